"""GPU parity of calls over the paged cache whose outcome must not follow from other sequences of the call or from arguments that
say nothing of the data, against the 64-bit oracle.

Tolerances, relative to the root mean square of the oracle's output. bf16 queries: half a step of the output, 2^-8
of its value; probabilities cut to 16 bits are 2^-15 of themselves off at most, scores' fp32 roundings below 60 2^-24 of
|q| |k| / sqrt(hd): 0.002 together with values of up to 5 times the root mean square, as in the other tests of this entry
point. Probabilities rounded to bf16 do not meet it: 2^-9 each, a thousandth of the root mean square at a deviation of one
for sums that a few rows carry, thrice that among ten thousand outputs.
"""

import numpy as np
import pytest

import oracle
from oracle import serve
from synth import bf16_bits
from gpu_util import say, dev_bf16, dev_f32, dev_i32, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


def _inputs(seed, before, new, page, h, hkv, hd):
    rng = np.random.default_rng(seed)
    need = [-(-(p + n) // page) for p, n in zip(before, new)]
    pages = sum(need) + 1
    order = rng.permutation(pages)
    table = np.full((len(before), max(need)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    q = bf16_bits(rng.standard_normal((sum(new), h, hd)).astype(np.float32))
    kp = bf16_bits(rng.standard_normal((pages, hkv, page, hd)).astype(np.float32))
    vp = bf16_bits(rng.standard_normal((pages, hkv, hd, page)).astype(np.float32))
    return rng, q, kp, vp, table, np.cumsum([0] + list(new)).astype(np.int32)


def _call(sr, q, kp, vp, table, before, start, **kw):
    out = sr.sirius_attn_paged(dev_bf16(q), dev_bf16(kp), dev_bf16(vp), dev_i32(table), dev_i32(np.array(before)),
                               tok_start=dev_i32(start), **kw)
    return oracle.widen_bf16(host(out)).astype(np.float64)


@pytest.mark.parametrize("h,hkv,hd", [(32, 8, 128), (12, 4, 96), (8, 2, 64)])
@pytest.mark.parametrize("kw", [dict(), dict(softcap=30.0), dict(window=150)])
def test_few_rows_keep_their_precision_whatever_the_call(sr, h, hkv, hd, kw):
    """Decoded tokens and short chunks beside a prompt, and without max_n, have 16 bits of their probabilities."""
    rng, q, kp, vp, table, start = _inputs(hd, [60, 7, 200, 300, 0, 33], [1, 5, 1, 3, 140, 1], 16, h, hkv, hd)
    before = [60, 7, 200, 300, 0, 33]
    want = serve.attn_paged(oracle.widen_bf16(q), kp, vp, table, before, start, **kw)
    got = _call(sr, q, kp, vp, table, before, start, **kw)
    few = np.r_[0:10, 150]  # every sequence but the prompt
    rms = float(np.sqrt(np.mean(want[few] ** 2)))
    err = float(np.max(np.abs(got[few] - want[few]) - 2.0 ** -8 * np.abs(want[few]))) / rms
    say(f"  H={h}/{hkv} hd={hd} {kw}: {err:.2e} x RMS beyond the output's rounding")
    assert err <= 0.002
    many = slice(10, 150)
    more = 2.0 ** -8 * (serve.attn_paged(oracle.widen_bf16(q), kp, vp & 0x7fff, table, before, start, **kw)[many] + 2 * np.abs(want[many]))
    assert (np.abs(got[many] - want[many]) <= more + 0.002 * float(np.sqrt(np.mean(want[many] ** 2)))).all()


def test_masked_trees_without_max_n(sr):
    """A batch of trees with more than 64 nodes in all: each has fewer, so their masks hold."""
    import torch
    before, new = [30, 0, 100, 5, 61], [16, 20, 16, 13, 64]
    rng, q, kp, vp, table, start = _inputs(21, before, new, 8, 8, 2, 64)
    mask = []
    for n in new:
        bits = []
        for i in range(n):
            bits.append((bits[rng.integers(i)] if i and rng.random() < 0.8 else 0) | 1 << i)
        mask += bits
    words = torch.from_numpy(np.array(mask, np.uint64).view(np.int64)).cuda()
    want = serve.attn_paged(oracle.widen_bf16(q), kp, vp, table, before, start, mask=mask)
    got = _call(sr, q, kp, vp, table, before, start, mask=words)
    rms = float(np.sqrt(np.mean(want ** 2)))
    more = 2.0 ** -8 * (np.abs(want) + serve.attn_paged(oracle.widen_bf16(q), kp, vp & 0x7fff, table, before, start, mask=mask))
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + more + 0.002 * rms).all()
    given = _call(sr, q, kp, vp, table, before, start, mask=words, max_n=64)
    assert np.array_equal(got, given)
    # 65 tokens of one sequence have no bits: NaN, the others as they are
    got = _call(sr, q, kp, vp, np.ascontiguousarray(table[:3]), [30, 0, 0], np.array([0, 16, 36, 36 + 65], np.int32), mask=words)
    assert np.isnan(got[36:101]).all() and np.isfinite(got[:36]).all()


def test_max_n_left_out_is_what_a_table_holds(sr):
    """Short tables: the call is made for their rows, and a sequence beyond them gets NaN with and without max_n."""
    before, new = [0, 3, 9], [6, 1, 5]
    rng, q, kp, vp, table, start = _inputs(22, before, new, 8, 4, 2, 64)
    short = np.ascontiguousarray(table[:, :1])
    start2 = np.array([0, 6, 7, 12], np.int32)
    a = _call(sr, q, kp, vp, short, before, start2)
    b = _call(sr, q, kp, vp, short, before, start2, max_n=12)
    assert np.isnan(a[7:]).all() and np.array_equal(a[7:], b[7:], equal_nan=True)
    want = serve.attn_paged(oracle.widen_bf16(q), kp, vp, short, before, start2)
    rms = float(np.sqrt(np.mean(want[:7] ** 2)))
    for got in (a, b):
        assert (np.abs(got[:7] - want[:7]) <= 2.0 ** -8 * np.abs(want[:7]) + 0.002 * rms).all()


@pytest.mark.parametrize("cap", [1e-45, 1e-39, 2.0 ** -127, 1.2e-38, 3e38])
def test_caps_at_the_ends_of_fp32(sr, cap):
    """The smallest caps leave every row the same score, the largest leave scores as they are; one token and a prompt."""
    for before, new in (([70, 3], [1, 1]), ([5], [80])):
        rng, q, kp, vp, table, start = _inputs(23, before, new, 16, 4, 2, 64)
        kp[table[0, 0], :, 2] = 0  # a score of 0
        want = serve.attn_paged(oracle.widen_bf16(q), kp, vp, table, before, start, softcap=float(np.float32(cap)))
        got = _call(sr, q, kp, vp, table, before, start, softcap=cap)
        rms = float(np.sqrt(np.mean(want ** 2)))
        more = 2.0 ** -8 * (np.abs(want) + serve.attn_paged(oracle.widen_bf16(q), kp, vp & 0x7fff, table, before, start,
                                                            softcap=float(np.float32(cap)))) if new == [80] else 0.0
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + more + 0.002 * rms).all(), (cap, new)


@pytest.mark.parametrize("before,new,page,kw", [
    ([100], [300], 24, dict()), ([100], [300], 24, dict(window=130, softcap=20.0)), ([3000, 90], [1, 3], 8, dict()),
    ([700], [20], 64, dict(window=600)), ([0], [40], 16, dict())])
@pytest.mark.parametrize("qt", ["f32", "bf16"])
def test_infinities_and_nans_that_are_seen(sr, before, new, page, kw, qt):
    """An infinite value stays in its column, a key of NaN in the rows and heads that see it; everything else is as without
    them, whichever rows the matrix units' pieces spoil."""
    h, hkv, hd = 8, 2, 96
    rng, q, kp, vp, table, start = _inputs(31, before, new, page, h, hkv, hd)
    seen = before[0] + new[0]
    at = lambda row: (table[0, row // page], row % page)
    v_row, k_row = (seen * 2 // 3, seen - new[0] // 2 - 1) if kw.get("window", 999) > 200 else (seen - 260, seen - 60)
    qq = oracle.widen_bf16(q).astype(np.float32)
    want = serve.attn_paged(qq, kp, vp, table, before, start, **kw)
    more = 2.0 ** -8 * (np.abs(want) + serve.attn_paged(qq, kp, vp & 0x7fff, table, before, start, **kw)) if qt == "bf16" else 0.0
    pg, off = at(v_row)
    v2 = vp.copy()
    v2[pg, 0, 5, off], v2[pg, 0, 70, off] = bf16_bits(np.array([np.inf, -np.inf], np.float32))
    k2 = kp.copy()
    pg, off = at(k_row)
    k2[pg, 1, off, 17] = bf16_bits(np.array([np.nan], np.float32))[0]
    out = sr.sirius_attn_paged(dev_f32(qq) if qt == "f32" else dev_bf16(q), dev_bf16(k2), dev_bf16(v2), dev_i32(table),
                               dev_i32(np.array(before)), tok_start=dev_i32(start), **kw)
    got = (host(out) if qt == "f32" else oracle.widen_bf16(host(out))).astype(np.float64)
    row = np.concatenate([p + np.arange(n) for p, n in zip(before, new)])
    mine = np.arange(sum(new)) < new[0]
    window = kw.get("window") or 1 << 30
    sees = lambda r: mine & (row >= r) & (row < r + window)
    heads = np.arange(h) // (h // hkv)
    bad = np.zeros(got.shape, bool)
    bad[np.ix_(sees(v_row), heads == 0, [5, 70])] = True
    bad[np.ix_(sees(k_row), heads == 1)] = True
    assert (got[np.ix_(sees(v_row), heads == 0, [5])] == np.inf).all() and (got[np.ix_(sees(v_row), heads == 0, [70])] == -np.inf).all()
    assert np.isnan(got[np.ix_(sees(k_row), heads == 1)]).all()
    rms = float(np.sqrt(np.mean(want ** 2)))
    tol = (2.0 ** -8 * np.abs(want) + more + 0.002 * rms) if qt == "bf16" else 1e-4 * rms
    ok = np.abs(got - want) <= tol
    assert ok[~bad].all(), float(np.max(np.abs(got - want)[~bad])) / rms
