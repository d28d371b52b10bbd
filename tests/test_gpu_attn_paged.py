"""GPU parity: attention over the paged cache against the 64-bit oracle.

Tolerances, relative to the root mean square of the oracle's output. fp32 queries: the scores' products
and sums round to about (hd + 4) 2^-24 |q| |k| / sqrt(hd), below 60 2^-24 here, weights and their sums to
a few more of it: 1e-4 is the bar of every fp32 attention in this suite. bf16 queries: out rounds to half
a step, 2^-8 of its value (values reach 5 times the root mean square: 0.02), probabilities to 16 bits and
scores as above, below 0.002 more.
"""

import numpy as np
import pytest

import oracle
from oracle import serve
from synth import bf16_bits
from gpu_util import say, dev_bf16, dev_f32, dev_i32, host

pytestmark = pytest.mark.gpu

TOL = {"f32": (0.0, 1e-4), "bf16": (2.0 ** -8, 0.002)}  # of the value, of the root mean square


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


def _table(rng, before, new, page, spare=2):
    need = [-(-(p + n) // page) for p, n in zip(before, new)]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table = np.full((len(before), max(need + [1]) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return pages, table


def _inputs(seed, before, new, page, h, hkv, hd, std=1.0):
    rng = np.random.default_rng(seed)
    pages, table = _table(rng, before, new, page)
    q = (std * rng.standard_normal((sum(new), h, hd))).astype(np.float32)
    kp = bf16_bits(rng.standard_normal((pages, hkv, page, hd)).astype(np.float32))
    vp = bf16_bits(rng.standard_normal((pages, hkv, hd, page)).astype(np.float32))
    return rng, q, kp, vp, table, np.cumsum([0] + list(new)).astype(np.int32)


def _dev_q(q, qt):
    return dev_f32(q) if qt == "f32" else dev_bf16(bf16_bits(q))


def _seen_q(q, qt):
    return q if qt == "f32" else oracle.widen_bf16(bf16_bits(q))


def _host(t):
    import torch
    a = host(t)
    return (oracle.widen_bf16(a) if t.dtype == torch.bfloat16 else a).astype(np.float64)


def _run(sr, q, kp, vp, table, before, start, qt, **kw):
    import torch
    dev = {k: (dev_f32(v) if k == "slopes" else v) for k, v in kw.items()}
    if kw.get("mask") is not None:
        dev["mask"] = torch.from_numpy(np.asarray(kw["mask"], np.uint64).view(np.int64)).cuda()
    return sr.sirius_attn_paged(_dev_q(q, qt), dev_bf16(kp), dev_bf16(vp), dev_i32(table), dev_i32(np.asarray(before)),
                                tok_start=None if start is None else dev_i32(start), **dev)


def _check(got, want, tol, more=0.0):
    rms = float(np.sqrt(np.mean(want * want)))
    err = float(np.max(np.abs(got - want) - tol[0] * np.abs(want) - more)) / max(rms, 1e-30)
    assert err <= tol[1], f"max-abs error {err:.3e} x RMS"
    return err


def _parity(sr, seed, before, new, page, h, hkv, hd, qt, std=1.0, uniform=False, **kw):
    rng, q, kp, vp, table, start = _inputs(seed, before, new, page, h, hkv, hd, std)
    got = _host(_run(sr, q, kp, vp, table, before, None if uniform else start, qt, **kw))
    okw = {k: v for k, v in kw.items() if k != "max_n"}
    want = serve.attn_paged(_seen_q(q, qt), kp, vp, table, before, start, **okw)
    more = 0.0
    n = kw.get("max_n") or (max(new) if uniform else sum(new))  # the call's max_n
    if qt == "bf16" and n * (h // hkv) > 64:
        more = 2.0 ** -8 * (serve.attn_paged(_seen_q(q, qt), kp, vp & 0x7fff, table, before, start, **okw) + np.abs(want))
    e = _check(got, want, TOL[qt], more)
    say(f"  before={before} new={new} page={page} H={h}/{hkv} hd={hd} {qt} {sorted(kw)}: {e:.2e} x RMS")


@pytest.mark.parametrize("qt", ["f32", "bf16"])
@pytest.mark.parametrize("before,new,page,h,hkv,hd", [
    ([0], [1], 8, 1, 1, 8),                              # the first token of all
    ([31, 32, 33, 0], [1, 1, 1, 1], 16, 4, 2, 64),        # around a tile
    ([127, 128, 129, 500], [1] * 4, 24, 32, 8, 128),      # around four tiles; pages that end inside them
    ([2047], [1], 64, 32, 8, 128),
    ([4000, 3, 700], [1, 1, 1], 200, 8, 1, 96),
    ([5, 0, 300], [3, 20, 16], 16, 12, 2, 80),            # ragged chunks
    ([0, 40], [70, 0], 32, 4, 4, 40),                     # a prompt, and a sequence without tokens
    ([900], [16], 64, 64, 8, 128),                        # 128 query rows per key/value head
    ([0], [200], 64, 8, 2, 128),
    ([50], [333], 40, 6, 2, 112),
    ([1000, 10], [130, 1], 4096, 16, 4, 64),
])
def test_shapes(sr, qt, before, new, page, h, hkv, hd):
    _parity(sr, len(before) * 7 + hd, before, new, page, h, hkv, hd, qt)


@pytest.mark.parametrize("qt", ["f32", "bf16"])
@pytest.mark.parametrize("before,new", [([700, 3], [1, 1]), ([90, 0, 1500], [6, 9, 2]), ([10], [150])])
def test_cap_bias_and_window(sr, qt, before, new):
    h, hkv, hd, page = 8, 2, 128, 16
    slopes = (2.0 ** -np.arange(1, h + 1)).astype(np.float32)
    for i, kw in enumerate((dict(softcap=5.0), dict(softcap=50.0, scale=0.4), dict(slopes=slopes), dict(window=1), dict(window=33),
                            dict(window=100, softcap=20.0, slopes=slopes), dict(scale=0.02))):
        _parity(sr, 50 + i, before, new, page, h, hkv, hd, qt, std=2.0, **kw)


@pytest.mark.parametrize("qt", ["f32", "bf16"])
@pytest.mark.parametrize("before,n,w,page,h,hkv", [([0, 100], 13, 3, 8, 4, 2), ([1000], 64, 4, 64, 32, 8), ([513, 31], 40, 8, 24, 8, 8)])
def test_tree_masks(sr, qt, before, n, w, page, h, hkv):
    rng = np.random.default_rng(n)
    mask = []
    for _ in before:
        bits = []
        for i in range(n):
            up = bits[(i // w - 1) * w + int(rng.integers(w))] if i >= w else 0
            bits.append(up | 1 << i)
        mask += bits
    _parity(sr, 70 + n, before, [n] * len(before), page, h, hkv, 64, qt, uniform=True, mask=mask)
    _parity(sr, 71 + n, before, [n] * len(before), page, h, hkv, 64, qt, mask=mask, window=20, softcap=30.0, max_n=n)


def test_tokens_that_see_nothing_get_zeros(sr):
    rng, q, kp, vp, table, start = _inputs(5, [0, 600], [4, 4], 8, 4, 2, 64)
    mask = [0, 0b10, 0b100, 0, 0, 0b1, 0, 0b1000]
    for window in (0, 1):
        got = _host(_run(sr, q, kp, vp, table, [0, 600], start, "f32", mask=mask, window=window))
        want = serve.attn_paged(q, kp, vp, table, [0, 600], start, mask=mask, window=window)
        _check(got, want, TOL["f32"])
        assert (got[[0, 3]] == 0.0).all()
        assert ((got[[4, 6]] == 0.0).all()) == (window == 1)


@pytest.mark.parametrize("qt", ["f32", "bf16"])
def test_hidden_rows_do_not_reach_a_token(sr, qt):
    """Infinities and NaN in rows that a token does not see: behind the last token in its page, later rows of the
    chunk, rows in front of the window, nodes that are no ancestors."""
    before, new, page = [100, 7], [5, 3], 24
    rng, q, kp, vp, table, start = _inputs(8, before, new, page, 4, 2, 64)
    mask = [0b00001, 0b00011, 0b00101, 0b01011, 0b10101, 0b001, 0b011, 0b101]
    cases = [dict(), dict(window=40), dict(mask=mask), dict(mask=mask, window=3, softcap=10.0)]
    for bad in (np.inf, -np.inf, np.nan):
        for kw in cases:
            k2, v2 = kp.copy(), vp.copy()
            junk = bf16_bits(np.array([bad], np.float32))[0]
            for b, (p, n) in enumerate(zip(before, new)):
                for row in range(p + n, (p + n + page - 1) // page * page):  # behind the last token
                    k2[table[b, row // page], :, row % page], v2[table[b, row // page], :, :, row % page] = junk, junk
            row = before[0] + 3  # seen by token 3 and, without masks, 4
            k2[table[0, row // page], :, row % page], v2[table[0, row // page], :, :, row % page] = junk, junk
            if kw.get("window"):
                for row in (0, 60):  # in front of every window
                    k2[table[0, row // page], :, row % page], v2[table[0, row // page], :, :, row % page] = junk, junk
            got = _host(_run(sr, q, k2, v2, table, before, start, qt, **kw))
            want = serve.attn_paged(_seen_q(q, qt), kp, vp, table, before, start, **kw)
            sees = [3] if kw.get("mask") else [3, 4]
            rest = [t for t in range(8) if t not in sees]
            _check(got[rest], want[rest], TOL[qt])


def test_infinite_keys_and_values_that_are_seen(sr):
    before, new, page = [40], [2], 8
    rng, q, kp, vp, table, start = _inputs(9, before, new, page, 2, 1, 64)
    q = np.abs(q)
    at = (table[0, 3], 0, 3)  # row 27
    k2 = kp.copy()
    k2[at] = bf16_bits(np.full(64, -np.inf, np.float32))  # score -inf: weighs nothing
    got = _host(_run(sr, q, k2, vp, table, before, start, "f32"))
    with np.errstate(invalid="ignore"):
        want = serve.attn_paged(q, k2, vp, table, before, start)
    _check(got, want, TOL["f32"])
    v2 = vp.copy()
    v2[table[0, 3], 0, 5, 3] = bf16_bits(np.array([np.inf], np.float32))[0]  # an infinite column stays in its column
    got = _host(_run(sr, q, kp, v2, table, before, start, "f32"))
    want = serve.attn_paged(q, kp, vp, table, before, start)
    assert (got[:, :, 5] == np.inf).all()
    rest = [c for c in range(64) if c != 5]
    _check(got[:, :, rest], want[:, :, rest], TOL["f32"])


def test_bad_places_give_nan_and_leave_the_rest(sr):
    before, new, page = [10, -1, 30, 3, 200], [2, 2, 2, 2, 2], 8
    rng, q, kp, vp, table, start = _inputs(10, [10, 1, 30, 3, 200], new, page, 4, 2, 64)
    table[3, 0] = kp.shape[0]
    table[4, 2] = -7  # in the middle of a long sequence
    before[2] = table.shape[1] * page - 1
    extra = 3  # tokens behind the last sequence
    q2 = np.concatenate([q, q[:extra]])
    import torch
    out = torch.full((len(q2), 4, 64), 5.0, device="cuda")
    got = _host(sr.sirius_attn_paged(dev_f32(q2), dev_bf16(kp), dev_bf16(vp), dev_i32(table), dev_i32(np.array(before)),
                                     tok_start=dev_i32(start), max_n=2, out=out))
    want = serve.attn_paged(q, kp, vp, table, before, start)
    _check(got[:2], want[:2], TOL["f32"])
    assert np.isnan(got[2:10]).all() and (got[10:] == 5.0).all()
    # a page in front of every window is not looked at
    got = _host(_run(sr, q, kp, vp, table, before, start, "f32", window=100, max_n=2))
    want = serve.attn_paged(q, kp, vp, table, before, start, window=100)
    _check(got[8:], want[8:], TOL["f32"])
    # more tokens than max_n
    got = _host(_run(sr, q, kp, vp, table, before, np.array([0, 2, 4, 6, 8, 10], np.int32), "f32", max_n=1))
    assert np.isnan(got).all()


def test_ragged_batch_long_and_short(sr):
    """Sequences of several units and of one in a call, by more sequences than one block counts."""
    rng = np.random.default_rng(3)
    before = (rng.integers(0, 40, 300)).tolist()
    before[7], before[150], before[299] = 6000, 9001, 3000
    new = [1] * 300
    new[20], new[250] = 0, 3
    _parity(sr, 31, before, new, 16, 2, 1, 64, "f32", max_n=3)


@pytest.mark.parametrize("qt", ["f32", "bf16"])
@pytest.mark.parametrize("before,new,page,h,hkv,hd", [
    ([24000, 16500], [1, 1], 16, 64, 64, 8),    # units longer than the pages staged at once
    ([5000], [600], 24, 64, 64, 8),             # whole sequences in tiles, their page ring wraps
    ([3000, 2500, 3100], [20, 20, 20], 8, 64, 64, 8),
])
def test_long_units(sr, qt, before, new, page, h, hkv, hd):
    _parity(sr, 40 + hd, before, new, page, h, hkv, hd, qt, max_n=max(new))


def test_strided_queries_and_streams(sr):
    import torch
    before, new, page = [300, 20], [3, 3], 16
    rng, q, kp, vp, table, start = _inputs(12, before, new, page, 4, 2, 64)
    args = [dev_bf16(kp), dev_bf16(vp), dev_i32(table), dev_i32(np.array(before))]
    wide = torch.zeros(6, 4 * 64 + 256, device="cuda")
    wide[:, : 4 * 64] = dev_f32(q).view(6, -1)
    one = sr.sirius_attn_paged(wide[:, : 4 * 64].view(6, 4, 64), *args)
    two = sr.sirius_attn_paged(dev_f32(q), *args)
    assert torch.equal(one, two)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    three = sr.sirius_attn_paged(dev_f32(q), *args, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(three, two)
    none = sr.sirius_attn_paged(dev_f32(q)[:0], *args)
    assert tuple(none.shape) == (0, 4, 64)
