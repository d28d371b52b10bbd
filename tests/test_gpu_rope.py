"""GPU parity: rotary positions with per-head norms, and the append of keys and values to the paged
cache, against the 64-bit oracle.

Tolerances. A result is a sum of two products of values below s = sqrt(hd) * max|w| (normalised) or max|x|,
times mscale: each product, the sum, the norm's factor (its sum of hd squares, root and division: under
hd / 2 + 4 half steps) and the sine (one ulp of 1) round in fp32, so |error| <= (hd / 2 + 12) 2^-24 of
the pair's magnitude |u| + |v| times mscale; bf16 results add half a step, 2^-8 of the value.
"""

import numpy as np
import pytest

from oracle import serve
from synth import bf16_bits
from gpu_util import say, dev_bf16, dev_f32, dev_i32, host
import oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


def _freqs(rot, theta=10000.0):
    import torch
    if rot == 0:
        return None, np.zeros(0)
    f = theta ** (-2.0 * np.arange(rot // 2) / rot)
    return torch.from_numpy(f).cuda(), f


def _dev(x, dtype):
    return dev_f32(x) if dtype == "f32" else dev_bf16(bf16_bits(x))


def _seen(x, dtype):
    return x if dtype == "f32" else oracle.widen_bf16(bf16_bits(x))


def _magnitude(x, rot, inter, eps, w):
    """|u| + |v| of each column's pair, of the normalised row."""
    y = np.abs(serve.rope(x, np.zeros(x.shape[0]), np.zeros(0), norm_eps=eps, weight=w))
    m = y.copy()
    half = rot // 2
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if inter else (j, j + half)
        m[..., a] = m[..., b] = y[..., a] + y[..., b]
    return m


def _check(got, want, x, rot, inter, eps, w, mscale, bf16):
    hd = x.shape[-1]
    tol = (hd / 2 + 12) * 2.0 ** -24 * _magnitude(x, rot, inter, eps, w) * max(1.0, abs(mscale))
    if bf16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    err = np.abs(np.asarray(got, np.float64) - want)
    assert (err <= tol + 1e-38).all(), f"{float((err / (tol + 1e-38)).max()):.3g} times the tolerance"


def _host(t):
    import torch
    a = host(t)
    return oracle.widen_bf16(a) if t.dtype == torch.bfloat16 else a


@pytest.mark.parametrize("t,h,hkv,hd,rot,inter,norm,qt,kt,far", [
    (1, 32, 8, 128, 128, False, False, "f32", "bf16", 2047),
    (1, 1, 1, 8, 2, False, True, "f32", "f32", 3),
    (3, 5, 1, 24, 10, False, True, "bf16", "f32", 900000),    # pairs that start on no vector
    (7, 4, 2, 80, 20, False, False, "f32", "bf16", 100),
    (7, 12, 2, 80, 22, True, True, "f32", "f32", 1000000),     # a vector of pairs turned in part
    (130, 3, 3, 64, 64, True, False, "bf16", "bf16", 131072),
    (1100, 6, 2, 96, 48, False, True, "bf16", "bf16", 40000),  # one workgroup per token
    (5, 2, 2, 40, 0, False, True, "f32", "f32", 10),           # the norm alone
    (2, 64, 8, 120, 118, True, True, "f32", "bf16", 1 << 30),
])
def test_rope(sr, t, h, hkv, hd, rot, inter, norm, qt, kt, far):
    say(f"rope T={t} H={h}/{hkv} hd={hd} rot={rot} inter={inter} norm={norm} {qt}/{kt}")
    rng = np.random.default_rng(t * 131 + hd)
    q, k = rng.standard_normal((t, h, hd)).astype(np.float32), rng.standard_normal((t, hkv, hd)).astype(np.float32)
    k *= 30.0
    wq, wk = (bf16_bits((1 + 0.3 * rng.standard_normal(hd)).astype(np.float32)) for _ in range(2))
    pos = (far - rng.integers(0, far + 1, t)).astype(np.int32)
    fd, f = _freqs(rot)
    eps, m = (1e-5 if norm else -1.0), 1.25
    kw = dict(interleaved=inter, mscale=m, norm_eps=eps)
    if norm:
        kw |= dict(q_weight=dev_bf16(wq), k_weight=dev_bf16(wk))
    qo, ko = sr.sirius_rope(_dev(q, qt), _dev(k, kt), dev_i32(pos), fd, **kw)
    q, k = _seen(q, qt), _seen(k, kt)
    want_q = serve.rope(q, pos, f, inter, m, eps, wq if norm else None)
    want_k = serve.rope(k, pos, f, inter, m, eps, wk if norm else None)
    _check(_host(qo), want_q, q, rot, inter, eps, wq if norm else None, m, qt == "bf16")
    _check(_host(ko), want_k, k, rot, inter, eps, wk if norm else None, m, True)


def test_rope_views_in_place_and_absent_inputs(sr):
    import torch
    rng = np.random.default_rng(9)
    t, h, hkv, hd = 9, 4, 2, 32
    x = rng.standard_normal((t, (h + 2 * hkv) * hd)).astype(np.float32)
    pos = dev_i32(rng.integers(0, 5000, t))
    fd, _ = _freqs(hd)
    X = dev_f32(x)
    q, k = X[:, : h * hd].view(t, h, hd), X[:, h * hd:(h + hkv) * hd].view(t, hkv, hd)
    qo, ko = sr.sirius_rope(q, k, pos, fd)
    q2, k2 = sr.sirius_rope(q.contiguous(), k.contiguous(), pos, fd)
    assert torch.equal(qo, q2) and torch.equal(ko, k2)
    only_q, none = sr.sirius_rope(q, None, pos, fd)
    none2, only_k = sr.sirius_rope(None, k, pos, fd)
    assert none is None and none2 is None and torch.equal(only_q, qo) and torch.equal(only_k, ko)
    c = q.contiguous()
    same, _ = sr.sirius_rope(c, None, pos, fd, q_out=c)
    assert same is c and torch.equal(c, qo)
    kb = k.to(torch.bfloat16)
    want = sr.sirius_rope(None, kb.contiguous(), pos, fd)[1]
    kb = kb.contiguous()
    sr.sirius_rope(None, kb, pos, fd, k_out=kb)
    assert torch.equal(kb, want)
    e, _ = sr.sirius_rope(q[:0], None, pos[:0], fd)
    assert tuple(e.shape) == (0, h, hd)


def test_rope_infinities_stay_where_they_are(sr):
    """A column behind the rotated ones passes whatever it holds; a pair with an infinity does not touch others."""
    x = np.ones((1, 1, 16), np.float32)
    x[0, 0, 12], x[0, 0, 13], x[0, 0, 1] = np.inf, np.nan, -np.inf
    for inter, pair in ((False, (1, 5)), (True, (0, 1))):
        fd, f = _freqs(8)
        got = host(sr.sirius_rope(dev_f32(x), None, dev_i32([3]), fd, interleaved=inter)[0])[0, 0]
        assert got[12] == np.inf and np.isnan(got[13])
        rest = [c for c in range(16) if c not in pair + (12, 13)]
        assert np.isfinite(got[rest]).all() and not np.isfinite(got[list(pair)]).any()


def _cache(rng, bsz, before, new, page, hkv, hd, spare=2):
    need = [-(-(p + n) // page) for p, n in zip(before, new)]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table = np.full((bsz, max(need + [1]) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    kp = bf16_bits(rng.standard_normal((pages, hkv, page, hd)).astype(np.float32))
    vp = bf16_bits(rng.standard_normal((pages, hkv, hd, page)).astype(np.float32))
    return kp, vp, table


@pytest.mark.parametrize("before,new,page,h,hkv,hd,rot,inter,norm,qt,kt,ragged", [
    ([0], [1], 8, 4, 2, 16, 16, False, False, "f32", "bf16", False),
    ([7, 8, 300], [1, 1, 1], 64, 32, 8, 128, 128, False, False, "f32", "bf16", False),
    ([3, 0, 50, 9, 1], [5, 0, 130, 1, 0], 24, 12, 2, 80, 40, True, True, "f32", "f32", True),
    ([0, 1000], [200, 77], 16, 4, 4, 64, 30, False, True, "bf16", "bf16", True),
    ([1], [1500], 32, 8, 1, 96, 96, False, True, "bf16", "f32", False),
    ([0, 0, 0], [0, 9, 0], 200, 2, 2, 8, 8, True, False, "f32", "f32", True),
])
def test_append(sr, before, new, page, h, hkv, hd, rot, inter, norm, qt, kt, ragged):
    say(f"append before={before} new={new} page={page} H={h}/{hkv} hd={hd} {qt}/{kt}")
    rng = np.random.default_rng(sum(new) + hd)
    bsz, t = len(before), sum(new)
    extra = 2 if ragged else 0  # tokens behind the last sequence
    kp, vp, table = _cache(rng, bsz, before, new, page, hkv, hd)
    q = rng.standard_normal((t + extra, h, hd)).astype(np.float32)
    k, v = rng.standard_normal((2, t + extra, hkv, hd)).astype(np.float32)
    w = bf16_bits((1 + 0.3 * rng.standard_normal(hd)).astype(np.float32))
    start = np.cumsum([0] + new).astype(np.int32)
    fd, f = _freqs(rot)
    eps = 1e-6 if norm else -1.0
    kw = dict(interleaved=inter, norm_eps=eps)
    if norm:
        kw |= dict(q_weight=dev_bf16(w), k_weight=dev_bf16(w))
    Kp, Vp = dev_bf16(kp), dev_bf16(vp)
    Q = _dev(q, qt)
    out = Q.clone().fill_(7.0)
    got = sr.sirius_kv_append(Q, _dev(k, kt), _dev(v, kt), Kp, Vp, dev_i32(table), dev_i32(before), fd,
                              tok_start=dev_i32(start) if ragged else None, q_out=out, **kw)
    assert got is out
    q, k, v = _seen(q, qt), _seen(k, kt), _seen(v, kt)
    rows = np.zeros(t, np.int64)
    want_k, want_v = kp.copy(), bf16_bits(np.zeros(1, np.float32)) * 0
    want_v = vp.copy()
    k2 = np.zeros((t, hkv, hd))
    hit = np.zeros(kp.shape, bool)
    for tok, b, row, pg in serve.places(before, start, table, page, kp.shape[0]):
        rows[tok] = row
        hit[pg, :, row % page] = True
        want_v[pg, :, :, row % page] = bf16_bits(v[tok].astype(np.float32))
    wn = w if norm else None
    want_q = serve.rope(q[:t], rows, f, inter, 1.0, eps, wn)
    k2 = serve.rope(k[:t], rows, f, inter, 1.0, eps, wn)
    res = _host(out)
    _check(res[:t], want_q, q[:t], rot, inter, eps, wn, 1.0, qt == "bf16")
    assert (res[t:] == 7.0).all()
    assert np.array_equal(host(Vp), want_v)
    k_got = host(Kp)
    assert np.array_equal(k_got[~hit], kp[~hit])  # every other row as it was
    wide = oracle.widen_bf16(k_got)
    for tok, b, row, pg in serve.places(before, start, table, page, kp.shape[0]):
        _check(wide[pg, :, row % page][None], k2[tok][None], k[tok][None], rot, inter, eps, wn, 1.0, True)


def test_append_positions_without_queries(sr):
    """Given positions turn the keys, the rows stay the cache's; without q nothing is returned."""
    import torch
    rng = np.random.default_rng(4)
    kp, vp, table = _cache(rng, 2, [4, 9], [3, 3], 8, 2, 16)
    k, v = rng.standard_normal((2, 6, 2, 16)).astype(np.float32)
    fd, f = _freqs(16)
    pos = np.array([4, 5, 5, 9, 10, 10], np.int32)
    Kp, Vp = dev_bf16(kp), dev_bf16(vp)
    assert sr.sirius_kv_append(None, dev_f32(k), dev_f32(v), Kp, Vp, dev_i32(table), dev_i32([4, 9]), fd,
                               positions=dev_i32(pos)) is None
    want = serve.rope(k, pos, f)
    got = oracle.widen_bf16(host(Kp))
    for tok, b, row, pg in serve.places([4, 9], [0, 3, 6], table, 8, kp.shape[0]):
        _check(got[pg, :, row % 8][None], want[tok][None], k[tok][None], 16, False, -1.0, None, 1.0, True)
    # no rotation at all: keys are copied
    Kp = dev_bf16(kp)
    sr.sirius_kv_append(None, dev_f32(k), dev_f32(v), Kp, Vp, dev_i32(table), dev_i32([4, 9]))
    for tok, b, row, pg in serve.places([4, 9], [0, 3, 6], table, 8, kp.shape[0]):
        assert np.array_equal(host(Kp)[pg, :, row % 8], bf16_bits(k[tok]))


def test_append_bad_places_write_nothing(sr):
    """Positions outside the table and pages outside the pool: the cache stays, other sequences are served."""
    rng = np.random.default_rng(6)
    kp, vp, table = _cache(rng, 4, [0, 4, 3, 6], [2, 2, 2, 2], 8, 1, 8)
    table[2, 0], table[3, 0] = kp.shape[0], -5
    cap = table.shape[1] * 8
    pos = np.array([-1, 4, 3, cap - 1], np.int32)
    k, v = rng.standard_normal((2, 8, 1, 8)).astype(np.float32)
    Kp, Vp = dev_bf16(kp), dev_bf16(vp)
    sr.sirius_kv_append(None, dev_f32(k), dev_f32(v), Kp, Vp, dev_i32(table), dev_i32(pos))
    want_k, want_v = kp.copy(), vp.copy()
    for i in range(2):
        want_k[table[1, 0], :, 4 + i] = bf16_bits(k[2 + i])
        want_v[table[1, 0], :, :, 4 + i] = bf16_bits(v[2 + i])
    assert np.array_equal(host(Kp), want_k) and np.array_equal(host(Vp), want_v)


def test_append_many_sequences(sr):
    """More sequences than one look at the offsets takes, most of them empty."""
    rng = np.random.default_rng(8)
    bsz = 5000
    new = (rng.random(bsz) < 0.1).astype(int) * rng.integers(1, 4, bsz)
    new[-1] = 0
    start = np.cumsum(np.concatenate(([0], new))).astype(np.int32)
    t = int(start[-1])
    table = np.arange(bsz, dtype=np.int32)[:, None]
    pos = rng.integers(0, 5, bsz).astype(np.int32)
    kp, vp = np.zeros((bsz, 1, 8, 8), np.uint16), np.zeros((bsz, 1, 8, 8), np.uint16)
    k, v = rng.standard_normal((2, t, 1, 8)).astype(np.float32)
    Kp, Vp = dev_bf16(kp), dev_bf16(vp)
    sr.sirius_kv_append(None, dev_f32(k), dev_f32(v), Kp, Vp, dev_i32(table), dev_i32(pos), tok_start=dev_i32(start))
    for tok, b, row, pg in serve.places(pos, start, table, 8, bsz):
        kp[pg, :, row], vp[pg, :, :, row] = bf16_bits(k[tok]), bf16_bits(v[tok])
    assert np.array_equal(host(Kp), kp) and np.array_equal(host(Vp), vp)
