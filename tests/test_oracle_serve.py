"""Pins of the serving-step oracle: rotary positions, places in the paged cache, attention over it,
sampling; and the host-side rotation frequencies."""

import ctypes
import math

import numpy as np
import pytest

import oracle
from oracle import serve


def test_a_quarter_turn_by_hand():
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    f = [math.pi / 2, 0.0]
    half = serve.rope(x, [1], f)  # pairs (0, 2) by a quarter turn, (1, 3) not at all
    np.testing.assert_allclose(half[0, 0], [-3, 2, 1, 4, 5, 6, 7, 8], atol=1e-15)
    inter = serve.rope(x, [1], f, interleaved=True)  # pairs (0, 1), (2, 3)
    np.testing.assert_allclose(inter[0, 0], [-2, 1, 3, 4, 5, 6, 7, 8], atol=1e-15)


def test_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 16))
    f = 100.0 ** (-np.arange(8) / 8)
    at = lambda i, j: float(np.sum(serve.rope(q, [i], f) * serve.rope(k, [j], f)))
    assert abs(at(7, 3) - at(1007, 1003)) < 1e-9


def test_norm_has_unit_mean_square():
    x = np.random.default_rng(2).standard_normal((3, 2, 24))
    y = serve.rope(x, [0, 5, 9], np.ones(6), norm_eps=0.0)  # a rotation keeps the norm
    np.testing.assert_allclose(np.mean(y * y, axis=-1), 1.0, rtol=1e-12)


def test_paged_attention_is_the_contiguous_one():
    rng = np.random.default_rng(3)
    h, hkv, hd, ps = 4, 2, 8, 8
    lens, new = [5, 0, 17], [3, 1, 2]
    q = rng.standard_normal((6, h, hd))
    kp, vp = rng.standard_normal((9, hkv, ps, hd)), rng.standard_normal((9, hkv, hd, ps))
    table = np.array([[4, -1, 0], [2, 9, 9], [7, 1, 3]])
    start = np.cumsum([0] + new)
    got = serve.attn_paged(q, kp, vp, table, lens, start)
    for b in range(3):
        length = lens[b] + new[b]
        keys = np.stack([kp[table[b, r // ps], :, r % ps] for r in range(length)])
        values = np.stack([vp[table[b, r // ps], :, :, r % ps] for r in range(length)])
        pad = np.zeros((1, 30, hkv, hd))
        kc, vc = pad.copy(), pad.copy()
        kc[0, :length], vc[0, :length] = keys, values
        want, _, _ = oracle.attn_kv(q[None, start[b]:start[b + 1]], keys[None, lens[b]:], values[None, lens[b]:], kc, vc, [lens[b]])
        np.testing.assert_allclose(got[start[b]:start[b + 1]], want[0], rtol=1e-12)


def test_masks_and_bad_pages_by_hand():
    kp, vp = np.zeros((2, 1, 8, 8)), np.zeros((2, 1, 8, 8))
    vp[0, 0, :, :] = np.arange(8.0)  # row r's value is r in every column
    q = np.ones((3, 1, 8))
    run = lambda **kw: serve.attn_paged(q, kp, vp, np.array([[0]]), [2], [0, 3], **kw)[:, 0, 0]
    np.testing.assert_allclose(run(), [1.0, 1.5, 2.0])          # means of 0..2, 0..3, 0..4
    np.testing.assert_allclose(run(window=1), [2.0, 3.0, 4.0])
    np.testing.assert_allclose(run(mask=[0b001, 0b010, 0b101]), [1.0, 4 / 3, 7 / 4])
    np.testing.assert_allclose(run(mask=[0, 0, 0], window=1), [0.0, 0.0, 0.0])
    slope = run(slopes=[math.log(2.0)])
    np.testing.assert_allclose(slope[0], (2 * 1 + 1 * 0.5) / 1.75)
    bad = serve.attn_paged(q, kp, vp, np.array([[2]]), [2], [0, 3])
    assert np.isnan(bad).all()


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.2, 0.1])
    tok = lambda u, **kw: serve.sample(x, u, **kw)[0]
    assert [tok(u) for u in (0.0, 0.0999, 0.1001, 0.4999, 0.5001, 0.95)] == [0, 0, 1, 1, 2, 4]
    assert serve.sample(x, 0.49, top_k=3)[:2] == (1, 3) and tok(0.999, top_k=3) == 3
    assert serve.sample(x, 0.999, top_k=2) [:2] == (2, 2)          # a tie goes to the lower index
    assert serve.sample(x, 0.0, top_p=0.39)[:2] == (1, 1)
    assert serve.sample(x, 0.999, top_p=0.41)[:2] == (2, 2)
    assert serve.sample(x, 0.0, min_p=0.49)[:2] == (1, 3)
    assert serve.sample(x, 0.3, temperature=0)[:2] == (1, 1)
    assert serve.sample(np.full(4, -np.inf), 0.3)[0] == -1
    assert serve.sample(np.array([np.nan, 1.0, -np.inf]), 0.9)[:2] == (1, 1)
    assert serve.sample(np.array([0.0, np.inf, np.inf]), 0.6)[:2] == (2, 2)


@pytest.fixture(scope="module")
def L():
    from paper_2409_03856_amd import _lib
    import os
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libsirius.so not built")
    return _lib.lib()


def _freqs(L, rot, theta, scaling=0, factor=1.0, low=0.0, high=0.0, orig=0.0):
    out = (ctypes.c_double * (rot // 2))()
    assert L.sirius_rope_freqs(out, rot, theta, scaling, factor, low, high, orig) == 0
    return np.array(out)


def test_frequencies(L):
    plain = _freqs(L, 8, 10000.0)
    np.testing.assert_allclose(plain, [1.0, 0.1, 0.01, 0.001], rtol=1e-14)
    np.testing.assert_allclose(_freqs(L, 8, 10000.0, 1, 4.0), plain / 4, rtol=1e-14)
    # the base form: the slowest pair is `factor` times as slow, the fastest as it was
    base = _freqs(L, 8, 10000.0, 2, 4.0)
    np.testing.assert_allclose(base[[0, 3]], [1.0, 0.001 / 4], rtol=1e-12)
    # smooth: pairs with over 4 turns in the original length stay, under 1 are divided, between is linear
    orig = 2 * math.pi * 100.0
    smooth = _freqs(L, 8, 10000.0, 3, 8.0, 1.0, 16.0, orig)  # turns 100, 10, 1, 0.1
    np.testing.assert_allclose(smooth, [1.0, 0.1 * (0.6 + 0.4 / 8), 0.01 / 8, 0.001 / 8], rtol=1e-12)
    # ramp: pair indices of 10 and 1 turns are 1 and 2
    ramp = _freqs(L, 8, 10000.0, 4, 8.0, 1.0, 10.0, orig * (1 + 1e-12))
    assert ramp[0] == 1.0 and ramp[3] == pytest.approx(0.001 / 8)


def test_frequency_refusals(L):
    out = (ctypes.c_double * 64)()
    err = lambda *a: L.sirius_rope_freqs(*a)
    assert err(None, 8, 1e4, 0, 1.0, 0.0, 0.0, 0.0) == -1
    for rot in (0, 7, 130, -2):
        assert err(out, rot, 1e4, 0, 1.0, 0.0, 0.0, 0.0) == -1
    for theta in (1.0, 0.0, float("nan"), float("inf")):
        assert err(out, 8, theta, 0, 1.0, 0.0, 0.0, 0.0) == -1
    assert err(out, 8, 1e4, 5, 1.0, 0.0, 0.0, 0.0) == -1
    assert err(out, 8, 1e4, 1, 0.5, 0.0, 0.0, 0.0) == -1
    assert err(out, 2, 1e4, 2, 2.0, 0.0, 0.0, 0.0) == -1
    assert err(out, 8, 1e4, 3, 2.0, 4.0, 1.0, 8192.0) == -1
    assert err(out, 8, 1e4, 3, 2.0, 1.0, 4.0, 0.0) == -1
    assert err(out, 8, 1e4, 4, 2.0, 0.0, 4.0, 8192.0) == -1
