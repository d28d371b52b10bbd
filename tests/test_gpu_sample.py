"""GPU parity: sampling against the 64-bit oracle.

Tokens and counts are whole numbers and have to be the oracle's, except where u (or the p-cut) lies within the
sums' own error of a border: weights are counted in units of 2^-(62 - log2 V) of the best one's, so a
border's share of the mass moves by at most V / 2 units, below 2^-25 for every V here. A row whose border
lies that close to its u counts as undecided; at most one row of a case may. prob is one rounding to
fp32 and those units off.
"""

import numpy as np
import pytest

from oracle import serve
from gpu_util import say, dev_f32, dev_i32, host

pytestmark = pytest.mark.gpu

BAND = 2.0 ** -25


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


def _logits(rng, b, v, std=2.5, ties=False):
    x = (std * rng.standard_normal((b, v))).astype(np.float32)
    x[:, rng.permutation(v)[: max(1, v // 500)]] += 5.0
    if ties:
        x = (np.round(x * 8) / 8).astype(np.float32)
    return x


def _check(sr, x, u, t, k, p, m, X=None):
    X = dev_f32(x) if X is None else X
    dev = lambda a, f: None if a is None else f(np.asarray(a))
    tok, kept, prob = sr.sirius_sample(X, dev_f32(u), temperature=dev(t, dev_f32), top_k=dev(k, dev_i32), top_p=dev(p, dev_f32),
                                       min_p=dev(m, dev_f32))
    tok, kept, prob = host(tok), host(kept), host(prob)
    undecided = 0
    at = lambda a, b, d: d if a is None else np.asarray(a, np.float64)[b]
    f32 = lambda a, b, d: d if a is None else float(np.float32(a[b]))
    for b in range(x.shape[0]):
        kw = dict(temperature=f32(t, b, 1.0), top_k=int(at(k, b, 0)), top_p=f32(p, b, 1.0), min_p=f32(m, b, 0.0))
        uu = float(np.float32(u[b]))
        want = serve.sample(x[b], uu, **kw)
        near = [serve.sample(x[b], min(max(uu + d, 0.0), 1.0), **(kw | dict(top_p=kw["top_p"] * (1 + e))))
                for d in (-BAND, BAND) for e in (-BAND, BAND)] if (tok[b], kept[b]) != want[:2] else []
        if near:
            undecided += 1
            assert (tok[b], kept[b]) in [n[:2] for n in near], (b, kw, uu, tok[b], kept[b], want)
            want = next(n for n in near if n[:2] == (tok[b], kept[b]))
        assert abs(prob[b] - want[2]) <= 2.0 ** -24 * want[2] + BAND, (b, prob[b], want)
    assert undecided <= 1
    return tok


@pytest.mark.parametrize("b,v,ties", [(1, 1, False), (3, 2, False), (5, 7, True), (4, 63, False), (4, 1000, True), (3, 1023, False),
                                      (2, 32000, False), (3, 50257, True), (2, 128256, False), (1, 300001, True)])
def test_filters(sr, b, v, ties):
    rng = np.random.default_rng(v)
    x = _logits(rng, b, v, ties=ties)
    for i, (t, k, p, m) in enumerate(((None, None, None, None), (0.7, None, None, None), (1.0, 5, None, None), (0.9, None, 0.9, None),
                                      (1.1, None, None, 0.05), (0.8, 50, 0.95, 0.02), (1.3, max(1, v // 3), 0.999, None),
                                      (1.0, v + 5, 0.5, 0.5), (0.05, 40, 0.99, None), (30.0, v // 2 + 1, 0.7, 0.9))):
        full = lambda a, d: None if a is None else np.full(b, a, d)
        u = rng.random(b).astype(np.float32)
        _check(sr, x, u, full(t, np.float32), full(k, np.int32), full(p, np.float32), full(m, np.float32))
    say(f"sample B={b} V={v} ties={ties}")


def test_mixed_batch_and_all_of_u(sr):
    rng = np.random.default_rng(2)
    b, v = 64, 2000
    x = np.repeat(_logits(rng, 1, v, ties=True), b, 0)
    u = np.linspace(0, 1, b).astype(np.float32)
    u[-2] = np.nextafter(np.float32(1), np.float32(0))
    _check(sr, x, u, None, None, None, None)
    t = rng.choice([0.0, 0.5, 1.0, 2.0], b).astype(np.float32)
    k = rng.choice([-1, 0, 1, 2, 17, 400, 2000, 5000], b).astype(np.int32)
    p = rng.choice([0.0, 0.1, 0.5, 0.9, 1.0, 1.5], b).astype(np.float32)
    m = rng.choice([-1.0, 0.0, 0.01, 0.5, 1.0, 1.5], b).astype(np.float32)
    _check(sr, _logits(rng, b, v, ties=True), rng.random(b), t, k, p, m)


def test_cuts_far_down_and_crowded(sr):
    """Cuts below what the bins hold, lists and bins with more tokens than their room, both cuts at once."""
    rng = np.random.default_rng(21)
    v = 40000
    x = _logits(rng, 12, v, std=3.0)
    x[1] = np.round(x[1])                      # a dozen values: thousands of ties at every cut
    x[2] = rng.choice([0.0, 1e-3], v)
    x[3, :20000] -= 200.0                      # half of the row weighs next to nothing
    x[4, 1:] -= 1000.0                         # more than 700 below: not counted
    x[5] = np.sort(x[5])
    x[6] = np.sort(x[6])[::-1]
    x[7, 5000:] = -np.inf
    x[8] *= 30.0
    u = rng.random(12).astype(np.float32)
    f = lambda a: np.full(12, a, np.float32)
    for t, k, p, m in ((1.0, 0, 1.0, 1e-15), (1.0, 0, 0.9999999, 0.0), (1.0, 0, 0.9999999, 1e-3), (1.0, 0, 0.3, 1e-20), (1.0, 200, 1.0, 0.0),
                       (1.0, 256, 0.99, 1e-9), (1.0, 257, 1.0, 0.0), (1.0, 39999, 1.0, 0.0), (1.0, 30000, 0.999, 0.0), (0.01, 300, 0.9, 0.1),
                       (1.0, 5000, 0.2, 0.3), (1.0, 0, 1.0, 0.0), (0.02, 0, 1.0, 0.0), (1e-6, 0, 0.9, 0.0), (1e-6, 3, 0.9, 0.0), (1e9, 0, 0.5, 0.0)):
        _check(sr, x, u, f(t), np.full(12, k), f(p), f(m))


def test_long_rows_of_many_chunks(sr):
    rng = np.random.default_rng(22)
    x = _logits(rng, 2, (1 << 21) + 77)
    for t, k, p, m in ((1.0, 100, 0.9, 0.0), (1.0, 0, 0.6, 0.0), (1.0, 0, 1.0, 0.02), (1.0, 0, 1.0, 0.0), (1.0, 3000, 0.9, 0.001)):
        f = lambda a: np.full(2, a, np.float32)
        _check(sr, x, rng.random(2).astype(np.float32), f(t), np.full(2, k), f(p), f(m))


def test_equal_logits(sr):
    """Every border is a tie: the lowest indices stay."""
    x = np.zeros((6, 1000), np.float32)
    x[3:] = -np.float32(3.4e38)
    u = np.array([0.0, 0.49995, 0.9999, 0.0, 0.49995, 0.9999], np.float32)
    for k, p in ((10, None), (None, 0.25), (333, 0.5), (None, 1.0)):
        _check(sr, x, u, None, None if k is None else np.full(6, k), None if p is None else np.full(6, p, np.float32), None)
    tok = _check(sr, x, u, None, np.full(6, 10), None, None)
    assert tok.tolist() == [0, 4, 9, 0, 4, 9]


def test_masked_infinite_and_nan_logits(sr):
    rng = np.random.default_rng(5)
    x = _logits(rng, 8, 5000)
    x[0, rng.random(5000) < 0.99] = -np.inf
    x[1, :] = -np.inf
    x[2, :] = np.nan
    x[3, ::2] = np.nan
    x[4, [7, 4000]] = np.inf
    x[5, 1:] = -np.inf
    x[6, :] = np.finfo(np.float32).min
    x[6, 123] = 0.0
    x[7, :] = np.finfo(np.float32).min
    u = np.full(8, 0.7, np.float32)
    for k, p in ((None, None), (50, 0.9), (4999, None), (None, 0.6)):
        tok = _check(sr, x, u, None, None if k is None else np.full(8, k), None if p is None else np.full(8, p, np.float32), None)
        assert tok[1] == -1 and tok[2] == -1 and tok[4] in (7, 4000) and tok[5] == 0 and tok[6] == 123


def test_masks_of_the_lowest_value_and_cold_rows(sr):
    """Tokens that weigh nothing (a mask's finite numbers, cold temperatures) are in no count, whatever share of a
    chunk or of the row they are; the end of the row masked as a padded vocabulary is."""
    rng = np.random.default_rng(15)
    v = 20000
    x = _logits(rng, 8, v)
    low = np.finfo(np.float32).min
    x[0, rng.random(v) < 0.5] = low
    x[1, 9000:] = low
    x[2, rng.random(v) < 0.999] = -1e9
    x[3, 16000:] = -1e4
    x[4, :8192] = low
    x[4, 8192:] -= 400.0
    x[5, ::2] -= 350.0
    x[5, 1::4] -= 695.0
    x[6, 1000:] = -np.inf
    x[6, ::7] = low
    u = rng.random(8).astype(np.float32)
    f = lambda a: np.full(8, a, np.float32)
    for t, k, p, m in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (1.0, 300, 1.0, 0.0), (1.0, 300, 0.8, 0.01),
                       (0.01, 0, 1.0, 0.0), (0.01, 0, 0.95, 0.0), (0.01, 300, 0.95, 0.0), (0.003, 0, 1.0, 0.001), (1.0, 40, 0.9, 0.0),
                       (1.0, 3, 1.0, 0.0), (1.0, 256, 1.0, 0.0), (0.01, 200, 1.0, 0.0)):
        _check(sr, x, u, f(t), np.full(8, k), f(p), f(m))


def test_cuts_beside_zero_at_hot_temperatures(sr):
    """All logits in one bin around zero, whose products with a hot temperature's scale vanish."""
    rng = np.random.default_rng(16)
    x = rng.standard_normal((5, 400)).astype(np.float32)
    x[1] = np.abs(x[1])
    x[2] = -np.abs(x[2])
    x[3] = rng.choice(np.array([0.0, -0.0, 1e-45, -1e-45, 1e-40, -1e-38], np.float32), 400)
    x[4] *= 1e30
    u = rng.random(5).astype(np.float32)
    for t in (1e3, 1e12, 1e30, 3e38):
        for k, p, m in ((0, 0.5, 0.0), (0, 1.0, 0.9), (300, 0.7, 0.5)):
            _check(sr, x, u, np.full(5, t, np.float32), np.full(5, k), np.full(5, p, np.float32), np.full(5, m, np.float32))


def test_smallest_parameters(sr):
    """Temperatures, shares and weights at the ends of fp32; u outside [0, 1] counts as its end."""
    rng = np.random.default_rng(19)
    x = np.round(_logits(rng, 6, 5000) * 2) / 2
    x[1] = np.where(rng.random(5000) < 0.01, np.float32(9.5), x[1])
    x[2] = 0.0
    u = np.array([-1.0, 0.5, 0.3, 2.0, 1.0, 0.0], np.float32)
    f = lambda a: np.full(6, a, np.float32)
    for t, k, p, m in ((1e-40, 0, 1.0, 0.0), (1e-45, 0, 0.9, 0.5), (1e-38, 300, 0.9, 0.0), (1e-40, 7, 1.0, 0.0), (1.0, 0, 1e-40, 0.0),
                       (1.0, 0, 1.0, 1.0), (1.0, 0, 1.0, 1e-40), (1.0, 5, 1e-45, 1.0), (0.5, 0, 0.99999994, 0.0)):
        _check(sr, x, u, f(t), np.full(6, k), f(p), f(m))


def test_all_of_u_with_a_tail_far_down(sr):
    """A last chunk whose tokens hold no unit of mass alone but some together: at u = 1 the last token that holds one."""
    rng = np.random.default_rng(18)
    x = np.full((1, 24576), -36.0, np.float32)
    x[:, :2000] = rng.standard_normal((1, 2000))
    for p in (1.0, 0.9999999):
        assert _check(sr, x, np.ones(1, np.float32), None, None, np.full(1, p, np.float32), None).tolist() == [1999]


def test_rows_beyond_32_bits(sr):
    """Rows so far apart that their offsets pass 2^32 elements; further apart than 2^31 they are refused."""
    import torch
    rng = np.random.default_rng(17)
    x = _logits(rng, 3, 5000)
    buf = torch.empty(2 * 2_200_000_000 + 5000, dtype=torch.float32, device="cuda")
    X = buf.as_strided((3, 5000), (2_200_000_000, 1))
    with pytest.raises(sr.SiriusError, match="apart"):
        sr.sirius_sample(X, dev_f32(np.zeros(3)))
    X = buf.as_strided((3, 5000), (2 ** 31, 1))
    X.copy_(dev_f32(x))
    _check(sr, x, rng.random(3), np.full(3, 0.9, np.float32), np.array([0, 20, 300]), np.array([0.9, 0.9, 1.0], np.float32), None, X=X)


def test_bad_parameters_give_no_token(sr):
    x = np.zeros((7, 10), np.float32)
    t = np.array([-1, np.nan, np.inf, 1, 1, 1, 1], np.float32)
    p = np.array([1, 1, 1, np.nan, 1, 1, 1], np.float32)
    m = np.array([0, 0, 0, 0, np.nan, 0, 0], np.float32)
    u = np.array([0.5, 0.5, 0.5, 0.5, 0.5, np.nan, 0.55], np.float32)
    tok, kept, prob = sr.sirius_sample(dev_f32(x), dev_f32(u), temperature=dev_f32(t), top_p=dev_f32(p), min_p=dev_f32(m))
    assert host(tok).tolist() == [-1] * 6 + [5] and host(kept).tolist() == [0] * 6 + [10] and (host(prob)[:6] == 0).all()


def test_strides_scalars_and_repeats(sr):
    import torch
    rng = np.random.default_rng(7)
    for wide, off in ((2051, 0), (2048, 4), (2500, 0)):
        x = _logits(rng, 9, wide)
        X = dev_f32(x)[:, off:off + 1999]
        u = rng.random(9)
        _check(sr, np.ascontiguousarray(x[:, off:off + 1999]), u, np.full(9, 0.8, np.float32), np.full(9, 60), np.full(9, 0.9, np.float32),
               None, X=X)
        one = sr.sirius_sample(X, dev_f32(u), temperature=0.8, top_k=60, top_p=0.9)
        two = sr.sirius_sample(X.contiguous(), dev_f32(u), temperature=0.8, top_k=60, top_p=0.9)
        for a, b in zip(one, two):
            assert torch.equal(a, b)
    t, k, p = sr.sirius_sample(dev_f32(np.zeros((0, 5), np.float32)), dev_f32(np.zeros(0)))
    assert t.numel() == 0


def test_frequencies_follow_the_probabilities(sr):
    """20000 draws from one row of six tokens: each share within five standard deviations."""
    x = np.log(np.array([0.05, 0.3, 0.1, 0.25, 0.2, 0.1])).astype(np.float32)
    n = 20000
    u = np.random.default_rng(11).random(n).astype(np.float32)
    tok = host(sr.sirius_sample(dev_f32(np.repeat(x[None], n, 0)), dev_f32(u), top_k=4)[0])
    share = np.bincount(tok, minlength=6) / n
    want = np.array([0, 0.3, 0.1, 0.25, 0.2, 0]) / 0.85
    assert (np.abs(share - want) <= 5 * np.sqrt(want * (1 - want) / n)).all(), share
