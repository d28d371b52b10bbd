"""GPU parity: long tails of weights that lie beside half a unit of the sums.

Weights are added as whole numbers of 2^-s of the best one's, s = min(50, 62 - ceil(log2 V)), so each is off by half a unit
at most and a sum over V tokens by V / 2 units. The kept mass is at least the best one's weight: a border of u, and a
token's share, move by V / 2 2^-s at most (2^-21 for 2^21 tokens, 2^-29 for 128256). A tail of equal weights just
beside half a unit reaches it. prob is rounded to fp32 once more. Counts are exact.
"""

import math

import numpy as np
import pytest

from oracle import serve
from gpu_util import say, dev_f32, dev_i32, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


@pytest.mark.parametrize("v", [8192, 128256, 1 << 21])
@pytest.mark.parametrize("beside", [0.99, 1.01])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.999), (1000, 1.0), (50, 1.0)])
def test_tails_beside_half_a_unit(sr, v, beside, k, p):
    s = min(50, 62 - math.ceil(math.log2(v)))
    off = v / 2 * 2.0 ** -s
    x = np.full((4, v), math.log(beside * 2.0 ** -(s + 1)), np.float32)
    x[0, 0] = x[1, v // 2] = x[2, v - 1] = x[3, 7] = 0.0
    u = np.array([1.0 - 2.0 ** -24, 0.5, 0.3, 1.0], np.float32)
    tok, kept, prob = (host(t) for t in sr.sirius_sample(dev_f32(x), dev_f32(u), top_k=dev_i32(np.full(4, k)),
                                                         top_p=dev_f32(np.full(4, p))))
    for b in range(4):
        want = serve.sample(x[b], float(u[b]), top_k=k, top_p=float(np.float32(p)))
        assert kept[b] == want[1], (b, kept[b], want)
        first, last = (serve.sample(x[b], min(max(float(u[b]) + d, 0.0), 1.0), top_k=k, top_p=float(np.float32(p)))[0] for d in (-2 * off, 2 * off))
        assert first <= tok[b] <= last, (b, tok[b], first, last)
        share = 1.0 / (1.0 + (want[1] - 1) * math.exp(float(x[b].min()))) if x[b, tok[b]] == 0.0 else 0.0
        assert abs(prob[b] - share) <= 2.0 ** -24 * share + 2 * off, (b, prob[b], share)
    say(f"  V={v} s={s} {beside} of half a unit, k={k} p={p}: tokens {tok.tolist()}")


@pytest.mark.parametrize("v", [9000, 128256, 1 << 21])
def test_the_last_token_of_positive_mass_at_one(sr, v):
    """A chunk's tokens of half a unit and more count as one each, so that they sum to more than the chunk's share of the
    row: u = 1 draws the last of them all the same, with every filter that leaves it."""
    s = min(50, 62 - math.ceil(math.log2(v)))
    x = np.full((3, v), math.log(1.01 * 2.0 ** -(s + 1)), np.float32)
    x[0, 0] = x[1, v // 2] = x[2, 7] = 0.0
    x[2, v - 100:] = -np.inf
    u = dev_f32(np.ones(3))
    for kw in (dict(), dict(min_p=1e-30), dict(top_k=v - 200), dict(temperature=0.999)):
        tok, kept, _ = (host(t).tolist() for t in sr.sirius_sample(dev_f32(x), u, **kw))
        if "temperature" in kw:  # each below half a unit then: the best one alone has mass
            assert tok == [0, v // 2, 7], (kw, tok)
        elif "top_k" in kw:  # the first of the tied ones stay
            assert tok == [v - 201] * 3, (kw, tok)
            assert kept == [v - 200] * 3
        else:
            assert tok == [v - 1, v - 1, v - 101], (kw, tok)
