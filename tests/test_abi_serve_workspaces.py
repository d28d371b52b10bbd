"""Workspace sizes of the serving step on the host: what is reserved for the largest call serves every smaller one."""

import ctypes
import os
import random
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(
    not os.path.exists(os.path.join(ROOT, "paper_2409_03856_amd", "libsirius.so")),
    reason="libsirius.so not built (run __graft_entry__.build())")

FAKE = ctypes.c_void_p(1 << 20)  # non-null, 16-byte aligned; these calls are refused before it is used


@pytest.fixture(scope="module")
def L():
    from paper_2409_03856_amd import _lib
    return _lib.lib()


def _needed(L, rc):
    """Bytes that a call with too small a workspace says it needs."""
    assert rc == -2
    return int(re.search(rb"< (\d+) needed", L.sirius_last_error()).group(1))


def test_sampling_workspace_of_the_largest_call_serves_the_smaller_ones(L):
    size = lambda b, v: L.sirius_workspace_size(11, b, 0, 0, v, 0)
    need = lambda b, v: _needed(L, L.sirius_sample(FAKE, v, b, v, FAKE, None, None, None, None, FAKE, None, None, FAKE, 0, None))
    for v in (1, 2048, 8193, 32000, 128256, 2097152, 2097153, 1 << 24):  # the chunks' size changes on the way
        sizes = [size(b, v) for b in range(1, 300)]
        assert sizes == sorted(sizes) and sizes[0] > 0, v
        assert all(need(b, v) <= sizes[b - 1] for b in range(1, 300)), v
    rng = random.Random(5)
    for _ in range(3000):
        b, v = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 20))
        most = size(b, v)
        for c in ((rng.randint(1, b), v), (b, rng.randint(1, v)), (rng.randint(1, b), rng.randint(1, v))):
            assert need(*c) <= size(*c) <= most, (c, b, v)
