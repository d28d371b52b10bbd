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


class PagedC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "page_table", "cache_pos", "tok_start")] + \
               [(n, ctypes.c_int) for n in ("B", "T", "max_n", "n_kv_heads", "head_dim", "n_pages", "page_size", "max_pages")]


def test_paged_attention_workspace_of_the_largest_call_serves_the_smaller_ones(L):
    size = lambda b, n, k, g, hd: L.sirius_workspace_size(10, b, n, (k * g << 16) + k, hd, 0)

    def need(b, n, k, g, hd):
        p = FAKE.value
        cache = PagedC(p, p, p, p, p, b, b * n, n, k, hd, 9, 16, 4)
        return max(_needed(L, L.sirius_attn_paged(FAKE, t, k * g * hd, ctypes.byref(cache), k * g, 0.0, 0.0, None, 0, None, FAKE, FAKE, 0,
                                                  None)) for t in (0, 1))

    for k, g, hd in ((8, 4, 128), (1, 1, 64), (1, 8, 128), (40, 1, 128), (3, 5, 80), (255, 1, 8), (257, 2, 8), (512, 1, 8)):
        sizes = [size(5, n, k, g, hd) for n in range(0, 1500)]
        assert sizes == sorted(sizes) and sizes[0] > 0, (k, g, hd)
        assert all(need(5, n, k, g, hd) <= sizes[n] for n in range(1, 1500)), (k, g, hd)
    rng = random.Random(6)
    for _ in range(4000):
        k, g, hd = rng.randint(1, 64), rng.randint(1, 16), 8 * rng.randint(1, 16)
        b, n = int(2 ** rng.uniform(0, 10)), int(2 ** rng.uniform(0, 10))
        most = size(b, n, k, g, hd)
        for c in ((rng.randint(1, b), n), (b, rng.randint(1, n)), (rng.randint(1, b), rng.randint(1, n))):
            assert need(*c, k, g, hd) <= size(*c, k, g, hd) <= most, (c, (b, n, k, g, hd))
