"""Refusals of the serving-step entry points, on the host before anything is enqueued."""

import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(
    not os.path.exists(os.path.join(ROOT, "paper_2409_03856_amd", "libsirius.so")),
    reason="libsirius.so not built (run __graft_entry__.build())")

FAKE = ctypes.c_void_p(1 << 20)  # non-null, 16-byte aligned; never dereferenced by these calls
ODD = ctypes.c_void_p((1 << 20) + 8)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2409_03856_amd import _lib
    return _lib


class RotationC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("freqs", "q_weight", "k_weight")] + \
               [("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int), ("mscale", ctypes.c_float), ("norm_eps", ctypes.c_float)]


class PagedC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "page_table", "cache_pos", "tok_start")] + \
               [(n, ctypes.c_int) for n in ("B", "T", "max_n", "n_kv_heads", "head_dim", "n_pages", "page_size", "max_pages")]


def test_the_binding_packs_the_structs(lib):
    assert lib._ROTATION.size == ctypes.sizeof(RotationC) and lib._PAGED.size == ctypes.sizeof(PagedC)
    r = RotationC.from_buffer_copy(lib._ROTATION.pack(8, 16, 24, 64, 1, 1.5, -1.0))
    assert (r.freqs, r.q_weight, r.k_weight, r.rot_dim, r.interleaved, r.mscale, r.norm_eps) == (8, 16, 24, 64, 1, 1.5, -1.0)
    c = PagedC.from_buffer_copy(lib._PAGED.pack(*range(1, 14)))
    assert [getattr(c, n) for n, _ in PagedC._fields_] == list(range(1, 14))


def _rotation(lib, **kw):
    r = dict(freqs=1 << 20, q_weight=None, k_weight=None, rot_dim=64, interleaved=0, mscale=1.0, norm_eps=-1.0)
    return RotationC(*(r | kw).values())


def _paged(lib, **kw):
    c = dict(k_pages=1 << 20, v_pages=1 << 21, page_table=1 << 20, cache_pos=1 << 20, tok_start=None, B=2, T=6, max_n=3,
             n_kv_heads=2, head_dim=64, n_pages=9, page_size=16, max_pages=4)
    return PagedC(*(c | kw).values())


BAD_ROTATIONS = [dict(rot_dim=7), dict(rot_dim=66), dict(rot_dim=-2), dict(freqs=None), dict(mscale=NAN), dict(mscale=INF),
                 dict(norm_eps=NAN), dict(norm_eps=INF), dict(q_weight=(1 << 20) + 2), dict(freqs=(1 << 20) + 8)]
BAD_CACHES = [dict(k_pages=None), dict(v_pages=None), dict(k_pages=(1 << 20) + 8), dict(page_table=None), dict(cache_pos=None),
              dict(B=-1), dict(B=65536, T=65536 * 3), dict(T=-1), dict(T=5), dict(T=(1 << 20) + 1, max_n=1 << 20, B=1),
              dict(max_n=-1), dict(n_kv_heads=0), dict(head_dim=12), dict(head_dim=136), dict(n_pages=0), dict(page_size=12),
              dict(page_size=0), dict(page_size=4104), dict(max_pages=0), dict(max_pages=65537)]


def test_rope_refusals(lib):
    L = lib.lib()
    base = dict(q=FAKE, qt=0, ldq=256, k=FAKE, kt=1, ldk=128, pos=FAKE, T=3, H=4, Hkv=2, hd=64, rot=_rotation(lib), qo=FAKE, ko=FAKE)

    def call(**kw):
        a = base | kw
        a["rot"] = None if a["rot"] is None else ctypes.byref(a["rot"])
        return L.sirius_rope(*a.values(), None)

    for kw in (dict(q=None, k=None), dict(q=ODD), dict(qo=None), dict(qo=ODD), dict(k=ODD), dict(ko=None), dict(pos=None), dict(qt=2),
               dict(kt=-1), dict(ldq=255), dict(ldq=252), dict(ldq=260), dict(ldk=64), dict(T=-1), dict(T=(1 << 20) + 1), dict(H=0),
               dict(H=4097), dict(Hkv=0), dict(hd=60), dict(hd=0), dict(hd=136), dict(rot=None)):
        assert call(**kw) == -1, kw
    for kw in BAD_ROTATIONS:
        assert call(rot=_rotation(lib, **kw)) == -1, kw
    assert call(T=0, q=None, k=None) == 0


def test_append_refusals(lib):
    L = lib.lib()
    base = dict(q=FAKE, qt=0, ldq=256, k=FAKE, v=FAKE, kt=1, ldk=128, ldv=128, cache=_paged(lib), pos=None, H=4,
                rot=_rotation(lib), qo=FAKE)

    def call(**kw):
        a = base | kw
        for n in ("rot", "cache"):
            a[n] = None if a[n] is None else ctypes.byref(a[n])
        return L.sirius_kv_append(*a.values(), None)

    for kw in (dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD), dict(q=ODD), dict(qo=None), dict(qt=3), dict(kt=2), dict(ldk=120),
               dict(ldv=132), dict(ldq=128), dict(H=0), dict(cache=None)):
        assert call(**kw) == -1, kw
    for kw in BAD_CACHES:
        assert call(cache=_paged(lib, **kw)) == -1, kw
    for kw in BAD_ROTATIONS:
        assert call(rot=_rotation(lib, **kw)) == -1, kw
    for kw in (dict(T=0, B=0), dict(T=0, max_n=0), dict(T=0, tok_start=1 << 20)):
        assert call(cache=_paged(lib, **kw), k=None) == 0, kw


def test_binding_refusals(lib):
    """Shapes and types that the binding turns away before the library sees them (tensors on the CPU are among them)."""
    import torch
    x = torch.zeros(3, 4, 64)
    pos = torch.zeros(3, dtype=torch.int32)
    f = torch.ones(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="GPU"):
        lib.sirius_rope(x, x, pos, f)
    with pytest.raises(ValueError):
        lib.sirius_rope(None, None, pos, f)
    with pytest.raises(ValueError):
        lib.sirius_rope(x[0], None, pos, f)
    pages, table = torch.zeros(2, 4, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        lib.sirius_kv_append(None, x, x, pages, pages.transpose(2, 3), table, pos[:1], f)
    with pytest.raises(ValueError):
        lib.sirius_rope_freqs(64, scaling="half")
    with pytest.raises(ValueError):
        lib.sirius_rope_freqs(0)
    with pytest.raises(lib.SiriusError):
        lib.sirius_rope_freqs(64, 0.5)


def test_attention_refusals(lib):
    L = lib.lib()
    base = dict(q=FAKE, qt=0, ldq=256, cache=_paged(lib), H=4, scale=0.0, cap=0.0, slopes=None, window=0, mask=None, out=FAKE,
                ws=FAKE, n=1 << 30)

    def call(**kw):
        a = base | kw
        a["cache"] = None if a["cache"] is None else ctypes.byref(a["cache"])
        return L.sirius_attn_paged(*a.values(), None)

    for kw in (dict(q=None), dict(q=ODD), dict(out=None), dict(out=ODD), dict(ws=None), dict(qt=2), dict(ldq=248), dict(H=3), dict(H=0),
               dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(cap=-1.0), dict(cap=NAN), dict(cap=INF), dict(window=-1),
               dict(cache=None), dict(mask=FAKE, cache=_paged(lib, max_n=65, T=130))):
        assert call(**kw) == -1, kw
    for kw in BAD_CACHES:
        assert call(cache=_paged(lib, **kw)) == -1, kw
    assert call(n=16) == -2
    for kw in (dict(T=0, B=0), dict(T=0, max_n=0), dict(T=0, tok_start=1 << 20)):
        assert call(cache=_paged(lib, **kw), q=None) == 0, kw
    size = lambda *a: L.sirius_workspace_size(10, *a)
    assert size(2, 3, 4 * 65536 + 2, 64, 0) > 0 and size(0, 0, 4 * 65536 + 2, 64, 0) > 0
    for a in ((-1, 3, 4 * 65536 + 2, 64, 0), (2, -1, 4 * 65536 + 2, 64, 0), (2, 3, 3 * 65536 + 2, 64, 0), (2, 3, 4 * 65536 + 2, 60, 0)):
        assert size(*a) == 0, a


def test_sampling_refusals(lib):
    L = lib.lib()
    base = dict(logits=FAKE, ld=100, B=2, V=100, u=FAKE, t=None, k=None, p=None, m=None, token=FAKE, kept=None, prob=None, ws=FAKE,
                n=1 << 30)
    call = lambda **kw: L.sirius_sample(*(base | kw).values(), None)
    for kw in (dict(logits=None), dict(logits=ODD), dict(u=None), dict(token=None), dict(ws=None), dict(B=-1), dict(B=65536), dict(V=0),
               dict(V=(1 << 24) + 1, ld=1 << 25), dict(ld=99), dict(ld=-1)):
        assert call(**kw) == -1, kw
    assert call(n=0) == -2
    assert call(B=0, logits=None) == 0
    assert L.sirius_workspace_size(11, 2, 0, 0, 100, 0) > 0 and L.sirius_workspace_size(11, 2, 0, 0, 0, 0) == 0
    import torch
    x = torch.zeros(2, 10)
    with pytest.raises(ValueError, match="GPU"):
        lib.sirius_sample(x, x[:, 0].contiguous())
    with pytest.raises(ValueError, match="fp32"):
        lib.sirius_sample(x.double(), x[:, 0].contiguous())


def test_calls_with_more_threads_than_a_launch_holds(lib):
    """Sizes inside every single limit whose product would pass 2^32 threads are refused, not launched."""
    L = lib.lib()
    wide = dict(B=1, T=1 << 20, max_n=1 << 20, n_kv_heads=4096, head_dim=8, max_pages=65536, page_size=16)
    cache = _paged(lib, **wide)
    rot = _rotation(lib, rot_dim=8)
    assert L.sirius_kv_append(None, 0, 0, FAKE, FAKE, 1, 32768, 32768, ctypes.byref(cache), None, 0, ctypes.byref(rot), None, None) == -1
    assert b"too many" in L.sirius_last_error()
    cache = _paged(lib, **(wide | dict(B=400, tok_start=1 << 20, n_kv_heads=64)))
    assert L.sirius_attn_paged(FAKE, 0, 512, ctypes.byref(cache), 64, 0.0, 0.0, None, 0, None, FAKE, FAKE, (1 << 63), None) == -1
    assert b"too many" in L.sirius_last_error()
    v = 1 << 24
    assert L.sirius_sample(FAKE, v, 65535, v, FAKE, None, None, None, None, FAKE, None, None, FAKE, (1 << 63), None) == -1
    assert b"too many" in L.sirius_last_error()
