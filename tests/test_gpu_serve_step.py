"""The serving step as it is used: append, attention, sampling and rollback, step after step over one paged cache,
against the 64-bit oracle; the same calls captured into a graph; calls on two streams and from two threads.
"""

import threading

import numpy as np
import pytest

import oracle
from oracle import serve
from synth import bf16_bits
from gpu_util import say, dev_bf16, dev_f32, dev_i32, host

pytestmark = pytest.mark.gpu

H, HKV, HD, PAGE, VOCAB = 8, 2, 64, 16, 501


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


class Step:
    """One layer's weights, a cache for `bsz` sequences, and both sides' steps."""

    def __init__(self, sr, bsz, rows, seed=1):
        self.sr, self.bsz = sr, bsz
        rng = np.random.default_rng(seed)
        self.rng = rng
        per = -(-rows // PAGE)
        pages = bsz * per + 1
        self.table = rng.permutation(pages)[: bsz * per].reshape(bsz, per).astype(np.int32)
        self.kp, self.vp = np.zeros((pages, HKV, PAGE, HD)), np.zeros((pages, HKV, HD, PAGE))
        self.Kp, self.Vp = (dev_bf16(np.zeros(s, np.uint16)) for s in (self.kp.shape, self.vp.shape))
        self.Table = dev_i32(self.table)
        self.wq, self.wk = (bf16_bits((1 + 0.2 * rng.standard_normal(HD)).astype(np.float32)) for _ in range(2))
        self.head = (rng.standard_normal((H * HD, VOCAB)) / 20).astype(np.float32)
        self.Wq, self.Wk, self.Head = dev_bf16(self.wq), dev_bf16(self.wk), dev_f32(self.head)
        self.freqs = sr.sirius_rope_freqs(HD, 500000.0, scaling="smooth", factor=8.0)
        self.f = host(self.freqs)
        self.norm = dict(norm_eps=1e-6, q_weight=self.Wq, k_weight=self.Wk)

    def inputs(self, t):
        q = self.rng.standard_normal((t, H, HD)).astype(np.float32)
        k, v = self.rng.standard_normal((2, t, HKV, HD)).astype(np.float32)
        return q, bf16_bits(k), bf16_bits(v)

    def device(self, q, k, v, pos, start=None, **attn):
        """The step on the GPU from device inputs: (attention, logits of every token)."""
        qr = self.sr.sirius_kv_append(q, k, v, self.Kp, self.Vp, self.Table, pos, self.freqs, tok_start=start, **self.norm)
        out = self.sr.sirius_attn_paged(qr, self.Kp, self.Vp, self.Table, pos, tok_start=start, **attn)
        return out, out.reshape(-1, H * HD) @ self.Head

    def plain(self, q, k, v, pos, start, **attn):
        """The same in 64 bits; keys and values are what the cache holds (the GPU's roundings of the oracle's)."""
        places = serve.places(pos, start, self.table, PAGE, self.kp.shape[0])
        rows = np.array([r for _, _, r, _ in places])
        qr = serve.rope(q, rows, self.f, norm_eps=1e-6, weight=self.wq)
        kr = serve.rope(k, rows, self.f, norm_eps=1e-6, weight=self.wk)
        held = oracle.widen_bf16(host(self.Kp))
        for t, b, row, pg in places:
            got = held[pg, :, row % PAGE]
            assert np.max(np.abs(got - kr[t])) <= 2.0 ** -8 * np.max(np.abs(kr[t])) + 1e-5
            self.kp[pg, :, row % PAGE] = got
            self.vp[pg, :, :, row % PAGE] = oracle.widen_bf16(v[t])
        assert np.array_equal(oracle.widen_bf16(host(self.Vp)), self.vp)
        return serve.attn_paged(qr, self.kp, self.vp, self.table, pos, start, **attn)


def _close(got, want):
    rms = float(np.sqrt(np.mean(want * want)))
    assert float(np.max(np.abs(got - want))) <= 1e-4 * rms


def test_prompt_drafts_check_and_sampling(sr):
    """Prompts of three lengths, four drafted tokens one by one, the check's pass over the chunk that rewrites their
    rows, rollback to what each accepts, a sampled token: the positions, the cache and every output follow."""
    s = Step(sr, 3, 80)
    prompts = [17, 1, 30]
    start = np.cumsum([0] + prompts).astype(np.int32)
    pos = np.zeros(3, np.int32)
    Pos = dev_i32(pos)
    q, k, v = s.inputs(sum(prompts))
    out, _ = s.device(dev_f32(q), dev_bf16(k), dev_bf16(v), Pos, dev_i32(start), max_n=30)
    _close(host(out), s.plain(q, k, v, pos, start))
    pos = pos + np.array(prompts, np.int32)
    Pos += dev_i32(np.array(prompts, np.int32))
    n = 4
    for period, accept in enumerate(([0, 2, 4], [3, 4, 1])):
        one = np.arange(4, dtype=np.int32)
        at = pos.copy()
        for i in range(n):
            q, k, v = s.inputs(3)
            out, logits = s.device(dev_f32(q), dev_bf16(k), dev_bf16(v), Pos)
            _close(host(out), s.plain(q, k, v, at, one))
            u = s.rng.random(3).astype(np.float32)
            tok, kept, prob = sr.sirius_sample(logits, dev_f32(u), temperature=0.8, top_k=40, top_p=0.95)
            lg = host(logits)
            for b in range(3):
                want = serve.sample(lg[b], float(u[b]), float(np.float32(0.8)), 40, float(np.float32(0.95)))
                assert (int(host(tok)[b]), int(host(kept)[b])) == want[:2]
            sr.sirius_kv_rollback(Pos, dev_i32(np.zeros(3, np.int32)), 1)
            at = at + 1
        Pos -= n
        q, k, v = s.inputs(3 * n)
        out, _ = s.device(dev_f32(q), dev_bf16(k), dev_bf16(v), Pos)
        _close(host(out), s.plain(q, k, v, pos, np.arange(4, dtype=np.int32) * n))
        sr.sirius_kv_rollback(Pos, dev_i32(np.array(accept, np.int32)), n)
        pos = oracle.kv_rollback(pos, accept, n).astype(np.int32)
        assert host(Pos).tolist() == pos.tolist()
        say(f"period {period}: positions {pos.tolist()}")


def test_tree_pass_feeds_the_tree_check(sr):
    """Nodes of a drafted tree at their depths' positions under their ancestors' bits: each node's output is that of
    its path run as a chain."""
    s = Step(sr, 1, 200, seed=3)
    q, k, v = s.inputs(50)
    s.device(dev_f32(q), dev_bf16(k), dev_bf16(v), dev_i32([0]))
    w, levels = 3, 4
    n = w * levels
    parents = np.array([[s.rng.integers(w) for _ in range(w)] for _ in range(levels)])
    bits = [0] * n
    for i in range(n):
        up = bits[(i // w - 1) * w + parents[i // w][i % w]] if i >= w else 0
        bits[i] = up | 1 << i
    q, k, v = s.inputs(n)
    import torch
    depth = np.array([50 + i // w for i in range(n)], np.int32)
    Pos = dev_i32([50])
    qr = sr.sirius_kv_append(dev_f32(q), dev_bf16(k), dev_bf16(v), s.Kp, s.Vp, s.Table, Pos, s.freqs, positions=dev_i32(depth), **s.norm)
    tree = host(sr.sirius_attn_paged(qr, s.Kp, s.Vp, s.Table, Pos, mask=torch.tensor(bits, dtype=torch.int64).cuda()))
    for leaf in range(n - w, n):
        path = [i for i in range(n) if bits[leaf] >> i & 1]
        out, _ = s.device(dev_f32(q[path]), dev_bf16(k[path]), dev_bf16(v[path]), Pos)
        _close(tree[path], host(out).astype(np.float64))


def test_captured_step_replays(sr):
    """A step captured once and replayed on new inputs with eager work between gives the eager results every time,
    while a second graph of the same calls lives."""
    import torch
    s = Step(sr, 4, 400, seed=5)
    q, k, v = s.inputs(4 * 90)
    Pos = dev_i32(np.zeros(4, np.int32))
    s.device(dev_f32(q), dev_bf16(k), dev_bf16(v), Pos)
    Pos += 90
    q, k, v = (dev_f32(x) if x.dtype == np.float32 else dev_bf16(x) for x in s.inputs(4))
    u = dev_f32(np.full(4, 0.5, np.float32))
    params = dict(temperature=dev_f32(np.full(4, 0.9, np.float32)), top_k=dev_i32(np.array([0, 5, 300, 50])),
                  top_p=dev_f32(np.array([0.9, 1.0, 0.8, 0.95], np.float32)), min_p=dev_f32(np.array([0.0, 0.0, 0.01, 0.1], np.float32)))

    def step():
        out, logits = s.device(q, k, v, Pos)
        return (out,) + tuple(sr.sirius_sample(logits, u, **params))

    step()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    for i in range(4):
        a, b, c = s.inputs(4)
        q.copy_(dev_f32(a))
        k.copy_(dev_bf16(b))
        v.copy_(dev_bf16(c))
        u.copy_(dev_f32(s.rng.random(4)))
        eager = [t.clone() for t in step()]
        for g, o in zip(graphs, outs):
            for t in o:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(eager, o)), i
        Pos += 1


def test_two_streams_and_two_threads(sr):
    """Calls that are not ordered to each other share no workspace: bit for bit what each gives alone."""
    import torch
    calls = []
    for i in range(2):
        s = Step(sr, 6, 900, seed=20 + i)
        q, k, v = s.inputs(6 * 700)
        Pos = dev_i32(np.zeros(6, np.int32))
        s.device(dev_f32(q), dev_bf16(k), dev_bf16(v), Pos)
        Pos += 700
        qd, x, u = dev_f32(s.inputs(6)[0]), dev_f32(3 * s.rng.standard_normal((40, 30000))), dev_f32(s.rng.random(40))

        def call(s=s, qd=qd, x=x, u=u, Pos=Pos, **kw):
            return (sr.sirius_attn_paged(qd, s.Kp, s.Vp, s.Table, Pos, **kw),) + tuple(sr.sirius_sample(x, u, top_p=0.9, **kw))

        calls.append(call)
    want = [[t.clone() for t in c()] for c in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [c(stream=st) for c, st in zip(calls, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    found = [None, None]

    def run(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(5):
                found[i] = calls[i]()
        streams[i].synchronize()

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    for a, b in zip(found, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_pages_beyond_32_bits(sr):
    """Pages whose elements lie beyond 2^32: what is appended there and read back is bit for bit a small pool's."""
    import torch
    rng = np.random.default_rng(9)
    hkv, hd, page = 8, 128, 64
    high = 2 ** 32 // (hkv * hd * page) + 3
    used = [high - 1, 0, high - 2, 1, high // 2 + 1, high - 3]
    shape = {"k": (hkv, page, hd), "v": (hkv, hd, page)}
    pos, start = np.array([70, 100], np.int32), np.array([0, 50, 51], np.int32)
    q = rng.standard_normal((51, 16, hd)).astype(np.float32)
    k, v = (bf16_bits(rng.standard_normal((51, hkv, hd)).astype(np.float32)) for _ in range(2))
    old = {n: dev_bf16(bf16_bits(rng.standard_normal((6,) + shape[n]).astype(np.float32))) for n in "kv"}
    got = []
    for ids, pages in ((used, high), (list(range(6)), 6)):
        pools = {n: torch.empty((pages,) + shape[n], dtype=torch.bfloat16, device="cuda") for n in "kv"}
        for n in "kv":
            for j, i in enumerate(ids):
                pools[n][i].copy_(old[n][j])
        table = dev_i32(np.array([ids[:3], ids[3:]], np.int32))
        kv = (pools["k"], pools["v"], table, dev_i32(pos))
        qr = sr.sirius_kv_append(dev_f32(q), dev_bf16(k), dev_bf16(v), *kv, sr.sirius_rope_freqs(hd, 10000.0), tok_start=dev_i32(start))
        out = sr.sirius_attn_paged(qr, *kv, tok_start=dev_i32(start), max_n=50)
        got.append([qr, out] + [pools[n][i].clone() for n in "kv" for i in ids])
        del pools, kv
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert bool(torch.isfinite(got[0][1]).all())
