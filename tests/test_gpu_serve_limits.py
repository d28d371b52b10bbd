"""GPU parity at the documented ends: a sequence of 2^20 cache rows, a vocabulary of 2^24, 4096 heads, 65535 sequences.

References are 64-bit torch operations on the GPU. Tolerances: fp32 attention 1e-4 of the output's root mean square, as
everywhere (each weight is off by its score's rounding, below 60 2^-24 here, and what a million of them sum to by as much
relative to the root mean square); the append writes roundings of the inputs; a token and its count are equal, u
lying further than V / 2 2^-38 = 2^-15 of the best weight from the token's borders.
"""

import numpy as np
import pytest

from oracle import serve
from gpu_util import dev_f32, dev_i32, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sr():
    import paper_2409_03856_amd as sr
    sr.lib()
    return sr


@pytest.mark.parametrize("page", [8, 4096])
def test_the_last_row_of_the_longest_sequence(sr, page):
    import torch
    rows, h, hd = 1 << 20, 4, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    kp = torch.randn(rows // page, 1, page, hd, generator=g, device="cuda", dtype=torch.bfloat16)
    vp = torch.randn(rows // page, 1, hd, page, generator=g, device="cuda", dtype=torch.bfloat16)
    table = torch.randperm(rows // page, generator=g, device="cuda").to(torch.int32)[None].contiguous()
    q, k, v = (torch.randn(2, n, hd, generator=g, device="cuda") for n in (h, 1, 1))
    pos = dev_i32(np.array([rows - 2]))
    assert sr.sirius_kv_append(None, k, v, kp, vp, table, pos) is None
    keys = kp[table[0].long()].reshape(rows, hd).double()
    values = vp[table[0].long()].transpose(2, 3).reshape(rows, hd).double()
    assert torch.equal(keys[-2:], k[:, 0].to(torch.bfloat16).double()) and torch.equal(values[-2:], v[:, 0].to(torch.bfloat16).double())
    got = sr.sirius_attn_paged(q, kp, vp, table, pos).double()
    for i in range(2):
        x = q[i].double() @ keys[: rows - 1 + i].T.contiguous() / 8.0
        want = torch.softmax(x, 1) @ values[: rows - 1 + i]
        assert float((got[i] - want).abs().max()) <= 1e-4 * float(want.square().mean().sqrt())
    # one row further there is no place
    pos += 1
    before = kp.clone()
    sr.sirius_kv_append(None, k, v, kp, vp, table, pos)
    assert torch.equal(before, kp) and bool(sr.sirius_attn_paged(q, kp, vp, table, pos).isnan().all())


def test_the_largest_vocabulary(sr):
    import torch
    n = 1 << 24
    g = torch.Generator(device="cuda").manual_seed(2)
    x = 2.5 * torch.randn(2, n, generator=g, device="cuda")
    x[:, torch.randperm(n, generator=g, device="cuda")[:2000]] += 8.0
    u = np.array([0.3, 0.8], np.float32)
    tok, kept, prob = (host(t) for t in sr.sirius_sample(x, dev_f32(u), top_k=50, top_p=0.9))
    for b in range(2):
        best = torch.topk(x[b], 200).indices.sort().values
        want = serve.sample(host(x[b][best]), float(u[b]), top_k=50, top_p=float(np.float32(0.9)))
        assert (int(tok[b]), int(kept[b])) == (int(best[want[0]]), want[1])
    tok, kept, prob = (host(t) for t in sr.sirius_sample(x, dev_f32(u)))
    for b in range(2):
        w = (x[b].double() - x[b].max().double()).exp()
        run = w.cumsum(0)
        t, at = int(tok[b]), float(u[b]) * float(run[-1])
        assert kept[b] == n and float(run[t - 1]) - 2.0 ** -15 <= at < float(run[t]) + 2.0 ** -15
        assert abs(float(prob[b]) - float(w[t] / run[-1])) <= 2.0 ** -24 * float(prob[b]) + 2.0 ** -15 / float(run[-1])


def test_the_most_heads_and_sequences(sr):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    for h, hkv, b, per in ((4096, 4096, 1, 3), (4096, 1, 2, 3), (2, 1, 65535, 1)):
        kp = torch.randn(b * per, hkv, 8, 8, generator=g, device="cuda", dtype=torch.bfloat16)
        vp = torch.randn(b * per, hkv, 8, 8, generator=g, device="cuda", dtype=torch.bfloat16)
        table = torch.randperm(b * per, generator=g, device="cuda").to(torch.int32).view(b, per)
        pos = torch.randint(0, 8 * per, (b,), generator=g, device="cuda").to(torch.int32)
        q = torch.randn(b, h, 8, generator=g, device="cuda")
        got = sr.sirius_attn_paged(q, kp, vp, table, pos).double()
        keys = kp[table.long()].double().transpose(1, 2).reshape(b, hkv, 8 * per, 8)
        values = vp[table.long()].double().permute(0, 2, 1, 4, 3).reshape(b, hkv, 8 * per, 8)
        x = torch.matmul(q.double().view(b, hkv, h // hkv, 8), keys.transpose(2, 3).contiguous()) / 8.0 ** 0.5
        x = x.masked_fill(torch.arange(8 * per, device="cuda") > pos[:, None, None, None], -torch.inf)
        want = torch.matmul(torch.softmax(x, -1), values).reshape(b, h, 8)
        assert float((got - want).abs().max()) <= 1e-4 * float(want.square().mean().sqrt())
