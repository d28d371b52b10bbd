"""The serving step's operators as they are measured: position rotation, the append to a paged cache, attention over that
cache, and sampling. Where `own` is false, run() computes them by elementary operations; where it is true, by the library.

A serving program holds a pool of cache pages, k_pages [pages, Hkv, page size, head size] and v_pages [pages, Hkv,
head size, page size] (values transposed), a table [sequences, pages per sequence] and each sequence's position. A step
rotates the new tokens' queries and keys, writes keys and values to their pages, attends, and samples from the logits.
Ragged sizes of a case come from the case alone, every value from the seed.
"""

import math
import random

import torch

own = False
DEV = "cuda"
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one decoded token's queries and keys before attention over the contiguous cache: the smallest call
        {"name": "rope_token", "op": "rope", "t": 1, "h": 32, "hkv": 8, "hd": 128, "rot": 128, "inter": False, "norm": False,
         "far": 2048, "scaled": False, "qt": "f32", "kt": "bf16"},
        # the nodes of drafted trees at far positions: part of the head, neighbouring pairs, norms, scaled frequencies
        {"name": "rope_tree", "op": "rope", "t": 520, "h": 24, "hkv": 8, "hd": 96, "rot": 48, "inter": True, "norm": True,
         "far": 900000, "scaled": True, "qt": "f32", "kt": "f32"},
        # a prompt's queries and keys with per-head norms
        {"name": "rope_prompt", "op": "rope", "t": 8192, "h": 32, "hkv": 8, "hd": 128, "rot": 128, "inter": False, "norm": True,
         "far": 8192, "scaled": True, "qt": "bf16", "kt": "bf16"},
        # one decoded token of each of 16 sequences into the cache, every layer and step
        {"name": "append_decode", "op": "append", "b": 16, "n": 1, "ragged": False, "len": 3000, "page": 64, "h": 32, "hkv": 8,
         "hd": 128, "rot": 128, "inter": False, "norm": False, "scaled": False, "qt": "f32", "kt": "bf16"},
        # drafted chunks and prompt pieces of odd lengths together, small odd pages, an odd head
        {"name": "append_ragged", "op": "append", "b": 9, "n": 201, "ragged": True, "len": 1500, "page": 24, "h": 12, "hkv": 2,
         "hd": 80, "rot": 40, "inter": True, "norm": True, "scaled": False, "qt": "f32", "kt": "f32"},
        # a long prompt
        {"name": "append_prompt", "op": "append", "b": 1, "n": 8192, "ragged": False, "len": 0, "page": 64, "h": 32, "hkv": 8,
         "hd": 128, "rot": 128, "inter": False, "norm": True, "scaled": True, "qt": "bf16", "kt": "bf16"},
        # one decoded token over 2048 rows
        {"name": "attn_token", "op": "attn", "b": 1, "n": 1, "ragged": False, "len": 2048, "page": 64, "h": 32, "hkv": 8,
         "hd": 128, "cap": 0.0, "alibi": False, "window": 0, "tree": 0, "qt": "f32"},
        # a decode batch whose contexts go from hundreds of rows to 30000
        {"name": "attn_decode", "op": "attn", "b": 48, "n": 1, "ragged": True, "len": 30000, "page": 16, "h": 32, "hkv": 8,
         "hd": 128, "cap": 0.0, "alibi": False, "window": 0, "tree": 0, "qt": "bf16"},
        # the full model's pass over the drafted trees of eight sequences, capped scores
        {"name": "attn_tree", "op": "attn", "b": 8, "n": 40, "ragged": False, "len": 6000, "page": 64, "h": 32, "hkv": 8,
         "hd": 128, "cap": 50.0, "alibi": False, "window": 0, "tree": 4, "qt": "f32"},
        # two prompts
        {"name": "attn_prompt", "op": "attn", "b": 2, "n": 4500, "ragged": True, "len": 0, "page": 64, "h": 32, "hkv": 8,
         "hd": 128, "cap": 0.0, "alibi": False, "window": 0, "tree": 0, "qt": "bf16"},
        # one token of a small vocabulary, all filters
        {"name": "sample_token", "op": "sample", "b": 1, "v": 32000, "k": 50, "p": 0.9, "m": 0.02, "mixed": False, "ties": False},
        # a batch whose requests ask for different things, from greedy to unfiltered; logits of a 16-bit product
        {"name": "sample_batch", "op": "sample", "b": 192, "v": 128256, "k": 100, "p": 0.95, "m": 0.05, "mixed": True, "ties": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((32, 8, 128), (64, 8, 128), (32, 32, 128), (40, 8, 128), (16, 4, 64), (24, 8, 96), (12, 2, 80), (8, 1, 128))


def _rotation(rng, hd):
    return {"rot": hd if rng.random() < 0.6 else 2 * rng.randint(1, hd // 2), "inter": rng.random() < 0.4, "norm": rng.random() < 0.5,
            "scaled": rng.random() < 0.5, "qt": rng.choice(("f32", "bf16")), "kt": rng.choice(("bf16", "bf16", "f32"))}


def draw(rng):
    op = rng.choice(("rope", "append", "append", "attn", "attn", "attn", "sample", "sample"))
    h, hkv, hd = rng.choice(_HEADS)
    page = rng.choice((8, 16, 24, 32, 64, 128, 200))
    if op == "rope":
        t = _log(rng, 1, 8192 * 32 * 128 // max(32 * 128, h * hd))
        return {"op": op, "t": t, "h": h, "hkv": hkv, "hd": hd, "far": _log(rng, t + 1, 1000000), **_rotation(rng, hd)}
    if op == "append":
        b = _log(rng, 1, 128)
        n = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, 8192 * 4096 // max(4096, h * hd) // b))
        return {"op": op, "b": b, "n": n, "ragged": rng.random() < 0.6, "len": _log(rng, 1, 4000), "page": page,
                "h": h, "hkv": hkv, "hd": hd, **_rotation(rng, hd)}
    if op == "sample":
        v = _log(rng, 500, 160000)
        return {"op": op, "b": _log(rng, 1, max(1, min(256, 24000000 // v))), "v": v, "k": rng.choice((0, _log(rng, 1, 2000))),
                "p": rng.choice((1.0, round(rng.uniform(0.5, 0.99), 3))), "m": rng.choice((0.0, round(rng.uniform(0.01, 0.2), 3))),
                "mixed": rng.random() < 0.5, "ties": rng.random() < 0.5}
    kind = rng.random()
    tree = 0
    if kind < 0.45:  # decode
        b, n, length = _log(rng, 1, 64), 1, _log(rng, 1, 32000)
    elif kind < 0.75:  # drafted chunks, half of them trees
        b, n, length = _log(rng, 1, 16), rng.randint(2, 64), _log(rng, 1, 12000)
        tree = rng.choice((0, rng.randint(2, 8)))
    else:  # prompts, some behind rows that are there already
        b, n = rng.randint(1, 4), _log(rng, 65, 4000)
        length = rng.choice((0, _log(rng, 1, 2000)))
    while b > 1 and b * (length + n) * hkv * hd > 48 * 12000 * 8 * 128:
        b //= 2
    case = {"op": op, "b": b, "n": n, "ragged": rng.random() < 0.6, "len": length, "page": page, "h": h, "hkv": hkv, "hd": hd,
            "cap": rng.choice((0.0, 0.0, 30.0, 50.0)), "alibi": tree == 0 and rng.random() < 0.25,
            "window": rng.choice((0, 0, _log(rng, 16, 4096))), "tree": tree, "qt": rng.choice(("f32", "bf16"))}
    while work(case)["flops"] > 2.0e11:  # what the listed prompts cost
        case["n"] = case["n"] * 4 // 5
    return case


def _ragged(case):
    """Rows in the cache before the step and new tokens of each sequence; the longest are the case's own figures."""
    r = random.Random("%d %d %d" % (case["b"], case["n"], case["len"]))
    before, new = [], []
    for i in range(case["b"]):
        f, g = math.exp(r.uniform(math.log(0.02), 0.0)), r.random()
        before.append(int(case["len"] * (f if i and case["ragged"] else 1.0)))
        new.append(max(1, int(case["n"] * (g if i and case["ragged"] and not case.get("tree") else 1.0))))
    return before, new


# ------------------------------------------------------------------------------------------------ inputs

_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _randn(g, *shape, dtype=torch.float32, std=1.0):
    x = torch.randn(*shape, generator=g, device=DEV, dtype=dtype)
    return x.mul_(std) if std != 1.0 else x


def _rotary(case, g):
    hd, rot = case["hd"], case["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = 500000.0 ** (-2.0 * i / rot)
    m = 1.0
    if case["scaled"]:  # long contexts: slow angles by a factor of 8, fast ones as they are
        turns = 8192.0 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        f, m = f * (keep + (1.0 - keep) / 8.0), 0.1 * math.log(8.0) + 1.0
    s = {"freqs": f.to(DEV), "inter": case["inter"], "mscale": m, "eps": EPS if case["norm"] else -1.0, "qw": None, "kw": None}
    if case["norm"]:
        s["qw"], s["kw"] = ((1.0 + 0.2 * _randn(g, hd)).to(torch.bfloat16) for _ in range(2))
    return s


def _cache(case, g):
    """The pool, the table in a random order of pages (-1 behind a sequence's last) and the sequences' places."""
    before, new = _ragged(case)
    page = case["page"]
    need = [-(-(p + n) // page) for p, n in zip(before, new)]
    pages, wide = sum(need) + 3, max(need) + 1
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).tolist()
    table = torch.full((case["b"], wide), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    start = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)
    hkv, hd = case["hkv"], case["hd"]
    return {"k_pages": _randn(g, pages, hkv, page, hd, dtype=torch.bfloat16), "v_pages": _randn(g, pages, hkv, hd, page, dtype=torch.bfloat16),
            "table": table.to(DEV), "pos": torch.tensor(before, dtype=torch.int32).to(DEV),
            "start": start.to(DEV) if case["ragged"] else None, "t": sum(new), "n": max(new)}


def _tree_bits(case, seed):
    """Each node's ancestors and itself as bits, for trees of `tree` nodes a level; a node's parent is any of the level above."""
    r, bits = random.Random(seed), []
    for _ in range(case["b"]):
        own_bits = []
        for i in range(case["n"]):
            w = case["tree"]
            up = own_bits[(i // w - 1) * w + r.randrange(w)] if i >= w else 0
            own_bits.append(up | 1 << i)
        bits += own_bits
    return torch.tensor([x - (1 << 64) if x >> 63 else x for x in bits], dtype=torch.int64).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op = case["op"]
    s = {"op": op}
    if op == "sample":
        b, v = case["b"], case["v"]
        x = _randn(g, b, v, std=2.5)
        x[:, : max(1, v // 2000)] += 6.0  # the few tokens that a context makes likely
        x = x[:, torch.randperm(v, generator=g, device=DEV)].contiguous()
        s["logits"] = x.to(torch.bfloat16).float() if case["ties"] else x
        s["u"] = torch.rand(b, generator=g, device=DEV)
        row = torch.arange(b, device=DEV)
        some = (lambda m, i: row % m == i) if case["mixed"] else (lambda m, i: row < 0)
        s["temperature"] = torch.where(some(5, 1), 0.0, 0.7 + 0.5 * torch.rand(b, generator=g, device=DEV))
        s["top_k"] = torch.where(some(3, 1), 0, torch.full_like(row, case["k"])).to(torch.int32)
        s["top_p"] = torch.where(some(4, 2), 1.0, torch.full((b,), case["p"], device=DEV))
        s["min_p"] = torch.where(some(2, 1), 0.0, torch.full((b,), case["m"], device=DEV))
        return s
    h, hkv, hd = case["h"], case["hkv"], case["hd"]
    if op == "rope":
        t = case["t"]
        s |= _rotary(case, g)
        s["q"], s["k"] = _randn(g, t, h, hd, dtype=_TYPE[case["qt"]]), _randn(g, t, hkv, hd, dtype=_TYPE[case["kt"]])
        s["positions"] = (torch.arange(t, device=DEV) + (case["far"] - t)).to(torch.int32)
        return s
    s |= _cache(case, g)
    t = s["t"]
    if op == "append":
        s |= _rotary(case, g)
        s["q"] = _randn(g, t, h, hd, dtype=_TYPE[case["qt"]])
        s["k"], s["v"] = (_randn(g, t, hkv, hd, dtype=_TYPE[case["kt"]]) for _ in range(2))
        return s
    s["q"] = _randn(g, t, h, hd, dtype=_TYPE[case["qt"]], std=1.5)
    s["cap"], s["window"] = case["cap"], case["window"]
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, h + 1, device=DEV, dtype=torch.float32) / h) if case["alibi"] else None
    s["bits"] = _tree_bits(case, seed) if case["tree"] else None
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _OWN[s["op"]](s)
    return _PLAIN[s["op"]](s)


def _own_rope(s):
    import paper_2409_03856_amd as sr
    return sr.sirius_rope(s["q"], s["k"], s["positions"], s["freqs"], interleaved=s["inter"], mscale=s["mscale"], norm_eps=s["eps"],
                          q_weight=s["qw"], k_weight=s["kw"])


def _own_append(s):
    import paper_2409_03856_amd as sr
    q = sr.sirius_kv_append(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["pos"], s["freqs"], tok_start=s["start"],
                            interleaved=s["inter"], mscale=s["mscale"], norm_eps=s["eps"], q_weight=s["qw"], k_weight=s["kw"])
    return q, s["k_pages"], s["v_pages"]


def _own_attn(s):
    import paper_2409_03856_amd as sr
    return sr.sirius_attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["pos"], tok_start=s["start"], max_n=s["n"],
                                softcap=s["cap"], slopes=s["slopes"], window=s["window"], mask=s["bits"])


def _own_sample(s):
    import paper_2409_03856_amd as sr
    return sr.sirius_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])


_OWN = {"rope": _own_rope, "append": _own_append, "attn": _own_attn, "sample": _own_sample}


def _rotated(x, weight, positions, s):
    """The norm and the rotation of x [T, heads, head size], in 32 bits; angles in 64."""
    x = x.float()
    if s["eps"] >= 0:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * weight.float()
    a = positions.double()[:, None] * s["freqs"]
    c, n = ((f(a) * s["mscale"]).float()[:, None] for f in (torch.cos, torch.sin))
    half = s["freqs"].numel()
    head, rest = x[..., : 2 * half], x[..., 2 * half:]
    if s["inter"]:
        u, v = head[..., 0::2], head[..., 1::2]
        head = torch.stack((u * c - v * n, u * n + v * c), -1).flatten(-2)
    else:
        u, v = head[..., :half], head[..., half:]
        head = torch.cat((u * c - v * n, u * n + v * c), -1)
    return torch.cat((head, rest), -1)


def _plain_rope(s):
    return (_rotated(s["q"], s["qw"], s["positions"], s).to(s["q"].dtype),
            _rotated(s["k"], s["kw"], s["positions"], s).to(torch.bfloat16))


def _places(s):
    """Each token's sequence, its number in it, and its cache row."""
    t, b = s["t"], s["pos"].numel()
    i = torch.arange(t, device=DEV)
    if s["start"] is None:
        seq, first = i // (t // b), i // (t // b) * (t // b)
    else:
        seq = (i[:, None] >= s["start"][None, 1:]).sum(1)
        first = s["start"].long()[seq]
    return seq, i - first, s["pos"].long()[seq] + i - first


def _plain_append(s):
    seq, _, row = _places(s)
    page = s["k_pages"].shape[2]
    at, off = s["table"].long()[seq, row // page], row % page
    q = _rotated(s["q"], s["qw"], row, s).to(s["q"].dtype)
    s["k_pages"][at, :, off] = _rotated(s["k"], s["kw"], row, s).to(torch.bfloat16)
    s["v_pages"][at, :, :, off] = s["v"].to(torch.bfloat16)
    return q, s["k_pages"], s["v_pages"]


def _plain_attn(s):
    seq, num, row = _places(s)
    t, h, hd = s["q"].shape
    _, hkv, page, _ = s["k_pages"].shape
    b, wide = s["table"].shape
    at = s["table"].long().clamp(min=0)
    length = wide * page
    k = s["k_pages"][at].float().transpose(1, 2).reshape(b, hkv, length, hd)
    v = s["v_pages"][at].float().permute(0, 2, 1, 4, 3).reshape(b, hkv, length, hd)
    n = s["n"]
    grid = torch.full((b, n), -1, dtype=torch.int64, device=DEV)
    grid[seq, num] = torch.arange(t, device=DEV)
    used = grid >= 0
    q = s["q"].float()[grid.clamp(min=0)].reshape(b, n, hkv, h // hkv, hd).transpose(1, 2).reshape(b, hkv, -1, hd)
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(hd))
    if s["cap"] > 0:
        x = s["cap"] * torch.tanh(x / s["cap"])
    x = x.view(b, hkv, n, h // hkv, length)
    place = torch.where(used, row[grid.clamp(min=0)], -1)
    j = torch.arange(length, device=DEV)
    away = place[:, :, None] - j
    if s["slopes"] is not None:
        x = x - s["slopes"].view(1, hkv, 1, h // hkv, 1) * away[:, None, :, None, :].float()
    seen = away >= 0
    if s["window"] > 0:
        seen = seen & (away < s["window"])
    if s["bits"] is not None:
        inside = j[None, None, :] - s["pos"].long()[:, None, None]
        bit = (s["bits"][grid.clamp(min=0)][:, :, None] >> inside.clamp(0, 63)) & 1
        seen = seen & ((inside < 0) | (bit != 0))
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    w = torch.exp(x - x.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(b, hkv, -1, length), v).view(b, hkv, n, h // hkv, hd).transpose(1, 2).reshape(b, n, h, hd)
    return out[seq, num].to(s["q"].dtype)


def _plain_sample(s):
    sv, si = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    sv = sv.double()
    temp = s["temperature"].double()[:, None]
    w = torch.exp((sv - sv[:, :1]) / torch.where(temp > 0, temp, 1.0))
    rank = torch.arange(sv.shape[1], device=DEV)[None]
    k = torch.where(s["top_k"] > 0, s["top_k"], sv.shape[1])[:, None]
    k = torch.where(temp > 0, k, 1)
    wk = torch.where(rank < k, w, 0.0)
    top = s["top_p"].double()[:, None]
    keep = (rank < k) & ((wk.cumsum(1) - wk < top * wk.sum(1, keepdim=True)) | (top >= 1)) & (w >= s["min_p"].double()[:, None])
    keep = keep | (rank == 0)
    kept = torch.zeros_like(w).scatter_(1, si, torch.where(keep, w, 0.0))
    run_sum = kept.cumsum(1)
    total = run_sum[:, -1:]
    token = (run_sum <= s["u"].double()[:, None] * total).sum(1)
    prob = (kept.gather(1, token[:, None]) / total)[:, 0]
    return token.to(torch.int32), keep.sum(1).to(torch.int32), prob.float()


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn, "sample": _plain_sample}


# ------------------------------------------------------------------------------------------------ what a pass needs

_SIZE = {"f32": 4, "bf16": 2}


def work(case):
    if case["op"] == "sample":
        return {"bytes": 4 * case["b"] * case["v"] + 32 * case["b"], "flops": 8 * case["b"] * case["v"]}
    h, hkv, hd = case["h"], case["hkv"], case["hd"]
    sq = _SIZE[case["qt"]]
    if case["op"] == "rope":
        return {"bytes": case["t"] * hd * (2 * sq * h + (_SIZE[case["kt"]] + 2) * hkv), "flops": 6 * case["t"] * (h + hkv) * hd}
    before, new = _ragged(case)
    t = sum(new)
    if case["op"] == "append":
        return {"bytes": t * hd * (2 * sq * h + 2 * (_SIZE[case["kt"]] + 2) * hkv), "flops": 6 * t * (h + hkv) * hd}
    pairs = rows = 0
    for p, n in zip(before, new):
        window = case["window"] or p + n
        rows += min(p + n, window + n - 1)
        if case["tree"]:
            depth = [i // case["tree"] + 1 for i in range(n)]  # the visible part of the chunk
            pairs += sum(min(p + d, window) for d in depth)
        else:
            pairs += sum(min(p + i + 1, window) for i in range(n))
    return {"bytes": 4 * rows * hkv * hd + 2 * t * h * hd * sq, "flops": 4 * pairs * h * hd}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """The same outputs from the definitions, sequence by sequence and row by row, in 64 bits."""
    return {"rope": _exact_rope, "append": _exact_append, "attn": _exact_attn, "sample": _exact_sample}[case["op"]](case, prepare(case, seed))


def _turned(x, weight, positions, s):
    """Norm and rotation as products of complex numbers."""
    x = x.double()
    if s["eps"] >= 0:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt() * weight.double()
    half = s["freqs"].numel()
    by = torch.polar(torch.full((positions.numel(), half), s["mscale"], dtype=torch.float64, device=DEV), torch.outer(positions.double(), s["freqs"]))
    one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["inter"] else (slice(0, half), slice(half, 2 * half))
    z = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * by[:, None]
    y = x.clone()
    y[..., one], y[..., two] = z.real, z.imag
    return y


def _exact_rope(case, s):
    return _turned(s["q"], s["qw"], s["positions"], s), _turned(s["k"], s["kw"], s["positions"], s)


def _exact_append(case, s):
    before, new = _ragged(case)
    page = case["page"]
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    q, at = [], 0
    for b, (p, n) in enumerate(zip(before, new)):
        rows = torch.arange(p, p + n, device=DEV)
        k = _turned(s["k"][at:at + n], s["kw"], rows, s)
        q.append(_turned(s["q"][at:at + n], s["qw"], rows, s))
        for first in range(p // page * page, p + n, page):
            lo, hi = max(first, p), min(first + page, p + n)
            place = int(s["table"][b, first // page])
            kp[place, :, lo - first:hi - first] = k[lo - p:hi - p].transpose(0, 1)
            vp[place, :, :, lo - first:hi - first] = s["v"][at + lo - p:at + hi - p].double().permute(1, 2, 0)
        at += n
    return torch.cat(q), kp, vp


def _exact_attn(case, s):
    before, new = _ragged(case)
    page, h, hkv, hd = case["page"], case["h"], case["hkv"], case["hd"]
    out, at = [], 0
    for b, (p, n) in enumerate(zip(before, new)):
        places = s["table"][b, : -(-(p + n) // page)].long()
        keys = s["k_pages"][places].double().transpose(0, 1).reshape(hkv, -1, hd)[:, : p + n]
        values = s["v_pages"][places].double().permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, : p + n]
        for i0 in range(0, n, 512):
            m = min(512, n - i0)
            q = s["q"][at + i0:at + i0 + m].double().view(m, hkv, h // hkv, hd).permute(1, 2, 0, 3).reshape(hkv, -1, hd)
            x = torch.bmm(q, keys.transpose(1, 2).contiguous()).view(hkv, h // hkv, m, -1) / math.sqrt(hd)
            if case["cap"] > 0:
                x = case["cap"] * torch.tanh(x / case["cap"])
            here, there = torch.arange(p + i0, p + i0 + m, device=DEV)[:, None], torch.arange(p + n, device=DEV)[None]
            if s["slopes"] is not None:
                x = x - s["slopes"].double().view(hkv, -1, 1, 1) * (here - there).double()
            hidden = there > here
            if case["window"]:
                hidden = hidden | (there <= here - case["window"])
            if s["bits"] is not None:
                bit = torch.stack([(s["bits"][at + i0:at + i0 + m] >> c) & 1 for c in range(n)], 1) == 0
                hidden[:, p:] |= bit
            x = x.masked_fill(hidden, -math.inf)
            w = torch.softmax(x, -1).view(hkv, -1, p + n)
            out.append(torch.bmm(w, values.contiguous()).view(hkv, h // hkv, m, hd).permute(2, 0, 1, 3).reshape(m, h, hd))
        at += n
    return torch.cat(out)


def _exact_sample(case, s):
    tokens, counts, probs = [], [], []
    for b in range(case["b"]):
        x = s["logits"][b].double()
        temp, k, p, m = (float(s[n][b]) for n in ("temperature", "top_k", "top_p", "min_p"))
        best = x.max()
        if temp == 0:
            first = int((x == best).nonzero()[0])
            tokens, counts, probs = tokens + [first], counts + [1], probs + [1.0]
            continue
        w = torch.exp((x - best) / temp)
        order = torch.argsort(-x, stable=True)
        if k > 0:
            order = order[: int(k)]
        mass = w[order]
        if p < 1:
            ahead = torch.cat((mass.new_zeros(1), mass.cumsum(0)[:-1]))
            order = order[: max(1, int((ahead < p * mass.sum()).sum()))]
        order = order[: max(1, int((w[order] >= m).sum()))]
        index = order.sort().values
        reach = w[index].cumsum(0)
        j = int((reach <= float(s["u"][b]) * reach[-1]).sum())
        tokens.append(int(index[j]))
        counts.append(index.numel())
        probs.append(float(w[index[j]] / reach[-1]))
    return (torch.tensor(tokens, dtype=torch.int32), torch.tensor(counts, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64))
