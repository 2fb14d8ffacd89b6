"""The operators of tree-drafted, sampled decoding, in their plain form and through the library.

Four operators: the rotary embedding of query and key rows with their per-head norms (``rope``), attention of a tree
of drafted tokens over the paged cache (``tree``), sampling from logits with given random numbers (``sample``) and the
commit of a tree's accepted path (``commit``).

``own`` is False: ``run`` computes them with elementary torch operations.  ``own`` is True: ``run`` makes the library's
calls.  Shapes are those of ``sdlm_synth``: 16 query heads over 2 key heads of 128 with 151936 tokens, 40 over 8 of
128 with 152064, and the tiny 4 over 2 of 64 with 1024.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

SHAPES = {"3b": (16, 2, 128), "32b": (40, 8, 128), "tiny": (4, 2, 64)}  # query heads, key heads, head size
VOCABS = {"3b": 151936, "32b": 152064, "tiny": 1024}
THETA, EPS = 1000000.0, 1e-6
TRAINED = 32768                # positions the unscaled rotary embedding was made for
BETA_FAST, BETA_SLOW = 32.0, 1.0


# ---- cases ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # one new token of one sequence: only latency counts
        dict(name="rope_token", op="rope", shape="3b", batch=1, n=1, rot=128, interleaved=False, scaling="none",
             factor=1.0, norm=True, fused=False, far=4096),
        # a verification pass over 32 small trees: neighbouring pairs, half of the head, rows out of the stacked q/k/v
        # product, positions stretched
        dict(name="rope_tree", op="rope", shape="3b", batch=32, n=21, rot=64, interleaved=True, scaling="linear",
             factor=4.0, norm=False, fused=True, far=16384),
        # a long prompt in the largest shape, past the trained length, frequencies scaled by band
        dict(name="rope_prompt", op="rope", shape="32b", batch=1, n=16381, rot=128, interleaved=False, scaling="yarn",
             factor=4.0, norm=True, fused=True, far=131072),
        # one sequence and a single token: the form without a draft
        dict(name="tree_token", op="tree", shape="3b", batch=1, n=1, lo=1024, hi=1024, ragged=False),
        # a batch of ragged prefixes with small trees of different sizes: the cache's bytes
        dict(name="tree_batch", op="tree", shape="3b", batch=32, n=13, lo=512, hi=4096, ragged=True),
        # few sequences with long prefixes
        dict(name="tree_long", op="tree", shape="3b", batch=8, n=32, lo=32768, hi=32768, ragged=False),
        # the largest shape with the widest trees: the products
        dict(name="tree_wide", op="tree", shape="32b", batch=64, n=64, lo=512, hi=4096, ragged=True),
        # one row with every filter
        dict(name="sample_row", op="sample", shape="3b", rows=1, dtype="bf16", peak=8.0, filters="all", banned=False),
        # a batch of verified positions with the filters of ordinary requests, some of them greedy, and banned tokens
        dict(name="sample_batch", op="sample", shape="3b", rows=128, dtype="bf16", peak=6.0, filters="all", banned=True),
        # many rows in 32 bits, flat distributions with a wide nucleus
        dict(name="sample_flat", op="sample", shape="32b", rows=256, dtype="fp32", peak=0.0, filters="top_p", banned=False),
        # one sequence's accepted path
        dict(name="commit_one", op="commit", shape="tiny", batch=1, n=16, lo=200, hi=200, p=0.8),
        # several sequences with the widest trees
        dict(name="commit_batch", op="commit", shape="3b", batch=8, n=64, lo=100, hi=700, p=0.9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _drawn(rng, op):
    shape = rng.choice(("3b", "32b", "tiny"))
    d = SHAPES[shape][2]
    if op == "rope":
        rot = rng.choice([r for r in (16, 32, 48, 64, 96, 128) if r <= d])
        scaling = rng.choice(("none", "linear", "ntk", "yarn"))
        return dict(op=op, shape=shape, batch=_log_int(rng, 1, 64), n=_log_int(rng, 1, 16384), rot=rot,
                    interleaved=rng.random() < 0.5, scaling=scaling,
                    factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 8.0), 2), norm=rng.random() < 0.6,
                    fused=rng.random() < 0.5, far=_log_int(rng, 1024, 1000000))
    if op == "tree":
        hi = _log_int(rng, 1, 32768)
        return dict(op=op, shape=shape, batch=_log_int(rng, 1, 64), n=rng.randint(1, 64), lo=rng.randint(0, hi), hi=hi,
                    ragged=rng.random() < 0.5)
    if op == "sample":
        return dict(op=op, shape=shape, rows=_log_int(rng, 1, 256), dtype=rng.choice(("bf16", "fp32")),
                    peak=rng.choice((0.0, 4.0, 6.0, 8.0)), filters=rng.choice(("all", "top_p", "top_k", "none")),
                    banned=rng.random() < 0.5)
    hi = _log_int(rng, 64, 2048)
    return dict(op=op, shape=shape, batch=rng.randint(1, 8), n=rng.randint(1, 64), lo=rng.randint(0, hi), hi=hi,
                p=round(rng.uniform(0.3, 1.0), 2))


def draw(rng):
    op = rng.choice(("rope", "tree", "tree", "sample", "sample", "commit"))
    most = [work(c) for c in listed() if c["op"] == op]
    while True:
        case = _drawn(rng, op)
        w = work(case)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most):
            return case


def _lens(case):
    """Prefix lengths, spread over lo..hi."""
    lo, hi = case["lo"], case["hi"]
    return [lo + int((hi - lo + 1) * ((b + 1) * 0.6180339887 % 1.0)) for b in range(case["batch"])]


def _nodes(case):
    """Nodes of each sequence's tree."""
    n = case["n"]
    return [n - (5 * b) % ((n + 1) // 2) if case.get("ragged") else n for b in range(case["batch"])]


# ---- inputs --------------------------------------------------------------------------------------------------
def _normal(g, shape, std=1.0, mean=0.0):
    """Normal bf16 values, drawn in pieces (the 32-bit draw of a whole cache would be as large again)."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 26):
        m = min(1 << 26, flat.numel() - i)
        flat[i:i + m] = torch.randn(m, generator=g, device="cuda") * std + mean
    return out


def _context(case, lens, extra, seed):
    import paper_2509_24007_b200 as pk
    hq, hk, d = SHAPES[case["shape"]]
    pages = [(x + extra + 63) // 64 + 1 for x in lens]
    sd = pk.Sdlm(pk.SdlmConfig(hq, hk, d, 256, VOCABS[case["shape"]], sum(pages), len(lens), max(pages), max_block=8))
    sd.kv_reset(np.random.default_rng(seed).permutation(sum(pages)).astype(np.int32))
    return pk, sd


def _tree(case, g):
    """Parents: each node hangs from one of the six before it (node 0 from the prefix)."""
    B, n = case["batch"], case["n"]
    j = torch.arange(n, device="cuda")
    lo = (j - 6).clamp(min=0)
    r = torch.rand((B, n), generator=g, device="cuda")
    parent = lo + (r * (j - lo)).long().clamp(max=5)
    parent = torch.minimum(parent, (j - 1).clamp(min=0)).to(torch.int32)
    parent[:, 0] = -1
    return parent.contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    hq, hk, d = SHAPES[case["shape"]]
    s = {"case": case}
    if case["op"] == "rope":
        B, n = case["batch"], case["n"]
        s["pos"] = torch.randint(0, case["far"], (B, n), generator=g, device="cuda", dtype=torch.int32)
        if case["fused"]:
            qkv = _normal(g, (B, n, hq + 2 * hk, d))
            s["q"], s["k"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
        else:
            s["q"], s["k"] = _normal(g, (B, n, hq, d)), _normal(g, (B, n, hk, d))
        s["wq"], s["wk"] = (_normal(g, (d,), 0.2, 1.0), _normal(g, (d,), 0.2, 1.0)) if case["norm"] else (None, None)
        if own:
            pk, s["sd"] = _context(case, [0] * B, 0, seed)
            kind = {"none": pk.ROPE_PLAIN, "linear": pk.ROPE_LINEAR, "ntk": pk.ROPE_NTK, "yarn": pk.ROPE_YARN}
            s["rope"] = pk.RopeConfig(theta=THETA, rot_dim=case["rot"], interleaved=case["interleaved"],
                                      scaling=kind[case["scaling"]], factor=case["factor"], trained_len=TRAINED,
                                      beta_fast=BETA_FAST, beta_slow=BETA_SLOW)
            s["q_out"] = torch.empty((B, n, hq, d), dtype=torch.bfloat16, device="cuda")
            s["k_out"] = torch.empty((B, n, hk, d), dtype=torch.bfloat16, device="cuda")
        return s
    if case["op"] == "sample":
        R, V = case["rows"], VOCABS[case["shape"]]
        x = torch.randn((R, V), generator=g, device="cuda") * 2.0
        if case["peak"]:  # a few likely tokens in every row, as a language model has them
            # (one in each fortieth of the vocabulary: of an index drawn twice either value might be left standing)
            at = torch.randint(0, V // 40, (R, 40), generator=g, device="cuda") + torch.arange(40, device="cuda") * (V // 40)
            up = case["peak"] + 2.0 * torch.randn((R, 40), generator=g, device="cuda")
            x.scatter_(1, at, up)
        if case["banned"]:  # the padding of the vocabulary, and single tokens
            x[:, V - V // 64:] = -math.inf
            x[:, torch.randint(0, V, (100,), generator=g, device="cuda")] = -math.inf
        s["logits"] = x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        del x
        s["u"] = torch.rand(R, generator=g, device="cuda")
        rnd = torch.rand((4, R), generator=g, device="cuda")
        one, f = torch.ones(R, device="cuda"), case["filters"]
        s["T"] = 0.6 + 0.8 * rnd[0]
        s["k"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["p"], s["m"] = one.clone(), 0.0 * one
        if f in ("all", "top_k"):
            ks = torch.tensor([0, 1, 20, 50, 200, 1000], dtype=torch.int32, device="cuda")
            s["k"] = ks[(rnd[1] * 6).long().clamp(max=5)] if f == "all" else 1 + (rnd[1] * 2000).int()
        if f in ("all", "top_p"):
            s["p"] = 0.7 + 0.35 * rnd[2]  # from 1 on: no limit
        if f == "all":
            s["m"] = torch.where(rnd[3] < 0.5, 0.0, 0.1 * rnd[3])
            s["T"] = torch.where(rnd[3] > 0.875, 0.0, s["T"])  # greedy
        if own:
            _, s["sd"] = _context(case, [0], 0, seed)
        return s
    B, n, lens, nodes = case["batch"], case["n"], _lens(case), _nodes(case)
    room = max(max(lens), 1) + (n if case["op"] == "commit" else 0)
    s["parent"] = _tree(case, g)
    s["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["nodes"] = torch.tensor(nodes, dtype=torch.int32, device="cuda")
    s["kt"], s["vt"] = _normal(g, (B, n, hk, d)), _normal(g, (B, n, hk, d))
    s["kh"], s["vh"] = _normal(g, (B, room, hk, d)), _normal(g, (B, room, hk, d))  # prefixes, rows behind them unused
    if case["op"] == "tree":
        s["q"] = _normal(g, (B, n, hq, d))
    else:
        s["draft"] = torch.randint(0, 50, (B, n), generator=g, device="cuda", dtype=torch.int32)
        s["next"] = torch.randint(1000, 1050, (B, n), generator=g, device="cuda", dtype=torch.int32)
        coin = torch.rand((B, n), generator=g, device="cuda") < case["p"]
        child = torch.arange(n, device="cuda") * coin
        child[:, 0] = 0
        kids = torch.zeros((B, n), dtype=torch.int64, device="cuda")
        kids.scatter_reduce_(1, s["parent"].long().clamp(min=0), child, "amax")
        s["next"] = torch.where(kids > 0, s["draft"].gather(1, kids), s["next"]).contiguous()
    if own:
        _, sd = _context(case, lens, n, seed)
        s["sd"] = sd
        for b, x in enumerate(lens):
            if x:
                sd.kv_add_seq(b, s["kh"][b, :x].contiguous(), s["vh"][b, :x].contiguous())
        if case["op"] == "tree":
            s["out"] = torch.zeros((B, n, hq, d), dtype=torch.bfloat16, device="cuda")
        else:
            s["saved"] = sd.kv_save()
            s["ka"], s["va"] = torch.zeros_like(s["kh"]), torch.zeros_like(s["vh"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------
def _bands(case, dtype):
    """Angle per position of each rotated pair, and the factor on cosine and sine."""
    r, s = case["rot"], case["factor"]
    i = torch.arange(r // 2, dtype=dtype, device="cuda")
    if case["scaling"] == "ntk":
        return (THETA * s ** (r / (r - 2.0))) ** (-2.0 * i / r), 1.0
    f = THETA ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "yarn":
        lo, hi = (r * math.log(TRAINED / (b * 2.0 * math.pi)) / (2.0 * math.log(THETA)) for b in (BETA_FAST, BETA_SLOW))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
        ramp = ((i - lo) / (hi - lo if hi > lo else 0.001)).clamp(0.0, 1.0)
        return f / s * ramp + f * (1.0 - ramp), 0.1 * math.log(s) + 1.0 if s > 1.0 else 1.0
    return f, 1.0


def _rotated(x, w, cos, sin, rot, interleaved):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    y, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, rest), dim=-1).to(torch.bfloat16)


def _rope(s):
    c = s["case"]
    if own:
        s["sd"].qk_norm_rope(s["q"], s["k"], s["rope"], positions=s["pos"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS,
                             q_out=s["q_out"], k_out=s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    f, m = _bands(c, torch.float64)
    a = s["pos"].double()[..., None, None] * f  # far positions: the angle in 64 bits
    cos, sin = (torch.cos(a) * m).float(), (torch.sin(a) * m).float()
    return {"q": _rotated(s["q"], s["wq"], cos, sin, c["rot"], c["interleaved"]),
            "k": _rotated(s["k"], s["wk"], cos, sin, c["rot"], c["interleaved"])}


def _reach(parent, dtype=torch.float32):
    """[.., j, i] = 1 where node i is node j or one before it on its path: (I - P)^-1 with P[j, parent[j]] = 1."""
    n = parent.shape[-1]
    i = torch.arange(n, device="cuda")
    eye = torch.eye(n, dtype=dtype, device="cuda")
    edges = (parent.long()[..., None] == i).to(dtype)
    return torch.linalg.solve_triangular(eye - edges, eye.expand_as(edges), upper=False, unitriangular=True) > 0.5


def _tree_attention(s):
    if own:
        s["sd"].tree_attn(s["q"], s["kt"], s["vt"], s["parent"], n_nodes=s["nodes"], out=s["out"])
        return s["out"]
    c, q = s["case"], s["q"].float()
    B, n, hq, d = q.shape
    L, hk = s["kh"].shape[1], s["kh"].shape[2]
    q = q.reshape(B, n, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(B, hk, -1, d) * d ** -0.5
    k = torch.cat((s["kh"], s["kt"]), 1).float().permute(0, 2, 3, 1)
    seen = (torch.arange(L, device="cuda") < s["len"][:, None])[:, None, :].expand(B, n, L)
    node = torch.arange(n, device="cuda") < s["nodes"][:, None]
    seen = torch.cat((seen, _reach(s["parent"])), 2)
    score = torch.matmul(q, k).view(B, hk, hq // hk, n, L + n)
    del k
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    v = torch.cat((s["vh"], s["vt"]), 1).float().permute(0, 2, 1, 3)
    out = torch.matmul(score.view(B, hk, -1, L + n), v).view(B, hk, hq // hk, n, d) / total
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)
    return torch.where(node[..., None, None], out, 0.0).to(torch.bfloat16)


def _sample(s):
    if own:
        token, prob, entropy, kept = s["sd"].sample(s["logits"], s["u"], temperature=s["T"], top_k=s["k"], top_p=s["p"],
                                                    min_p=s["m"])
        return {"token": token, "prob": prob, "entropy": entropy, "kept": kept}
    x = s["logits"].float()
    V = x.shape[1]
    greedy = s["T"] <= 0
    k = torch.where(greedy, 1, torch.where(s["k"] <= 0, V, s["k"]))
    v, order = torch.sort(x, dim=1, descending=True, stable=True)  # equal values: lowest index first
    z = (v - v[:, :1]).double() / torch.where(greedy, 1.0, s["T"]).double()[:, None]
    w = torch.exp(z)
    keep = (torch.arange(V, device="cuda") < k[:, None]) & (v > -math.inf)
    w = w * keep
    cum = torch.cumsum(w, 1)
    p = s["p"].double()[:, None]
    keep &= (p >= 1.0) | (cum - w < p * cum[:, -1:])
    keep &= w >= s["m"].double().clamp(max=1.0)[:, None]
    w = w * keep
    total = w.sum(1, keepdim=True)
    entropy = (torch.log(total) - torch.where(keep, w * z, 0.0).sum(1, keepdim=True) / total)[:, 0]
    by_index = torch.empty_like(w).scatter_(1, order, w)
    cum = torch.cumsum(by_index, 1)
    token = (cum <= s["u"].double()[:, None] * total).sum(1).clamp(max=V - 1)
    prob = by_index.gather(1, token[:, None])[:, 0] / total[:, 0]
    return {"token": token.to(torch.int32), "prob": prob.float(), "entropy": entropy.float(),
            "kept": keep.sum(1).to(torch.int32)}


def _commit(s):
    c = s["case"]
    if own:
        sd = s["sd"]
        sd.kv_restore(s["saved"])  # every pass starts from the same tables
        accepted, tokens, path = sd.tree_commit(s["draft"], s["next"], s["parent"], s["kt"], s["vt"], n_nodes=s["nodes"])
        sd.kv_gather_batch(s["ka"], s["va"])
        return {"accepted": accepted, "tokens": tokens, "path": path, "k": s["ka"], "v": s["va"]}
    B, n = s["parent"].shape
    room = s["kh"].shape[1]
    parent, j = s["parent"].long(), torch.arange(n, device="cuda")
    # a node is taken when its token is what its parent decided on, and it is the first such child, all along its path
    fits = (s["draft"] == s["next"].gather(1, parent.clamp(min=0))) & (j < s["nodes"][:, None])
    twin = (parent[:, :, None] == parent[:, None, :]) & (s["draft"][:, :, None] == s["draft"][:, None, :])
    fits &= ~(twin & (j[None, :] < j[:, None])).any(2)
    fits = torch.where(j == 0, j < s["nodes"][:, None], fits)
    taken = ~(_reach(s["parent"]) & ~fits[:, None, :]).any(2)
    accepted = taken.sum(1)
    place = torch.where(taken, taken.cumsum(1) - 1, n)
    path = torch.full((B, n + 1), -1, dtype=torch.int64, device="cuda").scatter_(1, place, j.expand(B, n))[:, :n]
    there = path >= 0
    tokens = torch.where(there, s["next"].gather(1, path.clamp(min=0)), -1)
    t = torch.arange(room, device="cuda") - s["len"][:, None]
    node = path.gather(1, t.clamp(0, n - 1))
    old, new = (t < 0)[..., None, None], ((t >= 0) & (t < accepted[:, None]))[..., None, None]
    at = node.clamp(min=0)[..., None, None].expand_as(s["kh"])
    k = torch.where(old, s["kh"], torch.where(new, s["kt"].gather(1, at), 0.0))
    v = torch.where(old, s["vh"], torch.where(new, s["vt"].gather(1, at), 0.0))
    return {"accepted": accepted.to(torch.int32), "tokens": tokens.to(torch.int32), "path": path.to(torch.int32),
            "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def run(state):
    op = state["case"]["op"]
    if op == "rope":
        return _rope(state)
    if op == "tree":
        return _tree_attention(state)
    if op == "sample":
        return _sample(state)
    return _commit(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def work(case):
    hq, hk, d = SHAPES[case["shape"]]
    if case["op"] == "rope":
        rows = case["batch"] * case["n"]
        each = rows * (hq + hk) * d
        return {"bytes": 4 * each + 4 * rows, "flops": (7 if case["norm"] else 3) * each}
    if case["op"] == "sample":
        each = case["rows"] * VOCABS[case["shape"]]
        return {"bytes": (2 if case["dtype"] == "bf16" else 4) * each + 36 * case["rows"], "flops": 4 * each}
    lens, nodes = _lens(case), _nodes(case)
    row = hk * d * 2
    if case["op"] == "tree":
        return {"bytes": sum(2 * row * (x + m) + 4 * m * hq * d for x, m in zip(lens, nodes)) + 4 * case["batch"] * case["n"],
                "flops": sum(4 * hq * d * m * (x + 1) for x, m in zip(lens, nodes))}
    # the committed sequences are read back: the prefix and at least one row of each
    return {"bytes": sum(4 * row * (x + 1) + 4 * row + 20 * m for x, m in zip(lens, nodes)), "flops": sum(nodes)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------
def _exact_rope(case, s):
    r, f, m = case["rot"], *_bands(case, torch.float64)
    angle = s["pos"].double().unsqueeze(-1) * f
    turn = torch.polar(torch.full_like(angle, m), angle).unsqueeze(2)

    def of(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
        y = x[..., :r]
        pair = y.unflatten(-1, (r // 2, 2)) if case["interleaved"] else y.unflatten(-1, (2, r // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x = x.clone()
        x[..., :r] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return x

    return {"q": of(s["q"], s["wq"]), "k": of(s["k"], s["wk"])}


def _exact_tree(case, s):
    hq, hk, d = SHAPES[case["shape"]]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    parents = s["parent"].tolist()
    for b, (x, m) in enumerate(zip(_lens(case), _nodes(case))):
        sees = np.zeros((m, x + m), dtype=bool)
        sees[:, :x] = True
        for j in range(m):
            i = j
            while i >= 0:
                sees[j, x + i] = True
                i = parents[b][i]
        hidden = torch.from_numpy(~sees).cuda()
        for h in range(hk):
            k = torch.cat((s["kh"][b, :x, h], s["kt"][b, :m, h])).double()
            v = torch.cat((s["vh"][b, :x, h], s["vt"][b, :m, h])).double()
            q = s["q"][b, :m, h * (hq // hk):(h + 1) * (hq // hk)].double()
            score = torch.einsum("jgd,td->gjt", q, k) / math.sqrt(d)
            score = score.masked_fill(hidden, -math.inf)
            weight = torch.exp(score - torch.logsumexp(score, -1, keepdim=True))
            out[b, :m, h * (hq // hk):(h + 1) * (hq // hk)] = torch.einsum("gjt,td->jgd", weight, v)
    return out


def _exact_sample(case, s):
    x = s["logits"].float().cpu().numpy()
    u, T, k, p, m = (s[a].cpu().numpy().astype(np.float64) for a in ("u", "T", "k", "p", "m"))
    tokens, probs, entropies, kepts = [], [], [], []
    for r in range(x.shape[0]):
        able = np.flatnonzero(x[r] > -np.inf)
        able = able[np.argsort(-x[r][able], kind="stable")]
        z = x[r][able].astype(np.float64)
        z = (z - z[0]) / (T[r] if T[r] > 0 else 1.0)
        n = 1 if T[r] <= 0 else int(k[r]) if 0 < k[r] < len(able) else len(able)
        w = np.exp(z[:n])
        if p[r] < 1.0:
            before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
            n = max(1, int(np.count_nonzero(before < p[r] * w.sum())))
        w = w[:n][w[:n] >= min(m[r], 1.0)]
        n = len(w)
        prob = w / w.sum()
        by_index = np.argsort(able[:n])
        at = by_index[min(n - 1, int(np.searchsorted(np.cumsum(w[by_index]), u[r] * w.sum(), side="right")))]
        tokens.append(int(able[at]))
        probs.append(prob[at])
        live = prob[prob > 0]
        entropies.append(-float(np.sum(live * np.log(live))))
        kepts.append(n)
    return {"token": np.array(tokens, np.int32), "prob": np.array(probs), "entropy": np.array(entropies),
            "kept": np.array(kepts, np.int32)}


def _exact_commit(case, s):
    n, lens, nodes = case["n"], _lens(case), _nodes(case)
    parent, draft, decided = (s[a].tolist() for a in ("parent", "draft", "next"))
    k, v = torch.zeros_like(s["kh"], dtype=torch.float64), torch.zeros_like(s["vh"], dtype=torch.float64)
    paths = []
    for b, (x, m) in enumerate(zip(lens, nodes)):
        way = [0]
        while True:
            nxt = [c for c in range(1, m) if parent[b][c] == way[-1] and draft[b][c] == decided[b][way[-1]]]
            if not nxt:
                break
            way.append(nxt[0])
        paths.append(way)
        k[b, :x], v[b, :x] = s["kh"][b, :x].double(), s["vh"][b, :x].double()
        k[b, x:x + len(way)], v[b, x:x + len(way)] = s["kt"][b, way].double(), s["vt"][b, way].double()
    pad = [w + [-1] * (n - len(w)) for w in paths]
    told = [[decided[b][i] if i >= 0 else -1 for i in w] for b, w in enumerate(pad)]
    return {"accepted": np.array([len(w) for w in paths], np.int32), "tokens": np.array(told, np.int32),
            "path": np.array(pad, np.int32), "k": k, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "tree": _exact_tree, "sample": _exact_sample, "commit": _exact_commit}[case["op"]](case, s)
