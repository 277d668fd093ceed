"""Timed cases of the token operators: the projection with per-camera adapters (project), the
norm and rotation of queries and keys (rotate) and the masked attention (attend).

A transformer that reads stitched canvases has one token per 16 x 16 pixels of canvas, so a
1280 x 1280 canvas is 6,400 tokens and a 1024 x 1024 one 4,096; the tokens of one RoI patch are
one document, the cells outside every patch have none, and each camera may have adapters of its
own. A model that describes what it sees goes on with single tokens against a cache.

The layout of a case (ragged lengths, documents, adapters of tokens) comes from its "layout"
number, the values of its tensors from the seed.

Kinds (`case["kind"]`):
  project  y = x w^T + scale_g (x a_g^T) b_g^T, adapter g by token
  rotate   per-head norm and rotation of q and k; with "cache", k and v go to rows of a cache
  attend   attention over ragged sequences: "single" is one query per sequence against its
           cache, otherwise queries and keys are the same tokens
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


# ------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one new token of each of 8 cameras through a small layer: latency
        dict(name="project_single_8cam", kind="project", tokens=8, k=1024, n=1536, adapters=8,
             rank=8, bare=0.0, type="bf16", layout=1),
        # odd sizes, tokens of mixed requests, a third of them without an adapter
        dict(name="project_odd", kind="project", tokens=1777, k=1160, n=2051, adapters=5, rank=12,
             bare=0.33, type="f16", layout=2),
        # the tokens of one 1280 x 1280 canvas, patches of 20 cameras
        dict(name="project_canvas", kind="project", tokens=6400, k=1024, n=1536, adapters=20,
             rank=16, bare=0.1, type="bf16", layout=3),
        # four such canvases through a large layer
        dict(name="project_4canvas", kind="project", tokens=25600, k=4096, n=4096, adapters=20,
             rank=32, bare=0.1, type="bf16", layout=4),
        # one new token of each of 20 cameras, keys and values into the cache
        dict(name="rotate_single_20cam", kind="rotate", tokens=20, heads=16, kv_heads=4, d=64,
             rot=64, axes=1, pairs="half", positions=4096, cache=True, type="bf16", layout=5),
        # odd counts, part of each head rotated, neighbouring pairs, two position axes
        dict(name="rotate_odd", kind="rotate", tokens=3333, heads=7, kv_heads=1, d=80, rot=40,
             axes=2, pairs="next", positions=512, cache=False, type="f16", layout=6),
        # a batch of 32 canvases of 4,096 tokens
        dict(name="rotate_32canvas", kind="rotate", tokens=131072, heads=16, kv_heads=2, d=128,
             rot=128, axes=2, pairs="half", positions=512, cache=False, type="bf16", layout=7),
        # one query of each of 20 cameras, caches of up to a quarter of a 1280 x 1280 canvas
        dict(name="attend_single_20cam", kind="attend", single=True, seqs=20, length=1600, heads=16,
             kv_heads=4, d=64, cap=30.0, slopes=False, positions=False, docs=0, prefix=False,
             causal=True, raster=False, type="bf16", layout=8),
        # 8 long caches, bias by distance
        dict(name="attend_single_long", kind="attend", single=True, seqs=8, length=100003, heads=16,
             kv_heads=2, d=128, cap=0.0, slopes=True, positions=False, docs=0, prefix=False,
             causal=True, raster=False, type="bf16", layout=9),
        # four 1280 x 1280 canvases of about 32 patches, bias by distance on the canvas
        dict(name="attend_canvas", kind="attend", single=False, seqs=4, length=6400, heads=16,
             kv_heads=16, d=64, cap=0.0, slopes=True, positions=True, docs=32, prefix=False,
             causal=False, raster=False, type="f16", layout=10),
        # ragged prompts whose first part is an image every token may see, capped scores
        dict(name="attend_prefix", kind="attend", single=False, seqs=7, length=2077, heads=16,
             kv_heads=4, d=128, cap=50.0, slopes=False, positions=False, docs=0, prefix=True,
             causal=True, raster=False, type="bf16", layout=11),
        # one long prompt
        dict(name="attend_causal", kind="attend", single=False, seqs=1, length=16384, heads=16,
             kv_heads=4, d=128, cap=0.0, slopes=True, positions=False, docs=0, prefix=False,
             causal=True, raster=False, type="bf16", layout=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["project", "rotate", "attend"])
    layout, kind_type = rng.randrange(1 << 30), rng.choice(["f16", "bf16"])
    if kind == "project":
        c = dict(kind=kind, tokens=_log(rng, 1, 25600), k=8 * _log(rng, 32, 512),
                 n=_log(rng, 200, 4096), adapters=_log(rng, 1, 40), rank=_log(rng, 1, 64),
                 bare=rng.choice([0.0, 0.1, 0.5]), type=kind_type, layout=layout)
        c["rank"] = min(c["rank"], 1024 // c["adapters"])
    elif kind == "rotate":
        kv = rng.choice([1, 2])
        d = 2 * rng.randint(16, 64) if rng.random() < 0.3 else rng.choice([32, 64, 80, 96, 128])
        axes = rng.choice([1, 2])
        rot = d if rng.random() < 0.6 else max(4, d // 2)
        c = dict(kind=kind, tokens=_log(rng, 1, 131072), heads=kv * rng.choice([1, 2, 4, 8]),
                 kv_heads=kv, d=d, rot=rot - rot % 4, axes=axes,
                 pairs=rng.choice(["half", "next"]), positions=rng.choice([512, 4096]),
                 cache=rng.random() < 0.4, type=kind_type, layout=layout)
    else:
        single, kv = rng.random() < 0.5, rng.choice([1, 2, 4])
        d = rng.choice([32, 40, 64, 72, 96, 128])
        heads = kv * rng.choice([1, 2, 4, 8])
        length = _log(rng, 1, 100003) if single else _log(rng, 1, 16384)
        seqs = _log(rng, 1, 64 if single else 8)
        heads = min(heads, 16)
        if single:
            seqs = max(1, min(seqs, 8 * 100003 // length))
        else:
            seqs = max(1, min(seqs, 16384 * 16384 // (length * length)))
        docs = rng.choice([0, 0, 3, 32])
        causal = single or rng.random() < 0.6
        c = dict(kind=kind, single=single, seqs=seqs, length=length, heads=heads, kv_heads=kv, d=d,
                 cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.5,
                 positions=rng.random() < 0.3, docs=docs, prefix=causal and rng.random() < 0.3,
                 causal=causal, raster=rng.random() < 0.5, type=kind_type, layout=layout)
    return c


# ----------------------------------------------------------------------------- the layouts

def _lengths(c):
    """Keys of each sequence: the first is the longest, the others spread below it."""
    r = random.Random(c["layout"])
    if c["docs"] and not c["single"]:
        return [c["length"]] * c["seqs"]
    return [c["length"]] + [r.randint(max(1, c["length"] // 8), c["length"])
                            for _ in range(c["seqs"] - 1)]


def _shelves(r, tokens, docs):
    """Documents and cells of a canvas of `tokens` cells, about `docs` patches on shelves: patch
    numbers run along a shelf, a tenth or so of the cells is on no patch (document -1)."""
    side = max(1, math.isqrt(tokens))
    rows = -(-tokens // side)
    grid = np.full((rows, side), -1, dtype=np.int32)
    edge = max(1, int(math.sqrt(rows * side / docs)))
    y = n = 0
    while y < rows:
        h = max(1, int(edge * r.uniform(0.6, 1.5)))
        x = 0
        while x < side:
            w = max(1, int(edge * r.uniform(0.5, 1.6)))
            grid[y:y + max(1, int(h * r.uniform(0.75, 1.0))), x:x + w] = n
            n, x = n + 1, x + w
        y += h
    flat = grid.reshape(-1)[:tokens]
    cells = np.stack([np.arange(tokens) % side, np.arange(tokens) // side], 1).astype(np.int32)
    return flat, cells


def _layout(c):
    """Per token of an attend case: documents and positions (numpy), key and query rows."""
    r = random.Random(c["layout"] + 1)
    lens = _lengths(c)
    docs, cells = [], []
    for n in lens:
        d, p = _shelves(r, n, c["docs"] or 1)
        if c["docs"] and not c["raster"]:  # patch by patch, the cells on no patch last
            order = np.argsort(np.where(d < 0, 1 << 30, d), kind="stable")
            d, p = d[order], p[order]
        docs.append(d)
        cells.append(p)
    prefix = [r.randint(0, n) // 2 for n in lens]
    return lens, docs, cells, prefix


def _adapters(c):
    """Adapter of each token: runs of tokens of one camera; a `bare` share without one."""
    r = random.Random(c["layout"])
    out = []
    while len(out) < c["tokens"]:
        run = 1 if c["tokens"] <= 64 else r.randint(1, max(2, c["tokens"] // 16))
        g = -1 if r.random() < c["bare"] else r.randrange(c["adapters"])
        if c["tokens"] <= 64 and g >= 0:
            g = len(out) % c["adapters"]
        out += [g] * run
    return out[:c["tokens"]]


def _slopes(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def _visible(c):
    """Visible (query, key) pairs of an attend case, and the rows of queries and keys."""
    lens, docs, _, prefix = _layout(c)
    pairs = 0
    for n, d, p in zip(lens, docs, prefix):
        p = p if c["prefix"] else 0
        if c["single"]:
            pairs += int((d == d[n - 1]).sum()) if c["docs"] and d[n - 1] >= 0 else n * (not c["docs"])
        elif c["docs"] and c["causal"]:
            i = np.arange(n)
            for v in np.unique(d[d >= 0]):
                at = i[d == v]  # sorted: the key at rank k is seen by later tokens and, in the
                pairs += len(at) * (len(at) + 1) // 2  # prefix, by the k earlier ones too
                inside = int((at < p).sum())
                pairs += inside * (inside - 1) // 2
        elif c["docs"]:
            pairs += int((np.bincount(d[d >= 0]).astype(np.int64) ** 2).sum()) if (d >= 0).any() else 0
        elif c["causal"]:
            pairs += n * (n + 1) // 2 + p * (p - 1) // 2
        else:
            pairs += n * n
    return pairs, (c["seqs"] if c["single"] else sum(lens)), sum(lens)


def work(case):
    c = case
    if c["kind"] == "project":
        got = [g for g in _adapters(c) if g >= 0]
        low = len(set(got)) * c["rank"] * (c["k"] + c["n"])
        return {"bytes": 2 * (c["tokens"] * (c["k"] + c["n"]) + c["n"] * c["k"] + low),
                "flops": 2 * c["tokens"] * c["k"] * c["n"]
                + 2 * len(got) * c["rank"] * (c["k"] + c["n"])}
    if c["kind"] == "rotate":
        rows = c["heads"] + c["kv_heads"] * (2 if c["cache"] else 1)
        values = c["tokens"] * rows * c["d"]
        table = 8 * min(c["positions"], c["tokens"] * c["axes"]) * c["rot"] // 2
        return {"bytes": 4 * values + 4 * c["tokens"] * (c["axes"] + 1) + table,
                "flops": 8 * values}
    pairs, q, k = _visible(c)
    return {"bytes": 4 * q * c["heads"] * c["d"] + 4 * k * c["kv_heads"] * c["d"]
            + (4 * (q + k) if c["docs"] else 0) + (8 * (q + k) if c["positions"] else 0),
            "flops": 4 * pairs * c["heads"] * c["d"]}


# ------------------------------------------------------------------------------ the inputs

def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = TYPES[c["type"]]

    def normal(*shape, gain=1.0):
        return torch.randn(shape, generator=gen, device=DEVICE).mul_(gain).to(dt)

    def ints(v):
        return torch.from_numpy(np.asarray(v, dtype=np.int32)).to(DEVICE)

    s = {"case": c}
    if c["kind"] == "project":
        s["x"] = normal(c["tokens"], c["k"])
        s["w"] = normal(c["n"], c["k"], gain=c["k"] ** -0.5)
        s["a"] = normal(c["adapters"], c["rank"], c["k"], gain=c["k"] ** -0.5)
        s["b"] = normal(c["adapters"], c["n"], c["rank"], gain=0.5 * c["rank"] ** -0.5)
        s["scale"] = 0.5 + torch.rand(c["adapters"], generator=gen, device=DEVICE)
        s["adapter"] = ints(_adapters(c))
    elif c["kind"] == "rotate":
        t, h, g, d = c["tokens"], c["heads"], c["kv_heads"], c["d"]
        qkv = normal(t, h + 2 * g, d)  # as one projection leaves them: q, k and v in one row
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]
        s["q_weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEVICE)).to(dt)
        s["k_weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEVICE)).to(dt)
        freq = 10000.0 ** (-torch.arange(c["rot"] // 2, device=DEVICE, dtype=torch.float64)
                           / (c["rot"] // 2))
        angle = torch.arange(c["positions"], device=DEVICE, dtype=torch.float64)[:, None] * freq
        s["table"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        s["pos"] = torch.randint(0, c["positions"], (t, c["axes"]), generator=gen, device=DEVICE,
                                 dtype=torch.int32)
        if c["cache"]:  # a cache with room for four times the tokens, each row of another token
            rows = 4 * t
            s["slot"] = torch.randperm(rows, generator=gen, device=DEVICE)[:t].contiguous()
            s["k_cache"], s["v_cache"] = normal(rows, g, d), normal(rows, g, d)
    else:
        lens, docs, cells, prefix = _layout(c)
        q_lens = [1] * c["seqs"] if c["single"] else lens
        q_rows, k_rows = sum(q_lens), sum(lens)
        s["q"] = normal(q_rows, c["heads"], c["d"], gain=3.0)
        s["k"] = normal(k_rows, c["kv_heads"], c["d"])
        s["v"] = normal(k_rows, c["kv_heads"], c["d"])
        begin = np.concatenate([[0], np.cumsum(lens)])
        s["q_begin"] = ints(np.concatenate([[0], np.cumsum(q_lens)]))
        s["kv_begin"] = torch.from_numpy(begin[:-1].astype(np.int64)).to(DEVICE)
        s["kv_len"] = ints(lens)
        s["max_q"], s["max_kv"] = max(q_lens), max(lens)
        last = begin[1:] - 1 if c["single"] else slice(None)
        docs, cells = np.concatenate(docs), np.concatenate(cells)
        s["k_doc"] = ints(docs) if c["docs"] else None
        s["q_doc"] = ints(docs[last]) if c["docs"] else None
        s["k_pos"] = ints(cells) if c["positions"] else None
        s["q_pos"] = ints(cells[last]) if c["positions"] else None
        s["prefix"] = ints(prefix) if c["prefix"] else None
        s["slope"] = (torch.tensor(_slopes(c["heads"]), device=DEVICE) if c["slopes"] else None)
        s["scale"] = c["d"] ** -0.5
    return s


# --------------------------------------------------------------------- the plain operators

def _project(s):
    x, w = s["x"].float(), s["w"].float()
    a, b = s["a"].float(), s["b"].float()
    groups, rank, k = a.shape
    h = (x @ a.reshape(groups * rank, k).t()).view(-1, groups, rank)
    mine = s["adapter"].long()[:, None] == torch.arange(groups, device=x.device)
    h = h * (mine * s["scale"])[:, :, None]
    low = h.view(-1, groups * rank) @ b.transpose(1, 2).reshape(groups * rank, -1)
    return (x @ w.t() + low).to(s["x"].dtype)


def _turn(s, v, weight):
    c = s["case"]
    rot, axes = c["rot"], c["axes"]
    half = rot // 2
    u = v.float()
    u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * weight.float()
    axis = torch.arange(half, device=v.device) * axes // half
    cs = s["table"][s["pos"].long()[:, axis], torch.arange(half, device=v.device)][:, None]
    cos, sin = cs[..., 0], cs[..., 1]
    if c["pairs"] == "half":
        one, two = u[..., :half], u[..., half:rot]
        turned = torch.cat([one * cos - two * sin, one * sin + two * cos], -1)
    else:
        one, two = u[..., 0:rot:2], u[..., 1:rot:2]
        turned = torch.stack([one * cos - two * sin, one * sin + two * cos], -1).flatten(-2)
    return torch.cat([turned, u[..., rot:]], -1).to(v.dtype)


def _rotate(s):
    q, k = _turn(s, s["q"], s["q_weight"]), _turn(s, s["k"], s["k_weight"])
    if not s["case"]["cache"]:
        return {"q": q, "k": k}
    s["k_cache"][s["slot"]] = k
    s["v_cache"][s["slot"]] = s["v"]
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"]}


def _attend(s):
    c = s["case"]
    group, max_q, max_kv = c["heads"] // c["kv_heads"], s["max_q"], s["max_kv"]
    dev = s["q"].device
    q_len = (s["q_begin"][1:] - s["q_begin"][:-1]).long()
    kv_len = s["kv_len"].long()
    i, j = torch.arange(max_q, device=dev), torch.arange(max_kv, device=dev)
    q_at = (s["q_begin"][:-1, None].long() + i).clamp(max=s["q"].shape[0] - 1)
    k_at = (s["kv_begin"][:, None] + j).clamp(max=s["k"].shape[0] - 1)
    # [sequence, kv head, query in group x query, d]
    q = s["q"].float()[q_at].view(-1, max_q, c["kv_heads"], group, c["d"])
    q = q.permute(0, 2, 3, 1, 4).reshape(-1, c["kv_heads"], group * max_q, c["d"])
    k = s["k"].float()[k_at].transpose(1, 2)
    v = s["v"].float()[k_at].transpose(1, 2)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    z = z.view(-1, c["kv_heads"], group, max_q, max_kv)
    if c["cap"] > 0:
        z = z.div_(c["cap"]).tanh_().mul_(c["cap"])
    at = (kv_len - q_len)[:, None] + i
    if s["slope"] is not None:
        if s["k_pos"] is not None:
            far = (s["q_pos"][q_at][:, :, None] - s["k_pos"][k_at][:, None]).abs().sum(-1)
        else:
            far = (at[:, :, None] - j).abs()
        slope = s["slope"].view(1, c["kv_heads"], group, 1, 1)
        z -= slope * far[:, None, None].float()
    see = (i < q_len[:, None])[:, :, None] & (j < kv_len[:, None])[:, None]
    if c["causal"]:
        early = j <= at[:, :, None]
        if s["prefix"] is not None:
            early = early | (j < s["prefix"][:, None])[:, None]
        see = see & early
    if s["k_doc"] is not None:
        d_q, d_k = s["q_doc"][q_at], s["k_doc"][k_at]
        see = see & (d_q[:, :, None] == d_k[:, None]) & (d_q >= 0)[:, :, None]
    z = z.masked_fill_(~see[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(-1, c["kv_heads"], group * max_q, max_kv), v)
    out = out.view(-1, c["kv_heads"], group, max_q, c["d"])
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    out = out.permute(0, 3, 1, 2, 4).reshape(-1, max_q, c["heads"], c["d"])
    return out[i < q_len[:, None]].to(s["q"].dtype)


PLAIN = {"project": _project, "rotate": _rotate, "attend": _attend}


# --------------------------------------------------------------------- the library's calls

def _bind(s):
    """Outputs, workspaces and argument blocks, which a serving program makes once."""
    from paper_2404_09267_amd import tg

    c = s["case"]
    if c["kind"] == "project":
        adapters = tg.Adapters(s["a"], s["b"], s["scale"])
        bufs = tg.ProjectBuffers(c["tokens"], c["k"], c["n"], TYPES[c["type"]], adapters)
        args = tg.project_args(s["x"], s["w"], bufs, adapters, s["adapter"])
        s["out"], s["call"], s["args"] = bufs.y, tg.project_raw, args
    elif c["kind"] == "rotate":
        q_out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        more = {}
        if c["cache"]:
            k_out = s["k_cache"]
            more = dict(v=s["v"], v_out=s["v_cache"], slot=s["slot"])
        else:
            k_out = torch.empty(s["k"].shape, dtype=s["k"].dtype, device=DEVICE)
        args = tg.rotate_args(s["q"], s["k"], s["q_weight"], s["k_weight"], s["table"], s["pos"],
                              q_out, k_out, eps=EPS, interleaved=c["pairs"] == "next", **more)
        s["out"] = {"q": q_out, "k": k_out}
        if c["cache"]:
            s["out"]["v"] = s["v_cache"]
        s["call"], s["args"] = tg.rotate_raw, args
    else:
        seqs = tg.Sequences(s["q_begin"], s["kv_begin"], s["kv_len"], s["max_q"], s["max_kv"],
                            prefix=s["prefix"])
        out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        bufs = tg.AttendBuffers(seqs, s["q"], s["k"])
        args = tg.attend_args(s["q"], s["k"], s["v"], seqs, out, bufs, scale=s["scale"],
                              cap=c["cap"], causal=c["causal"], q_doc=s["q_doc"],
                              k_doc=s["k_doc"], q_pos=s["q_pos"], k_pos=s["k_pos"],
                              slope=s["slope"])
        s["out"], s["call"], s["args"] = out, tg.attend_raw, args


def run(state):
    if not own:
        return PLAIN[state["case"]["kind"]](state)
    if "call" not in state:
        _bind(state)
    code = state["call"](state["args"])
    if code != 0:
        raise RuntimeError(f"{state['case']['kind']}: status {code}")
    return state["out"]


# ----------------------------------------------------------------------- 64-bit definitions

def _exact_project(s):
    x, w = s["x"].double(), s["w"].double()
    y = x @ w.t()
    for g in range(s["a"].shape[0]):
        rows = (s["adapter"] == g).nonzero()[:, 0]
        if len(rows):
            y[rows] += s["scale"][g].double() * ((x[rows] @ s["a"][g].double().t())
                                                 @ s["b"][g].double().t())
    return y


def _exact_turn(s, v, weight):
    c = s["case"]
    n = v.shape[-1]
    u = v.double()
    u = u / torch.sqrt(u.pow(2).sum(-1, keepdim=True) / n + EPS) * weight.double()
    out, half = u.clone(), c["rot"] // 2
    for p in range(half):
        i, j = (p, p + half) if c["pairs"] == "half" else (2 * p, 2 * p + 1)
        row = s["pos"][:, p * c["axes"] // half].long()
        cos, sin = s["table"][row, p, 0].double()[:, None], s["table"][row, p, 1].double()[:, None]
        out[..., i] = u[..., i] * cos - u[..., j] * sin
        out[..., j] = u[..., i] * sin + u[..., j] * cos
    return out


def _exact_rotate(s):
    q, k = _exact_turn(s, s["q"], s["q_weight"]), _exact_turn(s, s["k"], s["k_weight"])
    if not s["case"]["cache"]:
        return {"q": q, "k": k}
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    k_cache[s["slot"]], v_cache[s["slot"]] = k, s["v"].double()
    return {"q": q, "k": k_cache, "v": v_cache}


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    begin = s["q_begin"].tolist()
    for b, (first, n) in enumerate(zip(s["kv_begin"].tolist(), s["kv_len"].tolist())):
        q0, q1 = begin[b], begin[b + 1]
        j = torch.arange(n, device=out.device)
        i = torch.arange(n - (q1 - q0), n, device=out.device)
        see = torch.ones((q1 - q0, n), dtype=torch.bool, device=out.device)
        if c["causal"]:
            see &= j[None] <= i[:, None]
            if s["prefix"] is not None:
                see |= (j < s["prefix"][b])[None]
        if s["k_doc"] is not None:
            see &= s["q_doc"][q0:q1, None] == s["k_doc"][None, first:first + n]
            see &= s["q_doc"][q0:q1, None] >= 0
        if s["k_pos"] is not None:
            far = (s["q_pos"][q0:q1, None, 0] - s["k_pos"][None, first:first + n, 0]).abs()
            far = far + (s["q_pos"][q0:q1, None, 1] - s["k_pos"][None, first:first + n, 1]).abs()
        else:
            far = (i[:, None] - j[None]).abs()
        any_key = see.any(1)
        for h in range(c["heads"]):
            g = h * c["kv_heads"] // c["heads"]
            z = s["q"][q0:q1, h].double() @ s["k"][first:first + n, g].double().t() * s["scale"]
            if c["cap"] > 0:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if s["slope"] is not None:
                z = z - s["slope"][h].double() * far
            z = torch.where(see, z, torch.full_like(z, -math.inf))
            p = torch.softmax(z[any_key], -1)
            out[q0:q1, h][any_key] = p @ s["v"][first:first + n, g].double()
    return out


EXACT = {"project": _exact_project, "rotate": _exact_rotate, "attend": _exact_attend}


def exact(case, seed):
    s = prepare(case, seed)
    return EXACT[case["kind"]](s)
