"""Timed cases of the serving operators: page tables of a key-value cache (pages), attention of
single tokens over its pages (attend), the norms, gate and residual around a block (norm), rows
rounded to 8-bit integers (quantize) and the product of such rows (project_i8).

A program that serves many cameras keeps the keys and values of all requests in pages of one
cache. In a step every request brings one new token, or a prompt: the pages give each token its
row, its keys and values go there, and its query sees the rows of its own request. Between the
products of a layer lie the norms and the residual; the products themselves read weights of 8 bits.

The layout of a case (lengths, pages, gates) comes from its "layout" number, the values of its
tensors from the seed.

Kinds (`case["kind"]`):
  pages       from lengths and new tokens: pages given back and taken, tables, a row for each token
  attend      one query a sequence against its pages
  norm        x_scale x + y_scale gate norm(y), and the norm of that
  quantize    a row's values over its largest / 127, to the nearest integer
  project_i8  sums of products of 8-bit integers, times a token's and an output's scale
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
        # a step of 64 requests of one new token each: latency
        dict(name="pages_step_64", kind="pages", seqs=64, length=1600, page=16, prompts=0.0,
             prompt=1, ended=0.0, spare=1.0, layout=1),
        # requests in motion: some bring prompts of up to 4,096 tokens, some have ended
        dict(name="pages_mixed", kind="pages", seqs=512, length=8192, page=64, prompts=0.15,
             prompt=4096, ended=0.1, spare=1.0, layout=2),
        # one query of each of 20 cameras, up to a quarter of a 1280 x 1280 canvas each
        dict(name="attend_20cam", kind="attend", seqs=20, length=1600, page=16, heads=16,
             kv_heads=4, d=64, cap=30.0, slopes=False, window=0, type="bf16", layout=3),
        # odd counts, pages that end inside everything else, a window, bias by distance
        dict(name="attend_odd", kind="attend", seqs=33, length=3001, page=24, heads=14,
             kv_heads=2, d=80, cap=0.0, slopes=True, window=1111, type="f16", layout=4),
        # 8 long caches
        dict(name="attend_long", kind="attend", seqs=8, length=100003, page=64, heads=16,
             kv_heads=2, d=128, cap=0.0, slopes=False, window=0, type="bf16", layout=5),
        # one new token of each of 20 cameras, gates by camera: latency
        dict(name="norm_single_20cam", kind="norm", tokens=20, n=1024, first="rms", then="rms",
             bias=False, gates=20, type="bf16", layout=6),
        # the tokens of four 1280 x 1280 canvases through a large layer
        dict(name="norm_4canvas", kind="norm", tokens=25600, n=4096, first="layer", then="rms",
             bias=True, gates=20, type="bf16", layout=7),
        # odd sizes, as after a ragged batch of prompts
        dict(name="quantize_odd", kind="quantize", tokens=1777, k=1160, type="f16", layout=8),
        # the tokens of four canvases before a large layer
        dict(name="quantize_4canvas", kind="quantize", tokens=25600, k=4096, type="bf16", layout=9),
        # one new token of each of 8 cameras through a small layer: latency
        dict(name="i8_single_8cam", kind="project_i8", tokens=8, k=1024, n=1536, type="bf16",
             layout=10),
        # odd sizes
        dict(name="i8_odd", kind="project_i8", tokens=1777, k=1168, n=2051, type="f16", layout=11),
        # the tokens of four canvases through a large layer
        dict(name="i8_4canvas", kind="project_i8", tokens=25600, k=4096, n=4096, type="bf16",
             layout=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pages", "attend", "norm", "quantize", "project_i8"])
    layout, kind_type = rng.randrange(1 << 30), rng.choice(["f16", "bf16"])
    if kind == "pages":
        prompts = rng.choice([0.0, 0.1, 0.3])
        return dict(kind=kind, seqs=_log(rng, 1, 512), length=_log(rng, 1, 8192),
                    page=rng.choice([8, 16, 24, 32, 64, 128]), prompts=prompts,
                    prompt=_log(rng, 2, 4096) if prompts else 1, ended=rng.choice([0.0, 0.1]),
                    spare=rng.choice([1.0, 1.0, 0.5]), layout=layout)
    if kind == "attend":
        kv = rng.choice([1, 2, 4])
        heads, length = min(kv * rng.choice([1, 2, 4, 7, 8]), 16), _log(rng, 1, 100003)
        seqs = max(1, min(_log(rng, 1, 256), 8 * 100003 * 2 // (length * kv)))
        return dict(kind=kind, seqs=seqs, length=length, page=rng.choice([8, 16, 24, 32, 64, 128]),
                    heads=heads, kv_heads=kv, d=rng.choice([32, 40, 64, 72, 96, 128]),
                    cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.4,
                    window=rng.choice([0, 0, 0, 100, 4096]), type=kind_type, layout=layout)
    if kind == "norm":
        return dict(kind=kind, tokens=_log(rng, 1, 25600), n=rng.choice([1, 4, 8]) * _log(rng, 8, 512),
                    first=rng.choice(["none", "rms", "layer"]), then=rng.choice(["rms", "layer"]),
                    bias=rng.random() < 0.5, gates=rng.choice([0, 1, 20]), type=kind_type,
                    layout=layout)
    if kind == "quantize":
        return dict(kind=kind, tokens=_log(rng, 1, 25600), k=rng.choice([1, 8]) * _log(rng, 8, 512),
                    type=kind_type, layout=layout)
    return dict(kind=kind, tokens=_log(rng, 1, 25600), k=16 * _log(rng, 4, 256),
                n=_log(rng, 100, 4096), type=kind_type, layout=layout)


# ----------------------------------------------------------------------------- the layouts

def _spread(r, longest, count):
    """Lengths: the first is the longest, the others spread below it."""
    return [longest] + [r.randint(max(1, longest // 8), longest) for _ in range(count - 1)]


def _requests(c):
    """Rows held, new tokens and whether it has ended, of each request; spare pages."""
    r = random.Random(c["layout"])
    held = _spread(r, c["length"], c["seqs"])
    ended = [r.random() < c["ended"] for _ in held]
    new = [0 if e else r.randint(1, c["prompt"]) if r.random() < c["prompts"] else 1 for e in ended]
    held = [n if k < 2 else 0 for n, k in zip(held, new)]  # one with a prompt has just come
    page = c["page"]
    take = sum(-(-(n + k) // page) - -(-n // page) for n, k, e in zip(held, new, ended) if not e)
    give = sum(-(-n // page) for n, e in zip(held, ended) if e)
    # with spare 1 all find pages, with less the last requests do not
    spare = take + 8 if c["spare"] >= 1 else max(0, int(take * c["spare"]) - give)
    return held, new, ended, spare


def _key_counts(c):
    r = random.Random(c["layout"])
    return _spread(r, c["length"], c["seqs"])


def _gate_rows(c):
    """Gate of each token: runs of tokens of one camera."""
    r = random.Random(c["layout"])
    out = []
    while len(out) < c["tokens"]:
        run = 1 if c["tokens"] <= 64 else r.randint(1, max(2, c["tokens"] // 16))
        out += [r.randrange(c["gates"])] * run
    return out[:c["tokens"]]


def _pages_of(lens, page, spare, seed):
    """Tables (-1 where there is no page) and the other pages, in the order that a long run of
    requests leaves: none."""
    count = [-(-n // page) for n in lens]
    order = np.random.RandomState(seed % (1 << 31)).permutation(sum(count) + spare).astype(np.int32)
    table = np.full((len(lens), max(max(count), 1)), -1, dtype=np.int32)
    at = 0
    for row, n in zip(table, count):
        row[:n] = order[at:at + n]
        at += n
    return table, order[at:]


def work(case):
    c = case
    if c["kind"] == "pages":
        held, new, ended, spare = _requests(c)
        page = c["page"]
        moved = sum(-(-n // page) if e else -(-(n + k) // page) - -(-n // page)
                    for n, k, e in zip(held, new, ended))
        return {"bytes": 16 * c["seqs"] + 8 * moved + 12 * sum(new), "flops": 0}
    if c["kind"] == "attend":
        keys = sum(min(n, c["window"] or n) for n in _key_counts(c))
        return {"bytes": 4 * keys * c["kv_heads"] * c["d"] + 4 * keys // c["page"]
                + 4 * c["seqs"] * c["heads"] * c["d"],
                "flops": 4 * keys * c["heads"] * c["d"]}
    if c["kind"] == "norm":
        vectors = c["gates"] + (2 + 2 * c["bias"] if c["first"] != "none" else 1 + c["bias"])
        return {"bytes": 8 * c["tokens"] * c["n"] + 2 * vectors * c["n"],
                "flops": 12 * c["tokens"] * c["n"]}
    if c["kind"] == "quantize":
        return {"bytes": 3 * c["tokens"] * c["k"] + 4 * c["tokens"],
                "flops": 3 * c["tokens"] * c["k"]}
    return {"bytes": c["k"] * (c["tokens"] + c["n"]) + 2 * c["tokens"] * c["n"],
            "flops": 2 * c["tokens"] * c["k"] * c["n"]}


# ------------------------------------------------------------------------------ the inputs

def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = TYPES.get(c.get("type"))

    def normal(*shape, gain=1.0):
        return torch.randn(shape, generator=gen, device=DEVICE).mul_(gain).to(dt)

    def dev(v, kind=np.int32):
        return torch.from_numpy(np.ascontiguousarray(v, dtype=kind)).to(DEVICE)

    s = {"case": c}
    if c["kind"] == "pages":
        held, new, ended, spare = _requests(c)
        most = max(n + k for n, k in zip(held, new))
        table, free = _pages_of(held, c["page"], spare, int(seed))
        wide = np.full((c["seqs"], -(-most // c["page"])), -1, dtype=np.int32)
        wide[:, :table.shape[1]] = table[:, :wide.shape[1]]
        n_pages = int((table >= 0).sum()) + spare
        stack = np.full(n_pages, -1, dtype=np.int32)
        stack[:spare] = free
        s["n_tokens"] = sum(new)
        s["q_begin"] = dev(np.concatenate([[0], np.cumsum(new)]))
        s["kv_len"], s["table"], s["free"] = dev(held), dev(wide), dev(stack)
        s["n_free"] = dev([spare])
        s["release"] = dev(ended) if c["ended"] else None
    elif c["kind"] == "attend":
        lens = _key_counts(c)
        table, _ = _pages_of(lens, c["page"], 3, int(seed))
        rows = (int((table >= 0).sum()) + 3) * c["page"]
        s["table"], s["kv_len"], s["max_kv"] = dev(table), dev(lens), max(lens)
        s["q"] = normal(c["seqs"], c["heads"], c["d"], gain=3.0)
        s["k"] = normal(rows, c["kv_heads"], c["d"])
        s["v"] = normal(rows, c["kv_heads"], c["d"])
        s["slope"] = (torch.tensor([2.0 ** (-8.0 * (h + 1) / c["heads"])
                                    for h in range(c["heads"])], device=DEVICE)
                      if c["slopes"] else None)
        s["scale"] = c["d"] ** -0.5
    elif c["kind"] == "norm":
        t, n = c["tokens"], c["n"]
        s["x"], s["y"] = normal(t, n, gain=4.0), normal(t, n) + normal(n)
        s["weight"], s["y_weight"] = 1 + normal(n, gain=0.2), 1 + normal(n, gain=0.2)
        s["bias"], s["y_bias"] = ((normal(n, gain=0.1), normal(n, gain=0.1)) if c["bias"]
                                  else (None, None))
        if c["first"] == "none":
            s["y_weight"] = s["y_bias"] = None
        s["gate"] = 0.5 + normal(c["gates"], n, gain=0.2) if c["gates"] else None
        s["gate_row"] = dev(_gate_rows(c)) if c["gates"] > 1 else None
        s["x_scale"], s["y_scale"] = 0.9, 0.5
    elif c["kind"] == "quantize":
        loud = torch.rand(c["k"], generator=gen, device=DEVICE) < 0.01  # a few channels stand out
        s["x"] = normal(c["tokens"], c["k"]) * (1 + 20 * loud).to(dt)
    else:
        def ints(*shape):
            v = torch.randn(shape, generator=gen, device=DEVICE).mul_(36).round_()
            return v.clamp_(-127, 127).to(torch.int8)

        s["x"], s["w"] = ints(c["tokens"], c["k"]), ints(c["n"], c["k"])
        s["x_scale"] = (1 + torch.rand(c["tokens"], generator=gen, device=DEVICE)) / 36
        s["w_scale"] = (1 + torch.rand(c["n"], generator=gen, device=DEVICE)) / 36 * c["k"] ** -0.5
    return s


# --------------------------------------------------------------------- the plain operators

def _pages(s):
    c = s["case"]
    page, (seqs, cols) = c["page"], s["table"].shape
    table, kv_len, begin = s["table"].long(), s["kv_len"].long(), s["q_begin"].long()
    n_pages, col = s["free"].numel(), torch.arange(cols, device=DEVICE)
    ended = s["release"] != 0 if s["release"] is not None else torch.zeros_like(kv_len).bool()
    held = (kv_len + page - 1) // page
    back = (col < torch.where(ended, held, 0)[:, None]).view(-1)
    at = torch.where(back, s["n_free"].long() + torch.cumsum(back, 0) - 1, n_pages)
    stack = torch.cat([s["free"].long(), table.new_zeros(1)])
    stack = stack.scatter(0, at.clamp(max=n_pages), table.view(-1))
    top = (s["n_free"].long() + back.sum()).clamp(max=n_pages)
    start, have = torch.where(ended, 0, kv_len), torch.where(ended, 0, held)
    new = begin[1:] - begin[:-1]
    room = start + new <= cols * page
    need = torch.where(room, (start + new + page - 1) // page - have, 0)
    upto = torch.cumsum(need, 0)
    fits = room & ((need == 0) | (upto <= top))
    taken = torch.where(fits & (need > 0), upto, 0).amax(0, keepdim=True)
    which = (upto - need)[:, None] + col - have[:, None]
    mine = fits[:, None] & (col >= have[:, None]) & (col < (have + need)[:, None])
    table = torch.where(mine, stack[(top - 1 - which).clamp(0, n_pages)], table)
    token = torch.arange(s["n_tokens"], device=DEVICE)
    seq = torch.bucketize(token, begin[1:], right=True).clamp(max=seqs - 1)
    placed = fits[seq] & (token < begin[-1])
    pos = start[seq] + token - begin[seq]
    slot = table[seq, (pos // page).clamp(max=cols - 1)] * page + pos % page
    return {"table": table.int(), "kv_len": torch.where(fits, start + new, start).int(),
            "free": stack[:-1].int(), "n_free": (top - taken).int(),
            "refused": (~fits).sum(0, keepdim=True).int(),
            "slot": torch.where(placed, slot, -1), "pos": torch.where(placed, pos, 0).int()[:, None]}


def _attend(s):
    c = s["case"]
    group, n, page = c["heads"] // c["kv_heads"], s["max_kv"], c["page"]
    j = torch.arange(n, device=DEVICE)
    kv_len = s["kv_len"].long()[:, None]
    at = (s["table"].long()[:, j // page] * page + j % page).clamp(min=0)
    k, v = s["k"][at].float().transpose(1, 2), s["v"][at].float().transpose(1, 2)
    q = s["q"].float().view(-1, c["kv_heads"], group, c["d"])
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    if c["cap"] > 0:
        z = torch.tanh(z / c["cap"]) * c["cap"]
    if s["slope"] is not None:
        z = z - s["slope"].view(1, c["kv_heads"], group, 1) * (kv_len - 1 - j)[:, None, None].float()
    see = j < kv_len
    if c["window"]:
        see = see & (j >= kv_len - c["window"])
    z = z.masked_fill(~see[:, None, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    out = torch.matmul(p, v.contiguous()) / p.sum(-1, keepdim=True)
    return out.view(-1, c["heads"], c["d"]).to(s["q"].dtype)


def _normed(u, kind, weight, bias):
    if kind == "layer":
        u = u - u.mean(-1, keepdim=True)
    if kind != "none":
        u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS)
    u = u * weight.float() if weight is not None else u
    return u + bias.float() if bias is not None else u


def _norm(s):
    c = s["case"]
    y = _normed(s["y"].float(), c["first"], s["y_weight"], s["y_bias"])
    if s["gate"] is not None:
        y = y * (s["gate"].float()[s["gate_row"].long()] if s["gate_row"] is not None
                 else s["gate"].float()[:1])
    r = s["x_scale"] * s["x"].float() + s["y_scale"] * y
    h = _normed(r, c["then"], s["weight"], s["bias"])
    return {"x": r.to(s["x"].dtype), "h": h.to(s["x"].dtype)}


def _quantize(s):
    scale = (s["x"].abs().amax(1).double() / 127).float()
    q = torch.round(s["x"].double() / torch.where(scale > 0, scale, 1.0).double()[:, None])
    return {"q": q.to(torch.int8), "scale": scale}


def _project_i8(s):
    sums = s["x"].float() @ s["w"].float().t()
    return (sums * (s["x_scale"][:, None] * s["w_scale"])).to(TYPES[s["case"]["type"]])


PLAIN = {"pages": _pages, "attend": _attend, "norm": _norm, "quantize": _quantize,
         "project_i8": _project_i8}


# --------------------------------------------------------------------- the library's calls

def _bind(s):
    """Outputs, workspaces and argument blocks, which a serving program makes once."""
    from paper_2404_09267_amd import tg

    c = s["case"]
    like = dict(device=DEVICE, dtype=TYPES.get(c.get("type")))
    if c["kind"] == "pages":
        pages = tg.Pages(s["table"], s["kv_len"], c["page"], s["free"], s["n_free"])
        bufs = tg.PagesBuffers(pages, s["n_tokens"])
        after = tg.Pages(s["table"], torch.empty_like(s["kv_len"]), c["page"], s["free"],
                         torch.empty_like(s["n_free"]))
        s["out"] = {"table": s["table"], "kv_len": after.kv_len, "free": s["free"],
                    "n_free": after.n_free, "refused": bufs.refused, "slot": bufs.slot,
                    "pos": bufs.pos}
        s["call"] = tg.pages_raw
        s["args"] = tg.pages_args(pages, s["q_begin"], bufs, release=s["release"], after=after)
    elif c["kind"] == "attend":
        pages = tg.Pages(s["table"], s["kv_len"], c["page"])
        s["out"] = torch.empty(s["q"].shape, **like)
        bufs = tg.AttendPagesBuffers(s["q"], s["k"], s["max_kv"])
        s["call"] = tg.attend_pages_raw
        s["args"] = tg.attend_pages_args(s["q"], s["k"], s["v"], pages, s["out"], bufs,
                                         scale=s["scale"], cap=c["cap"], window=c["window"],
                                         slope=s["slope"])
    elif c["kind"] == "norm":
        kinds = {"none": tg.NORM_NONE, "rms": tg.NORM_RMS, "layer": tg.NORM_LAYER}
        x_out, h = torch.empty(s["x"].shape, **like), torch.empty(s["x"].shape, **like)
        s["out"], s["call"] = {"x": x_out, "h": h}, tg.norm_raw
        s["args"] = tg.norm_args(s["x"], x_out, h, y=s["y"], y_norm=kinds[c["first"]],
                                 y_weight=s["y_weight"], y_bias=s["y_bias"], gate=s["gate"],
                                 gate_row=s["gate_row"], x_scale=s["x_scale"],
                                 y_scale=s["y_scale"], norm=kinds[c["then"]], weight=s["weight"],
                                 bias=s["bias"], eps=EPS)
    elif c["kind"] == "quantize":
        q = torch.empty(s["x"].shape, dtype=torch.int8, device=DEVICE)
        scale = torch.empty(c["tokens"], device=DEVICE)
        s["out"], s["call"] = {"q": q, "scale": scale}, tg.quantize_raw
        s["args"] = tg.quantize_args(s["x"], q, scale)
    else:
        s["out"] = torch.empty((c["tokens"], c["n"]), **like)
        s["call"] = tg.project_i8_raw
        s["args"] = tg.project_i8_args(s["x"], s["x_scale"], s["w"], s["w_scale"], s["out"])


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

def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["kv_len"].tolist()):
        j = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device=DEVICE)
        rows = s["table"][b].long()[torch.div(j, c["page"], rounding_mode="floor")]
        rows = rows * c["page"] + j.remainder(c["page"])
        for h in range(c["heads"]):
            g = h * c["kv_heads"] // c["heads"]
            z = s["k"][rows, g].double() @ s["q"][b, h].double() * s["scale"]
            if c["cap"] > 0:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if s["slope"] is not None:
                z = z - s["slope"][h].double() * (n - 1 - j)
            out[b, h] = torch.softmax(z, 0) @ s["v"][rows, g].double()
    return out


def _exact_norm(s):
    c = s["case"]

    def normed(u, kind, weight, bias):
        if kind != "none":
            mean = u.sum(1, keepdim=True) / c["n"] if kind == "layer" else 0.0
            u = (u - mean) / torch.sqrt(((u - mean) ** 2).sum(1, keepdim=True) / c["n"] + EPS)
        if weight is not None:
            u = weight.double() * u
        return u if bias is None else u + bias.double()

    r = normed(s["y"].double(), c["first"], s["y_weight"], s["y_bias"])
    if s["gate"] is not None:
        rows = s["gate_row"].long() if s["gate_row"] is not None else torch.zeros(
            c["tokens"], dtype=torch.long, device=DEVICE)
        r = s["gate"].double().index_select(0, rows) * r
    r = s["x_scale"] * s["x"].double() + s["y_scale"] * r
    return {"x": r, "h": normed(r, c["then"], s["weight"], s["bias"])}


def exact(case, seed):
    c = case
    if c["kind"] == "pages":
        return None
    s = prepare(c, seed)
    if c["kind"] == "attend":
        return _exact_attend(s)
    if c["kind"] == "norm":
        return _exact_norm(s)
    if c["kind"] == "quantize":
        return {"q": None, "scale": s["x"].double().abs().max(1).values / 127}
    return s["x_scale"].double()[:, None] * (s["x"].double() @ s["w"].double().t()) * s["w_scale"].double()
