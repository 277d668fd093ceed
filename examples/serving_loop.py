"""Requests of many cameras through transformer layers over one paged cache, in 8-bit weights.

    python examples/serving_loop.py

A request is a prompt (a patch's tokens, say) and the tokens that come after it, one a step; which
those are a sampler would say from the results, here they are given. Requests come and go; each has
a place among the sequences while it lasts, and what it holds of the cache are pages that come from
whoever has ended. A step is

    tg_pages         pages given back and taken, a cache row and a position for every new token
  and per layer
    tg_norm          the norm before attention, of the residual that the layer before has left
    tg_quantize      rows to 8-bit integers
    tg_project_i8    queries, keys and values
    tg_rotate        norm and rotation of queries and keys; keys and values go to their cache rows
    tg_attend_pages  each request's newest token over its own rows; the tokens of prompts see each
                     other by tg_attend
    tg_quantize, tg_project_i8   heads -> embedding
    tg_norm          the norm after attention, the camera's gate, the residual, and the norm before
                     the feed-forward block, which is one more product here

Steps of single tokens have the same shapes whoever is there: they are captured once and replayed,
with lengths, ends and places read on the device.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2404_09267_amd import tg  # noqa: E402

DTYPE = torch.bfloat16


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


class Rows8:
    """Rows as 8-bit integers with a scale each: a weight's outputs, or tokens."""

    def __init__(self, x):
        self.q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
        self.scale = torch.empty(x.shape[0], device="cuda")
        tg.quantize(x, self.q, self.scale)


class Layer:
    """Random weights of one layer, with a gate per camera."""

    def __init__(self, cameras, heads, kv_heads, d, g):
        def normal(*shape, gain):
            return (torch.randn(shape, generator=g, device="cuda") * gain).to(DTYPE)

        width, qkv = heads * d, (heads + 2 * kv_heads) * d
        self.qkv = Rows8(normal(qkv, width, gain=width ** -0.5))
        self.out = Rows8(normal(width, width, gain=width ** -0.5))
        self.mix = Rows8(normal(width, width, gain=width ** -0.5))
        self.gate = 1 + normal(cameras, width, gain=0.2)
        self.norms = [1 + normal(width, gain=0.1) for _ in range(4)]
        self.q_weight, self.k_weight = (1 + normal(d, gain=0.1) for _ in range(2))


class Server:
    """Layers, a paged cache for `places` requests at once, and the step over them."""

    def __init__(self, cameras=6, places=8, n_layers=2, heads=8, kv_heads=2, d=64, page=16,
                 n_pages=96, most=512, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.d = heads, kv_heads, d
        self.width, self.most = heads * d, most
        self.layers = [Layer(cameras, heads, kv_heads, d, g) for _ in range(n_layers)]
        self.pages = tg.Pages.empty(places, most // page, n_pages, page)
        self.cache = [torch.zeros((2, n_pages * page, kv_heads, d), dtype=DTYPE, device="cuda")
                      for _ in range(n_layers)]
        angle = (torch.arange(most, device="cuda")[:, None].double()
                 * 1000.0 ** (-torch.arange(d // 2, device="cuda").double() / (d // 2)))
        self.table = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        self.refused = ints([0])  # of the last step: requests whose tokens found no pages
        self.graph = None

    def project(self, x, w):
        rows, y = Rows8(x), torch.empty((x.shape[0], w.q.shape[0]), dtype=DTYPE, device="cuda")
        tg.project_i8(rows.q, rows.scale, w.q, w.scale, y)
        return y

    def attend(self, q, layer, begin, slot, prompts):
        """Results of all new tokens: the newest of each request over its pages; of a prompt, which
        starts its request, all of them over each other."""
        k, v = self.cache[layer]
        out = torch.zeros_like(q)
        scale = self.d ** -0.5
        if prompts is not None:
            tokens = q.shape[0]
            seqs = tg.Sequences(begin, prompts[0], prompts[1], tokens, tokens)
            tg.attend(q, k[slot.clamp(min=0)], v[slot.clamp(min=0)], seqs, out,
                      tg.AttendBuffers(seqs, q, k), scale, causal=True)
        bufs = tg.AttendPagesBuffers(q, k, self.most, n_seqs=self.pages.n_seqs)
        tg.attend_pages(q, k, v, self.pages, out, bufs, scale, q_begin=begin)
        return out.view(-1, self.width)

    def forward(self, x, camera, begin, release, prompts=None):
        """New tokens x [tokens, width] of the requests, request by request; their results."""
        bufs = tg.PagesBuffers(self.pages, x.shape[0])
        bufs.refused = self.refused
        tg.pages(self.pages, begin, bufs, release=release)
        h, g, d = self.heads, self.kv_heads, self.d
        y = None  # what the layer before has made of x
        for i, layer in enumerate(self.layers):
            a, b, c, e = layer.norms
            n = torch.empty_like(x)
            r = torch.empty_like(x)
            tg.norm(x, r, n, y=y, weight=a)
            x = r
            qkv = self.project(n, layer.qkv).view(-1, h + 2 * g, d)
            q = torch.empty((x.shape[0], h, d), dtype=DTYPE, device="cuda")
            tg.rotate(qkv[:, :h], qkv[:, h:h + g], layer.q_weight, layer.k_weight, self.table,
                      bufs.pos, q, self.cache[i][0], qkv[:, h + g:], self.cache[i][1], bufs.slot)
            heads = self.attend(q, i, begin, bufs.slot, prompts)
            tg.norm(x, x, n, y=self.project(heads, layer.out), y_norm=tg.NORM_RMS, y_weight=b,
                    gate=layer.gate, gate_row=camera, weight=c)
            y = self.project(n, layer.mix)
        out = torch.empty_like(x)
        tg.norm(x, None, out, y=y, weight=e)
        return out

    def capture(self):
        """The step of single tokens as a graph over buffers of its own."""
        places = self.pages.n_seqs
        self.x = torch.zeros((places, self.width), dtype=DTYPE, device="cuda")
        self.camera, self.release = ints([0] * places), ints([0] * places)
        self.begin = ints([0] * (places + 1))
        # once outside the graph: nobody has a token, so that nothing changes
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.forward(self.x, self.camera, self.begin, self.release)
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.y = self.forward(self.x, self.camera, self.begin, self.release)

    def step(self, tokens, cameras, ended, replay=True):
        """One step: tokens[p] is the list of place p's new tokens ([width] each), None or empty for
        none; ended: places whose requests have ended before it. Returns, by place, the results;
        raises where a request found no pages for its tokens."""
        new = [t if t is not None else [] for t in tokens]
        begin = np.concatenate([[0], np.cumsum([len(t) for t in new])])
        flat = [row for t in new for row in t]
        release = [int(p in ended) for p in range(len(new))]
        camera = [cameras[p] for p, t in enumerate(new) for _ in t]
        if replay and all(len(t) <= 1 for t in new):
            if self.graph is None:
                self.capture()
            if flat:
                self.x[:len(flat)].copy_(torch.stack(flat))
                self.camera[:len(flat)].copy_(ints(camera))
            self.begin.copy_(ints(begin.tolist()))
            self.release.copy_(ints(release))
            self.graph.replay()
            y = self.y.clone()
        else:
            first = np.where(np.diff(begin) > 0, begin[:-1], 0)
            prompts = (ints(first.tolist(), torch.int64), ints(np.diff(begin).tolist()))
            if all(len(t) <= 1 for t in new):
                prompts = None
            y = self.forward(torch.stack(flat), ints(camera), ints(begin.tolist()),
                             ints(release), prompts)
        if int(self.refused):  # their tokens are nowhere, and no results
            raise RuntimeError("the cache is full")
        return [y[begin[p]:begin[p + 1]] for p in range(len(new))]


def requests(count, cameras, width, seed):
    """(camera, prompt, the tokens that follow) of each."""
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = lambda n: torch.randn((int(n), width), generator=g, device="cuda").to(DTYPE)
    return [(int(r.integers(cameras)), rows(r.integers(1, 90)), rows(r.integers(1, 30)))
            for _ in range(count)]


def serve(server, todo, replay=True):
    """All requests, as many at once as there are places. Results of each: its prompt's last token
    and all that follow."""
    places = server.pages.n_seqs
    waiting, at, ended = list(range(len(todo))), [None] * places, set()
    made = [[] for _ in todo]
    while waiting or any(i is not None for i in at):
        for p in range(places):
            if at[p] is None and waiting:
                at[p] = waiting.pop(0)
        tokens = [None] * places
        for p, i in enumerate(at):
            if i is not None:
                n = len(made[i])
                tokens[p] = list(todo[i][2][n - 1:n] if n else todo[i][1])
        if any(t is not None and len(t) > 1 for t in tokens):  # prompts are a step of their own
            tokens = [t if t is not None and len(t) > 1 else None for t in tokens]
        results = server.step(tokens, [todo[i][0] if i is not None else 0 for i in at], ended,
                              replay)
        ended = set()
        for p in range(places):
            if tokens[p]:
                i = at[p]
                made[i].append(results[p][-1])
                if len(made[i]) > len(todo[i][2]):
                    at[p] = None
                    ended.add(p)
    if replay:  # a step without tokens, in which the last requests give their pages back
        server.step([None] * places, [0] * places, ended)
    return [torch.stack(m) for m in made]


def main(seed: int = 0) -> float:
    cameras, count = 6, 20
    server = Server(cameras=cameras)
    todo = requests(count, cameras, server.width, seed)
    together = serve(server, todo)
    held = int(server.pages.free.shape[0]) - int(server.pages.n_free)
    worst = 0.0
    for i in range(0, count, 3):
        alone = serve(Server(cameras=cameras), todo[i:i + 1], replay=False)[0]
        worst = max(worst, float((together[i].float() - alone.float()).norm()
                                 / alone.float().norm()))
    print(f"{count} requests, {sum(len(t) for t in together)} results, {held} pages still held; "
          f"every third against itself alone: largest relative difference {worst:.1e}")
    return worst


if __name__ == "__main__":
    main()
