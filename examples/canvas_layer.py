"""One attention layer of a transformer over stitched canvases, and single tokens after it.

    python examples/canvas_layer.py

Patches of several cameras are packed and stitched as for any detector (tg_plan_pack,
tg_stitch). Each 16 x 16 cell of a canvas is a token. A cell belongs to the patch that holds its
centre, as a detector's box does; its position is that of its pixels in the patch's frame, and its
adapter that of the frame's camera. The layer is then

    tg_project  cells -> embedding;  embedding -> queries, keys and values, with the camera's adapter
    tg_rotate   norm of queries and keys per head, rotated by x and y in the frame
    tg_attend   a token sees the tokens of its own patch, nearer ones more
    tg_project  heads -> embedding, with the camera's adapter

so that a patch comes out as if it had been alone, whatever shares its canvas. Afterwards one new
token per patch (a query about it) goes through the same calls against the patch's keys and
values, which lie in a cache, row by row.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2404_09267_amd import tg  # noqa: E402
from paper_2404_09267_amd import workload as W  # noqa: E402

CELL = 16
DTYPE = torch.bfloat16


def cells(plan: tg.Plan, rois: np.ndarray, canvas: int):
    """Per cell of all canvases, patch by patch: (canvas, cell y, cell x), the patch (its place in
    plan.order), the frame and the position in the frame, in cells. Cells on no patch are left
    out: they would see nothing."""
    side = canvas // CELL
    centre = np.arange(side) * CELL + CELL // 2
    at, patch, frame, pos = [], [], [], []
    for p, i in enumerate(plan.order):
        c, dx, dy = plan.place[i]
        f, sx, sy, w, h = rois[i]
        xs = np.nonzero((centre >= dx) & (centre < dx + w))[0]
        ys = np.nonzero((centre >= dy) & (centre < dy + h))[0]
        y, x = (v.reshape(-1) for v in np.meshgrid(ys, xs, indexing="ij"))
        at.append(np.stack([np.full(len(x), c), y, x], 1))
        patch.append(np.full(len(x), p))
        frame.append(np.full(len(x), f))
        pos.append(np.stack([(centre[x] - dx + sx) // CELL, (centre[y] - dy + sy) // CELL], 1))
    one = lambda v: np.ascontiguousarray(np.concatenate(v), dtype=np.int32)
    return one(at), one(patch), one(frame), one(pos)


class Layer:
    """Random weights of one layer, with an adapter per camera."""

    def __init__(self, cameras: int, frame_cells: int, heads: int = 8, kv_heads: int = 2,
                 d: int = 64, rank: int = 8, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, gain):
            return (torch.randn(shape, generator=g, device="cuda") * gain).to(DTYPE)

        def adapters(k, n):
            return tg.Adapters(normal(cameras, rank, k, gain=k ** -0.5),
                               normal(cameras, n, rank, gain=0.2),
                               torch.ones(cameras, device="cuda"))

        self.heads, self.kv_heads, self.d, self.width = heads, kv_heads, d, heads * d
        cell = 3 * CELL * CELL
        qkv = (heads + 2 * kv_heads) * d
        self.embed = normal(self.width, cell, gain=cell ** -0.5)
        self.qkv, self.out = (normal(n, self.width, gain=self.width ** -0.5)
                              for n in (qkv, self.width))
        self.qkv_low, self.out_low = adapters(self.width, qkv), adapters(self.width, self.width)
        self.q_weight, self.k_weight = (1 + normal(d, gain=0.1) for _ in range(2))
        self.slope = 0.5 ** torch.arange(1, heads + 1, device="cuda").float()
        angle = (torch.arange(frame_cells, device="cuda")[:, None].double()
                 * 100.0 ** (-torch.arange(d // 2, device="cuda").double() / (d // 2)))
        self.table = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()

    def project(self, x, w, low=None, camera=None):
        bufs = tg.ProjectBuffers(x.shape[0], x.shape[1], w.shape[0], DTYPE, low)
        tg.project(x, w, bufs, low, camera)
        return bufs.y

    def queries(self, x, camera, pos, k_rows, v_rows, slot=None):
        """Rotated queries of tokens x; their keys and values go to k_rows and v_rows."""
        h, g, d = self.heads, self.kv_heads, self.d
        qkv = self.project(x, self.qkv, self.qkv_low, camera).view(-1, h + 2 * g, d)
        q = torch.empty((x.shape[0], h, d), dtype=DTYPE, device="cuda")
        tg.rotate(qkv[:, :h], qkv[:, h:h + g], self.q_weight, self.k_weight, self.table, pos, q,
                  k_rows, qkv[:, h + g:], v_rows, slot)
        return q

    def attend(self, q, k, v, seqs, camera, **masks):
        out = torch.empty_like(q)
        tg.attend(q, k, v, seqs, out, tg.AttendBuffers(seqs, q, k), self.d ** -0.5,
                  slope=self.slope, **masks)
        return self.project(out.view(-1, self.width), self.out, self.out_low, camera)


def stitched_cells(rois, frames, canvas):
    """Packs and stitches; returns the cells' pixels [tokens, 3 * 16 * 16] and cells()."""
    n, fh, fw, _ = frames.shape
    plan = tg.plan_pack(rois, canvas, canvas, fw, fh, n, tg.SHELF_FFDH)
    out = torch.empty((plan.n_canvases, 3, canvas, canvas), dtype=torch.float16, device="cuda")
    tg.stitch(frames, tg.DevicePlan(rois, plan), 0, plan.n_canvases, canvas, canvas, W.MEAN, W.STD,
              W.PAD, out)
    at, patch, frame, pos = cells(plan, rois, canvas)
    side = canvas // CELL
    grid = out.view(-1, 3, side, CELL, side, CELL).permute(0, 2, 4, 1, 3, 5)
    c, y, x = (torch.from_numpy(v.astype(np.int64)).cuda() for v in at.T)
    return grid[c, y, x].reshape(len(at), -1).to(DTYPE), plan, patch, frame, pos


def sequences(q_lens, kv_lens):
    """One sequence after the other, queries and keys."""
    q = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    k = np.concatenate([[0], np.cumsum(kv_lens)]).astype(np.int64)
    return tg.Sequences(torch.from_numpy(q).cuda(), torch.from_numpy(k[:-1].copy()).cuda(),
                        torch.from_numpy(np.asarray(kv_lens, dtype=np.int32)).cuda(),
                        int(max(q_lens)), int(max(kv_lens)))


def run(rois, frames, canvas, layer):
    """Tokens of every patch through the layer, then one new token per patch. Returns, by RoI id,
    the layer's results and the new token's."""
    x, plan, patch, frame, pos = stitched_cells(rois, frames, canvas)
    dev = lambda v: torch.from_numpy(v).cuda()
    camera, doc, position = dev(frame), dev(patch), dev(pos)
    tokens, n = len(patch), len(rois)
    canvas_of = plan.place[plan.order[patch], 0]
    per_canvas = np.bincount(canvas_of, minlength=plan.n_canvases)
    per_patch = np.bincount(patch, minlength=n)

    # the cache: each patch's tokens, and a row for the token that comes after them
    first = np.concatenate([[0], np.cumsum(per_patch + 1)])
    slot = dev((first[patch] + np.arange(tokens) - np.concatenate([[0], np.cumsum(per_patch)])[patch]
                ).astype(np.int64))
    cache = [torch.zeros((int(first[-1]), layer.kv_heads, layer.d), dtype=DTYPE, device="cuda")
             for _ in range(2)]
    e = layer.project(x, layer.embed)
    q = layer.queries(e, camera, position, *cache, slot)
    k, v = cache[0][slot], cache[1][slot]  # in the order of the queries
    seqs = sequences(per_canvas, per_canvas)
    y = layer.attend(q, k, v, seqs, camera, q_doc=doc, k_doc=doc, q_pos=position, k_pos=position)

    # one token per patch: a fixed word, at the patch's first cell, against the patch's own rows
    starts = np.concatenate([[0], np.cumsum(per_patch)])[:-1]
    some = np.nonzero(per_patch)[0]
    word = torch.sin(torch.arange(layer.width, device="cuda").float()).to(DTYPE)
    word = word.expand(len(some), -1).contiguous()
    at = dev(starts[some])
    new = layer.queries(word, camera[at].contiguous(), position[at].contiguous(), *cache,
                        dev((first[some] + per_patch[some]).astype(np.int64)))
    single = tg.Sequences(torch.arange(len(some) + 1, dtype=torch.int32, device="cuda"),
                          dev(first[some].astype(np.int64)),
                          dev((per_patch[some] + 1).astype(np.int32)), 1,
                          int(per_patch.max()) + 1)
    z = layer.attend(new, cache[0], cache[1], single, camera[at].contiguous(), causal=True)
    torch.cuda.synchronize()
    by_roi = {int(plan.order[p]): (y[starts[p]:starts[p] + per_patch[p]], z[j])
              for j, p in enumerate(some)}
    return by_roi, tokens, plan.n_canvases


def main(seed: int = 0) -> float:
    cameras, fw, fh, canvas, n = 6, 1280, 720, 512, 60
    rng = np.random.default_rng(seed)
    rois = W.random_rois(rng, n, cameras, fw, fh, 32, 200, 200)
    rois[:, 3:] -= rois[:, 3:] % CELL  # whole cells: shelves then start on cells, too
    frames = torch.from_numpy(W.random_frames_np(cameras, fh, fw, seed)).cuda()
    layer = Layer(cameras, max(fw, fh) // CELL + 1)
    together, tokens, canvases = run(rois, frames, canvas, layer)
    worst = 0.0
    for i in range(0, n, 4):
        alone, _, _ = run(rois[i:i + 1], frames, canvas, layer)
        for a, b in zip(alone[0], together[i]):
            worst = max(worst, float((a.float() - b.float()).norm() / b.float().norm()))
    print(f"{n} patches of {cameras} cameras on {canvases} canvases, {tokens} tokens; every fourth "
          f"against itself alone on a canvas: largest relative difference {worst:.1e}")
    return worst


if __name__ == "__main__":
    main()
