"""Plain implementations of the serving operators, straight from their definitions, and the bounds
on what 32-bit arithmetic and one rounding may differ from them (test infrastructure)."""
from __future__ import annotations

import numpy as np
import torch

from token_reference import E32, TINY, UNIT

RMS, LAYER = 1, 2


def pages(q_begin, kv_len, table, free, n_free, page, n_pages, n_tokens, release=None):
    """The state after a step, sequence by sequence: a dict of lists (free: the pages that nobody
    holds, in order; slot -1 and pos 0 where a token has no row)."""
    seqs, cols = len(kv_len), len(table[0]) if len(table) else 0
    table = [list(row) for row in table]
    stack = list(free[:n_free])
    lens = list(kv_len)
    for s in range(seqs):
        if release is not None and release[s]:
            stack += table[s][:-(-lens[s] // page)]
            lens[s] = 0
    slot, pos, refused, asked, taken = [-1] * n_tokens, [0] * n_tokens, 0, 0, 0
    top = len(stack)
    for s in range(seqs):
        new = q_begin[s + 1] - q_begin[s]
        have = -(-lens[s] // page)
        room = lens[s] + new <= cols * page
        need = -(-(lens[s] + new) // page) - have if room else 0
        asked += need
        if not room or (need > 0 and asked > top):
            refused += 1
            continue
        for i in range(need):
            table[s][have + i] = stack[top - 1 - (asked - need + i)]
        taken = max(taken, asked if need else 0)
        for i in range(new):
            p = lens[s] + i
            at = table[s][p // page]
            if 0 <= at < n_pages:
                slot[q_begin[s] + i], pos[q_begin[s] + i] = at * page + p % page, p
        lens[s] += new
    return dict(table=table, kv_len=lens, free=stack[:top - taken], slot=slot, pos=pos,
                refused=refused)


def attend_pages(q, k, v, table, kv_len, page, scale, cap=0.0, window=0, slope=None, max_kv=None):
    """(out, bound) for q [S, H, d], k and v [rows, Hk, d]. The bound: a score is off by the
    32-bit sum of its products and a few roundings of its parts, a weight by that (twice: it is
    divided by a sum) and by its rounding to the type, the result by its own rounding."""
    u = UNIT[q.dtype]
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.full(q.shape, TINY[q.dtype], dtype=torch.float64)
    group, d = q.shape[1] // k.shape[1], q.shape[2]
    n_pages = k.shape[0] // page
    for s in range(q.shape[0]):
        n = max(int(kv_len[s]), 0)
        end = min(n, table.shape[1] * page, n if max_kv is None else max_kv)
        j = torch.arange(max(0, n - window) if window else 0, max(end, 0))
        at = table[s].long()[j // page]
        j, at = j[(at >= 0) & (at < n_pages)], at[(at >= 0) & (at < n_pages)]
        if len(j) == 0:
            continue
        rows = at * page + j % page
        for h in range(q.shape[1]):
            kr, vr = k[rows, h // group].double(), v[rows, h // group].double()
            qi = q[s, h].double()
            z = scale * (kr @ qi)
            ez = (d + 4) * E32 * abs(scale) * (kr.abs() @ qi.abs())
            if cap > 0:
                z = cap * torch.tanh(z / cap)
                ez = ez + 8 * E32 * cap
            if slope is not None:
                far = (n - 1 - j).double()
                z = z - float(slope[h]) * far
                ez = ez + 4 * E32 * abs(float(slope[h])) * far
            p = torch.softmax(z, 0)
            # keys of next to no weight may be off by more without a part in the result
            ez = ez + 4 * E32 * (z[p > 1e-12].abs().max() + 1)
            e = float(torch.where(p > 1e-12, ez, torch.zeros_like(ez)).max())
            mag = p @ vr.abs()
            out[s, h] = p @ vr
            bound[s, h] += u * out[s, h].abs() + (u + 2 * np.expm1(2 * e)
                                                  + (len(j) + 8) * E32) * mag
    return out, bound


# A sum over a row passes at most 32 additions in a thread, 6 in a wave and 16 of waves, and what is
# summed a few roundings before it.
SUMS = 64


def _normed(u, err, kind, weight, bias, eps):
    """Norm of u, of which `err` is uncertain, and what is uncertain of it."""
    if kind:
        if kind == LAYER:
            mean = u.mean(1, keepdim=True)
            err = err + err.mean(1, keepdim=True) + SUMS * E32 * u.abs().mean(1, keepdim=True)
            err = err + E32 * (u.abs() + mean.abs())
            u = u - mean
        inv = 1 / torch.sqrt((u * u).mean(1, keepdim=True) + eps)
        rms_err = torch.sqrt((err * err).mean(1, keepdim=True))
        u, err = u * inv, err * inv + (u * inv).abs() * (rms_err * inv + (SUMS + 8) * E32)
    if weight is not None:
        u, err = u * weight.double(), err * weight.double().abs()
    if bias is not None:
        u = u + bias.double()
    return u, err + 4 * E32 * u.abs() + (4 * E32 * bias.double().abs() if bias is not None else 0)


def norm(x, y=None, y_norm=0, y_weight=None, y_bias=None, gate=None, gate_row=None, x_scale=1.0,
         y_scale=1.0, kind=RMS, weight=None, bias=None, eps=1e-6):
    """((x_out, bound), (h, bound)) of x, y [tokens, n]."""
    xs, ys = float(np.float32(x_scale)), float(np.float32(y_scale))
    eps = float(np.float32(eps))
    r = xs * x.double()
    err = E32 * r.abs()
    if y is not None:
        b, eb = _normed(y.double(), torch.zeros_like(r), y_norm, y_weight, y_bias, eps)
        has = torch.ones(len(x), dtype=torch.bool)
        if gate is not None:
            row = gate_row.long() if gate_row is not None else torch.zeros(len(x)).long()
            has = (row >= 0) & (row < gate.shape[0])
            g = gate.double()[row.clamp(0, gate.shape[0] - 1)]
            b, eb = b * g, eb * g.abs()
        b, eb = b[has] * ys, eb[has] * abs(ys)
        r[has] += b
        err[has] += eb + 4 * E32 * b.abs()
    h, eh = _normed(r, err, kind, weight, bias, eps)
    unit, tiny = UNIT[x.dtype], TINY[x.dtype]
    # errors of errors: twice the first order
    return (r, unit * r.abs() + 2 * err + tiny), (h, unit * h.abs() + 2 * eh + tiny)


def quantize(x):
    """(integers, scales): the quotient of 16-bit values by a scale of 24 bits, up to 127, lies
    2^-32 of its size from a tie or on it, so that 64 bits decide."""
    top = x.abs().amax(1).float().numpy()
    scale = top / np.float32(127)
    bad = ~np.isfinite(top)
    by = np.where((scale > 0) & ~bad, scale, 1).astype(np.float64)
    q = np.rint(np.where(bad[:, None], 0, x.double().numpy()) / by[:, None])
    q = np.where(scale[:, None] == 0, 0, q)
    assert np.abs(q).max(initial=0) <= 127
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(np.where(bad, np.nan, scale))


def project_i8(x, x_scale, w, w_scale, dtype):
    """(y, bound): the sum, the scales' product and their product rounded once each."""
    y = (x.double() @ w.double().t()) * (x_scale.double()[:, None] * w_scale.double())
    return y, (UNIT[dtype] + 2 * E32) * y.abs() + TINY[dtype]
