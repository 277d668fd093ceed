"""Plain 64-bit implementations of the token operators, straight from their formulas, and the
bounds on what 32-bit sums and one rounding may differ from them (test infrastructure)."""
from __future__ import annotations

import numpy as np
import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half an ulp, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half the smallest subnormal
E32 = 2.0 ** -23


def project(x, w, a, b, scale, adapter):
    """(y, bound on the error of y) for x [T, K], w [N, K]; a None: no adapters. A sum of K
    products in 32 bits is off by at most K E32 times the sum of magnitudes; h is kept as two
    values of the type, off by at most UNIT^2 of its row's largest."""
    u = UNIT[x.dtype]
    xd, wd = x.double(), w.double()
    y = xd @ wd.t()
    err = x.shape[1] * E32 * (xd.abs() @ wd.abs().t())
    for g in range(a.shape[0] if a is not None else 0):
        t = (adapter == g).nonzero()[:, 0]
        if len(t) == 0:
            continue
        s, ad, bd = float(scale[g]), a[g].double(), b[g].double()
        h = xd[t] @ ad.t()
        y[t] += s * (h @ bd.t())
        mag = xd[t].abs() @ ad.abs().t()
        err[t] += abs(s) * (((x.shape[1] + 2 * a.shape[1] + 4) * E32 * mag
                             + 2 * u * u * h.abs().amax(1, keepdim=True)) @ bd.abs().t())
    return y, err + u * y.abs() + TINY[x.dtype] + E32 * y.abs()


def rotate(v, weight, table, pos, eps, interleaved):
    """(result, bound) of norm and rotation for v [T, H, d], table [P, half, 2], pos [T, axes]."""
    d, half, axes = v.shape[2], table.shape[1], pos.shape[1]
    u = v.double()
    u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps)
    if weight is not None:
        u = u * weight.double()
    out, mag = u.clone(), u.abs()
    for i in range(half):
        x, y = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        p = pos[:, i * axes // half].long().clamp(0, table.shape[0] - 1)
        c, s = table[p, i, 0].double()[:, None], table[p, i, 1].double()[:, None]
        out[..., x] = u[..., x] * c - u[..., y] * s
        out[..., y] = u[..., x] * s + u[..., y] * c
        m = u[..., x].abs() + u[..., y].abs()
        mag[..., x] = m
        mag[..., y] = m
    unit = UNIT[v.dtype]
    return out, unit * out.abs() + (d + 16) * E32 * mag + TINY[v.dtype]


def attend(q, k, v, q_begin, kv_begin, kv_len, scale, cap=0.0, causal=False, prefix=None,
           q_doc=None, k_doc=None, q_pos=None, k_pos=None, slope=None):
    """(out, bound) for q [Tq, H, d], k and v [Tk, Hk, d]. The bound: a score is off by the
    32-bit sum of its products and a few roundings of its parts, a weight by that (twice: it is
    divided by a sum) and by its rounding to the type, the result by its own rounding."""
    u = UNIT[q.dtype]
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.full(q.shape, TINY[q.dtype], dtype=torch.float64)
    group, d = q.shape[1] // k.shape[1], q.shape[2]
    for s in range(len(kv_len)):
        q0, q1, k0, n = int(q_begin[s]), int(q_begin[s + 1]), int(kv_begin[s]), int(kv_len[s])
        for i in range(q0, q1):
            place = n - (q1 - q0) + i - q0
            j = torch.arange(n)
            see = torch.ones(n, dtype=torch.bool)
            if causal:
                see &= (j <= place) | (j < (int(prefix[s]) if prefix is not None else 0))
            if q_doc is not None:
                see &= (k_doc[k0:k0 + n] == q_doc[i]) & (q_doc[i] >= 0)
            if not see.any():
                continue
            js = j[see]
            far = (js - place).abs().double()
            if k_pos is not None:
                far = (k_pos[k0 + js].double() - q_pos[i].double()).abs().sum(-1)
            for h in range(q.shape[1]):
                kr, vr = k[k0 + js, h // group].double(), v[k0 + js, h // group].double()
                qi = q[i, h].double()
                z = scale * (kr @ qi)
                ez = (d + 4) * E32 * abs(scale) * (kr.abs() @ qi.abs())
                if cap > 0:
                    z = cap * torch.tanh(z / cap)
                    ez = ez + 8 * E32 * cap
                if slope is not None:
                    z = z - float(slope[h]) * far
                    ez = ez + 4 * E32 * abs(float(slope[h])) * far
                p = torch.exp(z - z.max())
                p = p / p.sum()
                ez = ez + 4 * E32 * (z.abs().max() + 1)
                # keys of next to no weight may be off by more without a part in the result
                e = float((ez + 0 * p).max()) if cap <= 0 and slope is None else float(
                    (torch.where(p > 1e-12, ez, torch.zeros_like(ez))).max())
                mag = p @ vr.abs()
                out[i, h] = p @ vr
                bound[i, h] += u * out[i, h].abs() + (u + 2 * np.expm1(2 * e)
                                                      + (n + 8) * E32) * mag
    return out, bound


def assert_within(got, want, bound, name):
    got = got.double().to(want.device)
    assert got.shape == want.shape
    assert torch.isfinite(got).all(), f"{name}: not finite"
    over = (got - want).abs() - bound
    worst = int(over.argmax()) if over.numel() else 0
    assert over.numel() == 0 or float(over.max()) <= 0, (
        f"{name}: {int((over > 0).sum())} of {over.numel()} values off, worst at "
        f"{tuple(int(x) for x in torch.unravel_index(torch.tensor(worst), over.shape))}: "
        f"{float(got.flatten()[worst])} for {float(want.flatten()[worst])}, "
        f"bound {float(bound.flatten()[worst])}")
