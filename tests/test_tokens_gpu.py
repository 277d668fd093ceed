"""The token operators (tg_project, tg_rotate, tg_attend) against plain 64-bit implementations,
through the C ABI: types, odd sizes, strides, lengths of zero and one, masks that leave a query
nothing, and values that a mask hides."""
import math

import pytest
import torch

from gpu_helpers import say
from paper_2404_09267_amd import tg
import token_reference as R

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype, gain=1.0):
    return (torch.randn(shape, generator=g) * gain).to(dtype)


def dev(t):
    return None if t is None else t.cuda()


# ------------------------------------------------------------------------------- project

def run_project(x, w, ad=None, adapter=None, bufs=None):
    xd, wd = (t if t.is_cuda else t.cuda() for t in (x, w))
    dad = tg.Adapters(*(dev(t) for t in ad)) if ad is not None else None
    bufs = bufs or tg.ProjectBuffers(x.shape[0], x.shape[1], w.shape[0], x.dtype, dad)
    bufs.y.fill_(NAN)
    tg.project(xd, wd, bufs, dad, dev(adapter))
    torch.cuda.synchronize()
    return bufs.y.cpu()


PROJECT = [
    # tokens, k, n, adapters, rank, kind of adapter ids
    (1, 8, 1, 1, 1, "one"), (1, 256, 300, 3, 8, "each"), (7, 64, 130, 7, 5, "each"),
    (8, 1024, 1536, 8, 8, "each"), (16, 72, 17, 2, 16, "runs"), (17, 120, 129, 4, 12, "mixed"),
    (33, 512, 64, 33, 4, "each"), (64, 200, 96, 5, 64, "mixed"), (65, 136, 257, 3, 33, "runs"),
    (128, 64, 128, 2, 16, "none"), (129, 328, 200, 6, 24, "mixed"), (200, 64, 40, 1, 16, "runs"),
    (300, 192, 384, 20, 17, "mixed"), (513, 88, 515, 3, 16, "runs"), (40, 2048, 96, 40, 16, "each"),
]


def adapter_ids(kind, tokens, n, g):
    if kind == "one":
        return torch.zeros(tokens, dtype=torch.int32)
    if kind == "none":
        return torch.full((tokens,), -1, dtype=torch.int32)
    if kind == "each":
        return (torch.arange(tokens) % n).int()
    if kind == "runs":
        return (torch.arange(tokens) * n // tokens).int()
    ids = torch.randint(-1, n + 1, (tokens,), generator=g, dtype=torch.int32)  # n: no adapter too
    return ids


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,k,n,adapters,rank,kind", PROJECT)
def test_project(tokens, k, n, adapters, rank, kind, dtype):
    say("project", tokens, k, n, adapters, rank, kind, dtype)
    g, dt = gen(tokens * 7 + k), DT[dtype]
    x = normal(g, tokens, k, dtype=dt)
    w = normal(g, n, k, dtype=dt, gain=k ** -0.5)
    a = normal(g, adapters, rank, k, dtype=dt, gain=k ** -0.5)
    b = normal(g, adapters, n, rank, dtype=dt)
    scale = 0.5 + torch.rand(adapters, generator=g)
    ids = adapter_ids(kind, tokens, adapters, g)
    want, bound = R.project(x, w, a, b, scale, ids)
    got = run_project(x, w, (a, b, scale), ids)
    R.assert_within(got, want, bound, "project")
    want, bound = R.project(x, w, None, None, None, None)
    R.assert_within(run_project(x, w), want, bound, "project without adapters")


@pytest.mark.parametrize("tokens", [3, 70, 300])
def test_project_strides_and_borders(tokens):
    """Rows inside wider tensors; nothing outside the result is written."""
    say("project strides", tokens)
    g, k, n = gen(5), 88, 133
    wide = normal(g, tokens + 2, k + 24, dtype=torch.bfloat16)
    ww = normal(g, n + 3, k + 8, dtype=torch.bfloat16)
    x, w = wide.cuda()[1:-1, 8:8 + k], ww.cuda()[2:-1, :k]
    out = torch.full((tokens + 2, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    bufs = tg.ProjectBuffers(tokens, k, n, torch.bfloat16)
    bufs.y = out[1:-1, 3:3 + n]
    tg.project(x, w, bufs)
    torch.cuda.synchronize()
    want, bound = R.project(x.cpu(), w.cpu(), None, None, None, None)
    R.assert_within(out[1:-1, 3:3 + n], want, bound, "project")
    out[1:-1, 3:3 + n] = 7.0
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("tokens", [5, 40, 150])
def test_project_keeps_adapters_apart(tokens):
    """Infinities and NaN in one adapter, or in one token, reach no other token."""
    say("project apart", tokens)
    g, k, n, dt = gen(6), 64, 80, torch.float16
    x, w = normal(g, tokens, k, dtype=dt), normal(g, n, k, dtype=dt, gain=0.1)
    a, b = normal(g, 3, 8, k, dtype=dt, gain=0.1), normal(g, 3, n, 8, dtype=dt)
    scale = torch.ones(3)
    ids = (torch.arange(tokens) % 4).int() - 1
    want, bound = R.project(x, w, a, b, scale, ids)
    b[1, :, 2], a[1, 3, :] = NAN, INF
    sick = 2  # a token of adapter 1: neither changes the others
    x[sick, 5] = NAN
    got = run_project(x, w, (a, b, scale), ids)
    rest = (ids != 1)
    assert int(ids[sick]) == 1
    R.assert_within(got[rest], want[rest], bound[rest], "project")
    assert bool(torch.isnan(got[~rest]).any(1).all())


# enough tiles of each size that the projection chooses from: 64 x 64, 128 x 64, 128 x 128 by 8
# waves and by 4, 160 x 128, 192 x 256, 256 x 256; each with k that ends inside a step
TILES = [(300, 1000, 200), (520, 4100, 72), (1777, 2051, 136), (2050, 2100, 72), (4000, 2100, 104),
         (12000, 1000, 136), (8192, 4096, 40), (862, 1317, 504), (2048, 2048, 136)]


@pytest.mark.parametrize("dtype,adapters,rank", [("bf16", 6, 16), ("f16", 40, 12), ("f16", 3, 64),
                                                 ("bf16", 4, 7)])
@pytest.mark.parametrize("tokens,n,k", TILES)
def test_project_tiles(tokens, n, k, dtype, adapters, rank):
    say("project tiles", tokens, n, k, dtype, adapters, rank)
    g, dt = gen(tokens + rank), DT[dtype]
    x, w = normal(g, tokens, k, dtype=dt).cuda(), normal(g, n, k, dtype=dt, gain=k ** -0.5).cuda()
    a = normal(g, adapters, rank, k, dtype=dt, gain=k ** -0.5).cuda()
    b, scale = normal(g, adapters, n, rank, dtype=dt).cuda(), 0.5 + torch.rand(adapters, generator=g)
    runs = torch.randint(-1, adapters, (tokens // 17 + 1,), generator=g, dtype=torch.int32)
    ids = runs.repeat_interleave(17)[:tokens].contiguous()
    want, bound = R.project(x, w, a, b, scale, ids.cuda())
    got = run_project(x, w, (a, b, scale), ids).cuda()
    R.assert_within(got, want, bound, "project")
    # one adapter and two tokens gone bad change no other token
    sick = [tokens // 2, tokens - 1]
    b[1, n // 2:, 0], a[1, 0, 0], x[sick, 0] = NAN, INF, INF
    rest = ids != 1
    rest[sick] = False
    got = run_project(x, w, (a, b, scale), ids)
    R.assert_within(got[rest].cuda(), want[rest.cuda()], bound[rest.cuda()], "project")


def test_project_large_and_small_rows():
    """Rows of h far from 1 in binary16: neither overflow nor lose their small values."""
    say("project range")
    g, k, n, dt = gen(7), 256, 64, torch.float16
    x = normal(g, 6, k, dtype=dt)
    x[1::2] *= 2.0 ** -10
    w = normal(g, n, k, dtype=dt, gain=0.01)
    a = normal(g, 2, 16, k, dtype=dt)
    a[0] *= 2.0 ** 10  # h about 2^14 .. 2^16
    b = normal(g, 2, n, 16, dtype=dt)
    b[0] *= 2.0 ** -8
    scale, ids = torch.tensor([1.5, 0.25]), torch.tensor([0, 0, 1, 1, 0, 1], dtype=torch.int32)
    a[0] *= 4.0
    x[0] *= 2.0
    want, bound = R.project(x, w, a, b, scale, ids)
    R.assert_within(run_project(x, w, (a, b, scale), ids), want, bound, "project")


def test_project_nothing():
    x = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    w = torch.zeros((32, 64), dtype=torch.float16, device="cuda")
    tg.project(x, w, tg.ProjectBuffers(0, 64, 32, torch.float16))
    torch.cuda.synchronize()


# -------------------------------------------------------------------------------- rotate

ROTATE = [
    # tokens, heads, kv heads, d, rot, axes
    (1, 1, 1, 2, 2, 1), (3, 2, 1, 6, 4, 2), (5, 4, 2, 16, 16, 1), (9, 7, 1, 80, 40, 2),
    (20, 16, 4, 64, 64, 1), (17, 3, 3, 128, 64, 2), (33, 8, 2, 128, 128, 2), (4, 2, 1, 96, 32, 2),
    (6, 5, 1, 256, 256, 1), (2, 3, 1, 510, 30, 2), (70, 16, 2, 48, 48, 2), (11, 4, 1, 64, 0, 1),
    (5000, 2, 1, 32, 32, 2), (3, 1, 2, 512, 512, 1),
]


def make_table(g, positions, half):
    angle = torch.rand((positions, half), generator=g, dtype=torch.float64) * 6.3
    return torch.stack([angle.cos(), angle.sin()], -1).float()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,heads,kv,d,rot,axes", ROTATE)
def test_rotate(tokens, heads, kv, d, rot, axes, dtype, interleaved):
    say("rotate", tokens, heads, kv, d, rot, axes, dtype, interleaved)
    g, dt = gen(tokens + d), DT[dtype]
    qkv = normal(g, tokens, heads + 2 * kv, d, dtype=dt, gain=3.0)
    qw, kw = normal(g, d, dtype=dt), normal(g, d, dtype=dt)
    table = make_table(g, 50, rot // 2)
    pos = torch.randint(-2, 53, (tokens, axes), generator=g, dtype=torch.int32)
    dq = qkv.cuda()
    q, k = dq[:, :heads], dq[:, heads:heads + kv]
    q_out = torch.full(q.shape, NAN, dtype=dt, device="cuda")
    k_out = torch.full(k.shape, NAN, dtype=dt, device="cuda")
    tg.rotate(q, k, qw.cuda(), kw.cuda(), table.cuda(), pos.cuda(), q_out, k_out, eps=1e-5,
              interleaved=interleaved)
    # in place, without weights
    tg.rotate(q, k, None, None, table.cuda(), pos.cuda(), q, k, eps=1e-5, interleaved=interleaved)
    torch.cuda.synchronize()
    hq, hk, hv = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    for got, x, w in ((q_out, hq, qw), (k_out, hk, kw), (q, hq, None), (k, hk, None)):
        want, bound = R.rotate(x, w, table, pos, 1e-5, interleaved)
        R.assert_within(got, want, bound, "rotate")
    assert torch.equal(dq[:, heads + kv:].cpu(), hv)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,kv,d", [(1, 1, 64), (20, 4, 64), (37, 2, 128), (13, 3, 34)])
def test_rotate_into_cache(tokens, kv, d, dtype):
    say("rotate cache", tokens, kv, d, dtype)
    g, dt, heads, rows = gen(tokens), DT[dtype], 4, 100
    q, k, v = (normal(g, tokens, h, d, dtype=dt) for h in (heads, kv, kv))
    v[0, 0, 0] = NAN  # values are copied, whatever they are
    table, pos = make_table(g, 30, d // 2), torch.randint(0, 30, (tokens, 1), generator=g,
                                                          dtype=torch.int32)
    slot = torch.randperm(rows, generator=g)[:tokens]
    if tokens > 4:
        slot[1], slot[3] = -1, rows  # written nowhere
    kc, vc = normal(g, rows, kv, d, dtype=dt), normal(g, rows, kv, d, dtype=dt)
    dk, dv = kc.cuda(), vc.cuda()
    q_out = torch.empty((tokens, heads, d), dtype=dt, device="cuda")
    tg.rotate(q.cuda(), k.cuda(), None, None, table.cuda(), pos.cuda(), q_out, dk, v.cuda(), dv,
              slot.cuda())
    torch.cuda.synchronize()
    want, bound = R.rotate(q, None, table, pos, 1e-6, False)
    R.assert_within(q_out, want, bound, "queries")
    want, bound = R.rotate(k, None, table, pos, 1e-6, False)
    dk, dv = dk.cpu(), dv.cpu()
    for t in range(tokens):
        if 0 <= slot[t] < rows:
            R.assert_within(dk[slot[t]], want[t], bound[t], "key")
            assert torch.equal(dv[slot[t]].view(torch.int16), v[t].view(torch.int16))
            kc[slot[t]], vc[slot[t]] = dk[slot[t]], dv[slot[t]]
    assert torch.equal(kc, dk) and torch.equal(vc.view(torch.int16), dv.view(torch.int16))


def test_rotate_zeros_and_huge():
    """A head of zeros stays zero, a head near the type's largest value does not overflow."""
    q = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda")
    q[1] = 60000.0
    table = torch.stack([torch.ones(1, 32), torch.zeros(1, 32)], -1).cuda()
    pos = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    out, k_out = torch.empty_like(q), torch.empty_like(q)
    tg.rotate(q, q.clone(), None, None, table, pos, out, k_out)
    torch.cuda.synchronize()
    assert bool((out[0] == 0).all()) and bool((out[1] == 1).all())


# -------------------------------------------------------------------------------- attend

def run_attend(q, k, v, q_begin, kv_begin, kv_len, scale, out=None, max_q=None, max_kv=None,
               stream=None, **more):
    prefix = more.pop("prefix", None)
    qb = torch.as_tensor(q_begin, dtype=torch.int32)
    kl = torch.as_tensor(kv_len, dtype=torch.int32)
    max_q = int((qb[1:] - qb[:-1]).max()) if max_q is None else max_q
    max_kv = int(kl.max()) if max_kv is None else max_kv
    seqs = tg.Sequences(qb.cuda(), torch.as_tensor(kv_begin, dtype=torch.int64).cuda(), kl.cuda(),
                        max_q, max_kv,
                        prefix=dev(None if prefix is None else
                                   torch.as_tensor(prefix, dtype=torch.int32)))
    q, k, v = (t if t.is_cuda else t.cuda() for t in (q, k, v))
    out = torch.full(q.shape, NAN, dtype=q.dtype, device="cuda") if out is None else out
    bufs = tg.AttendBuffers(seqs, q, k)
    bufs.workspace.fill_(255)
    flags = {n: dev(t) if isinstance(t, torch.Tensor) else t for n, t in more.items()}
    tg.attend(q, k, v, seqs, out, bufs, scale, stream=stream, **flags)
    torch.cuda.synchronize()
    return out


def ragged(lens):
    b = [0]
    for n in lens:
        b.append(b[-1] + n)
    return b


def make(seed, q_lens, kv_lens, heads, kv, d, dtype, gain=2.0, gap=0):
    g, dt = gen(seed), DT[dtype]
    begin = ragged([n + gap for n in kv_lens])
    q = normal(g, sum(q_lens), heads, d, dtype=dt, gain=gain)
    k = normal(g, max(begin[-1], 1), kv, d, dtype=dt)
    v = normal(g, max(begin[-1], 1), kv, d, dtype=dt)
    return g, q, k, v, ragged(q_lens), begin[:-1]


def features(name, g, q_rows, k_rows, heads, seqs, kv_lens):
    f = {}
    if "causal" in name:
        f["causal"] = True
    if "prefix" in name:
        f["prefix"] = [int(torch.randint(-3, n + 5, (1,), generator=g)) for n in kv_lens]
    if "cap" in name:
        f["cap"] = 3000.0 if "bigcap" in name else 5.0
    if "slope" in name:
        f["slope"] = 0.5 ** torch.arange(1, heads + 1).float()
    if "pos" in name:
        f["q_pos"] = torch.randint(-20, 20, (q_rows, 2), generator=g, dtype=torch.int32)
        f["k_pos"] = torch.randint(-20, 20, (k_rows, 2), generator=g, dtype=torch.int32)
    if "docs" in name:
        f["q_doc"] = torch.randint(-1, 4, (q_rows,), generator=g, dtype=torch.int32)
        f["k_doc"] = torch.randint(-1, 4, (k_rows,), generator=g, dtype=torch.int32)
    return f


SHAPES = [
    # query lengths, key lengths, heads, kv heads, d
    ([1], [1], 1, 1, 8), ([1, 1, 1], [1, 0, 33], 4, 2, 64), ([1, 2, 0, 3], [300, 64, 9, 700], 6, 2, 40),
    ([5, 1], [5, 1030], 8, 1, 128), ([17], [129], 12, 4, 72), ([3, 70], [200, 65], 3, 3, 96),
    ([70, 0, 129, 1], [70, 3, 129, 40], 4, 2, 64), ([200], [77], 2, 1, 128),
    ([33, 300], [500, 300], 4, 1, 128), ([65, 1, 64], [65, 0, 190], 2, 2, 32),
]
KINDS = ["plain", "causal", "causal prefix", "docs", "causal docs prefix", "cap", "causal bigcap",
         "causal slope", "slope pos", "cap causal slope pos docs prefix"]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attend(shape, kind, dtype):
    q_lens, kv_lens, heads, kv, d = SHAPES[shape]
    say("attend", SHAPES[shape], kind, dtype)
    g, q, k, v, qb, kb = make(shape, q_lens, kv_lens, heads, kv, d, dtype, gap=shape % 3)
    f = features(kind, g, q.shape[0], k.shape[0], heads, len(q_lens), kv_lens)
    want, bound = R.attend(q, k, v, qb, kb, kv_lens, d ** -0.5, **f)
    got = run_attend(q, k, v, qb, kb, kv_lens, d ** -0.5, **f)
    R.assert_within(got, want, bound, "attend")


@pytest.mark.parametrize("places", ["index", "pos"])
@pytest.mark.parametrize("q_len", [1, 90])
def test_attend_slopes_of_any_sign(q_len, places):
    """Nearer keys less, and heads without a bias, beside the usual ones; far and negative places."""
    say("attend slopes", q_len, places)
    g, q, k, v, qb, kb = make(21, [q_len], [150], 4, 2, 64, "bf16")
    f = dict(slope=torch.tensor([-0.05, 0.0, 0.3, -0.2]))
    if places == "pos":
        f["q_pos"] = torch.randint(-30, 30, (q_len, 2), generator=g, dtype=torch.int32) + 100000
        f["k_pos"] = torch.randint(-30, 30, (150, 2), generator=g, dtype=torch.int32) + 100000
        f["k_pos"][::7] -= 50
        f["k_pos"][3] = -(1 << 31)
    want, bound = R.attend(q, k, v, qb, kb, [150], 0.125, **f)
    R.assert_within(run_attend(q, k, v, qb, kb, [150], 0.125, **f), want, bound, "attend")


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("q_len", [1, 90])
def test_attend_scales(q_len, scale):
    say("attend scale", q_len, scale)
    _, q, k, v, qb, kb = make(3, [q_len], [150], 2, 1, 64, "f16")
    want, bound = R.attend(q, k, v, qb, kb, [150], scale)
    R.assert_within(run_attend(q, k, v, qb, kb, [150], scale), want, bound, "attend")


@pytest.mark.parametrize("what", ["k", "v", "both"])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("q_len,kind", [(1, "docs"), (3, "causal"), (3, "causal docs prefix"),
                                        (150, "causal"), (150, "docs"),
                                        (150, "causal docs prefix cap slope")])
def test_attend_hidden_values(q_len, kind, bad, what):
    """NaN and infinities in keys and values that a query does not see do not reach it."""
    say("attend hidden", q_len, kind, bad, what)
    n = 200
    g, q, k, v, qb, kb = make(4, [q_len], [n], 4, 2, 64, "bf16", gap=70)
    f = features(kind, g, q_len, n + 70, 4, 1, [n])
    if "prefix" in f:
        f["prefix"] = [20]
    if "docs" in kind:
        f["q_doc"][:] = torch.arange(q_len).int() % 3
        f["k_doc"][:] = torch.arange(n + 70).int() % 4  # nobody sees document 3
    want, bound = R.attend(q, k, v, qb, kb, [n], 0.125, **f)
    hidden = [n, n + 40]  # past the last key
    if "docs" in kind:
        hidden += [3, 7, 103, 199]
    for t, c in (k, 1), (v, 2):
        if what == "both" or what == ("k" if c == 1 else "v"):
            t[hidden] = bad
    seen = torch.ones(q_len, dtype=torch.bool)
    if "causal" in kind and "docs" not in kind:
        last = n - q_len + q_len // 2  # seen by the later queries only
        for t, c in (k, 1), (v, 2):
            if what == "both" or what == ("k" if c == 1 else "v"):
                t[last, :, 5] = bad
        seen = torch.arange(q_len) + n - q_len < last
    got = run_attend(q, k, v, qb, kb, [n], 0.125, **f)
    R.assert_within(got[seen.cuda()], want[seen], bound[seen], "attend")


@pytest.mark.parametrize("q_len", [1, 100])
def test_attend_seen_infinities(q_len):
    """An infinite value that is seen comes through where the sum is infinite, and nowhere else."""
    n = 130
    _, q, k, v, qb, kb = make(5, [q_len], [n], 2, 1, 64, "f16", gain=0.5)
    want, bound = R.attend(q, k, v, qb, kb, [n], 0.125)
    v[17, 0, 9] = INF
    got = run_attend(q, k, v, qb, kb, [n], 0.125).cpu()
    assert bool((got[:, :, 9] == INF).all())
    rest = [c for c in range(64) if c != 9]
    R.assert_within(got[:, :, rest], want[:, :, rest], bound[:, :, rest], "attend")


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [90, 300]), ([80, 130], [80, 200])])
def test_attend_strides_and_borders(q_lens, kv_lens):
    """Heads of one row of a fused projection; nothing outside the result is written."""
    say("attend strides", q_lens)
    g, dt, heads, kv, d = gen(8), torch.bfloat16, 4, 2, 40
    rows = sum(kv_lens)
    qkv = normal(g, rows, (heads + 2 * kv) * d + 8, dtype=dt).cuda()
    k = qkv[:, heads * d:(heads + kv) * d].view(rows, kv, d)
    v = qkv[:, (heads + kv) * d:(heads + 2 * kv) * d].view(rows, kv, d)
    q = qkv[:sum(q_lens), :heads * d].view(sum(q_lens), heads, d)
    wide = torch.full((sum(q_lens) + 2, heads, d + 16), 7.0, dtype=dt, device="cuda")
    out = wide[1:-1, :, 8:8 + d]
    qb, kb = ragged(q_lens), ragged(kv_lens)[:-1]
    run_attend(q, k, v, qb, kb, kv_lens, d ** -0.5, out=out, causal=True)
    want, bound = R.attend(q.cpu(), k.cpu(), v.cpu(), qb, kb, kv_lens, d ** -0.5, causal=True)
    R.assert_within(out, want, bound, "attend")
    out.fill_(7.0)
    assert bool((wide == 7.0).all())


def test_attend_heads_first_layout():
    """[heads, rows, d] tensors, as views."""
    _, q, k, v, qb, kb = make(9, [100], [100], 4, 2, 64, "f16")
    qt, kt, vt = (t.transpose(0, 1).contiguous().cuda().transpose(0, 1) for t in (q, k, v))
    want, bound = R.attend(q, k, v, qb, kb, [100], 0.125, causal=True)
    R.assert_within(run_attend(qt, kt, vt, qb, kb, [100], 0.125, causal=True), want, bound, "attend")


@pytest.mark.parametrize("q_len", [1, 4])
@pytest.mark.parametrize("n", [1, 255, 256, 257, 4000, 20011])
def test_attend_long_cache(n, q_len):
    """Key ranges cut over workgroups and joined; ragged, so that some have no key of a part."""
    say("attend long", n, q_len)
    lens = [n, max(q_len, n // 7), max(q_len, 3)]
    _, q, k, v, qb, kb = make(n, [q_len] * 3, lens, 4, 2, 64, "bf16")
    f = dict(causal=True, slope=torch.tensor([0.5, 0.01, 0.002, 0.0]))
    want, bound = R.attend(q, k, v, qb, kb, lens, 0.125, **f)
    got = run_attend(q, k, v, qb, kb, lens, 0.125, **f)
    R.assert_within(got, want, bound, "attend")
    assert torch.equal(got, run_attend(q, k, v, qb, kb, lens, 0.125, **f))


@pytest.mark.parametrize("q_lens,kv_lens", [([40, 7, 33], [5000, 4097, 40]), ([120], [6000])])
@pytest.mark.parametrize("kind", ["causal", "causal prefix cap slope", "docs slope pos"])
def test_attend_tens_of_queries_over_long_keys(q_lens, kv_lens, kind):
    """Several 16-row tiles of queries against keys that are cut into parts."""
    say("attend tens", q_lens, kind)
    g, q, k, v, qb, kb = make(20, q_lens, kv_lens, 4, 2, 64, "bf16")
    f = features(kind, g, q.shape[0], k.shape[0], 4, len(q_lens), kv_lens)
    want, bound = R.attend(q, k, v, qb, kb, kv_lens, 0.125, **f)
    R.assert_within(run_attend(q, k, v, qb, kb, kv_lens, 0.125, **f), want, bound, "attend")


CUT = [
    # few tiles and long keys: the keys of a tile are cut over workgroups
    ([100, 3, 0, 130], [4000, 3, 900, 2500], 4, 2, 64), ([300], [1600], 2, 1, 128),
    ([65, 70], [10, 3000], 2, 2, 72), ([129], [900], 1, 1, 40), ([900], [900], 2, 1, 128),
]


@pytest.mark.parametrize("kind", ["plain", "causal", "causal prefix", "cap", "causal bigcap",
                                  "causal slope", "slope pos", "docs",
                                  "cap causal slope pos prefix"])
@pytest.mark.parametrize("shape", range(len(CUT)))
def test_attend_tiles_whose_keys_are_cut(shape, kind):
    q_lens, kv_lens, heads, kv, d = CUT[shape]
    say("attend cut", CUT[shape], kind)
    dtype = ["f16", "bf16"][shape % 2]
    g, q, k, v, qb, kb = make(shape, q_lens, kv_lens, heads, kv, d, dtype, gap=shape % 3)
    f = features(kind, g, q.shape[0], k.shape[0], heads, len(q_lens), kv_lens)
    want, bound = R.attend(q, k, v, qb, kb, kv_lens, d ** -0.5, **f)
    got = run_attend(q, k, v, qb, kb, kv_lens, d ** -0.5, **f)
    R.assert_within(got, want, bound, "attend")


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("bad", [NAN, float("inf"), -float("inf")])
def test_attend_hidden_values_where_keys_are_cut(bad, what):
    say("attend cut hidden", bad, what)
    n, n_q, seen = 1700, 140, 1610  # the first 50 queries do not see key 1610
    g, q, k, v, qb, kb = make(7, [n_q], [n], 4, 2, 64, "bf16", gap=60)
    want, bound = R.attend(q, k, v, qb, kb, [n], 0.125, causal=True)
    (k if what == "k" else v)[[seen, seen + 1, n, n + 40]] = bad
    got = run_attend(q, k, v, qb, kb, [n], 0.125, causal=True)
    first = n_q - (n - seen)
    R.assert_within(got[:first], want[:first], bound[:first], "attend")


@pytest.mark.parametrize("n_seqs,longest,heads,kv,d", [(33, 1000, 4, 2, 64), (40, 1500, 16, 4, 40),
                                                      (20, 512, 4, 1, 128), (20, 513, 4, 1, 128)])
def test_attend_single_tokens_of_many_caches(n_seqs, longest, heads, kv, d):
    """Keys that are not cut, and parts of more keys than the fewest, with caches of every length."""
    say("attend many caches", n_seqs, longest)
    lens = [longest - (longest * i // n_seqs if i % 3 else i % 2) for i in range(n_seqs)]
    g, q, k, v, qb, kb = make(n_seqs, [1] * n_seqs, lens, heads, kv, d, "bf16", gap=3)
    f = features("cap causal slope", g, q.shape[0], k.shape[0], heads, n_seqs, lens)
    want, bound = R.attend(q, k, v, qb, kb, lens, d ** -0.5, **f)
    R.assert_within(run_attend(q, k, v, qb, kb, lens, d ** -0.5, **f), want, bound, "attend")


def test_attend_many_documents():
    """More key tiles than are looked through at once, few of them seen."""
    n, d = 300000, 64
    g, q, k, v, qb, kb = make(10, [70], [n], 1, 1, d, "f16")
    k_doc = torch.full((n,), 5, dtype=torch.int32)
    k_doc[100:140], k_doc[262140:262150], k_doc[-1] = 1, 1, 2
    q_doc = (torch.arange(70) % 3).int()  # document 0 has no key
    want, bound = R.attend(q, k, v, qb, kb, [n], 0.125, q_doc=q_doc, k_doc=k_doc)
    R.assert_within(run_attend(q, k, v, qb, kb, [n], 0.125, q_doc=q_doc, k_doc=k_doc), want, bound,
                    "attend")


@pytest.mark.parametrize("q_len", [1, 80])
def test_attend_offsets_past_32_bits(q_len):
    """Rows whose offset in the cache, in values, passes 2^32."""
    say("attend far rows", q_len)
    row, n = 2048, 150
    rows = 2 ** 32 // row + 1000
    if torch.cuda.get_device_properties(0).total_memory < 4 * rows * row + (8 << 30):
        pytest.skip("needs 17 GB of device memory")
    cache = torch.empty((rows, row), dtype=torch.float16, device="cuda")
    g, q, k, v, qb, _ = make(11, [q_len], [n], 2, 1, 64, "f16")
    first = rows - n - 20
    cache[first:first + n, :64], cache[first:first + n, 64:128] = k[:, 0].cuda(), v[:, 0].cuda()
    kd, vd = cache[:, :64].unsqueeze(1), cache[:, 64:128].unsqueeze(1)
    want, bound = R.attend(q, k, v, qb, [0], [n], 0.125, causal=True)
    got = run_attend(q, kd, vd, qb, [first], [n], 0.125, causal=True)
    R.assert_within(got, want, bound, "attend")


def test_attend_bounds_and_broken_tables():
    """Lengths beyond the caller's bounds and rows outside the tensors are left out."""
    say("attend bounds")
    _, q, k, v, qb, kb = make(12, [4, 3], [100, 60], 2, 1, 64, "f16")
    for qb, kb, kl, mq, mk in (
            ([0, 4, 7], [0, 100], [100, 1000], 4, 1000),       # runs past the last key row
            ([0, 4, 9999], [0, 100], [100, 60], 100, 100),     # runs past the last query row
            ([-5, 4, 2], [-3, 10 ** 12], [100, 60], 200, 100),  # broken
            ([0, 4, 7], [0, 100], [-1, -7], 4, 100)):
        out = run_attend(q, k, v, qb, kb, kl, 0.125, max_q=mq, max_kv=mk)
        assert out.shape == q.shape
    out = run_attend(q, k, v, [0, 4, 7], [0, 100], [100, 60], 0.125, max_q=4, max_kv=50)
    want, bound = R.attend(q, k, v, [0, 4, 7], [0, 100], [50, 50], 0.125)
    R.assert_within(out, want, bound, "attend")


@pytest.mark.parametrize("q_len", [2, 90])
def test_operators_on_another_stream(q_len):
    """Work enqueued on the caller's stream, after what that stream already holds."""
    say("streams", q_len)
    _, q, k, v, qb, kb = make(13, [q_len], [300], 4, 2, 64, "bf16")
    want, bound = R.attend(q, k, v, qb, kb, [300], 0.125)
    side = torch.cuda.Stream()
    kd = torch.full(k.shape, NAN, dtype=k.dtype, device="cuda")
    src = k.cuda()
    seqs = tg.Sequences(*(torch.as_tensor(t, dtype=d).cuda() for t, d in (
        (qb, torch.int32), (kb, torch.int64), ([300], torch.int32))), q_len, 300)
    dq, dv = q.cuda(), v.cuda()
    out, bufs = torch.empty_like(dq), tg.AttendBuffers(seqs, dq, kd)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1000000)
        kd.copy_(src)
        tg.attend(dq, kd, dv, seqs, out, bufs, 0.125)
    side.synchronize()
    R.assert_within(out, want, bound, "attend")


def test_operators_in_a_graph():
    """The three calls captured in a graph and replayed on new values, each replay checked."""
    say("graph")
    g, dt, tokens, heads, kv, d, k = gen(14), torch.bfloat16, 6, 4, 2, 64, 128
    width, rows = (heads + 2 * kv) * d, 64
    w = normal(g, width, k, dtype=dt, gain=k ** -0.5).cuda()
    ad = tg.Adapters(*(dev(t) for t in (normal(g, 3, 8, k, dtype=dt, gain=k ** -0.5),
                                        normal(g, 3, width, 8, dtype=dt), torch.ones(3))))
    x = torch.empty((tokens, k), dtype=dt, device="cuda")
    ids = torch.arange(tokens, dtype=torch.int32, device="cuda") % 4
    pb = tg.ProjectBuffers(tokens, k, width, dt, ad)
    table = make_table(g, 32, d // 2).cuda()
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")[:, None].contiguous()
    kc, vc = (torch.zeros((rows, kv, d), dtype=dt, device="cuda") for _ in range(2))
    slot = torch.arange(tokens, dtype=torch.int64, device="cuda") * 10 + 9
    seqs = tg.Sequences(torch.arange(tokens + 1, dtype=torch.int32, device="cuda"),
                        torch.arange(tokens, dtype=torch.int64, device="cuda") * 10,
                        torch.full((tokens,), 10, dtype=torch.int32, device="cuda"), 1, 10)
    qkv = pb.y.view(tokens, heads + 2 * kv, d)
    q_out, out = (torch.empty((tokens, heads, d), dtype=dt, device="cuda") for _ in range(2))
    ab = tg.AttendBuffers(seqs, q_out, kc)

    def step():
        tg.project(x, w, pb, ad, ids)
        tg.rotate(qkv[:, :heads], qkv[:, heads:heads + kv], None, None, table, pos, q_out, kc,
                  qkv[:, heads + kv:], vc, slot)
        tg.attend(q_out, kc, vc, seqs, out, ab, d ** -0.5, causal=True)

    x.copy_(normal(g, tokens, k, dtype=dt))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        x.copy_(normal(g, tokens, k, dtype=dt))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and bool(torch.isfinite(out).all())
