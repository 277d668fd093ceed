"""The token operators where sizes, masks and values are at their ends, against plain 64-bit
implementations: what the tests of single operators do not reach."""
import math

import pytest
import torch

from gpu_helpers import say
from paper_2404_09267_amd import tg
from test_tokens_gpu import DT, NAN, dev, features, gen, make, make_table, \
    normal, run_attend, run_project
import token_reference as R

pytestmark = pytest.mark.gpu


def room(gib):
    """Skips where the card has less memory than this."""
    if torch.cuda.get_device_properties(0).total_memory < gib << 30:
        pytest.skip(f"needs {gib} GB of device memory")


# ------------------------------------------------------------------------------- project

@pytest.mark.parametrize("rank", [8, 16, 20])
def test_project_adapters_past_one_buffer(rank):
    """2 GiB of b and more, which one buffer does not reach, and several adapters in a tile."""
    say("project far adapters", rank)
    room(40)
    tokens, k, n, dt = 300, 64, 32768, torch.bfloat16
    adapters = 2 ** 31 // (n * rank * 2) + 3
    g = gen(rank)
    x, w = normal(g, tokens, k, dtype=dt).cuda(), normal(g, n, k, dtype=dt, gain=0.125).cuda()
    a = normal(g, adapters, rank, k, dtype=dt, gain=0.125).cuda()
    b = torch.empty((adapters, n, rank), dtype=dt, device="cuda").normal_()
    ids = (torch.arange(tokens) // 9 * 131 % adapters).int()
    ids[:5], ids[-3:] = adapters - 1, 0
    ids[40:60] = -1
    scale = 0.5 + torch.rand(adapters, generator=g)
    want, bound = R.project(x, w, a, b, scale, ids.cuda())
    bufs = tg.ProjectBuffers(tokens, k, n, dt, tg.Adapters(a, b, scale.cuda()))
    bufs.y.fill_(NAN)
    tg.project(x, w, bufs, tg.Adapters(a, b, scale.cuda()), ids.cuda())
    torch.cuda.synchronize()
    R.assert_within(bufs.y, want, bound, "project")


@pytest.mark.parametrize("tokens", [200, 300, 2100])
def test_project_small_rows_of_h(tokens):
    """Rows of h far below binary16's smallest normal number, and b large: as exact as others."""
    say("project small h", tokens)
    g, k, n, dt = gen(31), 64, 160, torch.float16
    x, w = normal(g, tokens, k, dtype=dt), normal(g, n, k, dtype=dt) * 0
    a = normal(g, 3, 8, k, dtype=dt, gain=2.0 ** -6)
    x[::3] *= 2.0 ** -9
    b = normal(g, 3, n, 8, dtype=dt, gain=1024.0)
    scale = torch.tensor([2.0 ** -18, 1.0, 2.0 ** 9])
    a[2] *= 2.0 ** 9  # and rows of h past its largest, with a b to match
    b[2] *= 2.0 ** -20
    ids = (torch.arange(tokens) // 7 % 4).int() - 1
    w[::5] = normal(g, len(range(0, n, 5)), k, dtype=dt, gain=0.1)
    want, bound = R.project(x, w, a, b, scale, ids)
    R.assert_within(run_project(x, w, (a, b, scale), ids), want, bound, "project")


@pytest.mark.parametrize("case", ["odd rank, 70 MB of b", "b between boundaries"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_project_gathered_adapters(case, dtype):
    """Rows of b that loads to LDS cannot take and that are not laid out anew."""
    say("project gathered", case, dtype)
    room(8)
    g, dt = gen(32), DT[dtype]
    tokens, k, n, adapters, rank = ((300, 72, 28001, 40, 17) if "odd" in case else
                                    (333, 136, 515, 5, 12))
    x, w = normal(g, tokens, k, dtype=dt).cuda(), normal(g, n, k, dtype=dt, gain=k ** -0.5).cuda()
    a = normal(g, adapters, rank, k, dtype=dt, gain=k ** -0.5).cuda()
    b = torch.empty(1 + adapters * n * rank, dtype=dt, device="cuda").normal_()
    b = b[0 if "odd" in case else 1:][:adapters * n * rank].view(adapters, n, rank)
    scale = 0.5 + torch.rand(adapters, generator=g)
    ids = torch.randint(-1, adapters + 1, (tokens,), generator=g, dtype=torch.int32)
    want, bound = R.project(x, w, a, b, scale, ids.cuda())
    got = run_project(x, w, (a, b, scale), ids)
    R.assert_within(got.cuda(), want, bound, "project")


# -------------------------------------------------------------------------------- rotate

def test_rotate_more_heads_than_a_row_of_workgroups():
    """So many heads that their threads pass 2^32."""
    say("rotate many")
    room(24)
    tokens, d = 2 ** 26 + 5, 2
    q = torch.empty((tokens, 1, d), dtype=torch.bfloat16, device="cuda").normal_()
    pos = (torch.arange(tokens, device="cuda") % 3).int()[:, None].contiguous()
    table = torch.tensor([[[1.0, 0.0]], [[0.0, 1.0]], [[0.6, -0.8]]]).cuda()
    out = torch.full_like(q, NAN)
    none = q[:, :0]
    tg.rotate(q, none, None, None, table, pos, out, none)
    torch.cuda.synchronize()
    for first in (0, tokens // 2, tokens - 10000):
        t = slice(first, first + 10000)
        want, bound = R.rotate(q[t].cpu(), None, table.cpu(), pos[t].cpu(), 1e-6, False)
        R.assert_within(out[t].cpu(), want, bound, "rotate")
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("tokens,heads,d,rot", [(5, 3, 64, 64), (7, 2, 34, 20), (3, 1, 512, 512),
                                                (40, 8, 16, 0)])
def test_rotate_values_whose_squares_overflow(tokens, heads, d, rot):
    """bfloat16 reaches 3 * 10^38, squares of 2 * 10^19 pass it: the norm is that of the values."""
    say("rotate huge", tokens, heads, d, rot)
    g, dt = gen(45), torch.bfloat16
    q, k = normal(g, tokens, heads, d, dtype=dt), normal(g, tokens, 1, d, dtype=dt)
    q[1::2] *= 2.0 ** 70
    q[2] *= 2.0 ** 50
    k[::2] *= 2.0 ** 120
    k[1, 0, :5] = 2.0 ** 100  # and next to ordinary ones
    w = normal(g, d, dtype=dt)
    pos = torch.randint(0, 9, (tokens, 1), generator=g, dtype=torch.int32)
    table = make_table(g, 9, rot // 2)
    out, k_out = (torch.full(t.shape, NAN, dtype=dt, device="cuda") for t in (q, k))
    tg.rotate(q.cuda(), k.cuda(), w.cuda(), None, table.cuda(), pos.cuda(), out, k_out)
    torch.cuda.synchronize()
    for got, x, by in ((out, q, w), (k_out, k, None)):
        want, bound = R.rotate(x, by, table, pos, 1e-6, False)
        R.assert_within(got, want, bound, "rotate")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,rot", [(64, 0), (64, 32), (64, 36), (34, 0), (34, 10)])
def test_rotate_infinite_and_nan_heads(d, rot, dtype, interleaved):
    """An infinity leaves the rest of its head 0, NaN takes its head, and neither another one; a
    value that does not turn does not see those beside it."""
    say("rotate inf nan", d, rot, dtype, interleaved)
    g, dt = gen(46), DT[dtype]
    q, k = normal(g, 4, 2, d, dtype=dt), normal(g, 4, 1, d, dtype=dt)
    q[0, 0, d - 1], k[0, 0, 1] = math.inf, NAN  # the last value turns in no case
    table, pos = make_table(g, 3, rot // 2), torch.zeros((4, 1), dtype=torch.int32)
    out, k_out = (torch.full(t.shape, NAN, dtype=dt, device="cuda") for t in (q, k))
    tg.rotate(q.cuda(), k.cuda(), None, None, table.cuda(), pos.cuda(), out, k_out,
              interleaved=interleaved)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[0, 0, d - 1])) and bool((out[0, 0, :d - 1] == 0).all())
    assert bool(torch.isnan(k_out[0, 0]).all())
    for got, x in ((out[1:], q[1:]), (out[:1, 1:], q[:1, 1:]), (k_out[1:], k[1:])):
        want, bound = R.rotate(x, None, table, pos[:len(x)], 1e-6, interleaved)
        R.assert_within(got, want, bound, "rotate")


# -------------------------------------------------------------------------------- attend

@pytest.mark.parametrize("n_seqs,heads,kv,queries", [(2 ** 20 + 3, 32, 32, 1),
                                                     (2 ** 18 + 1, 64, 1, 2)])
def test_attend_more_rows_than_a_row_of_workgroups(n_seqs, heads, kv, queries):
    """So many sequences that the threads of both forms pass 2^32; each sees one key, or none."""
    say("attend many", n_seqs, heads, kv, queries)
    room(24)
    d, dt, keys = 8, torch.float16, 1000
    g = gen(33)
    k, v = normal(g, keys, kv, d, dtype=dt).cuda(), normal(g, keys, kv, d, dtype=dt).cuda()
    q = torch.empty((n_seqs * queries, heads, d), dtype=dt, device="cuda").normal_()
    at = torch.arange(n_seqs, device="cuda")
    seqs = tg.Sequences((torch.arange(n_seqs + 1, device="cuda") * queries).int(), at % keys,
                        (at % 7 > 0).int(), queries, 1)
    out = torch.full_like(q, NAN)
    tg.attend(q, k, v, seqs, out, tg.AttendBuffers(seqs, q, k), 0.5)
    torch.cuda.synchronize()
    want = v[at % keys].repeat_interleave(heads // kv, 1) * (at % 7 > 0)[:, None, None]
    out = out.view(n_seqs, queries, heads, d)
    for i in range(queries):
        assert bool((out[:, i] == want).all())


CUT_KEYS = [(300, 1600, 2, 1, 128, "bf16"), (140, 4000, 4, 2, 64, "f16")]


def finite_rest(got, want, bound, lost):
    """The rows `lost` are NaN throughout, all others within their bounds."""
    got = got.cpu()
    assert bool(torch.isnan(got[lost]).all())
    R.assert_within(got[~lost], want[~lost], bound[~lost], "attend")


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n_q,n,heads,kv,d,dtype", CUT_KEYS + [(1, 3000, 4, 2, 64, "bf16"),
                                                              (100, 300, 2, 1, 64, "f16"),
                                                              (1, 200, 4, 1, 40, "f16")])
def test_attend_seen_nan(n_q, n, heads, kv, d, dtype, causal):
    """A NaN in a query, or in keys it sees, is its result, however the keys are cut."""
    say("attend seen nan", n_q, n, dtype, causal)
    _, q, k, v, qb, kb = make(34, [n_q], [n], heads, kv, d, dtype)
    f = dict(causal=causal)
    want, bound = R.attend(q, k, v, qb, kb, [n], d ** -0.5, **f)
    place = torch.arange(n_q) + n - n_q
    bad = q.clone()
    bad[n_q // 2, :, 3] = NAN
    got = run_attend(bad, k, v, qb, kb, [n], d ** -0.5, **f)
    finite_rest(got, want, bound, torch.arange(n_q) == n_q // 2)
    # whole parts of the keys, and the first key of a tile as all that some queries see of it
    for keys in (slice(0, n // 2), slice(n // 2, n), slice(n - n_q // 2 & ~63, None)):
        bad = k.clone()
        bad[keys] = NAN
        first = torch.arange(n)[keys][0]
        lost = place >= first if causal else torch.ones(n_q, dtype=torch.bool)
        finite_rest(run_attend(q, bad, v, qb, kb, [n], d ** -0.5, **f), want, bound, lost)
    for j in range(n - n_q & ~63, n, 64):
        bad = k.clone()
        bad[max(j, 0)] = NAN
        lost = place >= j if causal else torch.ones(n_q, dtype=torch.bool)
        finite_rest(run_attend(q, bad, v, qb, kb, [n], d ** -0.5, **f), want, bound, lost)


@pytest.mark.parametrize("q_len", [3, 100])
def test_attend_documents_of_every_sign(q_len):
    """Documents below 0 see nothing, the lowest number among them; the highest sees its own."""
    say("attend documents", q_len)
    g, q, k, v, qb, kb = make(35, [q_len], [170], 4, 2, 64, "bf16")
    names = torch.tensor([-(1 << 31), -1, 0, (1 << 31) - 1, -(1 << 31) + 1], dtype=torch.int32)
    f = dict(q_doc=names[torch.arange(q_len) % 5], k_doc=names[torch.arange(170) * 7 // 3 % 5])
    want, bound = R.attend(q, k, v, qb, kb, [170], 0.125, **f)
    assert bool((want[0] == 0).all())
    R.assert_within(run_attend(q, k, v, qb, kb, [170], 0.125, **f), want, bound, "attend")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_len,n", [(1, 500), (70, 500), (1, 100003), (70, 100003)])
def test_attend_many_small_weights(q_len, n, dtype):
    """A key of weight 1 in every 64, whose value is 0, and many of weight e^-17.5, 0.84 of half
    binary16's smallest number, whose values add up. A weight is off by its rounding to the type;
    in binary16, with the largest weight at 2^7, by no less than 2^-32 of it."""
    say("attend small weights", q_len, n, dtype)
    _, q, k, v, qb, kb = make(36, [q_len], [n], 1, 1, 8, dtype)
    q[:], k[:] = 0, 0
    q[:, :, 0], k[:, :, 0] = 1.0, -17.5
    v = (v.abs() * 60).clamp(1.0, 200.0)
    k[::64], v[::64] = 0, 0
    want, _ = R.attend(q, k, v, qb, kb, [n], 1.0)
    small, u = math.exp(-17.5), R.UNIT[q.dtype]
    each = max(u * small, 2.0 ** -32) if dtype == "f16" else u * small
    # 64 keys' errors against a sum of 1, those of the exponent (26 in binary32) and of the sum
    bound = (u * want + R.TINY[q.dtype] + 64 * float(v.max()) * (each + 40 * R.E32 * small)
             + 2 * u * want + (n + 8) * R.E32 * want)
    R.assert_within(run_attend(q, k, v, qb, kb, [n], 1.0), want, bound, "attend")


@pytest.mark.parametrize("q_len", [1, 90, 300])
def test_attend_far_positions_are_exact(q_len):
    """Queries of one batch at places 2^30 apart: the distance to a key beside each is whole. Keys
    of the other places are too far to weigh anything."""
    say("attend far positions", q_len)
    n, heads = 400, 2
    g, q, k, v, qb, kb = make(37, [q_len], [n], heads, 1, 64, "bf16", gain=0.5)
    bases = torch.tensor([0, 1 << 30, -(1 << 30) - 77, (1 << 31) - 100, 1 << 25, -(1 << 31) + 9])
    qc, kc = torch.arange(q_len) % 6, torch.randint(0, 6, (n,), generator=g)
    if q_len == 1:
        qc[:] = 1
    f = dict(slope=torch.tensor([0.25, 1.0]))
    place = lambda c, rows: (bases[c][:, None] + torch.randint(0, 5, (rows, 2), generator=g)).int()
    f["q_pos"], f["k_pos"] = place(qc, q_len), place(kc, n)
    want, bound = R.attend(q, k, v, qb, kb, [n], 0.125, q_doc=qc.int(), k_doc=kc.int(), **f)
    got = run_attend(q, k, v, qb, kb, [n], 0.125, **f)
    R.assert_within(got, want, bound, "attend")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_len,n", [(1, 150), (1, 3000), (90, 150), (140, 3000)])
def test_attend_scores_of_any_size(q_len, n, dtype):
    """Scores so large that their rounding alone is many units of the exponent: the largest has
    all of the weight. They are whole multiples of the scale, so it is the same in any order."""
    say("attend large scores", q_len, n, dtype)
    g, q, k, v, qb, kb = make(38, [q_len], [n], 4, 2, 64, dtype)
    q[:], k[:] = 0, 0
    q[..., 0], q[..., 5] = 2.0, 1.0
    top = torch.randint(0, n, (2,), generator=g)
    k[..., 0] = -torch.randint(1, 9, (n, 2), generator=g).to(k.dtype)
    k[..., 5] = torch.randint(0, 2, (n, 2), generator=g).to(k.dtype)
    for h in range(2):
        k[top[h], h, 0], k[top[h], h, 5] = 50.0, 1.0
    want = torch.stack([v[top[h // 2], h // 2] for h in range(4)]).expand(q.shape)
    for scale in (1e6, 1.1e7, 3e8, 7.7e8, 1e9, 3.3e9, 1.7e10, 6e12, 1e20):
        got = run_attend(q, k, v, qb, kb, [n], scale).cpu()
        assert bool((got == want).all()), scale
    # the same by a bias that favours distance
    f = dict(slope=-torch.tensor([0.7, 1.25, 2.5, 5.0]),
             q_pos=torch.randint(0, 30, (q_len, 2), generator=g, dtype=torch.int32),
             k_pos=torch.randint(0, 30, (n, 2), generator=g, dtype=torch.int32))
    for far in (2 ** 31 - 1, 2 ** 31 - 12345, 2 ** 28 + 99):
        f["k_pos"][top] = -far
        both = v[top].float().mean(0) if top[0] != top[1] else v[top[0]].float()
        got = run_attend(q, k * 0, v, qb, kb, [n], 0.125, **f).cpu()
        bound = 4 * R.UNIT[q.dtype] * v[top].double().abs().amax(0)
        for h in range(4):
            R.assert_within(got[:, h], both[h // 2].double().expand(q_len, -1), bound[h // 2],
                            "attend")


@pytest.mark.parametrize("cap", [1e-40, 1e-30, 1e-6, 3e38])
@pytest.mark.parametrize("q_len,more", [(1, {}), (90, {}), (90, {"slope": True}),
                                        (1, {"slope": True})])
def test_attend_caps_of_every_size(q_len, more, cap):
    """Caps whose quotient with the scale leaves binary32, scores of 0 among them."""
    say("attend caps", q_len, cap)
    _, q, k, v, qb, kb = make(39, [q_len], [150], 2, 1, 64, "bf16")
    k[::9], q[::5] = 0, 0
    f = dict(cap=cap)
    if more:
        f["slope"] = torch.tensor([0.5, 0.01])
    # the bound has a share of the cap in it: tanh of next to nothing is straight
    straight = {n: t for n, t in f.items() if n != "cap"}
    want, bound = R.attend(q, k, v, qb, kb, [150], 0.125, **(straight if cap > 1e30 else f))
    R.assert_within(run_attend(q, k, v, qb, kb, [150], 0.125, **f), want, bound, "attend")


@pytest.mark.parametrize("q_len,n", [(0, 40), (3, 0), (80, 0)])
def test_attend_nothing_to_see_with_documents(q_len, n):
    """No queries, or no keys at all, beside documents and positions."""
    say("attend nothing", q_len, n)
    dt = torch.float16
    q = torch.ones((q_len, 2, 64), dtype=dt, device="cuda")
    k = torch.ones((n, 1, 64), dtype=dt, device="cuda")
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    f = dict(q_doc=ints(q_len), k_doc=ints(n), q_pos=ints(q_len, 2), k_pos=ints(n, 2),
             slope=torch.ones(2))
    out = run_attend(q, k, k, [0, q_len], [0], [n], 0.125, **f)
    assert out.shape == q.shape and bool((out == 0).all())


def test_one_row_or_head_of_any_stride():
    """A dimension of one element has a stride that nothing is reached by."""
    say("one row")
    g, dt, d, rows = gen(40), torch.bfloat16, 64, 90
    odd = lambda t, s: t.as_strided(t.shape, s)
    q, k, v = (normal(g, n, 1, d, dtype=dt).cuda() for n in (1, rows, rows))
    want, bound = R.attend(q.cpu(), k.cpu(), v.cpu(), [0, 1], [0], [rows], 0.125)
    out = odd(torch.empty_like(q), (1 << 40, 3, 1))
    run_attend(odd(q, (12345, 1 << 33, 1)), odd(k, (d, 7, 1)), v, [0, 1], [0], [rows], 0.125,
               out=out)
    R.assert_within(out, want, bound, "attend")
    one = odd(k[:1], (1 << 30, 1, 1))
    run_attend(q, one, one, [0, 1], [0], [1], 0.125, out=out)
    assert bool((out == one).all())


def clamped(q, k, v, qb, kb, kl, max_q, max_kv, scale):
    """What the operator documents for tables that leave the tensors or the bounds: results, their
    bounds, and which rows are written."""
    n_q, n_k = q.shape[0], k.shape[0]
    want = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.full(q.shape, R.TINY[q.dtype], dtype=torch.float64)
    written = torch.zeros(n_q, dtype=torch.bool)
    for s in range(len(kb)):
        a = min(max(qb[s], 0), n_q)
        b = min(max(qb[s + 1], a), n_q)
        k0 = kb[s] if 0 <= kb[s] < n_k else 0
        n = min(max(kl[s], 0), n_k - k0, max_kv) if 0 <= kb[s] < n_k else 0
        b = min(b, a + max_q)
        written[a:b] = True
        if n > 0 and b > a:
            want[a:b], bound[a:b] = R.attend(q[a:b], k[k0:k0 + n], v[k0:k0 + n], [0, b - a], [0],
                                             [n], scale)
    return want, bound, written


BROKEN = [  # queries and keys there are; q_begin, kv_begin, kv_len, max_q, max_kv
    (7, 160, [0, 4, 7], [0, 100], [100, 1000], 4, 1000),
    (7, 160, [0, 4, 9999], [0, 100], [100, 60], 30, 100),
    (7, 160, [-5, 4, 2], [-3, 10 ** 12], [100, 60], 30, 100),
    (7, 160, [0, 4, 7], [0, 100], [-1, -7], 4, 100),
    (7, 160, [0, 4, 7], [0, 159], [100, 60], 2, 50),
    (300, 500, [0, 130, 9999], [0, 400], [400, 1000], 400, 1000),
    (300, 500, [-70, 100, 290], [-3, 499], [100, 60], 250, 100),
    (300, 500, [10, 200, 250], [0, 10 ** 12], [500, 9], 90, 130),
    (300, 4000, [0, 150, 9999], [0, 2000], [4000, 4000], 300, 4000),
    (300, 4000, [5, 150, 300], [100, 3990], [2500, 10 ** 9], 129, 2400),
    (40, 3000, [0, 20, 9999], [500, 0], [9999, 3000], 25, 2900),
]


@pytest.mark.parametrize("case", range(len(BROKEN)))
def test_attend_broken_tables_reach_nothing_else(case):
    """Lengths and rows outside the tensors or the bounds count as documented; the rows of no
    sequence, and what lies around the result, stay as they were."""
    n_q, n_k, qb, kb, kl, max_q, max_kv = BROKEN[case]
    say("attend broken", BROKEN[case])
    g, dt, heads, d = gen(41), torch.float16, 2, 64
    q, k, v = (normal(g, n, h, d, dtype=dt) for n, h in ((n_q, heads), (n_k, 1), (n_k, 1)))
    wide = torch.full((n_q + 64, heads, d + 16), 7.0, dtype=dt, device="cuda")
    out = wide[32:-32, :, 8:8 + d]
    run_attend(q, k, v, qb, kb, kl, 0.125, out=out, max_q=max_q, max_kv=max_kv)
    want, bound, written = clamped(q, k, v, qb, kb, kl, max_q, max_kv, 0.125)
    R.assert_within(out.cpu()[written], want[written], bound[written], "attend")
    out[written.cuda()] = 7.0
    assert bool((wide == 7.0).all())


@pytest.mark.parametrize("kind", ["causal", "causal docs prefix", "slope pos"])
@pytest.mark.parametrize("n_seqs,q_most,kv_most,heads,kv", [
    (150, 1, 1500, 4, 2), (250, 2, 2000, 2, 2), (300, 3, 90, 4, 1), (100, 80, 60, 2, 1),
    (70, 40, 200, 4, 2), (65, 1, 3000, 8, 1)])
def test_attend_more_sequences_than_lanes(n_seqs, q_most, kv_most, heads, kv, kind):
    """More than 64 sequences, up to and past those whose keys are cut."""
    say("attend many sequences", n_seqs, q_most, kv_most, kind)
    g = gen(n_seqs)
    q_lens = [int(torch.randint(0, q_most + 1, (1,), generator=g)) for _ in range(n_seqs)]
    kv_lens = [int(torch.randint(0, kv_most + 1, (1,), generator=g)) for _ in range(n_seqs)]
    q_lens[3], kv_lens[5] = q_most, kv_most
    g, q, k, v, qb, kb = make(n_seqs, q_lens, kv_lens, heads, kv, 32, "bf16", gap=2)
    f = features(kind, g, q.shape[0], k.shape[0], heads, n_seqs, kv_lens)
    want, bound = R.attend(q, k, v, qb, kb, kv_lens, 0.2, **f)
    R.assert_within(run_attend(q, k, v, qb, kb, kv_lens, 0.2, **f), want, bound, "attend")


@pytest.mark.parametrize("lens,heads,kv,d", [([20011, 2858, 4], 4, 2, 64), ([9000], 8, 1, 128),
                                             ([1500 - 37 * i for i in range(40)], 4, 2, 40)])
@pytest.mark.parametrize("q_len", [1, 4])
def test_attend_long_caches_in_binary16(lens, heads, kv, d, q_len):
    say("attend long f16", len(lens), q_len)
    g, q, k, v, qb, kb = make(42, [q_len] * len(lens), lens, heads, kv, d, "f16")
    f = features("cap causal slope", g, q.shape[0], k.shape[0], heads, len(lens), lens)
    want, bound = R.attend(q, k, v, qb, kb, lens, d ** -0.5, **f)
    R.assert_within(run_attend(q, k, v, qb, kb, lens, d ** -0.5, **f), want, bound, "attend")


def test_operators_in_a_graph_are_right():
    """Each call's results in every replay of a captured graph against the formulas, with other
    work and synchronisations between the replays."""
    say("graph and formulas")
    g, dt, tokens, heads, kv, d, k = gen(43), torch.float16, 6, 4, 2, 64, 128
    width, rows, keys = (heads + 2 * kv) * d, 6 * 700, 700
    w = normal(g, width, k, dtype=dt, gain=k ** -0.5)
    ad = (normal(g, 3, 8, k, dtype=dt, gain=k ** -0.5), normal(g, 3, width, 8, dtype=dt),
          torch.ones(3))
    dad, dw = tg.Adapters(*(dev(t) for t in ad)), w.cuda()
    x = torch.empty((tokens, k), dtype=dt, device="cuda")
    ids = torch.arange(tokens, dtype=torch.int32) % 4
    pb = tg.ProjectBuffers(tokens, k, width, dt, dad)
    table = make_table(g, 32, d // 2)
    pos = torch.arange(tokens, dtype=torch.int32)[:, None].contiguous()
    kc, vc = (normal(g, rows, kv, d, dtype=dt).cuda() for _ in range(2))
    slot = torch.arange(tokens) * keys + keys - 1
    seqs = tg.Sequences(torch.arange(tokens + 1, dtype=torch.int32, device="cuda"),
                        torch.arange(tokens, dtype=torch.int64, device="cuda") * keys,
                        torch.full((tokens,), keys, dtype=torch.int32, device="cuda"), 1, keys)
    qkv = pb.y.view(tokens, heads + 2 * kv, d)
    q_out, out = (torch.empty((tokens, heads, d), dtype=dt, device="cuda") for _ in range(2))
    ab, dids, dtable, dpos, dslot = (tg.AttendBuffers(seqs, q_out, kc), ids.cuda(), table.cuda(),
                                     pos.cuda(), slot.cuda())

    def step():
        tg.project(x, dw, pb, dad, dids)
        tg.rotate(qkv[:, :heads], qkv[:, heads:heads + kv], None, None, dtable, dpos, q_out, kc,
                  qkv[:, heads + kv:], vc, dslot)
        tg.attend(q_out, kc, vc, seqs, out, ab, d ** -0.5, causal=True)

    x.zero_()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        hx = normal(g, tokens, k, dtype=dt)
        x.copy_(hx)
        scratch = (b.workspace.view(torch.float32) for b in (pb, ab))
        for t in (pb.y, q_out, out, *scratch):
            t.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        want, bound = R.project(hx, w, *ad, ids)
        R.assert_within(pb.y, want, bound, "project")
        h = qkv.cpu()
        want, bound = R.rotate(h[:, :heads], None, table, pos, 1e-6, False)
        R.assert_within(q_out, want, bound, "queries")
        want, bound = R.rotate(h[:, heads:heads + kv], None, table, pos, 1e-6, False)
        R.assert_within(kc[dslot], want, bound, "keys")
        assert torch.equal(vc[dslot].cpu(), h[:, heads + kv:])
        want, bound = R.attend(q_out.cpu(), kc.cpu(), vc.cpu(), list(range(tokens + 1)),
                               [i * keys for i in range(tokens)], [keys] * tokens, d ** -0.5,
                               causal=True)
        R.assert_within(out, want, bound, "attend")


def test_broken_values_do_not_stall():
    """All results NaN: formed again one by one, which must not take hundreds of times as long."""
    say("broken values")
    g, dt, n = gen(44), torch.bfloat16, 4096

    def took(call):
        call()
        best = math.inf
        for _ in range(3):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            call()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    q, k, v = (normal(g, n, h, 128, dtype=dt).cuda() for h in (8, 2, 2))
    seqs = tg.Sequences(*(torch.tensor(t, dtype=i).cuda() for t, i in (
        ([0, n], torch.int32), ([0], torch.int64), ([n], torch.int32))), n, n)
    out, bufs = torch.empty_like(q), tg.AttendBuffers(seqs, q, k)
    call = lambda: tg.attend(q, k, v, seqs, out, bufs, 0.1, causal=True)
    well = took(call)
    q[:, :, 7] = NAN
    assert took(call) < 60 * well and bool(torch.isnan(out).all())
    x, w = normal(g, n, 1024, dtype=dt).cuda(), normal(g, 1024, 1024, dtype=dt).cuda()
    low = tg.Adapters(normal(g, 2, 16, 1024, dtype=dt).cuda(),
                      normal(g, 2, 1024, 16, dtype=dt).cuda(), torch.ones(2, device="cuda"))
    ids = (torch.arange(n, device="cuda") // 100 % 2).int()
    pb = tg.ProjectBuffers(n, 1024, 1024, dt, low)
    call = lambda: tg.project(x, w, pb, low, ids)
    well = took(call)
    x[:, 7] = NAN
    assert took(call) < 60 * well and bool(torch.isnan(pb.y).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_len,n", [(1, 1), (1, 3000), (5, 90), (90, 1), (90, 150), (140, 3000)])
def test_attend_scores_of_minus_infinity(q_len, n, dtype):
    """A query whose every score is minus infinity has no weights: NaN, and not 0 as for no key."""
    say("attend minus infinity", q_len, n, dtype)
    _, q, k, v, qb, kb = make(47, [q_len], [n], 4, 2, 64, dtype)
    k[..., 0] = k[..., 0].abs() + 0.5
    f = dict(causal=True)
    want, bound = R.attend(q, k, v, qb, kb, [n], 0.125, **f)
    sick = torch.arange(q_len) == q_len - 1 if n < q_len else torch.arange(q_len) % 3 == 0
    q[sick, :, 0] = -math.inf
    finite_rest(run_attend(q, k, v, qb, kb, [n], 0.125, **f), want, bound, sick)
