"""The serving operators (tg_pages, tg_attend_pages, tg_norm, tg_quantize, tg_project_i8) against
plain implementations, through the C ABI: types, odd sizes, strides, lengths of zero and one, pages
that end anywhere, values that must not reach a result, streams and captured graphs."""
import math
import random

import pytest
import torch

from gpu_helpers import say
from paper_2404_09267_amd import tg
import serving_reference as R

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype, gain=1.0):
    return (torch.randn(shape, generator=g) * gain).to(dtype)


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def apart(t, rows=2, wide=16):
    """The values of t [n, ...] on the device inside a wider tensor of NaN (or 77), and that
    tensor; rows stay on 16-byte boundaries where the width allows."""
    shape = (t.shape[0] + rows, *t.shape[1:-1], t.shape[-1] + wide)
    whole = torch.full(shape, NAN if t.dtype.is_floating_point else 77, dtype=t.dtype,
                       device="cuda")
    view = whole[1:1 + t.shape[0], ..., wide // 2:wide // 2 + t.shape[-1]]
    view.copy_(t)
    return view, whole


def untouched(view, whole):
    """Nothing around `view` in `whole` (see apart) was written."""
    left = whole.clone()
    at = view.storage_offset() - whole.storage_offset()
    left.as_strided(view.shape, view.stride(), at).fill_(NAN if left.is_floating_point() else 77)
    return bool(torch.isnan(left).all() if left.is_floating_point() else (left == 77).all())


# --------------------------------------------------------------------------------- pages

class Step:
    """A cache's pages on the device and as lists, stepped together."""

    def __init__(self, seqs, cols, n_pages, page, seed=0, stride=None):
        r = random.Random(seed)
        self.page, self.n_pages, self.cols = page, n_pages, cols
        stack = list(range(n_pages))
        r.shuffle(stack)
        self.lens, self.free = [0] * seqs, stack
        self.table = [[-1] * cols for _ in range(seqs)]
        wide = torch.full((seqs, stride or cols), -7, dtype=torch.int32, device="cuda")
        wide[:, :cols] = -1
        self.wide = wide
        self.dev = tg.Pages(wide[:, :cols], ints(self.lens), page, ints(stack), ints([n_pages]))

    def step(self, new, release=None, pad=0, ahead=0, with_pos=True):
        begin = [ahead]
        for n in new:
            begin.append(begin[-1] + n)
        tokens = begin[-1] + pad
        bufs = tg.PagesBuffers(self.dev, tokens)
        bufs.slot.fill_(-99)
        bufs.pos.fill_(-99)
        want = R.pages(begin, self.lens, self.table, self.free, len(self.free), self.page,
                       self.n_pages, tokens, release)
        a = tg.pages_args(self.dev, ints(begin), bufs, ints(release) if release else None)
        if not with_pos:
            a.pos = None
        assert tg.pages_raw(a) == tg.OK
        torch.cuda.synchronize()
        assert self.dev.kv_len.tolist() == want["kv_len"]
        assert self.dev.table.tolist() == want["table"]
        n = int(self.dev.n_free)
        assert self.dev.free.tolist()[:n] == want["free"]
        assert bufs.slot.tolist() == want["slot"]
        assert bufs.pos[:, 0].tolist() == (want["pos"] if with_pos else [-99] * tokens)
        assert int(bufs.refused) == want["refused"]
        if self.wide.shape[1] > self.cols:
            assert bool((self.wide[:, self.cols:] == -7).all())
        self.lens, self.table, self.free = want["kv_len"], want["table"], want["free"]
        held = [p for row, m in zip(self.table, self.lens) for p in row[:-(-m // self.page)]]
        assert sorted(held + self.free) == list(range(self.n_pages))
        return want


@pytest.mark.parametrize("page", [1, 16, 24, 128])
@pytest.mark.parametrize("seqs", [1, 5, 64, 65, 1500])
def test_pages_steps(seqs, page):
    """Prompts, single tokens and ends, one step after the other, until pages run out."""
    say("pages", seqs, page)
    r = random.Random(seqs * 1000 + page)
    cols = max(3, 90 // page)
    s = Step(seqs, cols, max(2, seqs * cols * 2 // 3), page, seed=seqs, stride=cols + 3)
    refused = 0
    for step in range(9):
        new = [r.choice([0, 1, 1, 1, 2, page, page + 1, r.randint(1, 60)]) for _ in range(seqs)]
        ends = [int(r.random() < 0.15) for _ in range(seqs)] if step % 3 else None
        refused += s.step(new, ends, pad=r.choice([0, 5]), ahead=r.choice([0, 3]),
                          with_pos=step != 4)["refused"]
    assert refused > 0 or seqs < 64


@pytest.mark.parametrize("tokens", [4096, 4097, 20000])
def test_pages_long_prompts(tokens):
    """Both ways of giving tokens their rows: in the one launch and in a second one."""
    say("pages prompts", tokens)
    s = Step(7, 2000, 3000, 16, seed=3)
    s.step([1, 0, 5, 2, 0, 0, 1])
    s.step([1, 0, tokens // 2, 1, 0, tokens - tokens // 2 - 12, 1], pad=5, ahead=4)
    s.step([tokens - 1, 0, 0, 0, 0, 1, 0], [0, 0, 1, 0, 0, 1, 0])


def test_pages_many_short_prompts():
    """More tokens than the one launch serves, of more sequences than fit its list."""
    say("pages many")
    s = Step(5000, 2, 9000, 4, seed=4)
    s.step([1 + i % 4 for i in range(5000)], pad=100)
    s.step([i % 3 for i in range(5000)], [int(i % 7 == 0) for i in range(5000)])


def test_pages_without_tokens():
    """A step in which requests end and nobody brings a token."""
    say("pages without tokens")
    for seqs in (3, 1100):
        s = Step(seqs, 5, 5 * seqs, 8, seed=6)
        s.step([i % 39 for i in range(seqs)])
        s.step([0] * seqs, [i % 2 for i in range(seqs)])
        s.step([0] * seqs)
        s.step([0] * seqs, [1] * seqs)
        assert len(s.free) == 5 * seqs


def test_pages_nobody():
    """No sequences: padding alone."""
    say("pages nobody")
    table = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    p = tg.Pages(table, ints([]), 16, ints([4, 2]), ints([2]))
    for tokens in (3, 5000):
        bufs = tg.PagesBuffers(p, tokens)
        bufs.slot.fill_(9)
        tg.pages(p, ints([0]), bufs)
        assert set(bufs.slot.tolist()) == {-1} and set(bufs.pos[:, 0].tolist()) == {0}
        assert int(p.n_free) == 2 and int(bufs.refused) == 0


@pytest.mark.parametrize("tokens", [40, 6000])
def test_pages_bad_state(tokens):
    """Lengths, counts, tables and token ranges that are none: nothing outside the arrays is read
    or written, and the rows that come out are rows of the cache."""
    say("pages bad state", tokens)
    g = gen(tokens)
    seqs, cols, n_pages, page = 300, 5, 50, 8
    for turn in range(4):
        wild = torch.randint(-(1 << 31), (1 << 31) - 1, (seqs * cols,), generator=g)
        some = torch.randint(-2, n_pages + 2, (seqs * cols,), generator=g)
        table = torch.where(torch.rand(seqs * cols, generator=g) < 0.3, wild, some).int()
        lens = torch.randint(-9, 3 * page * cols, (seqs,), generator=g).int()
        lens[::7] = -(1 << 31)
        lens[1::7] = (1 << 31) - 1
        begin = torch.randint(-9, tokens + 9, (seqs + 1,), generator=g).int()
        if turn % 2:
            begin = begin.sort().values
        whole = torch.full((seqs * cols + 200,), 77, dtype=torch.int32, device="cuda")
        whole[100:-100] = table.cuda()
        stack = torch.full((n_pages + 200,), 77, dtype=torch.int32, device="cuda")
        stack[100:-100] = some[:n_pages].int().cuda()
        p = tg.Pages(whole[100:-100].view(seqs, cols), lens.cuda(), page, stack[100:-100],
                     ints([[1 << 30, -5, n_pages, 7][turn]]))
        bufs = tg.PagesBuffers(p, tokens)
        tg.pages(p, begin.cuda(), bufs, release=torch.randint(0, 2, (seqs,), generator=g).int().cuda())
        torch.cuda.synchronize()
        for t in (whole, stack):
            assert set(t[:100].tolist()) == set(t[-100:].tolist()) == {77}
        assert 0 <= int(p.n_free) <= n_pages
        assert int(p.kv_len.min()) >= 0 and int(p.kv_len.max()) <= page * cols
        if turn % 2:
            assert int(bufs.slot.min()) >= -1 and int(bufs.slot.max()) < n_pages * page


def test_pages_repeat_apart():
    """With lengths and count apart a call can be repeated, and gives the same."""
    say("pages repeat")
    s = Step(9, 6, 40, 8, seed=5)
    s.step([9, 1, 20, 8, 0, 3, 16, 1, 2])
    after = tg.Pages(s.dev.table, torch.empty_like(s.dev.kv_len), 8, s.dev.free, ints([0]))
    bufs = tg.PagesBuffers(s.dev, 7)
    a = tg.pages_args(s.dev, ints([0, 1, 2, 3, 4, 4, 5, 6, 7, 7]), bufs,
                      release=ints([0, 0, 0, 0, 1, 0, 0, 0, 1]), after=after)
    got = []
    for _ in range(3):
        assert tg.pages_raw(a) == tg.OK
        torch.cuda.synchronize()
        got.append((after.kv_len.tolist(), after.n_free.tolist(), bufs.slot.tolist(),
                    s.dev.table.tolist(), s.dev.free.tolist()))
    assert got[0] == got[1] == got[2]
    assert s.dev.kv_len.tolist() == s.lens


# ---------------------------------------------------------------------------- attend_pages

def cache(g, lens, page, kv_heads, d, dtype, spare=3, cols=None):
    """A paged cache on the CPU: k, v [rows, kv heads, d], table; pages in no order, and NaN in
    every row that no sequence holds."""
    count = [-(-n // page) for n in lens]
    n_pages = sum(count) + spare
    order = torch.randperm(n_pages, generator=g)
    cols = cols or max(max(count), 1)
    table = torch.full((len(lens), cols), -1, dtype=torch.int32)
    rows = n_pages * page
    k, v = (normal(g, rows, kv_heads, d, dtype=dtype) for _ in range(2))
    held = torch.zeros(rows, dtype=torch.bool)
    at = 0
    for s, (n, c) in enumerate(zip(lens, count)):
        table[s, :c] = order[at:at + c].int()
        j = torch.arange(n)
        held[table[s].long()[j // page] * page + j % page] = True
        at += c
    k[~held], v[~held] = NAN, NAN
    return k, v, table


def widened(table, page, most):
    """The table with entries that are no page, up to `most` rows: what a sequence may hold, and
    not what it holds, decides how a call is done."""
    more = 0 if most is None else -(-most // page) - table.shape[1]
    return torch.nn.functional.pad(table, (0, max(more, 0)), value=-1)


def run_attend(q, k, v, table, lens, page, max_kv=None, out=None, **more):
    pages = tg.Pages(table.cuda(), ints(list(lens)), page)
    qd, kd, vd = (t if t.is_cuda else t.cuda() for t in (q, k, v))
    out = torch.full(q.shape, NAN, dtype=q.dtype, device="cuda") if out is None else out
    bufs = tg.AttendPagesBuffers(qd, kd, max(lens) if max_kv is None else max_kv)
    bufs.workspace.fill_(255)
    if more.get("slope") is not None:
        more["slope"] = more["slope"].cuda()
    tg.attend_pages(qd, kd, vd, pages, out, bufs, **more)
    torch.cuda.synchronize()
    return out.cpu()


ATTEND = [
    # lengths, page, heads, kv heads, d, extras
    ([1], 16, 1, 1, 8, {}), ([0, 1, 2], 1, 2, 1, 64, {}), ([31, 32, 33, 0], 8, 8, 2, 32, {}),
    ([63, 64, 65, 129], 24, 14, 2, 80, dict(slope=True)), ([500, 7], 16, 16, 16, 128, {}),
    ([513, 1, 900], 16, 16, 4, 64, dict(cap=30.0)), ([2000], 7, 7, 1, 72, dict(slope=True)),
    ([700, 0, 1300, 64], 128, 40, 2, 128, dict(cap=2.0, slope=True)),
    ([1025] * 3 + [5], 64, 4, 4, 40, dict(window=100)), ([300, 40, 0, 90], 5, 4, 2, 96,
                                                        dict(window=64, slope=True)),
    ([1500, 1501, 1502], 32, 6, 2, 128, dict(window=1100, cap=50.0)),
    ([3000] + [3] * 70, 16, 8, 4, 64, {}), ([90] * 260, 16, 2, 1, 16, {}),
    ([90, 33, 64], 8, 6, 2, 128, {}), ([400, 39], 40, 5, 1, 72, {}),
    ([90, 5, 0] * 13, 16, 6, 2, 72, {}), ([64, 33, 100] * 11, 32, 36, 1, 40, dict(slope=True)),
]


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attend_pages(case, dtype, most):
    lens, page, heads, kv, d, extra = ATTEND[case]
    say("attend_pages", case, dtype)
    g, dt = gen(case), DT[dtype]
    k, v, table = cache(g, lens, page, kv, d, dt)
    table = widened(table, page, most)
    q = normal(g, len(lens), heads, d, dtype=dt, gain=2.0)
    more = dict(extra, scale=d ** -0.5)
    if more.get("slope"):
        more["slope"] = torch.linspace(-0.01, 0.3, heads)
    want, bound = R.attend_pages(q, k, v, table, lens, page, **more)
    got = run_attend(q, k, v, table, lens, page, most, **more)
    R_assert(got, want, bound, "attend_pages")


def R_assert(got, want, bound, name):
    from token_reference import assert_within

    assert_within(got, want, bound, name)


@pytest.mark.parametrize("max_kv", [0, 40, 5000, 1 << 30])
def test_attend_pages_bounds(max_kv):
    """A bound below, or far above, the lengths; lengths past the table; lengths below 0."""
    say("attend_pages bounds", max_kv)
    g, lens, page = gen(11), [700, 64, 0, 33], 16
    k, v, table = cache(g, lens, page, 2, 64, torch.bfloat16)
    q = normal(g, 4, 8, 64, dtype=torch.bfloat16)
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.1, max_kv=max_kv)
    R_assert(run_attend(q, k, v, table, lens, page, max_kv, scale=0.1), want, bound, "bound")
    long = [700, 64, -5, (1 << 31) - 1]
    table[3, 3:] = -1  # of the last one's claim, three pages are there
    k2, v2 = torch.nan_to_num(k, nan=0.5), torch.nan_to_num(v, nan=0.25)
    if max_kv < 1 << 30:
        want, bound = R.attend_pages(q[:3], k2, v2, table[:3], long[:3], page, 0.1, max_kv=max_kv)
        got = run_attend(q, k2, v2, table, long, page, max_kv, scale=0.1)
        R_assert(got[:3], want, bound, "long")
        j = min(48, max_kv)
        want, bound = R.attend_pages(q[3:], k2, v2, table[3:], [j], page, 0.1)
        R_assert(got[3:], want, bound, "past the table")


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("length", [60, 1500])
def test_attend_pages_hides(length, most):
    """Pages that are none, rows past the end and before the window hold NaN and infinities."""
    say("attend_pages hides", length)
    g, page = gen(12), 16
    lens = [length, length - 5, 20, 17]
    k, v, table = cache(g, lens, page, 2, 64, torch.float16)
    table = widened(table, page, most)
    q = normal(g, 4, 4, 64, dtype=torch.float16)
    n_pages = k.shape[0] // page
    for s, (at, bad) in enumerate(((1, -1), (0, n_pages), (0, 1 << 30), (1, -(1 << 31)))):
        j = torch.arange(at * page, min((at + 1) * page, lens[s]))
        rows = table[s, at].long() * page + j % page
        k[rows], v[rows] = INF, NAN
        table[s, at] = bad
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.2)
    R_assert(run_attend(q, k, v, table, lens, page, most, scale=0.2), want, bound, "bad pages")
    table[:] = -1
    assert bool((run_attend(q, k, v, table, lens, page, most, scale=0.2) == 0).all())
    k, v, table = cache(g, lens, page, 2, 64, torch.float16)
    table = widened(table, page, most)
    for s, n in enumerate(lens):
        j = torch.arange(n - 9)
        rows = table[s].long()[j // page] * page + j % page
        k[rows], v[rows] = NAN, INF
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.2, window=9)
    got = run_attend(q, k, v, table, lens, page, most, scale=0.2, window=9)
    R_assert(got, want, bound, "window")


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("length", [40, 1500])
def test_attend_pages_broken_values(length, most):
    """NaN that a query sees is its result, an infinite value its column's; scores that are all
    minus infinity leave no weights. Other sequences and heads do not see it."""
    say("attend_pages broken", length)
    g, page, d = gen(13), 16, 32
    lens = [length] * 5
    k, v, table = cache(g, lens, page, 2, d, torch.bfloat16)
    table = widened(table, page, most)
    k, v = torch.nan_to_num(k, nan=1.0), torch.nan_to_num(v, nan=1.0)
    q = normal(g, 5, 4, d, dtype=torch.bfloat16).abs() + 0.1
    row = lambda s, j: int(table[s, j // page]) * page + j % page
    clean, bound = R.attend_pages(q, k, v, table, lens, page, 0.1)
    k[row(1, length - 1), 0, 3] = NAN
    v[row(2, 3), 1, 5] = INF
    for j in range(length):
        k[row(3, j), 1, :] = -INF
    k[row(4, 7), 0, :] = -INF  # one score of minus infinity: no weight
    got = run_attend(q, k, v, table, lens, page, most, scale=0.1)
    assert bool(torch.isnan(got[1, :2]).all()) and bool((got[2, 2:, 5] == INF).all())
    assert bool(torch.isnan(got[3, 2:]).all())
    want4, bound4 = R.attend_pages(q[4:], torch.nan_to_num(k, nan=0, neginf=-3e38), v, table[4:],
                                   lens[4:], page, 0.1)
    R_assert(got[4:], want4, bound4, "minus infinity")
    fine = torch.ones(got.shape, dtype=torch.bool)
    fine[1, :2], fine[2, 2:, 5], fine[3, 2:], fine[4] = False, False, False, False
    R_assert(got[fine], clean[fine], bound[fine], "others")


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("length", [45, 1300])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attend_pages_large_scores(length, dtype, most):
    """Scores of 2^24 and more: the largest takes all, none is lost to rounding; factors at the
    ends of binary32; a factor of 0 and below 0."""
    say("attend_pages large", length, dtype)
    g, page, d, dt = gen(14), 16, 64, DT[dtype]
    k, v, table = cache(g, [length], page, 1, d, dt)
    table = widened(table, page, most)
    q = normal(g, 1, 3, d, dtype=dt)
    for scale in (0.0, -0.3, 3e7, 1e30):
        got = run_attend(q, k, v, table, [length], page, most, scale=scale).double()
        j = torch.arange(length)
        rows = table[0].long()[j // page] * page + j % page
        if abs(scale) < 1:
            want, bound = R.attend_pages(q, k, v, table, [length], page, scale)
            R_assert(got, want, bound, f"scale {scale}")
            continue
        for h in range(3):
            best = int((k[rows, 0].double() @ q[0, h].double()).argmax())
            assert torch.equal(got[0, h], v[rows[best], 0].double()), (scale, h)


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("cap", [1e-3, 5.0, 1e4, 1e30])
def test_attend_pages_caps(cap, most):
    say("attend_pages cap", cap)
    g, page, d, lens = gen(15), 16, 64, [50, 1100]
    k, v, table = cache(g, lens, page, 1, d, torch.float16)
    table = widened(table, page, most)
    q = normal(g, 2, 5, d, dtype=torch.float16, gain=3.0)
    # tanh does nothing to scores under 1e30, and the bound is then that of the plain score
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.2, cap=cap if cap < 1e15 else 0.0)
    R_assert(run_attend(q, k, v, table, lens, page, most, scale=0.2, cap=cap), want, bound, "cap")


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
def test_attend_pages_strides(most):
    """Heads and rows apart, inside wider tensors; nothing but the result is written."""
    say("attend_pages strides")
    g, page, lens = gen(16), 24, [70, 1200, 0]
    k, v, table = cache(g, lens, page, 2, 72, torch.bfloat16)
    table = widened(table, page, most)
    q = normal(g, 3, 6, 72, dtype=torch.bfloat16)
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.1)
    # k and v of one tensor, heads outside rows
    both = torch.full((2, 2, k.shape[0], 88), NAN, dtype=k.dtype, device="cuda")
    both[0, :, :, 8:80] = k.transpose(0, 1).cuda()
    both[1, :, :, 8:80] = v.transpose(0, 1).cuda()
    kd, vd = (both[i, :, :, 8:80].transpose(0, 1) for i in (0, 1))
    qd, _ = apart(q)
    out, whole = apart(torch.zeros(q.shape, dtype=q.dtype))
    wide = torch.full((3, table.shape[1] + 5), 0, dtype=torch.int32, device="cuda")
    wide[:, 2:-3] = table.cuda()
    pages = tg.Pages(wide[:, 2:-3], ints(lens), page)
    tg.attend_pages(qd, kd, vd, pages, out, tg.AttendPagesBuffers(qd, kd, most or 1200), 0.1)
    torch.cuda.synchronize()
    R_assert(out.cpu(), want, bound, "strides")
    assert untouched(out, whole)


def test_attend_pages_far_rows():
    """Rows past 2^31 values of the cache: 5 GiB of keys, of which a few pages are used."""
    say("attend_pages far")
    page, kv, d, n_pages = 64, 8, 128, 40960
    k = torch.zeros((n_pages * page, kv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((n_pages * page, kv, d), dtype=torch.bfloat16, device="cuda")
    g, lens = gen(17), [150, 900]
    sk, sv, table = cache(g, lens, page, kv, d, torch.bfloat16, spare=0)
    far = n_pages - sk.shape[0] // page
    k[far * page:], v[far * page:] = sk.cuda(), sv.cuda()
    q = normal(g, 2, 8, d, dtype=torch.bfloat16)
    want, bound = R.attend_pages(q, sk, sv, table, lens, page, 0.1)
    R_assert(run_attend(q, k, v, table + far, lens, page, scale=0.1), want, bound, "far")


@pytest.mark.parametrize("window", [0, 33, 2222])
@pytest.mark.parametrize("lens", [[0, 0, 2500, 0, 1, 31, 32, 33, 0, 4000, 64, 0, 0], [0] * 7,
                                  [1] * 40 + [0] * 40 + [4500], [4100, 0], [64] * 66 + [2100],
                                  [17000, 3]])
def test_attend_pages_ranges(lens, window):
    """Sequences of no keys and of few among long ones, where all keys are cut into ranges."""
    say("attend_pages ranges", len(lens), window)
    g, page = gen(19), 8
    k, v, table = cache(g, lens, page, 1, 32, torch.bfloat16)
    q = normal(g, len(lens), 2, 32, dtype=torch.bfloat16)
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.2, window=window)
    got = run_attend(q, k, v, table, lens, page, 17000, scale=0.2, window=window)
    R_assert(got, want, bound, "ranges")


@pytest.mark.parametrize("longest", [300, 3000])
def test_attend_pages_rows_of_tokens(longest):
    """Queries are the last tokens of sequences; those without tokens have none, and no other row
    is written."""
    say("attend_pages rows", longest)
    g, page, lens = gen(20), 16, [40, 7, longest, 0, 90, 64, 33]
    k, v, table = cache(g, lens, page, 2, 64, torch.float16)
    begin = [2, 3, 3, 8, 9, 9, 10, 14]  # the last one's row is outside
    q = normal(g, 12, 4, 64, dtype=torch.float16)
    has, rows = [0, 2, 3, 5], [2, 7, 8, 9]
    want, bound = R.attend_pages(q[rows], k, v, table[has], [lens[i] for i in has], page, 0.2)
    pages = tg.Pages(table.cuda(), ints(lens), page)
    out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
    bufs = tg.AttendPagesBuffers(q, k, longest, n_seqs=len(lens))
    tg.attend_pages(q.cuda(), k.cuda(), v.cuda(), pages, out, bufs, 0.2, q_begin=ints(begin))
    out = out.cpu()
    R_assert(out[rows], want, bound, "rows")
    out[rows] = 5.0
    assert bool((out == 5.0).all())
    begin = [-5, -1, 0, 0, 1 << 30, 3, 99, -(1 << 31)]
    bad = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
    tg.attend_pages(q.cuda(), k.cuda(), v.cuda(), pages, bad, bufs, 0.2, q_begin=ints(begin))
    assert bool((bad == 5.0).all())


@pytest.mark.parametrize("seqs", [1024, 1025])
def test_attend_pages_many_sequences(seqs):
    """As many sequences as are cut, and one more; one of them long."""
    say("attend_pages many", seqs)
    g, page = gen(18), 16
    lens = [5] * (seqs - 1) + [5000]
    k, v, table = cache(g, lens, page, 1, 16, torch.float16)
    q = normal(g, seqs, 1, 16, dtype=torch.float16)
    want, bound = R.attend_pages(q, k, v, table, lens, page, 0.25)
    R_assert(run_attend(q, k, v, table, lens, page, scale=0.25), want, bound, "many")


# ----------------------------------------------------------------------------------- norm

NORM = [(1, 1), (3, 7), (5, 64), (2, 100), (7, 512), (3, 513), (4, 1024), (2, 1160), (3, 2048),
        (2, 2049), (5, 4096), (2, 5000), (2, 8192), (1, 8200), (2, 16384), (1, 16385), (1, 32768),
        (66, 96)]


def norm_inputs(g, tokens, n, dt, gates):
    x, y = normal(g, tokens, n, dtype=dt, gain=3.0), normal(g, tokens, n, dtype=dt) + 1
    vec = lambda at: (at + normal(g, n, dtype=torch.float32, gain=0.3)).to(dt)
    gate = normal(g, gates, n, dtype=dt) if gates else None
    row = torch.randint(-1, gates + 1, (tokens,), generator=g).int() if gates > 1 else None
    return x, y, vec(1), vec(0), gate, row, vec(1), vec(0)


def run_norm(x, y=None, x_out=True, h=True, **more):
    dev = lambda t: t.cuda() if isinstance(t, torch.Tensor) else t
    xo, ho = (torch.full(x.shape, NAN, dtype=x.dtype, device="cuda") if want else None
              for want in (x_out, h))
    tg.norm(dev(x), xo, ho, y=dev(y), **{k: dev(t) for k, t in more.items()})
    torch.cuda.synchronize()
    return xo, ho


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,n", NORM)
def test_norm(tokens, n, dtype):
    say("norm", tokens, n, dtype)
    g, dt = gen(tokens * n), DT[dtype]
    for y_norm, kind, gates in ((1, 1, 3), (2, 2, 0), (0, 2, 1), (2, 0, 3)):
        x, y, yw, yb, gate, row, w, b = norm_inputs(g, tokens, n, dt, gates)
        more = dict(y_norm=y_norm, y_weight=yw, y_bias=yb if kind == 2 else None, gate=gate,
                    gate_row=row, x_scale=0.7, y_scale=-0.4, weight=w,
                    bias=b if kind != 1 else None, eps=1e-5)
        (r, er), (h, eh) = R.norm(x, y, kind=kind, **more)
        xo, ho = run_norm(x, y, norm=kind, **more)
        R_assert(xo.cpu(), r, er, f"x_out {y_norm} {kind}")
        R_assert(ho.cpu(), h, eh, f"h {y_norm} {kind}")
    (r, er), (h, eh) = R.norm(x, kind=1)
    _, ho = run_norm(x, x_out=False)
    R_assert(ho.cpu(), h, eh, "norm alone")
    xo, _ = run_norm(x, h=False, x_scale=0.5)
    R_assert(xo.cpu(), r / 2, er / 2 + 2.0 ** -24, "scale alone")


@pytest.mark.parametrize("n", [100, 1000, 4096])
def test_norm_in_place_and_strides(n):
    """x_out is x, h is y, rows apart; nothing around the results is written."""
    say("norm in place", n)
    g, dt = gen(n), torch.bfloat16
    x, y, yw, yb, gate, row, w, b = norm_inputs(g, 9, n, dt, 4)
    more = dict(y_norm=2, y_weight=yw, gate=gate, gate_row=row, weight=w, bias=b)
    (r, er), (h, eh) = R.norm(x, y, kind=1, **more)
    dev = {k: t.cuda() if isinstance(t, torch.Tensor) else t for k, t in more.items()}
    dev["gate"], _ = apart(gate)
    for odd in (16, 18):  # rows on 16-byte boundaries, and not
        xd, wx = apart(x, wide=odd)
        yd, wy = apart(y, wide=odd)
        tg.norm(xd, xd, yd, y=yd, norm=1, **dev)
        torch.cuda.synchronize()
        R_assert(xd.cpu(), r, er, "x in place")
        R_assert(yd.cpu(), h, eh, "h in y's place")
        assert untouched(xd, wx) and untouched(yd, wy)
    yd, xd = y.cuda(), x.cuda()
    tg.norm(xd, yd, xd, y=yd, norm=1, **dev)
    torch.cuda.synchronize()
    R_assert(yd.cpu(), r, er, "x_out in y's place")
    R_assert(xd.cpu(), h, eh, "h in x's place")


def test_norm_gates_keep_apart():
    """A token without a gate does not see y, and no token another's gate, whatever they hold."""
    say("norm gates")
    g, dt = gen(31), torch.float16
    x, y, yw, yb, gate, row, w, b = norm_inputs(g, 8, 640, dt, 3)
    row = torch.tensor([0, 1, 2, -1, 3, 0, -(1 << 31), (1 << 31) - 1]).int()
    want = R.norm(x, y, 1, yw, None, gate, row, kind=1, weight=w)
    none = row.clamp(0, 2) != row
    y[none], gate[1] = NAN, INF
    xo, ho = run_norm(x, y, y_norm=1, y_weight=yw, gate=gate, gate_row=row, norm=1, weight=w)
    fine = torch.arange(8) != 1
    for got, (exp, bound) in zip((xo, ho), want):
        R_assert(got.cpu()[fine], exp[fine], bound[fine], "gates")
    assert not bool(torch.isfinite(xo[1]).any())


@pytest.mark.parametrize("n", [96, 3000, 9000])
@pytest.mark.parametrize("kind", [1, 2])
def test_norm_far_from_one(n, kind):
    """bfloat16 whose squares leave binary32 at either end, with and without an eps to hide it."""
    say("norm far", n, kind)
    g = gen(n + kind)
    x = normal(g, 6, n, dtype=torch.float32)
    for eps, gains in ((0.0, (1e30, 1e-30, 1e37, 3e-38)), (1e-6, (1e30, 1e-30)),
                       (1e-30, (1e-12, 1e-18))):
        for gain in gains:
            v = (x * gain).to(torch.bfloat16)
            _, (h, eh) = R.norm(v, kind=kind, eps=eps)
            _, ho = run_norm(v, x_out=False, norm=kind, eps=eps)
            # values below 2^-126 have lost digits before the norm sees them
            R_assert(ho.cpu(), h, eh + (2.0 ** -7 if gain < 1e-37 else 0) * h.abs(), f"{gain} {eps}")
    _, ho = run_norm(torch.zeros((2, n)).bfloat16(), x_out=False, norm=kind, eps=1e-30)
    assert bool((ho == 0).all())
    flat = torch.full((2, n), 1e30).bfloat16()
    _, ho = run_norm(flat, x_out=False, norm=kind, eps=1e-6)
    assert bool(((ho - int(kind == 1)).abs() <= 2.0 ** -7).all())


@pytest.mark.parametrize("n", [1, 9, 60, 64, 100, 128, 129, 132, 200, 255, 256, 257])
def test_norm_narrow(n):
    """Many short rows, of which neighbours share a wave: far, flat, broken and without a gate."""
    say("norm narrow", n)
    g, dt, tokens = gen(n), torch.bfloat16, 1003
    for kind in (1, 2):
        x, y, yw, yb, gate, row, w, b = norm_inputs(g, tokens, n, dt, 3)
        gain = torch.tensor([1.0, 1e30, 1e-3, 0.0, 1.0, 1e25, 1.0])[torch.arange(tokens) % 7]
        x = (x.float() * gain[:, None]).to(dt)
        more = dict(y_norm=kind, y_weight=yw, gate=gate, gate_row=row, weight=w, bias=b, eps=1e-5)
        if n == 1 and kind == 2:  # all of a row is its mean
            more.update(y_norm=0)
        (r, er), (h, eh) = R.norm(x, y, kind=kind, **more)
        broken = torch.arange(tokens) % 11 == 5
        x[broken, n - 1] = NAN
        xo, ho = run_norm(x, y, norm=kind, **more)
        R_assert(xo.cpu()[~broken], r[~broken], er[~broken], "x_out")
        R_assert(ho.cpu()[~broken], h[~broken], eh[~broken], "h")
        assert bool(torch.isnan(ho.cpu()[broken]).all())


@pytest.mark.parametrize("n", [520, 1024, 1999, 2040, 4092, 4096, 8184, 8191])
def test_norm_many(n):
    """Rows of more than 2^22 values together, some of them with squares past binary32."""
    say("norm many", n)
    tokens = (1 << 22) // n + 3
    g, dt = gen(n), torch.bfloat16
    for kind in (1, 2):
        x, y, yw, yb, gate, row, w, b = norm_inputs(g, tokens, n, dt, 3)
        x[5], x[tokens - 1] = x[5] * 1e30, x[tokens - 1] * 1e30
        more = dict(y_norm=kind, y_weight=yw, gate=gate, gate_row=row, weight=w, bias=b, eps=1e-5)
        (r, er), (h, eh) = R.norm(x, y, kind=kind, **more)
        xo, ho = run_norm(x, y, norm=kind, **more)
        R_assert(xo.cpu(), r, er, "x_out")
        R_assert(ho.cpu(), h, eh, "h")


def test_norm_large_offset():
    """A mean far larger than the spread: variance from differences, not from sums of squares."""
    say("norm offset")
    x = (100 + torch.randn((4, 4096), generator=gen(33))).half()
    _, (h, eh) = R.norm(x, kind=2)
    _, ho = run_norm(x, x_out=False, norm=2)
    R_assert(ho.cpu(), h, eh, "offset")


def test_norm_broken_rows_stay_apart():
    say("norm broken")
    for n in (96, 2000):
        x = normal(gen(34), 6, n, dtype=torch.bfloat16)
        _, (h, eh) = R.norm(x, kind=2)
        x[1, 3], x[4, n - 1] = NAN, INF
        _, ho = run_norm(x, x_out=False, norm=2)
        fine = torch.tensor([0, 2, 3, 5])
        R_assert(ho.cpu()[fine], h[fine], eh[fine], "others")
        assert bool(torch.isnan(ho[1]).all()) and bool(torch.isnan(ho[4]).any())


# ------------------------------------------------------------------------------- quantize

QUANT = [(1, 1), (3, 7), (70, 8), (5, 100), (6, 512), (3, 520), (2, 1024), (9, 1160), (3, 2048),
         (2, 4096), (2, 4104), (1, 8192), (2, 10000), (1, 16384), (1, 32768), (2, 40000), (1, 5001)]


def run_quantize(x, q=None):
    q = torch.full(x.shape, 77, dtype=torch.int8, device="cuda") if q is None else q
    scale = torch.full((x.shape[0],), -1.0, device="cuda")
    tg.quantize(x if x.is_cuda else x.cuda(), q, scale)
    torch.cuda.synchronize()
    return q.cpu(), scale.cpu()


def same_rows(got, want):
    assert torch.equal(got[0], want[0])
    assert torch.equal(got[1].view(torch.int32)[~torch.isnan(want[1])],
                       want[1].view(torch.int32)[~torch.isnan(want[1])])
    assert torch.equal(torch.isnan(got[1]), torch.isnan(want[1]))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,k", QUANT)
def test_quantize(rows, k, dtype):
    say("quantize", rows, k, dtype)
    x = normal(gen(rows * k), rows, k, dtype=DT[dtype], gain=2.5)
    same_rows(run_quantize(x), R.quantize(x))
    wide, _ = apart(x, wide=18)  # rows off the 16-byte boundaries
    q, whole = apart(torch.zeros(x.shape, dtype=torch.int8), wide=7)
    same_rows(run_quantize(wide, q), R.quantize(x))
    assert untouched(q, whole)
    wide, _ = apart(x)
    q, whole = apart(torch.zeros(x.shape, dtype=torch.int8))
    same_rows(run_quantize(wide, q), R.quantize(x))
    assert untouched(q, whole)


@pytest.mark.parametrize("k", [1, 9, 60, 64, 100, 128, 129, 132, 200, 255, 256, 257])
def test_quantize_narrow(k):
    """Many short rows, of which neighbours share a wave: far, of zeros and broken."""
    say("quantize narrow", k)
    for dt in (torch.float16, torch.bfloat16):
        x = normal(gen(k), 1003, k, dtype=torch.float32)
        gain = torch.tensor([1.0, 1e4, 1e-6, 0.0, 1.0, 1e-37])[torch.arange(1003) % 6]
        x = (x * gain[:, None]).to(dt)
        x[torch.arange(1003) % 11 == 5, k - 1] = NAN
        x[torch.arange(1003) % 13 == 7, 0] = INF
        same_rows(run_quantize(x), R.quantize(x))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quantize_ties(dtype):
    """Quotients on ties and next to them, over the type's whole range, zeros and broken rows."""
    say("quantize ties", dtype)
    dt = DT[dtype]
    # a scale that is a power of two: halves are ties; all values of the type around them
    halves = torch.arange(-254, 255).float() / 2
    rows = [halves, halves * 3, torch.nextafter(halves, halves + 1)]
    x = torch.zeros((12, 1024))
    for i, e in enumerate((-20, -14, -3, 0, 4, 6, 8) if dt == torch.float16
                          else (-126, -100, -62, -1, 0, 60, 110)):
        x[i, :509] = rows[0] * 2.0 ** e
    x[7, :509] = halves + halves.sign() / 64
    x[8, 3] = INF
    x[9, 5] = NAN
    x = x.to(dt)
    x[10] = torch.randint(-(1 << 15), 1 << 15, (1024,), generator=gen(41)).short().view(dt)
    x[10] = torch.where(torch.isfinite(x[10]), x[10], torch.zeros_like(x[10]))
    want = R.quantize(x)
    same_rows(run_quantize(x), want)
    same_rows(run_quantize(x[:, :1021].contiguous()), R.quantize(x[:, :1021]))
    assert want[1][11] == 0 and math.isnan(want[1][8]) and math.isnan(want[1][9])
    # every value of the type, against scales of all sizes
    every = torch.arange(-(1 << 15), 1 << 15).short().view(dt)
    every = every[torch.isfinite(every)]
    every = every[every.float().abs().argsort()]
    n = len(every) // 2048
    x = every[:n * 2048].view(n, 2048).contiguous()
    same_rows(run_quantize(x), R.quantize(x))
    x = every[:n * 2048].view(2048, n).t().contiguous()
    same_rows(run_quantize(x), R.quantize(x))


# ----------------------------------------------------------------------------- project_i8

PROJECT = [(1, 16, 1), (1, 64, 300), (7, 1024, 130), (8, 1024, 1536), (16, 80, 17), (17, 112, 129),
           (33, 512, 64), (64, 208, 96), (64, 4096, 33), (65, 144, 257), (129, 320, 200),
           (300, 192, 384), (513, 96, 515), (700, 1024, 1000), (2048, 128, 2048), (3000, 272, 1500),
           (5000, 64, 1111), (2500, 64, 4100), (2100, 144, 2100), (4352, 64, 4096), (6400, 64, 1536),
           (3500, 80, 2048), (1500, 96, 1000),
           # several tiles of 256 x 256 a workgroup, of 2, 3 and 4 steps
           (6300, 144, 4200), (6400, 272, 4096), (6350, 400, 4099), (13200, 144, 4096)]


def signed(g, *shape):
    return torch.randint(-128, 128, shape, generator=g).to(torch.int8)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,k,n", PROJECT)
def test_project_i8(tokens, k, n, dtype):
    say("project_i8", tokens, k, n, dtype)
    g = gen(tokens + k + n)
    x, w = signed(g, tokens, k), signed(g, n, k)
    xs, ws = (torch.rand(m, generator=g) * 0.02 / k ** 0.5 + 1e-3 for m in (tokens, n))
    want, bound = R.project_i8(x, xs, w, ws, DT[dtype])
    y = torch.full((tokens, n), NAN, dtype=DT[dtype], device="cuda")
    tg.project_i8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y)
    torch.cuda.synchronize()
    R_assert(y.cpu(), want, bound, "project_i8")


@pytest.mark.parametrize("tokens", [3, 40, 70, 300])
def test_project_i8_strides_and_borders(tokens):
    say("project_i8 strides", tokens)
    g, k, n = gen(51), 96, 133
    wx, ww = signed(g, tokens + 2, k + 48).cuda(), signed(g, n + 3, k + 16).cuda()
    x, w = wx[1:-1, 16:16 + k], ww[2:-1, :k]
    xs, ws = torch.rand(tokens, generator=g) * 1e-3, torch.rand(n, generator=g)
    out, whole = apart(torch.zeros((tokens, n)).bfloat16(), wide=7)
    tg.project_i8(x, xs.cuda(), w, ws.cuda(), out)
    torch.cuda.synchronize()
    want, bound = R.project_i8(x.cpu(), xs, w.cpu(), ws, torch.bfloat16)
    R_assert(out.cpu(), want, bound, "project_i8")
    assert untouched(out, whole)


@pytest.mark.parametrize("tokens", [2, 200])
def test_project_i8_longest(tokens):
    """Sums at the end of 32 bits; scales that are NaN or infinite stay their token's and output's."""
    say("project_i8 longest", tokens)
    k, n = tg.PROJECT_I8_MAX_K, 40
    x = torch.full((tokens, k), -128, dtype=torch.int8)
    x[1] = 127
    w = torch.full((n, k), -128, dtype=torch.int8)
    w[3] = 1
    xs, ws = torch.full((tokens,), 2.0 ** -20), torch.ones(n)
    want, bound = R.project_i8(x, xs, w, ws, torch.bfloat16)
    xs[0], ws[7] = NAN, INF
    y = torch.full((tokens, n), 3.0, dtype=torch.bfloat16, device="cuda")
    tg.project_i8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y)
    torch.cuda.synchronize()
    y = y.cpu()
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isinf(y[1:, 7]).all())
    fine = torch.arange(n) != 7
    R_assert(y[1:, fine], want[1:, fine], bound[1:, fine], "longest")


def test_quantized_rows_through_the_product():
    """A row with a NaN makes its own results NaN and no others."""
    say("quantize and project_i8")
    g = gen(52)
    x, w = normal(g, 90, 320, dtype=torch.bfloat16), normal(g, 70, 320, dtype=torch.bfloat16)
    x[5, 7] = NAN
    (q, s), (wq, ws) = run_quantize(x), run_quantize(w)
    y = torch.empty((90, 70), dtype=torch.bfloat16, device="cuda")
    tg.project_i8(q.cuda(), s.cuda(), wq.cuda(), ws.cuda(), y)
    torch.cuda.synchronize()
    fine = torch.arange(90) != 5
    assert bool(torch.isnan(y[5]).all())
    want, bound = R.project_i8(q[fine], s[fine], wq, ws, torch.bfloat16)
    R_assert(y.cpu()[fine], want, bound, "product")
    # and the rounding to integers: half a scale of each operand, for each of the products
    plain = x[fine].double() @ w.double().t()
    off = (s[fine].double()[:, None] / 2) * w.double().abs().sum(1) + (
        ws.double() / 2) * (x[fine].double().abs().sum(1)[:, None] + 320 * s[fine].double()[:, None] / 2)
    assert bool(((want - plain).abs() <= off).all())


# --------------------------------------------------------------- sizes, streams and graphs

def test_rows_past_32_bits():
    """Arrays of more than 2^31 values: the last rows are where they belong."""
    say("far rows")
    g, n, rows = gen(61), 32768, 70000
    x = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    some = normal(g, 3, n, dtype=torch.bfloat16)
    at = torch.tensor([0, rows // 2 + 3, rows - 1])
    x[at.cuda()] = some.cuda()
    h = torch.full_like(x, 3.0)
    tg.norm(x, None, h, norm=tg.NORM_RMS)
    _, (want, bound) = R.norm(some, kind=1)
    R_assert(h[at.cuda()].cpu(), want, bound, "norm")
    q = torch.full((rows, n), 7, dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    tg.quantize(x, q, s)
    wq, ws = R.quantize(some)
    assert torch.equal(q[at.cuda()].cpu(), wq) and torch.equal(s[at.cuda()].cpu(), ws)
    assert int(q[1].abs().max()) == 0 and int(q[rows - 2].abs().max()) == 0
    del x, h
    w, scale = signed(g, 40, n), torch.full((40,), 1e-3)
    y = torch.full((rows, 40), NAN, dtype=torch.bfloat16, device="cuda")
    tg.project_i8(q, s, w.cuda(), scale.cuda(), y)
    torch.cuda.synchronize()
    want, bound = R.project_i8(wq, ws, w, scale, torch.bfloat16)
    R_assert(y[at.cuda()].cpu(), want, bound, "project_i8")
    assert int((y != 0).any(1).sum()) == 3


@pytest.mark.parametrize("n", [8, 128, 256, 512, 1024, 2048, 4096, 8192, 16384, 32768])
def test_rows_past_the_caches(n):
    """Results that pass the caches are those of the same rows in calls that do not."""
    say("past the caches", n)
    rows, part = (96 << 20) // n + 1, (20 << 20) // n  # of 2^22 values or more, each
    g = torch.Generator("cuda").manual_seed(n)
    x, y = (torch.randn((rows, n), generator=g, device="cuda").bfloat16() for _ in range(2))
    xo, h = torch.full_like(x, NAN), torch.full_like(x, NAN)
    q = torch.full((rows, n), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -1.0, device="cuda")
    more = dict(y_norm=tg.NORM_LAYER, norm=tg.NORM_RMS)
    tg.norm(x, xo, h, y=y, **more)
    tg.quantize(x, q, s)
    for t in range(0, rows, part):
        xs, hs, qs, ss = (torch.empty_like(a[t:t + part]) for a in (xo, h, q, s))
        tg.norm(x[t:t + part], xs, hs, y=y[t:t + part], **more)
        tg.quantize(x[t:t + part], qs, ss)
        for got, want in ((xo, xs), (h, hs), (q, qs), (s, ss)):
            assert torch.equal(got[t:t + part], want)


def operators(seed):
    """A call of each operator as (outputs, function of a stream), on inputs of its own."""
    g, dt = gen(seed), torch.bfloat16
    x, y = normal(g, 70, 1024, dtype=dt).cuda(), normal(g, 70, 1024, dtype=dt).cuda()
    xo, h = torch.empty_like(x), torch.empty_like(x)
    q8, s8 = torch.empty((70, 1024), dtype=torch.int8, device="cuda"), torch.empty(70, device="cuda")
    w8, sw = signed(g, 300, 1024).cuda(), torch.rand(300, generator=g).cuda()
    y8 = torch.empty((70, 300), dtype=dt, device="cuda")
    lens, page = [3000, 5, 0, 640, 1777], 16
    k, v, table = cache(g, lens, page, 2, 64, dt)
    pages = tg.Pages(table.cuda(), ints(lens), page)
    q = normal(g, 5, 8, 64, dtype=dt).cuda()
    k, v, out = k.cuda(), v.cuda(), torch.empty_like(q)
    bufs = tg.AttendPagesBuffers(q, k, 3000)
    free = tg.Pages.empty(40, 300, 9000, 16)
    after = tg.Pages(free.table, torch.empty_like(free.kv_len), 16, free.free,
                     torch.empty_like(free.n_free))
    begin = torch.cat([torch.zeros(1), torch.randint(0, 400, (40,), generator=g).cumsum(0)]).int()
    rows = tg.PagesBuffers(free, int(begin[-1]))
    begin = begin.cuda()
    return [
        ([xo, h], lambda s: tg.norm(x, xo, h, y=y, y_norm=tg.NORM_LAYER, stream=s)),
        ([q8, s8], lambda s: tg.quantize(x, q8, s8, stream=s)),
        ([y8], lambda s: tg.project_i8(q8, s8, w8, sw, y8, stream=s)),
        ([out], lambda s: tg.attend_pages(q, k, v, pages, out, bufs, 0.1, stream=s)),
        ([rows.slot, rows.pos, rows.refused, after.kv_len, after.n_free],  # the table: in and out
         lambda s: tg.pages(free, begin, rows, after=after, stream=s))]


def test_other_device_is_refused(monkeypatch):
    """A call goes to the current device's stream: tensors of another are refused."""
    say("other device")
    x, p = torch.zeros((2, 64), device="cuda").half(), tg.Pages.empty(2, 3, 4, 16)
    q8, one = torch.zeros((2, 64), dtype=torch.int8, device="cuda"), torch.zeros(2, device="cuda")
    bufs, q = tg.PagesBuffers(p, 2), x.view(2, 1, 64)
    scratch = tg.AttendPagesBuffers(q, q, 40)
    begin = ints([0, 1, 2])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for make in (lambda: tg.norm_args(x, x), lambda: tg.quantize_args(x, q8, one),
                 lambda: tg.project_i8_args(q8, one, q8, one, x[:, :2]),
                 lambda: tg.pages_args(p, begin, bufs),
                 lambda: tg.attend_pages_args(q, q, q, p, q, scratch, 1.0)):
        with pytest.raises(ValueError, match="current device"):
            make()
    seen = []
    monkeypatch.setattr(tg, "_here", lambda *tensors: seen.extend(tensors))
    after = tg.Pages(p.table, p.kv_len.clone(), 16, p.free, p.n_free.clone())
    ends = ints([0, 1])
    tg.pages_args(p, begin, bufs, ends, after)
    for t in (p.table, p.kv_len, p.free, p.n_free, begin, ends, bufs.slot, bufs.pos, bufs.refused,
              bufs.workspace, after.kv_len, after.n_free):
        assert any(t is u for u in seen)


def test_streams():
    """Two sets of calls at once on two streams give what each gives alone on the current one."""
    say("streams")
    sets = [operators(71), operators(72)]
    want = []
    for calls in sets:
        for outs, call in calls:
            call(None)
        want.append([[t.clone() for t in outs] for outs, _ in calls])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for turn in range(4):
        for calls in sets:
            for outs, _ in calls:
                for t in outs:
                    t.zero_()
        torch.cuda.synchronize()
        for i in range(len(sets[0])):
            for calls, s in zip(sets, streams):
                calls[i][1](s)
        torch.cuda.synchronize()
        for calls, exp in zip(sets, want):
            for (outs, _), ref in zip(calls, exp):
                assert all(torch.equal(a, b) for a, b in zip(outs, ref))


def test_graphs():
    """Captured calls, replayed with eager work between, of two graphs that share workspaces."""
    say("graphs")
    calls = operators(73)
    want = []
    for outs, call in calls:
        call(None)
        want.append([t.clone() for t in outs])
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _, call in calls:
                call(None)
        graphs.append(graph)
    for turn in range(6):
        for outs, _ in calls:
            for t in outs:
                t.zero_()
        graphs[turn % 2].replay()
        if turn % 3 == 2:
            torch.cuda.synchronize()
            for _, call in calls:
                call(None)
        torch.cuda.synchronize()
        for (outs, _), ref in zip(calls, want):
            assert all(torch.equal(a, b) for a, b in zip(outs, ref))


def test_the_same_call_gives_the_same_bits():
    say("repeat")
    calls = operators(74)
    first = None
    for _ in range(5):
        for _, call in calls:
            call(None)
        torch.cuda.synchronize()
        got = [t.clone() for outs, _ in calls for t in outs]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))
