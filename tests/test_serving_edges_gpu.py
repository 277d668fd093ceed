"""Serving operators where their other tests do not reach: the digits of attention weights,
lengths past every bound where keys are cut, and pages that are none on their way back to the
stack."""
import random

import pytest
import torch

from gpu_helpers import say
from paper_2404_09267_amd import tg
import serving_reference as R
from test_serving_gpu import DT, R_assert, cache, gen, ints, normal, run_attend, widened
from token_reference import UNIT

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------- attend_pages

def attend_bound(q, k, v, table, lens, page, **more):
    """(out, bound) with weights as a rounding to the type and, rounded as well, what that leaves:
    they are off by UNIT^2 of themselves (what is left is at most UNIT of a weight, and its rounding
    UNIT of that), which counts twice since their sum has it too. In binary16, what is left is a
    multiple of 2^-24, and the largest weight 2^7 or more: 2^-25 / 2^7 of it for each key."""
    want, bound = R.attend_pages(q, k, v, table, lens, page, **more)
    size, _ = R.attend_pages(q, k, v.abs(), table, lens, page, **more)  # what the weights act on
    u = UNIT[q.dtype]
    bound = bound - (u - 2 * u * u) * size
    if q.dtype == torch.float16:
        n = torch.tensor([float(max(m, 0)) for m in lens]).double()[:, None, None]
        most = torch.nan_to_num(v).abs().double().max()
        bound = bound + 2 * n * 2.0 ** -32 * most
    return want, bound


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens,page,heads,kv,d,extra", [
    ([2, 3, 5, 90], 16, 16, 2, 8, {}), ([40, 1, 333], 24, 7, 1, 64, dict(cap=3.0)),
    ([33, 900, 64, 0], 8, 40, 2, 128, dict(window=300)), ([2000, 17], 64, 4, 4, 72, dict(slope=True)),
    ([600] * 3, 16, 8, 4, 32, {}), ([1500, 31, 32], 128, 6, 2, 96, {})])
def test_attend_pages_keeps_the_weights_digits(lens, page, heads, kv, d, extra, dtype, most):
    """Where values of both signs cancel, a rounding of the weights is far more than one of the
    result."""
    say("attend_pages digits", lens, d, dtype, most)
    g, dt = gen(d + heads), DT[dtype]
    k, v, table = cache(g, lens, page, kv, d, dt)
    table = widened(table, page, most)
    q = normal(g, len(lens), heads, d, dtype=dt)
    more = dict(extra, scale=0.25 * d ** -0.5)
    if more.get("slope"):
        more["slope"] = torch.linspace(-0.002, 0.02, heads)
    want, bound = attend_bound(q, k, v, table, lens, page, **more)
    got = run_attend(q, k, v, table, lens, page, most, **more)
    R_assert(got, want, bound, "digits")


@pytest.mark.parametrize("most", [None, 20000])  # of the lengths; the larger has keys cut
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [1, 8, 9, 20])  # a weight's parts beside each other, or not
@pytest.mark.parametrize("even", [True, False])  # weights that are all 1, with nothing left, or not
def test_attend_pages_infinite_values(even, group, dtype, most):
    """An infinite value that has a weight is its column's result, whatever sign the weight's second
    part has, and NaN makes NaN; other columns do not see them."""
    say("attend_pages infinite", even, group, dtype, most)
    g, page, d, n, dt = gen(21), 16, 40, 170, DT[dtype]
    k, v, table = cache(g, [n], page, 1, d, dt)
    table = widened(table, page, most)
    q = normal(g, 1, group, d, dtype=dt, gain=0.0 if even else 1.0)
    row = lambda j: int(table[0, j // page]) * page + j % page
    want, bound = R.attend_pages(q, k, v, table, [n], page, 0.1)
    inf, nan = float("inf"), float("nan")
    for j, c, bad in ((3, 5, inf), (n - 1, 7, -inf), (77, 9, nan), (40, 11, inf), (41, 11, -inf)):
        v[row(j), 0, c] = bad
    got = run_attend(q, k, v, table, [n], page, most, scale=0.1)
    assert bool((got[0, :, 5] == inf).all()) and bool((got[0, :, 7] == -inf).all())
    assert bool(torch.isnan(got[0, :, [9, 11]]).all())
    fine = [c for c in range(d) if c not in (5, 7, 9, 11)]
    R_assert(got[:, :, fine], want[:, :, fine], bound[:, :, fine], "others")


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("max_kv", [5000, 20000, 1 << 30])
def test_attend_pages_lengths_past_the_bound(max_kv, window):
    """Lengths below 0 and up to 2^31 - 1 where keys are cut into ranges: the query stands at the
    last key that is claimed, and sees those that there are."""
    say("attend_pages lengths", max_kv, window)
    g, lens, page = gen(11), [700, 64, 0, 33], 16
    k, v, table = cache(g, lens, page, 2, 64, torch.bfloat16)
    table = widened(table, page, 20000)
    k, v = torch.nan_to_num(k, nan=0.5), torch.nan_to_num(v, nan=0.25)
    q = normal(g, 4, 8, 64, dtype=torch.bfloat16)
    claimed = [700, 64, -5, (1 << 31) - 1]
    got = run_attend(q, k, v, table, claimed, page, max_kv, scale=0.1, window=window)
    seen = 3 if window else 4
    want, bound = R.attend_pages(q[:seen], k, v, table[:seen], claimed[:seen], page, 0.1,
                                 window=window, max_kv=max_kv)
    R_assert(got[:seen], want, bound, "claimed")
    assert bool((got[seen:] == 0).all())  # the last 50 of what is claimed are not there


# --------------------------------------------------------------------------------- pages

def same(got, want, name):
    off = (got.cpu() != torch.tensor(want, dtype=got.dtype)).sum()
    assert int(off) == 0, f"{name}: {int(off)} differ"


def freed(table, lens, release, page, n_pages):
    """Pages that go back, in order: what is no page is left out."""
    back = [p for row, n, r in zip(table, lens, release) if r for p in row[:-(-n // page)]]
    return [p for p in back if 0 <= p < n_pages]


@pytest.mark.parametrize("seqs,cols", [(3, 3), (40, 100), (1500, 4), (2100, 2)])
def test_pages_that_are_none_do_not_go_back(seqs, cols):
    """A sequence that ends with entries that are no page gives back the others: nobody else is
    given what is none, and the count of free pages is of pages."""
    say("pages none", seqs, cols)
    r, page = random.Random(seqs), 4
    n_pages = seqs * cols
    order = list(range(n_pages))
    r.shuffle(order)
    lens = [r.randint(0, cols * page) for _ in range(seqs)]
    table = [[-1] * cols for _ in range(seqs)]
    for row, n in zip(table, lens):
        for i in range(-(-n // page)):
            row[i] = order.pop()
    release = [int(r.random() < 0.6) for _ in range(seqs)]
    release[0], lens[0] = 1, cols * page
    for row, ends in zip(table, release):
        for i in range(cols):
            if ends and r.random() < 0.2:
                row[i] = r.choice([-1, n_pages, -(1 << 31), (1 << 31) - 1])
    table[0][1] = n_pages
    free = order[:1]  # next to nothing but what goes back
    new = [r.choice([0, 1, 1, 2, page + 1]) for _ in range(seqs)]
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    stack = free + freed(table, lens, release, page, n_pages)
    want = R.pages(begin, [0 if e else n for e, n in zip(release, lens)], table, stack, len(stack),
                   page, n_pages, begin[-1])
    dev = tg.Pages(ints(table), ints(lens), page, ints(free + [-5] * (n_pages - len(free))),
                   ints([len(free)]))
    bufs = tg.PagesBuffers(dev, begin[-1])
    tg.pages(dev, ints(begin), bufs, release=ints(release))
    torch.cuda.synchronize()
    assert int(dev.n_free) == len(want["free"]) and int(bufs.refused) == want["refused"]
    same(dev.free[:len(want["free"])], want["free"], "free")
    same(dev.table, want["table"], "table")
    same(dev.kv_len, want["kv_len"], "kv_len")
    same(bufs.slot, want["slot"], "slot")
    same(bufs.pos[:, 0], want["pos"], "pos")


def test_pages_more_than_there_are_go_back():
    """Rows that name pages twice, and none among them: the stack holds as many as there are."""
    say("pages too many")
    table = [[i % 7 if i % 3 else 1 << 20 for i in range(s, s + 1200)] for s in range(5)]
    dev = tg.Pages(ints(table), ints([1200] * 5), 1, ints([3] * 2 + [-5] * 1998), ints([2]))
    bufs = tg.PagesBuffers(dev, 0)
    tg.pages(dev, ints([0] * 6), bufs, release=ints([1] * 5))
    torch.cuda.synchronize()
    assert int(dev.n_free) == 2000
    same(dev.free, ([3, 3] + freed(table, [1200] * 5, [1] * 5, 1, 2000))[:2000], "free")
