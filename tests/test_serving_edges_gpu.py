"""Serving operators where their other tests do not reach: the digits of attention weights."""
import pytest
import torch

from gpu_helpers import say
import serving_reference as R
from test_serving_gpu import DT, R_assert, cache, gen, normal, run_attend, widened
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
