"""The token operators where sizes, masks and values are at their ends, against plain 64-bit
implementations: what the tests of single operators do not reach."""
import pytest
import torch

from gpu_helpers import say
from paper_2404_09267_amd import tg
from test_tokens_gpu import NAN, gen, normal
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
