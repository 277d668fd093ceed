"""Limits of the token operators that the host checks before any HIP work (no GPU)."""
import numpy as np
import pytest

from paper_2404_09267_amd import tg
from test_tokens import attend, project, rotate


def test_project_more_than_one_launch():
    """Refused before anything is enqueued: the rows of h go first."""
    assert project(n_tokens=(1 << 28) + 1, workspace_bytes=1 << 50) == tg.E_INVAL
    assert project(n_tokens=1 << 28, n=1 << 23, y_stride=1 << 23,
                   workspace_bytes=1 << 50) == tg.E_INVAL


def test_rotate_more_than_one_launch():
    assert rotate(n_tokens=(1 << 31) - 1, n_heads=1 << 10, d=66, rot=66) == tg.E_INVAL


@pytest.mark.parametrize("queries", [1, 40])
def test_attend_more_than_one_launch(queries):
    assert attend(n_seqs=(1 << 31) - 1, max_q_len=queries, max_kv_len=1,
                  n_q_rows=(1 << 31) - 1) == tg.E_INVAL


@pytest.mark.parametrize("none", [dict(q_doc=None), dict(k_doc=None), dict(q_pos=None)])
def test_attend_arrays_of_no_rows(none):
    """An array of no rows is null as often as not: there is nothing to do."""
    assert attend(n_q_rows=0, **none) == tg.OK
    assert attend(n_seqs=0, **none) == tg.OK


def less(rng, sizes):
    """Sizes of which none is larger."""
    return [int(rng.integers(1, n + 1)) if rng.random() < 0.7 else n for n in sizes]


def test_attend_workspace_of_the_largest_batch_does_for_smaller_ones():
    """Scratch is made once, for the largest batch; fewer sequences or queries may be cut into more
    parts, and take another form."""
    need = lambda sizes, heads: int(tg.lib().tg_attend_workspace_bytes(*sizes, *heads))
    assert need((191, 191, 1, 4000), (32, 8, 128)) <= need((192, 192, 1, 4000), (32, 8, 128))
    assert need((4, 64, 16, 4000), (32, 8, 128)) <= need((4, 68, 17, 4000), (32, 8, 128))
    rng = np.random.default_rng(0)
    for _ in range(20000):
        kv = int(rng.choice([1, 2, 3, 4, 8, 16, 71, 1600]))
        group, d = int(rng.choice([1, 2, 4, 7, 8, 16, 71])), int(rng.choice([8, 64, 72, 128]))
        heads = (kv * group, kv, d)
        most = [int(2 ** rng.uniform(0, top)) for top in (10, 16, 13, 18)]
        assert need(less(rng, most), heads) <= need(most, heads), (most, heads)


def test_project_workspace_of_the_most_tokens_does_for_fewer():
    """Fewer tokens may have more cuts of k, fewer adapters be laid out anew."""
    need = lambda *sizes: int(tg.lib().tg_project_workspace_bytes(*sizes))
    assert need(64, 4096, 4096, 0, 0) <= need(200, 4096, 4096, 0, 0)
    assert need(300, 64, 28001, 30, 17) <= need(300, 64, 28001, 40, 17)
    rng = np.random.default_rng(0)
    for _ in range(20000):
        k, n = 8 * int(2 ** rng.uniform(0, 10)), int(2 ** rng.uniform(0, 17))
        rank = int(rng.integers(1, 65))
        tokens, adapters = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 7))
        t, g = less(rng, (tokens, adapters))
        assert need(t, k, n, g, rank) <= need(tokens, k, n, adapters, rank)
        assert need(t, k, n, 0, 0) <= need(tokens, k, n, 0, 0) <= need(tokens, k, n, adapters, rank)
