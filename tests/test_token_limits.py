"""Limits of the token operators that the host checks before any HIP work (no GPU)."""
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
