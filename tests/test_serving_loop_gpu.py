"""The example that runs the serving operators together: requests over one paged cache."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location(
        "serving_loop", os.path.join(ROOT, "examples", "serving_loop.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_requests_come_out_as_if_alone():
    """Who else is served does not change a request's results. Attention over a prompt may sum in
    another order: a rounding of its result to bfloat16 (2^-8) may fall the other way, and with it
    an 8-bit integer of the row (a step of 1 / 127 of its largest, 2^-7), in each of two layers; a
    row or a page of another request changes whole values."""
    assert load().main() <= 2 * (2.0 ** -8 + 2.0 ** -7)


def test_replayed_steps_are_the_eager_ones():
    """The same requests in the same order, single tokens replayed from a graph or not: the same
    bits, and every page is free in the end."""
    example = load()
    servers = [example.Server(places=5, n_pages=40, seed=3) for _ in range(2)]
    todo = example.requests(9, 6, servers[0].width, 3)
    replayed, eager = (example.serve(s, todo, replay=r) for s, r in zip(servers, (True, False)))
    assert all(torch.equal(a, b) for a, b in zip(replayed, eager))
    assert int(servers[0].pages.n_free) == 40
    assert sorted(servers[0].pages.free.tolist()) == list(range(40))


def test_two_graphs_share_a_cache():
    """Steps of one token and steps of none, captured apart over the same pages and replayed in turn
    with eager ones between, give what eager steps give."""
    example = load()
    servers = [example.Server(places=3, n_pages=30, seed=4) for _ in range(2)]
    todo = example.requests(3, 6, servers[0].width, 5)
    for s in servers:
        s.step([list(t[1]) for t in todo], [t[0] for t in todo], set(), replay=False)
    first = servers[0]
    first.capture()
    one = (first.graph, first.x, first.camera, first.begin, first.release, first.y)
    first.capture()
    two = (first.graph, first.x, first.camera, first.begin, first.release, first.y)
    for turn in range(9):
        tokens = [[t[2][turn % len(t[2])]] if (turn + p) % 4 else None for p, t in enumerate(todo)]
        if turn % 3 < 2:
            (first.graph, first.x, first.camera, first.begin, first.release,
             first.y) = (one, two)[turn % 3]
        got = first.step(tokens, [t[0] for t in todo], set(), replay=turn % 3 < 2)
        want = servers[1].step(tokens, [t[0] for t in todo], set(), replay=False)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("replay", [True, False])
def test_a_full_cache_is_said(replay):
    """A token that finds no page raises, in a replayed step as in an eager one; those who found
    theirs have moved on, and it goes on once somebody has ended."""
    example = load()
    server = example.Server(places=3, n_pages=3, page=16, most=64, seed=6)
    row = lambda: torch.ones(server.width, dtype=example.DTYPE, device="cuda")
    prompt = lambda n: [row() for _ in range(n)]
    server.step([prompt(15), prompt(16), prompt(9)], [0, 1, 2], set())
    server.step([[row()], None, None], [0, 1, 2], set(), replay)
    for _ in range(2):
        with pytest.raises(RuntimeError, match="cache is full"):
            server.step([None, [row()], [row()]], [0, 1, 2], set(), replay)
    assert server.pages.kv_len.tolist() == [16, 16, 11]
    server.step([None, [row()], None], [0, 1, 2], {0}, replay)
    assert server.pages.kv_len.tolist() == [0, 17, 11]
    assert int(server.pages.n_free) == 0
