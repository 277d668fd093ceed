"""What the token operators refuse, before any HIP work (no GPU), and what the 64-bit
references of the tests give in cases that can be worked by hand."""
import ctypes
import math

import pytest
import torch

from paper_2404_09267_amd import tg
import token_reference as R

P = 1 << 20  # a pointer that is never followed: every call below is refused


def project(**change):
    a = tg.ProjectArgs(x=P, x_stride=64, w=P, w_stride=64, adapter=P, a=P, b=P, scale=P, y=P,
                       y_stride=32, n_tokens=4, k=64, n=32, n_adapters=2, rank=8, type=tg.F16,
                       workspace=P, workspace_bytes=1 << 20)
    for n, v in change.items():
        setattr(a, n, v)
    return int(tg.lib().tg_project(ctypes.byref(a), None))


def rotate(**change):
    a = tg.RotateArgs(q=P, k=P, v=P, q_stride=64, q_head_stride=64, k_stride=64, k_head_stride=64,
                      v_stride=64, v_head_stride=64, q_weight=P, k_weight=P, table=P, pos=P,
                      q_out=P, k_out=P, v_out=P, q_out_stride=64, q_out_head_stride=64,
                      k_out_stride=64, k_out_head_stride=64, v_out_stride=64,
                      v_out_head_stride=64, slot=P, n_rows=9, eps=1e-6, n_tokens=4, n_heads=1,
                      n_kv_heads=1, d=64, rot=64, axes=1, interleaved=0, n_positions=10,
                      type=tg.BF16)
    for n, v in change.items():
        setattr(a, n, v)
    return int(tg.lib().tg_rotate(ctypes.byref(a), None))


def attend(**change):
    a = tg.AttendArgs(q=P, k=P, v=P, q_stride=64, q_head_stride=64, k_stride=64, k_head_stride=64,
                      v_stride=64, v_head_stride=64, out=P, out_stride=64, out_head_stride=64,
                      q_begin=P, kv_begin=P, kv_len=P, prefix=None, q_doc=P, k_doc=P, q_pos=P,
                      k_pos=P, slope=P, scale=0.1, cap=0.0, causal=1, n_seqs=2, n_q_rows=2,
                      n_k_rows=100, max_q_len=1, max_kv_len=4000, n_heads=4, n_kv_heads=2, d=64,
                      type=tg.F16, workspace=P, workspace_bytes=1 << 30)
    for n, v in change.items():
        setattr(a, n, v)
    return int(tg.lib().tg_attend(ctypes.byref(a), None))


@pytest.mark.parametrize("change", [
    dict(n_tokens=-1), dict(k=0), dict(k=60), dict(n=0), dict(n_adapters=-1), dict(type=2),
    dict(x_stride=56), dict(x_stride=65), dict(w_stride=56), dict(w_stride=68), dict(y_stride=31),
    dict(x_stride=1 << 23), dict(w_stride=1 << 23), dict(rank=0), dict(rank=65), dict(x=None),
    dict(w=None), dict(y=None), dict(x=P + 8), dict(w=P + 2), dict(a=P + 8), dict(a=None),
    dict(b=None), dict(scale=None)])
def test_project_refuses(change):
    assert project(**change) == tg.E_INVAL


def test_project_workspace():
    need = int(tg.lib().tg_project_workspace_bytes(4, 64, 32, 2, 8))
    assert need > 0
    assert project(workspace=None) == tg.E_WORKSPACE
    assert project(workspace=P + 8) == tg.E_WORKSPACE
    assert project(workspace_bytes=need - 1) == tg.E_WORKSPACE
    assert project(n_tokens=0) == tg.OK
    for bad in ((0, 64, 32, 2, 8), (4, 0, 32, 2, 8), (4, 64, 0, 2, 8), (4, 64, 32, 0, 8),
                (4, 64, 32, 2, 0), (-1, 64, 32, 2, 8)):
        assert int(tg.lib().tg_project_workspace_bytes(*bad)) == 0


@pytest.mark.parametrize("change", [
    dict(n_tokens=-1), dict(n_heads=-1), dict(n_kv_heads=-1), dict(type=-1), dict(d=0),
    dict(d=63, rot=2), dict(d=514), dict(rot=66), dict(rot=3), dict(rot=-2), dict(axes=0),
    dict(axes=3), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(n_positions=0),
    dict(n_rows=-1), dict(v=None), dict(v_out=None), dict(q=None), dict(k=None), dict(q_out=None),
    dict(k_out=None), dict(table=None), dict(pos=None)])
def test_rotate_refuses(change):
    assert rotate(**change) == tg.E_INVAL


def test_rotate_nothing():
    assert rotate(n_tokens=0) == tg.OK
    assert rotate(n_heads=0, n_kv_heads=0) == tg.OK


@pytest.mark.parametrize("change", [
    dict(n_seqs=-1), dict(n_q_rows=-1), dict(n_k_rows=-1), dict(max_q_len=-1),
    dict(max_kv_len=-1), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=3), dict(d=0),
    dict(d=4), dict(d=60), dict(d=136), dict(type=5), dict(scale=math.nan), dict(scale=math.inf),
    dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf), dict(q_doc=None), dict(k_doc=None),
    dict(q_pos=None), dict(k_pos=None), dict(prefix=P, causal=0), dict(q=None), dict(k=None),
    dict(v=None), dict(out=None), dict(q_begin=None), dict(kv_begin=None), dict(kv_len=None),
    dict(q=P + 2), dict(k=P + 8), dict(v=P + 4), dict(out=P + 8), dict(q_stride=60),
    dict(k_stride=-64), dict(v_stride=1 << 23), dict(k_head_stride=4), dict(out_head_stride=-8)])
def test_attend_refuses(change):
    assert attend(**change) == tg.E_INVAL


def test_attend_workspace():
    args = (2, 2, 1, 4000, 4, 2, 64)
    need = int(tg.lib().tg_attend_workspace_bytes(*args))
    assert need > 0
    assert attend(workspace=None) == tg.E_WORKSPACE
    assert attend(workspace=P + 4) == tg.E_WORKSPACE
    assert attend(workspace_bytes=need - 1) == tg.E_WORKSPACE
    assert attend(n_seqs=0) == tg.OK
    assert attend(n_q_rows=0) == tg.OK
    assert attend(max_q_len=0) == tg.OK
    assert int(tg.lib().tg_attend_workspace_bytes(2, 2, 1, 4000, 4, 3, 64)) == 0
    assert int(tg.lib().tg_attend_workspace_bytes(2, 0, 1, 4000, 4, 2, 64)) == 0


def test_null_arguments():
    L = tg.lib()
    for call in (L.tg_project, L.tg_rotate, L.tg_attend):
        assert int(call(None, None)) == tg.E_INVAL


def test_host_tensors_are_refused():
    x = torch.zeros((2, 64), dtype=torch.float16)
    with pytest.raises(ValueError, match="device tensor"):
        tg.project_args(x, x, None)
    q = torch.zeros((2, 1, 64), dtype=torch.float32)
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        tg.rotate_args(q, q, None, None, None, None, q, q)
    with pytest.raises(ValueError, match="device tensor"):
        tg.attend_args(q.half(), q.half(), q.half(), None, None, None, 1.0)


# the references, in cases worked by hand

def test_reference_project():
    x = torch.tensor([[1.0, 2.0], [3.0, -1.0]]).bfloat16()
    w = torch.tensor([[1.0, 1.0], [0.0, 2.0]]).bfloat16()
    a, b = torch.tensor([[[1.0, -1.0]]]).bfloat16(), torch.tensor([[[2.0], [4.0]]]).bfloat16()
    y, _ = R.project(x, w, a, b, torch.tensor([0.5]), torch.tensor([-1, 0]))
    # token 1: (2, -2) and h = 4: + 0.5 * 4 * (2, 4)
    assert y.tolist() == [[3.0, 4.0], [6.0, 6.0]]


def test_reference_rotate():
    v = torch.tensor([[[3.0, 4.0, 0.0, 0.0]]]).half()  # rms 2.5
    table = torch.tensor([[[0.0, 1.0]], [[1.0, 0.0]]])  # position 0: a quarter turn
    out, _ = R.rotate(v, None, table, torch.tensor([[0]]), 0.0, False)
    assert torch.allclose(out, torch.tensor([[[-1.6, 1.2, 0.0, 0.0]]], dtype=torch.float64))
    out, _ = R.rotate(v, None, table, torch.tensor([[7]]), 0.0, False)  # as the last position
    assert torch.allclose(out, torch.tensor([[[1.2, 1.6, 0.0, 0.0]]], dtype=torch.float64))


def test_reference_attend():
    q = torch.ones((2, 1, 8)).half()
    k = torch.zeros((3, 1, 8)).half()
    k[1] = math.log(3.0)  # score log 27 at scale 3 / 8
    v = torch.arange(3.0)[:, None, None].expand(3, 1, 8).half()
    out, _ = R.attend(q, k, v, [0, 2], [0], [3], 0.0)
    assert torch.allclose(out, torch.ones_like(out))  # equal weights
    out, _ = R.attend(q, k, v, [0, 2], [0], [3], 0.0, causal=True)
    assert torch.allclose(out[:, 0, 0], torch.tensor([0.5, 1.0], dtype=torch.float64))
    out, _ = R.attend(q, k, v, [0, 2], [0], [3], 0.0, q_doc=torch.tensor([1, -1]),
                      k_doc=torch.tensor([1, 0, 1]))
    assert torch.allclose(out[:, 0, 0], torch.tensor([1.0, 0.0], dtype=torch.float64))
    # bias by distance: the first query stands at key 1, weights 1/2, 1, 1/2
    out, _ = R.attend(q, k, v, [0, 2], [0], [3], 0.0, slope=torch.tensor([math.log(2.0)]))
    assert torch.allclose(out[0, 0], torch.ones(8, dtype=torch.float64), atol=1e-6)
    out, _ = R.attend(q, k, v, [0, 2], [0], [3], 3.0 / 8, causal=True)
    w = float(torch.exp(3.0 / 8 * (q[0, 0].double() @ k[1, 0].double())))
    assert abs(float(out[0, 0, 0]) - w / (1 + w)) < 1e-12
