"""What the serving operators refuse, before any HIP work (no GPU), and what the references of the
tests give in cases that can be worked by hand."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2404_09267_amd import tg
import serving_reference as R

P = 1 << 20  # a pointer that is never followed: every call below is refused
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def call(entry, a, change):
    for n, v in change.items():
        setattr(a, n, v)
    return int(getattr(tg.lib(), entry)(ctypes.byref(a), None))


def pages(**change):
    a = tg.PagesArgs(q_begin=P, kv_len=P, kv_len_out=P, release=P, table=P, table_stride=9,
                     free_pages=P, n_free=P, n_free_out=P, slot=P, pos=P, refused=P, n_seqs=4,
                     n_tokens=9000, n_pages=100, page_size=16, max_pages=9, workspace=P,
                     workspace_bytes=1 << 20)
    return call("tg_pages", a, change)


def attend(**change):
    a = tg.AttendPagesArgs(q=P, k=P, v=P, q_stride=256, q_head_stride=64, k_stride=128,
                           k_head_stride=64, v_stride=128, v_head_stride=64, out=P,
                           out_stride=256, out_head_stride=64, table=P, table_stride=99, kv_len=P,
                           slope=P, scale=0.1, cap=0.0, window=0, n_seqs=2, n_pages=200,
                           page_size=16, max_pages=99, max_kv_len=1500, n_heads=4, n_kv_heads=2,
                           d=64, type=tg.F16, workspace=P, workspace_bytes=1 << 30)
    return call("tg_attend_pages", a, change)


def norm(**change):
    a = tg.NormArgs(x=P, x_stride=64, y=P, y_stride=64, y_norm=1, y_weight=P, y_bias=P, gate=P,
                    gate_stride=64, gate_row=P, x_scale=1.0, y_scale=1.0, x_out=P,
                    x_out_stride=64, h=P, h_stride=64, norm=2, weight=P, bias=P, eps=1e-6,
                    n_tokens=3, n=64, n_gates=2, type=tg.BF16)
    return call("tg_norm", a, change)


def quantize(**change):
    a = tg.QuantizeArgs(x=P, x_stride=64, q=P, q_stride=64, scale=P, n_rows=3, k=64, type=tg.F16)
    return call("tg_quantize", a, change)


def project(**change):
    a = tg.ProjectI8Args(x=P, x_stride=64, x_scale=P, w=P, w_stride=64, w_scale=P, y=P,
                         y_stride=32, n_tokens=3, k=64, n=32, type=tg.BF16)
    return call("tg_project_i8", a, change)


@pytest.mark.parametrize("change", [
    dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(n_tokens=-1), dict(n_pages=-1),
    dict(page_size=0), dict(max_pages=0), dict(table_stride=8), dict(table_stride=-9),
    dict(max_pages=(1 << 20) + 1, table_stride=1 << 21),
    dict(n_pages=1 << 20, page_size=1 << 11), dict(q_begin=None), dict(kv_len=None),
    dict(kv_len_out=None), dict(table=None), dict(free_pages=None), dict(n_free=None),
    dict(n_free_out=None), dict(slot=None), dict(refused=None)])
def test_pages_refuses(change):
    assert pages(**change) == tg.E_INVAL


def test_pages_workspace():
    need = int(tg.lib().tg_pages_workspace_bytes(4, 9000))
    assert need > 0
    assert pages(workspace=None) == tg.E_WORKSPACE
    assert pages(workspace=P + 8) == tg.E_WORKSPACE
    assert pages(workspace_bytes=need - 1) == tg.E_WORKSPACE
    assert pages(n_seqs=0, n_tokens=0) == tg.OK
    most = [int(tg.lib().tg_pages_workspace_bytes(s, t)) for s in (1, 7, 500, 1 << 20)
            for t in (9000, 1 << 20)]
    assert most == sorted(most)
    for bad in ((0, 9000), (-1, 9000), (4, -1), ((1 << 20) + 1, 9000)):
        assert int(tg.lib().tg_pages_workspace_bytes(*bad)) == 0


@pytest.mark.parametrize("change", [
    dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(n_pages=-1), dict(page_size=0),
    dict(max_pages=0), dict(table_stride=98), dict(n_pages=1 << 20, page_size=1 << 11),
    dict(max_kv_len=-1), dict(max_kv_len=(1 << 30) + 1), dict(window=-1), dict(n_heads=0),
    dict(n_kv_heads=0), dict(n_heads=3), dict(d=0), dict(d=4), dict(d=60), dict(d=136),
    dict(type=2), dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0),
    dict(cap=math.nan), dict(cap=math.inf), dict(q=None), dict(k=None), dict(v=None),
    dict(out=None), dict(table=None), dict(kv_len=None), dict(q=P + 2), dict(k=P + 8),
    dict(v=P + 4), dict(out=P + 8), dict(q_stride=60), dict(k_stride=-64),
    dict(v_stride=1 << 23), dict(k_head_stride=4), dict(out_head_stride=-8)])
def test_attend_pages_refuses(change):
    assert attend(**change) == tg.E_INVAL


def test_attend_pages_workspace():
    need = int(tg.lib().tg_attend_pages_workspace_bytes(2, 1500, 4, 2, 64))
    assert need > 0
    assert attend(workspace=None) == tg.E_WORKSPACE
    assert attend(workspace=P + 4) == tg.E_WORKSPACE
    assert attend(workspace_bytes=need - 1) == tg.E_WORKSPACE
    assert attend(n_seqs=0) == tg.OK
    assert attend(q_begin=P, n_q_rows=0) == tg.OK
    assert attend(q_begin=P, n_q_rows=-1) == tg.E_INVAL
    for heads, kv, d in ((4, 2, 64), (16, 16, 128), (40, 1, 80), (4000, 2000, 8)):
        last = 0
        for seqs in (1, 2, 60, 400, 1024, 1025, 9000, 1 << 20):
            row = [int(tg.lib().tg_attend_pages_workspace_bytes(seqs, n, heads, kv, d))
                   for n in (0, 1, 512, 513, 1025, 5000, 1 << 30)]
            assert row == sorted(row) and row[-1] >= last
            last = row[-1]
    for bad in ((0, 1500, 4, 2, 64), (-1, 1500, 4, 2, 64), (2, -1, 4, 2, 64), (2, 1500, 4, 3, 64),
                (2, 1500, 4, 2, 60)):
        assert int(tg.lib().tg_attend_pages_workspace_bytes(*bad)) == 0


@pytest.mark.parametrize("change", [
    dict(n_tokens=-1), dict(n=0), dict(n=32769, x_stride=1 << 16), dict(n_gates=-1),
    dict(n_gates=0), dict(type=2), dict(y_norm=3), dict(norm=-1), dict(eps=-1.0),
    dict(eps=math.nan), dict(eps=math.inf), dict(x_scale=math.nan), dict(y_scale=math.inf),
    dict(y=None), dict(gate=None), dict(x=None), dict(x_out=None, h=None), dict(x_stride=63),
    dict(y_stride=63), dict(gate_stride=1), dict(x_out_stride=0), dict(h_stride=-64)])
def test_norm_refuses(change):
    assert norm(**change) == tg.E_INVAL


@pytest.mark.parametrize("change", [
    dict(n_rows=-1), dict(k=0), dict(type=-1), dict(x_stride=63), dict(q_stride=63), dict(x=None),
    dict(q=None), dict(scale=None)])
def test_quantize_refuses(change):
    assert quantize(**change) == tg.E_INVAL


@pytest.mark.parametrize("change", [
    dict(n_tokens=-1), dict(n_tokens=(1 << 30) + 1), dict(n=0), dict(n=(1 << 30) + 1), dict(k=0),
    dict(k=8), dict(k=72, x_stride=80, w_stride=80),
    dict(k=131072, x_stride=1 << 18, w_stride=1 << 18), dict(type=2), dict(x_stride=48),
    dict(w_stride=56), dict(x_stride=72), dict(w_stride=1 << 23), dict(y_stride=31), dict(x=None),
    dict(w=None), dict(y=None), dict(x_scale=None), dict(w_scale=None), dict(x=P + 8),
    dict(w=P + 4)])
def test_project_i8_refuses(change):
    assert project(**change) == tg.E_INVAL


def test_more_than_a_launch_holds():
    """Sizes within every other limit that no grid holds; no card holds their arrays either."""
    most = (1 << 31) - 1
    assert attend(n_seqs=1 << 20, n_heads=2048, n_kv_heads=2048, max_kv_len=500) == tg.E_INVAL
    assert norm(n_tokens=most, n=1100, x_stride=1100, y_stride=1100, gate_stride=1100,
                x_out_stride=1100, h_stride=1100) == tg.E_INVAL
    assert quantize(n_rows=most, k=1100, x_stride=1100, q_stride=1100) == tg.E_INVAL
    assert quantize(n_rows=most, k=40000, x_stride=40000, q_stride=40000) == tg.E_INVAL
    for tokens, n in ((1 << 30, 1 << 10), (1 << 20, 1 << 20), (300, 1 << 30), (1 << 30, 400)):
        assert project(n_tokens=tokens, n=n, y_stride=n) == tg.E_INVAL, (tokens, n)


def test_nothing():
    assert norm(n_tokens=0) == quantize(n_rows=0) == project(n_tokens=0) == tg.OK
    L = tg.lib()
    for entry in (L.tg_pages, L.tg_attend_pages, L.tg_norm, L.tg_quantize, L.tg_project_i8):
        assert int(entry(None, None)) == tg.E_INVAL


def test_host_tensors_are_refused():
    x = torch.zeros((2, 64), dtype=torch.float16)
    q = x.to(torch.int8)
    table, lens = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for make in (lambda: tg.Pages(table, lens, 16), lambda: tg.norm_args(x, x),
                 lambda: tg.quantize_args(x, q, torch.zeros(2)),
                 lambda: tg.project_i8_args(q, lens.float(), q, lens.float(), x)):
        with pytest.raises(ValueError, match="device tensor"):
            make()
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        tg.norm_args(x.float(), x)


STRUCTS = {"tg_pages_args": tg.PagesArgs, "tg_attend_pages_args": tg.AttendPagesArgs,
           "tg_norm_args": tg.NormArgs, "tg_quantize_args": tg.QuantizeArgs,
           "tg_project_i8_args": tg.ProjectI8Args}


def test_struct_layout_matches_header(tmp_path):
    lines = []
    for name, struct in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in struct._fields_]
    lines += [f'printf("{n} %d\\n", {n});' for n in ("TG_PAGES_MAX_SEQS", "TG_NORM_MAX_N",
                                                    "TG_PROJECT_I8_MAX_K", "TG_NORM_LAYER")]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tg.h"\nint main(void) {\n'
                   + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe],
                   check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    c = {k: int(v) for k, v in (line.split() for line in out.splitlines())}
    for name, struct in STRUCTS.items():
        assert c[name] == ctypes.sizeof(struct), name
        for f, _ in struct._fields_:
            assert c[f"{name}.{f}"] == getattr(struct, f).offset, f
    assert c["TG_PAGES_MAX_SEQS"] == tg.PAGES_MAX_SEQS and c["TG_NORM_MAX_N"] == tg.NORM_MAX_N
    assert c["TG_PROJECT_I8_MAX_K"] == tg.PROJECT_I8_MAX_K
    assert c["TG_NORM_LAYER"] == tg.NORM_LAYER


# the references, in cases worked by hand

def test_reference_pages():
    # pages of 4: the first ends inside its page, the second takes one, the third starts anew
    # with what it gave back on top of the stack, the last asks for more than is left
    got = R.pages([0, 1, 2, 7, 19], [2, 4, 5, 0], [[3, -1, -1], [5, -1, -1], [1, 2, -1],
                                                  [-1, -1, -1]], [0, 4, 6], 3, 4, 7, 20,
                  [0, 0, 1, 0])
    assert got["kv_len"] == [3, 5, 5, 0]
    assert got["table"] == [[3, -1, -1], [5, 2, -1], [1, 6, -1], [-1, -1, -1]]
    assert got["free"] == [0, 4] and got["refused"] == 1
    assert got["slot"][:7] == [14, 8, 4, 5, 6, 7, 24] and set(got["slot"][7:]) == {-1}
    assert got["pos"] == [2, 4, 0, 1, 2, 3, 4] + [0] * 13


def test_reference_attend_pages():
    q = torch.ones((2, 1, 8)).half()
    v = torch.arange(8.0)[:, None, None].expand(8, 1, 8).half()
    k = torch.zeros((8, 1, 8)).half()
    table = torch.tensor([[3, 0, 9], [1, -1, 2]])
    out, _ = R.attend_pages(q, k, v, table, [3, 0], 2, 1.0)
    # keys are rows 6, 7 and 0
    assert torch.allclose(out[0], torch.full((1, 8), 13 / 3, dtype=torch.float64))
    assert bool((out[1] == 0).all())
    out, _ = R.attend_pages(q, k, v, table, [6, 6], 2, 1.0)  # pages 9 and -1 are none
    assert torch.allclose(out[:, 0, 0], torch.tensor([3.5, 3.5], dtype=torch.float64))
    out, _ = R.attend_pages(q, k, v, table, [3, 4], 2, 1.0, window=2)
    assert torch.allclose(out[:, 0, 0], torch.tensor([3.5, 0.0], dtype=torch.float64))
    out, _ = R.attend_pages(q, k, v, table, [3, 1], 2, 1.0, slope=torch.tensor([math.log(2.0)]))
    assert torch.allclose(out[:, 0, 0], torch.tensor([(6 + 14 + 0) / 7, 2.0], dtype=torch.float64))


def test_reference_norm():
    x = torch.tensor([[3.0, 4.0, 0.0, 0.0]]).half()
    (r, _), (h, _) = R.norm(x, kind=R.RMS, eps=0.0)  # rms 2.5
    assert r.tolist() == [[3.0, 4.0, 0.0, 0.0]]
    assert torch.allclose(h, torch.tensor([[1.2, 1.6, 0.0, 0.0]], dtype=torch.float64))
    y = torch.tensor([[1.0, 3.0, 1.0, 3.0]]).half()  # mean 2, differences of 1
    gate = torch.tensor([[9.0] * 4, [2.0] * 4]).half()
    (r, _), _ = R.norm(x, y, R.LAYER, None, x[0], gate, torch.tensor([1]), 1.0, 0.5, eps=0.0)
    assert r.tolist() == [[3 + 2.0, 4 + 5.0, -1.0, 1.0]]
    (r, _), _ = R.norm(x, y, R.LAYER, None, x[0], gate, torch.tensor([2]), 2.0, 0.5, eps=0.0)
    assert r.tolist() == [[6.0, 8.0, 0.0, 0.0]]


def test_reference_quantize():
    q, scale = R.quantize(torch.tensor([[127.0, -0.5, 1.5, 2.5], [0, 0, 0, 0],
                                        [math.inf, 1, 2, 3], [254.0, 3.0, -254.0, 1.0]]).half())
    assert q.tolist() == [[127, 0, 2, 2], [0] * 4, [0] * 4, [127, 2, -127, 0]]
    assert scale[0] == 1 and scale[1] == 0 and math.isnan(scale[2]) and scale[3] == 2


def test_reference_project_i8():
    x, w = torch.tensor([[1, -2], [127, 127]]).char(), torch.tensor([[3, 4], [-128, 127]]).char()
    y, _ = R.project_i8(x, torch.tensor([1.0, 0.5]), w, torch.tensor([2.0, 1.0]), torch.half)
    assert y.tolist() == [[-10.0, -382.0], [889.0, -63.5]]
