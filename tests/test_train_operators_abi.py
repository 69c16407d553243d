"""CPU checks of the training operators' argument checks: every refusal comes
before any device work (there is no device here), on addresses that are never
read."""
import ctypes
import math

import pytest
import torch

from paper_2609_15160_amd import tlf, train

P, ODD = 0x1000, 0x1008  # a 16-byte and an 8-byte aligned address
BAD, UNS, F32, BF16 = tlf.E_INVALID_ARG, tlf.E_UNSUPPORTED, tlf.DTYPE_F32, tlf.DTYPE_BF16


@pytest.fixture(scope="module")
def lib():
    return tlf.load()


def _norm(lib, **kw):
    a = dict(x=P, xt=F32, gamma=P, group=P, groups=2, rows=3, d=8, eps=1e-5, y=P, yt=BF16, rstd=P)
    a.update(kw)
    return lib.tlf_rms_norm(a["x"], a["xt"], a["gamma"], a["group"], a["groups"], a["rows"], a["d"], a["eps"], a["y"],
                            a["yt"], a["rstd"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), BAD), (dict(y=None), BAD), (dict(x=ODD), BAD), (dict(y=ODD), BAD), (dict(gamma=ODD), BAD),
    (dict(xt=2), BAD), (dict(yt=-1), BAD), (dict(rows=-1), BAD), (dict(d=0), BAD), (dict(d=6), BAD),
    (dict(eps=0.0), BAD), (dict(eps=math.nan), BAD), (dict(groups=-1), BAD), (dict(groups=0), BAD),
    (dict(gamma=None), BAD), (dict(group=None), BAD), (dict(d=4100), UNS), (dict(groups=17), UNS),
])
def test_rms_norm_refusals(lib, kw, status):
    assert _norm(lib, **kw) == status


def test_rms_norm_without_rows_needs_no_device(lib):
    assert _norm(lib, rows=0, x=None, y=None) == tlf.OK


def _norm_grad(lib, **kw):
    a = dict(dy=P, yt=F32, x=P, xt=F32, gamma=P, group=P, groups=2, rstd=P, rows=3, d=8, dx=P, dgamma=P, ws=P, n=1 << 20)
    a.update(kw)
    return lib.tlf_rms_norm_grad(a["dy"], a["yt"], a["x"], a["xt"], a["gamma"], a["group"], a["groups"], a["rstd"],
                                 a["rows"], a["d"], a["dx"], a["dgamma"], a["ws"], a["n"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), BAD), (dict(x=None), BAD), (dict(rstd=None), BAD), (dict(group=None), BAD), (dict(dy=ODD), BAD),
    (dict(dx=ODD), BAD), (dict(dgamma=ODD), BAD), (dict(ws=None), BAD), (dict(ws=ODD), BAD), (dict(n=63), BAD),
    (dict(groups=0, gamma=None), BAD), (dict(gamma=None), BAD), (dict(d=10), BAD), (dict(yt=9), BAD), (dict(rows=-2), BAD),
    (dict(d=8192), UNS), (dict(groups=33), UNS),
])
def test_rms_norm_grad_refusals(lib, kw, status):
    assert _norm_grad(lib, **kw) == status


def test_rms_norm_grad_of_nothing(lib):
    assert _norm_grad(lib, dx=None, dgamma=None, dy=None) == tlf.OK


def _ffn(lib, **kw):
    a = dict(x=P, wgu=P, wd=P, t=BF16, rows=5, d=64, f=128, gu=P, a=P, y=P, ws=P, n=1 << 30)
    a.update(kw)
    return lib.tlf_ffn(a["x"], a["wgu"], a["wd"], a["t"], a["rows"], a["d"], a["f"], a["gu"], a["a"], a["y"], a["ws"],
                       a["n"], None)


WIDTHS = [(dict(d=0), BAD), (dict(f=-64), BAD), (dict(rows=-1), BAD), (dict(t=2), BAD), (dict(d=96), UNS),
          (dict(f=100), UNS), (dict(d=16384 + 64), UNS), (dict(f=16384 + 64), UNS)]


@pytest.mark.parametrize("kw,status", WIDTHS + [
    (dict(x=None), BAD), (dict(wgu=None), BAD), (dict(wd=None), BAD), (dict(a=None), BAD), (dict(y=None), BAD),
    (dict(x=ODD), BAD), (dict(wgu=ODD), BAD), (dict(wd=ODD), BAD), (dict(gu=ODD), BAD), (dict(a=ODD), BAD),
    (dict(y=ODD), BAD), (dict(ws=ODD), BAD),
])
def test_ffn_refusals(lib, kw, status):
    assert _ffn(lib, **kw) == status


def test_ffn_without_rows_needs_no_device(lib):
    assert _ffn(lib, rows=0, x=None, y=None) == tlf.OK


def _ffn_grad(lib, **kw):
    a = dict(dy=P, x=P, wgu=P, wd=P, gu=P, a=P, t=BF16, rows=5, d=64, f=128, dx=P, dwgu=P, dwd=P, ws=P, n=1 << 30)
    a.update(kw)
    return lib.tlf_ffn_grad(a["dy"], a["x"], a["wgu"], a["wd"], a["gu"], a["a"], a["t"], a["rows"], a["d"], a["f"],
                            a["dx"], a["dwgu"], a["dwd"], a["ws"], a["n"], None)


@pytest.mark.parametrize("kw,status", WIDTHS + [
    (dict(dy=None), BAD), (dict(x=None), BAD), (dict(wgu=None), BAD), (dict(wd=None), BAD), (dict(gu=None), BAD),
    (dict(a=None), BAD), (dict(ws=None), BAD), (dict(n=5 * 256 * 2 - 1), BAD), (dict(ws=ODD), BAD), (dict(dy=ODD), BAD),
    (dict(dx=ODD), BAD), (dict(dwgu=ODD), BAD), (dict(dwd=ODD), BAD), (dict(gu=ODD), BAD),
])
def test_ffn_grad_refusals(lib, kw, status):
    assert _ffn_grad(lib, **kw) == status


def test_ffn_grad_of_nothing(lib):
    assert _ffn_grad(lib, dx=None, dwgu=None, dwd=None, ws=None, n=0) == tlf.OK


def test_workspace_sizes_refuse_what_the_calls_refuse(lib):
    n = ctypes.c_size_t()
    assert lib.tlf_ffn_grad_ws_bytes(BF16, 5, 96, 128, ctypes.byref(n)) == UNS
    assert lib.tlf_ffn_grad_ws_bytes(BF16, 5, 64, 128, None) == BAD
    assert lib.tlf_rms_norm_grad_ws_bytes(17, 5, 64, ctypes.byref(n)) == UNS
    assert lib.tlf_rms_norm_grad_ws_bytes(1, 5, 64, None) == BAD
    # products of rows and widths past 32 bits
    assert lib.tlf_ffn_grad_ws_bytes(F32, 2 ** 31 - 1, 64, 16384, ctypes.byref(n)) == tlf.OK
    assert n.value >= (2 ** 31 - 1) * 2 * 16384 * 4


def _adamw(lib, count=1, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, table=True, **kw):
    a = dict(d_param=P, d_copy=None, d_grad=P, d_m=P, d_v=P, d_m_scale=P, d_v_scale=P, n=10, step=1, weight_decay=0.1,
             grad_dtype=F32, state_bits=32)
    a.update(kw)
    t = (tlf.AdamwTensor * 1)(tlf.AdamwTensor(**a))
    return lib.tlf_adamw(t if table else None, count, lr, b1, b2, eps, None)


@pytest.mark.parametrize("kw", [
    dict(count=-1), dict(table=False), dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(b1=1.0), dict(b1=-0.1),
    dict(b2=1.0), dict(b2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=1e-40), dict(eps=math.inf), dict(d_param=None),
    dict(d_grad=None), dict(d_m=None), dict(d_v=None), dict(n=-1), dict(step=0), dict(weight_decay=-0.1),
    dict(weight_decay=math.nan), dict(grad_dtype=7), dict(state_bits=16), dict(state_bits=8, d_m_scale=None),
    dict(state_bits=8, d_v_scale=None), dict(d_param=P + 2), dict(d_grad=P + 1), dict(d_m=P + 2), dict(d_copy=P + 1),
])
def test_adamw_refusals(lib, kw):
    assert _adamw(lib, **kw) == BAD


def test_adamw_of_nothing(lib):
    assert _adamw(lib, count=0, table=False) == tlf.OK
    assert _adamw(lib, n=0, d_param=None, d_grad=None) == tlf.OK


def test_adamw_struct_matches_the_header(tmp_path):
    import os
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tlf.h"\nint main(void){printf("%zu %zu %zu\\n",'
                   "sizeof(tlf_adamw_tensor),offsetof(tlf_adamw_tensor,weight_decay),"
                   "offsetof(tlf_adamw_tensor,state_bits));return 0;}")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c99", "-I", inc, str(src), "-o", str(tmp_path / "t")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    assert got == [ctypes.sizeof(tlf.AdamwTensor), tlf.AdamwTensor.weight_decay.offset, tlf.AdamwTensor.state_bits.offset]


def test_wrappers_refuse_host_tensors_and_wrong_shapes():
    x = torch.zeros(2, 64)
    with pytest.raises(ValueError):
        train.rms_norm(x)
    with pytest.raises(ValueError):
        train.ffn(x, torch.zeros(128, 64), torch.zeros(64, 64))
    with pytest.raises(ValueError):
        train.adamw_([x], [x], [x], [x], 1, lr=1e-3)
    with pytest.raises(ValueError):
        train.adamw_([x], [], [x], [x], 1, lr=1e-3)
    with pytest.raises(ValueError):
        train.AdamW([x.requires_grad_()], lr=1e-3)
    train.adamw_([], [], [], [], 1, lr=1e-3)


@pytest.mark.parametrize("rows", [2 ** 30 + 1, 2 ** 31 - 1])
def test_rms_norm_refuses_more_rows_than_it_counts(lib, rows):
    n = ctypes.c_size_t()
    assert _norm(lib, rows=rows) == UNS
    assert _norm_grad(lib, rows=rows) == UNS
    assert lib.tlf_rms_norm_grad_ws_bytes(2, rows, 8, ctypes.byref(n)) == UNS


@pytest.mark.parametrize("rows,d,f", [(2 ** 31 - 1, 64, 64), (2 ** 29, 64, 64), (2 ** 21, 64, 16384), (2 ** 21, 16384, 64)])
def test_ffn_refuses_more_elements_than_a_launch_covers(lib, rows, d, f):
    assert _ffn(lib, rows=rows, d=d, f=f) == UNS
    assert _ffn_grad(lib, rows=rows, d=d, f=f, n=1 << 60) == UNS


def test_adamw_refuses_more_elements_than_a_launch_covers(lib):
    assert _adamw(lib, n=2 ** 35 + 1) == UNS


def test_wrappers_refuse_dimensions_past_32_bits():
    x = torch.empty(2 ** 31, 4, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        train._int32("rms_norm", None, x)
