"""CPU checks of the argument checks of the training operators around the FFN half:
every refusal comes before any device work (there is no device here), on addresses
that are never read."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2609_15160_amd import tlf, train

INC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
P, ODD = 0x1000, 0x1008  # a 16-byte and an 8-byte aligned address
BAD, UNS, F32, BF16 = tlf.E_INVALID_ARG, tlf.E_UNSUPPORTED, tlf.DTYPE_F32, tlf.DTYPE_BF16
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return tlf.load()


def _shape(**kw):
    a = dict(dtype=BF16, batch=3, heads=4, kv_heads=2, head_dim=64, rows_q=100, rows_k=200, window=16, sinks=4, scale=0.125,
             q_stride=256, k_stride=128, v_stride=128, o_stride=256, d_q_offsets=P, d_k_offsets=P, d_k_lengths=None)
    a.update(kw)
    return tlf.AttnShape(**a)


SHAPES = [
    (dict(dtype=2), BAD), (dict(batch=-1), BAD), (dict(rows_q=-1), BAD), (dict(rows_k=-1), BAD), (dict(heads=0), BAD),
    (dict(kv_heads=0), BAD), (dict(kv_heads=3), BAD), (dict(head_dim=0), BAD), (dict(window=-1), BAD), (dict(sinks=-1), BAD),
    (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=math.nan), BAD), (dict(scale=math.inf), BAD), (dict(scale=1e-13), BAD), (dict(scale=1.1e12), BAD),
    (dict(q_stride=252), BAD), (dict(q_stride=248), BAD), (dict(k_stride=120), BAD), (dict(v_stride=-128), BAD),
    (dict(o_stride=0), BAD), (dict(d_q_offsets=None), BAD), (dict(d_k_offsets=None), BAD), (dict(head_dim=32), UNS),
    (dict(head_dim=16), UNS), (dict(sinks=65), UNS), (dict(q_stride=(1 << 21) + 8), UNS), (dict(rows_q=1 << 30), UNS),
    (dict(rows_k=1 << 30), UNS), (dict(rows_q=1 << 28), UNS), (dict(batch=1 << 21), UNS),
    (dict(heads=2048, kv_heads=2, q_stride=1 << 17, o_stride=1 << 17), UNS),
]


@pytest.mark.parametrize("kw,status", SHAPES)
def test_attention_shape_refusals(lib, kw, status):
    need, s = ctypes.c_size_t(), _shape(**kw)
    assert lib.tlf_attn_ws_bytes(s, need) == status and lib.tlf_attn_grad_ws_bytes(s, need) == status
    assert lib.tlf_attn(s, P, P, P, P, P, P, P, BIG, None) == status
    assert lib.tlf_attn_grad(s, P, P, P, P, P, P, P, P, 256, P, 128, P, 128, P, BIG, None) == status


@pytest.mark.parametrize("at", range(1, 5))
@pytest.mark.parametrize("bad", [None, ODD])
def test_attention_pointer_refusals(lib, at, bad):
    args = [_shape(), P, P, P, P, P, P, P, BIG, None]
    args[at] = bad
    assert lib.tlf_attn(*args) == BAD


def test_attention_other_refusals(lib):
    assert lib.tlf_attn(None, P, P, P, P, P, P, P, BIG, None) == BAD
    assert lib.tlf_attn_ws_bytes(_shape(), None) == BAD and lib.tlf_attn_grad_ws_bytes(_shape(), None) == BAD
    assert lib.tlf_attn(_shape(), P, P, P, P, 0x1002, P, P, BIG, None) == BAD
    assert lib.tlf_attn(_shape(d_q_offsets=0x1002), P, P, P, P, P, P, P, BIG, None) == BAD
    assert lib.tlf_attn(_shape(d_k_lengths=0x1001), P, P, P, P, P, P, P, BIG, None) == BAD
    need, few = ctypes.c_size_t(), _shape(rows_q=3, rows_k=300000, window=0)
    assert lib.tlf_attn_ws_bytes(few, need) == tlf.OK and need.value > 0
    assert lib.tlf_attn(few, P, P, P, P, None, None, P, need.value - 1, None) == BAD
    assert lib.tlf_attn(few, P, P, P, P, None, None, None, BIG, None) == BAD
    assert lib.tlf_attn(_shape(rows_q=0), None, P, P, None, None, None, None, 0, None) == tlf.OK
    assert lib.tlf_attn(_shape(), P, P, P, P, P, ODD, P, BIG, None) == BAD
    f32 = _shape(dtype=F32)  # whose o is not rounded
    assert lib.tlf_attn(f32, P, P, P, P, P, P, P, BIG, None) == BAD
    assert lib.tlf_attn_grad(f32, P, P, P, P, P, P, P, P, 256, P, 128, P, 128, P, BIG, None) == BAD


@pytest.mark.parametrize("at,bad", [(k, b) for k in (1, 2, 3, 4, 5, 8, 10, 12, 14) for b in (None, ODD)] +
                         [(6, None), (6, 0x1002), (7, ODD), (9, 248), (9, 257), (11, 120), (13, 120), (15, 4)])
def test_attention_gradient_refusals(lib, at, bad):
    args = [_shape(), P, P, P, P, P, P, P, P, 256, P, 128, P, 128, P, BIG, None]
    args[at] = bad
    assert lib.tlf_attn_grad(*args) == BAD


def test_attention_gradient_of_nothing(lib):
    s = _shape(rows_q=0, rows_k=0, batch=0)
    assert lib.tlf_attn_grad(s, None, None, None, None, None, None, None, None, 256, None, 128, None, 128, None, 0, None) == tlf.OK


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"tlf_attn_shape": tlf.AttnShape}
    src, want = "", []
    for name, s in structs.items():
        src += f'printf("%zu ", sizeof({name}));' + "".join(f'printf("%zu ", offsetof({name}, {f}));' for f, _ in s._fields_)
        want += [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tlf.h"\nint main(void){' + src + "return 0;}")
    subprocess.check_call(["gcc", "-std=c99", "-I", INC, str(tmp_path / "t.c"), "-o", str(tmp_path / "t")])
    assert [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()] == want
    text = open(os.path.join(INC, "tlf.h")).read()
    assert f"TLF_ATTN_MAX_SINKS {tlf.ATTN_MAX_SINKS}\n" in text and tlf.ATTN_MAX_STRIDE == 1 << 21


class _Cuda(torch.Tensor):
    """A CPU tensor that passes for one on a device: the checks of arguments come before any use."""
    is_cuda = True


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_Cuda)


def _off(*v):
    return _t(len(v), dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: train.attention(torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), _off(0, 3)),
    lambda: train.attention(_t(3, 128), _t(3, 2, 64), _t(3, 2, 64), _off(0, 3)),
    lambda: train.attention(_t(3, 2, 64), _t(3, 2, 64), _t(3, 1, 64), _off(0, 3)),
    lambda: train.attention(_t(3, 2, 64), _t(3, 2, 16), _t(3, 2, 16), _off(0, 3)),
    lambda: train.attention(_t(3, 3, 64), _t(3, 2, 64), _t(3, 2, 64), _off(0, 3)),
    lambda: train.attention(_t(3, 2, 64), _t(4, 2, 64), _t(4, 2, 64), _off(0, 3)),
    lambda: train.attention(_t(3, 2, 64), _t(3, 2, 64, dtype=torch.float32), _t(3, 2, 64), _off(0, 3)),
    lambda: train.attention(*[_t(3, 2, 64, dtype=torch.float16)] * 3, _off(0, 3)),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _t(2, dtype=torch.int64)),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _t(2, 1, dtype=torch.int32)),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _t(0, dtype=torch.int32)),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _off(0, 3), _off(0, 1, 3)),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _off(0, 3), None, _off(1, 2)),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _off(0, 3), window=0),
    lambda: train.attention(*[_t(3, 2, 64)] * 3, _off(0, 3), sinks=-1),
    lambda: train.self_attention(_t(3, 6, 64), _off(0, 3), 2),
    lambda: train.self_attention(_t(3, 384), _off(0, 3), 5),
    lambda: train.self_attention(_t(3, 384), _off(0, 3), 4, 3),
    lambda: train.self_attention(_t(3, 384), _off(0, 3), 0),
    lambda: train.self_attention(torch.zeros(3, 384), _off(0, 3), 2),
])
def test_attention_argument_errors(call):
    with pytest.raises(ValueError, match="attention"):
        call()


@pytest.mark.parametrize("sinks", [65, 1 << 31, (1 << 32) + 1, 1 << 40])
@pytest.mark.parametrize("window", [None, 5, (1 << 32) + 5])
def test_sinks_past_their_limit_are_refused_at_any_size(sinks, window):
    """A number that 32 bits do not hold is not taken for what is left of it."""
    for call in (lambda: train.attention(*[_t(3, 2, 64)] * 3, _off(0, 3), window=window, sinks=sinks),
                 lambda: train.self_attention(_t(3, 384), _off(0, 3), 2, window=window, sinks=sinks)):
        with pytest.raises(tlf.TlfError) as e:
            call()
        assert e.value.status == UNS


def test_offsets_past_32_bits_are_refused():
    off = torch.zeros(1, dtype=torch.int32).expand((1 << 32) + 1).as_subclass(_Cuda)
    with pytest.raises(ValueError, match="2.31"):
        train.attention(*[_t(3, 2, 64)] * 3, off)


def _resid(lib, **kw):
    a = dict(x=P, y=P, yt=BF16, alpha=P, gamma=P, group=P, groups=2, rows=3, d=8, post=0, eps=1e-5, h=P, z=P, rstd=P, ystd=P)
    a.update(kw)
    return lib.tlf_residual_norm(*(a[k] for k in ("x", "y", "yt", "alpha", "gamma", "group", "groups", "rows", "d", "post",
                                                  "eps", "h", "z", "rstd", "ystd")), None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), BAD), (dict(y=None), BAD), (dict(h=None), BAD), (dict(z=None), BAD), (dict(x=ODD), BAD), (dict(y=ODD), BAD),
    (dict(h=ODD), BAD), (dict(z=ODD), BAD), (dict(alpha=ODD), BAD), (dict(gamma=ODD), BAD), (dict(yt=2), BAD),
    (dict(rows=-1), BAD), (dict(d=0), BAD), (dict(d=6), BAD), (dict(eps=0.0), BAD), (dict(eps=math.nan), BAD),
    (dict(groups=-1), BAD), (dict(groups=0), BAD), (dict(alpha=None, gamma=None), BAD), (dict(group=None), BAD),
    (dict(group=0x1002), BAD), (dict(rstd=0x1002), BAD), (dict(ystd=0x1001), BAD), (dict(d=4100), UNS),
    (dict(groups=17), UNS), (dict(rows=(1 << 30) + 1), UNS),
])
def test_residual_norm_refusals(lib, kw, status):
    assert _resid(lib, **kw) == status


def test_residual_norm_without_rows_needs_no_device(lib):
    assert _resid(lib, rows=0, x=None, y=None, h=None, z=None) == tlf.OK


def _resid_grad(lib, **kw):
    a = dict(dh=P, dz=P, h=P, y=P, yt=F32, alpha=P, gamma=P, group=P, groups=2, rstd=P, ystd=P, rows=3, d=8, post=1, dx=P, dy=P,
             dalpha=P, dgamma=P, ws=P, n=1 << 20)
    a.update(kw)
    return lib.tlf_residual_norm_grad(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(h=None), BAD), (dict(y=None), BAD), (dict(rstd=None), BAD), (dict(ystd=None), BAD), (dict(dx=None), BAD),
    (dict(dy=None), BAD), (dict(group=None), BAD), (dict(ws=None), BAD), (dict(n=127), BAD), (dict(dalpha=None), BAD),
    (dict(dgamma=None), BAD), (dict(alpha=None), BAD), (dict(gamma=None), BAD), (dict(groups=0, alpha=None, gamma=None), BAD),
    *[({k: ODD}, BAD) for k in ("dh", "dz", "h", "y", "alpha", "gamma", "dx", "dy", "dalpha", "dgamma", "ws")],
    (dict(d=10), BAD), (dict(yt=9), BAD), (dict(rows=-2), BAD), (dict(d=8192), UNS), (dict(groups=33), UNS),
])
def test_residual_norm_grad_refusals(lib, kw, status):
    assert _resid_grad(lib, **kw) == status


def _grads(*t):
    return (tlf.Grad * max(1, len(t)))(*(tlf.Grad(*v, 0) for v in t))


@pytest.mark.parametrize("t,status", [
    ((None, 5, F32), BAD), ((P, -1, F32), BAD), ((P, 5, 2), BAD), ((0x1002, 5, F32), BAD), ((0x1001, 5, BF16), BAD),
    ((P, (1 << 35) + 1, F32), UNS),
])
def test_grad_norm_refusals(lib, t, status):
    need, g = ctypes.c_size_t(), _grads((P, 10, F32), t)
    assert lib.tlf_grad_norm_ws_bytes(g, 2, need) == status
    assert lib.tlf_grad_norm(g, 2, 1.0, P, P, P, BIG, None) == status
    assert lib.tlf_grad_clip(g, 2, 0x4000, None) == status


def test_grad_norm_other_refusals(lib):
    g, need = _grads((P, 10, F32), (None, 0, BF16)), ctypes.c_size_t()
    assert lib.tlf_grad_norm_ws_bytes(g, 2, need) == tlf.OK and need.value == 8
    for bad in (0.0, -1.0, math.nan):
        assert lib.tlf_grad_norm(g, 2, bad, P, P, P, 8, None) == BAD
    for norm, scale, ws, n in ((None, P, P, 8), (0x1002, P, P, 8), (P, 0x1002, P, 8), (P, P, None, 8), (P, P, 0x1004, 8), (P, P, P, 7)):
        assert lib.tlf_grad_norm(g, 2, 1.0, norm, scale, ws, n, None) == BAD
    assert lib.tlf_grad_norm(None, 2, 1.0, P, P, P, 8, None) == BAD and lib.tlf_grad_norm(g, -1, 1.0, P, P, P, 8, None) == BAD
    assert lib.tlf_grad_clip(g, 2, None, None) == BAD and lib.tlf_grad_clip(g, 2, 0x4002, None) == BAD


@pytest.mark.parametrize("b,scale", [((P, 10, F32), 0x4000), ((P + 36, 10, F32), 0x4000), ((P + 38, 1, BF16), 0x4000),
                                     ((P + 64, 10, F32), P + 36), ((P + 64, 10, F32), P + 64)])
def test_grad_clip_refuses_overlaps(lib, b, scale):
    assert lib.tlf_grad_clip(_grads((P, 10, F32), b), 2, scale, None) == BAD


def _adamw(scale, **kw):
    a = dict(d_param=0x10000, d_copy=None, d_grad=0x20000, d_m=0x30000, d_v=0x40000, n=64, step=1, weight_decay=0.0,
             grad_dtype=F32, state_bits=32)
    a.update(kw)
    t = (tlf.AdamwTensor * 1)()
    for k, v in a.items():
        setattr(t[0], k, v)
    return tlf.load().tlf_adamw_scaled(t, 1, 1e-3, 0.9, 0.95, 1e-8, scale, None)


@pytest.mark.parametrize("scale", [None, 0x1002, 0x10000, 0x100fc, 0x30010, 0x40000])
def test_scaled_adamw_refusals(scale):
    assert _adamw(scale) == BAD


def test_scaled_adamw_refuses_what_adamw_does():
    assert _adamw(0x1000, step=0) == BAD and _adamw(0x1000, n=(1 << 35) + 1) == UNS and _adamw(0x1000, d_m=0x10000) == BAD


def test_grad_struct_layout(tmp_path):
    src = 'printf("%zu ", sizeof(tlf_grad));' + "".join(f'printf("%zu ", offsetof(tlf_grad, {f}));' for f, _ in tlf.Grad._fields_)
    (tmp_path / "t.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tlf.h"\nint main(void){' + src + "return 0;}")
    subprocess.check_call(["gcc", "-std=c99", "-I", INC, str(tmp_path / "t.c"), "-o", str(tmp_path / "t")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    assert got == [ctypes.sizeof(tlf.Grad)] + [getattr(tlf.Grad, f).offset for f, _ in tlf.Grad._fields_]


F = torch.float32


@pytest.mark.parametrize("call", [
    lambda: train.residual_norm(torch.zeros(3, 8), torch.zeros(3, 8)),
    lambda: train.residual_norm(_t(3, 8), _t(3, 8)),
    lambda: train.residual_norm(_t(3, 2, 4, dtype=F), _t(3, 2, 4)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 4)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8, dtype=torch.float16)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), alpha=_t(8)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), alpha=_t(4, dtype=F)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), alpha=_t(2, 8, dtype=F)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), alpha=_t(0, 8, dtype=F), group=_t(3, dtype=torch.int32)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), alpha=_t(2, 8, dtype=F), gamma=_t(3, 8, dtype=F),
                                group=_t(3, dtype=torch.int32)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), group=_t(3, dtype=torch.int32)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), gamma=_t(2, 8, dtype=F), group=_t(3, dtype=torch.int64)),
    lambda: train.residual_norm(_t(3, 8, dtype=F), _t(3, 8), gamma=_t(2, 8, dtype=F), group=_t(2, dtype=torch.int32)),
])
def test_residual_norm_argument_errors(call):
    with pytest.raises(ValueError, match="residual_norm"):
        call()


@pytest.mark.parametrize("fn,args", [(train.grad_norm, ()), (train.clip_grad_norm_, (1.0,))])
@pytest.mark.parametrize("grads", [[], [torch.zeros(4)], [_t(4, dtype=torch.float16)], [_t(4, 4).T]])
def test_grad_norm_argument_errors(fn, args, grads):
    with pytest.raises(ValueError, match=fn.__name__):
        fn(grads, *args)


def test_limits_that_are_none():
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError, match="max_norm"):
            train.grad_norm([_t(4)], bad)
    with pytest.raises(ValueError, match="max_norm"):
        train.clip_grad_norm_([_t(4)], None)
    with pytest.raises(ValueError, match="grad_scale"):
        train.adamw_([_t(4, dtype=F)], [_t(4)], [_t(4, dtype=F)], [_t(4, dtype=F)], 1, 1e-3, grad_scale=_t(2, dtype=F))
