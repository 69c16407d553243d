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
    (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=math.nan), BAD), (dict(scale=math.inf), BAD),
    (dict(q_stride=252), BAD), (dict(q_stride=248), BAD), (dict(k_stride=120), BAD), (dict(v_stride=-128), BAD),
    (dict(o_stride=0), BAD), (dict(d_q_offsets=None), BAD), (dict(d_k_offsets=None), BAD), (dict(head_dim=32), UNS),
    (dict(head_dim=16), UNS), (dict(sinks=65), UNS), (dict(q_stride=(1 << 22) + 8), UNS), (dict(rows_q=1 << 30), UNS),
    (dict(rows_k=1 << 30), UNS), (dict(rows_q=1 << 28), UNS), (dict(batch=1 << 21), UNS),
    (dict(heads=2048, kv_heads=2, q_stride=1 << 17, o_stride=1 << 17), UNS),
]


@pytest.mark.parametrize("kw,status", SHAPES)
def test_attention_shape_refusals(lib, kw, status):
    need, s = ctypes.c_size_t(), _shape(**kw)
    assert lib.tlf_attn_ws_bytes(s, need) == status and lib.tlf_attn_grad_ws_bytes(s, need) == status
    assert lib.tlf_attn(s, P, P, P, P, P, P, BIG, None) == status
    assert lib.tlf_attn_grad(s, P, P, P, P, P, P, P, 256, P, 128, P, 128, P, BIG, None) == status


@pytest.mark.parametrize("at", range(1, 5))
@pytest.mark.parametrize("bad", [None, ODD])
def test_attention_pointer_refusals(lib, at, bad):
    args = [_shape(), P, P, P, P, P, P, BIG, None]
    args[at] = bad
    assert lib.tlf_attn(*args) == BAD


def test_attention_other_refusals(lib):
    assert lib.tlf_attn(None, P, P, P, P, P, P, BIG, None) == BAD
    assert lib.tlf_attn_ws_bytes(_shape(), None) == BAD and lib.tlf_attn_grad_ws_bytes(_shape(), None) == BAD
    assert lib.tlf_attn(_shape(), P, P, P, P, 0x1002, P, BIG, None) == BAD
    assert lib.tlf_attn(_shape(d_q_offsets=0x1002), P, P, P, P, P, P, BIG, None) == BAD
    assert lib.tlf_attn(_shape(d_k_lengths=0x1001), P, P, P, P, P, P, BIG, None) == BAD
    need, few = ctypes.c_size_t(), _shape(rows_q=3, rows_k=300000, window=0)
    assert lib.tlf_attn_ws_bytes(few, need) == tlf.OK and need.value > 0
    assert lib.tlf_attn(few, P, P, P, P, None, P, need.value - 1, None) == BAD
    assert lib.tlf_attn(few, P, P, P, P, None, None, BIG, None) == BAD
    assert lib.tlf_attn(_shape(rows_q=0), None, P, P, None, None, None, 0, None) == tlf.OK


@pytest.mark.parametrize("at,bad", [(k, b) for k in (1, 2, 3, 4, 5, 7, 9, 11, 13) for b in (None, ODD)] +
                         [(6, None), (6, 0x1002), (8, 248), (8, 257), (10, 120), (12, 120), (14, 4)])
def test_attention_gradient_refusals(lib, at, bad):
    args = [_shape(), P, P, P, P, P, P, P, 256, P, 128, P, 128, P, BIG, None]
    args[at] = bad
    assert lib.tlf_attn_grad(*args) == BAD


def test_attention_gradient_of_nothing(lib):
    s = _shape(rows_q=0, rows_k=0, batch=0)
    assert lib.tlf_attn_grad(s, None, None, None, None, None, None, None, 256, None, 128, None, 128, None, 0, None) == tlf.OK


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
    assert f"TLF_ATTN_MAX_SINKS {tlf.ATTN_MAX_SINKS}\n" in text and tlf.ATTN_MAX_STRIDE == 1 << 22


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
