"""CPU checks of the training operators' host side: sizes and what the Python
wrappers do around the kernels."""
import os
import subprocess

import pytest
import torch
import torch.utils.checkpoint

from paper_2609_15160_amd import tlf, train

INC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def test_kept_bytes_match_the_header(tmp_path):
    """18 bits for each of two values in bf16, 32 in float32, of whole 16 rows."""
    cases = [(t, rows, f) for t in (tlf.DTYPE_F32, tlf.DTYPE_BF16) for rows in (0, 1, 15, 16, 17, 66000, 2 ** 29)
             for f in (64, 192, 16384)]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "tlf.h"\nint main(void){' + "".join(
        f'printf("%zu\\n",tlf_ffn_kept_bytes({t},{rows},{f}));' for t, rows, f in cases) + "return 0;}")
    subprocess.check_call(["gcc", "-std=c99", "-I", INC, str(src), "-o", str(tmp_path / "t")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    for n, (t, rows, f) in zip(got, cases):
        bits = (rows + 15) // 16 * 16 * f * 2 * (18 if t == tlf.DTYPE_BF16 else 32)
        assert n == tlf.ffn_kept_bytes(t, rows, f) == bits // 8 and n % 16 == 0


@pytest.fixture
def no_kernels(monkeypatch):
    """The autograd functions without their kernels: what they compute is left as it is allocated."""
    monkeypatch.setattr(train, "_run", lambda *a: None)
    monkeypatch.setattr(train, "_workspace", lambda *a, **k: (None, 0))


def _operators():
    x = torch.ones(3, 64, requires_grad=True)
    gamma, wgu, wd = torch.ones(1, 64), torch.ones(128, 64), torch.ones(64, 64)
    yield x, lambda t: train._RmsNorm.apply(t, gamma, None, 1e-5, torch.float32, True)
    yield x, lambda t: train._Ffn.apply(t, wgu, wd, True)


def test_gradients_with_a_graph_under_checkpointing(no_kernels):
    """A recomputed activation can be taken once: a first gradient that keeps a graph takes it no second time."""
    for x, op in _operators():
        y = torch.utils.checkpoint.checkpoint(op, x, use_reentrant=False)
        dx, = torch.autograd.grad(y, x, torch.ones_like(y), create_graph=True)
        assert dx.shape == x.shape and dx.requires_grad
        with pytest.raises(RuntimeError, match="gradients of gradients"):
            torch.autograd.grad(dx, x, torch.ones_like(dx))


@pytest.mark.parametrize("create_graph", [False, True])
def test_saved_tensors_are_unpacked_once(no_kernels, create_graph):
    for x, op in _operators():
        packed, unpacked = [], []

        def pack(t):
            packed.append(t)
            return t

        def unpack(t):
            unpacked.append(t)
            return t

        with torch.autograd.graph.saved_tensors_hooks(pack, unpack):
            y = op(x)
        torch.autograd.grad(y, x, torch.ones_like(y), create_graph=create_graph)
        assert len(packed) == len(unpacked) >= 3


# ---------------------------------------------------------------------------
# AdamW: overlapping tensors are refused before any device work
# ---------------------------------------------------------------------------

def _at(tensor, buffer, offset=0):
    return ((tensor * 8 + buffer + 1) << 16) + offset


def _buffers(tensor):
    """A tensor of 1000 elements, each of its buffers 64 KiB from the next."""
    names = ("d_param", "d_copy", "d_grad", "d_m", "d_v", "d_m_scale", "d_v_scale")
    return dict({name: _at(tensor, i) for i, name in enumerate(names)}, n=1000, step=1, weight_decay=0.0,
                grad_dtype=tlf.DTYPE_F32, state_bits=8)


def _step(*tensors):
    table = (tlf.AdamwTensor * len(tensors))(*(tlf.AdamwTensor(**{**_buffers(k), **a}) for k, a in enumerate(tensors)))
    return tlf.load().tlf_adamw(table, len(tensors), 1e-3, 0.9, 0.95, 1e-8, None)


@pytest.mark.parametrize("kw", [
    dict(d_param=_at(0, 0)), dict(d_copy=_at(0, 1)), dict(d_m=_at(0, 3)), dict(d_v=_at(0, 4)), dict(d_m_scale=_at(0, 5)),
    dict(d_v_scale=_at(0, 6)),                                            # the same buffer in two tensors
    dict(d_param=_at(0, 0, 3996)), dict(d_copy=_at(0, 1, 1998)), dict(d_m=_at(0, 3, 999)), dict(d_v=_at(0, 4, -999)),
    dict(d_m_scale=_at(0, 5, 12)),                                        # their last or first element
    dict(d_m_scale=_at(1, 6)), dict(d_copy=_at(1, 0)), dict(d_m=_at(1, 4, 500)),  # within one tensor
    dict(d_grad=_at(0, 0)), dict(d_grad=_at(1, 0)), dict(d_grad=_at(0, 1, 1000)),  # a gradient that an update overwrites
])
def test_adamw_refuses_overlapping_buffers(kw):
    assert _step({}, kw) == tlf.E_INVALID_ARG


@pytest.mark.parametrize("kw,twice", [({}, False), (dict(d_copy=_at(0, 1)), True), (dict(d_m_scale=_at(0, 5)), True),
                                      (dict(d_v_scale=_at(1, 5)), True), (dict(d_grad=_at(0, 2)), False),
                                      (dict(d_copy=_at(0, 1), n=0), False)])
def test_adamw_wrapper_names_a_buffer_given_twice(kw, twice):
    table = (tlf.AdamwTensor * 2)(*(tlf.AdamwTensor(**{**_buffers(k), **a}) for k, a in enumerate(({}, kw))))
    assert train._given_twice(table) is twice


# ---------------------------------------------------------------------------
# AdamW's state
# ---------------------------------------------------------------------------

class _Cuda(torch.Tensor):
    """A host tensor that passes for a device one where nothing reaches a device."""
    is_cuda = True


def _optimizer(bits=32):
    leaves = [torch.ones(300, dtype=torch.bfloat16), torch.ones(7)]
    return train.AdamW([t.as_subclass(_Cuda).requires_grad_() for t in leaves], lr=1e-3, state_bits=bits)


def _flat(opt):
    pairs = [t for v in (opt.masters, opt.exp_avgs, opt.exp_avg_sqs) for s in v for t in (s if isinstance(s, tuple) else (s,))]
    return [t for t in pairs if t is not None]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("key", ["steps", "masters", "exp_avgs", "exp_avg_sqs"])
def test_a_refused_state_is_not_half_loaded(bits, key):
    opt, other = _optimizer(bits), _optimizer(bits)
    other.steps = [3, 4]
    for t in _flat(other):
        t.view(torch.uint8).fill_(1)
    state = other.state_dict()
    if key == "steps":
        state[key] = [3]
    elif key == "masters":
        state[key] = [None, state[key][0]]  # the float32 leaf's place instead of the bfloat16 one's
    else:
        state[key] = [state[key][0], (torch.zeros(9) if bits == 32 else (state[key][1][0], torch.zeros(2)))]
    before = [t.clone() for t in _flat(opt)]
    with pytest.raises(ValueError):
        opt.load_state_dict(state)
    assert opt.steps == [0, 0]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(_flat(opt), before))
    opt.load_state_dict(other.state_dict())
    assert opt.steps == [3, 4]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(_flat(opt), _flat(other)))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_loaded_state_reaches_the_bfloat16_leaves(bits):
    opt, other = _optimizer(bits), _optimizer(bits)
    other.masters[0].copy_(torch.linspace(-3, 3, 300))
    opt.load_state_dict(other.state_dict())
    assert torch.equal(opt.masters[0], other.masters[0])
    assert torch.equal(opt.params[0].detach(), opt.masters[0].to(torch.bfloat16))
    assert torch.equal(opt.params[1].detach(), torch.ones(7))  # a float32 leaf is the caller's to load


def _stepped(monkeypatch, opt):
    """opt.step() with a gradient for every leaf and a kernel that adds 2^-12 to each parameter, copies rounded."""
    def kernel(params, grads, m, v, steps, lr, betas, eps, decay, copies):
        for p, c in zip(params, copies):
            p += 2.0 ** -12
            if c is not None:
                c.copy_(p)

    monkeypatch.setattr(train, "adamw_", kernel)
    for p in opt.params:
        p.grad = torch.zeros_like(p)
    opt.step()


def test_weights_written_into_a_leaf_reach_its_master(monkeypatch):
    """What a bfloat16 leaf was set to between steps is what the next step goes on from; elements that are as the
    master rounded keep the master's bits, after a write of the same values too."""
    opt = _optimizer()
    for _ in range(3):
        _stepped(monkeypatch, opt)
    master, leaf = opt.masters[0], opt.params[0]
    kept = master.clone()
    assert torch.equal(kept, torch.full((300,), 1 + 3 * 2.0 ** -12))  # 1 in bfloat16
    with torch.no_grad():
        leaf[:100] = 5.0
        leaf[100:200] = leaf[100:200].clone()
    _stepped(monkeypatch, opt)
    assert torch.equal(master[:100], torch.full((100,), 5 + 2.0 ** -12))
    assert torch.equal(master[100:], kept[100:] + 2.0 ** -12)
    assert torch.equal(leaf.detach(), master.to(torch.bfloat16))
    with torch.no_grad():
        leaf.fill_(-2.0)
    assert torch.equal(opt.state_dict()["masters"][0], torch.full((300,), -2.0))
    with torch.no_grad():
        leaf.fill_(7.0)
    fresh = _optimizer()
    opt.load_state_dict(fresh.state_dict())  # a loaded state comes after what was written before it
    _stepped(monkeypatch, opt)
    assert torch.equal(master, torch.full((300,), 1 + 2.0 ** -12))
