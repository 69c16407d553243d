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
