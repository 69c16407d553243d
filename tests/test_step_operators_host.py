"""CPU checks of what the Python wrappers of the attention and of the residual with its
norm do around the kernels."""
import pytest
import torch
import torch.utils.checkpoint

from paper_2609_15160_amd import train


@pytest.fixture
def no_kernels(monkeypatch):
    """The autograd functions without their kernels: what they compute is left as it is allocated."""
    class Library:
        def __getattr__(self, name):
            return name
    monkeypatch.setattr(train, "_run", lambda *a: None)
    monkeypatch.setattr(train, "_workspace", lambda *a, **k: (None, 0))
    monkeypatch.setattr(train.tlf, "load", Library)


def _operators():
    off = torch.tensor([0, 2, 3], dtype=torch.int32)
    q, k = torch.ones(3, 4, 64, requires_grad=True), torch.ones(3, 2, 64)
    yield q, lambda t: train._Attention.apply(t, k, k, off, off, None, 4, 2, 64, 0, 0, 0.125, True)
    qkv = torch.ones(3, 8 * 64, requires_grad=True)
    yield qkv, lambda t: train._Attention.apply(t, None, None, off, off, None, 4, 2, 64, 5, 1, 0.125, True)
    x, y, scale = torch.ones(3, 64, requires_grad=True), torch.ones(3, 64), torch.ones(1, 64)
    yield x, lambda t: train._ResidualNorm.apply(t, y, scale, scale, None, 1e-5, False, True)[1]
    yield x, lambda t: train._ResidualNorm.apply(t, y, None, None, None, 1e-5, True, True)[0]


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


def test_a_step_with_clipping_takes_the_norm_once(monkeypatch):
    """AdamW.step(max_norm): one norm over all gradients, whose scale every group's update takes; none without."""
    calls = []
    monkeypatch.setattr(train, "grad_norm", lambda g, m: calls.append((len(list(g)), m)) or ("norm", "scale"))
    monkeypatch.setattr(train, "adamw_", lambda *a, **k: calls.append(k.get("grad_scale")))
    p = [torch.nn.Parameter(torch.ones(4)) for _ in range(3)]
    opt = object.__new__(train.AdamW)
    opt.params, opt.masters = p, [None] * 3
    opt.exp_avgs, opt.exp_avg_sqs, opt.steps = [None] * 3, [None] * 3, [0] * 3
    opt.weight_decay, opt.lr, opt.betas, opt.eps, opt._written = [0.0] * 3, 1e-3, (0.9, 0.95), 1e-8, [None] * 3
    monkeypatch.setattr(opt, "_take_written", lambda have: None, raising=False)
    monkeypatch.setattr(train, "_writes", lambda p: 0)
    assert opt.step(max_norm=1.0) is None and not calls  # no gradients yet
    for t in p[:2]:
        t.grad = torch.ones(4)
    assert opt.step(max_norm=1.0) == "norm" and calls[0] == (2, 1.0) and set(calls[1:]) == {"scale"}
    assert opt.steps == [1, 1, 0]
    calls.clear()
    assert opt.step() is None and set(calls) == {None}
