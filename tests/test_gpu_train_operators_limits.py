"""GPU tests of the training operators of the block's FFN half where their
arguments end: gates and products across float32's range, moments whose codes
are at the ends of the 8-bit formats, states that do not fit, tensors that
overlap, every tile shape against the formula with its roundings.

Bars as in test_gpu_train_operators.py: e = 2^-24 relative to the value for a
float32 rounding, 2^-8 for one to bf16, 2^-10 for what the gated FFN keeps
between its passes; (n + 2) e times the sum of magnitudes for a sum."""
import numpy as np
import pytest

from oracle import train_operators as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E32, E16, EKEPT = 2.0 ** -24, 2.0 ** -8, 2.0 ** -10


def _train():
    from paper_2609_15160_amd import train
    return train


def _say(*what):
    print("[train-op]", *what, flush=True)


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(v):
    """The values as bf16, and what those stand for."""
    t = torch.tensor(v, dtype=torch.float64).to(torch.bfloat16)
    return t, t.double().numpy()


def _close(got, want, bound, what):
    got = _np(got)
    over = np.abs(got - want) - bound
    assert got.shape == want.shape and np.all(over <= 0), (what, np.unravel_index(np.argmax(over), over.shape),
                                                           got.ravel()[np.argmax(over)], want.ravel()[np.argmax(over)])


# ---------------------------------------------------------------------------
# Gated FFN: the range of what it keeps
# ---------------------------------------------------------------------------

# gates and ups of bf16 operands: ordinary, past 2^32, near the top, below 2^-30 and far below
GATES = [0.5, -2.0, 3.0, -9.0, 1e10, 1e20, 1e33, 1.0, 2.0, 5.0, 1e-13, 2.0 ** -28, 2.0 ** -34, 2.0 ** -42, 1e-30, -1e-12]
UPS = [1.5, 0.25, -4.0, 8.0, 1.0, 1.0, 1.0, 1e10, -1e20, 3e33, 1e-13, 2.0 ** -29, 2.0 ** -33, 1.0, 1e-7, 1e-12]


@pytest.mark.parametrize("n,f", [
    (1, 64), (17, 64), (333, 192),
    (2000, 2688),  # gate/up and da on 128 x 128 tiles
    (4096, 2816),  # on 256 x 256 tiles
])
def test_ffn_gradients_over_the_range_of_bf16(n, f):
    """Column c's gate and up are x's first element times one weight each, W_down passes every 64th column on, dy is a
    power of two: the gradients are sums of dg and du themselves, whatever the column's magnitude.

    An element of dg or du is off by its own rounding, that of what was kept, and 2^-18 for the float32 arithmetic of
    the activation (1 - s next to 1 times a gate of 10: 10 2^-24, and exp and reciprocal in their last bits)."""
    train = _train()
    d = 64
    _say("ffn range", n, d, f)
    gate, up = _bf16(np.resize(GATES, f))[0], _bf16(np.resize(UPS, f))[0]
    x = torch.zeros(n, d, dtype=torch.bfloat16)
    x[:, 0] = 1.0
    x[1::2, 0] = -1.0  # the negative gates too
    wgu = torch.zeros(2 * f, d, dtype=torch.bfloat16)
    wgu[:f, 0], wgu[f:, 0] = gate, up
    wd = torch.eye(64, dtype=torch.bfloat16).repeat(1, f // 64).contiguous()
    dy = torch.full((n, d), 2.0 ** -6, dtype=torch.bfloat16)
    leaves = [t.cuda().requires_grad_() for t in (x, wgu, wd)]
    y = train.ffn(*leaves)
    got = torch.autograd.grad(y, leaves, dy.cuda())
    X, W, D, G = (t.double().numpy() for t in (x, wgu, wd, dy))
    A = np.abs
    with np.errstate(over="ignore"):
        g, u = X @ W[:f].T, X @ W[f:].T
        s = O.sigmoid(g)
        a = g * s * u
        da = G @ D
        dgu = np.concatenate([da * u * s * (1 + g * (1 - s)), da * g * s], 1)
        want = [dgu @ W, dgu.T @ X, G.T @ a]
    assert all(np.isfinite(w).all() for w in want)
    ea, ed = A(a) * (E16 + 2.0 ** -18), A(dgu) * (E16 + EKEPT + 2.0 ** -18)
    bounds = [ed @ A(W) + (2 * f + 2) * E32 * (A(dgu) @ A(W)), ed.T @ A(X) + (n + 2) * E32 * (A(dgu).T @ A(X)),
              A(G).T @ ea + (n + 2) * E32 * (A(G).T @ A(a))]
    _close(y, a @ D.T, 1.01 * (ea @ A(D).T + (f + 2) * E32 * (A(a) @ A(D).T) + E16 * A(a @ D.T)) + 1e-37, "y")
    for name, t, w, b in zip(("dx", "dw_gate_up", "dw_down"), got, want, bounds):
        _close(t, w, 1.01 * (b + E16 * A(w)) + 1e-37, name)


def test_ffn_infinities_reach_the_gradients():
    """An infinite up value gives infinite gradients, a NaN gives NaN, and neither leaves its columns."""
    train = _train()
    n, d, f = 3, 64, 64
    x = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 1.0
    wgu = torch.zeros(2 * f, d, dtype=torch.bfloat16, device="cuda")
    wgu[:, 0] = 0.5
    wgu[f + 1, 0], wgu[f + 2, 0], wgu[f + 3, 0] = float("inf"), float("-inf"), float("nan")
    wd = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    leaves = [t.requires_grad_() for t in (wgu, wd)]
    y = train.ffn(x, *leaves)
    dwgu, = torch.autograd.grad(y, leaves[:1], torch.ones_like(y))
    assert dwgu[1, 0] == float("inf") and dwgu[2, 0] == float("-inf") and torch.isnan(dwgu[3, 0])
    rest = [k for k in range(f) if k not in (1, 2, 3)]
    assert torch.isfinite(dwgu[:f][rest]).all() and torch.isfinite(dwgu[f:]).all()


def test_gradients_under_checkpointing():
    """Recomputed in the backward pass, with and without a graph of it: the gradients of a plain pass, to the bit."""
    from torch.utils.checkpoint import checkpoint
    train = _train()
    gen = torch.Generator(device="cuda").manual_seed(12)
    new = lambda *s, scale=1.0: (torch.randn(*s, generator=gen, device="cuda") * scale).requires_grad_()  # noqa: E731
    leaves = [new(70, 128), new(1, 128, scale=0.2), new(2 * 192, 128, scale=0.1), new(128, 192, scale=0.1)]

    def block(x, gamma, wgu, wd):
        return train.ffn(train.rms_norm(x, gamma), wgu, wd)

    y = block(*leaves)
    dy = torch.randn(y.shape, generator=gen, device="cuda")
    want = torch.autograd.grad(y, leaves, dy)
    for graph in (False, True):
        y = checkpoint(block, *leaves, use_reentrant=False)
        for a, b in zip(torch.autograd.grad(y, leaves, dy, create_graph=graph), want):
            assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------

def _fresh8(n):
    """Fresh 8-bit moments of n elements."""
    codes = lambda t: torch.zeros(n, dtype=torch.uint8, device="cuda").view(t)  # noqa: E731
    scales = lambda: torch.zeros(-(-n // O.BLOCK), device="cuda")  # noqa: E731
    return (codes(torch.float8_e4m3fn), scales()), (codes(torch.float8_e5m2), scales())


def test_adamw_smallest_second_moments():
    """Gradients so far below their block's largest that v over the scale is none in float32 keep the smallest code."""
    train = _train()
    n = 3 * 256 + 5
    g = np.zeros(n, np.float32)
    g[0], g[1:200] = 1.0, 1e-26
    g[256], g[257:400] = 1e15, 1e-30
    g[512], g[513:600] = 1e-3, 1e-45
    g[768], g[769:] = 1.0, 1e-38  # the last, short block
    p, (m, v) = torch.zeros(n, device="cuda"), _fresh8(n)
    _say("adamw tiny", n)
    train.adamw_([p], [torch.from_numpy(g).cuda()], [m], [v], 1, lr=1e-3)
    _, m1, v1 = O.adamw(np.zeros(n), g, np.zeros(n), np.zeros(n), 1, 1e-3, (0.9, 0.95), 1e-8, 0.0)
    for got, new, which in ((m, m1, "m"), (v, v1, "v")):
        codes, scales = O.encode(new, which)
        assert np.array_equal(got[1].cpu().numpy(), scales), which
        assert torch.equal(got[0].cpu().view(torch.uint8), codes.view(torch.uint8)), which
    assert torch.equal(v[0].float() > 0, torch.from_numpy(g > 0).cuda())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 1e38])
def test_adamw_spoilt_gradients_spoil_their_block(bad):
    """8 bits: one gradient that is not finite, or whose square is none in float32, makes the block's scale of the
    second moments (and, unless finite, of the first) infinite or NaN, as the formula's largest magnitude; the other
    blocks go on, and the next step shows NaN in the block."""
    train = _train()
    n = 3 * 256 + 100
    rng = np.random.default_rng(41)
    g = (rng.standard_normal(n) * 1e-3).astype(np.float32)
    g[256 + 77] = bad
    g[768 + 99] = bad  # the last, short block
    p, (m, v) = torch.zeros(n, device="cuda"), _fresh8(n)
    _say("adamw spoilt", bad)
    train.adamw_([p], [torch.from_numpy(g).cuda()], [m], [v], 1, lr=1e-3)
    with np.errstate(all="ignore"):
        _, m1, v1 = O.adamw(np.zeros(n), g, np.zeros(n), np.zeros(n), 1, 1e-3, (0.9, 0.95), 1e-8, 0.0)
        for got, new, which in ((m, m1, "m"), (v, v1, "v")):
            codes, scales = O.encode(new, which)
            assert np.array_equal(got[1].cpu().numpy(), scales, equal_nan=True), which
            want = O.decode(codes, scales)
            have = O.decode(got[0].cpu(), got[1].cpu().numpy())
            assert np.array_equal(have, want, equal_nan=True), which
    whole = torch.ones(n, dtype=torch.bool, device="cuda")
    whole[256:512] = whole[768:] = False
    assert not torch.isfinite(v[1][1]) and not torch.isfinite(v[1][3])
    train.adamw_([p], [torch.zeros(n, device="cuda")], [m], [v], 2, lr=1e-3)
    assert torch.isfinite(p[whole]).all() and torch.isnan(p[~whole]).all()


def test_adamw_neighbours_in_one_buffer_and_shared_gradients():
    """Tensors that touch without overlapping and gradients that two tensors share are as good as separate ones."""
    train = _train()
    rng = np.random.default_rng(43)
    new = lambda n: torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda()  # noqa: E731
    room, g = new(6 * 1000), new(1000)
    one = [t.abs() for t in room.split(1000)]
    room.abs_()
    parts = list(room.split(1000))
    for p in (one, parts):
        train.adamw_(p[:2], [g, g], p[2:4], p[4:], 3, lr=1e-2)
    assert all(torch.equal(a, b) for a, b in zip(one, parts))
    with pytest.raises((ValueError, RuntimeError)):
        train.adamw_([room[:1000], room[999:1999]], [g, g], [new(1000), new(1000)], [new(1000), new(1000)], 1, lr=1e-3)
    assert all(torch.equal(a, b) for a, b in zip(one, parts))


def test_adamw_refuses_copies_and_scales_given_twice():
    train = _train()
    new = lambda: torch.ones(300, device="cuda")  # noqa: E731
    copy = torch.ones(300, dtype=torch.bfloat16, device="cuda")
    p, q = new(), new()
    with pytest.raises(ValueError, match="twice"):
        train.adamw_([p, q], [new(), new()], [new(), new()], [new(), new()], 1, lr=1e-3, copies=[copy, copy])
    (m, v), (m2, v2) = _fresh8(300), _fresh8(300)
    with pytest.raises(ValueError, match="twice"):
        train.adamw_([p, q], [new(), new()], [m, (m2[0], m[1])], [v, v2], 1, lr=1e-3)
    with pytest.raises(ValueError, match="twice"):
        train.adamw_([p], [new()], [m], [(v[0], m[1])], 1, lr=1e-3)
    assert all(torch.equal(t.float(), torch.ones(300, device="cuda")) for t in (p, q, copy))


def test_adamw_class_goes_on_from_written_leaves():
    """Weights written into a bfloat16 leaf after the optimizer was made are the ones that the next step updates."""
    train = _train()
    rng = np.random.default_rng(47)
    leaf = torch.zeros(500, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    opt = train.AdamW([leaf], lr=1e-2)
    with torch.no_grad():
        leaf.copy_(torch.from_numpy(rng.standard_normal(500)))
    start = leaf.detach().float()
    leaf.grad = torch.from_numpy(rng.standard_normal(500)).to(torch.bfloat16).cuda()
    for _ in range(2):
        opt.step()
    p, m, v = _np(start), np.zeros(500), np.zeros(500)
    for t in (1, 2):
        p, m, v = O.adamw(p, _np(leaf.grad), m, v, t, 1e-2, (0.9, 0.95), 1e-8, 0.0)
    # each step moves by about 1e-2, off by some tens of roundings of it and of the parameter (below 4)
    assert np.max(np.abs(_np(opt.masters[0]) - p)) <= 2 * (2e-2 * 40 * E32 + 4 * 4 * E32)
    assert torch.equal(leaf.detach(), opt.masters[0].to(torch.bfloat16))
