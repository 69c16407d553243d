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


# ---------------------------------------------------------------------------
# Every kernel of the FFN and of the norm, at sizes that select it
# ---------------------------------------------------------------------------

FFN_SHAPES = [
    # bf16: gate/up, da, y, dx and the weights' gradients of 256 x 256 ...
    (6000, 512, 1856), (5500, 2048, 128), (40, 2048, 2560), (5300, 2048, 128),
    # ... of 128 x 128, the last for the weights' gradients ...
    (2600, 768, 2048), (2500, 2048, 64), (1500, 768, 2048), (333, 2048, 2048),
    # ... and of 64 x 64: by four waves, by 16, in ranges
    (3001, 640, 128), (1000, 768, 512), (20, 128, 4224), (5003, 256, 320),
]
FFN_SHAPES_F32 = [(1, 64, 64), (3001, 256, 192), (3001, 256, 512), (300, 256, 512), (5000, 256, 64), (20, 128, 2304),
                  (530, 64, 64)]


def _ffn_operands(n, d, f, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + n + 3 * d + f)
    new = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device="cuda") * std).to(dtype)  # noqa: E731
    return new(n, d), new(2 * f, d, std=1.5 / d ** 0.5), new(d, f, std=0.1), new(n, d, std=0.1)


def _ffn_and_gradients(x, wgu, wd, dy):
    leaves = [t.detach().requires_grad_() for t in (x, wgu, wd)]
    y = _train().ffn(*leaves)
    return (y.detach(), *torch.autograd.grad(y, leaves, dy))


@pytest.mark.parametrize("n,d,f", FFN_SHAPES)
def test_ffn_is_its_formula_with_its_roundings(n, d, f):
    """Each result in norm against float64 with the documented roundings at their places.  What is left is where a
    float32 sum falls to the other side of a rounding: its error is about sqrt(K) 2^-24 of a sum of K terms (K up to
    6000: 5e-6 relative to the value), so a value of 8 bits, steps of 2^-7 to 2^-8, flips with a probability of at most
    2 x 5e-6 / 2^-8 = 2.4e-3 by one step: sqrt(2.4e-3) 2^-8 = 2e-4 in norm, 4e-4 with three such roundings in a row and a
    kept value's; 2^-10 is the bar.  Keeping 8 bits instead of 10, or leaving out a row, moves more than that
    (test_oracle_train_operators.py)."""
    _say("ffn formula", n, d, f)
    x, wgu, wd, dy = _ffn_operands(n, d, f, torch.bfloat16)
    dy2 = dy.clone()
    dy2[: n - n % 64] = 0  # the weights' gradients from the rows of the last, short stage alone
    for dy in [dy] + ([dy2] if n % 64 else []):
        got = _ffn_and_gradients(x, wgu, wd, dy)
        for name, a, b in zip(("y", "dx", "dw_gate_up", "dw_down"), got, O.ffn_rounded(dy, x, wgu, wd)):
            off = float((a.double() - b).norm() / b.norm())
            _say(name, f"{off:.1e}")
            assert off <= 2.0 ** -10, (name, off)


def _kernels(prefix, calls):
    """Names of the kernels, of those whose name has the prefix, that the calls launch, and of those in the library."""
    import re
    import subprocess
    from paper_2609_15160_amd import tlf
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        for call in calls:
            call()
        torch.cuda.synchronize()
    with open(tlf.LIB_PATH, "rb") as f:
        built = {m.decode() for m in re.findall(rb"_ZN3tlf12_GLOBAL__N_1\d+" + prefix.encode() + rb"\w*", f.read())}
    names = sorted(n for n in built if "device_stub" not in n)
    plain = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True).stdout.split("\n")
    known = dict(zip(names, names)) | dict(zip(plain, names))
    return {known[e.name] for e in prof.events() if e.name in known}, set(names)


def test_every_ffn_kernel_is_reached():
    """The sizes above, and those of float32, launch every tile shape, transposition, epilogue and split there is."""
    _say("ffn kernels")
    calls = [lambda s=s, t=t: _ffn_and_gradients(*_ffn_operands(*s, t)) for t, shapes in
             ((torch.bfloat16, FFN_SHAPES), (torch.float32, FFN_SHAPES_F32)) for s in shapes]
    ran, built = _kernels("k_ffn", calls)
    assert len(built) >= 30 and ran == built, sorted(built - ran)


# Widths of 1, 2, 4, 8 and 16 vectors of a lane; one wave to sixteen for the sums of gamma's gradient.
NORM_TYPES = [(a, b) for a in (torch.float32, torch.bfloat16) for b in (torch.float32, torch.bfloat16)]
NORM_WIDTHS = [(256, (0,)), (512, (0,)), (1024, (0, 1, 8, 16)), (2048, (0, 1, 8, 16)), (4096, (0, 1, 8, 16))]
MANY = 300 << 20  # bytes of x and y, above what the rows of a call may have to be read through the caches


def _norm_operands(bytes_, d, groups, xt, yt):
    n = bytes_ // (d * (xt.itemsize + yt.itemsize)) | 1
    gen = torch.Generator(device="cuda").manual_seed(n + d + groups)
    new = lambda t, *s: torch.randn(*s, generator=gen, device="cuda").to(t)  # noqa: E731
    gamma = new(torch.float32, groups, d) * 0.3 if groups else None
    # with one group too, some rows belong to none
    group = torch.randint(-1, groups + 1, (n,), generator=gen, device="cuda", dtype=torch.int32) if groups else None
    return new(xt, n, d), gamma, group, new(yt, n, d)


def _norm_and_gradients(x, gamma, group, dy):
    leaves = [t.detach().requires_grad_() for t in (x, gamma) if t is not None]
    y = _train().rms_norm(leaves[0], leaves[1] if gamma is not None else None, group, dtype=dy.dtype)
    return (y.detach(), *torch.autograd.grad(y, leaves, dy))


@pytest.mark.parametrize("xt,yt", NORM_TYPES)
@pytest.mark.parametrize("d,groups", [(d, k) for d, ks in NORM_WIDTHS for k in ks])
def test_norm_of_many_bytes(xt, yt, d, groups):
    """A call of more bytes than the caches hold: its rows to the bit as those of a small call, which is held against
    float64 here; gamma's gradient against float64 over all rows.  The sum of a column goes over at most rows / 256 + 8
    rows in order, then 128 partial sums; r is off by (d + 12) 2^-24 of it."""
    _say("norm", d, groups, xt, yt)
    x, gamma, group, dy = _norm_operands(MANY, d, groups, xt, yt)
    n = x.shape[0]
    gen = torch.Generator(device="cuda").manual_seed(d + groups)
    at = torch.cat([torch.arange(9, device="cuda"), torch.randint(0, n, (100,), generator=gen, device="cuda"),
                    torch.arange(n - 9, n, device="cuda")])
    some = (x[at], gamma, None if group is None else group[at], dy[at])
    large, small = _norm_and_gradients(x, gamma, group, dy), _norm_and_gradients(*some)
    assert torch.equal(large[0][at], small[0]) and torch.equal(large[1][at], small[1])
    xs, gs = some[0].double(), some[3].double()
    gain = torch.ones_like(xs)
    if groups:
        known = (some[2] >= 0) & (some[2] < groups)
        gain[known] += gamma.double()[some[2][known].long()]
    r = (xs.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    h, e = gs * gain, (d + 12) * E32
    want, dx = xs * r * gain, r * (h - xs * r * r * (h * xs).mean(1, keepdim=True))
    mag = r * (h.abs() + xs.abs() * r * r * (h * xs).abs().mean(1, keepdim=True))
    half = lambda t: E16 if t == torch.bfloat16 else E32  # noqa: E731
    assert ((small[0].double() - want).abs() <= want.abs() * (2 * e + half(yt) * 1.001)).all()
    assert ((small[1].double() - dx).abs() <= 4 * e * mag + dx.abs() * half(xt) * 1.001).all()
    if groups:
        xr = x.double()
        xr *= (xr.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        xr *= dy
        for k in range(groups):
            one = xr[group == k]
            bound = one.abs().sum(0) * (n / 256 + 8 + 128 + d + 16) * E32
            assert ((large[2][k].double() - one.sum(0)).abs() <= bound).all(), k


def test_every_norm_kernel_is_reached():
    _say("norm kernels")
    calls = [lambda a=(b, d, k, xt, yt): _norm_and_gradients(*_norm_operands(*a))
             for b in (1 << 20, MANY) for d, ks in NORM_WIDTHS for k in ks for xt, yt in NORM_TYPES]
    ran, built = _kernels("k_norm", calls)
    assert len(built) >= 100 and ran == built, sorted(built - ran)


def test_ffn_weight_gradients_past_32_bit_offsets():
    """[dg | du] of 66000 x 32768 passes 2^31 elements, and 2^32 bytes lie before its last rows: the weights' gradients,
    which read it and `a` with rows as the sum, against float64 products of the formula's dg, du and a (as it rounds
    them) in columns from both ends of each half; y and dx of the last rows."""
    n, d, f = 66000, 64, 16384
    x, wgu, wd, dy = _ffn_operands(n, d, f, torch.bfloat16)
    _say("ffn", n, d, f)
    y, dx, dwgu, dwd = _ffn_and_gradients(x, wgu, wd, dy)
    pick = torch.tensor([0, 1, 77, 4095, 8192, f - 65, f - 2, f - 1], device="cuda")
    # the formula of these columns alone: their gates and ups, their part of W_down
    _, _, want_gu, want_d = O.ffn_rounded(dy, x, torch.cat([wgu[pick], wgu[f + pick]]), wd[:, pick].contiguous())
    for name, a, b in (("dw_gate", dwgu[pick], want_gu[:8]), ("dw_up", dwgu[f + pick], want_gu[8:]),
                       ("dw_down", dwd[:, pick], want_d)):
        off = float((a.double() - b).norm() / b.norm())
        _say(name, f"{off:.1e}")
        assert off <= 2.0 ** -10, name
    part = torch.arange(n - 300, n, device="cuda")
    want_y, want_dx, _, _ = O.ffn_rounded(dy[part], x[part], wgu, wd)
    for name, a, b in (("y", y[part], want_y), ("dx", dx[part], want_dx)):
        assert float((a.double() - b).norm() / b.norm()) <= 2.0 ** -10, name


def test_adamw_class_refused_under_capture_loses_no_written_leaf():
    """A step that is refused because it is captured takes nothing: the next one still goes on from the written leaf."""
    train = _train()
    leaf = torch.zeros(256, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    opt = train.AdamW([leaf], lr=0.0)
    leaf.grad = torch.ones_like(leaf)
    with torch.no_grad():
        leaf.fill_(3.0)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph):
        other.add_(1.0)
        with pytest.raises(RuntimeError, match="captured"):
            opt.step()
    opt.step()
    assert torch.equal(opt.masters[0], torch.full((256,), 3.0, device="cuda")) and opt.steps == [1]
    assert torch.equal(leaf.detach().float(), opt.masters[0])
