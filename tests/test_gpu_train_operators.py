"""GPU parity of the training operators of the block's FFN half (RMSNorm, the
gated FFN, AdamW) against the float64 oracle on the same inputs.

Bars, with e = 2^-24 (half a float32 step relative to the value) and, for bf16
results and stored values, 2^-8 per rounding: a sum of n products is off by at
most (n + 2) e times the sum of their magnitudes in any order; the bounds below
carry that through each formula to first order, doubled for the higher orders
and for the elementary functions' last bits.  8-bit moments are compared code
for code, the kernel and the oracle both rounding float64 values."""
import numpy as np
import pytest

from oracle import train_operators as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E32, E16 = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5


def _train():
    from paper_2609_15160_amd import train
    return train


def _say(*what):
    print("[train-op]", *what, flush=True)


def _dt(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _np(t):
    return t.detach().double().cpu().numpy()


def _normal(rng, *shape, std=1.0, dtype="f32"):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(_dt(dtype)).cuda()


def _within(got, want, bound, what):
    got = _np(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    over = np.abs(got - want) - bound
    assert np.all(over <= 0), (what, float(np.max(over)), int(np.argmax(over)), float(np.max(np.abs(got - want))))


# ---------------------------------------------------------------------------
# RMSNorm
# ---------------------------------------------------------------------------

def _check_norm(rows, d, groups, xt, yt, seed=0, group=None, x=None):
    train = _train()
    rng = np.random.default_rng(seed + rows * 7 + d)
    _say("norm", rows, d, groups, xt, yt)
    x = _normal(rng, rows, d, std=1.5, dtype=xt) if x is None else x
    gamma = _normal(rng, groups, d, std=0.3) if groups else None
    if groups > 1 and group is None:
        group = torch.from_numpy(rng.integers(-1, groups + 1, rows).astype(np.int32)).cuda()  # some rows without a scale
    dy = _normal(rng, rows, d, dtype=yt)
    leaves = [t.requires_grad_() for t in (x, gamma) if t is not None]
    y = train.rms_norm(x, gamma, group, eps=EPS, dtype=_dt(yt))
    assert y.dtype == _dt(yt)
    got = torch.autograd.grad(y, leaves, dy)
    g_np = None if group is None else group.cpu().numpy()
    gm = None if gamma is None else _np(gamma)
    xs, dys = _np(x), _np(dy)
    want, r = O.rms_norm(xs, gm, g_np, EPS)
    half = lambda t: E16 if t == "bf16" else 0.0  # noqa: E731
    n = (d + 12) * E32  # relative error of r and of a row's mean product, as a share of the magnitudes
    _within(y, want, 2 * n * np.abs(want) + half(yt) * np.abs(want) * (1 + 1e-6) + 1e-30, "y")
    dx, dgamma = O.rms_norm_backward(dys, xs, gm, g_np, EPS)
    h = np.abs(dys * O.scale_rows(gm, g_np, rows, d))
    mag = r[:, None] * (h + np.abs(xs) * r[:, None] ** 2 * (h * np.abs(xs)).mean(1, keepdims=True)) if rows else h
    _within(got[0], dx, 4 * n * mag + half(xt) * np.abs(dx) * (1 + 1e-6) + 1e-30, "dx")
    if groups:
        _, mags = O.rms_norm_backward(np.abs(dys), np.abs(xs), gm, g_np, EPS)
        _within(got[1], dgamma, ((rows + 4) * E32 + n) * 2 * mags + 1e-30, "dgamma")


@pytest.mark.parametrize("rows,d", [(1, 4), (1, 768), (3, 60), (5, 260), (7, 516), (130, 1024), (67, 1028), (33, 2048),
                                    (9, 2052), (17, 4096)])
@pytest.mark.parametrize("groups", [0, 1, 5])
def test_norm(rows, d, groups):
    _check_norm(rows, d, groups, "f32", "bf16")


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,d,groups", [(300, 256, 16), (2049, 64, 2), (41, 1364, 0)])
def test_norm_types(xt, yt, rows, d, groups):
    _check_norm(rows, d, groups, xt, yt)


@pytest.mark.parametrize("rows,d,groups", [(50, 2048, 16), (70, 2304, 16), (100, 4096, 9), (61, 4096, 16), (5000, 8, 3)])
def test_norm_many_scales(rows, d, groups):
    """Sums of 128 to 256 KB, around what fits LDS, and many rows of few columns."""
    _check_norm(rows, d, groups, "f32", "bf16")


def test_norm_without_rows():
    train = _train()
    x, gamma = torch.zeros(0, 128, device="cuda", requires_grad=True), torch.ones(2, 128, device="cuda", requires_grad=True)
    y = train.rms_norm(x, gamma, torch.zeros(0, dtype=torch.int32, device="cuda"))
    dx, dg = torch.autograd.grad(y, (x, gamma), torch.zeros_like(y))
    assert y.shape == dx.shape == (0, 128) and torch.equal(dg, torch.zeros_like(gamma))


def test_norm_zero_rows_and_empty_groups():
    """Rows of zeros (r = 1 / sqrt(eps)), a group that no row has, gamma as a vector."""
    x = torch.zeros(6, 128, device="cuda")
    x[3] = 2.0
    group = torch.full((6,), 2, dtype=torch.int32, device="cuda")
    _check_norm(6, 128, 4, "f32", "f32", group=group, x=x)
    train = _train()
    gamma = torch.full((128,), 0.5, device="cuda", requires_grad=True)
    y = train.rms_norm(x.detach(), gamma)
    g, = torch.autograd.grad(y, gamma, torch.ones_like(y))
    assert g.shape == gamma.shape
    want = O.rms_norm_backward(np.ones((6, 128)), _np(x), _np(gamma), None, EPS)[1].reshape(128)
    _within(g, want, 200 * E32 * np.abs(want), "dgamma")


def test_norm_partial_gradients_and_strided_input():
    train = _train()
    rng = np.random.default_rng(5)
    wide = _normal(rng, 40, 512)
    x, gamma, dy = wide[1::2, 100:356], _normal(rng, 1, 256), _normal(rng, 20, 256)
    y = train.rms_norm(x, gamma.requires_grad_())
    g, = torch.autograd.grad(y, gamma, dy)
    z = x.contiguous().requires_grad_()
    y2 = train.rms_norm(z, gamma)
    gx, g2 = torch.autograd.grad(y2, (z, gamma), dy.t().contiguous().t())
    assert torch.equal(y, y2) and torch.equal(g, g2)
    gx2, = torch.autograd.grad(train.rms_norm(z, gamma.detach()), z, dy)
    assert torch.equal(gx, gx2)


# ---------------------------------------------------------------------------
# Gated FFN
# ---------------------------------------------------------------------------

def _ffn_bounds(x, wgu, wd, dy, t):
    """Bounds on the errors of y, dx, dw_gate_up, dw_down (first order, magnitudes in float64)."""
    A = np.abs
    f, d, n = wd.shape[1], wd.shape[0], x.shape[0]
    q = E16 if t == "bf16" else 0.0
    fn = 8 * E32  # exp, division and the products of the activation, relative
    g, u = x @ wgu[:f].T, x @ wgu[f:].T
    s = O.sigmoid(g)
    d1 = A(s * (1 + g * (1 - s)))                     # derivative of silu; its own derivative is at most 1/2
    eg, eu = (d + 2) * E32 * (A(x) @ A(wgu[:f]).T), (d + 2) * E32 * (A(x) @ A(wgu[f:]).T)
    a = g * s * u
    ea = d1 * eg * A(u) + A(g * s) * eu + fn * A(a) + q * A(a)
    ey = ea @ A(wd).T + (f + 2) * E32 * (A(a) @ A(wd).T) + q * A(a @ wd.T)
    da = dy @ wd
    eda = (d + 2) * E32 * (A(dy) @ A(wd))
    hg, hu = eg + q * A(g), eu + q * A(u)             # g and u as they are stored
    edg = eda * A(u) * d1 + A(da) * (hu * d1 + A(u) * 0.5 * hg) + (fn + q) * A(da * u) * (d1 + s * A(g) * E32 + s)
    edu = eda * A(g * s) + A(da) * d1 * hg + (fn + q) * A(da * g * s)
    dgu = np.concatenate([da * u * s * (1 + g * (1 - s)), da * g * s], 1)
    edgu = np.concatenate([edg, edu], 1)
    edx = edgu @ A(wgu) + (2 * f + 2) * E32 * (A(dgu) @ A(wgu)) + q * A(dgu @ wgu)
    egu = edgu.T @ A(x) + (n + 2) * E32 * (A(dgu).T @ A(x)) + q * A(dgu.T @ x)
    edn = A(dy).T @ ea + (n + 2) * E32 * (A(dy).T @ A(a)) + q * A(dy.T @ a)
    return [2 * e + 1e-30 for e in (ey, edx, egu, edn)]


def _ffn_inputs(n, d, f, t, seed=0):
    rng = np.random.default_rng(seed + n + d * 3 + f)
    return (_normal(rng, n, d, dtype=t), _normal(rng, 2 * f, d, std=1.5 / np.sqrt(d), dtype=t),
            _normal(rng, d, f, std=0.1, dtype=t), _normal(rng, n, d, std=0.1, dtype=t))


def _check_ffn(n, d, f, t, seed=0):
    train = _train()
    _say("ffn", n, d, f, t)
    x, wgu, wd, dy = _ffn_inputs(n, d, f, t, seed)
    leaves = [v.requires_grad_() for v in (x, wgu, wd)]
    y = train.ffn(x, wgu, wd)
    got = [y, *torch.autograd.grad(y, leaves, dy)]
    args = [_np(v) for v in (x, wgu, wd)]
    want = [O.ffn(*args), *O.ffn_backward(_np(dy), *args)]
    for name, a, b, e in zip(("y", "dx", "dw_gate_up", "dw_down"), got, want, _ffn_bounds(*args, _np(dy), t)):
        assert a.dtype == _dt(t)
        _within(a, b, e, name)
    with torch.no_grad():  # the same result where nothing is kept for a gradient
        assert torch.equal(train.ffn(x, wgu, wd), y)
    return got


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129, 257, 300])
def test_ffn_rows(t, n):
    _check_ffn(n, 128, 192, t)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,f", [(5, 64, 64), (70, 64, 256), (130, 320, 64), (40, 192, 448), (200, 704, 320),
                                   (77, 1024, 832)])
def test_ffn_widths(t, n, d, f):
    _check_ffn(n, d, f, t)


@pytest.mark.parametrize("t,n,d,f", [("bf16", 1500, 768, 2048), ("bf16", 2600, 512, 1344), ("f32", 1100, 256, 512),
                                     ("bf16", 5003, 256, 320), ("f32", 4100, 64, 128)])
def test_ffn_many_rows(t, n, d, f):
    """Rows enough for the large tiles and for weight gradients summed over several ranges of rows."""
    _check_ffn(n, d, f, t)


@pytest.mark.parametrize("t,n,d,f", [
    ("bf16", 6000, 512, 1856),   # the fused products on 256 x 256 tiles, a ragged last row of them
    ("bf16", 5300, 2048, 128),   # y and dx on 256 x 256 tiles, weight gradients of few tiles split by rows
    ("bf16", 40, 2048, 2560),    # the weight gradient on 256 x 256 tiles
    ("bf16", 2500, 2048, 64),    # y and dx on 128 x 128 tiles
    ("bf16", 3001, 640, 128),    # y and dx on 64 x 64 tiles, by four waves
    ("bf16", 20, 128, 4224),     # y and dx split over the compute units
    ("f32", 20, 128, 2304),      # the same in float32
    ("f32", 530, 64, 64),        # fewer steps than workgroups they are split over
])
def test_ffn_tile_shapes(t, n, d, f):
    _check_ffn(n, d, f, t)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_ffn_without_rows(t):
    train = _train()
    x, wgu, wd, dy = _ffn_inputs(0, 128, 64, t)
    leaves = [v.requires_grad_() for v in (x, wgu, wd)]
    y = train.ffn(x, wgu, wd)
    dx, a, b = torch.autograd.grad(y, leaves, dy)
    assert y.shape == dx.shape == (0, 128)
    assert torch.equal(a, torch.zeros_like(wgu)) and torch.equal(b, torch.zeros_like(wd))


@pytest.mark.parametrize("n", [40, 700])
def test_ffn_partial_gradients_are_the_same(n):
    train = _train()
    x, wgu, wd, dy = _ffn_inputs(n, 256, 320, "bf16")
    full = torch.autograd.grad(train.ffn(x.requires_grad_(), wgu.requires_grad_(), wd.requires_grad_()), (x, wgu, wd), dy)
    for k, leaf in enumerate((x, wgu, wd)):
        args = [v.detach() for v in (x, wgu, wd)]
        args[k] = leaf
        got, = torch.autograd.grad(train.ffn(*args), leaf, dy)
        assert torch.equal(got, full[k])


def test_ffn_extreme_gates():
    """Gates of +-100 and beyond exp's range, zero inputs: silu and its derivative saturate, no NaN."""
    train = _train()
    for t in ("bf16", "f32"):
        x = torch.zeros(4, 64, device="cuda", dtype=_dt(t))
        x[0, 0], x[1, 0], x[2, 0] = 100.0, -100.0, -2000.0
        wgu = torch.zeros(128, 64, device="cuda", dtype=_dt(t))
        wgu[:64, 0], wgu[64:, 0] = 1.0, 0.5
        wd = torch.eye(64, device="cuda", dtype=_dt(t))
        leaves = [v.requires_grad_() for v in (x, wgu, wd)]
        y = train.ffn(*leaves)
        got = [y, *torch.autograd.grad(y, leaves, torch.ones_like(y))]
        args = [_np(v) for v in leaves]
        with np.errstate(over="ignore"):
            want = [O.ffn(*args), *O.ffn_backward(np.ones((4, 64)), *args)]
        for a, b in zip(got, want):
            assert torch.isfinite(a).all()
            np.testing.assert_allclose(_np(a), b, rtol=4 * E16, atol=1e-30)


def test_ffn_rows_do_not_depend_on_each_other():
    """NaN in one row stays in its row of y and dx."""
    train = _train()
    x, wgu, wd, dy = _ffn_inputs(90, 128, 192, "bf16")
    clean = train.ffn(x, wgu, wd)
    x2 = x.clone()
    x2[37] = float("nan")
    x2.requires_grad_()
    y = train.ffn(x2, wgu, wd)
    dx, = torch.autograd.grad(y, x2, dy)
    rest = torch.arange(90, device="cuda") != 37
    assert torch.isnan(y[37]).all() and torch.equal(y[rest], clean[rest])
    assert torch.isnan(dx[37]).all() and torch.isfinite(dx[rest]).all()


def test_ffn_past_32_bit_offsets():
    """gu of 66000 x 33024 elements passes 2^31; sampled rows against the oracle, and the rows' gradient."""
    train = _train()
    n, d, f = 66000, 64, 16384
    rng = np.random.default_rng(3)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(n, d, generator=g, device="cuda").to(torch.bfloat16)
    wgu = (torch.randn(2 * f, d, generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    wd = (torch.randn(d, f, generator=g, device="cuda") * 0.05).to(torch.bfloat16)
    dy = torch.randn(n, d, generator=g, device="cuda").to(torch.bfloat16)
    _say("ffn", n, d, f, "bf16")
    x.requires_grad_()
    y = train.ffn(x, wgu, wd)
    dx, = torch.autograd.grad(y, x, dy)
    pick = np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, 6)]))
    at = torch.from_numpy(pick).cuda()
    args = [_np(x[at]), _np(wgu), _np(wd)]
    want, wdx = O.ffn(*args), O.ffn_backward(_np(dy[at]), *args)[0]
    bounds = _ffn_bounds(*args, _np(dy[at]), "bf16")
    _within(y[at], want, bounds[0], "y")
    _within(dx[at], wdx, bounds[1], "dx")


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------

def _state8(rng, n, which, std):
    v = rng.standard_normal(n) * std
    codes, scales = O.encode(v if which == "m" else v ** 2, which)
    return codes.cuda(), torch.from_numpy(scales).cuda()


def _decode(s):
    return O.decode(s[0].cpu(), s[1].cpu().numpy())


def _adamw_case(sizes, bits, gt, copies, step, lr=6e-4, betas=(0.9, 0.95), eps=1e-8, wd=0.1, seed=0, offset=0):
    train = _train()
    rng = np.random.default_rng(seed + sum(sizes))
    _say("adamw", sizes if len(sizes) < 8 else len(sizes), bits, gt, copies, step, offset)
    take = lambda t: t if not offset else torch.cat([t[:offset], t])[offset:]  # noqa: E731  (off a 16-byte boundary)
    p = [take(_normal(rng, n, std=0.02)) for n in sizes]
    g = [take(_normal(rng, n, std=1e-3, dtype=gt)) for n in sizes]
    c = [take(torch.zeros(n, dtype=torch.bfloat16, device="cuda")) for n in sizes] if copies else None
    if bits == 32:
        m = [take(_normal(rng, n, std=3e-4)) for n in sizes]
        v = [take(_normal(rng, n, std=1e-3).square()) for n in sizes]
        old = [(_np(a), _np(b)) for a, b in zip(m, v)]
    else:
        m, v = [_state8(rng, n, "m", 3e-4) for n in sizes], [_state8(rng, n, "v", 1e-3) for n in sizes]
        old = [(_decode(a), _decode(b)) for a, b in zip(m, v)]
    before = [_np(t) for t in p]
    train.adamw_(p, g, m, v, step, lr=lr, betas=betas, eps=eps, weight_decay=wd, copies=c)
    for k, n in enumerate(sizes):
        want, m1, v1 = O.adamw(before[k], _np(g[k]), *old[k], step, lr, betas, eps, wd)
        if bits == 32:
            em = 4 * E32 * (betas[0] * np.abs(old[k][0]) + (1 - betas[0]) * np.abs(_np(g[k])))
            _within(m[k], m1, em + 1e-44, "m")
            _within(v[k], v1, 5 * E32 * v1 + 1e-44, "v")
        else:
            em = 2 * E32 * np.abs(m1)
            for got, new, which in ((m[k], m1, "m"), (v[k], v1, "v")):
                codes, scales = O.encode(new, which)
                assert np.array_equal(got[1].cpu().numpy(), scales), which
                assert torch.equal(got[0].cpu().view(torch.uint8), codes.view(torch.uint8)), which
        root = np.sqrt(v1 / (1 - betas[1] ** step)) + eps
        move = lr / (1 - betas[0] ** step) / root
        ep = 4 * E32 * np.abs(before[k]) + move * em + 16 * E32 * move * np.abs(m1) + E32 * np.abs(want)
        _within(p[k], want, ep + 1e-44, "p")
        if copies:
            assert torch.equal(c[k], p[k].to(torch.bfloat16))
    return p, m, v


SIZES = [[1], [3, 255, 256, 257], [4095, 4096, 4097, 5, 1024], [70001]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gt,copies", [("f32", False), ("bf16", True)])
@pytest.mark.parametrize("sizes", SIZES)
def test_adamw(bits, gt, copies, sizes):
    _adamw_case(sizes, bits, gt, copies, step=7)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_adamw_unaligned(bits, offset):
    _adamw_case([9000, 300, 8192], bits, "bf16", True, step=2, offset=offset)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(step=1), dict(step=10 ** 6), dict(step=3, betas=(0.0, 0.5)), dict(step=2, wd=0.0, lr=0.0),
                                dict(step=5, eps=1e-2, wd=1.0, lr=0.5)])
def test_adamw_constants(bits, kw):
    _adamw_case([777, 5000], bits, "f32", False, **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_more_tensors_than_a_launch_takes(bits):
    _adamw_case([(17 * k) % 700 + 1 for k in range(131)], bits, "f32", True, step=4)


def test_adamw_eight_bit_corners():
    """Zero state and gradient, one large value beside tiny ones, a zero gradient on a filled state, blocks whose scale
    underflows."""
    train = _train()
    n = 1024
    g = np.zeros(n, np.float32)
    g[256], g[257:512] = 1.0, 1e-9
    g[512:768] = np.linspace(-1, 1, 256)
    g[768:] = 1e-24
    p = torch.zeros(n, device="cuda")
    m = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.zeros(4, device="cuda"))
    v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e5m2), torch.zeros(4, device="cuda"))
    om, ov, op = np.zeros(n), np.zeros(n), np.zeros(n)
    for t in range(1, 6):
        if t == 4:
            g = np.zeros(n, np.float32)
        train.adamw_([p], [torch.from_numpy(g).cuda()], [m], [v], t, lr=1e-3, eps=1e-8)
        op, om, ov = O.adamw(op, g, om, ov, t, 1e-3, (0.9, 0.95), 1e-8, 0.0)
        (cm, sm), (cv, sv) = O.encode(om, "m"), O.encode(ov, "v")
        assert np.array_equal(m[1].cpu().numpy(), sm) and np.array_equal(v[1].cpu().numpy(), sv)
        assert torch.equal(m[0].cpu().view(torch.uint8), cm.view(torch.uint8))
        assert torch.equal(v[0].cpu().view(torch.uint8), cv.view(torch.uint8))
        om, ov = O.decode(cm, sm), O.decode(cv, sv)
        assert torch.isfinite(p).all()
        # the bar of a step (below 2 lr each, 40 roundings) times the steps so far
        assert np.max(np.abs(_np(p) - op)) <= t * 2e-3 * 40 * E32
        assert not p[:256].any()


def test_adamw_class_against_its_steps():
    """bf16 leaves with masters beside float32 ones, a leaf without a gradient, 32 and 8 bits, state saved and loaded."""
    train = _train()
    rng = np.random.default_rng(11)
    for bits in (32, 8):
        leaves = [_normal(rng, 130, 64, std=0.02, dtype="bf16").requires_grad_(), _normal(rng, 77, std=0.02).requires_grad_(),
                  _normal(rng, 5, std=0.02).requires_grad_()]
        twin = [t.detach().clone().requires_grad_() for t in leaves]
        opt = train.AdamW(leaves, lr=1e-2, weight_decay=[0.1, 0.0, 0.0], state_bits=bits)
        two = train.AdamW(twin, lr=1e-2, weight_decay=[0.1, 0.0, 0.0], state_bits=bits)
        kept, fixed = leaves[2].detach().clone(), leaves[0].detach().float()
        p, m, v = _np(fixed).reshape(-1), np.zeros(130 * 64), np.zeros(130 * 64)
        for t in range(1, 4):
            for a, b in zip(leaves[:2], twin[:2]):
                a.grad = torch.randn(a.shape, device="cuda").to(a.dtype)
                b.grad = a.grad.clone()
            opt.step()
            if t == 2:  # the twin goes on from the first one's state
                for a, b in zip(leaves, twin):
                    b.data.copy_(a.data)
                two.load_state_dict(opt.state_dict())
            elif t == 3:
                two.step()
            p, m, v = O.adamw(p, _np(leaves[0].grad).reshape(-1), m, v, t, 1e-2, (0.9, 0.95), 1e-8, 0.1)
            if bits == 8:
                m, v = O.decode(*O.encode(m, "m")), O.decode(*O.encode(v, "v"))
        assert torch.equal(leaves[2].detach(), kept) and opt.steps == [3, 3, 0]
        # each of the three steps moves by at most about 1e-2 times a few and is off by some tens of roundings of it
        assert np.max(np.abs(_np(opt.masters[0]).reshape(-1) - p)) <= 3 * (0.1 * 40 * E32 + 4 * E32)
        assert torch.equal(leaves[0].detach(), opt.masters[0].to(torch.bfloat16))
        for a, b in zip(leaves, twin):
            assert torch.equal(a, b)


def test_adamw_update_is_noticed_by_a_saved_graph():
    train = _train()
    x, wgu, wd, dy = _ffn_inputs(8, 64, 64, "f32")
    wd.requires_grad_()
    y = train.ffn(x.requires_grad_(), wgu, wd)
    opt = train.AdamW([wd], lr=1e-3)
    wd.grad = torch.ones_like(wd)
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(dy)


# ---------------------------------------------------------------------------
# Together, on other streams, captured
# ---------------------------------------------------------------------------

def _chain(train, depth, H, gamma, wgu, wd, batch, seq, loops):
    h = H
    for i in range(1, loops + 1):
        p = train.plan(depth, batch, seq, i)
        x = train.gather(h, p)
        n = train.rms_norm(x, gamma, depth[p.index.long()] - 1, dtype=wgu.dtype)
        h = train.scatter(h, train.ffn(n, wgu, wd).float(), p)
    return h


def test_training_step_together():
    """Three loops of gather, norm by depth, FFN, scatter in float32, gradients of everything, one optimizer step:
    against the oracle's forward and backward in float64."""
    import synth
    from oracle import gather_scatter as G
    train = _train()
    B, T, d, f, R = 2, 75, 64, 128, 3
    rows = B * T
    m = synth.make_train_depths(rows, R, seed=21)
    rng = np.random.default_rng(22)
    H, gamma, wgu, wd, W = (_normal(rng, *s, std=v).requires_grad_() for s, v in
                            (((rows, d), 1.0), ((R, d), 0.2), ((2 * f, d), 0.15), ((d, f), 0.1), ((rows, d), 1.0)))
    W = W.detach()
    depth = torch.from_numpy(m).cuda()
    out = _chain(train, depth, H, gamma, wgu, wd, B, T, R)
    grads = torch.autograd.grad(out, (H, gamma, wgu, wd), W)

    h, saved = _np(H), []
    gm, ga, gb = _np(gamma), _np(wgu), _np(wd)
    for i in range(1, R + 1):
        idx = G.active_rows(m, i)
        x = G.gather(h, idx)
        n, _ = O.rms_norm(x, gm, m[idx] - 1, EPS)
        saved.append((idx, x, n))
        h = G.scatter(h, O.ffn(n, ga, gb), idx)
    np.testing.assert_allclose(_np(out), h, rtol=1e-4, atol=1e-5)
    dh, dgm, dga, dgb = _np(W), 0, 0, 0
    for idx, x, n in reversed(saved):
        prev, dy = G.scatter_backward(dh, idx)
        dn, a, b = O.ffn_backward(dy, n, ga, gb)
        dx, c = O.rms_norm_backward(dn, x, gm, m[idx] - 1, EPS)
        dga, dgb, dgm = dga + a, dgb + b, dgm + c
        dh = prev + G.gather_backward(dx, idx, rows)
    for got, want in zip(grads, (dh, dgm, dga, dgb)):
        np.testing.assert_allclose(_np(got), want, rtol=1e-3, atol=1e-4 * np.abs(want).max())

    opt = train.AdamW([gamma, wgu, wd], lr=1e-3, weight_decay=0.1)
    before = [_np(t) for t in opt.params]
    for t, g in zip(opt.params, grads[1:]):
        t.grad = g
    opt.step()
    for t, b, g in zip(opt.params, before, grads[1:]):
        want, _, _ = O.adamw(b, _np(g), np.zeros(b.size), np.zeros(b.size), 1, 1e-3, (0.9, 0.95), 1e-8, 0.1)
        np.testing.assert_allclose(_np(t).reshape(-1), want, rtol=1e-5, atol=1e-3 * 2e-5)


def test_operators_on_another_stream():
    train = _train()
    x, wgu, wd, dy = _ffn_inputs(500, 256, 320, "bf16")
    gamma = torch.full((1, 256), 0.1, device="cuda")

    def work():
        leaves = [t.detach().clone().requires_grad_() for t in (x, gamma, wgu, wd)]
        y = train.ffn(train.rms_norm(leaves[0], leaves[1]), leaves[2], leaves[3])
        return [y.detach(), *torch.autograd.grad(y, leaves, dy)]

    want = work()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [work() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for g in got:
        for a, b in zip(g, want):
            assert torch.equal(a, b)


def test_operators_replayed_from_a_graph():
    """norm, FFN and their gradients through the C ABI in a captured graph, several replays on new inputs with the
    program's own eager work in between: each equals the eager result to the bit."""
    import ctypes
    from paper_2609_15160_amd import tlf
    train = _train()
    lib = tlf.load()
    n, d, f, G = 1300, 256, 320, 3
    x, wgu, wd, dy = _ffn_inputs(n, d, f, "bf16")
    gamma = torch.randn(G, d, device="cuda") * 0.1
    group = torch.randint(0, G, (n,), device="cuda", dtype=torch.int32)
    new = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device="cuda")  # noqa: E731
    y, rstd, a, z = new(n, d), new(n, dt=torch.float32), new(n, f), new(n, d)
    gu = new(tlf.ffn_kept_bytes(tlf.DTYPE_BF16, n, f), dt=torch.uint8)
    dyn, dwgu, dwd, dx, dgamma = new(n, d), new(2 * f, d), new(d, f), new(n, d), new(G, d, dt=torch.float32)
    size = ctypes.c_size_t()
    assert lib.tlf_ffn_grad_ws_bytes(tlf.DTYPE_BF16, n, d, f, ctypes.byref(size)) == tlf.OK
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    assert lib.tlf_rms_norm_grad_ws_bytes(G, n, d, ctypes.byref(size)) == tlf.OK
    ws2 = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    P = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    B = tlf.DTYPE_BF16

    def calls():
        s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        return [lib.tlf_rms_norm(P(x), B, P(gamma), P(group), G, n, d, EPS, P(y), B, P(rstd), s),
                lib.tlf_ffn(P(y), P(wgu), P(wd), B, n, d, f, P(gu), P(a), P(z), P(ws), ws.numel(), s),
                lib.tlf_ffn_grad(P(dy), P(y), P(wgu), P(wd), P(gu), P(a), B, n, d, f, P(dyn), P(dwgu), P(dwd), P(ws),
                                 ws.numel(), s),
                lib.tlf_rms_norm_grad(P(dyn), B, P(x), B, P(gamma), P(group), G, P(rstd), n, d, P(dx), P(dgamma), P(ws2),
                                      ws2.numel(), s)]

    assert calls() == [tlf.OK] * 4
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert calls() == [tlf.OK] * 4
    for k in range(4):
        x.copy_(_ffn_inputs(n, d, f, "bf16", seed=100 + k)[0])
        for t in (y, z, dyn, dwgu, dwd, dx, dgamma):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (z, dwgu, dwd, dx, dgamma)]
        xl, gl, al, bl = (t.detach().clone().requires_grad_() for t in (x, gamma, wgu, wd))
        zz = train.ffn(train.rms_norm(xl, gl, group), al, bl)
        gx, gg, ga, gb = torch.autograd.grad(zz, (xl, gl, al, bl), dy)
        for p, q in zip(got, (zz, ga, gb, gx, gg)):
            assert torch.equal(p, q)


def test_adamw_is_refused_under_capture():
    train = _train()
    p, g, m, v = (torch.zeros(64, device="cuda") for _ in range(4))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.add_(1.0)
        with pytest.raises(RuntimeError, match="captured"):
            train.adamw_([p], [g], [m], [v], 1, lr=1e-3)
    graph.replay()
    assert torch.equal(p, torch.ones_like(p))


def test_rows_behind_the_last_stay_as_they_were():
    """Outputs handed in with room behind them: the calls write their rows and columns only."""
    import ctypes
    from paper_2609_15160_amd import tlf
    lib = tlf.load()
    n, d, f = 37, 192, 64
    x, wgu, wd, dy = _ffn_inputs(n, d, f, "bf16")
    room = lambda r, c, dt=torch.bfloat16: torch.full((r + 3, c), 7.0, dtype=dt, device="cuda")  # noqa: E731
    a, y, dx, dwgu, dwd, h = room(n, f), room(n, d), room(n, d), room(2 * f, d), room(d, f), room(n, d)
    kept = tlf.ffn_kept_bytes(tlf.DTYPE_BF16, n, f)
    gu = torch.full((kept + 64,), 7, dtype=torch.uint8, device="cuda")
    rstd = torch.full((n + 3,), 7.0, device="cuda")
    P = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    s, B = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), tlf.DTYPE_BF16
    size = ctypes.c_size_t()
    assert lib.tlf_ffn_grad_ws_bytes(B, n, d, f, ctypes.byref(size)) == tlf.OK
    ws = torch.full((size.value + 64,), 7, dtype=torch.uint8, device="cuda")
    assert lib.tlf_rms_norm(P(x), B, None, None, 0, n, d, EPS, P(h), B, P(rstd), s) == tlf.OK
    assert lib.tlf_ffn(P(x), P(wgu), P(wd), B, n, d, f, P(gu), P(a), P(y), P(ws), size.value, s) == tlf.OK
    assert lib.tlf_ffn_grad(P(dy), P(x), P(wgu), P(wd), P(gu), P(a), B, n, d, f, P(dx), P(dwgu), P(dwd), P(ws),
                            size.value, s) == tlf.OK
    for t in (a, y, dx, dwgu, dwd, h):
        assert (t[-3:] == 7.0).all() and torch.isfinite(t.float()).all()
    assert (rstd[-3:] == 7.0).all() and (ws[size.value:] == 7).all() and (gu[kept:] == 7).all()


def test_adamw_eight_bit_ties():
    """Many blocks: some maxima fall on a tie between two float32 values, which a fused product and sum would break
    another way than the formula's own order (seen in about one of 2500 blocks)."""
    rng = np.random.default_rng(31)
    train = _train()
    n = 256 * 20000
    p, g = torch.zeros(n, device="cuda"), _normal(rng, n, std=1e-3, dtype="bf16")
    m, v = [_state8(rng, n, w, s) for w, s in (("m", 3e-4), ("v", 1e-3))]
    om, ov = _decode(m), _decode(v)
    train.adamw_([p], [g], [m], [v], 9, lr=1e-3)
    _, m1, v1 = O.adamw(np.zeros(n), _np(g), om, ov, 9, 1e-3, (0.9, 0.95), 1e-8, 0.0)
    for got, new, which in ((m, m1, "m"), (v, v1, "v")):
        codes, scales = O.encode(new, which)
        assert np.array_equal(got[1].cpu().numpy(), scales), which
        assert torch.equal(got[0].cpu().view(torch.uint8), codes.view(torch.uint8)), which


@pytest.mark.parametrize("scaled", [False, True])
def test_norm_of_more_rows_than_a_launch(scaled):
    """2^26 + 5 rows of 4, past the rows of one launch.  The expected values are float64 of the same bfloat16 inputs,
    rounded to bfloat16 by the comparison: half a step, 2^-8, and 2^-16 for the kernel's float32 arithmetic (a chain of
    about ten roundings of 2^-24, amplified at most tenfold where dx's two terms cancel, held against the row's largest
    |h| r)."""
    train = _train()
    n, d = 2 ** 26 + 5, 4
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n, d, generator=gen, device="cuda", dtype=torch.bfloat16).requires_grad_()
    dy = torch.randn(n, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    gamma = torch.tensor([[0.5, -0.25, 0.0, 1.0], [-0.5, 0.75, 0.125, 2.0]], device="cuda").requires_grad_() if scaled else None
    group = torch.randint(0, 3, (n,), generator=gen, device="cuda", dtype=torch.int32) if scaled else None  # 2: none
    _say("norm", n, d, scaled)
    y = train.rms_norm(x, gamma, group)
    got = torch.autograd.grad(y, [x] + ([gamma] if scaled else []), dy)
    at = torch.cat([torch.arange(0, n, 1009, device="cuda")] +
                   [torch.arange(k * 2 ** 24 - 3, k * 2 ** 24 + 3, device="cuda") for k in (1, 2, 3, 4)] +
                   [torch.arange(n - 9, n, device="cuda")]).clamp(max=n - 1)
    xs, gs = x.detach()[at].double(), dy[at].double()
    gain = 1.0
    if scaled:
        gain = torch.cat([1.0 + gamma.detach().double(), torch.ones(1, d, device="cuda", dtype=torch.float64)])[group[at].long()]
    r = (xs.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    h = gs * gain
    want = xs * r * gain
    dx = r * (h - xs * r * r * (h * xs).mean(1, keepdim=True))
    assert ((y.detach()[at].double() - want).abs() <= want.abs() * (2 ** -8 + 2 ** -16)).all()
    assert ((got[0][at].double() - dx).abs() <= dx.abs() * (2 ** -8 + 2 ** -16) +
            2 ** -16 * (r * h.abs().amax(1, keepdim=True))).all()
    if scaled:
        # float32 sums of n products: each workgroup's run of rows adds one rounding per row to the sum of |terms| at
        # worst, of which 2^14 rows make 2^14 2^-24; rounding errors' signs are mixed, so this is a wide bound
        xr = x.detach().double()
        xr *= (xr.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        xr *= dy
        for k in (0, 1):
            one = xr * (group == k)[:, None]
            bound = one.abs().sum(0) * (2 ** 14 + 512) * 2 ** -24
            assert ((got[1][k].double() - one.sum(0)).abs() <= bound).all()


def test_adamw_refuses_a_tensor_given_twice():
    train = _train()
    p, q, g, m, v, m2 = (torch.zeros(64, device="cuda") for _ in range(6))
    with pytest.raises(ValueError, match="twice"):
        train.adamw_([p, p], [g, g], [m, m2], [v, q], 1, lr=1e-3)
    with pytest.raises(ValueError, match="twice"):
        train.adamw_([p, q], [g, g], [m, m], [v, m2], 1, lr=1e-3)
    assert not any(t.any() for t in (p, q, m, v, m2))
    empty = torch.zeros(0, device="cuda")
    train.adamw_([empty, empty], [empty, empty], [empty, empty], [empty, empty], 1, lr=1e-3)


def test_forward_and_backward_captured_together():
    """The operators and their gradients recorded into a graph by leaves that no other graph holds, replayed with new
    contents between eager calls on tensors of their own: the same to the bit."""
    train = _train()
    n, d, f = 200, 256, 320
    gen = torch.Generator(device="cuda").manual_seed(8)
    new = lambda *s, scale=1.0, t=torch.float32: (torch.randn(*s, generator=gen, device="cuda") * scale).to(t)  # noqa: E731
    make = lambda: [new(n, d), new(4, d, scale=0.3), new(2 * f, d, scale=0.1, t=torch.bfloat16),  # noqa: E731
                    new(d, f, scale=0.1, t=torch.bfloat16), new(n, d, t=torch.bfloat16)]
    group = torch.randint(0, 4, (n,), generator=gen, device="cuda", dtype=torch.int32)

    def step(x, gamma, wgu, wd, dy):
        y = train.ffn(train.rms_norm(x, gamma, group, dtype=torch.bfloat16), wgu, wd)
        return [y.detach(), *torch.autograd.grad(y, (x, gamma, wgu, wd), dy)]

    leaves = lambda ts: [t.clone().requires_grad_() for t in ts[:4]] + [ts[4].clone()]  # noqa: E731
    sets = [make() for _ in range(4)]
    want = [[t.clone() for t in step(*leaves(s))] for s in sets]
    held = leaves(sets[0])
    _say("capture", n, d, f)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for k in (1, 2, 3, 0):
        with torch.no_grad():
            for t, s in zip(held, sets[k]):
                t.copy_(s)
        graph.replay()
        step(*leaves(sets[(k + 1) % 4]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[k])), k


@pytest.mark.parametrize("t,n,d,f", [
    ("bf16", 1000, 768, 512),    # y and dx by 16 waves that share the sum
    ("bf16", 700, 1024, 64),     # the same, fewer steps than waves share
    ("bf16", 12, 768, 1024),     # y and dx in ranges, an uneven number of steps in each
    ("bf16", 600, 1024, 2624),   # the same with more tiles
    ("bf16", 1700, 768, 256),    # more tiles than compute units, by four waves
    ("f32", 3001, 256, 192),     # float32 by 16 waves
    ("f32", 300, 256, 512),      # float32 in ranges
    ("f32", 5000, 256, 64),      # float32 weight gradients in ranges for two workgroups on each compute unit
    ("f32", 257, 64, 64),        # and in ranges of 64 rows
])
def test_ffn_few_tiles(t, n, d, f):
    _check_ffn(n, d, f, t)


def test_gradients_of_gradients_are_refused():
    train = _train()
    x, w, v = (torch.randn(64, 64, device="cuda").requires_grad_() for _ in range(3))
    gu = torch.cat([w, v])
    for out in (train.rms_norm(x), train.ffn(x, gu, v)):
        one, = torch.autograd.grad(out, x, torch.ones_like(out), retain_graph=True)
        dx, = torch.autograd.grad(out, x, torch.ones_like(out), create_graph=True)
        assert torch.equal(one, dx)
        with pytest.raises(RuntimeError, match="gradients of gradients"):
            torch.autograd.grad(dx, x, torch.ones_like(dx))


@pytest.mark.parametrize("n,d,groups,xt,yt", [(70000, 1024, 8, "f32", "bf16"), (50000, 2048, 0, "bf16", "bf16"),
                                              (30000, 2052, 3, "f32", "f32")])
def test_norm_rows_of_a_large_call_as_of_a_small_one(n, d, groups, xt, yt):
    """Rows do not depend on how many there are: a call of more bytes than the caches hold against one of some of its
    rows, to the bit."""
    train = _train()
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, d, generator=gen, device="cuda").to(_dt(xt)).requires_grad_()
    dy = torch.randn(n, d, generator=gen, device="cuda").to(_dt(yt))
    gamma = torch.randn(groups, d, generator=gen, device="cuda").requires_grad_() if groups else None
    group = torch.randint(0, groups, (n,), generator=gen, device="cuda", dtype=torch.int32) if groups else None
    _say("norm", n, d, groups, xt, yt)
    at = torch.cat([torch.arange(5, device="cuda"), torch.randint(0, n, (200,), generator=gen, device="cuda"),
                    torch.arange(n - 5, n, device="cuda")])

    def both(x, dy, group):
        y = train.rms_norm(x, gamma, group, dtype=_dt(yt))
        return y.detach(), torch.autograd.grad(y, [x] + ([gamma] if groups else []), dy)[0]

    small = both(x.detach()[at].requires_grad_(), dy[at], None if group is None else group[at])
    for a, b in zip(both(x, dy, group), small):
        assert torch.equal(a[at], b)
