"""GPU parity of the gated residual with its norm, of the gradients' norm and of
clipped AdamW steps against the float64 oracle on the same inputs, and of a training
step of the block through all its operators.

Bars, with e = 2^-24 (half a float32 step relative to the value) and E = 2^-8 for
bf16 results: a sum of n products is off by at most (n + 2) e times the sum of their
magnitudes in any order; carried through the formulas to first order, doubled for
the higher orders and the square roots and divisions."""
import numpy as np
import pytest

from oracle import step_operators as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E32, E16 = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5


def _train():
    from paper_2609_15160_amd import train
    return train


def _say(*what):
    print("[step-op]", *what, flush=True)


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
# The gated residual and its norm
# ---------------------------------------------------------------------------

def _check_resid(rows, d, groups, yt, post, which="ag", seed=0, x=None, y=None, group=None, use="hz"):
    """`which` scales there are (a, g), `use`: the outputs that have a gradient."""
    train = _train()
    rng = np.random.default_rng(seed + rows * 7 + d)
    _say("residual", rows, d, groups, yt, "post" if post else "", which, use)
    x = _normal(rng, rows, d, std=1.5) if x is None else x
    y = _normal(rng, rows, d, std=0.7, dtype=yt) if y is None else y
    alpha = _normal(rng, groups, d, std=0.3) if groups and "a" in which else None
    gamma = _normal(rng, groups, d, std=0.3) if groups and "g" in which else None
    if groups > 1 and group is None:
        group = torch.from_numpy(rng.integers(-1, groups + 1, rows).astype(np.int32)).cuda()  # some rows without a scale
    dh, dz = _normal(rng, rows, d), _normal(rng, rows, d, dtype=yt)
    leaves = [t.requires_grad_() for t in (x, y, alpha, gamma) if t is not None]
    h, z = train.residual_norm(x, y, alpha, gamma, group, eps=EPS, post_norm=post)
    assert h.dtype == torch.float32 and z.dtype == y.dtype
    pick = [(t, g) for t, g, n in ((h, dh, "h"), (z, dz, "z")) if n in use]
    got = dict(zip([n for n, t in (("dx", x), ("dy", y), ("dalpha", alpha), ("dgamma", gamma)) if t is not None],
                   torch.autograd.grad([t for t, _ in pick], leaves, [g for _, g in pick])))
    n = None if group is None else group.cpu().numpy()
    an, gn = (None if t is None else _np(t) for t in (alpha, gamma))
    dhn, dzn = (_np(t) if c in use else np.zeros((rows, d)) for t, c in ((dh, "h"), (dz, "z")))
    xs, ys = _np(x), _np(y)
    w = O.residual_norm(xs, ys, an, gn, n, EPS, post, dhn, dzn)
    E, k = (E16 if yt == "bf16" else 0.0), (d + 16) * E32
    # h: y's r (k), then a product and a sum; z: h's error again and its r
    at = np.abs(w["a"] * w["t"])
    eh = 2 * (2 * E32 * (np.abs(xs) + at) + (k * at if post else 0.0))
    _within(h, w["h"], eh + 1e-30, "h")
    mean = lambda v: v.mean(1, keepdims=True)  # noqa: E731
    ah, r = np.abs(w["h"]), w["r"]
    er = 2 * k + r ** 2 * mean(ah * eh)  # relative, of r
    _within(z, w["z"], 2 * np.abs(w["c"]) * r * (eh + ah * er) + E * np.abs(w["z"]) * (1 + 1e-6) + 1e-30, "z")
    # gradients: magnitudes of every product, each off by 4 k and by what h and r are off
    u = np.abs(dzn * w["c"])
    mag = np.abs(dhn) + r * (u + ah * r ** 2 * mean(u * ah))
    off = r * (u * er + r ** 2 * (eh * mean(u * ah) + ah * mean(u * eh) + 3 * ah * er * mean(u * ah)))
    ex = 4 * k * mag + 2 * off
    _within(got["dx"], w["dx"], ex + 1e-30, "dx")
    aa, ay, ry = np.abs(w["a"]), np.abs(ys), w["ry"]
    if post:  # the mean of dt y is taken of two sums, of (dh + r u) a y and of h a y
        e, m = np.abs(dhn) + r * u, r ** 3 * mean(u * ah)
        two = mean(e * aa * ay) + m * mean(ah * aa * ay)
        ey = ry * (aa * ex + ay * ry ** 2 * (mean(aa * ex * ay) + 6 * k * two + 6 * er.max() * two)) + 6 * k * ry * (aa * mag + ay * ry ** 2 * two)
    else:
        ey = aa * ex + 4 * E32 * aa * mag
    _within(got["dy"], w["dy"], 2 * ey + E * np.abs(w["dy"]) * (1 + 1e-6) + 1e-30, "dy")
    for name, table, each, err in (("dalpha", alpha, mag * np.abs(w["t"]), ex * np.abs(w["t"]) + k * mag * np.abs(w["t"])),
                                   ("dgamma", gamma, np.abs(dzn) * ah * r, np.abs(dzn) * r * (eh + ah * er))):
        if table is not None:
            bound = O.by_group((rows + 6) * E32 * each + err, n, groups)
            _within(got[name], w[name], 2 * bound + 1e-30, name)


@pytest.mark.parametrize("rows,d", [(1, 4), (1, 768), (3, 60), (5, 260), (130, 1024), (67, 1028), (33, 2048), (9, 2052), (17, 4096)])
@pytest.mark.parametrize("groups", [0, 1, 5])
@pytest.mark.parametrize("post", [False, True])
def test_residual_norm(rows, d, groups, post):
    _check_resid(rows, d, groups, "bf16", post)


@pytest.mark.parametrize("rows,d,groups", [(300, 256, 16), (2049, 64, 2), (41, 1364, 9), (50, 2304, 16), (35, 4096, 8)])
@pytest.mark.parametrize("post", [False, True])
def test_residual_norm_float32_and_many_groups(rows, d, groups, post):
    _check_resid(rows, d, groups, "f32", post)


@pytest.mark.parametrize("which", ["a", "g"])
@pytest.mark.parametrize("groups", [1, 3, 12])
def test_residual_norm_with_one_scale(which, groups):
    _check_resid(77, 512, groups, "bf16", False, which)
    _check_resid(77, 512, groups, "bf16", True, which)


@pytest.mark.parametrize("use", ["h", "z"])
@pytest.mark.parametrize("post", [False, True])
def test_residual_norm_with_one_gradient(use, post):
    _check_resid(40, 256, 3, "bf16", post, use=use)
    _check_resid(40, 256, 0, "f32", post, use=use)


def test_residual_norm_zero_rows_and_empty_groups():
    x, y = torch.zeros(6, 128, device="cuda"), torch.zeros(6, 128, device="cuda")
    x[3], y[4] = 2.0, -1.0
    group = torch.full((6,), 2, dtype=torch.int32, device="cuda")
    for post in (False, True):
        _check_resid(6, 128, 4, "f32", post, x=x.clone(), y=y.clone(), group=group)


@pytest.mark.parametrize("yt", ["f32", "bf16"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("groups", [0, 1, 5, 12])
def test_residual_norm_gradients_of_small_eps_and_rows_far_from_one(monkeypatch, yt, post, groups):
    """The cube of 1 / sqrt(mean + eps) leaves float32's range while the gradients do not: rows of zeros with a small eps,
    rows of large values."""
    rng = np.random.default_rng(14)
    x, y = _normal(rng, 9, 260), _normal(rng, 9, 260, dtype=yt)
    x[:2], y[0], y[2] = 0.0, 0.0, 0.0
    with monkeypatch.context() as m:
        m.setitem(globals(), "EPS", 1e-28)
        _check_resid(9, 260, groups, yt, post, x=x.clone(), y=y.clone())
        _check_resid(9, 260, groups, yt, post, x=torch.zeros_like(x), y=torch.zeros_like(y), use="z")
    for std in (1e13, 1e16):
        _check_resid(9, 260, groups, yt, post, x=_normal(rng, 9, 260, std=std), y=_normal(rng, 9, 260, std=std, dtype=yt), use="z")


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("groups", [0, 3])
def test_residual_norm_past_32_bits_of_elements(post, groups):
    """The last rows of tensors of more than 2^31 elements, zeros before them: h, z and the rows' gradients to the bit those
    of the last rows alone; the scales' to the order of their sums, of which the zeros have no part."""
    train = _train()
    rows, few, d = 1060000, 100, 2048
    assert (rows - few) * d > 1 << 31
    _say("residual past 2^31 elements", rows, d, groups, post)
    rng = np.random.default_rng(15)
    part = [_normal(rng, few, d), _normal(rng, few, d, dtype="bf16"), _normal(rng, few, d), _normal(rng, few, d, dtype="bf16")]
    scales = [_normal(rng, groups, d, std=0.3) if groups else None for _ in range(2)]
    group = torch.from_numpy(rng.integers(0, groups, few).astype(np.int32)).cuda() if groups else None

    def behind(t):
        out = torch.zeros((rows, *t.shape[1:]), dtype=t.dtype, device="cuda")
        out[-few:] = t
        return out

    def run(x, y, dh, dz, group):
        leaves = [t.detach().clone().requires_grad_() if t is not None and t.shape[0] == groups else t for t in scales]
        x.requires_grad_(), y.requires_grad_()
        h, z = train.residual_norm(x, y, *leaves, group, post_norm=post)
        return h.detach(), z.detach(), *torch.autograd.grad((h, z), [x, y] + [t for t in leaves if t is not None], (dh, dz))

    want = run(*part, group)
    got = run(*[behind(t.detach()) for t in part], None if group is None else behind(group))
    for a, b in zip(got[:4], want[:4]):
        assert torch.equal(a[-few:], b)
    if groups:
        x, y, dh, dz = map(_np, part)
        w = O.residual_norm(x, y, *map(_np, scales), group.cpu().numpy(), EPS, post, dh, dz)
        for a, b, each in ((got[4], want[4], w["dx"] * w["t"]), (got[5], want[5], dz * w["h"] * w["r"])):
            mag = O.by_group(np.abs(each), group.cpu().numpy(), groups)
            assert np.all(np.abs(_np(a) - _np(b)) <= 2 * (few + 2) * E32 * 1.01 * mag)


def test_residual_norm_without_rows():
    train = _train()
    x, y = torch.zeros(0, 128, device="cuda", requires_grad=True), torch.zeros(0, 128, device="cuda", requires_grad=True)
    a, g = (torch.ones(2, 128, device="cuda", requires_grad=True) for _ in range(2))
    h, z = train.residual_norm(x, y, a, g, torch.zeros(0, dtype=torch.int32, device="cuda"))
    got = torch.autograd.grad((h, z), (x, y, a, g), (torch.zeros_like(h), torch.zeros_like(z)))
    assert h.shape == z.shape == got[0].shape == got[1].shape == (0, 128) and not got[2].any() and not got[3].any()


def test_residual_norm_strided_and_partial():
    """Rows that are not 16-byte aligned are copied; scales that need no gradient have none."""
    train = _train()
    rng = np.random.default_rng(5)
    wide = _normal(rng, 40, 515)
    x, y, a, g = wide[1::2, 3:259], _normal(rng, 20, 256, dtype="bf16"), _normal(rng, 256), _normal(rng, 256)
    h, z = train.residual_norm(x, y, a, g)
    w = O.residual_norm(_np(x), _np(y), _np(a), _np(g), None, EPS, False)
    assert np.abs(_np(h) - w["h"]).max() <= 4 * E32 * np.abs(w["h"]).max() * 4
    h, z = train.residual_norm(x, y.requires_grad_(), a, g)
    dy, = torch.autograd.grad(z, y, torch.ones_like(z))
    assert dy.shape == y.shape and not x.requires_grad
    dy2, da = torch.autograd.grad(train.residual_norm(x, y, a.requires_grad_(), g)[1], (y, a), torch.ones_like(z))
    assert torch.equal(dy, dy2) and da.shape == a.shape


def test_residual_norm_gradients_by_differences():
    train = _train()
    rng = np.random.default_rng(8)
    x, y, a, g = _normal(rng, 5, 64), _normal(rng, 5, 64), _normal(rng, 2, 64, std=0.3), _normal(rng, 2, 64, std=0.3)
    group = torch.tensor([0, 1, 1, 0, 1], dtype=torch.int32, device="cuda")
    ch, cz = _normal(rng, 5, 64), _normal(rng, 5, 64)
    leaves = [t.requires_grad_() for t in (x, y, a, g)]
    h, z = train.residual_norm(*leaves, group, eps=EPS, post_norm=True)
    got = torch.autograd.grad((h, z), leaves, (ch, cz))
    vals = [_np(t) for t in leaves]
    for k, t in enumerate(got):
        step = rng.standard_normal(vals[k].shape)
        f = []
        for s in (1e-5, -1e-5):
            v = [b + (s * step if i == k else 0) for i, b in enumerate(vals)]
            w = O.residual_norm(*v, group.cpu().numpy(), EPS, True)
            f.append((w["h"] * _np(ch)).sum() + (w["z"] * _np(cz)).sum())
        slope, have = (f[0] - f[1]) / 2e-5, (_np(t) * step).sum()
        # the gradients' float32 rounding, and the differences' third-order term and cancellation in float64
        assert abs(slope - have) <= 300 * E32 * np.abs(_np(t) * step).sum() + 1e-5, (k, slope, have)


# ---------------------------------------------------------------------------
# Gradient norm, clipping, clipped steps
# ---------------------------------------------------------------------------

def _grads(rng, sizes, types, std=1.0):
    return [_normal(rng, n, std=std, dtype=t) for n, t in zip(sizes, types)]


def _near(got, want, n_roundings=2):
    assert abs(float(got) - want) <= n_roundings * E32 * abs(want), (float(got), want)


@pytest.mark.parametrize("sizes", [[1], [7], [8192], [8193, 3, 0, 16384], [100003, 1, 65536], [5] * 400, [3000000]])
@pytest.mark.parametrize("types", [("f32",), ("bf16",), ("f32", "bf16")])
def test_grad_norm(sizes, types):
    """float64 sums: the norm is the oracle's rounded to float32, the scale one more rounding."""
    train = _train()
    _say("norm", sizes[:4], types)
    g = _grads(np.random.default_rng(len(sizes)), sizes, (types * len(sizes))[:len(sizes)], std=0.01)
    for limit in (None, 1e-3, 1e9):
        norm, scale = train.grad_norm(g, limit)
        want = O.grad_norm([_np(t) for t in g], limit)
        _near(norm, want[0])
        _near(scale, want[1])
        assert norm.shape == scale.shape == ()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", [0, 1, 3])
def test_clip_grad_norm(dtype, at):
    """In place, from any alignment, the neighbours left alone; within the limit nothing changes."""
    train = _train()
    rng = np.random.default_rng(9)
    whole = [_normal(rng, n, dtype=dtype) for n in (20000, 50, 8192 + at, 1 + at)]
    before = [t.clone() for t in whole]
    g = [t[at:] for t in whole]
    norm, want = train.clip_grad_norm_(g, 1e6), O.grad_norm([_np(t[at:]) for t in before], 5.0)
    _near(norm, want[0])
    assert all(torch.equal(a, b) for a, b in zip(whole, before))
    versions = [t._version for t in g]
    norm = train.clip_grad_norm_(g, 5.0)
    _near(norm, want[0])
    assert all(t._version > v for t, v in zip(g, versions))
    for t, b in zip(whole, before):
        assert torch.equal(t[:at], b[:at])
        w = _np(b[at:]) * want[1]
        _within(t[at:], w, ((E16 if dtype == "bf16" else 0.0) + 4 * E32) * np.abs(w) + 1e-40, "clipped")
    _near(train.grad_norm(g)[0], 5.0, 2 if dtype == "f32" else 2 ** 17)  # each by E at most: norm by E


def test_norms_at_the_ends_of_the_range():
    train = _train()
    big, small = torch.full((1000,), 3e38, device="cuda"), torch.full((1000,), 1e-40, device="cuda")
    norm, scale = train.grad_norm([big], 1.0)
    assert float(norm) == float("inf")  # 3e38 sqrt(1000) is none of float32's values; the scale is taken in float64
    # 1.05e-40 is subnormal: float32's steps there are 2^-149, a rounding is off by half of one
    assert abs(float(scale) - 1.0 / (float(np.float32(3e38)) * 1000 ** 0.5)) <= 2.0 ** -150
    norm, scale = train.grad_norm([small], 1.0)
    want = float(small[0].double()) * 1000 ** 0.5
    assert abs(float(norm) - want) <= 2.0 ** -149 and float(scale) == 1.0  # subnormal: half a step
    norm, scale = train.grad_norm([torch.zeros(10, device="cuda")], 1e-3)
    assert float(norm) == 0.0 and float(scale) == 1.0
    norm, scale = train.grad_norm([torch.zeros(0, device="cuda")], 1e-3)
    assert float(norm) == 0.0 and float(scale) == 1.0
    for bad in (float("nan"), float("inf")):
        g = torch.ones(9000, device="cuda")
        g[8999] = bad
        norm, scale = train.grad_norm([g, torch.ones(3, device="cuda")], 1.0)
        assert not np.isfinite(float(norm)) and (float(scale) == 0.0 if bad == float("inf") else np.isnan(float(scale)))


@pytest.mark.parametrize("limit", [None, float("inf"), 3.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scale_of_a_norm_that_is_not_finite(limit, dtype):
    """0 or NaN, whatever the limit: what takes the scale cannot take such gradients for good ones."""
    train = _train()
    for bad in (float("inf"), -float("inf"), float("nan")):
        g = torch.ones(20000, device="cuda", dtype=_dt(dtype))
        g[17] = bad
        norm, scale = train.grad_norm([torch.ones(3, device="cuda"), g], limit)
        assert not np.isfinite(float(norm)) and (np.isnan(float(scale)) or float(scale) == 0.0), (bad, float(scale))
    norm, scale = train.grad_norm([torch.ones(9, device="cuda", dtype=_dt(dtype))], limit)
    assert float(norm) == 3.0 and float(scale) == 1.0


def test_norm_of_views_that_overlap_and_clip_refuses_them():
    train = _train()
    from paper_2609_15160_amd import tlf
    t = torch.ones(100, device="cuda")
    assert float(train.grad_norm([t, t[50:]])[0]) == np.float32(150 ** 0.5)
    with pytest.raises(tlf.TlfError):
        train.clip_grad_norm_([t, t[50:]], 1.0)
    assert torch.equal(t, torch.ones_like(t))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_past_32_bits_of_elements(dtype):
    """Ones around element 2^31 and at the end of a longer tensor: counted by the norm, scaled by the clipping."""
    train = _train()
    _say("gradient past 2^31 elements", dtype)
    g = torch.zeros((1 << 31) + 20005, dtype=_dt(dtype), device="cuda")
    g[(1 << 31) - 8:(1 << 31) + 9], g[-8:] = 1.0, 1.0
    assert float(train.clip_grad_norm_([g], 2.5)) == 5.0
    assert bool((g[(1 << 31) - 8:(1 << 31) + 9] == 0.5).all() and (g[-8:] == 0.5).all())
    assert float(train.grad_norm([g])[0]) == 2.5


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_scaled_adamw_equals_the_step_on_scaled_gradients(bits, grad):
    """A scale that is a power of two makes the scaled gradients exact, so both steps are of the same gradients.  8-bit
    moments round products and sums by themselves: the same to the bit.  In float32 b m + c g may be fused from either
    product, so the two are off by at most one rounding of each product (2 e of the sum of magnitudes between them, twice
    over two steps), which the update p - rate m / (root v + eps) takes with 4 and 6 e of its size, 0.1 at most."""
    train = _train()
    rng = np.random.default_rng(3)
    sizes = [5000, 255, 1, 256 * 40 + 7]

    def state():
        r = np.random.default_rng(4)
        zeros = lambda n, t: (torch.zeros(n, dtype=torch.uint8, device="cuda").view(t), torch.zeros(-(-n // 256), device="cuda"))  # noqa: E731
        m = [torch.zeros(n, device="cuda") if bits == 32 else zeros(n, torch.float8_e4m3fn) for n in sizes]
        v = [torch.zeros(n, device="cuda") if bits == 32 else zeros(n, torch.float8_e5m2) for n in sizes]
        return [_normal(r, n) for n in sizes], m, v, [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes]

    g = [_normal(rng, n, std=0.1, dtype=grad) for n in sizes]
    a, b = state(), state()
    for step in (1, 2):
        train.adamw_(a[0], g, a[1], a[2], step, 1e-2, weight_decay=0.1, copies=a[3], grad_scale=torch.tensor(0.25, device="cuda"))
        train.adamw_(b[0], [t * 0.25 for t in g], b[1], b[2], step, 1e-2, weight_decay=0.1, copies=b[3])
    if bits == 32:
        for name, x, y in zip("pmvc", a, b):
            for i, (t, u) in enumerate(zip(x, y)):
                size = {"m": 0.9 * _np(b[1][i]).__abs__() + 0.1 * _np(g[i]).__abs__(), "v": _np(b[2][i])}
                mag = {"p": np.abs(_np(u)) + 0.1 * 10, "m": size["m"], "v": size["v"], "c": np.abs(_np(u)) * E16 / E32 + 1}[name]
                assert np.all(np.abs(_np(t) - _np(u)) <= 2 * 4 * E32 * mag), (name, i)
        return
    flat = lambda s: [u.view(torch.uint8) if u.element_size() == 1 else u for t in s for e in t for u in (e if isinstance(e, tuple) else (e,))]  # noqa: E731
    assert all(torch.equal(x, y) for x, y in zip(flat(a), flat(b)))


def test_scaled_adamw_against_the_formula():
    train = _train()
    rng = np.random.default_rng(6)
    p, g, m, v = _normal(rng, 4099), _normal(rng, 4099, std=0.1), _normal(rng, 4099, std=0.01), _normal(rng, 4099).square() * 1e-3
    p0, g0, m0, v0 = map(_np, (p, g, m, v))
    norm, scale = train.grad_norm([g], 0.5)
    train.adamw_([p], [g], [m], [v], 7, 1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, grad_scale=scale)
    s = O.grad_norm([g0], 0.5)[1]
    m1, v1 = 0.9 * m0 + 0.1 * s * g0, 0.95 * v0 + 0.05 * (s * g0) ** 2
    _within(m, m1, 8 * E32 * (np.abs(0.9 * m0) + np.abs(0.1 * s * g0)), "m")
    _within(v, v1, 12 * E32 * v1, "v")
    upd = 1e-2 * (m1 / (1 - 0.9 ** 7)) / (np.sqrt(v1 / (1 - 0.95 ** 7)) + 1e-8)
    mag = 1e-2 * ((np.abs(0.9 * m0) + np.abs(0.1 * s * g0)) / (1 - 0.9 ** 7)) / (np.sqrt(v1 / (1 - 0.95 ** 7)) + 1e-8)
    _within(p, p0 * (1 - 1e-3) - upd, 4 * E32 * np.abs(p0) + 40 * E32 * mag, "p")
    assert torch.equal(g.double().cpu(), torch.from_numpy(g0))


def test_optimizer_steps_with_a_limit():
    """AdamW.step(max_norm): the leaves as with gradients clipped beforehand, the gradients left, the norm returned."""
    train = _train()
    rng = np.random.default_rng(2)
    shapes = [(300, 64), (64,), (1000,)]

    def make():
        r = np.random.default_rng(1)
        return [_normal(r, *s, dtype=t).requires_grad_() for s, t in zip(shapes, ("f32", "f32", "bf16"))]

    a, b = make(), make()
    oa, ob = train.AdamW(a, 1e-2), train.AdamW(b, 1e-2)
    assert oa.step(max_norm=1.0) is None  # no gradients yet
    for k in range(3):
        g = [_normal(rng, *s, std=10.0 ** k, dtype=t) for s, t in zip(shapes, ("f32", "f32", "bf16"))]
        for p, q, t in zip(a, b, g):
            p.grad, q.grad = t.clone(), t.clone()
        norm = oa.step(max_norm=20.0)
        assert all(torch.equal(p.grad, t) for p, t in zip(a, g))
        want = O.grad_norm([_np(t) for t in g], 20.0)
        _near(norm, want[0])
        for q, t in zip(b, g):  # the clipped gradients in float32, without a rounding to bf16
            q.grad = None
        ob_grads = [t.float() * float(np.float32(want[1])) for t in g]
        train.adamw_([ob.masters[i] if ob.masters[i] is not None else b[i].detach() for i in range(3)], ob_grads, ob.exp_avgs,
                     ob.exp_avg_sqs, k + 1, 1e-2)
    for i, (p, q) in enumerate(zip(a, b)):
        x, y = (oa.masters[i], ob.masters[i]) if oa.masters[i] is not None else (p, q)
        # both scales are the norm's quotient to one float32 rounding: moments by 4 e, each of 3 steps of at most 1e-2 by 16 e
        assert float((x.detach().double() - y.detach().double()).abs().max()) <= 3 * (E32 * 16) * 4
    with pytest.raises(ValueError, match="max_norm"):
        a[0].grad = torch.ones_like(a[0])
        oa.step(max_norm=0.0)


def test_two_streams_and_another_current_stream():
    train = _train()
    rng = np.random.default_rng(0)
    g = [_normal(rng, 100000), _normal(rng, 777, dtype="bf16")]
    want = float(train.grad_norm(g, 1.0)[0])
    x, y = _normal(rng, 3000, 256), _normal(rng, 3000, 256, dtype="bf16")
    h0, z0 = train.residual_norm(x, y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append((train.grad_norm(g, 1.0), train.residual_norm(x, y)))
    torch.cuda.synchronize()
    for (norm, _), (h, z) in got:
        assert float(norm) == want and torch.equal(h, h0) and torch.equal(z, z0)


# ---------------------------------------------------------------------------
# A training step of the block through all of them
# ---------------------------------------------------------------------------

class _Block:
    """One layer of the shared block with AdaLN scales: the operators, or (plain) float64 torch."""
    heads, kv, width, f, d, groups = 4, 2, 64, 128, 256, 4

    def __init__(self, dtype, seed=0):
        rng = np.random.default_rng(seed)
        qkv = (self.heads + 2 * self.kv) * self.width
        shapes = {"qkv": (qkv, self.d), "o": (self.d, self.heads * self.width), "gu": (2 * self.f, self.d), "down": (self.d, self.f)}
        self.w = {k: _normal(rng, *s, std=0.05, dtype=dtype).requires_grad_() for k, s in shapes.items()}
        for k in ("alpha_msa", "gamma_msa", "alpha_mlp", "gamma_mlp"):
            self.w[k] = _normal(rng, self.groups, self.d, std=0.2).requires_grad_()
        self.dtype = _dt(dtype)

    def __call__(self, h, plans, depth):
        train = _train()
        w = self.w
        for p in plans:
            x = train.gather(h, p)
            group = depth[p.index.long()] - 1
            y = train.rms_norm(x, w["gamma_msa"], group, dtype=self.dtype)
            o = train.self_attention(y @ w["qkv"].T, p.offsets, self.heads, self.kv, window=9, sinks=2)
            x2, z = train.residual_norm(x, o @ w["o"].T, w["alpha_msa"], w["gamma_mlp"], group)
            x3, _ = train.residual_norm(x2, train.ffn(z, w["gu"], w["down"]), w["alpha_mlp"], None, group)
            h = train.scatter(h, x3 - x, p)
        return h

    def plain(self, h, leaves, plans, depth):
        w = leaves
        norm = lambda t: t * (t.square().mean(1, keepdim=True) + 1e-5).rsqrt()  # noqa: E731
        for p in plans:
            idx = p.index.long()
            x, group = h[idx], (depth[idx] - 1).long()
            qkv = (norm(x) * (1 + w["gamma_msa"][group])) @ w["qkv"].T
            outs, at = [], p.offsets.tolist()
            for a, b in zip(at, at[1:]):
                if a == b:
                    continue
                t = qkv[a:b].reshape(b - a, self.heads + 2 * self.kv, self.width).transpose(0, 1)
                q, k, v = t[:self.heads], t[self.heads:self.heads + self.kv], t[self.heads + self.kv:]
                k, v = (u.repeat_interleave(self.heads // self.kv, 0) for u in (k, v))
                i = torch.arange(b - a, device=h.device)
                u = i[:, None] - i[None, :]
                s = (q @ k.transpose(1, 2)) / 8.0
                s = s.masked_fill(~((u >= 0) & ((u < 9) | (i[None, :] < 2))), float("-inf"))
                outs.append((torch.softmax(s, -1) @ v).transpose(0, 1).reshape(b - a, -1))
            x2 = x + (1 + w["alpha_msa"][group]) * (torch.cat(outs) @ w["o"].T)
            z = norm(x2) * (1 + w["gamma_mlp"][group])
            g, u = (z @ w["gu"].T).chunk(2, 1)
            x3 = x2 + (1 + w["alpha_mlp"][group]) * ((torch.nn.functional.silu(g) * u) @ w["down"].T)
            h = h.index_add(0, idx, x3 - x)
        return h


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_step_of_the_block(dtype):
    """Two loops over ragged sequences, loss, gradients, a clipped step.  The whole's gradients against float64: each
    of some 20 roundings on the way is E (or, of float32 tensors, sums of up to 640 products with 640 e) of its
    value in norm; twice their sum."""
    train = _train()
    rng = np.random.default_rng(11)
    B, T, d = 3, 37, _Block.d
    depth = torch.from_numpy(rng.integers(1, 5, B * T).astype(np.int32)).cuda()
    depth[T:2 * T] = 1  # one sequence has no rows in the second loop
    plans = [train.plan(depth, B, T, i) for i in (1, 2)]
    h = _normal(rng, B * T, d).requires_grad_()
    c = _normal(rng, B * T, d)
    block = _Block(dtype)
    out = block(h, plans, depth)
    names = list(block.w)
    got = torch.autograd.grad((out * c).sum(), [h] + [block.w[k] for k in names])
    h64 = h.detach().double().requires_grad_()
    w64 = {k: t.detach().double().requires_grad_() for k, t in block.w.items()}
    ref = block.plain(h64, w64, plans, depth)
    want = torch.autograd.grad((ref * c.double()).sum(), [h64] + [w64[k] for k in names])
    tol = 2 * 20 * (E16 if dtype == "bf16" else 640 * E32)
    for name, a, b in zip(["out", "h"] + names, [out, *got], [ref, *want]):
        rel = float((a.double() - b).norm() / b.norm())
        print("[step-op] block", dtype, name, "%.2g" % rel, "of", tol, flush=True)
        assert rel <= tol, (name, rel)
    leaves = [block.w[k] for k in names]
    opt = train.AdamW(leaves, 1e-3)
    for t, g in zip(leaves, got[1:]):
        t.grad = g
    before = [t.detach().clone() for t in leaves]
    norm = opt.step(max_norm=0.1)
    _near(norm, O.grad_norm([_np(g) for g in got[1:]])[0])
    assert all(not torch.equal(a, b) for a, b in zip(before, leaves))


def test_captured_and_replayed_with_its_gradients():
    """Attention, residual and norm, forward and backward, in one graph: every replay equals the eager result on the
    inputs of that replay, with eager work between."""
    train = _train()
    rng = np.random.default_rng(12)
    offsets = torch.tensor([0, 30, 30, 97], dtype=torch.int32, device="cuda")
    qkv = _normal(rng, 100, 3 * 128, dtype="bf16").requires_grad_()
    x = _normal(rng, 100, 128).requires_grad_()
    c, g = _normal(rng, 100, 128), _normal(rng, 300)

    def run():
        o = train.self_attention(qkv, offsets, 2, window=20, sinks=3)
        h, z = train.residual_norm(x, o)
        grads = torch.autograd.grad((h, z), (qkv, x), (c, c.to(torch.bfloat16)))
        return (h, z, *grads, *train.grad_norm([g, grads[1]], 1.0))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for k in range(4):
        with torch.no_grad():
            qkv.copy_(_normal(rng, 100, 3 * 128, dtype="bf16"))
            offsets.copy_(torch.tensor([0, 30 + k, 40 + k, 97 - k], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in out]
        want = run()
        assert all(torch.equal(a, b) for a, b in zip(have, want)), k
