"""CPU pins of oracle/step_operators.py: attention against torch's softmax and autograd
in float64 and against hand-worked masks, the residual with its norm and the
gradient norm against torch and differences."""
import numpy as np
import pytest
import torch

from oracle import step_operators as O

RNG = np.random.default_rng


def test_visible_by_hand():
    assert O.visible(2, 5, 2, 1).astype(int).tolist() == [[1, 0, 1, 1, 0], [1, 0, 0, 1, 1]]
    assert O.visible(3, 2, None, 0).astype(int).tolist() == [[0, 0], [1, 0], [1, 1]]
    assert O.visible(2, 2, 1, 0).astype(int).tolist() == [[1, 0], [0, 1]]


@pytest.mark.parametrize("nq,n,heads,kv,window,sinks,scale", [
    (6, 6, 4, 2, None, 0, None), (6, 6, 2, 2, 3, 0, 0.7), (5, 9, 4, 1, 2, 2, None), (1, 12, 3, 3, 4, 1, None)])
def test_attention_against_autograd(nq, n, heads, kv, window, sinks, scale):
    r, D = RNG(nq + n), 8
    q, k, v, do = (torch.from_numpy(r.standard_normal(s)).requires_grad_() for s in
                   ((nq, heads, D), (n, kv, D), (n, kv, D), (nq, heads, D)))
    p, x = n - nq + torch.arange(nq)[:, None], torch.arange(n)[None, :]
    seen = (x <= p) & ((p - x < (n if window is None else window)) | (x < sinks))
    kk, vv = (t.repeat_interleave(heads // kv, 1) for t in (k, v))
    s = torch.einsum("qhd,khd->hqk", q, kk) * (D ** -0.5 if scale is None else scale)
    o = torch.einsum("hqk,khd->qhd", s.masked_fill(~seen, -torch.inf).softmax(-1), vv)
    want = torch.autograd.grad(o, (q, k, v), do.detach())
    a = [t.detach().numpy() for t in (q, k, v)]
    got = O.attention(*a, window, sinks, scale, do.detach().numpy())
    np.testing.assert_allclose(got["o"], o.detach().numpy(), rtol=1e-12, atol=1e-12)
    for name, w in zip(("dq", "dk", "dv"), want):
        np.testing.assert_allclose(got[name], w.numpy(), rtol=1e-11, atol=1e-11)


def test_attention_without_a_visible_key_and_with_unseen_infinities():
    r = RNG(1)
    q, k, v, do = r.standard_normal((4, 1, 8)), r.standard_normal((2, 1, 8)), r.standard_normal((2, 1, 8)), np.ones((4, 1, 8))
    got = O.attention(q, k, v, None, 0, None, do)
    assert not got["o"][:2].any() and not got["dq"][:2].any() and got["o"][2:].all()
    clean = O.attention(q[:3], k, v, None, 0, None, do[:3])
    v2 = v.copy()
    v2[1] = np.inf  # seen by the last query alone, which is not there
    again = O.attention(q[2:3], k[:1], v[:1], None, 0, None, do[2:3])
    assert np.array_equal(again["o"], O.attention(q[2:3], k[:1], v2[:1], None, 0, None, do[2:3])["o"])
    assert not np.isfinite(O.attention(q[:3], k, v2, 1, 0, None, do[:3])["o"][2]).any() and np.isfinite(clean["o"]).all()
    assert np.isfinite(O.attention(q[:3], k, v2, 1, 0, None, do[:3])["o"][1]).all()


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("groups", [0, 1, 3])
def test_residual_norm_against_autograd(post, groups):
    r = RNG(10 * groups + post)
    rows, d, eps = 6, 8, 1e-5
    t = lambda *s: torch.from_numpy(r.standard_normal(s)).requires_grad_()  # noqa: E731
    x, y, wh, wz = t(rows, d), t(rows, d), t(rows, d), t(rows, d)
    alpha, gamma = (t(groups, d), t(groups, d)) if groups else (None, None)
    group = r.integers(-1, groups + 1, rows) if groups > 1 else None
    take = lambda s: 1.0 if s is None else 1 + (s[0] if group is None else torch.stack(  # noqa: E731
        [s[g] if 0 <= g < groups else torch.zeros(d, dtype=torch.float64) for g in group]))
    h = x + take(alpha) * (y / torch.sqrt((y * y).mean(1, keepdim=True) + eps) if post else y)
    z = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * take(gamma)
    leaves = [s for s in (x, y, alpha, gamma) if s is not None]
    want = torch.autograd.grad((h * wh).sum() + (z * wz).sum(), leaves)
    n_ = lambda s: None if s is None else s.detach().numpy()  # noqa: E731
    got = O.residual_norm(n_(x), n_(y), n_(alpha), n_(gamma), group, eps, post, n_(wh), n_(wz))
    np.testing.assert_allclose(got["h"], n_(h), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(got["z"], n_(z), rtol=1e-12, atol=1e-12)
    for name, w in zip(("dx", "dy", "dalpha", "dgamma"), want):
        np.testing.assert_allclose(got[name], n_(w), rtol=1e-10, atol=1e-11)


@pytest.mark.parametrize("post", [False, True])
def test_residual_norm_gradients_against_differences(post):
    r = RNG(5)
    rows, d, eps, h = 3, 8, 1e-5, 1e-6
    x, y, wh, wz = (r.standard_normal((rows, d)) for _ in range(4))
    alpha, gamma = 0.3 * r.standard_normal((1, d)), 0.3 * r.standard_normal((1, d))
    args = {"x": x, "y": y, "alpha": alpha, "gamma": gamma}

    def loss(**kw):
        o = O.residual_norm(*[kw.get(name, a) for name, a in args.items()], None, eps, post)
        return (o["h"] * wh).sum() + (o["z"] * wz).sum()

    g = O.residual_norm(x, y, alpha, gamma, None, eps, post, wh, wz)
    for name, a in args.items():
        for at in [(0, 0), (a.shape[0] - 1, 5)]:
            up, down = a.copy(), a.copy()
            up[at] += h
            down[at] -= h
            # central differences of a smooth function: h^2 and rounding errors below 1e-8
            assert abs((loss(**{name: up}) - loss(**{name: down})) / (2 * h) - g["d" + name][at]) < 1e-7, (name, at)


def test_grad_norm():
    grads = [np.array([3.0, 0.0]), np.array([[4.0]])]
    assert O.grad_norm(grads) == (5.0, 1.0)
    assert O.grad_norm(grads, 5.0) == (5.0, 1.0) and O.grad_norm(grads, 2.5) == (5.0, 0.5)
