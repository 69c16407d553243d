"""CPU pins of oracle/train_operators.py: gradients against differences and
against torch's autograd in float64, AdamW against its own definition run over
several steps by torch, the 8-bit formats against hand-worked values."""
import numpy as np
import pytest
import torch

from oracle import train_operators as O

RNG = np.random.default_rng


def _difference(f, x, at, h=1e-6):
    a, b = x.copy(), x.copy()
    a[at] += h
    b[at] -= h
    return (f(a) - f(b)) / (2 * h)


@pytest.mark.parametrize("groups", [0, 1, 3])
def test_norm_gradients_against_differences(groups):
    r = RNG(groups)
    rows, d, eps = 5, 8, 1e-5
    x, w = r.standard_normal((rows, d)), r.standard_normal((rows, d))
    gamma = r.standard_normal((groups, d)) * 0.3 if groups else None
    group = r.integers(-1, groups + 1, rows) if groups > 1 else None
    dx, dgamma = O.rms_norm_backward(w, x, gamma, group, eps)
    for at in [(0, 0), (2, 5), (4, 7)]:
        # central differences of a smooth function: h^2 and rounding errors below 1e-8
        assert abs(_difference(lambda t: (O.rms_norm(t, gamma, group, eps)[0] * w).sum(), x, at) - dx[at]) < 1e-7
    for k in range(groups):
        assert abs(_difference(lambda t: (O.rms_norm(x, t, group, eps)[0] * w).sum(), gamma, (k, 3)) - dgamma[k, 3]) < 1e-7


def test_norm_of_a_row_without_group_takes_no_scale():
    x = RNG(1).standard_normal((2, 4))
    y, _ = O.rms_norm(x, np.ones((2, 4)), np.array([1, 2]), 1e-5)
    plain, _ = O.rms_norm(x, None, None, 1e-5)
    assert np.array_equal(y[0], 2 * plain[0]) and np.array_equal(y[1], plain[1])


def test_ffn_gradients_against_autograd():
    r = RNG(2)
    n, d, f = 7, 6, 10
    x, wgu, wd, dy = (torch.from_numpy(r.standard_normal(s)).requires_grad_() for s in
                      ((n, d), (2 * f, d), (d, f), (n, d)))
    y = torch.nn.functional.linear(
        torch.nn.functional.silu(torch.nn.functional.linear(x, wgu[:f])) * torch.nn.functional.linear(x, wgu[f:]), wd)
    want = torch.autograd.grad(y, (x, wgu, wd), dy.detach())
    n_ = lambda t: t.detach().numpy()  # noqa: E731
    np.testing.assert_allclose(O.ffn(n_(x), n_(wgu), n_(wd)), n_(y), rtol=1e-12, atol=1e-12)
    for a, b in zip(O.ffn_backward(n_(dy), n_(x), n_(wgu), n_(wd)), want):
        np.testing.assert_allclose(a, n_(b), rtol=1e-11, atol=1e-11)


def test_adamw_against_torch():
    r = RNG(3)
    p = torch.from_numpy(r.standard_normal(50)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.3)
    q, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = r.standard_normal(50)
        p.grad = torch.from_numpy(g)
        opt.step()
        q, m, v = O.adamw(q, g, m, v, t, 1e-2, (0.8, 0.95), 1e-6, 0.3)
        np.testing.assert_allclose(q, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_eight_bit_moments_by_hand():
    v = np.zeros(300)
    v[:5] = [448.0, -224.0, 1.0, 17.0, 2.0 ** -11]   # e4m3: 16 and 18 are neighbours of 17, a tie to even
    v[256:259] = [-3.0, 1.5, 0.0]
    codes, scales = O.encode(v, "m")
    assert scales.tolist() == [1.0, np.float32(3.0 / 448.0)]
    assert O.decode(codes, scales)[:5].tolist() == [448.0, -224.0, 1.0, 16.0, 0.0]
    got = O.decode(codes, scales)[256:259]
    np.testing.assert_allclose(got, [-3.0, 1.5, 0.0], rtol=2.0 ** -23)
    w = np.zeros(4)
    w[:3] = [57344.0, 1e-30, 2.0 ** -15]             # a second moment above zero stays above zero
    codes, scales = O.encode(w, "v")
    assert scales[0] == 1.0 and O.decode(codes, scales).tolist() == [57344.0, 2.0 ** -16, 2.0 ** -15, 0.0]
    codes, scales = O.encode(np.zeros(3), "m")
    assert scales[0] == 0.0 and not O.decode(codes, scales).any()


@pytest.mark.parametrize("which", ["m", "v"])
def test_eight_bit_round_trip_is_within_half_a_step(which):
    r = RNG(4)
    v = r.standard_normal(1000) * 10.0 ** r.integers(-3, 2, 1000)
    if which == "v":
        v = v ** 2
    back = O.decode(*O.encode(v, which))
    half = 2.0 ** -4 if which == "m" else 2.0 ** -3
    smallest = {"m": 2.0 ** -9 / 448.0, "v": 2.0 ** -16 / 57344.0}[which]  # of the block's largest
    top = np.repeat([np.abs(v[b:b + 256]).max() for b in range(0, 1000, 256)], 256)[:1000]
    # half a step of the value or of the subnormal grid (a whole one for a v held above zero), and the
    # scale's own float32 rounding
    assert np.all(np.abs(back - v) <= np.maximum(half * np.abs(v), smallest * top) * (1 + 2.0 ** -20) + np.abs(v) * 2.0 ** -22)


def test_round_bits():
    one = torch.tensor([1.0, 1.0 + 2.0 ** -10, 1.0 + 2.0 ** -9, 1.0 + 3 * 2.0 ** -10, -1.0 - 2.0 ** -10 - 2.0 ** -40, 0.0,
                        3e-300], dtype=torch.float64)
    want = [1.0, 1.0, 1.0 + 2.0 ** -9, 1.0 + 2.0 ** -8, -1.0 - 2.0 ** -9, 0.0]
    got = O.round_bits(one, 10)
    assert got[:6].tolist() == want and abs(got[6] / 3e-300 - 1) <= 2.0 ** -10
    r = torch.from_numpy(RNG(8).standard_normal(1000))
    assert torch.equal(O.round_bits(r.float().double(), 24), r.float().double())
    assert torch.equal(O.round_bits(r, 8), r.to(torch.bfloat16).double())  # but for a tie of float32, of which there is none


def _difference_in_norm(got, want):
    return float((got - want).norm() / want.norm())


def test_rounded_ffn_and_what_a_norm_tells():
    """The rounded formula is the formula up to its roundings; a fault of the kind that a kernel may have moves some
    result by more than 2^-10 of its norm."""
    r = RNG(9)
    n, d, f = 1003, 64, 128
    new = lambda *s, std=1.0: torch.from_numpy(r.standard_normal(s) * std).to(torch.bfloat16)  # noqa: E731
    x, wgu, wd, dy = new(n, d), new(2 * f, d, std=1.5 / 8), new(d, f, std=0.1), new(n, d, std=0.1)
    args = [t.double().numpy() for t in (x, wgu, wd)]
    plain = [O.ffn(*args), *O.ffn_backward(dy.double().numpy(), *args)]
    right = O.ffn_rounded(dy, x, wgu, wd)
    for a, b in zip(right, plain):
        # at most three bf16 roundings and one of 2^-10 in a row, each up to 2^-8 of a value
        assert 1e-4 < _difference_in_norm(a, torch.from_numpy(b)) < 3 * 2.0 ** -8 + 2.0 ** -10
    worst = lambda other: max(_difference_in_norm(a, b) for a, b in zip(other, right))  # noqa: E731
    assert worst(O.ffn_rounded(dy, x, wgu, wd, kept_bits=8)) > 2.0 ** -10       # kept as bf16
    lost = dy.clone()
    lost[-1] = 0                                                                # one row left out of the sums
    assert worst(O.ffn_rounded(lost, x, wgu, wd)) > 2.0 ** -10
    part = dy.clone()
    part[: n - n % 64] = 0                                                      # the last, short stage alone
    assert worst(O.ffn_rounded(part * 0, x, wgu, wd)) > 2.0 ** -10
