"""Oracle for the training operators of the block's FFN half (Appendix A), CPU
test infrastructure only.

Plain numpy in float64 on the values given: RMSNorm with the AdaLN scale of a
row's group, the gated FFN, their gradients, and AdamW with moments in 32 or 8
bits (the 8-bit formats' own rounding is torch's float32 to float8 cast).
Shares no code with the HIP path."""
import numpy as np
import torch

BLOCK = 256
FORMATS = {"m": (torch.float8_e4m3fn, 448.0), "v": (torch.float8_e5m2, 57344.0)}


def scale_rows(gamma, group, rows, d):
    """1 + gamma of each row; 1 where the row's group is none of gamma's."""
    out = np.ones((rows, d))
    if gamma is not None:
        gamma = np.asarray(gamma, np.float64).reshape(-1, d)
        for r in range(rows):
            k = 0 if group is None else int(group[r])
            if 0 <= k < len(gamma):
                out[r] += gamma[k]
    return out


def rms_norm(x, gamma, group, eps):
    x = np.asarray(x, np.float64)
    r = 1.0 / np.sqrt((x ** 2).mean(1, keepdims=True) + eps)
    return x * r * scale_rows(gamma, group, *x.shape), r[:, 0]


def rms_norm_backward(dy, x, gamma, group, eps):
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    rows, d = x.shape
    r = 1.0 / np.sqrt((x ** 2).mean(1, keepdims=True) + eps)
    h = dy * scale_rows(gamma, group, rows, d)
    dx = r * (h - x * r ** 2 * (h * x).mean(1, keepdims=True))
    dgamma = None
    if gamma is not None:
        n = np.asarray(gamma).size // d
        dgamma = np.zeros((n, d))
        for row in range(rows):
            k = 0 if group is None else int(group[row])
            if 0 <= k < n:
                dgamma[k] += dy[row] * x[row] * r[row]
    return dx, dgamma


def sigmoid(g):
    return 1.0 / (1.0 + np.exp(-g))


def ffn(x, w_gate_up, w_down):
    x, wgu, wd = (np.asarray(t, np.float64) for t in (x, w_gate_up, w_down))
    f = wd.shape[1]
    g, u = x @ wgu[:f].T, x @ wgu[f:].T
    return (g * sigmoid(g) * u) @ wd.T


def ffn_backward(dy, x, w_gate_up, w_down):
    dy, x, wgu, wd = (np.asarray(t, np.float64) for t in (dy, x, w_gate_up, w_down))
    f = wd.shape[1]
    g, u = x @ wgu[:f].T, x @ wgu[f:].T
    s = sigmoid(g)
    da = dy @ wd
    dgu = np.concatenate([da * u * s * (1 + g * (1 - s)), da * g * s], 1)
    return dgu @ wgu, dgu.T @ x, dy.T @ (g * s * u)


def encode(v, which):
    """(float8 codes, float32 scales) of a flat float64 moment."""
    dtype, most = FORMATS[which]
    v = np.asarray(v, np.float64).reshape(-1)
    codes, scales = np.zeros(v.size, np.float32), []
    for b in range(0, v.size, BLOCK):
        part = v[b:b + BLOCK]
        s = np.float32(np.float64(np.abs(part).max().astype(np.float32)) / most)
        scales.append(s)
        if s > 0:
            t = np.clip(part / np.float64(s), -most, most)
            if which == "v":
                t = np.where((t > 0) & (t < 2.0 ** -16), 2.0 ** -16, t)
            codes[b:b + BLOCK] = t.astype(np.float32)
    return torch.from_numpy(codes).to(dtype), np.array(scales, np.float32)


def decode(codes, scales):
    c = codes.float().numpy().astype(np.float64).reshape(-1)
    return c * np.repeat(np.asarray(scales, np.float64), BLOCK)[: c.size]


def adamw(p, g, m, v, step, lr, betas, eps, weight_decay):
    """New (p, m, v) of flat float64 arrays."""
    p, g, m, v = (np.asarray(t, np.float64).reshape(-1) for t in (p, g, m, v))
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    mh, vh = m / (1 - b1 ** step), v / (1 - b2 ** step)
    return p * (1 - lr * weight_decay) - lr * mh / (np.sqrt(vh) + eps), m, v


# ---------------------------------------------------------------------------
# The gated FFN of bf16 tensors with the roundings that it documents, in torch
# (float64 on any device), so that large sizes can be compared
# ---------------------------------------------------------------------------

def round_bits(v, bits):
    """float64 values rounded to so many significant bits, ties to even."""
    drop = 53 - bits
    b = v.contiguous().view(torch.int64)
    b = b + ((1 << (drop - 1)) - 1) + ((b >> drop) & 1)
    return ((b >> drop) << drop).view(torch.float64)


def ffn_rounded(dy, x, w_gate_up, w_down, kept_bits=10):
    """(y, dx, dw_gate_up, dw_down): a, dg, du and the results rounded to bf16, silu(g) and u silu'(g) to `kept_bits`
    significant bits between the passes, everything else in float64."""
    half = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    dy, x, wgu, wd = (t.double() for t in (dy, x, w_gate_up, w_down))
    f = wd.shape[1]
    g, u = x @ wgu[:f].T, x @ wgu[f:].T
    s = 1.0 / (1.0 + torch.exp(-g))
    p, q = g * s, u * (s * (1.0 + g * (1.0 - s)))
    a = half(p * u)
    da = dy @ wd
    dgu = half(torch.cat([da * round_bits(q, kept_bits), da * round_bits(p, kept_bits)], 1))
    return tuple(half(t) for t in (a @ wd.T, dgu @ wgu, dgu.T @ x, dy.T @ a))
