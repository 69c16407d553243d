"""GPU parity of the attention of ragged rows (window, sinks, shared heads,
gradients, single tokens) against the float64 oracle on the same inputs.

Bars, with e = 2^-24 and, for bf16 tensors, E = 2^-8 per rounding (half a step
relative to the value); sums of n products are off by (n + 2) e times the sum of
their magnitudes in any order.  First-order bounds, doubled where float32's
elementary functions and higher orders come in:
  score       D products:              S = (D + 8) e scale sum|q||k| (base 2 exponent and its rounding included)
  weight P    exp of a difference:     relative 2 (2 max S + (n + 8) e) =: w
  o           P rounded (E), summed:   (E + w) sum P |v| + E |o|
  dv          the same over queries:   (E + w) sum P |do| + E |dv|
  delta       do . o with o as stored: sum |do| (bound of o) + (D + 2) e sum |do||o|
  dS          P (dP - delta):          P ((D + 2) e sum |do||v| + bound of delta) + (E + w) |dS|
  dq, dk      summed, scaled:          scale sum (bound of dS) |k| (|q|) + E |dq| (|dk|)"""
import numpy as np
import pytest

from oracle import step_operators as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E32, E16 = 2.0 ** -24, 2.0 ** -8


def _train():
    from paper_2609_15160_amd import train
    return train


def _say(*what):
    print("[attention]", *what, flush=True)


def _dt(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _np(t):
    return t.detach().double().cpu().numpy()


def _normal(rng, *shape, std=1.0, dtype="f32"):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(_dt(dtype)).cuda()


def _offsets(n):
    return torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32).cuda()


def _within(got, want, bound, what):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    over = np.abs(got - want) - bound
    assert np.all(over <= 0), (what, float(np.nanmax(over)), int(np.argmax(over)), float(np.nanmax(np.abs(got - want))))


def bounds(q, k, v, r, window, sinks, scale, dtype, do=None):
    """Bounds of one sequence's results (arrays as the oracle's), from the magnitudes."""
    E = E16 if dtype == "bf16" else 0.0
    nq, heads, D = q.shape
    n, kv = k.shape[:2]
    each = heads // kv
    aq, ak, av, p = np.abs(q), np.abs(k), np.abs(v), r["p"]
    out = {"o": np.zeros(q.shape), "dq": np.zeros(q.shape), "dk": np.zeros(k.shape), "dv": np.zeros(v.shape)}
    for h in range(heads):
        c = h // each
        seen = p[h] > 0
        S = (D + 8) * E32 * scale * np.where(seen, aq[:, h] @ ak[:, c].T, 0.0).max(1, initial=0.0)
        w = 2 * (2 * S + (n + 8) * E32)
        out["o"][:, h] = (E + w)[:, None] * (p[h] @ av[:, c]) + E * np.abs(r["o"][:, h])
        if do is None:
            continue
        ad, d = np.abs(do[:, h]), do[:, h]
        out["dv"][:, c] += p[h].T @ ((E + w)[:, None] * ad)
        delta = (ad * out["o"][:, h]).sum(1) + (D + 2) * E32 * (ad * np.abs(r["o"][:, h])).sum(1)
        dS = p[h] * (d @ v[:, c].T - (d * r["o"][:, h]).sum(1, keepdims=True))
        b = p[h] * ((D + 2) * E32 * (ad @ av[:, c].T) + delta[:, None]) + (E + w)[:, None] * np.abs(dS)
        b = b + (n + 2) * E32 * np.abs(dS)
        out["dq"][:, h] = scale * (b @ ak[:, c]) + E * np.abs(r["dq"][:, h])
        out["dk"][:, c] += scale * (b.T @ aq[:, h])
    if do is not None:
        out["dk"] += (E + (each * nq + 2) * E32) * np.abs(r["dk"])
        out["dv"] += (E + (each * nq + 2) * E32) * np.abs(r["dv"])
    return {name: 1.01 * b + 1e-30 for name, b in out.items()}


def _check(n, heads, kv, D, window=None, sinks=0, dtype="bf16", nq=None, tail=0, scale=None, grad=True, seed=0,
           room=None, std=1.0, packed=False):
    """Sequences of n keys and nq queries each (n by default), in `room` rows each, `tail` rows behind the last."""
    train = _train()
    nq, room = n if nq is None else nq, n if room is None else room
    _say("lengths", n, "queries", nq, "room", room, heads, kv, D, "window", window, sinks, dtype, "tail", tail, "packed", packed)
    rng = np.random.default_rng(seed + 31 * sum(n) + 7 * heads + D)
    q = _normal(rng, sum(nq) + tail, heads, D, std=std, dtype=dtype)
    k, v = (_normal(rng, sum(room) + tail, kv, D, std=s, dtype=dtype) for s in (std, 1.0))
    do = _normal(rng, sum(nq) + tail, heads, D, dtype=dtype)
    args = dict(window=window, sinks=sinks, scale=scale)
    if packed:
        qkv = torch.cat([t.flatten(1) for t in (q, k, v)], 1).contiguous().requires_grad_(grad)
        o = train.self_attention(qkv, _offsets(nq), heads, kv, **args)
        got = {"o": _np(o).reshape(q.shape)}
        if grad:
            g, = torch.autograd.grad(o, qkv, do.flatten(1))
            parts = np.split(_np(g).reshape(len(q), heads + 2 * kv, D), (heads, heads + kv), 1)
            got.update(dq=parts[0], dk=parts[1], dv=parts[2])
    else:
        for t in (q, k, v):
            t.requires_grad_(grad)
        lengths = torch.tensor(n, dtype=torch.int32).cuda() if room != n else None
        o = train.attention(q, k, v, _offsets(nq), _offsets(room), lengths, **args)
        got = {"o": _np(o)}
        if grad:
            got.update(zip(("dq", "dk", "dv"), map(_np, torch.autograd.grad(o, (q, k, v), do))))
    assert o.dtype == q.dtype
    q, k, v, do = map(_np, (q, k, v, do))
    a, b = np.cumsum([0] + list(nq)), np.cumsum([0] + list(room))
    for i in range(len(n)):
        mq, mk = slice(a[i], a[i + 1]), slice(b[i], b[i] + n[i])
        r = O.attention(q[mq], k[mk], v[mk], window, sinks, scale, do[mq] if grad else None)
        lim = bounds(q[mq], k[mk], v[mk], r, window, sinks, D ** -0.5 if scale is None else scale, dtype,
                     do[mq] if grad else None)
        _within(got["o"][mq], r["o"], lim["o"], ("o", i))
        if grad:
            _within(got["dq"][mq], r["dq"], lim["dq"], ("dq", i))
            _within(got["dk"][mk], r["dk"], lim["dk"], ("dk", i))
            _within(got["dv"][mk], r["dv"], lim["dv"], ("dv", i))
            for name in ("dk", "dv"):  # room without keys
                assert not got[name][b[i] + n[i]:b[i + 1]].any(), (name, i)
    for name, at in (("o", a), ("dq", a), ("dk", b), ("dv", b)):  # rows behind the last sequence
        if name in got:
            assert not got[name][at[-1]:].any(), name


TYPES = [("bf16", 64), ("bf16", 128), ("f32", 16), ("f32", 64), ("f32", 128)]


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("n", [[1], [2, 0, 1], [17, 64, 33], [65], [130, 5], [0, 0, 0, 97]])
def test_ragged_causal(dtype, D, n):
    _check(n, 2, 2, D, dtype=dtype)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (31, 3), (64, 4), (100, 64), (65, 1), (1000, 5)])
def test_window_and_sinks(dtype, D, window, sinks):
    _check([200, 3, 77], 2, 1, D, window=window, sinks=sinks, dtype=dtype, tail=3)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 2), (6, 1), (3, 3)])
def test_shared_heads(dtype, D, heads, kv):
    _check([70, 41], heads, kv, D, window=50, sinks=2, dtype=dtype)
    _check([70, 41], heads, kv, D, window=50, sinks=2, dtype=dtype, packed=True, tail=2)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("nq,n", [([5, 0, 40], [90, 20, 70]), ([40, 3, 9], [7, 3, 0]), ([64, 1], [64, 300])])
def test_queries_of_other_rows_than_keys(dtype, D, nq, n):
    """Chunks behind a cache; queries before the first key and sequences without keys see nothing."""
    _check(n, 2, 2, D, nq=nq, dtype=dtype)
    _check(n, 2, 1, D, nq=nq, room=[x + 13 for x in n], window=40, sinks=3, dtype=dtype, tail=1)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2), (17, 1), (40, 2)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (37, 4)])
def test_single_tokens(dtype, D, heads, kv, window, sinks):
    n = [1, 33, 0, 300, 64]
    _check(n, heads, kv, D, nq=[1] * 5, room=[300] * 5, window=window, sinks=sinks, dtype=dtype, grad=heads < 17)


@pytest.mark.parametrize("dtype,D", TYPES)
def test_single_tokens_over_a_long_axis(dtype, D):
    """Keys of a row split over workgroups, with sequences of fewer keys than ranges among them."""
    _check([3000, 5, 0, 2900, 1], 2, 1, D, nq=[1] * 5, dtype=dtype, grad=False)
    _check([5000, 40], 4, 1, D, nq=[1, 1], room=[5003, 2000], window=2500, sinks=7, dtype=dtype, grad=False)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_many_tiles(dtype, D):
    """Enough tiles for the workgroups of four waves, ragged, with sinks whose queries are split into ranges."""
    _check([1500, 0, 1390, 700], 16, 16, D, window=50, sinks=5, dtype=dtype, packed=True, tail=130)


def test_many_tiles_causal():
    _check([1030, 900, 1100, 1025], 16, 8, 64, dtype="bf16", packed=True)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 64)])
def test_sharp_and_growing_scores(dtype, D):
    """Scores of some hundred: the base of a row's softmax moves again and again as keys grow."""
    train = _train()
    rng = np.random.default_rng(4)
    n = 300
    q, k, v = (_normal(rng, n, 1, D, dtype=dtype) for _ in range(3))
    k = (k * torch.linspace(0.1, 30, n, device="cuda")[:, None, None]).to(k.dtype)
    o = train.attention(q, k, v, _offsets([n]), window=250, sinks=2)
    r = O.attention(_np(q), _np(k), _np(v), 250, 2)
    _within(o, r["o"], bounds(_np(q), _np(k), _np(v), r, 250, 2, D ** -0.5, dtype)["o"], "o")
