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


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("n,heads,kv,room", [([2500], 1, 1, None), ([1500, 3, 0, 700], 4, 2, [1500, 3, 5, 800])])
def test_sinks_of_long_sequences(dtype, D, n, heads, kv, room):
    """First tiles whose queries go in many ranges, joined afterwards; short and empty sequences and room among them."""
    _check(n, heads, kv, D, window=20, sinks=5, dtype=dtype, room=room)


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


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("scores", ["low", "lower", "lowest", "low first", "lowest first", "high first"])
def test_scores_far_from_zero(dtype, D, nq, scores):
    """Weights relative to any fixed base would leave float32's range, or reach its subnormal end."""
    train = _train()
    rng = np.random.default_rng(5)
    n = 200
    q = _normal(rng, nq, 1, D, std=0.1, dtype=dtype)
    k, v = (_normal(rng, n, 1, D, std=s, dtype=dtype) for s in (0.1, 1.0))
    do = _normal(rng, nq, 1, D, dtype=dtype)
    rest = {"low": -95.0, "lower": -110.0, "lowest": -900.0}.get(scores, 10.0)
    first = {"low first": -70.0, "lowest first": -1e4, "high first": 200.0}.get(scores, rest)
    q[:, 0, 0], k[:, 0, 0] = 8.0, rest / 8
    k[torch.arange(0, n, 50), 0, 0] = first / 8  # the first keys of several windows too
    for window, sinks in ((None, 0), (51, 0), (30, 3)):
        leaves = [t.detach().clone().requires_grad_() for t in (q, k, v)]
        o = train.attention(*leaves, _offsets([nq]), _offsets([n]), window=window, sinks=sinks, scale=1.0)
        got = dict(zip(("o", "dq", "dk", "dv"), (o, *torch.autograd.grad(o, leaves, do))))
        arrays = [_np(t) for t in (q, k, v)]
        r = O.attention(*arrays, window, sinks, 1.0, _np(do))
        lim = bounds(*arrays, r, window, sinks, 1.0, dtype, _np(do))
        for name in got:
            _within(got[name], r[name], lim[name], (name, window))


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("first", [0.0, -50.0])
@pytest.mark.parametrize("up", [60.0, 80.0, 84.0, 86.0, 87.0, 88.0, 100.0])
def test_scores_that_rise_between_tiles(dtype, D, nq, first, up):
    """Scores far above those of a row's first keys, twice: weights relative to what the first keys give are up to the end of
    float32's range, their sums beyond it, while sums of weights times small values, or values of both signs, are not."""
    train = _train()
    _say("rising scores", dtype, D, nq, first, up)
    rng = np.random.default_rng(9)
    n = 200
    q = _normal(rng, nq, 1, D, std=0.1, dtype=dtype)
    k = _normal(rng, n, 1, D, std=0.1, dtype=dtype)
    do = _normal(rng, nq, 1, D, dtype=dtype)
    at = torch.arange(n, device="cuda")
    q[:, 0, 0] = 8.0
    k[:, 0, 0] = ((first + up * ((at >= 40).float() + (at >= 120).float())) / 8).to(k.dtype)
    small = 0.01 + _normal(rng, n, 1, D, std=0.001)
    for v in (small, small * (1 - 2 * (at % 2))[:, None, None]):
        v = v.to(k.dtype)
        for window, sinks in ((None, 0), (51, 0), (30, 3)):
            leaves = [t.detach().clone().requires_grad_() for t in (q, k, v)]
            o = train.attention(*leaves, _offsets([nq]), _offsets([n]), window=window, sinks=sinks, scale=1.0)
            got = dict(zip(("o", "dq", "dk", "dv"), (o, *torch.autograd.grad(o, leaves, do))))
            arrays = [_np(t) for t in (q, k, v)]
            r = O.attention(*arrays, window, sinks, 1.0, _np(do))
            lim = bounds(*arrays, r, window, sinks, 1.0, dtype, _np(do))
            for name in got:
                _within(got[name], r[name], lim[name], (name, window))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nq,window,std", [(300, None, 1.0), (300, None, 2.0), (300, 40, 3.0), (4, None, 2.0), (1, None, 2.0)])
def test_roundings_are_those_of_the_operands(D, nq, window, std):
    """bfloat16 tensors, rows that few keys have most of the weight of: equal in norm to the formula with its operands
    (weights, gradients of scores) and results rounded and nothing else, o as the gradients take it among that, to 2^-10.
    Left over are values next to a rounding's border that float32's errors move across it: a score is off by less than
    (D + 8) 2^-24 of the sum of its magnitudes, some 2^-13 in all here, so that of the values at most 2^-13 / 2^-8 move by
    2^-8: in norm 2^-8 2^-2.5 at the very most, and with typical errors (2^-19 of a score) 2^-8 2^-5.5 = 2^-13.5.

    That is for weights relative to a whole base, whose power of two moves no rounding.  For few rows the base is a score:
    weights are rounded elsewhere, each by E = 2^-8 at most here and there, so that o, a mean by the rounded weights, differs
    by 2 E sum p |v - o|, delta by 2 E sum p |do . (v - o)| =: b, and what is rounded behind them by that and by 2 E of
    itself: dS by p b + 2 E |dS|, dq and dk by the sums of that, and 2 E of themselves."""
    train = _train()
    rng = np.random.default_rng(6)
    n, heads = 300, 4
    q = _normal(rng, nq, heads, D, std=std, dtype="bf16")
    k, v = (_normal(rng, n, heads, D, std=s, dtype="bf16") for s in (std, 1.0))
    do = _normal(rng, nq, heads, D, dtype="bf16")
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    o = train.attention(*leaves, _offsets([nq]), _offsets([n]), window=window)
    got = [_np(t) for t in (o, *torch.autograd.grad(o, leaves, do))]
    q, k, v, do = map(_np, (q, k, v, do))

    def bf(x):
        return torch.from_numpy(x).float().bfloat16().double().numpy()

    want, extra = ([np.zeros(t.shape) for t in (q, q, k, v)] for _ in range(2))
    scale, seen, E = D ** -0.5, O.visible(nq, n, window, 0), E16 if nq <= 8 else 0.0
    for h in range(heads):
        s = np.where(seen, scale * np.log2(np.e) * (q[:, h] @ k[:, h].T), -np.inf)
        w = np.exp2(s - np.ceil(s.max(1, keepdims=True)))
        p = w / w.sum(1, keepdims=True)
        oh = bf(w) @ v[:, h] / bf(w).sum(1, keepdims=True)
        ds = bf(p * (do[:, h] @ v[:, h].T - (do[:, h] * oh).sum(1, keepdims=True)))
        for t, x in zip(want, (oh, scale * ds @ k[:, h], scale * ds.T @ q[:, h], bf(p).T @ do[:, h])):
            t[:, h] = bf(x)
        far = v[None, :, h] - oh[:, None]
        b = 2 * E * (p * np.abs((do[:, None, h] * far).sum(2))).sum(1, keepdims=True)
        eds = p * b + 2 * E * np.abs(ds)
        for t, w, x in zip(extra, want, (2 * E * (p[:, :, None] * np.abs(far)).sum(1), scale * eds @ np.abs(k[:, h]),
                                         scale * eds.T @ np.abs(q[:, h]))):
            t[:, h] = x + 2 * E * np.abs(w[:, h])
    for name, a, b, x in zip(("o", "dq", "dk", "dv"), got, want, extra):
        off = np.linalg.norm(a - b), 2.0 ** -10 * np.linalg.norm(b) + np.linalg.norm(x)
        assert off[0] <= off[1], (name, off)


# ---------------------------------------------------------------------------
# What is not seen takes no part, whatever its values; layouts, streams, order
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_where_they_are_seen(dtype, D, bad):
    """One key's values, another's key and one query's gradient not finite: the rows that see none of them are the
    same as without, to the bounds; those that do are not finite."""
    train = _train()
    rng = np.random.default_rng(21)
    n, heads = 150, 2
    q, k, v, do = (_normal(rng, n, heads, D, dtype=dtype) for _ in range(4))
    for window, sinks in ((None, 0), (40, 0), (40, 3)):
        vb, kb, db = v.clone(), k.clone(), do.clone()
        vb[70, 0, 5] = bad
        kb[90, 1] = float("nan")
        db[100, 0, 3] = bad
        leaves = [t.clone().requires_grad_() for t in (q, kb, vb)]
        o = train.attention(*leaves, _offsets([n]), window=window, sinks=sinks)
        got = dict(zip(("o", "dq", "dk", "dv"), (o, *torch.autograd.grad(o, leaves, db))))
        r = O.attention(_np(q), _np(kb), _np(vb), window, sinks, None, _np(db))
        clean = O.attention(_np(q), _np(k), _np(v), window, sinks, None, _np(do))
        lim = bounds(_np(q), _np(k), _np(v), clean, window, sinks, D ** -0.5, dtype, _np(do))
        for name in ("o", "dq", "dk", "dv"):
            have, want = _np(got[name]), r[name]
            fine = np.isfinite(want)
            assert not fine.all()
            some = window is not None or name != "dk"  # without a window scores that are not finite reach every key
            assert fine.any() == some, name
            assert np.array_equal(np.isfinite(have), fine), (name, window, int((np.isfinite(have) != fine).sum()))
            # where a finite result has the same inputs as without them, the same bounds; else it is checked as finite
            with np.errstate(invalid="ignore"):
                same = fine & (np.abs(want - clean[name]) <= 1e-12 * np.abs(clean[name]))
            assert same.any() == some and np.all(np.abs(have[same] - want[same]) <= lim[name][same]), (name, window)


def _entry(q, k, v, do, offsets, k_offsets, window, sinks, scale=None):
    """Through the C entry points, their outputs full of NaN before: a dict of o, lse, low (bfloat16) and the gradients."""
    import ctypes

    from paper_2609_15160_amd import tlf
    train, lib = _train(), tlf.load()
    (rows, heads, D), (k_rows, kv) = q.shape, k.shape[:2]
    out = {name: torch.full_like(t, float("nan")) for name, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    out["lse"] = torch.full((heads, rows), float("nan"), device="cuda")
    out["low"] = torch.full_like(q, float("nan")) if q.dtype == torch.bfloat16 else None
    wide, kv_wide = heads * D, kv * D
    shape = tlf.AttnShape(train._DTYPE[q.dtype], len(offsets) - 1, heads, kv, D, rows, k_rows, window or 0, sinks,
                          D ** -0.5 if scale is None else scale, wide, kv_wide, kv_wide, wide, offsets.data_ptr(),
                          k_offsets.data_ptr(), None)
    ws, need = train._workspace(lib.tlf_attn_ws_bytes, shape, device=q.device)
    train._run(lib.tlf_attn, q.device, shape, q, k, v, out["o"], out["lse"], out["low"], ws, need)
    ws, need = train._workspace(lib.tlf_attn_grad_ws_bytes, shape, device=q.device)
    train._run(lib.tlf_attn_grad, q.device, shape, do, q, k, v, out["o"], out["lse"], out["low"], out["dq"], wide, out["dk"],
               kv_wide, out["dv"], kv_wide, ws, need)
    return out


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("nq,n", [(40, 7), (60, 40), (300, 130)])
def test_queries_before_the_first_key_give_zeros_whatever_the_values(dtype, D, nq, n):
    """Queries that see no key beside ones that do, in one tile and one wave; keys, values and the unseeing rows' own q
    and gradients not finite: zeros, an lse of +inf, and no part in any gradient."""
    rng = np.random.default_rng(27)
    heads, before = 2, nq - n
    q, do = (_normal(rng, nq, heads, D, dtype=dtype) for _ in range(2))
    k, v = (_normal(rng, n, heads, D, dtype=dtype) for _ in range(2))
    qb, kb, vb, db = (t.clone() for t in (q, k, v, do))
    qb[0], qb[before - 1, 0, 1] = float("nan"), float("inf")
    db[0, 0, 3], db[before - 1] = float("inf"), float("nan")
    kb[n - 1, 0] = float("nan")
    vb[0, 0, 5], vb[n // 2, 1, 2], vb[n // 2, 1, 3] = float("inf"), float("nan"), -float("inf")
    for window, sinks in ((None, 0), (5, 0), (5, 2)):
        _say("before the first key", dtype, D, nq, n, window, sinks)
        got = _entry(qb, kb, vb, db, _offsets([nq]), _offsets([n]), window, sinks)
        for name in ("o", "dq", "low"):
            assert got[name] is None or not got[name][:before].any(), (name, window)  # NaN counts as some
        assert bool((got["lse"][:, :before] == float("inf")).all()), window
        r = O.attention(_np(qb), _np(kb), _np(vb), window, sinks, None, _np(db))
        clean = O.attention(_np(q), _np(k), _np(v), window, sinks, None, _np(do))
        lim = bounds(_np(q), _np(k), _np(v), clean, window, sinks, D ** -0.5, dtype, _np(do))
        for name in ("o", "dq", "dk", "dv"):
            have, want = _np(got[name]), r[name]
            fine = np.isfinite(want)
            assert not fine.all() and np.array_equal(np.isfinite(have), fine), (name, window)
            with np.errstate(invalid="ignore"):
                same = fine & (np.abs(want - clean[name]) <= 1e-12 * np.abs(clean[name]))
            assert np.all(np.abs(have[same] - want[same]) <= lim[name][same]), (name, window)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("ahead,k_ahead", [(1, 0), (0, 1), (5, 63), (128, 64), (300, 200), (127, 129)])
@pytest.mark.parametrize("nq", [[25, 0, 17], [1, 0, 1], [140, 3, 0]])
def test_rows_ahead_of_the_first_sequence(dtype, D, ahead, k_ahead, nq):
    """Offsets that begin behind row 0: the rows ahead, as those behind, are written as zeros, and the sequences are what they
    are without them."""
    _say("rows ahead", dtype, D, ahead, k_ahead, nq)
    rng = np.random.default_rng(28)
    n, heads, kv, tail = [30, 70, 17], 4, 2, 3
    q, do = (_normal(rng, ahead + sum(nq) + tail, heads, D, dtype=dtype) for _ in range(2))
    k, v = (_normal(rng, k_ahead + sum(n) + tail, kv, D, dtype=dtype) for _ in range(2))
    for window, sinks in ((None, 0), (20, 3)):
        got = _entry(q, k, v, do, _offsets(nq) + ahead, _offsets(n) + k_ahead, window, sinks)
        a, b = ahead + np.cumsum([0] + nq), k_ahead + np.cumsum([0] + n)
        for name, at in (("o", a), ("low", a), ("dq", a), ("dk", b), ("dv", b)):
            assert got[name] is None or not (got[name][:at[0]].any() or got[name][at[-1]:].any()), (name, window)
        assert bool((got["lse"][:, :ahead] == float("inf")).all() and (got["lse"][:, a[-1]:] == float("inf")).all())
        for i in range(3):
            mq, mk = slice(a[i], a[i + 1]), slice(b[i], b[i + 1])
            arrays = [_np(t) for t in (q[mq], k[mk], v[mk])]
            r = O.attention(*arrays, window, sinks, None, _np(do[mq]))
            lim = bounds(*arrays, r, window, sinks, D ** -0.5, dtype, _np(do[mq]))
            for name, m in (("o", mq), ("dq", mq), ("dk", mk), ("dv", mk)):
                _within(got[name][m], r[name], lim[name], (name, i, window))


def test_self_attention_of_a_sequence_behind_other_rows():
    train = _train()
    rng = np.random.default_rng(29)
    qkv = _normal(rng, 500, 6 * 64, dtype="bf16")
    a, b = qkv.clone().requires_grad_(), qkv[200:450].clone().requires_grad_()
    oa, ob = (train.self_attention(t, torch.tensor(off, dtype=torch.int32, device="cuda"), 4, 1, window=40)
              for t, off in ((a, (200, 300, 450)), (b, (0, 100, 250))))
    do = _normal(rng, 500, 256, dtype="bf16")
    ga, = torch.autograd.grad(oa, a, do)
    gb, = torch.autograd.grad(ob, b, do[200:450])
    for whole, part in ((oa, ob), (ga, gb)):
        assert torch.equal(whole[200:450], part) and not whole[:200].any() and not whole[450:].any()


@pytest.mark.parametrize("nq", [1, 40])
def test_rows_behind_a_caches_end_are_not_read(nq):
    """Room of a cache that is not used yet holds NaN."""
    train = _train()
    rng = np.random.default_rng(22)
    room, n = 200, [150, 40, 64]
    q = _normal(rng, 3 * nq, 4, 64, dtype="bf16")
    k, v = (_normal(rng, 3 * room, 2, 64, dtype="bf16") for _ in range(2))
    lengths = torch.tensor(n, dtype=torch.int32).cuda()
    want = train.attention(q, k, v, _offsets([nq] * 3), _offsets([room] * 3), lengths, window=30, sinks=2)
    for i, m in enumerate(n):
        k[i * room + m:(i + 1) * room] = float("nan")
        v[i * room + m:(i + 1) * room] = float("nan")
    got = train.attention(q, k, v, _offsets([nq] * 3), _offsets([room] * 3), lengths, window=30, sinks=2)
    assert torch.isfinite(got).all() and torch.equal(got, want)


@pytest.mark.parametrize("nq", [1, 50])
def test_strided_and_misaligned_rows(nq):
    """Rows inside wider ones as they lie; other strides and alignments by a copy; the same results to the bit."""
    train = _train()
    rng = np.random.default_rng(23)
    n = 60
    wide = _normal(rng, n, 1000, dtype="bf16")
    q, k, v = (wide[:, a:a + 256].view(n, 4, 64) for a in (0, 256, 512))
    q = q[:2 * nq] if nq == 1 else q
    args = (_offsets([1, 1]), _offsets([20, 40])) if nq == 1 else (_offsets([20, 40]),)
    plain = [t.contiguous().requires_grad_() for t in (q, k, v)]
    want = train.attention(*plain, *args, window=17)
    do = _normal(rng, *want.shape, dtype="bf16")
    grads = torch.autograd.grad(want, plain, do)
    odd = torch.empty(n * 256 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(n, 4, 64)
    odd.copy_(k)
    ways = [(q, k, v), (q, odd, v), (q.transpose(0, 1).contiguous().transpose(0, 1), k, wide[:, 512:768].view(n, 4, 64))]
    for w in ways:
        leaves = [t.detach().requires_grad_() for t in w]
        got = train.attention(*leaves, *args, window=17)
        assert torch.equal(got, want)
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(got, leaves, do), grads))
    one = k[:, :1].expand(n, 4, 64)  # one head for all, a stride of zero
    a = train.attention(q, one, one, *args)
    b = train.attention(q, k[:, :1], k[:, :1], *args)
    assert torch.equal(a, b)


def test_self_attention_of_rows_inside_wider_ones():
    train = _train()
    rng = np.random.default_rng(24)
    wide = _normal(rng, 70, 800, dtype="bf16")
    qkv = wide[:, 8:8 + 6 * 64]
    a = qkv.detach().requires_grad_()
    b = qkv.detach().clone().requires_grad_()
    oa, ob = (train.self_attention(t, _offsets([30, 40]), 4, 1) for t in (a, b))
    assert torch.equal(oa, ob)
    assert torch.equal(torch.autograd.grad(oa.sum(), a)[0], torch.autograd.grad(ob.sum(), b)[0])


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("nq", [[700, 400], [1, 1]])
def test_rows_past_32_bits_of_elements(dtype, D, nq):
    """Rows at the largest stride, the last of them more than 2^31 elements behind the first, inputs and gradients: the same
    to the bit as rows that lie one behind the other."""
    import ctypes

    from paper_2609_15160_amd import tlf
    train, lib = _train(), tlf.load()
    _say("rows past 2^31 elements", dtype, D, nq)
    rng = np.random.default_rng(30)
    n, heads, kv, wide = [700, 400], 4, 2, tlf.ATTN_MAX_STRIDE
    assert (sum(n) - 1) * wide > 1 << 31
    q, do = (_normal(rng, sum(nq), heads, D, dtype=dtype) for _ in range(2))
    k, v = (_normal(rng, sum(n), kv, D, dtype=dtype) for _ in range(2))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    args = dict(window=90, sinks=3)
    want = train.attention(*leaves, _offsets(nq), _offsets(n), **args)
    grads = torch.autograd.grad(want, leaves, do)
    space = torch.empty(sum(n), wide, dtype=q.dtype, device="cuda")
    cut = lambda t, at: space[:len(t), at:at + t[0].numel()].view(t.shape)  # noqa: E731
    far = [cut(t, 1024 * i) for i, t in enumerate((q, k, v))]
    for t, f in zip((q, k, v), far):
        f.copy_(t)
    assert all(train._rows_of_heads(f, f.shape[1], D) is f for f in far)  # read as they lie
    got = train.attention(*[f.detach().requires_grad_() for f in far], _offsets(nq), _offsets(n), **args)
    assert torch.equal(got, want)
    out = [cut(t, 4096 + 1024 * i) for i, t in enumerate((q, k, v, q, q))]  # dq, dk, dv, o, low
    lse = torch.empty(heads, sum(nq), device="cuda")
    d_o = cut(do, 16384)
    d_o.copy_(do)
    off, k_off = _offsets(nq), _offsets(n)
    shape = tlf.AttnShape(train._DTYPE[q.dtype], 2, heads, kv, D, sum(nq), sum(n), 90, 3, D ** -0.5, wide, wide, wide, wide,
                          off.data_ptr(), k_off.data_ptr(), None)
    low = out[4] if dtype == "bf16" else None
    ws, need = train._workspace(lib.tlf_attn_ws_bytes, ctypes.byref(shape), device=q.device)
    train._run(lib.tlf_attn, q.device, shape, *far, out[3], lse, low, ws, need)
    ws, need = train._workspace(lib.tlf_attn_grad_ws_bytes, ctypes.byref(shape), device=q.device)
    train._run(lib.tlf_attn_grad, q.device, shape, d_o, *far, out[3], lse, low, out[0], wide, out[1], wide, out[2], wide, ws, need)
    assert all(torch.equal(a, b) for a, b in zip((out[3], *out[:3]), (want, *grads)))


def test_gradients_by_differences():
    train = _train()
    rng = np.random.default_rng(25)
    n = [9, 0, 21]
    q, k, v = (_normal(rng, 30, h, 16) for h in (4, 2, 2))
    leaves = [t.requires_grad_() for t in (q, k, v)]
    o = train.attention(*leaves, _offsets(n), window=6, sinks=2)
    c = _normal(rng, *o.shape)
    got = torch.autograd.grad(o, leaves, c)
    vals = [_np(t) for t in leaves]
    for i, g in enumerate(got):
        step = rng.standard_normal(vals[i].shape)
        f = []
        for s in (1e-5, -1e-5):
            t = [x + (s * step if j == i else 0) for j, x in enumerate(vals)]
            f.append(sum((O.attention(*(x[a:b] for x in t), 6, 2)["o"] * _np(c)[a:b]).sum() for a, b in ((0, 9), (9, 30))))
        slope, have = (f[0] - f[1]) / 2e-5, (_np(g) * step).sum()
        assert abs(slope - have) <= 300 * E32 * np.abs(_np(g) * step).sum() + 1e-5, (i, slope, have)


def test_same_from_call_to_call_and_on_other_streams():
    train = _train()
    rng = np.random.default_rng(26)
    qkv = _normal(rng, 3000, 3 * 512, dtype="bf16").requires_grad_()
    do = _normal(rng, 3000, 512, dtype="bf16")

    def run():
        o = train.self_attention(qkv, off, 8, window=100, sinks=4)
        return o, torch.autograd.grad(o, qkv, do)[0]

    off = _offsets([1200, 1, 1700])
    want = run()
    torch.cuda.synchronize()
    outs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            outs.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in outs for a, b in zip(got, want))


def test_no_rows_and_no_sequences():
    train = _train()
    e = torch.zeros(0, 4, 64, device="cuda", requires_grad=True)
    o = train.attention(e, e, e, _offsets([]))
    assert o.shape == (0, 4, 64)
    assert torch.autograd.grad(o.sum(), e)[0].shape == (0, 4, 64)
    t = torch.ones(5, 4, 64, device="cuda", requires_grad=True)
    o = train.attention(t, t, t, _offsets([]))  # rows of no sequence
    assert not o.any() and not torch.autograd.grad(o.sum(), t)[0].any()
    k = torch.ones(3, 4, 64, device="cuda", requires_grad=True)
    o = train.attention(e, k, k, _offsets([0]), _offsets([3]))
    assert o.shape == (0, 4, 64) and not torch.autograd.grad(o.sum(), k)[0].any()
    o = train.attention(t, e, e, _offsets([5]), _offsets([0]))
    assert not o.any() and not torch.autograd.grad(o.sum(), t)[0].any()


@pytest.mark.parametrize("D", [64, 128])
def test_gradients_from_o_alone(D):
    """The C entry points without what o's rounding takes: to the same bounds, which carry that rounding."""
    import ctypes

    from paper_2609_15160_amd import tlf
    train, lib = _train(), tlf.load()
    rng = np.random.default_rng(8)
    n, heads, kv, window, sinks = 200, 4, 2, 50, 3
    q, do = (_normal(rng, n, heads, D, dtype="bf16") for _ in range(2))
    k, v = (_normal(rng, n, kv, D, dtype="bf16") for _ in range(2))
    off = _offsets([n])
    o, dq, dk, dv = (torch.full_like(t, float("nan")) for t in (q, q, k, v))
    lse = torch.empty(heads, n, device="cuda")
    shape = tlf.AttnShape(tlf.DTYPE_BF16, 1, heads, kv, D, n, n, window, sinks, D ** -0.5, heads * D, kv * D, kv * D, heads * D,
                          off.data_ptr(), off.data_ptr(), None)
    need = ctypes.c_size_t()
    assert lib.tlf_attn_ws_bytes(shape, need) == tlf.OK and need.value == 0
    train._run(lib.tlf_attn, q.device, shape, q, k, v, o, lse, None, None, 0)
    assert lib.tlf_attn_grad_ws_bytes(shape, need) == tlf.OK
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    train._run(lib.tlf_attn_grad, q.device, shape, do, q, k, v, o, lse, None, dq, heads * D, dk, kv * D, dv, kv * D, ws,
               need.value)
    arrays = [_np(t) for t in (q, k, v)]
    r = O.attention(*arrays, window, sinks, None, _np(do))
    lim = bounds(*arrays, r, window, sinks, D ** -0.5, "bf16", _np(do))
    for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        _within(t, r[name], lim[name], name)


def test_gradients_of_gradients_are_refused():
    train = _train()
    t = torch.ones(5, 4, 64, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(train.attention(t, t, t, _offsets([5])).sum(), t, create_graph=True)
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        torch.autograd.grad(g.sum(), t)
