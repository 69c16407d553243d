"""The operators around the FFN half of a training step, as cases that can be measured.

  attn   train.self_attention: causal attention of ragged sequences with a sliding
         window and first tokens that stay visible, forward or with its gradients
  token  train.attention: one new token of each sequence against a cache of keys
         and values that has room for more than it holds
  resid  train.residual_norm: the gated residual sum and the next norm in one,
         with the AdaLN scales of each row's group, forward or with its gradients
  clip   train.clip_grad_norm_: the global norm of many gradients, and clipping
  step   train.grad_norm and train.adamw_: an AdamW step with clipped gradients

`run` gives the operators in plain form (float32 products, sums and elementary
functions, rounded once at the end), or, with `own`, through the framework.
"""
import math
import random

import torch

own = False

EPS = 1e-5
BETAS, ADAM_EPS, LR, DECAY = (0.9, 0.95), 1e-8, 6e-4, 0.1
GRAD_STD = 1e-3
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# width, SwiGLU width, layers, vocabulary, positions of the models that the framework is used with
MODELS = {
    "d64": (64, 256, 1, 512, 64),
    "d256": (256, 512, 2, 512, 256),
    "d768": (768, 2048, 2, 32000, 2304),
    "d1024": (1024, 2816, 2, 32000, 4096),
    "d2048": (2048, 5504, 2, 32000, 4352),
}


def attn_(batch, most, least, heads, kv_heads, width, window=0, sinks=0, dtype="bf16", train=True, tail=0, mix=0):
    """`batch` sequences of least to most rows (`mix` says which), `tail` rows behind the last; window 0: all before."""
    return dict(kind="attn", batch=batch, most=most, least=least, heads=heads, kv_heads=kv_heads, width=width,
                window=window, sinks=sinks, dtype=dtype, train=train, tail=tail, mix=mix)


def token_(batch, room, least, heads, kv_heads, width, window=0, sinks=0, dtype="bf16", mix=0):
    """One token each against caches of `room` rows that hold least to room."""
    return dict(kind="token", batch=batch, most=room, least=least, heads=heads, kv_heads=kv_heads, width=width,
                window=window, sinks=sinks, dtype=dtype, mix=mix)


def resid_(rows, d, groups=0, y="bf16", post=False, train=True):
    """The residual rows are float32; y: the type of what is added, and of the normalised rows."""
    return dict(kind="resid", rows=rows, d=d, groups=groups, y=y, post=post, train=train)


def clip_(model, grad="f32", limit=0.5):
    """limit: max_norm over the norm that the gradients have about."""
    return dict(kind="clip", model=model, grad=grad, limit=limit)


def step_(model, grad="f32", copies=False, limit=0.5, step=1000):
    return dict(kind="step", model=model, grad=grad, copies=copies, limit=limit, step=step)


def listed():
    named = lambda name, c: dict(c, name=name)  # noqa: E731
    return [
        # a late loop of the 32 x 512 training batch: few tokens of each sequence are left, of some none
        named("attn_d768_32x130", attn_(32, 130, 0, 12, 12, 64, window=64, sinks=4, tail=37, mix=3)),
        # the first loop of the 8 x 4096 training batch, with a window and sinks
        named("attn_d1024_8x4096_w1024", attn_(8, 4096, 4096, 16, 16, 64, window=1024, sinks=4)),
        # the larger model: long sequences of odd lengths, every earlier token visible
        named("attn_d2048_4x4099", attn_(4, 4099, 2500, 16, 16, 128, mix=5)),
        # the small float32 model of parity runs, with shared key and value heads and ragged sequences
        named("attn_d256_f32_9x300", attn_(9, 300, 1, 4, 2, 64, window=100, sinks=3, dtype="f32", mix=2)),
        # a generated token of every sequence of the 256 x 2048 batch, a window over caches of different lengths
        named("token_d768_256_w512", token_(256, 2304, 700, 12, 12, 64, window=512, sinks=4, mix=1)),
        # a token of two very long sequences with shared heads: one long axis, few rows
        named("token_2x65001", token_(2, 65001, 40000, 16, 2, 128, mix=4)),
        # the deepest loop of a few short sequences: a handful of rows, forward only
        named("resid_d768_7", resid_(7, 768, groups=1, train=False)),
        # between attention and FFN in the first loop of the 8 x 4096 batch: eight depths, float32 stream, bf16 operands
        named("resid_d1024_32768_g8", resid_(32768, 1024, groups=8)),
        # a block with norms before and after, float32 throughout, a row count that fits no tile
        named("resid_d2048_9999_post", resid_(9999, 2048, groups=3, y="f32", post=True)),
        # the tiny model's gradients: launches and latency
        named("clip_d64", clip_("d64", limit=2.0)),
        # the larger model's bf16 gradients within the limit, as in most steps: read, not written
        named("clip_d2048_bf16", clip_("d2048", grad="bf16", limit=2.0)),
        # a float32 step of the 768-wide model whose gradients are over the limit
        named("step_d768", step_("d768")),
    ]


def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("attn", "attn", "attn", "token", "token", "resid", "resid", "clip", "step"))
    if kind in ("attn", "token"):
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        width = rng.choice((64, 64, 128) if dtype == "bf16" else (16, 64, 128))
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 1, 2, 3, 4))
        window = rng.choice((0, log_int(rng, 1, 4096), log_int(rng, 16, 2048)))
        sinks = rng.choice((0, rng.randint(1, 4), rng.randint(1, 64))) if window else 0
        if kind == "token":
            room = log_int(rng, 1, 65536)
            batch = log_int(rng, 1, max(1, min(512, (1 << 27) // (room * kv_heads * width))))
            return token_(batch, room, rng.choice((0, 1, room // 2, room)), heads, kv_heads, width, window, sinks, dtype,
                          mix=rng.randint(1, 1000000))
        most = log_int(rng, 1, 4200)
        cells = (1 << 30) * 64 // width if dtype == "bf16" else 1 << 26
        batch = log_int(rng, 1, max(1, min(64, cells // (heads * most * most))))
        return attn_(batch, most, rng.choice((0, 1, most // 2, most)), heads, kv_heads, width, window, sinks, dtype,
                     train=rng.random() < 0.75, tail=rng.choice((0, 0, rng.randint(1, 200))), mix=rng.randint(1, 1000000))
    if kind == "resid":
        d = rng.choice((64, 256, 768, 1024, 2048, 4 * rng.randint(1, 1024)))
        return resid_(log_int(rng, 1, 33554432 // max(d, 1024)), d, groups=rng.choice((0, 1, rng.randint(2, 16))),
                      y=rng.choice(("bf16", "bf16", "f32")), post=rng.random() < 0.4, train=rng.random() < 0.75)
    model, grad = rng.choice(("d64", "d256", "d768", "d1024")), rng.choice(("f32", "bf16"))
    limit = round(rng.uniform(0.05, 0.9) if rng.random() < 0.6 else rng.uniform(1.1, 4.0), 3)
    if kind == "clip":
        return clip_(model, grad, limit)
    return step_(model, grad, rng.random() < 0.5, limit, step=log_int(rng, 1, 100000))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def generator(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + stream)


def lengths(case):
    """Rows of each sequence: uniform over their range, the first has one at least."""
    rng = random.Random(case["mix"])
    n = [rng.randint(case["least"], case["most"]) for _ in range(case["batch"])]
    return [max(1, n[0])] + n[1:]


def shapes(model):
    """The model's tensors: token and position embeddings in one table, the router's weights and biases in one
    vector, each layer's matrices."""
    d, f, layers, vocab, positions = MODELS[model]
    return [(vocab + positions, d), (8 * (d + 1),)] + [(3 * d, d), (d, d), (2 * f, d), (d, f)] * layers


def starts(n):
    at = torch.zeros(len(n) + 1, dtype=torch.int64)
    at[1:] = torch.tensor(n, dtype=torch.int64).cumsum(0)
    return at


def inputs(case, seed):
    g = generator(seed, 2)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    kind = case["kind"]
    if kind == "attn":
        n, w, t = lengths(case), case["width"], TYPES[case["dtype"]]
        rows = sum(n) + case["tail"]
        s = {"qkv": normal(rows, (case["heads"] + 2 * case["kv_heads"]) * w, dtype=t), "offsets": starts(n).int().cuda()}
        if case["train"]:
            s["do"] = normal(rows, case["heads"] * w, std=0.1, dtype=t)
        return s
    if kind == "token":
        b, w, t, room = case["batch"], case["width"], TYPES[case["dtype"]], case["most"]
        return {"q": normal(b, case["heads"], w, dtype=t), "k": normal(b * room, case["kv_heads"], w, dtype=t),
                "v": normal(b * room, case["kv_heads"], w, dtype=t),
                "offsets": torch.arange(b + 1, dtype=torch.int32, device="cuda"),
                "k_offsets": torch.arange(b + 1, dtype=torch.int32, device="cuda") * room,
                "k_lengths": torch.tensor(lengths(case), dtype=torch.int32, device="cuda")}
    if kind == "resid":
        rows, d, n = case["rows"], case["d"], case["groups"]
        s = {"x": normal(rows, d, std=1.5), "y": normal(rows, d, std=0.7, dtype=TYPES[case["y"]]),
             "alpha": normal(n, d, std=0.2) if n else None, "gamma": normal(n, d, std=0.2) if n else None,
             "group": torch.randint(0, n, (rows,), generator=g, device="cuda", dtype=torch.int32) if n > 1 else None}
        if case["train"]:
            s["dh"] = normal(rows, d, std=0.01)
            s["dz"] = normal(rows, d, std=0.01, dtype=TYPES[case["y"]])
        return s
    size = shapes(case["model"])
    s = {"grads": [normal(*n, std=GRAD_STD, dtype=TYPES[case["grad"]]) for n in size],
         "max_norm": case["limit"] * GRAD_STD * math.sqrt(sum(math.prod(n) for n in size))}
    if kind == "step":
        s["params"] = [normal(*n, std=0.02) for n in size]
        s["m"] = [normal(*n, std=3e-4) for n in size]
        s["v"] = [normal(*n, std=1e-3).square() for n in size]
        s["copies"] = [p.to(torch.bfloat16) for p in s["params"]] if case["copies"] else None
    return s


def prepare(case, seed):
    s = dict(inputs(case, seed), case=case)
    if case.get("train"):
        for k in ("qkv", "x", "y", "alpha", "gamma"):
            if s.get(k) is not None:
                s[k].requires_grad_()
    if case["kind"] == "attn":  # where sequence b's row t lies, and whether it is there
        n, most = torch.tensor(lengths(case)), max(1, max(lengths(case)))
        t = torch.arange(most)
        s["there"] = (t < n[:, None]).cuda()
        s["at"] = torch.where(t < n[:, None], starts(lengths(case))[:-1, None] + t, 0).cuda()
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return {"attn": run_attn, "token": run_token, "resid": run_resid, "clip": run_clip, "step": run_step}[s["case"]["kind"]](s)


def visible(p, j, case):
    """Whether the query at position p sees the key at position j."""
    seen = j <= p
    if case["window"]:
        seen = seen & ((p - j < case["window"]) | (j < case["sinks"]))
    return seen


def run_attn(s):
    case = s["case"]
    if own:
        from paper_2609_15160_amd import train
        o = train.self_attention(s["qkv"], s["offsets"], case["heads"], case["kv_heads"], window=case["window"] or None,
                                 sinks=case["sinks"])
        if not case["train"]:
            return {"o": o}
        return {"o": o.detach(), "dqkv": torch.autograd.grad(o, s["qkv"], s["do"])[0]}
    return plain_attn(case, s["qkv"].detach(), s["at"], s["there"], s.get("do"))


def plain_attn(case, qkv, at, there, do):
    """The sequences padded to one length, [batch, heads, length, width] each of q, k, v."""
    heads, kv, w = case["heads"], case["kv_heads"], case["width"]
    each, (batch, most), scale = heads // kv, at.shape, 1.0 / math.sqrt(w)
    x = torch.where(there[..., None], qkv.float()[at], 0.0).reshape(batch, most, heads + 2 * kv, w).transpose(1, 2)
    q = x[:, :heads].contiguous()
    k = x[:, heads:heads + kv].repeat_interleave(each, 1).contiguous()
    v = x[:, heads + kv:].repeat_interleave(each, 1).contiguous()
    t = torch.arange(most, device=qkv.device)
    seen = visible(t[:, None], t[None, :], case)
    p = (q @ k.transpose(2, 3).contiguous()) * scale
    p = torch.where(seen, p, -math.inf)
    p = torch.exp(p - p.amax(3, keepdim=True))
    p = p / p.sum(3, keepdim=True)

    def rows(x):  # back to the rows of the sequences, zeros behind them
        out = torch.zeros(qkv.shape[0], x.shape[1], w, dtype=torch.float32, device=qkv.device)
        out[at[there]] = x.transpose(1, 2)[there]
        return out.reshape(qkv.shape[0], -1).to(qkv.dtype)

    o = rows(p @ v)
    if do is None:
        return {"o": o}
    g = torch.where(there[..., None], do.float()[at], 0.0).reshape(batch, most, heads, w).transpose(1, 2).contiguous()
    dv = p.transpose(2, 3).contiguous() @ g
    dp = g @ v.transpose(2, 3).contiguous()
    ds = p * (dp - (p * dp).sum(3, keepdim=True)) * scale
    dk = ds.transpose(2, 3).contiguous() @ q
    shared = lambda x: x.reshape(batch, kv, each, most, w).sum(2)  # noqa: E731
    return {"o": o, "dqkv": rows(torch.cat([ds @ k, shared(dk), shared(dv)], 1))}


def run_token(s):
    case = s["case"]
    if own:
        from paper_2609_15160_amd import train
        return {"o": train.attention(s["q"], s["k"], s["v"], s["offsets"], s["k_offsets"], s["k_lengths"],
                                     window=case["window"] or None, sinks=case["sinks"])}
    b, room, heads, kv, w = case["batch"], case["most"], case["heads"], case["kv_heads"], case["width"]
    q = s["q"].float().reshape(b, kv, heads // kv, w)
    k, v = (s[x].float().reshape(b, room, kv, w).transpose(1, 2).contiguous() for x in ("k", "v"))
    j, n = torch.arange(room, device=q.device), s["k_lengths"].long()[:, None]
    seen = visible(n - 1, j, case)[:, None, None, :]
    p = torch.where(seen, (q @ k.transpose(2, 3).contiguous()) / math.sqrt(w), -math.inf)
    p = torch.where(seen, torch.exp(p - p.amax(3, keepdim=True)), 0.0)
    o = (p @ v) / torch.clamp(p.sum(3, keepdim=True), min=1e-30)  # an empty cache: zeros
    return {"o": o.reshape(b, heads, w).to(s["q"].dtype)}


def run_resid(s):
    case = s["case"]
    if own:
        from paper_2609_15160_amd import train
        h, z = train.residual_norm(s["x"], s["y"], s["alpha"], s["gamma"], s["group"], eps=EPS, post_norm=case["post"])
        if not case["train"]:
            return {"h": h, "z": z}
        wanted = [t for t in (s["x"], s["y"], s["alpha"], s["gamma"]) if t is not None]
        got = list(torch.autograd.grad((h, z), wanted, (s["dh"], s["dz"]))) + [None, None]
        return {"h": h.detach(), "z": z.detach(), "dx": got[0], "dy": got[1], "dalpha": got[2], "dgamma": got[3]}
    return plain_resid(case, s)


def plain_resid(case, s):
    x, y = s["x"].detach(), s["y"].detach()
    of_row = lambda t: 1.0 if t is None else 1.0 + (t.detach() if s["group"] is None else t.detach()[s["group"].long()])  # noqa: E731
    yf, a, c = y.float(), of_row(s["alpha"]), of_row(s["gamma"])
    ry = torch.rsqrt(yf.square().mean(1, keepdim=True) + EPS) if case["post"] else 1.0
    t = yf * ry
    h = x + a * t
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    z = (h * r * c).to(y.dtype)
    if not case["train"]:
        return {"h": h, "z": z}
    dz = s["dz"].float()
    u = dz * c
    dh = s["dh"] + r * (u - h * (r * r * (u * h).mean(1, keepdim=True)))
    dt = dh * a
    dy = ry * (dt - yf * (ry * ry * (dt * yf).mean(1, keepdim=True))) if case["post"] else dt
    out = {"h": h, "z": z, "dx": dh, "dy": dy.to(y.dtype), "dalpha": None, "dgamma": None}
    if s["alpha"] is not None:
        out["dalpha"], out["dgamma"] = by_group(dh * t, s), by_group(dz * h * r, s)
    return out


def by_group(v, s):
    if s["group"] is None:
        return v.sum(0, keepdim=True)
    return torch.zeros_like(s["alpha"]).index_add_(0, s["group"].long(), v)


def plain_norm(grads):
    """The norm, summed in 64 bits."""
    return torch.sqrt(sum(g.double().square().sum() for g in grads))


def run_clip(s):
    if own:
        from paper_2609_15160_amd import train
        norm = train.clip_grad_norm_(s["grads"], s["max_norm"])
    else:
        norm = plain_norm(s["grads"])
        scale = torch.clamp(s["max_norm"] / norm, max=1.0).float()
        [g.copy_(g.float() * scale) for g in s["grads"]]
        norm = norm.float()
    return {"norm": norm, "grads": s["grads"]}


def run_step(s):
    case = s["case"]
    if own:
        from paper_2609_15160_amd import train
        norm, scale = train.grad_norm(s["grads"], s["max_norm"])
        train.adamw_(s["params"], s["grads"], s["m"], s["v"], case["step"], lr=LR, betas=BETAS, eps=ADAM_EPS,
                     weight_decay=DECAY, copies=s["copies"], grad_scale=scale)
    else:
        norm = plain_norm(s["grads"])
        scale = torch.clamp(s["max_norm"] / norm, max=1.0).float()
        [plain_adamw(k, s, case["step"], scale) for k in range(len(s["params"]))]
        norm = norm.float()
    return {"norm": norm, "params": s["params"], "copies": s["copies"], "m": s["m"], "v": s["v"]}


def plain_adamw(k, s, step, scale):
    p, m, v, g = s["params"][k], s["m"][k], s["v"][k], s["grads"][k].float() * scale
    b1, b2 = BETAS
    m.mul_(b1).add_(g * (1.0 - b1))
    v.mul_(b2).add_(g.square() * (1.0 - b2))
    root = torch.sqrt(v) * (1.0 / math.sqrt(1.0 - b2 ** step))
    p.mul_(1.0 - LR * DECAY).sub_(m * (LR / (1.0 - b1 ** step)) / (root + ADAM_EPS))
    if s["copies"] is not None:
        s["copies"][k].copy_(p)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def seen_by(p, case):
    """Keys that the query at position p sees."""
    if not case["window"]:
        return p + 1
    near = min(p + 1, case["window"])
    return near + min(case["sinks"], p + 1 - near)


def work(case):
    """Bytes: each input read once, each output written once."""
    size = lambda t: {"f32": 4, "bf16": 2}[t]  # noqa: E731
    if case["kind"] == "attn":
        n, w, b = lengths(case), case["width"], size(case["dtype"])
        pairs = sum(seen_by(p, case) for length in n for p in range(length))
        q, kv = sum(n) * case["heads"] * w * b, sum(n) * case["kv_heads"] * w * b
        both = 2 if case["train"] else 1  # q, k, v and o, and their gradients
        return {"bytes": both * (2 * q + 2 * kv), "flops": (14 if case["train"] else 4) * w * case["heads"] * pairs}
    if case["kind"] == "token":
        w, b, pairs = case["width"], size(case["dtype"]), sum(seen_by(n - 1, case) for n in lengths(case))
        return {"bytes": b * w * (2 * case["batch"] * case["heads"] + 2 * case["kv_heads"] * pairs) + 12 * case["batch"],
                "flops": 4 * w * case["heads"] * pairs}
    if case["kind"] == "resid":
        one, both = case["rows"] * case["d"], 2 if case["train"] else 1  # x, y, h and z, and their gradients
        return {"bytes": both * (2 * one * (4 + size(case["y"])) + 8 * case["groups"] * case["d"]) +
                (4 * case["rows"] if case["groups"] > 1 else 0), "flops": one * (24 if case["train"] else 8)}
    n = sum(math.prod(s) for s in shapes(case["model"]))
    if case["kind"] == "clip":  # gradients over the limit are written too
        return {"bytes": n * size(case["grad"]) * (2 if case["limit"] < 1 else 1), "flops": 2 * n}
    return {"bytes": n * (24 + size(case["grad"]) + (2 if case["copies"] else 0)), "flops": 17 * n}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    return {"attn": exact_attn, "token": exact_token, "resid": exact_resid, "clip": exact_clip,
            "step": exact_step}[case["kind"]](case, inputs(case, seed))


def attend(q, k, v, case):
    """softmax of one sequence: q [heads, m, w] at its last positions, k and v [kv_heads, n, w]."""
    each, n = q.shape[0] // k.shape[0], k.shape[1]
    at = torch.arange(n, device=q.device)
    hidden = torch.logical_not(visible(at[n - q.shape[1]:, None], at[None, :], case))
    score = torch.matmul(q, k.repeat_interleave(each, 0).mT) / w_root(q)
    return torch.softmax(score.masked_fill(hidden, -math.inf), -1).matmul(v.repeat_interleave(each, 0))


def w_root(q):
    return float(q.shape[-1]) ** 0.5


def exact_attn(case, s):
    heads, kv, w = case["heads"], case["kv_heads"], case["width"]
    qkv = s["qkv"].double()
    o, dqkv = torch.zeros_like(qkv[:, :heads * w]), torch.zeros_like(qkv) if case["train"] else None
    first = 0
    for n in lengths(case):
        if n:
            mine = slice(first, first + n)
            x = qkv[mine].reshape(n, -1, w).transpose(0, 1).contiguous().requires_grad_(case["train"])
            y = attend(x[:heads], x[heads:heads + kv], x[heads + kv:], case)
            o[mine] = y.detach().transpose(0, 1).reshape(n, -1)
            if case["train"]:
                g = s["do"][mine].double().reshape(n, heads, w).transpose(0, 1)
                dqkv[mine] = torch.autograd.grad(y, x, g)[0].transpose(0, 1).reshape(n, -1)
        first += n
    return {"o": o, "dqkv": dqkv} if case["train"] else {"o": o}


def exact_token(case, s):
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths(case)):
        if n:
            k, v = (s[x][b * case["most"]:b * case["most"] + n].double().transpose(0, 1) for x in ("k", "v"))
            o[b] = attend(s["q"][b].double()[:, None], k, v, case)[:, 0]
    return {"o": o}


def exact_resid(case, s):
    x, y = s["x"].double(), s["y"].double()
    of_row = torch.zeros(x.shape[0], dtype=torch.int64, device="cuda") if s["group"] is None else s["group"].long()
    if case["train"]:
        x.requires_grad_()
        y.requires_grad_()
    scales = [None if s[k] is None else s[k].double().requires_grad_(case["train"]) for k in ("alpha", "gamma")]
    gain = [1.0 if p is None else 1.0 + p[of_row] for p in scales]
    h = x + gain[0] * (y * (y.pow(2).mean(1, keepdim=True) + EPS).pow(-0.5) if case["post"] else y)
    z = h * (h.pow(2).mean(1, keepdim=True) + EPS).pow(-0.5) * gain[1]
    if not case["train"]:
        return {"h": h, "z": z}
    wanted = [x, y] + [p for p in scales if p is not None]
    got = list(torch.autograd.grad((h, z), wanted, (s["dh"].double(), s["dz"].double()))) + [None, None]
    return {"h": h.detach(), "z": z.detach(), "dx": got[0], "dy": got[1], "dalpha": got[2], "dgamma": got[3]}


def exact_clip(case, s):
    norm = torch.cat([g.double().flatten() for g in s["grads"]]).norm()
    factor = min(1.0, s["max_norm"] / float(norm))
    return {"norm": norm, "grads": [g.double() * factor for g in s["grads"]]}


def exact_step(case, s):
    b1, b2 = BETAS
    clipped = exact_clip(case, s)
    out = {"norm": clipped["norm"], "params": [], "copies": [] if case["copies"] else None, "m": [], "v": []}
    for p, g, m, v in zip(s["params"], clipped["grads"], s["m"], s["v"]):
        m = m.double() * b1 + g * (1 - b1)
        v = v.double() * b2 + g * g * (1 - b2)
        p = p.double() * (1 - LR * DECAY) - LR * (m / (1 - b1 ** case["step"])) / ((v / (1 - b2 ** case["step"])).sqrt() + ADAM_EPS)
        out["params"].append(p)
        if case["copies"]:
            out["copies"].append(p)
        out["m"].append(m)
        out["v"].append(v)
    return out
