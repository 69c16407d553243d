"""The training operators of the FFN half of the block, as cases that can be measured.

  norm   train.rms_norm: RMSNorm of the float32 residual rows, with the AdaLN
         scale of each row's group or without, forward or with its gradients
  ffn    train.ffn: the SwiGLU feed-forward block, forward or with its gradients
  adamw  train.adamw_: one AdamW step over a model's tensors, moments in float32
         or in 8 bits (e4m3 and e5m2 with a float32 scale for 256 elements)

`run` gives the operators in plain form (float32 products, sums and elementary
functions, rounded once at the end), or, with `own`, through the framework.
"""
import math

import torch

own = False

EPS = 1e-5
BETAS, ADAM_EPS, LR, DECAY = (0.9, 0.95), 1e-8, 6e-4, 0.1
BLOCK = 256  # elements that share a scale of the 8-bit moments
M_MAX, V_MAX, V_MIN = 448.0, 57344.0, 2.0 ** -16  # largest e4m3, largest and smallest e5m2 value
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# width, SwiGLU width, layers, vocabulary, positions of the models that the framework is used with
MODELS = {
    "d64": (64, 256, 1, 512, 64),
    "d256": (256, 512, 2, 512, 256),
    "d768": (768, 2048, 2, 32000, 2304),
    "d1024": (1024, 2816, 2, 32000, 4096),
    "d2048": (2048, 5504, 2, 32000, 4352),
}


def norm_(rows, d, groups=0, out="bf16", train=True, x="f32"):
    return dict(kind="norm", rows=rows, d=d, groups=groups, x=x, out=out, train=train)


def ffn_(rows, d, f, dtype="bf16", train=True):
    return dict(kind="ffn", rows=rows, d=d, f=f, dtype=dtype, train=train)


def adamw_(model, bits=32, grad="f32", copies=False, step=1000):
    return dict(kind="adamw", model=model, bits=bits, grad=grad, copies=copies, step=step)


def listed():
    named = lambda name, c: dict(c, name=name)  # noqa: E731
    return [
        # the deepest loop of a few short sequences: a handful of rows, forward only
        named("norm_d768_7", norm_(7, 768, groups=1, train=False)),
        # the first loop of a training batch of 8 x 4096 tokens: eight depths, each with its own scale
        named("norm_d1024_32768_g8", norm_(32768, 1024, groups=8)),
        # no conditioning, float32 throughout, a row count that fits no tile
        named("norm_d2048_9999_f32", norm_(9999, 2048, out="f32")),
        # one token through the larger model's FFN (a generated token outside the decode path)
        named("ffn_d2048_1", ffn_(1, 2048, 5504, train=False)),
        # scoring: forward only over a batch
        named("ffn_d768_6000_forward", ffn_(6000, 768, 2048, train=False)),
        # a late loop of a small training batch, where few tokens are left
        named("ffn_d768_333", ffn_(333, 768, 2048)),
        # a loop of the 8 x 4096 training batch with half of its tokens active
        named("ffn_d1024_16384", ffn_(16384, 1024, 2816)),
        # the larger model, an odd number of active tokens
        named("ffn_d2048_8191", ffn_(8191, 2048, 5504)),
        # the small float32 model of the tests and of parity runs
        named("ffn_d256_3001_f32", ffn_(3001, 256, 512, dtype="f32")),
        # the tiny model's optimizer step: launches and latency
        named("adamw_d64", adamw_("d64")),
        # float32 training of the 768-wide model
        named("adamw_d768", adamw_("d768")),
        # mixed precision: bf16 gradients, float32 parameters with bf16 copies, moments in 8 bits
        named("adamw_d2048_8bit", adamw_("d2048", bits=8, grad="bf16", copies=True)),
    ]


def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "ffn", "ffn", "adamw"))
    if kind == "norm":
        d = rng.choice((64, 256, 768, 1024, 2048, 4 * rng.randint(1, 1024)))
        return norm_(log_int(rng, 1, 33554432 // max(d, 1024)), d, groups=rng.choice((0, 1, rng.randint(2, 16))),
                     out=rng.choice(("bf16", "bf16", "f32")), x=rng.choice(("f32", "f32", "bf16")),
                     train=rng.random() < 0.75)
    if kind == "ffn":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        if rng.random() < 0.6:
            d, f = MODELS[rng.choice(("d768", "d1024", "d2048") if dtype == "bf16" else ("d64", "d256"))][:2]
        else:
            d, f = 64 * rng.randint(1, 24), 64 * rng.randint(1, 48)
        most = 92000000000 if dtype == "bf16" else 4000000000
        return ffn_(log_int(rng, 1, max(1, min(32768, most // (d * f)))), d, f, dtype=dtype, train=rng.random() < 0.75)
    return adamw_(rng.choice(("d64", "d256", "d768", "d1024")), bits=rng.choice((8, 32)),
                  grad=rng.choice(("f32", "bf16")), copies=rng.random() < 0.5, step=log_int(rng, 1, 100000))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def generator(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + stream)


def shapes(model):
    """The model's tensors: token and position embeddings in one table, the router's weights and biases in one
    vector, each layer's matrices."""
    d, f, layers, vocab, positions = MODELS[model]
    return [(vocab + positions, d), (8 * (d + 1),)] + [(3 * d, d), (d, d), (2 * f, d), (d, f)] * layers


def inputs(case, seed):
    g = generator(seed, 1)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    if case["kind"] == "norm":
        rows, d, n = case["rows"], case["d"], case["groups"]
        s = {"x": normal(rows, d, std=1.5, dtype=TYPES[case["x"]]), "gamma": normal(n, d, std=0.2) if n else None,
             "group": torch.randint(0, n, (rows,), generator=g, device="cuda", dtype=torch.int32) if n > 1 else None}
        if case["train"]:
            s["dy"] = normal(rows, d, std=0.01, dtype=TYPES[case["out"]])
        return s
    if case["kind"] == "ffn":
        rows, d, f, t = case["rows"], case["d"], case["f"], TYPES[case["dtype"]]
        s = {"x": normal(rows, d, dtype=t), "w_gate_up": normal(2 * f, d, std=0.5 / math.sqrt(d) + 0.01, dtype=t),
             "w_down": normal(d, f, std=0.02, dtype=t)}
        if case["train"]:
            s["dy"] = normal(rows, d, std=0.01, dtype=t)
        return s
    size = shapes(case["model"])
    s = {"params": [normal(*n, std=0.02) for n in size],
         "grads": [normal(*n, std=1e-3, dtype=TYPES[case["grad"]]) for n in size],
         "m": [normal(*n, std=3e-4) for n in size], "v": [normal(*n, std=1e-3).square() for n in size]}
    s["copies"] = [p.to(torch.bfloat16) for p in s["params"]] if case["copies"] else None
    if case["bits"] == 8:
        s["m"] = [store(m.double(), M_MAX, torch.float8_e4m3fn) for m in s["m"]]
        s["v"] = [store(v.double(), V_MAX, torch.float8_e5m2) for v in s["v"]]
    return s


def prepare(case, seed):
    s = inputs(case, seed)
    leaves = {"norm": ("x", "gamma"), "ffn": ("x", "w_gate_up", "w_down"), "adamw": ()}[case["kind"]]
    if case.get("train"):
        for k in leaves:
            if s[k] is not None:
                s[k].requires_grad_()
    return dict(s, case=case)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return {"norm": run_norm, "ffn": run_ffn, "adamw": run_adamw}[s["case"]["kind"]](s)


def run_norm(s):
    case = s["case"]
    if own:
        from paper_2609_15160_amd import train
        if not case["train"]:
            return {"y": train.rms_norm(s["x"], s["gamma"], s["group"], eps=EPS, dtype=TYPES[case["out"]])}
        y = train.rms_norm(s["x"], s["gamma"], s["group"], eps=EPS, dtype=TYPES[case["out"]])
        wanted = [t for t in (s["x"], s["gamma"]) if t is not None]
        got = torch.autograd.grad(y, wanted, s["dy"])
        return {"y": y.detach(), "dx": got[0], "dgamma": got[1] if len(got) > 1 else None}
    return plain_norm(s["x"].detach(), s["gamma"], s["group"], s.get("dy"), TYPES[case["out"]])


def plain_norm(x, gamma, group, dy, out):
    xf = x.float()
    r = torch.rsqrt(xf.square().mean(1, keepdim=True) + EPS)
    scale = 1.0 if gamma is None else 1.0 + gamma.detach() if group is None else 1.0 + gamma.detach()[group.long()]
    y = (xf * r * scale).to(out)
    if dy is None:
        return {"y": y}
    g = dy.float()
    h = g * scale
    dx = (r * (h - xf * (r * r * (h * xf).mean(1, keepdim=True)))).to(x.dtype)
    dgamma = None
    if gamma is not None:
        part = g * xf * r
        if group is None:
            dgamma = part.sum(0, keepdim=True)
        else:
            dgamma = torch.zeros_like(gamma).index_add_(0, group.long(), part)
    return {"y": y, "dx": dx, "dgamma": dgamma}


def run_ffn(s):
    if own:
        from paper_2609_15160_amd import train
        y = train.ffn(s["x"], s["w_gate_up"], s["w_down"])
        if not s["case"]["train"]:
            return {"y": y}
        dx, dgu, dd = torch.autograd.grad(y, (s["x"], s["w_gate_up"], s["w_down"]), s["dy"])
        return {"y": y.detach(), "dx": dx, "dw_gate_up": dgu, "dw_down": dd}
    return plain_ffn(s["x"].detach(), s["w_gate_up"].detach(), s["w_down"].detach(), s.get("dy"))


def plain_ffn(x, w_gate_up, w_down, dy):
    t, f = x.dtype, w_down.shape[1]
    xf, wgu, wd = x.float(), w_gate_up.float(), w_down.float()
    gu = xf @ wgu.T
    g, u = gu[:, :f], gu[:, f:]
    sig = 1.0 / (1.0 + torch.exp(-g))
    act = g * sig
    a = act * u
    y = (a @ wd.T).to(t)
    if dy is None:
        return {"y": y}
    dyf = dy.float()
    da = dyf @ wd
    dgu = torch.cat([da * u * sig * (1.0 + g * (1.0 - sig)), da * act], 1)
    return {"y": y, "dx": (dgu @ wgu).to(t), "dw_gate_up": (dgu.T @ xf).to(t), "dw_down": (dyf.T @ a).to(t)}


def run_adamw(s):
    case = s["case"]
    if own:
        from paper_2609_15160_amd import train
        train.adamw_(s["params"], s["grads"], s["m"], s["v"], case["step"], lr=LR, betas=BETAS, eps=ADAM_EPS,
                     weight_decay=DECAY, copies=s["copies"])
    else:
        [plain_adamw(k, s, case) for k in range(len(s["params"]))]
    return {"params": s["params"], "copies": s["copies"], "m": s["m"], "v": s["v"]}


def plain_adamw(k, s, case):
    """One tensor's step in place; 8-bit moments in 64 bits up to their rounding, whose borders 32 bits would shift."""
    p, g, m, v = s["params"][k], s["grads"][k], s["m"][k], s["v"][k]
    b1, b2 = BETAS
    if case["bits"] == 8:
        gd = g.double()
        m1 = b1 * load(*m, p.shape) + (1.0 - b1) * gd
        v1 = b2 * load(*v, p.shape) + (1.0 - b2) * gd.square()
        [old.copy_(new) for old, new in zip(m, store(m1, M_MAX, torch.float8_e4m3fn))]
        [old.copy_(new) for old, new in zip(v, store(v1, V_MAX, torch.float8_e5m2))]
        m1, v1 = m1.float(), v1.float()
    else:
        gf = g.float()
        m1 = m.mul_(b1).add_(gf * (1.0 - b1))
        v1 = v.mul_(b2).add_(gf.square() * (1.0 - b2))
    root = torch.sqrt(v1) * (1.0 / math.sqrt(1.0 - b2 ** case["step"]))
    p.mul_(1.0 - LR * DECAY).sub_(m1 * (LR / (1.0 - b1 ** case["step"])) / (root + ADAM_EPS))
    if s["copies"] is not None:
        s["copies"][k].copy_(p)


def store(v, most, dtype):
    """(codes, scales) of a float64 tensor: 8-bit floats of v / scale, one float32 scale for each 256 elements."""
    n = v.numel()
    rows = torch.nn.functional.pad(v.reshape(-1), (0, -n % BLOCK)).reshape(-1, BLOCK)
    scale = (rows.abs().amax(1).float().double() / most).float()
    t = torch.where(scale[:, None] > 0, rows / scale[:, None].double(), 0.0).clamp(-most, most)
    if dtype == torch.float8_e5m2:  # a second moment that is not zero does not become zero
        t = torch.where(t > 0, t.clamp(min=V_MIN), t)
    return t.float().reshape(-1)[:n].to(dtype).reshape(v.shape), scale


def load(codes, scale, shape):
    return codes.reshape(-1).double().mul_(scale.double().repeat_interleave(BLOCK)[:codes.numel()]).reshape(shape)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Bytes: each input read once, each output written once."""
    size = lambda t: {"f32": 4, "bf16": 2}[t]  # noqa: E731
    if case["kind"] == "norm":
        one = case["rows"] * case["d"]
        both = 2 if case["train"] else 1  # x and y, and their gradients
        return {"bytes": both * (one * (size(case["x"]) + size(case["out"])) + 4 * case["groups"] * case["d"]) +
                (4 * case["rows"] if case["groups"] > 1 else 0), "flops": one * (12 if case["train"] else 4)}
    if case["kind"] == "ffn":
        n, d, f = case["rows"], case["d"], case["f"]
        both = 2 if case["train"] else 1
        return {"bytes": both * size(case["dtype"]) * (2 * n * d + 3 * d * f),
                "flops": (18 if case["train"] else 6) * n * d * f}
    n = sum(math.prod(s) for s in shapes(case["model"]))
    moments = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
    return {"bytes": n * (8 + size(case["grad"]) + moments + (2 if case["copies"] else 0)), "flops": 14 * n}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    return {"norm": exact_norm, "ffn": exact_ffn, "adamw": exact_adamw}[case["kind"]](case, inputs(case, seed))


def exact_norm(case, s):
    x = s["x"].double()
    rms = (x.pow(2).sum(1) / x.shape[1] + EPS).sqrt()
    unit = x / rms[:, None]
    gain = torch.ones_like(x)
    if s["gamma"] is not None:
        of_row = 0 if s["group"] is None else s["group"]
        gain = gain + s["gamma"].double()[torch.zeros_like(x[:, 0], dtype=torch.int64) + of_row]
    y = unit * gain
    if not case["train"]:
        return {"y": y}
    dy = s["dy"].double()
    du = dy * gain
    dx = (du - unit * (du * unit).sum(1, keepdim=True) / x.shape[1]) / rms[:, None]
    dgamma = None
    if s["gamma"] is not None:
        each = dy * unit
        at = torch.zeros(x.shape[0], dtype=torch.int32, device="cuda") if s["group"] is None else s["group"]
        dgamma = torch.stack([each[at == k].sum(0) for k in range(case["groups"])])
    return {"y": y, "dx": dx, "dgamma": dgamma}


def exact_ffn(case, s):
    x, f = s["x"].double(), case["f"]
    gate, up, down = s["w_gate_up"][:f].double(), s["w_gate_up"][f:].double(), s["w_down"].double()
    g, u = x.matmul(gate.T), x.matmul(up.T)
    open_ = torch.sigmoid(g)
    y = (u * g * open_).matmul(down.T)
    if not case["train"]:
        return {"y": y}
    dy = s["dy"].double()
    da = dy.matmul(down)
    dg, du = da * u * (open_ + g * open_ * (1 - open_)), da * g * open_
    return {"y": y, "dx": dg.matmul(gate) + du.matmul(up), "dw_gate_up": torch.cat([dg.T.matmul(x), du.T.matmul(x)]),
            "dw_down": dy.T.matmul(u * g * open_)}


def exact_adamw(case, s):
    b1, b2 = BETAS
    out = {"params": [], "copies": [] if case["copies"] else None, "m": [], "v": []}
    for p, g, m, v in zip(s["params"], s["grads"], s["m"], s["v"]):
        p, g = p.double(), g.double()
        if case["bits"] == 8:
            each = torch.arange(p.numel(), device="cuda").reshape(p.shape) // BLOCK
            m, v = m[0].double() * m[1].double()[each], v[0].double() * v[1].double()[each]
        m = m.double() * b1 + g * (1 - b1)
        v = v.double() * b2 + g * g * (1 - b2)
        step = (m / (1 - b1 ** case["step"])) / ((v / (1 - b2 ** case["step"])).sqrt() + ADAM_EPS)
        p = p - LR * DECAY * p - LR * step
        out["params"].append(p)
        if case["copies"]:
            out["copies"].append(p)
        out["m"].append(m if case["bits"] == 32 else exact_codes(m, M_MAX, torch.float8_e4m3fn))
        out["v"].append(v if case["bits"] == 32 else exact_codes(v, V_MAX, torch.float8_e5m2))
    return out


def exact_codes(v, most, dtype):
    """(values of the codes, scales): each block's largest magnitude is at the top of the 8-bit range."""
    flat = v.flatten()
    ids = torch.arange(flat.numel(), device="cuda") // BLOCK
    top = torch.zeros(int(ids[-1]) + 1, dtype=torch.float64, device="cuda").scatter_reduce(0, ids, flat.abs(), "amax")
    scale = (top.float().double() / most).float()
    t = torch.nan_to_num(flat / scale.double()[ids], nan=0.0)
    if dtype == torch.float8_e5m2:
        t = torch.where((t > 0) & (t < V_MIN), V_MIN, t)
    return t.clamp(-most, most).float().to(dtype).double().reshape(v.shape), scale.double()
