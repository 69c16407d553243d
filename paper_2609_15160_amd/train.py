"""Training-side gather-scatter (Section 3.2, Eq. 6-7) and the router's
straight-through estimator (Appendix B) as autograd functions over libtlf.

Argument marshalling only: the active set, the gather, the scatter, their
gradients and the estimator all run in libtlf's HIP kernels, on the current
torch stream.

    p = plan(depth, batch, seq_len, loop)     # loop i's active rows
    x = gather(h, p)                          # [p.count, d], Eq. 6
    h = scatter(h, block(x), p)               # Eq. 7 (scatter_ writes into h)

Of the block, all but its projections (torch.nn.functional.linear) is here: rms_norm
(with the AdaLN scale of each row's group), self_attention among the gathered rows
(Eq. 10; with a sliding window and sinks if asked), residual_norm (the gated residual
and the next norm in one pass), ffn, and the optimizer's step: adamw_ and AdamW, and
grad_norm and clip_grad_norm_.

    z = rms_norm(x, gamma_msa, group, dtype=torch.bfloat16)
    a = self_attention(linear(z, w_qkv), p.offsets, heads)
    x, z = residual_norm(x, linear(a, w_o), alpha_msa, gamma_mlp, group)
    x, z = residual_norm(x, ffn(z, w_gate_up, w_down), alpha_mlp, next_gamma_msa, group)
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass

import torch

from . import tlf


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(status: int, where: str):
    if status != tlf.OK:
        raise tlf.TlfError(status, where)


def _rows_tensor(h: torch.Tensor, name: str):
    if h.dtype != torch.float32 or h.dim() != 2 or not h.is_cuda or not h.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous float32 [rows, d] CUDA tensor")


@dataclass
class LoopPlan:
    """Active set of one loop: compact index -> row (`index`), row -> compact
    index or -1 (`slot`), each sequence's start in the compact tensor plus the
    total (`offsets`), the count on the device (`count_dev`) and on the host."""
    loop: int
    rows: int
    index: torch.Tensor
    slot: torch.Tensor
    offsets: torch.Tensor
    count_dev: torch.Tensor
    count: int


def plan_workspace(batch: int, seq_len: int, device="cuda") -> torch.Tensor:
    """Scratch for the multi-workgroup planner (one int32 count per chunk of rows)."""
    return torch.empty(max(tlf.gs_plan_ws_bytes(batch * seq_len), 4), dtype=torch.uint8, device=device)


def plan(depth: torch.Tensor, batch: int, seq_len: int, loop: int, workspace: torch.Tensor = None) -> LoopPlan:
    """Active rows of loop `loop`; reads the count back to the host (one
    synchronisation), since the compact tensor's size must be known there.
    With a `workspace` (plan_workspace) the multi-workgroup planner runs,
    otherwise the single-workgroup one; both give the same plan."""
    if depth.dtype != torch.int32 or not depth.is_cuda or not depth.is_contiguous():
        raise ValueError("depth: expected a contiguous int32 CUDA tensor")
    rows = batch * seq_len
    if depth.numel() != rows:
        raise ValueError(f"depth holds {depth.numel()} entries, batch * seq_len = {rows}")
    dev = depth.device
    index = torch.empty(max(rows, 1), dtype=torch.int32, device=dev)
    slot = torch.empty(max(rows, 1), dtype=torch.int32, device=dev)
    offsets = torch.empty(batch + 1, dtype=torch.int32, device=dev)
    count = torch.empty(1, dtype=torch.int32, device=dev)
    if workspace is None:
        _check(tlf.load().tlf_gs_plan(_ptr(depth), batch, seq_len, loop, _ptr(index), _ptr(slot), _ptr(offsets),
                                      _ptr(count), _stream()), "tlf_gs_plan")
    else:
        if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace: expected a contiguous uint8 CUDA tensor (plan_workspace)")
        _check(tlf.load().tlf_gs_plan_ws(_ptr(depth), batch, seq_len, loop, _ptr(index), _ptr(slot),
                                         _ptr(offsets), _ptr(count), _ptr(workspace), workspace.numel(),
                                         _stream()), "tlf_gs_plan_ws")
    n = int(count.item())
    return LoopPlan(loop, rows, index[:n], slot[:rows], offsets, count, n)


def gather_raw(h: torch.Tensor, p: LoopPlan, out: torch.Tensor = None) -> torch.Tensor:
    _rows_tensor(h, "h")
    d = h.shape[1]
    if out is None:
        out = torch.empty((p.count, d), dtype=h.dtype, device=h.device)
    _check(tlf.load().tlf_gs_gather(_ptr(h), _ptr(p.index), _ptr(p.count_dev), p.count, d, _ptr(out), _stream()),
           "tlf_gs_gather")
    return out


def scatter_raw(h_prev: torch.Tensor, y: torch.Tensor, p: LoopPlan, out: torch.Tensor = None) -> torch.Tensor:
    """Eq. 7 into `out` (a new tensor by default; `out is h_prev` updates in place)."""
    _rows_tensor(h_prev, "h_prev")
    _rows_tensor(y, "y")
    if h_prev.shape[0] != p.rows or y.shape != (p.count, h_prev.shape[1]):
        raise ValueError(f"scatter: h_prev {tuple(h_prev.shape)}, y {tuple(y.shape)}, plan rows {p.rows} "
                         f"count {p.count}")
    if out is None:
        out = torch.empty_like(h_prev)
    # with no active row y is empty (no address) and never read: pass h_prev's
    yp = _ptr(y) if y.numel() else _ptr(h_prev)
    _check(tlf.load().tlf_gs_scatter(_ptr(h_prev), yp, _ptr(p.slot), p.rows, h_prev.shape[1], _ptr(out),
                                     _stream()), "tlf_gs_scatter")
    return out


def expand_raw(y: torch.Tensor, p: LoopPlan) -> torch.Tensor:
    """The compact rows `y` at their rows of a new [rows, d] tensor, zeros elsewhere (the gather's gradient)."""
    _rows_tensor(y, "y")
    if y.shape[0] != p.count:
        raise ValueError(f"expand: y {tuple(y.shape)}, plan rows {p.rows} count {p.count}")
    out = torch.empty((p.rows, y.shape[1]), dtype=y.dtype, device=y.device)
    # with no active row y is empty (no address) and never read: pass out's
    yp = _ptr(y) if y.numel() else _ptr(out)
    _check(tlf.load().tlf_gs_expand(yp, _ptr(p.slot), p.rows, y.shape[1], _ptr(out), _stream()), "tlf_gs_expand")
    return out


class _Gather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, p):
        ctx.p = p
        ctx.shape = h.shape
        return gather_raw(h.contiguous(), p)

    @staticmethod
    def backward(ctx, g):
        if ctx.shape[0] != ctx.p.rows:
            raise ValueError(f"gather: h {tuple(ctx.shape)}, plan rows {ctx.p.rows} count {ctx.p.count}")
        return expand_raw(g.contiguous(), ctx.p), None


class _Scatter(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h_prev, y, p):
        ctx.p = p
        return scatter_raw(h_prev.contiguous(), y.contiguous(), p)

    @staticmethod
    def backward(ctx, g):
        g = g.contiguous()
        return g, gather_raw(g, ctx.p), None


class _ScatterInPlace(torch.autograd.Function):
    """Eq. 7 written into h_prev: neither gradient needs the previous state
    (the block's backward uses its own compact input), so the rows that no
    loop touches need not be copied."""
    @staticmethod
    def forward(ctx, h_prev, y, p):
        ctx.p = p
        scatter_raw(h_prev, y.contiguous(), p, out=h_prev)
        ctx.mark_dirty(h_prev)
        return h_prev

    @staticmethod
    def backward(ctx, g):
        g = g.contiguous()
        return g, gather_raw(g, ctx.p), None


class _Ste(torch.autograd.Function):
    @staticmethod
    def forward(ctx, score, depth):
        ctx.save_for_backward(score, depth)
        value = torch.empty(depth.shape, dtype=torch.float32, device=depth.device)
        _check(tlf.load().tlf_ste(_ptr(depth), None, None, depth.numel(), _ptr(value), None, _stream()), "tlf_ste")
        return value

    @staticmethod
    def backward(ctx, g):
        score, depth = ctx.saved_tensors
        g = g.contiguous().float()
        ds = torch.empty_like(score)
        _check(tlf.load().tlf_ste(None, _ptr(score), _ptr(g), score.numel(), None, _ptr(ds), _stream()), "tlf_ste")
        return ds, None


def gather(h: torch.Tensor, p: LoopPlan) -> torch.Tensor:
    """Eq. 6 with its gradient (the compact gradient added into the rows)."""
    return _Gather.apply(h, p)


def scatter(h_prev: torch.Tensor, y: torch.Tensor, p: LoopPlan) -> torch.Tensor:
    """Eq. 7 with its gradient (identity to h_prev, gathered rows to y)."""
    return _Scatter.apply(h_prev, y, p)


def scatter_(h_prev: torch.Tensor, y: torch.Tensor, p: LoopPlan) -> torch.Tensor:
    """Eq. 7 in place on h_prev (which must be contiguous and not a leaf that
    requires grad); same gradients as `scatter`, traffic only on active rows."""
    return _ScatterInPlace.apply(h_prev, y, p)


def ste(score: torch.Tensor, depth: torch.Tensor) -> torch.Tensor:
    """Appendix B: value `depth`, gradient sigma'(score) to `score`."""
    if score.dtype != torch.float32 or depth.dtype != torch.int32 or score.shape != depth.shape:
        raise ValueError("ste: float32 score and int32 depth of one shape expected")
    return _Ste.apply(score.contiguous(), depth.contiguous())


# ---------------------------------------------------------------------------
# The block's FFN half: RMSNorm, the gated FFN, and the optimizer's step
#
# rms_norm, ffn, residual_norm and the attention may be captured into a graph, their
# backward pass with them if no graph from before the capture holds the same leaves:
# autograd runs a leaf's gradient on the stream where the leaf was first used.
# grad_norm and clip_grad_norm_ may be captured too.
# ---------------------------------------------------------------------------

_DTYPE = {torch.float32: tlf.DTYPE_F32, torch.bfloat16: tlf.DTYPE_BF16}


def _run(fn, device: torch.device, *args) -> None:
    """fn(*args, stream) with `device` current, on that device's current stream; tensors among the arguments stand for
    their addresses."""
    args = [a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args]
    if device.index == torch.cuda.current_device():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    else:
        with torch.cuda.device(device):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    _check(status, fn.__name__)


def _same_device(t, *others):
    for o in others:
        if o is not None and o.device != t.device:
            raise ValueError(f"tensors on {t.device} and {o.device}: one device expected")


def _int32(name, *tensors):
    if any(n >= 1 << 31 for t in tensors if t is not None for n in t.shape):
        raise ValueError(f"{name}: a dimension of 2^31 or more")


def _wants_grad(*tensors) -> bool:
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _workspace(fn, *args, device):
    need = ctypes.c_size_t()
    _check(fn(*args, ctypes.byref(need)), fn.__name__)
    if need.value == 0:
        return None, 0
    return torch.empty(need.value, dtype=torch.uint8, device=device), need.value


class _NoSecond(torch.autograd.Function):
    """The first n tensors, gradients that depend on the rest: their own gradients are refused."""
    @staticmethod
    def forward(ctx, n, *tensors):
        return tensors[:n]

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("rms_norm, residual_norm, attention and ffn have no gradients of gradients")


def _first_order(backward):
    """A backward pass without one of its own, backward(ctx, saved tensors, *grads): where a graph of it is built
    (create_graph), differentiating that is refused.  The saved tensors are unpacked here, once: a recomputed one
    (checkpointing) is there for one taking only."""
    @functools.wraps(backward)
    def run(ctx, *grads):
        saved = ctx.saved_tensors
        if not torch.is_grad_enabled():
            return backward(ctx, saved, *grads)
        with torch.no_grad():
            out = backward(ctx, saved, *grads)
        return _NoSecond.apply(len(out), *out, *(t for t in (*saved, *grads) if t is not None))
    return run


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, group, eps, dtype, grad):
        rows, d = x.shape
        groups = 0 if gamma is None else gamma.numel() // d
        y = torch.empty((rows, d), dtype=dtype, device=x.device)
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device) if grad else None
        _run(tlf.load().tlf_rms_norm, x.device, x, _DTYPE[x.dtype], gamma, group, groups, rows, d, eps, y, _DTYPE[dtype],
             rstd)
        if grad:
            ctx.save_for_backward(x, gamma, group, rstd)
        return y

    @staticmethod
    @_first_order
    def backward(ctx, saved, dy):
        x, gamma, group, rstd = saved
        rows, d = x.shape
        groups = 0 if gamma is None else gamma.numel() // d
        dy = _aligned(dy)
        dx = torch.empty_like(x) if ctx.needs_input_grad[0] else None
        dgamma = torch.empty_like(gamma) if ctx.needs_input_grad[1] else None
        lib = tlf.load()
        ws, n = None, 0
        if dgamma is not None:
            ws, n = _workspace(lib.tlf_rms_norm_grad_ws_bytes, groups, rows, d, device=x.device)
        _run(lib.tlf_rms_norm_grad, x.device, dy, _DTYPE[dy.dtype], x, _DTYPE[x.dtype], gamma, group, groups, rstd, rows,
             d, dx, dgamma, ws, n)
        return dx, dgamma, None, None, None, None


def _aligned(t: torch.Tensor) -> torch.Tensor:
    """`t` contiguous and from a 16-byte boundary, copied where it is not."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def rms_norm(x: torch.Tensor, gamma: torch.Tensor = None, group: torch.Tensor = None, eps: float = 1e-5,
             dtype: torch.dtype = None) -> torch.Tensor:
    """RMSNorm of the rows of x ([rows, d], float32 or bfloat16) times 1 + gamma, with gradients to x and gamma.

    gamma is None, one [d] or [1, d] scale, or [groups, d] scales of which row r takes number group[r] (int32 [rows];
    a row whose number is none of them takes no scale): the AdaLN modulation of each token's depth.  The result has
    `dtype` (x's by default).  d is a multiple of 4 up to 4096, there are 16 groups and 2^30 rows at most.  Squares are
    summed in float32: a row whose sum of squares passes its range comes out as zeros."""
    if x.dim() != 2 or x.dtype not in _DTYPE or not x.is_cuda:
        raise ValueError("rms_norm: expected a float32 or bfloat16 [rows, d] CUDA tensor")
    dtype = dtype or x.dtype
    if dtype not in _DTYPE:
        raise ValueError(f"rms_norm: dtype {dtype}, expected float32 or bfloat16")
    d = x.shape[1]
    if gamma is not None:
        if gamma.dtype != torch.float32 or gamma.dim() not in (1, 2) or gamma.shape[-1] != d:
            raise ValueError(f"rms_norm: gamma {tuple(gamma.shape)} {gamma.dtype}, expected float32 [d] or [groups, d]")
        if group is None and gamma.numel() != d:
            raise ValueError("rms_norm: several scales need each row's group")
    if group is not None:
        if gamma is None or group.dtype != torch.int32 or group.shape != (x.shape[0],):
            raise ValueError("rms_norm: group is int32 [rows] and goes with gamma")
        group = group.contiguous()
    _int32("rms_norm", x, gamma)
    _same_device(x, gamma, group)
    return _RmsNorm.apply(_aligned(x), None if gamma is None else _aligned(gamma), group, float(eps), dtype,
                          _wants_grad(x, gamma))


class _Ffn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate_up, w_down, grad):
        rows, d = x.shape
        f = w_down.shape[1]
        code = _DTYPE[x.dtype]
        ws, n = _workspace(tlf.load().tlf_ffn_ws_bytes, code, rows, d, f, device=x.device)
        # what the backward pass keeps, then a (a multiple of 16 bytes), in one buffer
        size = tlf.ffn_kept_bytes(code, rows, f) if grad else 0
        kept = torch.empty(size + rows * f * x.element_size(), dtype=torch.uint8, device=x.device)
        y = torch.empty((rows, d), dtype=x.dtype, device=x.device)
        at = kept.data_ptr()
        _run(tlf.load().tlf_ffn, x.device, x, w_gate_up, w_down, code, rows, d, f, at if grad else None, at + size, y,
             ws, n)
        if grad:
            ctx.save_for_backward(x, w_gate_up, w_down, kept)
        return y

    @staticmethod
    @_first_order
    def backward(ctx, saved, dy):
        x, w_gate_up, w_down, kept = saved
        rows, d = x.shape
        f = w_down.shape[1]
        dy = _aligned(dy)
        outs = [torch.empty_like(t) if need else None
                for t, need in zip((x, w_gate_up, w_down), ctx.needs_input_grad)]
        lib = tlf.load()
        code = _DTYPE[x.dtype]
        ws, n = _workspace(lib.tlf_ffn_grad_ws_bytes, code, rows, d, f, device=x.device)
        at = kept.data_ptr()
        _run(lib.tlf_ffn_grad, x.device, dy, x, w_gate_up, w_down, at, at + tlf.ffn_kept_bytes(code, rows, f), code, rows,
             d, f, *outs, ws, n)
        return (*outs, None)


def ffn(x: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor) -> torch.Tensor:
    """The block's gated FFN, W_down (silu(W_gate x) * (W_up x)) of the rows of x ([rows, d]), with gradients.

    w_gate_up is [2f, d] (rows gate | up), w_down [d, f]; all three float32 or all bfloat16, d and f multiples of 64 up
    to 16384.  Sums are float32.  Of bfloat16 tensors the hidden activation and its gradient, operands of the next
    products, are rounded to bfloat16, and what the backward pass takes of the activation to 10 significant bits with
    float32's range; of float32 tensors nothing is rounded on the way."""
    if x.dim() != 2 or x.dtype not in _DTYPE or not x.is_cuda:
        raise ValueError("ffn: expected a float32 or bfloat16 [rows, d] CUDA tensor")
    d, f = x.shape[1], w_down.shape[-1]
    if w_gate_up.shape != (2 * f, d) or w_down.shape != (d, f):
        raise ValueError(f"ffn: x {tuple(x.shape)}, w_gate_up {tuple(w_gate_up.shape)}, w_down {tuple(w_down.shape)}; "
                         "expected [rows, d], [2f, d], [d, f]")
    if w_gate_up.dtype != x.dtype or w_down.dtype != x.dtype:
        raise ValueError("ffn: x and the weights are of one dtype")
    _int32("ffn", x, w_gate_up)
    _same_device(x, w_gate_up, w_down)
    return _Ffn.apply(_aligned(x), _aligned(w_gate_up), _aligned(w_down), _wants_grad(x, w_gate_up, w_down))


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, alpha, gamma, group, eps, post, grad):
        rows, d = x.shape
        groups = next((t.numel() // d for t in (alpha, gamma) if t is not None), 0)
        h, z = torch.empty_like(x), torch.empty_like(y)
        stats = torch.empty((2, rows), dtype=torch.float32, device=x.device) if grad else None
        rstd, ystd = (stats[0], stats[1] if post else None) if grad else (None, None)
        _run(tlf.load().tlf_residual_norm, x.device, x, y, _DTYPE[y.dtype], alpha, gamma, group, groups, rows, d, post, eps,
             h, z, rstd, ystd)
        ctx.set_materialize_grads(False)
        if grad:
            ctx.post, ctx.groups = post, groups
            ctx.save_for_backward(h, y, alpha, gamma, group, stats)
        return h, z

    @staticmethod
    @_first_order
    def backward(ctx, saved, dh, dz):
        h, y, alpha, gamma, group, stats = saved
        rows, d = h.shape
        if dh is None and dz is None:
            return (None,) * 8
        dh, dz = (None if t is None else _aligned(t) for t in (dh, dz))
        dx, dy = torch.empty_like(h), torch.empty_like(y)
        sums = any(ctx.needs_input_grad[2:4])
        dalpha, dgamma = (torch.empty_like(t) if sums and t is not None else None for t in (alpha, gamma))
        lib = tlf.load()
        ws, n = None, 0
        if sums:
            ws, n = _workspace(lib.tlf_residual_norm_grad_ws_bytes, ctx.groups, rows, d, device=h.device)
        _run(lib.tlf_residual_norm_grad, h.device, dh, dz, h, y, _DTYPE[y.dtype], alpha, gamma, group, ctx.groups, stats[0],
             stats[1] if ctx.post else None, rows, d, ctx.post, dx, dy, dalpha, dgamma, ws, n)
        return dx, dy, dalpha, dgamma, None, None, None, None


def residual_norm(x: torch.Tensor, y: torch.Tensor, alpha: torch.Tensor = None, gamma: torch.Tensor = None,
                  group: torch.Tensor = None, eps: float = 1e-5, post_norm: bool = False):
    """(h, z): the residual rows h = x + (1 + alpha) y, and their RMSNorm z times 1 + gamma, the next block's operand, in
    one pass, with gradients to x, y, alpha and gamma.

    x and h are float32 [rows, d], y and z float32 or bfloat16.  alpha and gamma are None, one [d] or [1, d] scale, or
    [groups, d] scales of which row r takes number group[r] (int32 [rows]; a row whose number is none of them takes none):
    the AdaLN gate and modulation of each token's depth.  With post_norm y is divided by its own root mean square first: a
    block with norms before and after.  Widths, groups, rows and sums as in rms_norm."""
    if x.dim() != 2 or x.dtype != torch.float32 or not x.is_cuda:
        raise ValueError("residual_norm: expected float32 [rows, d] CUDA residual rows")
    if y.shape != x.shape or y.dtype not in _DTYPE:
        raise ValueError(f"residual_norm: y {tuple(y.shape)} {y.dtype}, expected float32 or bfloat16 {tuple(x.shape)}")
    d, groups = x.shape[1], None
    for name, t in (("alpha", alpha), ("gamma", gamma)):
        if t is None:
            continue
        if t.dtype != torch.float32 or t.dim() not in (1, 2) or t.shape[-1] != d or t.numel() == 0:
            raise ValueError(f"residual_norm: {name} {tuple(t.shape)} {t.dtype}, expected float32 [d] or [groups, d]")
        if groups not in (None, t.numel() // d):
            raise ValueError("residual_norm: alpha and gamma are of the same groups")
        groups = t.numel() // d
        if group is None and groups != 1:
            raise ValueError("residual_norm: several scales need each row's group")
    if group is not None:
        if groups is None or group.dtype != torch.int32 or group.shape != (x.shape[0],):
            raise ValueError("residual_norm: group is int32 [rows] and goes with alpha or gamma")
        group = group.contiguous()
    _int32("residual_norm", x, alpha, gamma)
    _same_device(x, y, alpha, gamma, group)
    alpha, gamma = (None if t is None else _aligned(t) for t in (alpha, gamma))
    return _ResidualNorm.apply(_aligned(x), _aligned(y), alpha, gamma, group, float(eps), bool(post_norm),
                               _wants_grad(x, y, alpha, gamma))


# ---------------------------------------------------------------------------
# The block's attention: causal, over ragged rows, with a sliding window and sinks
# ---------------------------------------------------------------------------

def _rows_of_heads(t: torch.Tensor, heads: int, width: int) -> torch.Tensor:
    """`t` ([rows, heads, width], or [rows, heads * width]) as it lies if a row's elements are contiguous and its rows
    are 16-byte aligned, else copied."""
    want = (width, 1) if t.dim() == 3 else (1,)
    lies = all(n == 1 or s == w for n, s, w in zip(t.shape[1:], t.stride()[1:], want))
    each = t.element_size()
    if lies and t.data_ptr() % 16 == 0 and (t.shape[0] <= 1 or heads * width <= t.stride(0) <= tlf.ATTN_MAX_STRIDE and
                                            t.stride(0) * each % 16 == 0):
        return t
    return t.clone(memory_format=torch.contiguous_format)


def _row_stride(t: torch.Tensor, wide: int) -> int:
    return t.stride(0) if t.shape[0] > 1 else -(-wide // 8) * 8


class _Attention(torch.autograd.Function):
    """q, k and v as they lie in one tensor of rows q | k | v (self_attention), or as three."""
    @staticmethod
    def forward(ctx, x, k, v, offsets, k_offsets, k_lengths, heads, kv_heads, width, window, sinks, scale, grad):
        packed = k is None
        qw, kw = heads * width, kv_heads * width
        q = _rows_of_heads(x, heads + 2 * kv_heads if packed else heads, width)
        if packed:
            k, v = _key_rows(q, qw, kw)
            strides, rows_k = (_row_stride(q, qw + 2 * kw),) * 3, q.shape[0]
        else:
            k, v = _rows_of_heads(k, kv_heads, width), _rows_of_heads(v, kv_heads, width)
            strides, rows_k = (_row_stride(q, qw), _row_stride(k, kw), _row_stride(v, kw)), k.shape[0]
        o = torch.empty((q.shape[0], qw) if packed else (q.shape[0], heads, width), dtype=q.dtype, device=q.device)
        ctx.numbers = (_DTYPE[q.dtype], offsets.numel() - 1, heads, kv_heads, width, q.shape[0], rows_k, window, sinks, scale,
                       *strides, qw)
        shape = _attn_shape(ctx.numbers, offsets, k_offsets, k_lengths)
        lse = torch.empty((heads, q.shape[0]), dtype=torch.float32, device=q.device) if grad else None
        low = torch.empty_like(o) if grad and o.dtype == torch.bfloat16 else None  # what o's rounding takes
        ws, n = _workspace(tlf.load().tlf_attn_ws_bytes, shape, device=q.device)
        _run(tlf.load().tlf_attn, q.device, shape, q, k, v, o, lse, low, ws, n)
        if grad:
            ctx.packed = packed
            ctx.save_for_backward(q, None if packed else k, None if packed else v, offsets, k_offsets, k_lengths, o, lse, low)
        return o

    @staticmethod
    @_first_order
    def backward(ctx, saved, do):
        q, k, v, offsets, k_offsets, k_lengths, o, lse, low = saved
        _, _, heads, kv_heads, width = ctx.numbers[:5]
        qw, kw = heads * width, kv_heads * width
        do = _aligned(do)
        if ctx.packed:
            k, v = _key_rows(q, qw, kw)
            dq = torch.empty((q.shape[0], qw + 2 * kw), dtype=q.dtype, device=q.device)
            (dk, dv), strides = _key_rows(dq, qw, kw), (qw + 2 * kw,) * 3
        else:
            dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
            strides = (qw, kw, kw)
        shape = _attn_shape(ctx.numbers, offsets, k_offsets, k_lengths)
        ws, n = _workspace(tlf.load().tlf_attn_grad_ws_bytes, shape, device=q.device)
        _run(tlf.load().tlf_attn_grad, q.device, shape, do, q, k, v, o, lse, low, dq, strides[0], dk, strides[1], dv,
             strides[2], ws, n)
        grads = (dq, None, None) if ctx.packed else (dq, dk, dv)
        return (*grads, *(None,) * 10)


def _key_rows(rows: torch.Tensor, qw: int, kw: int):
    """Where k and v begin in rows q | k | v: addresses, which cost the host less than tensors of their own."""
    at, each = rows.data_ptr(), rows.element_size()
    return at + qw * each, at + (qw + kw) * each


def _attn_shape(numbers, offsets, k_offsets, k_lengths) -> tlf.AttnShape:
    return tlf.AttnShape(*numbers, offsets.data_ptr(), k_offsets.data_ptr(), None if k_lengths is None else k_lengths.data_ptr())


def _attend(name, q, k, v, offsets, k_offsets, k_lengths, heads, kv_heads, width, window, sinks, scale):
    if q.dtype not in _DTYPE or not q.is_cuda:
        raise ValueError(f"{name}: float32 or bfloat16 CUDA tensors expected")
    if heads < 1 or kv_heads < 1 or heads % kv_heads:
        raise ValueError(f"{name}: {heads} heads are no multiple of {kv_heads} key heads")
    k_offsets = offsets if k_offsets is None else k_offsets
    for t in (offsets, k_offsets, k_lengths):
        if t is not None and (t.dtype != torch.int32 or t.dim() != 1):
            raise ValueError(f"{name}: offsets and lengths are int32 vectors")
    if offsets.numel() < 1 or k_offsets.numel() != offsets.numel() or \
            (k_lengths is not None and k_lengths.numel() != offsets.numel() - 1):
        raise ValueError(f"{name}: one offset more than sequences, one length each")
    if window is not None and window < 1 or sinks < 0:
        raise ValueError(f"{name}: window {window}, sinks {sinks}")
    _int32(name, q, k, v, offsets)
    _same_device(q, k, v, offsets, k_offsets, k_lengths)
    window, sinks = (min(n, (1 << 31) - 1) for n in (window or 0, sinks))  # 32 bits each, as they are passed
    at = (offsets.contiguous(), k_offsets.contiguous(), None if k_lengths is None else k_lengths.contiguous())
    return _Attention.apply(q, k, v, *at, heads, kv_heads, width, window, sinks,
                            width ** -0.5 if scale is None else float(scale), _wants_grad(q, k, v))


def self_attention(qkv: torch.Tensor, offsets: torch.Tensor, heads: int, kv_heads: int = None, window: int = None,
                   sinks: int = 0, scale: float = None) -> torch.Tensor:
    """Causal attention within each sequence of rows q | k | v (qkv [rows, (heads + 2 kv_heads) * width], as the block's
    QKV projection gives them), with the gradient to qkv, one tensor.  Returns [rows, heads * width].

    offsets: int32, ascending, where each sequence's rows begin, and their end (LoopPlan.offsets).  With a `window` a row
    sees the last `window` rows of its sequence, itself included, and the first `sinks` ones; without it every earlier
    row.  heads is a multiple of kv_heads (heads by default): consecutive heads share a key head.  Width 64 or 128 (16 too
    in float32), sinks 64 at most, scale 1 / sqrt(width) by default.  Rows of no sequence, ahead of the first or behind
    the last, give zeros.  What a row does not see takes no part, whatever its values.  Scores, softmax and sums are
    float32; of bfloat16 tensors the weights, and in the backward pass the gradients of the scores, are rounded to
    bfloat16 as operands.

    Rows whose result is not finite, whose scores rise by more than some 80 above those of the first keys that they see, or
    whose scores are all below -78, are computed again one by one, which takes long where there are many of them."""
    kv_heads = heads if kv_heads is None else kv_heads
    if qkv.dim() != 2 or heads < 1 or kv_heads < 1 or qkv.shape[1] % (heads + 2 * kv_heads):
        raise ValueError(f"self_attention: qkv {tuple(qkv.shape)}, expected [rows, ({heads} + 2 x {kv_heads}) * width]")
    width = qkv.shape[1] // (heads + 2 * kv_heads)
    return _attend("self_attention", qkv, None, None, offsets, None, None, heads, kv_heads, width, window, sinks, scale)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, k_offsets: torch.Tensor = None,
              k_lengths: torch.Tensor = None, window: int = None, sinks: int = 0, scale: float = None) -> torch.Tensor:
    """Causal attention of each sequence's rows of q ([rows, heads, width]) to its rows of k and v ([k_rows, kv_heads,
    width]), with gradients to all three.  As self_attention; a sequence's last query stands at its last key.

    offsets, k_offsets: int32, ascending, where each sequence's rows of q, and of k and v, begin, and their ends
    (k_offsets: as offsets).  k_lengths: int32, how many rows each sequence holds of those up to the next one's begin (all by default):
    the new tokens' rows against a cache that has room for more.  A row that sees nothing gives zeros.  Rows of heads
    may lie in wider ones (a stride that is a multiple of 16 bytes); else they are copied."""
    if q.dim() != 3 or k.dim() != 3 or k.shape != v.shape or k.shape[2] != q.shape[2]:
        raise ValueError(f"attention: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}; expected [rows, heads, "
                         "width], twice [k_rows, kv_heads, width]")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("attention: q, k and v are of one dtype")
    if k_offsets is None and k.shape[0] != q.shape[0]:
        raise ValueError("attention: k and v of other rows than q need k_offsets")
    return _attend("attention", q, k, v, offsets, k_offsets, k_lengths, q.shape[1], k.shape[1], q.shape[2], window, sinks,
                   scale)


def _moment(state, like, dtype8, name):
    """(moment tensor, scales or None) of one parameter, checked."""
    t, s = state if isinstance(state, (tuple, list)) else (state, None)
    if t.numel() != like.numel() or not t.is_contiguous() or t.dtype != (torch.float32 if s is None else dtype8):
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype}, expected a contiguous float32 tensor or a pair of "
                         f"{dtype8} codes and float32 scales, of the parameter's size")
    if s is not None and (s.dtype != torch.float32 or not s.is_contiguous() or
                          s.numel() != -(-t.numel() // tlf.ADAMW_BLOCK)):
        raise ValueError(f"{name}: one contiguous float32 scale per {tlf.ADAMW_BLOCK} elements expected")
    return t, s


def _given_twice(table) -> bool:
    """Whether one address is updated twice by the tensors of an adamw_ call."""
    at = [a for t in table if t.n for a in (t.d_param, t.d_copy, t.d_m, t.d_v, t.d_m_scale, t.d_v_scale) if a]
    return len(set(at)) < len(at)


def _grad_table(name, grads):
    table = (tlf.Grad * len(grads))()
    for k, g in enumerate(grads):
        if g.dtype not in _DTYPE or not g.is_cuda or not g.is_contiguous():
            raise ValueError(f"{name}: gradients are contiguous float32 or bfloat16 CUDA tensors")
        if g.device != grads[0].device:
            raise ValueError(f"{name}: tensors on one device expected")
        table[k] = tlf.Grad(g.data_ptr(), g.numel(), _DTYPE[g.dtype], 0)
    return table


def _grad_norm(name, grads, table, max_norm):
    if max_norm is not None and not max_norm > 0:
        raise ValueError(f"{name}: max_norm {max_norm}")
    dev = grads[0].device
    ws, n = _workspace(tlf.load().tlf_grad_norm_ws_bytes, table, len(grads), device=dev)
    out = torch.empty(2, dtype=torch.float32, device=dev)
    _run(tlf.load().tlf_grad_norm, dev, table, len(grads), float("inf") if max_norm is None else max_norm, out,
         out.data_ptr() + 4, ws, n)
    return out[0], out[1]


def grad_norm(grads, max_norm: float = None):
    """(norm, scale) of a list of gradients (contiguous float32 or bfloat16 CUDA tensors), both float32 on the device: the
    norm of all their elements, summed in float64, and 1, or max_norm / norm where the norm is above max_norm (> 0).

    The host does not wait.  adamw_ takes the scale as it is: clipping then costs no pass over the gradients.  Gradients
    that are not finite give a scale of 0 or NaN, without a max_norm too."""
    grads = list(grads)
    if not grads:
        raise ValueError("grad_norm: no gradients")
    return _grad_norm("grad_norm", grads, _grad_table("grad_norm", grads), max_norm)


@torch.no_grad()
def clip_grad_norm_(grads, max_norm: float) -> torch.Tensor:
    """Multiplies the gradients by grad_norm's scale in place, rounded to their types, and returns the norm that they had.
    Gradients within the limit are not written.  They overlap nowhere."""
    grads = list(grads)
    if not grads:
        raise ValueError("clip_grad_norm_: no gradients")
    if max_norm is None:
        raise ValueError("clip_grad_norm_: max_norm None")
    table = _grad_table("clip_grad_norm_", grads)
    norm, scale = _grad_norm("clip_grad_norm_", grads, table, max_norm)
    _run(tlf.load().tlf_grad_clip, norm.device, table, len(grads), scale)
    torch.autograd.graph.increment_version(grads)
    return norm


def adamw_(params, grads, exp_avgs, exp_avg_sqs, step, lr: float, betas=(0.9, 0.95), eps: float = 1e-8,
           weight_decay=0.0, copies=None, grad_scale: torch.Tensor = None) -> None:
    """One AdamW step over many tensors, in place (tlf_adamw; few launches for all of them).

    params       contiguous float32 CUDA tensors, updated
    grads        their gradients, contiguous float32 or bfloat16
    exp_avgs     first moments, updated: a float32 tensor, or 8 bits as (torch.float8_e4m3fn codes, float32 scales)
    exp_avg_sqs  second moments, updated: a float32 tensor, or (torch.float8_e5m2 codes, float32 scales)
    step         the step's number from 1, or one number for each tensor; a value, as the rates are, so a step that is
                 captured into a graph is refused: its replays would repeat the corrections of one step
    weight_decay one value or one for each tensor
    copies       bfloat16 tensors that receive the updated parameters rounded, or None
    grad_scale   a float32 CUDA value that the gradients count times (grad_norm's scale), or None

    What is updated overlaps nothing else of the call; gradients may overlap each other.  eps is at least the smallest
    normal float32.
    """
    n = len(params)
    steps = [step] * n if isinstance(step, int) else list(step)
    decays = [weight_decay] * n if isinstance(weight_decay, (int, float)) else list(weight_decay)
    copies = [None] * n if copies is None else list(copies)
    if not n == len(grads) == len(exp_avgs) == len(exp_avg_sqs) == len(steps) == len(decays) == len(copies):
        raise ValueError("adamw_: one gradient, pair of moments, step, decay and copy for each parameter")
    if n == 0:
        return
    table = (tlf.AdamwTensor * n)()
    dev = params[0].device
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or grad_scale.device != dev):
        raise ValueError("adamw_: grad_scale is one float32 value on the parameters' device")
    for k, (p, g, c) in enumerate(zip(params, grads, copies)):
        if p.dtype != torch.float32 or not p.is_cuda or not p.is_contiguous():
            raise ValueError("adamw_: parameters are contiguous float32 CUDA tensors")
        if g.dtype not in _DTYPE or g.shape != p.shape or not g.is_contiguous():
            raise ValueError(f"adamw_: gradient {tuple(g.shape)} {g.dtype} of parameter {tuple(p.shape)}: contiguous "
                             "float32 or bfloat16 of its shape expected")
        if c is not None and (c.dtype != torch.bfloat16 or c.shape != p.shape or not c.is_contiguous()):
            raise ValueError("adamw_: copies are contiguous bfloat16 tensors of the parameters' shapes")
        m, ms = _moment(exp_avgs[k], p, torch.float8_e4m3fn, "exp_avg")
        v, vs = _moment(exp_avg_sqs[k], p, torch.float8_e5m2, "exp_avg_sq")
        if (ms is None) != (vs is None):
            raise ValueError("adamw_: both moments in 8 bits or both in float32")
        for t in (p, g, c, m, v, ms, vs):
            if t is not None and t.device != dev:
                raise ValueError("adamw_: tensors on one device expected")
        table[k] = tlf.AdamwTensor(p.data_ptr(), c.data_ptr() if c is not None else None, g.data_ptr(), m.data_ptr(),
                                   v.data_ptr(), ms.data_ptr() if ms is not None else None,
                                   vs.data_ptr() if vs is not None else None, p.numel(), steps[k], decays[k],
                                   _DTYPE[g.dtype], 32 if ms is None else 8)
    with torch.cuda.device(dev):
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("adamw_: the step number and rates are values and cannot be captured into a graph")
    try:
        if grad_scale is None:
            _run(tlf.load().tlf_adamw, dev, table, n, lr, betas[0], betas[1], eps)
        else:
            _run(tlf.load().tlf_adamw_scaled, dev, table, n, lr, betas[0], betas[1], eps, grad_scale)
    except tlf.TlfError as e:
        if e.status == tlf.E_INVALID_ARG and _given_twice(table):
            raise ValueError("adamw_: a parameter, copy, moment or scale appears twice") from None
        raise
    # a graph that saved a parameter or copy for its backward pass has to notice the update
    torch.autograd.graph.increment_version([*params, *(c for c in copies if c is not None)])


def _writes(t: torch.Tensor):
    """How often t was written, as autograd counts it (inference tensors are not counted)."""
    return None if t.is_inference() else t._version


class AdamW:
    """AdamW over leaf tensors, with moments of 32 or 8 bits.

    params: contiguous float32 or bfloat16 CUDA leaves.  A bfloat16 one is trained through a float32 master that the
    optimizer holds (masters[k]); the leaf receives it rounded.  Elements that are written into such a leaf afterwards
    go into the master at the next step or state_dict, but for writes through its .data, which autograd does not count
    and the step overwrites.  step() updates every parameter that has a gradient, each with its own count of steps.
    weight_decay is one value or one for each parameter.  lr may be set between steps.  state_dict and load_state_dict
    carry the masters, moments and counts; load_state_dict sets the bfloat16 leaves to the masters rounded and leaves
    float32 ones as they are."""

    def __init__(self, params, lr: float, betas=(0.9, 0.95), eps: float = 1e-8, weight_decay=0.0,
                 state_bits: int = 32):
        self.params = list(params)
        self.lr, self.betas, self.eps = lr, tuple(betas), eps
        n = len(self.params)
        self.weight_decay = [weight_decay] * n if isinstance(weight_decay, (int, float)) else list(weight_decay)
        if state_bits not in (8, 32) or len(self.weight_decay) != n:
            raise ValueError("AdamW: state_bits 8 or 32, weight_decay one value or one for each parameter")
        if len({id(p) for p in self.params}) != n:
            raise ValueError("AdamW: a parameter appears twice")
        for p in self.params:
            if p.dtype not in _DTYPE or not p.is_cuda or not p.is_contiguous() or not p.is_leaf:
                raise ValueError("AdamW: contiguous float32 or bfloat16 CUDA leaves expected")
        self.state_bits = state_bits
        self.masters = [p.detach().float() if p.dtype == torch.bfloat16 else None for p in self.params]
        self.exp_avgs = [self._zeros(p, torch.float8_e4m3fn) for p in self.params]
        self.exp_avg_sqs = [self._zeros(p, torch.float8_e5m2) for p in self.params]
        self.steps = [0] * n
        self._written = [_writes(p) for p in self.params]  # as far as the masters know the leaves

    def _zeros(self, p, dtype8):
        if self.state_bits == 32:
            return torch.zeros(p.shape, dtype=torch.float32, device=p.device)
        return (torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(dtype8),
                torch.zeros(-(-p.numel() // tlf.ADAMW_BLOCK), dtype=torch.float32, device=p.device))

    def _take_written(self, have) -> None:
        for k in have:
            p, m = self.params[k].detach(), self.masters[k]
            if m is not None and _writes(p) != self._written[k]:
                m.copy_(torch.where(m.to(p.dtype) == p, m, p.float()))  # the same again if no step follows

    @torch.no_grad()
    def step(self, max_norm: float = None):
        """One step; with max_norm the gradients, all on one device, count times grad_norm's scale (they are left as they
        are), and their norm is returned: a float32 value on the device, None without gradients."""
        have = [k for k, p in enumerate(self.params) if p.grad is not None]
        grads = {k: self.params[k].grad.contiguous() for k in have}
        norm = scale = None
        if max_norm is not None and have:
            norm, scale = grad_norm(grads.values(), max_norm)
        self._take_written(have)
        by = {}
        for k in have:
            by.setdefault(self.params[k].device, []).append(k)
        for at in by.values():
            pick = lambda v: [v[k] for k in at]  # noqa: E731
            real = [self.params[k].detach() if self.masters[k] is None else self.masters[k] for k in at]
            copies = [None if self.masters[k] is None else self.params[k].detach() for k in at]
            adamw_(real, pick(grads), pick(self.exp_avgs), pick(self.exp_avg_sqs), [self.steps[k] + 1 for k in at], self.lr,
                   self.betas, self.eps, pick(self.weight_decay), copies, **({} if scale is None else {"grad_scale": scale}))
            for k in at:
                self.steps[k] += 1
                self._written[k] = _writes(self.params[k])
        return norm

    def zero_grad(self) -> None:
        for p in self.params:
            p.grad = None

    @torch.no_grad()
    def state_dict(self) -> dict:
        self._take_written(range(len(self.params)))
        return {"steps": list(self.steps), "masters": list(self.masters), "exp_avgs": list(self.exp_avgs),
                "exp_avg_sqs": list(self.exp_avg_sqs), "state_bits": self.state_bits}

    @torch.no_grad()
    def load_state_dict(self, state: dict) -> None:
        if state["state_bits"] != self.state_bits or len(state["steps"]) != len(self.params):
            raise ValueError("AdamW: the state is of other parameters or another state_bits")
        parts = lambda s: () if s is None else tuple(s) if isinstance(s, (tuple, list)) else (s,)  # noqa: E731
        steps, pairs = [int(k) for k in state["steps"]], []
        for key in ("masters", "exp_avgs", "exp_avg_sqs"):
            mine, given = [[parts(s) for s in v] for v in (getattr(self, key), state[key])]
            if [[(t.shape, t.dtype) for t in s] for s in mine] != [[(t.shape, t.dtype) for t in s] for s in given]:
                raise ValueError(f"AdamW: {key} do not fit the parameters")
            pairs += [(t, g) for a, b in zip(mine, given) for t, g in zip(a, b)]
        for t, g in pairs:  # all of it fits
            t.copy_(g)
        for k, (p, m) in enumerate(zip(self.params, self.masters)):
            if m is not None:
                p.copy_(m)
                self._written[k] = _writes(p)
        self.steps = steps
