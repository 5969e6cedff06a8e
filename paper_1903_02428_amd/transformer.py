"""The parts of a graph transformer's block (ctypes marshalling only): attention
among the nodes of each graph with a learned bias by relative position, the norms around
a block with its gate and residual scale, and activations kept in 8 bits."""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
from dataclasses import dataclass

import torch

from .binding import (DTYPE, _aligned16, _Attention, _BlockNorm, _check, _need_cuda, _ptr, _size, _stream, _workspace,
                      dense_transform, library)

NORM = {"layer": 0, "rms": 1}


def _on(device):
    """Launches go to the tensors' device, whichever is current."""
    return contextlib.nullcontext() if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} must be on {device}, got {t.device}")


def _written(*tensors):
    """Kernels write through addresses, which autograd does not see: a caller's tensor that was written
    counts as modified in place, so that a backward that kept it says so."""
    for t in tensors:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


def _room(workspace, nbytes: int, device):
    """The caller's workspace where it is large enough, else one made here."""
    if workspace is not None:
        _need_cuda("workspace", workspace)  # adjacent bytes: as many as its elements have
        if not _aligned16(workspace):
            raise ValueError("workspace must be 16-byte aligned")
        if workspace.numel() * workspace.element_size() >= nbytes:
            return workspace
    return _workspace(nbytes, device)


class _Gradient(torch.autograd.Function):
    """A gradient that was asked for with create_graph, tied to what it depends on: differentiating
    it raises."""

    @staticmethod
    def forward(ctx, gradient, *depends):
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("this operator can be differentiated once: its gradients have none themselves")


def _once(backward):
    """For a backward that calls kernels, which autograd does not see: without this its results would
    count as constants in a second differentiation, and terms be left out silently."""
    @functools.wraps(backward)
    def wrapper(ctx, *grads):
        if not torch.is_grad_enabled():
            return backward(ctx, *grads)
        with torch.no_grad():
            out = backward(ctx, *grads)
        depends = [t for t in (*grads, *ctx.saved_tensors) if t is not None and t.requires_grad]
        return tuple(None if t is None else _Gradient.apply(t, *depends) for t in out)
    return wrapper


def relative_buckets(num_buckets: int = 32, max_distance: int = 128, bidirectional: bool = True,
                     device="cuda") -> torch.Tensor:
    """Bucket of every offset -max_distance .. max_distance (key position minus
    query position), int32 [2 * max_distance + 1], as global_attention reads it:
    half of the buckets hold one small distance each, the rest divide the
    distances up to max_distance by their logarithm, and what lies beyond shares the last.
    bidirectional: later keys have half of the buckets for themselves; otherwise they
    take bucket 0 (for causal attention)."""
    n = num_buckets // 2 if bidirectional else num_buckets
    if n < 1 or max_distance < 0 or (bidirectional and num_buckets % 2):
        raise ValueError("need at least one bucket for each direction and a distance of 0 or more")
    near = max(1, n // 2)
    if n > 1 and max_distance <= near:
        raise ValueError("max_distance must exceed the buckets of single distances")

    def bucket(d):
        a = abs(d)
        if a >= near:
            a = min(n - 1, near + int(math.log(a / near) / math.log(max_distance / near) * (n - near) + 1e-9)) if n > 1 else 0
        if not bidirectional:
            return 0 if d > 0 else a
        return a + n if d > 0 else a
    return torch.tensor([bucket(d) for d in range(-max_distance, max_distance + 1)], dtype=torch.int32, device=device)


def _heads(name, t, dtype=None, device=None):
    """A [rows, heads, D] tensor whose features are adjacent (rows and heads may be strided)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a HIP device, got {t.device}")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [rows, heads, features], got shape {tuple(t.shape)}")
    if t.dtype not in DTYPE or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be {dtype or 'float32 or bfloat16'}, got {t.dtype}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name}'s features must be adjacent in memory")
    return t


def _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, zero_rest, skip=0) -> _Attention:
    _heads("q", q)
    _heads("k", k, q.dtype)
    _heads("v", v, q.dtype)
    (Nq, H, D), (Nk, Hkv, Dk) = q.shape, k.shape
    if Dk != D or v.shape != k.shape:
        raise ValueError("k and v must both be [rows, key heads, D] with q's D")
    if Hkv == 0 or H % Hkv or H == 0 or D == 0:
        raise ValueError("q's heads must be a multiple of k's, and there must be features")
    k_ptr = ptr if k_ptr is None else k_ptr
    _need_cuda("ptr", ptr, torch.int64, 1)
    _need_cuda("k_ptr", k_ptr, torch.int64, 1)
    if ptr.shape[0] < 1 or ptr.shape != k_ptr.shape:
        raise ValueError("ptr and k_ptr must both be [graphs + 1]")
    if k_ptr is ptr and Nk != Nq:
        raise ValueError("k and q must have the same rows where they share ptr")
    if (table is None) != (buckets is None):
        raise ValueError("table and buckets come together")
    if table is not None:
        _need_cuda("table", table, q.dtype, 2)
        _need_cuda("buckets", buckets, torch.int32, 1)
        if table.shape[1] != H or table.shape[0] < 1:
            raise ValueError("table must be [buckets, heads]")
        if buckets.shape[0] % 2 == 0:
            raise ValueError("buckets must be [2 * reach + 1]")
    _same_device(q.device, k=k, v=v, ptr=ptr, k_ptr=k_ptr, table=table, buckets=buckets)
    scale = D ** -0.5 if scale is None else float(scale)
    if not 1e-30 <= scale <= 1e30:
        raise ValueError("scale must lie between 1e-30 and 1e30")
    return _Attention(ptr.data_ptr(), k_ptr.data_ptr(), ptr.shape[0] - 1, Nq, Nk, H, Hkv, D, q.stride(0), q.stride(1),
                      k.stride(0), k.stride(1), v.stride(0), v.stride(1), DTYPE[q.dtype], scale, int(bool(causal)),
                      _ptr(table), _ptr(buckets), 0 if table is None else table.shape[0],
                      0 if table is None else buckets.shape[0] // 2, int(zero_rest), skip)


def _bytes(fn, c) -> int:
    out = ctypes.c_size_t(0)
    _check(fn(ctypes.byref(c), ctypes.byref(out)), fn.__name__)
    return out.value


def global_attention_workspace_bytes(q, k, v, ptr, k_ptr=None, table=None, buckets=None, causal=False, scale=None) -> int:
    c = _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, False)
    return _bytes(library().pyg_global_attention_workspace, c)


def global_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, ptr: torch.Tensor,
                     k_ptr: torch.Tensor | None = None, table: torch.Tensor | None = None,
                     buckets: torch.Tensor | None = None, causal: bool = False, scale: float | None = None,
                     out: torch.Tensor | None = None, stat: torch.Tensor | None = None,
                     rest: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of each graph's nodes to one another (pyg_global_attention):
    out[i, h] = sum_j softmax_j(scale <q[i, h], k[j, h']> + table[buckets[offset], h])
    v[j, h'], over the keys j of i's graph.

    q [Nq, H, D], k and v [Nk, Hkv, D] (float32 or bfloat16, D <= 128, Hkv divides H; rows and
    heads may be strided views); ptr int64 [graphs + 1], the rows of each graph's queries,
    and k_ptr those of its keys (default: the same); table [buckets, H] and buckets as
    relative_buckets() makes it; causal: keys later than the query are not seen, whatever
    they hold (the last query is aligned with the last key); scale defaults to D ** -0.5. `stat` (float32
    [Nq, H, 2]) receives what global_attention_backward needs, `rest` (bfloat16, out's shape)
    what rounding took from out. Rows that belong to no graph
    get zeros, but are left as they were in an `out` that the caller brings."""
    lib = library()
    c = _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, out is None)
    dev, given = q.device, out
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    else:
        _need_cuda("out", out, q.dtype, 3)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if stat is not None:
        _need_cuda("stat", stat, torch.float32, 3)
        if stat.shape != (*q.shape[:2], 2):
            raise ValueError("stat must be [rows, heads, 2]")
    _rest(rest, q)
    _same_device(dev, out=out, stat=stat, rest=rest, workspace=workspace)
    with _on(dev):
        nbytes = _bytes(lib.pyg_global_attention_workspace, c)
        workspace = _room(workspace, nbytes, dev) if nbytes else None
        _check(lib.pyg_global_attention(ctypes.byref(c), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(stat),
                                        _ptr(rest), _ptr(workspace), nbytes, _stream(dev)), "pyg_global_attention")
    _written(given, stat, rest)
    return out


def _rest(rest, q):
    if rest is not None:
        _need_cuda("rest", rest, torch.bfloat16, 3)
        if q.dtype != torch.bfloat16 or rest.shape != q.shape:
            raise ValueError("rest must have q's shape, and q be bfloat16")


def global_attention_backward(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              out: torch.Tensor, stat: torch.Tensor, ptr: torch.Tensor,
                              k_ptr: torch.Tensor | None = None, table: torch.Tensor | None = None,
                              buckets: torch.Tensor | None = None, causal: bool = False, scale: float | None = None,
                              need_grad_table: bool = True, rest: torch.Tensor | None = None,
                              workspace: torch.Tensor | None = None, need_grad_q: bool = True,
                              need_grad_kv: bool = True):
    """Gradients of global_attention: (grad_q, grad_k, grad_v, grad_table), None for those
    that are not needed, from its result `out`, the `stat` and, if it was asked for, the `rest` it filled."""
    lib = library()
    need_grad_table = need_grad_table and table is not None
    c = _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, True,
                   (not need_grad_q) + 2 * (not need_grad_kv) + 4 * (not need_grad_table))
    dev = q.device
    for name, t in (("grad_out", grad_out), ("out", out)):
        _need_cuda(name, t, q.dtype, 3)
        if t.shape != q.shape:
            raise ValueError(f"{name} must have q's shape")
    _need_cuda("stat", stat, torch.float32, 3)
    if stat.shape != (*q.shape[:2], 2):
        raise ValueError("stat must be [rows, heads, 2]")
    _rest(rest, q)
    _same_device(dev, grad_out=grad_out, out=out, stat=stat, rest=rest, workspace=workspace)
    gq, gk, gv = (torch.empty(t.shape, dtype=t.dtype, device=dev) if need else None
                  for t, need in ((q, need_grad_q), (k, need_grad_kv), (v, need_grad_kv)))
    gt = torch.empty_like(table) if need_grad_table else None
    with _on(dev):
        nbytes = _bytes(lib.pyg_global_attention_backward_workspace, c)
        workspace = _room(workspace, nbytes, dev)
        _check(lib.pyg_global_attention_backward(ctypes.byref(c), _ptr(grad_out), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                                 _ptr(stat), _ptr(rest), _ptr(gq), _ptr(gk), _ptr(gv), _ptr(gt), _ptr(workspace),
                                                 nbytes, _stream(dev)), "pyg_global_attention_backward")
    return gq, gk, gv, gt


def _adjacent(t):
    """Features adjacent and no row or head standing for several, by a copy where it takes one."""
    fits = t.dim() != 3 or (t.shape[2] <= 1 or t.stride(2) == 1) and 0 not in t.stride()
    return t if fits else t.contiguous()


class GlobalAttention(torch.autograd.Function):
    """Differentiable global_attention. Use as GlobalAttention.apply(q, k, v, table_or_None,
    ptr, k_ptr_or_None, buckets_or_None, causal, scale); gradients for q, k, v and the table."""

    @staticmethod
    def forward(ctx, q, k, v, table, ptr, k_ptr=None, buckets=None, causal: bool = False, scale: float | None = None):
        qc, kc, vc = (_adjacent(t.detach()) for t in (q, k, v))
        tc = None if table is None else table.detach().contiguous()
        need = any(ctx.needs_input_grad[:4])
        stat = torch.empty((*q.shape[:2], 2), dtype=torch.float32, device=q.device) if need else None
        rest = torch.empty(q.shape, dtype=q.dtype, device=q.device) if need and q.dtype == torch.bfloat16 else None
        out = global_attention(qc, kc, vc, ptr, k_ptr, tc, buckets, causal, scale, stat=stat, rest=rest)
        ctx.causal, ctx.scale = causal, scale
        ctx.save_for_backward(q, k, v, table, out, stat, rest, ptr, k_ptr, buckets)
        return out

    @staticmethod
    @_once
    def backward(ctx, grad_out):
        q, k, v, table, out, stat, rest, ptr, k_ptr, buckets = ctx.saved_tensors
        qc, kc, vc = (_adjacent(t.detach()) for t in (q, k, v))
        tc = None if table is None else table.detach().contiguous()
        need = ctx.needs_input_grad
        grads = global_attention_backward(grad_out.to(q.dtype).contiguous(), qc, kc, vc, out.contiguous(), stat, ptr, k_ptr,
                                          tc, buckets, ctx.causal, ctx.scale, need_grad_table=need[3], rest=rest,
                                          need_grad_q=need[0], need_grad_kv=need[1] or need[2])
        return tuple(g if need else None for g, need in zip(grads, ctx.needs_input_grad)) + (None,) * 5


# ------------------------------------------------------- activations in 8 bits


@dataclass
class Checkpoint:
    """A matrix [N, F] kept in 8 bits (activation_checkpoint): int8 codes, 32 features of
    a row sharing a power-of-two step."""
    codes: torch.Tensor  # int8 [N, 32 * blocks]
    steps: torch.Tensor  # uint8 [N, blocks]: exponent of the step + 127
    F: int
    dtype: torch.dtype   # what it was made from

    @property
    def N(self) -> int:
        return self.steps.shape[0]


def _new_checkpoint(N: int, F: int, dtype, device) -> Checkpoint:
    blocks = -(-F // 32)
    return Checkpoint(torch.empty((N, blocks * 32), dtype=torch.int8, device=device),
                      torch.empty((N, blocks), dtype=torch.uint8, device=device), F, dtype)


def _checked(kept: Checkpoint, device=None):
    _need_cuda("codes", kept.codes, torch.int8, 2)
    _need_cuda("steps", kept.steps, torch.uint8, 2)
    blocks = -(-kept.F // 32)
    if kept.F < 1 or kept.steps.shape[1] != blocks or tuple(kept.codes.shape) != (kept.N, blocks * 32):
        raise ValueError("codes must be [N, 32 * blocks] and steps [N, blocks] with blocks = ceil(F / 32)")
    if not _aligned16(kept.codes):
        raise ValueError("codes must be 16-byte aligned")
    _same_device(device or kept.codes.device, codes=kept.codes, steps=kept.steps)
    return kept


def activation_checkpoint(x: torch.Tensor, out: Checkpoint | None = None) -> Checkpoint:
    """x [N, F] (float32 or bfloat16) in 8 bits: every 32 features of a row share a step, the smallest
    power of two that leaves the largest of them below 127.5 steps; a code is the
    nearest multiple (ties to even). Blocks with an infinity or NaN come back as NaN."""
    _need_cuda("x", x, None, 2)
    if x.dtype not in DTYPE:
        raise ValueError("x must be float32 or bfloat16")
    N, F = x.shape
    if F < 1:
        raise ValueError("x must have features")
    given = out
    if out is None:
        out = _new_checkpoint(N, F, x.dtype, x.device)
    elif (out.N, out.F, out.dtype) != (N, F, x.dtype):
        raise ValueError("out is the checkpoint of another shape or type")
    _checked(out, x.device)
    with _on(x.device):
        _check(library().pyg_activation_checkpoint(_ptr(x), DTYPE[x.dtype], N, F, _ptr(out.codes), _ptr(out.steps),
                                                   _stream(x.device)), "pyg_activation_checkpoint")
    if given is not None:
        _written(given.codes, given.steps)
    return out


def checkpoint_restore(kept: Checkpoint, dtype: torch.dtype | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """The matrix that a checkpoint stands for, exactly (in float32 or bfloat16)."""
    _checked(kept)
    dtype = (kept.dtype if out is None else out.dtype) if dtype is None else dtype
    if dtype not in DTYPE:
        raise ValueError("dtype must be float32 or bfloat16")
    dev, given = kept.codes.device, out
    if out is None:
        out = torch.empty((kept.N, kept.F), dtype=dtype, device=dev)
    else:
        _need_cuda("out", out, dtype, 2)
        if tuple(out.shape) != (kept.N, kept.F):
            raise ValueError("out must be [N, F]")
        _same_device(dev, out=out)
    with _on(dev):
        _check(library().pyg_checkpoint_restore(_ptr(kept.codes), _ptr(kept.steps), kept.N, kept.F, _ptr(out),
                                                DTYPE[dtype], _stream(dev)), "pyg_checkpoint_restore")
    _written(given)
    return out


def dense_transform_backward(grad_out: torch.Tensor, theta: torch.Tensor, kept: Checkpoint | None, need_grad_x: bool = True,
                             need_grad_theta: bool = True, workspace: torch.Tensor | None = None):
    """Gradients of dense_transform(x, theta) from grad_out [N, Fo] and x kept in 8 bits:
    (grad_x = grad_out theta^T or None, grad_theta = x^T grad_out or None), in theta's type. Without
    need_grad_theta nothing of x is read, and kept may be None."""
    lib = library()
    _need_cuda("grad_out", grad_out, None, 2)
    if grad_out.dtype not in DTYPE:
        raise ValueError("grad_out must be float32 or bfloat16")
    _need_cuda("theta", theta, grad_out.dtype, 2)
    dev = grad_out.device
    if kept is not None:
        _checked(kept, dev)
    elif need_grad_theta:
        raise ValueError("the gradient of theta needs x's checkpoint")
    (N, Fo), Fi = grad_out.shape, theta.shape[0]
    if theta.shape[1] != Fo or (kept is not None and (kept.N, kept.F) != (N, Fi)):
        raise ValueError("grad_out must be [N, Fo], theta [Fi, Fo] and the checkpoint [N, Fi]")
    if Fo < 1 or Fi < 1:
        raise ValueError("theta must have rows and columns")
    _same_device(dev, theta=theta, workspace=workspace)
    gx = torch.empty((N, Fi), dtype=theta.dtype, device=dev) if need_grad_x else None
    gt = torch.empty_like(theta) if need_grad_theta else None
    with _on(dev):
        nbytes = _size(lib.pyg_dense_transform_backward_workspace, DTYPE[theta.dtype], N, Fi, Fo) if need_grad_theta else 0
        workspace = _room(workspace, nbytes, dev) if nbytes else None
        _check(lib.pyg_dense_transform_backward(_ptr(grad_out), DTYPE[theta.dtype], N, Fo, _ptr(theta), Fi,
                                                _ptr(kept.codes) if kept else None, _ptr(kept.steps) if kept else None,
                                                _ptr(gx), _ptr(gt), _ptr(workspace), nbytes,
                                                _stream(dev)), "pyg_dense_transform_backward")
    return gx, gt


class DenseTransform(torch.autograd.Function):
    """Differentiable dense_transform whose input is kept in 8 bits for the backward: the
    gradient of theta is that of the kept values. Use as DenseTransform.apply(x, theta,
    kept): `kept` is x's checkpoint where there is one (block_norm makes it with y), else it is made
    here. x, theta and the result have one type."""

    @staticmethod
    def forward(ctx, x, theta, kept: Checkpoint | None = None):
        xc, tc = x.detach().contiguous(), theta.detach().contiguous()
        ctx.F = None
        if ctx.needs_input_grad[1]:
            kept = activation_checkpoint(xc) if kept is None else kept
            if (kept.N, kept.F) != tuple(x.shape):
                raise ValueError("kept must be the checkpoint of x")
            ctx.F = kept.F
        ctx.shape = tuple(x.shape)
        _need_cuda("x", xc, None, 2)
        _same_device(x.device, theta=tc)
        with _on(x.device):
            out = dense_transform(xc, tc, x.dtype)
        ctx.save_for_backward(theta, *((kept.codes, kept.steps) if ctx.F else ()))
        return out

    @staticmethod
    @_once
    def backward(ctx, grad_out):
        theta, *held = ctx.saved_tensors
        g, t = grad_out.to(theta.dtype).contiguous(), theta.detach().contiguous()
        # where theta needs no gradient nothing was kept
        kept = Checkpoint(*held, ctx.F, theta.dtype) if ctx.F else None
        gx, gt = dense_transform_backward(g, t, kept, ctx.needs_input_grad[0], kept is not None)
        return gx, gt, None


# ------------------------------------------------------- norms around a block


def _norm_args(h, residual, gate, scale, post_weight, post_bias, weight, bias, norm, eps) -> _BlockNorm:
    _need_cuda("h", h, None, 2)
    if h.dtype not in DTYPE:
        raise ValueError("h must be float32 or bfloat16")
    if norm not in NORM:
        raise ValueError("norm must be 'layer' or 'rms'")
    if not eps >= 0:
        raise ValueError("eps must not be negative")
    N, F = h.shape
    if F < 1:
        raise ValueError("h must have features")
    if residual is not None:
        _need_cuda("residual", residual, h.dtype, 2)
        if residual.shape != h.shape:
            raise ValueError("residual must have h's shape")
    if gate is not None:
        _need_cuda("gate", gate, h.dtype, 2)
        if gate.shape[0] != N or gate.shape[1] not in (1, F):
            raise ValueError("gate must be [N, F] or [N, 1]")
    for name, t in (("scale", scale), ("post_weight", post_weight), ("post_bias", post_bias), ("weight", weight),
                    ("bias", bias)):
        if t is not None:
            _need_cuda(name, t, torch.float32, 1)
            if t.shape[0] != F:
                raise ValueError(f"{name} must be [F]")
    if (post_bias is not None and post_weight is None) or (bias is not None and weight is None):
        raise ValueError("a bias needs its weight")
    _same_device(h.device, residual=residual, gate=gate, scale=scale, post_weight=post_weight, post_bias=post_bias,
                 weight=weight, bias=bias)
    return _BlockNorm(DTYPE[h.dtype], NORM[norm], N, F, eps, _ptr(h), _ptr(residual), _ptr(gate),
                      int(gate is not None and gate.shape[1] == 1), _ptr(scale), _ptr(post_weight), _ptr(post_bias),
                      _ptr(weight), _ptr(bias))


def block_norm(h: torch.Tensor, residual: torch.Tensor | None = None, gate: torch.Tensor | None = None,
               scale: torch.Tensor | None = None, post_weight: torch.Tensor | None = None,
               post_bias: torch.Tensor | None = None, weight: torch.Tensor | None = None,
               bias: torch.Tensor | None = None, norm: str = "layer", eps: float = 1e-5, checkpoint: bool = False):
    """What lies between two blocks of a transformer, in one pass over the rows: with h the
    first block's result and `residual` its input,
        u = norm(h) * post_weight + post_bias           (h without post_weight)
        r = residual + scale * sigmoid(gate) * u
        y = norm(r) * weight + bias                     (None without weight)
    h, residual [N, F], gate [N, F] or [N, 1] in one type (float32 or bfloat16), scale, weights and
    biases float32 [F]; norm "layer" or "rms"; F <= 8192. Returns (r, y, kept): kept is y's
    8-bit checkpoint with `checkpoint`, else None. Where all that is asked is a norm (no
    residual, gate, scale or post_weight), r is h itself."""
    a = _norm_args(h, residual, gate, scale, post_weight, post_bias, weight, bias, norm, eps)
    if checkpoint and weight is None:
        raise ValueError("a checkpoint is made of y: weight is needed")
    plain = residual is None and gate is None and scale is None and post_weight is None
    r = h if plain else torch.empty_like(h)
    y = torch.empty_like(h) if weight is not None else None
    kept = _new_checkpoint(a.N, a.F, h.dtype, h.device) if checkpoint else None
    if plain and y is None:
        return r, None, None
    with _on(h.device):
        _check(library().pyg_block_norm(ctypes.byref(a), None if plain else _ptr(r), _ptr(y),
                                        _ptr(kept.codes) if kept else None, _ptr(kept.steps) if kept else None,
                                        _stream(h.device)), "pyg_block_norm")
    return r, y, kept


def block_norm_backward(grad_r: torch.Tensor | None, grad_y: torch.Tensor | None, h, residual=None, gate=None, scale=None,
                        post_weight=None, post_bias=None, weight=None, bias=None, norm: str = "layer", eps: float = 1e-5,
                        need: tuple | None = None, workspace: torch.Tensor | None = None):
    """Gradients of block_norm for its eight tensors, in their order (None where one is
    missing or not needed), from the gradients of r and y (None: zeros)."""
    lib = library()
    a = _norm_args(h, residual, gate, scale, post_weight, post_bias, weight, bias, norm, eps)
    for name, g in (("grad_r", grad_r), ("grad_y", grad_y)):
        if g is not None:
            _need_cuda(name, g, h.dtype, 2)
            if g.shape != h.shape:
                raise ValueError(f"{name} must have h's shape")
    if grad_r is None and grad_y is None:
        raise ValueError("need grad_r or grad_y")
    if grad_y is not None and weight is None:
        raise ValueError("there is no y without weight")
    _same_device(h.device, grad_r=grad_r, grad_y=grad_y, workspace=workspace)
    tensors = (h, residual, gate, scale, post_weight, post_bias, weight, bias)
    need = need or (True,) * 8
    grads = tuple(torch.empty_like(t) if t is not None and n else None for t, n in zip(tensors, need))
    with _on(h.device):
        nbytes = _bytes(lib.pyg_block_norm_backward_workspace, a)
        workspace = _room(workspace, nbytes, h.device)
        _check(lib.pyg_block_norm_backward(ctypes.byref(a), _ptr(grad_r), _ptr(grad_y), *[_ptr(g) for g in grads],
                                           _ptr(workspace), nbytes, _stream(h.device)),
               "pyg_block_norm_backward")
    return grads


class BlockNorm(torch.autograd.Function):
    """Differentiable block_norm. Use as BlockNorm.apply(h, residual, gate, scale, post_weight,
    post_bias, weight, bias, norm, eps, checkpoint), None for the parts that are left out;
    returns (r, y, kept). Nothing but the inputs is kept for the backward."""

    @staticmethod
    def forward(ctx, h, residual=None, gate=None, scale=None, post_weight=None, post_bias=None, weight=None, bias=None,
                norm: str = "layer", eps: float = 1e-5, checkpoint: bool = False):
        tensors = (h, residual, gate, scale, post_weight, post_bias, weight, bias)
        c = [None if t is None else t.detach().contiguous() for t in tensors]
        r, y, kept = block_norm(*c, norm=norm, eps=eps, checkpoint=checkpoint)
        if r is c[0]:
            r = h.view_as(h)  # passed through: autograd wants an output of its own
        ctx.norm, ctx.eps = norm, eps
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(*tensors)
        return r, y, kept

    @staticmethod
    @_once
    def backward(ctx, grad_r, grad_y, _):
        tensors = ctx.saved_tensors
        if grad_r is None and grad_y is None:
            return (None,) * 11
        c = [None if t is None else t.detach().contiguous() for t in tensors]
        gr, gy = (None if g is None else g.to(c[0].dtype).contiguous() for g in (grad_r, grad_y))
        need = (ctx.needs_input_grad + (False,) * 8)[:8]  # of the arguments that were given
        return block_norm_backward(gr, gy, *c, norm=ctx.norm, eps=ctx.eps, need=need) + (None,) * 3
