"""The parts of a graph transformer's block (ctypes marshalling only): attention
among the nodes of each graph with a learned bias by relative position."""
from __future__ import annotations

import contextlib
import ctypes
import math

import torch

from .binding import DTYPE, _Attention, _check, _need_cuda, _ptr, _stream, _workspace, library


def _on(device):
    """Launches go to the tensors' device, whichever is current."""
    return contextlib.nullcontext() if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} must be on {device}, got {t.device}")


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


def _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, zero_rest) -> _Attention:
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
    if not 0.0 < scale <= 1e30:
        raise ValueError("scale must be positive and finite")
    return _Attention(ptr.data_ptr(), k_ptr.data_ptr(), ptr.shape[0] - 1, Nq, Nk, H, Hkv, D, q.stride(0), q.stride(1),
                      k.stride(0), k.stride(1), v.stride(0), v.stride(1), DTYPE[q.dtype], scale, int(bool(causal)),
                      _ptr(table), _ptr(buckets), 0 if table is None else table.shape[0],
                      0 if table is None else buckets.shape[0] // 2, int(zero_rest))


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
                     workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of each graph's nodes to one another (pyg_global_attention):
    out[i, h] = sum_j softmax_j(scale <q[i, h], k[j, h']> + table[buckets[offset], h])
    v[j, h'], over the keys j of i's graph.

    q [Nq, H, D], k and v [Nk, Hkv, D] (float32 or bfloat16, D <= 128, Hkv divides H; rows and
    heads may be strided views); ptr int64 [graphs + 1], the rows of each graph's queries,
    and k_ptr those of its keys (default: the same); table [buckets, H] and buckets as
    relative_buckets() makes it; causal: keys later than the query are not seen (the last
    query is aligned with the last key); scale defaults to D ** -0.5. `stat` (float32
    [Nq, H, 2]) receives what global_attention_backward needs. Rows that belong to no graph
    get zeros, but are left as they were in an `out` that the caller brings."""
    lib = library()
    c = _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, out is None)
    dev = q.device
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
    _same_device(dev, out=out, stat=stat, workspace=workspace)
    with _on(dev):
        nbytes = _bytes(lib.pyg_global_attention_workspace, c)
        if nbytes and (workspace is None or workspace.numel() < nbytes):
            workspace = _workspace(nbytes, dev)
        _check(lib.pyg_global_attention(ctypes.byref(c), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(stat),
                                        _ptr(workspace), nbytes, _stream(dev)), "pyg_global_attention")
    return out


def global_attention_backward(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              out: torch.Tensor, stat: torch.Tensor, ptr: torch.Tensor,
                              k_ptr: torch.Tensor | None = None, table: torch.Tensor | None = None,
                              buckets: torch.Tensor | None = None, causal: bool = False, scale: float | None = None,
                              need_grad_table: bool = True, workspace: torch.Tensor | None = None):
    """Gradients of global_attention: (grad_q, grad_k, grad_v, grad_table or
    None), from its result `out` and the `stat` it filled."""
    lib = library()
    c = _attention(q, k, v, ptr, k_ptr, table, buckets, causal, scale, True)
    dev = q.device
    for name, t in (("grad_out", grad_out), ("out", out)):
        _need_cuda(name, t, q.dtype, 3)
        if t.shape != q.shape:
            raise ValueError(f"{name} must have q's shape")
    _need_cuda("stat", stat, torch.float32, 3)
    if stat.shape != (*q.shape[:2], 2):
        raise ValueError("stat must be [rows, heads, 2]")
    _same_device(dev, grad_out=grad_out, out=out, stat=stat, workspace=workspace)
    gq, gk, gv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
    gt = torch.empty_like(table) if table is not None and need_grad_table else None
    with _on(dev):
        nbytes = _bytes(lib.pyg_global_attention_backward_workspace, c)
        if workspace is None or workspace.numel() < nbytes:
            workspace = _workspace(nbytes, dev)
        _check(lib.pyg_global_attention_backward(ctypes.byref(c), _ptr(grad_out), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                                 _ptr(stat), _ptr(gq), _ptr(gk), _ptr(gv), _ptr(gt), _ptr(workspace),
                                                 workspace.numel(), _stream(dev)), "pyg_global_attention_backward")
    return gq, gk, gv, gt


def _adjacent(t):
    return t if t.dim() != 3 or t.shape[2] <= 1 or t.stride(2) == 1 and 0 not in t.stride() else t.contiguous()


class GlobalAttention(torch.autograd.Function):
    """Differentiable global_attention. Use as GlobalAttention.apply(q, k, v, table_or_None,
    ptr, k_ptr_or_None, buckets_or_None, causal, scale); gradients for q, k, v and the table."""

    @staticmethod
    def forward(ctx, q, k, v, table, ptr, k_ptr=None, buckets=None, causal: bool = False, scale: float | None = None):
        qc, kc, vc = (_adjacent(t.detach()) for t in (q, k, v))
        tc = None if table is None else table.detach().contiguous()
        need = any(ctx.needs_input_grad[:4])
        stat = torch.empty((*q.shape[:2], 2), dtype=torch.float32, device=q.device) if need else None
        out = global_attention(qc, kc, vc, ptr, k_ptr, tc, buckets, causal, scale, stat=stat)
        ctx.causal, ctx.scale = causal, scale
        ctx.save_for_backward(q, k, v, table, out, stat, ptr, k_ptr, buckets)
        return out

    @staticmethod
    def backward(ctx, grad_out):
        q, k, v, table, out, stat, ptr, k_ptr, buckets = ctx.saved_tensors
        qc, kc, vc = (_adjacent(t.detach()) for t in (q, k, v))
        tc = None if table is None else table.detach().contiguous()
        grads = global_attention_backward(grad_out.to(q.dtype).contiguous(), qc, kc, vc, out.contiguous(), stat, ptr, k_ptr,
                                          tc, buckets, ctx.causal, ctx.scale, need_grad_table=ctx.needs_input_grad[3])
        return tuple(g if need else None for g, need in zip(grads, ctx.needs_input_grad)) + (None,) * 5
