"""Fitting the router and the pool, for torch users: the training-side calls of the C ABI with their outputs and workspaces
allocated.  Work goes to the current stream of the tensors' device; no arithmetic here.  The results are no part of an autograd
graph: while gradients are recorded, tensors that require them are refused; call under `torch.no_grad()` (or with detached tensors) and
take the gradients from the calls that end in `_grad`.

A step of one side (keys or values), behind `ckv_route`:

    loss, lse, score, mean = route_loss(x, W, bias, idx)
    K = gather(pool, idx, user, score)                       # the model's keys; d_K from its backward pass
    ordered = sort_indices(idx, pool.shape[1])
    d_pool, d_user, d_score = gather_grad(pool, ordered, score, d_K)
    dx, dW, dbias = route_loss_grad(x, W, bias, idx, ordered, lse, score, mean, 1.0, 0.01, d_score)
"""
from __future__ import annotations

import functools
from typing import Optional, Tuple

import torch

from . import binding as B
from .session import _DT

# what the workspaces take: functions of the sizes alone
_sort_bytes = functools.lru_cache(maxsize=512)(B.ckv_sort_indices_bytes)
_loss_bytes = functools.lru_cache(maxsize=512)(B.ckv_route_loss_bytes)
_gather_bytes = functools.lru_cache(maxsize=512)(B.ckv_gather_bytes)
_gather_grad_bytes = functools.lru_cache(maxsize=512)(B.ckv_gather_grad_bytes)


def _refuse(name: str, t: torch.Tensor, shape, dtype, device):
    raise ValueError(f"{name} must be {dtype} {tuple(shape)} on cuda:{device}: got {t.dtype} {tuple(t.shape)} on {t.device}")


def _check(name: str, t: Optional[torch.Tensor], shape, dtype, device: int) -> None:
    if t is not None and (t.shape != shape or t.dtype is not dtype or t.get_device() != device):
        _refuse(name, t, shape, dtype, device)


def _no_graph(*tensors: Optional[torch.Tensor]) -> None:
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError("a tensor requires a gradient, which this call does not record: call it under torch.no_grad() and take the "
                             "gradients from route_loss_grad and gather_grad")


def _where(t: torch.Tensor) -> Tuple[int, int]:
    """Ordinal of the tensor's device, and the handle of the stream that is current there."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("the arguments must be CUDA tensors")
    return dev, _stream_of(dev)


def _stream_of(dev: int) -> int:
    # (the handle alone: torch.cuda.current_stream() builds a Stream object around it)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(dev) if raw is not None else torch.cuda.current_stream(dev).cuda_stream


def sort_indices(idx: torch.Tensor, n_entries: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """order [G][n], offset [G][n_entries + 1] (int32) of idx [n][G]: the positions by the entry they picked, those without
    one last; entry j's are order[g][offset[j]:offset[j + 1]]."""
    dev, stream = _where(idx)
    n, G = idx.shape
    _check("idx", idx, (n, G), torch.int32, dev)
    nbytes = _sort_bytes(n, G, n_entries)
    order, offset = idx.new_empty((G, n)), idx.new_empty((G, n_entries + 1))
    ws = idx.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    B.ckv_sort_indices(dev, n, G, n_entries, idx, order, offset, ws, nbytes, stream)
    return order, offset


def _check_router(x, W, bias, idx, dev):
    (n, d), (G, m, dw) = x.shape, W.shape
    _check("x", x, (n, dw), torch.bfloat16, dev)
    _check("W", W, (G, m, d), torch.bfloat16, dev)
    _check("bias", bias, (G, m), torch.float32, dev)
    _check("idx", idx, (n, G), torch.int32, dev)
    return n, d, G, m


def route_loss(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor], idx: torch.Tensor):
    """loss [G][2] (load balance, peak), lse [n][G], score [n][G], mean [G][m], all fp32, of router inputs x [n][d_in] and
    weights W [G][m][d_in] (bf16), bias [G][m] fp32 or None and the picked entries idx [n][G]."""
    _no_graph(x, W, bias)
    dev, stream = _where(x)
    n, d, G, m = _check_router(x, W, bias, idx, dev)
    nbytes = _loss_bytes(n, G, d, m)[0]
    f32 = torch.float32
    loss, lse = x.new_empty((G, 2), dtype=f32), x.new_empty((n, G), dtype=f32)
    score = torch.empty_like(lse)  # (less of the host's time than spelling it out)
    mean = x.new_empty((G, m), dtype=f32) if bias is None else torch.empty_like(bias)
    B.ckv_route_loss(dev, n, G, d, m, x, W, bias, idx, loss, lse, score, mean, x.new_empty(nbytes, dtype=torch.uint8), nbytes, stream)
    return loss, lse, score, mean


def route_loss_grad(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor], idx: torch.Tensor,
                    ordered: Tuple[torch.Tensor, torch.Tensor], lse: torch.Tensor, score: torch.Tensor, mean: torch.Tensor,
                    balance_weight: float, peak_weight: float, d_score: Optional[torch.Tensor] = None):
    """dx [n][d_in], dW [G][m][d_in] (bf16), dbias [G][m] (fp32) of sum_g (balance_weight balance_g + peak_weight peak_g) and of
    what else depends on the picked scores (d_score [n][G] or None); `ordered` is sort_indices(idx, m)."""
    _no_graph(x, W, bias, lse, score, mean, d_score)
    dev, stream = _where(x)
    n, d, G, m = _check_router(x, W, bias, idx, dev)
    order, offset = ordered
    i32, f32 = torch.int32, torch.float32
    _check("order", order, (G, n), i32, dev)
    _check("offset", offset, (G, m + 1), i32, dev)
    _check("lse", lse, (n, G), f32, dev)
    _check("score", score, (n, G), f32, dev)
    _check("mean", mean, (G, m), f32, dev)
    _check("d_score", d_score, (n, G), f32, dev)
    nbytes = _loss_bytes(n, G, d, m)[1]
    dx, dW, dbias = torch.empty_like(x), torch.empty_like(W), torch.empty_like(mean)
    B.ckv_route_loss_grad(dev, n, G, d, m, x, W, bias, idx, order, offset, lse, score, mean, balance_weight, peak_weight, d_score,
                          dx, dW, dbias, x.new_empty(nbytes, dtype=torch.uint8), nbytes, stream)
    return dx, dW, dbias


def _dtype_of(pool: torch.Tensor) -> int:
    dt = _DT.get(pool.dtype)
    if dt is None:
        raise ValueError(f"pool must be one of {list(_DT)}: got {pool.dtype}")
    return dt


def gather(pool: torch.Tensor, idx: torch.Tensor, user: Optional[torch.Tensor], score: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[n][G][d_user + d_shared]: user part (user [n][G][d_user] or None) and picked row of pool [G][m][d_shared], the latter times
    sigmoid(score [n][G]) if given; zeros for a position without an entry."""
    _no_graph(pool, user, score)
    dev, stream = _where(pool)
    dt = _dtype_of(pool)
    G, m, ds = pool.shape
    n = idx.shape[0]
    du = 0 if user is None else user.shape[2]
    _check("idx", idx, (n, G), torch.int32, dev)
    _check("user", user, (n, G, du), pool.dtype, dev)
    _check("score", score, (n, G), torch.float32, dev)
    out = pool.new_empty((n, G, du + ds))
    nbytes = _gather_bytes(dt, n, G, du + ds, ds, m)
    ws = pool.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    B.ckv_gather(dev, dt, n, G, du + ds, ds, m, pool, idx, user if du else None, score, out, ws, nbytes, stream)
    return out


def gather_grad(pool: torch.Tensor, ordered: Tuple[torch.Tensor, torch.Tensor], score: Optional[torch.Tensor], d_out: torch.Tensor):
    """d_pool [G][m][d_shared] (fp32), d_user [n][G][d_user] (None without a user part), d_score [n][G] (fp32; None without a
    gate) of `gather`, from d_out [n][G][d_user + d_shared] and `ordered` = sort_indices(idx, m)."""
    _no_graph(pool, score, d_out)
    dev, stream = _where(pool)
    dt = _dtype_of(pool)
    G, m, ds = pool.shape
    n, _, D = d_out.shape
    if D < ds:
        raise ValueError("d_out is narrower than the pool's rows")
    order, offset = ordered
    f32 = torch.float32
    _check("d_out", d_out, (n, G, D), pool.dtype, dev)
    _check("order", order, (G, n), torch.int32, dev)
    _check("offset", offset, (G, m + 1), torch.int32, dev)
    _check("score", score, (n, G), f32, dev)
    nbytes = _gather_grad_bytes(n, G, D)
    d_pool = pool.new_empty((G, m, ds), dtype=f32)
    d_user = pool.new_empty((n, G, D - ds)) if D > ds else None
    d_score = None if score is None else torch.empty_like(score)
    ws = pool.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    B.ckv_gather_grad(dev, dt, n, G, D, ds, m, pool, order, offset, score, d_out, d_pool, d_user, d_score, ws, nbytes, stream)
    return d_pool, d_user, d_score
