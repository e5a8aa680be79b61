"""Fitting the router and the pool, for torch users: the training-side calls of the C ABI with their outputs and workspaces
allocated.  Work goes to the current stream of the tensors' device; no arithmetic here.

A step of one side (keys or values), behind `ckv_route`:

    loss, lse, score, mean = route_loss(x, W, bias, idx)
    K = gather(pool, idx, user, score)                       # the model's keys; d_K from its backward pass
    ordered = sort_indices(idx, pool.shape[1])
    d_pool, d_user, d_score = gather_grad(pool, ordered, score, d_K)
    dx, dW, dbias = route_loss_grad(x, W, bias, idx, ordered, lse, score, mean, 1.0, 0.01, d_score)
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as B
from .session import _DT


def _check(name: str, t: Optional[torch.Tensor], shape, dtype, device) -> None:
    if t is None:
        return
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on {device}: got {t.dtype} {tuple(t.shape)} on {t.device}")


def _where(t: torch.Tensor) -> Tuple[int, int]:
    """Ordinal of the tensor's device, and the handle of the stream that is current there."""
    if t.device.type != "cuda":
        raise ValueError("the arguments must be CUDA tensors")
    return t.device.index, torch.cuda.current_stream(t.device).cuda_stream


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def sort_indices(idx: torch.Tensor, n_entries: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """order [G][n], offset [G][n_entries + 1] (int32) of idx [n][G]: the positions by the entry they picked, those without
    one last; entry j's are order[g][offset[j]:offset[j + 1]]."""
    dev, stream = _where(idx)
    n, G = idx.shape
    _check("idx", idx, (n, G), torch.int32, idx.device)
    order = torch.empty((G, n), dtype=torch.int32, device=idx.device)
    offset = torch.empty((G, n_entries + 1), dtype=torch.int32, device=idx.device)
    nbytes = B.ckv_sort_indices_bytes(n, G, n_entries)
    B.ckv_sort_indices(dev, n, G, n_entries, idx, order, offset, _workspace(nbytes, idx.device), nbytes, stream)
    return order, offset


def _check_router(x, W, bias, idx):
    (n, d), (G, m, dw) = x.shape, W.shape
    _check("x", x, (n, dw), torch.bfloat16, x.device)
    _check("W", W, (G, m, d), torch.bfloat16, x.device)
    _check("bias", bias, (G, m), torch.float32, x.device)
    _check("idx", idx, (n, G), torch.int32, x.device)
    return n, d, G, m


def route_loss(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor], idx: torch.Tensor):
    """loss [G][2] (load balance, peak), lse [n][G], score [n][G], mean [G][m], all fp32, of router inputs x [n][d_in] and
    weights W [G][m][d_in] (bf16), bias [G][m] fp32 or None and the picked entries idx [n][G]."""
    dev, stream = _where(x)
    n, d, G, m = _check_router(x, W, bias, idx)

    def empty(*shape):
        return torch.empty(shape, dtype=torch.float32, device=x.device)

    loss, lse, score, mean = empty(G, 2), empty(n, G), empty(n, G), empty(G, m)
    nbytes = B.ckv_route_loss_bytes(n, G, d, m)[0]
    B.ckv_route_loss(dev, n, G, d, m, x, W, bias, idx, loss, lse, score, mean, _workspace(nbytes, x.device), nbytes, stream)
    return loss, lse, score, mean


def route_loss_grad(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor], idx: torch.Tensor,
                    ordered: Tuple[torch.Tensor, torch.Tensor], lse: torch.Tensor, score: torch.Tensor, mean: torch.Tensor,
                    balance_weight: float, peak_weight: float, d_score: Optional[torch.Tensor] = None):
    """dx [n][d_in], dW [G][m][d_in] (bf16), dbias [G][m] (fp32) of sum_g (balance_weight balance_g + peak_weight peak_g) and of
    what else depends on the picked scores (d_score [n][G] or None); `ordered` is sort_indices(idx, m)."""
    dev, stream = _where(x)
    n, d, G, m = _check_router(x, W, bias, idx)
    for name, t, shape, dtype in (("order", ordered[0], (G, n), torch.int32), ("offset", ordered[1], (G, m + 1), torch.int32),
                                  ("lse", lse, (n, G), torch.float32), ("score", score, (n, G), torch.float32),
                                  ("mean", mean, (G, m), torch.float32), ("d_score", d_score, (n, G), torch.float32)):
        _check(name, t, shape, dtype, x.device)
    dx, dW = torch.empty_like(x, memory_format=torch.contiguous_format), torch.empty_like(W, memory_format=torch.contiguous_format)
    dbias = torch.empty((G, m), dtype=torch.float32, device=x.device)
    nbytes = B.ckv_route_loss_bytes(n, G, d, m)[1]
    B.ckv_route_loss_grad(dev, n, G, d, m, x, W, bias, idx, ordered[0], ordered[1], lse, score, mean, balance_weight, peak_weight,
                          d_score, dx, dW, dbias, _workspace(nbytes, x.device), nbytes, stream)
    return dx, dW, dbias


def _check_pool(pool):
    if pool.dtype not in _DT:
        raise ValueError(f"pool must be one of {list(_DT)}: got {pool.dtype}")
    return pool.shape


def gather(pool: torch.Tensor, idx: torch.Tensor, user: Optional[torch.Tensor], score: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[n][G][d_user + d_shared]: user part (user [n][G][d_user] or None) and picked row of pool [G][m][d_shared], the latter times
    sigmoid(score [n][G]) if given; zeros for a position without an entry."""
    dev, stream = _where(pool)
    G, m, ds = _check_pool(pool)
    n = idx.shape[0]
    du = 0 if user is None else user.shape[2]
    _check("idx", idx, (n, G), torch.int32, pool.device)
    _check("user", user, (n, G, du), pool.dtype, pool.device)
    _check("score", score, (n, G), torch.float32, pool.device)
    out = torch.empty((n, G, du + ds), dtype=pool.dtype, device=pool.device)
    B.ckv_gather(dev, _DT[pool.dtype], n, G, du + ds, ds, m, pool, idx, user if du else None, score, out, stream)
    return out


def gather_grad(pool: torch.Tensor, ordered: Tuple[torch.Tensor, torch.Tensor], score: Optional[torch.Tensor], d_out: torch.Tensor):
    """d_pool [G][m][d_shared] (fp32), d_user [n][G][d_user] (None without a user part), d_score [n][G] (fp32; None without a
    gate) of `gather`, from d_out [n][G][d_user + d_shared] and `ordered` = sort_indices(idx, m)."""
    dev, stream = _where(pool)
    G, m, ds = _check_pool(pool)
    n, _, D = d_out.shape
    if D < ds:
        raise ValueError("d_out is narrower than the pool's rows")
    for name, t, shape, dtype in (("d_out", d_out, (n, G, D), pool.dtype), ("order", ordered[0], (G, n), torch.int32),
                                  ("offset", ordered[1], (G, m + 1), torch.int32), ("score", score, (n, G), torch.float32)):
        _check(name, t, shape, dtype, pool.device)
    d_pool = torch.empty((G, m, ds), dtype=torch.float32, device=pool.device)
    d_user = torch.empty((n, G, D - ds), dtype=pool.dtype, device=pool.device) if D > ds else None
    d_score = None if score is None else torch.empty((n, G), dtype=torch.float32, device=pool.device)
    nbytes = B.ckv_gather_grad_bytes(n, G, D)
    B.ckv_gather_grad(dev, _DT[pool.dtype], n, G, D, ds, m, pool, ordered[0], ordered[1], score, d_out, d_pool, d_user, d_score,
                      _workspace(nbytes, pool.device), nbytes, stream)
    return d_pool, d_user, d_score
