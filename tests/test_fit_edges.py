"""Inputs of the training-side calls at the edges of what their documentation allows, against the oracle.

Tolerances as in test_fit.py: a rounding to fp32 is off by 2^-24 of the value, to bf16 by 2^-8; S is the size of a score.
"""
import numpy as np
import pytest

from oracle import fit_oracle as F
from test_fit import _check_grad, _check_loss, _close, _dev, _gather_case, _host, _loss_case, _router

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("high", [1e5, 1e6, 1e7, 1e9, 1e10, 1e30, 3e38])
def test_an_entry_forced_in_by_its_bias_takes_all_weight(d, high):
    """One entry's bias outweighs all others': its softmax weight is one.  A score rounded to fp32 less itself is zero, whose exponential is off
    by 1.6e-7 at most (the passes' polynomial), and a mean of such weights by two roundings more."""
    import paper_2601_19178_b200 as ckv
    n, m, G = 500, 700, 3
    x, W, b, idx = _router(21, n, m, G, d, pad=0.1)
    at = [0, 130, 699]
    for g in range(G):
        b[g, at[g]] = high
    idx[idx[:, 0] >= 0, 0] = at[0]
    real = idx >= 0
    rows = real.sum(0)
    got = [_host(t) for t in _loss_case(x, W, b, idx)]
    one = 1.6e-7 + 2 * 2.0 ** -23
    want = F.route_loss(x, W, b, idx)
    assert np.isfinite(got[1]).all()
    _close(got[1], want[1], (d + 2) * 2.0 ** -23 * np.abs(want[1]), "lse")
    others = np.ones((G, m), bool)
    for g in range(G):
        _close(got[3][g, at[g]], 1.0, one, "mean")
        others[g, at[g]] = False
    assert not got[3][others].any()
    _close(got[0][:, 0], np.log(m), one * (1 + np.log(m)) + 2.0 ** -23 * np.log(m), "balance")
    # the gradient: T vanishes, the picked entries' terms stay
    w_peak = 0.5
    d_score = (np.random.default_rng(1).standard_normal((n, G)) / n).astype(np.float32)
    f32 = [v.astype(np.float32) for v in got[1:]]
    order = ckv.sort_indices(_dev(idx), m)
    grads = ckv.route_loss_grad(_dev(x), _dev(W), _dev(b), _dev(idx), order, *[_dev(v) for v in f32], 1.0, w_peak, _dev(d_score))
    dx, dW, db, size = F.route_loss_grad(x, W, b, idx, want[3], 1.0, w_peak, d_score.astype(np.float64))
    # what the picked entries' coefficients are made of, before it cancels: the sigmoid is off by 2^-21 and by a quarter of its score's error
    whole = F.route_loss_grad(x, W, b, idx, want[3], 0.0, -w_peak, np.abs(d_score).astype(np.float64))[3]
    es = (d + 2) * 2.0 ** -23 * np.abs(F.f64(x)[:, None, None, :] * F.f64(W)[None, :, ::7]).sum(3).max() * 2
    X, Wf = np.abs(F.f64(x)), np.abs(F.f64(W))
    # |T| of the forced entry: |p (h - r)| with p and sum p h off by 1e-4 (the polynomial of degree 3) at most
    T = 4 * 1e-4 * np.log(m) / rows
    left = {"dx": sum(real[:, g, None] * T[g] * Wf[g, at[g]][None] for g in range(G)), "dW": np.zeros((G, m, d)), "db": np.zeros((G, m))}
    for g in range(G):
        left["dW"][g, at[g]] = T[g] * X[real[:, g]].sum(0)
        left["db"][g, at[g]] = T[g] * rows[g]
    for name, g, w in (("dx", grads[0], dx), ("dW", grads[1], dW), ("db", grads[2], db)):
        half = 2.0 ** -8 if name != "db" else 0
        _close(_host(g), w, left[name] * (1 + 2 * half) + half * np.abs(w) + (2.0 ** -18 + es / 4) * whole[name][2] + 1e-37, name)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("shift", [2000.0, 1e5, -1e5, -1e6])
def test_a_shift_of_all_biases_changes_only_their_rounding(d, shift):
    """Scores of size S are off by 2^-23 S for each of the bias' three parts and of their own rounding, lse by one rounding more, and a weight
    by both."""
    n, m, G = 300, 500, 2
    x, W, b, idx = _router(22, n, m, G, d, pad=0.1)
    b = (b + np.float32(shift)).astype(np.float32)
    got = [_host(t) for t in _loss_case(x, W, b, idx)]
    want = F.route_loss(x, W, b, idx)
    S = np.abs(want[1]).max()
    es = 4 * 2.0 ** -23 * S + (d + 2) * 2.0 ** -23 * np.abs(F.scores(x, W, None, 0)).max() * 8
    assert np.isfinite(got[1]).all()
    _close(got[1], want[1], es + 2.0 ** -23 * S + 2.0 ** -21, "lse")
    e = np.expm1(2 * es + 2.0 ** -23 * S + 2.0 ** -19)
    _close(got[3], want[3], e * want[3] + 1e-37, "mean")
    _check_grad(x, W, b, idx, what=f"shift {shift}")


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("bad", [0x7fc0, 0x7f80, 0xff80])  # NaN, infinities of either sign
def test_inputs_that_are_no_numbers_stay_in_the_groups_that_take_part(d, bad):
    """Positions with an entry in group 1 alone, whose inputs are not finite: groups 0 and 2 have the same bits as if they were padding."""
    import paper_2601_19178_b200 as ckv
    n, m, G = 400, 300, 3
    x, W, b, idx = _router(23, n, m, G, d, pad=0.1)
    some = np.arange(3, n, 50)
    idx[some] = [-1, 7, m]
    x[some[::2]], x[some[1::2], 1] = bad, bad              # the whole row, or one number of it
    results = []
    for one in (idx, np.where(np.isin(np.arange(n), some)[:, None], -1, idx).astype(np.int32)):
        loss, lse, score, mean = _loss_case(x, W, b, one)
        order = ckv.sort_indices(_dev(one), m)
        grads = ckv.route_loss_grad(_dev(x), _dev(W), _dev(b), _dev(one), order, lse, score, mean, 1.0, 0.1)
        results.append([_host(t) for t in (loss, lse.t(), score.t(), mean, grads[1], grads[2])])
    for got, want in zip(*results):
        for g in (0, 2):
            assert np.isfinite(want[g]).all() and np.array_equal(got[g], want[g])
    assert np.isnan(results[0][0][1, 0]) and np.isnan(results[0][1][1, some]).all() and np.isnan(results[0][3][1]).all()


def test_scores_that_are_no_numbers_make_lse_none():
    x, W, b, idx = _router(24, 200, 300, 2, 64)
    x[5] = 0x7fc0
    loss, lse, score, mean = [_host(t) for t in _loss_case(x, W, b, idx)]
    other = np.arange(200) != 5
    assert np.isnan(lse[5]).all() and np.isfinite(lse[other]).all() and np.isnan(score[5]).all() and np.isnan(mean).all() and np.isnan(loss[:, 0]).all()


@pytest.mark.parametrize("n,m,G,d", [(20000, 300, 4, 32), (20000, 300, 4, 64), (15000, 200, 5, 128), (700, 15000, 4, 64), (300, 9000, 7, 128)])
def test_passes_of_more_blocks_than_run_at_a_time(n, m, G, d):
    """Partial results that a launch of their own joins: of LSE and R (more than 148 blocks of 384 positions), of MEAN (of as many entries)."""
    x, W, b, idx = _router(n + d, n, m, G, d, pad=0.1)
    idx[::11, 1] = m
    _check_loss(x, W, b, idx, f"n={n} m={m} G={G} d={d}")
    _check_grad(x, W, b, idx, what=f"n={n} m={m} G={G} d={d}")


def _inside(t, fill):
    """The tensor's values in the middle of a larger array of `fill`, 256 bytes from either end; the array, and its part."""
    import torch
    pad = 256 // t.element_size()
    flat = torch.full((t.numel() + 2 * pad,), fill, dtype=t.dtype, device="cuda")
    part = flat[pad:pad + t.numel()].view(t.shape)
    part.copy_(t)
    return flat, part


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [500, 3000])
def test_places_outside_of_the_arrays_are_left_out(n, dtype):
    """Positions just outside of [0, n) in a sorted order: they add nothing (NaN lies there), and nothing is written for them, around the
    results, or for the positions that do not appear."""
    import torch
    import paper_2601_19178_b200 as ckv
    G, m, D, du = 2, 40, 32, 2
    pool, idx, user, score, d_out = _gather_case(6, dtype, n, G, m, D, du, True)
    order, offset = F.sort_indices(idx, m)
    rng = np.random.default_rng(n)
    missing = np.zeros((n, G), bool)
    for g in range(G):
        at = rng.choice(n, 40, replace=False)
        missing[order[g, at], g] = True
        order[g, at] = rng.choice([-3, -1, n, n + 1, n + 5], 40)
    nan = float("nan")
    into = [_inside(t, 7.0) for t in (torch.full((G, m, D - du), 3.0, device="cuda"), torch.full((n, G, du), 3.0, device="cuda", dtype=_dev(pool).dtype),
                                      torch.full((n, G), 3.0, device="cuda"))]
    args = [_inside(_dev(pool), nan)[1], _inside(_dev(order), -1)[1], _inside(_dev(offset), -1)[1], _inside(_dev(score), nan)[1], _inside(_dev(d_out), nan)[1]]
    need = ckv.ckv_gather_grad_bytes(n, G, D)
    ws_flat, ws = _inside(torch.zeros(need, dtype=torch.uint8, device="cuda"), 9)
    ckv.ckv_gather_grad(0, ckv.CKV_BF16 if dtype == "bf16" else ckv.CKV_F32, n, G, D, D - du, m, *args, *[part for _, part in into],
                        ws if need else None, need)
    gone = np.where(missing, -1, idx).astype(np.int32)
    w_pool, w_user, w_score, a_pool, a_score = F.gather_grad(pool, gone, score, d_out)
    d_pool, d_user, d_score = [_host(part) for _, part in into]
    _close(d_pool, w_pool, (n * 2.0 ** -24 + 2.0 ** -20) * a_pool, "d_pool")
    assert np.array_equal(d_user, np.where(missing[:, :, None], 3.0, w_user))
    _close(d_score, np.where(missing, 3.0, w_score), (D * 2.0 ** -24 + 2.0 ** -19) * a_score, "d_score")
    for flat, part in (*into, (ws_flat, ws)):
        pad = 256 // flat.element_size()
        want = 9 if flat is ws_flat else 7
        assert (flat[:pad] == want).all() and (flat[flat.numel() - pad:] == want).all()


@pytest.mark.parametrize("n", [500, 3000])
def test_runs_outside_of_the_arrays_write_nothing_around_the_results(n):
    """Offsets that are no offsets, somewhat past the ends and out of order, for both gradients."""
    import torch
    import paper_2601_19178_b200 as ckv
    G, m, D, du, d = 2, 40, 32, 2, 64
    pool, idx, user, score, d_out = [_dev(t) for t in _gather_case(8, "bf16", n, G, m, D, du, True)]
    x, W, b, _ = [_dev(t) for t in _router(3, n, m, G, d)]
    _, lse, s, mean = ckv.route_loss(x, W, b, idx)
    order, offset = ckv.sort_indices(idx, m)
    g = torch.Generator(device="cuda").manual_seed(n)
    for wild in (torch.randint(-30, n + 30, (G, m + 1), generator=g, device="cuda", dtype=torch.int32), offset + 25, offset - 25, offset.flip(1).contiguous()):
        into = [_inside(t, 7.0) for t in (torch.zeros((G, m, D - du), device="cuda"), torch.zeros_like(user), torch.zeros((n, G), device="cuda"),
                                          torch.zeros_like(x), torch.zeros_like(W), torch.zeros_like(b))]
        need, need_route = ckv.ckv_gather_grad_bytes(n, G, D), ckv.ckv_route_loss_bytes(n, G, d, m)[1]
        ws_flat, ws = _inside(torch.zeros(max(need, need_route), dtype=torch.uint8, device="cuda"), 9)
        o = [_inside(order, -1)[1], _inside(wild, 2 ** 30)[1]]
        ckv.ckv_gather_grad(0, ckv.CKV_BF16, n, G, D, D - du, m, pool, *o, score, d_out, *[part for _, part in into[:3]], ws, ws.numel())
        ckv.ckv_route_loss_grad(0, n, G, d, m, x, W, b, idx, *o, lse, s, mean, 1.0, 1.0, None, *[part for _, part in into[3:]], ws, ws.numel())
        for flat, part in (*into, (ws_flat, ws)):
            pad = 256 // flat.element_size()
            want = 9 if flat is ws_flat else 7
            assert (flat[:pad] == want).all() and (flat[flat.numel() - pad:] == want).all()


def test_calls_from_several_threads():
    """First calls of fresh threads, for pools of different sizes: each kernel's shared memory differs between them."""
    import torch
    import paper_2601_19178_b200 as ckv
    from test_gpu_threads import _together
    sizes = [(5000, 5000), (8000, 20000), (9000, 24000), (300, 13000), (12000, 700), (8192, 24998)]
    threads = 24
    inputs = []
    for k in range(threads):
        n, m = sizes[k % len(sizes)]
        x, W, b, idx = _router(30 + k, n // 20 + 1, 90 + k, 2, (32, 64, 128)[k % 3])
        rng = np.random.default_rng(k)
        picked = rng.integers(-1, m + 1, (n, 2)).astype(np.int32)
        inputs.append((m, picked, _dev(picked), [_dev(t) for t in (x, W, b, idx)]))
    got, want = [None] * threads, []
    for m, picked, _, r in inputs:
        want.append([*F.sort_indices(picked, m), *[t.cpu() for t in ckv.route_loss(*r)]])
    torch.cuda.synchronize()

    def work(k):
        m, _, idx, r = inputs[k]
        for _ in range(5):
            got[k] = [*ckv.sort_indices(idx, m), *ckv.route_loss(*r)]
        torch.cuda.current_stream().synchronize()

    _together(threads, work)
    for g, w in zip(got, want):
        assert all(np.array_equal(a.cpu().numpy(), np.asarray(c)) for a, c in zip(g, w))


@pytest.mark.parametrize("n", [300, 3000])
@pytest.mark.parametrize("dtype,D,du", [("bf16", 64, 1), ("bf16", 64, 4), ("bf16", 64, 8), ("bf16", 128, 27), ("bf16", 16, 3), ("f32", 32, 1), ("f32", 32, 4), ("f32", 128, 13)])
def test_user_gradients_that_are_no_numbers_stay_in_d_user(n, dtype, D, du):
    """d_score is the product with the pool's part of the row alone."""
    import paper_2601_19178_b200 as ckv
    pool, idx, user, score, d_out = _gather_case(n + D, dtype, n, 2, 90, D, du, True)
    as_bits = np.asarray([0x7fc0, 0x7f80, 0xff80], np.uint16) if dtype == "bf16" else np.asarray([np.nan, np.inf, -np.inf], np.float32)
    for k in range(3):
        d_out[k::7, :, :du] = as_bits[k]
    d_pool, d_user, d_score = [_host(t) for t in ckv.gather_grad(_dev(pool), ckv.sort_indices(_dev(idx), 90), _dev(score), _dev(d_out))]
    w_pool, w_user, w_score, a_pool, a_score = F.gather_grad(pool, idx, score, d_out)
    assert np.array_equal(d_user, w_user, equal_nan=True)
    _close(d_pool, w_pool, (n * 2.0 ** -24 + 2.0 ** -20) * a_pool, "d_pool")
    _close(d_score, w_score, (D * 2.0 ** -24 + 2.0 ** -19) * a_score, "d_score")
