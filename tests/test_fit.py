"""Training side of the router and the pool: oracle pins and refusals on the CPU, CUDA kernels against the oracle on the GPU.

Tolerances.  A rounding to fp32 is off by at most 2^-24 of the value, to bf16 by 2^-8.  S bounds sum_k |x_k w_k| + |b| of a
score, whose fp32 sum of d + 1 terms is off by at most (d + 2) 2^-23 S (the tensor core cuts instead of rounding); `e` below, the
relative error of a softmax weight, is twice that (score and lse) and 2^-19 for the exponential of arguments of some tens.
"""
import ctypes
import ctypes as C
import os

import numpy as np
import pytest

import synth
from oracle import fit_oracle as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
bits = synth.f32_to_bf16_bits


# ---- the oracle -------------------------------------------------------------------------------------------------

def _router(seed, n, m, G, d, spread=1.0, bias=True, pad=0.0):
    rng = np.random.default_rng(seed)
    x = bits((rng.standard_normal((n, d)) / np.sqrt(d)).astype(np.float32))
    W = bits((spread * rng.standard_normal((G, m, d))).astype(np.float32))
    b = (0.3 * rng.standard_normal((G, m))).astype(np.float32) if bias else None
    idx = np.stack([F.scores(x, W, b, g).argmax(1) for g in range(G)], 1).astype(np.int32)
    far = rng.random((n, G)) < 0.2                     # not every index is the arg-max: the calls do not ask for it
    idx[far] = rng.integers(0, m, int(far.sum()))
    idx[rng.random(n) < pad] = -1
    return x, W, b, idx


def test_oracle_losses_of_hand_worked_cases():
    # two entries, one position, scores (log 3, 0): p = (3/4, 1/4)
    x = np.array([[1.0, 0.0]], np.float32)
    W = np.array([[[np.log(3.0), 5.0], [0.0, 7.0]]], np.float32)
    loss, lse, score, mean = F.route_loss(x, W, None, np.array([[0]], np.int32))
    assert np.allclose(mean, [[0.75, 0.25]], atol=1e-7) and np.allclose(lse, np.log(4.0)) and np.allclose(score, np.log(3.0))
    assert np.allclose(loss, [[0.75 * np.log(1.5) + 0.25 * np.log(0.5), -np.log(0.75)]])
    # equal scores are balanced; a position without an entry changes nothing
    loss, *_ = F.route_loss(np.zeros((3, 2), np.float32), W, None, np.array([[0], [-1], [1]], np.int32))
    assert np.allclose(loss, [[0.0, np.log(2.0)]])


def test_oracle_gradient_equals_differences():
    n, m, G, d = 6, 5, 2, 3
    rng = np.random.default_rng(3)
    x, W, b = rng.standard_normal((n, d)), rng.standard_normal((G, m, d)), rng.standard_normal((G, m))
    idx = rng.integers(0, m, (n, G)).astype(np.int32)
    idx[2] = -1
    idx[4, 1] = m
    c = rng.standard_normal((n, G))

    def total(x, W, b):
        loss, _, score, _ = F.route_loss(x, W, b, idx)
        return 0.7 * loss[:, 0].sum() + 0.3 * loss[:, 1].sum() + (c * score).sum()

    mean = F.route_loss(x, W, b, idx)[3]
    dx, dW, db, _ = F.route_loss_grad(x, W, b, idx, mean, 0.7, 0.3, c)
    for a, da in ((x, dx), (W, dW), (b, db)):
        for k in range(a.size):
            at = np.unravel_index(k, a.shape)
            keep = a[at]
            a[at] = keep + 1e-5
            up = total(x, W, b)
            a[at] = keep - 1e-5
            down = total(x, W, b)
            a[at] = keep
            assert abs((up - down) / 2e-5 - da[at]) < 1e-8 + 1e-6 * abs(da[at])


def test_oracle_gather_gradient_equals_differences():
    n, m, G, ds, du = 5, 4, 2, 3, 2
    rng = np.random.default_rng(4)
    pool, user, score = rng.standard_normal((G, m, ds)), rng.standard_normal((n, G, du)), rng.standard_normal((n, G))
    idx = rng.integers(-1, m + 1, (n, G)).astype(np.int32)
    d_out = rng.standard_normal((n, G, du + ds))
    d_pool, d_user, d_score, _, _ = F.gather_grad(pool, idx, score, d_out)
    for a, da in ((pool, d_pool), (user, d_user), (score, d_score)):
        for k in range(a.size):
            at = np.unravel_index(k, a.shape)
            keep, v = a[at], []
            for e in (1e-6, -1e-6):
                a[at] = keep + e
                v.append((F.gather(pool, idx, user, score) * d_out).sum())
            a[at] = keep
            assert abs((v[0] - v[1]) / 2e-6 - da[at]) < 1e-7


def test_oracle_sort():
    idx = np.array([[2, 0], [-1, 1], [0, 7], [2, 1], [3, 0]], np.int32)
    order, offset = F.sort_indices(idx, 3)
    assert order.tolist() == [[2, 0, 3, 1, 4], [0, 4, 1, 3, 2]] and offset.tolist() == [[0, 1, 1, 3], [0, 2, 4, 4]]


# ---- refusals that need no GPU ----------------------------------------------------------------------------------

def test_sizes_are_refused_without_a_gpu():
    import paper_2601_19178_b200 as ckv
    L, v, w = ckv.lib, ctypes.c_int64(), ctypes.c_int64()
    bad, no = ckv.CKV_ERR_INVALID_ARG, ckv.CKV_ERR_UNSUPPORTED
    for n, G, m, want in ((-1, 1, 1, bad), (1, 0, 1, bad), (1, 1, 0, bad), (1, 65536, 1, no), (5, 2, 7, 0), (0, 1, 1, 0)):
        assert L.ckv_sort_indices_bytes(n, G, m, ctypes.byref(v)) == want
        assert L.ckv_route_loss_bytes(n, G, 64, m, ctypes.byref(v), ctypes.byref(w)) == want
        if want:
            assert L.ckv_sort_indices(0, n, G, m, None, None, None, None, 0, None) == want
            assert L.ckv_route_loss(0, n, G, 64, m, *[None] * 9, 0, None) == want
            assert L.ckv_route_loss_grad(0, n, G, 64, m, *[None] * 9, 0.0, 0.0, *[None] * 5, 0, None) == want
            assert L.ckv_gather(0, 1, n, G, 32, 30, m, *[None] * 6, 0, None) == want
            assert L.ckv_gather_bytes(1, n, G, 32, 30, m, ctypes.byref(v)) == want
            assert L.ckv_gather_grad(0, 1, n, G, 32, 30, m, *[None] * 9, 0, None) == want
    assert L.ckv_sort_indices_bytes(1, 1, 1, None) == bad
    for d in (0, 16, 48, 256):
        assert L.ckv_route_loss_bytes(1, 1, d, 1, ctypes.byref(v), ctypes.byref(w)) == no
        assert L.ckv_route_loss(0, 1, 1, d, 1, *[None] * 9, 0, None) == no
    assert L.ckv_gather(0, 1, 1, 1, 48, 30, 4, *[None] * 6, 0, None) == no
    assert L.ckv_gather(0, 2, 1, 1, 32, 30, 4, *[None] * 6, 0, None) == bad
    assert L.ckv_gather(0, 1, 1, 3, 32, 30, 2 ** 31 - 1, *[None] * 6, 0, None) == no              # more pool rows than 32 bits count
    for ds in (0, 33, -1):
        assert L.ckv_gather(0, 1, 1, 1, 32, ds, 4, *[None] * 6, 0, None) == ckv.CKV_ERR_SHAPE
        assert L.ckv_gather_grad(0, 1, 1, 1, 32, ds, 4, *[None] * 9, 0, None) == ckv.CKV_ERR_SHAPE


def test_wrong_tensors_are_refused_without_a_gpu():
    import torch
    import paper_2601_19178_b200 as ckv
    z = torch.zeros
    with pytest.raises(ValueError, match="CUDA"):
        ckv.sort_indices(z(3, 2, dtype=torch.int32), 5)
    with pytest.raises(ValueError, match="CUDA"):
        ckv.route_loss(z(3, 32, dtype=torch.bfloat16), z(1, 4, 32, dtype=torch.bfloat16), None, z(3, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        ckv.gather(z(1, 4, 30), z(3, 1, dtype=torch.int32), None)


from test_host_side import device_block, lib, objects, ptr  # noqa: E402,F401  (the library's host side on a stand-in for the CUDA runtime)


def _calls(lib):
    """Every call with arguments that it takes (sizes n = 20, G = 2, m = 30), as (function, arguments): device blocks for the arrays."""
    d = device_block(lib, 1 << 20)
    w = C.c_void_p((d.value + 255) // 256 * 256)
    big = C.c_int64(1 << 19)
    f = C.c_float
    return d, w, {
        "sort": (lib.ckv_sort_indices, [0, 20, 2, 30, d, d, d, w, big, None]),
        "loss": (lib.ckv_route_loss, [0, 20, 2, 64, 30, d, d, None, d, d, d, d, d, w, big, None]),
        "grad": (lib.ckv_route_loss_grad, [0, 20, 2, 64, 30, d, d, None, d, d, d, d, d, d, f(1), f(1), None, d, d, None, w, big, None]),
        "gather": (lib.ckv_gather, [0, 1, 20, 2, 32, 30, 30, d, d, d, None, d, w, big, None]),
        "gather_grad": (lib.ckv_gather_grad, [0, 1, 20, 2, 32, 30, 30, d, d, d, d, d, d, d, d, w, big, None])}


REQUIRED = {"sort": (4, 5, 6), "loss": (5, 6, 8, 9, 10, 11, 12, 13), "grad": (5, 6, 8, 9, 10, 11, 12, 13, 17, 18, 20),
            "gather": (7, 8, 9, 11), "gather_grad": (7, 8, 9, 11, 12, 14)}
OPTIONAL = {"loss": (7,), "grad": (7, 16, 19), "gather": (10,), "gather_grad": (13,)}


@pytest.mark.parametrize("name", list(REQUIRED))
def test_pointers_are_refused_without_a_gpu(lib, name):
    d, w, calls = _calls(lib)
    fn, args = calls[name]
    assert fn(*args) == 0
    host = np.zeros(1 << 20, np.uint8)
    odd = C.c_void_p(d.value + 1)
    for at in REQUIRED[name]:
        for wrong in (None, ptr(host), odd):
            assert fn(*args[:at], wrong, *args[at + 1:]) == 1, (at, wrong)
    for at in OPTIONAL.get(name, ()):
        for wrong in (ptr(host), odd):
            assert fn(*args[:at], wrong, *args[at + 1:]) == 1, (at, wrong)
    assert fn(-1, *args[1:]) == 1
    assert lib.fake_count(b"cudaLaunchKernelExC") >= 1


def test_workspaces_are_refused_without_a_gpu(lib):
    d, w, calls = _calls(lib)
    v, u = C.c_int64(), C.c_int64()
    assert lib.ckv_route_loss_bytes(20, 2, 64, 30, C.byref(v), C.byref(u)) == 0
    need = {"loss": (13, v.value), "grad": (20, u.value)}
    assert lib.ckv_gather_bytes(1, 70, 2, 32, 30, 30, C.byref(v)) == 0 and v.value > 0
    calls["gather"][1][2] = 70                                            # (rows enough for a copy of the pool)
    need["gather"] = (12, v.value)
    assert lib.ckv_sort_indices_bytes(9000, 2, 30, C.byref(v)) == 0 and v.value > 0
    calls["sort"][1][1] = 9000
    need["sort"] = (7, v.value)
    assert lib.ckv_gather_grad_bytes(600, 2, 32, C.byref(v)) == 0 and v.value > 0
    calls["gather_grad"][1][2] = 600
    need["gather_grad"] = (15, v.value)
    for name, (at, size) in need.items():
        fn, args = calls[name]
        assert fn(*args[:at], w, C.c_int64(size), *args[at + 2:]) == 0
        assert fn(*args[:at], w, C.c_int64(size - 1), *args[at + 2:]) == 1, name
        assert fn(*args[:at], C.c_void_p(w.value + 128), *args[at + 1:]) == 1, name


def test_calls_allocate_nothing_and_launch_few_kernels(lib):
    d, w, calls = _calls(lib)
    for name, launches in (("sort", 1), ("loss", 3), ("grad", 5), ("gather", 1), ("gather_grad", 1)):
        fn, args = calls[name]
        assert fn(*args) == 0
        lib.fake_reset()
        assert fn(*args) == 0
        assert lib.fake_count(b"cudaLaunchKernelExC") == launches, name
        for other in (b"cudaMalloc", b"cudaMallocHost", b"cudaHostAlloc", b"cudaFree", b"cudaStreamSynchronize", b"cudaMemcpyAsync", b"cudaFuncSetAttribute"):
            assert lib.fake_count(other) == 0, (name, other)


def test_a_launch_that_fails_is_reported(lib):
    d, w, calls = _calls(lib)
    for name in calls:
        fn, args = calls[name]
        lib.fake_reset()
        lib.fake_fail(b"cudaLaunchKernelExC", 1)
        assert fn(*args) != 0, name
        lib.fake_reset()
        assert fn(*args) == 0, name


# ---- the kernels ------------------------------------------------------------------------------------------------

def _dev(a):
    import torch
    from paper_2601_19178_b200.session import as_device_tensor
    return None if a is None else as_device_tensor(np.ascontiguousarray(a), "bf16" if a.dtype == np.uint16 else "i")


def _host(t):
    import torch
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _close(got, want, tol, what):
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - tol
    assert (over <= 0).all(), f"{what}: off by {np.abs(got - want).max():.3e}, {over.max():.3e} more than allowed at {np.unravel_index(over.argmax(), over.shape)}"


@pytest.mark.gpu
@pytest.mark.parametrize("n,G,m", [(0, 2, 5), (1, 1, 1), (2, 3, 70000), (37, 2, 5), (1000, 1, 1), (1023, 2, 32766), (1025, 2, 32768),
                                   (4097, 5, 255), (100003, 3, 4099), (300000, 1, 40000)])
def test_gpu_sort(n, G, m):
    import torch
    import paper_2601_19178_b200 as ckv
    rng = np.random.default_rng(n + m)
    for skew in (False, True):
        idx = (rng.integers(-2, m + 2, (n, G)) if not skew else np.minimum(rng.zipf(1.3, (n, G)) - 1, m + 3)).astype(np.int32)
        order, offset = ckv.sort_indices(_dev(idx), m)
        want_order, want_offset = F.sort_indices(idx, m)
        assert np.array_equal(offset.cpu().numpy(), want_offset) and np.array_equal(order.cpu().numpy(), want_order)


def _loss_case(x, W, b, idx):
    import paper_2601_19178_b200 as ckv
    loss, lse, score, mean = ckv.route_loss(_dev(x), _dev(W), _dev(b), _dev(idx))
    return loss, lse, score, mean


def _weight_error(x, W, b):
    X = F.f64(x)
    S = np.abs(X[np.isfinite(X)]).max(initial=0) * np.abs(F.f64(W)).sum(2).max()   # (padding may hold anything)
    S = S + (0 if b is None else np.abs(b[np.isfinite(b)]).max(initial=0))
    return (x.shape[1] + 2) * 2.0 ** -23 * S, 2 * (x.shape[1] + 2) * 2.0 ** -23 * S + 2.0 ** -19


def _check_loss(x, W, b, idx, what=""):
    m = W.shape[1]
    got = [_host(t) for t in _loss_case(x, W, b, idx)]
    want = F.route_loss(x, W, b, idx)
    es, e = _weight_error(x, W, b)
    for name, g, w in zip(("lse", "score"), got[1:3], want[1:3]):
        assert np.array_equal(np.isneginf(g), np.isneginf(w)), f"{what} {name}"
        fin = np.isfinite(w)
        _close(g[fin], w[fin], es + 2.0 ** -21 * (1 + np.abs(w[fin])), f"{what} {name}")
    _close(got[3], want[3], e * want[3] + 1e-37, f"{what} mean")
    used = np.where(want[3] > 0, want[3], 1)
    scale = (want[3] * np.abs(np.log(np.where(want[3] > 0, used * m, 1)))).sum(1)
    _close(got[0][:, 0], want[0][:, 0], e * (scale + e) + 2.0 ** -23 * want[0][:, 0], f"{what} balance")
    if np.isfinite(want[0][:, 1]).all():
        _close(got[0][:, 1], want[0][:, 1], es + 2.0 ** -21 * (1 + want[0][:, 1]), f"{what} peak")
    return got


SHAPES = [(1, 1, 1), (1, 300, 2), (37, 5, 2), (200, 1024, 2), (129, 127, 3), (513, 4100, 1), (1000, 64, 5), (2500, 700, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("n,m,G", SHAPES)
def test_gpu_route_loss(n, m, G, d):
    for spread, bias, pad in ((1.0, True, 0.0), (4.0, False, 0.4)):
        x, W, b, idx = _router(n + m + d, n, m, G, d, spread, bias, pad)
        _check_loss(x, W, b, idx, f"n={n} m={m} G={G} d={d} spread={spread}")


def _check_grad(x, W, b, idx, w_balance=1.0, w_peak=0.01, with_d=True, seed=0, what=""):
    import paper_2601_19178_b200 as ckv
    (n, d), (G, m, _) = x.shape, W.shape
    rng = np.random.default_rng(seed)
    d_score = (rng.standard_normal((n, G)) * 0.01 / max(n, 1)).astype(np.float32) if with_d else None
    _, lse, score, mean = F.route_loss(x, W, b, idx)
    f32 = [v.astype(np.float32) for v in (lse, score, mean)]
    order = ckv.sort_indices(_dev(idx), m)
    got = ckv.route_loss_grad(_dev(x), _dev(W), _dev(b), _dev(idx), order, *[_dev(v) for v in f32], w_balance, w_peak, _dev(d_score))
    dx, dW, db, size = F.route_loss_grad(x, W, b, idx, f32[2].astype(np.float64), w_balance, w_peak, None if d_score is None else d_score.astype(np.float64))
    _, e = _weight_error(x, W, b)
    e += 2.0 ** -23 * np.abs(f32[0][np.isfinite(f32[0])]).max(initial=0)        # lse comes rounded to fp32
    half = 2.0 ** -8
    for name, g, w, terms in (("dx", got[0], dx, m * G), ("dW", got[1], dW, n), ("db", got[2], db, n)):
        T, A, picked = size[name]
        sums = min(terms, 4096) * 2.0 ** -24 + 2.0 ** -20                        # fp32 sums of blocks of terms, and of the blocks
        tol = 2 * e * A + sums * (T + picked) + (half * T + half * np.abs(w) + half * half * T if name != "db" else 0) + 1e-37
        _close(_host(g), w, tol, f"{what} {name}")
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("n,m,G", SHAPES)
def test_gpu_route_loss_grad(n, m, G, d):
    for spread, bias, pad, with_d in ((1.0, True, 0.0, True), (4.0, False, 0.4, False)):
        x, W, b, idx = _router(n + m + d, n, m, G, d, spread, bias, pad)
        _check_grad(x, W, b, idx, with_d=with_d, what=f"n={n} m={m} G={G} d={d} spread={spread}")


@pytest.mark.gpu
def test_gpu_route_loss_of_padding_and_excluded_entries():
    """Positions that take part nowhere may hold anything; groups without a position, entries taken out by their bias,
    positions whose scores are all -inf."""
    x, W, b, idx = _router(5, 300, 200, 3, 64)
    idx[::3] = -1
    idx[1::7] = 200
    out = (idx < 0).all(1) | (idx >= 200).all(1)
    x[out] = 0x7fc0                                    # NaN
    x[np.nonzero(out)[0][::2]] = 0xff80                # -inf
    b[1, ::2] = -np.inf
    idx[:, 1] = np.where((idx[:, 1] >= 0) & (idx[:, 1] < 200), idx[:, 1] | 1, idx[:, 1])
    _check_loss(x, W, b, idx, "padding")
    got = _check_grad(x, W, b, idx, what="padding")
    assert not _host(got[0])[out].any() and not _host(got[1])[1, ::2].any()
    idx[:, 2] = -1
    loss = _check_loss(x, W, b, idx, "an empty group")[0]
    assert not loss[2].any()
    got = _check_grad(x, W, b, idx, what="an empty group")
    assert not _host(got[1])[2].any() and not _host(got[2])[2].any()
    idx[:] = -1
    assert not any(np.any(t) for t in _check_loss(x, W, b, idx, "no position"))
    assert not any(_host(t).any() for t in _check_grad(x, W, b, idx, what="no position"))
    # a group whose every entry is out: no weight anywhere
    x, W, b, idx = _router(6, 40, 30, 2, 32)
    b[0] = -np.inf
    got = _check_loss(x, W, b, idx, "every entry out")
    assert np.isneginf(got[1][:, 0]).all() and not got[3][0].any()


def test_oracle_takes_entries_out_by_their_bias():
    x, W, b, idx = _router(8, 30, 20, 2, 32)
    idx %= 7
    out, low = b.copy(), b.copy()
    out[:, 7:], low[:, 7:] = -np.inf, np.finfo(np.float32).min
    low[1, 9:] = -2.0 ** 20
    want = F.route_loss(x, W, out, idx)
    for g, w in zip(F.route_loss(x, W, low, idx), want):
        assert np.array_equal(g, w)
    part = F.route_loss(x, W[:, :7], b[:, :7], idx)
    assert np.allclose(part[1], want[1]) and np.allclose(part[3], want[3][:, :7]) and not want[3][:, 7:].any()
    grads = [F.route_loss_grad(x, W, v, idx, want[3], 1.0, 0.1)[:3] for v in (out, low)]
    assert all(np.array_equal(g, w) for g, w in zip(*grads))


@pytest.mark.gpu
@pytest.mark.parametrize("low", [-65504.0, -2.0 ** 20, -1e10, -1e30, float(np.finfo(np.float32).min)])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_gpu_router_entries_masked_by_a_large_bias_are_out(d, low):
    """Whole tiles of masked entries in front of the others, behind them, and all of a group: the bits that -inf gives."""
    import paper_2601_19178_b200 as ckv
    n, m, G = 150, 700, 3
    x, W, b, idx = _router(12, n, m, G, d)
    idx = (300 + idx % 40).astype(np.int32)
    results = []
    for v in (low, -np.inf):
        b[0, :300] = b[1, 340:] = v
        if low <= -2.0 ** 20:                          # (-65504 for all entries alike is no mask, but a shift)
            b[2] = v
        loss, lse, score, mean = _loss_case(x, W, b, idx)
        order = ckv.sort_indices(_dev(idx), m)
        grads = ckv.route_loss_grad(_dev(x), _dev(W), _dev(b), _dev(idx), order, lse, score, mean, 1.0, 0.0)
        results.append([_host(t) for t in (loss[:, 0], lse, mean, *grads)])
    for name, g, w in zip(("balance", "lse", "mean", "dx", "dW", "db"), *results):
        assert not np.isnan(w).any() and np.array_equal(g, w), name


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 128])
def test_gpu_router_inputs_and_gradients_off_the_16_byte_boundary(d):
    import torch
    import paper_2601_19178_b200 as ckv
    n, m, G = 77, 90, 2
    x, W, b, idx = [_dev(t) for t in _router(9, n, m, G, d)]

    def moved(t):                                       # the same values, two bytes further on
        flat = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")[1:t.numel() + 1]
        return flat.view(t.shape).copy_(t)

    want = ckv.route_loss(x, W, b, idx)
    got = ckv.route_loss(moved(x), W, b, idx)
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    order = ckv.sort_indices(idx, m)
    want_grad = ckv.route_loss_grad(x, W, b, idx, order, *want[1:], 1.0, 0.1)
    dx, dW, dbias = moved(x), moved(W), torch.empty((G, m), device="cuda")
    need = ckv.ckv_route_loss_bytes(n, G, d, m)[1]
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    ckv.ckv_route_loss_grad(0, n, G, d, m, moved(x), W, b, idx, *order, *want[1:], 1.0, 0.1, None, dx, dW, dbias, ws, need)
    assert all(torch.equal(a, c) for a, c in zip(want_grad, (dx, dW, dbias)))


@pytest.mark.gpu
def test_gpu_gather_off_the_word_boundary():
    """bf16 arrays on odd multiples of two bytes."""
    import torch
    import paper_2601_19178_b200 as ckv
    pool, idx, user, score, d_out = [_dev(t) for t in _gather_case(2, "bf16", 333, 2, 40, 32, 2, True)]

    def moved(t):
        return torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")[1:t.numel() + 1].view(t.shape).copy_(t)

    want = ckv.gather(pool, idx, user, score)
    for p, u in ((moved(pool), user), (pool, moved(user)), (moved(pool), moved(user))):
        assert torch.equal(ckv.gather(p, idx, u, score), want)
        out = moved(torch.zeros_like(want))
        need = ckv.ckv_gather_bytes(ckv.CKV_BF16, 333, 2, 32, 30, 40)
        ckv.ckv_gather(0, ckv.CKV_BF16, 333, 2, 32, 30, 40, p, idx, u, score, out, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
        assert torch.equal(out, want)
    order = ckv.sort_indices(idx, 40)
    want = ckv.gather_grad(pool, order, score, d_out)
    assert all(torch.equal(a, c) for a, c in zip(ckv.gather_grad(moved(pool), order, score, d_out), want))
    with pytest.raises(ckv.CkvError) as e:
        ckv.gather_grad(pool, order, score, moved(d_out))
    assert e.value.status == ckv.CKV_ERR_INVALID_ARG


@pytest.mark.gpu
def test_gpu_route_loss_without_positions():
    import torch
    import paper_2601_19178_b200 as ckv
    x, W, b, idx = _router(1, 4, 50, 2, 64)
    x, idx = x[:0], idx[:0]
    loss, lse, score, mean = _loss_case(x, W, b, idx)
    assert not loss.any() and not mean.any() and lse.shape == score.shape == (0, 2)
    got = ckv.route_loss_grad(_dev(x), _dev(W), _dev(b), _dev(idx), ckv.sort_indices(_dev(idx), 50), lse, score, mean, 1.0, 1.0)
    assert got[0].shape == (0, 64) and not got[1].any() and not got[2].any()


@pytest.mark.gpu
def test_gpu_route_loss_of_large_scores():
    """Scores of several hundreds, either sign: the running maximum, weights that vanish, a decided router."""
    rng = np.random.default_rng(8)
    x = bits((rng.standard_normal((200, 64)) * 4).astype(np.float32))
    W = bits((rng.standard_normal((2, 333, 64)) * 6).astype(np.float32))
    idx = rng.integers(0, 333, (200, 2)).astype(np.int32)
    got = [_host(t) for t in _loss_case(x, W, None, idx)]
    want = F.route_loss(x, W, None, idx)
    for g, w in zip(got[1:3], want[1:3]):
        _close(g, w, 66 * 2.0 ** -23 * np.abs(F.f64(x))[:, :, None].sum(1) * np.abs(F.f64(W)).max() + 2.0 ** -21 * np.abs(w), "large scores")
    assert abs(got[3].sum(1) - 1).max() < 1e-3


def _gather_case(seed, dtype, n, G, m, D, du, gated, pad=0.2):
    rng = np.random.default_rng(seed)
    cast = bits if dtype == "bf16" else (lambda a: a)
    pool = cast(rng.standard_normal((G, m, D - du)).astype(np.float32))
    user = cast(rng.standard_normal((n, G, du)).astype(np.float32)) if du else None
    idx = np.minimum(rng.zipf(1.2, (n, G)) - 1, m - 1).astype(np.int32) if seed % 2 else rng.integers(0, m, (n, G)).astype(np.int32)
    idx[rng.random((n, G)) < pad] = -1
    score = (3 * rng.standard_normal((n, G))).astype(np.float32) if gated else None
    d_out = cast(rng.standard_normal((n, G, D)).astype(np.float32))
    return pool, idx, user, score, d_out


GATHERS = [("bf16", 1, 1, 1, 16, 0), ("bf16", 200, 2, 1024, 32, 4), ("f32", 200, 2, 1024, 32, 4), ("bf16", 1000, 3, 77, 64, 1),
           ("bf16", 3001, 1, 5000, 64, 4), ("bf16", 777, 2, 3, 128, 8), ("f32", 999, 4, 50, 16, 3), ("f32", 300, 1, 9, 128, 127),
           ("bf16", 129, 5, 130, 32, 31), ("bf16", 50, 3, 900, 32, 1), ("f32", 400, 2, 90, 32, 20), ("bf16", 400, 2, 90, 64, 24), ("bf16", 700, 2, 3000, 128, 2), ("bf16", 65, 8, 64, 128, 0), ("f32", 5000, 1, 1, 64, 2), ("bf16", 40000, 2, 300, 32, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,G,m,D,du", GATHERS)
def test_gpu_gather(dtype, n, G, m, D, du):
    import paper_2601_19178_b200 as ckv
    for gated in (True, False):
        pool, idx, user, score, _ = _gather_case(n + D, dtype, n, G, m, D, du, gated)
        got = _host(ckv.gather(_dev(pool), _dev(idx), _dev(user), _dev(score)))
        want = F.gather(pool, idx, user, score)
        rel = (2.0 ** -20 if gated else 0) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (1 if gated else 0)
        _close(got, want, rel * np.abs(want), f"gated={gated}")
        if du:
            assert np.array_equal(got[:, :, :du], F.f64(user))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,G,m,D,du", GATHERS)
def test_gpu_gather_grad(dtype, n, G, m, D, du):
    import paper_2601_19178_b200 as ckv
    for gated in (True, False):
        pool, idx, user, score, d_out = _gather_case(n + D, dtype, n, G, m, D, du, gated)
        d_pool, d_user, d_score = ckv.gather_grad(_dev(pool), ckv.sort_indices(_dev(idx), m), _dev(score), _dev(d_out))
        w_pool, w_user, w_score, a_pool, a_score = F.gather_grad(pool, idx, score, d_out)
        _close(_host(d_pool), w_pool, (n * 2.0 ** -24 + 2.0 ** -20) * a_pool, "d_pool")
        if du:
            assert np.array_equal(_host(d_user), w_user)
        else:
            assert d_user is None
        if gated:
            _close(_host(d_score), w_score, (D * 2.0 ** -24 + 2.0 ** -19) * a_score, "d_score")
        else:
            assert d_score is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D,du", [("bf16", 64, 0), ("bf16", 64, 1), ("bf16", 64, 2), ("bf16", 64, 24), ("f32", 64, 4), ("f32", 64, 1)])
def test_gpu_gather_from_a_large_pool(dtype, D, du):
    """Pools of 8 MB and more, whose rows lie on elements, words or pieces, with fewer rows than twice the entries and with more."""
    import paper_2601_19178_b200 as ckv
    m = 40000
    pool, idx, user, score, _ = _gather_case(2, dtype, 2 * m + 5, 2, m, D, du, True)
    for n in (777, 2 * m + 5):
        i, u, s = idx[:n], None if user is None else user[:n], score[:n]
        got = _host(ckv.gather(_dev(pool), _dev(i), _dev(u), _dev(s)))
        want = F.gather(pool, i, u, s)
        _close(got, want, (2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)) * np.abs(want), f"n={n}")


@pytest.mark.gpu
@pytest.mark.parametrize("n", [300, 2000])
@pytest.mark.parametrize("dtype,D,du", [("bf16", 64, 1), ("bf16", 64, 4), ("bf16", 64, 8), ("bf16", 128, 24), ("bf16", 16, 3), ("f32", 32, 2), ("f32", 32, 4),
                                        ("f32", 128, 12)])
def test_gpu_gather_gradient_into_arrays_off_their_pieces(n, dtype, D, du):
    """Results an element further on: the bits of the aligned ones.  NaN where no position has an entry, and in rows nobody picked."""
    import torch
    import paper_2601_19178_b200 as ckv
    G, m = 3, 200
    pool, idx, user, score, d_out = _gather_case(n + du, dtype, n, G, m, D, du, True)
    nan = 0x7fc0 if dtype == "bf16" else np.nan
    d_out[:, :, du:][(idx < 0) | (idx >= m)] = nan
    for g in range(G):
        pool[g, np.setdiff1d(np.arange(m), idx[:, g])] = nan
    p, s, d = _dev(pool), _dev(score), _dev(d_out)
    order = ckv.sort_indices(_dev(idx), m)
    want = ckv.gather_grad(p, order, s, d)
    assert all(torch.isfinite(t).all() for t in (want[0], want[2]))
    moved = [torch.full((t.numel() + 8,), 7.0, dtype=t.dtype, device="cuda") for t in want]
    into = [f[1:t.numel() + 1].view(t.shape) for f, t in zip(moved, want)]
    need = ckv.ckv_gather_grad_bytes(n, G, D)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    ckv.ckv_gather_grad(0, ckv.CKV_BF16 if dtype == "bf16" else ckv.CKV_F32, n, G, D, D - du, m, p, *order, s, d, *into, ws, need)
    for f, t, w in zip(moved, into, want):
        assert torch.equal(t, w) and f[0] == 7 and (f[t.numel() + 1:] == 7).all()


@pytest.mark.gpu
def test_gpu_gather_and_gradient_without_positions():
    import torch
    import paper_2601_19178_b200 as ckv
    pool, idx, user, score, d_out = _gather_case(0, "bf16", 3, 2, 9, 32, 2, True)
    p, i = _dev(pool), _dev(idx[:0])
    assert ckv.gather(p, i, _dev(user[:0]), _dev(score[:0])).shape == (0, 2, 32)
    d_pool, d_user, d_score = ckv.gather_grad(p, ckv.sort_indices(i, 9), _dev(score[:0]), _dev(d_out[:0]))
    assert not d_pool.any() and d_pool.shape == (2, 9, 30) and d_user.shape == (0, 2, 2) and d_score.shape == (0, 2)


@pytest.mark.gpu
def test_gpu_refusals():
    import torch
    import paper_2601_19178_b200 as ckv
    x, W, b, idx = [_dev(t) for t in _router(1, 20, 30, 2, 64)]
    order = ckv.sort_indices(idx, 30)
    loss, lse, score, mean = ckv.route_loss(x, W, b, idx)
    need, need_grad = ckv.ckv_route_loss_bytes(20, 2, 64, 30)
    ws = torch.empty(max(need, need_grad), dtype=torch.uint8, device="cuda")

    def status(fn, *a):
        with pytest.raises(ckv.CkvError) as e:
            fn(*a)
        return e.value.status

    outs = [torch.empty_like(t) for t in (loss, lse, score, mean)]
    call = [0, 20, 2, 64, 30, x, W, b, idx, *outs, ws, need]
    ckv.ckv_route_loss(*call)
    for at in (5, 6, 8, 9, 10, 11, 12, 13):
        for wrong in (None, np.zeros(1 << 16, np.uint8)):
            assert status(ckv.ckv_route_loss, *call[:at], wrong, *call[at + 1:]) == ckv.CKV_ERR_INVALID_ARG
    assert status(ckv.ckv_route_loss, *call[:-1], need - 1) == ckv.CKV_ERR_INVALID_ARG
    flat = torch.empty(W.numel() + 4, dtype=torch.bfloat16, device="cuda")
    assert status(ckv.ckv_route_loss, *call[:6], flat[4:], *call[7:]) == ckv.CKV_ERR_INVALID_ARG       # W on 8 bytes
    assert status(ckv.ckv_route_loss, *call[:13], ws[16:], *call[14:]) == ckv.CKV_ERR_INVALID_ARG      # workspace on 16
    for wrong in (dict(x=x[:, :32].contiguous()), dict(x=x.float()), dict(idx=idx.long()), dict(idx=idx[:, :1].contiguous()), dict(b=b[:, 1:].contiguous())):
        with pytest.raises(ValueError):
            ckv.route_loss(wrong.get("x", x), W, wrong.get("b", b), wrong.get("idx", idx))
    with pytest.raises(ValueError):
        ckv.route_loss(x.t().contiguous().t(), W, b, idx)                                              # not contiguous
    with pytest.raises(ValueError):
        ckv.route_loss_grad(x, W, b, idx, (order[0][:, 1:].contiguous(), order[1]), lse, score, mean, 1.0, 1.0)
    pool = torch.zeros(2, 30, 28, device="cuda")
    with pytest.raises(ValueError):
        ckv.gather(pool.half(), idx, None)
    with pytest.raises(ValueError):
        ckv.gather(pool, idx, torch.zeros(20, 2, 4, device="cuda", dtype=torch.bfloat16))
    assert status(ckv.gather, pool, idx, None) == ckv.CKV_ERR_UNSUPPORTED                              # rows of 28
    d_out = torch.zeros(20, 2, 32, device="cuda")
    got = [torch.empty(2, 30, 28, device="cuda"), torch.empty(20, 2, 4, device="cuda"), torch.empty(20, 2, device="cuda")]
    n_ws = ckv.ckv_gather_grad_bytes(20, 2, 32)
    for s, d in ((score, None), (None, got[2])):                                                       # d_score iff score
        assert status(ckv.ckv_gather_grad, 0, ckv.CKV_F32, 20, 2, 32, 28, 30, pool, *order, s, d_out, got[0], got[1], d, ws, n_ws) == ckv.CKV_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("n", [500, 3000])
def test_gpu_an_order_that_is_none_reads_and_writes_in_bounds(n):
    """order and offset come from ckv_sort_indices; whatever else lies there, the calls stay inside their arrays."""
    import torch
    import paper_2601_19178_b200 as ckv
    pool, idx, user, score, d_out = [_dev(t) for t in _gather_case(0, "bf16", n, 2, 40, 32, 2, True)]
    x, W, b, picked = [_dev(t) for t in _router(2, n, 40, 2, 32)]
    _, lse, s, mean = ckv.route_loss(x, W, b, picked)
    g = torch.Generator(device="cuda").manual_seed(1)
    for lo, hi in ((-5, n + 100), (-2 ** 31, 2 ** 31 - 1)):
        order = torch.randint(lo, hi, (2, n), generator=g, device="cuda", dtype=torch.int32)
        offset = torch.randint(lo, hi, (2, 41), generator=g, device="cuda", dtype=torch.int32)
        for o in ((order, offset), (order, torch.sort(offset)[0]), (order, ckv.sort_indices(idx, 40)[1])):
            ckv.gather_grad(pool, o, score, d_out)
            ckv.route_loss_grad(x, W, b, picked, o, lse, s, mean, 1.0, 1.0, s)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("n,m", [(512, 7), (513, 7), (9000, 33), (60000, 20000)])
def test_gpu_a_collapsed_router(n, m):
    """Nearly all positions pick one entry: its run goes through many blocks; most entries have none."""
    import paper_2601_19178_b200 as ckv
    rng = np.random.default_rng(n)
    idx = np.full((n, 2), m // 2, np.int32)
    few = rng.random((n, 2)) < 0.02
    idx[few] = rng.integers(-1, m, int(few.sum()))
    order, offset = ckv.sort_indices(_dev(idx), m)
    want_order, want_offset = F.sort_indices(idx, m)
    assert np.array_equal(order.cpu().numpy(), want_order) and np.array_equal(offset.cpu().numpy(), want_offset)
    pool, _, _, score, d_out = _gather_case(4, "bf16", n, 2, m, 64, 3, True)
    d_pool, d_user, d_score = ckv.gather_grad(_dev(pool), (order, offset), _dev(score), _dev(d_out))
    w_pool, w_user, w_score, a_pool, a_score = F.gather_grad(pool, idx, score, d_out)
    _close(_host(d_pool), w_pool, (4096 * 2.0 ** -24 + 2.0 ** -20) * a_pool, "d_pool")      # sums of blocks of rows, and of the blocks
    assert np.array_equal(_host(d_user), w_user)
    _close(_host(d_score), w_score, (64 * 2.0 ** -24 + 2.0 ** -19) * a_score, "d_score")
    if n <= 9000:
        x, W, b, _ = _router(5, n, m, 2, 64)
        _check_loss(x, W, b, idx, "collapsed")
        _check_grad(x, W, b, idx, what="collapsed")


@pytest.mark.gpu
def test_gpu_arrays_of_more_than_2_to_the_31_elements():
    import torch
    import paper_2601_19178_b200 as ckv
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = torch.Generator(device="cuda").manual_seed(3)
    n, G, m, D = 700001, 25, 300, 128                                       # rows of d_out and out: 2.24e9 elements
    idx = torch.randint(-1, m, (n, G), generator=g, device="cuda", dtype=torch.int32)
    pool = torch.randn((G, m, D - 2), generator=g, device="cuda").bfloat16()
    user = torch.randn((n, G, 2), generator=g, device="cuda").bfloat16()
    out = ckv.gather(pool, idx, user)
    order = ckv.sort_indices(idx, m)
    last = slice(n - 5000, n)
    for k in (0, G - 1):
        i = idx[last, k].long()
        want = torch.cat([user[last, k], torch.where((i >= 0)[:, None], pool[k][i.clamp(min=0)], torch.zeros((), dtype=pool.dtype, device="cuda"))], 1)
        assert torch.equal(out[last, k], want)
    d_pool, d_user, d_score = ckv.gather_grad(pool, order, None, out)         # (the rows themselves as gradient: sums of equal rows)
    assert torch.equal(d_user, user) and d_score is None
    count = (order[1][:, 1:] - order[1][:, :-1]).float()[:, :, None]
    want = pool.float() * count
    assert ((d_pool - want).abs() <= 4096 * 2.0 ** -24 * want.abs()).all()
    del out, user, d_pool, d_user, want
    n, G, m, d = 70, 33, 1 << 20, 64                                        # W and dW: 2.2e9 elements
    x = (torch.randn((n, d), generator=g, device="cuda") / 8).bfloat16()
    W = torch.empty((G, m, d), dtype=torch.bfloat16, device="cuda")
    for k in range(G):
        W[k] = torch.randn((m, d), generator=g, device="cuda").bfloat16()
    idx = torch.randint(0, m, (n, G), generator=g, device="cuda", dtype=torch.int32)
    order = ckv.sort_indices(idx, m)
    loss, lse, score, mean = ckv.route_loss(x, W, None, idx)
    dx, dW, dbias = ckv.route_loss_grad(x, W, None, idx, order, lse, score, mean, 1.0, 1.0)
    k = G - 1                                                               # the last group, by the definition in 64 bits
    s = x.double() @ W[k].double().t()
    p = torch.softmax(s, 1)
    S = (x.double().abs().max() * W[k].double().abs().sum(1).max()).item()
    es = (d + 2) * 2.0 ** -23 * S                                            # of a score, and of a weight, see above
    e = 2 * es + 2.0 ** -19
    assert ((lse[:, k] - torch.logsumexp(s, 1)).abs() <= es + 2.0 ** -21 * (1 + lse[:, k].abs())).all()
    assert ((mean[k] - p.mean(0)).abs() <= e * p.mean(0)).all()
    h = torch.log(mean[k].double() * m) / n
    t = p * (h - (p @ h)[:, None])
    t[torch.arange(n, device="cuda"), idx[:, k].long()] -= torch.sigmoid(-score[:, k].double()) / n
    A = p * (h.abs() + (p @ h.abs())[:, None])
    half = 2.0 ** -8
    tol = 2 * e * (A.t() @ x.double().abs()) + (2 * half + 2.0 ** -18) * (t.abs().t() @ x.double().abs()) + 1e-37
    assert ((dW[k].double() - t.t() @ x.double()).abs() <= tol).all()
    assert ((dbias[k] - t.sum(0)).abs() <= 2 * e * A.sum(0) + 2.0 ** -18 * t.abs().sum(0)).all()


@pytest.mark.gpu
def test_gpu_results_are_the_same_bits_on_any_stream_and_replayed():
    import torch
    import paper_2601_19178_b200 as ckv
    x, W, b, idx = [_dev(t) for t in _router(2, 3000, 900, 2, 64, pad=0.1)]
    pool, _, user, _, d_out = [_dev(t) for t in _gather_case(1, "bf16", 3000, 2, 900, 32, 2, False)]

    def step():
        loss, lse, score, mean = ckv.route_loss(x, W, b, idx)
        K = ckv.gather(pool, idx, user, score)
        order = ckv.sort_indices(idx, 900)
        d_pool, d_user, d_score = ckv.gather_grad(pool, order, score, d_out)
        return [loss, lse, score, mean, K, *order, d_pool, d_user, d_score,
                *ckv.route_loss_grad(x, W, b, idx, order, lse, score, mean, 1.0, 0.01, d_score)]

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    assert all(torch.equal(a, w) for a, w in zip(again, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for t in held:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for a, w in zip(held, want))
    two = [torch.cuda.Stream() for _ in range(2)]           # two at once
    torch.cuda.synchronize()
    outs = []
    for s in two:
        with torch.cuda.stream(s):
            outs.append(step())
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for o in outs for a, w in zip(o, want))


@pytest.mark.gpu
def test_gpu_a_training_step_feeds_the_serving_calls():
    """Route, fit, refresh the pool, serve: the gated rows' attention loss falls along its gradient as differences say."""
    import torch
    import paper_2601_19178_b200 as ckv
    G, m, D, du, d, n = 2, 100, 32, 2, 64, 160
    x, W, b, _ = [_dev(t) for t in _router(7, n, m, G, d)]
    pool, _, user, _, target = _gather_case(3, "f32", n, G, m, D, du, True)
    pool, user, target = _dev(pool), _dev(user), _dev(target)
    idx = torch.empty((n, G), dtype=torch.int32, device="cuda")
    ckv.ckv_route(0, n, G, d, m, x, W, b, idx)
    loss, lse, score, mean = ckv.route_loss(x, W, b, idx)

    def task(p, s):
        return 0.5 * ((ckv.gather(p, idx, user, s) - target).double() ** 2).sum().item()

    out = ckv.gather(pool, idx, user, score)
    order = ckv.sort_indices(idx, m)
    d_pool, d_user, d_score = ckv.gather_grad(pool, order, score, out - target)
    assert torch.equal(d_user, (out - target)[:, :, :du])
    # central differences along random directions; second-order terms cancel, third-order ones are of the size of step^2
    g = torch.Generator(device="cuda").manual_seed(0)
    for t, dt in ((pool, d_pool), (score, d_score)):
        v = torch.randn(t.shape, generator=g, device="cuda") * 1e-2
        a, c = (task(t + v, score), task(t - v, score)) if t is pool else (task(pool, t + v), task(pool, t - v))
        slope = (dt.double() * v.double()).sum().item()
        assert abs((a - c) / 2 - slope) <= 1e-3 * abs(slope) + 1e-4 * dt.double().norm().item() * v.double().norm().item()
    dx, dW, db = ckv.route_loss_grad(x, W, b, idx, order, lse, score, mean, 1.0, 0.01, d_score)
    assert all(torch.isfinite(t.float()).all() for t in (dx, dW, db))
    # the refreshed pool serves: materialised rows are the ungated lookup
    s = ckv.CollectiveKV(G, D, torch.float32)
    new = pool - 0.1 * d_pool
    s.pool_load(new, new)
    s.cache_put(5, idx, idx, user, user)
    K, V = s.materialize(5)
    assert torch.equal(K, ckv.gather(new, idx, user)) and torch.equal(V, K)
    s.close()
