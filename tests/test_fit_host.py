"""What the training-side calls do on the host, on the CPU: the library's object files linked with a stand-in for the CUDA runtime."""
import ctypes as C
import os
import re
import subprocess
import threading

import numpy as np
import pytest

from test_fit import OPTIONAL, REQUIRED, _calls
from test_host_side import ROOT, device_block, objects  # noqa: F401


def _stand_in(objects, tmp, source):
    so = str(tmp / ("lib" + source.replace(".cpp", ".so")))
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I/usr/local/cuda/include", "-o", so,
                    *objects, os.path.join(ROOT, "tests", source)], check=True)
    return C.CDLL(so)


@pytest.fixture(scope="module")
def lib2(objects, tmp_path_factory):
    return _stand_in(objects, tmp_path_factory.mktemp("fit"), "fake_fit.cpp")


def _in_a_thread(work):
    got = []
    t = threading.Thread(target=lambda: got.append(work()))
    t.start()
    t.join(60)
    assert not t.is_alive()
    return got[0]


@pytest.mark.parametrize("n,large,small", [(5000, 20000, 13000), (9000, 24000, 14000)])
def test_a_sort_leaves_other_threads_their_shared_memory(lib2, n, large, small):
    """A thread's first sort, while another thread's first one, with fewer entries, runs between its permission and its launch."""
    lib = lib2
    need, other = C.c_int64(), C.c_int64()
    assert lib.ckv_sort_indices_bytes(n, 2, large, C.byref(need)) == lib.ckv_sort_indices_bytes(n, 2, small, C.byref(other)) == 0
    need.value = max(need.value, other.value)
    d, w = device_block(lib, 1 << 20), device_block(lib, max(need.value, 1) + 256)
    ws = C.c_void_p((w.value + 255) // 256 * 256)

    def sort(m):
        return lib.ckv_sort_indices(0, n, 2, m, d, d, d, ws, C.c_int64(need.value), None)

    inner = []
    hook = C.CFUNCTYPE(None)(lambda: inner.append(_in_a_thread(lambda: sort(small))))

    def outer():
        lib.fake_before_launch(hook)
        return sort(large)

    assert _in_a_thread(outer) == 0 and inner == [0]


def test_lanes_that_share_a_counter_read_it_before_it_moves_on():
    """Lanes with equal keys read the key's next place, and one of them writes the new one: the warp meets in between, for nothing else
    keeps its lanes together.  No result tells, so the source is read."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(ROOT, "paper_2601_19178_b200", "csrc", "kernels_sort.cu")).read())
    bodies = re.findall(r"int32_t take_places\(.*?\n\{(.*?)\n\}", code, re.S)
    assert len(bodies) == 2
    for body in bodies:
        read = max(m.start() for m in re.finditer(r"(= next\[d\]|volatile unsigned long long\*>\(slots \+ d\);)", body))
        write = re.search(r"next\[d\] = |slots \+ d\) = ", body).start()
        assert "__syncwarp();" in body[read:write], body


@pytest.mark.parametrize("name", list(REQUIRED))
def test_arrays_of_another_device_are_refused(lib2, name):
    """Every array has to lie on the call's device, or in managed memory."""
    lib = lib2
    d, w, calls = _calls(lib)
    fn, args = calls[name]
    managed, far = device_block(lib, 1 << 20), device_block(lib, 1 << 20)
    assert managed.value % 256 == far.value % 256 == 0
    lib.fake_block_of(managed, -1)
    lib.fake_block_of(far, 1)
    workspace = {"loss": 13, "grad": 20}.get(name)
    for at in (*REQUIRED[name], *OPTIONAL.get(name, ())):
        assert fn(*args[:at], managed, *args[at + 1:]) == 0, at
        assert fn(*args[:at], far, *args[at + 1:]) == 1, at
        if at != workspace:
            assert fn(1, *args[1:at], far, *args[at + 1:]) == 1, at      # (and the others on device 0)


def test_tensors_of_a_graph_are_refused():
    """The calls leave no graph behind: a tensor that wants gradients would get none without a word."""
    import torch
    import paper_2601_19178_b200 as ckv

    z = torch.zeros
    n, G, m, d = 3, 1, 4, 32
    idx, order, offset = z(n, G, dtype=torch.int32), z(G, n, dtype=torch.int32), z(G, m + 1, dtype=torch.int32)
    x, W, bias = z(n, d, dtype=torch.bfloat16), z(G, m, d, dtype=torch.bfloat16), z(G, m)
    per, mean, pool, user, d_out = z(n, G), z(G, m), z(G, m, 30), z(n, G, 2), z(n, G, 32)
    calls = [(ckv.route_loss, [x, W, bias, idx], (0, 1, 2)),
             (ckv.route_loss_grad, [x, W, bias, idx, (order, offset), per, per, mean, 1.0, 1.0, per], (0, 1, 2, 5, 6, 7, 10)),
             (ckv.gather, [pool, idx, user, per], (0, 2, 3)),
             (ckv.gather_grad, [pool, (order, offset), per, d_out], (0, 2, 3))]
    for fn, args, wants in calls:
        for at in wants:
            wanted = [a.clone().requires_grad_() if k == at else a for k, a in enumerate(args)]
            with pytest.raises(ValueError, match="no_grad"):
                fn(*wanted)
            with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):     # (further than that needs a GPU)
                fn(*wanted)
        with pytest.raises(ValueError, match="CUDA"):
            fn(*args)


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 5, 2 ** 63, -2 ** 31 - 1])
def test_sizes_of_more_than_32_bits_are_refused(n):
    """ctypes keeps the low 32 bits of a number: 2^32 + 5 positions would be five."""
    import paper_2601_19178_b200 as ckv
    for call in (lambda: ckv.ckv_sort_indices_bytes(n, 1, 1), lambda: ckv.ckv_sort_indices_bytes(5, 1, n),
                 lambda: ckv.ckv_sort_indices(0, n, 1, 1, None, None, None, None, 0, 1),
                 lambda: ckv.ckv_route_loss_bytes(n, 1, 64, 1), lambda: ckv.ckv_gather_bytes(1, n, 1, 32, 30, 1),
                 lambda: ckv.ckv_gather_grad_bytes(n, 1, 32), lambda: ckv.ckv_route(0, n, 1, 64, 4, None, None, None, None, stream=1)):
        with pytest.raises((C.ArgumentError, OverflowError), match="32 bits|too large"):
            call()


def test_polynomials_of_the_exponential_have_the_errors_stated_beside_them():
    """The coefficients as the kernels have them, 2^f on [-1/2, 1/2] in 64 bits; degree 5, which the losses' sums take, on average as well."""
    src = open(os.path.join(ROOT, "paper_2601_19178_b200", "csrc", "kernels_route_sweep.cu")).read()
    body = src[src.index("struct Exp2"):]
    body = body[:body.index("scale = {")]
    stated = [float(v) for v in re.search(r"\((\S+), (\S+), (\S+) for degrees 3 to 5", src).groups()]
    f = np.linspace(-0.5, 0.5, 20001)
    forms = [[np.float32(c) for c in re.findall(r"both\(([\d.]+)f\)", line)] for line in re.findall(r"p = (fma2.*?);", body, re.S)]
    assert sorted(len(c) for c in forms) == [4, 5, 6]
    for coefficients in forms:
        p = 0.0
        for c in coefficients:
            p = p * f + np.float64(c)
        error = p / np.exp2(f) - 1
        assert abs(error).max() <= stated[len(coefficients) - 4] * 1.01, len(coefficients) - 1
        if len(coefficients) == 6:
            assert abs(error.mean()) <= 2e-8
