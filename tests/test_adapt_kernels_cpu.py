"""Which kernels the large calls of the operators that adapt a model launch, without a GPU: against a HIP runtime that logs launches
(launch_log.cpp).  The sizes are those that test_gpu_adapt_kernels.py checks against 64-bit results, so that every kernel that a
rule may choose for large calls is one that a test runs."""
import os
import subprocess
import sys

import pytest

from paper_1502_00512_amd import binding
from test_gpu_adapt_kernels import GRAD, MEET, words

HERE = os.path.dirname(os.path.abspath(__file__))

# (ctypes alone: torch would bring the real runtime along)
DRIVER = """
import ctypes as C, sys
C.CDLL(sys.argv[1], C.RTLD_GLOBAL)
lib = C.CDLL(sys.argv[2])
at = [1 << 44]
def dev():
    at[0] += 1 << 40
    return C.c_void_p(at[0])
i64, f, z = C.c_int64, C.c_float, C.c_size_t(1 << 39)
class Adapters(C.Structure):
    _fields_ = [("down", C.c_void_p), ("up", C.c_void_p), ("scale", C.c_void_p), ("n", C.c_int32), ("R", C.c_int32)]
def grad(dtype, rows, K, N, n, R):
    a = Adapters(dev(), dev(), None, n, R)
    return lib.rnnlm_adapter_backward(dev(), i64(N), dev(), i64(K), dev(), dtype, i64(rows), K, N, C.byref(a), dev(), dev(), dev(), dev(), i64(K), None, dev(), z, None)
def meet(dtype, T, P, V):
    return lib.rnnlm_preference_loss(dev(), dtype, T, P, V, i64(V), dev(), None, None, 0, f(0.1), f(0), 0, f(1), dev(), None, None, dev(), i64(V), None, dev(), z, None)
rc = eval(sys.argv[3])
assert rc == 0, rc
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    if not os.path.exists(binding.LIB_PATH):
        from paper_1502_00512_amd.build import build
        build()
    so = str(tmp_path_factory.mktemp("runtime") / "liblaunch_log.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_log.cpp")], check=True)
    return so


def kernels(runtime, tmp_path, call):
    log = str(tmp_path / "log")
    r = subprocess.run([sys.executable, "-c", DRIVER, runtime, binding.LIB_PATH, call], env=dict(os.environ, LAUNCH_LOG=log), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return [line.split()[2] for line in open(log) if line.startswith("L")]


def of(dtype, *numbers):
    """The template's arguments as a symbol spells them."""
    return "I" + {"fp32": "f", "bf16": "DF16b"}[dtype] + "".join(f"Li{i}E" for i in numbers)


@pytest.mark.parametrize("dtype,M,N,n,R,kernel", GRAD)
def test_gradients_of_wide_windows(runtime, tmp_path, dtype, M, N, n, R, kernel):
    names = [k for k in kernels(runtime, tmp_path, f"grad({int(dtype == 'bf16')}, {M}, 61, {N}, {n}, {R})") if "adapter_grad_kernel" in k]
    assert len(names) == 1 and "adapter_grad_kernel" + of(dtype, *kernel) + "Lb0E" in names[0]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,P,V,shape", MEET)
def test_rows_that_meet(runtime, tmp_path, T, P, V, shape, dtype):
    names = [k for k in kernels(runtime, tmp_path, f"meet({int(dtype == 'bf16')}, {T}, {P}, {words(dtype, V)})") if "preference_meet_kernel" in k]
    assert len(names) == (0 if shape is None else 1)
    assert shape is None or "preference_meet_kernel" + of(dtype, *shape) in names[0]


def test_every_kernel_of_large_calls_is_among_them():
    assert {(d, *k) for d, *_, k in GRAD} >= {("bf16", j, 4) for j in (1, 2, 3, 4)} | {("fp32", j, v) for j, v in ((1, 2), (1, 4), (2, 4), (3, 2), (4, 2))} | {("bf16", 1, 8)}
    assert {s for *_, s in MEET if s} == {(256, 6), (256, 8), (512, 6), (512, 8), (512, 12), (512, 16), (512, 20), (512, 25), (1024, 18), (1024, 25)}
