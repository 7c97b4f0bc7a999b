"""The host code of the gated recurrence, layer norm and sampling on a runtime without a GPU: a CUDA call that fails ends the call with
TCU_ERR_CUDA, nothing is queued behind it, no error is left for a later call; what is refused is refused before anything is queued."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libtcu_more_fake.so")
    csrc = os.path.join(ROOT, "paper_2411_17887_b200", "csrc")
    subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O0", "--threads", "0", "--cudart", "none", "-shared", "-Xcompiler", "-fPIC",
                    "-Xlinker", "-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-o", out, *(os.path.join(csrc, name) for name in ("tcu_gated.cu", "tcu_norm.cu", "tcu_sample.cu")),
                    os.path.join(HERE, "fake_cudart.cpp")], check=True)
    lib = ctypes.CDLL(out, mode=os.RTLD_LOCAL | os.RTLD_NOW)
    lib.tcu_layer_norm_workspace_bytes.restype = ctypes.c_size_t
    lib.tcu_layer_norm_workspace_bytes.argtypes = [ctypes.c_size_t] * 2
    return lib


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


def at(i):
    return i << 36


def p(x):
    return ctypes.c_void_p(x)


def n(x):
    return ctypes.c_size_t(x)


def gated(lib, B, call, batch=3, tokens=700, channels=200, dtype=2, packed=False):
    rows = lambda i: (at(i), 0 if packed else tokens * channels, channels)  # noqa: E731
    marks = B.tcu_gated_marks_bytes(batch, tokens if packed else batch * tokens, channels)
    args = B.tcu_gated_args(dtype, 0, channels, batch, tokens, rows(1), rows(2), rows(3), d_offsets=at(9) if packed else 0, d_marks=at(4), marks_bytes=marks, d_y=rows(5), d_x=rows(6),
                            d_gate=rows(7), d_state_out=at(8))
    return getattr(lib, f"tcu_gated_{call}")(args, None)


def step(lib, B):
    return lib.tcu_gated_step(B.tcu_gated_args(2, 1, 77, 5, 1, (at(1), 77, 0), (at(2), 77, 0), (at(3), 77, 0), d_state_out=at(4), pool_slots=5), None)


def norm_forward(lib, B, rows=100, d=2048):
    return lib.tcu_layer_norm_forward(p(at(1)), n(rows), n(d), n(d), 2, p(at(2)), p(at(3)), 0, ctypes.c_float(1e-5), p(at(4)), None)


def norm_backward(lib, B, rows=100, d=2048):
    size = lib.tcu_layer_norm_workspace_bytes(rows, d)
    return lib.tcu_layer_norm_backward(p(at(1)), n(d), p(at(2)), n(d), n(rows), n(d), 2, p(at(3)), 0, ctypes.c_float(1e-5), p(at(4)), p(at(5)), p(at(6)), p(at(7)), n(size), None)


def sample(lib, B, rows=10, vocabulary=50000, **more):
    return lib.tcu_sample(B.tcu_sample_args(more.pop("dtype", 0), rows, vocabulary, at(1), vocabulary, at(2), 0, at(3), at(4), **more), None)


CALLS = {
    "recurrence": lambda lib, B: gated(lib, B, "forward"),
    "recurrence of one channel at a time": lambda lib, B: gated(lib, B, "forward", channels=201),
    "recurrence, packed": lambda lib, B: gated(lib, B, "forward", batch=40, packed=True),
    "gradients of the recurrence": lambda lib, B: gated(lib, B, "backward", dtype=0),
    "single tokens": step,
    "norm": norm_forward,
    "gradients of the norm": norm_backward,
    "gradients of the norm without rows": lambda lib, B: norm_backward(lib, B, rows=0),
    "sampling": sample,
    "sampling from many tokens": lambda lib, B: sample(lib, B, vocabulary=1 << 18),
}
FAILS = ("cudaLaunchKernel", "cudaLaunchKernelExC", "cudaFuncSetAttribute", "cudaMemsetAsync", "cudaGetDevice")


@pytest.mark.parametrize("what", CALLS)
def test_nothing_follows_a_call_that_failed(lib, B, what):
    run = CALLS[what]
    met = 0
    for name in FAILS:
        for k in range(1, 10):
            lib.fake_reset(name.encode(), k)
            status = run(lib, B)
            if not lib.fake_failed():
                break
            met += 1
            assert status == B.TCU_ERR_CUDA, (name, k)
            assert lib.fake_launches_after_failure() == 0, (name, k)
            lib.fake_reset(b"", 0)
            assert norm_forward(lib, B, rows=3, d=64) == B.TCU_OK                      # its launch is checked: no error is left
    assert met > 0
    lib.fake_reset(b"", 0)
    assert run(lib, B) == B.TCU_OK


def test_launches(lib, B):
    """How many launches a call has, and that one without work has none."""
    for what, count in (("recurrence", 1), ("gradients of the recurrence", 1), ("norm", 1), ("gradients of the norm", 2), ("gradients of the norm without rows", 0), ("sampling", 1)):
        lib.fake_reset(b"", 0)
        assert CALLS[what](lib, B) == B.TCU_OK and lib.fake_launches() == count, what
    lib.fake_reset(b"", 0)
    assert gated(lib, B, "forward", batch=0) == B.TCU_OK and sample(lib, B, rows=0) == B.TCU_OK and norm_forward(lib, B, rows=0) == B.TCU_OK
    assert lib.fake_launches() == 0


def test_refused_before_anything_is_queued(lib, B):
    lib.fake_reset(b"", 0)
    assert gated(lib, B, "forward", batch=1 << 31) == B.TCU_ERR_UNSUPPORTED
    assert gated(lib, B, "forward", batch=(1 << 63) + 1, channels=1 << 29) == B.TCU_ERR_UNSUPPORTED
    assert gated(lib, B, "backward", tokens=(1 << 31) - 8191) == B.TCU_ERR_UNSUPPORTED
    assert norm_forward(lib, B, d=16385) == B.TCU_ERR_UNSUPPORTED
    assert norm_forward(lib, B, rows=1 << 31) == B.TCU_ERR_UNSUPPORTED
    assert sample(lib, B, vocabulary=(1 << 18) + 1) == B.TCU_ERR_UNSUPPORTED
    assert sample(lib, B, top_p=float("nan")) == B.TCU_ERR_INVALID_ARG
    assert lib.fake_launches() == 0


def test_arrays_as_large_as_the_addresses(lib, B):
    """An array whose last byte has no address overlaps whatever lies behind its first one."""
    big = (at(1), (1 << 38) - 8, 64)
    args = B.tcu_gated_args(2, 0, 64, (1 << 24) + 1, 1, big, (at(1) >> 1, 0, 64), (at(1) + (1 << 30), 64, 64))
    lib.fake_reset(b"", 0)
    assert lib.tcu_gated_forward(args, None) == B.TCU_ERR_INVALID_ARG
    assert lib.fake_launches() == 0
