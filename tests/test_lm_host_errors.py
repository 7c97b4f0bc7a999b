"""The host code of the language-model operators on a runtime without a GPU.  A CUDA call that fails on the host ends a call of the language-model operators: nothing is queued behind it (the kernels of a
sequence index memory by what the ones before have written), and the caller gets TCU_ERR_CUDA.  And what is refused is refused before anything is queued."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libtcu_lm_fake.so")
    subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O0", "--cudart", "none", "-shared", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic",
                    "-I", os.path.join(ROOT, "include"), "-o", out, os.path.join(ROOT, "paper_2411_17887_b200", "csrc", "tcu_lm.cu"),
                    os.path.join(HERE, "fake_cudart.cpp")], check=True)
    return ctypes.CDLL(out, mode=os.RTLD_LOCAL | os.RTLD_NOW)


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


def p(x):
    return ctypes.c_void_p(x)


def gradient(lib, n, id_bytes, table=1 << 32):
    rows, d = 30000, 64
    size = lib.tcu_embedding_workspace_bytes
    size.restype, size.argtypes = ctypes.c_size_t, [ctypes.c_size_t] * 3
    return lib.tcu_embedding_backward(p(2 << 32), 2, p(3 << 32), id_bytes, ctypes.c_size_t(n), ctypes.c_size_t(rows), ctypes.c_size_t(d), ctypes.c_float(1.0), 0,
                                      p(table), 0, p(4 << 32), ctypes.c_size_t(size(n, rows, d)), None)


def attention(lib, B, backward, batch, tokens, heads, packed):
    at = lambda i: (i << 36, 0 if packed else tokens * heads * 64, heads * 64, 64)  # noqa: E731
    args = B.tcu_linattn_args(B.TCU_BF16, batch, tokens, heads, 64, 64, 1.0, 1 << 35, at(1), at(2), at(3), at(4), d_o=at(5), d_q=at(6), d_k=at(7), d_v=at(8),
                              d_offsets=(1 << 34) if packed else 0)
    size = lib.tcu_linattn_scratch_bytes
    size.restype = ctypes.c_size_t
    scratch = size(args, backward)
    args = B.tcu_linattn_with_scratch(args, (1 << 33) if scratch else 0, scratch)
    return (lib.tcu_linattn_backward if backward else lib.tcu_linattn_forward)(args, p(1 << 32), ctypes.c_size_t(256), None)


CALLS = {
    "gradient of 2000 tokens": lambda lib, B: gradient(lib, 2000, 8),            # sorted in one block
    "gradient of 2001 tokens": lambda lib, B: gradient(lib, 2001, 4),
    "gradient of 9000 tokens": lambda lib, B: gradient(lib, 9000, 8),            # counts added up by every block
    "gradient of 90000 tokens": lambda lib, B: gradient(lib, 90000, 4),          # and scanned
    "gradient of 40 tokens": lambda lib, B: gradient(lib, 40, 8),                # one launch
    "packed sequences in order": lambda lib, B: attention(lib, B, 0, 20, 3000, 16, True),
    "packed sequences": lambda lib, B: attention(lib, B, 0, 2, 3000, 16, True),
    "whole walks": lambda lib, B: attention(lib, B, 0, 1, 700, 3, False),
    "gradients": lambda lib, B: attention(lib, B, 1, 1, 700, 3, False),
}
FAILS = ("cudaLaunchKernel", "cudaLaunchKernelExC", "cudaFuncSetAttribute", "cudaGetDevice")


@pytest.mark.parametrize("what", CALLS)
def test_nothing_follows_a_call_that_failed(lib, B, what):
    run = CALLS[what]
    met = 0
    for name in FAILS:
        # (what a first call sets and remembers has to fail before any call that succeeds)
        for at in range(1, 20):
            lib.fake_reset(name.encode(), at)
            status = run(lib, B)
            if not lib.fake_failed():
                break
            met += 1
            assert status == B.TCU_ERR_CUDA, (name, at)
            assert lib.fake_launches_after_failure() == 0, (name, at)
    assert met > 0
    lib.fake_reset(b"", 0)
    assert run(lib, B) == B.TCU_OK
    assert lib.fake_launches() > 0


def test_walks_that_cannot_be_cut_run_whole(lib, B):
    """A cooperative launch that does not fit is no error: the walks run whole."""
    run = lambda: attention(lib, B, 0, 2, 700, 80, False)  # noqa: E731
    lib.fake_reset(b"", 0)
    assert run() == B.TCU_OK and lib.fake_launches() == 1
    lib.fake_reset(b"cudaLaunchKernelExC", 1)
    assert run() == B.TCU_OK and lib.fake_launches() == 2


@pytest.mark.parametrize("batch,heads", [(1 << 31, 1 << 30), (1 << 31, 1), (1 << 26, 2), (3, (1 << 32) - 1), ((1 << 63) + 1, 2), ((1 << 64) - 1, (1 << 32) - 1)])
def test_more_walks_than_a_grid_has_blocks(lib, B, batch, heads):
    """Also where batch times heads wraps around in 64 bits to a small number."""
    at = lambda i: (i << 36, 1 << 20, 64, 64)  # noqa: E731
    args = B.tcu_linattn_args(B.TCU_BF16, batch, 100, heads, 64, 64, 1.0, 1 << 35, at(1), at(2), at(3), at(4), d_o=at(5), d_q=at(6), d_k=at(7), d_v=at(8))
    lib.fake_reset(b"", 0)
    for fn in (lib.tcu_linattn_forward, lib.tcu_linattn_backward):
        assert fn(args, p(1 << 32), ctypes.c_size_t(256), None) == B.TCU_ERR_UNSUPPORTED
    for backward in (0, 1):
        assert lib.tcu_linattn_scratch_bytes(args, backward) == 0
    assert lib.fake_launches() == 0


def test_arrays_as_large_as_the_addresses(lib, B):
    """An array whose last byte has no address overlaps whatever lies behind its first one."""
    big = (1 << 36, (1 << 38) - 8, 64, 64)                               # 2^25 sequences of 2^39 bytes each
    o = ((1 << 36) + (1 << 30), 64, 64, 64)
    args = B.tcu_linattn_args(B.TCU_BF16, (1 << 25) + 1, 1, 1, 64, 64, 1.0, 1 << 35, big, (1 << 60, 0, 0, 0), (1 << 60, 0, 0, 0), o)
    lib.fake_reset(b"", 0)
    assert lib.tcu_linattn_forward(args, p(1 << 32), ctypes.c_size_t(256), None) == B.TCU_ERR_INVALID_ARG
    assert lib.fake_launches() == 0
    table = lambda stride, rows: lib.tcu_embedding_forward(p(3 << 32), 8, ctypes.c_size_t(10), p(2 << 40), ctypes.c_size_t(rows), ctypes.c_size_t(8),  # noqa: E731
                                                           ctypes.c_size_t(stride), 2, ctypes.c_float(1.0), p((2 << 40) + 4096), None)
    assert table(1 << 62, 9) == B.TCU_ERR_INVALID_ARG
    assert lib.fake_launches() == 0
    assert table(1 << 62, 1) == B.TCU_OK                                 # one row: no stride


def test_a_step_does_not_write_over_what_other_blocks_read(lib, B):
    """From 65 columns on a head's blocks read all of q and k while another writes its part of o."""
    q, k, v = ((i << 36, 2 * 128, 0, 128) for i in range(1, 4))
    for dv in (64, 65, 128):
        for o, ok in (((4 << 36, 2 * 128, 0, 128), True), (v, True), (q, dv <= 64), (k, dv <= 64)):
            args = B.tcu_linattn_args(B.TCU_BF16, 3, 1, 2, 128, dv, 1.0, 1 << 35, q, k, v, o, d_state_out=5 << 36, pool_slots=3)
            lib.fake_reset(b"", 0)
            assert lib.tcu_linattn_step(args, None) == (B.TCU_OK if ok else B.TCU_ERR_INVALID_ARG)
            assert lib.fake_launches() == ok


def test_no_error_is_left_for_a_later_call(lib, B, tmp_path):
    """Errors that a call has reported, or has found a way around, are not found again by the launch check of the next one.  (A library of
    its own, that remembers nothing.)"""
    import shutil
    for name in ("cudaOccupancyMaxActiveClusters", "cudaFuncSetAttribute", "cudaGetDevice", "cudaDeviceGetAttribute", "cudaMemsetAsync", "cudaMemcpyAsync"):
        one = str(tmp_path / f"{name}.so")
        shutil.copy(lib._name, one)
        one = ctypes.CDLL(one, mode=os.RTLD_LOCAL | os.RTLD_NOW)
        one.fake_reset(name.encode(), 1)
        calls = [CALLS[what] for what in ("packed sequences in order", "gradient of 2000 tokens")] + [lambda lib, B: attention(lib, B, 0, 2, 700, 80, False)]
        calls.append(lambda lib, B: lib.tcu_linattn_forward(B.tcu_linattn_args(B.TCU_BF16, 1, 0, 1, 64, 64, 1.0, 1 << 35, *[(0, 0, 0, 0)] * 4, d_state_in=1 << 36,
                                                                               d_state_out=1 << 37), p(1 << 32), ctypes.c_size_t(256), None))
        for call in calls:
            call(one, B)
        assert one.fake_failed()
        one.fake_reset(b"", 0)
        assert gradient(one, 40, 8) == B.TCU_OK, name                    # its one launch is checked
        assert [call(one, B) for call in calls] == [B.TCU_OK] * 4
        if name == "cudaOccupancyMaxActiveClusters":
            one = str(tmp_path / "again.so")
            shutil.copy(lib._name, one)
            one = ctypes.CDLL(one, mode=os.RTLD_LOCAL | os.RTLD_NOW)
            one.fake_reset(name.encode(), 3)
            assert calls[0](one, B) == B.TCU_OK                          # clusters of that size are not used, that is all


def test_results_do_not_overlap(lib, B):
    """States that overlap without being the same, and two gradients in one place, are written by blocks in any order."""
    at = lambda i: (i << 36, 0, 64, 64)  # noqa: E731
    lib.fake_reset(b"", 0)

    def call(backward=0, tokens=100, d_q=at(6), d_k=at(7), d_v=at(8), **states):
        args = B.tcu_linattn_args(B.TCU_BF16, 1, tokens, 1, 64, 64, 1.0, 1 << 35, at(1), at(2), at(3), at(4), d_o=at(5), d_q=d_q, d_k=d_k, d_v=d_v, **states)
        return (lib.tcu_linattn_backward if backward else lib.tcu_linattn_forward)(args, p(1 << 32), ctypes.c_size_t(256), None)

    s0, size = 1 << 37, 64 * 64 * 4
    for tokens in (0, 100):
        assert call(tokens=tokens, d_state_in=s0, d_state_out=s0) == B.TCU_OK
        assert call(tokens=tokens, d_state_in=s0, d_state_out=s0 + size) == B.TCU_OK
        for off in (16, size - 16, -16):
            assert call(tokens=tokens, d_state_in=s0, d_state_out=s0 + off) == B.TCU_ERR_INVALID_ARG
    assert call(backward=1) == B.TCU_OK
    joined = [(6 << 36 | 128 * i, 0, 192, 192) for i in range(3)]
    assert call(backward=1, d_q=joined[0], d_k=joined[1], d_v=joined[2]) == B.TCU_OK
    for bad in (dict(d_q=at(7)), dict(d_q=at(8)), dict(d_v=at(7))):
        assert call(backward=1, **bad) == B.TCU_ERR_INVALID_ARG
