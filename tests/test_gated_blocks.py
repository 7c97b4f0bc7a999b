"""How many blocks walk a sequence of the gated recurrence together: as many as an SM's shared memory lets run at once, whatever the kernel's own needs."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SMS, OF_SM, OF_BLOCK = 148, 228 * 1024, 1024


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libtcu_gated_fake.so")
    subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O0", "-Xcicc", "-O0", "--cudart", "none", "-shared", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic",
                    "-I", os.path.join(ROOT, "include"), "-o", out, os.path.join(ROOT, "paper_2411_17887_b200", "csrc", "tcu_gated.cu"), os.path.join(HERE, "fake_launches.cpp")], check=True)
    lib = ctypes.CDLL(out, mode=os.RTLD_LOCAL | os.RTLD_NOW)
    lib.fake_last_shared.restype = ctypes.c_size_t
    return lib


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


def launch(lib, B, call, dtype, batch, tokens, channels, packed):
    rows = lambda i: (i << 36, 0 if packed else tokens * channels, channels)  # noqa: E731
    marks = B.tcu_gated_marks_bytes(batch, tokens if packed else batch * tokens, channels)
    args = B.tcu_gated_args(dtype, 0, channels, batch, tokens, rows(1), rows(2), rows(3), d_offsets=9 << 36 if packed else 0, d_marks=4 << 36, marks_bytes=marks, d_y=rows(5), d_x=rows(6),
                            d_gate=rows(7), d_state_out=8 << 36)
    lib.fake_reset(b"", 0)
    assert getattr(lib, f"tcu_gated_{call}")(args, None) == B.TCU_OK and lib.fake_launches() == 1
    return lib.fake_last_grid(), lib.fake_last_cluster(), lib.fake_last_shared()


@pytest.mark.parametrize("call", ["forward", "backward"])
@pytest.mark.parametrize("dtype", [0, 1, 2], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("channels", [1024, 1022, 1023], ids=["aligned", "even", "odd"])
def test_blocks_of_clusters_run_at_once(lib, B, call, dtype, channels):
    strips = (channels + 63) // 64
    met = set()
    for packed in (False, True):
        for batch in (1, 2, 3, 4, 5, 8, 9, 12, 18, 19, 40, 100):
            tokens = 4096 * (batch if packed else 1)
            grid, cluster, shared = launch(lib, B, call, dtype, batch, tokens, channels, packed)
            assert grid == batch * strips * cluster and cluster in (1, 2, 4, 8) and shared <= 227 * 1024
            met.add(cluster)
            # (registers: two blocks an SM)
            at_once = SMS * min(2, OF_SM // (shared + OF_BLOCK)) * (4 if packed else 1)
            assert cluster == 1 or grid <= at_once, (packed, batch, grid, cluster, shared)
            if cluster < 8 and grid * 2 <= SMS * (4 if packed else 1):
                raise AssertionError(("more blocks would run at once", packed, batch, grid, cluster))
    assert {1, 8} <= met
