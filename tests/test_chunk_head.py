"""The header of a chunk plan: what was laid out, or, where the room did not hold it, a plan of nothing that fits no call
(the kernels compare the key, tests/test_gpu_chunk_plans.py).  Host code only."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_19242_amd", "csrc")


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("head") / "chunk_head_harness")
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-x", "hip", "-I", CSRC,
                    "-I", os.path.join(os.path.dirname(HERE), "include"), os.path.join(HERE, "chunk_head_harness.cpp"),
                    "-o", exe], check=True, capture_output=True)
    return exe


KEY = 0x89abcdef01234567


@pytest.mark.parametrize("longer,others,units,rows,written", [(3, 4, 2, 70, 1), (0, 0, 0, 0, 1), (1 << 20, 1 << 20, 5, 99, 1),
                                                             (3, 4, 2, 70, 0), (1 << 21, 0, 1 << 20, 200, 0)])
def test_headers(harness, longer, others, units, rows, written):
    line = f"{longer << 32 | others} {units << 32 | 1000} {rows} 100 4096 {KEY} {written}\n"
    got = [int(x) for x in subprocess.run([harness], input=line, capture_output=True, text=True, check=True).stdout.split()]
    key = (got[4] & 0xffffffff) | (got[5] & 0xffffffff) << 32
    want = (longer + others, units, KEY) if written else (0, 0, 0)
    assert (got[0], got[1], key) == want and got[2:4] == [min(rows, 100), 4096]
