"""How many blocks serve the backward pass of the layer norm (tests/norm_dispatch_check.cu; nvcc, no GPU)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dispatch(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("norm") / "norm_dispatch_check")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17",
                           "-I", os.path.join(ROOT, "paper_2301_08527_b200", "csrc"), "-I", os.path.join(ROOT, "include"),
                           os.path.join(ROOT, "tests", "norm_dispatch_check.cu"), "-o", exe, "-lpthread"])

    def ask(*rows):
        out = subprocess.run([exe], input="".join("%d %d %d\n" % r for r in rows), capture_output=True, text=True, check=True)
        return [tuple(map(int, line.split())) for line in out.stdout.splitlines()]
    return ask


def test_dx_alone_has_all_blocks(dispatch):
    # as many blocks as there are rows for, with two at least on an SM
    cases = [(128, 4096, 128), (128, 1001, 128), (64, 4096, 64), (4096, 128, 128), (2048, 256, 128), (1024, 512, 128), (20, 1000, 20), (4, 1000, 4), (1, 5, 1)]
    assert dispatch(*[(N, P, 0) for N, P, _ in cases]) == [(owners, 0) for _, _, owners in cases]
