"""The grids of the layer operators: a launch holds fewer than 2^32 work items in a dimension, and every workgroup that is
asked for has to be in it (host code; no GPU needed)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2508_18182_amd import build as B

SOURCE = r"""
#include "layer_ops.h"
extern "C" void grid(long long n, int threads, unsigned* out) {
  const dim3 g = adloco::launch_grid(n, threads);
  out[0] = g.x; out[1] = g.y; out[2] = g.z;
}
"""


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("grid")
    (d / "g.hip").write_text(SOURCE)
    subprocess.run([hipcc, *B.HIPCC_FLAGS, "-shared", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, str(d / "g.hip"),
                    "-o", str(d / "g.so")], check=True, capture_output=True)
    lib = C.CDLL(str(d / "g.so"))

    def call(n, threads):
        out = (C.c_uint * 3)()
        lib.grid(C.c_longlong(n), threads, out)
        return list(out)
    return call


@pytest.mark.parametrize("threads", [64, 128, 256, 512])
def test_grid_holds_every_workgroup(grid, threads):
    most = (2**32 - 1) // threads                      # the most that one dimension holds
    for n in [1, 2, 7, most - 1, most, most + 1, most + 2, 2 * most, 2 * most + 1, 2**31 - 1]:
        x, y, z = grid(n, threads)
        assert z == 1 and 1 <= y < 65536 and x * threads < 2**32
        assert x * y >= n > x * y - x                  # all of them, and no row of the grid without one
        if n <= most:
            assert (x, y) == (n, 1)
