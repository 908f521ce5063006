"""What adloco_block_product makes of its flags before any device work (no GPU needed)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

import paper_2508_18182_amd as A
from paper_2508_18182_amd import binding as bind
from paper_2508_18182_amd import build as B

HELPER = r"""
#include "common.h"
extern "C" void* new_context() { return new adloco_ctx(); }
extern "C" void delete_context(void* p) { delete static_cast<adloco_ctx*>(p); }
extern "C" unsigned exact_products() { return ADLOCO_EXACT_PRODUCTS; }
"""

EINVAL, EUNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("flags")
    (d / "h.hip").write_text(HELPER)
    A.load_library()
    subprocess.run([hipcc, *B.HIPCC_FLAGS, "-shared", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, str(d / "h.hip"),
                    "-o", str(d / "h.so")], check=True, capture_output=True)
    lib = C.CDLL(str(d / "h.so"))
    lib.new_context.restype = C.c_void_p
    lib.delete_context.argtypes = [C.c_void_p]
    p = lib.new_context()
    yield lib, C.c_void_p(p)
    lib.delete_context(p)


@pytest.mark.parametrize("dtype", [A.ADLOCO_F32, A.ADLOCO_BF16, A.ADLOCO_F16])
@pytest.mark.parametrize("flags", range(16))
def test_flags(host, flags, dtype):
    """Without rows there is nothing to launch: a call that is sound succeeds."""
    none, b = (bind.Blocks8Desc(1 << 40, 1 << 41, rows, 256, 256, 64) for rows in (0, 64))
    got = A.load_library().adloco_block_product(host[1], none, b, 1 << 42, 0, dtype, flags, None)
    known = flags & ~(A.ADLOCO_ACCUMULATE | A.ADLOCO_EXACT_PRODUCTS) == 0
    assert got == (EINVAL if not known else EUNSUPPORTED if flags & A.ADLOCO_ACCUMULATE and dtype != A.ADLOCO_F32 else 0)


def test_the_binding_has_the_headers_value(host):
    assert host[0].exact_products() == A.ADLOCO_EXACT_PRODUCTS
