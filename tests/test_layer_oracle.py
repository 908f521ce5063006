"""CPU pins of the layer operators' oracle, and the refusals of their entry points (no GPU: they return before any device
work)."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2508_18182_amd as A
from oracle import layer_oracle as lo
from paper_2508_18182_amd import binding as bind
from paper_2508_18182_amd import build as B


@pytest.mark.parametrize("counter,key,want", [
    # the generator's published known answers
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, want):
    assert tuple(int(w) for w in lo.philox(counter, key)) == want


def test_dropout_share_and_slices():
    keep = lo.dropout_keep(4096, 200, 0.1, 0x0123456789ABCDEF)
    n = keep.size                                     # binomial: five standard deviations
    assert abs(keep.mean() - (1 - lo.dropout_threshold(0.1) / 65536)) < 5 * np.sqrt(0.09 / n)
    assert abs(np.corrcoef(keep[:, :-1].ravel(), keep[:, 1:].ravel())[0, 1]) < 5 / np.sqrt(n)
    assert np.array_equal(keep[100:200, :77], lo.dropout_keep(100, 77, 0.1, 0x0123456789ABCDEF, 100))
    assert not np.array_equal(keep, lo.dropout_keep(4096, 200, 0.1, 0x0123456789ABCDEE))


def test_norm_gradient_against_differences():
    r = np.random.default_rng(3)
    h, gain, dy, eps = r.normal(size=(4, 7)), r.normal(size=7), r.normal(size=(4, 7)), 1e-3
    dh, rows = lo.rms_norm_backward(h, gain, dy, eps)
    step = 1e-6
    for i in range(4):
        for j in range(7):
            up, down = h.copy(), h.copy()
            up[i, j] += step
            down[i, j] -= step
            diff = ((lo.rms_norm(up, gain, eps) - lo.rms_norm(down, gain, eps)) * dy).sum() / (2 * step)
            assert abs(diff - dh[i, j]) < 1e-7 * (1 + abs(diff))
    for j in range(7):
        up, down = gain.copy(), gain.copy()
        up[j] += step
        down[j] -= step
        diff = ((lo.rms_norm(h, up, eps) - lo.rms_norm(h, down, eps)) * dy).sum() / (2 * step)
        assert abs(diff - rows.sum(axis=0)[j]) < 1e-7 * (1 + abs(diff))


def test_e4m3_values_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(lo.e4m3_table(), want)


def test_blocks_by_hand():
    assert lo.block_exponent([0.0, 448.0, 448.1, 1.75, 1.76, 2.0**-140, 3.0e38]).tolist() == [1, 127, 128, 119, 120, 1, 247]
    x = np.zeros((1, 130))
    x[0, :4] = [448.0, 17.0, 1.0 + 1 / 16, np.inf]     # 17 and 1 + 1/16 lie half way: to the even neighbour
    x[0, 129] = -3.0
    q, e = lo.pack(x)
    assert q.shape == (1, 256) and e.tolist() == [[127], [120]]
    assert q[0, :3].tolist() == [448.0, 16.0, 1.0] and np.isnan(q[0, 3]) and q[0, 129] == -384.0 and not q[0, 130:].any()
    r = np.random.default_rng(5).normal(size=(9, 300)).astype(np.float32)
    q, e = lo.pack(r)
    codes = torch.from_numpy(q).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(lo.e4m3_table()[codes], q)           # every value is one of the type's
    back = lo.unpack(codes, e, 300)
    assert np.all(np.abs(back - r) <= np.abs(r) * 2.0**-4 + np.repeat(np.exp2(e.T - 127.0), 128, axis=1)[:, :300] * 2.0**-10)


# ---- refusals -------------------------------------------------------------------------------

HELPER = r"""
#include "common.h"
extern "C" void* new_context() { return new adloco_ctx(); }
extern "C" void delete_context(void* p) { delete static_cast<adloco_ctx*>(p); }
extern "C" const char* reason(void* p) { return static_cast<adloco_ctx*>(p)->err.c_str(); }
extern "C" void sizes(int* out) {
  out[0] = sizeof(adloco_dropout_mask); out[1] = sizeof(adloco_blocks8);
  out[2] = sizeof(adloco_norm_io); out[3] = sizeof(adloco_norm_backward_io);
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    """A context that owns no device, for the checks that come before any device work."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("host")
    (d / "h.hip").write_text(HELPER)
    A.load_library()
    subprocess.run([hipcc, *B.HIPCC_FLAGS, "-shared", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, str(d / "h.hip"),
                    "-o", str(d / "h.so")], check=True, capture_output=True)
    lib = C.CDLL(str(d / "h.so"))
    lib.new_context.restype = C.c_void_p
    lib.reason.restype = C.c_char_p
    lib.reason.argtypes = lib.delete_context.argtypes = [C.c_void_p]
    p = lib.new_context()
    yield lib, C.c_void_p(p)
    lib.delete_context(p)


def test_structs_match_the_header(host):
    got = (C.c_int * 4)()
    host[0].sizes(got)
    assert list(got) == [C.sizeof(t) for t in (bind.DropoutMask, bind.Blocks8Desc, bind.NormIo, bind.NormBackwardIo)]


BASE = 1 << 40          # addresses that nothing ever looks at


def _blocks(rows=64, cols=256, data=BASE, exponent=BASE + (1 << 30), row_stride=256, exponent_stride=64):
    return bind.Blocks8Desc(data, exponent, rows, cols, row_stride, exponent_stride)


def _code(host, name, *args):
    code = getattr(A.load_library(), name)(host[1], *args)
    if code:
        assert host[0].reason(host[1]).decode().startswith(name[len("adloco_"):] + ":"), host[0].reason(host[1])
    return code


EINVAL, EUNSUPPORTED = 1, 2


def _mask(p=0.1, seed=1, first_row=0):
    return C.byref(bind.DropoutMask(p, seed, first_row))


@pytest.mark.parametrize("change,want", [
    (dict(rows=0), 0), (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(rows=-1), EINVAL), (dict(d=0), EINVAL),
    (dict(dtype=7), EUNSUPPORTED), (dict(mask=None), EINVAL), (dict(mask=_mask(1.0)), EINVAL), (dict(mask=_mask(-0.1)), EINVAL),
    (dict(mask=_mask(float("nan"))), EINVAL), (dict(mask=_mask(1 - 2.0**-18)), EINVAL), (dict(mask=_mask(first_row=-1)), EINVAL),
    (dict(xs=63), EINVAL), (dict(os=32), EINVAL), (dict(x=BASE + 1), EINVAL), (dict(out=BASE + 2), EINVAL),
    (dict(out=BASE, os=65), EINVAL), (dict(residual=BASE + 200, out=BASE + 128), EINVAL), (dict(rows=1 << 60), EUNSUPPORTED),
])
def test_dropout_refuses(host, change, want):
    a = dict(x=BASE, xs=0, residual=None, rs=0, out=BASE + (1 << 33), os=0, rows=8, d=64, dtype=A.ADLOCO_BF16, mask=_mask())
    a.update(change)
    assert _code(host, "adloco_dropout", a["x"], a["xs"], a["residual"], a["rs"], a["out"], a["os"], a["rows"], a["d"], a["dtype"],
                 a["mask"], None) == want


@pytest.mark.parametrize("change,want", [
    (dict(rows=0), 0), (dict(cols=0), 0), (dict(along=None), EINVAL), (dict(dtype=3), EUNSUPPORTED), (dict(x=None), EINVAL),
    (dict(xs=255), EINVAL), (dict(rows=-1), EINVAL), (dict(x=BASE + (1 << 32) + 1), EINVAL),
    (dict(along=_blocks(rows=63)), EINVAL), (dict(along=_blocks(cols=255)), EINVAL), (dict(along=_blocks(data=BASE + 8)), EINVAL),
    (dict(along=_blocks(exponent=BASE + 8)), EINVAL), (dict(along=_blocks(row_stride=240)), EINVAL),
    (dict(along=_blocks(row_stride=264)), EINVAL), (dict(along=_blocks(exponent_stride=48)), EINVAL),
    (dict(along=_blocks(exponent_stride=72)), EINVAL), (dict(along=_blocks(data=None)), EINVAL),
    (dict(along=_blocks(exponent=BASE + 256)), EINVAL), (dict(x=BASE), EINVAL),
    (dict(across=_blocks()), EINVAL), (dict(across=_blocks(rows=256, cols=64, row_stride=128, exponent_stride=256)), EINVAL),
])
def test_pack_blocks_refuses(host, change, want):
    a = dict(x=BASE + (1 << 32), xs=0, rows=64, cols=256, dtype=A.ADLOCO_F32, along=_blocks(), across=None)
    a.update(change)
    assert _code(host, "adloco_pack_blocks", a["x"], a["xs"], a["rows"], a["cols"], a["dtype"], a["along"], a["across"], None) == want


@pytest.mark.parametrize("change,want", [
    (dict(a=_blocks(rows=0)), 0), (dict(b=_blocks(rows=0)), 0), (dict(a=None), EINVAL), (dict(b=None), EINVAL),
    (dict(dtype=9), EUNSUPPORTED), (dict(flags=2), EINVAL), (dict(flags=1), EUNSUPPORTED), (dict(b=_blocks(cols=250)), EINVAL),
    (dict(a=_blocks(row_stride=128)), EINVAL), (dict(b=_blocks(exponent_stride=16)), EINVAL), (dict(out=None), EINVAL),
    (dict(os=63), EINVAL), (dict(out=BASE + (1 << 32) + 1), EINVAL), (dict(out=BASE + 64), EINVAL),
])
def test_block_product_refuses(host, change, want):
    a = dict(a=_blocks(), b=_blocks(), out=BASE + (1 << 32), os=0, dtype=A.ADLOCO_BF16, flags=0)
    a.update(change)
    assert _code(host, "adloco_block_product", a["a"], a["b"], a["out"], a["os"], a["dtype"], a["flags"], None) == want


def _io(kind, **change):
    far = iter(range(1, 20))
    fields = [n for n, t in kind._fields_ if t is C.c_void_p]
    io = kind(**{n: BASE + next(far) * (1 << 32) for n in fields})
    for n, v in change.items():
        setattr(io, n, v)
    return io


@pytest.mark.parametrize("io,change,want", [
    ({}, dict(rows=0), 0), ({}, dict(rows=-1), EINVAL), ({}, dict(d=0), EINVAL), ({}, dict(d=16385), EUNSUPPORTED),
    ({}, dict(dtype=5), EUNSUPPORTED), ({}, dict(eps=0.0), EINVAL), ({}, dict(eps=float("nan")), EINVAL),
    ({}, dict(eps=float("inf")), EINVAL), ({}, dict(eps=1e-40), EINVAL), ({}, dict(rows=1 << 32), EUNSUPPORTED),
    ({}, dict(mask=_mask(2.0)), EINVAL), (dict(x=None), {}, EINVAL), (dict(h=None, y=None), {}, EINVAL),
    (dict(x=BASE + 1), {}, EINVAL), (dict(gain=BASE + 2), {}, EINVAL), (dict(h_row_stride=63), {}, EINVAL),
    (dict(h=BASE, y=BASE), {}, EINVAL), (dict(x=BASE, h=BASE + 2), {}, EINVAL), (dict(gain=BASE, y=BASE + 64), {}, EINVAL),
    ({}, dict(y8=_blocks(rows=8, cols=63)), EINVAL), ({}, dict(y8=_blocks(rows=9, cols=64)), EINVAL),
    (dict(x=BASE), dict(y8=_blocks(rows=8, cols=64)), EINVAL),
])
def test_rms_norm_refuses(host, io, change, want):
    a = dict(rows=8, d=64, dtype=A.ADLOCO_BF16, eps=1e-5, mask=None, y8=None)
    a.update(change)
    assert _code(host, "adloco_rms_norm", C.byref(_io(bind.NormIo, **io)), a["rows"], a["d"], a["dtype"], a["eps"], a["mask"], a["y8"],
                 None) == want


@pytest.mark.parametrize("io,change,want", [
    ({}, dict(B=0), 0), (dict(gain_sums=None), dict(T=0), 0), ({}, dict(B=-1), EINVAL), ({}, dict(T=-1), EINVAL),
    ({}, dict(d=0), EINVAL), ({}, dict(d=16385), EUNSUPPORTED), ({}, dict(dtype=5), EUNSUPPORTED), ({}, dict(eps=0.0), EINVAL),
    ({}, dict(B=1 << 16, T=1 << 16), EUNSUPPORTED), ({}, dict(mask=_mask(1.0)), EINVAL), (dict(h=None), {}, EINVAL),
    (dict(dy=None), {}, EINVAL), (dict(dh=None, dx=None, gain_sums=None), {}, EINVAL), (dict(dy_row_stride=3), {}, EINVAL),
    (dict(dh=BASE, dx=BASE), {}, EINVAL), (dict(dh=BASE, dy=BASE + 128, dy_row_stride=65), {}, EINVAL),
    (dict(gain_sums=BASE, dx=BASE + 64), {}, EINVAL), (dict(gain_sums=BASE + 2), {}, EINVAL), (dict(h=BASE, gain_sums=BASE), {}, EINVAL),
])
def test_rms_norm_backward_refuses(host, io, change, want):
    a = dict(B=2, T=4, d=64, dtype=A.ADLOCO_BF16, eps=1e-5, mask=None)
    a.update(change)
    assert _code(host, "adloco_rms_norm_backward", C.byref(_io(bind.NormBackwardIo, **io)), a["B"], a["T"], a["d"], a["dtype"],
                 a["eps"], a["mask"], None) == want


def test_strides_beyond_all_memory_are_refused(host):
    """Rows times stride beyond 64 bits: the check for overlaps would be made on what is left of the product."""
    far, many = 1 << 40, 1 << 30
    assert _code(host, "adloco_dropout", BASE, far, None, 0, BASE, far, many, 64, A.ADLOCO_F32, _mask(), None) == EINVAL
    io = _io(bind.NormIo, residual=None, h=None, x_row_stride=far, y_row_stride=far)
    assert _code(host, "adloco_rms_norm", C.byref(io), many, 64, A.ADLOCO_F32, 1e-5, None, None, None) == EINVAL
    io = _io(bind.NormBackwardIo, dh_row_stride=far)
    assert _code(host, "adloco_rms_norm_backward", C.byref(io), 1, many, 64, A.ADLOCO_F32, 1e-5, None, None) == EINVAL
    wide, tall = _blocks(rows=many, row_stride=far, exponent_stride=many), _blocks(cols=many, row_stride=many, exponent_stride=far)
    small = _blocks(data=BASE + (1 << 50), exponent=BASE + (1 << 51))
    for b in (wide, tall):
        assert _code(host, "adloco_pack_blocks", BASE, 0, b.rows, b.cols, A.ADLOCO_F32, b, None, None) == EINVAL
        assert _code(host, "adloco_block_product", b, b, BASE, 0, A.ADLOCO_F32, 0, None) == EINVAL
    assert _code(host, "adloco_pack_blocks", BASE, far, many, 256, A.ADLOCO_F32, _blocks(rows=many, exponent_stride=many), None, None) == EINVAL
    assert _code(host, "adloco_block_product", _blocks(rows=many, exponent_stride=many), small, BASE, far, A.ADLOCO_F32, 0, None) == EINVAL


def test_rms_norm_refuses_blocks_that_overlap_themselves(host):
    y8 = _blocks(rows=8, cols=64, row_stride=128, exponent_stride=16, exponent=BASE + 16)
    io = _io(bind.NormIo)
    assert _code(host, "adloco_rms_norm", C.byref(io), 8, 64, A.ADLOCO_BF16, 1e-5, None, y8, None) == EINVAL


def test_binding_refuses_before_the_library():
    class Ctx:
        device, _h = 0, None
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        A.adloco_dropout(Ctx, x, x, 0.1, 0)
    with pytest.raises(TypeError, match="float64"):
        A.adloco_rms_norm(Ctx, x.double(), None, 1e-5, y=x)
    with pytest.raises(ValueError, match="GPU"):
        A.adloco_block_product(Ctx, A.Blocks8.empty(4, 8, "cpu"), A.Blocks8.empty(4, 8, "cpu"), x)
    b = A.Blocks8.empty(5, 130, "cpu")
    assert tuple(b.data.shape) == (5, 256) and tuple(b.exponent.shape) == (2, 16)
