"""The RMS norm and its backward pass at the ends of fp32: outputs that overflow, values next to the middle of two 8-bit or
16-bit ones, gradients and rows whose products leave the range that their quotients stay in."""
import numpy as np
import pytest
import torch

import paper_2508_18182_amd as A
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0**-24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def host(t):
    return t.detach().cpu().double().numpy()


def codes_of(b):
    wide = -(-b.cols // 128) * 128
    return lo.e4m3_table()[b.data[:, :wide].cpu().numpy()], b.exponent[:, :b.rows].cpu().numpy()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [128, 300, 2048])
def test_outputs_beyond_fp32(ctx, d, dtype):
    """y where it overflows is infinite and NaN in 8 bits, as packing it in fp32 gives; the rest of its block keeps its own
    exponent.  Rows of 16 values +- 9, 5, 3, 3, 1, 1, 1, 1 (mean square 16, twice) and zeros: n is what h is, over a power of
    two or the square root of one."""
    eight = torch.tensor([9.0, -5, 3, 3, 1, -1, 1, 1])
    h = torch.zeros(3, d)
    h[:, :16] = eight.repeat(2)
    h[1] = -h[1]
    h[2, 0] = 0.0                                      # (0 times a large gain)
    x = h.to(TYPES[dtype]).to(DEV)
    gain = torch.full((d,), 0.5)
    gain[0], gain[1], gain[9] = 3.0e38, -3.0e38, 3.4e38
    y, y32, y8, again = torch.empty_like(x), torch.empty(3, d, device=DEV), A.Blocks8.empty(3, d, DEV), A.Blocks8.empty(3, d, DEV)
    A.adloco_rms_norm(ctx, x, gain.to(DEV), 1e-30, y=y, y8=y8)
    A.adloco_rms_norm(ctx, x.float(), gain.to(DEV), 1e-30, y=y32)
    want = lo.rms_norm(h.double().numpy(), gain.double().numpy(), 1e-30)
    over = np.abs(want) > 3.4028235e38                 # (the nearest of them are a factor of 1.2 away)
    assert over.sum() >= 5
    got = host(y32)
    assert np.array_equal(np.isinf(got), over) and np.array_equal(np.sign(got[over]), np.sign(want[over]))
    assert np.array_equal(np.isinf(host(y))[over], np.ones(over.sum(), bool)) and not np.isnan(host(y)).any()
    codes, exps = codes_of(y8)
    A.adloco_pack_blocks(ctx, y32, again)
    assert np.array_equal(np.isnan(codes[:, :d]), over)
    assert np.array_equal(np.isnan(codes_of(again)[0][:, :d]), over) and np.array_equal(exps, codes_of(again)[1])
    finite = np.where(over, 0.0, want)
    power = np.repeat(np.exp2(exps.astype(np.float64) - 127).T, 128, axis=1)[:, :d]
    assert np.array_equal(exps, lo.pack(finite)[1])
    off = np.abs(codes[:, :d] * power - finite)
    assert (off[~over] <= ((2.0**-4 * (1 + 64 * U) + 64 * U) * np.abs(finite) + 2.0**-10 * power)[~over]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_gains_that_are_not_finite(ctx, dtype):
    x = torch.tensor([[9.0, -5, 3, 3, 1, -1, 1, 0] * 3], dtype=TYPES[dtype], device=DEV)
    x = x * torch.tensor([1.0, 0.37], device=DEV)[:, None].to(x.dtype)
    gain = torch.full((24,), 0.3, device=DEV)
    gain[0:3], gain[5], gain[7], gain[15], gain[16] = float("inf"), float("-inf"), float("inf"), 0.0, float("nan")
    y, y8 = torch.empty_like(x), A.Blocks8.empty(2, 24, DEV)
    A.adloco_rms_norm(ctx, x, gain, 1e-5, y=y, y8=y8)
    with np.errstate(invalid="ignore"):
        want = lo.rms_norm(host(x), host(gain), 1e-5)
    got = host(y)
    wild = ~np.isfinite(want)
    assert np.array_equal(got[wild], want[wild], equal_nan=True) and np.isfinite(got[~wild]).all()
    np.testing.assert_allclose(got[~wild], want[~wild], rtol=torch.finfo(y.dtype).eps / 2 * (1 + 64 * U) + 64 * U)
    assert np.array_equal(np.isnan(codes_of(y8)[0][:, :24]), wild)


def next_to_middles(bits):
    """Gains such that a value 5/4 (or 3/4, 9/4) times one lies within 2^-24 of the middle of two neighbouring numbers of `bits`
    mantissa bits, on either side of it and never on it: rounded to fp32 first, it often is that middle."""
    out = []
    for over in (9, 5, 3):
        for i in range(2**bits) if bits < 4 else range(0, 2**bits, 5):
            middle = 1 + (2 * i + 1) * 2.0**-(bits + 1)
            g = np.float32(middle * 4 / over)
            out += [(over, v) for v in (g, np.nextafter(g, np.float32(0)), np.nextafter(g, np.float32(9)))
                    if float(v) * over / 4 != middle]
    return out


@pytest.mark.parametrize("out,dtype", [("y8", "f32"), ("y8", "bf16"), ("y", "bf16"), ("y", "f16")])
def test_values_next_to_the_middle_of_two_are_rounded_once(ctx, out, dtype):
    """Rows of +- 9, 5, 3, 3, 1, 1, 1, 1: their mean square is 16 (eps 2^-126 is lost beside it even in fp64), n = h / 4 is exact,
    and n times a gain of 24 bits is exact in fp64, so that the oracle's rounding of it is the rounding of the value itself."""
    bits = {"y8": 3, "bf16": 7, "f16": 10}[out if out == "y8" else dtype]
    cases = next_to_middles(bits)
    d = 1 << (8 * len(cases) - 1).bit_length()
    h, gain = np.tile([9.0, -5, 3, 3, 1, -1, 1, 1], d // 8), np.ones(d, np.float32)
    at = {9: 0, 5: 1, 3: 2}
    for k, (over, g) in enumerate(cases):
        gain[8 * k + at[over]] = g
    x = torch.from_numpy(np.stack([h, -h])).to(TYPES[dtype]).to(DEV)
    want = np.stack([h, -h]) / 4 * gain.astype(np.float64)
    twice = np.float32(want).astype(np.float64)        # what a first rounding to fp32 makes of them
    if out == "y8":
        y8 = A.Blocks8.empty(2, d, DEV)
        A.adloco_rms_norm(ctx, x, torch.from_numpy(gain).to(DEV), 2.0**-126, y8=y8)
        codes, exps = codes_of(y8)
        right, other = lo.pack(want), lo.pack(twice)
        np.testing.assert_array_equal(exps, right[1])
        np.testing.assert_array_equal(codes, right[0])
        assert (right[0] != other[0]).sum() >= 8       # (the inputs tell one from the other)
    else:
        y = torch.empty_like(x)
        A.adloco_rms_norm(ctx, x, torch.from_numpy(gain).to(DEV), 2.0**-126, y=y)

        def rounded(v):
            step = np.exp2(np.floor(np.log2(np.abs(v))) - bits)
            return np.rint(v / step) * step
        np.testing.assert_array_equal(host(y), rounded(want))
        assert (rounded(want) != rounded(twice)).sum() >= 8


# ---- backward -------------------------------------------------------------------------------
# u = 2^-24.  A sum over a row is 64 terms in a row and 8 in a tree, all its terms are off by three roundings: with n and r off by
# six each, w - n mean(w n) is off by 90 u (|w| + |n| mean|w n|) at most (the bound of ordinary rows, 80 u, and the scales').

BACK_TOL = 90 * U


def backward(ctx, h, gain, dy, eps, dtype=torch.float32):
    h, dy = (torch.from_numpy(np.asarray(v, np.float32)).to(dtype).to(DEV) for v in (h, dy))
    g = None if gain is None else torch.from_numpy(np.asarray(gain, np.float32)).to(DEV)
    dh, sums = torch.empty_like(h), torch.empty(h.shape, device=DEV)
    A.adloco_rms_norm_backward(ctx, h, g, dy, eps, dh, gain_sums=sums)
    hh, yy, gg = host(h), host(dy), np.ones(h.shape[1]) if g is None else host(g)
    grad, parts = lo.rms_norm_backward(hh, gg, yy, eps)
    r = 1 / np.sqrt((hh * hh).mean(1, keepdims=True) + eps)
    n, w = hh * r, gg * yy
    assert np.abs(grad).max() < 1e38 and np.abs(parts).max() < 1e38    # (the gradients are finite)
    half = torch.finfo(dtype).eps / 2
    tol = BACK_TOL * r * (np.abs(w) + np.abs(n) * np.abs(w * n).mean(1, keepdims=True))
    least = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    off = np.abs(host(dh) - grad)
    assert (off <= tol + half * np.abs(grad) * (1 + 1e-4) + least).all(), (off / tol).max(1)
    np.testing.assert_array_less(np.abs(host(sums) - parts), BACK_TOL * np.abs(parts) + 2.0**-148)
    return host(dh)


def normal(seed, *shape):
    return np.random.default_rng(seed).normal(size=shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [96, 771, 3000, 16384])
def test_backward_where_only_the_product_overflows(ctx, d, dtype):
    """Sums of h^2 within fp32, of w h beyond it."""
    h, dy = normal(1, 6, d), normal(2, 6, d)
    for i, (a, b) in enumerate([(1e15, 1e24), (1e10, 1e29), (1e15, 1e29), (3.0, 5e36), (1e2, 1e35), (1.0, 1.0)]):
        h[i] *= a
        dy[i] *= b
    h[5, ::3] = 0
    dy[0] = np.abs(dy[0]) * np.sign(h[0])              # every term of one sign
    backward(ctx, h, 1 + 0.1 * normal(3, d), dy, 1e-5, TYPES[dtype])


@pytest.mark.parametrize("d", [96, 3000])
def test_backward_of_large_rows_with_large_gradients(ctx, d):
    """h^2 beyond fp32 as well, with small, ordinary and large gradients, and terms that cancel."""
    h, dy = normal(4, 7, d), normal(5, 7, d)
    for i, (a, b) in enumerate([(1e25, 1e20), (1e30, 1e36), (5e37, 1.0), (1e22, 1e-10), (3e19, 1e18), (1e37, 1e-3)]):
        h[i] *= a
        dy[i] *= b
    dy[4, d // 2:] = -dy[4, :d // 2]
    h[4, d // 2:] = h[4, :d // 2]
    backward(ctx, h, None, dy, 1e-5)


@pytest.mark.parametrize("d", [96, 3000])
def test_backward_of_small_rows_with_a_small_eps(ctx, d):
    """Products of w and h below fp32, of w and n within it."""
    h, dy = normal(6, 6, d), normal(7, 6, d)
    for i, (a, b) in enumerate([(1e-17, 1e-24), (1e-16, 1e-28), (1e-18, 1e-10), (1e-18, 1.0), (1e-17, 1e-20)]):
        h[i] *= a
        dy[i] *= b
    h[4], dy[5] = 0, 0
    got = backward(ctx, h, 1 + 0.1 * normal(8, d), dy, 2e-38)
    assert not got[5].any()


@pytest.mark.parametrize("d", [8192, 16384])
def test_eps_counts_beside_large_rows(ctx, d):
    """eps 1e30 beside the smallest mean squares whose sum leaves fp32, 2.6e34 to 7.7e34: it moves the root by 100 to 300 u."""
    h = np.sign(normal(9, 3, d)) * np.sqrt(4.3e38 / d) * np.array([[1.0], [1.1], [1.2]])
    backward(ctx, h, None, normal(10, 3, d) * 1e10, 1e30)


# ---- gain sums of long samples ----------------------------------------------------------------
# A run of L rows is added up in pieces of p rows, p the power of two from 256 on whose square reaches L, the runs' sums in
# sixteen parts: with values of one sign the sum is off by (p + L / p + runs / 16 + 16) u of itself, and 8 u for n and the products.

def sums_of_one_sign(ctx, T, d, dtype, runs):
    h = torch.ones(T, d, dtype=dtype, device=DEV)
    h[:, 1::2] = -1
    dy = torch.full((T, d), 0.1, dtype=dtype, device=DEV)
    sums = torch.full((1, d), 9.0, device=DEV)
    A.adloco_rms_norm_backward(ctx, h, None, dy, 1e-5, gain_sums=sums)
    L, piece = -(-T // runs), 256
    while piece * piece < L:
        piece *= 2
    want = T * float(dy[0, 0]) / np.sqrt(1 + 1e-5)
    off = np.abs(host(sums)[0] * np.where(np.arange(d) % 2, -1, 1) - want)
    assert off.max() <= (piece + L / piece + runs / 16 + 24) * U * want, off.max() / want
    again = torch.empty_like(sums)
    A.adloco_rms_norm_backward(ctx, h, None, dy, 1e-5, gain_sums=again)
    assert torch.equal(again, sums)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", [(255, 8), (256, 9), (257, 8), (512, 24), (513, 8), (131149, 24), (70000, 1030), (66000, 8200)])
def test_gain_sums_in_one_run(T, d, dtype):
    """Without memory for scratch a sample is one run."""
    ctx = A.Context(0)
    ctx.set_tuning("scratch_limit_kb", 1)
    sums_of_one_sign(ctx, T, d, TYPES[dtype], 1)
    ctx.close()


@pytest.mark.parametrize("T,d,waves", [((1 << 20) + 3, 520, 2), ((1 << 21) + 5, 2056, 8)])
def test_gain_sums_of_a_long_sample(ctx, T, d, waves):
    sums_of_one_sign(ctx, T, d, torch.bfloat16, 256 * (16 if d <= 1024 else 8) // waves)
