"""Products of 8-bit blocks whose largest terms cancel, in whole numbers: the sum of the others is what is left, and every
partial sum is below 2^24, so that exact products give the exact sum, rounded once."""
import numpy as np
import pytest
import torch

import paper_2508_18182_amd as A

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def cancelling(m, n, k, seed=0):
    """Whole numbers from -8 to 8, and up to three pairs of neighbouring columns with 448 * 448 - 448 * 448: (a, b, a b^T)."""
    r = np.random.default_rng(1000 * m + n + k + seed)
    a, b = r.integers(-8, 9, (m, k)).astype(np.float64), r.integers(-8, 9, (n, k)).astype(np.float64)
    for at in sorted({0, k // 2 // 2 * 2, (k - 2) // 2 * 2}):
        if at + 1 < k:
            a[:, at:at + 2], b[:, at], b[:, at + 1] = 448, 448, -448
    return a, b, a @ b.T


def blocks(v):
    b = A.Blocks8.empty(*v.shape, DEV)
    b.data.zero_()
    b.data[:, :v.shape[1]] = torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
    b.exponent.fill_(127)
    return b


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(1, 1, 2), (1, 70, 128), (3, 5632, 2048), (16, 33, 640), (17, 100, 300), (32, 4096, 1024)])
def test_few_rows(ctx, m, n, k, dtype):
    a, b, want = cancelling(m, n, k)
    ctx.set_tuning("product_blocks", 1)
    try:
        out = torch.full((m, n), float("nan"), dtype=TYPES[dtype], device=DEV)
        A.adloco_block_product(ctx, blocks(a), blocks(b), out)
    finally:
        ctx.set_tuning("product_blocks", 0)
    assert torch.equal(out.cpu(), torch.from_numpy(want).to(TYPES[dtype]))


@pytest.mark.parametrize("m,n,k", [(1, 5632, 2048), (3, 5632, 2048), (32, 8192, 4096)])
def test_few_rows_by_the_sizes(ctx, m, n, k):
    """The kernel that the library chooses for them."""
    a, b, want = cancelling(m, n, k, 1)
    out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    A.adloco_block_product(ctx, blocks(a), blocks(b), out)
    assert torch.equal(out.cpu(), torch.from_numpy(want).to(torch.bfloat16))


# (16 x 16 blocks per wave and side, pieces of the contraction); 0: the library's choice
@pytest.mark.parametrize("variant", [(0, 0), (1, 0), (4, 1), (4, 3), (8, 1), (8, 7)], ids=lambda v: f"{v[0]}x{v[1]}")
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(1, 1, 2), (20, 70, 300), (33, 129, 1000), (128, 128, 128), (130, 1000, 250), (300, 513, 4000), (257, 260, 9000)])
def test_by_request(ctx, m, n, k, dtype, variant):
    """ADLOCO_EXACT_PRODUCTS, whatever the kernel: rows that are aligned and rows that are not, nothing between them."""
    a, b, want = cancelling(m, n, k)
    ctx.set_tuning("product_blocks", variant[0])
    ctx.set_tuning("product_pieces", variant[1])
    try:
        for pad in (0, 3, 8):
            buf = torch.full((m, n + pad), 7.0, dtype=TYPES[dtype], device=DEV)
            A.adloco_block_product(ctx, blocks(a), blocks(b), buf[:, :n], A.ADLOCO_EXACT_PRODUCTS)
            assert torch.equal(buf[:, :n].cpu(), torch.from_numpy(want).to(TYPES[dtype]))
            assert bool((buf[:, n:] == 7).all())
        if dtype == "f32":
            out = torch.full((m, n), 5.0, device=DEV)
            A.adloco_block_product(ctx, blocks(a), blocks(b), out, A.ADLOCO_EXACT_PRODUCTS | A.ADLOCO_ACCUMULATE)
            assert torch.equal(out.cpu(), torch.from_numpy(want + 5).float())
    finally:
        ctx.set_tuning("product_blocks", 0)
        ctx.set_tuning("product_pieces", 0)


@pytest.mark.parametrize("m,n,k", [(4200, 4100, 1024), (65281, 256, 512)])
def test_large_outputs_by_request(ctx, m, n, k):
    a, b, _ = cancelling(m, n, k)
    out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    A.adloco_block_product(ctx, blocks(a), blocks(b), out, A.ADLOCO_EXACT_PRODUCTS)
    want = torch.from_numpy(a).to(DEV) @ torch.from_numpy(b).to(DEV).T.contiguous()
    assert torch.equal(out, want.to(torch.bfloat16))


@pytest.mark.parametrize("variant", [(4, 1), (4, 3), (8, 1), (8, 2)], ids=lambda v: f"{v[0]}x{v[1]}")
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(33, 129, 1000), (300, 260, 2000)])
def test_what_the_8_bit_instruction_leaves(ctx, m, n, k, dtype, variant):
    """Without it: each product is cut off below 2^-13 of the largest of a group of at most 32, so that a group is off by 32 times
    2^-13 of its largest product, and all of them by that of the sum of their largest ones: the pairs of 448 lie in six groups at
    most, every other group's products are 64 at most."""
    a, b, want = cancelling(m, n, k)
    ctx.set_tuning("product_blocks", variant[0])
    ctx.set_tuning("product_pieces", variant[1])
    try:
        out = torch.empty((m, n), dtype=TYPES[dtype], device=DEV)
        A.adloco_block_product(ctx, blocks(a), blocks(b), out)
    finally:
        ctx.set_tuning("product_blocks", 0)
        ctx.set_tuning("product_pieces", 0)
    largest = 6 * 448.0**2 + 64.0 * (-(-k // 128) * 128 // 32 * 4)              # (groups of eight at least)
    half = torch.finfo(TYPES[dtype]).eps / 2
    off = np.abs(out.cpu().double().numpy() - want)
    cut = 32 * 2.0**-13 * largest
    assert (off <= half * np.abs(want) + cut * (1 + half)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ea,eb,top", [(0, 200, 448), (1, 200, 448), (2, 230, 448), (3, 200, 448), (200, 1, 448), (246, 60, 448),
                                       (60, 246, 448), (247, 60, 240), (254, 20, 1.75), (3, 246, 448), (255, 127, 448)])
def test_few_rows_of_extreme_exponents(ctx, ea, eb, top, dtype):
    """fp32 sums of exact products of what the operands are in bf16: 2 k u of the sum of magnitudes (u = 2^-24), half a step of
    2^-133 for an operand below that, and the output's rounding."""
    m, n, k, dt = 20, 48, 200, TYPES[dtype]
    r = np.random.default_rng(ea + eb)
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = torch.nonzero(every.abs() <= top).flatten().to(torch.uint8)
    a, b = A.Blocks8.empty(m, k, DEV), A.Blocks8.empty(n, k, DEV)
    values = []
    for x, e in ((a, ea), (b, eb)):
        c = codes[torch.from_numpy(r.integers(0, len(codes), (x.rows, k)))]
        x.data.zero_()
        x.data[:, :k] = c.to(DEV)
        x.exponent.fill_(e)
        values.append(c.view(torch.float8_e4m3fn).double().numpy() * 2.0**(e - 127))
    av, bv = values
    out = torch.empty(m, n, dtype=dt, device=DEV)
    ctx.set_tuning("product_blocks", 1)
    try:
        A.adloco_block_product(ctx, a, b, out)
    finally:
        ctx.set_tuning("product_blocks", 0)
    if ea == 255:
        assert bool(out.isnan().all())
        return
    want, size = av @ bv.T, np.abs(av) @ np.abs(bv).T
    lost = 2.0**-134 * ((ea < 3) * np.abs(bv).sum(1)[None] + (eb < 3) * np.abs(av).sum(1)[:, None])
    half, least = torch.finfo(dt).eps / 2, torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    off = np.abs(out.cpu().double().numpy() - want)
    assert (off <= half * np.abs(want) + (lost + 2 * k * 2.0**-24 * size) * (1 + half) + least).all()
