// 8-bit blocks: packing of a matrix along its rows and / or across them, and the product of two packed matrices on the
// scaled matrix instructions.
#include "layer_ops.h"

namespace adloco {

const char* check_blocks8(const adloco_blocks8* b) {
  if (b->rows < 0 || b->cols < 1 || b->rows > 0x7fffffffLL || b->cols > 0x7fffff80LL) return "rows or cols out of range";
  const int64_t wide = (b->cols + 127) / 128 * 128;
  if (b->rows > 0 && (!b->data || !b->exponent)) return "data or exponent is NULL";
  if (reinterpret_cast<uintptr_t>(b->data) % 16 || reinterpret_cast<uintptr_t>(b->exponent) % 16)
    return "data and exponent must be 16-byte aligned";
  if (b->row_stride < wide || b->row_stride % 16 || b->row_stride > (int64_t(1) << 40))
    return "row_stride must hold whole blocks of 128 and be a multiple of 16";
  if (b->exponent_stride < b->rows || b->exponent_stride % 16 || b->exponent_stride > (int64_t(1) << 40))
    return "exponent_stride must be a multiple of 16 and at least rows";
  return nullptr;
}

namespace {

// ---------------------------------------------------------------------------------------------------------------------
// Packing.  A workgroup takes 128 x 128 values, a lane 8 x 8 of them in registers: blocks along the rows are 16 lanes of a
// row, blocks across them the 16 groups of eight rows.  x is read once whichever of the two outputs are asked for; the
// transposed one goes through LDS, so that both are stored in whole lines.
// ---------------------------------------------------------------------------------------------------------------------
struct PackArgs {
  const void* x;
  long long xs;
  long long rows, cols;
  unsigned char *q, *e, *qt, *et;      // along the rows, across them; NULL: not asked for
  long long qs, es, qts, ets;
  unsigned col_tiles;
};

template <typename E, bool FAST> __global__ __launch_bounds__(256) void pack_blocks_kernel(PackArgs a) {
  __shared__ float big_lds[4][128];
  __shared__ uint2 turn[128][16];
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const long long rt = blockIdx.x / a.col_tiles, ct = blockIdx.x - rt * a.col_tiles;
  const long long r0 = rt * 128 + rg * 8, c0 = ct * 128;
  const int left = int(a.cols - c0 < 128 ? a.cols - c0 : 128);
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (r0 + i < a.rows) {
      load_eight<E, FAST>(static_cast<const E*>(a.x) + (r0 + i) * a.xs + c0, cg * 8, left, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
  }
  if (a.q) {
    unsigned long long exps = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float big = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) big = fmaxf(big, finite_abs(v[i][j]));
      const unsigned e = block_exponent(max16(big));
      exps |= (unsigned long long)e << (8 * i);
      if (r0 + i < a.rows) *reinterpret_cast<uint2*>(a.q + (r0 + i) * a.qs + c0 + cg * 8) = pack_eight(v[i], block_inverse(e));
    }
    if (cg == 0) {
      unsigned char* p = a.e + ct * a.es + r0;
      if (r0 + 8 <= a.rows) *reinterpret_cast<unsigned long long*>(p) = exps;
      else
        for (int i = 0; r0 + i < a.rows; ++i) p[i] = (unsigned char)(exps >> (8 * i));
    }
  }
  if (!a.qt) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = fmaxf(big, finite_abs(v[i][j]));
    big = fmaxf(big, __shfl_xor(big, 16, 64));
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    if ((threadIdx.x & 63) < 16) big_lds[threadIdx.x >> 6][cg * 8 + j] = big;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = cg * 8 + j;
    const unsigned e = block_exponent(fmaxf(fmaxf(big_lds[0][c], big_lds[1][c]), fmaxf(big_lds[2][c], big_lds[3][c])));
    float col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) col[i] = v[i][j];
    turn[c][rg ^ (c & 15)] = pack_eight(col, block_inverse(e));
    if (rg == 0 && c0 + c < a.cols) a.et[rt * a.ets + c0 + c] = (unsigned char)e;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = i * 16 + rg;
    if (c < left) *reinterpret_cast<uint2*>(a.qt + (c0 + c) * a.qts + rt * 128 + cg * 8) = turn[c][cg ^ (c & 15)];
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Product.  out[m][n] = sum_k 2^(ea[k / 128][m] - 127) 2^(eb[k / 128][n] - 127) a[m][k] b[n][k]: both operands hold k
// contiguously.  One v_mfma_scale_f32_16x16x128 multiplies 16 rows by 16 columns over one block of 128 and applies the two
// powers of two by itself; products are exact, sums in fp32.  Which 32 of the 128 values of k a lane holds does not matter
// as long as both operands agree; which 16 rows make a block of the tile is free too, and a lane takes neighbouring rows
// for the blocks (row = lane * MB + block), so that their exponents are one load and a lane's outputs of a row one store.
// ---------------------------------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) int mfma_i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

struct ProductArgs {
  const unsigned char *a, *b, *ea, *eb;
  long long as, bs, eas, ebs;
  void* out;
  long long os;
  int M, N, steps;             // steps: blocks of k
  int tiles_n;
  int accumulate;
};

template <typename E> __device__ __forceinline__ void put_out(E* p, float v, bool accumulate) {
  if constexpr (std::is_same<E, float>::value) *p = accumulate ? *p + v : v;
  else *p = E(v);
}

constexpr int kProductTile = 128;

template <typename E> __global__ __launch_bounds__(256) void product_kernel(ProductArgs p) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][kProductTile * 128];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int l16 = lane & 15, kg = lane >> 4;
  const long long m0 = (long long)(blockIdx.x / p.tiles_n) * kProductTile, n0 = (long long)(blockIdx.x % p.tiles_n) * kProductTile;
  const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  mfma_f32x4 acc[4][4] = {};
  const long long ra = m0 + wm + l16 * 4 < p.M ? m0 + wm + l16 * 4 : 0, rb = n0 + wn + l16 * 4 < p.N ? n0 + wn + l16 * 4 : 0;
  for (int s = 0; s < p.steps; ++s) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (tid >> 3) + i * 32, ch = tid & 7;
      const long long am = m0 + r < p.M ? m0 + r : p.M - 1, bn = n0 + r < p.N ? n0 + r : p.N - 1;
      const int at = r * 128 + ((ch ^ ((r >> 2) & 7)) * 16);
      *reinterpret_cast<i32x4*>(lds[0] + at) = *reinterpret_cast<const i32x4*>(p.a + am * p.as + (long long)s * 128 + ch * 16);
      *reinterpret_cast<i32x4*>(lds[1] + at) = *reinterpret_cast<const i32x4*>(p.b + bn * p.bs + (long long)s * 128 + ch * 16);
    }
    const int ea = *reinterpret_cast<const int*>(p.ea + s * p.eas + ra), eb = *reinterpret_cast<const int*>(p.eb + s * p.ebs + rb);
    __syncthreads();
    mfma_i32x8 fa[4], fb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = wm + l16 * 4 + i, y = wn + l16 * 4 + i;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const i32x4 u = *reinterpret_cast<const i32x4*>(lds[0] + x * 128 + (((kg * 2 + h) ^ ((x >> 2) & 7)) * 16));
        const i32x4 w = *reinterpret_cast<const i32x4*>(lds[1] + y * 128 + (((kg * 2 + h) ^ ((y >> 2) & 7)) * 16));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          fa[i][h * 4 + j] = u[j];
          fb[i][h * 4 + j] = w[j];
        }
      }
    }
#define ADLOCO_STEP(m, n) \
  acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[m], fb[n], acc[m][n], 0, 0, m, ea, n, eb)
#define ADLOCO_ROW(m) ADLOCO_STEP(m, 0); ADLOCO_STEP(m, 1); ADLOCO_STEP(m, 2); ADLOCO_STEP(m, 3)
    ADLOCO_ROW(0); ADLOCO_ROW(1); ADLOCO_ROW(2); ADLOCO_ROW(3);
#undef ADLOCO_ROW
#undef ADLOCO_STEP
  }
  E* out = static_cast<E*>(p.out);
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long r = m0 + wm + (kg * 4 + j) * 4 + m;
      if (r >= p.M) continue;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const long long c = n0 + wn + l16 * 4 + n;
        if (c < p.N) put_out(out + r * p.os + c, acc[m][n][j], p.accumulate != 0);
      }
    }
}

size_t size_of(int dtype) { return is_16bit(dtype) ? 2 : 4; }

template <typename E, bool FAST> hipError_t launch_pack(const PackArgs& a, unsigned blocks, hipStream_t st) {
  hipLaunchKernelGGL((pack_blocks_kernel<E, FAST>), dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename E> hipError_t launch_product(const ProductArgs& a, unsigned blocks, hipStream_t st) {
  hipLaunchKernelGGL((product_kernel<E>), dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

RowSpan values_of(const adloco_blocks8* b) {
  return RowSpan{b ? b->data : nullptr, b ? b->rows : 0, b ? (b->cols + 127) / 128 * 128 : 0, b ? b->row_stride : 0};
}
RowSpan exponents_of(const adloco_blocks8* b) {
  return RowSpan{b ? b->exponent : nullptr, b ? (b->cols + 127) / 128 : 0, b ? b->rows : 0, b ? b->exponent_stride : 0};
}

}  // namespace
}  // namespace adloco

using namespace adloco;

extern "C" int adloco_pack_blocks(adloco_ctx* ctx, const void* x, int64_t x_row_stride, int64_t rows, int64_t cols, int dtype,
                                  const adloco_blocks8* along, const adloco_blocks8* across, void* stream) {
  if (!ctx) return ADLOCO_EINVAL;
  if (dtype != ADLOCO_F32 && !is_16bit(dtype)) return fail(ctx, ADLOCO_EUNSUPPORTED, "pack_blocks: dtype %d not supported", dtype);
  if (rows < 0 || cols < 0 || rows > 0x7fffff80LL || cols > 0x7fffff80LL)
    return fail(ctx, ADLOCO_EINVAL, "pack_blocks: rows = %lld, cols = %lld", (long long)rows, (long long)cols);
  if (!along && !across) return fail(ctx, ADLOCO_EINVAL, "pack_blocks: there is no output");
  if (rows == 0 || cols == 0) return ADLOCO_OK;
  if (along) {
    if (const char* why = check_blocks8(along)) return fail(ctx, ADLOCO_EINVAL, "pack_blocks: along: %s", why);
    if (along->rows != rows || along->cols != cols) return fail(ctx, ADLOCO_EINVAL, "pack_blocks: along is not of rows x cols values");
  }
  if (across) {
    if (const char* why = check_blocks8(across)) return fail(ctx, ADLOCO_EINVAL, "pack_blocks: across: %s", why);
    if (across->rows != cols || across->cols != rows) return fail(ctx, ADLOCO_EINVAL, "pack_blocks: across is not of cols x rows values");
  }
  const size_t es = size_of(dtype);
  const int64_t xs = x_row_stride ? x_row_stride : cols;
  if (!x || xs < cols || xs > (int64_t(1) << 40) || reinterpret_cast<uintptr_t>(x) % es)
    return fail(ctx, ADLOCO_EINVAL, "pack_blocks: x is NULL or misaligned, or its row stride is smaller than the row or out of range");
  const RowSpan s[5] = {{x, rows, (long long)(cols * es), (long long)(xs * es)}, values_of(along), exponents_of(along),
                        values_of(across), exponents_of(across)};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (spans_overlap(s[i], s[j])) return fail(ctx, ADLOCO_EINVAL, "pack_blocks: two arguments overlap");
  const int64_t rt = (rows + 127) / 128, ct = (cols + 127) / 128;
  if (rt * ct > 0x7fffffffLL) return fail(ctx, ADLOCO_EUNSUPPORTED, "pack_blocks: too many values for one launch");
  PackArgs a{};
  a.x = x;
  a.xs = xs;
  a.rows = rows;
  a.cols = cols;
  a.col_tiles = unsigned(ct);
  if (along) {
    a.q = static_cast<unsigned char*>(along->data);
    a.e = along->exponent;
    a.qs = along->row_stride;
    a.es = along->exponent_stride;
  }
  if (across) {
    a.qt = static_cast<unsigned char*>(across->data);
    a.et = across->exponent;
    a.qts = across->row_stride;
    a.ets = across->exponent_stride;
  }
  const bool fast = reinterpret_cast<uintptr_t>(x) % 16 == 0 && xs * (int64_t)es % 16 == 0 && cols % 8 == 0;
  DeviceScope scope(ctx);
  if (!scope.ok()) return fail(ctx, ADLOCO_EHIP, "pack_blocks: device %d cannot be made current", ctx->device);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const unsigned n = unsigned(rt * ct);
  hipEvent_t ev = prof_begin(ctx, st);
  hipError_t e;
  if (dtype == ADLOCO_BF16) e = fast ? launch_pack<__bf16, true>(a, n, st) : launch_pack<__bf16, false>(a, n, st);
  else if (dtype == ADLOCO_F16) e = fast ? launch_pack<_Float16, true>(a, n, st) : launch_pack<_Float16, false>(a, n, st);
  else e = fast ? launch_pack<float, true>(a, n, st) : launch_pack<float, false>(a, n, st);
  prof_end(ctx, kProfPack, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "pack_blocks launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}

extern "C" int adloco_block_product(adloco_ctx* ctx, const adloco_blocks8* a, const adloco_blocks8* b, void* out, int64_t out_row_stride,
                                    int dtype, uint32_t flags, void* stream) {
  if (!ctx) return ADLOCO_EINVAL;
  if (dtype != ADLOCO_F32 && !is_16bit(dtype)) return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: dtype %d not supported", dtype);
  if (!a || !b) return fail(ctx, ADLOCO_EINVAL, "block_product: a or b is NULL");
  if (flags & ~ADLOCO_ACCUMULATE) return fail(ctx, ADLOCO_EINVAL, "block_product: unknown flags");
  if ((flags & ADLOCO_ACCUMULATE) && dtype != ADLOCO_F32)
    return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: only an fp32 output accumulates");
  if (const char* why = check_blocks8(a)) return fail(ctx, ADLOCO_EINVAL, "block_product: a: %s", why);
  if (const char* why = check_blocks8(b)) return fail(ctx, ADLOCO_EINVAL, "block_product: b: %s", why);
  if (a->cols != b->cols) return fail(ctx, ADLOCO_EINVAL, "block_product: rows of a hold %lld values, of b %lld", (long long)a->cols, (long long)b->cols);
  if (a->rows == 0 || b->rows == 0) return ADLOCO_OK;
  const size_t es = size_of(dtype);
  const int64_t os = out_row_stride ? out_row_stride : b->rows;
  if (!out || os < b->rows || os > (int64_t(1) << 40) || reinterpret_cast<uintptr_t>(out) % es)
    return fail(ctx, ADLOCO_EINVAL, "block_product: out is NULL or misaligned, or its row stride is smaller than the row or out of range");
  const RowSpan so{out, a->rows, (long long)(b->rows * es), (long long)(os * es)};
  for (const adloco_blocks8* x : {a, b})
    if (spans_overlap(so, values_of(x)) || spans_overlap(so, exponents_of(x)))
      return fail(ctx, ADLOCO_EINVAL, "block_product: out overlaps an operand");
  const int64_t tm = (a->rows + kProductTile - 1) / kProductTile, tn = (b->rows + kProductTile - 1) / kProductTile;
  if (tm * tn > 0x7fffffffLL) return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: too many tiles for one launch");
  ProductArgs p{};
  p.a = static_cast<const unsigned char*>(a->data);
  p.b = static_cast<const unsigned char*>(b->data);
  p.ea = a->exponent;
  p.eb = b->exponent;
  p.as = a->row_stride;
  p.bs = b->row_stride;
  p.eas = a->exponent_stride;
  p.ebs = b->exponent_stride;
  p.out = out;
  p.os = os;
  p.M = int(a->rows);
  p.N = int(b->rows);
  p.steps = int((a->cols + 127) / 128);
  p.tiles_n = int(tn);
  p.accumulate = flags & ADLOCO_ACCUMULATE ? 1 : 0;
  DeviceScope scope(ctx);
  if (!scope.ok()) return fail(ctx, ADLOCO_EHIP, "block_product: device %d cannot be made current", ctx->device);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const unsigned n = unsigned(tm * tn);
  hipEvent_t ev = prof_begin(ctx, st);
  const hipError_t e = dtype == ADLOCO_BF16 ? launch_product<__bf16>(p, n, st)
                       : dtype == ADLOCO_F16 ? launch_product<_Float16>(p, n, st) : launch_product<float>(p, n, st);
  prof_end(ctx, kProfProduct, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "block_product launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}
