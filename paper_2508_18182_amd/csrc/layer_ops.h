// Device arithmetic shared by the layer operators: rows of eight values, the dropout mask, 8-bit blocks.
#pragma once

#include <type_traits>

#include "common.h"

namespace adloco {

// Number of a workgroup in a grid of launch_grid.
__device__ __forceinline__ long long launch_index() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// ---- eight consecutive values of a row -----------------------------------------------------------------------------
// FAST: rows are 16-byte aligned and whole multiples of eight long, so that a lane's eight are all there or all not.
// Others are loaded eight at a time all the same, at element alignment: the last ones of a row as the last eight, moved down
// when they are used (as the fetched values are not needed yet, nothing waits here).  Loaded and stored singly, those few took
// as long as all the others: 32768 x 1023 bf16, dropout 78 / 45 us, norm 98 / 64, its backward 103 / 56, packing 62 / 32.
template <typename E> using eight = E __attribute__((ext_vector_type(8)));
template <typename E, bool FAST> __device__ __forceinline__ eight<E> fetch_eight(const E* row, int c, int d) {
  eight<E> r = {};
  if constexpr (FAST) {
    if (c < d) r = __builtin_nontemporal_load(reinterpret_cast<const eight<E>*>(row + c));
  } else if (d >= 8) {
    __builtin_memcpy(&r, row + (c < d - 8 ? c : d - 8), sizeof r);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < d) r[j] = row[c + j];
  }
  return r;
}
// The fetched values in fp32, zeros behind the last column.
template <typename E, bool FAST> __device__ __forceinline__ void widen_eight(const eight<E>& r, int c, int d, float (&v)[8]) {
  if constexpr (FAST) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = float(r[j]);
  } else {
    constexpr int words = 2 * sizeof(E);               // 32-bit words, two or one values each
    typedef __attribute__((ext_vector_type(words))) unsigned raw;
    raw w = __builtin_bit_cast(raw, r);
    const int down = d >= 8 && c > d - 8 ? c - (d - 8) : 0;
    if (down) {                                        // (most waves have no such lane)
#pragma unroll
      for (int by = 4; by >= int(4 / sizeof(E)); by >>= 1) {
        const int step = by * int(sizeof(E)) / 4;
#pragma unroll
        for (int j = 0; j < words; ++j) w[j] = (down & by) ? (j + step < words ? w[j + step] : 0u) : w[j];
      }
      if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int j = 0; j < words; ++j) w[j] = (down & 1) ? w[j] >> 16 | (j + 1 < words ? w[j + 1] << 16 : 0u) : w[j];
      }
    }
    const eight<E> o = __builtin_bit_cast(eight<E>, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = down < 8 ? float(o[j]) : 0.f;
  }
}
template <typename E, bool FAST> __device__ __forceinline__ void load_eight(const E* row, int c, int d, float (&v)[8]) {
  widen_eight<E, FAST>(fetch_eight<E, FAST>(row, c, d), c, d, v);
}
template <typename E, bool FAST> __device__ __forceinline__ void store_eight(E* row, int c, int d, const float (&v)[8]) {
  eight<E> r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = E(v[j]);
  if constexpr (FAST) {
    if (c < d) __builtin_nontemporal_store(r, reinterpret_cast<eight<E>*>(row + c));
  } else if (c <= d - 8) {                             // (d may be 2^31 - 1: c + 8 would overflow)
    __builtin_memcpy(row + c, &r, sizeof r);
  } else if (c < d) {                                  // four, two and one of them
    const int n = d - c;
    E* to = row + c;
    if (n & 4) __builtin_memcpy(to, &r, 4 * sizeof(E));
    if (n & 2) {
      const E two[2] = {(n & 4) ? r[4] : r[0], (n & 4) ? r[5] : r[1]};
      __builtin_memcpy(to + (n & 4), two, sizeof two);
    }
    if (n & 1) to[n & 6] = (n & 4) ? ((n & 2) ? r[6] : r[4]) : ((n & 2) ? r[2] : r[0]);
  }
}

// ---- dropout -------------------------------------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 x 32 -> 64 bit products each turn a counter and a key into 128 random bits.  Eight columns of a row take one counter
// (column / 8, row, row >> 32, 0) and 16 bits each: the mask of an element depends on its row number and column alone,
// whatever the launch, so that it is formed again in the backward pass and never stored.  16 bits instead of 32 halve the
// integer work, which otherwise takes longer than the memory traffic of a 16-bit tensor.
struct DropoutArgs {
  unsigned k0, k1;           // key: the seed
  unsigned threshold;        // dropped below it; 0: no dropout
  float scale;               // 65536 / (65536 - threshold)
  unsigned long long first_row;
};
__device__ __forceinline__ void drop_eight(const DropoutArgs& m, long long row, int c, float (&v)[8]) {
  const unsigned long long r = m.first_row + (unsigned long long)row;
  unsigned c0 = unsigned(c) >> 3, c1 = unsigned(r), c2 = unsigned(r >> 32), c3 = 0;
  unsigned k0 = m.k0, k1 = m.k1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = unsigned(p1 >> 32) ^ c1 ^ k0;
    c1 = unsigned(p1);
    c2 = unsigned(p0 >> 32) ^ c3 ^ k1;
    c3 = unsigned(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  const unsigned w[4] = {c0, c1, c2, c3};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned u = (j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu;
    v[j] = u < m.threshold ? 0.f : v[j] * m.scale;        // (selected, not multiplied: a dropped NaN is gone)
  }
}

// ---- 8-bit blocks --------------------------------------------------------------------------------------------------
// Magnitudes are compared as bits: their order is that of the numbers, with infinities and NaN above them all, so that one
// maximum serves both the exponent and the question whether a block holds any of those.
constexpr unsigned kNotFinite = 0x7f800000u;
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
// Largest magnitude of eight values; FINITE: infinities and NaN, which have no say in a block's exponent, left out.
template <bool FINITE> __device__ __forceinline__ unsigned largest(const float (&v)[8]) {
  unsigned big = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned m = magnitude(v[j]);
    big = larger(big, FINITE && m >= kNotFinite ? 0u : m);
  }
  return big;
}
// Biased exponent of the smallest power of two s >= 2^-126 with x <= 448 s for the finite magnitude x of these bits,
// 448 = 1.75 * 2^8 the largest e4m3 value: read off the bits, hence exact.
__device__ __forceinline__ unsigned block_exponent(unsigned big) {
  const int e = int(big >> 23) - 8 + ((big & 0x7fffffu) > 0x600000u ? 1 : 0);
  return unsigned(e < 1 ? 1 : e);
}
// Four values over the block's power of two (exact) to e4m3, round to nearest even: at most half a step, 2^-4 of a value
// that is not below 2^-6.  The largest is 448 by the choice of the exponent, so that nothing saturates.
__device__ __forceinline__ unsigned pack_four(float a, float b, float c, float d, unsigned exponent) {
  typedef __attribute__((ext_vector_type(2))) short i16x2;
  const float s = __uint_as_float(exponent << 23);
  i16x2 w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, s, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, s, true);
  return __builtin_bit_cast(unsigned, w);
}
// Values that are not finite become NaN (e4m3 has no infinity).
__device__ __forceinline__ void mark_four(float a, float b, float c, float d, unsigned& o) {
  if (magnitude(a) >= kNotFinite) o |= 0x7fu;
  if (magnitude(b) >= kNotFinite) o |= 0x7f00u;
  if (magnitude(c) >= kNotFinite) o |= 0x7f0000u;
  if (magnitude(d) >= kNotFinite) o |= 0x7f000000u;
}
__device__ __forceinline__ uint2 pack_eight(const float (&v)[8], unsigned exponent) {
  return make_uint2(pack_four(v[0], v[1], v[2], v[3], exponent), pack_four(v[4], v[5], v[6], v[7], exponent));
}
__device__ __forceinline__ void mark_eight(const float (&v)[8], uint2& o) {
  mark_four(v[0], v[1], v[2], v[3], o.x);
  mark_four(v[4], v[5], v[6], v[7], o.y);
}
// y, the fp32 rounding of y + rest, with its last bit set where something was rounded away (towards what it was): rounded
// once more to fewer bits, it gives what y + rest gives.  Without it, one value in 2^20 comes to lie just between two e4m3
// values by its first rounding, and goes a whole step the wrong way half the time.  An infinite or NaN y (whose
// rest is not finite either) stays what it is.
__device__ __forceinline__ float round_to_odd(float y, float rest) {
  const unsigned u = __float_as_uint(y);
  const int towards = int((__float_as_uint(rest) ^ u)) >> 31 | 1;        // away from zero: 1, towards it: -1
  constexpr int finite = 0x198;                         // class of rest: normal or subnormal, of either sign, and not zero
  const bool cut = __builtin_amdgcn_classf(rest, finite) && (u & 1u) == 0u && (u & 0x7fffffffu) != 0u;
  return __uint_as_float(cut ? u + unsigned(towards) : u);
}
// Maximum over groups of 16 lanes, in all of them.  All lanes of a group have to be there.
__device__ __forceinline__ unsigned max16(unsigned v) {
#define ADLOCO_ROR_MAX(n) v = larger(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x120 + n, 0xf, 0xf, false)))
  ADLOCO_ROR_MAX(8);
  ADLOCO_ROR_MAX(4);
  ADLOCO_ROR_MAX(2);
  ADLOCO_ROR_MAX(1);
#undef ADLOCO_ROR_MAX
  return v;
}
// Biased exponent of the block that 16 lanes hold eight values each of.  any (the same for the wave): some value of the wave
// is not finite.
__device__ __forceinline__ unsigned row_block(const float (&v)[8], bool& any) {
  unsigned big = max16(largest<false>(v));
  any = __builtin_amdgcn_ballot_w64(big >= kNotFinite) != 0;
  if (any) big = max16(largest<true>(v));
  return block_exponent(big);
}
__device__ __forceinline__ float sum64(float v) {
#define ADLOCO_ROR_ADD(n) \
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + n, 0xf, 0xf, false))
  ADLOCO_ROR_ADD(8);
  ADLOCO_ROR_ADD(4);
  ADLOCO_ROR_ADD(2);
  ADLOCO_ROR_ADD(1);
#undef ADLOCO_ROR_ADD
  v += __shfl_xor(v, 16, 64);
  v += __shfl_xor(v, 32, 64);
  return v;
}

// The same in fp64.
__device__ __forceinline__ double sum64(double v) {
  auto ror = [](double x, auto n) {
    const unsigned long long u = __double_as_longlong(x);
    const unsigned lo = __builtin_amdgcn_update_dpp(0, int(unsigned(u)), 0x120 + decltype(n)::value, 0xf, 0xf, false);
    const unsigned hi = __builtin_amdgcn_update_dpp(0, int(unsigned(u >> 32)), 0x120 + decltype(n)::value, 0xf, 0xf, false);
    return __longlong_as_double((unsigned long long)hi << 32 | lo);
  };
  v += ror(v, std::integral_constant<int, 8>{});
  v += ror(v, std::integral_constant<int, 4>{});
  v += ror(v, std::integral_constant<int, 2>{});
  v += ror(v, std::integral_constant<int, 1>{});
  v += __shfl_xor(v, 16, 64);
  v += __shfl_xor(v, 32, 64);
  return v;
}

// ---- host side -----------------------------------------------------------------------------------------------------
// The context's device made current for a call, the caller's restored behind it.
class DeviceScope {
 public:
  explicit DeviceScope(const adloco_ctx* ctx) {
    int now = -1;
    if (hipGetDevice(&now) == hipSuccess && now != ctx->device) {
      before_ = now;
      ok_ = hipSetDevice(ctx->device) == hipSuccess;
    }
  }
  ~DeviceScope() {
    if (before_ >= 0) (void)hipSetDevice(before_);
  }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  bool ok() const { return ok_; }

 private:
  int before_ = -1;
  bool ok_ = true;
};

// Grid of n workgroups: a launch holds fewer than 2^32 work items in a dimension, so many small workgroups take a second one.
// The last ones, from launch_index() >= n on, have nothing to do.
inline dim3 launch_grid(long long n, int threads) {
  const long long most = 0xffffffffLL / threads, y = (n + most - 1) / most;
  return y <= 1 ? dim3(unsigned(n)) : dim3(unsigned((n + y - 1) / y), unsigned(y));
}

// One matrix argument as the checks see it: `rows` rows of `width` bytes, `stride` bytes apart.
struct RowSpan {
  const void* p;
  long long rows, width, stride;
  bool same(const RowSpan& o) const { return p == o.p && (stride == o.stride || rows <= 1); }
};
// Whether its size fits the arithmetic of addresses.
inline bool span_in_reach(long long rows, long long stride) { return rows <= 1 || stride <= (1LL << 56) / rows; }
// Whether two of them may share a byte.  Column ranges of one buffer (equal strides) do not.
inline bool spans_overlap(const RowSpan& x, const RowSpan& y) {
  if (!x.p || !y.p || x.rows <= 0 || y.rows <= 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
  const uintptr_t ae = a + uintptr_t((x.rows - 1) * x.stride + x.width), be = b + uintptr_t((y.rows - 1) * y.stride + y.width);
  if (ae <= b || be <= a) return false;
  if (x.stride != y.stride || x.stride <= 0) return true;
  const uintptr_t s = uintptr_t(x.stride), off = a <= b ? (b - a) % s : (s - (a - b) % s) % s;   // of y's rows within x's
  return off < uintptr_t(x.width) || s - off < uintptr_t(y.width);
}

// Scratch of the layer operators: one block of a fixed size, taken by the first call that needs it and never moved, so
// that captured calls keep it.  NULL if there is none and the stream is being captured, or there is no memory.
constexpr size_t kLayerScratch = size_t(64) << 20;
inline float* layer_scratch(adloco_ctx* ctx, hipStream_t st) {
  return obtain_scratch(ctx, ctx->layer_part, kLayerScratch, st) ? static_cast<float*>(ctx->layer_part.ptr) : nullptr;
}
const char* check_blocks8(const adloco_blocks8* b);

}  // namespace adloco
