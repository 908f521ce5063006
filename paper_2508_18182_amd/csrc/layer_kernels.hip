// Dropout and the root-mean-square norm of a transformer layer, forward and backward.  All of it is bound by memory: every
// input is read once and every output written once, rows stay in registers between the two passes that a norm makes.
#include <cmath>
#include <type_traits>

#include "layer_ops.h"

namespace adloco {
namespace {

// ---------------------------------------------------------------------------------------------------------------------
// out = residual + dropout(x).  One lane: eight columns of a row, one counter of the generator.  32768 x 1024 bf16 with a
// residual: 32 us, 6.3 TB/s; the generator's integer products hide behind the traffic.
// ---------------------------------------------------------------------------------------------------------------------
struct DropArgs {
  const void* x;
  const void* residual;      // or NULL
  void* out;
  long long xs, rs, os;      // row strides, elements
  long long rows, total;     // total: rows * per_row
  int d;
  unsigned per_row;          // groups of eight columns
  DropoutArgs m;
};

template <typename E, bool FAST> __global__ __launch_bounds__(64) void dropout_kernel(DropArgs a) {
  const long long i = launch_index() * 64 + threadIdx.x;
  if (i >= a.total) return;
  const long long row = a.total <= 0xffffffffLL ? unsigned(i) / a.per_row : i / a.per_row;
  const int c = int(i - row * a.per_row) * 8;
  float v[8], r[8];
  load_eight<E, FAST>(static_cast<const E*>(a.x) + row * a.xs, c, a.d, v);
  if (a.residual) load_eight<E, FAST>(static_cast<const E*>(a.residual) + row * a.rs, c, a.d, r);
  if (a.m.threshold) drop_eight(a.m, row, c, v);
  if (a.residual) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += r[j];
  }
  store_eight<E, FAST>(static_cast<E*>(a.out) + row * a.os, c, a.d, v);
}

// ---------------------------------------------------------------------------------------------------------------------
// h = residual + dropout(x);  y = h * rsqrt(mean(h^2) + eps) * gain, in the type of x and / or in 8-bit blocks.
// A row belongs to WAVES waves, a lane holds NV groups of eight columns of it in registers.  The statistics are of h in
// fp32, before it is rounded for the store.  Where the squares of a row leave fp32 (|h| > 1.8e19), they are formed again of
// 2^-96 h: a row of large finite values keeps its norm.  32768 x 2048 bf16 with residual, h, y and y8: 98 us, 6.2 TB/s;
// 5005 x 771 fp32, whose rows share no alignment: 13 us, 4.7 TB/s; one row: 3 us, four dependent trips to memory and back.
// ---------------------------------------------------------------------------------------------------------------------
struct NormArgs {
  const void* x;
  const void* residual;
  const float* gain;
  void* h;
  void* y;
  long long xs, rs, hs, ys;
  unsigned char* q;          // 8-bit blocks: values, row stride, width (whole blocks); NULL: none
  unsigned char* e;
  long long qs, es;
  long long rows;
  int d, wide;               // wide: d up to whole blocks where they are written, else d
  double inv_d, eps;
  DropoutArgs m;
};

constexpr float kLargest = 3.402823466e38f;       // the largest fp32 number
constexpr float kTiny = 1.262177448353619e-29f;   // 2^-96: 16384 squares of the largest fp32 number fit

// Sums over the row of a few values at once; `slot` alternates from row to row, so that one barrier is enough.
template <int WAVES, int N, typename F> __device__ __forceinline__ void row_sums(F (&s)[N], F (*lds)[8][N], int slot) {
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = sum64(s[k]);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) lds[slot][threadIdx.x >> 6][k] = s[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      s[k] = lds[slot][0][k];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s[k] += lds[slot][w][k];
    }
  }
}
// A lane's eight gains of one group; 0 behind the last column.
__device__ __forceinline__ void load_gain(const float* gain, int c, int d, bool vec, float (&g)[8]) {
  if (gain && vec && c + 8 <= d) {
    const float4 a = *reinterpret_cast<const float4*>(gain + c), b = *reinterpret_cast<const float4*>(gain + c + 4);
    g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w;
    g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = c + j >= d ? 0.f : gain ? gain[c + j] : 1.f;
}

template <typename E, int NV, int WAVES, bool FAST> __global__ __launch_bounds__(64 * WAVES) void rms_norm_kernel(NormArgs a) {
  __shared__ double lds[4][8][1];
  int slot = 0;
  const int c0 = threadIdx.x * 8;
  float g[NV][8];
  const bool gain_vec = reinterpret_cast<unsigned long long>(a.gain) % 16 == 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) load_gain(a.gain, c0 + i * 512 * WAVES, a.d, gain_vec, g[i]);
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float h[NV][8], r[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) load_eight<E, FAST>(static_cast<const E*>(a.x) + row * a.xs, c0 + i * 512 * WAVES, a.d, h[i]);
    if (a.residual)
#pragma unroll
      for (int i = 0; i < NV; ++i)
        load_eight<E, FAST>(static_cast<const E*>(a.residual) + row * a.rs, c0 + i * 512 * WAVES, a.d, r[i]);
    if (a.m.threshold)
#pragma unroll
      for (int i = 0; i < NV; ++i) drop_eight(a.m, row, c0 + i * 512 * WAVES, h[i]);
    if (a.residual)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += r[i][j];
    if (a.h)
#pragma unroll
      for (int i = 0; i < NV; ++i) store_eight<E, FAST>(static_cast<E*>(a.h) + row * a.hs, c0 + i * 512 * WAVES, a.d, h[i]);
    // One factor for the whole row, and 8-bit outputs that change by a whole step where a value lies next to the middle of two:
    // the sum over the lanes and the root are formed in fp64 (once per row), and the products with the root's and their own
    // rounding errors carried along, up to the one rounding of the output.
    auto squares = [&] {
      float q = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) q = fmaf(h[i][j], h[i][j], q);
      return q;
    };
    double s[1] = {squares()}, eps = a.eps;
    row_sums<WAVES, 1>(s, lds, slot++ & 3);
    if (!(s[0] <= 3.402823466e38)) {                // (the same for the whole row)
      eps *= double(kTiny) * kTiny;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] *= kTiny;
      s[0] = squares();
      row_sums<WAVES, 1>(s, lds, slot++ & 3);
    }
    const double root = rsqrt(s[0] * a.inv_d + eps);
    const float r_hi = float(root), r_lo = float(root - double(r_hi));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float odd[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (clamped: an infinite gain would make it infinite, of either sign, or NaN)
        const float n = h[i][j] * r_hi, error = fmaf(h[i][j], r_lo, fmaf(h[i][j], r_hi, -n));
        const float rest = __builtin_amdgcn_fmed3f(error * g[i][j], -kLargest, kLargest);
        h[i][j] = fmaf(n, g[i][j], rest);
        odd[j] = round_to_odd(h[i][j], fmaf(n, g[i][j], -h[i][j]) + rest);
      }
      const int c = c0 + i * 512 * WAVES;
      if (a.y) {
        if constexpr (std::is_same<E, float>::value) store_eight<E, FAST>(static_cast<E*>(a.y) + row * a.ys, c, a.d, h[i]);
        else store_eight<E, FAST>(static_cast<E*>(a.y) + row * a.ys, c, a.d, odd);
      }
      if (a.q) {
#pragma unroll
        for (int j = 0; j < 8; ++j) odd[j] = c + j < a.d ? odd[j] : 0.f;       // (in a row whose norm is not finite, 0 * NaN)
        bool any;
        const unsigned e = row_block(odd, any);
        if (c < a.wide) {
          uint2 o = pack_eight(odd, e);
          if (any) mark_eight(odd, o);
          *reinterpret_cast<uint2*>(a.q + row * a.qs + c) = o;
          if ((threadIdx.x & 15) == 0) a.e[(long long)(c >> 7) * a.es + row] = (unsigned char)e;
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Backward of the norm.  With r = rsqrt(mean(h^2) + eps), n = h r and w = gain dy:
//   dh = dh_in + r (w - n mean(w n)),  dx = dropout(dh),  gain_sums[sample] = sum_t dy n.
// Both sums of a row are formed in one pass, r again from h, which is here anyway.  A group of WAVES waves takes a run of one
// sample's rows in order and keeps its columns of sum dy n in registers; runs are added up in order by a second kernel.
// Rows whose sums leave fp32 make further passes over their registers.  A long run puts its sums into memory every `piece` rows,
// about the root of its length: rounding errors grow with that.
// 32768 x 1024 bf16 with dh_in and dropout, 32 samples: 66 us, 5.1 TB/s, and 4.5 us for the runs (8 MB written and read again);
// two rows ahead instead of one: the same (70.7 and 70.9 us in all), at 2048 columns worse (99 and 104).
// ---------------------------------------------------------------------------------------------------------------------
struct NormBackArgs {
  const void* h;
  const void* dy;
  const void* dh_in;
  const float* gain;
  void* dh;
  void* dx;
  float* sums;               // [samples][runs][d], or NULL
  long long hs, ys, is, os, xs;
  long long T;
  int runs;                  // per sample
  unsigned groups;           // samples * runs
  int piece;                 // rows that are added up in registers, a power of two
  int d;
  float inv_d, eps;
  DropoutArgs m;
};

template <typename E, int NV, int WAVES, bool FAST>
__global__ __launch_bounds__(64 * WAVES) void rms_norm_backward_kernel(NormBackArgs a) {
  __shared__ float lds[4][8][2];
  int slot = 0;
  const int c0 = threadIdx.x * 8;
  const unsigned group = unsigned(launch_index());
  if (group >= a.groups) return;
  const long long sample = group / unsigned(a.runs);
  const int run = int(group - sample * a.runs);
  const long long first = sample * a.T + a.T * run / a.runs, last = sample * a.T + a.T * (run + 1) / a.runs;
  float acc[NV][8], g[NV][8];
  const bool gain_vec = reinterpret_cast<unsigned long long>(a.gain) % 16 == 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    load_gain(a.gain, c0 + i * 512 * WAVES, a.d, gain_vec, g[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
  }
  // the next row is fetched behind the work on this one: two reductions and a store would expose its latency
  eight<E> rh[NV], ry[NV], ri[NV];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = c0 + i * 512 * WAVES;
      rh[i] = fetch_eight<E, FAST>(static_cast<const E*>(a.h) + row * a.hs, c, a.d);
      ry[i] = fetch_eight<E, FAST>(static_cast<const E*>(a.dy) + row * a.ys, c, a.d);
      if (a.dh_in) ri[i] = fetch_eight<E, FAST>(static_cast<const E*>(a.dh_in) + row * a.is, c, a.d);
    }
  };
  constexpr bool ahead = NV < 4;                    // (wider rows have no registers left for it)
  if (ahead && first < last) fetch(first);
  long long row = first;
  do {                                              // (once without a row: sums of nothing)
    const long long end = last - row < a.piece ? last : row + a.piece;
    for (; row < end; ++row) {
      if (!ahead) fetch(row);
      float h[NV][8], y[NV][8], in[NV][8];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        widen_eight<E, FAST>(rh[i], c0 + i * 512 * WAVES, a.d, h[i]);
        widen_eight<E, FAST>(ry[i], c0 + i * 512 * WAVES, a.d, y[i]);
        if (a.dh_in) widen_eight<E, FAST>(ri[i], c0 + i * 512 * WAVES, a.d, in[i]);
      }
      if (ahead && row + 1 < last) fetch(row + 1);
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s[0] = fmaf(h[i][j], h[i][j], s[0]);
          s[1] = fmaf(g[i][j] * y[i][j], h[i][j], s[1]);
        }
      row_sums<WAVES, 2>(s, lds, slot++ & 3);
      float r = rsqrtf(fmaf(s[0], a.inv_d, a.eps)), mean = s[1] * r * a.inv_d, out = r;
      // Sums that left fp32 (the same for the whole row).  w h may where w n does not: above it, or below it if r is large, when a
      // sum of 0 may be one of lost products.
      if (!(s[0] <= kLargest && fabsf(mean) <= kLargest && (r <= 1024.f || fabsf(s[1]) >= 0x1p-100f))) {
        const float down = fabsf(s[1]) < 1.f ? 1.f : 0x1p-24f;         // w may be as large as fp32, and |n| adds up to d
        if (!(s[0] <= kLargest)) {
          s[0] = s[1] = 0.f;
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              h[i][j] *= kTiny;
              s[0] = fmaf(h[i][j], h[i][j], s[0]);
            }
          row_sums<WAVES, 2>(s, lds, slot++ & 3);
          r = rsqrtf(fmaf(s[0], a.inv_d, float(double(a.eps) * (double(kTiny) * kTiny))));
          out = r * kTiny;
        }
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) s[1] = fmaf(g[i][j] * y[i][j] * down, h[i][j] * r, s[1]);
        row_sums<WAVES, 2>(s, lds, slot++ & 3);
        mean = s[1] * a.inv_d / down;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = c0 + i * 512 * WAVES;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float n = h[i][j] * r;
          acc[i][j] = fmaf(y[i][j], n, acc[i][j]);
          v[j] = out * fmaf(-n, mean, g[i][j] * y[i][j]);
          if (a.dh_in) v[j] += in[i][j];
        }
        if (a.dh) store_eight<E, FAST>(static_cast<E*>(a.dh) + row * a.os, c, a.d, v);
        if (a.dx) {
          if (a.m.threshold) drop_eight(a.m, row, c, v);
          store_eight<E, FAST>(static_cast<E*>(a.dx) + row * a.xs, c, a.d, v);
        }
      }
    }
    if (a.sums) {
      const bool more = end - first > a.piece;        // there are sums of the pieces before
      int at = c0;
      asm volatile("" : "+v"(at));                    // (addresses formed here: kept through the rows, they cost their registers)
      float* out = a.sums + (sample * a.runs + run) * a.d;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = at + i * 512 * WAVES + j;
          if (c < a.d) out[c] = more ? out[c] + acc[i][j] : acc[i][j];
          acc[i][j] = 0.f;
        }
    }
  } while (row < last);
}

// Adds up a sample's runs: 64 columns per workgroup, a sixteenth of the runs per wave in order, then the sixteen in order.
constexpr int kRunWaves = 16;
__global__ __launch_bounds__(64 * kRunWaves) void gain_runs_kernel(const float* parts, int runs, int d, int slabs, float* out) {
  __shared__ float lds[kRunWaves][64];
  const long long sample = blockIdx.x / slabs;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = int(blockIdx.x - sample * slabs) * 64 + lane, cc = c < d ? c : d - 1;
  const float* p = parts + sample * runs * d + cc;
  const int first = runs * wave / kRunWaves, last = runs * (wave + 1) / kRunWaves;
  float s = 0.f;
#pragma unroll 8
  for (int k = first; k < last; ++k) s += p[(long long)k * d];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave > 0 || c >= d) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < kRunWaves; ++k) s += lds[k][lane];
  out[sample * d + c] = s;
}

// ---------------------------------------------------------------------------------------------------------------------
bool known_dtype(int dtype) { return dtype == ADLOCO_F32 || is_16bit(dtype); }
size_t size_of(int dtype) { return is_16bit(dtype) ? 2 : 4; }
bool fast_rows(const void* p, long long stride, int d, size_t esize) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (long long)esize % 16 == 0 && d % 8 == 0);
}

// NULL if the mask is sound, else what is wrong with it.
const char* dropout_args(const adloco_dropout_mask* m, DropoutArgs& out) {
  out = DropoutArgs{0, 0, 0, 1.f, 0};
  if (!m) return nullptr;
  if (!(m->p >= 0.0) || !(m->p < 1.0)) return "p must be in [0, 1)";
  if (m->first_row < 0) return "first_row must not be negative";
  const double t = std::nearbyint(m->p * 65536.0);
  if (t > 65535.0) return "p rounds to 1 (steps of 2^-16)";
  out.k0 = unsigned(m->seed);
  out.k1 = unsigned(m->seed >> 32);
  out.threshold = unsigned(t);
  out.scale = float(65536.0 / (65536.0 - t));
  out.first_row = (unsigned long long)m->first_row;
  return nullptr;
}

// Row strides (0: d) of up to eight matrix arguments; false with the reason in the context.
struct Matrix {
  const char* name;
  const void* p;
  int64_t stride;
  bool written;
};
bool check_matrices(adloco_ctx* ctx, const char* who, Matrix* m, int n, int64_t rows, int32_t d, int dtype, bool& fast) {
  const size_t es = size_of(dtype);
  fast = true;
  for (int i = 0; i < n; ++i) {
    if (m[i].stride == 0) m[i].stride = d;
    if (!m[i].p) continue;
    if (m[i].stride < d || m[i].stride > (int64_t(1) << 40) || !span_in_reach(rows, m[i].stride * (int64_t)es)) {
      fail(ctx, ADLOCO_EINVAL, "%s: row stride of %s is smaller than the row or out of range", who, m[i].name);
      return false;
    }
    if (reinterpret_cast<uintptr_t>(m[i].p) % es) {
      fail(ctx, ADLOCO_EINVAL, "%s: %s is not aligned to its element size", who, m[i].name);
      return false;
    }
    fast = fast && fast_rows(m[i].p, m[i].stride, d, es);
  }
  auto span = [&](const Matrix& x) { return RowSpan{x.p, rows, (long long)(d * es), (long long)(x.stride * es)}; };
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j) {
      if (i == j || !m[i].written || !m[i].p || !m[j].p || (m[j].written && j < i)) continue;
      const RowSpan a = span(m[i]), b = span(m[j]);
      if (m[j].written ? spans_overlap(a, b) : !a.same(b) && spans_overlap(a, b)) {     // (in place: the very same rows)
        fail(ctx, ADLOCO_EINVAL, "%s: %s overlaps %s", who, m[i].name, m[j].name);
        return false;
      }
    }
  return true;
}

template <template <typename, bool> class F, typename... A> hipError_t by_type(int dtype, bool fast, A&&... args) {
  if (dtype == ADLOCO_BF16) return fast ? F<__bf16, true>::run(args...) : F<__bf16, false>::run(args...);
  if (dtype == ADLOCO_F16) return fast ? F<_Float16, true>::run(args...) : F<_Float16, false>::run(args...);
  return fast ? F<float, true>::run(args...) : F<float, false>::run(args...);
}

template <typename E, bool FAST> struct LaunchDropout {
  static hipError_t run(const DropArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((dropout_kernel<E, FAST>), launch_grid((a.total + 63) / 64, 64), dim3(64), 0, st, a);
    return hipGetLastError();
  }
};

// Waves per row and groups of eight columns per lane.  As many waves as the row fills: with 2048 columns on one wave (four
// groups a lane) the forward pass of 32768 rows takes 118 us, on two 101, on four 99.
constexpr int kNormWidth = 16384;
constexpr int norm_waves(int wide) { return wide <= 512 ? 1 : wide <= 1024 ? 2 : wide <= 2048 ? 4 : 8; }
#define ADLOCO_NORM_SHAPE(wide, CALL)         \
  do {                                        \
    if (wide <= 512) CALL(1, 1);              \
    else if (wide <= 1024) CALL(1, 2);        \
    else if (wide <= 2048) CALL(1, 4);        \
    else if (wide <= 4096) CALL(1, 8);        \
    else if (wide <= 8192) CALL(2, 8);        \
    else CALL(4, 8);                          \
  } while (0)

template <typename E, bool FAST> struct LaunchNorm {
  static hipError_t run(const NormArgs& a, hipStream_t st) {
    // Sixteen waves per compute unit, which all run at once; where that leaves a workgroup eight rows or more, four each, dealt out
    // as others end (at once / dealt out: 32768 x 2048 110 / 103 us, 32768 x 768 with dropout 51 / 46, one row each 107 / 49; at
    // five rows, 2500 x 5000, at once 26, dealt out 27).
    const long long most = (long long)kNumCu * 16 / norm_waves(a.wide);
    const long long groups = a.rows < most ? a.rows : a.rows < 8 * most ? most : (a.rows + 3) / 4;
    const long long limit = 0xffffffffLL / (64 * norm_waves(a.wide));      // (a launch holds fewer than 2^32 work items)
    const dim3 grid(unsigned(groups < limit ? groups : limit));
#define ADLOCO_CALL(NV, WAVES) hipLaunchKernelGGL((rms_norm_kernel<E, NV, WAVES, FAST>), grid, dim3(64 * WAVES), 0, st, a)
    ADLOCO_NORM_SHAPE(a.wide, ADLOCO_CALL);
#undef ADLOCO_CALL
    return hipGetLastError();
  }
};

template <typename E, bool FAST> struct LaunchNormBack {
  static hipError_t run(const NormBackArgs& a, hipStream_t st) {
#define ADLOCO_CALL(NV, WAVES) \
  hipLaunchKernelGGL((rms_norm_backward_kernel<E, NV, WAVES, FAST>), launch_grid(a.groups, 64 * WAVES), dim3(64 * WAVES), 0, st, a)
    ADLOCO_NORM_SHAPE(a.d, ADLOCO_CALL);
#undef ADLOCO_CALL
    return hipGetLastError();
  }
};

}  // namespace
}  // namespace adloco

using namespace adloco;

extern "C" int adloco_dropout(adloco_ctx* ctx, const void* x, int64_t x_row_stride, const void* residual,
                              int64_t residual_row_stride, void* out, int64_t out_row_stride, int64_t rows, int32_t d, int dtype,
                              const adloco_dropout_mask* mask, void* stream) {
  if (!ctx) return ADLOCO_EINVAL;
  if (!known_dtype(dtype)) return fail(ctx, ADLOCO_EUNSUPPORTED, "dropout: dtype %d not supported", dtype);
  if (rows < 0 || d < 1) return fail(ctx, ADLOCO_EINVAL, "dropout: rows = %lld, d = %d", (long long)rows, d);
  if (!mask) return fail(ctx, ADLOCO_EINVAL, "dropout: mask is NULL");
  DropArgs a{};
  if (const char* why = dropout_args(mask, a.m)) return fail(ctx, ADLOCO_EINVAL, "dropout: %s", why);
  if (rows == 0) return ADLOCO_OK;
  if (!x || !out) return fail(ctx, ADLOCO_EINVAL, "dropout: x or out is NULL");
  a.per_row = unsigned((d + 7LL) / 8);
  if (rows > (0x7fffffffLL * 64) / a.per_row) return fail(ctx, ADLOCO_EUNSUPPORTED, "dropout: too many elements for one launch");
  Matrix m[] = {{"x", x, x_row_stride, false}, {"residual", residual, residual_row_stride, false}, {"out", out, out_row_stride, true}};
  bool fast;
  if (!check_matrices(ctx, "dropout", m, 3, rows, d, dtype, fast)) return ADLOCO_EINVAL;
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.xs = m[0].stride;
  a.rs = m[1].stride;
  a.os = m[2].stride;
  a.rows = rows;
  a.total = rows * a.per_row;
  a.d = d;
  DeviceScope scope(ctx);
  if (!scope.ok()) return fail(ctx, ADLOCO_EHIP, "dropout: device %d cannot be made current", ctx->device);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipEvent_t ev = prof_begin(ctx, st);
  const hipError_t e = by_type<LaunchDropout>(dtype, fast, a, st);
  prof_end(ctx, kProfDropout, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "dropout launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}

extern "C" int adloco_rms_norm(adloco_ctx* ctx, const adloco_norm_io* io, int64_t rows, int32_t d, int dtype, double eps,
                               const adloco_dropout_mask* mask, const adloco_blocks8* y8, void* stream) {
  if (!ctx) return ADLOCO_EINVAL;
  if (!known_dtype(dtype)) return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm: dtype %d not supported", dtype);
  if (!io || rows < 0 || d < 1) return fail(ctx, ADLOCO_EINVAL, "rms_norm: no matrices, or rows = %lld, d = %d", (long long)rows, d);
  if (d > kNormWidth) return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm: d = %d exceeds %d", d, kNormWidth);
  if (rows > 0x7fffffffLL) return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm: too many rows for one launch");
  if (!(eps >= 1.1754943508222875e-38) || !(eps <= 1e30)) return fail(ctx, ADLOCO_EINVAL, "rms_norm: eps must be positive and finite in fp32");
  NormArgs a{};
  if (const char* why = dropout_args(mask, a.m)) return fail(ctx, ADLOCO_EINVAL, "rms_norm: %s", why);
  if (y8) {
    if (const char* why = check_blocks8(y8)) return fail(ctx, ADLOCO_EINVAL, "rms_norm: y8: %s", why);
    if (y8->rows != rows || y8->cols != d) return fail(ctx, ADLOCO_EINVAL, "rms_norm: y8 is not of rows x d values");
  }
  if (rows == 0) return ADLOCO_OK;
  if (!io->x || (!io->h && !io->y && !y8)) return fail(ctx, ADLOCO_EINVAL, "rms_norm: x is NULL, or there is no output");
  if (reinterpret_cast<uintptr_t>(io->gain) % 4) return fail(ctx, ADLOCO_EINVAL, "rms_norm: gain is not 4-byte aligned");
  Matrix m[] = {{"x", io->x, io->x_row_stride, false}, {"residual", io->residual, io->residual_row_stride, false},
                {"h", io->h, io->h_row_stride, true}, {"y", io->y, io->y_row_stride, true}};
  bool fast;
  if (!check_matrices(ctx, "rms_norm", m, 4, rows, d, dtype, fast)) return ADLOCO_EINVAL;
  const size_t es = size_of(dtype);
  const RowSpan gain{io->gain, 1, 4LL * d, 4LL * d};
  const RowSpan q{y8 ? y8->data : nullptr, rows, (d + 127LL) / 128 * 128, y8 ? (long long)y8->row_stride : 0};
  const RowSpan ex{y8 ? y8->exponent : nullptr, (d + 127LL) / 128, (long long)rows, y8 ? (long long)y8->exponent_stride : 0};
  for (const Matrix& x : m) {
    const RowSpan s{x.p, rows, (long long)(d * es), (long long)(x.stride * es)};
    if (spans_overlap(s, q) || spans_overlap(s, ex) || (x.written && spans_overlap(s, gain)))
      return fail(ctx, ADLOCO_EINVAL, "rms_norm: %s overlaps y8 or gain", x.name);
  }
  if (spans_overlap(gain, q) || spans_overlap(gain, ex) || spans_overlap(q, ex))
    return fail(ctx, ADLOCO_EINVAL, "rms_norm: y8 overlaps gain or itself");
  a.x = io->x;
  a.residual = io->residual;
  a.gain = io->gain;
  a.h = io->h;
  a.y = io->y;
  a.xs = m[0].stride;
  a.rs = m[1].stride;
  a.hs = m[2].stride;
  a.ys = m[3].stride;
  a.rows = rows;
  a.d = a.wide = d;
  if (y8) {
    a.q = static_cast<unsigned char*>(y8->data);
    a.e = y8->exponent;
    a.qs = y8->row_stride;
    a.es = y8->exponent_stride;
    a.wide = int((d + 127LL) / 128 * 128);
  }
  a.inv_d = 1.0 / d;
  a.eps = eps;
  DeviceScope scope(ctx);
  if (!scope.ok()) return fail(ctx, ADLOCO_EHIP, "rms_norm: device %d cannot be made current", ctx->device);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipEvent_t ev = prof_begin(ctx, st);
  const hipError_t e = by_type<LaunchNorm>(dtype, fast, a, st);
  prof_end(ctx, kProfNorm, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "rms_norm launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}

extern "C" int adloco_rms_norm_backward(adloco_ctx* ctx, const adloco_norm_backward_io* io, int64_t B, int64_t T, int32_t d,
                                        int dtype, double eps, const adloco_dropout_mask* mask, void* stream) {
  if (!ctx) return ADLOCO_EINVAL;
  if (!known_dtype(dtype)) return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm_backward: dtype %d not supported", dtype);
  if (!io || B < 0 || T < 0 || d < 1)
    return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: no matrices, or B = %lld, T = %lld, d = %d", (long long)B, (long long)T, d);
  if (d > kNormWidth) return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm_backward: d = %d exceeds %d", d, kNormWidth);
  if (B > 0x7fffffffLL || T > 0x7fffffffLL || B * T > 0x7fffffffLL)
    return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm_backward: too many rows for one launch");
  if (!(eps >= 1.1754943508222875e-38) || !(eps <= 1e30))
    return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: eps must be positive and finite in fp32");
  NormBackArgs a{};
  if (const char* why = dropout_args(mask, a.m)) return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: %s", why);
  const int64_t rows = B * T;
  if (B == 0 || (T == 0 && !io->gain_sums)) return ADLOCO_OK;
  if (T > 0 && (!io->h || !io->dy || (!io->dh && !io->dx && !io->gain_sums)))
    return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: h or dy is NULL, or there is no output");
  if (reinterpret_cast<uintptr_t>(io->gain) % 4 || reinterpret_cast<uintptr_t>(io->gain_sums) % 4)
    return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: gain or gain_sums is not 4-byte aligned");
  Matrix m[] = {{"h", io->h, io->h_row_stride, false}, {"dy", io->dy, io->dy_row_stride, false},
                {"dh_in", io->dh_in, io->dh_in_row_stride, false}, {"dh", io->dh, io->dh_row_stride, true},
                {"dx", io->dx, io->dx_row_stride, true}};
  bool fast;
  if (!check_matrices(ctx, "rms_norm_backward", m, 5, rows, d, dtype, fast)) return ADLOCO_EINVAL;
  const size_t es = size_of(dtype);
  const RowSpan gain{io->gain, 1, 4LL * d, 4LL * d}, sums{io->gain_sums, B, 4LL * d, 4LL * d};
  for (const Matrix& x : m) {
    const RowSpan s{x.p, rows, (long long)(d * es), (long long)(x.stride * es)};
    if (spans_overlap(s, sums) || (x.written && spans_overlap(s, gain)))
      return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: %s overlaps gain or gain_sums", x.name);
  }
  if (spans_overlap(gain, sums)) return fail(ctx, ADLOCO_EINVAL, "rms_norm_backward: gain overlaps gain_sums");
  DeviceScope scope(ctx);
  if (!scope.ok()) return fail(ctx, ADLOCO_EHIP, "rms_norm_backward: device %d cannot be made current", ctx->device);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // Runs per sample: enough workgroups to fill the chip, runs of 4 rows at least, their sums within the scratch.  Waves per
  // compute unit, measured: 32768 x 1024 with dropout 8: 78 us, 16: 70, 20: 74; 32768 x 2048 8: 99, 16: 111; 4096 x 8192 58, 64.
  const long long least = 4;
  const long long wanted = (long long)kNumCu * (d <= 1024 ? 16 : 8) / norm_waves(d);
  long long runs = (wanted + B - 1) / B;
  if (runs > (T + least - 1) / least) runs = (T + least - 1) / least;
  if (runs < 1) runs = 1;
  float* parts = io->gain_sums;
  if (io->gain_sums && runs > 1) {
    const long long fit = (long long)(kLayerScratch / 4) / (B * d);
    if (runs > fit) runs = fit;
    float* scratch = runs > 1 ? layer_scratch(ctx, st) : nullptr;
    if (scratch) parts = scratch; else runs = 1;
  }
  a.h = io->h;
  a.dy = io->dy;
  a.dh_in = io->dh_in;
  a.gain = io->gain;
  a.dh = io->dh;
  a.dx = io->dx;
  a.sums = io->gain_sums ? parts : nullptr;
  a.hs = m[0].stride;
  a.ys = m[1].stride;
  a.is = m[2].stride;
  a.os = m[3].stride;
  a.xs = m[4].stride;
  a.T = T;
  a.runs = int(runs);
  a.piece = 256;
  while ((long long)a.piece * a.piece < T / runs) a.piece *= 2;
  a.d = d;
  a.inv_d = float(1.0 / d);
  a.eps = float(eps);
  const int slabs = (d + 63) / 64;
  if (B * runs > 0x7fffffffLL || (runs > 1 && B * slabs > 0x7fffffffLL))
    return fail(ctx, ADLOCO_EUNSUPPORTED, "rms_norm_backward: too many samples for one launch");
  hipEvent_t ev = prof_begin(ctx, st);
  a.groups = unsigned(B * runs);
  hipError_t e = by_type<LaunchNormBack>(dtype, fast, a, st);
  if (e == hipSuccess && io->gain_sums && runs > 1) {
    hipLaunchKernelGGL(gain_runs_kernel, dim3(unsigned(B * slabs)), dim3(64 * kRunWaves), 0, st, parts, int(runs), d, slabs, io->gain_sums);
    e = hipGetLastError();
  }
  prof_end(ctx, kProfNormBack, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "rms_norm_backward launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}
