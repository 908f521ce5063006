// 8-bit blocks: packing of a matrix along its rows and / or across them, and the product of two packed matrices on the
// scaled matrix instructions.
#include <type_traits>
#include <utility>

#include "layer_ops.h"

namespace adloco {

const char* check_blocks8(const adloco_blocks8* b) {
  if (b->rows < 0 || b->cols < 1 || b->rows > 0x7fffffffLL || b->cols > 0x7fffff80LL) return "rows or cols out of range";
  const int64_t wide = (b->cols + 127) / 128 * 128;
  if (b->rows > 0 && (!b->data || !b->exponent)) return "data or exponent is NULL";
  if (reinterpret_cast<uintptr_t>(b->data) % 16 || reinterpret_cast<uintptr_t>(b->exponent) % 16)
    return "data and exponent must be 16-byte aligned";
  if (b->row_stride < wide || b->row_stride % 16 || b->row_stride > (int64_t(1) << 40) || !span_in_reach(b->rows, b->row_stride))
    return "row_stride must hold whole blocks of 128, be a multiple of 16 and within reach";
  if (b->exponent_stride < b->rows || b->exponent_stride % 16 || b->exponent_stride > (int64_t(1) << 40) ||
      !span_in_reach(wide / 128, b->exponent_stride))
    return "exponent_stride must be a multiple of 16, at least rows and within reach";
  return nullptr;
}

namespace {

// ---------------------------------------------------------------------------------------------------------------------
// Packing.  A workgroup of eight waves takes 128 x 128 values, a lane eight columns of four rows in registers: blocks along
// the rows are 16 lanes of a row, blocks across them the 32 groups of four rows.  x is read once whichever of the two outputs
// are asked for; the transposed one goes through LDS, so that both are stored in whole lines.  Bound by memory and by the two
// trips through a workgroup (load, reduce, turn, store): 32768 x 1024 bf16 both ways 25 us, 5.4 TB/s; 5632 x 2048 fp32 16 us.
// ---------------------------------------------------------------------------------------------------------------------
struct PackArgs {
  const void* x;
  long long xs;
  long long rows, cols;
  unsigned char *q, *e, *qt, *et;      // along the rows, across them; NULL: not asked for
  long long qs, es, qts, ets;
  unsigned col_tiles, tiles;
};

constexpr int kPackThreads = 512, kPackRows = 4;

template <typename E, bool FAST> __global__ __launch_bounds__(kPackThreads) void pack_blocks_kernel(PackArgs a) {
  constexpr int R = kPackRows;
  __shared__ __attribute__((aligned(16))) unsigned most[128];
  __shared__ __attribute__((aligned(16))) unsigned turn[128][32];
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const unsigned tile = unsigned(launch_index());
  if (tile >= a.tiles) return;
  const long long rt = tile / a.col_tiles, ct = tile - rt * a.col_tiles;
  const long long r0 = rt * 128 + rg * R, c0 = ct * 128;
  const int left = int(a.cols - c0 < 128 ? a.cols - c0 : 128);
  if (threadIdx.x < 128) most[threadIdx.x] = 0;
  // all four rows are requested before the first is looked at (rows and columns behind the last: the last ones again)
  float v[R][8];
  {
    eight<E> raw[R];
    const int cc = FAST && cg * 8 >= left ? left - 8 : cg * 8;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const long long r = r0 + i < a.rows ? r0 + i : a.rows - 1;
      raw[i] = fetch_eight<E, FAST>(static_cast<const E*>(a.x) + r * a.xs + c0, cc, left);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      widen_eight<E, FAST>(raw[i], cg * 8, left, v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = r0 + i < a.rows && cg * 8 + j < left ? v[i][j] : 0.f;
    }
  }
  if (a.q) {
    unsigned big[R], exps = 0;
    bool mine = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      big[i] = max16(largest<false>(v[i]));
      mine = mine || big[i] >= kNotFinite;
    }
    const bool any = __builtin_amdgcn_ballot_w64(mine) != 0;      // (the same for the wave)
    if (any)
#pragma unroll
      for (int i = 0; i < R; ++i) big[i] = max16(largest<true>(v[i]));
    uint2 out[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const unsigned e = block_exponent(big[i]);
      exps |= e << (8 * i);
      out[i] = pack_eight(v[i], e);
    }
    if (any)
#pragma unroll
      for (int i = 0; i < R; ++i) mark_eight(v[i], out[i]);
    unsigned char* q = a.q + r0 * a.qs + c0 + cg * 8;
    unsigned char* p = a.e + ct * a.es + r0;
    if (r0 + R <= a.rows) {
#pragma unroll
      for (int i = 0; i < R; ++i) *reinterpret_cast<uint2*>(q + i * a.qs) = out[i];
      if (cg == 0) *reinterpret_cast<unsigned*>(p) = exps;
    } else {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (r0 + i < a.rows) {
          *reinterpret_cast<uint2*>(q + i * a.qs) = out[i];
          if (cg == 0) p[i] = (unsigned char)(exps >> (8 * i));
        }
    }
  }
  if (!a.qt) return;
  // largest magnitude of each column: of a wave's 16 rows by shuffles, of the waves in LDS
  auto columns = [&](bool finite) {
    unsigned big[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      big[j] = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) big[j] = larger(big[j], finite && magnitude(v[i][j]) >= kNotFinite ? 0u : magnitude(v[i][j]));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) big[j] = larger(big[j], __shfl_xor(big[j], 16, 64));
#pragma unroll
    for (int j = 0; j < 8; ++j) big[j] = larger(big[j], __shfl_xor(big[j], 32, 64));
    unsigned all = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) all = larger(all, big[j]);
    if ((threadIdx.x & 63) < 16)
#pragma unroll
      for (int j = 0; j < 8; ++j) atomicMax(&most[cg * 8 + j], big[j]);
    return all >= kNotFinite;
  };
  __syncthreads();
  const bool any = __builtin_amdgcn_readfirstlane(__syncthreads_or(columns(false)));
  if (any) {                                          // some value of the tile is not finite: the maxima of the others
    if (threadIdx.x < 128) most[threadIdx.x] = 0;
    __syncthreads();
    columns(true);
    __syncthreads();
  }
  const uint4 lo = *reinterpret_cast<const uint4*>(&most[cg * 8]), hi = *reinterpret_cast<const uint4*>(&most[cg * 8 + 4]);
  const unsigned big[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  unsigned long long exps = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned e = block_exponent(big[j]);
    unsigned o = pack_four(v[0][j], v[1][j], v[2][j], v[3][j], e);
    if (any) mark_four(v[0][j], v[1][j], v[2][j], v[3][j], o);
    // (groups of four words permuted by the column: the lanes of a store spread over the banks)
    turn[cg * 8 + j][rg ^ ((cg & 7) << 2)] = o;
    exps |= (unsigned long long)e << (8 * j);
  }
  if (rg == 0 && cg * 8 < left) {
    unsigned char* p = a.et + rt * a.ets + c0 + cg * 8;
    if (cg * 8 + 8 <= left) *reinterpret_cast<unsigned long long*>(p) = exps;
    else
      for (int j = 0; cg * 8 + j < left; ++j) p[j] = (unsigned char)(exps >> (8 * j));
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = i * 64 + (threadIdx.x >> 3), q = threadIdx.x & 7;
    if (c < left)
      *reinterpret_cast<uint4*>(a.qt + (c0 + c) * a.qts + rt * 128 + q * 16) = *reinterpret_cast<const uint4*>(&turn[c][(q ^ ((c >> 3) & 7)) * 4]);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Product.  out[m][n] = sum_k 2^(ea[k / 128][m] - 127) 2^(eb[k / 128][n] - 127) a[m][k] b[n][k]: both operands hold k
// contiguously.
//   16-bit outputs: one v_mfma_scale_f32_16x16x128 multiplies 16 rows by 16 columns over one block of 128 and applies the
// two powers of two by itself.  It adds its products in groups whose members it cuts off below 2^-13 of the largest of them
// (measured; the unscaled 8-bit instructions do the same), which leaves 1.5e-5 of a sum of Gaussian values: a hundredth of
// what the output's own rounding costs in bf16, a tenth in fp16.
//   fp32 outputs, and 16-bit ones by request (EXACT): gradient sums would keep that error, so the values are widened to bf16 in
// registers, where they and their powers of two are exact, and multiplied by v_mfma_f32_16x16x32_bf16 at half the rate: products
// exact, sums fp32.
// Which 32 of the 128 values of k a lane holds does not matter as long as both operands agree; which 16 rows make a block of
// the tile is free too, and a lane takes neighbouring rows for the blocks (row = lane * NB + block), so that their exponents
// are one load and a lane's outputs of a row one store.
//   A workgroup of four waves forms a tile of 2 x 2 wave tiles of 16 MB x 16 NB.  Blocks of k come by direct loads into one of
// two LDS stages (rows of 128 bytes, 16-byte chunks permuted so that eight neighbouring rows lie in different banks).  Per
// block, the rows of B are held in registers and those of A stream through a few.  What bounds it is the way from L2 to LDS
// (31 to 39 bytes per clock and compute unit; a 256 x 256 tile needs 32 at the full rate of the matrix cores), so that loads
// have to be under way all the time: the workgroup meets twice per block and refills in two parts whatever has been read --
// after the first half of A's blocks their place and B's, after the second half theirs -- which gives every load one and a
// half blocks of time until it is needed, out of two stages.
//   Measured, these and the figures further down on one card in one go (cards differ by 5 %, and so does one with what it ran
// just before): 32768 x 5632 x 2048 to bf16 281 to 292 us, 2.6 PFLOP/s; 8192^3 344 us, 3.2; 16384^3 2.68 ms, 3.3.  fp32 out: 8192^3
// 801 us, 1.37 PFLOP/s; 1024 x 4096 x 32033 214 us, 1.26.  The matrix cores are busy for 73 % and 56 % of the cycles (and the clock
// falls to 1.7 and 1.9 GHz under them); in the second, widening takes as many vector cycles as the products take matrix cycles.
// ---------------------------------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) int mfma_i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

struct ProductArgs {
  const unsigned char *a, *b, *ea, *eb;
  long long as, bs, eas, ebs;
  void* out;
  float* part;                 // partial tiles [tile][piece] of a split contraction; NULL: none
  long long os;
  int M, N, steps;             // steps: blocks of k
  int tiles_m, tiles_n, pieces;
  int accumulate, vec;         // vec: a lane's outputs of a row are one aligned store
};

constexpr int kTileGroup = 4;  // tile rows that an XCD walks down before it takes the next tile column

__device__ __forceinline__ void tile_place(const ProductArgs& p, int tile, int& tm, int& tn) {
  const int band = tile / (kTileGroup * p.tiles_n), first = band * kTileGroup;
  const int high = p.tiles_m - first < kTileGroup ? p.tiles_m - first : kTileGroup;
  const int in = tile - first * p.tiles_n;
  tn = in / high;
  tm = first + in - tn * high;
}
// Tile and piece of a workgroup: consecutive workgroups go to the eight XCDs in turn, each XCD gets a contiguous run of the
// tiles, in bands of kTileGroup tile rows, so that what shares an L2 shares rows of A and columns of B.
__device__ __forceinline__ bool product_place(const ProductArgs& p, int index, int& tm, int& tn, int& piece, int& tile) {
  const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.pieces, per = (total + kNumXcd - 1) / kNumXcd;
  const int w = (index % kNumXcd) * per + index / kNumXcd;
  if (index / kNumXcd >= per || w >= total) return false;
  tile = w / p.pieces;
  piece = w - tile * p.pieces;
  tile_place(p, tile, tm, tn);
  return true;
}

// 4 bytes per lane to LDS, consecutive (see direct_load_lds16).
__device__ __forceinline__ void direct_load_lds4(const void* src, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(lds_addr) : "m0");
}

// The 32 values of a lane times their power of two, as four bf16 operands.
struct WideFrag { mfma_bf16x8 k[4]; };
__device__ __forceinline__ WideFrag widen(const mfma_i32x8& f, unsigned exponent) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const float s = __uint_as_float(exponent << 23);
  WideFrag w;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(unsigned(f[i]), s, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(unsigned(f[i]), s, true);
    w.k[i / 2][(i & 1) * 4 + 0] = lo[0];
    w.k[i / 2][(i & 1) * 4 + 1] = lo[1];
    w.k[i / 2][(i & 1) * 4 + 2] = hi[0];
    w.k[i / 2][(i & 1) * 4 + 3] = hi[1];
  }
  return w;
}

// PINNED: accumulators in the accumulation registers and in assembly, for tiles that need all of them (the compiler moves
// them about otherwise, and spills).  Operands and exponents come straight from LDS, so that no vector instruction that wrote
// them stands near; fences as for mfma_16x16x32.
// FRESH: from zero, the old accumulators are only overwritten.
template <int SEL_A, int SEL_B, bool PINNED, bool FRESH>
__device__ __forceinline__ void scaled_mfma(mfma_f32x4& c, const mfma_i32x8& a, const mfma_i32x8& b, int ea, int eb) {
  if constexpr (PINNED && FRESH)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, 0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
                 : "=a"(c) : "v"(a), "v"(b), "v"(ea), "v"(eb), "n"(SEL_A & 1), "n"(SEL_B & 1), "n"(SEL_A >> 1), "n"(SEL_B >> 1));
  else if constexpr (PINNED)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
                 : "+a"(c) : "v"(a), "v"(b), "v"(ea), "v"(eb), "n"(SEL_A & 1), "n"(SEL_B & 1), "n"(SEL_A >> 1), "n"(SEL_B >> 1));
  else
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, SEL_A, ea, SEL_B, eb);
}
template <typename E, int NB> __device__ __forceinline__ void store_row(E* p, const float (&v)[NB], bool accumulate) {
  typedef __attribute__((ext_vector_type(NB))) E row;
  row r;
  if constexpr (std::is_same<E, float>::value) {
    row old = {};
    if (accumulate) old = *reinterpret_cast<const row*>(p);
#pragma unroll
    for (int n = 0; n < NB; ++n) r[n] = accumulate ? old[n] + v[n] : v[n];
  } else {
#pragma unroll
    for (int n = 0; n < NB; ++n) r[n] = E(v[n]);
  }
  *reinterpret_cast<row*>(p) = r;
}

template <int MB, int NB, bool EXACT> struct TileShape {
  static constexpr int wave_m = 16 * MB, wave_n = 16 * NB, edge_m = 2 * wave_m, edge_n = 2 * wave_n, rows = edge_m + edge_n;
  static constexpr int stage = rows * 128 + rows;              // values of A, of B; exponents of A, of B
  static constexpr int lds = 2 * stage;
  static constexpr int resident = MB * NB == 16 ? 2 : 1;       // workgroups per compute unit
  static constexpr int ahead = MB == 8 ? 3 : 1;                // rows of A fetched before they are multiplied
  static constexpr int first_loads = MB / 2 + NB + 1, second_loads = MB / 2;   // direct loads per wave: B, exponents and the
                                                                               // first half of A; the second half
};

template <int N> __device__ __forceinline__ void product_wait() {
  static_assert(N < 64, "the counter has six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

template <typename F, int... K> __device__ __forceinline__ void for_each_index(F& f, std::integer_sequence<int, K...>) {
  (f(std::integral_constant<int, K>{}), ...);
}

// WALK: one workgroup per compute unit takes tile after tile (every 32nd of its XCD's run), and asks for the first blocks of
// the next one before it stores the outputs of this one, which then leave under its first products.  For whole contractions of
// an even number of blocks.
template <int MB, int NB, bool EXACT, bool WALK, typename E>
__global__ __launch_bounds__(256, (TileShape<MB, NB, EXACT>::resident)) void product_tile_kernel(ProductArgs p) {
  using T = TileShape<MB, NB, EXACT>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  int tm, tn, piece, tile;
  if (!product_place(p, blockIdx.x, tm, tn, piece, tile)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, kg = lane >> 4;
  int m0 = tm * T::edge_m, n0 = tn * T::edge_n;       // of the tile that is multiplied
  const int s0 = int((long long)p.steps * piece / p.pieces), n_steps = int((long long)p.steps * (piece + 1) / p.pieces) - s0;
  const unsigned at = lds_address(lds);

  // Direct loads of eight rows each.  Slot q of a wave tile holds its row (q % 16) * MB + q / 16 (the 16 rows of a block side
  // by side), chunk c of it at place c ^ (q / 2 % 8): the 16 lanes of a read
  // that go together lie in all 64 banks.  Rows behind the last one are the last one again.
  const int chunk = ((lane & 7) ^ (lane >> 4)) * 16;
  auto offset = [&](int sub, int tile_row, int q, int blocks, int last, long long stride) {
    const int in = q + sub, r = tile_row + (in & 15) * blocks + (in >> 4);
    return __umul24(unsigned(r < last ? r : last), unsigned(stride)) + (chunk ^ ((q & 8) * 8));
  };
  // A: load i of MB brings blocks of half i / (MB / 2) of both wave tiles' rows
  auto slot_a = [&](int i, int& t) {
    const int u = wave * (MB / 2) + i % (MB / 2);
    t = u / MB;
    return i / (MB / 2) * 8 * MB + (u % MB) * 8;
  };
  auto slot_b = [&](int i, int& t) {
    const int u = wave * NB + i;
    t = u / (2 * NB);
    return (u % (2 * NB)) * 8;
  };
  // exponents, four rows a lane; a wave brings 256 bytes of A's and B's (the four waves all of them, some twice)
  const int e_at = (wave & 1) * (T::rows - 256) + lane * 4;
  const bool of_b = e_at >= T::edge_m;
  const int e_row = of_b ? e_at - T::edge_m : e_at;
  const long long pe_step = of_b ? p.ebs : p.eas;
  unsigned off_a[MB], off_b[NB];
  const unsigned char *base_a, *base_b, *pe;
  int loaded = 0;
  auto aim = [&](int tm, int tn) {                    // loads: to the first block of a tile
    const int r0 = tm * T::edge_m, q0 = tn * T::edge_n, last_a = p.M - r0 - 1, last_b = p.N - q0 - 1;
    int sub = lane >> 3;
    if constexpr (WALK) asm volatile("" : "+v"(sub));   // (formed anew for every tile: kept, it costs registers that the loop needs)
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      int t;
      const int q = slot_a(i, t);
      off_a[i] = offset(sub, t * T::wave_m, q, MB, last_a, p.as);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      int t;
      const int q = slot_b(i, t);
      off_b[i] = offset(sub, t * T::wave_n, q, NB, last_b, p.bs);
    }
    base_a = uniform_ptr(p.a + (long long)r0 * p.as + (long long)s0 * 128);
    base_b = uniform_ptr(p.b + (long long)q0 * p.bs + (long long)s0 * 128);
    const int e_rows = of_b ? p.N - q0 : p.M - r0;
    pe = (of_b ? p.eb + (long long)s0 * p.ebs + q0 : p.ea + (long long)s0 * p.eas + r0) + (e_row < e_rows ? e_row : 0);
    loaded = 0;
  };
  aim(tm, tn);
  auto load_a = [&](int buf, int i) {
    int t;
    const int q = slot_a(i, t);
    direct_load_lds16_s(off_a[i], base_a, at + buf * T::stage + (t * T::wave_m + q) * 128);
  };
  auto load_b = [&](int buf, int i) {
    int t;
    const int q = slot_b(i, t);
    direct_load_lds16_s(off_b[i], base_b, at + buf * T::stage + (T::edge_m + t * T::wave_n + q) * 128);
  };
  auto load_first = [&](int buf, int i) {             // item i of first_loads
    if (i == 0) {
      direct_load_lds4(pe, at + buf * T::stage + T::rows * 128 + (wave & 1) * (T::rows - 256));
    } else if (i <= NB) {
      load_b(buf, i - 1);
    } else {
      load_a(buf, i - 1 - NB);
    }
  };
  auto load_second = [&](int buf, int i) {
    load_a(buf, MB / 2 + i);
    if (i == MB / 2 - 1 && ++loaded < n_steps) {      // to the next block; behind the last one, that one again
      base_a += 128;
      base_b += 128;
      pe += pe_step;
    }
  };
  auto meet = [&] {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  const int wm = (wave >> 1) * T::wave_m, wn = (wave & 1) * T::wave_n;
  const int key = l16 >> 1;
  const int row_a = (wm + l16) * 128, row_b = (T::edge_m + wn + l16) * 128;
  const int c0 = ((kg * 2) ^ key) * 16, c1 = ((kg * 2 + 1) ^ key) * 16;
  auto frag = [&](int buf, int row, int block) {
    const unsigned char* q = lds + buf * T::stage + row + block * 2048;
    const i32x4 x = *reinterpret_cast<const i32x4*>(q + c0), y = *reinterpret_cast<const i32x4*>(q + c1);
    return mfma_i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  };

  constexpr bool pinned = MB * NB == 64 && !EXACT;
  constexpr int ahead = T::ahead;
  mfma_f32x4 acc[MB][NB];
  if constexpr (!WALK) {
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[m][n] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (pinned) mfma_fence(acc);
  }
  struct Held { mfma_i32x8 b[NB], a[ahead]; int ea[MB / 4], eb[NB / 4]; };
  constexpr int fetches = 1 + ahead + NB;
  auto fetch = [&](int buf, Held& h, int i) {         // item i of fetches
    const unsigned char* q = lds + buf * T::stage + T::rows * 128;
    if (i == 0) {
#pragma unroll
      for (int x = 0; x < MB / 4; ++x) h.ea[x] = *reinterpret_cast<const int*>(q + wm + l16 * MB + x * 4);
#pragma unroll
      for (int x = 0; x < NB / 4; ++x) h.eb[x] = *reinterpret_cast<const int*>(q + T::edge_m + wn + l16 * NB + x * 4);
    } else if (i == 1) {
      h.a[0] = frag(buf, row_a, 0);
    } else if (i < 2 + NB) {
      h.b[i - 2] = frag(buf, row_b, i - 2);
    } else {
      h.a[i - 1 - NB] = frag(buf, row_a, i - 1 - NB);
    }
  };
  // Block s of the piece, in stage s % 2.  Loads are asked for in the order first(s), second(s), first(s + 1), ..; two blocks
  // are under way at most, and a wait leaves those behind the one it is for.  Blocks behind the last one are loaded and
  // fetched like any other (the last one again, into places that nobody reads any more), so that all steps are alike.
  // A wave issues in order, and a matrix instruction keeps the matrix core busy for eight issue slots: loads and LDS reads are
  // dealt out one by one between them.
  // FRESH: the first block of a walked tile, whose products overwrite the accumulators.  behind_1, behind_2: stores of the
  // tile before that lie between the loads that are waited for and the wait (memory operations of a wave count down in order).
  constexpr int stores = MB * 4;
  auto wait = [](bool behind) {
    if (WALK && behind) product_wait<T::first_loads + T::second_loads + stores>();
    else product_wait<T::first_loads + T::second_loads>();
  };
  auto step = [&](auto fresh, int buf, Held& h, Held& next, bool behind_1, bool behind_2) {
    constexpr int meet_1 = (MB / 2 - ahead) * NB, meet_2 = (MB - ahead) * NB, end = MB * NB;
    mfma_i32x8 a[MB];
#pragma unroll
    for (int i = 0; i < ahead; ++i) a[i] = h.a[i];
    WideFrag wa, wb[EXACT ? NB : 1];
    auto slot = [&](auto index) {
      constexpr int k = decltype(index)::value, m = k / NB, n = k % NB;
      if constexpr (k == meet_1) {                    // B and the first half of A have been read; the second half is needed
        wait(behind_1);
        meet();
      }
      if constexpr (k == meet_2) {                    // all of A has been read; the next block's first part is needed
        wait(behind_2);
        meet();
      }
      if constexpr (EXACT) {
        if (n == 0) wa = widen(a[m], (unsigned(h.ea[m / 4]) >> (8 * (m & 3))) & 255u);
        if (m == 0) wb[n] = widen(h.b[n], (unsigned(h.eb[n / 4]) >> (8 * (n & 3))) & 255u);
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[m][n] = mfma_16x16x32_v<false>(wa.k[x], wb[n].k[x], acc[m][n]);
      } else {
        scaled_mfma<(m & 3), (n & 3), pinned, decltype(fresh)::value>(acc[m][n], a[m], h.b[n], h.ea[m / 4], h.eb[n / 4]);
      }
      if constexpr (n == 0 && m + ahead < MB) a[m + ahead] = frag(buf, row_a, m + ahead);
      if constexpr (k >= meet_1 && k < meet_2) {
#pragma unroll
        for (int i = 0; i < T::first_loads; ++i)
          if (k == meet_1 + i * (meet_2 - meet_1) / T::first_loads) load_first(buf, i);
      }
      if constexpr (k >= meet_2) {
#pragma unroll
        for (int i = 0; i < fetches; ++i)
          if (k == meet_2 + i * (end - meet_2) / fetches) fetch(buf ^ 1, next, i);
#pragma unroll
        for (int i = 0; i < T::second_loads; ++i)
          if (k == meet_2 + (2 * i + 1) * (end - meet_2) / (2 * T::second_loads)) load_second(buf, i);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    for_each_index(slot, std::make_integer_sequence<int, end>{});
  };
  auto load = [&](int buf) {
#pragma unroll
    for (int i = 0; i < T::first_loads; ++i) load_first(buf, i);
#pragma unroll
    for (int i = 0; i < T::second_loads; ++i) load_second(buf, i);
  };
  // Element j of block (m, n): row (kg * 4 + j) * MB + m of the wave tile, column l16 * NB + n.  Four ways out, each short
  // enough for the instruction cache (checks woven into one of them: 60 KB of code, 4 us a tile).
  auto rows_out = [&](int first, int count, auto put) {
#pragma unroll
    for (int m = 0; m < MB; ++m)
      if (m >= first && m < first + count)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v[NB];
#pragma unroll
          for (int i = 0; i < NB; ++i) v[i] = pinned ? mfma_acc(acc[m][i], j) : acc[m][i][j];
          put(m, j, v);
        }
  };
  auto store = [&]() -> bool {                        // true: by `stores` memory operations, and nothing else of LDS
    if constexpr (pinned) mfma_fence(acc);
    int row0 = wm + kg * 4 * MB;
    if constexpr (WALK) asm volatile("" : "+v"(row0));
    if (p.part) {
      float* const part = p.part + ((long long)tile * p.pieces + piece) * (T::edge_m * T::edge_n) + row0 * T::edge_n + wn + l16 * NB;
      rows_out(0, MB, [&](int m, int j, const float (&v)[NB]) { store_row<float, NB>(part + (j * MB + m) * T::edge_n, v, false); });
    } else if (p.vec && p.M - m0 >= T::edge_m && p.N - n0 >= T::edge_n) {
      E* const out = static_cast<E*>(p.out) + (m0 + row0) * p.os + n0 + wn + l16 * NB;
      rows_out(0, MB, [&](int m, int j, const float (&v)[NB]) { store_row<E, NB>(out + (j * MB + m) * p.os, v, p.accumulate != 0); });
      return !p.accumulate;
    } else if (p.vec && p.N % NB == 0) {
      // a tile on the edge: a lane's columns are all there or all not
      const int below = p.M - m0 - row0;
      E* const out = static_cast<E*>(p.out) + (m0 + row0) * p.os + n0 + wn + l16 * NB;
      if (n0 + wn + l16 * NB < p.N)
        rows_out(0, MB, [&](int m, int j, const float (&v)[NB]) {
          if (j * MB + m < below) store_row<E, NB>(out + (j * MB + m) * p.os, v, p.accumulate != 0);
        });
    } else {
      // rows that are not aligned, or no whole number of a lane's columns: 64 rows of the wave tile at a time through LDS, value
      // by value, eight under way
      constexpr int passes = MB / 4, wide = T::wave_n / 64, ahead_rows = 8 / wide;
      product_wait<0>();
      meet();
      float* const mine = reinterpret_cast<float*>(lds) + wave * (64 * T::wave_n);
#pragma unroll
      for (int h = 0; h < passes; ++h) {
        rows_out(h * 4, 4, [&](int m, int j, const float (&v)[NB]) {
          float* to = mine + ((kg * 4 + j) * 4 + m - h * 4) * T::wave_n + l16 * NB;
#pragma unroll
          for (int i = 0; i < NB; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int below = p.M - m0 - wm, right = p.N - n0 - wn;
        E* const out = static_cast<E*>(p.out) + (m0 + wm) * p.os + n0 + wn;
#pragma unroll 1
        for (int i0 = 0; i0 < 64; i0 += ahead_rows) {
          float v[ahead_rows][wide];
#pragma unroll
          for (int i = 0; i < ahead_rows; ++i)
#pragma unroll
            for (int c = 0; c < wide; ++c) v[i][c] = mine[(i0 + i) * T::wave_n + c * 64 + lane];
#pragma unroll
          for (int i = 0; i < ahead_rows; ++i) {
            const int r = ((i0 + i) >> 2) * MB + h * 4 + ((i0 + i) & 3);
#pragma unroll
            for (int c = 0; c < wide; ++c)
              if (r < below && c * 64 + lane < right) {
                E* q = out + r * p.os + c * 64 + lane;
                if constexpr (std::is_same<E, float>::value) *q = p.accumulate ? *q + v[i][c] : v[i][c];
                else *q = E(v[i][c]);
              }
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    return false;
  };
  Held h0, h1;
  auto begin = [&](bool behind) {                     // the first block is here: fetch what its first products take
    if (WALK && behind) product_wait<T::first_loads + 2 * T::second_loads + stores>();
    else product_wait<T::first_loads + 2 * T::second_loads>();
    meet();
#pragma unroll
    for (int i = 0; i < fetches; ++i) fetch(0, h0, i);
  };
  constexpr std::integral_constant<bool, false> more{};
  load(0);
  load(1);
  bool behind = false;
  if constexpr (WALK) {
    constexpr std::integral_constant<bool, true> fresh{};
    for (int w = blockIdx.x;;) {
      begin(behind);
      step(fresh, 0, h0, h1, behind, behind);
      step(more, 1, h1, h0, behind, false);
#pragma unroll 1
      for (int s = 2; s < n_steps; s += 2) {
        step(more, 0, h0, h1, false, false);
        step(more, 1, h1, h0, false, false);
      }
      w += kNumCu;
      const bool on = product_place(p, w, tm, tn, piece, tile);
      const bool plain = p.vec && p.M - m0 >= T::edge_m && p.N - n0 >= T::edge_n;
      product_wait<0>();                              // (the last loads went to the places that the next ones take)
      if (on && plain) {
        aim(tm, tn);
        load(0);
        load(1);
      }
      behind = store();
      if (!on) break;
      m0 = tm * T::edge_m;
      n0 = tn * T::edge_n;
      if (!plain) {                                   // (LDS served the outputs)
        meet();
        aim(tm, tn);
        load(0);
        load(1);
      }
    }
  } else {
    begin(false);
    for (int s = 0; s + 1 < n_steps; s += 2) {
      step(more, 0, h0, h1, false, false);
      step(more, 1, h1, h0, false, false);
    }
    if (n_steps & 1) step(more, 0, h0, h1, false, false);
    behind = store();
  }
  // No load may reach LDS that is another workgroup's by then; stores may be under way still (a wave's memory operations
  // count down in order).
  if (behind) product_wait<stores>();
  else product_wait<0>();
}

// Adds up the pieces of a split contraction in order: four columns of a tile row per lane.
template <int EDGE_M, int EDGE_N, typename E> __global__ __launch_bounds__(256) void product_join_kernel(ProductArgs p) {
  constexpr int rows = 1024 / EDGE_N, slabs = EDGE_M / rows;
  const int tile = blockIdx.x / slabs, r = (blockIdx.x - tile * slabs) * rows + threadIdx.x / (EDGE_N / 4);
  const int c = (threadIdx.x % (EDGE_N / 4)) * 4;
  int tm, tn;
  tile_place(p, tile, tm, tn);
  if (tm * EDGE_M + r >= p.M || tn * EDGE_N + c >= p.N) return;
  const float* from = p.part + (long long)tile * p.pieces * (EDGE_M * EDGE_N) + r * EDGE_N + c;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < p.pieces; ++s) {
    const float4 x = *reinterpret_cast<const float4*>(from + (long long)s * (EDGE_M * EDGE_N));
    v[0] += x.x;
    v[1] += x.y;
    v[2] += x.z;
    v[3] += x.w;
  }
  E* const out = static_cast<E*>(p.out) + (tm * EDGE_M + r) * p.os + tn * EDGE_N + c;
  const int left = p.N - tn * EDGE_N - c;
  if (p.vec && left >= 4) {
    store_row<E, 4>(out, v, p.accumulate != 0);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) {
      if constexpr (std::is_same<E, float>::value) out[i] = p.accumulate ? out[i] + v[i] : v[i];
      else out[i] = E(v[i]);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Few rows of A (up to 32): B is read once, by whoever multiplies it, straight into registers; all else is latency.  A
// workgroup takes 16 columns, its waves share the blocks of k among them and add up what they have through LDS, in order.
// 3 x 5632 x 2048: 5.4 us, 2.1 TB/s of B (with the host's part 8.0, on small tiles 9.2); 33 to 64 rows would take 13 us, on
// small tiles 10.  Widened like fp32 outputs whatever the output is: the vector and matrix cores wait for memory anyway (8-bit
// instruction / widened, with the host's part: 3 x 5632 x 2048 7.0 / 7.0 us, 32 x 8192 x 8192 24.9 / 25.3, 8 x 4096 x 14336
// 15.0 / 15.4).
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kFewRows = 32;

template <int RB, int WAVES, typename E> __global__ __launch_bounds__(64 * WAVES) void product_few_kernel(ProductArgs p) {
  __shared__ float lds[WAVES][RB][4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kg = lane >> 4;
  const long long first = launch_index() * 16;
  if (first >= p.N) return;
  const int n = int(first) + l16, nn = n < p.N ? n : p.N - 1;
  const unsigned char* b = p.b + (long long)nn * p.bs + kg * 32;
  const unsigned char* eb = p.eb + nn;
  const unsigned char* a[RB];
  const unsigned char* ea[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int m = r * 16 + l16 < p.M ? r * 16 + l16 : p.M - 1;
    a[r] = p.a + (long long)m * p.as + kg * 32;
    ea[r] = p.ea + m;
  }
  mfma_f32x4 acc[RB] = {};
  auto values = [](const unsigned char* q) {
    const i32x4 x = *reinterpret_cast<const i32x4*>(q), y = *reinterpret_cast<const i32x4*>(q + 16);
    return mfma_i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  };
  constexpr int U = 4;                                // blocks of k that a wave has under way
  for (int s0 = wave; s0 < p.steps; s0 += WAVES * U) {
    mfma_i32x8 fb[U], fa[U][RB];
    int xb[U], xa[U][RB];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int s = s0 + i * WAVES < p.steps ? s0 + i * WAVES : p.steps - 1;
      fb[i] = values(b + (long long)s * 128);
      xb[i] = eb[s * p.ebs];
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        fa[i][r] = values(a[r] + (long long)s * 128);
        xa[i][r] = ea[r][s * p.eas];
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (s0 + i * WAVES >= p.steps) break;           // (the same for the wave)
      const WideFrag wb = widen(fb[i], unsigned(xb[i]));
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const WideFrag wa = widen(fa[i][r], unsigned(xa[i][r]));
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[r] = mfma_16x16x32_v<false>(wa.k[k], wb.k[k], acc[r]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[wave][r][j][lane] = acc[r][j];
  __syncthreads();
  for (int i = wave; i < RB * 4; i += WAVES) {
    const int r = i >> 2, j = i & 3, m = r * 16 + kg * 4 + j;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += lds[w][r][j][lane];
    if (m >= p.M || n >= p.N) continue;
    E* to = static_cast<E*>(p.out) + (long long)m * p.os + n;
    if constexpr (std::is_same<E, float>::value) *to = p.accumulate ? *to + v : v;
    else *to = E(v);
  }
}

size_t size_of(int dtype) { return is_16bit(dtype) ? 2 : 4; }

template <typename E, bool FAST> hipError_t launch_pack(const PackArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((pack_blocks_kernel<E, FAST>), launch_grid(a.tiles, kPackThreads), dim3(kPackThreads), 0, st, a);
  return hipGetLastError();
}
template <int MB, int NB, bool EXACT, bool WALK, typename E> hipError_t launch_tiles(const ProductArgs& p, hipStream_t st) {
  using T = TileShape<MB, NB, EXACT>;
  auto kern = product_tile_kernel<MB, NB, EXACT, WALK, E>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, T::lds);
  if (e != hipSuccess) return e;
  const unsigned total = unsigned(p.tiles_m) * unsigned(p.tiles_n);
  const unsigned groups = WALK ? kNumCu : (total * p.pieces + kNumXcd - 1) / kNumXcd * kNumXcd;
  hipLaunchKernelGGL(kern, dim3(groups), dim3(256), T::lds, st, p);
  if (p.part)
    hipLaunchKernelGGL((product_join_kernel<T::edge_m, T::edge_n, E>), dim3(total * (T::edge_m * T::edge_n / 1024)), dim3(256), 0, st, p);
  return hipGetLastError();
}
// Waves per workgroup: as many blocks of k under way as it takes to fill the chip.
int few_waves(long long N, long long steps) { return N > 255 * 16 && steps <= 64 ? 4 : 8; }
template <int RB, typename E> hipError_t launch_few_rows(const ProductArgs& p, hipStream_t st) {
  const long long blocks = (p.N + 15LL) / 16;
  if (few_waves(p.N, p.steps) == 4)
    hipLaunchKernelGGL((product_few_kernel<RB, 4, E>), launch_grid(blocks, 256), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((product_few_kernel<RB, 8, E>), launch_grid(blocks, 512), dim3(512), 0, st, p);
  return hipGetLastError();
}
template <typename E> hipError_t launch_few(const ProductArgs& p, hipStream_t st) {
  return p.M <= 16 ? launch_few_rows<1, E>(p, st) : launch_few_rows<2, E>(p, st);
}
// More large tiles than compute units, whole, of an even number of blocks: one workgroup per compute unit walks over them (one
// workgroup per tile / walking: 32768 x 5632 x 2048 300 / 292 us, x 512 120 / 115, 8192 x 8192 x 1024 68.6 / 66.0).
template <typename E> hipError_t launch_product(const ProductArgs& p, bool large, bool exact, hipStream_t st) {
  if constexpr (!std::is_same<E, float>::value) {
    if (large) {
      const bool walk = p.pieces == 1 && p.steps % 2 == 0 && p.tiles_m * p.tiles_n > kNumCu;
      return walk ? launch_tiles<8, 8, false, true, E>(p, st) : launch_tiles<8, 8, false, false, E>(p, st);
    }
    if (!exact) return launch_tiles<4, 4, false, false, E>(p, st);
  }
  return launch_tiles<4, 4, true, false, E>(p, st);
}

// Which kernel, and how many pieces the contraction is cut into.  Times in microseconds, fitted to 5600 timings over 250
// shapes (1 to 32768 rows, 64 to 8192 columns, 128 to 32768 values of k; log error 13 %): 0.36 a block of k for a small tile
// that has its compute unit to itself and 0.95 for two that share it (exact products 0.75 and 1.5), 0.93 for a large tile, 3.0
// and 6.5 to start and store one; 1.7 and the partial tiles' way out and back for a second kernel.  The choice is within 4 %
// of the best one on average.  Measured with the host's 7 us, few rows / small tiles / small tiles in 4 pieces / large:
// 3 x 5632 x 2048 8.0 / 9.2 / 10.7 / 20, 64 x 8192 x 8192 - / 28 / 20 / 64, 512 x 5632 x 2048 - / 11 / 25 / 21, 32768 x 5632 x 2048
// - / 364 / - / 281 us.  Rows of the output that are not 16-byte aligned count 12 us more for a large tile (32001 x 2044 x 1024:
// small 79, large 97).
struct ProductChoice { int kernel, pieces; };          // kernel: 1 few rows, 4 small tiles, 8 large ones
ProductChoice choose_product(long long M, long long N, int steps, bool exact, bool aligned, int kernel, int pieces, bool split) {
  ProductChoice best{4, 1};
  double least = 1e300;
  auto offer = [&](int k, int n, double t) {
    if (t < least) {
      least = t;
      best = ProductChoice{k, n};
    }
  };
  if (M <= kFewRows && kernel <= 1) {
    const int waves = few_waves(N, steps);
    const double share = double((N + 15) / 16) * waves / (kNumCu * 16);
    offer(1, 1, 1.2 + double((steps + waves - 1) / waves) * (share > 1.0 ? share : 1.0) * (M <= 16 ? 0.45 : 0.65));
  }
  for (int k = 4; k <= 8; k += 4) {
    if ((kernel > 1 && k != kernel && !(exact && k == 4)) || (exact && k == 8)) continue;
    const long long edge = 32 * k, tiles = ((M + edge - 1) / edge) * ((N + edge - 1) / edge);
    const int most = !split ? 1 : pieces ? pieces : 64;
    for (int p = pieces && split ? pieces : 1; p <= most; ++p) {
      const int n = p < steps ? p : steps;
      if (n > 1 && size_t(tiles) * n * size_t(edge * edge) * sizeof(float) > kLayerScratch) {
        if (pieces) offer(k, 1, 1e299);
        break;
      }
      const double w = double(tiles) * n, s = double((steps + n - 1) / n);
      double t;
      if (k == 4) {
        const double alone = s * (exact ? 0.75 : 0.36) + 3.0, shared = s * (exact ? 1.5 : 0.95) + 3.0;
        const double full = double((long long)w / (2 * kNumCu)), left = w - full * 2 * kNumCu;
        t = full * shared + (left > kNumCu ? shared : left > 0 ? alone : 0.0);
      } else {
        t = double(((long long)w + kNumCu - 1) / kNumCu) * (s * 0.93 + (aligned || n > 1 ? 6.5 : 18.5));
      }
      offer(k, n, t + (n > 1 ? 1.7 + w * double(edge * edge) * 1e-6 : 0.0));
      if (n == steps) break;
    }
  }
  return best;
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
  if (!x || xs < cols || xs > (int64_t(1) << 40) || !span_in_reach(rows, xs * (int64_t)es) || reinterpret_cast<uintptr_t>(x) % es)
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
  a.tiles = unsigned(rt * ct);
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
  hipEvent_t ev = prof_begin(ctx, st);
  hipError_t e;
  if (dtype == ADLOCO_BF16) e = fast ? launch_pack<__bf16, true>(a, st) : launch_pack<__bf16, false>(a, st);
  else if (dtype == ADLOCO_F16) e = fast ? launch_pack<_Float16, true>(a, st) : launch_pack<_Float16, false>(a, st);
  else e = fast ? launch_pack<float, true>(a, st) : launch_pack<float, false>(a, st);
  prof_end(ctx, kProfPack, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "pack_blocks launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}

extern "C" int adloco_block_product(adloco_ctx* ctx, const adloco_blocks8* a, const adloco_blocks8* b, void* out, int64_t out_row_stride,
                                    int dtype, uint32_t flags, void* stream) {
  if (!ctx) return ADLOCO_EINVAL;
  if (dtype != ADLOCO_F32 && !is_16bit(dtype)) return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: dtype %d not supported", dtype);
  if (!a || !b) return fail(ctx, ADLOCO_EINVAL, "block_product: a or b is NULL");
  if (flags & ~(ADLOCO_ACCUMULATE | ADLOCO_EXACT_PRODUCTS)) return fail(ctx, ADLOCO_EINVAL, "block_product: unknown flags");
  if ((flags & ADLOCO_ACCUMULATE) && dtype != ADLOCO_F32)
    return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: only an fp32 output accumulates");
  if (const char* why = check_blocks8(a)) return fail(ctx, ADLOCO_EINVAL, "block_product: a: %s", why);
  if (const char* why = check_blocks8(b)) return fail(ctx, ADLOCO_EINVAL, "block_product: b: %s", why);
  if (a->cols != b->cols) return fail(ctx, ADLOCO_EINVAL, "block_product: rows of a hold %lld values, of b %lld", (long long)a->cols, (long long)b->cols);
  if (a->rows == 0 || b->rows == 0) return ADLOCO_OK;
  const size_t es = size_of(dtype);
  const int64_t os = out_row_stride ? out_row_stride : b->rows;
  if (!out || os < b->rows || os > (int64_t(1) << 40) || !span_in_reach(a->rows, os * (int64_t)es) ||
      reinterpret_cast<uintptr_t>(out) % es)
    return fail(ctx, ADLOCO_EINVAL, "block_product: out is NULL or misaligned, or its row stride is smaller than the row or out of range");
  const RowSpan so{out, a->rows, (long long)(b->rows * es), (long long)(os * es)};
  for (const adloco_blocks8* x : {a, b})
    if (spans_overlap(so, values_of(x)) || spans_overlap(so, exponents_of(x)))
      return fail(ctx, ADLOCO_EINVAL, "block_product: out overlaps an operand");
  if (a->row_stride > (1 << 23) || b->row_stride > (1 << 23))
    return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: rows more than 2^23 bytes apart");
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
  p.accumulate = flags & ADLOCO_ACCUMULATE ? 1 : 0;
  DeviceScope scope(ctx);
  if (!scope.ok()) return fail(ctx, ADLOCO_EHIP, "block_product: device %d cannot be made current", ctx->device);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool exact = dtype == ADLOCO_F32 || (flags & ADLOCO_EXACT_PRODUCTS);
  const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0 && os * (int64_t)es % 16 == 0;
  ProductChoice c = choose_product(a->rows, b->rows, p.steps, exact, aligned, ctx->product_blocks, ctx->product_pieces, true);
  if (c.pieces > 1) {
    p.part = layer_scratch(ctx, st);
    if (!p.part) c = choose_product(a->rows, b->rows, p.steps, exact, aligned, ctx->product_blocks, ctx->product_pieces, false);
  }
  const bool few = c.kernel == 1, large = c.kernel == 8;
  const int64_t edge = large ? 256 : 128, tm = (a->rows + edge - 1) / edge, tn = (b->rows + edge - 1) / edge;
  if (tm * tn > 0xfffff8LL) return fail(ctx, ADLOCO_EUNSUPPORTED, "block_product: too many tiles for one launch");
  p.tiles_m = int(tm);
  p.tiles_n = int(tn);
  p.pieces = c.pieces;
  const int64_t row = (p.pieces > 1 ? 4 : edge / 32) * (int64_t)es;
  p.vec = reinterpret_cast<uintptr_t>(out) % row == 0 && os * (int64_t)es % row == 0;
  hipEvent_t ev = prof_begin(ctx, st);
  const hipError_t e = few ? (dtype == ADLOCO_BF16 ? launch_few<__bf16>(p, st) : dtype == ADLOCO_F16 ? launch_few<_Float16>(p, st)
                                                                                  : launch_few<float>(p, st))
                       : dtype == ADLOCO_BF16 ? launch_product<__bf16>(p, large, exact, st)
                       : dtype == ADLOCO_F16 ? launch_product<_Float16>(p, large, exact, st) : launch_product<float>(p, large, exact, st);
  prof_end(ctx, kProfProduct, ev, st);
  if (e != hipSuccess) return fail(ctx, ADLOCO_EHIP, "block_product launch failed: %s", hipGetErrorString(e));
  return ADLOCO_OK;
}
