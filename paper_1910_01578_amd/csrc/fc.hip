// FC layers with bias, activation and residual in the product's epilogue, and their
// backward.  x [M, K], W [N, K]:
//   a = act(x W^T + b),  y = a + residual
//   dP = dy where a > 0 (ReLU) or dy,  dx = dP W,  dW = dP^T x,  db = sum_rows dP
//
// fp32 goes through the update step's products (train_gemm.hip: three bf16 planes an
// operand), or k_fc_any_f32 (the same planes, any width and alignment).  bf16 has two
// kernels here:
//   k_fc_tile  128 x 128 to 256 x 256 tiles, k in stages of 32 filled by direct loads.
//              The operands stay in their memory order; one whose contraction dimension
//              is not the fast one (W in dx, both in dW) is read by transposing LDS reads.
//              (k_fc_any: the same through registers, for operands of odd alignment.)
//   k_fc_few   few results: 16 outputs of up to 64 rows a work-group, k dealt to its 8
//              waves, no LDS but for the waves' sums.  What bounds it: reading W.
// Measured, bf16: 52,000 rows of 256 to 1,024 with ReLU 43 us (614 TFLOP/s; its 134 MB at the
// rate of a copy, 27); 16,384 of 2,048 to 2,048 with a residual 118 to 135 us (1,020 to 1,160
// TFLOP/s, as the clock holds); dX and dW of the former 41 and 42 us, dy's selection 49; one
// row of 256 to 1,024 2.8 us, a launch.  fp32, 2,503 rows of 131 to 517: 9.6 us.
// Both add in fp32 and round once.  dP has no rounding of its own (a selection), so dW
// and db, which are fp32, are sums of exact products.
#include <algorithm>
#include <type_traits>

#include "lds_dma.h"
#include "op_common.h"
#include "op_kernels.h"
#include "train_kernels.h"

namespace gdp {
namespace op {

namespace {

// C(m, n) = sum_k A(m, k) B(n, k).
struct FcProduct {
  const bf16 *a, *b;
  int64_t lda, ldb;
  int M, N, K;
  int mt, nt;                          // tiles
  int splits, k_per_split;             // pieces of the contraction
  // epilogue of bf16 results
  const bf16 *bias, *res;
  int64_t ldr;
  bf16 *c, *act_out;
  int64_t ldc, ldact;
  int relu;
  // fp32 results (dW): split z's sums at f + z M N; row sums of A (db) at rowsum + z M, or NULL
  float *f, *rowsum;
};

constexpr int kStep = 32;              // k of one LDS stage
__device__ const uint4 kZeros = {0, 0, 0, 0};

// One operand's stage in LDS: R rows x 32 k.  TR false: k is the fast dimension, an LDS
// row is 32 k of one row; true: an LDS row is R rows of one k.  16-byte granules of an LDS
// row are permuted so that fragment reads (plain: 16 rows x 4 granules; transposing: rows
// {8 g + 0..3} x 2 granules) fall in distinct banks.
template <bool TR, int R, int NT>
struct OpTile {
  static constexpr int GPR = TR ? R / 8 : kStep / 8, PER = R * kStep / 8 / NT, kBytes = R * kStep * 2;
  static __device__ __forceinline__ int key(int r) { return TR ? ((r & 3) | ((r >> 1) & 4)) << 1 : ((r >> 2) ^ (r >> 1)) & 3; }
  static __device__ __forceinline__ int pos(int i) { return ((int)(threadIdx.x >> 6) * PER + i) * 64 + (int)(threadIdx.x & 63); }
  static __device__ __forceinline__ int row(int i) { return pos(i) / GPR; }
  static __device__ __forceinline__ int gran(int i) { return (pos(i) % GPR) ^ key(row(i)); }
  // rows r0 + (lane & 15), k = 8 (lane / 16) + [0, 8)
  static __device__ __forceinline__ bf16x8 frag(const char* lds, int r0, int col, int g4) {
    if constexpr (!TR) {
      const int r = r0 + col;
      return *reinterpret_cast<const bf16x8*>(lds + r * (kStep * 2) + ((g4 ^ key(r)) << 4));
    } else {
      const int k = 8 * g4 + (col >> 2), c = r0 + 4 * (col & 3);
      const char* p = lds + (c % 8) * 2;
      return join8(read_tr16(p + k * (R * 2) + (((c / 8) ^ key(k)) << 4)),
                   read_tr16(p + (k + 4) * (R * 2) + (((c / 8) ^ key(k + 4)) << 4)));
    }
  }
};

// A WM x WN block of C in a wave's registers: 16 x 16 blocks formed transposed, so that a
// lane holds 4 consecutive columns of one row.
template <int WM, int WN, bool F32>
struct Block {
  static constexpr int NI = WM / 16, NJ = WN / 16;
  f32x4 acc[NI][NJ], ones[F32 ? NI : 1];
  // bias(j, v): the lane's 4 columns of blocks j (bf16 results), else zeros
  template <typename Bias>
  __device__ __forceinline__ void clear(Bias bias) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      f32x4 v = zero4();
      if constexpr (!F32) bias(j, v);
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i][j] = v;
    }
#pragma unroll
    for (int i = 0; i < (F32 ? NI : 1); ++i) ones[i] = zero4();
  }
  // row block i of one stage; sums: rowsum too
  __device__ __forceinline__ void add(int i, const bf16x8& a, const bf16x8 (&b)[NJ], bool sums) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = mma16(b[j], a, acc[i][j]);
    if constexpr (F32) {
      if (sums) {
        bf16x8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = (bf16)1.0f;
        ones[i] = mma16(one, a, ones[i]);
      }
    }
  }
  // Activation, residual and stores, rows from m0, columns from n0.  Two neighbouring 16 x 16
  // blocks exchange lane rows so that a lane holds 8 consecutive columns: 16-byte accesses,
  // 64 bytes a row.  PART: N may end inside a vector.  PLAIN: neither residual nor act_out.  A residual is loaded in
  // batches before their stores: a load behind a store that may alias it waits.
  template <bool PART, bool PLAIN>
  __device__ __forceinline__ void store_as(const FcProduct& g, int m0, int n0, int z, int col, int g4, bool sums) const {
    constexpr int NP = NJ / 2, NR = 8 / NP;                // 8 vectors of residual at a time
    const int n = n0 + 16 * (g4 & 1) + 8 * (g4 >> 1);      // of pair 0; pair p: 32 p further
    const float least = g.relu ? 0.f : -INFINITY;
    bf16* c = F32 ? nullptr : g.c + (int64_t)(m0 + col) * g.ldc + n;
#pragma unroll
    for (int h = 0; h < NI; h += NR) {
      Vec16<bf16> res[PLAIN ? 1 : NR][PLAIN ? 1 : NP];
      if constexpr (!PLAIN) {
        if (g.res) {
#pragma unroll
          for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int jp = 0; jp < NP; ++jp) {
              const int m = m0 + 16 * (h + i) + col, left = g.N - n - 32 * jp;
              if (m < g.M && left > 0) res[i][jp] = load16_part(g.res + (int64_t)m * g.ldr + n + 32 * jp, PART ? left : 8);
            }
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int m = m0 + 16 * (h + i) + col;
#pragma unroll
        for (int jp = 0; jp < NP; ++jp) {
          float v[8];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float lo = acc[h + i][2 * jp][r], hi = acc[h + i][2 * jp + 1][r];
            const auto t = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi),
                                                            false, false);
            const uint32_t own = t[0], other = t[1];       // (a bit cast of the element itself takes element 0)
            v[r] = __builtin_bit_cast(float, own);
            v[4 + r] = __builtin_bit_cast(float, other);
          }
          if (m >= g.M || n + 32 * jp >= g.N) continue;
          const int left = PART ? g.N - n - 32 * jp : 8;
          if constexpr (F32) {
            float* p = g.f + ((int64_t)z * g.M + m) * g.N + n + 32 * jp;
            Vec16<float> lo, hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              lo.v[e] = v[e];
              hi.v[e] = v[4 + e];
            }
            store16_part(p, lo, left);
            if (left > 4) store16_part(p + 4, hi, left - 4);
          } else {
            Vec16<bf16> o;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = __builtin_elementwise_maximum(v[e], least);             // NaN stays
              o.v[e] = (bf16)v[e];
            }
            if constexpr (!PLAIN) {
              if (g.act_out) store16_part(g.act_out + (int64_t)m * g.ldact + n + 32 * jp, o, left);
              if (g.res) {
#pragma unroll
                for (int e = 0; e < 8; ++e) o.v[e] = (bf16)(v[e] + to_f32(res[i][jp].v[e]));
              }
            }
            store16_part(c + 32 * jp, o, left);
          }
        }
        if constexpr (F32) {
          if (sums && g4 == 0 && m < g.M) g.rowsum[(int64_t)z * g.M + m] = ones[h + i][0];
        } else {
          c += 16 * g.ldc;
        }
      }
    }
  }
  template <bool PART>
  __device__ __forceinline__ void store(const FcProduct& g, int m0, int n0, int z, int col, int g4, bool sums) const {
    if (F32 || (!g.res && !g.act_out)) store_as<PART, true>(g, m0, n0, z, col, g4, sums);
    else store_as<PART, false>(g, m0, n0, z, col, g4, sums);
  }
};

// Four columns' bias by single loads.
__device__ __forceinline__ f32x4 bias_at_column(const FcProduct& g, int n) {
  f32x4 v = zero4();
  if (g.bias) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = to_f32(g.bias[min(n + r, g.N - 1)]);
  }
  return v;
}

// Tile t of the product, columns first, then rows, then pieces: neighbours share A's rows
// (dW: the rows of both).
template <int BM, int BN>
struct TileAt {
  int m0, n0, z, kb, K;
  __device__ __forceinline__ TileAt(const FcProduct& g, int t) {
    n0 = t % g.nt * BN;
    m0 = t / g.nt % g.mt * BM;
    z = t / (g.nt * g.mt);
    kb = z * g.k_per_split;
    K = min(g.K - kb, g.k_per_split);
  }
};

// One operand's way from memory to a work-group's stages: the granules of this lane, each
// load's place a constant past M0 and past the address alike.
template <typename O>
struct Feed {
  static constexpr bool TR = O::GPR > 4;
  static constexpr int kBack = 4096;                       // keeps 32-bit offsets less those constants positive
  const char* p;                                           // the next stage, less kBack
  int64_t step;                                            // bytes from stage to stage
  uint32_t off[O::PER];
  __device__ __forceinline__ void aim(const bf16* first, int64_t ld, int rows) {
    p = reinterpret_cast<const char*>(first) - kBack;
    step = TR ? ld * (kStep * 2) : kStep * 2;
    // past the edge: the last row (granule) again, its results are not stored
#pragma unroll
    for (int i = 0; i < O::PER; ++i)
      off[i] = (uint32_t)((TR ? O::row(i) * ld + min(O::gran(i) * 8, (rows - 1) & ~7)
                              : min(O::row(i), rows - 1) * ld + O::gran(i) * 8) * 2) + kBack - i * 1024;
  }
  // the next stage to LDS address `to` (of this wave's first granule); left: k from there on
  __device__ __forceinline__ void fetch(uint32_t to, int left) {
    static_assert(O::PER == 2 || O::PER == 4, "loads a lane");
    if (left >= kStep) {
      const dma::gptr_t base = dma::uniform_base(p);
      if constexpr (O::PER == 2) dma::dma16x2(base, off[0], off[1], to);
      else dma::dma16x4(base, off[0], off[1], off[2], off[3], to);
    } else {
      const char* at[O::PER];
#pragma unroll
      for (int i = 0; i < O::PER; ++i)
        at[i] = (TR ? O::row(i) : O::gran(i) * 8) < left ? p + off[i] : reinterpret_cast<const char*>(&kZeros) - i * 1024;
      if constexpr (O::PER == 2) dma::dma16x2(at[0], at[1], to);
      else dma::dma16x4(at[0], at[1], at[2], at[3], to);
    }
    p += step;
  }
};

// Aligned operands.  A work-group walks its tiles in one stream of 32-k stages: direct
// loads run NS - 1 stages ahead of the matrix instructions, across the ends of tiles, so
// that a short contraction does not wait for its first loads and an epilogue overlaps the
// next tile's.  A stage past the contraction's end reads zeros.  The bias comes with the
// stages.  Fragments of A are read two row blocks ahead of their products.
// A step is short (16 or 32 matrix instructions a wave): what it does beside them, scalar
// instructions too, shows.  PART: the results' columns may end inside a vector (the bias then
// comes by single loads).
template <bool ATR, bool BTR, bool PART, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64, 2) void k_fc_tile(FcProduct g, int tiles) {
  constexpr int NT = BM / WM * (BN / WN) * 64;
  constexpr bool F32 = ATR;            // dW
  using TA = OpTile<ATR, BM, NT>;
  using TB = OpTile<BTR, BN, NT>;
  constexpr int kStage = TA::kBytes + TB::kBytes, kLoads = TA::PER + TB::PER;
  constexpr int NI = WM / 16, NJ = WN / 16;
  __shared__ __attribute__((aligned(1024))) char lds[NS * kStage];
  __shared__ __attribute__((aligned(16))) char s_bias[2][F32 ? 16 : BN * 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g4 = lane >> 4;
  const int mw = wave / (BN / WN) * WM, nw = wave % (BN / WN) * WN;
  // each XCD takes a run of tiles, its work-groups take them in turn
  const int groups = (int)gridDim.x / kNumXcd, xcd = blockIdx.x % kNumXcd;
  const int per = tiles / kNumXcd, rem = tiles % kNumXcd;
  const int t_end = (xcd + 1) * per + min(xcd + 1, rem);
  const int t_first = xcd * per + min(xcd, rem) + (int)blockIdx.x / kNumXcd;
  if (t_first >= t_end) return;

  Feed<TA> feed_a;
  Feed<TB> feed_b;
  int left = 0, parity = 0;                                // of the tile that is loaded
  auto aim = [&](int tile) {
    const TileAt<BM, BN> t(g, tile);
    left = t.K;
    feed_a.aim(g.a + (ATR ? (int64_t)t.kb * g.lda + t.m0 : (int64_t)t.m0 * g.lda + t.kb), g.lda, g.M - t.m0);
    feed_b.aim(g.b + (BTR ? (int64_t)t.kb * g.ldb + t.n0 : (int64_t)t.n0 * g.ldb + t.kb), g.ldb, g.N - t.n0);
    if constexpr (!F32 && !PART) {
      if (wave == 0 && lane < BN / 8) {                    // this tile's bias, older than its first stage
        const int n = t.n0 + lane * 8;
        const void* from = g.bias && n < g.N ? static_cast<const void*>(g.bias + n) : &kZeros;
        dma::dma16_lane(from, s_bias[parity]);
      }
      parity ^= 1;
    }
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;          // (a generic LDS address's low word is the LDS offset)
  auto fetch = [&](int at) {                               // the next stage to byte `at` of the ring
    feed_a.fetch(lds0 + at + wave * (TA::PER * 1024), left);
    feed_b.fetch(lds0 + at + TA::kBytes + wave * (TB::PER * 1024), left);
    left -= kStep;
  };
  int now = 0, free = (NS - 1) * kStage, bias_at = 0;      // the stage to be multiplied, the one before it
  auto turn = [&]() {
    free = now;
    now = now == (NS - 1) * kStage ? 0 : now + kStage;
  };
  Block<WM, WN, F32> b;
  bf16x8 fa[4];
  auto read_b = [&](const char* p, int j) { return TB::frag(p + TA::kBytes, nw + 16 * j, col, g4); };
  auto step = [&](bool sums) {
    dma::wait_vm_barrier<(NS - 2) * kLoads>();             // this stage is in, the last one has been read
    fetch(free);
    const char* p = lds + now;
    bf16x8 fb[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) fb[j] = read_b(p, j);
    fa[0] = TA::frag(p, mw, col, g4);
    fa[1] = TA::frag(p, mw + 16, col, g4);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (i + 2 < NI) fa[(i + 2) % 4] = TA::frag(p, mw + 16 * (i + 2), col, g4);
      b.add(i, fa[i % 4], fb, sums);
    }
    turn();
  };
  aim(t_first);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) fetch(s * kStage);
  // the first tile's bias is in (a later one is older than a stage waited for)
  if constexpr (!F32 && !PART) dma::wait_vm_barrier<(NS - 1) * kLoads>();
  for (int t = t_first; t < t_end; t += groups) {
    const TileAt<BM, BN> at(g, t);
    const bool sums = F32 && g.rowsum && at.n0 == 0 && nw == 0;
    b.clear([&](int j, f32x4& v) {
      if constexpr (PART) {
        v = bias_at_column(g, at.n0 + nw + 16 * j + 4 * g4);
      } else {
        union {
          uint2 u;
          bf16 h[4];
        } x;
        x.u = *reinterpret_cast<const uint2*>(s_bias[bias_at] + (nw + 16 * j + 4 * g4) * 2);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = to_f32(x.h[r]);
      }
    });
    // the last NS - 1 steps load the next tile's first stages (behind the last tile: zeros)
    const int steps = max(NS - 1, (at.K + kStep - 1) / kStep);
    for (int s = 0; s < steps - (NS - 1); ++s) step(sums);
    left = 0;
    if (t + groups < t_end) aim(t + groups);
    for (int s = 0; s < NS - 1; ++s) step(sums);
    b.template store<PART>(g, at.m0 + mw, at.n0 + nw, at.z, col, g4, sums);
    bias_at ^= 1;
  }
  dma::wait_loads_then_barrier();                          // no direct load outlives the work-group
}

// Operands of any alignment and contraction length: 128 x 128 tiles, stages through
// registers, two LDS buffers.
template <bool ATR, bool BTR>
__global__ __launch_bounds__(256, 2) void k_fc_any(FcProduct g) {
  constexpr int BT = 128;
  constexpr bool F32 = ATR;
  using TA = OpTile<ATR, BT, 256>;
  using TB = OpTile<BTR, BT, 256>;
  __shared__ __attribute__((aligned(1024))) char lds[2 * (TA::kBytes + TB::kBytes)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int mw = (wave >> 1) * 64, nw = (wave & 1) * 64;
  const TileAt<BT, BT> at(g, xcd_remap(blockIdx.x, gridDim.x));
  const bf16* pa = g.a + (ATR ? (int64_t)at.kb * g.lda + at.m0 : (int64_t)at.m0 * g.lda + at.kb);
  const bf16* pb = g.b + (BTR ? (int64_t)at.kb * g.ldb + at.n0 : (int64_t)at.n0 * g.ldb + at.kb);
  Vec16<bf16> va[TA::PER], vb[TB::PER];
  auto load = [&](auto tile, const bf16* p, int64_t ld, int rows, int s, auto& v) {
    using O = decltype(tile);
    constexpr bool TR = O::GPR > 4;
#pragma unroll
    for (int i = 0; i < O::PER; ++i) {
      const int k = s * kStep + (TR ? O::row(i) : O::gran(i) * 8), r = TR ? O::gran(i) * 8 : min(O::row(i), rows - 1);
      const int left = TR ? (k < at.K ? rows - r : 0) : at.K - k;
      if (left > 0) v[i] = load16_part(p + (TR ? (int64_t)k * ld + r : (int64_t)r * ld + k), left);
      else *reinterpret_cast<uint4*>(&v[i]) = make_uint4(0, 0, 0, 0);
    }
  };
  auto fetch = [&](int s) {
    load(TA(), pa, g.lda, g.M - at.m0, s, va);
    load(TB(), pb, g.ldb, g.N - at.n0, s, vb);
  };
  auto put = [&](int s) {
    char* p = lds + (s & 1) * (TA::kBytes + TB::kBytes);
#pragma unroll
    for (int i = 0; i < TA::PER; ++i) *reinterpret_cast<uint4*>(p + TA::pos(i) * 16) = *reinterpret_cast<const uint4*>(&va[i]);
    p += TA::kBytes;
#pragma unroll
    for (int i = 0; i < TB::PER; ++i) *reinterpret_cast<uint4*>(p + TB::pos(i) * 16) = *reinterpret_cast<const uint4*>(&vb[i]);
  };
  const int steps = (at.K + kStep - 1) / kStep;
  const bool sums = F32 && g.rowsum && at.n0 == 0 && nw == 0;
  Block<64, 64, F32> b;
  b.clear([&](int j, f32x4& v) { v = bias_at_column(g, at.n0 + nw + 16 * j + 4 * g4); });
  fetch(0);
  put(0);
  if (steps > 1) fetch(1);
  for (int s = 0; s < steps; ++s) {
    __syncthreads();
    if (s + 1 < steps) put(s + 1);
    if (s + 2 < steps) fetch(s + 2);
    const char* p = lds + (s & 1) * (TA::kBytes + TB::kBytes);
    bf16x8 fb[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) fb[j] = TB::frag(p + TA::kBytes, nw + 16 * j, col, g4);
#pragma unroll
    for (int i = 0; i < 4; ++i) b.add(i, TA::frag(p, mw + 16 * i, col, g4), fb, sums);
  }
  b.template store<true>(g, at.m0 + mw, at.n0 + nw, at.z, col, g4, sums);
}

// fp32 of any alignment, both results from one product: 64 x 64 tiles, a wave 32 x 32 of
// them, k in stages of 32 through registers into two LDS buffers, three bf16 planes each.
// What bounds it: six products and two splits a stage between barriers, three work-groups a
// CU (12,001 rows of 515 to 1,003: 101 us, 123 TFLOP/s).
template <typename T>
struct FewArgs {
  const T *x, *w, *bias, *res;
  T *y, *act_out;
  int64_t ldx, ldr, ldy, ldact;
  int M, N, K, relu;
};
__global__ __launch_bounds__(256) void k_fc_any_f32(FewArgs<float> g) {
  constexpr int BT = 64;
  using O = OpTile<false, BT, 256>;
  constexpr int kOperand = 3 * O::kBytes;
  __shared__ __attribute__((aligned(1024))) char lds[4 * kOperand];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int mw = (wave >> 1) * 32, nw = (wave & 1) * 32;
  const int logical = xcd_remap(blockIdx.x, gridDim.x), nt = (g.N + BT - 1) / BT;
  const int m0 = logical / nt * BT, n0 = logical % nt * BT;
  const int k0 = O::gran(0) * 8;
  const float* px = g.x + (int64_t)min(m0 + O::row(0), g.M - 1) * g.ldx;
  const float* pw = g.w + (int64_t)min(n0 + O::row(0), g.N - 1) * g.K;
  Vec16<float> vx[2], vw[2];
  auto load = [&](const float* p, int k, Vec16<float> (&v)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = k + 4 * i;
      if (at < g.K) v[i] = load16_part(p + at, g.K - at);
      else *reinterpret_cast<uint4*>(&v[i]) = make_uint4(0, 0, 0, 0);
    }
  };
  auto fetch = [&](int s) {
    load(px, s * kStep + k0, vx);
    load(pw, s * kStep + k0, vw);
  };
  auto put_one = [&](char* to, const Vec16<float> (&v)[2]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = v[0].v[i];
      f[4 + i] = v[1].v[i];
    }
    const Operand<3> o = operand(f);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<bf16x8*>(to + q * O::kBytes + O::pos(0) * 16) = o.p[q];
  };
  auto put = [&](int s) {
    char* p = lds + (s & 1) * (2 * kOperand);
    put_one(p, vx);
    put_one(p + kOperand, vw);
  };
  auto frag = [&](const char* p, int r0) {
    Operand<3> o;
#pragma unroll
    for (int q = 0; q < 3; ++q) o.p[q] = O::frag(p + q * O::kBytes, r0, col, g4);
    return o;
  };
  f32x4 top[2][2], low[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) top[i][j] = low[i][j] = zero4();
  const int steps = (g.K + kStep - 1) / kStep;
  fetch(0);
  put(0);
  if (steps > 1) fetch(1);
  for (int s = 0; s < steps; ++s) {
    __syncthreads();
    if (s + 1 < steps) put(s + 1);
    if (s + 2 < steps) fetch(s + 2);
    const char* p = lds + (s & 1) * (2 * kOperand);
    const Operand<3> b[2] = {frag(p + kOperand, nw), frag(p + kOperand, nw + 16)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const Operand<3> a = frag(p, mw + 16 * i);
#pragma unroll
      for (int j = 0; j < 2; ++j) mma_planes(b[j], a, top[i][j], low[i][j]);
    }
  }
  const float least = g.relu ? 0.f : -INFINITY;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int n = n0 + nw + 16 * j + 4 * g4, left = g.N - n;
    if (left <= 0) continue;
    Vec16<float> bias = {};
    if (g.bias) bias = load16_part(g.bias + n, left);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int m = m0 + mw + 16 * i + col;
      if (m >= g.M) continue;
      Vec16<float> v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float sum = top[i][j][r] + low[i][j][r];
        if (!(sum * 0.f == 0.f) && r < left) {             // an infinity, or a value that rounds to a bf16 one, has no planes
          const float *x = g.x + (int64_t)m * g.ldx, *w = g.w + (int64_t)(n + r) * g.K;
          sum = 0.f;
          for (int k = 0; k < g.K; ++k) sum = fmaf(x[k], w[k], sum);
        }
        v.v[r] = __builtin_elementwise_maximum(sum + bias.v[r], least);      // NaN stays
      }
      if (g.act_out) store16_part(g.act_out + (int64_t)m * g.ldact + n, v, left);
      if (g.res) {
        const Vec16<float> t = load16_part(g.res + (int64_t)m * g.ldr + n, left);
#pragma unroll
        for (int r = 0; r < 4; ++r) v.v[r] += t.v[r];
      }
      store16_part(g.y + (int64_t)m * g.ldy + n, v, left);
    }
  }
}

// The splits' sums in order, in double.  entries of dW, then of db.
__global__ __launch_bounds__(256) void k_fc_join(const float* __restrict__ f, const float* __restrict__ rowsum, int splits,
                                                 int64_t mn, int m, float* __restrict__ dw, float* __restrict__ db) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= mn + m) return;
  const bool w = i < mn;
  if (w ? !dw : !db) return;
  const float* p = w ? f + i : rowsum + (i - mn);
  const int64_t step = w ? mn : m;
  double t = 0.0;
#pragma unroll 8
  for (int z = 0; z < splits; ++z) t += (double)p[z * step];
  if (w) dw[i] = (float)t;
  else db[i - mn] = (float)t;
}

// Copies of operands in the workspace: rows of ldd elements with zeros behind the cols-th,
// and with a gate only the elements where that is above 0 (dP; NaN is not).
template <typename T>
struct PadJob {
  const T *src, *gate;
  int64_t ld, ldgate, ldd;
  int rows, cols;
  T* dst;
};
template <typename T>
struct PadJobs {
  PadJob<T> job[3];
};
template <typename T>
__global__ __launch_bounds__(256) void k_fc_pad(PadJobs<T> jobs) {
  constexpr int V = Vec16<T>::N;
  const PadJob<T>& j = jobs.job[blockIdx.z];
  const int n = (blockIdx.x * 64 + (threadIdx.x & 63)) * V;
  if (n >= j.ldd) return;
  for (int64_t r = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6); r < j.rows; r += (int64_t)gridDim.y * 4) {
    Vec16<T> t = load16_part(j.src + r * j.ld + n, j.cols - n);
    if (j.gate) {
      const Vec16<T> x = load16_part(j.gate + r * j.ldgate + n, j.cols - n);
#pragma unroll
      for (int e = 0; e < V; ++e) t.v[e] = to_f32(x.v[e]) > 0.f ? t.v[e] : (T)0.f;
    }
    store16(j.dst + r * j.ldd + n, t);
  }
}
template <typename T>
hipError_t launch_pad(const PadJobs<T>& jobs, int n, hipStream_t s) {
  if (n == 0) return hipSuccess;
  int64_t wide = 0, rows = 0;
  for (int i = 0; i < n; ++i) {
    wide = std::max(wide, jobs.job[i].ldd);
    rows = std::max<int64_t>(rows, jobs.job[i].rows);
  }
  const unsigned cols = (unsigned)((wide + 64 * Vec16<T>::N - 1) / (64 * Vec16<T>::N));
  const unsigned groups = (unsigned)std::max<int64_t>(1, std::min<int64_t>((rows + 3) / 4, std::max<int64_t>(64, 8192 / cols)));
  hipLaunchKernelGGL((k_fc_pad<T>), dim3(cols, groups, n), dim3(256), 0, s, jobs);
  return hipGetLastError();
}

template <typename T>
__global__ __launch_bounds__(256) void k_fc_add(const T* a, int64_t lda, const T* res, int64_t ldr, int64_t rows, int N, T* y,
                                                int64_t ldy) {
  const int64_t total = rows * N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / N, n = i - r * N;
    y[r * ldy + n] = from_f32<T>(to_f32(a[r * lda + n]) + to_f32(res[r * ldr + n]));
  }
}

// k steps of a wave: 32 bf16 or 16 fp32 values of 16 outputs' and 16 MB rows'; a lane holds
// 16 consecutive bytes of one row of each.  fp32: four 16x16x4 instructions, the i-th
// contracting over element i of the lanes' vectors.
template <typename T> constexpr int few_k() { return 4 * Vec16<T>::N; }
template <typename T>
__device__ __forceinline__ f32x4 few_mma(const Vec16<T>& a, const Vec16<T>& b, f32x4 c) {
  if constexpr (sizeof(T) == 2) {
    c = mma16(as_bf16x8(a), as_bf16x8(b), c);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
  }
  return c;
}

constexpr int kFewWaves = 8;
template <typename T, int MB>
__global__ __launch_bounds__(64 * kFewWaves) void k_fc_few(FewArgs<T> g) {
  constexpr int KS = few_k<T>(), V = Vec16<T>::N, U = MB == 4 ? 2 : 4;
  __shared__ float part[kFewWaves][MB * 16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (MB * 16);
  const T* w = g.w + (int64_t)min(n0 + col, g.N - 1) * g.K + g4 * V;
  const T* x[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) x[b] = g.x + (int64_t)min(m0 + 16 * b + col, g.M - 1) * g.ldx + g4 * V;
  f32x4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) acc[b] = zero4();
  auto fetch = [&](const T* p, int k) {
    const int left = g.K - k - g4 * V;
    Vec16<T> t = {};
    if (left > 0) t = load16_part(p + k, left);
    return t;
  };
  for (int k = wave * KS; k < g.K; k += kFewWaves * KS * U) {
    Vec16<T> fw[U], fx[U][MB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fw[u] = fetch(w, k + u * kFewWaves * KS);
#pragma unroll
      for (int b = 0; b < MB; ++b) fx[u][b] = fetch(x[b], k + u * kFewWaves * KS);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < MB; ++b) acc[b] = few_mma(fw[u], fx[u][b], acc[b]);
  }
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) part[wave][16 * b + col][4 * g4 + r] = acc[b][r];
  __syncthreads();
  for (int i = threadIdx.x; i < MB * 256; i += 64 * kFewWaves) {
    const int row = i / 16, m = m0 + row, n = n0 + i % 16;
    if (m >= g.M || n >= g.N) continue;
    float v = 0.f;
#pragma unroll
    for (int p = 0; p < kFewWaves; ++p) v += part[p][row][i % 16];
    if (g.bias) v += to_f32(g.bias[n]);
    if (g.relu) v = v < 0.f ? 0.f : v;
    if (g.act_out) g.act_out[m * g.ldact + n] = from_f32<T>(v);
    if (g.res) v += to_f32(g.res[m * g.ldr + n]);
    g.y[m * g.ldy + n] = from_f32<T>(v);
  }
}

// Direct loads: 16-byte granules, and a tile's rows within 32-bit offsets of its first.
bool dma_ok(const bf16* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1 << 23); }

// Tiles of 256 x 256 (8 waves of 128 x 64, one work-group a CU) and 128 x 256 (4 of 64 x
// 128) do more products a step and LDS byte than 128 x 128 (4 of 64 x 64), where they fill
// the chip.  16,384 rows of 2,048 to 2,048: 118, 139 and 161 us; 52,000 of 256 to 1,024: -,
// 44 and 50 us; of 1,024 to 256 (203 large tiles): -, 38 and 45 us.
template <bool ATR, bool BTR>
hipError_t launch_product(FcProduct g, bool aligned, hipStream_t s) {
  int n = 0;
  auto tiles = [&](int bm, int bn) {
    g.mt = (g.M + bm - 1) / bm;
    g.nt = (g.N + bn - 1) / bn;
    n = (int)((int64_t)g.mt * g.nt * g.splits);
    return n;
  };
  auto grid = [&](int most) { return dim3((unsigned)std::min(most, (n + kNumXcd - 1) / kNumXcd * kNumXcd)); };
  if (!aligned) {
    tiles(128, 128);
    hipLaunchKernelGGL((k_fc_any<ATR, BTR>), dim3((unsigned)n), dim3(256), 0, s, g);
  } else if (g.N % 8 != 0 || (uintptr_t)g.bias % 16 != 0) {
    tiles(128, 128);
    hipLaunchKernelGGL((k_fc_tile<ATR, BTR, true, 128, 128, 64, 64, 4>), grid(512), dim3(256), 0, s, g, n);
  } else if (!ATR && g.K >= 512 && tiles(256, 256) >= 256) {
    if constexpr (!ATR) hipLaunchKernelGGL((k_fc_tile<ATR, BTR, false, 256, 256, 128, 64, 4>), grid(256), dim3(512), 0, s, g, n);
  } else if (!ATR && tiles(128, 256) >= 256) {
    if constexpr (!ATR) hipLaunchKernelGGL((k_fc_tile<ATR, BTR, false, 128, 256, 64, 128, 3>), grid(512), dim3(256), 0, s, g, n);
  } else {
    tiles(128, 128);
    hipLaunchKernelGGL((k_fc_tile<ATR, BTR, false, 128, 128, 64, 64, 4>), grid(512), dim3(256), 0, s, g, n);
  }
  return hipGetLastError();
}

}  // namespace

// Up to 16 rows, or while there are few 16 x 16 blocks of results, k is dealt to a
// work-group's waves instead of walked by one tile's.  bf16, by blocks (of 64 rows a
// work-group) and by tiles: 64 rows of 2,048 to 2,048 11.5 and 21 us, 256 rows (2,048
// blocks) 20.7 and 21.8, 512 rows 38 and 22.5; 512 of 515 to 1,003 12.9 and 24.5; 64 of 256
// to 1,024 3.9 and 5.8.  fp32: 128 rows of 2,048 to 2,048 (1,024 blocks) 24 and 39, 256 rows 45
// and 39; 256 of 256 to 1,024 5.6 and 8.2, 1,024 rows 14.9 and 9.1.
static bool few_rows(int M, int N, size_t bytes) {
  return M <= 16 || (int64_t)((M + 15) / 16) * ((N + 15) / 16) <= (bytes == 2 ? 2048 : 1024);
}

template <typename T>
hipError_t launch_fc(const gdp_fc_layer& f, const T* x, const T* w, const T* b, const T* residual, T* y, T* act_out,
                     hipStream_t s) {
  const int M = (int)f.rows, K = f.in_dim, N = f.out_dim, relu = f.act == GDP_ACT_RELU;
  if (M == 0) return hipSuccess;
  if (few_rows(M, N, sizeof(T))) {
    const FewArgs<T> g = {x, w, b, residual, y, act_out, f.ld_x, f.ld_res, f.ld_y, f.ld_act, M, N, K, relu};
    const dim3 grid((unsigned)(N + 15) / 16, (unsigned)(M + 63) / 64), block(64 * kFewWaves);
    if (M <= 16) hipLaunchKernelGGL((k_fc_few<T, 1>), grid, block, 0, s, g);
    else if (M <= 32) hipLaunchKernelGGL((k_fc_few<T, 2>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((k_fc_few<T, 4>), grid, block, 0, s, g);
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 4) {
    // the update step's product loads and stores whole vectors and takes k in whole stages;
    // element by element it is the slower one (relu of 2,503 rows of 131 to 517: 21 us there, 10
    // here; 12,001 of 515 to 1,003: 213 and 101; 12,000 of 512 to 1,000, whole: 76 and 95)
    auto whole = [](const void* p, int64_t ld) { return !p || (((uintptr_t)p & 15) == 0 && ld % 4 == 0); };
    if (K % 32 != 0 || N % 4 != 0 || !whole(x, f.ld_x) || !whole(w, K) || !whole(y, f.ld_y) || !whole(residual, f.ld_res) ||
        !whole(act_out, f.ld_act)) {
      const FewArgs<T> g = {x, w, b, residual, y, act_out, f.ld_x, f.ld_res, f.ld_y, f.ld_act, M, N, K, relu};
      const int64_t tiles = (int64_t)((M + 63) / 64) * ((N + 63) / 64);
      hipLaunchKernelGGL(k_fc_any_f32, dim3((unsigned)tiles), dim3(256), 0, s, g);
      return hipGetLastError();
    }
    tr::GemmStrided<float, float> g = {x, f.ld_x, 1, w, 1, K, M, N, K, y, f.ld_y};
    g.bias_f = b;
    g.act = relu ? tr::ACT_GATE : tr::ACT_NONE;
    if (residual && act_out) {
      // both arrays from one product: the activation's output, then the sum
      g.c = act_out;
      g.ldc = f.ld_act;
      const hipError_t e = tr::launch_gemm_strided(g, nullptr, 0, s);
      if (e != hipSuccess) return e;
      const int64_t blocks = std::min<int64_t>(((int64_t)M * N + 255) / 256, 8192);
      hipLaunchKernelGGL((k_fc_add<T>), dim3((unsigned)blocks), dim3(256), 0, s, (const T*)act_out, f.ld_act, residual, f.ld_res,
                         f.rows, N, y, f.ld_y);
      return hipGetLastError();
    }
    g.res = residual;
    g.ldr = f.ld_res;
    const hipError_t e = tr::launch_gemm_strided(g, nullptr, 0, s);
    if (e != hipSuccess || !act_out) return e;
    g.c = act_out;                                         // no residual: the output once more
    g.ldc = f.ld_act;
    return tr::launch_gemm_strided(g, nullptr, 0, s);
  } else {
    FcProduct g = {};
    g.a = x;
    g.lda = f.ld_x;
    g.b = w;
    g.ldb = K;
    g.M = M;
    g.N = N;
    g.K = g.k_per_split = K;
    g.splits = 1;
    g.bias = b;
    g.res = residual;
    g.ldr = f.ld_res;
    g.c = y;
    g.ldc = f.ld_y;
    g.act_out = act_out;
    g.ldact = f.ld_act;
    g.relu = relu;
    return launch_product<false, false>(g, dma_ok(x, f.ld_x) && dma_ok(w, K), s);
  }
}

template <typename T>
hipError_t launch_fc_backward(const gdp_fc_layer& f, const FcPlan& p, const T* dy, const T* x, const T* w,
                              const T* act_out, const T* dx_add, T* dx, float* dw, float* db, void* ws, hipStream_t s) {
  const int M = (int)f.rows, K = f.in_dim, N = f.out_dim;
  char* base = static_cast<char*>(ws);
  float* part = reinterpret_cast<float*>(base + p.partial);
  const int64_t mn = (int64_t)N * K;
  if (M == 0) {                                            // no rows: gradients of zero
    hipLaunchKernelGGL(k_fc_join, dim3((unsigned)((mn + N + 255) / 256)), dim3(256), 0, s, (const float*)nullptr,
                       (const float*)nullptr, 0, mn, N, dw, db);
    return hipGetLastError();
  }
  // the operands, or their copies
  int64_t lddy = f.ld_dy, ldx = f.ld_x, ldw = K;
  PadJobs<T> jobs = {};
  int n = 0;
  auto copy = [&](const T*& src, int64_t& ld, const T* gate, int rows, int cols, int64_t ldd, size_t at) {
    if (ldd == 0) return;
    T* dst = reinterpret_cast<T*>(base + at);
    jobs.job[n++] = {src, gate, ld, f.ld_act, ldd, rows, cols, dst};
    src = dst;
    ld = ldd;
  };
  copy(dy, lddy, f.act == GDP_ACT_RELU ? act_out : nullptr, M, N, p.ldp, p.dp);
  if (dw || db) copy(x, ldx, nullptr, M, K, p.ldx, p.x);
  if (dx) copy(w, ldw, nullptr, N, K, p.ldw, p.w);
  hipError_t e = launch_pad(jobs, n, s);
  if (e != hipSuccess) return e;
  if constexpr (sizeof(T) == 4) {
    if (dx) {
      tr::GemmStrided<float, float> g = {dy, lddy, 1, w, ldw, 1, M, K, N, dx, f.ld_dx};
      g.res = dx_add;
      g.ldr = f.ld_dx_add;
      e = tr::launch_gemm_strided(g, nullptr, 0, s);
    }
    if (e != hipSuccess || (!dw && !db)) return e;
    float* out = dw ? dw : part + p.partial_floats;        // db alone: the product's place is scratch
    tr::GemmStrided<float, float> g = {dy, 1, lddy, x, ldx, 1, N, K, M, out, K};
    g.rowsum = db;
    return tr::launch_gemm_strided(g, part, p.partial_floats, s);
  } else {
    FcProduct g = {};
    g.a = dy;
    g.lda = lddy;
    if (dx) {
      FcProduct d = g;
      d.b = w;
      d.ldb = ldw;
      d.M = M;
      d.N = K;
      d.K = d.k_per_split = N;
      d.splits = 1;
      d.res = dx_add;
      d.ldr = f.ld_dx_add;
      d.c = dx;
      d.ldc = f.ld_dx;
      e = launch_product<false, true>(d, dma_ok(dy, lddy) && dma_ok(w, ldw), s);
      if (e != hipSuccess) return e;
    }
    if (!dw && !db) return hipSuccess;
    g.b = x;
    g.ldb = ldx;
    g.M = N;
    g.N = K;
    g.K = M;
    g.splits = p.splits;
    g.k_per_split = p.rows_per_split;
    g.f = part;
    g.rowsum = part + p.splits * mn;
    e = launch_product<true, true>(g, dma_ok(dy, lddy) && dma_ok(x, ldx), s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_fc_join, dim3((unsigned)((mn + N + 255) / 256)), dim3(256), 0, s, (const float*)part,
                       (const float*)g.rowsum, p.splits, mn, N, dw, db);
    return hipGetLastError();
  }
}

#define GDP_FC_INST(T)                                                                                                \
  template hipError_t launch_fc<T>(const gdp_fc_layer&, const T*, const T*, const T*, const T*, T*, T*, hipStream_t); \
  template hipError_t launch_fc_backward<T>(const gdp_fc_layer&, const FcPlan&, const T*, const T*, const T*,         \
                                            const T*, const T*, T*, float*, float*, void*, hipStream_t);
GDP_FC_INST(float)
GDP_FC_INST(bf16)
#undef GDP_FC_INST

}  // namespace op
}  // namespace gdp
