// FC layers with bias, activation and residual in the product's epilogue, and their
// backward.  x [M, K], W [N, K]:
//   a = act(x W^T + b),  y = a + residual
//   dP = dy where a > 0 (ReLU) or dy,  dx = dP W,  dW = dP^T x,  db = sum_rows dP
//
// fp32 goes through the update step's products (train_gemm.hip: three bf16 planes an
// operand).  bf16 has two kernels here:
//   k_fc_tile  128 x 128 or 256 x 256 tiles, k in stages of 32 filled by direct loads.
//              The operands stay in their memory order; one whose contraction dimension
//              is not the fast one (W in dx, both in dW) is read by transposing LDS reads.
//              (k_fc_any: the same through registers, for operands of odd alignment.)
//   k_fc_few   up to 64 rows: 16 outputs a work-group, k dealt to its 8 waves, no LDS
//              but for the waves' sums.  What bounds it: reading W.
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
  const bf16 *a, *b, *gate;            // gate (or NULL): A's elements count where it is above 0
  int64_t lda, ldb, ldgate;
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
      return join8(read_tr16(p + k * (R * 2) + (((c / 8) ^ key(k)) << 4)), read_tr16(p + (k + 4) * (R * 2) + (((c / 8) ^ key(k + 4)) << 4)));
    }
  }
};

// bf16 values of x where g is above 0 (NaN is not), else 0: packed 16-bit integer
// operations on the bits, as the values above 0 are 0x0001 .. 0x7f80.
__device__ __forceinline__ bf16x8 gated(const bf16x8& x, const bf16x8& g) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
  union V {
    bf16x8 q;
    u16x2 h[4];
    uint32_t u[4];
  } v, m;
  v.q = x;
  m.q = g;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u16x2 t = __builtin_elementwise_min((u16x2)(m.h[i] - (uint16_t)1), (u16x2)(uint16_t)0x7f80) - (uint16_t)0x7f80;
    const i16x2 keep = __builtin_bit_cast(i16x2, t) >> (int16_t)15;
    v.u[i] &= __builtin_bit_cast(uint32_t, keep);
  }
  return v.q;
}

// A WM x WN block of C in a wave's registers: 16 x 16 blocks formed transposed, so that a
// lane holds 4 consecutive columns of one row.
template <int WM, int WN, bool F32>
struct Block {
  static constexpr int NI = WM / 16, NJ = WN / 16;
  f32x4 acc[NI][NJ], ones[F32 ? NI : 1];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = zero4();
#pragma unroll
    for (int i = 0; i < (F32 ? NI : 1); ++i) ones[i] = zero4();
  }
  // one stage; sums: rowsum too
  template <typename TA, typename TB>
  __device__ __forceinline__ void step(const char* sa, const char* sb, const char* sg, int mw, int nw, int col, int g4, bool sums) {
    bf16x8 fa[NI], fb[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) fb[j] = TB::frag(sb, nw + 16 * j, col, g4);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      fa[i] = TA::frag(sa, mw + 16 * i, col, g4);
      if (sg) fa[i] = gated(fa[i], TA::frag(sg, mw + 16 * i, col, g4));
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = mma16(fb[j], fa[i], acc[i][j]);
    if constexpr (F32) {
      if (sums) {
        bf16x8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = (bf16)1.0f;
#pragma unroll
        for (int i = 0; i < NI; ++i) ones[i] = mma16(one, fa[i], ones[i]);
      }
    }
  }
  // Bias, activation, residual and stores.  Two neighbouring 16 x 16 blocks exchange lane
  // rows so that a lane holds 8 consecutive columns: 16-byte accesses, 64 bytes a row.
  __device__ __forceinline__ void store(const FcProduct& g, int m0, int n0, int z, int col, int g4, bool sums) const {
    float bias[NJ][4];
    if constexpr (!F32) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int n = n0 + 16 * j + 4 * g4 + r;
          bias[j][r] = g.bias && n < g.N ? to_f32(g.bias[n]) : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int m = m0 + 16 * i + col;
#pragma unroll
      for (int jp = 0; jp < NJ / 2; ++jp) {
        float v[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = acc[i][2 * jp][r] + (F32 ? 0.f : bias[2 * jp][r]), y = acc[i][2 * jp + 1][r] + (F32 ? 0.f : bias[2 * jp + 1][r]);
          const auto t = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y), false, false);
          const uint32_t own = t[0], other = t[1];         // (a bit cast of the element itself takes element 0)
          v[r] = __builtin_bit_cast(float, own);
          v[4 + r] = __builtin_bit_cast(float, other);
        }
        const int n = n0 + 32 * jp + 16 * (g4 & 1) + 8 * (g4 >> 1), left = g.N - n;
        if (m >= g.M || left <= 0) continue;
        if constexpr (F32) {
          float* p = g.f + ((int64_t)z * g.M + m) * g.N + n;
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
            if (g.relu) v[e] = v[e] < 0.f ? 0.f : v[e];    // NaN stays
            o.v[e] = (bf16)v[e];
          }
          if (g.act_out) store16_part(g.act_out + (int64_t)m * g.ldact + n, o, left);
          if (g.res) {
            const Vec16<bf16> r = load16_part(g.res + (int64_t)m * g.ldr + n, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) o.v[e] = (bf16)(v[e] + to_f32(r.v[e]));
          }
          store16_part(g.c + (int64_t)m * g.ldc + n, o, left);
        }
      }
      if constexpr (F32) {
        if (sums && g4 == 0 && m < g.M) g.rowsum[(int64_t)z * g.M + m] = ones[i][0];
      }
    }
  }
};

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

// Aligned operands.  A work-group walks its tiles in one stream of 32-k stages: direct
// loads run NS - 1 stages ahead of the matrix instructions, across the ends of tiles, so
// that a short contraction does not wait for its first loads and its epilogue overlaps the
// next tile's.  A stage past the contraction's end reads zeros.
template <bool ATR, bool BTR, bool GATE, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64, 2) void k_fc_tile(FcProduct g, int tiles) {
  constexpr int NT = BM / WM * (BN / WN) * 64;
  constexpr bool F32 = ATR;            // dW
  using TA = OpTile<ATR, BM, NT>;
  using TB = OpTile<BTR, BN, NT>;
  constexpr int kStage = TA::kBytes * (GATE ? 2 : 1) + TB::kBytes, kLoads = TA::PER * (GATE ? 2 : 1) + TB::PER;
  __shared__ __attribute__((aligned(1024))) char lds[NS * kStage];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g4 = lane >> 4;
  const int mw = wave / (BN / WN) * WM, nw = wave % (BN / WN) * WN;
  // each XCD takes a run of tiles, its work-groups take them in turn
  const int groups = (int)gridDim.x / kNumXcd, xcd = blockIdx.x % kNumXcd;
  const int per = tiles / kNumXcd, rem = tiles % kNumXcd;
  const int t_end = (xcd + 1) * per + min(xcd + 1, rem);
  const int t_first = xcd * per + min(xcd, rem) + (int)blockIdx.x / kNumXcd;
  if (t_first >= t_end) return;

  // where the loads are: tile lt, stage ls of it
  int lt = t_first, ls = 0, lsteps = 0, lk = 0;
  const bf16 *pa = nullptr, *pb = nullptr, *pg = nullptr;
  uint32_t oa[TA::PER], ob[TB::PER], og[TA::PER];
  auto aim = [&]() {
    const TileAt<BM, BN> t(g, lt);
    lsteps = (t.K + kStep - 1) / kStep;
    lk = t.K;
    ls = 0;
    auto offsets = [&](auto tile, int64_t ld, int rows, auto& off) {
      using O = decltype(tile);
      // past the edge: the last row (granule) again, its results are not stored
#pragma unroll
      for (int i = 0; i < O::PER; ++i)
        off[i] = O::GPR > 4 ? (uint32_t)((O::row(i) * ld + min(O::gran(i) * 8, (rows - 1) & ~7)) * 2)
                            : (uint32_t)((min(O::row(i), rows - 1) * ld + O::gran(i) * 8) * 2);
    };
    pa = g.a + (ATR ? (int64_t)t.kb * g.lda + t.m0 : (int64_t)t.m0 * g.lda + t.kb);
    pb = g.b + (BTR ? (int64_t)t.kb * g.ldb + t.n0 : (int64_t)t.n0 * g.ldb + t.kb);
    offsets(TA(), g.lda, g.M - t.m0, oa);
    offsets(TB(), g.ldb, g.N - t.n0, ob);
    if constexpr (GATE) {
      pg = g.gate + (ATR ? (int64_t)t.kb * g.ldgate + t.m0 : (int64_t)t.m0 * g.ldgate + t.kb);
      offsets(TA(), g.ldgate, g.M - t.m0, og);
    }
  };
  auto fetch = [&](int slot) {                             // the next stage; past the last one: that one again
    char* to = lds + slot * kStage;
    auto load = [&](auto tile, const bf16* p, int64_t ld, const auto& off, char* at) {
      using O = decltype(tile);
      const bf16* q = p + (int64_t)ls * kStep * (O::GPR > 4 ? ld : 1);
      if ((ls + 1) * kStep <= lk) {
        const dma::gptr_t base = dma::uniform_base(q);
#pragma unroll
        for (int i = 0; i < O::PER; ++i) dma::dma16(base, off[i], at + (wave * O::PER + i) * 1024);
      } else {
        const int left = lk - ls * kStep;
#pragma unroll
        for (int i = 0; i < O::PER; ++i) {
          const bool in = (O::GPR > 4 ? O::row(i) : O::gran(i) * 8) < left;
          dma::dma16_lane(in ? reinterpret_cast<const char*>(q) + off[i] : reinterpret_cast<const char*>(&kZeros), at + (wave * O::PER + i) * 1024);
        }
      }
    };
    load(TA(), pa, g.lda, oa, to);
    load(TB(), pb, g.ldb, ob, to + TA::kBytes);
    if constexpr (GATE) load(TA(), pg, g.ldgate, og, to + TA::kBytes + TB::kBytes);
    if (ls + 1 < lsteps) ++ls;
    else if (lt + groups < t_end) {
      lt += groups;
      aim();
    }
  };
  aim();
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) fetch(s);
  int slot = 0;
  Block<WM, WN, F32> b;
  for (int t = t_first; t < t_end; t += groups) {
    const TileAt<BM, BN> at(g, t);
    const int steps = (at.K + kStep - 1) / kStep;
    const bool sums = F32 && g.rowsum && at.n0 == 0 && nw == 0;
    b.clear();
    for (int s = 0; s < steps; ++s) {
      // this stage's loads are in (NS - 2 stages are younger), the last stage has been read
      dma::wait_vm_barrier<(NS - 2) * kLoads>();
      fetch(slot == 0 ? NS - 1 : slot - 1);
      const char* p = lds + slot * kStage;
      b.template step<TA, TB>(p, p + TA::kBytes, GATE ? p + TA::kBytes + TB::kBytes : nullptr, mw, nw, col, g4, sums);
      slot = slot == NS - 1 ? 0 : slot + 1;
    }
    b.store(g, at.m0 + mw, at.n0 + nw, at.z, col, g4, sums);
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
  const bf16* pg = g.gate ? g.gate + (ATR ? (int64_t)at.kb * g.ldgate + at.m0 : (int64_t)at.m0 * g.ldgate + at.kb) : nullptr;
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
    if (pg) {
      Vec16<bf16> vg[TA::PER];
      load(TA(), pg, g.ldgate, g.M - at.m0, s, vg);
#pragma unroll
      for (int i = 0; i < TA::PER; ++i) {
        const bf16x8 t = gated(as_bf16x8(va[i]), as_bf16x8(vg[i]));
        va[i] = __builtin_bit_cast(Vec16<bf16>, t);
      }
    }
  };
  auto put = [&](int s) {
    char* p = lds + (s & 1) * (TA::kBytes + TB::kBytes);
#pragma unroll
    for (int i = 0; i < TA::PER; ++i) *reinterpret_cast<uint4*>(p + TA::pos(i) * 16) = *reinterpret_cast<const uint4*>(&va[i]);
#pragma unroll
    for (int i = 0; i < TB::PER; ++i) *reinterpret_cast<uint4*>(p + TA::kBytes + TB::pos(i) * 16) = *reinterpret_cast<const uint4*>(&vb[i]);
  };
  const int steps = (at.K + kStep - 1) / kStep;
  const bool sums = F32 && g.rowsum && at.n0 == 0 && nw == 0;
  Block<64, 64, F32> b;
  b.clear();
  fetch(0);
  put(0);
  if (steps > 1) fetch(1);
  for (int s = 0; s < steps; ++s) {
    __syncthreads();
    if (s + 1 < steps) put(s + 1);
    if (s + 2 < steps) fetch(s + 2);
    const char* p = lds + (s & 1) * (TA::kBytes + TB::kBytes);
    b.template step<TA, TB>(p, p + TA::kBytes, nullptr, mw, nw, col, g4, sums);
  }
  b.store(g, at.m0 + mw, at.n0 + nw, at.z, col, g4, sums);
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

// fp32: dP = dy where act_out > 0 (act_out NULL: dy), rows of ldp elements with zeros behind the N-th.
__global__ __launch_bounds__(256) void k_fc_mask(const float* __restrict__ dy, int64_t lddy, const float* __restrict__ a, int64_t lda,
                                                 int rows, int N, float* __restrict__ dp, int64_t ldp) {
  const int n = (blockIdx.x * 64 + (threadIdx.x & 63)) * 4;
  if (n >= ldp) return;
  for (int64_t r = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.y * 4) {
    Vec16<float> t = load16_part(dy + r * lddy + n, N - n);
    if (a) {
      const Vec16<float> x = load16_part(a + r * lda + n, N - n);
#pragma unroll
      for (int e = 0; e < 4; ++e) t.v[e] = x.v[e] > 0.f ? t.v[e] : 0.f;
    }
    store16(dp + r * ldp + n, t);
  }
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

template <typename T>
struct FewArgs {
  const T *x, *w, *bias, *res;
  T *y, *act_out;
  int64_t ldx, ldr, ldy, ldact;
  int M, N, K, relu;
};

constexpr int kFewWaves = 8;
template <typename T, int MB>
__global__ __launch_bounds__(64 * kFewWaves) void k_fc_few(FewArgs<T> g) {
  constexpr int KS = few_k<T>(), V = Vec16<T>::N, U = MB == 4 ? 2 : 4;
  __shared__ float part[kFewWaves][MB * 16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const T* w = g.w + (int64_t)min(n0 + col, g.N - 1) * g.K + g4 * V;
  const T* x[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) x[b] = g.x + (int64_t)min(16 * b + col, g.M - 1) * g.ldx + g4 * V;
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
    const int m = i / 16, n = n0 + i % 16;
    if (m >= g.M || n >= g.N) continue;
    float v = 0.f;
#pragma unroll
    for (int p = 0; p < kFewWaves; ++p) v += part[p][m][i % 16];
    if (g.bias) v += to_f32(g.bias[n]);
    if (g.relu) v = v < 0.f ? 0.f : v;
    if (g.act_out) g.act_out[m * g.ldact + n] = from_f32<T>(v);
    if (g.res) v += to_f32(g.res[m * g.ldr + n]);
    g.y[m * g.ldy + n] = from_f32<T>(v);
  }
}

// Direct loads: 16-byte granules, and a tile's rows within 32-bit offsets of its first.
bool dma_ok(const bf16* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1 << 23); }
// The same where the granules run along `cols` columns: the last one is whole.
bool dma_ok(const bf16* p, int64_t ld, int cols) { return dma_ok(p, ld) && cols % 8 == 0; }

// Large tiles (256 x 256, 8 waves, one work-group a CU) read LDS less per product, where
// they fill the chip.
template <bool ATR, bool BTR>
hipError_t launch_product(FcProduct g, bool aligned, hipStream_t s) {
  auto tiles = [&](int bm, int bn) {
    g.mt = (g.M + bm - 1) / bm;
    g.nt = (g.N + bn - 1) / bn;
    return (int64_t)g.mt * g.nt * g.splits;
  };
  if (!aligned || (g.gate && !dma_ok(g.gate, g.ldgate))) {
    const dim3 grid((unsigned)tiles(128, 128)), block(256);
    hipLaunchKernelGGL((k_fc_any<ATR, BTR>), grid, block, 0, s, g);
    return hipGetLastError();
  }
  if constexpr (!ATR) {
    if (!g.gate && g.K >= 512 && tiles(256, 256) >= 256) {
      const int n = (int)tiles(256, 256);
      hipLaunchKernelGGL((k_fc_tile<ATR, BTR, false, 256, 256, 128, 64, 4>), dim3(256), dim3(512), 0, s, g, n);
      return hipGetLastError();
    }
  }
  const int n = (int)tiles(128, 128);
  const dim3 grid((unsigned)std::min(512, (n + kNumXcd - 1) / kNumXcd * kNumXcd)), block(256);
  if constexpr (ATR || BTR) {
    if (g.gate) {
      hipLaunchKernelGGL((k_fc_tile<ATR, BTR, true, 128, 128, 64, 64, 3>), grid, block, 0, s, g, n);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((k_fc_tile<ATR, BTR, false, 128, 128, 64, 64, 4>), grid, block, 0, s, g, n);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_fc(const gdp_fc_layer& f, const T* x, const T* w, const T* b, const T* residual, T* y, T* act_out,
                     hipStream_t s) {
  const int M = (int)f.rows, K = f.in_dim, N = f.out_dim, relu = f.act == GDP_ACT_RELU;
  if (M == 0) return hipSuccess;
  if (M <= kFcFewRows) {
    const FewArgs<T> g = {x, w, b, residual, y, act_out, f.ld_x, f.ld_res, f.ld_y, f.ld_act, M, N, K, relu};
    const dim3 grid((unsigned)(N + 15) / 16), block(64 * kFewWaves);
    if (M <= 16) hipLaunchKernelGGL((k_fc_few<T, 1>), grid, block, 0, s, g);
    else if (M <= 32) hipLaunchKernelGGL((k_fc_few<T, 2>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((k_fc_few<T, 4>), grid, block, 0, s, g);
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 4) {
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
  const T* gate = f.act == GDP_ACT_RELU ? act_out : nullptr;
  if constexpr (sizeof(T) == 4) {
    const T* dp = dy;
    int64_t ldp = f.ld_dy;
    hipError_t e = hipSuccess;
    if (p.ldp > 0) {
      float* t = reinterpret_cast<float*>(base + p.dp);
      const dim3 grid((unsigned)(p.ldp / 4 + 63) / 64, (unsigned)std::min((M + 3) / 4, 4096));
      hipLaunchKernelGGL(k_fc_mask, grid, dim3(256), 0, s, dy, f.ld_dy, gate, f.ld_act, M, N, t, p.ldp);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      dp = t;
      ldp = p.ldp;
    }
    if (dx) {
      tr::GemmStrided<float, float> g = {dp, ldp, 1, w, K, 1, M, K, N, dx, f.ld_dx};
      g.res = dx_add;
      g.ldr = f.ld_dx_add;
      e = tr::launch_gemm_strided(g, nullptr, 0, s);
    }
    if (e != hipSuccess || (!dw && !db)) return e;
    float* out = dw ? dw : part + p.partial_floats;        // db alone: the product's place is scratch
    tr::GemmStrided<float, float> g = {dp, 1, ldp, x, f.ld_x, 1, N, K, M, out, K};
    g.rowsum = db;
    return tr::launch_gemm_strided(g, part, p.partial_floats, s);
  } else {
    FcProduct g = {};
    g.a = dy;
    g.lda = f.ld_dy;
    g.gate = gate;
    g.ldgate = f.ld_act;
    const bool rows_ok = dma_ok(dy, f.ld_dy);
    if (dx) {
      FcProduct d = g;
      d.b = w;
      d.ldb = K;
      d.M = M;
      d.N = K;
      d.K = d.k_per_split = N;
      d.splits = 1;
      d.res = dx_add;
      d.ldr = f.ld_dx_add;
      d.c = dx;
      d.ldc = f.ld_dx;
      const hipError_t e = launch_product<false, true>(d, rows_ok && N % 8 == 0 && dma_ok(w, K, K), s);
      if (e != hipSuccess) return e;
    }
    if (!dw && !db) return hipSuccess;
    g.b = x;
    g.ldb = f.ld_x;
    g.M = N;
    g.N = K;
    g.K = M;
    g.splits = p.splits;
    g.k_per_split = p.rows_per_split;
    g.f = part;
    g.rowsum = part + p.splits * mn;
    const hipError_t e = launch_product<true, true>(g, rows_ok && N % 8 == 0 && dma_ok(x, f.ld_x, K), s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_fc_join, dim3((unsigned)((mn + N + 255) / 256)), dim3(256), 0, s, (const float*)part,
                       (const float*)g.rowsum, p.splits, mn, N, dw, db);
    return hipGetLastError();
  }
}

#define GDP_FC_INST(T)                                                                                              \
  template hipError_t launch_fc<T>(const gdp_fc_layer&, const T*, const T*, const T*, const T*, T*, T*, hipStream_t); \
  template hipError_t launch_fc_backward<T>(const gdp_fc_layer&, const FcPlan&, const T*, const T*, const T*, const T*, const T*, T*, \
                                            float*, float*, void*, hipStream_t);
GDP_FC_INST(float)
GDP_FC_INST(bf16)
#undef GDP_FC_INST

}  // namespace op
}  // namespace gdp
