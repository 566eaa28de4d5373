// FC layers with bias, activation and residual in the product's epilogue, and their
// backward.  x [M, K], W [N, K]:
//   a = act(x W^T + b),  y = a + residual
//   dP = dy where a > 0 (ReLU) or dy,  dx = dP W,  dW = dP^T x,  db = sum_rows dP
//
// fp32 goes through the update step's products (train_gemm.hip: three bf16 planes an
// operand).  bf16 has two kernels here:
//   k_fc_tile  128 x 128 tiles, 4 waves of 64 x 64, k in steps of 64 through two LDS
//              buffers filled by direct loads one step ahead.  The operands stay in
//              their memory order; one whose contraction dimension is not the fast one
//              (W in dx, both in dW) is read by transposing LDS reads.
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

constexpr int kBM = 128, kBK = 64;
constexpr int kTileBytes = kBM * kBK * 2;

// One operand's tile: 128 rows (of C's rows or columns) x 64 k.  TR false: k is the fast
// dimension, an LDS row is 64 k of one row; true: an LDS row is 128 rows of one k.
// 16-byte granules of an LDS row are permuted so that fragment reads (plain: 16 rows x 4
// granules; transposing: rows {8 g + 0..3} x 2 granules) fall in distinct banks.
template <bool TR>
struct OpTile {
  static constexpr int GPR = TR ? kBM / 8 : kBK / 8, PER = 4;
  static __device__ __forceinline__ int key(int r) { return TR ? ((r & 3) | ((r >> 1) & 4)) << 1 : r & 7; }
  const bf16* base;                    // the tile's first element at k = 0
  int64_t ld;
  int rows, K;                         // rows left from the tile's first; contraction length
  uint32_t off[PER];                   // of this lane's granules in one full step, bytes
  static __device__ __forceinline__ int pos(int i) { return ((int)(threadIdx.x >> 6) * PER + i) * 64 + (int)(threadIdx.x & 63); }
  static __device__ __forceinline__ int row(int i) { return pos(i) / GPR; }
  static __device__ __forceinline__ int gran(int i) { return (pos(i) % GPR) ^ key(row(i)); }
  __device__ __forceinline__ OpTile(const bf16* p, int64_t ld_, int rows_, int K_) : base(p), ld(ld_), rows(rows_), K(K_) {
    // past the edge: the last row (granule) again, its results are not stored
#pragma unroll
    for (int i = 0; i < PER; ++i)
      off[i] = TR ? (uint32_t)(((int64_t)row(i) * ld + min(gran(i) * 8, (rows - 1) & ~7)) * 2)
                  : (uint32_t)(((int64_t)min(row(i), rows - 1) * ld + gran(i) * 8) * 2);
  }
  __device__ __forceinline__ void dma(char* lds, int step) const {
    const dma::gptr_t b = dma::uniform_base(base + (int64_t)step * kBK * (TR ? ld : 1));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < PER; ++i) dma::dma16(b, off[i], lds + (wave * PER + i) * 1024);
  }
  // any alignment, zeros past the contraction's end
  Vec16<bf16> v[PER];
  __device__ __forceinline__ void load(int step) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int k = step * kBK + (TR ? row(i) : gran(i) * 8), r = TR ? gran(i) * 8 : min(row(i), rows - 1);
      const int left = TR ? (k < K ? rows - r : 0) : K - k;
      const bf16* p = base + (TR ? (int64_t)k * ld + r : (int64_t)r * ld + k);
      if (left > 0) v[i] = load16_part(p, left);
      else *reinterpret_cast<uint4*>(&v[i]) = make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<uint4*>(lds + pos(i) * 16) = *reinterpret_cast<const uint4*>(&v[i]);
  }
  // rows r0 + (lane & 15), k = 32 ks + 8 (lane / 16) + [0, 8)
  static __device__ __forceinline__ bf16x8 frag(const char* lds, int r0, int ks, int col, int g4) {
    if constexpr (!TR) {
      const int r = r0 + col;
      return *reinterpret_cast<const bf16x8*>(lds + r * 128 + (((ks * 4 + g4) ^ key(r)) << 4));
    } else {
      const int k = 32 * ks + 8 * g4 + (col >> 2), c = r0 + 4 * (col & 3);
      const char* p = lds + (c % 8) * 2;
      return join8(read_tr16(p + k * 256 + (((c / 8) ^ key(k)) << 4)), read_tr16(p + (k + 4) * 256 + (((c / 8) ^ key(k + 4)) << 4)));
    }
  }
};

// C(m, n) = sum_k A(m, k) B(n, k).
struct FcProduct {
  const bf16 *a, *b;
  int64_t lda, ldb;
  int M, N, K;
  int mt, nt, k_per_split;             // tiles; contraction length of one split (a multiple of 64)
  // epilogue of bf16 results
  const bf16 *bias, *res;
  int64_t ldr;
  bf16 *c, *act_out;
  int64_t ldc, ldact;
  int relu;
  // fp32 results (dW): split z's sums at f + z M N; row sums of A (db) at rowsum + z M, or NULL
  float *f, *rowsum;
};

template <bool ATR, bool BTR, bool DMA>
__global__ __launch_bounds__(256, 2) void k_fc_tile(FcProduct g) {
  constexpr bool F32 = ATR;            // dW
  __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int mw = (wave >> 1) * 64, nw = (wave & 1) * 64;
  // consecutive tiles share A's rows (dW: the rows of both): keep them on one XCD
  const int tile = xcd_remap(blockIdx.x, gridDim.x);
  const int n0 = tile % g.nt * kBM, m0 = tile / g.nt % g.mt * kBM, z = tile / (g.nt * g.mt);
  const int kb = z * g.k_per_split, K = min(g.K - kb, g.k_per_split);
  OpTile<ATR> A(g.a + (ATR ? (int64_t)kb * g.lda + m0 : (int64_t)m0 * g.lda + kb), g.lda, g.M - m0, K);
  OpTile<BTR> B(g.b + (BTR ? (int64_t)kb * g.ldb + n0 : (int64_t)n0 * g.ldb + kb), g.ldb, g.N - n0, K);
  f32x4 acc[4][4], ones_acc[F32 ? 4 : 1];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = zero4();
  const bool sums = F32 && g.rowsum && n0 == 0 && nw == 0;
  bf16x8 one;
#pragma unroll
  for (int i = 0; i < 8; ++i) one[i] = (bf16)1.0f;
#pragma unroll
  for (int i = 0; i < (F32 ? 4 : 1); ++i) ones_acc[i] = zero4();
  auto buf_a = [&](int s) { return lds + (s & 1) * 2 * kTileBytes; };
  auto compute = [&](int s) {
    const char *sa = buf_a(s), *sb = sa + kTileBytes;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 fa[4], fb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) fa[i] = OpTile<ATR>::frag(sa, mw + 16 * i, ks, col, g4);
#pragma unroll
      for (int j = 0; j < 4; ++j) fb[j] = OpTile<BTR>::frag(sb, nw + 16 * j, ks, col, g4);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mma16(fb[j], fa[i], acc[i][j]);
      if constexpr (F32) {
        if (sums) {
#pragma unroll
          for (int i = 0; i < 4; ++i) ones_acc[i] = mma16(one, fa[i], ones_acc[i]);
        }
      }
    }
  };
  if constexpr (DMA) {
    const int full = K / kBK;
    if (full > 0) {
      A.dma(buf_a(0), 0);
      B.dma(buf_a(0) + kTileBytes, 0);
    }
    for (int s = 0; s < full; ++s) {
      dma::wait_loads_then_barrier();                      // step s is in; step s - 1 has been read
      if (s + 1 < full) {
        A.dma(buf_a(s + 1), s + 1);
        B.dma(buf_a(s + 1) + kTileBytes, s + 1);
      }
      compute(s);
    }
    if (K % kBK) {                                         // the rest through registers, with zeros
      A.load(full);
      B.load(full);
      A.store(buf_a(full));
      B.store(buf_a(full) + kTileBytes);
      __syncthreads();
      compute(full);
    }
  } else {
    const int steps = (K + kBK - 1) / kBK;
    A.load(0);
    B.load(0);
    A.store(buf_a(0));
    B.store(buf_a(0) + kTileBytes);
    if (steps > 1) {
      A.load(1);
      B.load(1);
    }
    for (int s = 0; s < steps; ++s) {
      __syncthreads();
      if (s + 1 < steps) {
        A.store(buf_a(s + 1));
        B.store(buf_a(s + 1) + kTileBytes);
      }
      if (s + 2 < steps) {
        A.load(s + 2);
        B.load(s + 2);
      }
      compute(s);
    }
  }
  __syncthreads();
  // Each wave turns its 64 x 64 block through its quarter of LDS, so that a lane holds 8
  // consecutive columns and 8 lanes a row's 64.
  char* mine = lds + wave * (64 * 64 * 4);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = 16 * i + col;
      *reinterpret_cast<f32x4*>(mine + m * 256 + (((4 * j + g4) ^ (m & 15)) << 4)) = acc[i][j];
    }
  __syncthreads();
  const int n = n0 + nw + (lane & 7) * 8, left = g.N - n;
  float bias[8];
  if constexpr (!F32) {
    const Vec16<bf16> t = g.bias && left > 0 ? load16_part(g.bias + n, left) : Vec16<bf16>{};
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = to_f32(t.v[e]);
  }
  if (left > 0) {
#pragma unroll 2
    for (int t = 0; t < 8; ++t) {
      const int ml = t * 8 + (lane >> 3), m = m0 + mw + ml;
      if (m >= g.M) break;
      float v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(mine + ml * 256 + (((2 * (lane & 7) + h) ^ (ml & 15)) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = x[e];
      }
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
          v[e] += bias[e];
          if (g.relu) v[e] = v[e] < 0.f ? 0.f : v[e];      // NaN stays
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
  }
  if constexpr (F32) {
    if (sums && g4 == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = m0 + mw + 16 * i + col;
        if (m < g.M) g.rowsum[(int64_t)z * g.M + m] = ones_acc[i][0];
      }
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

// dP = dy where act_out > 0 (act_out NULL: dy), rows of ldp elements with zeros behind the N-th.
template <typename T>
__global__ __launch_bounds__(256) void k_fc_mask(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ a, int64_t lda,
                                                 int64_t rows, int N, T* __restrict__ dp, int64_t ldp) {
  constexpr int V = Vec16<T>::N;
  const int64_t per = ldp / V, total = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per;
    const int n = (int)(i - r * per) * V;
    Vec16<T> t = load16_part(dy + r * lddy + n, N - n);
    if (a) {
      const Vec16<T> x = load16_part(a + r * lda + n, N - n);
#pragma unroll
      for (int e = 0; e < V; ++e) t.v[e] = to_f32(x.v[e]) > 0.f ? t.v[e] : (T)0.f;
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

template <bool ATR, bool BTR>
hipError_t launch_tile(const FcProduct& g, int splits, bool dma, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)g.mt * g.nt * splits)), block(256);
  if (dma) hipLaunchKernelGGL((k_fc_tile<ATR, BTR, true>), grid, block, 0, s, g);
  else hipLaunchKernelGGL((k_fc_tile<ATR, BTR, false>), grid, block, 0, s, g);
  return hipGetLastError();
}

int tiles_of(int n) { return (n + kBM - 1) / kBM; }

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
    g.K = K;
    g.mt = tiles_of(M);
    g.nt = tiles_of(N);
    g.k_per_split = (K + kBK - 1) / kBK * kBK;
    g.bias = b;
    g.res = residual;
    g.ldr = f.ld_res;
    g.c = y;
    g.ldc = f.ld_y;
    g.act_out = act_out;
    g.ldact = f.ld_act;
    g.relu = relu;
    return launch_tile<false, false>(g, 1, dma_ok(x, f.ld_x) && dma_ok(w, K), s);
  }
}

template <typename T>
hipError_t launch_fc_backward(const gdp_fc_layer& f, const FcPlan& p, const T* dy, const T* x, const T* w,
                              const T* act_out, const T* dx_add, T* dx, float* dw, float* db, void* ws, hipStream_t s) {
  const int M = (int)f.rows, K = f.in_dim, N = f.out_dim;
  char* base = static_cast<char*>(ws);
  const T* dp = dy;
  int64_t ldp = f.ld_dy;
  if (p.ldp > 0 && M > 0) {
    T* t = reinterpret_cast<T*>(base + p.dp);
    const int64_t blocks = std::min<int64_t>((f.rows * (p.ldp / Vec16<T>::N) + 255) / 256, 8192);
    hipLaunchKernelGGL((k_fc_mask<T>), dim3((unsigned)blocks), dim3(256), 0, s, dy, f.ld_dy,
                       f.act == GDP_ACT_RELU ? act_out : (const T*)nullptr, f.ld_act, f.rows, N, t, p.ldp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    dp = t;
    ldp = p.ldp;
  }
  float* part = reinterpret_cast<float*>(base + p.partial);
  const int64_t mn = (int64_t)N * K;
  if (M == 0) {                                            // no rows: gradients of zero
    hipLaunchKernelGGL(k_fc_join, dim3((unsigned)((mn + N + 255) / 256)), dim3(256), 0, s, (const float*)nullptr,
                       (const float*)nullptr, 0, mn, N, dw, db);
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 4) {
    hipError_t e = hipSuccess;
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
    if (dx) {
      FcProduct g = {};
      g.a = dp;
      g.lda = ldp;
      g.b = w;
      g.ldb = K;
      g.M = M;
      g.N = K;
      g.K = N;
      g.mt = tiles_of(M);
      g.nt = tiles_of(K);
      g.k_per_split = (N + kBK - 1) / kBK * kBK;
      g.res = dx_add;
      g.ldr = f.ld_dx_add;
      g.c = dx;
      g.ldc = f.ld_dx;
      const hipError_t e = launch_tile<false, true>(g, 1, dma_ok(dp, ldp) && dma_ok(w, K, K), s);
      if (e != hipSuccess) return e;
    }
    if (!dw && !db) return hipSuccess;
    FcProduct g = {};
    g.a = dp;
    g.lda = ldp;
    g.b = x;
    g.ldb = f.ld_x;
    g.M = N;
    g.N = K;
    g.K = M;
    g.mt = tiles_of(N);
    g.nt = tiles_of(K);
    g.k_per_split = p.rows_per_split;
    g.f = part;
    g.rowsum = part + p.splits * mn;
    const hipError_t e = launch_tile<true, true>(g, p.splits, dma_ok(dp, ldp, p.ldp > 0 ? 8 : N) && dma_ok(x, f.ld_x, K), s);
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
