// Segment attention with a learned relative position bias by buckets, forward and
// backward, for bf16 and fp32.
//
// A query at position p of its graph, s0 = floor(p / seg) seg, sees the keys j of
// [max(0, s0 - mem), s0 + seg) (j <= p with causal order) whose mask byte is not 0:
//   z = scale q . k_j + table[h][bucket(j - p)],  P = softmax(z),  o = sum_j P v_j
//   dP = dO . v,  D = sum_j P dP,  dS = P (dP - D)
//   dq = scale sum_j dS k_j,  dk = scale sum dS q,  dv = sum P dO,  dtable[h][b] = sum of dS in bucket b
// The bias depends on j - p alone, so a tile of 64 keys and the work-group's queries has
// one value a diagonal: they are put into LDS beside the tile, or, where the whole tile
// lies in one bucket (most tiles beyond the last bound), the value is one number.
//
// A work-group is 4 waves and 64 COLS queries (or keys, for dK and dV); the other side
// passes through LDS in tiles of 64 rows, one tile ahead, and one more in registers.
// Scores are formed transposed, so that a lane owns one query (one key): its row maximum
// is an in-lane maximum and two exchanges, and its probabilities are the next product's
// operand without leaving its registers; that product's other operand comes from
// transposing LDS reads.  bf16 operands go to the matrix cores as they are, fp32 ones as
// three bf16 planes (six products).  Probabilities and dS are rounded to one plane for
// bf16 data: their rounding is the size of the outputs' own.  What is summed over many
// rows into fp32 (row sums, D, dtable) is never rounded to bf16.
//
// D: the dQ pass starts from D0 = dO . o with the given o, and forms D = sum P dP beside
// its products, for the dK pass and dtable: a rounded o would be the largest error of
// dtable (which sums differences whose leading parts cancel).  For bf16 data dq takes what
// D0 leaves, (D0 - D) sum P k, from a product of its own, and its dS as two planes: a row's
// dS add up to zero, so the part that its keys have in common cancels and leaves their
// roundings (with one plane dq's error was 1.5 roundings of the exact dq, so 1.1).
//
// A column whose result is not finite is formed again, key by key over what it sees: a
// NaN or infinity in a row that it does not see meets a probability of zero in a tile
// they share, and must not reach it.
#include <algorithm>
#include <type_traits>

#include "op_common.h"
#include "op_kernels.h"

namespace gdp {
namespace op {

namespace {

constexpr int kTile = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescale = 8.0f;       // a row maximum is raised once scores pass it by 2^8
constexpr float kLargest = 0x1p100f;   // of a row's sum whose maximum is not raised

// What a kernel needs besides its arrays.
struct Geo {
  int heads, share;                    // query heads; query heads per key head
  int seg, mem, causal, buckets;
  float scale, sc;                     // scale; scale * log2(e)
  int64_t ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T> constexpr int planes() { return sizeof(T) == 2 ? 1 : 3; }

// A table entry in log2 units; what is below -1e30 excludes its bucket.
template <typename T>
__device__ __forceinline__ float bias_of(T t) {
  const float b = to_f32(t);
  return b < -1e30f ? -INFINITY : b * kLog2e;
}

// ---------------------------------------------------------------------------
// Buckets.
// ---------------------------------------------------------------------------
struct Buckets {
  int n, causal;
  const int* at;                       // LDS: the bounds, then INT_MAX up to 64
  int mine;                            // at[lane]
  __device__ __forceinline__ static void stage(int* lds, const RelBounds& b) {
    if (threadIdx.x < 64) lds[threadIdx.x] = bound(b, threadIdx.x);
  }
  __device__ __forceinline__ static int bound(const RelBounds& b, int i) { return i < b.n ? b.at[i] : INT32_MAX; }
  __device__ __forceinline__ Buckets(const int* lds, const RelBounds& b, int causal_)
      : n(b.n), causal(causal_), at(lds), mine(bound(b, threadIdx.x & 63)) {}
  __device__ __forceinline__ int side(int rel) const { return rel > 0 && !causal ? n + 1 : 0; }
  // of one distance a lane
  __device__ __forceinline__ int of(int rel) const {
    const int d = abs(rel);
    int lo = 0;                        // bounds at or below d
#pragma unroll
    for (int step = 32; step > 0; step >>= 1)
      if (at[lo + step - 1] <= d) lo += step;
    return lo + side(rel);
  }
  // of one distance for the whole wave
  __device__ __forceinline__ int of_uniform(int rel) const {
    const int d = abs(rel);
    return __popcll(__ballot(mine <= d)) + side(rel);
  }
  // The bucket that holds all of [lo, hi], or -1.
  __device__ __forceinline__ int common(int lo, int hi) const {
    if (lo <= 0 && hi > 0) return -1;
    const int a = of_uniform(lo);
    return a == of_uniform(hi) ? a : -1;
  }
};

// ---------------------------------------------------------------------------
// 64 rows of one head's columns as 1 or 3 bf16 planes in LDS.
// ---------------------------------------------------------------------------
template <typename T, int DH>
struct Tile {
  static constexpr int NP = planes<T>();
  static constexpr int G = DH / 8;                        // 16-byte granules per row
  static constexpr int kPlane = kTile * DH * 2;
  static constexpr int kBytes = NP * kPlane;
  static constexpr int U = kTile * G > 256 ? kTile * G / 256 : 1;
  // eight consecutive rows of a fragment read fall in distinct granules modulo 128 bytes
  static __device__ __forceinline__ int at(int row, int g) {
    if constexpr (DH == 16) return row * 32 + ((g ^ ((row >> 2) & 1)) << 4);
    else if constexpr (DH == 32) return row * 64 + ((g ^ (((row >> 2) ^ (row >> 1)) & 3)) << 4);
    else return row * 128 + ((g ^ (row & 7)) << 4);
  }
  Vec16<T> v[U][NP == 3 ? 2 : 1];
  static __device__ __forceinline__ int unit(int u) { return ((int)threadIdx.x + 256 * u) % (kTile * G); }
  // Where a work-group's tiles come from: rows [t0, t0 + 64), [t0 + 64, ..) of src, rows at or
  // past t1 as copies of row t1 - 1; place is this thread's first element in a tile.
  struct From {
    const T* tile;                     // the next tile's first element (uniform)
    int64_t ld;
    int left;                          // rows from there on
    int64_t place;
    __device__ __forceinline__ From(const T* src, int64_t ld_, int t0, int t1)
        : tile(src + (size_t)t0 * ld_), ld(ld_), left(t1 - t0), place(unit(0) / G * ld_ + unit(0) % G * 8) {}
  };
  __device__ __forceinline__ void load(From& f) {          // past the end: nothing that is used
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* p = f.tile + f.place + (int64_t)u * (256 / G) * f.ld;
      if (f.left < kTile) p = f.tile + (int64_t)min(unit(u) / G, f.left - 1) * f.ld + unit(u) % G * 8;
#pragma unroll
      for (int i = 0; i < (NP == 3 ? 2 : 1); ++i) v[u][i] = load16_any(p + i * Vec16<T>::N);
    }
    if (f.left > kTile) {
      f.tile += kTile * f.ld;
      f.left -= kTile;
    }
  }
  __device__ __forceinline__ void store(char* s) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int o = at(unit(u) / G, unit(u) % G);
      if constexpr (NP == 1) {
        *reinterpret_cast<bf16x8*>(s + o) = as_bf16x8(v[u][0]);
      } else {
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[i] = v[u][0].v[i];
          f[4 + i] = v[u][1].v[i];
        }
        const Operand<3> p = operand(f);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<bf16x8*>(s + q * kPlane + o) = p.p[q];
      }
    }
  }
  static __device__ __forceinline__ Operand<NP> granule(const char* s, int row, int g) {
    Operand<NP> o;
#pragma unroll
    for (int q = 0; q < NP; ++q) o.p[q] = *reinterpret_cast<const bf16x8*>(s + q * kPlane + at(row, g));
    return o;
  }
  // rows row0 + {4 g4 + i, 16 + 4 g4 + i} of column dim0 + (lane & 15), as an operand's eight k slots
  static __device__ __forceinline__ Operand<NP> transposed(const char* s, int row0, int dim0, int col, int g4) {
    const int r = row0 + 4 * g4 + (col >> 2), dim = dim0 + 4 * (col & 3);
    Operand<NP> o;
#pragma unroll
    for (int q = 0; q < NP; ++q)
      o.p[q] = join8(read_tr16(s + q * kPlane + at(r, dim / 8) + (dim % 8) * 2),
                     read_tr16(s + q * kPlane + at(r + 16, dim / 8) + (dim % 8) * 2));
    return o;
  }
};

// A lane's own row for products over the head dimension (d_h = 16: lane groups 2 and 3
// hold zeros, half of the instruction's k).
template <typename T, int DH>
struct Row {
  static constexpr int NP = planes<T>(), NK = DH == 64 ? 2 : 1;
  Operand<NP> k[NK];
  __device__ __forceinline__ void load(const T* row, int g4) {
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const T* p = row + (DH == 16 ? (g4 & 1) * 8 : s * 32 + g4 * 8);
      const bool on = DH != 16 || g4 < 2;
      if constexpr (NP == 1) {
        Vec16<T> t = load16_any(p);
        if (!on) *reinterpret_cast<uint4*>(&t) = make_uint4(0, 0, 0, 0);
        k[s] = operand(as_bf16x8(t));
      } else {
        const Vec16<T> a = load16_any(p), b = load16_any(p + 4);
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[i] = on ? a.v[i] : 0.f;
          f[4 + i] = on ? b.v[i] : 0.f;
        }
        k[s] = operand(f);
      }
    }
  }
};

// acc[c] = tile rows [row0, row0 + 16) . the columns' rows.  (What is added to them later,
// the bias less the log-sum-exp, -D, is not made the instruction's addend: beside it the
// products lose their low bits, dtable's error was 2.4e-6 instead of 4e-7.)
template <typename T, int DH, int COLS>
__device__ __forceinline__ void dot_rows(f32x4 (&acc)[COLS], const char* tile, int row0, const Row<T, DH> (&y)[COLS], int col,
                                         int g4) {
  f32x4 low[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) acc[c] = low[c] = zero4();
#pragma unroll
  for (int s = 0; s < Row<T, DH>::NK; ++s) {
    const auto a = Tile<T, DH>::granule(tile, row0 + col, DH == 16 ? (g4 & 1) : s * 4 + g4);
#pragma unroll
    for (int c = 0; c < COLS; ++c) mma_planes(a, y[c].k[s], acc[c], low[c]);
  }
  if constexpr (planes<T>() == 3) {
#pragma unroll
    for (int c = 0; c < COLS; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[c][r] += low[c][r];
  }
}

// acc[db][c] += tile^T . w over the tile's rows [row0, row0 + 32); w[c]: the lane's
// values of rows row0 + 4 g4 + i and row0 + 16 + 4 g4 + i.
template <typename T, int DH, int COLS, int NW>
__device__ __forceinline__ void acc_rows(f32x4 (&acc)[DH / 16][COLS], const char* tile, int row0, const Operand<NW> (&w)[COLS],
                                         int col, int g4) {
#pragma unroll
  for (int db = 0; db < DH / 16; ++db) {
    const auto a = Tile<T, DH>::transposed(tile, row0, 16 * db, col, g4);
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      if constexpr (planes<T>() == 1) {
        acc[db][c] = mma16(a.p[0], w[c].p[0], acc[db][c]);
      } else {
        f32x4 top = zero4(), low = zero4();
        mma_planes(a, w[c], top, low);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[db][c][r] += top[r] + low[r];
      }
    }
  }
}

template <typename T, int DH>
constexpr int buffers() { return planes<T>() == 3 && DH == 64 ? 1 : 2; }
template <typename T, int DH>
constexpr int tile_lds() { return buffers<T, DH>() * 2 * Tile<T, DH>::kBytes; }

// Two arrays' tiles through LDS: from fx and fy, prep(i) fills what else tile i needs in
// LDS (into buffer i & 1 of its own), work(x, y, i) uses both.  Ends with a barrier, so
// that the caller may start again.
template <typename T, int DH, typename Prep, typename Work>
__device__ __forceinline__ void for_tiles(char* lds, int tiles, typename Tile<T, DH>::From fx, typename Tile<T, DH>::From fy,
                                          Prep prep, Work work) {
  constexpr int NB = buffers<T, DH>(), kBuf = 2 * Tile<T, DH>::kBytes;
  Tile<T, DH> x, y;
  auto load = [&]() {
    x.load(fx);
    y.load(fy);
  };
  load();
  auto now = prep(0);
  if constexpr (NB == 2) {
    x.store(lds);
    y.store(lds + Tile<T, DH>::kBytes);
    load();
  }
  for (int i = 0; i < tiles; ++i) {
    __syncthreads();
    char* cur = lds + (NB == 2 ? (i & 1) * kBuf : 0);
    if constexpr (NB == 2) {
      char* nxt = lds + ((i + 1) & 1) * kBuf;
      x.store(nxt);
      y.store(nxt + Tile<T, DH>::kBytes);
      load();
    } else {
      x.store(cur);
      y.store(cur + Tile<T, DH>::kBytes);
      load();
      __syncthreads();
    }
    auto next = now;
    if (i + 1 < tiles) next = prep(i + 1);
    work(cur, cur + Tile<T, DH>::kBytes, i, now);
    now = next;
  }
  __syncthreads();
}

// What a tile's scores need to know of its keys: the bucket that holds all of them, or -1,
// and those that the key mask admits.
struct Keys {
  int bucket;
  uint64_t seen;
};

// f(whether a tile's pairs need masking, whether its biases are a diagonal's each), as constants
template <typename F>
__device__ __forceinline__ void by_tile(bool masked, bool diagonals, F f) {
  if (!masked && !diagonals) f(std::false_type(), std::false_type());
  else if (!masked) f(std::false_type(), std::true_type());
  else if (!diagonals) f(std::true_type(), std::false_type());
  else f(std::true_type(), std::true_type());
}

// Rows of a work block: graph g, queries (or keys) [i0, i0 + rows) of it.
struct Block {
  int g, i0;
};
__device__ __forceinline__ Block block_of(const RelTable& t, int b, int rows) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.blk[mid] <= b) lo = mid;
    else hi = mid - 1;
  }
  return {lo, (b - t.blk[lo]) * rows};
}

// The keys that position p sees, before the key mask.
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span span_of(const Geo& e, int p, int len) {
  const int s0 = p / e.seg * e.seg;
  return {max(0, s0 - e.mem), e.causal ? p + 1 : min(s0 + e.seg, len)};
}

// Bits [a, b) of a tile's 64 rows (a and b relative to it, any integers).
__device__ __forceinline__ uint64_t row_bits(int a, int b) {
  a = min(max(a, 0), 64);
  b = min(max(b, 0), 64);
  const uint64_t up = b >= 64 ? ~0ull : (1ull << b) - 1ull;
  return a >= 64 ? 0ull : up & ~((1ull << a) - 1ull);
}

template <typename T, int DH>
__device__ __forceinline__ float dot_f32(const T* x, const T* y) {
  float t = 0.f;
  for (int i = 0; i < DH; ++i) t = fmaf(to_f32(x[i]), to_f32(y[i]), t);
  return t;
}
// A lane's values 16 db + 4 g4 + r: o += w * row.
template <typename T, int DB>
__device__ __forceinline__ void add_row(f32x4 (&o)[DB], float w, const T* row, int g4) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) o[db][r] = fmaf(w, to_f32(row[db * 16 + 4 * g4 + r]), o[db][r]);
}
template <int DB, int COLS>
__device__ __forceinline__ bool finite_column(const f32x4 (&o)[DB][COLS], int c) {
  float any = 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) any = fmaf(o[db][c][r], 0.f, any);
  return any == any;
}
// Four consecutive values to any element address.
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) {
  Vec16<float> t;
#pragma unroll
  for (int r = 0; r < 4; ++r) t.v[r] = v[r];
  store16_any(p, t);
}
__device__ __forceinline__ void store4(bf16* p, const float (&v)[4]) {
  union {
    bf16 h[4];
    uint2 u;
  } t;
#pragma unroll
  for (int r = 0; r < 4; ++r) t.h[r] = (bf16)v[r];
  *reinterpret_cast<u32x2_any*>(p) = u32x2_any{t.u.x, t.u.y};
}

// Orders a wave's own LDS writes before its other lanes' reads.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A lane's value from N lanes on (before it) in its row of 16, 0 past the row's end.
template <int N>
__device__ __forceinline__ float row_left(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x100 + N, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ float row_right(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x110 + N, 0xf, 0xf, true));
}

// The biases of a tile's diagonals: value i belongs to the distance first + i.
template <int N>
struct Diagonals {
  float bias[2][N];
};

// Scores, forward ------------------------------------------------------------------------

// Bound by vector instructions: a score takes one FMA, one exponential (a quarter of the
// FMA's rate), one add to its row's sum and half a conversion.  A wave takes 32 of a tile's
// keys at a time, scores to products with V: few registers hold scores, so a SIMD holds four
// waves (d_h <= 32, bf16) whose matrix and vector work overlap.  52,000 queries, 8 heads of
// 32, 1,024 keys a query: 133 us (with all 64 keys at once and two waves: 157); 26 us of it
// do not depend on the number of keys (106 MB of arrays), each 64 keys cost 6.
template <typename T, int DH, int COLS>
constexpr int fwd_waves() { return planes<T>() == 1 && DH <= 32 ? 4 : 2; }

template <typename T, int DH, int COLS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(fwd_waves<T, DH, COLS>())))
void k_rel_fwd(RelTable rt, RelBounds rb, Geo e, const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
               const T* __restrict__ table, const uint8_t* __restrict__ key_mask, T* __restrict__ o, float* __restrict__ lse) {
  constexpr int DB = DH / 16, BQ = 64 * COLS, ND = kTile + BQ - 1;
  __shared__ __attribute__((aligned(16))) char lds[tile_lds<T, DH>()];
  __shared__ int s_bounds[64];
  __shared__ float s_table[2 * GDP_MAX_REL_BOUNDS + 2];
  __shared__ float s_diag[3][ND + 1];                      // a tile's biases by distance, tile i in buffer i % 3
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int head = logical % e.heads, kvh = head / e.share;
  const Block b = block_of(rt, logical / e.heads, BQ);
  const int len = rt.len[b.g], nq = rt.q0[b.g + 1] - rt.q0[b.g];
  const int count = min(BQ, nq - b.i0), p0 = len - nq + b.i0;
  const T* kg = k + (size_t)rt.start[b.g] * e.ldk + kvh * DH;
  const T* vg = v + (size_t)rt.start[b.g] * e.ldv + kvh * DH;
  const uint8_t* mg = key_mask ? key_mask + rt.start[b.g] : nullptr;
  const float bias = bias_of(table[(size_t)head * e.buckets + min((int)threadIdx.x, e.buckets - 1)]);
  const Buckets bk(s_bounds, rb, e.causal);
  const Span first = span_of(e, p0, len), last = span_of(e, p0 + count - 1, len);
  const int k0 = first.lo, k1 = last.hi, tiles = (k1 - k0 + kTile - 1) / kTile;
  auto query_of = [&](int c) { return (wave * COLS + c) * 16 + col; };
  auto row_of = [&](int c) { return (size_t)(rt.q0[b.g] + b.i0 + min(query_of(c), count - 1)); };

  Row<T, DH> qf[COLS];
  f32x4 oacc[DB][COLS];
  float m[COLS], lsum[COLS];
  Span span[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    span[c] = span_of(e, p0 + min(query_of(c), count - 1), len);
    qf[c].load(q + row_of(c) * e.ldq + head * DH, g4);
  }
  auto prep = [&](int i) {
    if (i == 0) {                                          // the first tiles are on their way
      Buckets::stage(s_bounds, rb);
      if ((int)threadIdx.x < e.buckets) s_table[threadIdx.x] = bias;
      __syncthreads();
    }
    const int t0 = k0 + i * kTile;
    const int u = bk.common(t0 - (p0 + BQ - 1), t0 + kTile - 1 - p0);
    if (u < 0 && (int)threadIdx.x < ND) s_diag[i % 3][threadIdx.x] = s_table[bk.of(t0 - (p0 + BQ - 1) + (int)threadIdx.x)];
    const uint64_t s = mg ? __ballot(mg[min(t0 + lane, k1 - 1)] != 0) : ~0ull;
    return Keys{u, s};
  };
  // Tile i's products -> probabilities, their sums added up.  CAREFUL: the maximum follows
  // the scores.  Else a row keeps the maximum of the first tile that shows it a key; scores
  // further above than fp32 reaches make its sum leave kLargest, and the work-group starts
  // again.
  // 32 keys' products -> probabilities, their sums added up.  CAREFUL: the maximum follows
  // the scores.  Else a row keeps the maximum of the first keys that it sees; scores further
  // above than fp32 reaches make its sum leave kLargest, and the work-group starts again.
  auto soften = [&](auto careful, f32x4 (&s)[2][COLS], int i, int h, const Keys& keys) {
    constexpr bool CAREFUL = decltype(careful)::value;
    const int t0 = k0 + i * kTile + 32 * h, u = keys.bucket;
    const uint32_t admitted = (uint32_t)(keys.seen >> (32 * h));
    const bool full = t0 >= last.lo && t0 + 32 <= first.hi && admitted == ~0u;
    float base[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) base[c] = m[c] == -INFINITY ? 0.f : m[c];
    if (u >= 0) {
#pragma unroll
      for (int c = 0; c < COLS; ++c) {
        const float add = s_table[u] - base[c];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[kb][c][r] = fmaf(s[kb][c][r], e.sc, add);
      }
    } else {
      // column c is 16 queries later than c - 1, block kb 16 keys: one shift of both is one value
      const float* d = s_diag[i % 3] + (BQ - 1) - (wave * COLS * 16 + col) + 4 * g4 + 32 * h;
      float t[COLS + 1][4];
#pragma unroll
      for (int w = 0; w <= COLS; ++w)
#pragma unroll
        for (int r = 0; r < 4; ++r) t[w][r] = d[(w - COLS + 1) * 16 + r];
#pragma unroll
      for (int c = 0; c < COLS; ++c)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[kb][c][r] = fmaf(s[kb][c][r], e.sc, t[kb - c + COLS - 1][r] - base[c]);
    }
    if (!full) {
#pragma unroll
      for (int c = 0; c < COLS; ++c) {
        const uint32_t on = ((uint32_t)row_bits(span[c].lo - t0, span[c].hi - t0) & admitted) >> (4 * g4);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[kb][c][r] = (on >> (kb * 16 + r)) & 1u ? s[kb][c][r] : -INFINITY;
      }
    }
    bool unset = false;
#pragma unroll
    for (int c = 0; c < COLS; ++c) unset = unset || m[c] == -INFINITY;
    if (CAREFUL || __any(unset)) {
      bool raise = false;
      float top[COLS];
#pragma unroll
      for (int c = 0; c < COLS; ++c) {
        float t = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r) t = fmaxf(t, s[kb][c][r]);
        t = fmaxf(t, xor_shfl(t, 16));
        top[c] = fmaxf(t, xor_shfl(t, 32));
        raise = raise || top[c] > (m[c] == -INFINITY ? -INFINITY : CAREFUL ? kRescale : INFINITY);
      }
      if (__any(raise)) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
          const bool up = top[c] > (m[c] == -INFINITY ? -INFINITY : CAREFUL ? kRescale : INFINITY);
          const float by = up ? top[c] : 0.f, corr = !up ? 1.f : m[c] == -INFINITY ? 0.f : exp2_fast(-by);
          m[c] = up ? base[c] + by : m[c];
          lsum[c] *= corr;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[kb][c][r] -= by;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 4; ++r) oacc[db][c][r] *= corr;
        }
      }
    }
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      float sum[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[kb][c][r] = exp2_fast(s[kb][c][r]);
        sum[kb] = (s[kb][c][0] + s[kb][c][1]) + (s[kb][c][2] + s[kb][c][3]);
      }
      lsum[c] += sum[0] + sum[1];
    }
  };
  auto pass = [&](auto careful) {
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      m[c] = -INFINITY;
      lsum[c] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db][c] = zero4();
    }
    const typename Tile<T, DH>::From fk{kg, e.ldk, k0, k1}, fv{vg, e.ldv, k0, k1};
    for_tiles<T, DH>(lds, tiles, fk, fv, prep, [&](const char* sK, const char* sV, int i, const Keys& keys) {
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        f32x4 s[2][COLS];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) dot_rows<T, DH, COLS>(s[kb], sK, 32 * h + kb * 16, qf, col, g4);
        soften(careful, s, i, h, keys);
        Operand<planes<T>()> p[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
          float t[8];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            t[r] = s[0][c][r];
            t[4 + r] = s[1][c][r];
          }
          p[c] = operand_of<planes<T>()>(t);
        }
        acc_rows<T, DH, COLS>(oacc, sV, 32 * h, p, col, g4);
      }
    });
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      lsum[c] += xor_shfl(lsum[c], 16);
      lsum[c] += xor_shfl(lsum[c], 32);
    }
  };
  pass(std::false_type());
  bool far = false;
#pragma unroll
  for (int c = 0; c < COLS; ++c) far = far || !(lsum[c] < kLargest && finite_column(oacc, c));
  if (__syncthreads_or(far)) pass(std::true_type());
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    if (query_of(c) >= count) continue;
    const size_t row = row_of(c);
    if (!(lsum[c] * 0.f == 0.f) || !finite_column(oacc, c)) {
      const T* qr = q + row * e.ldq + head * DH;
      const int p = p0 + query_of(c);
      auto score = [&](int j) { return fmaf(dot_f32<T, DH>(qr, kg + (size_t)j * e.ldk), e.sc, s_table[bk.of(j - p)]); };
      f32x4 t[DB];
#pragma unroll
      for (int db = 0; db < DB; ++db) t[db] = zero4();
      float mx = -INFINITY, sum = 0.f;
      for (int j = span[c].lo; j < span[c].hi; ++j)
        if (!mg || mg[j]) mx = fmaxf(mx, score(j));
      for (int j = span[c].lo; j < span[c].hi; ++j)
        if (!mg || mg[j]) {
          const float w = exp2f(score(j) - (mx == -INFINITY ? 0.f : mx));
          sum += w;
          add_row<T, DB>(t, w, vg + (size_t)j * e.ldv, g4);
        }
      m[c] = mx;
      lsum[c] = sum;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db][c] = t[db];
    }
    const bool none = lsum[c] == 0.f;                      // no key seen: zeros
    const float inv = none ? 0.f : 1.0f / lsum[c];
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const float t[4] = {oacc[db][c][0] * inv, oacc[db][c][1] * inv, oacc[db][c][2] * inv, oacc[db][c][3] * inv};
      store4(o + row * e.ldo + head * DH + db * 16 + 4 * g4, t);
    }
    if (lse && g4 == 0) lse[row * e.heads + head] = none ? -INFINITY : m[c] + log2f(lsum[c]);
  }
}

// Few queries over long keys --------------------------------------------------------------
//
// What bounds it: reading K and V once.  A work-group takes one key head of one graph, 16
// columns (a query and one of the heads that share the keys), and one part of the keys;
// its 4 waves take every fourth tile of 64 keys on their own, K straight from memory in
// operand layout, V through LDS of the wave's own for the transposing reads, the next
// tile's loads in flight meanwhile.  No barrier until the waves' results are joined.  With
// more parts than one, those go to the workspace and k_rel_join adds them.  The matrix
// cores are idle enough for probabilities of two planes (their rounding does not show).
// One query of each of 8 graphs of 12,000 keys, 8 heads of 64 on 2: 14 us and 4 for the
// join (49 MB, which a copy's rate moves in 10).

template <typename T, int DH>
struct FewTile {
  static constexpr int NP = planes<T>(), NK = DH == 64 ? 2 : 1, NV = NP == 3 ? 2 : 1;
  static constexpr int PER = DH / 8;                       // 8-value granules of V a lane loads: 64 rows of DH / 8
  Vec16<T> k[4][NK][NV], v[PER][NV];
  __device__ __forceinline__ void load(const T* kg, int64_t ldk, const T* vg, int64_t ldv, int t0, int k1, int lane) {
    const int col = lane & 15, g4 = lane >> 4;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const T* p = kg + (size_t)min(t0 + kb * 16 + col, k1 - 1) * ldk;
#pragma unroll
      for (int s = 0; s < NK; ++s)
#pragma unroll
        for (int i = 0; i < NV; ++i) k[kb][s][i] = load16_any(p + (DH == 16 ? (g4 & 1) * 8 : s * 32 + g4 * 8) + i * Vec16<T>::N);
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int at = u * 64 + lane;
      const T* p = vg + (size_t)min(t0 + at / PER, k1 - 1) * ldv + at % PER * 8;
#pragma unroll
      for (int i = 0; i < NV; ++i) v[u][i] = load16_any(p + i * Vec16<T>::N);
    }
  }
  static __device__ __forceinline__ Operand<NP> as_operand(const Vec16<T> (&x)[NV]) {
    if constexpr (NP == 1) {
      return operand(as_bf16x8(x[0]));
    } else {
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = x[0].v[i];
        f[4 + i] = x[1].v[i];
      }
      return operand(f);
    }
  }
  __device__ __forceinline__ void store_v(char* lds, int lane) const {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int at = u * 64 + lane;
      const Operand<NP> o = as_operand(v[u]);
#pragma unroll
      for (int q = 0; q < NP; ++q)
        *reinterpret_cast<bf16x8*>(lds + q * Tile<T, DH>::kPlane + Tile<T, DH>::at(at / PER, at % PER)) = o.p[q];
    }
  }
};

// One output column from its maximum, sum and weighted values; formed again over the keys
// where that is not finite.  Values dim, dim + 1, .. dim + N - 1.
template <typename T, int DH, int N>
__device__ __forceinline__ void finish_few(float (&o)[N], float m, float l, int dim, const T* qr, const T* kg, int64_t ldk,
                                           const T* vg, int64_t ldv, const uint8_t* mg, Span s, int p, float sc,
                                           const Buckets& bk, const T* table, T* out, float* lse) {
  float any = l * 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) any = fmaf(o[i], 0.f, any);
  if (any != any) {
    auto score = [&](int j) { return fmaf(dot_f32<T, DH>(qr, kg + (size_t)j * ldk), sc, bias_of(table[bk.of(j - p)])); };
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
    for (int j = s.lo; j < s.hi; ++j)
      if (!mg || mg[j]) m = fmaxf(m, score(j));
    for (int j = s.lo; j < s.hi; ++j)
      if (!mg || mg[j]) {
        const float w = exp2f(score(j) - (m == -INFINITY ? 0.f : m));
        l += w;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = fmaf(w, to_f32(vg[(size_t)j * ldv + dim + i]), o[i]);
      }
  }
  const bool none = l == 0.f;
  const float inv = none ? 0.f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < N; ++i) out[dim + i] = from_f32<T>(o[i] * inv);
  if (lse && dim == 0) *lse = none ? -INFINITY : m + log2f(l);
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void k_rel_few(RelTable rt, RelBounds rb, Geo e, int parts, const T* __restrict__ q,
                                                 const T* __restrict__ k, const T* __restrict__ v,
                                                 const T* __restrict__ table, const uint8_t* __restrict__ key_mask,
                                                 T* __restrict__ o, float* __restrict__ lse, float* __restrict__ partial) {
  constexpr int DB = DH / 16, NP = planes<T>(), kV = NP * Tile<T, DH>::kPlane, ROW = DH + 4;
  constexpr int kBytes = 4 * kV > 4 * 16 * ROW * 4 ? 4 * kV : 4 * 16 * ROW * 4;
  __shared__ __attribute__((aligned(16))) char lds[kBytes];
  __shared__ int s_bounds[64];
  __shared__ float s_table[16][2 * GDP_MAX_REL_BOUNDS + 3];
  __shared__ uint8_t s_bucket[4][kTile + kRelFewQueries];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  // the parts of one graph and key head side by side
  const int logical = xcd_remap(blockIdx.x, gridDim.x), kv_heads = e.heads / e.share;
  const int part = logical % parts, kvh = logical / parts % kv_heads;
  const Block b = block_of(rt, logical / parts / kv_heads, 16);
  const int len = rt.len[b.g], nq = rt.q0[b.g + 1] - rt.q0[b.g], pos0 = len - nq;
  const int columns = min(16, nq * e.share - b.i0);
  const T* kg = k + (size_t)rt.start[b.g] * e.ldk + kvh * DH;
  const T* vg = v + (size_t)rt.start[b.g] * e.ldv + kvh * DH;
  const uint8_t* mg = key_mask ? key_mask + rt.start[b.g] : nullptr;
  auto query_of = [&](int c) { return (b.i0 + min(c, columns - 1)) / e.share; };
  auto head_of = [&](int c) { return kvh * e.share + (b.i0 + min(c, columns - 1)) % e.share; };
  Buckets::stage(s_bounds, rb);
  for (int i = threadIdx.x; i < 16 * e.buckets; i += 256)
    s_table[i / e.buckets][i % e.buckets] = bias_of(table[(size_t)head_of(i / e.buckets) * e.buckets + i % e.buckets]);
  __syncthreads();
  const Buckets bk(s_bounds, rb, e.causal);
  const int pf = pos0 + query_of(0), pl = pos0 + query_of(15);
  const int k0 = span_of(e, pf, len).lo, k1 = span_of(e, pl, len).hi;
  const int tiles = (k1 - k0 + kTile - 1) / kTile, per = (tiles + parts - 1) / parts;
  const int end = min(tiles, (part + 1) * per);
  const int p = pos0 + query_of(col);
  const size_t row = (size_t)(rt.q0[b.g] + query_of(col));
  const int head = head_of(col);
  const Span span = span_of(e, p, len);
  Row<T, DH> qf[1];
  qf[0].load(q + row * e.ldq + head * DH, g4);
  f32x4 oacc[DB][1];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db][0] = zero4();
  float m = -INFINITY, lsum = 0.f;
  char* sV = lds + wave * kV;
  FewTile<T, DH> next;
  int i = part * per + wave;
  if (i < end) next.load(kg, e.ldk, vg, e.ldv, k0 + i * kTile, k1, lane);
  for (; i < end; i += 4) {
    const int t0 = k0 + i * kTile;
    f32x4 s[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      f32x4 low = zero4();
      s[kb] = zero4();
#pragma unroll
      for (int x = 0; x < FewTile<T, DH>::NK; ++x)
        mma_planes(FewTile<T, DH>::as_operand(next.k[kb][x]), qf[0].k[x], s[kb], low);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[kb][r] += low[r];
    }
    wave_lds_sync();                                       // the tile before this one has been read
    next.store_v(sV, lane);
    const uint64_t admitted = mg ? __ballot(mg[min(t0 + lane, k1 - 1)] != 0) : ~0ull;
    if (i + 4 < end) next.load(kg, e.ldk, vg, e.ldv, t0 + 4 * kTile, k1, lane);
    const int u = bk.common(t0 - pl, t0 + kTile - 1 - pf);
    if (u < 0) {                                           // buckets of the distances from t0 - pl on
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x * 64 + lane < kTile + pl - pf) s_bucket[wave][x * 64 + lane] = (uint8_t)bk.of(t0 - pl + x * 64 + lane);
    }
    wave_lds_sync();
    const float base = m == -INFINITY ? 0.f : m;
    const uint64_t on = (row_bits(span.lo - t0, span.hi - t0) & admitted) >> (4 * g4);
    const float bias = u >= 0 ? s_table[col][u] : 0.f;
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float add = u >= 0 ? bias : s_table[col][s_bucket[wave][kb * 16 + 4 * g4 + r + pl - p]];
        const float z = fmaf(s[kb][r], e.sc, add - base);
        s[kb][r] = (on >> (kb * 16 + r)) & 1ull ? z : -INFINITY;
        top = fmaxf(top, s[kb][r]);
      }
    top = fmaxf(top, xor_shfl(top, 16));
    top = fmaxf(top, xor_shfl(top, 32));
    const bool up = top > (m == -INFINITY ? -INFINITY : kRescale);
    const float by = up ? top : 0.f, corr = !up ? 1.f : m == -INFINITY ? 0.f : exp2_fast(-by);
    if (up) m = base + by;
    lsum *= corr;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) oacc[db][0][r] *= corr;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[kb][r] = exp2_fast(s[kb][r] - by);
        lsum += s[kb][r];
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float t[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        t[r] = s[2 * h][r];
        t[4 + r] = s[2 * h + 1][r];
      }
      Operand<NP> w[1] = {operand_of<NP>(t)};
      acc_rows<T, DH, 1>(oacc, sV, 32 * h, w, col, g4);
      if constexpr (NP == 1) {
#pragma unroll
        for (int r = 0; r < 8; ++r) t[r] -= to_f32(w[0].p[0][r]);
        w[0] = operand_of<NP>(t);
        acc_rows<T, DH, 1>(oacc, sV, 32 * h, w, col, g4);
      }
    }
  }
  lsum += xor_shfl(lsum, 16);
  lsum += xor_shfl(lsum, 32);
  // the waves' columns, joined: 16 threads a column, DB values each
  __syncthreads();
  float* mine = reinterpret_cast<float*>(lds) + wave * 16 * ROW + col * ROW;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) mine[16 * db + 4 * g4 + r] = oacc[db][0][r];
  if (g4 == 0) {
    mine[DH] = m;
    mine[DH + 1] = lsum;
  }
  __syncthreads();
  const int c = threadIdx.x >> 4, dim = (threadIdx.x & 15) * DB;
  if (c >= columns) return;
  const float* all = reinterpret_cast<const float*>(lds) + c * ROW;
  float M = -INFINITY, L = 0.f, out[DB];
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, all[w * 16 * ROW + DH]);
#pragma unroll
  for (int x = 0; x < DB; ++x) out[x] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = all[w * 16 * ROW + DH], f = mw == -INFINITY ? 0.f : exp2_fast(mw - M);
    L += f * all[w * 16 * ROW + DH + 1];
#pragma unroll
    for (int x = 0; x < DB; ++x) out[x] += f * all[w * 16 * ROW + dim + x];
  }
  const size_t orow = (size_t)(rt.q0[b.g] + query_of(c));
  const int oh = head_of(c);
  if (parts > 1) {
    float* to = partial + ((orow * e.heads + oh) * parts + part) * ROW;
#pragma unroll
    for (int x = 0; x < DB; ++x) to[dim + x] = out[x];
    if (dim == 0) {
      to[DH] = M;
      to[DH + 1] = L;
    }
  } else {
    const int op = pos0 + query_of(c);
    finish_few<T, DH, DB>(out, M, L, dim, q + orow * e.ldq + oh * DH, kg, e.ldk, vg, e.ldv, mg, span_of(e, op, len), op, e.sc, bk,
                          table + (size_t)oh * e.buckets, o + orow * e.ldo + oh * DH, lse ? lse + orow * e.heads + oh : nullptr);
  }
}

// One query and head a work-group: the parts' results, weighted by their maxima.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_rel_join(RelTable rt, RelBounds rb, Geo e, int parts, const T* __restrict__ q,
                                                  const T* __restrict__ k, const T* __restrict__ v,
                                                  const T* __restrict__ table, const uint8_t* __restrict__ key_mask,
                                                  T* __restrict__ o, float* __restrict__ lse,
                                                  const float* __restrict__ partial) {
  constexpr int ROW = DH + 4, NG = 256 / DH;
  __shared__ int s_bounds[64];
  __shared__ float s_m[4], s_l[NG], s_o[NG][DH];
  Buckets::stage(s_bounds, rb);
  const int head = blockIdx.x % e.heads, kvh = head / e.share, lane = threadIdx.x & 63;
  const size_t row = blockIdx.x / e.heads;
  const float* from = partial + (row * e.heads + head) * parts * ROW;
  float M = -INFINITY;
  for (int p = threadIdx.x; p < parts; p += 256) M = fmaxf(M, from[(size_t)p * ROW + DH]);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) M = fmaxf(M, xor_shfl(M, x));
  if (lane == 0) s_m[threadIdx.x >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  const int dim = threadIdx.x % DH, group = threadIdx.x / DH;
  float acc[1] = {0.f}, L = 0.f;
#pragma unroll 4
  for (int p = group; p < parts; p += NG) {
    const float mp = from[(size_t)p * ROW + DH], f = mp == -INFINITY ? 0.f : exp2_fast(mp - M);
    L += f * from[(size_t)p * ROW + DH + 1];
    acc[0] += f * from[(size_t)p * ROW + dim];
  }
  s_o[group][dim] = acc[0];
  if (dim == 0) s_l[group] = L;
  __syncthreads();
  if (group > 0) return;
  acc[0] = L = 0.f;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    acc[0] += s_o[g][dim];
    L += s_l[g];
  }
  int g = 0;                                               // the graph of the query
  for (int step = 64; step > 0; step >>= 1)
    if (g + step < rt.n && rt.q0[g + step] <= (int)row) g += step;
  const int len = rt.len[g], p = len - (rt.q0[g + 1] - rt.q0[g]) + (int)row - rt.q0[g];
  const Buckets bk(s_bounds, rb, e.causal);
  finish_few<T, DH, 1>(acc, M, L, dim, q + row * e.ldq + head * DH, k + (size_t)rt.start[g] * e.ldk + kvh * DH, e.ldk,
                       v + (size_t)rt.start[g] * e.ldv + kvh * DH, e.ldv, key_mask ? key_mask + rt.start[g] : nullptr,
                       span_of(e, p, len), p, e.sc, bk, table + (size_t)head * e.buckets, o + row * e.ldo + head * DH,
                       lse ? lse + row * e.heads + head : nullptr);
}

// dQ, and D for the other kernel ---------------------------------------------------------------

template <typename T, int DH, int COLS>
__global__ __launch_bounds__(256, 2) void k_rel_bwd_q(RelTable rt, RelBounds rb, Geo e, const T* __restrict__ dout,
                                                   const T* __restrict__ q, const T* __restrict__ k,
                                                   const T* __restrict__ v, const T* __restrict__ table,
                                                   const uint8_t* __restrict__ key_mask, const T* __restrict__ o,
                                                   const float* __restrict__ lse, T* __restrict__ dq,
                                                   float* __restrict__ D) {
  constexpr int DB = DH / 16, BQ = 64 * COLS, ND = kTile + BQ - 1;
  __shared__ __attribute__((aligned(16))) char lds[tile_lds<T, DH>()];
  __shared__ int s_bounds[64];
  __shared__ float s_table[2 * GDP_MAX_REL_BOUNDS + 2];
  __shared__ Diagonals<ND + 1> diag;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int head = logical % e.heads, kvh = head / e.share;
  const Block b = block_of(rt, logical / e.heads, BQ);
  const int len = rt.len[b.g], nq = rt.q0[b.g + 1] - rt.q0[b.g], pos0 = len - nq;
  const int count = min(BQ, nq - b.i0), p0 = pos0 + b.i0;
  const T* kg = k + (size_t)rt.start[b.g] * e.ldk + kvh * DH;
  const T* vg = v + (size_t)rt.start[b.g] * e.ldv + kvh * DH;
  const uint8_t* mg = key_mask ? key_mask + rt.start[b.g] : nullptr;
  Buckets::stage(s_bounds, rb);
  if ((int)threadIdx.x < e.buckets) s_table[threadIdx.x] = bias_of(table[(size_t)head * e.buckets + threadIdx.x]);
  __syncthreads();
  const Buckets bk(s_bounds, rb, e.causal);
  const Span first = span_of(e, p0, len), last = span_of(e, p0 + count - 1, len);
  const int k0 = first.lo, k1 = last.hi, tiles = (k1 - k0 + kTile - 1) / kTile;

  Row<T, DH> qf[COLS];
  Row<T, DH> df[COLS];
  constexpr bool REST = planes<T>() == 1;                  // an fp32 o leaves no rest
  f32x4 acc[DB][COLS], pk[DB][COLS];
  float L[COLS], D0[COLS], dsum[COLS];
  Span span[COLS];
  size_t row[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    const int i = min((wave * COLS + c) * 16 + col, count - 1);
    row[c] = (size_t)(rt.q0[b.g] + b.i0 + i);
    span[c] = span_of(e, p0 + i, len);
    qf[c].load(q + row[c] * e.ldq + head * DH, g4);
    df[c].load(dout + row[c] * e.lddo + head * DH, g4);
    L[c] = lse[row[c] * e.heads + head];
    if (L[c] == -INFINITY) L[c] = INFINITY;                // no key seen: every probability 0
    const T *po = o + row[c] * e.ldo + head * DH, *pd = dout + row[c] * e.lddo + head * DH;
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < DH / 4; ++j) t = fmaf(to_f32(po[g4 * (DH / 4) + j]), to_f32(pd[g4 * (DH / 4) + j]), t);
    t += xor_shfl(t, 16);
    D0[c] = t + xor_shfl(t, 32);
    dsum[c] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db][c] = pk[db][c] = zero4();
  }
  for_tiles<T, DH>(
      lds, tiles, {kg, e.ldk, k0, k1}, {vg, e.ldv, k0, k1},
      [&](int i) {
        const int t0 = k0 + i * kTile;
        const int u = bk.common(t0 - (p0 + BQ - 1), t0 + kTile - 1 - p0);
        if (u < 0 && (int)threadIdx.x < ND) diag.bias[i & 1][threadIdx.x] = s_table[bk.of(t0 - (p0 + BQ - 1) + (int)threadIdx.x)];
        const uint64_t s = mg ? __ballot(mg[min(t0 + lane, k1 - 1)] != 0) : ~0ull;
        return Keys{u, s};
      },
      [&](const char* sK, const char* sV, int i, const Keys& keys) {
        const int t0 = k0 + i * kTile, u = keys.bucket;
        const uint64_t admitted = keys.seen;
        const bool full = t0 >= last.lo && t0 + kTile <= first.hi && admitted == ~0ull;
        const float* d = diag.bias[i & 1] + (BQ - 1) - (wave * COLS * 16 + col) + 4 * g4;
        by_tile(!full, u < 0, [&](auto masked, auto diagonals) {
          constexpr bool MASKED = decltype(masked)::value, DIAG = decltype(diagonals)::value;
          const float bias = DIAG ? 0.f : s_table[u];
          uint64_t on[COLS];
          float less[COLS];
#pragma unroll
          for (int c = 0; c < COLS; ++c) {
            on[c] = MASKED ? (row_bits(span[c].lo - t0, span[c].hi - t0) & admitted) >> (4 * g4) : 0;
            less[c] = bias - L[c];
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float t[COLS][8], tp[COLS][8];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int kb = 2 * h + x;
              f32x4 s[COLS], dp[COLS];
              dot_rows<T, DH, COLS>(s, sK, kb * 16, qf, col, g4);
              dot_rows<T, DH, COLS>(dp, sV, kb * 16, df, col, g4);
#pragma unroll
              for (int c = 0; c < COLS; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  float p = exp2_fast(fmaf(s[c][r], e.sc, DIAG ? d[(kb - c) * 16 + r] - L[c] : less[c])), g = dp[c][r];
                  if (MASKED && !((on[c] >> (kb * 16 + r)) & 1ull)) p = g = 0.f;
                  dsum[c] = fmaf(p, g, dsum[c]);
                  t[c][4 * x + r] = p * (g - D0[c]);
                  tp[c][4 * x + r] = p;
                }
            }
            Operand<planes<T>()> w[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) w[c] = operand_of<planes<T>()>(t[c]);
            acc_rows<T, DH, COLS>(acc, sK, 32 * h, w, col, g4);
            if constexpr (REST) {
#pragma unroll
              for (int c = 0; c < COLS; ++c) {
#pragma unroll
                for (int r = 0; r < 8; ++r) t[c][r] -= to_f32(w[c].p[0][r]);
                w[c] = operand_of<1>(t[c]);
              }
              acc_rows<T, DH, COLS>(acc, sK, 32 * h, w, col, g4);
#pragma unroll
              for (int c = 0; c < COLS; ++c) w[c] = operand_of<1>(tp[c]);
              acc_rows<T, DH, COLS>(pk, sK, 32 * h, w, col, g4);
            }
          }
        });
      });
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    dsum[c] += xor_shfl(dsum[c], 16);
    dsum[c] += xor_shfl(dsum[c], 32);
    if ((wave * COLS + c) * 16 + col >= count) continue;
    if constexpr (REST) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[db][c][r] = fmaf(D0[c] - dsum[c], pk[db][c][r], acc[db][c][r]);
    }
    if (!(dsum[c] * 0.f == 0.f) || !finite_column(acc, c)) {
      const T *qr = q + row[c] * e.ldq + head * DH, *dr = dout + row[c] * e.lddo + head * DH;
      const int p = p0 + (wave * COLS + c) * 16 + col;
      f32x4 t[DB];
#pragma unroll
      for (int db = 0; db < DB; ++db) t[db] = zero4();
      auto pair = [&](int j, float& w) {                   // P and dP
        w = exp2f(fmaf(dot_f32<T, DH>(qr, kg + (size_t)j * e.ldk), e.sc, s_table[bk.of(j - p)] - L[c]));
        return dot_f32<T, DH>(dr, vg + (size_t)j * e.ldv);
      };
      float w;
      dsum[c] = 0.f;
      for (int j = span[c].lo; j < span[c].hi; ++j)
        if (!mg || mg[j]) {
          const float g = pair(j, w);
          dsum[c] = fmaf(w, g, dsum[c]);
        }
      for (int j = span[c].lo; j < span[c].hi; ++j)
        if (!mg || mg[j]) {
          const float g = pair(j, w);
          add_row<T, DB>(t, w * (g - dsum[c]), kg + (size_t)j * e.ldk, g4);
        }
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db][c] = t[db];
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const float t[4] = {acc[db][c][0] * e.scale, acc[db][c][1] * e.scale, acc[db][c][2] * e.scale, acc[db][c][3] * e.scale};
      store4(dq + row[c] * e.lddq + head * DH + db * 16 + 4 * g4, t);
    }
    if (g4 == 0) D[row[c] * e.heads + head] = dsum[c];
  }
}

// x of the lane N before this one in its row of 16, if that lane's bucket is this one's
template <int N>
__device__ __forceinline__ float row_right_if(float x, int bucket) {
  const int b = __builtin_amdgcn_update_dpp(-2, bucket, 0x110 + N, 0xf, 0xf, false);
  const float t = row_right<N>(x);
  return b == bucket ? t : 0.f;
}

// dK, dV and the table's gradient --------------------------------------------------------------

// The work-group's keys against every query that sees one of them, head after head of
// those that share the keys.  dtable: where a tile lies in one bucket its dS are added
// up in a lane's register until the bucket changes.  Elsewhere sums go along diagonals: the
// dS of row r of a block move r lanes within their 16 keys (a lane crossing keeps the value
// for the next block), so that one register adds up a block's 16 rows of four, and each
// wave and lane group leaves 80 sums a tile in LDS.  While the next tile is worked on, a
// thread a distance adds up the 16 that belong to it, and a scan over 16 distances adds
// those of one bucket.  Per work-group and head the sums go to partial in a fixed order.
// 29,000 queries of 4 graphs, 8 heads of 16, 512 keys a query, most tiles on diagonals: 109 us,
// the dQ pass 71; about half of it vector instructions, 14 a score.  (Diagonals through an LDS
// transpose of every 32 rows and a scan of 64 lanes each: 129.)
template <typename T, int DH, int COLS>
__global__ __launch_bounds__(256, planes<T>() == 1 && DH <= 32 ? 3 : 2)
void k_rel_bwd_kv(RelTable rt, RelBounds rb, Geo e, const T* __restrict__ dout, const T* __restrict__ q,
                  const T* __restrict__ k, const T* __restrict__ v, const T* __restrict__ table,
                  const uint8_t* __restrict__ key_mask, const float* __restrict__ lse, const float* __restrict__ D,
                  T* __restrict__ dk, T* __restrict__ dv, float* __restrict__ partial) {
  static_assert(COLS == 1, "a wave's diagonals are those of 16 keys");
  constexpr int DB = DH / 16, BK = 64, ND = kTile + BK - 1, KW = 16, NBK = 2 * GDP_MAX_REL_BOUNDS + 2;
  constexpr int NG = kTile + KW;                           // a lane group's diagonals of a tile: key - row + 64 in [0, NG)
  __shared__ __attribute__((aligned(16))) char lds[tile_lds<T, DH>()];
  __shared__ int s_bounds[64];
  __shared__ float s_table[NBK];
  __shared__ Diagonals<ND + 1> diag;
  __shared__ __attribute__((aligned(16))) float s_l[2][kTile], s_d[2][kTile];
  __shared__ int s_lo[2][kTile], s_hi[2][kTile];
  __shared__ float s_ds[2][16][NG];                        // by tile & 1, wave and lane group
  __shared__ int8_t s_bucket[4][ND + 1];                   // of tile i's distances in i & 3
  __shared__ float s_far[4][NBK], s_near[8][NBK];          // sums by bucket: of the waves' tiles; of rows of 16 distances
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
  const int logical = xcd_remap(blockIdx.x, gridDim.x);
  const int kv_heads = e.heads / e.share, kvh = logical % kv_heads, blk = logical / kv_heads;
  const Block b = block_of(rt, blk, BK);
  const int len = rt.len[b.g], q0 = rt.q0[b.g], nq = rt.q0[b.g + 1] - q0, pos0 = len - nq;
  const int kf0 = b.i0, kf1 = min(b.i0 + BK, len);         // the work-group's keys (positions)
  const size_t kbase = (size_t)rt.start[b.g];
  const uint8_t* mg = key_mask ? key_mask + kbase : nullptr;
  Buckets::stage(s_bounds, rb);
  for (int i = threadIdx.x; i < 4 * NBK; i += 256) s_far[i / NBK][i % NBK] = 0.f;
  for (int i = threadIdx.x; i < 8 * NBK; i += 256) s_near[i / NBK][i % NBK] = 0.f;
  __syncthreads();
  const Buckets bk(s_bounds, rb, e.causal);
  // queries that may see one of the keys: positions [pf, pl)
  const int pf = max(pos0, e.causal ? kf0 : kf0 / e.seg * e.seg);
  const int pl = min(len, (kf1 - 1 + e.mem) / e.seg * e.seg + e.seg);
  const int tiles = pl > pf ? (pl - pf + kTile - 1) / kTile : 0;

  Row<T, DH> kf[COLS];
  Row<T, DH> vf[COLS];
  f32x4 ak[DB][COLS], av[DB][COLS];
  int key[COLS];
  bool live[COLS];
  bool all = kf1 - kf0 == BK;
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    key[c] = kf0 + (wave * COLS + c) * 16 + col;
    live[c] = key[c] < kf1 && (!mg || mg[min(key[c], len - 1)] != 0);
    const size_t r = kbase + min(key[c], kf1 - 1);
    kf[c].load(k + r * e.ldk + kvh * DH, g4);
    vf[c].load(v + r * e.ldv + kvh * DH, g4);
    all = all && __all(live[c]);
#pragma unroll
    for (int db = 0; db < DB; ++db) ak[db][c] = av[db][c] = zero4();
  }
  for (int sh = 0; sh < e.share; ++sh) {
    const int head = kvh * e.share + sh;
    if ((int)threadIdx.x < e.buckets) s_table[threadIdx.x] = bias_of(table[(size_t)head * e.buckets + threadIdx.x]);
    __syncthreads();
    int cur = -1, last = 0;                                // the buckets of far, and of the tile before
    float far = 0.f;
    auto flush = [&]() {
      const float t = wave_sum(far);
      if (cur >= 0 && lane == 0) s_far[wave][cur] += t;
      far = 0.f;
      wave_lds_sync();
    };
    // wave 3's: lse and D of the next tile's row `lane`
    float row_l = 0.f, row_d = 0.f;
    auto load_row = [&](int i) {
      const size_t r = (size_t)(q0 + min(pf + i * kTile + lane, pl - 1) - pos0) * e.heads + head;
      row_l = lse[r];
      row_d = D[r];
    };
    if (wave == 3 && tiles > 0) load_row(0);
    auto collect = [&](int i) {                            // tile i's sums, all in LDS since a barrier: waves 2 and 3
      if (last >= 0 || wave < 2) return;
      int j = (int)threadIdx.x - 128;
      asm volatile("" : "+v"(j));                          // else 16 addresses and masks live through the loop
      const int bu = s_bucket[i & 3][j];
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int p = j + 1 - KW * w + 4 * g;
          const float z = s_ds[i & 1][4 * w + g][min(max(p, 0), NG - 1)];
          t += p >= 0 && p < NG ? z : 0.f;
        }
      // within a row of 16, the sum of a bucket's distances so far; its last one has all
      t += row_right_if<1>(t, bu);
      t += row_right_if<2>(t, bu);
      t += row_right_if<4>(t, bu);
      t += row_right_if<8>(t, bu);
      const int nb = __builtin_amdgcn_update_dpp(-2, bu, 0x101, 0xf, 0xf, false);
      if (bu >= 0 && nb != bu) s_near[j >> 4][bu] += t;
    };
    if (tiles > 0) {
      for_tiles<T, DH>(
          lds, tiles, {q + (size_t)q0 * e.ldq + head * DH, e.ldq, pf - pos0, pl - pos0},
          {dout + (size_t)q0 * e.lddo + head * DH, e.lddo, pf - pos0, pl - pos0},
          [&](int i) {
            const int t0 = pf + i * kTile, at = i & 1;
            const int u = bk.common(kf0 - (t0 + kTile - 1), kf0 + BK - 1 - t0);
            if (u < 0 && wave < 2) {
              const int j = threadIdx.x, rel = kf0 - (t0 + kTile - 1) + j, bu = bk.of(rel);
              if (j < ND) diag.bias[at][j] = s_table[bu];
              s_bucket[i & 3][j] = (int8_t)(j >= ND || (e.causal && rel > 0) ? -1 : bu);
            }
            if (wave == 3) {
              const int p = t0 + lane;
              const Span s = span_of(e, min(p, pl - 1), len);
              s_l[at][lane] = row_l == -INFINITY ? INFINITY : row_l;
              s_d[at][lane] = row_d;
              s_lo[at][lane] = p < pl ? s.lo : INT32_MAX;
              s_hi[at][lane] = p < pl ? s.hi : 0;
              load_row(i + 1);
            }
            return u;
          },
          [&](const char* sQ, const char* sD, int i, int u) {
            const int t0 = pf + i * kTile, at = i & 1;
            if (i > 0) collect(i - 1);
            last = u;
            const bool full = all && t0 + kTile <= pl && kf0 >= s_lo[at][kTile - 1] && kf1 <= s_hi[at][0];
            const float* d = diag.bias[at] + (kTile - 1) + wave * KW + col - 4 * g4;
            if (u >= 0 && u != cur) {
              flush();
              cur = u;
            }
            float* const sums = s_ds[at][4 * wave + g4] + col;
            by_tile(!full, u < 0, [&](auto masked, auto diagonals) {
              constexpr bool MASKED = decltype(masked)::value, DIAG = decltype(diagonals)::value;
              const float bias = DIAG ? 0.f : s_table[u];
              float next = 0.f;                            // of the 16 diagonals below the block's
#pragma unroll planes<T>() == 1 ? 2 : 1
              for (int h = 0; h < 2; ++h) {
                float tp[8], ts[8];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  const int row0 = 32 * h + 16 * x;
                  const float4 l4 = *reinterpret_cast<const float4*>(&s_l[at][row0 + 4 * g4]);
                  const float4 d4 = *reinterpret_cast<const float4*>(&s_d[at][row0 + 4 * g4]);
                  const float lr[4] = {l4.x, l4.y, l4.z, l4.w}, dr[4] = {d4.x, d4.y, d4.z, d4.w};
                  f32x4 s[1], dp[1];
                  dot_rows<T, DH, 1>(s, sQ, row0, kf, col, g4);
                  dot_rows<T, DH, 1>(dp, sD, row0, vf, col, g4);
#pragma unroll
                  for (int r = 0; r < 4; ++r) {
                    float p = exp2_fast(fmaf(s[0][r], e.sc, (DIAG ? d[-row0 - r] : bias) - lr[r])), g = dp[0][r] - dr[r];
                    if constexpr (MASKED) {
                      const int w = row0 + 4 * g4 + r;
                      const bool on = live[0] && key[0] >= s_lo[at][w] && key[0] < s_hi[at][w];
                      p = on ? p : 0.f;
                      g = on ? g : 0.f;
                    }
                    tp[4 * x + r] = p;
                    ts[4 * x + r] = p * g;
                  }
                  if constexpr (DIAG) {
                    const float* z = ts + 4 * x;
                    sums[kTile - row0] = (next + z[0]) + (row_left<1>(z[1]) + (row_left<2>(z[2]) + row_left<3>(z[3])));
                    next = row_right<15>(z[1]) + (row_right<14>(z[2]) + row_right<13>(z[3]));
                  } else {
                    far += (ts[4 * x] + ts[4 * x + 1]) + (ts[4 * x + 2] + ts[4 * x + 3]);
                  }
                }
                Operand<planes<T>()> w[1] = {operand_of<planes<T>()>(tp)};
                acc_rows<T, DH, 1>(av, sD, 32 * h, w, col, g4);
                w[0] = operand_of<planes<T>()>(ts);
                acc_rows<T, DH, 1>(ak, sQ, 32 * h, w, col, g4);
              }
              if constexpr (DIAG) sums[0] = next;
            });
          });
      collect(tiles - 1);
    }
    flush();
    __syncthreads();
    if ((int)threadIdx.x < e.buckets) {
      const int i = threadIdx.x;
      float sum = (s_far[0][i] + s_far[1][i]) + (s_far[2][i] + s_far[3][i]);
#pragma unroll
      for (int w = 0; w < 4; ++w) s_far[w][i] = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        sum += s_near[w][i];
        s_near[w][i] = 0.f;
      }
      partial[((size_t)blk * e.heads + head) * e.buckets + i] = sum;
    }
    __syncthreads();
  }
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    if (key[c] >= kf1) continue;
    if (!live[c]) {
#pragma unroll
      for (int db = 0; db < DB; ++db) ak[db][c] = av[db][c] = zero4();
    } else if (!finite_column(ak, c) || !finite_column(av, c)) {
      f32x4 tk[DB], tv[DB];
#pragma unroll
      for (int db = 0; db < DB; ++db) tk[db] = tv[db] = zero4();
      const T *kr = k + (kbase + key[c]) * e.ldk + kvh * DH, *vr = v + (kbase + key[c]) * e.ldv + kvh * DH;
      for (int sh = 0; sh < e.share; ++sh) {
        const int head = kvh * e.share + sh;
        for (int p = pf; p < pl; ++p) {
          const Span s = span_of(e, p, len);
          if (key[c] < s.lo || key[c] >= s.hi) continue;
          const size_t r = (size_t)(q0 + p - pos0);
          const T *qr = q + r * e.ldq + head * DH, *dr = dout + r * e.lddo + head * DH;
          const float bias = bias_of(table[(size_t)head * e.buckets + bk.of(key[c] - p)]);
          const float w = exp2f(fmaf(dot_f32<T, DH>(qr, kr), e.sc, bias - lse[r * e.heads + head]));
          add_row<T, DB>(tv, w, dr, g4);
          add_row<T, DB>(tk, w * (dot_f32<T, DH>(dr, vr) - D[r * e.heads + head]), qr, g4);
        }
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        ak[db][c] = tk[db];
        av[db][c] = tv[db];
      }
    }
    const size_t r = kbase + key[c];
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const float tk[4] = {ak[db][c][0] * e.scale, ak[db][c][1] * e.scale, ak[db][c][2] * e.scale, ak[db][c][3] * e.scale};
      const float tv[4] = {av[db][c][0], av[db][c][1], av[db][c][2], av[db][c][3]};
      store4(dk + r * e.lddk + kvh * DH + db * 16 + 4 * g4, tk);
      store4(dv + r * e.lddv + kvh * DH + db * 16 + 4 * g4, tv);
    }
  }
}

// dtable[h][b]: the work-groups' sums in order, in double.  A work-group takes 16
// entries, 16 threads each.
__global__ __launch_bounds__(256) void k_rel_table_grad(const float* __restrict__ partial, int blocks, int entries,
                                                        float* __restrict__ dtable) {
  __shared__ double s[16][17];
  const int x = threadIdx.x & 15, part = threadIdx.x >> 4, i = blockIdx.x * 16 + x;
  double t = 0.0;
  if (i < entries) {
    const int per = (blocks + 15) / 16, e = min(blocks, (part + 1) * per);
#pragma unroll 8
    for (int b = part * per; b < e; ++b) t += (double)partial[(size_t)b * entries + i];
  }
  s[part][x] = t;
  __syncthreads();
  if (part == 0 && i < entries) {
    double r = 0.0;
    for (int w = 0; w < 16; ++w) r += s[w][x];
    dtable[i] = (float)r;
  }
}

Geo geo_of(const gdp_rel_attn& a, const RelPlan& p) {
  Geo e;
  e.heads = a.n_heads;
  e.share = a.n_heads / a.n_kv_heads;
  e.seg = p.seg;
  e.mem = p.mem;
  e.causal = a.causal;
  e.buckets = p.buckets;
  e.scale = a.scale;
  e.sc = a.scale * kLog2e;
  e.ldq = a.ld_q;
  e.ldk = a.ld_k;
  e.ldv = a.ld_v;
  e.ldo = a.ld_o;
  e.lddo = a.ld_do;
  e.lddq = a.ld_dq;
  e.lddk = a.ld_dk;
  e.lddv = a.ld_dv;
  return e;
}

// The call's sequences with blocks of `rows` queries (or keys).
RelTable table_of(const gdp_rel_attn& a, int rows, bool keys) {
  RelTable t = {};
  t.n = a.n_graphs;
  for (int g = 0; g < a.n_graphs; ++g) {
    const int nq = a.n_query_h ? a.n_query_h[g] : a.len_h[g];
    t.start[g] = a.key_start_h[g];
    t.len[g] = a.len_h[g];
    t.q0[g + 1] = t.q0[g] + nq;
    t.blk[g + 1] = t.blk[g] + ((keys ? a.len_h[g] : nq) + rows - 1) / rows;
  }
  return t;
}
RelBounds bounds_of(const gdp_rel_attn& a) {
  RelBounds b = {};
  b.n = a.n_bounds;
  for (int i = 0; i < a.n_bounds; ++i) b.at[i] = a.bounds_h[i];
  return b;
}

// f(d_h as a constant, columns as a constant); TWO: the largest d_h with two columns
template <int TWO, typename F>
hipError_t by_shape(int dh, int cols, F f) {
  using std::integral_constant;
  constexpr integral_constant<int, 1> one{};
  constexpr integral_constant<int, 2> two{};
  if (cols == 2) {
    if constexpr (TWO >= 16)
      if (dh == 16) return f(integral_constant<int, 16>(), two);
    if constexpr (TWO >= 32)
      if (dh == 32) return f(integral_constant<int, 32>(), two);
    if constexpr (TWO >= 64)
      if (dh == 64) return f(integral_constant<int, 64>(), two);
    return hipErrorInvalidValue;
  }
  if (dh == 16) return f(integral_constant<int, 16>(), one);
  if (dh == 32) return f(integral_constant<int, 32>(), one);
  if (dh == 64) return f(integral_constant<int, 64>(), one);
  return hipErrorInvalidValue;
}

}  // namespace

template <typename T>
hipError_t launch_rel_attention(const gdp_rel_attn& a, const RelPlan& p, const T* q, const T* k, const T* v,
                                const T* table, const uint8_t* key_mask, T* o, float* lse, void* ws, hipStream_t s) {
  const Geo e = geo_of(a, p);
  const RelBounds rb = bounds_of(a);
  if (p.parts > 0) {
    float* partial = reinterpret_cast<float*>(ws);
    return by_shape<0>(a.head_dim, 1, [&](auto dh, auto) {
      RelTable rt = table_of(a, 1, false);
      for (int g = 0; g < rt.n; ++g) rt.blk[g + 1] = rt.blk[g] + ((rt.q0[g + 1] - rt.q0[g]) * e.share + 15) / 16;
      hipLaunchKernelGGL((k_rel_few<T, dh>), dim3((unsigned)rt.blk[rt.n] * a.n_kv_heads * p.parts), dim3(256), 0, s, rt, rb, e,
                         p.parts, q, k, v, table, key_mask, o, lse, partial);
      hipError_t err = hipGetLastError();
      if (err != hipSuccess || p.parts == 1) return err;
      hipLaunchKernelGGL((k_rel_join<T, dh>), dim3((unsigned)(p.queries * e.heads)), dim3(256), 0, s, rt, rb, e, p.parts, q, k, v,
                         table, key_mask, o, lse, (const float*)partial);
      return hipGetLastError();
    });
  }
  return by_shape<sizeof(T) == 2 ? 64 : 32>(a.head_dim, p.cols, [&](auto dh, auto cols) {
    const RelTable rt = table_of(a, 64 * cols, false);
    const int blocks = rt.blk[rt.n];
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL((k_rel_fwd<T, dh, cols>), dim3((unsigned)blocks * e.heads), dim3(256), 0, s, rt, rb, e, q, k, v, table,
                       key_mask, o, lse);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_rel_attention_backward(const gdp_rel_attn& a, const RelPlan& p, const T* dout, const T* q, const T* k,
                                         const T* v, const T* table, const uint8_t* key_mask, const T* o,
                                         const float* lse, T* dq, T* dk, T* dv, float* dtable, void* ws, hipStream_t s) {
  const Geo e = geo_of(a, p);
  const RelBounds rb = bounds_of(a);
  float* D = reinterpret_cast<float*>(static_cast<char*>(ws) + p.d);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(ws) + p.table_partial);
  hipError_t err = by_shape<0>(a.head_dim, 1, [&](auto dh, auto cols) {
    const RelTable rq = table_of(a, 64 * cols, false), rk = table_of(a, 64 * cols, true);
    const int bq = rq.blk[rq.n], bkv = rk.blk[rk.n];
    if (bq > 0) {
      hipLaunchKernelGGL((k_rel_bwd_q<T, dh, cols>), dim3((unsigned)bq * e.heads), dim3(256), 0, s, rq, rb, e, dout, q, k, v,
                         table, key_mask, o, lse, dq, D);
      const hipError_t r = hipGetLastError();
      if (r != hipSuccess) return r;
    }
    if (bkv > 0)
      hipLaunchKernelGGL((k_rel_bwd_kv<T, dh, cols>), dim3((unsigned)bkv * a.n_kv_heads), dim3(256), 0, s, rk, rb, e, dout, q,
                         k, v, table, key_mask, lse, D, dk, dv, partial);
    return hipGetLastError();
  });
  if (err != hipSuccess) return err;
  const int entries = a.n_heads * p.buckets;
  hipLaunchKernelGGL(k_rel_table_grad, dim3((unsigned)(entries + 15) / 16), dim3(256), 0, s, (const float*)partial, p.key_blocks,
                     entries, dtable);
  return hipGetLastError();
}

#define GDP_REL_INST(T)                                                                                                   \
  template hipError_t launch_rel_attention<T>(const gdp_rel_attn&, const RelPlan&, const T*, const T*, const T*, const T*, \
                                              const uint8_t*, T*, float*, void*, hipStream_t);                            \
  template hipError_t launch_rel_attention_backward<T>(const gdp_rel_attn&, const RelPlan&, const T*, const T*, const T*, \
                                                       const T*, const T*, const uint8_t*, const T*, const float*, T*, T*, \
                                                       T*, float*, void*, hipStream_t);
GDP_REL_INST(float)
GDP_REL_INST(bf16)
#undef GDP_REL_INST

}  // namespace op
}  // namespace gdp
