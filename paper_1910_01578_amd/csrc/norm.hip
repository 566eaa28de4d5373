// LayerNorm of a sum, forward and backward.
//
//   h = x + residual,  mean and variance of h's row,  xhat = (h - mean) rstd,  y = xhat gamma + beta
//   g = dy gamma,  dh = rstd (g - mean(g) - xhat mean(g xhat)) + dsum,  dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
//
// A row is held by LPR lanes (8 to 64 of a wave, or a work-group's 256), C vectors of 16
// bytes each, so that it is read once: the mean, then the squares about it, come from
// registers.  The backward forms both again from h, which costs no memory traffic and
// leaves nothing but h to keep.  All in fp32.
//
// The weights' gradients: a lane adds up its columns over the rows that its group walks,
// the groups of a work-group are added through LDS, and each work-group leaves one row of
// partial sums; k_norm_weights adds those in a fixed order, in double.
//
// What bounds it: memory.  52,000 rows of 256, bf16: forward with a residual and the sum kept
// 18 us (106 MB, 5.8 TB/s; what another kernel just wrote comes from the last cache), backward
// 22.6 us and 3.8 for the weights' sums (4.0 TB/s in all); 4,099 rows of 1,001, which no
// vector load fits: 9.3 and 19.5 us; 256 rows of 64, fp32: 3.6 us, a launch.
#include <algorithm>

#include "op_common.h"
#include "op_kernels.h"

namespace gdp {
namespace op {

namespace {

// Sum over the LPR lanes of a row (LPR = 256: the work-group, through red[4]).
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int m = 1; m < (LPR < 64 ? LPR : 64); m <<= 1) v += xor_shfl(v, m);
  if constexpr (LPR == 256) {
    __syncthreads();                                       // the sum before this one has been read
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[0] + red[1]) + (red[2] + red[3]);
  }
  return v;
}

// A lane's elements of one row: vector c holds columns (c LPR + lane) V and on.
template <typename T, int LPR, int C>
struct RowPart {
  static constexpr int V = Vec16<T>::N;
  static __device__ __forceinline__ int column(int c, int l) { return (c * LPR + l) * V; }
  // zeros past the row's end
  static __device__ __forceinline__ void load(const T* p, int width, int l, float (&f)[C][V]) {
    Vec16<T> t[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int j = column(c, l);
      if (j < width) t[c] = load16_part(p + j, width - j);
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) f[c][i] = column(c, l) < width ? to_f32(t[c].v[i]) : 0.f;
  }
  static __device__ __forceinline__ void store(T* p, int width, int l, const float (&f)[C][V]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int j = column(c, l);
      if (j >= width) continue;
      Vec16<T> t;
#pragma unroll
      for (int i = 0; i < V; ++i) t.v[i] = from_f32<T>(f[c][i]);
      store16_part(p + j, t, width - j);
    }
  }
};

// h -> h - mean (zeros stay zeros past the row's end); returns rstd
template <typename T, int LPR, int C>
__device__ __forceinline__ float centre(float (&h)[C][Vec16<T>::N], int width, int l, float eps, float* red) {
  constexpr int V = Vec16<T>::N;
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) s += h[c][i];
  const float mean = row_sum<LPR>(s, red) / (float)width;
  s = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      h[c][i] = RowPart<T, LPR, C>::column(c, l) + i < width ? h[c][i] - mean : 0.f;
      s = fmaf(h[c][i], h[c][i], s);
    }
  return 1.0f / sqrtf(row_sum<LPR>(s, red) / (float)width + eps);
}

template <typename T, int LPR, int C>
__global__ __launch_bounds__(256) void k_norm(NormArgs<T> a) {
  constexpr int V = Vec16<T>::N, RPW = 256 / LPR;
  using R = RowPart<T, LPR, C>;
  __shared__ float red[4];
  const int l = threadIdx.x % LPR;
  float gamma[C][V], beta[C][V];
  R::load(a.gamma, a.width, l, gamma);
  R::load(a.beta, a.width, l, beta);
  for (int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / LPR; r < a.rows; r += (int64_t)gridDim.x * RPW) {
    float h[C][V];
    R::load(a.x + r * a.ldx, a.width, l, h);
    if (a.res) {
      float t[C][V];
      R::load(a.res + r * a.ldr, a.width, l, t);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) h[c][i] += t[c][i];
    }
    if (a.sum) R::store(a.sum + r * a.lds, a.width, l, h);
    const float rstd = centre<T, LPR, C>(h, a.width, l, a.eps, red);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) h[c][i] = fmaf(h[c][i] * rstd, gamma[c][i], beta[c][i]);
    R::store(a.y + r * a.ldy, a.width, l, h);
  }
}

template <typename T, int LPR, int C>
__global__ __launch_bounds__(256) void k_norm_bwd(NormArgs<T> a, float* __restrict__ partial) {
  constexpr int V = Vec16<T>::N, RPW = 256 / LPR;
  using R = RowPart<T, LPR, C>;
  __shared__ float red[4];
  __shared__ float s_part[RPW > 1 ? RPW : 1][RPW > 1 ? LPR * C * V : 1];
  const int l = threadIdx.x % LPR, group = threadIdx.x / LPR;
  float gamma[C][V], dg[C][V], db[C][V];
  R::load(a.gamma, a.width, l, gamma);
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) dg[c][i] = db[c][i] = 0.f;
  const float inv = 1.0f / (float)a.width;
  for (int64_t r = (int64_t)blockIdx.x * RPW + group; r < a.rows; r += (int64_t)gridDim.x * RPW) {
    float h[C][V], g[C][V], t[C][V];
    R::load(a.x + r * a.ldx, a.width, l, h);
    R::load(a.dy + r * a.lddy, a.width, l, g);
    if (a.res) R::load(a.res + r * a.ldr, a.width, l, t);
    const float rstd = centre<T, LPR, C>(h, a.width, l, a.eps, red);
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[c][i] *= rstd;                                   // xhat
        dg[c][i] = fmaf(g[c][i], h[c][i], dg[c][i]);
        db[c][i] += g[c][i];
        g[c][i] *= gamma[c][i];
        s += g[c][i];
        q = fmaf(g[c][i], h[c][i], q);
      }
    s = row_sum<LPR>(s, red) * inv;
    q = row_sum<LPR>(q, red) * inv;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        g[c][i] = rstd * (g[c][i] - s - h[c][i] * q);
        if (a.res) g[c][i] += t[c][i];
      }
    R::store(a.y + r * a.ldy, a.width, l, g);
  }
  float* out = partial + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float(&d)[C][V] = which ? db : dg;
    if constexpr (RPW > 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) s_part[group][R::column(c, l) + i] = d[c][i];
      __syncthreads();
      for (int j = threadIdx.x; j < a.width; j += 256) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < RPW; ++w) t += s_part[w][j];
        out[which * a.width + j] = t;
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (R::column(c, l) + i < a.width) out[which * a.width + R::column(c, l) + i] = d[c][i];
    }
  }
}

// 16 of the 2 width columns a work-group, 64 threads each.
__global__ __launch_bounds__(1024) void k_norm_weights(const float* __restrict__ partial, int blocks, int width,
                                                       float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ double s[64][17];
  const int x = threadIdx.x & 15, part = threadIdx.x >> 4, j = blockIdx.x * 16 + x, n = 2 * width;
  double t = 0.0;
  if (j < n) {
#pragma unroll 8
    for (int b = part; b < blocks; b += 64) t += (double)partial[(size_t)b * n + j];
  }
  s[part][x] = t;
  __syncthreads();
  if (part == 0 && j < n) {
    double r = 0.0;
    for (int w = 0; w < 64; ++w) r += s[w][x];
    if (j < width) dgamma[j] = (float)r;
    else dbeta[j - width] = (float)r;
  }
}

// The least vectors a lane, then the least group, that hold a row: f(lanes, vectors a lane).
// (52,000 rows of 256, 32 lanes of one vector against 16 of two: 18.5 and 19.1 us, backward
// 25.1 and 30.1.  Above a wave's vectors two a lane come before a work-group's barriers, 64 of
// two against 256 of one at a width of 1,024: 85 and 92 us, backward 126 and 170.)
template <typename T, typename F>
hipError_t by_width(int width, F f) {
  using std::integral_constant;
  const int vecs = (width + Vec16<T>::N - 1) / Vec16<T>::N;
#define GDP_NORM_CASE(LPR, C) \
  if (vecs <= LPR * C) return f(integral_constant<int, LPR>(), integral_constant<int, C>())
  GDP_NORM_CASE(8, 1);
  GDP_NORM_CASE(16, 1);
  GDP_NORM_CASE(32, 1);
  GDP_NORM_CASE(64, 1);
  GDP_NORM_CASE(64, 2);
  GDP_NORM_CASE(256, 1);
  GDP_NORM_CASE(256, 2);
  GDP_NORM_CASE(256, 4);
  if constexpr (sizeof(T) == 4) GDP_NORM_CASE(256, 8);
#undef GDP_NORM_CASE
  return hipErrorInvalidValue;
}

}  // namespace

template <typename T>
hipError_t launch_norm(const NormArgs<T>& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return by_width<T>(a.width, [&](auto lpr, auto c) {
    const int64_t groups = (a.rows + 256 / lpr - 1) / (256 / lpr);
    hipLaunchKernelGGL((k_norm<T, lpr, c>), dim3((unsigned)std::min<int64_t>(groups, 2048)), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_norm_backward(const NormArgs<T>& a, float* partial, float* dgamma, float* dbeta, hipStream_t s) {
  int blocks = norm_backward_blocks(a.rows, a.width);
  // bf16 rows of two vectors a lane fill the registers of three work-groups a CU: two of them
  // each, in one round (4,099 rows of 1,001: 24.9 us with 1,001 groups, 20.8 with 768, 19.5 so;
  // 52,000 of 1,024: 124 and 120; fp32, whose vectors are half as long: 140 and 232)
  if (sizeof(T) == 2 && a.width > 64 * Vec16<T>::N && a.width <= 128 * Vec16<T>::N) blocks = std::min(blocks, 512);
  if (blocks > 0) {
    const hipError_t e = by_width<T>(a.width, [&](auto lpr, auto c) {
      hipLaunchKernelGGL((k_norm_bwd<T, lpr, c>), dim3((unsigned)blocks), dim3(256), 0, s, a, partial);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_norm_weights, dim3((unsigned)(2 * a.width + 15) / 16), dim3(1024), 0, s, (const float*)partial, blocks,
                     a.width, dgamma, dbeta);
  return hipGetLastError();
}

#define GDP_NORM_INST(T)                                                    \
  template hipError_t launch_norm<T>(const NormArgs<T>&, hipStream_t);      \
  template hipError_t launch_norm_backward<T>(const NormArgs<T>&, float*, float*, float*, hipStream_t);
GDP_NORM_INST(float)
GDP_NORM_INST(bf16)
#undef GDP_NORM_INST

}  // namespace op
}  // namespace gdp
