// Launch interface of the layer operators: LayerNorm (norm.hip), FC layers (fc.hip)
// and position-biased segment attention (rel_attention.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gdp.h"
#include "host_plan.h"

namespace gdp {
namespace op {

// ---- LayerNorm -----------------------------------------------------------------
template <typename T>
struct NormArgs {
  int64_t rows;
  int width;
  const T* x;        // forward: x; backward: the stored sum h
  int64_t ldx;
  const T* res;      // forward: residual or NULL; backward: dsum or NULL
  int64_t ldr;
  const T *gamma, *beta;
  float eps;
  const T* dy;       // backward
  int64_t lddy;
  T* y;              // forward: y; backward: dh
  int64_t ldy;
  T* sum;            // forward: the sum, or NULL
  int64_t lds;
};
template <typename T>
hipError_t launch_norm(const NormArgs<T>& a, hipStream_t s);
// partial: norm_backward_blocks() rows of 2 width floats.
template <typename T>
hipError_t launch_norm_backward(const NormArgs<T>& a, float* partial, float* dgamma, float* dbeta, hipStream_t s);

// ---- FC layers -------------------------------------------------------------------
// y = act(x W^T + b) + residual; act_out (may be NULL) = act(...)
template <typename T>
hipError_t launch_fc(const gdp_fc_layer& f, const T* x, const T* w, const T* b, const T* residual, T* y, T* act_out,
                     hipStream_t s);
template <typename T>
hipError_t launch_fc_backward(const gdp_fc_layer& f, const FcPlan& p, const T* dy, const T* x, const T* w,
                              const T* act_out, const T* dx_add, T* dx, float* dw, float* db, void* ws, hipStream_t s);

// ---- attention ---------------------------------------------------------------------
// The sequences of a call by value: keys of graph g in rows [start, start + len), its
// queries (the last count positions) in rows [q0[g], q0[g + 1]); blk: prefix of the
// work blocks of the kernel it is made for.
struct RelTable {
  int n;
  int start[GDP_MAX_GRAPHS], len[GDP_MAX_GRAPHS], q0[GDP_MAX_GRAPHS + 1], blk[GDP_MAX_GRAPHS + 1];
};
struct RelBounds {
  int n;
  int at[GDP_MAX_REL_BOUNDS];
};
template <typename T>
hipError_t launch_rel_attention(const gdp_rel_attn& a, const RelPlan& p, const T* q, const T* k, const T* v,
                                const T* table, const uint8_t* key_mask, T* o, float* lse, void* ws, hipStream_t s);
template <typename T>
hipError_t launch_rel_attention_backward(const gdp_rel_attn& a, const RelPlan& p, const T* dout, const T* q, const T* k,
                                         const T* v, const T* table, const uint8_t* key_mask, const T* o,
                                         const float* lse, T* dq, T* dk, T* dv, float* dtable, void* ws, hipStream_t s);

}  // namespace op
}  // namespace gdp
