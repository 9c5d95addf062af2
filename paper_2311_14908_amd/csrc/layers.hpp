// layers.hpp -- the operators that turn tokens into rows of a machine and take its gradient back
// (layers.cpp checks the arguments, embed.hip, norm.hip, adamw.hip and svgrad.hip hold the kernels).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svmx.h"

namespace svmx {

// ---- embedding bags (embed.hip)
struct EmbedCall {
  const void *tokens;  // [T], int32 or int64 (wide)
  int32_t wide;
  int32_t mean;
  int64_t T;
  const int64_t *bags;  // [B + 1], or NULL: position i is bag i (B == T)
  int64_t B;
  int64_t padding;  // tokens of this value are left out (negative: none)
  int64_t V, d;
  float scale;
};
int64_t embed_scratch_bytes(int64_t T, int64_t d, int64_t B, bool bags);
hipError_t launch_embed(const EmbedCall &c, const void *table, int32_t table_type, int64_t ld_table, void *out,
                        int32_t out_type, int64_t ld_out, void *ws, hipStream_t s);
int64_t embed_grad_scratch_bytes(int64_t T, int64_t d, int64_t B);
hipError_t launch_embed_grad(const EmbedCall &c, const void *dy, int32_t dy_type, int64_t ld_dy, void *de,
                             int32_t de_type, int64_t ld_de, bool accumulate, void *ws, hipStream_t s);
// *invalid = 1 where a token that is not the padding lies outside 0 .. V-1, or the bags do not run from 0
// to T without decreasing (left as it is otherwise).
hipError_t launch_embed_check(const EmbedCall &c, int32_t *invalid, hipStream_t s);

// ---- layer norm (norm.hip)
struct NormCall {
  int64_t n, d;
  const void *x;
  int32_t x_type;
  int64_t ld_x;
  const void *w, *b;  // NULL: 1 and 0
  int32_t w_type;
};
hipError_t launch_layernorm(const NormCall &c, float eps, void *y, int32_t y_type, int64_t ld_y, float *mean, float *rstd,
                            hipStream_t s);
int64_t layernorm_grad_scratch_bytes(int64_t n, int64_t d, int32_t x_type);
hipError_t launch_layernorm_grad(const NormCall &c, const void *dy, int32_t dy_type, int64_t ld_dy, const float *mean,
                                 const float *rstd, void *dx, int64_t ld_dx, void *dw, void *db, void *ws, hipStream_t s);

// ---- AdamW (adamw.hip)
hipError_t launch_adamw(const svm_adamw_tensor *tensors, int64_t count, const svm_adamw_params &p, hipStream_t s);

// ---- gradients of a machine in rows (svgrad.hip)
struct SvGradCall {
  const float *X;  // [n][d]
  const int32_t *y;
  const double *alpha;
  int64_t n, d;
  double gamma;
  const float *Q;      // [m][d], or NULL: the objective's gradient in X itself
  const double *up;    // [m] or NULL (1)
  int64_t m;
  float *out;          // [m][d]
};
int64_t sv_grad_scratch_bytes(int64_t n, int64_t d, int64_t m, bool objective);
hipError_t launch_sv_grad(const SvGradCall &c, void *ws, hipStream_t s);

}  // namespace svmx
