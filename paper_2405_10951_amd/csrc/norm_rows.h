// LayerNorm of rows as an operator (k_norm_rows.hip): raw device pointers and a stream, no allocation, no wait.
#pragma once
#include "bsr_internal.h"

namespace bsr {

struct NormRows {
  const void* x = nullptr; int64_t M = 0; int D = 0; int64_t ldx = 0;
  bool f32 = false;                                 // type of x and y
  const float *gamma = nullptr, *beta = nullptr;
  float eps = 0.f;
  void* y = nullptr; int64_t ldy = 0;               // null: none
  void* q = nullptr; uint8_t* scale = nullptr;      // the same rows in 8 bits (fp8.h); null: none
  float *mean = nullptr, *rstd = nullptr;           // null: none
};
void norm_rows_fwd(const NormRows& a, hipStream_t s);

constexpr int NORM_PARTIALS = 512;                  // most partial rows
struct NormRowsBwd {
  const void *dy = nullptr, *x = nullptr, *res = nullptr; int64_t lddy = 0, ldx = 0, ldr = 0;      // res null: none
  int64_t M = 0; int D = 0;
  bool f32 = false;                                 // type of dy, x, res and dx
  const float *mean = nullptr, *rstd = nullptr, *gamma = nullptr;
  void* dx = nullptr; int64_t lddx = 0;             // null: none
  float *dgamma = nullptr, *dbeta = nullptr;        // both or none
  float* partial = nullptr;                         // scratch of norm_rows_bwd_floats(D), where dgamma is given
};
inline size_t norm_rows_bwd_floats(int D) { return (size_t)NORM_PARTIALS * 2 * (((size_t)D + 7) / 8 * 8); }      // (partial rows are whole chunks)
void norm_rows_bwd(const NormRowsBwd& a, hipStream_t s);

}  // namespace bsr
