// RMSNorm of rows with the residual's addition (k_rms_rows.hip): raw device pointers and a stream, no allocation, no wait.
#pragma once
#include "bsr_internal.h"

namespace bsr {

struct RmsRows {
  const void *x = nullptr, *res = nullptr; int64_t ldx = 0, ldr = 0;      // res null: none
  int64_t M = 0; int D = 0;
  bool f32 = false;                                 // type of x, res, sum and y
  const float* gamma = nullptr;
  float eps = 0.f;
  void* sum = nullptr; int64_t lds = 0;             // x + res; null: not wanted
  void* y = nullptr; int64_t ldy = 0;               // null: none
  void* q = nullptr; uint8_t* scale = nullptr;      // the same rows in 8 bits (fp8.h); null: none
  float* rstd = nullptr;                            // null: not wanted
};
void rms_rows_fwd(const RmsRows& a, hipStream_t s);

constexpr int RMS_PARTIALS = 512;                   // most partial rows
struct RmsRowsBwd {
  const void *dy = nullptr, *x = nullptr, *res = nullptr; int64_t lddy = 0, ldx = 0, ldr = 0;      // res null: none
  int64_t M = 0; int D = 0;
  bool f32 = false;                                 // type of dy, x, res and dx
  const float *rstd = nullptr, *gamma = nullptr;
  void* dx = nullptr; int64_t lddx = 0;             // null: none
  float* dgamma = nullptr;                          // null: none
  float* partial = nullptr;                         // scratch of rms_rows_bwd_floats(D), where dgamma is given
};
inline size_t rms_rows_bwd_floats(int D) { return (size_t)RMS_PARTIALS * (((size_t)D + 7) / 8 * 8); }      // (partial rows are whole chunks)
void rms_rows_bwd(const RmsRowsBwd& a, hipStream_t s);

}  // namespace bsr
