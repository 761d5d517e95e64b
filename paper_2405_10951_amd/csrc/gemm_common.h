// What the matrix-product kernels share: GELU, compile-time loops, the LDS chunk swizzle, the order of tiles over the XCDs, waits.
#pragma once
#include <utility>

#include "bsr_internal.h"

namespace bsr {

constexpr int NXCD = 8;

// GELU(u) = u Phi(u) and its derivative Phi(u) + u phi(u), for bf16 results.  erf comes from
// the rational-exponential form of Abramowitz & Stegun 7.1.26, |error| <= 1.5e-7: Phi is within 5e-7 in fp32 arithmetic, at a
// fraction of the instructions of erff.  That is below half an ulp of the bf16 result wherever Phi is above 2.6e-4 (u > -3.5); further out, where
// GELU is below 9e-4 in size, it is an absolute error and no longer a relative one (4 % of GELU at u = -5, which is 1.4e-6).  Its exp(-x^2) with x = u / sqrt(2) is the Gaussian
// that phi(u) needs as well.  Its coefficients are halved, so that it is Phi that comes out: exact, and one product of 22 less.
__device__ inline float phi_as(float u, float& gauss) {
  const float x = u * 0.70710678118654752f, ax = fabsf(x);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, ax, 1.0f));
  float p = fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
  p = fmaf(p, t, 0.5f * 1.421413741f);
  p = fmaf(p, t, 0.5f * -0.284496736f);
  p = fmaf(p, t, 0.5f * 0.254829592f);
  gauss = __expf(-ax * ax);
  return 0.5f + copysignf(fmaf(-p * t, gauss, 0.5f), x);
}
__device__ inline float gelu_f(float u) {
  float gauss;
  return u * phi_as(u, gauss);
}
__device__ inline float gelu_grad_f(float u) {
  float gauss;
  const float cdf = phi_as(u, gauss);
  return fmaf(u * 0.39894228040143268f, gauss, cdf);
}

// The same for fp32 results: Phi within 6.3e-8, as 0.5 (1 + erff(u / sqrt(2))) has it, and on the negative side, where that form has nothing left below u = -5.4, to
// a relative error of u^2 2^-24 and a few units in the last place.  Near 0 an odd polynomial about 1/2, further out Phi(-|u|) = t P(t) exp(-u^2 / 2) with
// t = 1 / (1 + 0.4 |u| / sqrt(2)); both fitted to the least largest error (1e-10, and 4e-8 of the value), in 64 bits.  Both sides are worked out and one is chosen; a
// wavefront would take the cases of erfcf one after the other (6304 x 768 x 2304 to fp32 with GELU 37 us, with that 49, with the form above 34).
__device__ inline float phi_fp32(float u, float& gauss) {
  const float s = u * u, t = __builtin_amdgcn_rcpf(fmaf(0.282842712f, fabsf(u), 1.0f));
  gauss = __builtin_amdgcn_exp2f(s * -0.72134752044448170f);
  float n = fmaf(4.77419268e-07f, s, -9.06477662e-06f);
  n = fmaf(n, s, 0.000115043367f);
  n = fmaf(n, s, -0.00118711877f);
  n = fmaf(n, s, 0.00997350332f);
  n = fmaf(n, s, -0.0664903749f);
  n = fmaf(n, s, 0.39894228f);
  float p = fmaf(-0.0581641248f, t, 0.121886168f);
  p = fmaf(p, t, 0.00404896604f);
  p = fmaf(p, t, 0.106566807f);
  p = fmaf(p, t, 0.0993798277f);
  p = fmaf(p, t, 0.113347899f);
  p = fmaf(p, t, 0.112813417f);
  const float far = p * t * gauss;
  return fabsf(u) < 1.25f ? fmaf(u, n, 0.5f) : u < 0.f ? far : 1.0f - far;
}
__device__ inline float gelu_fp32(float u) {
  float gauss;
  return u * phi_fp32(u, gauss);
}
__device__ inline float gelu_grad_fp32(float u) {
  float gauss;
  const float cdf = phi_fp32(u, gauss);
  return fmaf(u * 0.39894228040143268f, gauss, cdf);
}
template <bool FP32> __device__ __forceinline__ float gelu_to(float u) {
  if constexpr (FP32) return gelu_fp32(u);
  else return gelu_f(u);
}
template <bool FP32> __device__ __forceinline__ float gelu_grad_to(float u) {
  if constexpr (FP32) return gelu_grad_fp32(u);
  else return gelu_grad_f(u);
}

template <int V> struct IC { static constexpr int value = V; };   // compile-time flag for generic lambdas
// f(IC<0>{}), ..., f(IC<N-1>{}): a loop whose index is a compile-time constant in the body
template <class F, int... I> __device__ __forceinline__ void sfor_impl(F&& f, std::integer_sequence<int, I...>) { (f(IC<I>{}), ...); }
template <int N, class F> __device__ __forceinline__ void sfor(F&& f) { sfor_impl(f, std::make_integer_sequence<int, N>{}); }

// LDS chunk swizzle: 16 consecutive rows reading the same logical 16-byte chunk hit 16 different
// (row parity, chunk position) pairs, i.e. all 64 banks once; 8 consecutive rows hit 8 positions.
__device__ inline int swz(int row) { return (row & 7) ^ ((row >> 3) & 1); }

// Logical tile id of this workgroup: XCD x owns the contiguous range [start(x), start(x+1)).
__device__ inline int xcd_remap(int pid, int nblocks) {
  const int base = nblocks / NXCD, rem = nblocks % NXCD;
  const int x = pid % NXCD, local = pid / NXCD;
  return x * base + min(x, rem) + local;
}

template <int N> __device__ __forceinline__ void wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}
__device__ __forceinline__ void wait_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4)); }
#define BSR_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)
#define BSR_GLOBAL_PTR(p) ((const void __attribute__((address_space(1)))*)(p))
#define BSR_LDS_VOID(p) ((void __attribute__((address_space(3)))*)(p))

}  // namespace bsr
