// 8-bit operands: e4m3 values with a power-of-two scale (an E8M0 byte, exponent + 127) for each block of 128.
//   e = the smallest integer >= -127 with max|x| 2^-e <= 448 (the largest e4m3 value; e = 0 for a block of zeros),
//   q = x 2^-e rounded to e4m3, to nearest, ties to even.
// Powers of two, because then everything but that one rounding is exact (any implementation gives the same bits) and because the matrix
// instructions of gfx950 take such scales beside their operands: dividing them out costs nothing.
// Non-finite values do not count towards the maximum and become NaN, which the products then show.
// Rows are padded with zeros to whole blocks (leading dimension ld8), scales to whole dwords (ld8s).
#pragma once
#include "rowops.h"

namespace bsr {

constexpr int BLOCK8 = 128;
__host__ __device__ inline int64_t ld8(int64_t k) { return (k + BLOCK8 - 1) / BLOCK8 * BLOCK8; }
__host__ __device__ inline int64_t ld8s(int64_t k) { return ((k + BLOCK8 - 1) / BLOCK8 + 3) / 4 * 4; }

// bits of |x|, 0 where x is not finite
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// the scale byte of a block from the bits of its largest |x|: 448 = 1.75 2^8
__device__ __forceinline__ uint32_t scale8_of(uint32_t bits) {
  return bits == 0 ? 127u : (uint32_t)max((int)(bits >> 23) - 8 + (int)((bits & 0x7fffffu) > 0x600000u), 0);
}
__device__ __forceinline__ float inverse_of(uint32_t scale8) { return __uint_as_float((254u - scale8) << 23); }      // 2^-e
// four values, brought into range by inv
__device__ __forceinline__ uint32_t pack8(float a, float b, float c, float d, float inv) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, lo, true);
}

// ---- launchers (device pointers, no allocation, no wait) -----------------------------------------------------------------------
// x [M,K] (bf16 or fp32, row stride ldx) -> q [M, ld8(K)], scale [M, ld8s(K)]
void quantize8_rows(const void* x, bool f32, int64_t M, int K, int64_t ldx, void* q, uint8_t* scale, hipStream_t s);
// w [in,out] (row stride ldw) -> blocks of 128 x 128, as [out, ld8(in)] with scales [ceil(out / 128), ld8s(in)] and, where q_back is given,
// as [in, ld8(out)] with scales [ceil(in / 128), ld8s(out)]
void quantize8_weight(const void* w, bool f32, int in, int out, int64_t ldw, void* q, uint8_t* scale, void* q_back, uint8_t* scale_back,
                      hipStream_t s);

// C[M,N] = epilogue(sum_k A(m,k) B(n,k)), A rows of 128-blocks, B blocks of 128 x 128
struct Gemm8Desc {
  const void* A = nullptr; const uint8_t* a_scale = nullptr;
  const void* B = nullptr; const uint8_t* b_scale = nullptr;
  int M = 0, N = 0, K = 0;
  int64_t lda = 0;                 // elements between rows of A (few-row form with a_type other than 8 bits)
  int a_type = 2;                  // 0 bf16, 1 fp32 (few-row form: brought to 8 bits on the way in), 2 e4m3
  bool out_f32 = false;            // type of C, res and aux: fp32, else bf16; all of row stride ldc
  bool cut = false;                // bf16 results: the 8-bit instructions may add the products (k_gemm8.hip: what that cuts)
  void* C = nullptr; int64_t ldc = 0;
  const float* bias = nullptr;     // [N]
  int act = 0;                     // Act
  void* aux = nullptr;             // ACT_GELU: receives the pre-activation where given; ACT_GELU_BWD: the stored one
  const void* res = nullptr;       // added last
};
bool gemm8_few_takes(int64_t M);   // products that the few-row form runs (it takes operands of any a_type)
void gemm8(const Gemm8Desc& g, hipStream_t s);

}  // namespace bsr
