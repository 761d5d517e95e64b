// Rows and weight matrices brought to 8 bits (fp8.h).  Bound by memory: 3 bytes move per bf16 element.
#include <algorithm>

#include "fp8.h"

namespace bsr {

namespace {

__device__ __forceinline__ uint32_t umax_dpp(uint32_t v, uint32_t o) { return v > o ? v : o; }
// maximum over each eight lanes (the pairs of eight_sum in rowops.h)
__device__ __forceinline__ uint32_t eight_max(uint32_t v) {
  v = umax_dpp(v, __float_as_uint(dpp_move<0xB1>(__uint_as_float(v))));
  v = umax_dpp(v, __float_as_uint(dpp_move<0x4E>(__uint_as_float(v))));
  return umax_dpp(v, __float_as_uint(dpp_move<0x141>(__uint_as_float(v))));
}

// Eight lanes take a block, 16 elements each; blocks count row after row, the padding of the scales included, so that a wavefront's
// scales are consecutive bytes.  16384 x 4096 bf16: 31 us (200 MB, 39 at the rate of a large copy: the rows fit the caches), 16384 x 4095 (rows at any address) 32.
template <typename T>
__global__ __launch_bounds__(256) void quantize8_rows_kernel(const T* __restrict__ x, int64_t blocks, int K, int64_t ldx, int per_row,
                                                             int real_blocks, uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  const int64_t b = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
  if (b >= blocks) return;
  const int64_t row = b / per_row;
  const int kb = (int)(b - row * per_row), part = threadIdx.x & 7, k0 = kb * BLOCK8 + part * 16;
  float v[16];
  const T* src = x + row * ldx + k0;
  if (k0 + 16 <= K) {
    constexpr int V = Chunk<T>::V;
    typename Chunk<T>::vec raw[16 / V];
#pragma unroll
    for (int i = 0; i < 16 / V; ++i) raw[i] = *(const typename Loose<T>::vec*)(src + i * V);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)raw[i / V][i % V];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)x[row * ldx + min(k0 + i, K - 1)];           // (no branch around a load)
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = k0 + i < K ? v[i] : 0.f;
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = umax_dpp(most, finite_bits(v[i]));
  const uint32_t s8 = scale8_of(eight_max(most));
  if (kb < real_blocks) {
    const float inv = inverse_of(s8);
    *(uint4*)(q + row * (int64_t)real_blocks * BLOCK8 + k0) =
        make_uint4(pack8(v[0], v[1], v[2], v[3], inv), pack8(v[4], v[5], v[6], v[7], inv), pack8(v[8], v[9], v[10], v[11], inv),
                   pack8(v[12], v[13], v[14], v[15], inv));
  }
  if (part == 0) scale[b] = (uint8_t)s8;
}

// A workgroup per block, 64 values a thread: piece t % P of rows t / P, t / P + 256 / P, ... (P 16-byte pieces a row of the
// block).  The transposed copy goes through LDS.  Once per weight matrix.  4096 x 8192 bf16: 24 us, with both copies.
template <typename T>
__global__ __launch_bounds__(256) void quantize8_weight_kernel(const T* __restrict__ w, int in, int out, int64_t ldw, uint8_t* __restrict__ q,
                                                               uint8_t* __restrict__ scale, uint8_t* __restrict__ q_back,
                                                               uint8_t* __restrict__ scale_back) {
  constexpr int V = Chunk<T>::V, P = BLOCK8 / V, STEP = 256 / P, N = BLOCK8 / STEP;
  __shared__ uint8_t tile[BLOCK8][BLOCK8 + 4];
  __shared__ uint32_t wave_most[4];
  const int i0 = blockIdx.y * BLOCK8, n0 = blockIdx.x * BLOCK8;
  const int r0 = threadIdx.x / P, c = threadIdx.x % P * V;
  float v[N][V];
  uint32_t most = 0;
  typename Chunk<T>::vec raw[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int i = i0 + r0 + k * STEP;
    const T* src = w + (int64_t)min(i, in - 1) * ldw + n0 + c;
    if (n0 + c + V <= out) raw[k] = *(const typename Loose<T>::vec*)src;
    else
#pragma unroll
      for (int e = 0; e < V; ++e) raw[k][e] = n0 + c + e < out ? src[e] : (T)0.f;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[k][e] = i0 + r0 + k * STEP < in ? (float)raw[k][e] : 0.f;
      most = umax_dpp(most, finite_bits(v[k][e]));
    }
  // bits of non-negative floats order as the floats do
  most = __float_as_uint(wave_max(__uint_as_float(most)));
  if ((threadIdx.x & 63) == 0) wave_most[threadIdx.x >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) most = umax_dpp(most, wave_most[i]);
  const uint32_t s8 = scale8_of(most);
  const float inv = inverse_of(s8);
  const int64_t ldq = ld8(in), ldb = ld8(out), lds = ld8s(in), ldbs = ld8s(out);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int r = r0 + k * STEP;
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const uint32_t p = pack8(v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3], inv);
      *(uint32_t*)&tile[r][c + e] = p;
      if (q_back && i0 + r < in) *(uint32_t*)(q_back + (int64_t)(i0 + r) * ldb + n0 + c + e) = p;
    }
  }
  __syncthreads();
  // eight neighbouring threads write a row of the other copy, 16 bytes each
  const int part = threadIdx.x % 8 * 16;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = threadIdx.x / 8 + k * 32;
    uint32_t p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      p[j] = tile[part + 4 * j][r] | (uint32_t)tile[part + 4 * j + 1][r] << 8 | (uint32_t)tile[part + 4 * j + 2][r] << 16 | (uint32_t)tile[part + 4 * j + 3][r] << 24;
    if (n0 + r < out) *(uint4*)(q + (int64_t)(n0 + r) * ldq + i0 + part) = make_uint4(p[0], p[1], p[2], p[3]);
  }
  if (threadIdx.x == 0) {
    const int bi = blockIdx.y, bn = blockIdx.x;
    scale[bn * lds + bi] = (uint8_t)s8;
    if (bi == (int)gridDim.y - 1)
      for (int64_t p = bi + 1; p < lds; ++p) scale[bn * lds + p] = 127;
    if (q_back) {
      scale_back[bi * ldbs + bn] = (uint8_t)s8;
      if (bn == (int)gridDim.x - 1)
        for (int64_t p = bn + 1; p < ldbs; ++p) scale_back[bi * ldbs + p] = 127;
    }
  }
}

template <typename T>
void rows_t(const void* x, int64_t M, int K, int64_t ldx, void* q, uint8_t* scale, hipStream_t s) {
  const int per_row = (int)ld8s(K), real = (int)(ld8(K) / BLOCK8);
  const int64_t step = std::max<int64_t>(1, (int64_t(1) << 28) / per_row);          // (a launch has fewer than 2^32 threads, and a block eight)
  for (int64_t m = 0; m < M; m += step) {
    const int64_t blocks = std::min(step, M - m) * per_row;
    quantize8_rows_kernel<T><<<(unsigned)((blocks * 8 + 255) / 256), 256, 0, s>>>((const T*)x + m * ldx, blocks, K, ldx, per_row, real,
                                                                                (uint8_t*)q + m * ld8(K), scale + m * per_row);
  }
}

}  // namespace

void quantize8_rows(const void* x, bool f32, int64_t M, int K, int64_t ldx, void* q, uint8_t* scale, hipStream_t s) {
  if (M <= 0) return;
  if (f32) rows_t<float>(x, M, K, ldx, q, scale, s);
  else rows_t<bf16>(x, M, K, ldx, q, scale, s);
}

void quantize8_weight(const void* w, bool f32, int in, int out, int64_t ldw, void* q, uint8_t* scale, void* q_back, uint8_t* scale_back,
                      hipStream_t s) {
  const dim3 grid((out + BLOCK8 - 1) / BLOCK8, (in + BLOCK8 - 1) / BLOCK8);
  auto go = [&](auto kern, auto* p) { kern<<<grid, 256, 0, s>>>(p, in, out, ldw, (uint8_t*)q, scale, (uint8_t*)q_back, scale_back); };
  if (f32) go(quantize8_weight_kernel<float>, (const float*)w);
  else go(quantize8_weight_kernel<bf16>, (const bf16*)w);
}

}  // namespace bsr
