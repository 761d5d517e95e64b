// What the kernels of rows of any length and stride share (k_norm_rows.hip, k_rms_rows.hip): chunks of 16 bytes at any address, sums over a row's
// threads, a chunk in 8 bits.
#pragma once
#include "fp8.h"

namespace bsr {

constexpr int64_t ROWS_A_LAUNCH = 1 << 21;                 // (a launch has fewer than 2^32 threads, and a row up to 1024)

// Results go past the caches, a wavefront's store being whole lines (16384 x 8192: forward 130 -> 94 us, backward 174 -> 170; 25216 x 768 backward 32 -> 26)
// A row lies in chunks of 16 bytes.  WHOLE: it is whole chunks on 16-byte boundaries; otherwise chunks lie at any element's address, and what is left
// behind the whole ones is the end of a chunk that ends with the row: its thread holds `skip` values of the chunk before it as well, which do
// not count.  So every load is one vector without a branch (value by value, a row of 5001 bf16 took 2.5 times as long).
template <int V> __device__ __forceinline__ int chunk_at(int c, int D) { return min(c * V, D - V); }
template <bool WHOLE, typename T> __device__ __forceinline__ typename Chunk<T>::vec get_chunk(const T* row, int c, int D) {
  const T* p = row + chunk_at<Chunk<T>::V>(c, D);
  if constexpr (WHOLE) return *(const typename Chunk<T>::vec*)p;
  else return *(const typename Loose<T>::vec*)p;
}
// (whole: chunk c is one; else its last V - skip values count)
template <bool WHOLE, typename T> __device__ __forceinline__ void put_chunk(T* row, int c, int D, bool whole, int skip, typename Chunk<T>::vec v) {
  constexpr int V = Chunk<T>::V;
  if (WHOLE) __builtin_nontemporal_store(v, (typename Chunk<T>::vec*)(row + c * V));
  else if (whole) *(typename Loose<T>::vec*)(row + c * V) = v;
  else
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e >= skip) row[D - V + e] = v[e];
}
template <bool WHOLE, int V> __device__ __forceinline__ void get_params(const float* p, int c, int D, float (&o)[V]) {
  p += chunk_at<V>(c, D);
  if constexpr (WHOLE) load_params<V>(p, o);
  else
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const Loose<float>::vec t = *(const Loose<float>::vec*)(p + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[4 * q + e] = t[e];
    }
}

// sums of a and b over the threads of a row: a wavefront, or all of a workgroup (red: two floats a wavefront; a second buffer in turn, so that
// one barrier a row is enough)
template <int TPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float (*red)[2]) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (TPR > WAVE) {
    const int w = threadIdx.x / WAVE;
    if (threadIdx.x % WAVE == 0) { red[w][0] = a; red[w][1] = b; }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / WAVE; ++i) { a += red[i][0]; b += red[i][1]; }
  }
}

// maximum over each 16 or 32 lanes, of values that are not negative (on the vector unit, as wave_all in rowops.h)
template <int N> __device__ __forceinline__ float lanes_max(float v) {
  static_assert(N == 16 || N == 32, "");
  if constexpr (N == 32) {
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
  }
  v = fmaxf(v, dpp_move<0x128>(v));
  v = fmaxf(v, dpp_move<0x124>(v));
  v = fmaxf(v, dpp_move<0x4E>(v));
  return fmaxf(v, dpp_move<0xB1>(v));
}

template <int TPR> constexpr int block_threads() { return TPR > 256 ? TPR : 256; }

// A row's chunk c (the i-th of its thread) in 8 bits: BLOCK8 / V neighbouring lanes hold a block.  o: zero where nothing counts.
// (8-bit rows stay in the caches for the product behind: LayerNorm of 16384 x 8192 takes 108 us past them against 127, but 25216 x 768 with its product, cut sums, 47 against 44)
template <bool WHOLE, int TPR, int V>
__device__ __forceinline__ void put_chunk8(const float (&o)[V], int i, int c, int nch, int all, int skip, int64_t ldq, uint8_t* q, uint8_t* scale) {
  if (i * TPR * V >= ldq) return;
  // (fmaxf passes NaN over; a block with an infinity goes through its values again)
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) most = fmaxf(most, fabsf(o[e]));
  most = lanes_max<BLOCK8 / V>(most);
  if (most == INFINITY) {
    most = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) most = fmaxf(most, __uint_as_float(finite_bits(o[e])));
    most = lanes_max<BLOCK8 / V>(most);
  }
  const uint32_t s8 = scale8_of(__float_as_uint(most));
  const float inv = inverse_of(s8);
  if (c * V < ldq) {
    uint32_t* to = (uint32_t*)(q + c * V);
    const int down = !WHOLE && c == nch && c < all ? 8 * skip : 0;          // (what does not count goes, zeros come behind)
    if constexpr (V == 8) {
      const uint64_t eight = (pack8(o[0], o[1], o[2], o[3], inv) | (uint64_t)pack8(o[4], o[5], o[6], o[7], inv) << 32) >> down;
      *(uint2*)to = make_uint2((uint32_t)eight, (uint32_t)(eight >> 32));
    } else {
      *to = pack8(o[0], o[1], o[2], o[3], inv) >> down;
    }
    if (c * V % BLOCK8 == 0) scale[c * V / BLOCK8] = (uint8_t)s8;
  }
}

// f(threads per row, chunks per thread) for a row of n chunks; false: too long.  Two chunks a thread leave registers for
// four wavefronts a SIMD in the backward pass.
template <class F> bool with_row_chunks_of(int n, F&& f) {
  if (n <= 64) f(RowC<64>{}, RowC<1>{});
  else if (n <= 128) f(RowC<64>{}, RowC<2>{});
  else if (n <= 256) f(RowC<256>{}, RowC<1>{});
  else if (n <= 512) f(RowC<256>{}, RowC<2>{});
  else if (n <= 1024) f(RowC<512>{}, RowC<2>{});
  else if (n <= 2048) f(RowC<1024>{}, RowC<2>{});
  else return false;
  return true;
}

template <typename T> bool in_chunks(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0; }

}  // namespace bsr
