// The norm of many tensors taken together, sqrt(sum over tensors, sum over values of g^2), and out = g min(1, max_norm / norm).
// Bound by memory: every value is read twice and written once.  Pass one: at most 2048 workgroups a launch walk the pieces of all tensors and leave a sum of squares each; pass
// two: every workgroup adds these up for itself, in the same order, while its first piece is on its way (a launch between the passes would cost as much as a few MB), and walks the pieces
// backwards, the last read first, for what the caches still hold.  Results that lie where the gradients do are left alone when nothing is to be scaled.
// Squares and sums are fp64: squares of fp32 gradients leave fp32's range, and sums of 10^9 of them its precision; the vector unit does them at several times the rate
// at which values arrive.  No atomics, fixed orders.
// Measured: 28.4 million fp32 values in 54 tensors 19 and 37 us while the caches hold them (341 MB read, read and written), 74 from memory; 2^29 values in 400 tensors, bf16 and fp32, 1050 us (5.1 TB/s),
// the two passes 303 + 11 (few small tensors) and 631 + 11 a launch.
#include <algorithm>

#include "clip.h"
#include "rowops.h"

namespace bsr {

namespace {

constexpr int NT = 256, WAVES = NT / WAVE;

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = WAVE / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}
// over the workgroup, in every thread; wavefronts in order
__device__ __forceinline__ double block_sum64(double v, double* red) {
  v = wave_sum64(v);
  if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) v += red[i];
  return v;
}

// the tensor that piece p belongs to
__device__ __forceinline__ int tensor_of(const ClipTable& t, int p) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.start[mid] <= p) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// f(values, how many of them, their place) for a thread's shares of a piece of n values: chunks of 16 bytes at any address, then single values
template <typename T, class F> __device__ __forceinline__ void for_piece(const T* g, int n, F&& f) {
  constexpr int V = Chunk<T>::V, AT_ONCE = 4;
  const int whole = n / V;
  for (int c = threadIdx.x; c < whole; c += AT_ONCE * NT) {
    typename Loose<T>::vec v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) v[i] = *(const typename Loose<T>::vec*)(g + min(c + i * NT, whole - 1) * V);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      if (c + i * NT < whole) f(v[i], (c + i * NT) * V);
  }
  for (int j = whole * V + threadIdx.x; j < n; j += NT) f(g[j], j);
}

__global__ __launch_bounds__(NT) void clip_norm_kernel(ClipTable t, double* __restrict__ parts) {
  __shared__ double red[WAVES];
  double s = 0.0;
  auto add = [&](auto v, int) __attribute__((always_inline)) {
    if constexpr (sizeof(v) < 16) {
      const double d = (double)(float)v;
      s = fma(d, d, s);
    } else
#pragma unroll
      for (int e = 0; e < (int)(16 / sizeof(v[0])); ++e) {
        const double d = (double)(float)v[e];
        s = fma(d, d, s);
      }
  };
  for (int p = blockIdx.x; p < t.pieces; p += gridDim.x) {
    const int i = tensor_of(t, p);
    const int64_t at = (int64_t)(p - t.start[i]) * CLIP_PIECE, n = t.n[i];
    if (n < 0) for_piece((const bf16*)t.g[i] + at, (int)min(-n - at, (int64_t)CLIP_PIECE), add);
    else for_piece((const float*)t.g[i] + at, (int)min(n - at, (int64_t)CLIP_PIECE), add);
  }
  s = block_sum64(s, red);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// adds the parts up: the norm, in every thread
__device__ __forceinline__ double norm_of(const double* __restrict__ parts, int n, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += NT) s += parts[i];
  return sqrt(block_sum64(s, red));
}

__global__ __launch_bounds__(NT) void clip_scale_kernel(ClipTable t, const double* __restrict__ parts, int nparts, float max_norm, float* norm) {
  __shared__ double red[WAVES];
  const double length = norm_of(parts, nparts, red);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)length;
  // (a norm that is no number, or infinite where it is told, scales nothing; fp64: the factor may lie below fp32's normal numbers)
  const double by = length > (double)max_norm && (float)length < INFINITY ? (double)max_norm / length : 1.0;
  for (int k = blockIdx.x; k < t.pieces; k += gridDim.x) {
    const int p = t.pieces - 1 - k, i = tensor_of(t, p);
    if (by == 1.0 && t.out[i] == t.g[i]) continue;
    const int64_t at = (int64_t)(p - t.start[i]) * CLIP_PIECE, n = t.n[i];
    auto put = [&](auto* out) __attribute__((always_inline)) {
      return [=](auto v, int j) __attribute__((always_inline)) {
        typedef decltype(v) V;
        if constexpr (sizeof(V) < 16) out[j] = (V)(float)((double)(float)v * by);
        else {
#pragma unroll
          for (int e = 0; e < (int)(16 / sizeof(v[0])); ++e) v[e] = (float)((double)(float)v[e] * by);
          *(typename Loose<std::remove_reference_t<decltype(*out)>>::vec*)(out + j) = v;
        }
      };
    };
    if (n < 0) for_piece((const bf16*)t.g[i] + at, (int)min(-n - at, (int64_t)CLIP_PIECE), put((bf16*)t.out[i] + at));
    else for_piece((const float*)t.g[i] + at, (int)min(n - at, (int64_t)CLIP_PIECE), put((float*)t.out[i] + at));
  }
}

__global__ __launch_bounds__(NT) void clip_norm_only_kernel(const double* __restrict__ parts, int nparts, float* norm) {
  __shared__ double red[WAVES];
  const double length = norm_of(parts, nparts, red);
  if (threadIdx.x == 0) *norm = (float)length;
}

// tensors [from, from + CLIP_TENSORS) as a table
int fill(ClipTable& t, const ClipArgs& a, int from) {
  t.count = std::min(CLIP_TENSORS, a.count - from);
  t.pieces = 0;
  for (int i = 0; i < t.count; ++i) {
    t.g[i] = a.g[from + i];
    t.out[i] = a.out ? a.out[from + i] : nullptr;
    t.n[i] = a.f32[from + i] ? a.n[from + i] : -a.n[from + i];
    t.start[i] = t.pieces;
    t.pieces += (int)((a.n[from + i] + CLIP_PIECE - 1) / CLIP_PIECE);
  }
  return t.pieces;
}

}  // namespace

void clip(const ClipArgs& a, hipStream_t s) {
  const int launches = clip_launches(a.count), share = clip_share(a.count);
  ClipTable t;
  int parts = 0;
  for (int l = 0; l < launches; ++l) {
    const int blocks = std::min(fill(t, a, l * CLIP_TENSORS), share);
    if (blocks > 0) clip_norm_kernel<<<blocks, NT, 0, s>>>(t, a.parts + parts);
    parts += blocks;
  }
  if (!a.out || parts == 0) {
    if (a.norm) clip_norm_only_kernel<<<1, NT, 0, s>>>(a.parts, parts, a.norm);
    return;
  }
  bool told = false;
  for (int l = launches - 1; l >= 0; --l) {
    if (launches > 1 && fill(t, a, l * CLIP_TENSORS) == 0) continue;
    clip_scale_kernel<<<std::min(t.pieces, 2048), NT, 0, s>>>(t, a.parts, parts, a.max_norm, told ? nullptr : a.norm);
    told = true;
  }
}

}  // namespace bsr
