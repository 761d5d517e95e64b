// Softmax cross-entropy of a linear layer and its gradients where there is little to do, or few rows: a few launches instead of tiles that fill the chip.  (The other sizes: k_linear_ce.hip.)
// The logits, or G, are left in scratch in fp32, 16 MB at most; the products take their fragments straight from the caller's tensors, whatever their type, stride and alignment.
//   logits   16 classes x 16 or 32 tokens a workgroup, the features split over its eight wavefronts, whole cache lines each (bf16 16 x 16 x 32, fp32 16 x 16 x 4 matrix instructions, both exact products
//            added in fp32); for the gradients they leave as G
//   rows     a workgroup a token: maximum, sum, loss
//   grads    up to 32 tokens: dx and dw in one pass over w, multiplied in fp32 (16 x 16 x 4)
// A launch is a chain of a few trips to memory; that, the calls and, for few rows of many classes, the bytes of w and dw are what bounds it.
#include <algorithm>

#include "linear_ce.h"
#include "rowops.h"

namespace bsr {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
constexpr float LOG2E = 1.4426950408889634f;

int over(int64_t n, int by) { return (int)((n + by - 1) / by); }

// V values of a row from k on, zero past its end
template <typename T> __device__ __forceinline__ typename Chunk<T>::vec piece(const T* row, int k, int D) {
  constexpr int V = Chunk<T>::V;
  if (k + V <= D) return *(const typename Loose<T>::vec*)(row + k);
  typename Chunk<T>::vec v;
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = k + e < D ? row[k + e] : (T)0.f;
  return v;
}
__device__ __forceinline__ f32x4 multiplied(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// (element e of the four lanes that hold a row's 16 values: any order of k will do that both operands have)
__device__ __forceinline__ f32x4 multiplied(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// what a token's logits become G by; counts: whether it has a gradient at all
struct Tokens {
  const int32_t* labels = nullptr; const float2* stats = nullptr; const float* row_grad = nullptr; float scale = 1.f;      // stats null: the logits stay what they are
  bool weighted = true;                            // G with its row's weight
  int N = 0, V = 0;
  __device__ __forceinline__ bool counts(int n) const {
    const int m = min(n, N - 1), label = labels[m];
    const float2 st = stats[m];
    return n < N && label >= 0 && label < V && (!row_grad || row_grad[m] != 0.f) && !(st.x == -INFINITY && st.y == 0.f);
  }
};

// z or G [N, ldz]: lane l has V features of class l % 16 and of token l % 16
constexpr int LOGIT_WAVES = 8;
template <typename T, int TILES>
__global__ __launch_bounds__(LOGIT_WAVES * WAVE) void small_logits_kernel(const T* __restrict__ x, int64_t ldx, const T* __restrict__ w, int64_t ldw, int D, const float* __restrict__ bias, Tokens tk,
                                                           float* __restrict__ z, int64_t ldz) {
  constexpr int C = Chunk<T>::V, STEP = 4 * C, AT_ONCE = 4;
  typedef typename Chunk<T>::vec vec;
  __shared__ f32x4 red[LOGIT_WAVES - 1][TILES][WAVE];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, v0 = blockIdx.x * 16, n0 = blockIdx.y * 16 * TILES, part = lane / 16 * C, N = tk.N, V = tk.V;
  const T* wr = w + (int64_t)min(v0 + lane % 16, V - 1) * ldw;
  const T* xr[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) xr[t] = x + (int64_t)min(n0 + t * 16 + lane % 16, N - 1) * ldx;
  f32x4 acc[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = wave * STEP * AT_ONCE; k < D; k += LOGIT_WAVES * STEP * AT_ONCE) {
    vec a[AT_ONCE], b[AT_ONCE][TILES];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int at = k + i * STEP + part;
      a[i] = piece(wr, at, D);
#pragma unroll
      for (int t = 0; t < TILES; ++t) b[i][t] = piece(xr[t], at, D);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
      for (int t = 0; t < TILES; ++t) acc[t] = multiplied(a[i], b[i][t], acc[t]);
  }
  if (wave > 0)
#pragma unroll
    for (int t = 0; t < TILES; ++t) red[wave - 1][t][lane] = acc[t];
  __syncthreads();
  if (wave > 0) return;
  const int v = v0 + lane / 16 * 4;
  f32x4 b;
#pragma unroll
  for (int j = 0; j < 4; ++j) b[j] = bias && v + j < V ? bias[v + j] : 0.f;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int n = n0 + t * 16 + lane % 16;
    if (n >= N || v >= V) continue;
    f32x4 o = acc[t];
#pragma unroll
    for (int i = 0; i < LOGIT_WAVES - 1; ++i) o += red[i][t][lane];
    o += b;
    if (tk.stats) {
      const bool counts = tk.counts(n);
      const float2 st = tk.stats[n];
      const float by = tk.scale * (tk.weighted && tk.row_grad ? tk.row_grad[n] : 1.f);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        o[j] = counts ? by * (__builtin_amdgcn_exp2f(fmaf(o[j] - st.x, LOG2E, -st.y * LOG2E)) - (v + j == tk.labels[n] ? 1.f : 0.f)) : 0.f;
    }
    *(f32x4*)(z + n * ldz + v) = o;                          // (ldz: whole fours)
  }
}

// a workgroup a token.  grad: the logits become G
__global__ __launch_bounds__(256) void small_rows_kernel(float* __restrict__ z, int64_t ldz, Tokens tk, float* __restrict__ loss, float2* __restrict__ stats, bool grad) {
  __shared__ float red[2][4];
  const int m = blockIdx.x, wave = threadIdx.x / WAVE, V = tk.V;
  float* row = z + m * ldz;
  float most = -INFINITY;
#pragma unroll 4
  for (int v = threadIdx.x; v < V; v += 256) most = fmaxf(most, row[v]);
  most = wave_max(most);
  if (threadIdx.x % WAVE == 0) red[0][wave] = most;
  __syncthreads();
  most = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  // (fmaxf passes NaN over, the sum does not; a row of -inf alone has sum 0)
  const float ref = most == -INFINITY ? 0.f : most;
  float s = 0.f;
#pragma unroll 4
  for (int v = threadIdx.x; v < V; v += 256) s += __builtin_amdgcn_exp2f((row[v] - ref) * LOG2E);
  s = wave_sum(s);
  if (threadIdx.x % WAVE == 0) red[1][wave] = s;
  __syncthreads();
  s = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const float ls = s == 0.f ? 0.f : logf(s);
  const int label = tk.labels[m];
  const bool there = label >= 0 && label < V && !(most == -INFINITY && s == 0.f);
  const float mine = there && threadIdx.x == 0 ? row[label] : 0.f;       // (before it becomes G)
  if (threadIdx.x == 0) {
    if (stats) stats[m] = make_float2(most, ls);
    if (loss) loss[m] = there ? (most - mine) + ls : 0.f;
  }
  if (!grad) return;
  __syncthreads();
  const float weight = tk.row_grad ? tk.row_grad[m] : 1.f, by = tk.weighted ? tk.scale * weight : 1.f;
#pragma unroll 4
  for (int v = threadIdx.x; v < V; v += 256) row[v] = there && weight != 0.f ? by * (__builtin_amdgcn_exp2f(fmaf(row[v] - most, LOG2E, -ls * LOG2E)) - (v == label ? 1.f : 0.f)) : 0.f;
}

// K values of a row from d on, zero past its end
template <int K, typename T> struct Some { typedef T vec __attribute__((ext_vector_type(K), aligned(sizeof(T)))); };
template <int K, typename T> __device__ __forceinline__ typename Some<K, T>::vec some(const T* row, int d, int D) {
  if (d + K <= D) return *(const typename Some<K, T>::vec*)(row + d);
  typename Some<K, T>::vec v;
#pragma unroll
  for (int e = 0; e < K; ++e) v[e] = d + e < D ? row[d + e] : (T)0.f;
  return v;
}
template <int K, typename T> __device__ __forceinline__ void put(T* row, int d, int D, typename Some<K, T>::vec v) {
  if (d + K <= D) *(typename Some<K, T>::vec*)(row + d) = v;
  else
#pragma unroll
    for (int e = 0; e < K; ++e)
      if (d + e < D) row[d + e] = v[e];
}

// features of a lane: 16 bytes; with two tiles of tokens 8, or they would not leave registers for a second wavefront a SIMD
template <typename T> constexpr int few_features(int tiles) { return tiles == 2 ? 4 : Chunk<T>::V; }

// dx = G w, dw = G^T x and db of up to 16 TILES tokens and any number of classes, w read and dw written once.  A workgroup takes 16 K features and a range of the classes, a wavefront every
// fourth 16 of these, in products of 16 x 16 whose column l % 16 of product i is feature K (l % 16) + i: a lane reads and writes K features together.  x's part stays in
// registers; dx's is added up over the range and leaves as a part.
template <typename T, typename TW, int TILES>
__global__ __launch_bounds__(256) void few_grads_kernel(const float* __restrict__ G, int64_t ldz, Tokens tk, int D, const T* __restrict__ x, int64_t ldx, const T* __restrict__ w, int64_t ldw,
                                                        float* __restrict__ parts, int64_t ldp, int per, TW* __restrict__ dw, int64_t lddw, float* __restrict__ db) {
  constexpr int K = few_features<T>(TILES);
  typedef typename Some<K, T>::vec vec;
  __shared__ f32x4 red[3][K][WAVE];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, lm = lane % 16, lq = lane / 16, d = (blockIdx.x * 16 + lm) * K, N = tk.N, V = tk.V;
  const int begin = blockIdx.y * per, end = min(begin + per, V);
  float xb[TILES][4][K];
  f32x4 acc[TILES][K];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = t * 16 + 4 * lq + j;
      const bool counts = tk.counts(n);                            // (a row that does not count may hold anything)
      const vec v = some<K>(x + (int64_t)min(n, N - 1) * ldx, d, D);
#pragma unroll
      for (int i = 0; i < K; ++i) xb[t][j][i] = counts ? (float)v[i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < K; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // G by rows (four classes of token l % 16) and by columns (four tokens of class l % 16)
  const float* gr[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) gr[t] = G + (int64_t)min(t * 16 + lm, N - 1) * ldz;
  vec nb[4];
  f32x4 nr[TILES];
  float nc[TILES][4];
  auto fetch = [&](int v0) __attribute__((always_inline)) {        // (a step ahead)
    const int v = v0 + 4 * lq, vc = min(v0 + lm, V - 1);
    if (parts) {
#pragma unroll
      for (int j = 0; j < 4; ++j) nb[j] = some<K>(w + (int64_t)min(v + j, V - 1) * ldw, d, D);
#pragma unroll
      for (int t = 0; t < TILES; ++t) nr[t] = v < V ? *(const f32x4*)(gr[t] + v) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) nc[t][j] = G[(int64_t)min(t * 16 + 4 * lq + j, N - 1) * ldz + vc];
  };
  if (begin + wave * 16 < end) fetch(begin + wave * 16);
  for (int v0 = begin + wave * 16; v0 < end; v0 += 64) {
    const int v = v0 + 4 * lq;
    vec b[4];
    f32x4 row[TILES];
    float col[TILES][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = nb[j];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      row[t] = nr[t];
#pragma unroll
      for (int j = 0; j < 4; ++j) col[t][j] = t * 16 + 4 * lq + j < N ? nc[t][j] : 0.f;
    }
    if (v0 + 64 < end) fetch(v0 + 64);
    if (parts)
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float g = v + j < end ? row[t][j] : 0.f;           // (what lies behind the last class is not written)
#pragma unroll
          for (int i = 0; i < K; ++i) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(g, (float)b[j][i], acc[t][i], 0, 0, 0);
        }
    if (dw) {
      f32x4 out[K];
#pragma unroll
      for (int i = 0; i < K; ++i) out[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < K; ++i) out[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(col[t][j], xb[t][j][i], out[i], 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (v + r < end) {
          typename Some<K, TW>::vec o;
#pragma unroll
          for (int i = 0; i < K; ++i) o[i] = (TW)out[i][r];
          put<K>(dw + (int64_t)(v + r) * lddw, d, D, o);
        }
    }
    if (db && blockIdx.x == 0) {
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += col[t][j];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (lq == 0 && v0 + lm < end) db[v0 + lm] = sum;
    }
  }
  if (!parts) return;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    if (t) __syncthreads();
    if (wave > 0)
#pragma unroll
      for (int i = 0; i < K; ++i) red[wave - 1][i][lane] = acc[t][i];
    __syncthreads();
    if (wave == 0)
#pragma unroll
      for (int i = 0; i < K; ++i) acc[t][i] = ((acc[t][i] + red[0][i][lane]) + red[1][i][lane]) + red[2][i][lane];
    if (wave == 0)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = t * 16 + 4 * lq + r;
        if (n < N)
#pragma unroll
          for (int i = 0; i < K; i += 4)
            if (d + i < D) *(f32x4*)(parts + ((int64_t)blockIdx.y * N + n) * ldp + d + i) = f32x4{acc[t][i][r], acc[t][i + 1][r], acc[t][i + 2][r], acc[t][i + 3][r]};
      }
  }
}
// dx from its parts, in order
template <typename T> __global__ __launch_bounds__(256) void few_sums_kernel(const float* __restrict__ parts, int count, int64_t ldp, Tokens tk, int D, T* __restrict__ dx, int64_t lddx) {
  const int d = (blockIdx.x * 64 + threadIdx.x % 64) * 4, n = blockIdx.y;
  __shared__ f32x4 red[3][64];
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (d < D)
#pragma unroll 8
    for (int p = threadIdx.x / 64; p < count; p += 4) v += *(const f32x4*)(parts + ((int64_t)p * tk.N + n) * ldp + d);
  if (threadIdx.x >= 64) red[threadIdx.x / 64 - 1][threadIdx.x % 64] = v;
  __syncthreads();
  if (threadIdx.x >= 64 || d >= D) return;
  v = ((v + red[0][threadIdx.x]) + red[1][threadIdx.x]) + red[2][threadIdx.x];
  if (!tk.counts(n)) v = f32x4{0.f, 0.f, 0.f, 0.f};                // (whatever w holds)
  put<4>(dx + n * lddx, d, D, typename Some<4, T>::vec{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
}

int64_t small_ldz(const LinearCe& a) { return ((int64_t)a.V + 3) / 4 * 4; }
template <typename T> void logits_as(const LinearCe& a, const Tokens& tk, float* z, hipStream_t s) {
  if (a.N <= 16) small_logits_kernel<T, 1><<<dim3(over(a.V, 16), 1), LOGIT_WAVES * WAVE, 0, s>>>((const T*)a.x, a.ldx, (const T*)a.w, a.ldw, a.D, a.bias, tk, z, small_ldz(a));
  else small_logits_kernel<T, 2><<<dim3(over(a.V, 16), over(a.N, 32)), LOGIT_WAVES * WAVE, 0, s>>>((const T*)a.x, a.ldx, (const T*)a.w, a.ldw, a.D, a.bias, tk, z, small_ldz(a));
}
// workgroups over the classes
int few_wide(bool f32, int N) { return 16 * (N > 16 ? few_features<float>(2) : f32 ? few_features<float>(1) : few_features<bf16>(1)); }
int few_ranges(bool f32, int N, int V, int D) { return std::min(over(V, 64), std::max(1, 1024 / over(D, few_wide(f32, N)))); }

template <typename T, typename TW> void grads_as(const LinearCe& a, const Tokens& tk, const float* G, float* parts, hipStream_t s) {
  const int wide = few_wide(a.f32, a.N);
  const int64_t ldp = ((int64_t)a.D + 3) / 4 * 4;
  const int per = over(over(a.V, few_ranges(a.f32, a.N, a.V, a.D)), 64) * 64, ranges = over(a.V, per);
  if (!a.dx) parts = nullptr;
  const dim3 grid(a.dx || a.dw ? over(a.D, wide) : 1, ranges);
  if (a.N <= 16) few_grads_kernel<T, TW, 1><<<grid, 256, 0, s>>>(G, small_ldz(a), tk, a.D, (const T*)a.x, a.ldx, (const T*)a.w, a.ldw, parts, ldp, per, (TW*)a.dw, a.lddw, a.db);
  else few_grads_kernel<T, TW, 2><<<grid, 256, 0, s>>>(G, small_ldz(a), tk, a.D, (const T*)a.x, a.ldx, (const T*)a.w, a.ldw, parts, ldp, per, (TW*)a.dw, a.lddw, a.db);
  if (a.dx) few_sums_kernel<T><<<dim3(over(a.D, 256), a.N), 256, 0, s>>>(parts, ranges, ldp, tk, a.D, (T*)a.dx, a.lddx);
}

}  // namespace

static Tokens tokens_of(const LinearCe& a, bool weighted) {
  Tokens tk;
  tk.N = a.N; tk.V = a.V; tk.labels = a.labels; tk.row_grad = a.row_grad; tk.weighted = weighted; tk.scale = weighted ? a.grad_scale : 1.f;
  return tk;
}
static void logits_of(const LinearCe& a, const Tokens& tk, float* z, hipStream_t s) {
  if (a.f32) logits_as<float>(a, tk, z, s);
  else logits_as<bf16>(a, tk, z, s);
}

void small_ce_forward(const LinearCe& a, float* z, SmallGrad grad, hipStream_t s) {
  const Tokens tk = tokens_of(a, grad == GRAD_WEIGHTED);
  logits_of(a, tk, z, s);
  small_rows_kernel<<<a.N, 256, 0, s>>>(z, small_ldz(a), tk, a.loss, (float2*)a.stats, grad != GRAD_NONE);
}

void small_ce_gradient(const LinearCe& a, bool weighted, float* G, hipStream_t s) {
  Tokens tk = tokens_of(a, weighted);
  tk.stats = (const float2*)a.stats;
  logits_of(a, tk, G, s);
}

static size_t few_parts_at(int N, int V) { return (small_ce_bytes(N, V) + 255) / 256 * 256; }
size_t few_ce_bytes(bool f32, int N, int V, int D) { return few_parts_at(N, V) + sizeof(float) * (size_t)few_ranges(f32, N, V, D) * N * (((size_t)D + 3) / 4 * 4); }
void few_ce_backward(const LinearCe& a, bool ready, hipStream_t s) {
  float *G = (float*)a.workspace, *parts = (float*)((char*)a.workspace + few_parts_at(a.N, a.V));
  if (!ready) small_ce_gradient(a, true, G, s);
  Tokens tk = tokens_of(a, true);
  tk.stats = (const float2*)a.stats;
  if (a.f32) grads_as<float, float>(a, tk, G, parts, s);
  else if (a.dw_f32) grads_as<bf16, float>(a, tk, G, parts, s);
  else grads_as<bf16, bf16>(a, tk, G, parts, s);
}

}  // namespace bsr
