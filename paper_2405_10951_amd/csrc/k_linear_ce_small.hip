// Softmax cross-entropy of a linear layer and its gradients where there is little to do, or few rows: a few launches instead of tiles that fill the chip.  (The other sizes: k_linear_ce.hip.)
// The logits, or G, are left in scratch in fp32, 16 MB at most; the products take their fragments straight from the caller's tensors, whatever their type, stride and alignment.
//   logits   16 classes x 16 or 32 tokens a workgroup, the features split over its eight wavefronts, whole cache lines each (bf16 16 x 16 x 32, fp32 16 x 16 x 4 matrix instructions, both exact products
//            added in fp32); for the gradients they leave as G
//   rows     a workgroup a token: maximum, sum, loss
//   grads    up to 64 tokens: dx and dw in one pass over w, multiplied in fp32 (16 x 16 x 4), or beside bf16 with G in two bf16 terms (16 x 16 x 32) and, for dw in fp32, a third (16 x 16 x 16)
// A launch is a chain of a few trips to memory; that, the calls and, for few rows of many classes, the bytes of w and dw are what bounds it.
// Measured: 32 x 768 x 100 fp32 8 + 11 us; loss and gradients of 48 x 2048 x 100000 fp32 987 to 1062 (by tiles 2360), of 1 x 100 x 100000 bf16 50 to 54; gradients of 32 x 4096 x 100000 bf16 348 (1.6 GB of w and dw: 4.7 TB/s; with fp32 products 728), of 64 rows 580 (two wavefronts a SIMD, of which each waits for a
// half as long rows' piece; G by columns from memory instead of LDS: 673; 8 features a lane and one wavefront: 660; four wavefronts side by side on G: 690).
// The third term of G for dw in fp32: loss and gradients of 64 x 4096 x 100000 949 us, of two terms 930; 32 x 4096 x 100000 749 with either; 33 x 2048 x 8000, gradients, 64 and 62.
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
  int N = 0, V = 0;
  float* loss = nullptr; float2* stats_out = nullptr;            // where a kernel that makes them leaves them
  int rows = 0;                                    // of G; those from N on, and classes from V on, are zero
  __device__ __forceinline__ bool counts(int n) const {
    const int m = min(n, N - 1), label = labels[m];
    const float2 st = stats[m];
    return n < N && label >= 0 && label < V && (!row_grad || row_grad[m] != 0.f) && !(st.x == -INFINITY && st.y == 0.f);
  }
};

// z or G [N, ldz]: lane l has V features of CT classes l % 16 and of TILES tokens l % 16.  KW of the eight wavefronts share the features of 16 CT classes.  (Every workgroup reads x from the caches: with many
// tokens for several classes at a time, or that would take longer than w's bytes: forward of 48 x 2048 x 100000 fp32 465 us with two times 16 classes and four times 16 tokens, 582 with one times 16
// classes, 32 x 2048 x 100000 328 and 387)
constexpr int LOGIT_WAVES = 8;
template <typename T, int TILES, int KW, int CT>
__global__ __launch_bounds__(LOGIT_WAVES * WAVE) void small_logits_kernel(const T* __restrict__ x, int64_t ldx, const T* __restrict__ w, int64_t ldw, int D, const float* __restrict__ bias, Tokens tk,
                                                           float* __restrict__ z, int64_t ldz) {
  constexpr int C = Chunk<T>::V, STEP = 4 * C, AT_ONCE = TILES * CT > 4 ? 2 : 4;
  typedef typename Chunk<T>::vec vec;
  __shared__ f32x4 red[KW > 1 ? KW - 1 : 1][CT][TILES][WAVE];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE % KW, v0 = (blockIdx.x * (LOGIT_WAVES / KW) + threadIdx.x / WAVE / KW) * 16 * CT, n0 = blockIdx.y * 16 * TILES,
            part = lane / 16 * C, N = tk.N, V = tk.V;
  const T *wr[CT], *xr[TILES];
#pragma unroll
  for (int c = 0; c < CT; ++c) wr[c] = w + (int64_t)min(v0 + c * 16 + lane % 16, V - 1) * ldw;
#pragma unroll
  for (int t = 0; t < TILES; ++t) xr[t] = x + (int64_t)min(n0 + t * 16 + lane % 16, N - 1) * ldx;
  f32x4 acc[CT][TILES];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = wave * STEP * AT_ONCE; k < D; k += KW * STEP * AT_ONCE) {
    vec a[AT_ONCE][CT], b[AT_ONCE][TILES];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int at = k + i * STEP + part;
#pragma unroll
      for (int c = 0; c < CT; ++c) a[i][c] = piece(wr[c], at, D);
#pragma unroll
      for (int t = 0; t < TILES; ++t) b[i][t] = piece(xr[t], at, D);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[c][t] = multiplied(a[i][c], b[i][t], acc[c][t]);
  }
  static_assert(KW == 1 || KW == LOGIT_WAVES, "");
  if constexpr (KW > 1) {
    if (wave > 0)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < TILES; ++t) red[wave - 1][c][t][lane] = acc[c][t];
    __syncthreads();
    if (wave > 0) return;
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int v = v0 + c * 16 + lane / 16 * 4;
    f32x4 b;
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = bias && v + j < V ? bias[v + j] : 0.f;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int n = n0 + t * 16 + lane % 16;
      if (n >= tk.rows || v >= ldz) continue;
      f32x4 o = acc[c][t];
      if constexpr (KW > 1)
#pragma unroll
        for (int i = 0; i < KW - 1; ++i) o += red[i][c][t][lane];
      o += b;
      if (tk.stats) {
        const bool counts = tk.counts(n);
        const int m = min(n, N - 1);
        const float2 st = tk.stats[m];
        const float by = tk.scale * (tk.row_grad ? tk.row_grad[m] : 1.f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[j] = counts && v + j < V ? by * (__builtin_amdgcn_exp2f(fmaf(o[j] - st.x, LOG2E, -st.y * LOG2E)) - (v + j == tk.labels[m] ? 1.f : 0.f)) : 0.f;
      }
      *(f32x4*)(z + n * ldz + v) = o;                        // (ldz: whole fours)
    }
  }
}

// a workgroup a token.  grad: the logits become G (of tk.rows rows)
template <int NT>
__global__ __launch_bounds__(NT) void small_rows_kernel(float* __restrict__ z, int64_t ldz, Tokens tk, float* __restrict__ loss, float2* __restrict__ stats, bool grad) {
  constexpr int WAVES = NT / WAVE;
  __shared__ float red[2][WAVES];
  const int m = blockIdx.x, wave = threadIdx.x / WAVE, V = tk.V;
  float* row = z + m * ldz;
  if (m >= tk.N) {
    for (int v = threadIdx.x; v < ldz; v += NT) row[v] = 0.f;
    return;
  }
  auto four = [&](int v) __attribute__((always_inline)) {          // (ldz: whole fours)
    f32x4 p = *(const f32x4*)(row + v);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = v + j < V ? p[j] : -INFINITY;
    return p;
  };
  float most = -INFINITY;
#pragma unroll 4
  for (int v = threadIdx.x * 4; v < V; v += NT * 4) {
    const f32x4 p = four(v);
    most = fmaxf(most, fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])));
  }
  most = wave_max(most);
  if (threadIdx.x % WAVE == 0) red[0][wave] = most;
  __syncthreads();
  most = red[0][0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) most = fmaxf(most, red[0][i]);
  // (fmaxf passes NaN over, the sum does not; a row of -inf alone has sum 0)
  const float ref = most == -INFINITY ? 0.f : most;
  float s = 0.f;
#pragma unroll 4
  for (int v = threadIdx.x * 4; v < V; v += NT * 4) {
    const f32x4 p = four(v);
#pragma unroll
    for (int j = 0; j < 4; ++j) s += __builtin_amdgcn_exp2f((p[j] - ref) * LOG2E);
  }
  s = wave_sum(s);
  if (threadIdx.x % WAVE == 0) red[1][wave] = s;
  __syncthreads();
  s = red[1][0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) s += red[1][i];
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
  const float weight = tk.row_grad ? tk.row_grad[m] : 1.f, by = tk.scale * weight;
  const bool counts = there && weight != 0.f;
#pragma unroll 4
  for (int v = threadIdx.x * 4; v < ldz; v += NT * 4) {
    f32x4 p = *(const f32x4*)(row + v);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = counts && v + j < V ? by * (__builtin_amdgcn_exp2f(fmaf(p[j] - most, LOG2E, -ls * LOG2E)) - (v + j == label ? 1.f : 0.f)) : 0.f;
    *(f32x4*)(row + v) = p;
  }
}

// logits to G in their place, with the row's weight: four classes a thread
__global__ __launch_bounds__(256) void small_turn_kernel(float* __restrict__ z, int64_t ldz, Tokens tk) {
  const int n = blockIdx.y, v = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (v >= ldz) return;
  const bool counts = tk.counts(n);
  const int m = min(n, tk.N - 1);
  const float2 st = tk.stats[m];
  const float by = tk.scale * (tk.row_grad ? tk.row_grad[m] : 1.f);
  f32x4 p = *(const f32x4*)(z + n * ldz + v);
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = counts && v + j < tk.V ? by * (__builtin_amdgcn_exp2f(fmaf(p[j] - st.x, LOG2E, -st.y * LOG2E)) - (v + j == tk.labels[m] ? 1.f : 0.f)) : 0.f;
  *(f32x4*)(z + n * ldz + v) = p;
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

// Classes that a workgroup takes alone, with the maxima and sums of its rows: two launches instead of four.  (Loss and gradients of 32 x 768 x 100 fp32 18.7 us against 21.5, of 250 classes 23.7 against
// 22.5; 64 x 4096 x 250 bf16 33 against 37)
constexpr int fused_classes(bool f32) { return f32 ? 128 : 256; }
// features of a lane: as many as leave registers for two wavefronts a SIMD
constexpr int few_features(bool f32, int tiles) { return f32 || tiles > 2 ? 4 : 8; }

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
// Four values of G, and what they are multiplied by, of the four k of a lane.  fp32: as they are, four products of 16 x 16 x 4.  Beside bf16: G in two bf16 terms, off by 2^-17 of itself, which take
// the eight k of one product of 16 x 16 x 32 and meet the other operand twice
template <typename T> struct Four;
template <> struct Four<float> {
  typedef f32x4 Other;
  f32x4 v;
  Four() = default;
  __device__ __forceinline__ explicit Four(f32x4 g) : v(g) {}
  // four classes of token lm to a tile; four tokens of class lm from it
  __device__ __forceinline__ void put(float (*tile)[16][20], int lm, int lq) const { *(f32x4*)&tile[0][lm][4 * lq] = v; }
  __device__ __forceinline__ Four(const float (*tile)[16][20], int lm, int lq) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = tile[0][4 * lq + j][lm];
  }
};
template <> struct Four<bf16> {
  typedef bf16x4 Other;
  bf16x8 v;
  Four() = default;
  __device__ __forceinline__ void put(bf16 (*tile)[16][16], int lm, int lq) const {
    *(bf16x4*)&tile[0][lm][4 * lq] = bf16x4{v[0], v[1], v[2], v[3]};
    *(bf16x4*)&tile[1][lm][4 * lq] = bf16x4{v[4], v[5], v[6], v[7]};
  }
  // (lanes 4 e + q of 16 name the address of classes 4 q .. of token e, and get a class each, four tokens of it)
  __device__ __forceinline__ Four(bf16 (*tile)[16][16], int lm, int lq) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef s16x4 __attribute__((address_space(3))) * at;
    const bf16x4 h = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)&tile[0][4 * lq + lm / 4][lm % 4 * 4]));
    const bf16x4 l = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)&tile[1][4 * lq + lm / 4][lm % 4 * 4]));
    v = bf16x8{h[0], h[1], h[2], h[3], l[0], l[1], l[2], l[3]};
  }
  __device__ __forceinline__ explicit Four(f32x4 g) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float h = __uint_as_float(__float_as_uint(g[j]) & 0xffff0000u);
      v[j] = (bf16)h;
      v[4 + j] = (bf16)(g[j] - h);
    }
  }
};
// What two terms leave of G, 8 bits more, for dw in fp32 beside bf16: the third term, of four classes of a token to a tile, and of four tokens of a class from it (as above)
__device__ __forceinline__ bf16x4 third(f32x4 g, const Four<bf16>& two) {
  bf16x4 m;
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = (bf16)((g[j] - (float)two.v[j]) - (float)two.v[4 + j]);
  return m;
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ s16x4 third_from(bf16 (*tile)[16], int lm, int lq) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)&tile[4 * lq + lm / 4][lm % 4 * 4]);
}
__device__ __forceinline__ f32x4 times(const Four<float>& g, f32x4 b, f32x4 c) { return multiplied(g.v, b, c); }
__device__ __forceinline__ f32x4 times(const Four<bf16>& g, bf16x4 b, f32x4 c) { return multiplied(g.v, bf16x8{b[0], b[1], b[2], b[3], b[0], b[1], b[2], b[3]}, c); }

// dx = G w, dw = G^T x and db of up to 16 TILES tokens and any number of classes, w read and dw written once.  A workgroup takes 16 K features and a range of the classes, a wavefront every
// fourth 16 of these, in products of 16 x 16 whose column l % 16 of product i is feature K (l % 16) + i: a lane reads and writes K features together.  x's part stays in
// registers; dx's is added up over the range and leaves as a part, or, of one range, as it is.  G: [16 TILES, ldz], ldz whole sixteens, zero behind the last token and class.
// LOGITS (of fused_classes() at most): G is still logits; every workgroup works out the rows' maxima and sums for itself, the first one leaves them and the losses.
template <typename T, typename TW, int TILES, bool LOGITS>
__global__ __launch_bounds__(256, 2) void few_grads_kernel(const float* __restrict__ G, int64_t ldz, Tokens tk, int D, const T* __restrict__ x, int64_t ldx,
                                                                               const T* __restrict__ w, int64_t ldw, float* __restrict__ parts, int64_t ldp, int per, T* __restrict__ dx,
                                                                               int64_t lddx, TW* __restrict__ dw, int64_t lddw, float* __restrict__ db) {
  constexpr int K = few_features(sizeof(T) == 4, TILES), STEP = 64;
  typedef typename Some<K, T>::vec vec;
  typedef typename Four<T>::Other other;
  __shared__ f32x4 red[3][K][WAVE];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, lm = lane % 16, lq = lane / 16, d = (blockIdx.x * 16 + lm) * K, N = tk.N, V = tk.V;
  const int begin = blockIdx.y * per, end = min(begin + per, V);
  const bool whole = (int)(blockIdx.x + 1) * 16 * K <= D;        // no feature of the workgroup lies behind the last
  const bool want_dx = parts || dx;
  __shared__ float4 rows[LOGITS ? 16 * TILES : 1];               // maximum, -log2 of the sum, weight, label (-1: the row does not count)
  if constexpr (LOGITS) {
    constexpr int MINE = 4 * TILES, EACH = fused_classes(sizeof(T) == 4) / WAVE;
    float z[MINE][EACH], most[MINE], s[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i)
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        const int n = i * 4 + wave, v = k * WAVE + lane;
        z[i][k] = n < N && v < V ? G[n * ldz + v] : -INFINITY;
      }
    // (thread n has token n's label, weight and logit on their way meanwhile)
    const int n = threadIdx.x, label = n < N ? tk.labels[n] : -1;
    const bool known = label >= 0 && label < V;
    const float weight = n < N && tk.row_grad ? tk.row_grad[n] : 1.f, mine = known ? G[n * ldz + label] : 0.f;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      most[i] = z[i][0];
#pragma unroll
      for (int k = 1; k < EACH; ++k) most[i] = fmaxf(most[i], z[i][k]);
      most[i] = wave_max(most[i]);
    }
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const float ref = most[i] == -INFINITY ? 0.f : most[i];      // (as small_rows_kernel)
      s[i] = 0.f;
#pragma unroll
      for (int k = 0; k < EACH; ++k) s[i] += __builtin_amdgcn_exp2f((z[i][k] - ref) * LOG2E);
      s[i] = wave_sum(s[i]);
    }
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < MINE; ++i) *(float2*)&rows[i * 4 + wave] = make_float2(most[i], s[i]);
    __syncthreads();
    if (n < 16 * TILES) {
      const float top = rows[n].x, sum = rows[n].y, ls = sum == 0.f ? 0.f : logf(sum);
      const bool there = known && !(top == -INFINITY && sum == 0.f);
      rows[n] = make_float4(top, -ls * LOG2E, tk.scale * weight, __int_as_float(there && weight != 0.f ? label : -1));
      if (n < N && blockIdx.x == 0) {
        if (tk.stats_out) tk.stats_out[n] = make_float2(top, ls);
        tk.loss[n] = there ? (top - mine) + ls : 0.f;
      }
    }
    __syncthreads();
  }
  auto counting = [&](int n) __attribute__((always_inline)) { return LOGITS ? __float_as_int(rows[n].w) >= 0 : tk.counts(n); };
  auto gradient = [&](float z, int n, int v) __attribute__((always_inline)) {     // of token n and class v
    const float4 r = rows[LOGITS ? n : 0];
    const int label = __float_as_int(r.w);
    return label >= 0 && v < V ? r.z * (__builtin_amdgcn_exp2f(fmaf(z - r.x, LOG2E, r.y)) - (v == label ? 1.f : 0.f)) : 0.f;
  };
  other xb[TILES][K];                              // of four tokens
  f32x4 acc[TILES][K];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = t * 16 + 4 * lq + j;
      const bool counts = counting(n);                             // (a row that does not count may hold anything)
      const vec v = some<K>(x + (int64_t)min(n, N - 1) * ldx, d, D);
#pragma unroll
      for (int i = 0; i < K; ++i) xb[t][i][j] = counts ? v[i] : (T)0.f;
    }
#pragma unroll
    for (int i = 0; i < K; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // G by rows (four classes of token l % 16), 256 MB at most: places in 32 bits; by columns (four tokens of class l % 16) through LDS, in bf16 with its transposing reads
  constexpr bool FINE = sizeof(T) == 2 && sizeof(TW) == 4;         // dw keeps more bits than two terms of G have
  constexpr int TERMS = sizeof(T) == 2 ? 2 + FINE : 1, LD = sizeof(T) == 2 ? 16 : 20;
  __shared__ __attribute__((aligned(16))) T turn[4][TILES][TERMS][16][LD];
  const unsigned by_row = lm * (unsigned)ldz + 4 * lq;
  vec nb[4];
  f32x4 nr[TILES];
  auto fetch = [&](int v0) __attribute__((always_inline)) {        // (a step ahead)
    if (v0 >= end) return;
    if (want_dx) {
      if (whole)
#pragma unroll
        for (int j = 0; j < 4; ++j) nb[j] = *(const vec*)(w + (int64_t)min(v0 + 4 * lq + j, V - 1) * ldw + d);
      else
#pragma unroll
        for (int j = 0; j < 4; ++j) nb[j] = some<K>(w + (int64_t)min(v0 + 4 * lq + j, V - 1) * ldw, d, D);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) nr[t] = *(const f32x4*)(G + (size_t)t * 16 * ldz + (by_row + (unsigned)v0));
  };
  fetch(begin + wave * 16);
  for (int v0 = begin + wave * 16; v0 < end; v0 += STEP) {
    const int v = v0 + 4 * lq;
    other b[K];                                    // of four classes
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) b[i][j] = nb[j][i];
    Four<T> row[TILES];
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if constexpr (LOGITS)
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) nr[t][j] = gradient(nr[t][j], t * 16 + lm, v + j);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      row[t] = Four<T>(nr[t]);
      sum += nr[t];
      row[t].put(turn[wave][t], lm, lq);
      if constexpr (FINE) *(bf16x4*)&turn[wave][t][TERMS - 1][lm][4 * lq] = third(nr[t], row[t]);
    }
    fetch(v0 + STEP);
    if (want_dx)
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < K; ++i) acc[t][i] = times(row[t], b[i], acc[t][i]);
    if (dw) {
      f32x4 out[K];
#pragma unroll
      for (int i = 0; i < K; ++i) out[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      wave_fence();
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const Four<T> g(turn[wave][t], lm, lq);
#pragma unroll
        for (int i = 0; i < K; ++i) out[i] = times(g, xb[t][i], out[i]);
        if constexpr (FINE) {
          const s16x4 m = third_from(turn[wave][t][TERMS - 1], lm, lq);
#pragma unroll
          for (int i = 0; i < K; ++i) out[i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(m, __builtin_bit_cast(s16x4, xb[t][i]), out[i], 0, 0, 0);
        }
      }
      wave_fence();
      auto put_row = [&](int r, bool all) __attribute__((always_inline)) {
        typename Some<K, TW>::vec o;
#pragma unroll
        for (int i = 0; i < K; ++i) o[i] = (TW)out[i][r];
        TW* to = dw + (int64_t)(v + r) * lddw;
        if (all) *(typename Some<K, TW>::vec*)(to + d) = o;
        else if (v + r < end) put<K>(to, d, D, o);
      };
      const bool all = whole && v0 + 16 <= end;
      if (all)
#pragma unroll
        for (int r = 0; r < 4; ++r) put_row(r, true);
      else
#pragma unroll
        for (int r = 0; r < 4; ++r) put_row(r, false);
    }
    if (db && blockIdx.x == 0) {                   // over the tokens, 16 lanes
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int o = 1; o < 16; o *= 2) sum[j] += __shfl_xor(sum[j], o);
        if (lm == j && v + j < end) db[v + j] = sum[j];
      }
    }
  }
  if (!want_dx) return;
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
        if (dx && n < N) {
          typename Some<K, T>::vec o;
#pragma unroll
          for (int i = 0; i < K; ++i) o[i] = counting(n) ? (T)acc[t][i][r] : (T)0.f;
          put<K>(dx + n * lddx, d, D, o);
        } else if (n < N)
#pragma unroll
          for (int i = 0; i < K; i += 4)
            if (d + i < D) *(f32x4*)(parts + ((int64_t)blockIdx.y * N + n) * ldp + d + i) = f32x4{acc[t][i][r], acc[t][i + 1][r], acc[t][i + 2][r], acc[t][i + 3][r]};
      }
  }
}
// dx from its parts, in order
template <typename T> __global__ __launch_bounds__(1024) void few_sums_kernel(const float* __restrict__ parts, int count, int64_t ldp, Tokens tk, int D, T* __restrict__ dx, int64_t lddx) {
  constexpr int WAVES = 16;
  const int t = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, d = (blockIdx.x * WAVE + t) * 4, n = blockIdx.y;
  __shared__ f32x4 red[WAVES][WAVE];
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (d < D)
#pragma unroll 8
    for (int p = wave; p < count; p += WAVES) v += *(const f32x4*)(parts + ((int64_t)p * tk.N + n) * ldp + d);
  red[wave][t] = v;
  __syncthreads();
  if (wave > 0 || d >= D) return;
#pragma unroll
  for (int i = 1; i < WAVES; ++i) v += red[i][t];
  if (!tk.counts(n)) v = f32x4{0.f, 0.f, 0.f, 0.f};                // (whatever w holds)
  put<4>(dx + n * lddx, d, D, typename Some<4, T>::vec{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
}

int64_t small_ldz(const LinearCe& a) { return small_ce_stride(a.N, a.V); }
// Two times 16 classes a workgroup (and four times 16 tokens, fp32) from 2^13 classes on, which fill the CUs then: forward of 32 x 1024 fp32 and 4096 classes 16.1 us, one times 16 14.4; 8192 17.1 and 19.6;
// 32768 52 and 61; 48 rows of 8192 24.0 and 30.6; 32 x 1000 x 8192 bf16 15.8 and 19.2.
// Every wavefront with classes of its own (KW 1) for rows of up to 256 bytes of so many, which would leave most of eight without features: 48 x 64 x 100000 fp32 36 us against 42, 500 x 40 x 8192 22.4 and 34.4, 400 x 64
// x 8192 bf16 23.7 and 34.9; longer rows 48 x 128 x 40000 fp32 29.4 and 24.9, 1 x 250 x 40000 bf16 19.0 and 15.7.
template <typename T> void logits_as(const LinearCe& a, const Tokens& tk, float* z, hipStream_t s) {
  auto go = [&](auto kernel, int classes, int tokens) {
    kernel<<<dim3(over(a.V, classes), over(a.N, tokens)), LOGIT_WAVES * WAVE, 0, s>>>((const T*)a.x, a.ldx, (const T*)a.w, a.ldw, a.D, a.bias, tk, z, small_ldz(a));
  };
  const bool many = a.V >= 1 << 13, narrow = many && a.D * sizeof(T) <= 256;
  if constexpr (sizeof(T) == 4)                    // (as many tokens beside bf16 rows of more features: tiles)
    if (a.N > 32 && many && !narrow) return go(small_logits_kernel<T, 4, 8, 2>, 32, 64);
  if (a.N <= 16) narrow ? go(small_logits_kernel<T, 1, 1, 1>, 128, 16) : many ? go(small_logits_kernel<T, 1, 8, 2>, 32, 16) : go(small_logits_kernel<T, 1, 8, 1>, 16, 16);
  else if (a.N > 32 && narrow) go(small_logits_kernel<T, 4, 1, 1>, 128, 64);
  else narrow ? go(small_logits_kernel<T, 2, 1, 1>, 128, 32) : many ? go(small_logits_kernel<T, 2, 8, 2>, 32, 32) : go(small_logits_kernel<T, 2, 8, 1>, 16, 32);
}
int few_tiles_of(int N) { return N > 32 ? 4 : N > 16 ? 2 : 1; }
int few_wide(bool f32, int N) { return 16 * few_features(f32, few_tiles_of(N)); }
// workgroups over the classes
int few_ranges(bool f32, int N, int V, int D) { return V <= fused_classes(f32) ? 1 : std::min(over(V, 64), std::max(1, 1024 / over(D, few_wide(f32, N)))); }

template <typename T, typename TW, bool LOGITS> void grads_as(const LinearCe& a, const Tokens& tk, const float* G, float* parts, hipStream_t s) {
  const int wide = few_wide(a.f32, a.N);
  const int64_t ldp = ((int64_t)a.D + 3) / 4 * 4;
  const int per = over(over(a.V, few_ranges(a.f32, a.N, a.V, a.D)), 64) * 64, ranges = over(a.V, per);
  const bool direct = ranges == 1;
  if (!a.dx || direct) parts = nullptr;
  auto go = [&](auto kernel) {
    kernel<<<dim3(a.dx || a.dw ? over(a.D, wide) : 1, ranges), 256, 0, s>>>(G, small_ldz(a), tk, a.D, (const T*)a.x, a.ldx, (const T*)a.w, a.ldw, parts, ldp, per, direct ? (T*)a.dx : nullptr, a.lddx,
                                                                          (TW*)a.dw, a.lddw, a.db);
  };
  if (a.N <= 16) go(few_grads_kernel<T, TW, 1, LOGITS>);
  else if (a.N <= 32) go(few_grads_kernel<T, TW, 2, LOGITS>);
  else go(few_grads_kernel<T, TW, 4, LOGITS>);
  if (parts) few_sums_kernel<T><<<dim3(over(a.D, 256), a.N), 1024, 0, s>>>(parts, ranges, ldp, tk, a.D, (T*)a.dx, a.lddx);
}
template <bool LOGITS> void grads(const LinearCe& a, const Tokens& tk, const float* G, float* parts, hipStream_t s) {
  if (a.f32) grads_as<float, float, LOGITS>(a, tk, G, parts, s);
  else if (a.dw_f32) grads_as<bf16, float, LOGITS>(a, tk, G, parts, s);
  else grads_as<bf16, bf16, LOGITS>(a, tk, G, parts, s);
}

}  // namespace

static Tokens tokens_of(const LinearCe& a) {
  Tokens tk;
  tk.N = tk.rows = a.N; tk.V = a.V; tk.labels = a.labels; tk.row_grad = a.row_grad; tk.scale = a.grad_scale;
  return tk;
}
static void logits_of(const LinearCe& a, const Tokens& tk, float* z, hipStream_t s) {
  if (a.f32) logits_as<float>(a, tk, z, s);
  else logits_as<bf16>(a, tk, z, s);
}

void small_ce_logits(const LinearCe& a, float* z, hipStream_t s) { logits_of(a, tokens_of(a), z, s); }

void small_ce_forward(const LinearCe& a, float* z, bool grad, hipStream_t s) {
  Tokens tk = tokens_of(a);
  logits_of(a, tk, z, s);
  if (grad) tk.rows = 16 * few_tiles_of(a.N);
  // (forward of 300 x 300 x 2000 fp32 15.5 us with 1024 threads a row, 15.2 with 256; 500 x 60 x 8192 23.2 and 22.8; 4 x 256 x 40000 18.2 and 21.7; 32 x 64 x 100000 27.9 and 35.2; loss and gradients of 16 x 512 x
  // 8192 27.4 and 28.4, of 16384 36.4 and 40.1)
  if (a.V > 4096) small_rows_kernel<1024><<<tk.rows, 1024, 0, s>>>(z, small_ldz(a), tk, a.loss, (float2*)a.stats, grad);
  else small_rows_kernel<256><<<tk.rows, 256, 0, s>>>(z, small_ldz(a), tk, a.loss, (float2*)a.stats, grad);
}

size_t few_parts_at(int N, int V) { return (small_ce_bytes(16 * few_tiles_of(N), V) + 255) / 256 * 256; }
size_t few_ce_bytes(bool f32, int N, int V, int D) { return sizeof(float) * (size_t)few_ranges(f32, N, V, D) * N * (((size_t)D + 3) / 4 * 4); }
void few_ce_backward(const LinearCe& a, Few there, hipStream_t s) {
  float *G = (float*)a.workspace, *parts = (float*)((char*)a.workspace + few_parts_at(a.N, a.V));
  Tokens tk = tokens_of(a);
  tk.stats = (const float2*)a.stats;
  tk.rows = 16 * few_tiles_of(a.N);
  if (there == FEW_NOTHING) logits_of(a, tk, G, s);
  if (there == FEW_LOGITS) small_turn_kernel<<<dim3(over(small_ldz(a), 1024), tk.rows), 256, 0, s>>>(G, small_ldz(a), tk);
  if (there == FEW_FUSED) {
    tk.stats = nullptr;                            // (and the logits as they are)
    logits_of(a, tk, G, s);
    tk.loss = a.loss; tk.stats_out = (float2*)a.stats;
    grads<true>(a, tk, G, parts, s);
  } else grads<false>(a, tk, G, parts, s);
}

bool few_fused(bool f32, int V) { return V <= fused_classes(f32); }

}  // namespace bsr
