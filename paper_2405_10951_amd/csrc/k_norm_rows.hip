// LayerNorm as an operator of its own: rows of any length and stride, forward to rows of the input's type and / or to 8-bit rows (fp8.h), and
// backward with the sums over rows that are the gradients of gamma and beta.  (The LayerNorms inside the step, whose rows lie together and whose
// sums over rows wait for one another, are in k_layernorm.hip.)
//   y = (x - mu) rstd gamma + beta;   dx = res + rstd (g - mean(g) - xhat mean(g xhat)), g = dy gamma;   dgamma = sum dy xhat, dbeta = sum dy
// Bound by memory: a row is read once, into registers, by 64 or 256 threads; statistics and sums are fp32, two-pass within the registers, sums over
// rows in a fixed order.  Rows that are no whole 16-byte chunks, are not aligned to them or are longer than the registers take are read again for
// every pass over them (`any` kernels).
#include <algorithm>

#include "fp8.h"
#include "norm_rows.h"

namespace bsr {

namespace {

constexpr int FINAL_WAVES = 16;

// A piece of a row: V values, V 16-byte chunks' worth or 1 (rows that are no whole chunks, or are not aligned to them)
template <typename T, int V> struct Piece { typedef T vec __attribute__((ext_vector_type(V))); };
template <typename T> struct Piece<T, 1> { struct vec { T v; __device__ __forceinline__ T& operator[](int) { return v; } __device__ __forceinline__ T operator[](int) const { return v; } }; };
// Results go past the caches, a wavefront's store being whole lines (16384 x 8192: forward 130 -> 94 us, backward 174 -> 170; 25216 x 768 backward 32 -> 26)
template <class P> __device__ __forceinline__ void put_past(P* to, const P& v) {
  if constexpr (sizeof(P) == 16) __builtin_nontemporal_store(v, to);
  else *to = v;
}
template <int V> __device__ __forceinline__ void params(const float* p, float (&o)[V]) {
  if constexpr (V == 1) o[0] = *p;
  else load_params<V>(p, o);
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

template <typename T, int V, int TPR, int MAXC, bool OUT, bool OUT8>
__global__ __launch_bounds__(block_threads<TPR>()) void rows_fwd_kernel(const T* __restrict__ x, int64_t M, int D, int64_t ldx,
                                                                        const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                                        T* __restrict__ y, int64_t ldy, uint8_t* __restrict__ q,
                                                                        uint8_t* __restrict__ scale, float* __restrict__ mean,
                                                                        float* __restrict__ rstd) {
  typedef typename Piece<T, V>::vec vec;
  constexpr int NT = block_threads<TPR>();
  constexpr bool AHEAD = V * MAXC <= 16;                   // gamma and beta asked for with the row (more would cost wavefronts)
  __shared__ float red[2][NT / WAVE][2];
  const int t = threadIdx.x % TPR;
  const int64_t m = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
  if (m >= M) return;                                     // (whole wavefronts, or the whole workgroup)
  const int nch = D / V;
  const T* xr = x + m * ldx;
  vec raw[MAXC];
  float v[MAXC][V], g[AHEAD ? MAXC : 1][V], b[AHEAD ? MAXC : 1][V];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) raw[i] = *(const vec*)(xr + min(t + i * TPR, nch - 1) * V);
  if constexpr (AHEAD)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = min(t + i * TPR, nch - 1) * V;
      params<V>(gamma + c, g[i]);
      params<V>(beta + c, b[i]);
    }
  float s = 0.f, none = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) { v[i][e] = t + i * TPR < nch ? (float)raw[i][e] : 0.f; s += v[i][e]; }
  row_sums<TPR>(s, none, red[0]);
  const float mu = s / (float)D;
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) { const float d = t + i * TPR < nch ? v[i][e] - mu : 0.f; sq += d * d; }
  row_sums<TPR>(sq, none, red[1]);
  const float rs = rsqrtf(sq / (float)D + eps);
  if (t == 0) {
    if (mean) mean[m] = mu;
    if (rstd) rstd[m] = rs;
  }
  const int64_t ldq = ld8(D), lds = ld8s(D);
  float o1[OUT8 && V == 1 ? MAXC : 1];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = t + i * TPR;
    float o[V];
    if (c < nch) {
      if constexpr (!AHEAD) {
        params<V>(gamma + c * V, g[0]);
        params<V>(beta + c * V, b[0]);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = (v[i][e] - mu) * rs * g[AHEAD ? i : 0][e] + b[AHEAD ? i : 0][e];
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = 0.f;
    }
    if (OUT && c < nch) {
      vec w;
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = (T)o[e];
      put_past((vec*)(y + m * ldy + c * V), w);
    }
    if constexpr (OUT8 && V == 1) {                       // two pieces of a wavefront hold a block
      static_assert(TPR == WAVE && MAXC % 2 == 0, "");
      o1[i] = o[0];
      if (i % 2 == 1 && (i - 1) * TPR < ldq) {
        const uint32_t s8 = scale8_of(__float_as_uint(wave_max(__uint_as_float(max(finite_bits(o1[i - 1]), finite_bits(o1[i]))))));
        const float inv = inverse_of(s8);
        uint8_t* to = q + m * ldq + (i - 1) * TPR + t;
        const uint32_t two = pack8(o1[i - 1], o1[i], 0.f, 0.f, inv);
        to[0] = (uint8_t)two;
        to[TPR] = (uint8_t)(two >> 8);
        if (t == 0) scale[m * lds + i / 2] = (uint8_t)s8;
      }
    } else if constexpr (OUT8) {                          // BLOCK8 / V neighbouring lanes hold a block
      if (i * TPR * V < ldq) {
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
          uint32_t* to = (uint32_t*)(q + m * ldq + c * V);
          if constexpr (V == 8) *(uint2*)to = make_uint2(pack8(o[0], o[1], o[2], o[3], inv), pack8(o[4], o[5], o[6], o[7], inv));
          else *to = pack8(o[0], o[1], o[2], o[3], inv);
          if (c * V % BLOCK8 == 0) scale[m * lds + c * V / BLOCK8] = (uint8_t)s8;
        }
      }
    }
  }
  if (OUT8 && t < lds - ldq / BLOCK8) scale[m * lds + ldq / BLOCK8 + t] = 127;
}

// any row: a wavefront each, read three times
template <typename T, bool OUT, bool OUT8>
__global__ __launch_bounds__(256) void rows_fwd_any_kernel(const T* __restrict__ x, int64_t M, int D, int64_t ldx, const float* __restrict__ gamma,
                                                           const float* __restrict__ beta, float eps, T* __restrict__ y, int64_t ldy,
                                                           uint8_t* __restrict__ q, uint8_t* __restrict__ scale, float* __restrict__ mean,
                                                           float* __restrict__ rstd) {
  const int lane = threadIdx.x % WAVE;
  const int64_t m = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
  if (m >= M) return;
  const T* xr = x + m * ldx;
  float s = 0.f;
  for (int j = lane; j < D; j += WAVE) s += (float)xr[j];
  const float mu = wave_sum(s) / (float)D;
  float sq = 0.f;
  for (int j = lane; j < D; j += WAVE) {
    const float d = (float)xr[j] - mu;
    sq += d * d;
  }
  const float rs = rsqrtf(wave_sum(sq) / (float)D + eps);
  if (lane == 0) {
    if (mean) mean[m] = mu;
    if (rstd) rstd[m] = rs;
  }
  const int64_t ldq = ld8(D), lds = ld8s(D);
  for (int64_t j0 = 0; j0 < ldq; j0 += BLOCK8) {          // a block at a time, two values a lane
    float o[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t j = j0 + 2 * lane + e;
      o[e] = j < D ? ((float)xr[j] - mu) * rs * gamma[j] + beta[j] : 0.f;
      if (OUT && j < D) y[m * ldy + j] = (T)o[e];
    }
    if constexpr (OUT8) {
      const uint32_t s8 = scale8_of(__float_as_uint(wave_max(__uint_as_float(max(finite_bits(o[0]), finite_bits(o[1]))))));
      *(uint16_t*)(q + m * ldq + j0 + 2 * lane) = (uint16_t)pack8(o[0], o[1], 0.f, 0.f, inverse_of(s8));
      if (lane == 0) scale[m * lds + j0 / BLOCK8] = (uint8_t)s8;
    }
  }
  if (OUT8 && lane < lds - ldq / BLOCK8) scale[m * lds + ldq / BLOCK8 + lane] = 127;
}

// Backward, with the next row's loads in flight.  Each group of TPR threads walks every gridDim.x (NT / TPR)-th row and keeps
// its sums for dgamma and dbeta in registers; the wavefronts of a workgroup then add theirs in a fixed order and leave them in
// partial[blockIdx.x] = [dgamma | dbeta].
template <typename T, int V, int TPR, int MAXC, bool DX, bool PARAMS, bool RES>
__global__ __launch_bounds__(block_threads<TPR>(), TPR == 512 ? 4 : 1) void rows_bwd_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
                                                                        const T* __restrict__ res, int64_t ldr, int64_t M, int D,
                                                                        const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                        const float* __restrict__ gamma, T* __restrict__ dx, int64_t lddx,
                                                                        float* __restrict__ partial) {
  constexpr int NT = block_threads<TPR>(), RPB = NT / TPR;
  typedef typename Piece<T, V>::vec vec;
  constexpr bool KEEP = NT <= 256;                        // gamma in registers (larger workgroups: more wavefronts on the CU count for more)
  constexpr bool RES_EARLY = TPR < 512;                   // the residual a row ahead as well
  extern __shared__ __attribute__((aligned(16))) float lds_sums[];                     // [RPB / 2][2][D]
  __shared__ float red[2][NT / WAVE][2];
  const int t = threadIdx.x % TPR, r = threadIdx.x / TPR, nch = D / V;
  const int64_t stride = (int64_t)gridDim.x * RPB;
  float dg[PARAMS ? MAXC : 1][V], db[PARAMS ? MAXC : 1][V], gk[KEEP ? MAXC : 1][V];
#pragma unroll
  for (int i = 0; i < (PARAMS ? MAXC : 1); ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dg[i][e] = db[i][e] = 0.f;
  if constexpr (KEEP)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) params<V>(gamma + min(t + i * TPR, nch - 1) * V, gk[i]);
  vec na[MAXC], nx[MAXC], nr[RES && RES_EARLY ? MAXC : 1];
  float nmu = 0.f, nrs = 0.f;
  auto prefetch = [&](int64_t m) __attribute__((always_inline)) {
    if (m >= M) return;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = min(t + i * TPR, nch - 1) * V;
      na[i] = *(const vec*)(dy + m * lddy + c);
      nx[i] = *(const vec*)(x + m * ldx + c);
      if constexpr (RES && RES_EARLY) nr[i] = *(const vec*)(res + m * ldr + c);
    }
    nmu = mean[m];
    nrs = rstd[m];
  };
  int64_t m = (int64_t)blockIdx.x * RPB + r;
  prefetch(m);
  for (int turn = 0; m < M; m += stride, turn ^= 1) {
    vec a[MAXC], b[MAXC], c[RES ? MAXC : 1];
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      a[i] = na[i];
      b[i] = nx[i];
      if constexpr (RES && RES_EARLY) c[i] = nr[i];
    }
    const float mu = nmu, rs = nrs;
    prefetch(m + stride);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < MAXC; ++i)
      if (t + i * TPR < nch) {
        float g[V];
        if constexpr (!KEEP) params<V>(gamma + (t + i * TPR) * V, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = (float)a[i][e], xh = ((float)b[i][e] - mu) * rs, gd = d * (KEEP ? gk[KEEP ? i : 0][e] : g[e]);
          if constexpr (PARAMS) { dg[i][e] += d * xh; db[i][e] += d; }
          s1 += gd;
          s2 += gd * xh;
        }
      }
    if constexpr (DX) {
      row_sums<TPR>(s1, s2, red[turn]);
      if constexpr (RES && !RES_EARLY)
#pragma unroll
        for (int i = 0; i < MAXC; ++i) c[i] = *(const vec*)(res + m * ldr + min(t + i * TPR, nch - 1) * V);
      const float m1 = s1 / (float)D, m2 = s2 / (float)D;
#pragma unroll
      for (int i = 0; i < MAXC; ++i) {
        const int ch = t + i * TPR;
        if (ch < nch) {
          float g[V];
          if constexpr (!KEEP) params<V>(gamma + ch * V, g);
          vec o;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float xh = ((float)b[i][e] - mu) * rs;
            float v = rs * ((float)a[i][e] * (KEEP ? gk[KEEP ? i : 0][e] : g[e]) - m1 - xh * m2);
            if constexpr (RES) v += (float)c[i][e];
            o[e] = (T)v;
          }
          put_past((vec*)(dx + m * lddx + ch * V), o);
        }
      }
    }
  }
  if constexpr (PARAMS) {
    // the sums to p = [dgamma | dbeta], or those at p added to them; four at a time where pieces are whole chunks
    auto leave = [&](float* p) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MAXC; ++i)
        if (t + i * TPR < nch) {
          float* to = p + (t + i * TPR) * V;
          if constexpr (V == 1) { to[0] = dg[i][0]; to[D] = db[i][0]; }
          else
#pragma unroll
            for (int e = 0; e < V; e += 4) {
              *(float4*)(to + e) = make_float4(dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]);
              *(float4*)(to + D + e) = make_float4(db[i][e], db[i][e + 1], db[i][e + 2], db[i][e + 3]);
            }
        }
    };
    auto add = [&](const float* p) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MAXC; ++i)
        if (t + i * TPR < nch) {
          float u[V], w[V];
          params<V>(p + (t + i * TPR) * V, u);
          params<V>(p + D + (t + i * TPR) * V, w);
#pragma unroll
          for (int e = 0; e < V; ++e) { dg[i][e] += u[e]; db[i][e] += w[e]; }
        }
    };
#pragma unroll
    for (int half = RPB / 2; half > 0; half /= 2) {       // (pairwise: a fixed tree)
      if (r >= half && r < 2 * half) leave(lds_sums + (size_t)(r - half) * 2 * D);
      __syncthreads();
      if (r < half) add(lds_sums + (size_t)r * 2 * D);
      __syncthreads();
    }
    if (r == 0) leave(partial + (int64_t)blockIdx.x * 2 * D);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rows_bwd_dx_any_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
                                                              const T* __restrict__ res, int64_t ldr, int64_t M, int D,
                                                              const float* __restrict__ mean, const float* __restrict__ rstd,
                                                              const float* __restrict__ gamma, T* __restrict__ dx, int64_t lddx) {
  const int lane = threadIdx.x % WAVE;
  const int64_t m = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
  if (m >= M) return;
  const float mu = mean[m], rs = rstd[m];
  const T *dr = dy + m * lddy, *xr = x + m * ldx;
  float s1 = 0.f, s2 = 0.f;
  for (int j = lane; j < D; j += WAVE) {
    const float g = (float)dr[j] * gamma[j];
    s1 += g;
    s2 += g * (((float)xr[j] - mu) * rs);
  }
  const float m1 = wave_sum(s1) / (float)D, m2 = wave_sum(s2) / (float)D;
  for (int j = lane; j < D; j += WAVE) {
    const float g = (float)dr[j] * gamma[j], xh = ((float)xr[j] - mu) * rs;
    float v = rs * (g - m1 - xh * m2);
    if (res) v += (float)res[m * ldr + j];
    dx[m * lddx + j] = (T)v;
  }
}

// sums over the rows of chunk blockIdx.y for 64 columns
template <typename T>
__global__ __launch_bounds__(256) void rows_bwd_params_any_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
                                                                  int64_t M, int D, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, int64_t per_chunk, float* __restrict__ partial) {
  __shared__ float red[2][4][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, col = blockIdx.x * WAVE + lane;
  const int64_t r0 = (int64_t)blockIdx.y * per_chunk, r1 = min(r0 + per_chunk, M);
  float s0 = 0.f, s1 = 0.f;
  if (col < D)
    for (int64_t m = r0 + w; m < r1; m += 4) {
      const float d = (float)dy[m * lddy + col];
      s0 += d * (((float)x[m * ldx + col] - mean[m]) * rstd[m]);
      s1 += d;
    }
  red[0][w][lane] = s0;
  red[1][w][lane] = s1;
  __syncthreads();
  if (w == 0 && col < D) {
    float* p = partial + (int64_t)blockIdx.y * 2 * D;
    p[col] = red[0][0][lane] + red[0][1][lane] + red[0][2][lane] + red[0][3][lane];
    p[D + col] = red[1][0][lane] + red[1][1][lane] + red[1][2][lane] + red[1][3][lane];
  }
}

// the 2 D sums over the partial rows, 64 a workgroup: wavefront w adds rows w, w + 16, ..., then the wavefronts in order
__global__ __launch_bounds__(FINAL_WAVES * WAVE) void rows_bwd_final_kernel(const float* __restrict__ partial, int D, int rows,
                                                                            float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float red[FINAL_WAVES][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE;
  const int64_t col = (int64_t)blockIdx.x * WAVE + lane;
  float s = 0.f;
  if (col < 2 * (int64_t)D) {
    // all rows of a wavefront on their way at once, those past the last one again and not counted (one by one they would each be a trip to memory)
    constexpr int K = NORM_PARTIALS / FINAL_WAVES;
    for (int r0 = w; r0 < rows; r0 += K * FINAL_WAVES) {
      float v[K];
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = partial[(int64_t)min(r0 + k * FINAL_WAVES, rows - 1) * 2 * D + col];
#pragma unroll
      for (int k = 0; k < K; ++k) s += r0 + k * FINAL_WAVES < rows ? v[k] : 0.f;
    }
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < 2 * (int64_t)D) {
    s = red[0][lane];
#pragma unroll
    for (int i = 1; i < FINAL_WAVES; ++i) s += red[i][lane];
    if (col < D) dgamma[col] = s;
    else dbeta[col - D] = s;
  }
}

// f(values per piece, threads per row, pieces per thread) for a row of whole 16-byte chunks; false: too long.  Two chunks a thread leave registers for
// four wavefronts a SIMD in the backward pass.
template <typename T, class F> bool with_row_chunks_of(int D, F&& f) {
  constexpr int V = Chunk<T>::V;
  const int n = D / V;
  if (n <= 64) f(RowC<V>{}, RowC<64>{}, RowC<1>{});
  else if (n <= 128) f(RowC<V>{}, RowC<64>{}, RowC<2>{});
  else if (n <= 256) f(RowC<V>{}, RowC<256>{}, RowC<1>{});
  else if (n <= 512) f(RowC<V>{}, RowC<256>{}, RowC<2>{});
  else if (n <= 1024) f(RowC<V>{}, RowC<512>{}, RowC<2>{});
  else if (n <= 2048) f(RowC<V>{}, RowC<1024>{}, RowC<2>{});
  else return false;
  return true;
}
// the backward pass of rows that are no whole chunks: a value a piece
template <class F> bool with_row_values(int D, F&& f) {
  if (D <= 512) f(RowC<1>{}, RowC<64>{}, RowC<8>{});
  else if (D <= 2048) f(RowC<1>{}, RowC<256>{}, RowC<8>{});
  else if (D <= 8192) f(RowC<1>{}, RowC<1024>{}, RowC<8>{});
  else return false;
  return true;
}

template <typename T> bool in_chunks(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0; }

template <typename T, bool OUT, bool OUT8>
void fwd_as(const NormRows& a, hipStream_t s) {
  const bool whole = a.D % Chunk<T>::V == 0 && in_chunks<T>(a.x, a.ldx) && (!OUT || in_chunks<T>(a.y, a.ldy));
  auto go = [&](auto P, auto TPR, auto C) {
    constexpr int v = decltype(P)::value, tpr = decltype(TPR)::value, nt = block_threads<tpr>(), rpb = nt / tpr;
    rows_fwd_kernel<T, v, tpr, decltype(C)::value, OUT, OUT8><<<(unsigned)((a.M + rpb - 1) / rpb), nt, 0, s>>>(
          (const T*)a.x, a.M, a.D, a.ldx, a.gamma, a.beta, a.eps, (T*)a.y, a.ldy, (uint8_t*)a.q, a.scale, a.mean, a.rstd);
  };
  bool done = true;
  // (8-bit blocks are put together from neighbouring chunks, or from two values of every lane of a wavefront; with and without them a row is summed the
  // same way)
  if (whole) done = with_row_chunks_of<T>(a.D, go);
  else if (a.D <= 512) go(RowC<1>{}, RowC<64>{}, RowC<8>{});
  else if (a.D <= 2048) go(RowC<1>{}, RowC<64>{}, RowC<32>{});
  else if (a.D <= 6144) go(RowC<1>{}, RowC<64>{}, RowC<96>{});
  else done = false;
  if (!done)
    rows_fwd_any_kernel<T, OUT, OUT8><<<(unsigned)((a.M + 3) / 4), 256, 0, s>>>((const T*)a.x, a.M, a.D, a.ldx, a.gamma, a.beta, a.eps, (T*)a.y, a.ldy,
                                                                              (uint8_t*)a.q, a.scale, a.mean, a.rstd);
}
template <typename T>
void fwd(const NormRows& a, hipStream_t s) {
  if (a.y && a.q) fwd_as<T, true, true>(a, s);
  else if (a.q) fwd_as<T, false, true>(a, s);
  else fwd_as<T, true, false>(a, s);
}

template <typename T>
void bwd(const NormRowsBwd& a, hipStream_t s) {
  const bool params = a.dgamma != nullptr;
  int rows = 0;                                           // partial rows
  if (a.M > 0) {
    const bool whole = a.D % Chunk<T>::V == 0 && in_chunks<T>(a.dy, a.lddy) && in_chunks<T>(a.x, a.ldx) && (!a.res || in_chunks<T>(a.res, a.ldr)) &&
                       (!a.dx || in_chunks<T>(a.dx, a.lddx));
    auto shaped = [&](auto P, auto TPR, auto C) {
      constexpr int v = decltype(P)::value, tpr = decltype(TPR)::value, maxc = decltype(C)::value;
      auto go = [&](auto DX, auto PARAMS, auto RES) {
        constexpr bool p = decltype(PARAMS)::value != 0;
        constexpr int nt = block_threads<tpr>(), rpb = nt / tpr;
        const int64_t need = (a.M + rpb - 1) / rpb;
        const unsigned grid = (unsigned)(p ? std::min<int64_t>(need, NORM_PARTIALS) : need);
        rows_bwd_kernel<T, v, tpr, maxc, decltype(DX)::value != 0, p, decltype(RES)::value != 0>
            <<<grid, nt, p ? rpb / 2 * 2 * a.D * sizeof(float) : 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, (const T*)a.res, a.ldr, a.M, a.D,
                                                                       a.mean, a.rstd, a.gamma, (T*)a.dx, a.lddx, a.partial);
        if (p) rows = (int)grid;
      };
      if (!a.dx) go(RowC<0>{}, RowC<1>{}, RowC<0>{});
      else if (a.res && params) go(RowC<1>{}, RowC<1>{}, RowC<1>{});
      else if (a.res) go(RowC<1>{}, RowC<0>{}, RowC<1>{});
      else if (params) go(RowC<1>{}, RowC<1>{}, RowC<0>{});
      else go(RowC<1>{}, RowC<0>{}, RowC<0>{});
    };
    const bool done = whole ? with_row_chunks_of<T>(a.D, shaped) : with_row_values(a.D, shaped);
    if (!done) {
      if (a.dx)
        rows_bwd_dx_any_kernel<T><<<(unsigned)((a.M + 3) / 4), 256, 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, (const T*)a.res, a.ldr, a.M,
                                                                          a.D, a.mean, a.rstd, a.gamma, (T*)a.dx, a.lddx);
      if (params) {
        const int64_t per_chunk = (a.M + 63) / 64;
        rows = (int)((a.M + per_chunk - 1) / per_chunk);
        rows_bwd_params_any_kernel<T><<<dim3((a.D + WAVE - 1) / WAVE, rows), 256, 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, a.M, a.D,
                                                                                        a.mean, a.rstd, per_chunk, a.partial);
      }
    }
  }
  if (params) rows_bwd_final_kernel<<<(unsigned)((2 * (int64_t)a.D + WAVE - 1) / WAVE), FINAL_WAVES * WAVE, 0, s>>>(a.partial, a.D, rows, a.dgamma, a.dbeta);
}

}  // namespace

void norm_rows_fwd(const NormRows& a, hipStream_t s) {
  if (a.M <= 0) return;
  if (a.f32) fwd<float>(a, s);
  else fwd<bf16>(a, s);
}

void norm_rows_bwd(const NormRowsBwd& a, hipStream_t s) {
  if (a.f32) bwd<float>(a, s);
  else bwd<bf16>(a, s);
}

}  // namespace bsr
