// LayerNorm as an operator of its own: rows of any length and stride, forward to rows of the input's type and / or to 8-bit rows (fp8.h), and
// backward with the sums over rows that are the gradients of gamma and beta.  (The LayerNorms inside the step, whose rows lie together and whose
// sums over rows wait for one another, are in k_layernorm.hip.)
//   y = (x - mu) rstd gamma + beta;   dx = res + rstd (g - mean(g) - xhat mean(g xhat)), g = dy gamma;   dgamma = sum dy xhat, dbeta = sum dy
// Bound by memory: a row is read once, into registers, by 64 to 1024 threads (two 16-byte chunks each at most); statistics and sums are fp32, two-pass
// within the registers, sums over rows in a fixed order.  Rows longer than the registers take (16384 bf16, 8192 fp32), or shorter than a chunk, are read
// again for every pass over them (`any` kernels).
// Measured, in chains of calls (us; bytes at the rate of a large copy in brackets): 6304 x 768 bf16 forward 5.6 (3.8), to 8 bits 6.3, backward 13.2 (5.7) in two
// launches; 16384 x 8192 bf16 94 (105), 125, 171 (158); 4096 x 5001 bf16, at any address, 26 (16), 26, 47 (24); 1031 x 1777 fp32 4.6 (2.9), 4.7, 12.6 (4.3).
#include <algorithm>

#include "norm_rows.h"
#include "row_chunks.h"

namespace bsr {

namespace {

constexpr int FINAL_WAVES = 16;

template <typename T, bool WHOLE, int TPR, int MAXC, bool OUT, bool OUT8>
__global__ __launch_bounds__(block_threads<TPR>()) void rows_fwd_kernel(const T* __restrict__ x, int64_t M, int D, int64_t ldx,
                                                                        const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                                        T* __restrict__ y, int64_t ldy, uint8_t* __restrict__ q,
                                                                        uint8_t* __restrict__ scale, float* __restrict__ mean,
                                                                        float* __restrict__ rstd) {
  typedef typename Chunk<T>::vec vec;
  constexpr int V = Chunk<T>::V, NT = block_threads<TPR>();
  constexpr bool AHEAD = V * MAXC <= 16;                   // gamma and beta asked for with the row (more would cost wavefronts)
  __shared__ float red[2][NT / WAVE][2];
  const int t = threadIdx.x % TPR;
  const int64_t m = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
  if (m >= M) return;                                     // (whole wavefronts, or the whole workgroup)
  const int nch = D / V, skip = WHOLE ? 0 : V - (D - nch * V), all = nch + (!WHOLE && skip < V);      // whole chunks; all
  auto has = [&](int c, int e) __attribute__((always_inline)) { return c < nch || (!WHOLE && c < all && e >= skip); };
  const T* xr = x + m * ldx;
  vec raw[MAXC];
  float v[MAXC][V], g[AHEAD ? MAXC : 1][V], b[AHEAD ? MAXC : 1][V];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) raw[i] = get_chunk<WHOLE>(xr, t + i * TPR, D);
  if constexpr (AHEAD)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      get_params<WHOLE>(gamma, t + i * TPR, D, g[i]);
      get_params<WHOLE>(beta, t + i * TPR, D, b[i]);
    }
  float s = 0.f, none = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) { v[i][e] = has(t + i * TPR, e) ? (float)raw[i][e] : 0.f; s += v[i][e]; }
  row_sums<TPR>(s, none, red[0]);
  const float mu = s / (float)D;
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) { const float d = has(t + i * TPR, e) ? v[i][e] - mu : 0.f; sq += d * d; }
  row_sums<TPR>(sq, none, red[1]);
  const float rs = rsqrtf(sq / (float)D + eps);
  if (t == 0) {
    if (mean) mean[m] = mu;
    if (rstd) rstd[m] = rs;
  }
  const int64_t ldq = ld8(D), lds = ld8s(D);
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = t + i * TPR;
    float o[V];
    if (c < all) {
      if constexpr (!AHEAD) {
        get_params<WHOLE>(gamma, c, D, g[0]);
        get_params<WHOLE>(beta, c, D, b[0]);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = has(c, e) ? (v[i][e] - mu) * rs * g[AHEAD ? i : 0][e] + b[AHEAD ? i : 0][e] : 0.f;
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = 0.f;
    }
    if (OUT && c < all) {
      vec w;
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = (T)o[e];
      put_chunk<WHOLE>(y + m * ldy, c, D, c < nch, skip, w);
    }
    if constexpr (OUT8) put_chunk8<WHOLE, TPR, V>(o, i, c, nch, all, skip, ldq, q + m * ldq, scale + m * lds);
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
template <typename T, bool WHOLE, int TPR, int MAXC, bool DX, bool PARAMS, bool RES>
__global__ __launch_bounds__(block_threads<TPR>(), TPR == 512 ? 4 : 1) void rows_bwd_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
                                                                        const T* __restrict__ res, int64_t ldr, int64_t M, int D,
                                                                        const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                        const float* __restrict__ gamma, T* __restrict__ dx, int64_t lddx,
                                                                        float* __restrict__ partial) {
  constexpr int V = Chunk<T>::V, NT = block_threads<TPR>(), RPB = NT / TPR;
  typedef typename Chunk<T>::vec vec;
  constexpr bool KEEP = NT <= 256;                        // gamma in registers (larger workgroups: more wavefronts on the CU count for more)
  constexpr bool RES_EARLY = TPR < 512;                   // the residual a row ahead as well
  extern __shared__ __attribute__((aligned(16))) float lds_sums[];                     // [RPB / 2][2][D in whole chunks]
  __shared__ float red[2][NT / WAVE][2];
  const int t = threadIdx.x % TPR, r = threadIdx.x / TPR, nch = D / V;
  const int skip = WHOLE ? 0 : V - (D - nch * V), all = nch + (!WHOLE && skip < V), P = all * V;
  auto has = [&](int c, int e) __attribute__((always_inline)) { return c < nch || (!WHOLE && c < all && e >= skip); };
  const int64_t stride = (int64_t)gridDim.x * RPB;
  float dg[PARAMS ? MAXC : 1][V], db[PARAMS ? MAXC : 1][V], gk[KEEP ? MAXC : 1][V];
#pragma unroll
  for (int i = 0; i < (PARAMS ? MAXC : 1); ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dg[i][e] = db[i][e] = 0.f;
  if constexpr (KEEP)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) get_params<WHOLE>(gamma, t + i * TPR, D, gk[i]);
  vec na[MAXC], nx[MAXC], nr[RES && RES_EARLY ? MAXC : 1];
  float nmu = 0.f, nrs = 0.f;
  auto prefetch = [&](int64_t m) __attribute__((always_inline)) {
    if (m >= M) return;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      na[i] = get_chunk<WHOLE>(dy + m * lddy, t + i * TPR, D);
      nx[i] = get_chunk<WHOLE>(x + m * ldx, t + i * TPR, D);
      if constexpr (RES && RES_EARLY) nr[i] = get_chunk<WHOLE>(res + m * ldr, t + i * TPR, D);
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
      if (t + i * TPR < all) {
        float g[V];
        if constexpr (!KEEP) get_params<WHOLE>(gamma, t + i * TPR, D, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const bool counts = WHOLE || has(t + i * TPR, e);
          const float d = counts ? (float)a[i][e] : 0.f, xh = counts ? ((float)b[i][e] - mu) * rs : 0.f, gd = d * (KEEP ? gk[KEEP ? i : 0][e] : g[e]);
          if constexpr (PARAMS) { dg[i][e] += d * xh; db[i][e] += d; }
          s1 += gd;
          s2 += gd * xh;
        }
      }
    if constexpr (DX) {
      row_sums<TPR>(s1, s2, red[turn]);
      if constexpr (RES && !RES_EARLY)
#pragma unroll
        for (int i = 0; i < MAXC; ++i) c[i] = get_chunk<WHOLE>(res + m * ldr, t + i * TPR, D);
      const float m1 = s1 / (float)D, m2 = s2 / (float)D;
#pragma unroll
      for (int i = 0; i < MAXC; ++i) {
        const int ch = t + i * TPR;
        if (ch < all) {
          float g[V];
          if constexpr (!KEEP) get_params<WHOLE>(gamma, ch, D, g);
          vec o;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float xh = ((float)b[i][e] - mu) * rs;
            float v = rs * ((float)a[i][e] * (KEEP ? gk[KEEP ? i : 0][e] : g[e]) - m1 - xh * m2);
            if constexpr (RES) v += (float)c[i][e];
            o[e] = (T)v;
          }
          put_chunk<WHOLE>(dx + m * lddx, ch, D, ch < nch, skip, o);
        }
      }
    }
  }
  if constexpr (PARAMS) {
    // the sums to p = [dgamma | dbeta], or those at p added to them
    auto leave = [&](float* p) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MAXC; ++i)
        if (t + i * TPR < all) {
          float* to = p + (t + i * TPR) * V;
#pragma unroll
          for (int e = 0; e < V; e += 4) {
            *(float4*)(to + e) = make_float4(dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]);
            *(float4*)(to + P + e) = make_float4(db[i][e], db[i][e + 1], db[i][e + 2], db[i][e + 3]);
          }
        }
    };
    auto add = [&](const float* p) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MAXC; ++i)
        if (t + i * TPR < all) {
          float u[V], w[V];
          load_params<V>(p + (t + i * TPR) * V, u);
          load_params<V>(p + P + (t + i * TPR) * V, w);
#pragma unroll
          for (int e = 0; e < V; ++e) { dg[i][e] += u[e]; db[i][e] += w[e]; }
        }
    };
#pragma unroll
    for (int half = RPB / 2; half > 0; half /= 2) {       // (pairwise: a fixed tree)
      if (r >= half && r < 2 * half) leave(lds_sums + (size_t)(r - half) * 2 * P);
      __syncthreads();
      if (r < half) add(lds_sums + (size_t)r * 2 * P);
      __syncthreads();
    }
    if (r == 0) leave(partial + (int64_t)blockIdx.x * 2 * P);
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

// where a partial row of P floats has column col: the last part of a row lies at the end of its chunk
template <typename T> __device__ __forceinline__ int part_at(int col, int D, int P) { return col < D / Chunk<T>::V * Chunk<T>::V ? col : col + P - D; }

// sums over the rows of chunk blockIdx.y for 64 columns
template <typename T>
__global__ __launch_bounds__(256) void rows_bwd_params_any_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
                                                                  int64_t M, int D, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, int64_t per_chunk, int P, float* __restrict__ partial) {
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
    float* p = partial + (int64_t)blockIdx.y * 2 * P;
    const int at = part_at<T>(col, D, P);
    p[at] = red[0][0][lane] + red[0][1][lane] + red[0][2][lane] + red[0][3][lane];
    p[P + at] = red[1][0][lane] + red[1][1][lane] + red[1][2][lane] + red[1][3][lane];
  }
}

// the sums over the partial rows [dgamma | dbeta], P floats each (those from `whole` on at their ends), 64 sums a workgroup: wavefront w adds rows w, w + 16, ..., then the wavefronts in order
__global__ __launch_bounds__(FINAL_WAVES * WAVE) void rows_bwd_final_kernel(const float* __restrict__ partial, int D, int P, int whole, int rows,
                                                                            float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float red[FINAL_WAVES][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE;
  const int64_t col = (int64_t)blockIdx.x * WAVE + lane;
  float s = 0.f;
  if (col < 2 * (int64_t)P) {
    // all rows of a wavefront on their way at once, those past the last one again and not counted (one by one they would each be a trip to memory)
    constexpr int K = NORM_PARTIALS / FINAL_WAVES;
    for (int r0 = w; r0 < rows; r0 += K * FINAL_WAVES) {
      float v[K];
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = partial[(int64_t)min(r0 + k * FINAL_WAVES, rows - 1) * 2 * P + col];
#pragma unroll
      for (int k = 0; k < K; ++k) s += r0 + k * FINAL_WAVES < rows ? v[k] : 0.f;
    }
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < 2 * (int64_t)P) {
    s = red[0][lane];
#pragma unroll
    for (int i = 1; i < FINAL_WAVES; ++i) s += red[i][lane];
    const int at = (int)(col < P ? col : col - P), j = at < whole ? at : at - (P - D);
    if (at < whole || j >= whole) (col < P ? dgamma : dbeta)[j] = s;
  }
}

template <typename T, bool OUT, bool OUT8>
void fwd_as(const NormRows& a, hipStream_t s) {
  const bool whole = a.D % Chunk<T>::V == 0 && in_chunks<T>(a.x, a.ldx) && (!OUT || in_chunks<T>(a.y, a.ldy));
  const int n = (a.D + Chunk<T>::V - 1) / Chunk<T>::V;
  auto go = [&](auto WHOLE, auto TPR, auto C) {
    constexpr int tpr = decltype(TPR)::value, nt = block_threads<tpr>(), rpb = nt / tpr;
    rows_fwd_kernel<T, decltype(WHOLE)::value != 0, tpr, decltype(C)::value, OUT, OUT8><<<(unsigned)((a.M + rpb - 1) / rpb), nt, 0, s>>>(
          (const T*)a.x, a.M, a.D, a.ldx, a.gamma, a.beta, a.eps, (T*)a.y, a.ldy, (uint8_t*)a.q, a.scale, a.mean, a.rstd);
  };
  // (a row shorter than a chunk has no whole one to read)
  const bool done = whole ? with_row_chunks_of(n, [&](auto TPR, auto C) { go(RowC<1>{}, TPR, C); })
                          : a.D >= Chunk<T>::V && with_row_chunks_of(n, [&](auto TPR, auto C) { go(RowC<0>{}, TPR, C); });
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
  const int n = (a.D + Chunk<T>::V - 1) / Chunk<T>::V, P = n * Chunk<T>::V;
  if (a.M > 0) {
    const bool whole = a.D % Chunk<T>::V == 0 && in_chunks<T>(a.dy, a.lddy) && in_chunks<T>(a.x, a.ldx) && (!a.res || in_chunks<T>(a.res, a.ldr)) &&
                       (!a.dx || in_chunks<T>(a.dx, a.lddx));
    auto shaped = [&](auto WHOLE, auto TPR, auto C) {
      constexpr int tpr = decltype(TPR)::value, maxc = decltype(C)::value;
      auto go = [&](auto DX, auto PARAMS, auto RES) {
        constexpr bool p = decltype(PARAMS)::value != 0;
        constexpr int nt = block_threads<tpr>(), rpb = nt / tpr;
        const int64_t need = (a.M + rpb - 1) / rpb;
        const unsigned grid = (unsigned)(p ? std::min<int64_t>(need, NORM_PARTIALS) : need);
        rows_bwd_kernel<T, decltype(WHOLE)::value != 0, tpr, maxc, decltype(DX)::value != 0, p, decltype(RES)::value != 0>
            <<<grid, nt, p ? rpb / 2 * 2 * P * sizeof(float) : 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, (const T*)a.res, a.ldr, a.M, a.D,
                                                                       a.mean, a.rstd, a.gamma, (T*)a.dx, a.lddx, a.partial);
        if (p) rows = (int)grid;
      };
      if (!a.dx) go(RowC<0>{}, RowC<1>{}, RowC<0>{});
      else if (a.res && params) go(RowC<1>{}, RowC<1>{}, RowC<1>{});
      else if (a.res) go(RowC<1>{}, RowC<0>{}, RowC<1>{});
      else if (params) go(RowC<1>{}, RowC<1>{}, RowC<0>{});
      else go(RowC<1>{}, RowC<0>{}, RowC<0>{});
    };
    const bool done = whole ? with_row_chunks_of(n, [&](auto TPR, auto C) { shaped(RowC<1>{}, TPR, C); })
                            : a.D >= Chunk<T>::V && with_row_chunks_of(n, [&](auto TPR, auto C) { shaped(RowC<0>{}, TPR, C); });
    if (!done) {
      if (params) {                                       // (first: dx may take the place of dy)
        const int64_t per_chunk = (a.M + 63) / 64;
        rows = (int)((a.M + per_chunk - 1) / per_chunk);
        rows_bwd_params_any_kernel<T><<<dim3((a.D + WAVE - 1) / WAVE, rows), 256, 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, a.M, a.D,
                                                                                        a.mean, a.rstd, per_chunk, P, a.partial);
      }
      for (int64_t m = 0; a.dx && m < a.M; m += ROWS_A_LAUNCH) {
        const int64_t here = std::min(ROWS_A_LAUNCH, a.M - m);
        rows_bwd_dx_any_kernel<T><<<(unsigned)((here + 3) / 4), 256, 0, s>>>((const T*)a.dy + m * a.lddy, a.lddy, (const T*)a.x + m * a.ldx, a.ldx,
                                                                           a.res ? (const T*)a.res + m * a.ldr : nullptr, a.ldr, here, a.D, a.mean + m,
                                                                           a.rstd + m, a.gamma, (T*)a.dx + m * a.lddx, a.lddx);
      }
    }
  }
  if (params) rows_bwd_final_kernel<<<(unsigned)((2 * (int64_t)P + WAVE - 1) / WAVE), FINAL_WAVES * WAVE, 0, s>>>(a.partial, a.D, P, a.D / Chunk<T>::V * Chunk<T>::V, rows, a.dgamma, a.dbeta);
}

}  // namespace

void norm_rows_fwd(const NormRows& a, hipStream_t s) {
  const int64_t size = a.f32 ? 4 : 2;
  for (int64_t m = 0; m < a.M; m += ROWS_A_LAUNCH) {
    NormRows b = a;
    b.M = std::min(ROWS_A_LAUNCH, a.M - m);
    b.x = (const char*)a.x + m * a.ldx * size;
    if (a.y) b.y = (char*)a.y + m * a.ldy * size;
    if (a.q) { b.q = (uint8_t*)a.q + m * ld8(a.D); b.scale = a.scale + m * ld8s(a.D); }
    if (a.mean) b.mean = a.mean + m;
    if (a.rstd) b.rstd = a.rstd + m;
    if (a.f32) fwd<float>(b, s);
    else fwd<bf16>(b, s);
  }
}

void norm_rows_bwd(const NormRowsBwd& a, hipStream_t s) {
  const int64_t size = a.f32 ? 4 : 2;
  if (a.dgamma || a.M <= ROWS_A_LAUNCH) {                  // (with sums the workgroups are few and walk the rows)
    if (a.f32) bwd<float>(a, s);
    else bwd<bf16>(a, s);
    return;
  }
  for (int64_t m = 0; m < a.M; m += ROWS_A_LAUNCH) {
    NormRowsBwd b = a;
    b.M = std::min(ROWS_A_LAUNCH, a.M - m);
    b.dy = (const char*)a.dy + m * a.lddy * size;
    b.x = (const char*)a.x + m * a.ldx * size;
    if (a.res) b.res = (const char*)a.res + m * a.ldr * size;
    b.dx = (char*)a.dx + m * a.lddx * size;
    b.mean = a.mean + m;
    b.rstd = a.rstd + m;
    if (a.f32) bwd<float>(b, s);
    else bwd<bf16>(b, s);
  }
}

}  // namespace bsr
