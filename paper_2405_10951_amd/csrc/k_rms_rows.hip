// RMSNorm of rows of any length and stride with the residual's addition in front, to rows of the input's type and / or to 8-bit rows (fp8.h), and its backward.
//   s = x + r;   y = s rstd gamma, rstd = 1 / sqrt(mean(s^2) + eps);   backward from h, the s that was kept:
//   dh = res + rstd (g - xhat mean(g xhat)), g = dy gamma, xhat = h rstd;   dgamma = sum over rows of dy xhat
// The sum is held in fp32 for the norm and rounded once where it is kept: the norm does not see that rounding (a backward pass does, as any does that keeps its
// activations in 16 bits).
// Bound by memory: a row is read once, into registers, by 64 to 1024 threads (two 16-byte chunks each at most), sums are fp32, over rows in a fixed order.
// Rows longer than the registers take (16384 bf16, 8192 fp32), or shorter than a chunk, are read again for every pass over them (`any` kernels).
// Measured: 16384 x 8192 bf16 with the residual, forward 182 us, backward 204, each 1.07 GB (5.9 and 5.3 TB/s; a copy of 2 GiB 4.96: more of this is reading); 6304 x 768 bf16 with residual to 8-bit
// rows 8.0; 1031 x 1777 fp32 backward 6.4 and 4.6 for the sums over its 512 partial rows; 1 x 4096 bf16 1.9.
#include <algorithm>

#include "rms_rows.h"
#include "row_chunks.h"

namespace bsr {

namespace {

constexpr int FINAL_WAVES = 16;

template <typename T, bool WHOLE, int TPR, int MAXC, bool RES, bool OUT, bool OUT8>
__global__ __launch_bounds__(block_threads<TPR>()) void rms_fwd_kernel(const T* x, const T* res, int64_t M, int D, int64_t ldx, int64_t ldr,
                                                                       const float* __restrict__ gamma, float eps, T* sum, int64_t lds, T* y, int64_t ldy,
                                                                       uint8_t* __restrict__ q, uint8_t* __restrict__ scale, float* __restrict__ rstd) {
  typedef typename Chunk<T>::vec vec;
  constexpr int V = Chunk<T>::V, NT = block_threads<TPR>();
  constexpr bool AHEAD = V * MAXC <= 16;                   // gamma asked for with the row (more would cost wavefronts)
  __shared__ float red[NT / WAVE][2];
  const int t = threadIdx.x % TPR;
  const int64_t m = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
  if (m >= M) return;                                     // (whole wavefronts, or the whole workgroup)
  const int nch = D / V, skip = WHOLE ? 0 : V - (D - nch * V), all = nch + (!WHOLE && skip < V);      // whole chunks; all
  auto has = [&](int c, int e) __attribute__((always_inline)) { return c < nch || (!WHOLE && c < all && e >= skip); };
  vec raw[MAXC], more[RES ? MAXC : 1];
  float v[MAXC][V], g[AHEAD ? MAXC : 1][V];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) raw[i] = get_chunk<WHOLE>(x + m * ldx, t + i * TPR, D);
  if constexpr (RES)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) more[i] = get_chunk<WHOLE>(res + m * ldr, t + i * TPR, D);
  if constexpr (AHEAD)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) get_params<WHOLE>(gamma, t + i * TPR, D, g[i]);
  float sq = 0.f, none = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[i][e] = has(t + i * TPR, e) ? (float)raw[i][e] : 0.f;
      if constexpr (RES) v[i][e] += has(t + i * TPR, e) ? (float)more[i][e] : 0.f;
      sq += v[i][e] * v[i][e];
    }
  row_sums<TPR>(sq, none, red);                           // (behind it nobody reads x or res any more: results may take their places)
  const float rs = rsqrtf(sq / (float)D + eps);
  if (t == 0 && rstd) rstd[m] = rs;
  const int64_t ldq = ld8(D), lds8 = ld8s(D);
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = t + i * TPR;
    if (RES && sum && c < all) {
      vec w;
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = (T)v[i][e];
      put_chunk<WHOLE>(sum + m * lds, c, D, c < nch, skip, w);
    }
    float o[V];
    if (c < all) {
      if constexpr (!AHEAD) get_params<WHOLE>(gamma, c, D, g[0]);
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = has(c, e) ? v[i][e] * rs * g[AHEAD ? i : 0][e] : 0.f;
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
    if constexpr (OUT8) put_chunk8<WHOLE, TPR, V>(o, i, c, nch, all, skip, ldq, q + m * ldq, scale + m * lds8);
  }
  if (OUT8 && t < lds8 - ldq / BLOCK8) scale[m * lds8 + ldq / BLOCK8 + t] = 127;
}

// any row: a wavefront each, read twice (an element is read and written by the same lane, so results may take the inputs' places)
template <typename T, bool OUT, bool OUT8>
__global__ __launch_bounds__(256) void rms_fwd_any_kernel(const T* x, const T* res, int64_t M, int D, int64_t ldx, int64_t ldr, const float* __restrict__ gamma,
                                                          float eps, T* sum, int64_t lds, T* y, int64_t ldy, uint8_t* __restrict__ q, uint8_t* __restrict__ scale,
                                                          float* __restrict__ rstd) {
  const int lane = threadIdx.x % WAVE;
  const int64_t m = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
  if (m >= M) return;
  auto at = [&](int64_t j) __attribute__((always_inline)) { return (float)x[m * ldx + j] + (res ? (float)res[m * ldr + j] : 0.f); };
  float sq = 0.f;
  for (int j = lane; j < D; j += WAVE) {
    const float v = at(j);
    sq += v * v;
  }
  const float rs = rsqrtf(wave_sum(sq) / (float)D + eps);
  if (lane == 0 && rstd) rstd[m] = rs;
  const int64_t ldq = ld8(D), lds8 = ld8s(D);
  for (int64_t j0 = 0; j0 < ldq; j0 += BLOCK8) {          // a block at a time, two values a lane
    float o[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t j = j0 + 2 * lane + e;
      const float v = j < D ? at(j) : 0.f;
      o[e] = j < D ? v * rs * gamma[j] : 0.f;
      if (res && sum && j < D) sum[m * lds + j] = (T)v;
      if (OUT && j < D) y[m * ldy + j] = (T)o[e];
    }
    if constexpr (OUT8) {
      const uint32_t s8 = scale8_of(__float_as_uint(wave_max(__uint_as_float(max(finite_bits(o[0]), finite_bits(o[1]))))));
      *(uint16_t*)(q + m * ldq + j0 + 2 * lane) = (uint16_t)pack8(o[0], o[1], 0.f, 0.f, inverse_of(s8));
      if (lane == 0) scale[m * lds8 + j0 / BLOCK8] = (uint8_t)s8;
    }
  }
  if (OUT8 && lane < lds8 - ldq / BLOCK8) scale[m * lds8 + ldq / BLOCK8 + lane] = 127;
}

// Backward, with the next row's loads in flight.  Each group of TPR threads walks every gridDim.x (NT / TPR)-th row and keeps its sums for dgamma in registers;
// the wavefronts of a workgroup then add theirs in a fixed order and leave them in partial[blockIdx.x].  (dx may take the place of an input: a thread writes the
// values that it alone uses; those in front of them in the last chunk, which another thread may have written by then, do not count.)
template <typename T, bool WHOLE, int TPR, int MAXC, bool DX, bool PARAMS, bool RES>
__global__ __launch_bounds__(block_threads<TPR>(), TPR == 512 ? 4 : 1) void rms_bwd_kernel(const T* dy, int64_t lddy, const T* x, int64_t ldx, const T* res, int64_t ldr,
                                                                                         int64_t M, int D, const float* __restrict__ rstd,
                                                                                         const float* __restrict__ gamma, T* dx, int64_t lddx,
                                                                                         float* __restrict__ partial) {
  constexpr int V = Chunk<T>::V, NT = block_threads<TPR>(), RPB = NT / TPR;
  typedef typename Chunk<T>::vec vec;
  constexpr bool KEEP = NT <= 256;                        // gamma in registers (larger workgroups: more wavefronts on the CU count for more)
  constexpr bool RES_EARLY = TPR < 512;                   // the residual a row ahead as well
  extern __shared__ __attribute__((aligned(16))) float lds_sums[];                     // [RPB / 2][D in whole chunks]
  __shared__ float red[2][NT / WAVE][2];
  const int t = threadIdx.x % TPR, r = threadIdx.x / TPR, nch = D / V;
  const int skip = WHOLE ? 0 : V - (D - nch * V), all = nch + (!WHOLE && skip < V), P = all * V;
  auto has = [&](int c, int e) __attribute__((always_inline)) { return c < nch || (!WHOLE && c < all && e >= skip); };
  const int64_t stride = (int64_t)gridDim.x * RPB;
  float dg[PARAMS ? MAXC : 1][V], gk[KEEP ? MAXC : 1][V];
#pragma unroll
  for (int i = 0; i < (PARAMS ? MAXC : 1); ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dg[i][e] = 0.f;
  if constexpr (KEEP && DX)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) get_params<WHOLE>(gamma, t + i * TPR, D, gk[i]);
  vec na[MAXC], nx[MAXC], nr[RES && RES_EARLY ? MAXC : 1];
  float nrs = 0.f;
  auto prefetch = [&](int64_t m) __attribute__((always_inline)) {
    if (m >= M) return;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      na[i] = get_chunk<WHOLE>(dy + m * lddy, t + i * TPR, D);
      nx[i] = get_chunk<WHOLE>(x + m * ldx, t + i * TPR, D);
      if constexpr (RES && RES_EARLY) nr[i] = get_chunk<WHOLE>(res + m * ldr, t + i * TPR, D);
    }
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
    const float rs = nrs;
    prefetch(m + stride);
    float s2 = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < MAXC; ++i)
      if (t + i * TPR < all) {
        float g[V];
        if constexpr (!KEEP && DX) get_params<WHOLE>(gamma, t + i * TPR, D, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const bool counts = WHOLE || has(t + i * TPR, e);
          const float dxh = counts ? (float)a[i][e] * ((float)b[i][e] * rs) : 0.f;
          if constexpr (PARAMS) dg[i][e] += dxh;
          if constexpr (DX) s2 += dxh * (KEEP ? gk[KEEP ? i : 0][e] : g[e]);
        }
      }
    if constexpr (DX) {
      row_sums<TPR>(s2, none, red[turn]);
      if constexpr (RES && !RES_EARLY)
#pragma unroll
        for (int i = 0; i < MAXC; ++i) c[i] = get_chunk<WHOLE>(res + m * ldr, t + i * TPR, D);
      const float m2 = s2 / (float)D;
#pragma unroll
      for (int i = 0; i < MAXC; ++i) {
        const int ch = t + i * TPR;
        if (ch < all) {
          float g[V];
          if constexpr (!KEEP) get_params<WHOLE>(gamma, ch, D, g);
          vec o;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            float v = rs * ((float)a[i][e] * (KEEP ? gk[KEEP ? i : 0][e] : g[e]) - (float)b[i][e] * rs * m2);
            if constexpr (RES) v += (float)c[i][e];
            o[e] = (T)v;
          }
          put_chunk<WHOLE>(dx + m * lddx, ch, D, ch < nch, skip, o);
        }
      }
    }
  }
  if constexpr (PARAMS) {
#pragma unroll
    for (int half = RPB / 2; half > 0; half /= 2) {       // (pairwise: a fixed tree)
      if (r >= half && r < 2 * half)
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
          if (t + i * TPR < all)
#pragma unroll
            for (int e = 0; e < V; e += 4)
              *(float4*)(lds_sums + (size_t)(r - half) * P + (t + i * TPR) * V + e) = make_float4(dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]);
      __syncthreads();
      if (r < half)
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
          if (t + i * TPR < all) {
            float u[V];
            load_params<V>(lds_sums + (size_t)r * P + (t + i * TPR) * V, u);
#pragma unroll
            for (int e = 0; e < V; ++e) dg[i][e] += u[e];
          }
      __syncthreads();
    }
    if (r == 0)
#pragma unroll
      for (int i = 0; i < MAXC; ++i)
        if (t + i * TPR < all)
#pragma unroll
          for (int e = 0; e < V; e += 4)
            *(float4*)(partial + (int64_t)blockIdx.x * P + (t + i * TPR) * V + e) = make_float4(dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rms_bwd_dx_any_kernel(const T* dy, int64_t lddy, const T* x, int64_t ldx, const T* res, int64_t ldr, int64_t M, int D,
                                                             const float* __restrict__ rstd, const float* __restrict__ gamma, T* dx, int64_t lddx) {
  const int lane = threadIdx.x % WAVE;
  const int64_t m = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
  if (m >= M) return;
  const float rs = rstd[m];
  const T *dr = dy + m * lddy, *xr = x + m * ldx;
  float s2 = 0.f;
  for (int j = lane; j < D; j += WAVE) s2 += (float)dr[j] * gamma[j] * ((float)xr[j] * rs);
  const float m2 = wave_sum(s2) / (float)D;
  for (int j = lane; j < D; j += WAVE) {
    float v = rs * ((float)dr[j] * gamma[j] - (float)xr[j] * rs * m2);
    if (res) v += (float)res[m * ldr + j];
    dx[m * lddx + j] = (T)v;
  }
}

// where a partial row of P floats has column col: the last part of a row lies at the end of its chunk
template <typename T> __device__ __forceinline__ int part_at(int col, int D, int P) { return col < D / Chunk<T>::V * Chunk<T>::V ? col : col + P - D; }

// sums over the rows of chunk blockIdx.y for 64 columns
template <typename T>
__global__ __launch_bounds__(256) void rms_bwd_params_any_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, int64_t M, int D,
                                                                 const float* __restrict__ rstd, int64_t per_chunk, int P, float* __restrict__ partial) {
  __shared__ float red[4][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, col = blockIdx.x * WAVE + lane;
  const int64_t r0 = (int64_t)blockIdx.y * per_chunk, r1 = min(r0 + per_chunk, M);
  float s = 0.f;
  if (col < D)
    for (int64_t m = r0 + w; m < r1; m += 4) s += (float)dy[m * lddy + col] * ((float)x[m * ldx + col] * rstd[m]);
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < D) partial[(int64_t)blockIdx.y * P + part_at<T>(col, D, P)] = red[0][lane] + red[1][lane] + red[2][lane] + red[3][lane];
}

// the sums over the partial rows of P floats (those from `whole` on at their ends), 64 sums a workgroup: wavefront w adds rows w, w + 16, ..., then the wavefronts in order
__global__ __launch_bounds__(FINAL_WAVES * WAVE) void rms_bwd_final_kernel(const float* __restrict__ partial, int D, int P, int whole, int rows, float* __restrict__ dgamma) {
  __shared__ float red[FINAL_WAVES][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE;
  const int64_t col = (int64_t)blockIdx.x * WAVE + lane;
  float s = 0.f;
  if (col < P) {
    // all rows of a wavefront on their way at once, those past the last one again and not counted (one by one they would each be a trip to memory)
    constexpr int K = RMS_PARTIALS / FINAL_WAVES;
    float v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = rows > 0 ? partial[(int64_t)min(w + k * FINAL_WAVES, rows - 1) * P + col] : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) s += w + k * FINAL_WAVES < rows ? v[k] : 0.f;
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < P) {
    s = red[0][lane];
#pragma unroll
    for (int i = 1; i < FINAL_WAVES; ++i) s += red[i][lane];
    const int at = (int)col, j = at < whole ? at : at - (P - D);
    if (at < whole || j >= whole) dgamma[j] = s;
  }
}

template <typename T, bool OUT, bool OUT8>
void fwd_as(const RmsRows& a, hipStream_t s) {
  const bool whole = a.D % Chunk<T>::V == 0 && in_chunks<T>(a.x, a.ldx) && (!a.res || (in_chunks<T>(a.res, a.ldr) && (!a.sum || in_chunks<T>(a.sum, a.lds)))) &&
                     (!OUT || in_chunks<T>(a.y, a.ldy));
  const int n = (a.D + Chunk<T>::V - 1) / Chunk<T>::V;
  auto go = [&](auto WHOLE, auto TPR, auto C) {
    constexpr int tpr = decltype(TPR)::value, nt = block_threads<tpr>(), rpb = nt / tpr;
    auto as = [&](auto RES) {
      rms_fwd_kernel<T, decltype(WHOLE)::value != 0, tpr, decltype(C)::value, decltype(RES)::value != 0, OUT, OUT8><<<(unsigned)((a.M + rpb - 1) / rpb), nt, 0, s>>>(
          (const T*)a.x, (const T*)a.res, a.M, a.D, a.ldx, a.ldr, a.gamma, a.eps, (T*)a.sum, a.lds, (T*)a.y, a.ldy, (uint8_t*)a.q, a.scale, a.rstd);
    };
    if (a.res) as(RowC<1>{});
    else as(RowC<0>{});
  };
  // (a row shorter than a chunk has no whole one to read)
  const bool done = whole ? with_row_chunks_of(n, [&](auto TPR, auto C) { go(RowC<1>{}, TPR, C); })
                          : a.D >= Chunk<T>::V && with_row_chunks_of(n, [&](auto TPR, auto C) { go(RowC<0>{}, TPR, C); });
  if (!done)
    rms_fwd_any_kernel<T, OUT, OUT8><<<(unsigned)((a.M + 3) / 4), 256, 0, s>>>((const T*)a.x, (const T*)a.res, a.M, a.D, a.ldx, a.ldr, a.gamma, a.eps, (T*)a.sum, a.lds,
                                                                             (T*)a.y, a.ldy, (uint8_t*)a.q, a.scale, a.rstd);
}
template <typename T>
void fwd(const RmsRows& a, hipStream_t s) {
  if (a.y && a.q) fwd_as<T, true, true>(a, s);
  else if (a.q) fwd_as<T, false, true>(a, s);
  else fwd_as<T, true, false>(a, s);
}

template <typename T>
void bwd(const RmsRowsBwd& a, hipStream_t s) {
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
        const unsigned grid = (unsigned)(p ? std::min<int64_t>(need, RMS_PARTIALS) : need);
        rms_bwd_kernel<T, decltype(WHOLE)::value != 0, tpr, maxc, decltype(DX)::value != 0, p, decltype(RES)::value != 0>
            <<<grid, nt, p ? rpb / 2 * P * sizeof(float) : 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, (const T*)a.res, a.ldr, a.M, a.D, a.rstd, a.gamma, (T*)a.dx,
                                                                  a.lddx, a.partial);
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
        rms_bwd_params_any_kernel<T><<<dim3((a.D + WAVE - 1) / WAVE, rows), 256, 0, s>>>((const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, a.M, a.D, a.rstd, per_chunk, P,
                                                                                       a.partial);
      }
      for (int64_t m = 0; a.dx && m < a.M; m += ROWS_A_LAUNCH) {
        const int64_t here = std::min(ROWS_A_LAUNCH, a.M - m);
        rms_bwd_dx_any_kernel<T><<<(unsigned)((here + 3) / 4), 256, 0, s>>>((const T*)a.dy + m * a.lddy, a.lddy, (const T*)a.x + m * a.ldx, a.ldx,
                                                                          a.res ? (const T*)a.res + m * a.ldr : nullptr, a.ldr, here, a.D, a.rstd + m, a.gamma,
                                                                          (T*)a.dx + m * a.lddx, a.lddx);
      }
    }
  }
  if (params) rms_bwd_final_kernel<<<(unsigned)((P + WAVE - 1) / WAVE), FINAL_WAVES * WAVE, 0, s>>>(a.partial, a.D, P, a.D / Chunk<T>::V * Chunk<T>::V, rows, a.dgamma);
}

}  // namespace

void rms_rows_fwd(const RmsRows& a, hipStream_t s) {
  const int64_t size = a.f32 ? 4 : 2;
  for (int64_t m = 0; m < a.M; m += ROWS_A_LAUNCH) {
    RmsRows b = a;
    b.M = std::min(ROWS_A_LAUNCH, a.M - m);
    b.x = (const char*)a.x + m * a.ldx * size;
    if (a.res) b.res = (const char*)a.res + m * a.ldr * size;
    if (a.sum) b.sum = (char*)a.sum + m * a.lds * size;
    if (a.y) b.y = (char*)a.y + m * a.ldy * size;
    if (a.q) { b.q = (uint8_t*)a.q + m * ld8(a.D); b.scale = a.scale + m * ld8s(a.D); }
    if (a.rstd) b.rstd = a.rstd + m;
    if (a.f32) fwd<float>(b, s);
    else fwd<bf16>(b, s);
  }
}

void rms_rows_bwd(const RmsRowsBwd& a, hipStream_t s) {
  const int64_t size = a.f32 ? 4 : 2;
  if (a.dgamma || a.M <= ROWS_A_LAUNCH) {                  // (with sums the workgroups are few and walk the rows)
    if (a.f32) bwd<float>(a, s);
    else bwd<bf16>(a, s);
    return;
  }
  for (int64_t m = 0; m < a.M; m += ROWS_A_LAUNCH) {
    RmsRowsBwd b = a;
    b.M = std::min(ROWS_A_LAUNCH, a.M - m);
    b.dy = (const char*)a.dy + m * a.lddy * size;
    b.x = (const char*)a.x + m * a.ldx * size;
    if (a.res) b.res = (const char*)a.res + m * a.ldr * size;
    b.dx = (char*)a.dx + m * a.lddx * size;
    b.rstd = a.rstd + m;
    if (a.f32) bwd<float>(b, s);
    else bwd<bf16>(b, s);
  }
}

}  // namespace bsr
