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

// sums of a and b over the threads of a row: a wavefront, or the four of a workgroup (red: two floats a wavefront; a second buffer in turn, so that
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

// maximum over each N lanes (16 or 32, a power of two), bits of non-negative floats
template <int N> __device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < N; o *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}

template <typename T, int TPR, int MAXC, bool OUT, bool OUT8>
__global__ __launch_bounds__(256) void rows_fwd_kernel(const T* __restrict__ x, int64_t M, int D, int64_t ldx, const float* __restrict__ gamma,
                                                       const float* __restrict__ beta, float eps, T* __restrict__ y, int64_t ldy,
                                                       uint8_t* __restrict__ q, uint8_t* __restrict__ scale, float* __restrict__ mean,
                                                       float* __restrict__ rstd) {
  constexpr int V = Chunk<T>::V;
  typedef typename Chunk<T>::vec vec;
  __shared__ float red[2][4][2];
  const int t = threadIdx.x % TPR;
  const int64_t m = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (m >= M) return;                                     // (whole wavefronts, or the whole workgroup)
  const int nch = D / V;
  const T* xr = x + m * ldx;
  vec raw[MAXC];
  float v[MAXC][V];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) raw[i] = *(const vec*)(xr + min(t + i * TPR, nch - 1) * V);
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
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = t + i * TPR;
    float o[V];
    if (c < nch) {
      float g[V], b[V];
      load_params<V>(gamma + c * V, g);
      load_params<V>(beta + c * V, b);
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = (v[i][e] - mu) * rs * g[e] + b[e];
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = 0.f;
    }
    if (OUT && c < nch) {
      vec w;
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = (T)o[e];
      *(vec*)(y + m * ldy + c * V) = w;
    }
    if constexpr (OUT8) {                                 // BLOCK8 / V neighbouring lanes hold a block
      if (i * TPR * V < ldq) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) most = max(most, finite_bits(o[e]));
        const uint32_t s8 = scale8_of(lanes_max<BLOCK8 / V>(most));
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

// Backward, with the next row's loads in flight.  256 / TPR rows of a workgroup at a time; each walks every gridDim.x (256 / TPR)-th row and keeps
// its sums for dgamma and dbeta in registers; the wavefronts of a workgroup then add theirs in a fixed order and leave them in
// partial[blockIdx.x] = [dgamma | dbeta].
template <typename T, int TPR, int MAXC, bool DX, bool PARAMS>
__global__ __launch_bounds__(256) void rows_bwd_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
                                                       const T* __restrict__ res, int64_t ldr, int64_t M, int D, const float* __restrict__ mean,
                                                       const float* __restrict__ rstd, const float* __restrict__ gamma, T* __restrict__ dx,
                                                       int64_t lddx, float* __restrict__ partial) {
  constexpr int V = Chunk<T>::V, RPB = 256 / TPR;
  typedef typename Chunk<T>::vec vec;
  extern __shared__ float lds_sums[];                     // [RPB - 1][2][D]
  __shared__ float red[2][4][2];
  const int t = threadIdx.x % TPR, r = threadIdx.x / TPR, nch = D / V;
  const int64_t stride = (int64_t)gridDim.x * RPB;
  float dg[MAXC][V], db[MAXC][V];
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) dg[i][e] = db[i][e] = 0.f;
  vec na[MAXC], nx[MAXC];
  float nmu = 0.f, nrs = 0.f;
  auto prefetch = [&](int64_t m) __attribute__((always_inline)) {
    if (m >= M) return;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = min(t + i * TPR, nch - 1) * V;
      na[i] = *(const vec*)(dy + m * lddy + c);
      nx[i] = *(const vec*)(x + m * ldx + c);
    }
    nmu = mean[m];
    nrs = rstd[m];
  };
  int64_t m = (int64_t)blockIdx.x * RPB + r;
  prefetch(m);
  for (int turn = 0; m < M; m += stride, turn ^= 1) {
    vec a[MAXC], b[MAXC];
#pragma unroll
    for (int i = 0; i < MAXC; ++i) { a[i] = na[i]; b[i] = nx[i]; }
    const float mu = nmu, rs = nrs;
    prefetch(m + stride);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < MAXC; ++i)
      if (t + i * TPR < nch) {
        float g[V];
        load_params<V>(gamma + (t + i * TPR) * V, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = (float)a[i][e], xh = ((float)b[i][e] - mu) * rs;
          if (PARAMS) { dg[i][e] += d * xh; db[i][e] += d; }
          s1 += d * g[e];
          s2 += d * g[e] * xh;
        }
      }
    if constexpr (DX) {
      row_sums<TPR>(s1, s2, red[turn]);
      const float m1 = s1 / (float)D, m2 = s2 / (float)D;
#pragma unroll
      for (int i = 0; i < MAXC; ++i) {
        const int c = t + i * TPR;
        if (c < nch) {
          float g[V];
          load_params<V>(gamma + c * V, g);
          vec rr, o;
          if (res) rr = *(const vec*)(res + m * ldr + c * V);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float xh = ((float)b[i][e] - mu) * rs;
            float v = rs * ((float)a[i][e] * g[e] - m1 - xh * m2);
            if (res) v += (float)rr[e];
            o[e] = (T)v;
          }
          *(vec*)(dx + m * lddx + c * V) = o;
        }
      }
    }
  }
  if constexpr (PARAMS) {
    auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MAXC; ++i)
        if (t + i * TPR < nch)
#pragma unroll
          for (int e = 0; e < V; ++e) f((t + i * TPR) * V + e, i, e);
    };
    if constexpr (RPB > 1) {
      if (r > 0) {
        float* p = lds_sums + (size_t)(r - 1) * 2 * D;
        each([&](int j, int i, int e) { p[j] = dg[i][e]; p[D + j] = db[i][e]; });
      }
      __syncthreads();
      if (r > 0) return;
      for (int k = 0; k < RPB - 1; ++k) {
        const float* p = lds_sums + (size_t)k * 2 * D;
        each([&](int j, int i, int e) { dg[i][e] += p[j]; db[i][e] += p[D + j]; });
      }
    }
    float* p = partial + (int64_t)blockIdx.x * 2 * D;
    each([&](int j, int i, int e) { p[j] = dg[i][e]; p[D + j] = db[i][e]; });
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
#pragma unroll 8
    for (int r = w; r < rows; r += FINAL_WAVES) s += partial[(int64_t)r * 2 * D + col];
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

// f(threads per row, chunks per thread) for rows of n chunks; false: too long
template <class F> bool with_row_shape(int n, F&& f) {
  if (n <= 64) f(RowC<64>{}, RowC<1>{});
  else if (n <= 128) f(RowC<64>{}, RowC<2>{});
  else if (n <= 256) f(RowC<64>{}, RowC<4>{});
  else if (n <= 512) f(RowC<256>{}, RowC<2>{});
  else if (n <= 1024) f(RowC<256>{}, RowC<4>{});
  else if (n <= 2048) f(RowC<256>{}, RowC<8>{});
  else return false;
  return true;
}

template <typename T> bool in_chunks(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0; }

template <typename T, bool OUT, bool OUT8>
void fwd_as(const NormRows& a, hipStream_t s) {
  constexpr int V = Chunk<T>::V;
  const bool vec = a.D % V == 0 && in_chunks<T>(a.x, a.ldx) && (!OUT || in_chunks<T>(a.y, a.ldy)) &&
                   with_row_shape(a.D / V, [&](auto TPR, auto C) {
                     constexpr int tpr = decltype(TPR)::value, rpb = 256 / tpr;
                     rows_fwd_kernel<T, tpr, decltype(C)::value, OUT, OUT8><<<(unsigned)((a.M + rpb - 1) / rpb), 256, 0, s>>>(
                         (const T*)a.x, a.M, a.D, a.ldx, a.gamma, a.beta, a.eps, (T*)a.y, a.ldy, (uint8_t*)a.q, a.scale, a.mean, a.rstd);
                   });
  if (!vec)
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
  constexpr int V = Chunk<T>::V;
  const bool params = a.dgamma != nullptr;
  int rows = 0;                                           // partial rows
  if (a.M > 0) {
    const bool vec = a.D % V == 0 && in_chunks<T>(a.dy, a.lddy) && in_chunks<T>(a.x, a.ldx) && (!a.res || in_chunks<T>(a.res, a.ldr)) &&
                     (!a.dx || in_chunks<T>(a.dx, a.lddx)) && with_row_shape(a.D / V, [&](auto TPR, auto C) {
                       constexpr int tpr = decltype(TPR)::value, rpb = 256 / tpr, maxc = decltype(C)::value;
                       const int64_t need = (a.M + rpb - 1) / rpb;
                       auto go = [&](auto DX, auto PARAMS) {
                         constexpr bool p = decltype(PARAMS)::value != 0;
                         const unsigned grid = (unsigned)(p ? std::min<int64_t>(need, NORM_PARTIALS) : need);
                         rows_bwd_kernel<T, tpr, maxc, decltype(DX)::value != 0, p><<<grid, 256, p ? (rpb - 1) * 2 * a.D * sizeof(float) : 0, s>>>(
                             (const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, (const T*)a.res, a.ldr, a.M, a.D, a.mean, a.rstd, a.gamma, (T*)a.dx, a.lddx,
                             a.partial);
                         if (p) rows = (int)grid;
                       };
                       if (!params) go(RowC<1>{}, RowC<0>{});
                       else if (a.dx) go(RowC<1>{}, RowC<1>{});
                       else go(RowC<0>{}, RowC<1>{});
                     });
    if (!vec) {
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
