// Loss of a classifier against a teacher's top logits, mixed with the label's cross-entropy, and its gradient.  Per row, with temperature T, hard
// weight a, the entries (c_j, t_j) that the teacher gave and the student's logits z:
//   p = softmax(t / T) over the entries,  q = softmax(z / T),  r = softmax(z)
//   L = (1 - a) T^2 sum_j p_j (log p_j - log q_{c_j}) + a (-log r_label)
//   dL/dz_v = (1 - a) T (q_v - sum_{j: c_j = v} p_j) + a (r_v - [v = label])
// A row without entries lacks the first part, one without a label the second; one whose logits are all -inf has loss and gradient 0.
// Bound by memory: a workgroup takes a row, asks for all of it at once, keeps it in registers (rows of up to 131072 bf16 or 65536 fp32 values), takes the
// maximum and both sums together and writes dz; longer rows are read a second time for dz.  The teacher's list is worked on while the row is on its way.  The few places that p and the label touch are
// written again behind a barrier by a thread each, duplicates added in the order of the list: no atomics, the same bits every time.
#include <cfloat>

#include "distill.h"
#include "rowops.h"

namespace bsr {

namespace {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// A row of n values as a workgroup of NT threads goes over it: single values up to the first 16-byte boundary (head of them), whole chunks, single
// values.  C > 0: a thread's C chunks and its single values stay in registers; C = 0: the row is read anew at every pass.
template <typename T, int NT, int C> struct Row {
  static constexpr int V = Chunk<T>::V, MOST = C * NT * V;       // longest row it holds, but for its ends
  typedef typename Chunk<T>::vec vec;
  const T* p;
  int n, head, chunks;
  vec raw[C > 0 ? C : 1];
  float first, last;
  __device__ __forceinline__ void start(const T* p_, int n_, int head_) {
    p = p_; n = n_; head = head_; chunks = (n - head) / V;
    if constexpr (C > 0) {
      const int t = threadIdx.x;
      if (chunks > 0)
#pragma unroll
        for (int i = 0; i < C; ++i) raw[i] = *(const vec*)(p + head + min(t + i * NT, chunks - 1) * (int64_t)V);
      first = t < head ? (float)p[t] : 0.f;
      last = head + chunks * V + t < n ? (float)p[head + chunks * V + t] : 0.f;
    }
  }
  template <class One, class Many> __device__ __forceinline__ void pass(One&& one, Many&& many) const {
    const int t = threadIdx.x;
    if constexpr (C > 0) {                             // (both ends are shorter than a chunk, and NT is not)
      if (t < head) one(t, first);
#pragma unroll
      for (int i = 0; i < C; ++i)
        if (t + i * NT < chunks) {
          float v[V];
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = (float)raw[i][e];
          many(head + (t + i * NT) * V, v);
        }
      if (head + chunks * V + t < n) one(head + chunks * V + t, last);
    } else {
      for (int i = t; i < head; i += NT) one(i, (float)p[i]);
      for (int c = t; c < chunks; c += NT) {
        const vec r = *(const vec*)(p + head + c * (int64_t)V);
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)r[e];
        many(head + c * V, v);
      }
      for (int i = head + chunks * V + t; i < n; i += NT) one(i, (float)p[i]);
    }
  }
};

// maximum m, sums of 2^((z - m) ct) and 2^((z - m) c1)
struct Stats { float m, st, s1; };
template <bool TWO> __device__ __forceinline__ void rescale(Stats& a, float m, float ct, float c1) {
  const float d = a.m - m;
  a.st *= exp2_(d * ct);
  if (TWO) a.s1 *= exp2_(d * c1);
  a.m = m;
}
template <int NT, bool TWO>
__device__ __forceinline__ void join(Stats& a, float ct, float c1, float (*red)[3]) {
  rescale<TWO>(a, wave_max(a.m), ct, c1);
  a.st = wave_sum(a.st);
  if (TWO) a.s1 = wave_sum(a.s1);
  if constexpr (NT > WAVE) {
    const int w = threadIdx.x / WAVE;
    if (threadIdx.x % WAVE == 0) { red[w][0] = a.m; red[w][1] = a.st; red[w][2] = a.s1; }
    __syncthreads();
    float m = red[0][0];
#pragma unroll
    for (int i = 1; i < NT / WAVE; ++i) m = fmaxf(m, red[i][0]);
    float st = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < NT / WAVE; ++i) {
      const float d = red[i][0] - m;
      st += red[i][1] * exp2_(d * ct);
      if (TWO) s1 += red[i][2] * exp2_(d * c1);
    }
    a = Stats{m, st, s1};
  }
}

// sum over the workgroup, in every thread
template <int NT> __device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (NT > WAVE) {
    if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < NT / WAVE; ++i) v += red[i];
  }
  return v;
}

// BWD: the statistics come from a.stats instead of a pass.  TWO: temperature other than 1 and a hard part, two sums
template <typename T, int NT, int C, bool BWD, bool TWO>
__global__ __launch_bounds__(NT) void distill_kernel(DistillArgs a) {
  extern __shared__ unsigned char dyn[];
  __shared__ float red[NT / WAVE][3], red_w[NT / WAVE], red_l[NT / WAVE];
  int* li = (int*)dyn;                              // [k] the classes, -1 where absent
  float* lp = (float*)(li + a.k);                   // [k] first t, then p
  float* lz = lp + a.k;                             // [k] the student's logits there
  const int tid = threadIdx.x, n = a.classes;
  const int64_t row = blockIdx.x;
  const T* z = (const T*)a.z + row * a.ldz;
  T* dz = a.dz ? (T*)a.dz + row * a.ldd : nullptr;
  constexpr int V = Chunk<T>::V;
  // (rows that lie differently within 16 bytes in z and dz go value by value: C = 0)
  int head = min(n, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T));
  if (C == 0 && dz && (((uintptr_t)z ^ (uintptr_t)dz) & 15)) head = n;
  Row<T, NT, C> held;
  held.start(z, n, head);
  const float inv_t = 1.f / a.temperature, ct = LOG2E * inv_t, c1 = LOG2E;
  const int label = a.labels && a.hard > 0.f ? a.labels[row] : -1;
  const bool labelled = label >= 0 && label < n;
  const float zl = labelled ? (float)z[label] : 0.f;
  // the teacher's list; its maximum and its sum
  float tm = -FLT_MAX;
  for (int j = tid; j < a.k; j += NT) {
    const int c = a.index[row * a.ldi + j];
    const bool there = c >= 0 && c < n;
    const float t = a.top_f32 ? ((const float*)a.top)[row * a.ldt + j] : (float)((const bf16*)a.top)[row * a.ldt + j];
    li[j] = there ? c : -1;
    lp[j] = t;
    lz[j] = there ? (float)z[c] : 0.f;
    if (there) tm = fmaxf(tm, t);
  }
  Stats st{-FLT_MAX, 0.f, 0.f};
  if constexpr (!BWD) {
    held.pass([&](int, float v) __attribute__((always_inline)) {
                      if (v > st.m) rescale<TWO>(st, v, ct, c1);
                      st.st += exp2_((v - st.m) * ct);
                      if (TWO) st.s1 += exp2_((v - st.m) * c1);
                    },
                    [&](int, const float (&v)[V]) __attribute__((always_inline)) {
                      float m = v[0];
#pragma unroll
                      for (int e = 1; e < V; ++e) m = fmaxf(m, v[e]);
                      if (m > st.m) rescale<TWO>(st, m, ct, c1);
#pragma unroll
                      for (int e = 0; e < V; ++e) {
                        st.st += exp2_((v[e] - st.m) * ct);
                        if (TWO) st.s1 += exp2_((v[e] - st.m) * c1);
                      }
                    });
    join<NT, TWO>(st, ct, c1, red);
    if (!TWO) st.s1 = st.st;                        // (temperature 1, or nobody asks)
  }
  // p in place of t
  float tmax = wave_max(tm);
  if constexpr (NT > WAVE) {
    if (tid % WAVE == 0) red_w[tid / WAVE] = tmax;
    __syncthreads();
    tmax = red_w[0];
#pragma unroll
    for (int i = 1; i < NT / WAVE; ++i) tmax = fmaxf(tmax, red_w[i]);
    __syncthreads();
  }
  float w = 0.f;
  for (int j = tid; j < a.k; j += NT)
    if (li[j] >= 0) w += exp2_((lp[j] - tmax) * ct);
  w = block_sum<NT>(w, red_w);
  const bool taught = w != 0.f;                      // (NaN goes on)
  // log-sum-exp at the temperature and at 1, as (m, log of the sum): differences to m first, they are small
  float lt, l1;
  if (BWD) {
    st.m = a.stats[3 * row];
    lt = a.stats[3 * row + 1];
    l1 = a.stats[3 * row + 2];
  } else {
    lt = logf(st.st);
    l1 = logf(st.s1);
  }
  const bool empty = lt == -INFINITY;
  float part = 0.f;
  const float lw = logf(w);
  for (int j = tid; j < a.k; j += NT) {
    if (li[j] < 0) continue;
    const float lq = (lz[j] - st.m) * inv_t - lt, lpj = (lp[j] - tmax) * inv_t - lw, p = taught ? expf(lpj) : 0.f;
    if (p != 0.f) part += p * (lpj - lq);
    lp[j] = p;
  }
  if constexpr (!BWD) {
    if (a.loss) {
      part = block_sum<NT>(part, red_l);
      float loss = (1.f - a.hard) * a.temperature * a.temperature * part;
      if (labelled) loss += a.hard * (l1 - (zl - st.m));
      if (tid == 0) a.loss[row] = empty ? 0.f : loss;
    }
    if (a.stats && tid == 0) {
      a.stats[3 * row] = st.m;
      a.stats[3 * row + 1] = lt;
      a.stats[3 * row + 2] = TWO || a.temperature == 1.f ? l1 : 0.f;
    }
  }
  if (!dz) return;
  __syncthreads();                                   // the list is whole; with dz = z, everybody has read its logits
  const float g = a.grad_scale * (a.row_grad ? a.row_grad[row] : 1.f);
  const float soft = taught && !empty ? (1.f - a.hard) * a.temperature * g : 0.f, mix = labelled && !empty ? a.hard * g : 0.f;
  const float bt = lt * LOG2E, b1 = l1 * LOG2E;
  auto grad = [&](float v) __attribute__((always_inline)) {
    const float d = v - st.m;
    if (TWO) return soft * exp2_(d * ct - bt) + mix * exp2_(d * c1 - b1);
    return (soft + mix) * exp2_(d * ct - bt);
  };
  if (empty) {
    for (int i = tid; i < n; i += NT) dz[i] = (T)0.f;
    return;
  }
  held.pass([&](int i, float v) __attribute__((always_inline)) { dz[i] = (T)grad(v); },
                  [&](int i, const float (&v)[V]) __attribute__((always_inline)) {
                    typename Chunk<T>::vec o;
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] = (T)grad(v[e]);
                    *(typename Chunk<T>::vec*)(dz + i) = o;
                  });
  __syncthreads();                                   // the row is out: now the places that p and the label touch
  bool label_listed = false;
  for (int j = tid; j < a.k; j += NT) {
    const int c = li[j];
    if (c < 0) continue;
    float p = 0.f;
    bool first = true;
    for (int i = 0; i < a.k; ++i)
      if (li[i] == c) {
        p += lp[i];
        if (i < j) first = false;
      }
    if (first) dz[c] = (T)(grad(lz[j]) - soft * p - (labelled && c == label ? mix : 0.f));
  }
  if (labelled && tid == 0) {
    for (int i = 0; i < a.k; ++i) label_listed |= li[i] == label;
    if (!label_listed) dz[label] = (T)(grad(zl) - mix);
  }
}

template <typename T, int NT, int C, bool BWD>
void go(const DistillArgs& a, hipStream_t s) {
  const size_t lds = (size_t)a.k * 12;
  if (a.hard > 0.f && a.temperature != 1.f) distill_kernel<T, NT, C, BWD, true><<<(unsigned)a.rows, NT, lds, s>>>(a);
  else distill_kernel<T, NT, C, BWD, false><<<(unsigned)a.rows, NT, lds, s>>>(a);
}
// Whether every row lies within 16 bytes in dz as it does in z
bool alike(const DistillArgs& a) {
  const int64_t e = a.f32 ? 4 : 2;
  return !a.dz || ((((uintptr_t)a.z ^ (uintptr_t)a.dz) & 15) == 0 && (a.rows == 1 || (a.ldz - a.ldd) * e % 16 == 0));
}
// Small workgroups: more rows at once on a CU, whose lists, sums and barriers then pass unseen behind one another's memory traffic.
template <typename T, bool BWD>
void go_size(const DistillArgs& a, hipStream_t s) {
  const int n = alike(a) ? (a.classes + Chunk<T>::V - 1) / Chunk<T>::V : INT32_MAX;        // chunks
  if (n <= 128) go<T, 64, 2, BWD>(a, s);
  else if (n <= 1024) go<T, 256, 4, BWD>(a, s);
  else if (n <= 4096) go<T, 256, 16, BWD>(a, s);
  else if (n <= 8192) go<T, 1024, 8, BWD>(a, s);
  else if (n <= 16384) go<T, 1024, 16, BWD>(a, s);
  else if (a.classes <= 1024) go<T, 64, 0, BWD>(a, s);
  else go<T, 1024, 0, BWD>(a, s);
}

}  // namespace

void distill_forward(const DistillArgs& a, hipStream_t s) {
  if (a.rows <= 0) return;
  if (a.f32) go_size<float, false>(a, s);
  else go_size<bf16, false>(a, s);
}

void distill_backward(const DistillArgs& a, hipStream_t s) {
  if (a.rows <= 0) return;
  if (a.f32) go_size<float, true>(a, s);
  else go_size<bf16, true>(a, s);
}

}  // namespace bsr
