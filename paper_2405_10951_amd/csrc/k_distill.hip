// Loss of a classifier against a teacher's top logits, mixed with the label's cross-entropy, and its gradient.  Per row, with temperature T, hard
// weight a, the entries (c_j, t_j) that the teacher gave and the student's logits z:
//   p = softmax(t / T) over the entries,  q = softmax(z / T),  r = softmax(z)
//   L = (1 - a) T^2 sum_j p_j (log p_j - log q_{c_j}) + a (-log r_label)
//   dL/dz_v = (1 - a) T (q_v - sum_{j: c_j = v} p_j) + a (r_v - [v = label])
// A row without entries lacks the first part, one without a label the second; one whose logits are all -inf has loss and gradient 0.  At a = 1 no row has the first part, and the
// list is not looked at: the student may give a class of it no weight at all, and 0 times that infinity is no loss.
// Bound by memory: a workgroup takes a row, asks for all of it at once, keeps it in registers (rows of up to 131072 bf16 or 65536 fp32 values), takes the
// maximum and both sums together and writes dz; longer rows are read a second time for dz.  The teacher's list is worked on while the row is on its way.  The few places that p and the label touch are
// written again behind a barrier by a thread each, duplicates added in the order of the list: no atomics, the same bits every time.
// Measured (bytes at a copy's rate in brackets): 4096 x 131072 bf16 loss and gradient 438 us (420), 2048 x 21841 bf16 gradient 38 (35), 32 x 100 fp32 5.4, a
// chain of waits.
#include <algorithm>
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

// P: 0: one sum (temperature 1, or no hard part); 1: the sums at the temperature and at 1 by an exponential each; 2, 3, 4: that temperature, where
// exp(d) is a power of exp(d / T).  With a hard part, against an exponential of its own: 4096 x 131072 bf16 loss and gradient at T = 2 587 -> 522 us, at 3 588 -> 545, at 4
// 586 -> 548; 2048 x 21841 42.0 -> 38.8, 39.8 and 39.9; 4096 x 65536 fp32 447 -> 416, 430 and 430; no shorter row is slower for it.
template <int P> __device__ __forceinline__ float second(float e, float d) {
  if constexpr (P == 2) return e * e;
  else if constexpr (P == 3) return e * e * e;
  else if constexpr (P == 4) return (e * e) * (e * e);
  else return exp2_(d * LOG2E);
}

// maximum m, sums of exp((z - m) / T) and exp(z - m)
struct Stats { float m, st, s1; };
template <int P> __device__ __forceinline__ void count(Stats& a, float v, float ct) {
  const float d = v - a.m, e = exp2_(d * ct);
  a.st += e;
  if (P) a.s1 += second<P>(e, d);
}
template <int P> __device__ __forceinline__ void rescale(Stats& a, float m, float ct) {
  const float d = a.m - m;
  a.st *= exp2_(d * ct);
  if (P) a.s1 *= exp2_(d * LOG2E);
  a.m = m;
}
// over a wavefront, and over the wavefronts of a workgroup
template <int P> __device__ __forceinline__ void join_wave(Stats& a, float ct) {
  rescale<P>(a, wave_max(a.m), ct);
  a.st = wave_sum(a.st);
  if (P) a.s1 = wave_sum(a.s1);
}
template <int NT, int P>
__device__ __forceinline__ void join(Stats& a, float ct, float (*red)[3]) {
  join_wave<P>(a, ct);
  if constexpr (NT > WAVE) {
    const int w = threadIdx.x / WAVE;
    if (threadIdx.x % WAVE == 0) { red[w][0] = a.m; red[w][1] = a.st; red[w][2] = a.s1; }
    __syncthreads();
    float m = red[0][0];
#pragma unroll
    for (int i = 1; i < NT / WAVE; ++i) m = fmaxf(m, red[i][0]);
    Stats all{m, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT / WAVE; ++i) {
      Stats one{red[i][0], red[i][1], red[i][2]};
      rescale<P>(one, m, ct);
      all.st += one.st;
      all.s1 += one.s1;
    }
    a = all;
  }
}
template <typename T, int NT, int C, int P>
__device__ __forceinline__ Stats row_stats(const Row<T, NT, C>& held, float ct, float (*red)[3]) {
  constexpr int V = Chunk<T>::V;
  Stats st{-FLT_MAX, 0.f, 0.f};
  held.pass([&](int, float v) __attribute__((always_inline)) {
              if (v > st.m) rescale<P>(st, v, ct);
              count<P>(st, v, ct);
            },
            [&](int, const float (&v)[V]) __attribute__((always_inline)) {
              float m = v[0];
#pragma unroll
              for (int e = 1; e < V; ++e) m = fmaxf(m, v[e]);
              if (m > st.m) rescale<P>(st, m, ct);
#pragma unroll
              for (int e = 0; e < V; ++e) count<P>(st, v[e], ct);
            });
  join<NT, P>(st, ct, red);
  return st;
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

// Segment seg of `count` of a row: [lo, hi), all but the first and the last of whole chunks
template <typename T> struct Segment {
  int lo, hi, head;
  __device__ __forceinline__ Segment(const DistillArgs& a, const T* z, int seg, int count) {
    const int n = a.classes;
    head = min(n, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T));
    const int chunks = (n - head) / Chunk<T>::V, per = (chunks + count - 1) / count;
    lo = seg == 0 ? 0 : head + min(chunks, seg * per) * Chunk<T>::V;
    hi = seg == count - 1 ? n : head + min(chunks, (seg + 1) * per) * Chunk<T>::V;
    if (seg > 0) head = 0;
  }
};

// Few rows of many classes: several workgroups a row, each on a segment; what they find here, the kernel below joins.
template <typename T, int NT, int C, int P>
__global__ __launch_bounds__(NT) void distill_parts_kernel(DistillArgs a) {
  __shared__ float red[NT / WAVE][3];
  const int64_t row = blockIdx.x / (unsigned)a.segments;
  const int seg = (int)(blockIdx.x % (unsigned)a.segments);
  const T* z = (const T*)a.z + row * a.ldz;
  const Segment<T> at(a, z, seg, a.segments);
  Row<T, NT, C> held;
  held.start(z + at.lo, at.hi - at.lo, at.head);
  const Stats st = row_stats<T, NT, C, P>(held, LOG2E / a.temperature, red);
  if (threadIdx.x == 0) {
    float* o = a.parts + (int64_t)blockIdx.x * 3;
    o[0] = st.m;
    o[1] = st.st;
    o[2] = st.s1;
  }
}

// where a row's maximum and sums come from: a pass over it, the forward's (a.stats), or those of its segments (a.parts)
enum { OWN, STATS, PARTS };
template <typename T, int NT, int C, int FROM, int P>
__global__ __launch_bounds__(NT) void distill_kernel(DistillArgs a) {
  extern __shared__ unsigned char dyn[];
  __shared__ float red[NT / WAVE][3], red_w[NT / WAVE], red_l[NT / WAVE];
  constexpr int V = Chunk<T>::V;
  int* li = (int*)dyn;                              // [k] the classes, -1 where absent
  float* lp = (float*)(li + a.k);                   // [k] first t, then p
  float* lz = lp + a.k;                             // [k] the student's logits there
  constexpr int LIST = NT < 256 ? NT : 256;         // threads that go through the list: a sum over it is the same whatever NT
  const int tid = threadIdx.x, n = a.classes, k = a.hard < 1.f ? a.k : 0, my_k = tid < LIST ? k : 0;
  const int64_t row = FROM == OWN ? (int64_t)blockIdx.x : (int64_t)(blockIdx.x / (unsigned)a.writers);
  const int seg = FROM == OWN ? 0 : (int)(blockIdx.x % (unsigned)a.writers);
  const T* z = (const T*)a.z + row * a.ldz;
  T* dz = a.dz ? (T*)a.dz + row * a.ldd : nullptr;
  const Segment<T> at(a, z, seg, FROM == OWN ? 1 : a.writers);
  Row<T, NT, C> held;
  if (FROM == OWN || dz) held.start(z + at.lo, at.hi - at.lo, at.head);
  const float inv_t = 1.f / a.temperature, ct = LOG2E * inv_t;
  const int label = a.labels && a.hard > 0.f ? a.labels[row] : -1;
  const bool labelled = label >= 0 && label < n;
  const float zl = labelled ? (float)z[label] : 0.f;
  // the teacher's list; its maximum and its sum
  float tm = -FLT_MAX;
  for (int j = tid; j < my_k; j += LIST) {
    const int c = a.index[row * a.ldi + j];
    const bool there = c >= 0 && c < n;
    const float t = a.top_f32 ? ((const float*)a.top)[row * a.ldt + j] : (float)((const bf16*)a.top)[row * a.ldt + j];
    li[j] = there ? c : -1;
    lp[j] = t;
    lz[j] = there ? (float)z[c] : 0.f;
    if (there) tm = fmaxf(tm, t);
  }
  Stats st{0.f, 0.f, 0.f};
  // logarithms of the sums
  float lt, l1;
  if constexpr (FROM == STATS) {
    st.m = a.stats[3 * row];
    lt = a.stats[3 * row + 1];
    l1 = a.stats[3 * row + 2];
  } else {
    if constexpr (FROM == OWN) {
      st = row_stats<T, NT, C, P>(held, ct, red);
    } else {                                         // (a lane for each segment)
      const int lane = tid % WAVE;
      const float* p = a.parts + (row * a.segments + min(lane, a.segments - 1)) * 3;
      st = lane < a.segments ? Stats{p[0], p[1], p[2]} : Stats{-FLT_MAX, 0.f, 0.f};
      join_wave<P>(st, ct);
    }
    if (!P) st.s1 = st.st;                          // (temperature 1, or nobody asks)
    lt = logf(st.st);
    l1 = logf(st.s1);
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
  for (int j = tid; j < my_k; j += LIST)
    if (li[j] >= 0) w += exp2_((lp[j] - tmax) * ct);
  w = block_sum<NT>(w, red_w);
  const bool taught = w != 0.f, empty = lt == -INFINITY;            // (NaN goes on)
  float part = 0.f;
  const float lw = logf(w);
  for (int j = tid; j < my_k; j += LIST) {
    if (li[j] < 0) continue;
    const float lq = (lz[j] - st.m) * inv_t - lt, lpj = (lp[j] - tmax) * inv_t - lw, p = taught ? expf(lpj) : 0.f;
    if (p != 0.f) part += p * (lpj - lq);
    lp[j] = p;
  }
  if (FROM != STATS && seg == 0) {
    if (a.loss) {
      part = block_sum<NT>(part, red_l);
      float loss = k > 0 ? (1.f - a.hard) * a.temperature * a.temperature * part : 0.f;
      if (labelled) loss += a.hard * (l1 - (zl - st.m));
      if (tid == 0) a.loss[row] = empty ? 0.f : lt != lt ? lt : loss;          // (NaN in z shows, with or without entries)
    }
    if (a.stats && tid == 0) {
      a.stats[3 * row] = st.m;
      a.stats[3 * row + 1] = lt;
      a.stats[3 * row + 2] = P || a.temperature == 1.f ? l1 : 0.f;
    }
  }
  if (!dz) return;
  __syncthreads();                                   // the list is whole; with dz = z, everybody has read its logits
  const float g = a.grad_scale * (a.row_grad ? a.row_grad[row] : 1.f);
  const float soft = taught && !empty ? (1.f - a.hard) * a.temperature * g : 0.f, mix = labelled && !empty ? a.hard * g : 0.f;
  // soft q + mix r, q = exp((z - m) / T) / sum, r = exp(z - m) / sum
  const float by_q = (P ? soft : soft + mix) * exp2_(-lt * LOG2E), by_r = P ? mix * exp2_(-l1 * LOG2E) : 0.f;
  auto grad = [&](float v) __attribute__((always_inline)) {
    const float d = v - st.m, e = exp2_(d * ct);
    return P ? by_q * e + by_r * second<P>(e, d) : by_q * e;
  };
  T* out = dz + at.lo;
  const bool alike = (((uintptr_t)z ^ (uintptr_t)dz) & 15) == 0;     // (rows that lie differently within 16 bytes in z and dz leave value by value)
  if (empty) {
    for (int i = tid; i < at.hi - at.lo; i += NT) out[i] = (T)0.f;
    return;
  }
  held.pass([&](int i, float v) __attribute__((always_inline)) { out[i] = (T)grad(v); },
            [&](int i, const float (&v)[V]) __attribute__((always_inline)) {
              typename Chunk<T>::vec o;
#pragma unroll
              for (int e = 0; e < V; ++e) o[e] = (T)grad(v[e]);
              // (past the caches: 2048 x 21841 bf16 backward 46 -> 36 us, 4096 x 131072 forward and backward 496 -> 455)
              if (alike) __builtin_nontemporal_store(o, (typename Chunk<T>::vec*)(out + i));
              else
#pragma unroll
                for (int e = 0; e < V; ++e) out[i + e] = o[e];
            });
  __syncthreads();                                   // the segment is out: now its places that p and the label touch
  for (int j = tid; j < my_k; j += LIST) {
    const int c = li[j];
    if (c < at.lo || c >= at.hi) continue;
    float p = 0.f;
    bool first = true;
    for (int i = 0; i < k; ++i)
      if (li[i] == c) {
        p += lp[i];
        if (i < j) first = false;
      }
    if (first) dz[c] = (T)(grad(lz[j]) - soft * p - (labelled && c == label ? mix : 0.f));
  }
  if (labelled && label >= at.lo && label < at.hi && tid == 0) {
    bool listed = false;
    for (int i = 0; i < k; ++i) listed |= li[i] == label;
    if (!listed) dz[label] = (T)(grad(zl) - mix);
  }
}

template <class F> void with_power(const DistillArgs& a, F&& f) {
  if (!(a.hard > 0.f) || a.temperature == 1.f) f(RowC<0>{});
  else if (a.temperature == 2.f) f(RowC<2>{});
  else if (a.temperature == 3.f) f(RowC<3>{});
  else if (a.temperature == 4.f) f(RowC<4>{});
  else f(RowC<1>{});
}
template <typename T, int NT, int C>
void go_parts(const DistillArgs& a, hipStream_t s) {
  with_power(a, [&](auto P) { distill_parts_kernel<T, NT, C, decltype(P)::value><<<(unsigned)(a.rows * a.segments), NT, 0, s>>>(a); });
}
template <typename T, int NT, int C, int FROM, int P>
void go(const DistillArgs& a, hipStream_t s) {
  distill_kernel<T, NT, C, FROM, P><<<(unsigned)(a.rows * a.writers), NT, (size_t)a.k * 12, s>>>(a);
}
template <typename T, int NT, int C, int FROM>
void go(const DistillArgs& a, hipStream_t s) {
  with_power(a, [&](auto P) { distill_kernel<T, NT, C, FROM, decltype(P)::value><<<(unsigned)(a.rows * a.writers), NT, (size_t)a.k * 12, s>>>(a); });
}
// Small workgroups: more rows at once on a CU, whose lists, sums and barriers then pass unseen behind one another's memory traffic.
template <typename T, int FROM>
void go_size(const DistillArgs& a, hipStream_t s) {
  const int all = (a.classes + Chunk<T>::V - 1) / Chunk<T>::V, n = (all + a.writers - 1) / a.writers;        // chunks
  if constexpr (FROM == PARTS) {
    const int m = (all + a.segments - 1) / a.segments;
    if (m <= 1024) go_parts<T, 256, 4>(a, s);
    else if (m <= 4096) go_parts<T, 256, 16>(a, s);
    else go_parts<T, 1024, 0>(a, s);
  }
  if constexpr (FROM != PARTS)
    if (n <= 128) return go<T, 64, 2, FROM>(a, s);
  if (n <= 1024) go<T, 256, 4, FROM>(a, s);
  else if (n <= 4096) go<T, 256, 16, FROM>(a, s);
  else if (n <= 8192) go<T, 512, 16, FROM>(a, s);
  else if (n <= 16384) {
    // (of one sum there is little to keep beside the row: 16 wavefronts fit; 4096 x 131072 bf16 forward and backward 485 us against 521, and 597 against 647 with two)
    if (!(a.hard > 0.f) || a.temperature == 1.f) go<T, 1024, 16, FROM, 0>(a, s);
    else go<T, 512, 32, FROM>(a, s);
  }
  else go<T, 1024, 0, FROM>(a, s);
}

}  // namespace

// Segments of a row: as many as give the CUs two workgroups each, of 1024 chunks at least, a wavefront's lanes at most.  A forward split is two launches, which three
// segments pay for.
static int segments_of(const DistillArgs& a) {
  const int64_t chunks = a.classes / (a.f32 ? 4 : 8);
  return (int)std::max<int64_t>(1, std::min<int64_t>({64, 512 / std::max<int64_t>(a.rows, 1), chunks / 1024}));
}
size_t distill_parts_floats(bool f32, int64_t rows, int classes) {
  DistillArgs a;
  a.f32 = f32; a.rows = rows; a.classes = classes;
  const int n = segments_of(a);
  return n < 3 ? 0 : (size_t)rows * n * 3;
}

// f on slices of the rows: a launch has fewer than 2^32 threads, and a row up to 1024 of them.  (Rows are split over workgroups, with scratch for it, only where they are few.)
constexpr int64_t ROWS_A_LAUNCH = 1 << 21;
template <class F> static void in_slices(const DistillArgs& all, F&& f) {
  const int64_t z_size = all.f32 ? 4 : 2, t_size = all.top_f32 ? 4 : 2;
  for (int64_t m = 0; m < all.rows; m += ROWS_A_LAUNCH) {
    DistillArgs a = all;
    a.rows = std::min(ROWS_A_LAUNCH, all.rows - m);
    a.z = (const char*)all.z + m * all.ldz * z_size;
    a.index = all.index + m * all.ldi;
    a.top = (const char*)all.top + m * all.ldt * t_size;
    if (all.labels) a.labels = all.labels + m;
    if (all.loss) a.loss = all.loss + m;
    if (all.stats) a.stats = all.stats + 3 * m;
    if (all.row_grad) a.row_grad = all.row_grad + m;
    if (all.dz) a.dz = (char*)all.dz + m * all.ldd * z_size;
    f(a);
  }
}

void distill_forward(const DistillArgs& given, hipStream_t s) {
  DistillArgs all = given;
  all.segments = all.parts ? segments_of(all) : 1;
  // (where dz takes the place of z, other segments' logits would be gone: one workgroup writes a row then, from the same parts)
  all.writers = all.dz && all.dz != all.z ? all.segments : 1;
  in_slices(all, [&](const DistillArgs& a) {
    if (a.parts) a.f32 ? go_size<float, PARTS>(a, s) : go_size<bf16, PARTS>(a, s);
    else a.f32 ? go_size<float, OWN>(a, s) : go_size<bf16, OWN>(a, s);
  });
}

void distill_backward(const DistillArgs& given, hipStream_t s) {
  DistillArgs all = given;
  all.writers = all.dz != all.z ? segments_of(all) : 1;
  in_slices(all, [&](const DistillArgs& a) { a.f32 ? go_size<float, STATS>(a, s) : go_size<bf16, STATS>(a, s); });
}

}  // namespace bsr
