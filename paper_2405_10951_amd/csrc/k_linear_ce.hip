// Softmax cross-entropy of a linear layer over many classes, and its gradients, without keeping the logits:
//   z = x w^T + b;   loss = log sum exp z - z_label;   G = softmax(z) - onehot(label);   dx = g G w;   dw = G^T (g x);   db = G^T g
// Forward: tiles of z stay in the accumulators of the product; a tile leaves each row's maximum and its sum of exp(z - maximum), and a second kernel joins the tiles of a row.
// Backward: z is made again, a piece of the classes at a time; the tile's end turns it into G and leaves that as it lies and transposed, so that both products behind it
// contract over contiguous memory like the first.  What they need transposed beside it (x once, the piece's rows of w) is transposed in a pass of its own.
//
// Numbers.  bf16 x and w are multiplied as they are and added in fp32.  G is kept in fp16, not bf16: it lies within -1 .. 1, and scaled by 2^14 its values keep 11 bits down to
// 2^-28 and are off by 2^-39 at most below, where bf16 would keep 8; x and w join it in fp16, each feature (a row of the transposed operand) scaled by a power of two so that its
// largest value lies in 2^14 .. 2^15, which is exact for bf16 values down to 2^-29 of the feature's largest.  The matrix instructions take both types at one rate.  fp32 operands are two fp16 terms each,
// h + l with h = fp16(v), l = fp16(v - h), off by 2^-22 of the value, and the products h h, h l, l h, added in fp32, are three runs over the contraction index.
// The row's weight g scales x in dw and the result in dx; rows whose label is absent or whose weight is 0 have G = 0 and, in the transposed x, zeros.
#include <algorithm>

#include "gemm_common.h"
#include "linear_ce.h"
#include "rowops.h"

namespace bsr {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16;
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int BK = 64;
constexpr int G_SHIFT = 14;                        // G is kept times 2^14

// ------------------------------------------------------------------------------------------ the products
enum Mode { STATS, GRAD, OUT };

// C(m,n) = sum_k A(m,k) B(n,k): rows of 64-element k-tiles, whole ones, 16-byte aligned.  SEG = 3: two terms each, ta and tb elements apart, products h h, h l, l h.
struct CeGemm {
  const void *A = nullptr, *B = nullptr;
  int64_t lda = 0, ldb = 0, ta = 0, tb = 0;
  int M = 0, N = 0, nk = 0;                        // nk: k-tiles of a term
  int splits = 1, per = 0;                         // workgroups over the k-tiles of a tile, k-tiles (of all terms) of each
  const int *ea = nullptr, *eb = nullptr;          // powers of two of A's and B's rows, null: 0
  // STATS, GRAD: m is a token, n a class of the piece that begins at class v0
  const float* bias = nullptr;                     // of the piece
  const int32_t* labels = nullptr;
  int v0 = 0, classes = 0;                         // classes of the whole layer
  float2* parts = nullptr; float* zlabel = nullptr;                        // STATS: [tile of classes][M] maximum and sum; [M]
  const float2* stats = nullptr; const float* row_grad = nullptr;          // GRAD: [M] maximum, log of the sum; weights or null
  f16 *G = nullptr, *GT = nullptr;                 // GRAD: [terms][M][ldg], [terms][N][ldgt], columns behind the last one zero; null: not wanted
  int64_t ldg = 0, ldgt = 0, tg = 0, tgt = 0;
  float* dbp = nullptr;                            // GRAD: [tile of tokens][N] sums of g G; null: not wanted
  // OUT
  float* part = nullptr; int64_t ldp = 0, tp = 0; bool add = false;        // [split][M][ldp] fp32 (of what was there as well)
  void* out = nullptr; int64_t ldo = 0; bool out_f32 = false, out_vec = false;   // or the result itself: times scale and, where given, its row's weight
  float scale = 1.f; const float* row_scale = nullptr;
};

template <int BM_, int BN_, int WM_, int WN_, int NST_> struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NST = NST_, NT = WM * WN * 64;
  static constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 32, NI = TN / 32;
  static constexpr size_t stages = (size_t)NST * (BM + BN) * 128;
  static constexpr int LDT = TM * 2 + 16, LDR = TN * 2 + 16, LDF = TN * 4 + 16;           // patch rows in bytes
  static constexpr int patch = TN * LDT > 32 * LDF ? TN * LDT : 32 * LDF;                  // of a wavefront
  static constexpr size_t lds = stages > (size_t)patch * WM * WN ? stages : (size_t)patch * WM * WN;
};
typedef Shape<256, 256, 2, 4, 2> Large;
typedef Shape<128, 128, 2, 4, 3> Small;
typedef Shape<32, 256, 1, 4, 4> Few;

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// tiles band after band of eight row tiles, row tile fastest: what an XCD works on at a time shares rows of A and of B
constexpr int BAND = 8;
__device__ __forceinline__ void tile_at(int t, int mt, int nt, int& m, int& n) {
  const int band = t / (BAND * nt), in = t - band * BAND * nt, rows = min(BAND, mt - band * BAND);
  n = in / rows;
  m = band * BAND + in - n * rows;
}

// The k-loop is the one of the step's products (operands straight into LDS, one barrier a k-tile, every matrix instruction followed by at most one
// fragment read or a few loads, the order pinned): accumulators hold transposed 32 x 32 tiles, element r of acc[mi][ni] is row mi 32 + lane % 32, column ni 32 + 8 (r / 4) + 4 (lane / 32) + r % 4.
template <class S, bool F16, int SEG>
__device__ __forceinline__ void multiply(const CeGemm& g, int m0, int n0, int kt0, int nk, unsigned char* smem, f32x16 (&acc)[S::MI][S::NI]) {
  constexpr int BM = S::BM, WN = S::WN, NST = S::NST, TM = S::TM, TN = S::TN, MI = S::MI, NI = S::NI, NMF = MI * NI, NFR = MI + NI;
  constexpr int RPI = S::NT / 8, AL = BM / RPI, BL = S::BN / RPI, LPT = AL + BL, STAGE = (BM + S::BN) * 128;
  static_assert(BM % RPI == 0 && S::BN % RPI == 0 && RPI % 16 == 0, "a load instruction covers whole groups of 16 rows");
  static_assert(NST >= 2 && NST <= 4 && (NST - 1) * LPT <= 60 && NMF >= 2, "vmcnt has 6 bits");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const f16* __restrict__ A = (const f16*)g.A + (int64_t)m0 * g.lda;
  const f16* __restrict__ B = (const f16*)g.B + (int64_t)n0 * g.ldb;
  // rows past the last one repeat it: they only feed accumulators that count for nothing
  const int lrow = tid >> 3, kc = (tid & 7) ^ swz(lrow);
  unsigned off[LPT];
#pragma unroll
  for (int i = 0; i < AL; ++i) off[i] = (unsigned)min(i * RPI + lrow, g.M - 1 - m0) * (unsigned)g.lda + kc * 8;
#pragma unroll
  for (int i = 0; i < BL; ++i) off[AL + i] = (unsigned)min(i * RPI + lrow, g.N - 1 - n0) * (unsigned)g.ldb + kc * 8;
  auto issue1 = [&](auto I, int kt, int st) __attribute__((always_inline)) {
    constexpr int i = decltype(I)::value;
    const f16* src;
    if constexpr (SEG == 1) src = (i < AL ? A : B) + (int64_t)(kt0 + kt) * BK;
    else {
      const int k = kt0 + kt, seg = (k >= g.nk) + (k >= 2 * g.nk);
      src = (i < AL ? A + (seg == 2 ? g.ta : 0) : B + (seg == 1 ? g.tb : 0)) + (int64_t)(k - seg * g.nk) * BK;
    }
    unsigned char* dst = smem + st * STAGE + wave * 1024 + (i < AL ? i * RPI * 128 : BM * 128 + (i - AL) * RPI * 128);
    __builtin_amdgcn_global_load_lds(BSR_GLOBAL_PTR(src + off[i]), BSR_LDS_VOID(dst), 16, 0, 0);
  };
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mi][ni][r] = 0.f;
  // fragments: read order A0, B0 .. B(NI-1), A1 .. A(MI-1), so that the first matrix instructions of a k-step can start early
  const int lr = lane & 31, lh = lane >> 5, sw = swz(lr);
  int offr[NFR];
  f16x8 fr[2][NFR];
#pragma unroll
  for (int j = 0; j < NFR; ++j) {
    const bool isA = j == 0 || j > NI;
    const int idx = j == 0 ? 0 : (j <= NI ? j - 1 : j - NI);
    offr[j] = isA ? (wm * TM + idx * 32 + lr) * 128 : BM * 128 + (wn * TN + idx * 32 + lr) * 128;
  }
  auto rd1 = [&](auto SET, auto J, int st, int ks) __attribute__((always_inline)) {
    constexpr int set = decltype(SET)::value, j = decltype(J)::value;
    fr[set][j] = *(const f16x8*)(smem + st * STAGE + (((ks * 2 + lh) ^ sw) << 4) + offr[j]);
  };
  auto mf1 = [&](auto SET, auto J) __attribute__((always_inline)) {
    constexpr int set = decltype(SET)::value, j = decltype(J)::value, mi = j / NI, ni = j % NI, ja = mi == 0 ? 0 : NI + mi, jb = 1 + ni;
    if constexpr (F16) acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[set][jb], fr[set][ja], acc[mi][ni], 0, 0, 0);
    else acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fr[set][jb]), __builtin_bit_cast(bf16x8, fr[set][ja]), acc[mi][ni], 0, 0, 0);
  };
  constexpr int PRE = NMF >= 16 ? 4 : (NMF >= 8 ? 2 : 1), POST = NMF - PRE;          // matrix instructions of the last k-step in front of the barrier, and behind it
  constexpr int SPAN = POST + (NST == 2 ? NMF >= 8 : NMF >= 4 ? 3 : NMF == 3 ? 2 : 0) * NMF;    // over which the loads of a k-tile are spread
  auto loads_at = [&](auto P, int kt, int st) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value, lo = p >= SPAN ? LPT : (p * LPT + SPAN - 1) / SPAN, hi = p + 1 >= SPAN ? LPT : ((p + 1) * LPT + SPAN - 1) / SPAN;
    sfor<hi - lo>([&](auto L) __attribute__((always_inline)) { issue1(IC<lo + decltype(L)::value>{}, kt, st); });
  };
  constexpr bool LATE = SPAN > POST;
  auto kstep = [&](auto SET, auto LOADS, auto KS, int st, int ktl, int stl) __attribute__((always_inline)) {
    constexpr int set = decltype(SET)::value, ks = decltype(KS)::value;
    sfor<NMF>([&](auto J) __attribute__((always_inline)) {
      constexpr int j = decltype(J)::value, RPM = (NFR + NMF - 1) / NMF;
      mf1(IC<set>{}, J);
      sfor<RPM>([&](auto R) __attribute__((always_inline)) {
        constexpr int r = j * RPM + decltype(R)::value;
        if constexpr (r < NFR) rd1(IC<set ^ 1>{}, IC<r>{}, st, ks);
      });
      if constexpr (decltype(LOADS)::value) loads_at(IC<POST + (ks - 1) * NMF + j>{}, ktl, stl);
      BSR_SCHED_FENCE();
    });
  };
  // the last k-step of k-tile kt, with the barrier.  VMW >= 0: loads that may stay in flight there; < 0: nothing is issued any more, the count follows from what is left
  auto klast = [&](auto VMW, int kt, int st, int stn, int rem) __attribute__((always_inline)) {
    constexpr int vmw = decltype(VMW)::value, RPP = (NFR + POST - 1) / POST;
    sfor<PRE>([&](auto J) __attribute__((always_inline)) { mf1(IC<1>{}, J); BSR_SCHED_FENCE(); });
    wait_lgkmcnt0();
    if constexpr (vmw >= 0) wait_vmcnt<vmw>();
    else if (rem >= 3) wait_vmcnt<2 * LPT>();
    else if (rem == 2) wait_vmcnt<LPT>();
    else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    BSR_SCHED_FENCE();
    sfor<POST>([&](auto P) __attribute__((always_inline)) {
      constexpr int p = decltype(P)::value;
      mf1(IC<1>{}, IC<PRE + p>{});
      sfor<RPP>([&](auto R) __attribute__((always_inline)) {
        constexpr int r = p * RPP + decltype(R)::value;
        if constexpr (r < NFR) rd1(IC<0>{}, IC<r>{}, stn, 0);
      });
      if constexpr (vmw >= 0) loads_at(P, kt + NST, st);
      BSR_SCHED_FENCE();
    });
  };
#pragma unroll
  for (int j = 0; j < NST; ++j)
    if (j < nk) sfor<LPT>([&](auto I) __attribute__((always_inline)) { issue1(I, j, j); });
  {
    const int fl = min(nk, NST) - 1;               // k-tiles that may stay in flight
    if (fl >= 3) wait_vmcnt<3 * LPT>(); else if (fl == 2) wait_vmcnt<2 * LPT>(); else if (fl == 1) wait_vmcnt<LPT>(); else wait_vmcnt<0>();
  }
  __builtin_amdgcn_s_barrier();
  sfor<NFR>([&](auto J) __attribute__((always_inline)) { rd1(IC<0>{}, J, 0, 0); });
  int st = 0, kt = 0;
  auto ktile = [&](auto LOADS, auto VMW) __attribute__((always_inline)) {
    const int stn = (st + 1 == NST) ? 0 : st + 1, stl = st == 0 ? NST - 1 : st - 1;
    kstep(IC<0>{}, LOADS, IC<1>{}, st, kt + NST - 1, stl);
    kstep(IC<1>{}, LOADS, IC<2>{}, st, kt + NST - 1, stl);
    kstep(IC<0>{}, LOADS, IC<3>{}, st, kt + NST - 1, stl);
    klast(VMW, kt, st, stn, nk - 1 - kt);
    st = stn;
    ++kt;
  };
  constexpr IC<(NST - 2) * LPT> steady{};
  if constexpr (LATE) {
    if (kt + NST < nk) ktile(IC<0>{}, steady);
    while (kt + NST < nk) ktile(IC<1>{}, steady);
    if (kt > 0) ktile(IC<1>{}, IC<-1>{});
  } else {
    while (kt + NST < nk) ktile(IC<0>{}, steady);
  }
  while (kt < nk) ktile(IC<0>{}, IC<-1>{});
  // every wavefront is past the last barrier, i.e. has read its last fragments of the tiles (the reads behind it are idle): wait for those before the stages are used for anything else
  wait_lgkmcnt0();
}

template <class S, Mode MODE, bool F16, int SEG>
__global__ __launch_bounds__(S::NT, S::lds <= 80 * 1024 ? S::NT / 128 : 1) void ce_kernel(CeGemm g, int mt, int nt) {
  constexpr int MI = S::MI, NI = S::NI, TM = S::TM, TN = S::TN;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
  const int lm = lane & 31, lh = lane >> 5;
  const int id = xcd_remap(blockIdx.x, gridDim.x), split = MODE == OUT ? id / (mt * nt) : 0;
  int tm, tn;
  tile_at(MODE == OUT ? id - split * mt * nt : id, mt, nt, tm, tn);
  const int m0 = tm * S::BM, n0 = tn * S::BN;
  const int kt0 = MODE == OUT ? split * g.per : 0, nk = MODE == OUT ? min(g.per, SEG * g.nk - kt0) : m0 < g.M ? SEG * g.nk : 0;      // (tokens that only fill GT's last k-tile: zeros)
  f32x16 acc[MI][NI];
  multiply<S, F16, SEG>(g, m0, n0, kt0, nk, smem, acc);
  __syncthreads();
  unsigned char* patch = smem + wave * S::patch;
  const int row0 = m0 + wm * TM, col0 = n0 + wn * TN;

  if constexpr (MODE == STATS || MODE == GRAD) {
    // a lane has 16 NI classes of MI tokens: what belongs to the classes, once
    float b[NI][16];
    int e[F16 ? NI : 1][16];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = col0 + ni * 32 + 8 * (r / 4) + 4 * lh + r % 4;
        b[ni][r] = n < g.N ? (g.bias ? g.bias[n] : 0.f) : -INFINITY;
        if constexpr (F16) e[ni][r] = n < g.N ? g.eb[n] : 0;
      }
    if constexpr (MODE == STATS) {
      float2* red = (float2*)smem;                 // [WN][BM]
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int m = row0 + mi * 32 + lm;
        const int at = m < g.M ? max(g.labels[m], -1) - g.v0 - col0 : -1, ea = F16 && m < g.M ? g.ea[m] : 0;
        float most = -INFINITY, zl = 0.f;
        bool mine = false;
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float z = acc[mi][ni][r];
            if constexpr (F16) z = ldexpf(z, ea + e[ni][r]);
            z += b[ni][r];
            // (a class past the last one: whatever the product of a repeated row is, it does not count)
            if (b[ni][r] == -INFINITY && col0 + ni * 32 + 8 * (r / 4) + 4 * lh + r % 4 >= g.N) z = -INFINITY;
            acc[mi][ni][r] = z;
            most = fmaxf(most, z);
            const bool here = at == ni * 32 + 8 * (r / 4) + 4 * lh + r % 4;
            zl = here ? z : zl;
            mine |= here;
          }
        most = half_max(most);
        const float ref = most == -INFINITY ? 0.f : most;
        float s = 0.f;
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int r = 0; r < 16; ++r) s += __expf(acc[mi][ni][r] - ref);
        s = half_sum(s);
        if (lh == 0) red[wn * S::BM + wm * TM + mi * 32 + lm] = make_float2(most, s);
        if (mine && at + col0 < g.N) g.zlabel[m] = zl;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < S::BM && m0 + i < g.M; i += S::NT) {
        float2 p = red[i];
#pragma unroll
        for (int j = 1; j < S::WN; ++j) {
          const float2 q = red[j * S::BM + i];
          const float most = fmaxf(p.x, q.x), ref = most == -INFINITY ? 0.f : most;
          p = make_float2(most, p.y * __expf(p.x - ref) + q.y * __expf(q.x - ref));
        }
        g.parts[(int64_t)tn * g.M + m0 + i] = p;
      }
    } else {
      constexpr int TERMS = SEG == 3 ? 2 : 1;
      f16x4 t[TERMS][MI][NI][4];
      float sum[NI][16];
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[ni][r] = 0.f;
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int m = row0 + mi * 32 + lm, mc = min(m, g.M - 1);
        const int label = g.labels[mc], ea = F16 ? g.ea[mc] : 0, at = max(label, -1) - g.v0 - col0;
        const float2 st = g.stats[mc];
        const float weight = g.row_grad ? g.row_grad[mc] : 1.f;
        // (label: of the whole layer; a row of logits that are all -inf has no gradient; of those that are all NaN the logarithm is NaN)
        const bool counts = m < g.M && label >= 0 && label < g.classes && weight != 0.f && !(st.x == -INFINITY && st.y == 0.f);
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int c = ni * 32 + 8 * (r / 4) + 4 * lh + r % 4;
            float z = acc[mi][ni][r];
            if constexpr (F16) z = ldexpf(z, ea + e[ni][r]);
            z += b[ni][r];
            float p = __expf((z - st.x) - st.y) - (at == c ? 1.f : 0.f);
            p = counts && col0 + c < g.N ? p : 0.f;
            sum[ni][r] += weight * p;
            p *= (float)(1 << G_SHIFT);
            const f16 h = (f16)p;
            t[0][mi][ni][r / 4][r % 4] = h;
            if constexpr (TERMS == 2) t[TERMS - 1][mi][ni][r / 4][r % 4] = (f16)(p - (float)h);
          }
      }
      (void)sum;
#pragma unroll
      for (int term = 0; term < TERMS; ++term) {
        if (g.GT) {
#pragma unroll
          for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                *(f16*)(patch + (ni * 32 + 8 * (r / 4) + 4 * lh + r % 4) * S::LDT + (mi * 32 + lm) * 2) = t[term][mi][ni][r / 4][r % 4];
          wave_fence();
          constexpr int CPR = TM / 8, RPP = 64 / CPR;            // 16-byte chunks of a patch row, rows at a time
          f16* to = g.GT + term * g.tgt;
          const int c = lane % CPR;
#pragma unroll 4
          for (int p = 0; p < TN / RPP; ++p) {
            const int r = p * RPP + lane / CPR, n = col0 + r, m = row0 + c * 8;
            if (n < g.N && m < g.ldgt) *(f16x8*)(to + (int64_t)n * g.ldgt + m) = *(const f16x8*)(patch + r * S::LDT + c * 16);
          }
          wave_fence();
        }
        if (g.G) {
          constexpr int CPR = TN / 8, RPP = 64 / CPR;
          f16* to = g.G + term * g.tg;
          const int c = lane % CPR;
#pragma unroll
          for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
#pragma unroll
              for (int q = 0; q < 4; ++q) *(f16x4*)(patch + lm * S::LDR + (ni * 32 + 8 * q + 4 * lh) * 2) = t[term][mi][ni][q];
            wave_fence();
#pragma unroll
            for (int p = 0; p < 32 / RPP; ++p) {
              const int r = p * RPP + lane / CPR, m = row0 + mi * 32 + r, n = col0 + c * 8;
              if (m < g.M && n < g.ldg) *(f16x8*)(to + (int64_t)m * g.ldg + n) = *(const f16x8*)(patch + r * S::LDR + c * 16);
            }
            wave_fence();
          }
        }
      }
      if (g.dbp) {
        // sums over the tile's tokens: the 32 lanes of a half, then the wavefronts, in order
        __syncthreads();
        float* red = (float*)smem;                 // [WM][BN]
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float v = sum[ni][r];
#pragma unroll
            for (int d = 16; d > 0; d /= 2) v += __shfl_xor(v, d);
            if (lm == 0) red[wm * S::BN + wn * TN + ni * 32 + 8 * (r / 4) + 4 * lh + r % 4] = v;
          }
        __syncthreads();
        for (int i = threadIdx.x; i < S::BN && n0 + i < g.N; i += S::NT) {
          float v = red[i];
#pragma unroll
          for (int j = 1; j < S::WM; ++j) v += red[j * S::BN + i];
          g.dbp[(int64_t)tm * g.N + n0 + i] = v;
        }
      }
    }
  } else {
    constexpr int CPR = TN / 4, RPP = 64 / CPR;                  // 4-column chunks of a patch row, rows at a time
    const int c = lane % CPR, n = col0 + c * 4;
    int e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = (n + j < g.N ? g.eb[n + j] : 0) - G_SHIFT;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(f32x4*)(patch + lm * S::LDF + (ni * 32 + 8 * q + 4 * lh) * 4) = f32x4{acc[mi][ni][4 * q], acc[mi][ni][4 * q + 1], acc[mi][ni][4 * q + 2], acc[mi][ni][4 * q + 3]};
      wave_fence();
#pragma unroll 4
      for (int p = 0; p < 32 / RPP; ++p) {
        const int r = p * RPP + lane / CPR, m = row0 + mi * 32 + r;
        f32x4 v = *(const f32x4*)(patch + r * S::LDF + c * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = ldexpf(v[j], e[j]);
        if (m < g.M && n < g.N) {
          if (g.part) {
            f32x4* to = (f32x4*)(g.part + split * g.tp + (int64_t)m * g.ldp + n);
            *to = g.add ? *to + v : v;
          } else {
            const float by = g.row_scale ? g.scale * g.row_scale[m] : g.scale;
            v *= by;
            if (g.out_f32) {
              float* to = (float*)g.out + (int64_t)m * g.ldo + n;
              if (g.out_vec) *(f32x4*)to = v;
              else
                for (int j = 0; j < 4; ++j)
                  if (n + j < g.N) to[j] = v[j];
            } else {
              bf16* to = (bf16*)g.out + (int64_t)m * g.ldo + n;
              typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
              const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
              if (g.out_vec) *(bf16x4*)to = o;
              else
                for (int j = 0; j < 4; ++j)
                  if (n + j < g.N) to[j] = o[j];
            }
          }
        }
      }
      wave_fence();
    }
  }
}

// ------------------------------------------------------------------------------------------ operands
// the power of two of a row whose largest finite |value| has these bits: that value times 2^-e lies in 2^14 .. 2^15
__device__ __forceinline__ int exponent_of(uint32_t bits) { return bits ? (int)(bits >> 23) - 127 - 14 : 0; }
__device__ __forceinline__ uint32_t bits_if_finite(float v) {
  const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// rows of D values to rows of whole k-tiles: bf16 as they are, fp32 in two fp16 terms (`term` elements apart) with a power of two a row.  A wavefront a row
template <typename T>
__global__ __launch_bounds__(256) void ce_pack_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows, int D, int Dp, uint16_t* __restrict__ to, int64_t term, int* __restrict__ exps) {
  const int lane = threadIdx.x % WAVE;
  const int64_t m = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE;
  if (m >= rows) return;
  const T* row = x + m * ldx;
  uint16_t* out = to + m * Dp;
  if constexpr (sizeof(T) == 2) {
    for (int j = lane; j < Dp; j += WAVE) out[j] = j < D ? __builtin_bit_cast(uint16_t, row[j]) : (uint16_t)0;
  } else {
    float most = 0.f;
    for (int j = lane; j < D; j += WAVE) most = fmaxf(most, __uint_as_float(bits_if_finite(row[j])));
    const int e = exponent_of(__float_as_uint(wave_max(most)));
    if (lane == 0) exps[m] = e;
    for (int j = lane; j < Dp; j += WAVE) {
      const float v = j < D ? ldexpf(row[j], -e) : 0.f;
      const f16 h = (f16)v, l = (f16)(v - (float)h);
      out[j] = __builtin_bit_cast(uint16_t, h);
      out[term + j] = __builtin_bit_cast(uint16_t, l);
    }
  }
}

// what a row of x counts with in dw
struct RowWeights { const int32_t* labels; const float* row_grad; int classes; };
__device__ __forceinline__ float weight_of(const RowWeights& w, int64_t m) {
  if (!w.labels) return 1.f;
  const int label = w.labels[m];
  return label >= 0 && label < w.classes ? w.row_grad ? w.row_grad[m] : 1.f : 0.f;
}
template <typename T> __device__ __forceinline__ float weighted(T v, float by) { return by == 0.f ? 0.f : (float)v * by; }

__global__ __launch_bounds__(256) void ce_zero_kernel(uint32_t* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0u;
}

// bits of the largest |value| of each column (maxima: their order changes nothing)
template <typename T>
__global__ __launch_bounds__(256) void ce_colmax_kernel(const T* __restrict__ x, int64_t ldx, int rows, int D, int per, RowWeights rw, uint32_t* __restrict__ most) {
  __shared__ uint32_t red[4][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, col = blockIdx.x * WAVE + lane, r1 = min((int)(blockIdx.y + 1) * per, rows);
  uint32_t b = 0;
  if (col < D)
#pragma unroll 8
    for (int m = blockIdx.y * per + w; m < r1; m += 4) b = max(b, bits_if_finite(weighted(x[m * ldx + col], weight_of(rw, m))));
  red[w][lane] = b;
  __syncthreads();
  if (w == 0 && col < D) atomicMax(most + col, max(max(red[0][lane], red[1][lane]), max(red[2][lane], red[3][lane])));
}

// [rows, D] -> [terms][D][ld] fp16, a power of two each of the D rows; what lies between rows and ld is zero
template <typename T>
__global__ __launch_bounds__(256) void ce_transpose_kernel(const T* __restrict__ x, int64_t ldx, int rows, int D, RowWeights rw, const uint32_t* __restrict__ most, f16* __restrict__ to,
                                                           int64_t ld, int64_t term, int* __restrict__ exps) {
  constexpr int TERMS = sizeof(T) / 2;
  __shared__ f16 tile[TERMS][64][64 + 8];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, c0 = blockIdx.y * 64, col = c0 + lane;
  const int m0 = blockIdx.x * 64, e = col < D ? exponent_of(most[col]) : 0;
  if (blockIdx.x == 0 && w == 0 && col < D) exps[col] = e;
#pragma unroll 4
  for (int r = w; r < 64; r += 4) {
    const int m = m0 + r;
    const float v = m < rows && col < D ? ldexpf(weighted(x[m * ldx + col], weight_of(rw, m)), -e) : 0.f;
    const f16 h = (f16)v;
    tile[0][lane][r] = h;
    if constexpr (TERMS == 2) tile[TERMS - 1][lane][r] = (f16)(v - (float)h);
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < TERMS; ++t)
#pragma unroll
    for (int i = threadIdx.x; i < 512; i += 256) {
      const int c = i / 8, m = m0 + i % 8 * 8;
      if (c0 + c < D && m < ld) *(f16x8*)(to + t * term + (int64_t)(c0 + c) * ld + m) = *(const f16x8*)&tile[t][c][i % 8 * 8];
    }
}

// ------------------------------------------------------------------------------------------ joining
// 64 rows a workgroup: wavefront w joins tiles w, w + 16, ..., then the wavefronts in order; first and last piece of the classes: begin, end
__global__ __launch_bounds__(1024) void ce_join_kernel(const float2* __restrict__ parts, int tiles, int M, float2* __restrict__ run, int begin, int end, const float* __restrict__ zlabel,
                                                       const int32_t* __restrict__ labels, int classes, float* __restrict__ loss, float2* __restrict__ stats) {
  __shared__ float2 red[16][WAVE];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, m = blockIdx.x * WAVE + lane, mc = min(m, M - 1);
  auto join = [](float2 p, float2 q) __attribute__((always_inline)) {
    const float most = fmaxf(p.x, q.x), ref = most == -INFINITY ? 0.f : most;
    return make_float2(most, p.y * __expf(p.x - ref) + q.y * __expf(q.x - ref));
  };
  float2 p = make_float2(-INFINITY, 0.f);
#pragma unroll 8
  for (int t = w; t < tiles; t += 16) p = join(p, parts[(int64_t)t * M + mc]);
  red[w][lane] = p;
  __syncthreads();
  if (w != 0 || m >= M) return;
  if (!begin) p = join(run[m], p);
#pragma unroll
  for (int i = 1; i < 16; ++i) p = join(p, red[i][lane]);
  if (!end) {
    run[m] = p;
    return;
  }
  // (a row of logits that are all -inf, and nothing else: sum 0)
  const float ls = p.y == 0.f ? 0.f : logf(p.y);
  if (stats) stats[m] = make_float2(p.x, ls);
  if (loss) {
    const int label = labels[m];
    const bool counts = label >= 0 && label < classes && !(p.x == -INFINITY && p.y == 0.f);
    loss[m] = counts ? (p.x - zlabel[m]) + ls : 0.f;
  }
}

// out = scale row_scale[m] (sum over the parts, in order)
template <typename T>
__global__ __launch_bounds__(256) void ce_reduce_kernel(const float* __restrict__ part, int splits, int64_t tp, int64_t ldp, int64_t M, int N, float scale, const float* __restrict__ row_scale,
                                                        T* __restrict__ out, int64_t ldo) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, chunks = (N + 3) / 4, m = i / chunks;
  const int n = (int)(i - m * chunks) * 4;
  if (m >= M) return;
  f32x4 v = *(const f32x4*)(part + m * ldp + n);
  for (int s = 1; s < splits; ++s) v += *(const f32x4*)(part + s * tp + m * ldp + n);
  v *= row_scale ? scale * row_scale[m] : scale;
  T* to = out + m * ldo + n;
  if (n + 4 <= N && ((uintptr_t)to & (4 * sizeof(T) - 1)) == 0) {
    typedef T vec __attribute__((ext_vector_type(4)));
    *(vec*)to = vec{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
    for (int j = 0; j < 4; ++j)
      if (n + j < N) to[j] = (T)v[j];
  }
}

__global__ __launch_bounds__(256) void ce_db_kernel(const float* __restrict__ dbp, int tiles, int n, float scale, float* __restrict__ db) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float v = 0.f;
#pragma unroll 8
  for (int t = 0; t < tiles; ++t) v += dbp[(int64_t)t * n + i];
  db[i] = scale * v;
}

// no tokens: no gradients
template <typename T> __global__ __launch_bounds__(256) void ce_fill_kernel(T* __restrict__ out, int64_t ld, int64_t rows, int cols) {
  for (int64_t m = blockIdx.x; m < rows; m += gridDim.x)
    for (int j = threadIdx.x; j < cols; j += 256) out[m * ld + j] = (T)0.f;
}

// ------------------------------------------------------------------------------------------ host
int up(int64_t n, int to) { return (int)((n + to - 1) / to * to); }
int over(int64_t n, int by) { return (int)((n + by - 1) / by); }

template <class S, Mode MODE, bool F16, int SEG> void launch(const CeGemm& g, int mt, int nt, hipStream_t s) {
  auto kern = ce_kernel<S, MODE, F16, SEG>;
  static uint64_t known = 0;                       // devices on which the kernel has its LDS
  int dev = 0;
  (void)hipGetDevice(&dev);
  if (!(__atomic_load_n(&known, __ATOMIC_RELAXED) >> (dev & 63) & 1)) {
    (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::lds);
    __atomic_fetch_or(&known, (uint64_t)1 << (dev & 63), __ATOMIC_RELAXED);
  }
  kern<<<mt * nt * g.splits, S::NT, S::lds, s>>>(g, mt, nt);
}
enum { LARGE, SMALL, FEW };
template <Mode MODE, bool F16, int SEG> void launch_as(int shape, const CeGemm& g, int rows, hipStream_t s) {
  // (rows: those that tiles have to cover)
  if (shape == FEW) launch<Few, MODE, F16, SEG>(g, over(rows, Few::BM), over(g.N, Few::BN), s);
  else if (shape == SMALL || (SEG == 3 && MODE == GRAD)) launch<Small, MODE, F16, SEG>(g, over(rows, Small::BM), over(g.N, Small::BN), s);
  else if constexpr (SEG == 1 || MODE != GRAD) launch<Large, MODE, F16, SEG>(g, over(rows, Large::BM), over(g.N, Large::BN), s);
}
int rows_of(int shape) { return shape == FEW ? Few::BM : shape == SMALL ? Small::BM : Large::BM; }
int cols_of(int shape) { return shape == FEW ? Few::BN : shape == SMALL ? Small::BN : Large::BN; }

// the shape and the workgroups over k of a product, by a model of its time in rounds over the 256 CUs (us)
struct Pick { int shape, splits, per; };
Pick pick(int64_t M, int64_t N, int kt, bool split, bool large) {
  static const double tile[3] = {1.15, 0.40, 0.30}, start[3] = {7, 4, 4};
  Pick best = {SMALL, 1, kt};
  double least = 1e30;
  for (int shape = 0; shape < 3; ++shape) {
    if ((shape == FEW && M > 32) || (shape == LARGE && !large)) continue;
    const int64_t tiles = (int64_t)over(M, rows_of(shape)) * over(N, cols_of(shape));
    for (int n = 1; n <= (split ? 64 : 1); ++n) {
      const int per = over(kt, n), splits = over(kt, per);
      if (splits != n || (n > 1 && per < 4)) continue;
      const double us = (double)((tiles * n + 255) / 256) * (per * tile[shape] + start[shape]) + (n > 1 ? 3 + n * M * N * 8e-6 / 4 : 0);
      if (us < least) { least = us; best = {shape, n, per}; }
    }
  }
  return best;
}

// sizes, and places in the workspace
struct Plan {
  int T, Dp, Np, Vs, Vp, Vc, dx_parts, dw_parts, Dq;
  size_t xp, ex, wp, ew, parts, run, zlabel, G, GT, xT, wT, exT, ewT, most, dxp, dwp, dbp, bytes;
  Plan(bool f32, int N, int D, int V, bool backward) {
    T = f32 ? 2 : 1;
    Dp = up(D, BK); Np = up(N, BK); Dq = up(D, 4);
    // Pieces of the classes, whole tiles and alike in size.  Forward: the tiles' maxima and sums take at most 64 MB (Vs) and what is packed 256 (Vp, where something is).
    // Backward: G, twice, takes at most 256 MB, and so does the transposed piece of w.
    auto piece = [&](double most) {
      const int64_t c = std::max<int64_t>(256, (int64_t)std::min(most, 1e9) / 256 * 256);
      return up(over(V, over(V, (int)c)), 256);
    };
    constexpr double MB = 1 << 20;
    Vs = piece(64 * MB * 128 / (8.0 * N));
    Vp = std::min(Vs, piece(256 * MB / (2.0 * T * Dp)));
    Vc = std::min(piece(256 * MB / (4.0 * T * Np)), piece(256 * MB / (2.0 * T * Dp)));
    bytes = 0;
    auto take = [&](size_t n) { const size_t at = bytes; bytes += (n + 255) / 256 * 256; return at; };
    const int Vm = backward ? Vc : Vp;
    xp = take((size_t)2 * T * N * Dp); ex = take(sizeof(int) * (size_t)N);
    wp = take((size_t)2 * T * Vm * Dp); ew = take(sizeof(int) * (size_t)Vm);
    if (!backward) {
      parts = take(sizeof(float2) * (size_t)over(Vs, 128) * N); run = take(sizeof(float2) * (size_t)N); zlabel = take(sizeof(float) * (size_t)N);
      return;
    }
    G = take((size_t)2 * T * N * Vc); GT = take((size_t)2 * T * Vc * Np);
    xT = take((size_t)2 * T * D * Np); exT = take(sizeof(int) * (size_t)D);
    wT = take((size_t)2 * T * D * Vc); ewT = take(sizeof(int) * (size_t)D);
    most = take(sizeof(uint32_t) * (size_t)D);
    dx_parts = pick(N, D, over(std::min(Vc, up(V, BK)), BK) * (T == 2 ? 3 : 1), true, true).splits;
    dw_parts = pick(std::min(V, Vc), D, Np / BK * (T == 2 ? 3 : 1), true, true).splits;
    dxp = take(sizeof(float) * (size_t)dx_parts * N * Dq);
    dwp = take(dw_parts > 1 ? sizeof(float) * (size_t)dw_parts * Vc * Dq : 0);
    dbp = take(sizeof(float) * (size_t)over(Np, 32) * Vc);
  }
};

// (a tile's rows are addressed in 32 bits)
bool whole_rows(const void* p, int64_t ld, int D) { return D % BK == 0 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld <= 1 << 23; }

// An operand of the logits: as it lies, or packed
struct Rows { const void* p; int64_t ld, term; const int* exps; };
Rows rows_operand(const void* p, int64_t ld, bool f32, int64_t rows, int D, int Dp, void* packed, int* exps, bool as_it_lies, hipStream_t s) {
  if (as_it_lies) return {p, ld, 0, nullptr};
  const int64_t term = rows * Dp;
  const unsigned grid = (unsigned)((rows + 3) / 4);
  if (f32) ce_pack_kernel<float><<<grid, 256, 0, s>>>((const float*)p, ld, rows, D, Dp, (uint16_t*)packed, term, exps);
  else ce_pack_kernel<bf16><<<grid, 256, 0, s>>>((const bf16*)p, ld, rows, D, Dp, (uint16_t*)packed, term, nullptr);
  return {packed, Dp, term, f32 ? exps : nullptr};
}

template <typename T>
void transposed(const void* x, int64_t ldx, int rows, int D, const RowWeights& rw, uint32_t* most, f16* to, int64_t ld, int64_t term, int* exps, hipStream_t s) {
  ce_zero_kernel<<<over(D, 256), 256, 0, s>>>(most, D);
  const int per = std::max(64, over(rows, std::max(1, 2048 / over(D, 64))));
  ce_colmax_kernel<T><<<dim3(over(D, 64), over(rows, per)), 256, 0, s>>>((const T*)x, ldx, rows, D, per, rw, most);
  ce_transpose_kernel<T><<<dim3(over(ld, 64), over(D, 64)), 256, 0, s>>>((const T*)x, ldx, rows, D, rw, most, to, ld, term, exps);
}

}  // namespace

size_t linear_ce_workspace_bytes(bool f32, int N, int D, int V, bool backward) { return Plan(f32, N, D, V, backward).bytes; }

void linear_ce_forward(const LinearCe& a, hipStream_t s) {
  const Plan p(a.f32, a.N, a.D, a.V, false);
  char* ws = (char*)a.workspace;
  const int64_t size = a.f32 ? 4 : 2;
  const bool direct_x = !a.f32 && whole_rows(a.x, a.ldx, a.D), direct_w = !a.f32 && whole_rows(a.w, a.ldw, a.D);
  const Rows x = rows_operand(a.x, a.ldx, a.f32, a.N, a.D, p.Dp, ws + p.xp, (int*)(ws + p.ex), direct_x, s);
  const int step = direct_w ? p.Vs : p.Vp;
  for (int v0 = 0; v0 < a.V; v0 += step) {
    const int n = std::min(step, a.V - v0);
    const Rows w = rows_operand((const char*)a.w + v0 * a.ldw * size, a.ldw, a.f32, n, a.D, p.Dp, ws + p.wp, (int*)(ws + p.ew), direct_w, s);
    CeGemm g;
    g.A = x.p; g.lda = x.ld; g.ta = x.term; g.ea = x.exps; g.B = w.p; g.ldb = w.ld; g.tb = w.term; g.eb = w.exps;
    g.M = a.N; g.N = n; g.nk = p.Dp / BK; g.bias = a.bias ? a.bias + v0 : nullptr; g.labels = a.labels; g.v0 = v0; g.classes = a.V;
    g.parts = (float2*)(ws + p.parts); g.zlabel = (float*)(ws + p.zlabel);
    const Pick k = pick(a.N, n, g.nk * (a.f32 ? 3 : 1), false, true);
    if (a.f32) launch_as<STATS, true, 3>(k.shape, g, a.N, s);
    else launch_as<STATS, false, 1>(k.shape, g, a.N, s);
    ce_join_kernel<<<over(a.N, WAVE), 1024, 0, s>>>(g.parts, over(n, cols_of(k.shape)), a.N, (float2*)(ws + p.run), v0 == 0, v0 + n == a.V, g.zlabel, a.labels, a.V, a.loss, (float2*)a.stats);
  }
}

template <typename T>
void backward_as(const LinearCe& a, hipStream_t s) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int SEG = F32 ? 3 : 1;
  const Plan p(F32, a.N, a.D, a.V, true);
  char* ws = (char*)a.workspace;
  const bool direct_x = !F32 && whole_rows(a.x, a.ldx, a.D), direct_w = !F32 && whole_rows(a.w, a.ldw, a.D);
  const Rows x = rows_operand(a.x, a.ldx, F32, a.N, a.D, p.Dp, ws + p.xp, (int*)(ws + p.ex), direct_x, s);
  f16 *xT = (f16*)(ws + p.xT), *wT = (f16*)(ws + p.wT), *G = (f16*)(ws + p.G), *GT = (f16*)(ws + p.GT);
  if (a.dw) transposed<T>(a.x, a.ldx, a.N, a.D, {a.labels, a.row_grad, a.V}, (uint32_t*)(ws + p.most), xT, p.Np, (int64_t)a.D * p.Np, (int*)(ws + p.exT), s);
  Pick kx = {SMALL, 1, 1};
  for (int v0 = 0; v0 < a.V; v0 += p.Vc) {
    const int n = std::min(p.Vc, a.V - v0), np = up(n, BK);
    const T* wv = (const T*)a.w + v0 * a.ldw;
    const Rows w = rows_operand(wv, a.ldw, F32, n, a.D, p.Dp, ws + p.wp, (int*)(ws + p.ew), direct_w, s);
    CeGemm g;
    g.A = x.p; g.lda = x.ld; g.ta = x.term; g.ea = x.exps; g.B = w.p; g.ldb = w.ld; g.tb = w.term; g.eb = w.exps;
    g.M = a.N; g.N = n; g.nk = p.Dp / BK; g.bias = a.bias ? a.bias + v0 : nullptr; g.labels = a.labels; g.v0 = v0; g.classes = a.V;
    g.stats = (const float2*)a.stats; g.row_grad = a.row_grad;
    if (a.dx) { g.G = G; g.ldg = np; g.tg = (int64_t)a.N * np; }
    if (a.dw) { g.GT = GT; g.ldgt = p.Np; g.tgt = (int64_t)n * p.Np; }
    if (a.db) g.dbp = (float*)(ws + p.dbp);
    const Pick kg = pick(a.N, n, g.nk * SEG, false, !F32);
    launch_as<GRAD, F32, SEG>(kg.shape, g, a.dw ? p.Np : a.N, s);
    if (a.db) ce_db_kernel<<<over(n, 256), 256, 0, s>>>(g.dbp, over(a.dw ? p.Np : a.N, rows_of(kg.shape)), n, a.grad_scale, a.db + v0);
    if (a.dx) {
      transposed<T>(wv, a.ldw, n, a.D, {nullptr, nullptr, 0}, (uint32_t*)(ws + p.most), wT, np, (int64_t)a.D * np, (int*)(ws + p.ewT), s);
      CeGemm o;
      o.A = G; o.lda = np; o.ta = g.tg; o.B = wT; o.ldb = np; o.tb = (int64_t)a.D * np; o.eb = (int*)(ws + p.ewT);
      o.M = a.N; o.N = a.D; o.nk = np / BK;
      // one shape and number of parts for all pieces: the parts are added to
      if (v0 == 0) kx = pick(a.N, a.D, o.nk * SEG, true, true);
      o.splits = kx.splits; o.per = over(o.nk * SEG, kx.splits);
      o.part = (float*)(ws + p.dxp); o.ldp = p.Dq; o.tp = (int64_t)a.N * p.Dq; o.add = v0 > 0;
      launch_as<OUT, true, SEG>(kx.shape, o, a.N, s);
    }
    if (a.dw) {
      CeGemm o;
      o.A = GT; o.lda = p.Np; o.ta = g.tgt; o.B = xT; o.ldb = p.Np; o.tb = (int64_t)a.D * p.Np; o.eb = (int*)(ws + p.exT);
      o.M = n; o.N = a.D; o.nk = p.Np / BK;
      const Pick k = pick(std::min(a.V, p.Vc), a.D, o.nk * SEG, true, true);
      o.splits = k.splits; o.per = k.per; o.scale = a.grad_scale;
      char* dw = (char*)a.dw + v0 * a.lddw * (a.dw_f32 ? 4 : 2);
      if (k.splits > 1) { o.part = (float*)(ws + p.dwp); o.ldp = p.Dq; o.tp = (int64_t)n * p.Dq; }
      else { o.out = dw; o.ldo = a.lddw; o.out_f32 = a.dw_f32; o.out_vec = a.D % 4 == 0 && a.lddw % 4 == 0 && ((uintptr_t)dw & (a.dw_f32 ? 15 : 7)) == 0; }
      launch_as<OUT, true, SEG>(k.shape, o, n, s);
      if (k.splits > 1) {
        const unsigned grid = (unsigned)over((int64_t)n * over(a.D, 4), 256);
        if (a.dw_f32) ce_reduce_kernel<float><<<grid, 256, 0, s>>>(o.part, k.splits, o.tp, o.ldp, n, a.D, a.grad_scale, nullptr, (float*)dw, a.lddw);
        else ce_reduce_kernel<bf16><<<grid, 256, 0, s>>>(o.part, k.splits, o.tp, o.ldp, n, a.D, a.grad_scale, nullptr, (bf16*)dw, a.lddw);
      }
    }
  }
  if (a.dx)
    ce_reduce_kernel<T><<<(unsigned)over((int64_t)a.N * over(a.D, 4), 256), 256, 0, s>>>((const float*)(ws + p.dxp), kx.splits, (int64_t)a.N * p.Dq, p.Dq, a.N, a.D, a.grad_scale, a.row_grad,
                                                                                       (T*)a.dx, a.lddx);
}
void linear_ce_backward(const LinearCe& a, hipStream_t s) {
  if (a.N == 0) {
    const unsigned grid = (unsigned)std::min(a.V, 4096);
    if (a.dw && a.dw_f32) ce_fill_kernel<float><<<grid, 256, 0, s>>>((float*)a.dw, a.lddw, a.V, a.D);
    else if (a.dw) ce_fill_kernel<bf16><<<grid, 256, 0, s>>>((bf16*)a.dw, a.lddw, a.V, a.D);
    if (a.db) ce_fill_kernel<float><<<1, 256, 0, s>>>(a.db, 0, 1, a.V);
    return;
  }
  if (a.f32) backward_as<float>(a, s);
  else backward_as<bf16>(a, s);
}

}  // namespace bsr
