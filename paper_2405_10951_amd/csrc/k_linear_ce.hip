// Softmax cross-entropy of a linear layer over many classes, and its gradients, without keeping the logits:
//   z = x w^T + b;   loss = log sum exp z - z_label;   G = softmax(z) - onehot(label);   dx = g G w;   dw = G^T (g x);   db = G^T g
// Forward: tiles of z stay in the accumulators of the product; a tile leaves each row's maximum and its sum of exp(z - maximum), and a second kernel joins the tiles of a row.
// Backward: z is made again (or, in one call for both, read where 16 MB hold it), a piece of the classes at a time; the tile's end turns it into G and leaves that as it lies and transposed, so that both products behind it
// contract over contiguous memory like the first.  What they need transposed beside it (x once, the piece's rows of w) is transposed in a pass of its own.
//
// Numbers.  bf16 x and w are multiplied as they are and added in fp32.  G is kept in fp16, not bf16: it lies within -1 .. 1, and scaled by 2^14 its values keep 11 bits down to
// 2^-28 and are off by 2^-39 at most below, where bf16 would keep 8; x and w join it in fp16, each feature (a row of the transposed operand) scaled by a power of two so that its
// largest value lies in 2^14 .. 2^15, which is exact for bf16 values down to 2^-29 of the feature's largest.  The matrix instructions take both types at one rate.  fp32 operands are two fp16 terms each,
// h + l with h = fp16(v), l = fp16(v - h), off by 2^-22 of the value, and the products h h, l h, h l are added in fp32.  A k-tile holds both terms of 32 k: it is loaded
// once for the three of them (333 x 1001 x 5003 loss and gradients 93 us in the run in which one product after another over the whole contraction took 109 and k-tile by k-tile 107; 93 to 102 from card to card).
// dw in fp32 beside bf16 operands: one fp16 term of G would show in it (with weights off by 8e-5 of its norm, two terms by 4.5e-7, at 2048 x 768 x 21841), so the transposed G has two, and so has x times a weight; the products
// h h, l h and, with weights, h l follow one another over a contraction of two or three times the tokens (6304 x 768 x 21841 loss and gradients 1423 us, with weights 1670; dw in bf16 1072).  In a bf16 result G's
// one term does not show: 2048 x 768 x 21841 dw is off by 1.662e-3 of its norm, from exact G by 1.659e-3, the rounding of the result.
// Bound by the matrix unit's power where it is large: at 4096 x 4096 x 131072 bf16 a tile of 16 x 16 x 32 instructions runs at 1.7 - 1.8 GHz (32 x 32 x 16 at 1.46, 6 % slower in all), the forward at
// 1350 TFLOP/s (3.25 ms), a piece's G at 1225 (450 us), both products of G at 1250 (880 us); transposing a piece takes 38 + 59 us.  2048 x 768 x 21841, gradients, best and median of
// twenty: maxima 12 and 14, transposing 16 and 18, G 94 and 111 (688 tiles of 12 k-tiles on 256 CUs: beginnings and ends count as much as the products), products 121 and 147, sums 9.  333 x 1001 x 5003 fp32: packing 11,
// logits 19, joining 5, maxima 10, transposing 13, G 9, products 35, sums 4.
// The row's weight g scales x in dw and the result in dx; rows whose label is absent or whose weight is 0 have G = 0 and, in the transposed x, zeros.
#include <algorithm>

#include "gemm_common.h"
#include "linear_ce.h"
#include "rowops.h"

namespace bsr {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16;
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

int up(int64_t n, int to) { return (int)((n + to - 1) / to * to); }
int over(int64_t n, int by) { return (int)((n + by - 1) / by); }

constexpr int BK = 64;
// where element k of a row lies: of two terms 32 h and 32 l in turn
template <int TERMS> __host__ __device__ constexpr int64_t spot(int64_t k, int term = 0) { return TERMS == 2 ? k / 32 * 64 + k % 32 + 32 * term : k; }
constexpr int G_SHIFT = 14;                        // G is kept times 2^14

// ------------------------------------------------------------------------------------------ the products
enum Mode { STATS, GRAD };

// C(m,n) = sum_k A(m,k) B(n,k): rows of 64-element k-tiles, whole ones, 16-byte aligned.  TERMS 2: a k-tile holds 32 k, first their h, then their l, and the products are h h, l h, h l.
struct CeGemm {
  const void *A = nullptr, *B = nullptr;
  int64_t lda = 0, ldb = 0;
  int M = 0, N = 0, nk = 0;                        // nk: k-tiles
  int splits = 1, per = 0;                         // products of G: workgroups over the k-tiles of a tile, k-tiles of each
  int pass = 0;                                    // PASSES: k-tiles of a pass; A's rows are h, then l, and so are B's where there are three passes: h h, l h, h l
  const int *ea = nullptr, *eb = nullptr;          // powers of two of A's and B's rows, null: 0
  // STATS, GRAD: m is a token, n a class of the piece that begins at class v0
  const float* bias = nullptr;                     // of the piece
  const int32_t* labels = nullptr;
  int v0 = 0, classes = 0;                         // classes of the whole layer
  float2* parts = nullptr; float* zlabel = nullptr;                        // STATS: [tile of classes][M] maximum and sum; [M]
  float* z = nullptr; int64_t ldz = 0;             // STATS: the logits as well, [M][ldz], ldz whole fours; null: not wanted
  const float2* stats = nullptr; const float* row_grad = nullptr;          // GRAD: [M] maximum, log of the sum; weights or null
  f16 *G = nullptr, *GT = nullptr;                 // GRAD: [M][ldg], [N][ldgt], of which kg and kgt columns (of one or both terms) are written, zero behind the last one; null: not wanted
  int64_t ldg = 0, ldgt = 0; int kg = 0, kgt = 0;
  float* dbp = nullptr; int64_t ldd = 0;           // GRAD: [tile of tokens][ldd] sums of g G; null: not wanted
  // products of G
  float* part = nullptr; int64_t ldp = 0, tp = 0; bool add = false;        // [split][M][ldp] fp32 (of what was there as well)
  void* out = nullptr; int64_t ldo = 0; bool out_f32 = false, out_vec = false;   // or the result itself, times scale
  float scale = 1.f;
};

template <int BM_, int BN_, int WM_, int WN_, int NST_> struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NST = NST_, NT = WM * WN * 64;
  static constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;              // a wavefront's part, in tiles of 16 x 16
  static constexpr size_t stages = (size_t)NST * (BM + BN) * 128;
  static constexpr int LDR = TN * 2 + 16, LDF = TN * 4 + 16;     // patch rows in bytes: fp16, fp32
  static constexpr int patch = 32 * (2 * LDR > LDF ? 2 * LDR : LDF);                       // of a wavefront: 32 rows, of one or two terms
  static constexpr size_t lds = stages > (size_t)patch * WM * WN ? stages : (size_t)patch * WM * WN;
  static constexpr int at_once = (int)(160 * 1024 / lds), wavefronts = at_once * (NT / 64) / 4;       // workgroups a CU, wavefronts a SIMD
};
typedef Shape<256, 256, 2, 4, 2> Large;
typedef Shape<256, 256, 2, 2, 2> LargeForward;     // (bf16: four wavefronts read a third less of LDS for the product, eight share the work of ending a tile; of two terms eight are faster,
                                                   // 2048 x 768 x 21841 196 us against 224, and need no register that four would spill)
typedef Shape<128, 128, 2, 4, 3> Small;
typedef Shape<64, 128, 2, 2, 3> Mid;                  // (logits only: where larger tiles would leave CUs idle)
typedef Shape<128, 128, 2, 4, 2> Short;               // (logits only: of few k-tiles, two workgroups a CU, so that one's products cover the other's beginning and end)
typedef Shape<32, 256, 1, 4, 4> Few;

// tiles band after band of eight row tiles, row tile fastest: what an XCD works on at a time shares rows of A and of B
constexpr int BAND = 8;
__device__ __forceinline__ void tile_at(int t, int mt, int nt, int& m, int& n) {
  const int band = t / (BAND * nt), in = t - band * BAND * nt, rows = min(BAND, mt - band * BAND);
  n = in / rows;
  m = band * BAND + in - n * rows;
}

// Where a row's chunks of 16 bytes lie in LDS: chunk kc at position kc ^ place(row).  A fragment is read 16 lanes at a time, of which some have one chunk and some its neighbour (lanes 0 - 3, 12 - 15
// and 20 - 27 go together), of 16 different rows: all 64 banks once.
__device__ __forceinline__ int place(int row) { return row >> 1 & 7; }

// Operands go straight into LDS (global_load_lds: rows of 8 chunks of 16 bytes, their order in LDS made by the address that a lane reads), NST stages of a
// k-tile of 64, one barrier a k-tile.  A k-tile is 2 MI groups (of two terms: 3 MI, h and l of each with B's h, then h again with B's l) of NI matrix instructions 16 x 16 x 32, each group with one fragment
// of A: fragments of A come DIST groups ahead through a ring of RING, those of B a half ahead.  DIST groups before the k-tile's end every wavefront has read all of it: there is the barrier, and behind it the loads of k-tile kt + NST go out into its stage, one or two a group.
// 16 x 16 x 32, not 32 x 32 x 16: under full load the clock is what the power allows, and the smaller tile, which touches half as many accumulators a product, draws less.
// The operands are swapped (B's rows first): accumulators hold transposed tiles, element r of acc[mi][ni] is row mi 16 + lane % 16, column ni 16 + 4 (lane / 16) + r.
// PASSES: rows of two terms lie one term behind the other, and the contraction goes over them as one longer one of up to three passes.
template <class S, bool F16, int TERMS, bool PASSES = false>
__device__ __forceinline__ void multiply(const CeGemm& g, int m0, int n0, int kt0, int nk, unsigned char* smem, f32x4 (&acc)[S::MI][S::NI]) {
  constexpr int BM = S::BM, WN = S::WN, NST = S::NST, TM = S::TM, TN = S::TN, MI = S::MI, NI = S::NI, HALF = TERMS * MI, NG = HALF + MI;
  constexpr int RPI = S::NT / 8, AL = BM / RPI, BL = S::BN / RPI, LPT = AL + BL, STAGE = (BM + S::BN) * 128;
  constexpr int RING = NG % 4 == 0 ? 4 : 3, DIST = RING - 1;
  static_assert(BM % RPI == 0 && S::BN % RPI == 0 && RPI % 16 == 0, "a load instruction covers whole groups of 16 rows");
  static_assert(NST >= 2 && NST <= 4 && (NST - 1) * LPT <= 60, "vmcnt has 6 bits");
  static_assert(NG % RING == 0 && NG > DIST, "the ring comes round with the k-tile");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const f16* __restrict__ A = (const f16*)g.A + (int64_t)m0 * g.lda;
  const f16* __restrict__ B = (const f16*)g.B + (int64_t)n0 * g.ldb;
  // rows past the last one repeat it: they only feed accumulators that count for nothing
  const int lrow = tid >> 3, kc = (tid & 7) ^ place(lrow);
  unsigned off[LPT];                               // in bytes: beside an address that the wavefront shares they cost no arithmetic
#pragma unroll
  for (int i = 0; i < AL; ++i) off[i] = (unsigned)min(i * RPI + lrow, g.M - 1 - m0) * (unsigned)g.lda * 2 + kc * 16;
#pragma unroll
  for (int i = 0; i < BL; ++i) off[AL + i] = (unsigned)min(i * RPI + lrow, g.N - 1 - n0) * (unsigned)g.ldb * 2 + kc * 16;
  auto issue1 = [&](auto I, int kt, int st) __attribute__((always_inline)) {
    constexpr int i = decltype(I)::value;
    const f16* src = i < AL ? A : B;
    int k = kt0 + kt;
    if constexpr (PASSES) {
      if (i < AL) k -= k >= 2 * g.pass ? 2 * g.pass : 0;
      else k -= k >= g.pass ? g.pass : 0;
    }
    // (a buffer: address of the tile in scalar registers, the row's bytes in a vector register, the k-tile's in a scalar one, and no arithmetic)
    unsigned char* dst = smem + st * STAGE + wave * 1024 + (i < AL ? i * RPI * 128 : BM * 128 + (i - AL) * RPI * 128);
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)src, 0, -1, 0x00020000), BSR_LDS_VOID(dst), 16, off[i], k * BK * 2, 0, 0);
#else
    (void)src; (void)dst; (void)k;                 // (the host's pass does not know these instructions)
#endif
  };
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
  // a fragment: 16 rows, a lane 8 k of one: chunk 4 ks + lane / 16 of row lane % 16
  const int lr = lane & 15, lq = lane >> 4, sw = place(lr);
  const unsigned char *fa = smem + (wm * TM + lr) * 128, *fb = smem + BM * 128 + (wn * TN + lr) * 128;
  f16x8 a[RING], b[2][NI];
  // group gi (0 .. NG - 1) of a k-tile: half of B, 32 k of A (or its term), rows of A
  auto half_of = [](int gi) constexpr { return gi >= HALF; };
  auto ks_of = [](int gi) constexpr { return TERMS == 2 ? (gi < HALF ? gi % 2 : 0) : gi / MI; };
  auto mi_of = [](int gi) constexpr { return gi >= HALF ? gi - HALF : TERMS == 2 ? gi / 2 : gi; };
  auto read_a = [&](auto GI, int st) __attribute__((always_inline)) {
    constexpr int gi = decltype(GI)::value, ks = ks_of(gi), mi = mi_of(gi);
    a[gi % RING] = *(const f16x8*)(fa + st * STAGE + mi * 16 * 128 + (((ks * 4 + lq) ^ sw) << 4));
  };
  auto read_b = [&](auto KS, auto J, int st) __attribute__((always_inline)) {
    constexpr int ks = decltype(KS)::value, j = decltype(J)::value;
    b[ks][j] = *(const f16x8*)(fb + st * STAGE + j * 16 * 128 + (((ks * 4 + lq) ^ sw) << 4));
  };
  // loads of k-tile ktl's number p .. : spread evenly over SPAN groups behind the barrier
  constexpr int SPAN = NG > 8 ? 8 : NG;
  auto loads = [&](auto P, int kt, int st) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value, lo = p >= SPAN ? LPT : (p * LPT + SPAN - 1) / SPAN, hi = p + 1 >= SPAN ? LPT : ((p + 1) * LPT + SPAN - 1) / SPAN;
    sfor<hi - lo>([&](auto L) __attribute__((always_inline)) { issue1(IC<lo + decltype(L)::value>{}, kt, st); });
  };
  // A k-tile in stage st; its successor in stn.  EARLY: the rest of the loads of k-tile kt + NST - 1 goes out into stage stl (the one in front of st);  VMW: loads that may stay in flight at the
  // barrier, behind which the first loads of k-tile kt + NST follow;  < 0: nothing more to load, the count follows from rem, the number of k-tiles behind this one
  auto ktile = [&](auto EARLY, auto VMW, int kt, int st, int stn, int stl, int rem) __attribute__((always_inline)) {
    constexpr int vmw = decltype(VMW)::value, LAST = NG - DIST;
    sfor<NG>([&](auto GI) __attribute__((always_inline)) {
      constexpr int gi = decltype(GI)::value, ks = half_of(gi), mi = mi_of(gi);
      if constexpr (gi == LAST) {
        wait_lgkmcnt0();
        if constexpr (vmw >= 0) wait_vmcnt<vmw>();
        else if (rem >= 3) wait_vmcnt<2 * LPT>();
        else if (rem == 2) wait_vmcnt<LPT>();
        else wait_vmcnt<0>();
        __builtin_amdgcn_s_barrier();
        BSR_SCHED_FENCE();
      }
      sfor<NI>([&](auto J) __attribute__((always_inline)) {
        constexpr int j = decltype(J)::value;
        if constexpr (F16) acc[mi][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[ks][j], a[gi % RING], acc[mi][j], 0, 0, 0);
        else acc[mi][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[ks][j]), __builtin_bit_cast(bf16x8, a[gi % RING]), acc[mi][j], 0, 0, 0);
        if constexpr (j == 0) {                    // (into the place of the group before, whose instructions have been issued)
          if constexpr (gi + DIST < NG) read_a(IC<gi + DIST>{}, st);
          else read_a(IC<gi + DIST - NG>{}, stn);
        }
        // the next k-step's fragments of B: a few a group, those of the next k-tile right behind the barrier, those of this one's second half in the middle of its first
        constexpr int at = ks == 0 ? gi - (HALF / 2 - 1) : gi - (LAST > HALF ? LAST : HALF);
        constexpr int BPG = (NI + DIST - 1) / DIST, jb = BPG * at + j;
        if constexpr (j < BPG && at >= 0 && jb < NI && (ks == 1 || HALF >= 4)) {
          if constexpr (ks == 0) read_b(IC<1>{}, IC<jb>{}, st);
          else read_b(IC<0>{}, IC<jb>{}, stn);
        }
        if constexpr (HALF < 4 && ks == 0 && gi == 0 && j == NI - 1) sfor<NI>([&](auto Q) __attribute__((always_inline)) { read_b(IC<1>{}, Q, st); });
        BSR_SCHED_FENCE();
      });
      if constexpr (gi >= LAST) {
        if constexpr (vmw >= 0) loads(IC<gi - LAST>{}, kt + NST, st);
      } else if constexpr (decltype(EARLY)::value) loads(IC<gi + DIST>{}, kt + NST - 1, stl);
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
  sfor<DIST>([&](auto I) __attribute__((always_inline)) { read_a(I, 0); });
  sfor<NI>([&](auto J) __attribute__((always_inline)) { read_b(IC<0>{}, J, 0); });
  int st = 0, kt = 0;
  auto step = [&](auto EARLY, auto VMW) __attribute__((always_inline)) {
    const int stn = st + 1 == NST ? 0 : st + 1, stl = st == 0 ? NST - 1 : st - 1;
    ktile(EARLY, VMW, kt, st, stn, stl, nk - 1 - kt);
    st = stn;
    ++kt;
  };
  constexpr IC<(NST - 2) * LPT> steady{};
  if (kt + NST < nk) step(IC<0>{}, steady);        // (the first stages' loads are all out)
  while (kt + NST < nk) step(IC<1>{}, steady);
  if (kt > 0 && kt < nk) step(IC<1>{}, IC<-1>{});  // the rest of the last loads
  while (kt < nk) step(IC<0>{}, IC<-1>{});
  // every wavefront is past the last barrier, i.e. has read its last fragments of the tiles (the reads behind it are idle): wait for those before the stages are used for anything else
  wait_lgkmcnt0();
}

template <class S> struct Wave {                   // where a wavefront's part of a tile lies
  int lane, lm, lq, wm, wn, row0, col0;
  __device__ __forceinline__ Wave(int m0, int n0) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63; lm = lane & 15; lq = lane >> 4; wm = wave / S::WN; wn = wave % S::WN;
    row0 = m0 + wm * S::TM; col0 = n0 + wn * S::TN;
  }
  // column (in the wavefront's part) of element r of acc[..][ni]
  __device__ __forceinline__ int col(int ni, int r) const { return ni * 16 + 4 * lq + r; }
  __device__ __forceinline__ unsigned char* patch(unsigned char* smem) const { return smem + (wm * S::WN + wn) * S::patch; }
};

// bias and powers of two of a lane's 4 NI classes; classes past the last one: -inf
template <class S, bool F16> struct Classes {
  float b[S::NI][4];
  int e[F16 ? S::NI : 1][4];
  bool edge;                                       // some lie past the last one (of the whole wavefront)
  __device__ __forceinline__ Classes(const CeGemm& g, const Wave<S>& w) {
    edge = w.col0 + S::TN > g.N;
#pragma unroll
    for (int ni = 0; ni < S::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = w.col0 + w.col(ni, r), nc = min(n, g.N - 1);
        b[ni][r] = g.bias ? g.bias[nc] : 0.f;
        if constexpr (F16) e[ni][r] = g.eb[nc];
      }
  }
  __device__ __forceinline__ float logit(float acc, int ea, int ni, int r) const {
    if constexpr (F16) acc = ldexpf(acc, ea + e[ni][r]);
    return acc + b[ni][r];
  }
};

// of lanes l, l ^ 16, l ^ 32 and l ^ 48
template <class Op> __device__ __forceinline__ float quarters_all(float v, Op op) {
  v = halves_all(v, op);
  const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
}

constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float2 joined(float2 p, float2 q) {   // two maxima with their sums of exp(z - maximum)
  const float most = fmaxf(p.x, q.x), ref = most == -INFINITY ? 0.f : most;
  return make_float2(most, p.y * __expf(p.x - ref) + q.y * __expf(q.x - ref));
}

// Forward: a row's maximum and sum over the tile's classes.  (fmaxf passes NaN over, the sum does not; a row of -inf alone has sum 0.)
template <class S, bool F16>
__device__ __forceinline__ void end_stats(const CeGemm& g, f32x4 (&acc)[S::MI][S::NI], int m0, int n0, int tn, unsigned char* smem) {
  const Wave<S> w(m0, n0);
  const Classes<S, F16> cl(g, w);
  float2* red = (float2*)smem;                     // [WN][BM]
#pragma unroll
  for (int mi = 0; mi < S::MI; ++mi) {
    const int m = w.row0 + mi * 16 + w.lm;
    const int at = m < g.M ? max(g.labels[m], -1) - g.v0 - w.col0 : -1, ea = F16 && m < g.M ? g.ea[m] : 0;
    float most = -INFINITY;
#pragma unroll
    for (int ni = 0; ni < S::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[mi][ni][r] = cl.logit(acc[mi][ni][r], ea, ni, r);
    if (g.z && m < g.M)
#pragma unroll
      for (int ni = 0; ni < S::NI; ++ni)
        if (w.col0 + w.col(ni, 0) < g.N) *(f32x4*)(g.z + (int64_t)m * g.ldz + w.col0 + w.col(ni, 0)) = acc[mi][ni];
    if (cl.edge)                                   // (whatever the product of a repeated row is, it does not count)
#pragma unroll
      for (int ni = 0; ni < S::NI; ++ni)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (w.col0 + w.col(ni, r) >= g.N) acc[mi][ni][r] = -INFINITY;
#pragma unroll
    for (int ni = 0; ni < S::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 4; ++r) most = fmaxf(most, acc[mi][ni][r]);
    if (__any(at >= 0 && at < S::TN))              // (few wavefronts hold a label)
#pragma unroll
      for (int ni = 0; ni < S::NI; ++ni)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (at == w.col(ni, r) && at + w.col0 < g.N) g.zlabel[m] = acc[mi][ni][r];
    most = quarters_all(most, [](float p, float q) { return fmaxf(p, q); });
    const float ref = most == -INFINITY ? 0.f : most;
    float s = 0.f;
#pragma unroll
    for (int ni = 0; ni < S::NI; ++ni)
#pragma unroll
      for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f((acc[mi][ni][r] - ref) * LOG2E);
    s = quarters_all(s, [](float p, float q) { return p + q; });
    if (w.lq == 0) red[w.wn * S::BM + w.wm * S::TM + mi * 16 + w.lm] = make_float2(most, s);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < S::BM && m0 + i < g.M; i += S::NT) {
    float2 p = red[i];
#pragma unroll
    for (int j = 1; j < S::WN; ++j) p = joined(p, red[j * S::BM + i]);
    g.parts[(int64_t)tn * g.M + m0 + i] = p;
  }
}

// sums of 16 (or 8) values over each 16 lanes: lane l gets that of value l % 16 (l % 8).  Each step halves the values a lane holds
template <int N> __device__ __forceinline__ float lanes16_sums(float (&v)[N]) {
  static_assert(N == 16 || N == 8, "");
  const int l = threadIdx.x;
  if constexpr (N == 16)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (l & 8 ? v[i + 8] : v[i]) + dpp_move<0x128>(l & 8 ? v[i] : v[i + 8]);        // lane ^ 8
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += dpp_move<0x128>(v[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (l & 4 ? v[i + 4] : v[i]) + dpp_move<0x141>(l & 4 ? v[i] : v[i + 4]);          // lane ^ 7, which holds the same values so far
#pragma unroll
  for (int i = 0; i < 2; ++i) v[i] = (l & 2 ? v[i + 2] : v[i]) + dpp_move<0x4E>(l & 2 ? v[i] : v[i + 2]);           // lane ^ 2
  return (l & 1 ? v[1] : v[0]) + dpp_move<0xB1>(l & 1 ? v[0] : v[1]);                                              // lane ^ 1
}

// Backward: the tile as G, in fp16 times 2^14, rows of 32 tokens at a time through a patch of LDS, from which rows are read as they lie and, with the transposing reads, columns
// FINE (of bf16 operands): the transposed G in two terms, one behind the other.  dw is wanted in fp32, and one fp16 term would be off by up to 2^-11 of itself
template <class S, bool F16, int TERMS, bool DB, bool FINE>
__device__ __forceinline__ void end_grad(const CeGemm& g, f32x4 (&acc)[S::MI][S::NI], int m0, int n0, int tm, unsigned char* smem) {
  constexpr int NI = S::NI, TERM = 32 * S::LDR, KEPT = FINE ? 2 : TERMS;
  const Wave<S> w(m0, n0);
  const Classes<S, F16> cl(g, w);
  unsigned char* patch = w.patch(smem);
  float sum[DB ? NI * 4 : 1];
  if constexpr (DB)
#pragma unroll
    for (int i = 0; i < NI * 4; ++i) sum[i] = 0.f;
#pragma unroll
  for (int mi = 0; mi < S::MI; ++mi) {
    const int m = w.row0 + mi * 16 + w.lm, mc = min(m, g.M - 1);
    const int label = max(g.labels[mc], -1), ea = F16 ? g.ea[mc] : 0, at = label - g.v0 - w.col0;
    const float2 st = g.stats[mc];
    const float weight = g.row_grad ? g.row_grad[mc] : 1.f;
    // (label: of the whole layer; a row of logits that are all -inf has no gradient; of those that are all NaN the logarithm is NaN)
    const bool counts = m < g.M && label >= 0 && label < g.classes && weight != 0.f && !(st.x == -INFINITY && st.y == 0.f);
    const float c = fmaf(st.y, -LOG2E, (float)G_SHIFT);
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[mi][ni][r] = __builtin_amdgcn_exp2f(fmaf(cl.logit(acc[mi][ni][r], ea, ni, r) - st.x, LOG2E, c));
    if (__any(at >= 0 && at < S::TN))              // (few wavefronts hold a label)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[mi][ni][r] -= at == w.col(ni, r) ? (float)(1 << G_SHIFT) : 0.f;
    if (!__all(counts) || cl.edge)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[mi][ni][r] = counts && w.col0 + w.col(ni, r) < g.N ? acc[mi][ni][r] : 0.f;
    if constexpr (DB) {
      const float by = counts ? weight : 0.f;
#pragma unroll
      for (int i = 0; i < NI * 4; ++i) sum[i] = fmaf(by, acc[mi][i / 4][i % 4], sum[i]);
    }
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      f16x4 h, l;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = acc[mi][ni][j];
        h[j] = (f16)p;
        if constexpr (KEPT == 2) l[j] = (f16)(p - (float)h[j]);
      }
      unsigned char* to = patch + (mi % 2 * 16 + w.lm) * S::LDR + w.col(ni, 0) * 2;
      *(f16x4*)to = h;
      if constexpr (KEPT == 2) *(f16x4*)(to + TERM) = l;
    }
    if (mi % 2 == 0) continue;
    const int first = w.row0 + (mi - 1) * 16;      // the patch's 32 tokens
    wave_fence();
#pragma unroll
    for (int term = 0; term < KEPT; ++term) {
      if (term < TERMS && g.G) {
        constexpr int CPR = S::TN / 8, RPP = 64 / CPR;           // 16-byte chunks of a patch row, rows at a time
        const int k = w.lane % CPR, n = w.col0 + k * 8;
#pragma unroll
        for (int p = 0; p < 32 / RPP; ++p) {
          const int r = p * RPP + w.lane / CPR, row = first + r;
          if (row < g.M && n < g.kg) *(f16x8*)(g.G + (int64_t)row * g.ldg + spot<TERMS>(n, term)) = *(const f16x8*)(patch + term * TERM + r * S::LDR + k * 16);
        }
      }
      if (g.GT) {
        // 16 lanes read 4 tokens x 16 classes (lane 4 e + q names the address of classes 4 q .. of token e) and get a class each, four tokens of it; two such reads are 16 bytes of GT
        const int j = w.lane & 15, octet = w.lane >> 4, token = first + octet * 8;
        const unsigned char* from = patch + term * TERM + (octet * 8 + (j >> 2)) * S::LDR + (j & 3) * 8;
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
#pragma unroll
        for (int cb = 0; cb < S::TN / 16; ++cb) {
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(from + cb * 32));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(from + cb * 32 + 4 * S::LDR));
          const int n = w.col0 + cb * 16 + j;
          if (n < g.N && token < g.kgt) *(s16x8*)(g.GT + (int64_t)n * g.ldgt + (FINE ? token + (int64_t)term * g.kgt : spot<TERMS>(token, term))) = s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        }
      }
    }
    wave_fence();
  }
  if constexpr (DB) {
    // sums over the tile's tokens: lanes, then the wavefronts in order
    constexpr int K = NI * 4 > 16 ? 16 : NI * 4;   // values at a time
    __syncthreads();
    float* red = (float*)smem;                     // [WM][BN]
#pragma unroll
    for (int i = 0; i < NI * 4; i += K) {
      float part[K];
#pragma unroll
      for (int j = 0; j < K; ++j) part[j] = sum[i + j];
      const float v = lanes16_sums<K>(part);
      if (w.lm < K) red[w.wm * S::BN + w.wn * S::TN + w.col((i + w.lm) / 4, w.lm % 4)] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < S::BN && n0 + i < g.N; i += S::NT) {
      float t = red[i];
#pragma unroll
      for (int j = 1; j < S::WM; ++j) t += red[j * S::BN + i];
      g.dbp[tm * g.ldd + n0 + i] = ldexpf(t, -G_SHIFT);
    }
  }
}

template <class S, Mode MODE, bool F16, int TERMS, bool DB, bool FINE>
__global__ __launch_bounds__(S::NT, S::wavefronts) void ce_logits_kernel(CeGemm g, int mt, int nt) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int tm, tn;
  tile_at(xcd_remap(blockIdx.x, gridDim.x), mt, nt, tm, tn);
  const int m0 = tm * S::BM, n0 = tn * S::BN;
  f32x4 acc[S::MI][S::NI];
  multiply<S, F16, TERMS>(g, m0, n0, 0, m0 < g.M ? g.nk : 0, smem, acc);      // (tokens that only fill GT's last k-tile: zeros)
  __syncthreads();
  if constexpr (MODE == STATS) end_stats<S, F16>(g, acc, m0, n0, tn, smem);
  else end_grad<S, F16, TERMS, DB, FINE>(g, acc, m0, n0, tm, smem);
}

// Up to two products of G in one launch (a, then b, na workgroups of the first): dx and dw of a piece fill the CUs together
template <class S, int TERMS, bool PASSES>
__global__ __launch_bounds__(S::NT, 1) void ce_grads_kernel(CeGemm a, CeGemm b, int na) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const bool first = (int)blockIdx.x < na;
  CeGemm g;
  if (first) g = a;
  else g = b;
  const int mt = (g.M + S::BM - 1) / S::BM, nt = (g.N + S::BN - 1) / S::BN, here = first ? na : (int)gridDim.x - na;
  const int id = xcd_remap(first ? blockIdx.x : blockIdx.x - na, here), split = id / (mt * nt);
  int tm, tn;
  tile_at(id - split * mt * nt, mt, nt, tm, tn);
  const int m0 = tm * S::BM, n0 = tn * S::BN, kt0 = split * g.per;
  f32x4 acc[S::MI][S::NI];
  multiply<S, true, TERMS, PASSES>(g, m0, n0, kt0, min(g.per, g.nk - kt0), smem, acc);
  __syncthreads();
  const Wave<S> w(m0, n0);
  unsigned char* patch = w.patch(smem);
  constexpr int CPR = S::TN / 4, RPP = 64 / CPR;                 // 4-column chunks of a patch row, rows at a time
  const int c = w.lane % CPR, n = w.col0 + c * 4;
  int e[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) e[j] = (n + j < g.N ? g.eb[n + j] : 0) - G_SHIFT;
#pragma unroll
  for (int mi = 0; mi < S::MI; ++mi) {
#pragma unroll
    for (int ni = 0; ni < S::NI; ++ni)
      *(f32x4*)(patch + (mi % 2 * 16 + w.lm) * S::LDF + w.col(ni, 0) * 4) = acc[mi][ni];
    if (mi % 2 == 0) continue;
    wave_fence();
#pragma unroll 4
    for (int p = 0; p < 32 / RPP; ++p) {
      const int r = p * RPP + w.lane / CPR, m = w.row0 + (mi - 1) * 16 + r;
      f32x4 v = *(const f32x4*)(patch + r * S::LDF + c * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = ldexpf(v[j], e[j]);
      if (m < g.M && n < g.N) {
        if (g.part) {
          f32x4* to = (f32x4*)(g.part + split * g.tp + (int64_t)m * g.ldp + n);
          *to = g.add ? *to + v : v;
        } else {
          v *= g.scale;
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

// ------------------------------------------------------------------------------------------ operands
// the power of two of a row whose largest finite |value| has these bits: that value times 2^-e lies in 2^14 .. 2^15
__device__ __forceinline__ int exponent_of(uint32_t bits) { return bits ? (int)(bits >> 23) - 127 - 14 : 0; }
__device__ __forceinline__ uint32_t bits_if_finite(float v) {
  const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// x, w or both (a launch handles up to two; the first `blocks` workgroups the first)
struct PackJob { const void* x = nullptr; int64_t ldx = 0, rows = 0; uint16_t* to = nullptr; int* exps = nullptr; };
// rows of D values to rows of whole k-tiles: bf16 as they are, a thread 8 of them, fp32 in two fp16 terms with a power of two a row, LANES lanes a row
template <typename T, int LANES> int pack_blocks(int64_t rows, int Dp) { return sizeof(T) == 2 ? over(rows * (Dp / 8), 256) : over(rows, 256 / LANES); }
template <typename T, int LANES>
__global__ __launch_bounds__(256) void ce_pack_kernel(PackJob a, PackJob b, int blocks, int D, int Dp) {
  const bool first = (int)blockIdx.x < blocks;
  const PackJob j = first ? a : b;
  const int block = first ? blockIdx.x : blockIdx.x - blocks;
  constexpr int V = Chunk<T>::V;
  auto load = [&](const T* row, int k) __attribute__((always_inline)) {
    typename Chunk<T>::vec v;
    if (k + V <= D) v = *(const typename Loose<T>::vec*)(row + k);
    else
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = k + e < D ? row[k + e] : (T)0.f;
    return v;
  };
  if constexpr (sizeof(T) == 2) {
    const unsigned chunks = Dp / V, i = (unsigned)block * 256 + threadIdx.x, m = i / chunks;       // (2^33 values at most)
    if (m < j.rows) *(typename Chunk<T>::vec*)(j.to + (int64_t)m * Dp + (i - m * chunks) * V) = load((const T*)j.x + (int64_t)m * j.ldx, (i - m * chunks) * V);
  } else {
    const int lane = threadIdx.x % LANES;
    const int64_t m = (int64_t)block * (256 / LANES) + threadIdx.x / LANES;
    const bool there = m < j.rows;                 // (lanes of other rows take part in the maximum)
    const T* row = (const T*)j.x + (there ? m : j.rows - 1) * j.ldx;
    uint16_t* out = j.to + m * Dp * 2;
    // rows of up to 2048 values stay in registers, longer ones are read twice
    constexpr int KEEP = LANES == WAVE ? 8 : 1;
    f32x4 v[KEEP];
    float most = 0.f;
    const bool kept = LANES < WAVE || Dp <= KEEP * WAVE * V;      // (fewer lanes: of rows that they hold)
    auto most_of = [&](f32x4 p) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < V; ++e) most = fmaxf(most, __uint_as_float(bits_if_finite(p[e])));
    };
    if (kept) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i) v[i] = load(row, (lane + i * LANES) * V);
#pragma unroll
      for (int i = 0; i < KEEP; ++i) most_of(v[i]);
    } else {
#pragma unroll 4
      for (int k = lane * V; k < D; k += WAVE * V) most_of(load(row, k));
    }
    if constexpr (LANES == WAVE) most = wave_max(most);
    else
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    if (!there) return;
    const int e = exponent_of(__float_as_uint(most));
    if (lane == 0) j.exps[m] = e;
    auto put = [&](int k, f32x4 x) __attribute__((always_inline)) {
      f16x4 h, l;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float s = ldexpf(x[i], -e);
        h[i] = (f16)s;
        l[i] = (f16)(s - (float)h[i]);
      }
      *(f16x4*)(out + spot<2>(k)) = h;
      *(f16x4*)(out + spot<2>(k, 1)) = l;
    };
    if (kept) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i)
        if ((lane + i * LANES) * V < Dp) put((lane + i * LANES) * V, v[i]);
    } else {
#pragma unroll 4
      for (int k = lane * V; k < Dp; k += WAVE * V) put(k, load(row, k));
    }
  }
}

// what a row of x counts with in dw
struct RowWeights { const int32_t* labels = nullptr; const float* row_grad = nullptr; int classes = 0; };
__device__ __forceinline__ float weight_of(const RowWeights& w, int64_t m) {
  if (!w.labels) return 1.f;
  const int label = w.labels[m];
  return label >= 0 && label < w.classes ? w.row_grad ? w.row_grad[m] : 1.f : 0.f;
}
__device__ __forceinline__ float weighted(float v, float by) { return by == 0.f ? 0.f : v * by; }

// A masked class has G 0 but where it is a row's label: its bias is -inf, or below -2^120 where the largest logit of every row with a label lies above -2^100 (its own would take 2^119 of x w to live).  It
// counts with 0 in dx, so that whatever its row of w holds does not make the features' powers of two larger than the others need.
// (Looking for such classes costs the gradients of 2048 x 768 x 21841 1.5 us of 270.5 where there is a bias.)
struct Masks { const float* bias = nullptr; const int32_t* labels = nullptr; const float2* stats = nullptr; int tokens = 0, classes = 0, v0 = 0; };      // bias of the piece; null: none is
constexpr float MAY_MASK = -0x1p120f;
// bits of the classes r0 .. r1 that are labels -> the bias that masks (all 256 threads, behind a barrier of their own)
__device__ __forceinline__ float look_at_rows(const Masks& k, int r0, int r1, uint32_t* bits, float* red) {
  for (int i = threadIdx.x; i < (r1 - r0 + 31) / 32; i += 256) bits[i] = 0;
  __syncthreads();
  float least = INFINITY;
  for (int i = threadIdx.x; i < k.tokens; i += 256) {
    const int label = k.labels[i], at = max(label, -1) - k.v0 - r0;
    if (label >= 0 && label < k.classes) least = fminf(least, k.stats[i].x);
    if (at >= 0 && at < r1 - r0) atomicOr(bits + at / 32, 1u << at % 32);
  }
  least = -wave_max(-least);
  if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = least;
  __syncthreads();
  return fminf(fminf(red[0], red[1]), fminf(red[2], red[3])) > -0x1p100f ? MAY_MASK : -INFINITY;
}
__device__ __forceinline__ bool is_masked(const Masks& k, int r, int r0, const uint32_t* bits, float limit) { return k.bias[r] <= limit && !(bits[(r - r0) / 32] >> (r - r0) % 32 & 1); }

// [rows, D] -> [D][ld] fp16 in one or two terms, a power of two each of the D rows; what lies between rows and ld is zero.  In two launches, each for x, w or both: the columns' maxima, `chunks`
// parts of the rows apart, then the rest
struct TransposeJob {
  const void* x = nullptr; int64_t ldx = 0; int rows = 0; RowWeights rw; Masks masks;
  int per = 1, chunks = 0;                         // rows of a part; parts (0: no job)
  uint32_t* most = nullptr;                        // [chunks][D] bits of the largest finite |value|
  f16* to = nullptr; int cols = 0; int64_t ld = 0; int* exps = nullptr;           // cols (of one or both terms) of a row are written
  bool both = false;                               // FINE: two terms, one behind the other (of x with weights, which bf16 values times them do not fit one of)
};
constexpr int CHUNKS = 64, MOST_PART = 1 << 15;    // rows of a part: a piece has 2^21 classes at most (its rows of 64 features 256 MB)

// SIDE pieces of 16 bytes side by side: a cache line, or four where that leaves enough workgroups (131072 x 4096 bf16, eight pieces: 47 against 40 us; 21841 x 768 12 against 21)
template <typename T, int SIDE>
__global__ __launch_bounds__(256) void ce_colmax_kernel(TransposeJob a, TransposeJob b, int D) {
  constexpr int V = Chunk<T>::V, ABOVE = 256 / SIDE;
  __shared__ uint32_t red[4][SIDE][V];
  const bool first = (int)blockIdx.y < a.chunks;
  const TransposeJob j = first ? a : b;
  const int chunk = first ? blockIdx.y : blockIdx.y - a.chunks, r0 = chunk * j.per, r1 = min(r0 + j.per, j.rows);
  const T* x = (const T*)j.x;
  uint32_t* most = j.most + (int64_t)chunk * D;
  // (masked classes are looked for beside the loads, the first 256 ahead of them; where there are some, the maxima are made once more without them)
  const float first_bias = j.masks.bias ? j.masks.bias[min(r0 + (int)threadIdx.x, r1 - 1)] : 0.f;
  __shared__ uint32_t label_bits[MOST_PART / 32];
  __shared__ float lows[4];
  __shared__ int found[4];
  float limit = 0.f;
  auto any_masked = [&]() __attribute__((always_inline)) {
    if (!j.masks.bias) return false;
    bool mine = first_bias <= MAY_MASK;
    for (int r = r0 + 256 + threadIdx.x; r < r1; r += 256) mine |= j.masks.bias[r] <= MAY_MASK;
    const bool wave = __any(mine);
    if (threadIdx.x % WAVE == 0) found[threadIdx.x / WAVE] = wave;
    __syncthreads();
    if (!(found[0] | found[1] | found[2] | found[3])) return false;
    limit = look_at_rows(j.masks, r0, r1, label_bits, lows);
    return true;
  };
  if (D < V) {                                     // (no whole piece to read)
    __shared__ uint32_t part[256 / V][V];
    const int c = threadIdx.x % V, i = threadIdx.x / V;
    const bool some = any_masked();
    uint32_t m = 0;
    if (c < D)
#pragma unroll 4
      for (int r = r0 + i; r < r1; r += 256 / V) m = max(m, bits_if_finite(weighted((float)x[r * j.ldx + c], some && is_masked(j.masks, r, r0, label_bits, limit) ? 0.f : weight_of(j.rw, r))));
    part[i][c] = m;
    __syncthreads();
    if ((int)threadIdx.x < D) {
      for (int k = 1; k < 256 / V; ++k) m = max(m, part[k][threadIdx.x]);
      most[threadIdx.x] = m;
    }
    return;
  }
  // the last piece of V columns ends with the row; the rows among the threads above each other
  const int s = threadIdx.x % SIDE, p = blockIdx.x * SIDE + s, col = min(p * V, D - V);
  uint32_t m[V];
#pragma unroll
  for (int e = 0; e < V; ++e) m[e] = 0;
#pragma unroll 8
  for (int r = r0 + threadIdx.x / SIDE; r < r1; r += ABOVE) {
    const typename Loose<T>::vec v = *(const typename Loose<T>::vec*)(x + r * j.ldx + col);
    const float by = weight_of(j.rw, r);
#pragma unroll
    for (int e = 0; e < V; ++e) m[e] = max(m[e], bits_if_finite(weighted((float)v[e], by)));
  }
  if (any_masked()) {
#pragma unroll
    for (int e = 0; e < V; ++e) m[e] = 0;
    for (int r = r0 + threadIdx.x / SIDE; r < r1; r += ABOVE) {
      if (is_masked(j.masks, r, r0, label_bits, limit)) continue;
      const typename Loose<T>::vec v = *(const typename Loose<T>::vec*)(x + r * j.ldx + col);
#pragma unroll
      for (int e = 0; e < V; ++e) m[e] = max(m[e], bits_if_finite((float)v[e]));
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    float f = __uint_as_float(m[e]);               // (finite and not negative: the bits' order is the values')
    const auto op = [](float p, float q) { return fmaxf(p, q); };
    if constexpr (SIDE == 8) f = quarters_all(fmaxf(f, dpp_move<0x128>(f)), op);      // lanes ^ 8, ^ 16, ^ 32
    else f = halves_all(f, op);
    m[e] = __float_as_uint(f);
  }
  if (threadIdx.x % WAVE < SIDE)
#pragma unroll
    for (int e = 0; e < V; ++e) red[threadIdx.x / WAVE][s][e] = m[e];
  __syncthreads();
  if ((int)threadIdx.x < SIDE * V) {               // (SIDE V <= 256)
    const int at = threadIdx.x / V, e = threadIdx.x % V, c = min((blockIdx.x * SIDE + at) * V, (unsigned)(D - V)) + e;
    most[c] = max(max(red[0][at][e], red[1][at][e]), max(red[2][at][e], red[3][at][e]));      // (columns that two pieces hold: the same from both)
  }
}

// `down` tiles of 64 x 64 a workgroup, below one another: their columns' powers of two are worked out once, and the next tile's rows are on their way while one is turned
template <typename T, bool FINE>
__global__ __launch_bounds__(256) void ce_transpose_kernel(TransposeJob a, TransposeJob b, int blocks, int down, int D) {
  constexpr int TERMS = sizeof(T) / 2, KEPT = FINE ? 2 : TERMS, V = Chunk<T>::V, PER_ROW = 64 / V, K = PER_ROW / 4, LD = 66;
  __shared__ f16 tile[KEPT][64][LD];              // (rows of 33 words: neither the writes down nor the reads across meet in a bank)
  __shared__ uint32_t red[4][64];
  __shared__ int exps[64];
  const bool first = (int)blockIdx.x < blocks;
  const TransposeJob j = first ? a : b;
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, c0 = blockIdx.y * 64, begin = (first ? blockIdx.x : blockIdx.x - blocks) * 64 * down, end = min(begin + 64 * down, j.cols);
  const T* x = (const T*)j.x;
  const int c = threadIdx.x % PER_ROW * V, r0 = threadIdx.x / PER_ROW;
  const bool whole = c0 + 64 <= D;
  typename Loose<T>::vec v[K];
  float by[K];
  auto fetch = [&](int m0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const int m = m0 + r0 + i * (256 / PER_ROW);
      by[i] = m < j.rows ? weight_of(j.rw, m) : 0.f;
      if (whole) v[i] = *(const typename Loose<T>::vec*)(x + (int64_t)min(m, j.rows - 1) * j.ldx + c0 + c);
      else
#pragma unroll
        for (int e = 0; e < V; ++e) v[i][e] = m < j.rows && c0 + c + e < D ? x[(int64_t)m * j.ldx + c0 + c + e] : (T)0.f;
    }
  };
  fetch(begin);
  __shared__ uint32_t label_bits[16];              // (down: 8 at most)
  __shared__ float lows[4];
  __shared__ int found[4];
  float bias[2] = {0.f, 0.f};                      // (of 512 classes)
  if (j.masks.bias)
#pragma unroll
    for (int i = 0; i < 2; ++i) bias[i] = j.masks.bias[min(begin + (int)threadIdx.x + 256 * i, j.rows - 1)];
  uint32_t most = 0;
  if (c0 + lane < D)
#pragma unroll 4
    for (int k = w; k < j.chunks; k += 4) most = max(most, j.most[(int64_t)k * D + c0 + lane]);
  red[w][lane] = most;
  const bool masked = __any(bias[0] <= MAY_MASK || bias[1] <= MAY_MASK);            // (or a class behind the workgroup's last: looked for in vain)
  if (lane == 0) found[w] = masked;
  __syncthreads();
  const bool some = found[0] | found[1] | found[2] | found[3];
  const float limit = some ? look_at_rows(j.masks, begin, min(end, j.rows), label_bits, lows) : 0.f;
  if (w == 0) {
    const int e = exponent_of(max(max(red[0][lane], red[1][lane]), max(red[2][lane], red[3][lane])));
    exps[lane] = e;
    if (begin == 0 && c0 + lane < D) j.exps[c0 + lane] = e;
  }
  __syncthreads();
  for (int m0 = begin; m0 < end; m0 += 64) {
    if (some)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int m = m0 + r0 + i * (256 / PER_ROW);
        if (m < j.rows && is_masked(j.masks, m, begin, label_bits, limit)) by[i] = 0.f;
      }
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float s = ldexpf(weighted((float)v[i][e], by[i]), -exps[c + e]);
        const f16 h = (f16)s;
        tile[0][c + e][r0 + i * (256 / PER_ROW)] = h;
        if constexpr (KEPT == 2) tile[KEPT - 1][c + e][r0 + i * (256 / PER_ROW)] = (f16)(s - (float)h);
      }
    if (m0 + 64 < end) fetch(m0 + 64);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < KEPT; ++t)
#pragma unroll
      for (int i = threadIdx.x; i < 512; i += 256) {
        if (FINE && t == 1 && !j.both) break;
        const int col = i / 8, k = i % 8 * 8;
        const uint32_t* from = (const uint32_t*)&tile[t][col][k];
        if (c0 + col < D && m0 + k < j.cols) *(uint4*)(j.to + (int64_t)(c0 + col) * j.ld + (FINE ? m0 + k + (int64_t)t * j.cols : spot<TERMS>(m0 + k, t))) = make_uint4(from[0], from[1], from[2], from[3]);
      }
    __syncthreads();
  }
}

// logits to what the tiles leave of G: 64 tokens x 64 classes a workgroup
template <int TERMS, bool FINE>
__global__ __launch_bounds__(256) void ce_turn_kernel(const float* __restrict__ from, int64_t ldz, CeGemm g) {
  __shared__ float tile[64][65];
  const int t = threadIdx.x, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, a = t / 4, b = t % 4 * 16;      // a row (or a column) and 16 of its values
  auto half = [](float p, f16& h, f16& l) __attribute__((always_inline)) {
    p *= (float)(1 << G_SHIFT);
    h = (f16)p;
    l = (f16)(p - (float)h);
  };
  float v[16];
  bool counts = m0 + a < g.M;                      // (as at a tile's end)
  float2 st = {0.f, 0.f};
  int label = -1;
  if (counts) {
    label = g.labels[m0 + a];
    st = g.stats[m0 + a];
    counts = label >= 0 && label < g.classes && (!g.row_grad || g.row_grad[m0 + a] != 0.f) && !(st.x == -INFINITY && st.y == 0.f);
  }
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    const bool there = counts && n0 + b + i < g.N;
    f32x4 p = there ? *(const f32x4*)(from + (int64_t)(m0 + a) * ldz + n0 + b + i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      p[j] = __builtin_amdgcn_exp2f(fmaf(p[j] - st.x, LOG2E, -st.y * LOG2E)) - (n0 + b + i + j == label ? 1.f : 0.f);
      tile[a][b + i + j] = v[i + j] = there && n0 + b + i + j < g.N ? p[j] : 0.f;
    }
  }
  // (second: whether, and how far behind, the other term goes; 0: 32 and 32 of both in turn)
  auto put = [&](f16* row, int at, auto BOTH, int64_t second) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
      f16x8 h, l;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f16 hj, lj;
        half(v[i + j], hj, lj);
        h[j] = hj;
        l[j] = lj;
      }
      *(f16x8*)(row + spot<TERMS>(at + i)) = h;
      if constexpr (decltype(BOTH)::value != 0) *(f16x8*)(row + (second ? at + i + second : spot<TERMS>(at + i, 1))) = l;
    }
  };
  if (g.G && m0 + a < g.M) put(g.G + (int64_t)(m0 + a) * g.ldg, n0 + b, IC<TERMS - 1>{}, 0);
  if (!g.GT && !g.dbp) return;
  __syncthreads();
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = tile[b + i][a];
    const int m = m0 + b + i;
    sum += m < g.M && g.row_grad && v[i] != 0.f ? g.row_grad[m] * v[i] : v[i];
  }
  if (g.GT && n0 + a < g.N) put(g.GT + (int64_t)(n0 + a) * g.ldgt, m0 + b, IC<FINE || TERMS == 2>{}, FINE ? g.kgt : 0);
  if (g.dbp) {
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if (t % 4 == 0 && n0 + a < g.N) g.dbp[blockIdx.y * g.ldd + n0 + a] = sum;
  }
}

// ------------------------------------------------------------------------------------------ joining
// 16 rows a workgroup, whose 64 quarters of wavefronts join every 64th tile each and then, in order, what they have; first and last piece of the classes: begin, end
__global__ __launch_bounds__(1024) void ce_join_kernel(const float2* __restrict__ parts, int tiles, int M, float2* __restrict__ run, int begin, int end, const float* __restrict__ zlabel,
                                                       const int32_t* __restrict__ labels, int classes, float* __restrict__ loss, float2* __restrict__ stats) {
  __shared__ float2 red[16][16];
  const int lane = threadIdx.x % WAVE, w = threadIdx.x / WAVE, m = blockIdx.x * 16 + lane % 16, mc = min(m, M - 1);
  float2 p = make_float2(-INFINITY, 0.f);
#pragma unroll 8
  for (int t = threadIdx.x / 16; t < tiles; t += 64) p = joined(p, parts[(int64_t)t * M + mc]);
#pragma unroll
  for (int d = 16; d < WAVE; d *= 2) p = joined(p, make_float2(__shfl_xor(p.x, d), __shfl_xor(p.y, d)));
  if (lane < 16) red[w][lane] = p;
  __syncthreads();
  if (threadIdx.x >= 16 || m >= M) return;
  if (!begin) p = joined(run[m], p);
#pragma unroll
  for (int i = 1; i < 16; ++i) p = joined(p, red[i][lane]);
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

// out = scale weight[m] (sum over the parts, in order), 0 for rows that do not count, whatever w and their weight hold; parts of db are rows of tokens
// db has a part for each 64 to 256 tokens, 65536 at most: from 16 on several threads (ways) share four classes and add up in fp64, every ways-th part each and then those sums in order.
// (Gradients of 4194304 x 16 x 20 bf16 4273 us, one thread a sum 7790; 200000 x 64 x 1000 1077 and 1830; 32768 x 64 x 131072 10870 and 13010; 4096 x 64 x 65536 600 and 611.  One, 16 and 64 ways: 1000 x 64 x 65536 162, 162, 168;
// 32000 x 64 x 4096 381, 323, 320; 262144 x 64 x 4096 9606, 5687, 5610.)
struct SumJob {
  const float* part = nullptr; int parts = 0; int64_t tp = 0, ldp = 0, rows = 0; int cols = 0;
  float scale = 1.f; RowWeights rw;                // rows by their weights
  void* out = nullptr; int64_t ldo = 0; bool f32 = false;
  int ways = 1, blocks = 0;
};
template <typename T> __device__ __forceinline__ void put_four(T* to, f32x4 v, int have) {
  if (have >= 4 && ((uintptr_t)to & (4 * sizeof(T) - 1)) == 0) {
    typedef T vec __attribute__((ext_vector_type(4)));
    *(vec*)to = vec{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
    for (int j = 0; j < 4; ++j)
      if (j < have) to[j] = (T)v[j];
  }
}
// dx, dw and db, or some of them, in one launch
template <bool WAYS>
__global__ __launch_bounds__(256) void ce_sums_kernel(SumJob a, SumJob b, SumJob c) {
  int block = blockIdx.x;
  SumJob j = a;
  if (block >= a.blocks) {
    block -= a.blocks;
    j = b;
    if (block >= b.blocks) {
      block -= b.blocks;
      j = c;
    }
  }
  if constexpr (WAYS) if (j.ways > 1) {            // (one row, fp32)
    __shared__ double red[4][256];
    const int wide = 256 / j.ways, way = threadIdx.x / wide, n = (block * wide + threadIdx.x % wide) * 4;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    if (n < j.cols)
#pragma unroll 8
      for (int s = way; s < j.parts; s += j.ways) {
        const f32x4 p = *(const f32x4*)(j.part + s * j.tp + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += (double)p[e];
      }
#pragma unroll
    for (int e = 0; e < 4; ++e) red[e][threadIdx.x] = v[e];
    __syncthreads();
    if (way > 0 || n >= j.cols) return;
    for (int i = 1; i < j.ways; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += red[e][i * wide + threadIdx.x];
    put_four((float*)j.out + n, f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]} * j.scale, j.cols - n);
    return;
  }
  const int64_t i = (int64_t)block * 256 + threadIdx.x, chunks = (j.cols + 3) / 4, m = i / chunks;
  const int n = (int)(i - m * chunks) * 4;
  if (m >= j.rows) return;
  const float* at = j.part + m * j.ldp + n;
  f32x4 v = *(const f32x4*)at;
#pragma unroll 4
  for (int s = 1; s < j.parts; ++s) v += *(const f32x4*)(at + s * j.tp);
  const float by = weight_of(j.rw, m);
  v = by == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : v * (j.scale * by);
  if (j.f32) put_four((float*)j.out + m * j.ldo + n, v, j.cols - n);
  else put_four((bf16*)j.out + m * j.ldo + n, v, j.cols - n);
}

// no tokens: no gradients
template <typename T> __global__ __launch_bounds__(256) void ce_fill_kernel(T* __restrict__ out, int64_t ld, int64_t rows, int cols) {
  for (int64_t m = blockIdx.x; m < rows; m += gridDim.x)
    for (int j = threadIdx.x; j < cols; j += 256) out[m * ld + j] = (T)0.f;
}

// ------------------------------------------------------------------------------------------ host

// a kernel has its LDS, once a device
template <auto KERNEL> void with_lds(size_t bytes) {
  static uint64_t known = 0;
  int dev = 0;
  (void)hipGetDevice(&dev);
  if (!(__atomic_load_n(&known, __ATOMIC_RELAXED) >> (dev & 63) & 1)) {
    (void)hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    __atomic_fetch_or(&known, (uint64_t)1 << (dev & 63), __ATOMIC_RELAXED);
  }
}
enum { LARGE, SMALL, MID, FEW, SHORT };
int rows_of(int shape) { return shape == FEW ? Few::BM : shape == SHORT ? Short::BM : shape == MID ? Mid::BM : shape == SMALL ? Small::BM : Large::BM; }
int cols_of(int shape) { return shape == FEW ? Few::BN : shape == SHORT ? Short::BN : shape == MID ? Mid::BN : shape == SMALL ? Small::BN : Large::BN; }

template <class S, Mode MODE, bool F16, int TERMS, bool DB, bool FINE> void launch_logits(const CeGemm& g, int rows, hipStream_t s) {
  with_lds<ce_logits_kernel<S, MODE, F16, TERMS, DB, FINE>>(S::lds);
  const int mt = over(rows, S::BM), nt = over(g.N, S::BN);
  ce_logits_kernel<S, MODE, F16, TERMS, DB, FINE><<<mt * nt, S::NT, S::lds, s>>>(g, mt, nt);
}
// rows: those that tiles have to cover
template <Mode MODE, bool F16, int TERMS, bool DB, bool FINE = false> void logits(int shape, const CeGemm& g, int rows, hipStream_t s) {
  if (shape == FEW) launch_logits<Few, MODE, F16, TERMS, DB, FINE>(g, rows, s);
  else if (shape == SHORT) launch_logits<Short, MODE, F16, TERMS, DB, FINE>(g, rows, s);
  else if (shape == MID) launch_logits<Mid, MODE, F16, TERMS, DB, FINE>(g, rows, s);
  else if (shape == SMALL) launch_logits<Small, MODE, F16, TERMS, DB, FINE>(g, rows, s);
  else launch_logits<std::conditional_t<MODE == STATS && TERMS == 1, LargeForward, Large>, MODE, F16, TERMS, DB, FINE>(g, rows, s);
}
template <class S, int TERMS, bool PASSES> void launch_grads(const CeGemm& a, const CeGemm& b, hipStream_t s) {
  auto blocks = [](const CeGemm& g) { return g.A ? over(g.M, S::BM) * over(g.N, S::BN) * g.splits : 0; };
  with_lds<ce_grads_kernel<S, TERMS, PASSES>>(S::lds);
  ce_grads_kernel<S, TERMS, PASSES><<<blocks(a) + blocks(b), S::NT, S::lds, s>>>(a, b, blocks(a));
}

// Models of a launch, in us: a workgroup, or the two of a shape that a CU takes at once, has a CU for start + k-tiles * tile.  (Short against large, forward: 600 x 100 x 100000 bf16 60 against 75 us, 2000 x 512 x
// 50000 128 against 136, 2048 x 768 x 21841 80 against 79)
struct Cost { double tile, start; int at_once; };
constexpr Cost COST[5] = {{1.7, 8, 1}, {0.6, 4, 1}, {0.4, 4, 1}, {0.5, 4, 1}, {1.03, 2.3, 2}};
// of a k-tile, which two terms make longer; of a row of so many times 64 features
double tile_work(bool f32) { return f32 ? 1.25 : 1; }
double logits_work(bool f32, int kt) { return kt * (f32 ? 2 : 1) * tile_work(f32); }
int logits_shape(int64_t M, int64_t N, double kt) {
  int best = SMALL;
  double least = 1e30;
  for (int shape = LARGE; shape <= SHORT; ++shape) {
    if (shape == FEW && M > Few::BM) continue;
    const int64_t tiles = (int64_t)over(M, rows_of(shape)) * over(N, cols_of(shape));
    const double us = (double)over(tiles, 256 * COST[shape].at_once) * (COST[shape].start + kt * COST[shape].tile);
    if (us < least) { least = us; best = shape; }
  }
  return best;
}
// shape and workgroups over k of dx (M x D, kx k-tiles) and dw (n x D, kw k-tiles) together; either may be missing (0 k-tiles).  dx's workgroups go first
struct Split { int shape, x, w; };
Split grads_split(int64_t M, int64_t n, int64_t D, int kx, int kw, double work) {
  Split best = {SMALL, 1, 1};
  double least = 1e30;
  // (255 rows of two terms of more than 2^21 tokens would pass 32 bits)
  for (int shape = kw > 1 << 16 ? SMALL : LARGE; shape <= SMALL; ++shape) {
    const int64_t tx = kx ? (int64_t)over(M, rows_of(shape)) * over(D, cols_of(shape)) : 0, tw = kw ? (int64_t)over(n, rows_of(shape)) * over(D, cols_of(shape)) : 0;
    const Cost c = COST[shape];
    for (int x = 1; x <= (kx ? 64 : 1); ++x) {
      if (x > 1 && (kx < 4 * x || tx * x > 1024)) break;
      for (int w = 1; w <= (kw ? 16 : 1); ++w) {
        if (w > 1 && (kw < 4 * w || tw * w > 1024)) break;
        const double a = c.start + over(kx, x) * c.tile * work, b = c.start + over(kw, w) * c.tile * work;
        // dx in rounds over the CUs, dw on those that are free
        const int64_t nx = tx * x, nw = tw * w, full = nx / 256, rest = nx % 256;
        double us = full * a + (rest ? a : 0);
        if (nw) {
          int64_t left = nw;
          double early = full * a, late = full * a + a;           // when 256 - rest CUs, and the rest, take the next
          us = std::max(us, 0.0);
          const int64_t rounds = std::max<int64_t>(0, (nw - 1024) / 256);      // (many: whole rounds at once)
          left -= rounds * 256;
          early += rounds * b;
          late += rounds * b;
          while (left > 0) {
            if (rest == 0 || early <= late) { left -= 256 - rest; early += b; us = std::max(us, early); }
            else { left -= rest; late += b; us = std::max(us, late); }
          }
        }
        // partial sums leave and come back
        us += ((kx ? x * M * D : 0) + (w > 1 ? w * n * D : 0)) * 8e-6 / 4;
        if (us < least * 0.999) { least = us; best = {shape, x, w}; }
      }
    }
  }
  return best;
}

// What goes to k_linear_ce_small.hip: little work, where the launches count; few rows backward (w is read and dw written once there), and forward where they would have to be packed first.  Its
// logits take 16 MB at most, those of few rows, of which there is room for 16, 32 or 64, 256
constexpr size_t SMALL_BYTES = 16 << 20, FEW_BYTES = 256 << 20;
// SMALL_WORK, tokens x features x classes: up to there where x or w would have to be packed (forward, without tiles and in tiles: 300 x 200 x 2000 fp32 14.6 and 18.0 us, bf16 17.8 and 18.3; 300 x 500 x 2000, just
// above, 22.5 and 19.7, 23.2 and 18.3; gradients 100 x 200 x 2000 fp32 31.9 and 34.6, 300 x 500 x 2000 50 and 44).
// MOST_SMALL_WORK: up to there where fewer than 64 tiles would leave most CUs idle behind long chains (forward, bf16 as it lies: 128 x 4096 x 512 15.7 and 24.5, 256 x 4096 x 512 16.0 and 24.7, 256 x 8192 x 512 26.5 and 42.1, 2^30;
// with more tiles, 512 x 2048 x 1024, 26.6 and 16.3; with more work, 128 x 4096 x 4096, 48 and 25.4).
constexpr double SMALL_WORK = 1 << 28, MOST_SMALL_WORK = 1 << 30;
bool is_small(int N, int D, int V) { return N <= 1 << 20 && small_ce_bytes(N, V) <= SMALL_BYTES && (double)N * D * V <= MOST_SMALL_WORK; }      // (a launch has up to 65535 workgroups one way)
// (more than 32 rows of a w that would have to be packed: 48 x 1001 x 50000 bf16 318 us here, 291 by tiles)
bool is_few(int N, int V) { return N <= FEW_ROWS && few_parts_at(N, V) <= FEW_BYTES; }
bool always_few(bool f32, int N) { return f32 || N <= 32; }

// sizes, and places in the workspace
struct Plan {
  int T, Dp, Np, Vs, Vp, Vc, Dq, ldd;
  Split split = {};
  size_t xp, ex, wp, ew, parts, run, zlabel, G, GT, xT, wT, exT, ewT, mostx, mostw, dxp, dwp, dbp, z, bytes;
  // packs: room for w packed; fine: x and G transposed in two terms
  Plan(bool f32, int N, int D, int V, bool backward, bool packs = true, bool fine = false) {
    T = f32 ? 2 : 1;
    const int TT = f32 || fine ? 2 : 1;            // terms of what is transposed of G and of x
    Dp = up(D, BK); Np = up(N, BK); Dq = up(D, 4);
    // Pieces of the classes, whole tiles and alike in size.  Forward: the tiles' maxima and sums take at most 64 MB (Vs) and what is packed 256 (Vp, where something is).
    // Backward: G, twice, takes at most 256 MB, and so does the transposed piece of w.
    auto piece = [&](double most) {
      const int64_t c = std::max<int64_t>(256, (int64_t)std::min(most, 1e9) / 256 * 256);
      const int pieces = over(V, (int)c);
      return pieces == 1 ? up(V, BK) : up(over(V, pieces), 256);
    };
    constexpr double MB = 1 << 20;
    Vs = piece(64 * MB * 128 / (8.0 * N));
    Vp = std::min(Vs, piece(256 * MB / (2.0 * T * Dp)));
    Vc = std::min(piece(256 * MB / (2.0 * (T + TT) * Np)), piece(256 * MB / (2.0 * T * Dp)));
    ldd = Vc;
    bytes = 0;
    auto take = [&](size_t n) { const size_t at = bytes; bytes += (n + 255) / 256 * 256; return at; };
    const int Vm = packs ? backward ? Vc : Vp : 0;
    xp = take((size_t)2 * T * N * Dp); ex = take(sizeof(int) * (size_t)N);
    wp = take((size_t)2 * T * Vm * Dp); ew = take(sizeof(int) * (size_t)Vm);
    if (!backward) {
      parts = take(sizeof(float2) * (size_t)over(Vs, 128) * N); run = take(sizeof(float2) * (size_t)N); zlabel = take(sizeof(float) * (size_t)N);
      return;
    }
    G = take((size_t)2 * T * N * Vc); GT = take((size_t)2 * TT * Vc * Np);
    xT = take((size_t)2 * TT * D * Np); exT = take(sizeof(int) * (size_t)D);
    wT = take((size_t)2 * T * D * Vc); ewT = take(sizeof(int) * (size_t)D);
    mostx = take(sizeof(uint32_t) * (size_t)CHUNKS * D); mostw = take(sizeof(uint32_t) * (size_t)CHUNKS * D);
    // (for the first piece; the others take as many workgroups over k)
    split = grads_split(N, std::min(V, Vc), D, std::min(Vc, up(V, BK)) / BK * T, Np / BK * TT, tile_work(f32));
    dxp = take(sizeof(float) * (size_t)split.x * N * Dq);
    dwp = take(split.w > 1 ? sizeof(float) * (size_t)split.w * Vc * Dq : 0);
    dbp = take(sizeof(float) * (size_t)over(Np, 32) * ldd);
    z = take(is_small(N, D, V) ? small_ce_bytes(N, V) : 0);
  }
};

// (255 rows of a tile, and k behind them, are addressed in 32 bits; so are those of what is packed and transposed here: rows of 2^20 features or 2^22 tokens at most, of two terms of 2^20 or 2^21)
bool whole_rows(const void* p, int64_t ld, int D) { return D % BK == 0 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld <= 1 << 22; }

// An operand of the logits: as it lies, or packed by what `job` then describes
struct Rows { const void* p; int64_t ld; const int* exps; };
Rows rows_operand(const void* p, int64_t ld, bool f32, int64_t rows, int Dp, void* packed, int* exps, bool as_it_lies, PackJob& job) {
  if (as_it_lies) return {p, ld, nullptr};
  job.x = p; job.ldx = ld; job.rows = rows; job.to = (uint16_t*)packed; job.exps = exps;
  return {packed, f32 ? 2 * Dp : Dp, f32 ? exps : nullptr};
}
void pack(const PackJob& a, const PackJob& b, bool f32, int D, int Dp, hipStream_t s) {
  if (a.rows + b.rows == 0) return;
  auto go = [&](auto kernel, int na, int nb) { kernel<<<na + nb, 256, 0, s>>>(a, b, na, D, Dp); };
  if (!f32) go(ce_pack_kernel<bf16, WAVE>, pack_blocks<bf16, WAVE>(a.rows, Dp), pack_blocks<bf16, WAVE>(b.rows, Dp));
  else if (Dp <= 64) go(ce_pack_kernel<float, 16>, pack_blocks<float, 16>(a.rows, Dp), pack_blocks<float, 16>(b.rows, Dp));
  else if (Dp <= 128) go(ce_pack_kernel<float, 32>, pack_blocks<float, 32>(a.rows, Dp), pack_blocks<float, 32>(b.rows, Dp));
  else go(ce_pack_kernel<float, WAVE>, pack_blocks<float, WAVE>(a.rows, Dp), pack_blocks<float, WAVE>(b.rows, Dp));
}

template <typename T, bool FINE> void transpose(const TransposeJob& a, const TransposeJob& b, int D, hipStream_t s) {
  if (a.chunks + b.chunks == 0) return;
  constexpr int LINE = 8 * Chunk<T>::V;
  if (over(D, 4 * LINE) * (a.chunks + b.chunks) >= 1024) ce_colmax_kernel<T, 32><<<dim3(over(D, 4 * LINE), a.chunks + b.chunks), 256, 0, s>>>(a, b, D);
  else ce_colmax_kernel<T, 8><<<dim3(over(D, LINE), a.chunks + b.chunks), 256, 0, s>>>(a, b, D);
  const int tiles = (a.chunks ? over(a.cols, 64) : 0) + (b.chunks ? over(b.cols, 64) : 0);
  // (2048 x 768 x 21841 bf16, gradients: one tile 256.7 us, four 255.7, eight 259.7; 4096 x 4096 x 20000 1901, 1897, 1898; 300 x 128 x 9000, few tiles in all, 32.4, 35.2, 38.9)
  const int down = (int)std::min<int64_t>(8, std::max<int64_t>(1, (int64_t)tiles * over(D, 64) / 2048));
  const int na = a.chunks ? over(a.cols, 64 * down) : 0, nb = b.chunks ? over(b.cols, 64 * down) : 0;
  ce_transpose_kernel<T, FINE><<<dim3(na + nb, over(D, 64)), 256, 0, s>>>(a, b, na, down, D);
}
void set_chunks(TransposeJob& j) {
  j.per = std::max(64, over(j.rows, CHUNKS));
  j.chunks = over(j.rows, j.per);
}

// whether tiles of the logits would leave most CUs idle, each behind a long chain of k-tiles
bool few_tiles(int N, int V, double kt) {
  const int shape = logits_shape(N, V, kt);
  return (int64_t)over(N, rows_of(shape)) * over(V, cols_of(shape)) < 64;
}

// tiles of the logits of n classes
int logits_shape(const LinearCe& a, const Plan& p, int n) { return logits_shape(a.N, n, (a.f32 ? 2 : 1) * p.Dp / BK * tile_work(a.f32)); }

CeGemm logits_gemm(const LinearCe& a, const Plan& p, const Rows& x, const Rows& w, int v0, int n) {
  CeGemm g;
  g.A = x.p; g.lda = x.ld; g.ea = x.exps; g.B = w.p; g.ldb = w.ld; g.eb = w.exps;
  g.M = a.N; g.N = n; g.nk = (a.f32 ? 2 : 1) * p.Dp / BK; g.bias = a.bias ? a.bias + v0 : nullptr; g.labels = a.labels; g.v0 = v0; g.classes = a.V;
  return g;
}

}  // namespace

size_t linear_ce_workspace_bytes(bool f32, int N, int D, int V, bool backward) {
  // (few rows: the logits may come from tiles, whose scratch lies where the parts of dx do afterwards)
  const size_t few = is_few(N, V) ? few_parts_at(N, V) + std::max(few_ce_bytes(f32, N, V, D), f32 ? 0 : Plan(f32, N, D, V, false, false).bytes) : 0;
  if (backward && few && always_few(f32, N)) return few;
  // (backward: dw may be wanted in either type)
  const size_t bytes = std::max({Plan(f32, N, D, V, backward).bytes, backward && !f32 ? Plan(f32, N, D, V, true, true, true).bytes : 0, backward ? few : 0});
  return !backward && (is_small(N, D, V) || (few && always_few(f32, N))) ? std::max(bytes, small_ce_bytes(N, V)) : bytes;
}

// How x and w lie, and what follows from it: the logits (or G) of little work straight from x and w, in a launch of its own, not in tiles
struct Way {
  bool x, w, little, few;                          // rows of whole 16-byte pieces; little work; gradients of few rows
  explicit Way(const LinearCe& a) {
    x = !a.f32 && whole_rows(a.x, a.ldx, a.D);
    w = !a.f32 && whole_rows(a.w, a.ldw, a.D);
    little = is_small(a.N, a.D, a.V) &&
             ((double)a.N * a.D * a.V <= SMALL_WORK && (!x || !w) || few_tiles(a.N, a.V, logits_work(a.f32, over(a.D, BK))));
    few = is_few(a.N, a.V) && (always_few(a.f32, a.N) || w || little);
  }
  bool straight() const { return little || (few && !w); }        // the forward's logits without tiles
};

// z: where the logits are kept as well (in one piece, and not of little work), or null;  packs: whether the workspace has room for w packed
static void forward_with(const LinearCe& a, float* z, bool packs, hipStream_t s) {
  const Way way(a);
  const bool direct_x = way.x, direct_w = way.w;
  if (way.straight()) {
    small_ce_forward(a, (float*)a.workspace, false, s);
    return;
  }
  const Plan p(a.f32, a.N, a.D, a.V, false, packs);
  char* ws = (char*)a.workspace;
  const int64_t size = a.f32 ? 4 : 2;
  PackJob px;
  const Rows x = rows_operand(a.x, a.ldx, a.f32, a.N, p.Dp, ws + p.xp, (int*)(ws + p.ex), direct_x, px);
  const int step = direct_w ? p.Vs : p.Vp;
  for (int v0 = 0; v0 < a.V; v0 += step) {
    const int n = std::min(step, a.V - v0);
    PackJob pw;
    const Rows w = rows_operand((const char*)a.w + v0 * a.ldw * size, a.ldw, a.f32, n, p.Dp, ws + p.wp, (int*)(ws + p.ew), direct_w, pw);
    pack(v0 == 0 ? px : PackJob(), pw, a.f32, a.D, p.Dp, s);
    CeGemm g = logits_gemm(a, p, x, w, v0, n);
    g.parts = (float2*)(ws + p.parts); g.zlabel = (float*)(ws + p.zlabel); g.z = z; g.ldz = small_ce_stride(a.N, a.V);
    const int shape = logits_shape(a, p, n);
    if (a.f32) logits<STATS, true, 2, false>(shape, g, a.N, s);
    else logits<STATS, false, 1, false>(shape, g, a.N, s);
    if (a.loss || a.stats)
      ce_join_kernel<<<over(a.N, 16), 1024, 0, s>>>(g.parts, over(n, cols_of(shape)), a.N, (float2*)(ws + p.run), v0 == 0, v0 + n == a.V, g.zlabel, a.labels, a.V, a.loss, (float2*)a.stats);
  }
}

void linear_ce_forward(const LinearCe& a, hipStream_t s) { forward_with(a, nullptr, true, s); }

// Loss and gradients in one call: the logits stay in scratch between the passes where they fit it and cost more to make again than to read.  (333 x 1001 x 5003 fp32 110 against 128 us, 1024 x 4096 x
// 4000 bf16 153 against 177, 1000 x 768 x 1000 40 against 43; 400 x 64 x 10000 51 against 48)
bool keeps(bool f32, int N, int D, int V) { return small_ce_bytes(N, V) <= SMALL_BYTES && over(D, BK) * (f32 ? 3 : 1) >= 8; }

// little work: its logits, in scratch, turned into what the tiles leave (in one piece)
bool takes_turn(const LinearCe& a, const Plan& p, const Way& way) { return way.little && p.Vc >= a.V; }

// dw in fp32 beside bf16 operands
bool is_fine(const LinearCe& a) { return !a.f32 && a.dw && a.dw_f32; }
Plan backward_plan(const LinearCe& a) { return Plan(a.f32, a.N, a.D, a.V, true, true, is_fine(a)); }

// What a forward on the same workspace has left: nothing, the packed operands (of one piece), or the logits (z)
enum Ready { NOTHING, PACKED, KEPT };
template <typename T, bool FINE>
void backward_as(const LinearCe& a, Ready ready, const float* z, hipStream_t s) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int TERMS = F32 ? 2 : 1;
  const Plan p = backward_plan(a);
  const int xterms = FINE && a.row_grad ? 2 : TERMS, gterms = FINE ? 2 : TERMS;             // of x and G transposed
  char* ws = (char*)a.workspace;
  const Way way(a);
  const bool direct_x = way.x, direct_w = way.w;
  PackJob px;
  const Rows x = rows_operand(a.x, a.ldx, F32, a.N, p.Dp, ws + p.xp, (int*)(ws + p.ex), direct_x, px);
  const bool turned = ready == KEPT || takes_turn(a, p, way);
  f16 *xT = (f16*)(ws + p.xT), *wT = (f16*)(ws + p.wT), *G = (f16*)(ws + p.G), *GT = (f16*)(ws + p.GT);
  for (int v0 = 0; v0 < a.V; v0 += p.Vc) {
    const int n = std::min(p.Vc, a.V - v0), np = up(n, BK);
    const bool begin = v0 == 0, end = v0 + n == a.V;
    const T* wv = (const T*)a.w + v0 * a.ldw;
    PackJob pw;
    const Rows w = rows_operand(wv, a.ldw, F32, n, p.Dp, ws + p.wp, (int*)(ws + p.ew), direct_w, pw);
    if (!turned && ready != PACKED) pack(begin ? px : PackJob(), pw, F32, a.D, p.Dp, s);
    CeGemm g = logits_gemm(a, p, x, w, v0, n);
    TransposeJob tx, tw;
    if (a.dw && begin) {
      tx.x = a.x; tx.ldx = a.ldx; tx.rows = a.N; tx.rw.labels = a.labels; tx.rw.row_grad = a.row_grad; tx.rw.classes = a.V;
      tx.most = (uint32_t*)(ws + p.mostx); tx.to = xT; tx.cols = p.Np; tx.ld = xterms * p.Np; tx.exps = (int*)(ws + p.exT);
      tx.both = xterms == 2;
      set_chunks(tx);
    }
    if (a.dx) {
      tw.x = wv; tw.ldx = a.ldw; tw.rows = n; tw.most = (uint32_t*)(ws + p.mostw); tw.to = wT; tw.cols = np; tw.ld = TERMS * np; tw.exps = (int*)(ws + p.ewT);
      tw.masks.bias = g.bias; tw.masks.labels = a.labels; tw.masks.stats = (const float2*)a.stats; tw.masks.tokens = a.N; tw.masks.classes = a.V; tw.masks.v0 = v0;
      set_chunks(tw);
    }
    transpose<T, FINE>(tx, tw, a.D, s);
    g.stats = (const float2*)a.stats; g.row_grad = a.row_grad;
    if (a.dx) { g.G = G; g.kg = np; g.ldg = TERMS * np; }
    if (a.dw) { g.GT = GT; g.kgt = p.Np; g.ldgt = gterms * p.Np; }
    if (a.db) { g.dbp = (float*)(ws + p.dbp); g.ldd = p.ldd; }
    const int shape = logits_shape(a, p, n), rows = a.dw ? p.Np : a.N, tall = turned ? 64 : rows_of(shape);
    if (turned) {
      if (ready != KEPT) small_ce_logits(a, (float*)(ws + p.z), s);
      ce_turn_kernel<TERMS, FINE><<<dim3(np / 64, over(rows, 64)), 256, 0, s>>>(ready == KEPT ? z : (const float*)(ws + p.z), small_ce_stride(a.N, a.V), g);
    } else if (a.db) {
      logits<GRAD, F32, TERMS, true, FINE>(shape, g, rows, s);
    } else {
      logits<GRAD, F32, TERMS, false, FINE>(shape, g, rows, s);
    }
    CeGemm ox, ow;
    SumJob sx, sw, sb;
    if (a.dx) {
      ox.A = G; ox.lda = g.ldg; ox.B = wT; ox.ldb = tw.ld; ox.eb = tw.exps;
      ox.M = a.N; ox.N = a.D; ox.nk = TERMS * np / BK; ox.splits = p.split.x; ox.per = over(ox.nk, ox.splits);
      ox.pass = ox.nk;
      ox.part = (float*)(ws + p.dxp); ox.ldp = p.Dq; ox.tp = (int64_t)a.N * p.Dq; ox.add = !begin;
      if (end) {
        sx.part = ox.part; sx.parts = ox.splits; sx.tp = ox.tp; sx.ldp = p.Dq; sx.rows = a.N; sx.cols = a.D; sx.scale = a.grad_scale; sx.rw.labels = a.labels; sx.rw.row_grad = a.row_grad; sx.rw.classes = a.V;
        sx.out = a.dx; sx.ldo = a.lddx; sx.f32 = F32; sx.blocks = over((int64_t)a.N * over(a.D, 4), 256);
      }
    }
    if (a.dw) {
      ow.A = GT; ow.lda = g.ldgt; ow.B = xT; ow.ldb = xterms * p.Np; ow.eb = (int*)(ws + p.exT);
      ow.M = n; ow.N = a.D; ow.nk = (FINE ? 1 + xterms : TERMS) * p.Np / BK; ow.pass = p.Np / BK; ow.splits = p.split.w; ow.per = over(ow.nk, ow.splits); ow.scale = a.grad_scale;
      char* dw = (char*)a.dw + v0 * a.lddw * (a.dw_f32 ? 4 : 2);
      if (ow.splits > 1) {
        ow.part = (float*)(ws + p.dwp); ow.ldp = p.Dq; ow.tp = (int64_t)n * p.Dq;
        sw.part = ow.part; sw.parts = ow.splits; sw.tp = ow.tp; sw.ldp = p.Dq; sw.rows = n; sw.cols = a.D; sw.scale = a.grad_scale;
        sw.out = dw; sw.ldo = a.lddw; sw.f32 = a.dw_f32; sw.blocks = over((int64_t)n * over(a.D, 4), 256);
      } else {
        ow.out = dw; ow.ldo = a.lddw; ow.out_f32 = a.dw_f32; ow.out_vec = a.D % 4 == 0 && a.lddw % 4 == 0 && ((uintptr_t)dw & (a.dw_f32 ? 15 : 7)) == 0;
      }
    }
    if (a.dx || a.dw) {
      if (p.split.shape == SMALL) launch_grads<Small, TERMS, FINE>(ox, ow, s);
      else launch_grads<Large, TERMS, FINE>(ox, ow, s);
    }
    if (a.db) {
      sb.part = g.dbp; sb.parts = over(rows, tall); sb.tp = p.ldd; sb.rows = 1; sb.cols = n; sb.scale = a.grad_scale; sb.out = a.db + v0; sb.f32 = true;
      sb.ways = sb.parts < 16 ? 1 : sb.parts < 512 ? 16 : 64; sb.blocks = over(over(n, 4), 256 / sb.ways);
    }
    const int blocks = sx.blocks + sw.blocks + sb.blocks;
    if (sb.ways > 1) ce_sums_kernel<true><<<blocks, 256, 0, s>>>(sx, sw, sb);
    else if (blocks > 0) ce_sums_kernel<false><<<blocks, 256, 0, s>>>(sx, sw, sb);
  }
}
static void backward_with(const LinearCe& a, Ready ready, const float* z, hipStream_t s) {
  if (a.f32) backward_as<float, false>(a, ready, z, s);
  else if (is_fine(a)) backward_as<bf16, true>(a, ready, z, s);
  else backward_as<bf16, false>(a, ready, z, s);
}
static void no_tokens(const LinearCe& a, hipStream_t s) {
  const unsigned grid = (unsigned)std::min(a.V, 4096);
  if (a.dw && a.dw_f32) ce_fill_kernel<float><<<grid, 256, 0, s>>>((float*)a.dw, a.lddw, a.V, a.D);
  else if (a.dw) ce_fill_kernel<bf16><<<grid, 256, 0, s>>>((bf16*)a.dw, a.lddw, a.V, a.D);
  if (a.db) ce_fill_kernel<float><<<1, 256, 0, s>>>(a.db, 0, 1, a.V);
}
// few rows; both: the forward as well
static void few_backward(const LinearCe& a, bool both, hipStream_t s) {
  const Way way(a);
  if (way.little || !way.w) {
    const bool fused = both && few_fused(a.f32, a.V);
    // (a launch of its own turns logits of very many classes into G faster than a workgroup a row: loss and gradients of 16 x 512 x 16384 fp32 37.4 us, in the rows' launch 36.4; 32 x 512 x 40000 99.3 and 98.8; 1 x 64 x
    // 100000 45.6 and 52.0; 32 x 64 x 300000 142 and 169)
    const bool many = a.V > 1 << 15;
    if (both && !fused) small_ce_forward(a, (float*)a.workspace, !many, s);
    few_ce_backward(a, fused ? FEW_FUSED : !both ? FEW_NOTHING : many ? FEW_LOGITS : FEW_GRADIENT, s);
  } else {
    LinearCe f = a;
    f.workspace = (char*)a.workspace + few_parts_at(a.N, a.V);
    if (!both) f.loss = f.stats = nullptr;
    forward_with(f, (float*)a.workspace, false, s);
    few_ce_backward(a, FEW_LOGITS, s);
  }
}
void linear_ce_backward(const LinearCe& a, hipStream_t s) {
  if (a.N == 0) no_tokens(a, s);
  else if (Way(a).few) few_backward(a, false, s);
  else backward_with(a, NOTHING, nullptr, s);
}

void linear_ce_tiles(const LinearCe& a, LinearCeTiles& t) {
  const Way way(a);
  const int id[] = {2256256, 3128128, 3064128, 4032256, 2128128};
  if (!way.straight()) {
    const Plan p(a.f32, a.N, a.D, a.V, false);
    const int step = std::min(a.V, way.w ? p.Vs : p.Vp);
    t.forward_pieces = over(a.V, step);
    t.forward = id[logits_shape(a, p, step)];
    t.forward_last = id[logits_shape(a, p, a.V - (t.forward_pieces - 1) * step)];
  }
  if (way.few) return;
  const Plan p = backward_plan(a);
  const int step = std::min(a.V, p.Vc);
  t.pieces = over(a.V, step);
  if (!takes_turn(a, p, way)) {
    t.gradient = id[logits_shape(a, p, step)];
    t.gradient_last = id[logits_shape(a, p, a.V - (t.pieces - 1) * step)];
  }
  t.products = id[p.split.shape == SMALL ? SMALL : LARGE];
  t.splits_x = p.split.x;
  t.splits_w = p.split.w;
}

static size_t both_kept_at(bool f32, int N, int D, int V) {
  return (std::max(linear_ce_workspace_bytes(f32, N, D, V, false), linear_ce_workspace_bytes(f32, N, D, V, true)) + 255) / 256 * 256;
}
size_t linear_ce_both_bytes(bool f32, int N, int D, int V) { return both_kept_at(f32, N, D, V) + (keeps(f32, N, D, V) && !(is_few(N, V) && always_few(f32, N)) ? small_ce_bytes(N, V) : 0); }
void linear_ce_both(const LinearCe& a, hipStream_t s) {
  const Way way(a);
  if (a.N == 0) {
    no_tokens(a, s);
  } else if (way.few) {
    few_backward(a, true, s);
  } else {
    const Plan f(a.f32, a.N, a.D, a.V, false), p = backward_plan(a);
    const bool one = p.Vc >= a.V && (way.w ? f.Vs : f.Vp) >= a.V;        // one piece in both
    if (takes_turn(a, p, way)) {
      float* z = (float*)((char*)a.workspace + p.z);
      small_ce_forward(a, z, false, s);
      backward_with(a, KEPT, z, s);
    } else if (one && keeps(a.f32, a.N, a.D, a.V) && !way.little) {
      float* z = (float*)((char*)a.workspace + both_kept_at(a.f32, a.N, a.D, a.V));
      forward_with(a, z, true, s);
      backward_with(a, KEPT, z, s);
    } else {
      linear_ce_forward(a, s);
      // (the packed operands lie at the same places)
      const bool packed = !way.little && (!way.x || !way.w) && one && f.xp == p.xp && f.ex == p.ex && f.wp == p.wp && f.ew == p.ew;
      backward_with(a, packed ? PACKED : NOTHING, nullptr, s);
    }
  }
}

}  // namespace bsr
