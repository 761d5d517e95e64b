// Products of 8-bit operands with a scale for each block of 128 (fp8.h): forward and input gradient of frozen linear layers.
//
// C(m,n) = epilogue(sum over blocks b of 2^(ea(m,b) + eb(n/128,b)) sum_{k in b} A(m,k) B(n,k)), fp32 accumulation, in two forms:
//   exact  v_mfma_f32_32x32x16_bf16 (16x16x32 for few rows) on operands that are brought to bf16, scale and all, on the way from LDS to the instruction
//   cut    v_mfma_scale_f32_32x32x64_f8f6f4, which multiplies by the scales of its operands on the way: a scale is a byte that each lane passes for its row
// A k-tile is one block of 128, so the bytes of a tile row (128) and the LDS layout are those of the bf16
// products with their k-tiles of 64, and so is the way operands come: straight from global memory into LDS.  Any order of k within a block
// is as good as another as long as both operands use it, the scale being one for all of it.
//
// How exactly that adds up (measured, one large product among small ones in an instruction).  Of the products that the 8-bit instructions add at
// a time, those smaller than 2^-13 of the largest are cut to nothing and the others to that place; between such groups, and to the accumulator, the sum is fp32.
// On random operands the result is off by about 3e-5 of its size, whatever K, but an outlier takes up to all of its group's small products with it: where two
// outliers cancel, what is left may be gone.  An element can be off by 2^-13 of the largest product for each product, 2^-6 of the largest in each block of
// 128.  The bf16 instructions add the same products to 24 bits, at half the rate; an e4m3 value times a power of two is a bf16 value, but at the ends of the range (2^128 is infinite,
// below 2^-126 there are fewer bits).  So exact sums are what runs, and a caller who wants bf16 results may choose the others (BSR_SUMS_CUT).  Few rows
// have the exact form alone, trips to memory being what they wait for: 1 x 4096 x 4096 5.5 us against 5.7 from 8-bit rows and 6.5 against 6.3 from bf16.
//
// Measured, in chains of launches, exact and cut: 8192^3 889 us (1237 TFLOP/s; to fp32 902) and 409 (2690), 16384 x 4096 x 8192 909 (with GELU 953, times GELU' 987) and
// 435 (480, 534), 4096^3 116 and 57, 6304 x 768 x 2304 26 and 15.5, 100 x 4096 x 4096 11.4 and 8.2.  Large products are bound by the card's power: on zeros 16384 x 4096 x 8192
// takes 688 us exact and 341 cut, at the same instructions and bytes.  Exact ones reach 86 % of the rate of the library's largest bf16 product.  Short sums are bound by the way
// into LDS, the conversions and the way out of the registers, few rows by the latency of a k-tile.
#include <algorithm>
#include <type_traits>

#include "fp8.h"
#include "gemm_common.h"

namespace bsr {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row of results, at the address of any element, of which n columns exist
template <typename T> __device__ __forceinline__ typename Chunk<T>::vec get16(const T* p, int n) {
  if (n >= Chunk<T>::V) return *(const typename Loose<T>::vec*)p;
  typename Chunk<T>::vec o;
#pragma unroll
  for (int i = 0; i < Chunk<T>::V; ++i) o[i] = i < n ? p[i] : (T)0.f;
  return o;
}
// past: past the caches, where rows lie on lines
template <typename T> __device__ __forceinline__ void put16(T* p, int n, bool past, typename Chunk<T>::vec v) {
  if (n >= Chunk<T>::V && past) __builtin_nontemporal_store(__builtin_bit_cast(i32x4, v), (i32x4*)p);
  else if (n >= Chunk<T>::V) *(typename Loose<T>::vec*)p = v;
  else
#pragma unroll
    for (int i = 0; i < Chunk<T>::V; ++i)
      if (i < n) p[i] = v[i];
}

// What follows the products of a wave tile: bias, GELU (with its stored input) or GELU', residual.  Bias and GELU are finished where the
// accumulators are; 32 rows at a time then go through a patch of LDS, rounded where nothing is to be added any more, and come back with a lane owning
// 16 bytes of a row.  bias: that of the wave tile's columns, in LDS.  What is added or multiplied there is asked for a row block ahead.  The row blocks are a
// loop: code that is written out once is fetched once.
// Stores.  A row of a wave tile is one or two 128-byte lines, or half of one, where rows lie on lines; such stores go past the caches, which
// otherwise lose the operands' panels to results that nobody reads here (cut sums, 16384 x 4096 x 8192: 509 -> 460 us; 6304 x 768 x 2304: 17.7 -> 15.7).  Smaller pieces of lines must not:
// results stored 32 bytes of a row at a time straight from the accumulators took 509 us the ordinary way and 688 past the caches.
template <int MI, int NI, typename T, int ACT>
__device__ __forceinline__ void epilogue8(const Gemm8Desc& g, f32x16 (&acc)[MI][NI], int row0, int col0, int lane, unsigned char* patch,
                                          const float* bias) {
  typedef typename Chunk<T>::vec vecT;
  constexpr int P = Chunk<T>::V, TN = NI * 32, CPR = TN / P, RPP = 64 / CPR, NPASS = 32 / RPP, LDF = (TN + 4) * 4, LDT = TN * (int)sizeof(T) + 16;
  const int lr = lane & 31, lh = lane >> 5, my_row = lane / CPR, col = col0 + lane % CPR * P, n = g.N - col;
  const bool past = g.ldc * (int64_t)sizeof(T) % 128 == 0;
  auto fence = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  typedef T vec4 __attribute__((ext_vector_type(4)));
  // the row block in blk, rounded, to dst
  auto out = [&](const f32x16 (&blk)[NI], T* dst, int mi) __attribute__((always_inline)) {
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        vec4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (T)blk[ni][4 * rg + e];
        *(vec4*)(patch + lr * LDT + (ni * 32 + 8 * rg + 4 * lh) * (int)sizeof(T)) = o;
      }
    fence();
#pragma unroll
    for (int p = 0; p < NPASS; ++p) {
      const int r = p * RPP + my_row, m = row0 + mi * 32 + r;
      const vecT v = *(const vecT*)(patch + r * LDT + lane % CPR * 16);
      if (m < g.M && n > 0) put16(dst + (int64_t)m * g.ldc + col, n, past, v);
    }
    fence();
  };
  const T* extra = (const T*)(ACT == ACT_GELU_BWD ? g.aux : g.res);
  const bool add = ACT == ACT_GELU_BWD || g.res;
  vecT next[NPASS];                                  // of the row block after this one
  auto ask = [&](int mi) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < NPASS; ++p) {
      const int m = row0 + mi * 32 + p * RPP + my_row;
      if (m < g.M && n > 0) next[p] = get16(extra + (int64_t)m * g.ldc + col, n);
    }
  };
  if (add) ask(0);
#pragma nounroll
  for (int mi = 0; mi < MI; ++mi) {
    f32x16 blk[NI];
    sfor<MI>([&](auto I) __attribute__((always_inline)) {
      constexpr int i = decltype(I)::value;
      if (mi == i)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) blk[ni] = acc[i][ni];
    });
    vecT more[NPASS];
#pragma unroll
    for (int p = 0; p < NPASS; ++p) more[p] = next[p];
    if (add && mi + 1 < MI) ask(mi + 1);
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const f32x4 b = *(const f32x4*)(bias + ni * 32 + 8 * rg + 4 * lh);
#pragma unroll
        for (int e = 0; e < 4; ++e) blk[ni][4 * rg + e] += b[e];
      }
    if constexpr (ACT == ACT_GELU) {
      if (g.aux) out(blk, (T*)g.aux, mi);
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int r = 0; r < 16; ++r) blk[ni][r] = gelu_to<sizeof(T) == 4>(blk[ni][r]);
    }
    if (!add) {
      out(blk, (T*)g.C, mi);
      continue;
    }
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg)
        *(f32x4*)(patch + lr * LDF + (ni * 32 + 8 * rg + 4 * lh) * 4) = f32x4{blk[ni][4 * rg], blk[ni][4 * rg + 1], blk[ni][4 * rg + 2], blk[ni][4 * rg + 3]};
    fence();
#pragma unroll
    for (int p = 0; p < NPASS; ++p) {
      const int r = p * RPP + my_row, m = row0 + mi * 32 + r;
      const float* src = (const float*)(patch + r * LDF) + lane % CPR * P;
      vecT v;
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = (T)(ACT == ACT_GELU_BWD ? src[i] * gelu_grad_to<sizeof(T) == 4>((float)more[p][i]) : src[i] + (float)more[p][i]);
      if (m < g.M && n > 0) put16((T*)g.C + (int64_t)m * g.ldc + col, n, past, v);
    }
    fence();
  }
}

// eight e4m3 values (two dwords) times the power of two whose E8M0 byte is s8: exact in bf16
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, int s8) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float s = __uint_as_float((unsigned)s8 << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ i32x8 join8(i32x4 a, i32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// Row and column of tile t: column after column within bands of eight tile rows, so that the tiles that an XCD works on at a time (neighbours, by
// xcd_remap) share rows and columns alike and its L2 reads each once.  16384 x 4096 x 8192: row after row, an XCD's 32 tiles read 33 panels a round, like this 12.
constexpr int BAND = 8;
__device__ __forceinline__ void place(int t, int ntm, int ntn, int& tm, int& tn) {
  const int band = t / (BAND * ntn), first = band * BAND, high = min(BAND, ntm - first), in = t - first * ntn;
  tm = first + in % high;
  tn = in / high;
}

// Block tile BM x BN x 128, WM x WN wavefronts, NST stages of LDS.  The weights are the first operand of the instruction, so an accumulator
// holds the transposed output tile: lane l owns output row l % 32 and four runs of four columns.
// A stage is (BM + BN) rows of 128 bytes (eight chunks of 16, chunk c of row r in slot c ^ swz(r)) and behind them a dword of scales for
// each row: the scales of four k-tiles, of which each k-tile reads its byte (each k-tile fetches the dword anew, 1/32 more bytes, so that
// every k-tile is the same number of loads and can be waited for by count).
// KG groups of wavefronts, each with stages of its own, share the k-tiles of a block tile (few tiles, long sums); the groups behind the first leave their
// sums in LDS, and the first adds them in their order.
template <int BM, int BN, int NT, int NST, int KG> constexpr size_t lds_of() {      // of a workgroup: stages and bias
  return (size_t)KG * NST * ((BM + BN) * 128 + (BM + BN + NT - 1) / NT * NT * 4) + BN * 4;
}
// (held to the registers that let as many workgroups share a CU as its LDS has room for, up to three)
template <int BM, int BN, int WM, int WN, int NST, int KG, typename T, int ACT, bool EXACT>
__global__ __launch_bounds__(WM * WN * KG * 64, std::max<int>(1, std::min<int>(3, 160 * 1024 / lds_of<BM, BN, WM * WN * 64, NST, KG>()) * WM * WN * KG / 4))
void gemm8_kernel(const void* hA, const void* hB, const void* hsa, const void* hsb, int hM, int hN, int hK,
                                                                int tiles, Gemm8Desc g) {
  constexpr int NW = WM * WN, NT = NW * 64, ROWS = BM + BN;
  constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 32, NI = TN / 32, NMF = MI * NI;
  constexpr int RPI = NT / 8;                        // tile rows that a load instruction of the workgroup fills
  constexpr int AL = BM / RPI, BL = BN / RPI;
  constexpr int SL = (ROWS + NT - 1) / NT;           // scale loads of a thread
  constexpr int LPT = AL + BL + SL;
  constexpr int SCALES = ROWS * 128;                 // where the scales of a stage start
  constexpr int STAGE = SCALES + SL * NT * 4;
  static_assert(BM % RPI == 0 && BN % RPI == 0 && RPI % 16 == 0, "a load instruction covers whole groups of 16 rows");
  static_assert(NST >= 2 && NST <= 4 && (NST - 1) * LPT <= 60, "vmcnt has 6 bits");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_all[];
  const int M = hM, N = hN;
  const int group = KG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
  unsigned char* smem = smem_all + group * NST * STAGE;
  float* bias = (float*)(smem_all + KG * NST * STAGE);
  const int tid = threadIdx.x - group * NT, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int tile = xcd_remap(blockIdx.x, tiles);
  int tm, tn;
  place(tile, (M + BM - 1) / BM, (N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int nall = (hK + BLOCK8 - 1) / BLOCK8;
  const unsigned ld = (unsigned)nall * BLOCK8, lds = (unsigned)(nall + 3) / 4 * 4;
  // the group's k-tiles: `mine` from `first` on, in nk turns (the barriers are everybody's; a group with one k-tile less passes over the last turn)
  const int first = KG > 1 ? group * (nall / KG) + min(group, nall % KG) : 0, mine = KG > 1 ? nall / KG + (group < nall % KG) : nall;
  const int nk = KG > 1 ? (nall + KG - 1) / KG : nall;
  const uint8_t* __restrict__ A = (const uint8_t*)hA + (int64_t)m0 * ld;
  const uint8_t* __restrict__ B = (const uint8_t*)hB + (int64_t)n0 * ld;

  // rows past the end repeat the last one: they only feed accumulators that are never stored
  const int lrow = tid >> 3, chunk = ((tid & 7) ^ swz(lrow)) * 16;
  constexpr bool TIGHT = MI * NI >= 8;               // no registers to keep the offsets of the loads in: worked out at each
  const int a_rows = M - 1 - m0, b_rows = N - 1 - n0;
  auto row_off = [&](auto I, int row) __attribute__((always_inline)) {
    constexpr int i = decltype(I)::value;
    return (unsigned)min((i < AL ? i : i - AL) * RPI + row, i < AL ? a_rows : b_rows) * ld + chunk;
  };
  unsigned off[TIGHT ? 1 : AL + BL];
  if constexpr (!TIGHT) sfor<AL + BL>([&](auto I) __attribute__((always_inline)) { off[decltype(I)::value] = row_off(I, lrow); });
  const uint8_t* soff[SL];
#pragma unroll
  for (int i = 0; i < SL; ++i) {
    const int r = i * NT + tid;
    soff[i] = r < BM ? (const uint8_t*)hsa + (int64_t)min(m0 + r, M - 1) * lds
                     : (const uint8_t*)hsb + (int64_t)(min(n0 + r - BM, N - 1) / BLOCK8) * lds;
  }
  auto issue1 = [&](auto I, int turn, int st) __attribute__((always_inline)) {
    constexpr int i = decltype(I)::value;
    const int kt = KG > 1 ? min(first + turn, nall - 1) : turn;
    unsigned char* base = smem + st * STAGE;
    if constexpr (i < AL + BL) {
      const uint8_t* src = (i < AL ? A : B) + (size_t)kt * BLOCK8;
      unsigned char* dst = base + wave * 1024 + (i < AL ? i * RPI * 128 : BM * 128 + (i - AL) * RPI * 128);
      unsigned o;
      if constexpr (TIGHT) {
        int row = lrow;
        asm volatile("" : "+v"(row));                // (not before the loop)
        o = row_off(I, row);
      } else {
        o = off[i];
      }
      __builtin_amdgcn_global_load_lds(BSR_GLOBAL_PTR(src + o), BSR_LDS_VOID(dst), 16, 0, 0);
    } else {
      constexpr int j = i - AL - BL;
      __builtin_amdgcn_global_load_lds(BSR_GLOBAL_PTR(soff[j] + (kt & ~3)), BSR_LDS_VOID(base + SCALES + (j * NT + wave * 64) * 4), 4, 0, 0);
    }
  };

  f32x16 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mi][ni][r] = 0.f;

  // Fragments: rows of A one set, each read for the next k-step once its products are done; rows of B two sets, of k-steps in turn (a second set
  // of A as well would spill in the largest tile).  Row r's bytes of k-step ks lie in chunks 4 ks + lh and 4 ks + 2 + lh, slot chunk ^ swz(r): the
  // address of the lane's first chunk, bits flipped for the others.
  const int lr = lane & 31, lh = lane >> 5;
  const int slot0 = lr * 128 + ((lh ^ swz(lr)) << 4);
  const int a_at = wm * TM * 128 + slot0, b_at = (BM + wn * TN) * 128 + slot0;
  const int as_at = SCALES + (wm * TM + lr) * 4, bs_at = SCALES + (BM + wn * TN + lr) * 4;
  i32x8 fa[MI], fb[2][NI];
  bf16x8 wa[EXACT ? MI : 1][4], wb[EXACT ? NI : 1][4];
  int sa[MI], sb[NI], sbn[NI];
  auto frag = [&](int at, int ks) __attribute__((always_inline)) {
    return join8(*(const i32x4*)(smem + (at ^ (ks << 6))), *(const i32x4*)(smem + (at ^ (ks << 6) ^ 32)));
  };
  auto rda = [&](auto I, int st, int ks) __attribute__((always_inline)) {
    constexpr int i = decltype(I)::value;
    fa[i] = frag(st * STAGE + i * 4096 + a_at, ks);
  };
  auto rdb = [&](auto SET, auto I, int st, int ks) __attribute__((always_inline)) {
    constexpr int set = decltype(SET)::value, i = decltype(I)::value;
    fb[set][i] = frag(st * STAGE + i * 4096 + b_at, ks);
  };
  auto rdsa = [&](auto I, int st, int kt) __attribute__((always_inline)) {
    constexpr int i = decltype(I)::value;
    sa[i] = smem[st * STAGE + as_at + i * 128 + (first + kt & 3)];
  };
  auto rdsb = [&](int st, int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) sbn[i] = smem[st * STAGE + bs_at + i * 128 + (first + kt & 3)];
  };
  auto next_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) sb[i] = sbn[i];
  };
  auto widen = [&](auto SET) __attribute__((always_inline)) {
    constexpr int set = decltype(SET)::value;
    if constexpr (EXACT) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int i = 0; i < MI; ++i) wa[i][q] = widen8(fa[i][2 * q], fa[i][2 * q + 1], sa[i]);
#pragma unroll
        for (int i = 0; i < NI; ++i) wb[i][q] = widen8(fb[set][i][2 * q], fb[set][i][2 * q + 1], sb[i]);
      }
    }
  };
  auto mf1 = [&](auto SET, auto J) __attribute__((always_inline)) {
    constexpr int set = decltype(SET)::value, mi = decltype(J)::value / NI, ni = decltype(J)::value % NI;
    if constexpr (EXACT) {
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[ni][q], wa[mi][q], acc[mi][ni], 0, 0, 0);
    } else {
      acc[mi][ni] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[set][ni], fa[mi], acc[mi][ni], 0, 0, 0, sb[ni], 0, sa[mi]);
    }
  };
  constexpr int PRE = NI;                            // MFMAs of the second k-step in front of the barrier: those of the first rows
  constexpr int POST = NMF - PRE;
  constexpr int SPAN = POST + (NST > 2 && NMF >= 4 ? NMF : 0);       // MFMAs that the loads of a k-tile are spread over
  constexpr bool LATE = SPAN > POST;                 // some follow in the next k-tile
  auto loads_at = [&](auto P, int kt, int st) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value, lo = p >= SPAN ? LPT : (p * LPT + SPAN - 1) / SPAN, hi = p + 1 >= SPAN ? LPT : ((p + 1) * LPT + SPAN - 1) / SPAN;
    sfor<hi - lo>([&](auto L) __attribute__((always_inline)) { issue1(IC<lo + decltype(L)::value>{}, kt, st); });
  };
  // what is read behind MFMA j of a k-step for the next one: B in the first MFMAs, the rows of A whose last product this was
  auto reads_at = [&](auto SETN, auto J, int st, int ks, int kt) __attribute__((always_inline)) {
    constexpr int j = decltype(J)::value;
    if constexpr (j % NI == NI - 1) {
      rda(IC<j / NI>{}, st, ks);
      if constexpr (decltype(SETN)::value == 0) rdsa(IC<j / NI>{}, st, kt);
    }
    constexpr int from = PRE < NMF ? PRE : 0;        // (behind the barrier, where there is one)
    if constexpr (j >= from && j - from < NI) rdb(SETN, IC<j - from>{}, st, ks);
  };
  // the first k-step of a k-tile: MFMAs on set 0 of B, the fragments of the second k-step
  auto kfirst = [&](auto LOADS, int st, int ktl, int stl) __attribute__((always_inline)) {
    widen(IC<0>{});
    sfor<NMF>([&](auto J) __attribute__((always_inline)) {
      mf1(IC<0>{}, J);
      reads_at(IC<1>{}, J, st, 1, 0);
      if constexpr (decltype(LOADS)::value) loads_at(IC<POST + decltype(J)::value>{}, ktl, stl);
      BSR_SCHED_FENCE();
    });
  };
  // the second, with the barrier.  VMW >= 0: loads that may stay in flight there (steady state, those of k-tile kt + NST follow it); VMW < 0:
  // nothing is issued any more and the count follows from rem, the k-tiles behind this one
  auto klast = [&](auto VMW, int kt, int st, int stn, int rem) __attribute__((always_inline)) {
    constexpr int vmw = decltype(VMW)::value;
    if constexpr (EXACT) widen(IC<1>{});
    sfor<PRE>([&](auto J) __attribute__((always_inline)) { mf1(IC<1>{}, J); BSR_SCHED_FENCE(); });
    wait_lgkmcnt0();
    if constexpr (vmw >= 0) wait_vmcnt<vmw>();
    else if (rem >= 3) wait_vmcnt<2 * LPT>();
    else if (rem == 2) wait_vmcnt<LPT>();
    else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    BSR_SCHED_FENCE();
    rda(IC<0>{}, stn, 0);                            // (its products were in front of the barrier)
    rdsa(IC<0>{}, stn, kt + 1);
    rdsb(stn, kt + 1);
    if constexpr (POST == 0) sfor<NI>([&](auto I) __attribute__((always_inline)) { rdb(IC<0>{}, I, stn, 0); });
    sfor<POST>([&](auto Q) __attribute__((always_inline)) {
      constexpr int q = decltype(Q)::value;
      mf1(IC<1>{}, IC<PRE + q>{});
      reads_at(IC<0>{}, IC<PRE + q>{}, stn, 0, kt + 1);
      if constexpr (vmw >= 0) loads_at(Q, kt + NST, st);
      BSR_SCHED_FENCE();
    });
    if constexpr (POST == 0 && vmw >= 0) sfor<LPT>([&](auto I) __attribute__((always_inline)) { issue1(I, kt + NST, st); });
    next_scales();
  };

  // the bias goes behind the stages, ahead of the first k-tile: it has landed when that has
  if (g.bias) {
    if (group == 0 && wave < BN / 64) __builtin_amdgcn_global_load_lds(BSR_GLOBAL_PTR(g.bias + min(n0 + tid, N - 1)), BSR_LDS_VOID(bias + wave * 64), 4, 0, 0);
  } else if (group == 0 && tid < BN) {
    bias[tid] = 0.f;
  }
#pragma unroll
  for (int j = 0; j < NST; ++j)
    if (j < nk) sfor<LPT>([&](auto I) __attribute__((always_inline)) { issue1(I, j, j); });
  {
    const int fl = min(nk, NST) - 1;
    if (fl >= 3) wait_vmcnt<3 * LPT>(); else if (fl == 2) wait_vmcnt<2 * LPT>(); else if (fl == 1) wait_vmcnt<LPT>(); else wait_vmcnt<0>();
  }
  wait_lgkmcnt0();
  __builtin_amdgcn_s_barrier();
  rdsb(0, 0);
  sfor<MI>([&](auto I) __attribute__((always_inline)) { rda(I, 0, 0); rdsa(I, 0, 0); });
  sfor<NI>([&](auto I) __attribute__((always_inline)) { rdb(IC<0>{}, I, 0, 0); });
  next_scales();
  int st = 0, kt = 0;
  auto ktile = [&](auto LOADS, auto VMW) __attribute__((always_inline)) {
    const int stn = (st + 1 == NST) ? 0 : st + 1, stl = st == 0 ? NST - 1 : st - 1;
    kfirst(LOADS, st, kt + NST - 1, stl);
    klast(VMW, kt, st, stn, nk - 1 - kt);
    st = stn;
    ++kt;
  };
  constexpr IC<(NST - 2) * LPT> steady{};
  if constexpr (LATE) {
    if (kt + NST < nk) ktile(IC<0>{}, steady);                    // (the prologue's loads are all out)
    while (kt + NST < nk) ktile(IC<1>{}, steady);
    if (kt > 0) ktile(IC<1>{}, IC<-1>{});                         // the last late loads
  } else {
    while (kt + NST < nk) ktile(IC<0>{}, steady);
  }
  if constexpr (KG == 1) {
    while (kt < nk) ktile(IC<0>{}, IC<-1>{});                     // nothing left to issue
  } else {
    static_assert(!LATE, "loads end with the k-tiles that issue them");
    while (kt < nk - 1) ktile(IC<0>{}, IC<-1>{});
    if (mine == nk) {
      kfirst(IC<0>{}, st, 0, 0);
      widen(IC<1>{});
      sfor<NMF>([&](auto J) __attribute__((always_inline)) { mf1(IC<1>{}, J); });
    }
    // behind the patches of the epilogue: [group - 1][wave][accumulator][16 floats in fours][lane]
    constexpr int PATCHES = NW * 32 * (TN + 4) * 4, PART = BM * BN * 4;
    static_assert(PATCHES + (KG - 1) * PART <= KG * NST * STAGE, "the sums of the groups lie in the stages");
    __syncthreads();
    auto part = [&](int of, int mi, int ni, int q) __attribute__((always_inline)) {
      return (f32x4*)(smem_all + PATCHES + (of - 1) * PART) + (((wave * MI + mi) * NI + ni) * 4 + q) * 64 + lane;
    };
    if (group > 0)
      sfor<MI * NI * 4>([&](auto I) __attribute__((always_inline)) {
        constexpr int q = decltype(I)::value % 4, ni = decltype(I)::value / 4 % NI, mi = decltype(I)::value / 4 / NI;
        *part(group, mi, ni, q) = f32x4{acc[mi][ni][4 * q], acc[mi][ni][4 * q + 1], acc[mi][ni][4 * q + 2], acc[mi][ni][4 * q + 3]};
      });
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int of = 1; of < KG; ++of)
      sfor<MI * NI * 4>([&](auto I) __attribute__((always_inline)) {
        constexpr int q = decltype(I)::value % 4, ni = decltype(I)::value / 4 % NI, mi = decltype(I)::value / 4 / NI;
        const f32x4 p = *part(of, mi, ni, q);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mi][ni][4 * q + e] += p[e];
      });
  }
  // every wavefront is past the last barrier: the stages are free, a patch of them for each wavefront
  epilogue8<MI, NI, T, ACT>(g, acc, m0 + wm * TM, n0 + wn * TN, lane, smem_all + wave * (32 * (TN + 4) * 4), bias + wn * TN);
}

// maximum over lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ uint32_t quarters_max(uint32_t v) {
  const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = max((uint32_t)h[0], (uint32_t)h[1]);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max((uint32_t)r[0], (uint32_t)r[1]);
}
// 32 values of a block whose other three quarters lanes l ^ 16, l ^ 32 and l ^ 48 hold -> 8 bits, and the block's scale byte.  The maximum is taken of
// the bits (two bf16 at a time), which non-finite values top: blocks that hold one go through the values again.
template <typename T>
__device__ __forceinline__ int quantize32(const typename Chunk<T>::vec (&v)[32 / Chunk<T>::V], i32x8& q) {
  constexpr int V = Chunk<T>::V;
  uint32_t most;
  if constexpr (sizeof(T) == 2) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t d = __builtin_bit_cast(u32x4, v[i / 4])[i % 4] & 0x7fff7fffu;
      m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, d));
    }
    most = quarters_max((uint32_t)max(m[0], m[1]) << 16);
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(v[i / V][i % V]) & 0x7fffffffu);
    most = quarters_max(m);
  }
  if (most >= 0x7f800000u) {
    most = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) most = max(most, finite_bits((float)v[i / V][i % V]));
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    const float inv = inverse_of(scale8_of(most));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = (float)v[4 * i / V][4 * i % V], b = (float)v[4 * i / V][(4 * i + 1) % V], c = (float)v[4 * i / V][(4 * i + 2) % V], d = (float)v[4 * i / V][(4 * i + 3) % V];
      q[i] = (int)pack8(a, b, c, d, inv);
    }
    return (int)scale8_of(most);
  }
  const int s8 = (int)scale8_of(most);
  const float s = __uint_as_float((uint32_t)s8 << 23);        // 2^e, what the instruction divides by
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s16x2 r = {0, 0};
    if constexpr (sizeof(T) == 2) {
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, bf16x2{v[i / 2][4 * (i % 2)], v[i / 2][4 * (i % 2) + 1]}, s, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, bf16x2{v[i / 2][4 * (i % 2) + 2], v[i / 2][4 * (i % 2) + 3]}, s, true);
    } else {
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v[i][0], v[i][1], s, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v[i][2], v[i][3], s, true);
    }
    q[i] = __builtin_bit_cast(int, r);
  }
  return s8;
}

// 32 bytes without the first n (< 32), zeros behind them
__device__ __forceinline__ i32x8 bytes_down(i32x8 q, int n) {
#pragma unroll
  for (int step = 4; step > 0; step /= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = n & 4 * step ? (i + step < 8 ? q[i + step] : 0) : q[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = (int)__builtin_amdgcn_alignbyte(i < 7 ? q[i + 1] : 0, q[i], n & 3);
  return q;
}

// Few rows: what counts is that the weights come once and at once.  A workgroup owns 16 columns and all rows (16 MI of them); its eight
// wavefronts share the k-tiles, each with its own straight from global memory into registers (a weight row's 128 bytes of a k-tile are a
// cache line that four lanes read whole), AHEAD of them asked for before the first is looked at, and their sums meet in LDS in wavefront
// order.  Rows of bf16 or fp32 are brought to 8 bits here by every workgroup for itself: they are
// few, and it saves the launch.  Bound by the latency of one trip to memory, then by the weights' bytes:
// 1 x 4096 x 4096 6.5 us from bf16 and 5.5 from 8-bit rows (the weights' bytes at a copy's rate: 3.3), 1 x 8192 x 8192 17.6 and 13.9 (13.2), 16 x 4096 x 4096 8.6 and 6.8.
enum { X_E4, X_BF16, X_F32 };                      // type of the rows
enum { ROWS_WHOLE, ROWS_PART, ROWS_SHORT };        // of whole pieces of 32 values; with a part of one at the end; of less than one
constexpr int FEW_WAVES = 8, FEW_ROWS = 32;
template <int X, int MI, int ROWS>
__global__ __launch_bounds__(FEW_WAVES * 64, 1) void gemm8_few_kernel(const void* hA, const void* hB, const void* hsa, const void* hsb, int hM, int hN,
                                                                      int hK, int64_t lda, Gemm8Desc g) {
  typedef typename std::conditional<X == X_F32, float, bf16>::type TX;
  constexpr int V = Chunk<TX>::V, AHEAD = X == X_E4 ? 4 : 4 / MI;
  __shared__ float part[FEW_WAVES][MI * 16][16 + 1];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int nk = (hK + BLOCK8 - 1) / BLOCK8;
  const int64_t ld = (int64_t)nk * BLOCK8, lds = (nk + 3) / 4 * 4;
  const uint8_t* wrow = (const uint8_t*)hB + (int64_t)min(n0 + lr, hN - 1) * ld + lg * 32;
  const uint8_t* wscale = (const uint8_t*)hsb + (int64_t)(n0 / BLOCK8) * lds;       // (16 columns lie in one block)
  f32x4 acc[MI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) acc[mi] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kt0 = wave; kt0 < nk; kt0 += FEW_WAVES * AHEAD) {
    i32x8 w[AHEAD], x8[X == X_E4 ? AHEAD : 1][MI];
    int ws[AHEAD], xs[X == X_E4 ? AHEAD : 1][MI];
    typename Chunk<TX>::vec raw[X == X_E4 ? 1 : AHEAD][MI][32 / V];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {                      // (past the end: the last k-tile again, not used)
      const int kt = min(kt0 + a * FEW_WAVES, nk - 1);
      w[a] = join8(*(const i32x4*)(wrow + (int64_t)kt * BLOCK8), *(const i32x4*)(wrow + (int64_t)kt * BLOCK8 + 16));
      ws[a] = wscale[kt];
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int64_t m = min(mi * 16 + lr, hM - 1);
        if constexpr (X == X_E4) {
          const uint8_t* p = (const uint8_t*)hA + m * ld + (int64_t)kt * BLOCK8 + lg * 32;
          x8[a][mi] = join8(*(const i32x4*)p, *(const i32x4*)(p + 16));
          xs[a][mi] = ((const uint8_t*)hsa)[m * lds + kt];
        } else if constexpr (ROWS != ROWS_SHORT) {         // (a piece past the end: the last 32 values)
          const TX* p = (const TX*)hA + m * lda + min(kt * BLOCK8 + lg * 32, hK - 32);
#pragma unroll
          for (int i = 0; i < 32 / V; ++i) raw[a][mi][i] = *(const typename Loose<TX>::vec*)(p + i * V);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) raw[a][mi][i / V][i % V] = ((const TX*)hA)[m * lda + min(i, hK - 1)];
        }
      }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int kt = kt0 + a * FEW_WAVES;
      if (kt >= nk) break;
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        i32x8 x;
        int s8;
        if constexpr (X == X_E4) {
          x = x8[a][mi];
          s8 = xs[a][mi];
        } else {
          const int k0 = kt * BLOCK8 + lg * 32;
          typename Chunk<TX>::vec v[32 / V];
#pragma unroll
          for (int i = 0; i < 32 / V; ++i) v[i] = ROWS == ROWS_WHOLE && k0 >= hK ? typename Chunk<TX>::vec{} : raw[a][mi][i];
          if constexpr (ROWS == ROWS_WHOLE) {
            s8 = quantize32<TX>(v, x);
          } else if constexpr (ROWS == ROWS_PART) {        // the values that are another piece's do not count, and leave
            const int skip = min(max(k0 - (hK - 32), 0), 32);
            if (kt == nk - 1)
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i / V][i % V] = i < skip ? (TX)0.f : v[i / V][i % V];
            s8 = quantize32<TX>(v, x);
            if (kt == nk - 1) x = bytes_down(x, skip & 31);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i / V][i % V] = k0 + i < hK ? v[i / V][i % V] : (TX)0.f;
            s8 = quantize32<TX>(v, x);
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[mi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[a][2 * q], w[a][2 * q + 1], ws[a]), widen8(x[2 * q], x[2 * q + 1], s8), acc[mi], 0, 0, 0);
      }
    }
  }
  // lane l holds columns 4 (l / 16) .. + 3 of row l % 16
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][mi * 16 + lr][4 * lg + e] = acc[mi][e];
  __syncthreads();
  auto get = [&](const void* p, int64_t at) __attribute__((always_inline)) { return g.out_f32 ? ((const float*)p)[at] : (float)((const bf16*)p)[at]; };
  auto put = [&](void* p, int64_t at, float v) __attribute__((always_inline)) {
    if (g.out_f32) ((float*)p)[at] = v;
    else ((bf16*)p)[at] = (bf16)v;
  };
  for (int i = tid; i < MI * 16 * 16; i += FEW_WAVES * 64) {
    const int m = i / 16, col = n0 + i % 16;
    if (m >= hM || col >= hN) continue;
    float v = part[0][m][i % 16];
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) v += part[w][m][i % 16];
    const int64_t at = (int64_t)m * g.ldc + col;
    if (g.bias) v += g.bias[col];
    if (g.act == ACT_GELU) {
      if (g.aux) put(g.aux, at, v);
      v = g.out_f32 ? gelu_fp32(v) : gelu_f(v);
    } else if (g.act == ACT_GELU_BWD) {
      v *= g.out_f32 ? gelu_grad_fp32(get(g.aux, at)) : gelu_grad_f(get(g.aux, at));
    }
    if (g.res) v += get(g.res, at);
    put(g.C, at, v);
  }
}

template <int BM, int BN, int WM, int WN, int NST, int KG, typename T, int ACT, bool EXACT>
void launch_tiled(const Gemm8Desc& g, hipStream_t s) {
  constexpr int NT = WM * WN * 64;
  constexpr size_t stages = lds_of<BM, BN, NT, NST, KG>();
  static_assert(BN <= NT, "a thread for each column of the bias");
  constexpr size_t patches = (size_t)WM * WN * 32 * (BN / WN + 4) * 4;
  static_assert(patches <= stages && stages <= 160 * 1024, "the epilogue patches live in the stages");
  auto kern = gemm8_kernel<BM, BN, WM, WN, NST, KG, T, ACT, EXACT>;
  static bool attr_set = false;
  if (!attr_set) {
    (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)stages);
    attr_set = true;
  }
  const int tiles = (int)((int64_t)((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN));
  kern<<<tiles, NT * KG, stages, s>>>(g.A, g.B, g.a_scale, g.b_scale, g.M, g.N, g.K, tiles, g);
}

// What a product takes in each block tile, in microseconds: c[0] + rounds (c[1] + c[2] k) + tiles per CU (c[3] + c[4] k), k the k-tiles (of a group) and rounds the
// turns of workgroups that the tiles make over the CUs, `sharing` of them on one at a time.  Least squares over 67 products timed in every tile
// (65 .. 16384 rows, 128 .. 8192 by 64 .. 8192, in chains of launches), one table for each arithmetic and type of result; the tile that comes out
// best took 1.01 times as long as the fastest of ten tiles on the mean, 1.20 times at worst (to fp32 1.13).
// Tiles whose k-tiles `groups` of wavefronts share (fitted over 60 products of up to 8 M results) are for one round of sums of two turns and more: with more tiles the
// CUs are full without them.  64 x 64 tiles, one group -> shared: 100 x 4096 x 4096 9.7 -> 8.4 us cut, 15.0 -> 11.6 exact and, to fp32, 15.7 -> 11.6; 64 x 8192 x 1024 15.9 -> 13.5 cut
// and 27.7 -> 19.0 to fp32; over the 60 products 5 % and 7 % on the mean.
struct Tile8 { int bm, bn, sharing, groups; float c[5]; };
constexpr Tile8 TILES_CUT[] = {
    {256, 256, 1, 1, {0.591f, 5.94f, 1.04f, 0.f, 0.544f}},
    {256, 128, 1, 1, {1.48f, 3.06f, 0.546f, 0.256f, 0.366f}},
    {128, 128, 2, 1, {2.04f, 0.f, 0.496f, 1.08f, 0.315f}},
    {128, 64, 2, 1, {1.32f, 1.44f, 0.315f, 0.f, 0.178f}},
    {64, 64, 3, 1, {1.77f, 0.697f, 0.19f, 0.0343f, 0.137f}},
    {64, 64, 1, 2, {0.f, 2.76f, 0.327f, 0.192f, 0.0601f}}};
constexpr Tile8 TILES_EXACT_BF16[] = {                        // (106 products of 64 .. 7430 by 64 .. 8192: 1.01, 1.11 at worst)
    {128, 128, 2, 1, {1.87f, 2.09f, 0.685f, 0.683f, 0.447f}},
    {64, 128, 3, 1, {1.49f, 1.17f, 0.526f, 0.517f, 0.264f}},
    {64, 64, 3, 1, {2.05f, 0.334f, 0.362f, 0.356f, 0.154f}},
    {128, 64, 1, 2, {0.f, 3.52f, 0.821f, 0.f, 0.199f}},
    {64, 64, 1, 4, {3.22f, 0.f, 0.957f, 0.f, 0.186f}}};
constexpr Tile8 TILES_EXACT_F32[] = {
    {128, 128, 2, 1, {1.04f, 3.67f, 0.718f, 0.695f, 0.478f}},
    {128, 64, 3, 1, {0.876f, 2.71f, 0.462f, 0.154f, 0.342f}},
    {64, 64, 3, 1, {2.61f, 0.152f, 0.335f, 0.525f, 0.186f}},
    {128, 64, 1, 2, {0.f, 3.81f, 0.814f, 0.692f, 0.126f}},
    {64, 64, 1, 4, {0.f, 3.42f, 0.948f, 0.643f, 0.0971f}}};
template <int N>
int pick(const Tile8 (&table)[N], const Gemm8Desc& g) {
  const int nk = (g.K + BLOCK8 - 1) / BLOCK8;
  int best = 0;
  float least = 0.f;
  for (int i = 0; i < N; ++i) {
    const Tile8& t = table[i];
    const int64_t tiles = (int64_t)((g.M + t.bm - 1) / t.bm) * ((g.N + t.bn - 1) / t.bn), slots = 256 * t.sharing;
    if (t.groups > 1 && (tiles > slots || nk < 2 * t.groups)) continue;
    const float k = (float)((nk + t.groups - 1) / t.groups);
    const float us = t.c[0] + (float)((tiles + slots - 1) / slots) * (t.c[1] + t.c[2] * k) + (float)tiles / 256.f * (t.c[3] + t.c[4] * k);
    if (i == 0 || us < least) { least = us; best = i; }
  }
  return best;
}

template <typename T, int ACT, bool EXACT>
void tiled(const Gemm8Desc& g, hipStream_t s) {
  if constexpr (!EXACT) {
    switch (pick(TILES_CUT, g)) {
      case 0: launch_tiled<256, 256, 2, 4, 2, 1, T, ACT, false>(g, s); break;
      case 1: launch_tiled<256, 128, 4, 2, 3, 1, T, ACT, false>(g, s); break;
      case 2: launch_tiled<128, 128, 2, 4, 2, 1, T, ACT, false>(g, s); break;
      case 3: launch_tiled<128, 64, 4, 1, 3, 1, T, ACT, false>(g, s); break;
      case 4: launch_tiled<64, 64, 2, 2, 3, 1, T, ACT, false>(g, s); break;
      default: launch_tiled<64, 64, 2, 2, 3, 2, T, ACT, false>(g, s); break;
    }
  } else {
    if constexpr (sizeof(T) == 2) {
      switch (pick(TILES_EXACT_BF16, g)) {
        case 0: launch_tiled<128, 128, 2, 2, 2, 1, T, ACT, true>(g, s); break;
        case 1: launch_tiled<64, 128, 2, 2, 2, 1, T, ACT, true>(g, s); break;
        case 2: launch_tiled<64, 64, 2, 2, 2, 1, T, ACT, true>(g, s); break;
        case 3: launch_tiled<128, 64, 2, 2, 2, 2, T, ACT, true>(g, s); break;
        default: launch_tiled<64, 64, 2, 2, 2, 4, T, ACT, true>(g, s); break;
      }
    } else {
      switch (pick(TILES_EXACT_F32, g)) {
        case 0: launch_tiled<128, 128, 2, 2, 2, 1, T, ACT, true>(g, s); break;
        case 1: launch_tiled<128, 64, 2, 2, 2, 1, T, ACT, true>(g, s); break;
        case 2: launch_tiled<64, 64, 2, 2, 3, 1, T, ACT, true>(g, s); break;
        case 3: launch_tiled<128, 64, 2, 2, 2, 2, T, ACT, true>(g, s); break;
        default: launch_tiled<64, 64, 2, 2, 2, 4, T, ACT, true>(g, s); break;
      }
    }
  }
}

template <int X, int ROWS>
void few_as(const Gemm8Desc& g, hipStream_t s) {
  const unsigned grid = (unsigned)((g.N + 15) / 16);
  auto go = [&](auto MI) {
    gemm8_few_kernel<X, decltype(MI)::value, ROWS><<<grid, FEW_WAVES * 64, 0, s>>>(g.A, g.B, g.a_scale, g.b_scale, g.M, g.N, g.K, g.lda, g);
  };
  if (g.M <= 16) go(IC<1>{});
  else go(IC<2>{});
}
void few(const Gemm8Desc& g, hipStream_t s) {
  auto of = [&](auto X) {
    constexpr int x = decltype(X)::value;
    if (g.K % 32 == 0) few_as<x, ROWS_WHOLE>(g, s);
    else if (g.K > 32) few_as<x, ROWS_PART>(g, s);
    else few_as<x, ROWS_SHORT>(g, s);
  };
  if (g.a_type == 2) few_as<X_E4, ROWS_WHOLE>(g, s);
  else if (g.a_type == 1) of(IC<X_F32>{});
  else of(IC<X_BF16>{});
}

template <typename T, bool EXACT>
void tiled_act(const Gemm8Desc& g, hipStream_t s) {
  if (g.act == ACT_GELU) tiled<T, ACT_GELU, EXACT>(g, s);
  else if (g.act == ACT_GELU_BWD) tiled<T, ACT_GELU_BWD, EXACT>(g, s);
  else tiled<T, ACT_NONE, EXACT>(g, s);
}

}  // namespace

bool gemm8_few_takes(int64_t M) { return M <= FEW_ROWS; }

void gemm8(const Gemm8Desc& g, hipStream_t s) {
  if (g.M <= 0) return;
  if (g.M <= FEW_ROWS) few(g, s);
  else if (g.out_f32) tiled_act<float, true>(g, s);
  else if (g.cut) tiled_act<bf16, false>(g, s);
  else tiled_act<bf16, true>(g, s);
}

}  // namespace bsr
