// Tile core of the products of block-scaled 8-bit tensors (quant_format.h): v_mfma_scale_f32_16x16x128_f8f6f4 with operands staged
// through LDS.  Both operands are rows of K codes; a K step is one block of 128, so one exponent an operand row, which the instruction
// applies.  C[m][n] = sum_k A[m][k] B[n][k], BM x 256 outputs of one product or BM x 128 of each of two that share A, four wavefronts.
#pragma once

#include "gemm_cores.h"
#include "quant_gemm.h"

namespace moe {

// An epilogue E whose last NQ outputs are quantised, too (128 columns of a row are the pieces of sixteen lanes), as moe_quant_rows would quantise the
// bf16 values.  KEEP: the bf16 outputs are written.
template <class E, int NQ, bool KEEP>
struct QuantOut : E {
  typedef void quantises;
  static constexpr bool STORES = KEEP;
  uint8_t *q[NQ], *s[NQ];  // codes and exponents, from the tile's first row and column on
  uint32_t ldq, lds;
  int q_valid;             // columns from the tile's first one on that rows of codes have (whole blocks)
  // Rows and columns that do not exist are dropped by the descriptors' bounds: the offsets of lanes whose column is beyond the row of codes, and for exponents of
  // all but one lane of a row, start at 2 GiB (256 rows of codes take less).
  static constexpr uint32_t kDrop = 0x80000000u;
  // pieces of rows row, row + step, ..
  template <int x, int N>
  __device__ __forceinline__ void quantise(const u32x4_t (&piece)[N], int row, int step, int col) const {
    if constexpr (x >= E::NOUT - NQ) {
      constexpr int n = x - (E::NOUT - NQ);
      // (beyond the last column there may be what other rows' NaN left)
      uint32_t v[N][4];
#pragma unroll
      for (int p = 0; p < N; p++)
#pragma unroll
        for (int i = 0; i < 4; i++) v[p][i] = piece[p][i];
      uint2 c[N];
      int e[N];
      quant_blocks_bf16(v, col < E::n_valid ? 0xffffffffu : 0u, c, e);
      const uint32_t at = col < q_valid ? (uint32_t)col : kDrop;
      const uint32_t at_s = col < q_valid && (col & (kQuantBlock - 1)) == 0 ? (uint32_t)col / kQuantBlock : kDrop;
      typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
      const uint32_t last = (uint32_t)E::rows - 1;
#pragma unroll
      for (int p = 0; p < N; p++) {
        const uint32_t r = (uint32_t)(row + p * step);
        __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{c[p].x, c[p].y}, make_rsrc(q[n], last * ldq + (uint32_t)q_valid), at + r * ldq, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b8((uint8_t)e[p], make_rsrc(s[n], last * lds + (uint32_t)q_valid / kQuantBlock), at_s + r * lds, 0, 0);
      }
    }
  }
};

// The rows of a tile: its valid ones, and where they are.
struct QuantTile {
  const uint8_t *a, *as;           // gathered rows: of the whole operand, else of the tile
  uint32_t a_bytes, as_bytes;      // from there to the end of the valid data
  RowMap map;
  const uint8_t *b[2], *bs[2];     // first row of the tile; exponents of the tile's first 128 columns
  int n_valid;                     // columns of the tile that there are
};

// An iteration t multiplies the tiles of block t of K.  A wave's fragments of A (8 registers each: 32 codes a lane) are all in registers, those
// of B in two halves, `lo` (the first product of a dual one) and `hi`.  The waves of a dual product lie one below the other, so that each has whole blocks
// of 128 columns of what it computes from both, which it may have to quantise.
//   phase 1: A x lo, meanwhile hi(t) is read;
//   barrier: every wave has read all it needs of t, and the tiles of t + 1 have landed;
//   phase 2: A x hi, meanwhile lo(t + 1) is read, A(t + 1) fragment by fragment behind the last use of A(t)'s, and the loads of
//            t + SLOTS are issued into the slot of t.
// (The loads of t + SLOTS start in phase 1 already, behind a barrier of their own once the fragments of t have been read.)
// Every fragment is read from LDS once, and no register holds two blocks' values of the same fragment.  MFMAs are inline assembly with a memory
// clobber, so that the order is the one written here (see MfmaDmaCore, whose loads, LDS layout and epilogue these are).
//
// What bounds it: matrix instructions that share their cycles with loads and LDS reads, at a clock that power holds down.  In the launch of 8192 x 4096 x 6400 the pipe is busy in
// 61 % of a unit's cycles at 1.8 GHz, in the K loop in 69 %; waits for LDS are 0.6 % of a wave's time.  A block of K of a 256 x 256 tile (64 MFMAs a wave, 2048 cycles) takes 1.4 to 1.7 us by card.  Where it took
// 1.70: with loads that all hit L2 1.58, without the loads 1.40, without LDS reads too 1.26, i.e. 2048 cycles at 1.6 GHz.  A tile costs
// 7 us besides (first loads, epilogue).  Products of 8192 x 4096 x 6400 172 to 179 us by card (2.40 to 2.50 PFLOP/s), of 16384 x 8192 x 8192 779 us (2.82); the
// register-resident loop of this instruction sustains 3.5 to 4.4 by operands, the vendor library (one scale a tensor) takes 235 us for the former and reaches
// 2.70 on 8192 x 8192 x 8192, where this core reaches 2.65.
// EXACT: the products are computed from the bf16 values that the codes stand for (a code times a power of two is one, but for the ends of bf16's range), whose
// instruction loses none of their bits to an alignment.  A quarter of the rate and a conversion of every fragment, one block of K after the other: for calls of
// few values (quant_exact).
template <int BM_, int NB, int SLOTS, bool EXACT = false>
struct QuantCore {
  static constexpr int BM = BM_, BN = 256 / NB, BK = kQuantBlock;
  static constexpr int WN = NB == 2 ? 1 : 2, WM = 4 / WN, NW = 4, NT = 256;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16, HB = NB * TN / 2;  // HB: B tiles of a half
  static constexpr int A_NI = BM / 32, B_NI = BN / 32;                // wave-wide 16-byte loads a wave and tile
  static constexpr int A_BYTES = BM * BK, B_BYTES = BN * BK;
  // a slot: A, B (both products), then a word per row of A with its exponent, and 64 words per wave and product with that of its columns
  static constexpr int SA_AT = A_BYTES + NB * B_BYTES, SB_AT = SA_AT + BM * 4, SLOT_BYTES = SB_AT + NW * NB * 256;
  static constexpr int LDS_BYTES = SLOTS * SLOT_BYTES;
  static constexpr int L = A_NI + NB * B_NI + 1 + NB;  // loads a wave and iteration
  static constexpr int H = TM * HB;                    // MFMAs of a phase
  // MFMA ahead of which the fragments of t have been read; the loads of t + SLOTS are spread from there on, up to END
  static constexpr int FREE = std::min(HB * std::max(H / (2 * HB), 1), H), END = 2 * H - (SLOTS == 2 ? H * 3 / 8 : 0);
  static constexpr int loads_before(int s) { return s <= FREE ? 0 : s >= END ? L : (s - FREE) * L / (END - FREE); }
  static_assert(LDS_BYTES <= 160 * 1024, "LDS of a compute unit");
  static_assert((SLOTS - 1) * L <= 63, "the wait count must be encodable");
  static_assert(BN / WN == kQuantBlock, "the columns of a wave are one block");
  typedef __attribute__((ext_vector_type(8))) int32_t frag_t;
  typedef __attribute__((ext_vector_type(4))) int rsrc_t;
  static constexpr uint32_t kNowhere = 0xffffff00u;

  __device__ static __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

  // (the words go through v_readfirstlane: see MfmaDmaCore::seek for the wait behind them)
  __device__ static __forceinline__ rsrc_t desc(const uint8_t* base, uint32_t bytes) {
    const uint64_t p = (uint64_t)base;
    rsrc_t r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)p);
    r[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu));
    r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    r[3] = 0x00020000;
    return r;
  }
  __device__ static __forceinline__ void move(rsrc_t& r, uint32_t step) {
    const uint64_t p = (((uint64_t)(uint32_t)r[1] << 32) | (uint32_t)r[0]) + step;
    r[0] = (int)(uint32_t)p;
    r[1] = (int)(uint32_t)(p >> 32);
  }
  // Descriptors of the loads of one iteration.  Their bases step along K; what lies beyond the valid rows stays out of their range, because a row's
  // stride is at least the bytes of K.  Once K is exhausted they are empty: loads deliver zeros.
  struct Cursor {
    rsrc_t a, as, b[NB], bs[NB];
    int left;
  };
  __device__ static __forceinline__ void next(Cursor& c) {
    move(c.a, BK);
    move(c.as, 1);
#pragma unroll
    for (int x = 0; x < NB; x++) {
      move(c.b[x], BK);
      move(c.bs[x], 1);
    }
    if (--c.left == 0) {
      c.a[2] = c.as[2] = 0;
#pragma unroll
      for (int x = 0; x < NB; x++) c.b[x][2] = c.bs[x][2] = 0;
    }
  }

  // C += B A with operands exchanged, as in MfmaDmaCore: register r of lane l is C[m = l % 16][n = 4 * (l / 16) + r].
  __device__ static __forceinline__ void mfma(f32x4_t& acc, const frag_t& b, const frag_t& a, int sb, int sa) {
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                 : "+a"(acc)
                 : "v"(b), "v"(a), "v"(sb), "v"(sa)
                 : "memory");
  }
  __device__ static __forceinline__ void mfma_values(f32x4_t& acc, const bf16x8_t& b, const bf16x8_t& a) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a) : "memory");
  }
  // with a tile load in its shadow: the MFMA is the wait state between the write of M0 and the load
  template <int plus, bool WORD>
  __device__ static __forceinline__ void mfma_load(f32x4_t& acc, const frag_t& b, const frag_t& a, int sb, int sa, const rsrc_t& rsrc, uint32_t base,
                                                   uint32_t voff) {
    if constexpr (WORD)
      asm volatile("s_add_u32 m0, %5, %6\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]\n\t"
                   "buffer_load_ubyte %7, %8, 0 offen lds"
                   : "+a"(acc)
                   : "v"(b), "v"(a), "v"(sb), "v"(sa), "s"(base), "n"(plus), "v"(voff), "s"(rsrc)
                   : "memory", "scc");
    else
      asm volatile("s_add_u32 m0, %5, %6\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]\n\t"
                   "buffer_load_dwordx4 %7, %8, 0 offen lds"
                   : "+a"(acc)
                   : "v"(b), "v"(a), "v"(sb), "v"(sa), "s"(base), "n"(plus), "v"(voff), "s"(rsrc)
                   : "memory", "scc");
  }
  template <int plus, bool WORD>
  __device__ static __forceinline__ void load(const rsrc_t& rsrc, uint32_t base, uint32_t voff) {
    if constexpr (WORD)
      asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_ubyte %2, %3, 0 offen lds" : : "s"(base), "n"(plus), "v"(voff), "s"(rsrc) : "memory", "scc");
    else
      asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds" : : "s"(base), "n"(plus), "v"(voff), "s"(rsrc) : "memory", "scc");
  }

  template <typename P> __device__ static __forceinline__ P lds(uint32_t at) {
    return *(const __attribute__((address_space(3))) P*)(uintptr_t)at;
  }

  template <class Epi>
  __device__ static __forceinline__ void run(char* smem, int nk, const QuantTile& t, int64_t lda, int64_t las, int64_t ldb, int64_t lbs, const Epi& epi) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm0 = (wave / WN) * (BM / WM), wn0 = (wave % WN) * (BN / WN);
    f32x4_t acc[NB][TM][TN];

    // ---- loads: the j-th of a wave fills the 1 KB piece wave + 4 j of a tile, eight rows, lane by lane; pieces swizzled as in MfmaDmaCore
    const int row = wave * 8 + (lane >> 3);
    const uint32_t col = (uint32_t)(((lane & 7) ^ swizzle(row)) << 4);
    uint32_t voa[A_NI], vob[B_NI];
    const int srow = (wave * 64 + lane) & (BM - 1);  // waves beyond the rows load them again
    uint32_t vos;
    if (t.map.gathered()) {
#pragma unroll
      for (int j = 0; j < A_NI; j++) {
        const int r = row + 32 * j;
        voa[j] = r < t.map.rows ? (uint32_t)t.map(r) * (uint32_t)lda + col : kNowhere;
      }
      vos = srow < t.map.rows ? (uint32_t)t.map(srow) * (uint32_t)las : kNowhere;
    } else {
#pragma unroll
      for (int j = 0; j < A_NI; j++) voa[j] = (uint32_t)(row + 32 * j) * (uint32_t)lda + col;
      vos = srow < t.map.rows ? (uint32_t)srow * (uint32_t)las : kNowhere;
    }
#pragma unroll
    for (int j = 0; j < B_NI; j++) vob[j] = (uint32_t)(row + 32 * j) * (uint32_t)ldb + col;
    const uint32_t zero = 0;
    Cursor c;
    const uint32_t k_bytes = (uint32_t)nk * BK;
    c.a = desc(t.a, t.a_bytes);
    c.as = desc(t.as, t.as_bytes);
#pragma unroll
    for (int x = 0; x < NB; x++) {
      c.b[x] = desc(t.b[x], (uint32_t)(t.n_valid - 1) * (uint32_t)ldb + k_bytes);
      // columns of this wave that do not exist have no exponents either
      c.bs[x] = desc(t.bs[x] + (NB == 1 ? (wn0 / kQuantBlock) * lbs : 0), wn0 < t.n_valid ? (uint32_t)nk : 0u);
    }
    c.left = nk;
#pragma unroll
    for (int x = 0; x < NB; x++) asm volatile("" : "+s"(c.b[x]), "+s"(c.bs[x]) : : "memory");
    asm volatile("s_nop 4" : "+s"(c.a), "+s"(c.as) : : "memory");
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    // LDS addresses of a slot's pieces of this wave (16-byte loads, words of A's exponents, of B's)
    const uint32_t p16 = lds0 + (uint32_t)wave * 1024u, pa = lds0 + SA_AT + (uint32_t)((wave * 64) & (BM - 1)) * 4u, pb = lds0 + SB_AT + (uint32_t)wave * (NB * 256u);
    // load number n of an iteration: A, then B, then the exponents; `at`: the slot's offset
    auto each_load = [&](auto n_c, uint32_t at, auto&& f) __attribute__((always_inline)) {
      constexpr int n = decltype(n_c)::value;
      if constexpr (n < A_NI) f(std::integral_constant<int, n * 4096>(), std::false_type(), c.a, p16 + at, voa[n]);
      else if constexpr (n < A_NI + NB * B_NI) {
        constexpr int x = (n - A_NI) / B_NI, j = (n - A_NI) % B_NI;
        f(std::integral_constant<int, A_BYTES + x * B_BYTES + j * 4096>(), std::false_type(), c.b[x], p16 + at, vob[j]);
      } else if constexpr (n == A_NI + NB * B_NI) f(std::integral_constant<int, 0>(), std::true_type(), c.as, pa + at, vos);
      else {
        constexpr int x = n - (A_NI + NB * B_NI + 1);
        f(std::integral_constant<int, x * 256>(), std::true_type(), c.bs[x], pb + at, zero);
      }
    };
    auto issue = [&](auto n_c, uint32_t at) __attribute__((always_inline)) {
      each_load(n_c, at, [&](auto plus, auto word, const rsrc_t& r, uint32_t base, uint32_t vo) __attribute__((always_inline)) {
        load<decltype(plus)::value, decltype(word)::value>(r, base, vo);
      });
    };
    for (int s = 0; s < SLOTS; s++) {
      static_for<L>([&](auto n) __attribute__((always_inline)) { issue(n, (uint32_t)(s * SLOT_BYTES)); });
      next(c);
    }
#pragma unroll
    for (int x = 0; x < NB; x++)
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[x][i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // (pinned: see MfmaDmaCore)
#pragma unroll
    for (int x = 0; x < NB; x++)
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) asm volatile("" : "+a"(acc[x][i][j])::"memory");
    asm volatile("s_nop 7" ::: "memory");

    // ---- fragments: lane l holds 32 codes of row l % 16: the 16-byte pieces l / 16 and 4 + l / 16 (any order of K that both operands share will do)
    const int fr = lane & 15, h = lane >> 4;
    // (EXACT: where only the first of the WM strips of rows has any, its waves share K with the others)
    const bool share = EXACT && WM > 1 && t.map.rows <= BM / WM;
    const int am0 = share ? 0 : wm0;
    uint32_t ao[2], bo[2];
#pragma unroll
    for (int q = 0; q < 2; q++) {
      ao[q] = lds0 + (uint32_t)((am0 + fr) * BK + (((4 * q + h) ^ swizzle(am0 + fr)) << 4));
      bo[q] = lds0 + A_BYTES + (uint32_t)((wn0 + fr) * BK + (((4 * q + h) ^ swizzle(wn0 + fr)) << 4));
    }
    const uint32_t sao = lds0 + SA_AT + (uint32_t)(am0 + fr) * 4u, sbo = pb + (uint32_t)lane * 4u;
    frag_t fa[TM], fl[HB], fh[HB];
    int sa[TM], sl, sh;
    auto frag = [&](const uint32_t (&o)[2], uint32_t at, uint32_t plus) __attribute__((always_inline)) {
      const u32x4_t p = lds<u32x4_t>(o[0] + at + plus), q = lds<u32x4_t>(o[1] + at + plus);
      return __builtin_bit_cast(frag_t, __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_a = [&](auto i_c, uint32_t at) __attribute__((always_inline)) {
      constexpr int i = decltype(i_c)::value;
      sa[i] = lds<int32_t>(sao + at + i * 64);
      fa[i] = frag(ao, at, i * 16 * BK);
    };
    auto read_lo = [&](auto j_c, uint32_t at) __attribute__((always_inline)) {
      constexpr int j = decltype(j_c)::value;
      if constexpr (j == 0) sl = lds<int32_t>(sbo + at);
      fl[j] = frag(bo, at, j * 16 * BK);
    };
    auto read_hi = [&](auto j_c, uint32_t at) __attribute__((always_inline)) {
      constexpr int j = decltype(j_c)::value;
      if constexpr (j == 0) sh = lds<int32_t>(sbo + at + (NB - 1) * 256);
      fh[j] = frag(bo, at, NB == 2 ? B_BYTES + j * 16 * BK : (HB + j) * 16 * BK);
    };
    auto landed = [&](auto n) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(n)::value) : "memory");
      __syncthreads();
    };
    uint32_t cur = 0;
    if constexpr (EXACT) {
      // the bf16 values of a quarter of a fragment: an operand of v_mfma_f32_16x16x32_bf16
      auto values = [](const frag_t& f, auto q_c, int byte) __attribute__((always_inline)) {
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
        constexpr int q = decltype(q_c)::value;
        const float scale = __uint_as_float((uint32_t)byte << 23);
        const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * q], scale, false),
                       b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * q], scale, true),
                       c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * q + 1], scale, false),
                       d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)f[2 * q + 1], scale, true);
        bf16x8_t v = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
        asm volatile("s_nop 1" : "+v"(v));  // two wait states between the conversions and the matrix instructions
        return v;
      };
      for (int it = 0; it < nk; it++) {
        landed(std::integral_constant<int, (SLOTS - 1) * L>());
        static_for<TM>([&](auto i) __attribute__((always_inline)) { read_a(i, cur); });
        static_for<HB>([&](auto j) __attribute__((always_inline)) { read_lo(j, cur); });
        static_for<HB>([&](auto j) __attribute__((always_inline)) { read_hi(j, cur); });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __syncthreads();  // every wave has read the slot: the loads of it + SLOTS may overwrite it
        static_for<L>([&](auto n) __attribute__((always_inline)) { issue(n, cur); });
        next(c);
        static_for<4>([&](auto q_c) __attribute__((always_inline)) {
          if (share && decltype(q_c)::value / (4 / WM) != wave / WN) return;
          bf16x8_t va[TM];
          static_for<TM>([&](auto i) __attribute__((always_inline)) { va[decltype(i)::value] = values(fa[decltype(i)::value], q_c, sa[decltype(i)::value]); });
          static_for<2 * HB>([&](auto t_c) __attribute__((always_inline)) {
            constexpr int t = decltype(t_c)::value, j = t % HB;
            const bf16x8_t vb = values(t < HB ? fl[j] : fh[j], q_c, t < HB ? sl : sh);
            static_for<TM>([&](auto i_c) __attribute__((always_inline)) {
              constexpr int i = decltype(i_c)::value;
              mfma_values(t < HB ? acc[0][i][j] : NB == 2 ? acc[NB - 1][i][j] : acc[0][i][TN - HB + j], vb, va[i]);
            });
          });
        });
        cur = cur == (SLOTS - 1) * SLOT_BYTES ? 0u : cur + SLOT_BYTES;
      }
    } else {
      landed(std::integral_constant<int, (SLOTS - 1) * L>());
      static_for<HB>([&](auto j) __attribute__((always_inline)) { read_lo(j, 0); });
      static_for<TM - 1>([&](auto i) __attribute__((always_inline)) { read_a(i, 0); });
      for (int it = 0; it < nk; it++) {
        const uint32_t nxt = cur == (SLOTS - 1) * SLOT_BYTES ? 0u : cur + SLOT_BYTES;
        static_for<2 * H>([&](auto slot_c) __attribute__((always_inline)) {
          constexpr int s = decltype(slot_c)::value, m = s % H, i = m / HB, j = m % HB, step = std::max(H / (2 * HB), 1);
          constexpr int n0 = loads_before(s), n1 = loads_before(s + 1);
          if constexpr (s == FREE && FREE < H) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __syncthreads();
          }
          if constexpr (s == H) landed(std::integral_constant<int, (SLOTS - 2) * L + n0>());
          if constexpr (s < H) {
            if constexpr (s == 0) read_a(std::integral_constant<int, TM - 1>(), cur);
            if constexpr (m % step == 0 && m / step < HB) read_hi(std::integral_constant<int, m / step>(), cur);
          } else {
            if constexpr (m % step == 0 && m / step < HB) read_lo(std::integral_constant<int, m / step>(), nxt);
            if constexpr (m > 0 && j == 0) read_a(std::integral_constant<int, i - 1>(), nxt);
          }
          f32x4_t& x = s < H ? acc[0][i][j] : NB == 2 ? acc[NB - 1][i][j] : acc[0][i][TN - HB + j];
          const frag_t& fb = s < H ? fl[j] : fh[j];
          const int sb = s < H ? sl : sh;
          if constexpr (n1 > n0) {
            each_load(std::integral_constant<int, n0>(), cur, [&](auto plus, auto word, const rsrc_t& r, uint32_t base, uint32_t vo) __attribute__((always_inline)) {
              mfma_load<decltype(plus)::value, decltype(word)::value>(x, fb, fa[i], sb, sa[i], r, base, vo);
            });
            static_for<n1 - n0 - 1>([&](auto y) __attribute__((always_inline)) { issue(std::integral_constant<int, n0 + 1 + decltype(y)::value>(), cur); });
          } else {
            mfma(x, fb, fa[i], sb, sa[i]);
          }
        });
        next(c);
        cur = nxt;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // (the wait behind the last MFMA, and the order of accumulator copies behind it: see MfmaDmaCore; these MFMAs take twice as long)
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15"
                 : "+a"(acc[NB - 1][TM - 1][TN - 1])
                 :
                 : "memory");
#pragma unroll
    for (int x = 0; x < NB; x++)
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) asm volatile("" : "+a"(acc[x][i][j])::"memory");
    __syncthreads();
    if constexpr (EXACT)
      if (share) {
        constexpr int kSums = NB * TM * TN * 1024;  // bytes of a wave's accumulators
        static_assert((WM - 1) * WN * kSums <= LDS_BYTES, "sums of the waves that share K");
        const uint32_t at = lds0 + (uint32_t)(lane * 16);
        auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
          for (int x = 0; x < NB; x++)
#pragma unroll
            for (int i = 0; i < TM; i++)
#pragma unroll
              for (int j = 0; j < TN; j++) f(acc[x][i][j], at + (uint32_t)(((x * TM + i) * TN + j) * 1024));
        };
        if (wave >= WN)
          each([&](f32x4_t& v, uint32_t o) __attribute__((always_inline)) { *(__attribute__((address_space(3))) f32x4_t*)(uintptr_t)(o + (wave - WN) * kSums) = v; });
        __syncthreads();
        if (wave < WN)
          for (int w = 0; w < WM - 1; w++)
            each([&](f32x4_t& v, uint32_t o) __attribute__((always_inline)) { v += lds<f32x4_t>(o + (w * WN + wave) * kSums); });
        __syncthreads();
      }
    TileEpilogue<NB, TM, TN, NW, LDS_BYTES, true, TM == 1 ? 16 : 32>::run(smem, acc, epi, wave, lane, wm0, wn0);
  }
};

}  // namespace moe
