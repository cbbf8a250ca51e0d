// moe_quant_gemm, moe_quant_expert_fwd / _bwd: grouped products of block-scaled 8-bit tensors.
#include "expert_impl.h"
#include "quant_core.h"

namespace moe {

// ------------------------------------------------------------------------------------------ kernel
template <int NB, int EPI> using Epi8 = Epilogue<bf16_t, NB, EPI>;
// Of an epilogue's outputs the last one alone: H of a forward pass that keeps nothing for a backward pass.
template <class E>
struct LastOutput : E {
  static constexpr int NOUT = 1;
  template <int NB, int NA>
  __device__ __forceinline__ void apply(const float (&v)[NB][4], const float (&a)[NA][4], float sc, float (&o)[1][4]) const {
    float all[E::NOUT][4];
    E::apply(v, a, sc, all);
#pragma unroll
    for (int q = 0; q < 4; q++) o[0][q] = all[E::NOUT - 1][q];
  }
};

template <class E, int NQ, bool KEEP>
__device__ __forceinline__ void set_quantised(QuantOut<E, NQ, KEEP>& epi, const QuantGemm& p, int64_t row0, int n0) {
#pragma unroll
  for (int x = 0; x < NQ; x++) {
    epi.q[x] = p.q[x] + row0 * p.ldq + n0;
    epi.s[x] = p.qs[x] + row0 * p.lds + n0 / kQuantBlock;
  }
  epi.ldq = (uint32_t)p.ldq;
  epi.lds = (uint32_t)p.lds;
  epi.q_valid = (p.N + kQuantBlock - 1) / kQuantBlock * kQuantBlock - n0;
}
template <class E>
__device__ __forceinline__ void set_quantised(E&, const QuantGemm&, int64_t, int) {}

// Blocks [k0, k0 + nk) of K; a part of a sum: `part`.
template <class Core, class Epi, int NB, bool PART = false>
__device__ __forceinline__ void quant_tile(const QuantGemm& p, const RowTile& t, int nt, char* smem, int part = 0) {
  const int rows = tile_rows(t), n0 = nt * Core::BN;
  const int k0 = PART ? part * p.k_part : 0, nk = PART ? min(p.k_part, p.nk - k0) : p.nk;
  QuantTile q;
  q.map = {p.a_index, p.a_index ? p.a_index_div : 1, t.row0_in, rows};
  const int64_t row0 = p.a_index ? 0 : t.row0_in;
  const uint32_t last = (uint32_t)((p.a_index ? p.a_src_rows : rows) - 1);
  q.a = p.A + row0 * p.lda + k0 * kQuantBlock;
  q.as = p.As + row0 * p.las + k0;
  q.a_bytes = last * (uint32_t)p.lda + (uint32_t)nk * kQuantBlock;
  q.as_bytes = last * (uint32_t)p.las + (uint32_t)nk;
#pragma unroll
  for (int x = 0; x < NB; x++) {
    q.b[x] = p.B[x] + t.group * p.b_group + n0 * p.ldb + k0 * kQuantBlock;
    q.bs[x] = p.Bs[x] + t.group * p.bs_group + n0 / kQuantBlock * p.lbs + k0;
  }
  q.n_valid = min(Core::BN, p.N - n0);
  Epi epi;
  const int64_t c_off = ((int64_t)t.row0_out * p.ldc + n0) * Epi::OES;
#pragma unroll
  for (int x = 0; x < Epi::NOUT; x++)
    epi.out[x] = (PART ? (char*)(p.part + (int64_t)(part * NB + x) * p.n_rows * p.N) : (char*)p.out[x]) + c_off;
#pragma unroll
  for (int x = 0; x < Epi::NAUX; x++) epi.in[x] = (const char*)p.in[x] + c_off;
  epi.ldc = p.ldc;
  epi.rows = rows;
  epi.n_valid = q.n_valid;
  epi.scale = p.c_scale;
  epi.index = p.a_index + t.row0_in;
  set_quantised(epi, p, t.row0_out, n0);
  Core::run(smem, nk, q, p.lda, p.las, p.ldb, p.lbs, epi);
}

// Heights of the tiles: 256, and for what is left of a group 128 and 64 (tiles of up to 64 rows are bound by streaming the matrix, whatever
// their height).
template <int NB> using QuantTall = QuantCore<256, NB, 2>;
template <int NB> using QuantMid = QuantCore<128, NB, 3>;
template <int NB, bool EXACT = false> using QuantShort = QuantCore<64, NB, 3, EXACT>;

// Tiles are dealt to the XCDs as in row_gemm_block: band by band of kBandRows row tiles, column by column within a band, runs of 32 (launches of
// few rounds: of 8) consecutive tiles to an XCD.
template <int NB, class Epi>
__device__ __forceinline__ void quant_gemm_block(const QuantGemm& p, int block, char* smem) {
  constexpr int BN = 256 / NB;
  const int ntn = (p.N + BN - 1) / BN;
  const int n_mt = *p.n_tiles;
  const int total = n_mt * ntn, q = dealt_tile(block, total);
  if (q >= total) return;
  // Launches of four rounds and more take bands two from the front, one from the back, until a third of them have come from the back: short tiles, bound
  // by streaming their matrices, beside tall ones.  (The last band, which may have fewer rows, stays the last.  Longest first and so, us: gate/up of
  // 16384 rows, d = 2048, 60 experts of 1408, Zipf loads, 202 and 184, of 32768 264 and 252, down 137 and 136; 16384 rows, d = 7168, 128 experts of 2048 870
  // and 876, down 472 and 457; launches of two to three rounds lose, gate/up of 9003 rows, d = 1000, 24 experts of 1368, 74 and 83, dH 75 and 93.)
  const TilePlace at = band_tile(q, n_mt, ntn, total >> 8 >= 4 ? n_mt / kBandRows / 3 : 0);
  RowTile t = p.tiles[at.mt];
  t.group = __builtin_amdgcn_readfirstlane(t.group);
  t.row0_in = __builtin_amdgcn_readfirstlane(t.row0_in);
  t.rows = __builtin_amdgcn_readfirstlane(t.rows);
  t.row0_out = __builtin_amdgcn_readfirstlane(t.row0_out);
  if (tile_rows(t) > 128) quant_tile<QuantTall<NB>, Epi, NB>(p, t, at.nt, smem);
  else if (tile_rows(t) > 64) quant_tile<QuantMid<NB>, Epi, NB>(p, t, at.nt, smem);
  else quant_tile<QuantShort<NB>, Epi, NB>(p, t, at.nt, smem);
}
template <int NB, class Epi>
__global__ __launch_bounds__(256, 1) void quant_gemm_kernel(QuantGemm p) {
  extern __shared__ __align__(16) char smem[];
  quant_gemm_block<NB, Epi>(p, blockIdx.x, smem);
}
// An input gradient and a weight gradient that does not depend on it (bf16) in one launch, as in row_w_gemm_kernel: the tiles of the one fill the units
// that the last tiles of the other leave idle.  (Training steps apart and together, us: T = 3001, d = 1000, 24 experts of 1368 537 and 501; T = 4096, d = 2048,
// 60 of 1408 1432 and 1418; T = 1426, d = 2688, one of 3584 289 and 231.)
template <class Epi, class WCore, int WNB>
__global__ __launch_bounds__(256, 1) void quant_w_gemm_kernel(QuantGemm p, WGemm w, int first_w, int rows, int w_blocks) {
  extern __shared__ __align__(16) char smem[];
  const int b = (int)blockIdx.x, row = b - first_w, wb = row < 0 ? b : row - rows;
  if (row >= 0 && row < rows) quant_gemm_block<1, Epi>(p, row, smem);
  else if (wb < w_blocks) w_gemm_block<WCore, WNB, true>(w, wb, smem);
}

// Calls of few rows (quant_small): tiles of 64 rows, found in the offsets by the blocks themselves, which costs about a microsecond where a plan takes a
// launch of seven.
template <int NB, class Epi, bool EXACT>
__global__ __launch_bounds__(256, 1) void quant_small_gemm_kernel(QuantGemm p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int BN = 256 / NB, BM = 64;
  const int ntn = (p.N + BN - 1) / BN, mt = blockIdx.x / ntn, nt = blockIdx.x - mt * ntn;
  // four groups a thread: the tiles before them, by shuffles and through LDS
  __shared__ int32_t wsum[4], found[3];
  const int g0 = threadIdx.x * 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int off[5], n = 0;
#pragma unroll
  for (int i = 0; i < 5; i++) off[i] = p.offsets[min(g0 + i, p.n_groups)];
#pragma unroll
  for (int i = 0; i < 4; i++) n += (max(off[i + 1] - off[i], 0) + BM - 1) / BM;
  int end = n;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int u = __shfl_up(end, m, kWave);
    if (lane >= m) end += u;
  }
  if (lane == kWave - 1) wsum[wave] = end;
  if (threadIdx.x < 3) found[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 3; w++) end += w < wave ? wsum[w] : 0;
  int first = end - n;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int c = max(off[i + 1] - off[i], 0), k = (c + BM - 1) / BM;
    if (mt >= first && mt < first + k) {
      found[0] = g0 + i;
      found[1] = off[i] + (mt - first) * BM;
      found[2] = min(BM, c - (mt - first) * BM);
    }
    first += k;
  }
  __syncthreads();
  RowTile t;
  t.group = __builtin_amdgcn_readfirstlane(found[0]);
  t.row0_in = __builtin_amdgcn_readfirstlane(found[1]);
  t.rows = __builtin_amdgcn_readfirstlane(found[2]);
  if (t.rows == 0) return;
  t.row0_out = t.row0_in;
  quant_tile<QuantShort<NB, EXACT>, Epi, NB>(p, t, nt, smem);
}

// One group of n_rows rows: tiles of one height, in parts along K or not; those of a last round that is not full cut into 2 or 4 lower ones.
template <class Epi, bool PART>
__global__ __launch_bounds__(256, 1) void quant_direct_gemm_kernel(QuantGemm p) {
  extern __shared__ __align__(16) char smem[];
  const int ntn = (p.N + 255) / 256, n_mt = (p.n_rows + p.height - 1) / p.height;
  const int part = PART ? blockIdx.x / p.part_blocks : 0, block = PART ? blockIdx.x - part * p.part_blocks : blockIdx.x;
  const int total = n_mt * ntn;
  const CutTile cut = cut_tile(block, total, PART ? 1 : p.tail);
  if (cut.q >= total) return;
  const TilePlace at = band_tile(cut.q, n_mt, ntn, 0);
  const int height = p.height / cut.pieces;
  RowTile t;
  t.group = 0;
  t.row0_in = t.row0_out = at.mt * p.height + cut.piece * height;
  t.rows = min(height, p.n_rows - t.row0_in);
  if (t.rows <= 0) return;
  if (t.rows > 128) quant_tile<QuantTall<1>, Epi, 1, PART>(p, t, at.nt, smem, part);
  else if (t.rows > 64) quant_tile<QuantMid<1>, Epi, 1, PART>(p, t, at.nt, smem, part);
  else quant_tile<QuantShort<1>, Epi, 1, PART>(p, t, at.nt, smem, part);
}

// Calls of up to 512 rows, of up to 1024 over eight groups or more: above, a group's tiles read its matrix too often.  (Forward passes with a plan and so, us:
// d = 2048, 60 experts of 1408, 32 rows 36 and 32, 512 90 and 82, 1024 98 and 98, 2048 124 and 134; d = 1024, 8 experts of 2816, 32 rows 34 and 32,
// 512 46 and 45, 1024 65 and 48, 2048 75 and 70, 4096 100 and 109; products of K = 4096, N = 6400, 4 groups, 512 rows 50 and 40, 1024 59 and 72.
// Sums in parts, joined by another launch, gain where a call has four rows (K = 2048, N = 1408: 13.8 and 11.6 us) and lose from eight on.)
static bool quant_small(int n_groups, int n_rows) { return n_rows <= 512 || (n_groups >= 8 && n_rows <= 1024); }
// Products whose outputs are quantised, of up to 2^16 values of them: computed from bf16 values, in tiles of 64 rows.  The 8-bit instruction's error, 1.5e-5, moves one
// in 600 of the outputs of silu(G) U to the other side of a border between codes, one in 1000 of gelu(G): small ones above all, by their share of the sum of squares one
// in 5000 to 15000.  Over many that adds 1e-3 to the 1.7e-3 of the next product's rounding to bf16, but where few of them carry weight, the error is that of the one which
// carries most (0.0056 of a training step's dX, 0.0051 of a forward pass's Y of 2 tokens; from bf16 values 0.0017; 1800 random calls of 2^16 to 2^20 values on the 8-bit
// instruction at most 0.0038).  The line is one for the tensor: a row of d_ff values of which one is moved may be off by more (see moe_hip.h).  Gate and up of 64 rows, 60 experts of
// 2048 x 1408, which are more than that: 28 us from bf16 values, 21 on the 8-bit instruction.
static bool quant_exact(int64_t n_rows, int cols) { return n_rows * cols <= 1 << 16; }
template <int NB, class Epi, bool EXACT = false>
static void launch_small(const char* label, const QuantGemm& p, hipStream_t st) {
  const int tiles = p.n_rows / 64 + std::min(p.n_groups, p.n_rows);  // at most
  launch_gemm<quant_small_gemm_kernel<NB, Epi, EXACT>>(label, (unsigned)(tiles * ceil_div(p.N, 256 / NB)), 256, QuantShort<NB, EXACT>::LDS_BYTES, st, p);
}

// A product of one group: height and parts by an estimate in microseconds, of a block of K (`iter`) and of what a tile takes besides (`fixed`).
// (Tall tiles in one part, and by this rule, us: 16 x 7168 x 2048 32 and 15, 256 x 7168 x 2048 34 and 21, 1024 x 7168 x 2048 37 and 30, 512 x 4096 x 6400 33 and 33; rounds
// of tall tiles only, and the last one cut: 8192 x 4096 x 6400 195 and 177, 2048 x 7168 x 2048 71 and 39.  Over 18 sizes it was within 10 % of the best choice.)
struct DirectQuant {
  int height = 256, parts = 1, tail = 1;
  double us = 0;
};
static DirectQuant direct_quant(int n_rows, int N, int nk) {
  static const int kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  static const double kIter[] = {1.45, 0.9, 0.6}, kFixed[] = {7, 6, 5};
  DirectQuant best;
  for (int h = 0; h < 3; h++)
    for (int parts : kParts) {
      if (parts > 1 && (2 * parts > nk || (int64_t)n_rows * N > (int64_t)1 << 24)) continue;
      DirectQuant c;
      c.height = 256 >> h;
      const int its = ceil_div(nk, parts);
      c.parts = ceil_div(nk, its);
      const int64_t tiles = (int64_t)ceil_div(n_rows, c.height) * ceil_div(N, 256), blocks = tiles * c.parts;
      const auto tile_us = [&](int k) { return kFixed[k] + its * kIter[k]; };
      c.us = (double)(blocks / 256) * tile_us(h);
      const int rest = (int)(blocks % 256);
      if (rest > 0) {
        double last = tile_us(h);
        if (c.parts == 1)
          for (int k = h + 1; k < 3; k++)
            if ((rest << (k - h)) <= 256 && tile_us(k) < last) {
              last = tile_us(k);
              c.tail = 1 << (k - h);
            }
        c.us += last;
      }
      if (c.parts > 1) c.us += 7 + 4e-6 / 4 * c.parts * n_rows * N;
      if (best.us == 0 || c.us < best.us) best = c;
    }
  return best;
}
static size_t direct_part_bytes(int n_rows, int N, int nk) {
  if (n_rows == 0) return 0;
  const int parts = direct_quant(n_rows, N, nk).parts;
  return parts == 1 ? 0 : align_up((size_t)parts * n_rows * N * 4, 256);
}
static void launch_direct(const char* label, QuantGemm p, float* part, hipStream_t st) {
  const DirectQuant c = direct_quant(p.n_rows, p.N, p.nk);
  p.height = c.height;
  p.tail = c.tail;
  p.n_parts = c.parts;
  p.k_part = ceil_div(p.nk, c.parts);
  p.part = part;
  const int tiles = ceil_div(p.n_rows, c.height) * ceil_div(p.N, 256);
  p.part_blocks = cut_tile_blocks(tiles, c.tail);
  constexpr int kLds = std::max({QuantTall<1>::LDS_BYTES, QuantMid<1>::LDS_BYTES, QuantShort<1>::LDS_BYTES});
  if (c.parts == 1) {
    launch_gemm<quant_direct_gemm_kernel<Epi8<1, EPI_STORE>, false>>(label, (unsigned)p.part_blocks, 256, kLds, st, p);
    return;
  }
  p.part_blocks = tiles;
  QuantGemm q = p;
  q.ldc = p.N;
  launch_gemm<quant_direct_gemm_kernel<Epi8<1, EPI_PART>, true>>(label, (unsigned)(tiles * c.parts), 256, kLds, st, q);
  launch_reduce<bf16_t, 1, EPI_STORE>(part, c.parts, (int64_t)p.n_rows * p.N, p.out, nullptr, st);
}

// At most max_tiles row tiles (the device knows how many there are).
template <int NB, class Epi>
static void launch_quant(const char* label, const QuantGemm& p, int max_tiles, hipStream_t st) {
  const unsigned blocks = row_block_count(max_tiles, p.N, 256 / NB);
  if (blocks == 0) return;
  constexpr int kLds = std::max({QuantTall<NB>::LDS_BYTES, QuantMid<NB>::LDS_BYTES, QuantShort<NB>::LDS_BYTES});
  launch_gemm<quant_gemm_kernel<NB, Epi>>(label, blocks, 256, kLds, st, p);
}
// w_first: the tiles of the weight gradient come first (first_w blocks, a multiple of 8, so that the row tiles keep their XCDs), else last.
template <class Epi, class WCore, int WNB>
static void launch_quant_w(const char* label, const QuantGemm& p, int max_tiles, const WGemm& w, bool w_first, hipStream_t st) {
  constexpr int kLds = std::max({QuantTall<1>::LDS_BYTES, QuantMid<1>::LDS_BYTES, QuantShort<1>::LDS_BYTES, WCore::LDS_BYTES});
  const unsigned rows = row_block_count(max_tiles, p.N, 256), w_blocks = w_block_count<WCore>(w);
  const unsigned first_w = w_first ? (w_blocks + 7) / 8 * 8 : 0;
  launch_gemm<quant_w_gemm_kernel<Epi, WCore, WNB>>(label, rows + (w_first ? first_w : w_blocks), 256, kLds, st, p, w, (int)first_w, (int)rows, (int)w_blocks);
}

// ------------------------------------------------------------------------------------ one product
static int quant_tiles(int n_groups, int n_rows) { return max_row_tiles(MOE_BF16, n_groups, n_rows, INT32_MAX); }
static size_t quant_plan_size(int n_groups, int n_rows) { return align_up(plan_bytes(n_groups, plan_cap(n_groups, n_rows) + 1), 256); }

static int check_groups(int n_groups, int n_rows, const char* who) {
  if (n_groups >= 1 && n_groups <= MOE_MAX_EXPERTS && n_rows >= 0 && n_rows < 1 << 30) return MOE_OK;
  set_error("%s: bad n_groups=%d n_rows=%d", who, n_groups, n_rows);
  return MOE_EINVAL;
}
// the tiles of a launch are counted in 32 bits
static int check_launch(int n_groups, int n_rows, int64_t cols, const char* who) {
  if ((quant_tiles(n_groups, n_rows) + 1) * (cols / 128 + 1) < (int64_t)1 << 31) return MOE_OK;
  set_error("%s: %d rows of %lld columns are too many", who, n_rows, (long long)cols);
  return MOE_EINVAL;
}

}  // namespace moe

extern "C" size_t moe_quant_gemm_workspace_bytes(int32_t n_groups, int32_t n_rows, int32_t K, int32_t N) {
  using namespace moe;
  if (n_groups < 1 || n_groups > MOE_MAX_EXPERTS || n_rows < 0 || K < 1 || N < 1) return 0;
  return std::max(quant_plan_size(n_groups, n_rows), n_groups == 1 ? direct_part_bytes(n_rows, N, (int)quant_blocks(K)) : 0);
}

extern "C" int moe_quant_gemm(int32_t n_groups, const int32_t* offsets, int32_t n_rows, int32_t K, int32_t N, const void* A, const void* As,
                              const void* B, const void* Bs, void* C, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  const int rc = check_groups(n_groups, n_rows, "moe_quant_gemm");
  if (rc) return rc;
  if (K < 1 || N < 1 || N % 8 || K > 1 << 22 || N > 1 << 22 || (!offsets && n_groups != 1)) {
    set_error("moe_quant_gemm: bad K=%d N=%d n_groups=%d (N a multiple of 8; one group where there are no offsets)", K, N, n_groups);
    return MOE_EINVAL;
  }
  if (!B || !Bs || !ws || (n_rows > 0 && (!A || !As || !C))) {
    set_error("moe_quant_gemm: null pointer");
    return MOE_EINVAL;
  }
  if (!aligned16(A) || !aligned16(B) || !aligned16(C) || !aligned16(ws)) {
    set_error("moe_quant_gemm: every tensor must be 16-byte aligned");
    return MOE_EINVAL;
  }
  const int rl = check_launch(n_groups, n_rows, N, "moe_quant_gemm");
  if (rl) return rl;
  const size_t need = moe_quant_gemm_workspace_bytes(n_groups, n_rows, K, N);
  if (ws_bytes < need) {
    set_error("moe_quant_gemm: workspace of %zu bytes, need %zu", ws_bytes, need);
    return MOE_EWS;
  }
  if (n_rows == 0) return MOE_OK;
  hipStream_t st = (hipStream_t)stream;
  QuantGemm p = {};
  p.n_rows = n_rows; p.n_groups = n_groups; p.N = N; p.nk = (int)quant_blocks(K);
  p.A = (const uint8_t*)A; p.As = (const uint8_t*)As; p.lda = quant_row(K); p.las = p.nk;
  p.B[0] = (const uint8_t*)B; p.Bs[0] = (const uint8_t*)Bs; p.ldb = p.lda; p.b_group = N * p.ldb; p.lbs = p.nk; p.bs_group = quant_blocks(N) * p.lbs;
  p.out[0] = C; p.ldc = N;
  if (!offsets) {
    launch_direct("quant_gemm", p, (float*)ws, st);
  } else if (quant_small(n_groups, n_rows)) {
    p.offsets = offsets;
    launch_small<1, Epi8<1, EPI_STORE>>("quant_gemm", p, st);
  } else {
    const Plan pl = carve_plan(ws, n_groups, plan_cap(n_groups, n_rows));
    launch_plan(offsets, n_groups, 256, pl, nullptr, nullptr, st);
    p.tiles = pl.tiles; p.n_tiles = pl.n_tiles;
    launch_quant<1, Epi8<1, EPI_STORE>>("quant_gemm", p, quant_tiles(n_groups, n_rows), st);
  }
  return launch_status("moe_quant_gemm");
}

// ---------------------------------------------------------------------------------------- experts
namespace moe {

extern template void expert_dw_impl<PATH_BF16_SMALL>(const BwdArgs&, hipStream_t);

// Workspace: plan; codes and exponents of H (forward) or of [dG | dU]; backward: dG and dU in bf16, for the weight gradients.
struct QuantSpace {
  size_t plan, act, codes, scales;
  QuantSpace(const moe_shape_t* s, int n_groups, int n_rows, int mats)
      : plan(quant_plan_size(n_groups, n_rows)), act(align_up((size_t)n_rows * s->d_ff * 2, 256)),
        codes(align_up((size_t)n_rows * mats * quant_row(s->d_ff), 256)), scales(align_up((size_t)n_rows * mats * quant_blocks(s->d_ff), 256)) {}
  size_t fwd() const { return plan + codes + scales; }
  size_t bwd() const { return plan + 2 * act + codes + scales; }
};

static int check_quant_expert(const moe_shape_t* s, int n_groups, const int32_t* offsets, int n_rows, const int32_t* src_of,
                              const moe_quant_weights_t* W, bool bwd, const char* who) {
  int rc = check_shape(s, who);
  if (rc) return rc;
  if (s->dtype != MOE_BF16) {
    set_error("%s: the experts' saved tensors are bf16", who);
    return MOE_EDTYPE;
  }
  rc = check_groups(n_groups, n_rows, who);
  if (rc) return rc;
  rc = check_launch(n_groups, n_rows, std::max(s->d, s->d_ff), who);
  if (rc) return rc;
  // (256 rows of [dG | dU] codes, and of bf16 outputs, within 2 GiB: QuantOut)
  if (512 * quant_row(std::max(s->d, s->d_ff)) >= (int64_t)1 << 31) {
    set_error("%s: rows of d=%d, d_ff=%d values are too long", who, s->d, s->d_ff);
    return MOE_EINVAL;
  }
  if (!offsets || !W) {
    set_error("%s: null pointer", who);
    return MOE_EINVAL;
  }
  if (src_of && n_rows != s->T * s->k) {
    set_error("%s: rows read in place are T*k rows", who);
    return MOE_EINVAL;
  }
  if (src_of && (int64_t)s->T * quant_row(s->d) >= ((int64_t)1 << 32) - 4096) {
    set_error("%s: rows read in place must take less than 4 GiB (32-bit byte offsets)", who);
    return MOE_EINVAL;
  }
  const void* fwd_ptrs[] = {W->WgT, W->WgT_s, W->WdT, W->WdT_s, W->WuT, W->WuT_s};
  const void* bwd_ptrs[] = {W->Wgu, W->Wgu_s, W->Wd, W->Wd_s};
  bool null = false, aligned = true;
  if (bwd) {
    for (const void* p : bwd_ptrs) null = null || !p;
    aligned = aligned16(W->Wgu) && aligned16(W->Wd);
  } else {
    for (int i = 0; i < (W->gated ? 6 : 4); i++) null = null || !fwd_ptrs[i];
    aligned = aligned16(W->WgT) && aligned16(W->WuT) && aligned16(W->WdT);
  }
  if (null || !aligned) {
    set_error(null ? "%s: null pointer among the weights" : "%s: every tensor must be 16-byte aligned", who);
    return MOE_EINVAL;
  }
  return MOE_OK;
}
static int fail_null(const char* who) {
  set_error("%s: null pointer", who);
  return MOE_EINVAL;
}

}  // namespace moe

extern "C" size_t moe_quant_expert_fwd_workspace_bytes(const moe_shape_t* shape, int32_t n_groups, int32_t n_rows) {
  using namespace moe;
  if (!shape || n_groups < 1 || n_rows < 0 || shape->d < 1 || shape->d_ff < 1) return 0;
  return QuantSpace(shape, n_groups, n_rows, 1).fwd();
}
extern "C" size_t moe_quant_expert_bwd_workspace_bytes(const moe_shape_t* shape, int32_t n_groups, int32_t n_rows) {
  using namespace moe;
  if (!shape || n_groups < 1 || n_rows < 0 || shape->d < 1 || shape->d_ff < 1) return 0;
  return QuantSpace(shape, n_groups, n_rows, 2).bwd();
}

extern "C" int moe_quant_expert_fwd(const moe_shape_t* shape, int32_t n_groups, const int32_t* offsets, int32_t n_rows, const int32_t* src_of,
                                    const void* XQ, const void* XS, const moe_quant_weights_t* W, void* G, void* U, void* H, void* Yout,
                                    const void* plan, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  static const char* who = "moe_quant_expert_fwd";
  const int rc = check_quant_expert(shape, n_groups, offsets, n_rows, src_of, W, false, who);
  if (rc) return rc;
  const bool gated = W->gated != 0;
  if (!ws || (n_rows > 0 && (!XQ || !XS || !Yout || (G && (!H || (gated && !U))) || (!G && H)))) return fail_null(who);
  const void* ptrs[] = {XQ, G, U, H, Yout, plan, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) {
      set_error("%s: every tensor must be 16-byte aligned", who);
      return MOE_EINVAL;
    }
  if (plan && (n_groups != shape->E || n_rows != shape->T * shape->k)) {
    set_error("%s: a plan is that of the shape: E groups, T*k rows", who);
    return MOE_EINVAL;
  }
  const QuantSpace sp(shape, n_groups, n_rows, 1);
  if (ws_bytes < sp.fwd()) {
    set_error("%s: workspace of %zu bytes, need %zu", who, ws_bytes, sp.fwd());
    return MOE_EWS;
  }
  if (n_rows == 0) return MOE_OK;
  hipStream_t st = (hipStream_t)stream;
  const int d = shape->d, F = shape->d_ff, tiles = max_row_tiles(MOE_BF16, n_groups, n_rows, d);
  const bool exact = quant_exact(n_rows, F), small = exact || quant_small(n_groups, n_rows);
  const Plan pl = carve_plan(plan ? (void*)plan : ws, n_groups, plan_cap(n_groups, n_rows));
  if (!plan && !small) launch_plan(offsets, n_groups, 256, pl, nullptr, nullptr, st);
  uint8_t *HQ = (uint8_t*)ws + sp.plan, *HS = HQ + sp.codes;
  QuantGemm p = {};
  p.tiles = pl.tiles; p.n_tiles = pl.n_tiles; p.offsets = offsets; p.n_rows = n_rows; p.n_groups = n_groups;
  p.N = F; p.nk = (int)quant_blocks(d);
  p.A = (const uint8_t*)XQ; p.As = (const uint8_t*)XS; p.lda = quant_row(d); p.las = p.nk;
  p.a_index = src_of; p.a_index_div = shape->k; p.a_src_rows = shape->T;
  p.B[0] = (const uint8_t*)W->WgT; p.Bs[0] = (const uint8_t*)W->WgT_s; p.B[1] = (const uint8_t*)W->WuT; p.Bs[1] = (const uint8_t*)W->WuT_s;
  p.ldb = p.lda; p.b_group = F * p.ldb; p.lbs = p.nk; p.bs_group = quant_blocks(F) * p.lbs;
  p.ldc = F;
  p.q[0] = HQ; p.qs[0] = HS; p.ldq = quant_row(F); p.lds = quant_blocks(F);
  typedef Epi8<2, EPI_SWIGLU_FWD> Gated;
  typedef Epi8<1, EPI_GELU_FWD> Plain;
  auto gate_up = [&](auto nb, auto epi) {
    if (exact) launch_small<decltype(nb)::value, decltype(epi), true>("quant_fwd_gate_up", p, st);
    else if (small) launch_small<decltype(nb)::value, decltype(epi)>("quant_fwd_gate_up", p, st);
    else launch_quant<decltype(nb)::value, decltype(epi)>("quant_fwd_gate_up", p, tiles, st);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  if (G) {
    p.out[0] = G; p.out[1] = gated ? U : H; p.out[2] = H;
    if (gated) gate_up(two, QuantOut<Gated, 1, true>());
    else gate_up(one, QuantOut<Plain, 1, true>());
  } else if (gated) {
    gate_up(two, QuantOut<LastOutput<Gated>, 1, false>());
  } else {
    gate_up(one, QuantOut<LastOutput<Plain>, 1, false>());
  }
  QuantGemm q = {};
  q.tiles = pl.tiles; q.n_tiles = pl.n_tiles; q.offsets = offsets; q.n_rows = n_rows; q.n_groups = n_groups;
  q.N = d; q.nk = (int)quant_blocks(F);
  q.A = HQ; q.As = HS; q.lda = quant_row(F); q.las = q.nk;
  q.B[0] = (const uint8_t*)W->WdT; q.Bs[0] = (const uint8_t*)W->WdT_s;
  q.ldb = q.lda; q.b_group = d * q.ldb; q.lbs = q.nk; q.bs_group = quant_blocks(d) * q.lbs;
  q.out[0] = Yout; q.ldc = d;
  if (small) launch_small<1, Epi8<1, EPI_STORE>>("quant_fwd_down", q, st);
  else launch_quant<1, Epi8<1, EPI_STORE>>("quant_fwd_down", q, tiles, st);
  return launch_status(who);
}

extern "C" int moe_quant_expert_bwd(const moe_shape_t* shape, int32_t n_groups, const int32_t* offsets, int32_t n_rows, const int32_t* src_of,
                                    const float* row_w, const void* dYQ, const void* dYS, const void* Xin, const moe_quant_weights_t* W,
                                    const void* G, const void* U, const void* H, const void* dYin, void* dXin, int32_t* active_ids,
                                    int32_t* n_active, void* dWg_c, void* dWu_c, void* dWd_c, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  static const char* who = "moe_quant_expert_bwd";
  const int rc = check_quant_expert(shape, n_groups, offsets, n_rows, src_of, W, true, who);
  if (rc) return rc;
  const bool gated = W->gated != 0;
  if (!ws || !active_ids || !n_active || !dWg_c || (gated && !dWu_c) || !dWd_c || (!src_of != !row_w) ||
      (n_rows > 0 && (!dYQ || !dYS || !Xin || !G || (gated && !U) || !H || !dYin || !dXin)))
    return fail_null(who);
  const void* ptrs[] = {dYQ, Xin, G, U, H, dYin, dXin, dWg_c, dWu_c, dWd_c, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) {
      set_error("%s: every tensor must be 16-byte aligned", who);
      return MOE_EINVAL;
    }
  const QuantSpace sp(shape, n_groups, n_rows, 2);
  if (ws_bytes < sp.bwd()) {
    set_error("%s: workspace of %zu bytes, need %zu", who, ws_bytes, sp.bwd());
    return MOE_EWS;
  }
  hipStream_t st = (hipStream_t)stream;
  const int d = shape->d, F = shape->d_ff, tiles = max_row_tiles(MOE_BF16, n_groups, n_rows, d);
  const Plan pl = carve_plan(ws, n_groups, plan_cap(n_groups, n_rows));
  launch_plan(offsets, n_groups, 256, pl, active_ids, n_active, st);
  if (n_rows == 0) return launch_status(who);
  char* dG = (char*)ws + sp.plan;
  char* dU = dG + sp.act;
  uint8_t *Q = (uint8_t*)dU + sp.act, *S = Q + sp.codes;  // a row of [dG | dU]
  const int mats = gated ? 2 : 1;
  QuantGemm p = {};
  p.tiles = pl.tiles; p.n_tiles = pl.n_tiles; p.offsets = offsets; p.n_rows = n_rows; p.n_groups = n_groups;
  p.N = F; p.nk = (int)quant_blocks(d);
  p.A = (const uint8_t*)dYQ; p.As = (const uint8_t*)dYS; p.lda = quant_row(d); p.las = p.nk;
  p.a_index = src_of; p.a_index_div = shape->k; p.a_src_rows = shape->T; p.c_scale = row_w;
  p.B[0] = (const uint8_t*)W->Wd; p.Bs[0] = (const uint8_t*)W->Wd_s;
  p.ldb = p.lda; p.b_group = F * p.ldb; p.lbs = p.nk; p.bs_group = quant_blocks(F) * p.lbs;
  p.in[0] = G; p.in[1] = U; p.out[0] = dG; p.out[1] = dU; p.ldc = F;
  p.q[0] = Q; p.qs[0] = S; p.q[1] = Q + quant_row(F); p.qs[1] = S + quant_blocks(F);
  p.ldq = mats * quant_row(F); p.lds = mats * quant_blocks(F);
  QuantGemm q = {};
  q.tiles = pl.tiles; q.n_tiles = pl.n_tiles; q.n_rows = n_rows;
  q.N = d; q.nk = mats * (int)quant_blocks(F);
  q.A = Q; q.As = S; q.lda = mats * quant_row(F); q.las = q.nk;
  q.B[0] = (const uint8_t*)W->Wgu; q.Bs[0] = (const uint8_t*)W->Wgu_s;
  q.ldb = q.lda; q.b_group = d * q.ldb; q.lbs = q.nk; q.bs_group = quant_blocks(d) * q.lbs;
  q.out[0] = dXin; q.ldc = d;
  BwdArgs a = {};
  a.d = d; a.F = F; a.n_groups = n_groups; a.n_rows = n_rows; a.offsets = offsets;
  a.Xin = Xin; a.Wu = gated ? W->Wgu : nullptr; a.G = G; a.U = U; a.H = H; a.dYin = dYin;
  a.dWg = dWg_c; a.dWu = dWu_c; a.dWd = dWd_c; a.ws = (char*)ws; a.dG = dG; a.dU = dU;
  typedef QuantOut<Epi8<1, EPI_SWIGLU_BWD>, 2, true> Gated;
  typedef QuantOut<Epi8<1, EPI_GELU_BWD>, 1, true> Plain;
  typedef Epi8<1, EPI_STORE> Store;
  const bool exact = quant_exact(n_rows, F);
  if (exact) {
    if (gated) launch_small<1, Gated, true>("quant_bwd_dh", p, st);
    else launch_small<1, Plain, true>("quant_bwd_dh", p, st);
  }
  if (small_tiles(MOE_BF16, n_groups, n_rows, d, F)) {  // (two of their weight-gradient blocks fit a compute unit: launches of their own)
    if (!exact && gated) launch_quant<1, Gated>("quant_bwd_dh", p, tiles, st);
    if (!exact && !gated) launch_quant<1, Plain>("quant_bwd_dh", p, tiles, st);
    launch_quant<1, Store>("quant_bwd_dx", q, tiles, st);
    expert_dw_impl<PATH_BF16_SMALL>(a, st);
    return launch_status(who);
  }
  typedef Cores<PATH_BF16> C;  // (the weight gradients of sizes with a K tail run on the same cores)
  typedef C::core<1, false, false> W1;
  typedef C::core<2, false, false> W2;
  const DwGemms g = dw_gemms<PATH_BF16>(a);
  // Row tiles of dH over up to eight blocks of K are shorter than the weight gradient's tiles of any group that counts.  (Whole steps with the row tiles first and
  // last, Zipf loads, us: d = 512, 32 experts of 1408 558 and 514, d = 768, 64 of 2816 1308 and 1269, two-matrix ones 982 and 937, even loads 984 and 1002,
  // d = 1000 503 and 492; d = 2048 1427 and 1426, d = 4096 6080 and 6121.  dX last: 0 to 3 % more, but for the two-matrix experts, 982 and 946.)
  const bool w_first = p.nk <= 8;
  const int dh_tiles = exact ? 0 : tiles;  // (computed above)
  if (gated) {
    launch_quant_w<Gated, W1, 1>("quant_bwd_dh_dwd", p, dh_tiles, g.dwd, w_first, st);
    launch_quant_w<Store, W2, 2>("quant_bwd_dx_dwgu", q, tiles, g.dwgu, false, st);
  } else {
    launch_quant_w<Plain, W1, 1>("quant_bwd_dh_dwd", p, dh_tiles, g.dwd, w_first, st);
    launch_quant_w<Store, W1, 1>("quant_bwd_dx_dwgu", q, tiles, g.dwgu, false, st);
  }
  launch_w_light<C::core_light<1>>("gemm_bwd_dw_light", g.dwd_light, g.dwgu_light, gated ? 2 : 1, st);
  return launch_status(who);
}
