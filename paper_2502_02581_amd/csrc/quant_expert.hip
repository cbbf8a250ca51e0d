// moe_quant_gemm, moe_quant_expert_fwd / _bwd: grouped products of block-scaled 8-bit tensors.
#include "expert_impl.h"
#include "quant_core.h"

namespace moe {

// ------------------------------------------------------------------------------------------ kernel
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

template <class Core, class Epi, int NB>
__device__ __forceinline__ void quant_tile(const QuantGemm& p, const RowTile& t, int nt, char* smem) {
  const int rows = tile_rows(t), n0 = nt * Core::BN;
  QuantTile q;
  q.map = {p.a_index, p.a_index ? p.a_index_div : 1, t.row0_in, rows};
  const int64_t row0 = p.a_index ? 0 : t.row0_in;
  const uint32_t last = (uint32_t)((p.a_index ? p.a_src_rows : rows) - 1);
  q.a = p.A + row0 * p.lda;
  q.as = p.As + row0 * p.las;
  q.a_bytes = last * (uint32_t)p.lda + (uint32_t)p.nk * kQuantBlock;
  q.as_bytes = last * (uint32_t)p.las + (uint32_t)p.nk;
#pragma unroll
  for (int x = 0; x < NB; x++) {
    q.b[x] = p.B[x] + t.group * p.b_group + n0 * p.ldb;
    q.bs[x] = p.Bs[x] + t.group * p.bs_group + n0 / kQuantBlock * p.lbs;
  }
  q.n_valid = min(Core::BN, p.N - n0);
  Epi epi;
  const int64_t c_off = ((int64_t)t.row0_out * p.ldc + n0) * Epi::OES;
#pragma unroll
  for (int x = 0; x < Epi::NOUT; x++) epi.out[x] = (char*)p.out[x] + c_off;
#pragma unroll
  for (int x = 0; x < Epi::NAUX; x++) epi.in[x] = (const char*)p.in[x] + c_off;
  epi.ldc = p.ldc;
  epi.rows = rows;
  epi.n_valid = q.n_valid;
  epi.scale = p.c_scale;
  epi.index = p.a_index + t.row0_in;
  set_quantised(epi, p, t.row0_out, n0);
  Core::run(smem, p.nk, q, p.lda, p.las, p.ldb, epi);
}

// Heights of the tiles: 256, and for what is left of a group 128 and 64 (tiles of up to 64 rows are bound by streaming the matrix, whatever
// their height).
template <int NB> using QuantTall = QuantCore<256, NB, 2>;
template <int NB> using QuantMid = QuantCore<128, NB, 3>;
template <int NB> using QuantShort = QuantCore<64, NB, 3>;

// Tiles are dealt to the XCDs as in row_gemm_block: band by band of kBandRows row tiles, column by column within a band, runs of 32 (launches of
// few rounds: of 8) consecutive tiles to an XCD.
template <int NB, class Epi>
__global__ __launch_bounds__(256, 1) void quant_gemm_kernel(QuantGemm p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int BN = 256 / NB;
  const int ntn = (p.N + BN - 1) / BN;
  const int n_mt = p.tiles ? *p.n_tiles : (p.n_rows + 255) / 256;
  const int total = n_mt * ntn, rounds = total >> 8, per_band = kBandRows * ntn;
  const int xcd = blockIdx.x & 7, round = blockIdx.x >> 8, b = (blockIdx.x >> 3) & 31;
  int q = round << 8;
  if (round < rounds) q += rounds > kFineRounds && round < rounds - 1 ? (xcd << 5) + b : ((b >> 3) << 6) + (xcd << 3) + (b & 7);
  else q += (b << 3) + xcd;
  if (q >= total) return;
  const int band = q / per_band, r = q - band * per_band, high = min(kBandRows, n_mt - band * kBandRows);
  const int mt = band * kBandRows + r % high, nt = r / high;
  RowTile t;
  if (p.tiles) t = p.tiles[mt];
  else { t.group = 0; t.row0_in = t.row0_out = mt * 256; t.rows = min(256, p.n_rows - t.row0_in); }
  t.group = __builtin_amdgcn_readfirstlane(t.group);
  t.row0_in = __builtin_amdgcn_readfirstlane(t.row0_in);
  t.rows = __builtin_amdgcn_readfirstlane(t.rows);
  t.row0_out = __builtin_amdgcn_readfirstlane(t.row0_out);
  if (tile_rows(t) > 128) quant_tile<QuantTall<NB>, Epi, NB>(p, t, nt, smem);
  else if (tile_rows(t) > 64) quant_tile<QuantMid<NB>, Epi, NB>(p, t, nt, smem);
  else quant_tile<QuantShort<NB>, Epi, NB>(p, t, nt, smem);
}

// At most max_tiles row tiles (the device knows how many there are).
template <int NB, class Epi>
static void launch_quant(const char* label, const QuantGemm& p, int max_tiles, hipStream_t st) {
  const unsigned blocks = row_block_count(max_tiles, p.N, 256 / NB);
  if (blocks == 0) return;
  constexpr int kLds = std::max({QuantTall<NB>::LDS_BYTES, QuantMid<NB>::LDS_BYTES, QuantShort<NB>::LDS_BYTES});
  launch_gemm<quant_gemm_kernel<NB, Epi>>(label, blocks, 256, kLds, st, p);
}
template <int NB, int EPI> using Epi8 = Epilogue<bf16_t, NB, EPI>;

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
  return quant_plan_size(n_groups, n_rows);
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
  int tiles = ceil_div(n_rows, 256);
  if (offsets) {
    const Plan pl = carve_plan(ws, n_groups, plan_cap(n_groups, n_rows));
    launch_plan(offsets, n_groups, 256, pl, nullptr, nullptr, st);
    p.tiles = pl.tiles; p.n_tiles = pl.n_tiles;
    tiles = quant_tiles(n_groups, n_rows);
  }
  p.n_rows = n_rows; p.N = N; p.nk = (int)quant_blocks(K);
  p.A = (const uint8_t*)A; p.As = (const uint8_t*)As; p.lda = quant_row(K); p.las = p.nk;
  p.B[0] = (const uint8_t*)B; p.Bs[0] = (const uint8_t*)Bs; p.ldb = p.lda; p.b_group = N * p.ldb; p.lbs = p.nk; p.bs_group = quant_blocks(N) * p.lbs;
  p.out[0] = C; p.ldc = N;
  launch_quant<1, Epi8<1, EPI_STORE>>("quant_gemm", p, tiles, st);
  return launch_status("moe_quant_gemm");
}

// ---------------------------------------------------------------------------------------- experts
namespace moe {

extern template void expert_dw_impl<PATH_BF16>(const BwdArgs&, hipStream_t);
extern template void expert_dw_impl<PATH_BF16_TAIL>(const BwdArgs&, hipStream_t);
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
  // (256 rows of [dG | dU] codes, and of bf16 outputs, within 32-bit byte offsets)
  if (512 * quant_row(std::max(s->d, s->d_ff)) >= ((int64_t)1 << 32) - 4096) {
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
  if (!shape || n_groups < 1 || n_rows < 0 || shape->d_ff < 1) return 0;
  return QuantSpace(shape, n_groups, n_rows, 1).fwd();
}
extern "C" size_t moe_quant_expert_bwd_workspace_bytes(const moe_shape_t* shape, int32_t n_groups, int32_t n_rows) {
  using namespace moe;
  if (!shape || n_groups < 1 || n_rows < 0 || shape->d_ff < 1) return 0;
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
  const Plan pl = carve_plan(plan ? (void*)plan : ws, n_groups, plan_cap(n_groups, n_rows));
  if (!plan) launch_plan(offsets, n_groups, 256, pl, nullptr, nullptr, st);
  uint8_t *HQ = (uint8_t*)ws + sp.plan, *HS = HQ + sp.codes;
  QuantGemm p = {};
  p.tiles = pl.tiles; p.n_tiles = pl.n_tiles; p.n_rows = n_rows;
  p.N = F; p.nk = (int)quant_blocks(d);
  p.A = (const uint8_t*)XQ; p.As = (const uint8_t*)XS; p.lda = quant_row(d); p.las = p.nk;
  p.a_index = src_of; p.a_index_div = shape->k; p.a_src_rows = shape->T;
  p.B[0] = (const uint8_t*)W->WgT; p.Bs[0] = (const uint8_t*)W->WgT_s; p.B[1] = (const uint8_t*)W->WuT; p.Bs[1] = (const uint8_t*)W->WuT_s;
  p.ldb = p.lda; p.b_group = F * p.ldb; p.lbs = p.nk; p.bs_group = quant_blocks(F) * p.lbs;
  p.ldc = F;
  p.q[0] = HQ; p.qs[0] = HS; p.ldq = quant_row(F); p.lds = quant_blocks(F);
  typedef Epi8<2, EPI_SWIGLU_FWD> Gated;
  typedef Epi8<1, EPI_GELU_FWD> Plain;
  if (G) {
    p.out[0] = G; p.out[1] = gated ? U : H; p.out[2] = H;
    if (gated) launch_quant<2, QuantOut<Gated, 1, true>>("quant_fwd_gate_up", p, tiles, st);
    else launch_quant<1, QuantOut<Plain, 1, true>>("quant_fwd_gate_up", p, tiles, st);
  } else if (gated) {
    launch_quant<2, QuantOut<LastOutput<Gated>, 1, false>>("quant_fwd_gate_up", p, tiles, st);
  } else {
    launch_quant<1, QuantOut<LastOutput<Plain>, 1, false>>("quant_fwd_gate_up", p, tiles, st);
  }
  QuantGemm q = {};
  q.tiles = pl.tiles; q.n_tiles = pl.n_tiles; q.n_rows = n_rows;
  q.N = d; q.nk = (int)quant_blocks(F);
  q.A = HQ; q.As = HS; q.lda = quant_row(F); q.las = q.nk;
  q.B[0] = (const uint8_t*)W->WdT; q.Bs[0] = (const uint8_t*)W->WdT_s;
  q.ldb = q.lda; q.b_group = d * q.ldb; q.lbs = q.nk; q.bs_group = quant_blocks(d) * q.lbs;
  q.out[0] = Yout; q.ldc = d;
  launch_quant<1, Epi8<1, EPI_STORE>>("quant_fwd_down", q, tiles, st);
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
  p.tiles = pl.tiles; p.n_tiles = pl.n_tiles; p.n_rows = n_rows;
  p.N = F; p.nk = (int)quant_blocks(d);
  p.A = (const uint8_t*)dYQ; p.As = (const uint8_t*)dYS; p.lda = quant_row(d); p.las = p.nk;
  p.a_index = src_of; p.a_index_div = shape->k; p.a_src_rows = shape->T; p.c_scale = row_w;
  p.B[0] = (const uint8_t*)W->Wd; p.Bs[0] = (const uint8_t*)W->Wd_s;
  p.ldb = p.lda; p.b_group = F * p.ldb; p.lbs = p.nk; p.bs_group = quant_blocks(F) * p.lbs;
  p.in[0] = G; p.in[1] = U; p.out[0] = dG; p.out[1] = dU; p.ldc = F;
  p.q[0] = Q; p.qs[0] = S; p.q[1] = Q + quant_row(F); p.qs[1] = S + quant_blocks(F);
  p.ldq = mats * quant_row(F); p.lds = mats * quant_blocks(F);
  if (gated) launch_quant<1, QuantOut<Epi8<1, EPI_SWIGLU_BWD>, 2, true>>("quant_bwd_dh", p, tiles, st);
  else launch_quant<1, QuantOut<Epi8<1, EPI_GELU_BWD>, 1, true>>("quant_bwd_dh", p, tiles, st);
  QuantGemm q = {};
  q.tiles = pl.tiles; q.n_tiles = pl.n_tiles; q.n_rows = n_rows;
  q.N = d; q.nk = mats * (int)quant_blocks(F);
  q.A = Q; q.As = S; q.lda = mats * quant_row(F); q.las = q.nk;
  q.B[0] = (const uint8_t*)W->Wgu; q.Bs[0] = (const uint8_t*)W->Wgu_s;
  q.ldb = q.lda; q.b_group = d * q.ldb; q.lbs = q.nk; q.bs_group = quant_blocks(d) * q.lbs;
  q.out[0] = dXin; q.ldc = d;
  launch_quant<1, Epi8<1, EPI_STORE>>("quant_bwd_dx", q, tiles, st);
  BwdArgs a = {};
  a.d = d; a.F = F; a.n_groups = n_groups; a.n_rows = n_rows; a.offsets = offsets;
  a.Xin = Xin; a.Wu = gated ? W->Wgu : nullptr; a.G = G; a.U = U; a.H = H; a.dYin = dYin;
  a.dWg = dWg_c; a.dWu = dWu_c; a.dWd = dWd_c; a.ws = (char*)ws; a.dG = dG; a.dU = dU;
  if (small_tiles(MOE_BF16, n_groups, n_rows, d, F)) expert_dw_impl<PATH_BF16_SMALL>(a, st);
  else if (d % 64 == 0 && F % 64 == 0) expert_dw_impl<PATH_BF16>(a, st);
  else expert_dw_impl<PATH_BF16_TAIL>(a, st);
  return launch_status(who);
}
