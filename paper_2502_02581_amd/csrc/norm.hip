// moe_norm_fwd / moe_norm_bwd: layer norm and RMS norm of token rows, with the addition (and the dropout) of a branch in front of it.
//
//   z = r + drop(x);   layer: m = mean z, v = mean (z - m)^2;   rms: m = 0, v = mean z^2;   s = 1 / sqrt(v + eps);   h = (z - m) s;   y = h w + b
//   g = dy w;   dz = dz_in + s (g - mean g [layer] - h mean(g h));   dr = dz;   dx = drop'(dz);   dw = sum over rows of dy h;   db = sum over rows of dy
//
// Both passes are bound by HBM.  A row stays in the registers of its team (a wavefront, or the wavefronts of a block) from its one load to its one store.
#include "rows.h"

namespace moe {

constexpr int kNormMaxD = 16384;

struct NormFwd {
  const void *X, *R, *w, *b;
  void *Z, *Y;
  float *mean, *rstd;
  int64_t ldx, ldr, ldz, ldy;
  int n_rows, d, layer, wf32;
  float eps;
  Dropout drop;
};
struct NormBwd {
  const void *dY, *Z, *w, *dZ;
  const float *mean, *rstd;
  void *dR, *dX;
  float* partial;  // [blocks][2][d]: sums of dw, db; NULL: not wanted
  int64_t lddy, ldz, lddz, lddr, lddx;
  int n_rows, d, layer, wf32;
  Dropout drop;
};

// eight values of the weights, `fill` where there are none
__device__ __forceinline__ void load_weights(const void* w, int wf32, int col, int valid, float fill, float (&v)[8]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = fill;
  } else if (wf32) {
    Piece<float> p;
    load_piece(p, (const float*)w + col, valid);
    p.values(v);
  } else {
    Piece<bf16_t> p;
    load_piece(p, (const bf16_t*)w + col, valid);
    p.values(v);
  }
}

// The mean's rounding error would be that of every value of the row: delta, the mean of z - m, puts it right, so that rows far from zero (mean 1e4, deviation 1, fp32)
// lose nothing but what their own values have lost.
enum { kPlain = 0, kAdd = 1, kDrop = 2 };

// WIDE: a block is a team; otherwise each of its wavefronts is one.
template <typename T, int V, bool WIDE, int MODE>
__global__ __launch_bounds__(V == 1 ? 1024 : V == 2 ? 512 : 512) void norm_fwd_kernel(NormFwd a) {
  __shared__ RowSums<2> sums;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
  const int team = WIDE ? blockIdx.x : blockIdx.x * n_waves + wave, n_teams = WIDE ? gridDim.x : gridDim.x * n_waves;
  const int first = WIDE ? threadIdx.x : lane, step = WIDE ? blockDim.x : kWave;
  const T *X = (const T*)a.X, *R = (const T*)a.R;
  T *Z = (T*)a.Z, *Y = (T*)a.Y;
  const DropKey key = MODE == kDrop ? drop_key(a.drop) : DropKey{};
  int turn = 0, valid[V];
  float w[V][8], b[V][8];
#pragma unroll
  for (int v = 0; v < V; v++) {
    const int col = 8 * (first + v * step);
    valid[v] = a.d - col;
    load_weights(a.w, a.wf32, col, valid[v], 1.f, w[v]);
    load_weights(a.b, a.wf32, col, valid[v], 0.f, b[v]);
  }
  const float inv_d = 1.f / (float)a.d;
  for (int row = team; row < a.n_rows; row += n_teams) {
    float z[V][8];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int c = first + v * step;
      Piece<T> x, r;
      load_piece(x, X + row * a.ldx + 8 * c, valid[v]);
      if (MODE != kPlain) {
        r.clear();
        if (R) load_piece(r, R + row * a.ldr + 8 * c, valid[v]);
        float add[8];
        x.values(z[v]);
        r.values(add);
        if (MODE == kDrop) {
          drop_piece(a.drop, key, c, row, z[v], add);
        } else {
#pragma unroll
          for (int j = 0; j < 8; j++) z[v][j] += add[j];
        }
        x.set(z[v]);  // the norm is of the values that are kept
        store_piece(x, Z + row * a.ldz + 8 * c, valid[v]);
      }
      x.values(z[v]);
    }
    float m = 0.f, delta = 0.f, var;
    if (a.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; v++)
#pragma unroll
        for (int j = 0; j < 8; j++) s[0] += z[v][j];
      if (WIDE) sums.sum(s, wave, n_waves, turn);
      else s[0] = lanes_sum(s[0]);
      m = s[0] * inv_d;
      float t[2] = {0.f, 0.f};
#pragma unroll
      for (int v = 0; v < V; v++) {
#pragma unroll
        for (int j = 0; j < 8; j++) z[v][j] = j < valid[v] ? z[v][j] - m : 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          t[0] += z[v][j];
          t[1] = fmaf(z[v][j], z[v][j], t[1]);
        }
      }
      if (WIDE) {
        sums.sum(t, wave, n_waves, turn);
      } else {
        t[0] = lanes_sum(t[0]);
        t[1] = lanes_sum(t[1]);
      }
      delta = t[0] * inv_d;
      var = fmaxf(t[1] / (float)a.d - delta * delta, 0.f);
      if (!(t[1] == t[1])) var = t[1];  // (the maximum would lose a NaN)
    } else {
      float t[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; v++)
#pragma unroll
        for (int j = 0; j < 8; j++) t[0] = fmaf(z[v][j], z[v][j], t[0]);
      if (WIDE) sums.sum(t, wave, n_waves, turn);
      else t[0] = lanes_sum(t[0]);
      var = t[0] / (float)a.d;
    }
    const float rstd = 1.f / sqrtf(var + a.eps);
    if (first == 0) {
      if (a.mean) a.mean[row] = m + delta;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int v = 0; v < V; v++) {
      Piece<T> y;
#pragma unroll
      for (int j = 0; j < 8; j++) z[v][j] = fmaf((z[v][j] - delta) * rstd, w[v][j], b[v][j]);
      y.set(z[v]);
      store_piece(y, Y + row * a.ldy + 8 * (first + v * step), valid[v]);
    }
  }
}

template <typename T, int V, bool WIDE, bool DROP>
__global__ __launch_bounds__(V == 1 ? 1024 : 512) void norm_bwd_kernel(NormBwd a) {
  __shared__ RowSums<3> sums;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
  const int team = WIDE ? blockIdx.x : blockIdx.x * n_waves + wave, n_teams = WIDE ? gridDim.x : gridDim.x * n_waves;
  const int first = WIDE ? threadIdx.x : lane, step = WIDE ? blockDim.x : kWave;
  const T *dY = (const T*)a.dY, *Z = (const T*)a.Z, *dZ = (const T*)a.dZ;
  T *dR = (T*)a.dR, *dX = (T*)a.dX;
  const DropKey key = DROP ? drop_key(a.drop) : DropKey{};
  int turn = 0, valid[V];
  float w[V][8], dw[V][8], db[V][8];
#pragma unroll
  for (int v = 0; v < V; v++) {
    const int col = 8 * (first + v * step);
    valid[v] = a.d - col;
    load_weights(a.w, a.wf32, col, valid[v], 1.f, w[v]);
#pragma unroll
    for (int j = 0; j < 8; j++) dw[v][j] = db[v][j] = 0.f;
  }
  const float inv_d = 1.f / (float)a.d;
  for (int row = team; row < a.n_rows; row += n_teams) {
    Piece<T> y[V], z[V], in[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int col = 8 * (first + v * step);
      load_piece(y[v], dY + row * a.lddy + col, valid[v]);
      load_piece(z[v], Z + row * a.ldz + col, valid[v]);
      if (dZ) load_piece(in[v], dZ + row * a.lddz + col, valid[v]);
      else in[v].clear();
    }
    const float m = a.layer ? a.mean[row] : 0.f, rstd = a.rstd[row];
    // sums of g, of g (z - m) and, for the mean's rounding error as in the forward pass, of z - m
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; v++) {
      float dy[8], x[8];
      y[v].values(dy);
      z[v].values(x);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float g = dy[j] * w[v][j], c = x[j] - m;
        s[0] += g;
        s[1] = fmaf(g, c, s[1]);
        s[2] += j < valid[v] ? c : 0.f;
      }
    }
    if (WIDE) {
      sums.sum(s, wave, n_waves, turn);
    } else {
#pragma unroll
      for (int i = 0; i < 3; i++) s[i] = lanes_sum(s[i]);
    }
    const float delta = a.layer ? s[2] * inv_d : 0.f, centre = m + delta;
    const float s1 = a.layer ? s[0] * inv_d : 0.f, s2 = (s[1] - delta * s[0]) * rstd * inv_d;
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int c = first + v * step;
      float dy[8], x[8], o[8];
      y[v].values(dy);
      z[v].values(x);
      in[v].values(o);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float h = ((x[j] - m) - delta) * rstd;
        o[j] = fmaf(rstd, dy[j] * w[v][j] - s1 - h * s2, o[j]);
        dw[v][j] = fmaf(dy[j], h, dw[v][j]);
        db[v][j] += dy[j];
      }
      Piece<T> out;
      if (dR) {
        out.set(o);
        store_piece(out, dR + row * a.lddr + 8 * c, valid[v]);
      }
      if (DROP) {
        const float zero[8] = {};
        drop_piece(a.drop, key, c, row, o, zero);
        out.set(o);
        store_piece(out, dX + row * a.lddx + 8 * c, valid[v]);
      }
    }
    (void)centre;
  }
  if (!a.partial) return;
  if (WIDE) {
    float* p = a.partial + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int col = 8 * (first + v * step);
      Piece<float> o;
      o.set(dw[v]);
      store_piece(o, p + col, valid[v]);
      o.set(db[v]);
      store_piece(o, p + a.d + col, valid[v]);
    }
  } else {  // the wavefronts of the block, one after the other
    __shared__ float all[2][64 * 8 * V];
    for (int q = 0; q < n_waves; q++) {
      if (wave == q) {
#pragma unroll
        for (int v = 0; v < V; v++)
#pragma unroll
          for (int j = 0; j < 8; j++) {
            const int at = (v * 8 + j) * 64 + lane;
            all[0][at] = q ? all[0][at] + dw[v][j] : dw[v][j];
            all[1][at] = q ? all[1][at] + db[v][j] : db[v][j];
          }
      }
      __syncthreads();
    }
    float* p = a.partial + (size_t)blockIdx.x * 2 * a.d;
    for (int col = threadIdx.x; col < a.d; col += blockDim.x) {
      const int c = col >> 3, at = ((c >> 6) * 8 + (col & 7)) * 64 + (c & 63);
      p[col] = all[0][at];
      p[a.d + col] = all[1][at];
    }
  }
}

// dw (blockIdx.y = 0) and db (1) from the blocks' sums: 32 columns x 8 runs, in a fixed order
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* partial, int blocks, int d, int wf32, void* dw, void* db) {
  __shared__ float part[8][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
  void* out = blockIdx.y ? db : dw;
  if (!out) return;
  float s = 0.f;
  if (col < d) {
    const float* p = partial + (size_t)blockIdx.y * d + col;
#pragma unroll 8
    for (int q = run; q < blocks; q += 8) s += p[(size_t)q * 2 * d];
  }
  part[run][threadIdx.x & 31] = s;
  __syncthreads();
  if (run == 0 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < 8; r++) t += part[r][threadIdx.x & 31];
    if (wf32) ((float*)out)[col] = t;
    else Elem<bf16_t>::store((bf16_t*)out + col, t);
  }
}

// pieces of a lane, wavefronts of a row
struct NormPlan {
  int V, waves, blocks;  // waves == 1: four teams in a block
};
static NormPlan norm_plan(const moe_norm_t* n, bool backward) {
  const int pieces = (n->d + 7) / 8;
  NormPlan p;
  if (pieces <= 64) p = {1, 1, 0};
  else if (pieces <= 128) p = {2, 1, 0};
  else if (pieces <= 1024) p = {2, (pieces + 127) / 128, 0};
  else p = {4, (pieces + 255) / 256, 0};
  const int rows = p.waves == 1 ? (n->n_rows + 3) / 4 : n->n_rows;
  const int most = backward ? 512 : 2048;
  p.blocks = rows < most ? rows : most;
  return p;
}

static int check_norm(const moe_norm_t* n, const char* who) {
  if (!n) {
    set_error("%s: norm is NULL", who);
    return MOE_EINVAL;
  }
  if ((n->dtype != MOE_F32 && n->dtype != MOE_BF16) || (n->wdtype != MOE_F32 && n->wdtype != MOE_BF16)) {
    set_error("%s: unknown dtype %d or %d", who, n->dtype, n->wdtype);
    return MOE_EDTYPE;
  }
  if (n->kind != MOE_NORM_LAYER && n->kind != MOE_NORM_RMS) {
    set_error("%s: unknown kind %d", who, n->kind);
    return MOE_EDTYPE;
  }
  if (n->n_rows < 0 || n->d < 1 || n->d > kNormMaxD || !(n->eps >= 0.f) || n->eps > 3.4e38f) {
    set_error("%s: bad sizes: %d rows of %d (1 to %d), eps %g", who, n->n_rows, n->d, kNormMaxD, (double)n->eps);
    return MOE_EINVAL;
  }
  return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_norm_bwd_workspace_bytes(const moe_norm_t* norm) {
  if (check_norm(norm, "moe_norm_bwd_workspace_bytes")) return 0;
  return (size_t)norm_plan(norm, true).blocks * 2 * (size_t)norm->d * sizeof(float) + 256;
}

extern "C" int moe_norm_fwd(const moe_norm_t* norm, const void* X, int64_t ldx, const void* R, int64_t ldr, const moe_drop_t* drop, const void* w,
                            const void* b, void* Z, int64_t ldz, void* Y, int64_t ldy, float* mean, float* rstd, void* stream) {
  const char* who = "moe_norm_fwd";
  int rc = check_norm(norm, who);
  Dropout dr;
  if (!rc) rc = make_dropout(drop, dr, who);
  if (rc) return rc;
  const int n = norm->n_rows, d = norm->d;
  const size_t e = elem_size(norm->dtype), we = elem_size(norm->wdtype);
  const bool sum = R || drop;
  if ((rc = check_rows(who, "X", X, ldx, n, d, e, true)) || (rc = check_rows(who, "R", R, ldr, n, d, e, false)) ||
      (rc = check_rows(who, "Z", Z, ldz, n, d, e, sum)) || (rc = check_rows(who, "Y", Y, ldy, n, d, e, true)) ||
      (rc = check_rows(who, "w", w, d, 1, d, we, false)) || (rc = check_rows(who, "b", b, d, 1, d, we, false)) ||
      (rc = check_rows(who, "mean", mean, 1, 1, 1, 4, false)) || (rc = check_rows(who, "rstd", rstd, 1, 1, 1, 4, false)))
    return rc;
  if (Z && !sum) {
    set_error("%s: Z goes with R or drop; without them it would be X", who);
    return MOE_EINVAL;
  }
  if (mean && norm->kind == MOE_NORM_RMS) {
    set_error("%s: an RMS norm has no mean", who);
    return MOE_EINVAL;
  }
  if (n == 0) return MOE_OK;
  const NormPlan p = norm_plan(norm, false);
  const NormFwd a = {X, R, w, b, Z, Y, mean, rstd, ldx, ldr, ldz, ldy, n, d, norm->kind == MOE_NORM_LAYER, norm->wdtype == MOE_F32, norm->eps, dr};
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid(p.blocks), block(p.waves == 1 ? 256 : 64 * p.waves);
  ProfScope prof("norm_fwd_kernel", st);
#define MOE_NORM_FWD(T, V, WIDE)                                                                           \
  do {                                                                                                     \
    if (!sum) hipLaunchKernelGGL((norm_fwd_kernel<T, V, WIDE, kPlain>), grid, block, 0, st, a);             \
    else if (dr.threshold == 0) hipLaunchKernelGGL((norm_fwd_kernel<T, V, WIDE, kAdd>), grid, block, 0, st, a); \
    else hipLaunchKernelGGL((norm_fwd_kernel<T, V, WIDE, kDrop>), grid, block, 0, st, a);                   \
  } while (0)
#define MOE_NORM_BY_PLAN(CALL, T)                                   \
  do {                                                              \
    if (p.waves == 1 && p.V == 1) CALL(T, 1, false);                \
    else if (p.waves == 1) CALL(T, 2, false);                       \
    else if (p.V == 2) CALL(T, 2, true);                            \
    else CALL(T, 4, true);                                          \
  } while (0)
  if (norm->dtype == MOE_F32) MOE_NORM_BY_PLAN(MOE_NORM_FWD, float);
  else MOE_NORM_BY_PLAN(MOE_NORM_FWD, bf16_t);
#undef MOE_NORM_FWD
  return launch_status(who);
}

extern "C" int moe_norm_bwd(const moe_norm_t* norm, const void* dY, int64_t lddy, const void* Z, int64_t ldz, const void* w, const float* mean,
                            const float* rstd, const void* dZ, int64_t lddz, const moe_drop_t* drop, void* dR, int64_t lddr, void* dX, int64_t lddx,
                            void* dw, void* db, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "moe_norm_bwd";
  int rc = check_norm(norm, who);
  Dropout dr;
  if (!rc) rc = make_dropout(drop, dr, who);
  if (rc) return rc;
  const int n = norm->n_rows, d = norm->d;
  const size_t e = elem_size(norm->dtype), we = elem_size(norm->wdtype);
  if ((rc = check_rows(who, "dY", dY, lddy, n, d, e, true)) || (rc = check_rows(who, "Z", Z, ldz, n, d, e, true)) ||
      (rc = check_rows(who, "dZ", dZ, lddz, n, d, e, false)) || (rc = check_rows(who, "dR", dR, lddr, n, d, e, !dX)) ||
      (rc = check_rows(who, "dX", dX, lddx, n, d, e, drop != nullptr)) || (rc = check_rows(who, "w", w, d, 1, d, we, false)) ||
      (rc = check_rows(who, "dw", dw, d, 1, d, we, false)) || (rc = check_rows(who, "db", db, d, 1, d, we, false)) ||
      (rc = check_rows(who, "mean", mean, 1, n, 1, 4, norm->kind == MOE_NORM_LAYER)) || (rc = check_rows(who, "rstd", rstd, 1, n, 1, 4, true)))
    return rc;
  if (dX && !drop) {
    set_error("%s: dX goes with drop; without it the gradient of the branch is dR", who);
    return MOE_EINVAL;
  }
  const bool weights = dw || db;
  const NormPlan p = norm_plan(norm, true);
  if (weights) {
    const size_t need = moe_norm_bwd_workspace_bytes(norm);
    if (!ws || !aligned16(ws)) {
      set_error("%s: null pointer or workspace not 16-byte aligned", who);
      return MOE_EINVAL;
    }
    if (ws_bytes < need) {
      set_error("%s: workspace of %zu bytes, need %zu", who, ws_bytes, need);
      return MOE_EWS;
    }
  }
  hipStream_t st = (hipStream_t)stream;
  if (n > 0) {
    const NormBwd a = {dY, Z, w, dZ, mean, rstd, dR, dX, weights ? (float*)ws : nullptr, lddy, ldz, lddz, lddr, lddx, n, d,
                       norm->kind == MOE_NORM_LAYER, norm->wdtype == MOE_F32, dr};
    const dim3 grid(p.blocks), block(p.waves == 1 ? 256 : 64 * p.waves);
    ProfScope prof("norm_bwd_kernel", st);
#define MOE_NORM_BWD(T, V, WIDE)                                                                          \
  do {                                                                                                    \
    if (drop) hipLaunchKernelGGL((norm_bwd_kernel<T, V, WIDE, true>), grid, block, 0, st, a);              \
    else hipLaunchKernelGGL((norm_bwd_kernel<T, V, WIDE, false>), grid, block, 0, st, a);                  \
  } while (0)
    if (norm->dtype == MOE_F32) MOE_NORM_BY_PLAN(MOE_NORM_BWD, float);
    else MOE_NORM_BY_PLAN(MOE_NORM_BWD, bf16_t);
#undef MOE_NORM_BWD
  }
  if (weights) {
    ProfScope prof("norm_weights_kernel", st);
    hipLaunchKernelGGL(norm_weights_kernel, dim3((d + 31) / 32, 2), dim3(256), 0, st, (const float*)ws, n > 0 ? p.blocks : 0, d, (int)(norm->wdtype == MOE_F32),
                       dw, db);
  }
  return n > 0 || weights ? launch_status(who) : MOE_OK;
}
