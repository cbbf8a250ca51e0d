// moe_norm_fwd / moe_norm_bwd: layer norm and RMS norm of token rows, with the addition (and the dropout) of a branch in front of it.
//
//   z = r + drop(x);   layer: m = mean z, v = mean (z - m)^2;   rms: m = 0, v = mean z^2;   s = 1 / sqrt(v + eps);   h = (z - m) s;   y = h w + b
//   g = dy w;   dz = dz_in + s (g - mean g [layer] - h mean(g h));   dr = dz;   dx = drop'(dz);   dw = sum over rows of dy h;   db = sum over rows of dy
//
// Both passes are bound by HBM.  A row stays in the registers of its team (16 or 32 lanes, a wavefront, or the wavefronts of a block) from its one load to its one store; but in
// the backward pass rows of more than 8192 values are read twice, and so are those beside which blocks of columns add up the weights' gradients.
#include "norm_plan.h"
#include "rows.h"

namespace moe {

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
  float* partial;  // [blocks][2][d]: sums of dw, db; NULL: not wanted, or
  void *dw, *db;   // written by the blocks behind the first row_blocks
  int64_t lddy, ldz, lddz, lddr, lddx;
  int n_rows, d, layer, wf32, row_blocks;
  Dropout drop;
};

// eight values of the weights, `fill` where there are none
__device__ __forceinline__ void load_weights(const void* w, int wf32, int col, int valid, float fill, float (&v)[8]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = fill;
  } else if (wf32) {
    Piece<float> p;
    load_piece<kByValue>(p, (const float*)w + col, valid, 0);
    p.values(v);
  } else {
    Piece<bf16_t> p;
    const int back = piece_back<kTinyTail>(col, valid);
    load_piece<kTinyTail>(p, (const bf16_t*)w + col, valid, back);
    settle<kTinyTail>(p, back);
    p.values(v);
  }
}

// z = x, r + x, r + drop(x); kPass: z = x, and no statistics are kept, so no backward pass will read x again (with kPlain it will: no streaming hint on its loads, or
// the backward pass of 1000 x 4096 right behind takes 15.7 us for 13.0)
enum { kPlain = 0, kAdd = 1, kDrop = 2, kPass = 3 };

// over the lanes of a team that is no block (whose lanes are active alike)
template <int TEAM>
__device__ __forceinline__ float team_sum(float x) {
  return TEAM == kLanes16Team ? row16_sum(x) : TEAM == kLanes32Team ? add_rows16(row16_sum(x)) : lanes_sum(x);
}

// Rows far from zero: the rounding error of the mean would be that of every value of the row.  delta, the mean of z - m, puts it right, so that they lose nothing but
// what their own values have lost (mean 1e4, deviation 1, fp32).  Where the mean is below the deviation its error is below the deviation's, and delta would bring in the
// roundings of z - m, which have one sign for all z of a binade; there it is left out.
template <typename T, int TAIL, int V, int TEAM, int MODE>
__global__ __launch_bounds__(!wide_team(TEAM) ? 256 : TEAM == kBlockTeam && V == 2 ? 512 : 1024) void norm_fwd_kernel(NormFwd a) {
  constexpr bool WIDE = wide_team(TEAM), ADD = MODE == kAdd || MODE == kDrop;
  constexpr int LANES = lanes_of(TEAM);
  __shared__ RowSums<2> sums;
  const int wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6, block_teams = WIDE ? 1 : blockDim.x / LANES;
  const int team = WIDE ? blockIdx.x : blockIdx.x * block_teams + threadIdx.x / LANES, n_teams = gridDim.x * block_teams;
  const int first = WIDE ? threadIdx.x : threadIdx.x % LANES, step = WIDE ? blockDim.x : LANES;
  const T *X = (const T*)a.X, *R = (const T*)a.R;
  T *Z = (T*)a.Z, *Y = (T*)a.Y;
  const DropKey key = MODE == kDrop ? drop_key(a.drop) : DropKey{};
  int turn = 0, valid[V], back[V];
  float w[V][8], b[V][8];
#pragma unroll
  for (int v = 0; v < V; v++) {
    const int col = 8 * (first + v * step);
    valid[v] = a.d - col;
    back[v] = piece_back<TAIL>(col, valid[v]);
    load_weights(a.w, a.wf32, col, valid[v], 1.f, w[v]);
    load_weights(a.b, a.wf32, col, valid[v], 0.f, b[v]);
  }
  const float inv_d = 1.f / (float)a.d;
  Piece<T> x[V], r[V];  // the next row: its loads are under way while the one before is worked on
  auto load = [&](int row) {
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int col = 8 * (first + v * step);
      load_piece<TAIL, MODE != kPlain>(x[v], X + row * a.ldx + col, valid[v], back[v]);
      if (ADD) {
        r[v].clear();
        if (R) load_piece<TAIL, true>(r[v], R + row * a.ldr + col, valid[v], back[v]);
      }
    }
  };
  if (TEAM != kLongTeam && team < a.n_rows) load(team);
  for (int row = team; row < a.n_rows; row += n_teams) {
    if (TEAM == kLongTeam) load(row);
    float z[V][8];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int c = first + v * step;
      settle<TAIL>(x[v], back[v]);
      x[v].values(z[v]);
      if (ADD) {
        float add[8];
        settle<TAIL>(r[v], back[v]);
        r[v].values(add);
        if (MODE == kDrop) {
          drop_piece(a.drop, key, c, row, z[v], add);
        } else {
#pragma unroll
          for (int j = 0; j < 8; j++) z[v][j] += add[j];
        }
        x[v].set(z[v]);  // the norm is of the values that are kept
        store_piece<TAIL>(x[v], Z + row * a.ldz + 8 * c, valid[v]);
        x[v].values(z[v]);
      }
    }
    if (TEAM != kLongTeam && row + n_teams < a.n_rows) load(row + n_teams);
    float m = 0.f, delta = 0.f, var;
    if (a.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; v++)
#pragma unroll
        for (int j = 0; j < 8; j++) s[0] += z[v][j];
      if (WIDE) sums.sum(s, wave, n_waves, turn);
      else s[0] = team_sum<TEAM>(s[0]);
      m = s[0] * inv_d;
      // Once, but for rows whose squares are the mean's error for the most part (constant ones of 1e9: 3600 for 0), where delta takes nearly all of them away and leaves its
      // rounding: again around the better mean, whose error is 2^-18 of that at most.  (The lanes of a team go round alike, their sums have the same bits.)
      float step = m;
#pragma unroll 1
      for (int round = 0;; round++) {
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; v++) {
#pragma unroll
          for (int j = 0; j < 8; j++) z[v][j] = j < valid[v] ? z[v][j] - step : 0.f;
#pragma unroll
          for (int j = 0; j < 8; j++) {
            t[0] += z[v][j];
            t[1] = fmaf(z[v][j], z[v][j], t[1]);
          }
        }
        if (WIDE) {
          sums.sum(t, wave, n_waves, turn);
        } else {
          t[0] = team_sum<TEAM>(t[0]);
          t[1] = team_sum<TEAM>(t[1]);
        }
        var = t[1] / (float)a.d;
        if (!(m * m > var)) break;
        step = t[0] * inv_d;
        const float left = var - step * step;
        if (left >= 0.5f * var || round == 2) {
          delta = step;
          var = left < 0.f ? 0.f : left;
          break;
        }
        m += step;
      }
    } else {
      float t[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; v++)
#pragma unroll
        for (int j = 0; j < 8; j++) t[0] = fmaf(z[v][j], z[v][j], t[0]);
      if (WIDE) sums.sum(t, wave, n_waves, turn);
      else t[0] = team_sum<TEAM>(t[0]);
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
      store_piece<TAIL>(y, Y + row * a.ldy + 8 * (first + v * step), valid[v]);
    }
  }
}

// dw and db of 128 bytes' worth of columns, over all rows: for calls of few rows, where reading these again costs less than another launch.  P lanes side by side hold a row's pieces,
// as many rows at once as the block has P lanes.  The mean's rounding error, 2^-24 of it, is less than 8 of the deviation's where the mean is below 8 deviations; other rows'
// lanes look at the whole row for it.
template <typename T, int TAIL>
__device__ __forceinline__ void norm_columns(const NormBwd& a, int block) {
  constexpr int P = sizeof(T) == 2 ? 8 : 4, U = 4;
  __shared__ float part[16][2][8 * P];
  const T *dY = (const T*)a.dY, *Z = (const T*)a.Z;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
  const int p = threadIdx.x & (P - 1), col = 8 * (block * P + p), valid = a.d - col, back = piece_back<TAIL>(col, valid), runs = blockDim.x / P;
  float dw[8], db[8];
#pragma unroll
  for (int j = 0; j < 8; j++) dw[j] = db[j] = 0.f;
  for (int row0 = threadIdx.x / P; row0 < a.n_rows; row0 += U * runs) {
    Piece<T> y[U], z[U];
    float m[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int row = row0 + u * runs;
      const bool there = row < a.n_rows;
      load_piece<TAIL>(y[u], dY + row * a.lddy + col, there ? valid : 0, there ? back : 0);
      load_piece<TAIL>(z[u], Z + row * a.ldz + col, there ? valid : 0, there ? back : 0);
      m[u] = there && a.layer ? a.mean[row] : 0.f;
      rstd[u] = there ? a.rstd[row] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int row = row0 + u * runs;
      if (row >= a.n_rows) break;
      float delta = 0.f;
      if (fabsf(m[u]) * rstd[u] > 8.f) {
        float s = 0.f;
        for (int c = p; 8 * c < a.d; c += P) {
          Piece<T> x;
          float v[8];
          const int short_of = piece_back<TAIL>(8 * c, a.d - 8 * c);
          load_piece<TAIL>(x, Z + row * a.ldz + 8 * c, a.d - 8 * c, short_of);
          settle<TAIL>(x, short_of);
          x.values(v);
#pragma unroll
          for (int j = 0; j < 8; j++) s += 8 * c + j < a.d ? v[j] - m[u] : 0.f;
        }
        s = add_lanes2(add_lanes1(s));
        if (P == 8) s = add_lanes4(s);
        delta = s / (float)a.d;
      }
      float dy[8], x[8];
      settle<TAIL>(y[u], back);
      settle<TAIL>(z[u], back);
      y[u].values(dy);
      z[u].values(x);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        dw[j] = fmaf(dy[j], ((x[j] - m[u]) - delta) * rstd[u], dw[j]);
        db[j] += dy[j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; j++) {
    if (P == 4) {
      dw[j] = add_quads(dw[j]);
      db[j] = add_quads(db[j]);
    } else {
      dw[j] += dpp<0x128>(dw[j]);  // a rotation of sixteen by eight
      db[j] += dpp<0x128>(db[j]);
    }
    dw[j] = add_rows32(add_rows16(dw[j]));
    db[j] = add_rows32(add_rows16(db[j]));
    if (lane < P) {
      part[wave][0][8 * p + j] = dw[j];
      part[wave][1][8 * p + j] = db[j];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * 8 * P; i += blockDim.x) {
    const int which = i / (8 * P), c = i % (8 * P), at = 8 * block * P + c;
    void* out = which ? a.db : a.dw;
    if (!out || at >= a.d) continue;
    float t = 0.f;
    for (int w = 0; w < n_waves; w++) t += part[w][which][c];
    if (a.wf32) ((float*)out)[at] = t;
    else Elem<bf16_t>::store((bf16_t*)out + at, t);
  }
}

// ONCE: streaming hints on the loads of rows.  With a dZ the rows are a residual stream's, four arrays of them, and the hints make the pass quicker (8192 x 4096: 60 us for
// 61.5); without one they make the forward pass behind it slower by more (8192 x 4096: 37.7 us for 28.5, both passes 82 for 73; 8192 x 7168 both 138 for 136).  Blocks of
// columns read the rows beside those of rows: no hints there.
template <typename T, int TAIL, int V, int TEAM, bool DROP, bool ONCE>
__global__ __launch_bounds__(!wide_team(TEAM) || (TEAM == kBlockTeam && V == 2) ? 512 : 1024) void norm_bwd_kernel(NormBwd a) {
  constexpr bool WIDE = wide_team(TEAM);
  constexpr int LANES = lanes_of(TEAM);
  if ((!WIDE || V == 1) && (int)blockIdx.x >= a.row_blocks) return norm_columns<T, TAIL>(a, blockIdx.x - a.row_blocks);
  __shared__ RowSums<3> sums;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6, block_teams = WIDE ? 1 : blockDim.x / LANES;
  const int team = WIDE ? blockIdx.x : blockIdx.x * block_teams + threadIdx.x / LANES, n_teams = a.row_blocks * block_teams;
  const int first = WIDE ? threadIdx.x : threadIdx.x % LANES, step = WIDE ? blockDim.x : LANES;
  const T *dY = (const T*)a.dY, *Z = (const T*)a.Z, *dZ = (const T*)a.dZ;
  T *dR = (T*)a.dR, *dX = (T*)a.dX;
  const DropKey key = DROP ? drop_key(a.drop) : DropKey{};
  int turn = 0, valid[V], back[V];
  float w[V][8], dw[V][8], db[V][8];
#pragma unroll
  for (int v = 0; v < V; v++) {
    const int col = 8 * (first + v * step);
    valid[v] = a.d - col;
    back[v] = piece_back<TAIL>(col, valid[v]);
    load_weights(a.w, a.wf32, col, valid[v], 1.f, w[v]);
#pragma unroll
    for (int j = 0; j < 8; j++) dw[v][j] = db[v][j] = 0.f;
  }
  const float inv_d = 1.f / (float)a.d;
  struct Loads {
    Piece<T> y, z, in;
  };
  auto load = [&](Loads& p, int row, int v, bool all) {
    const int col = 8 * (first + v * step);
    load_piece<TAIL, ONCE>(p.y, dY + row * a.lddy + col, valid[v], back[v]);
    load_piece<TAIL, ONCE>(p.z, Z + row * a.ldz + col, valid[v], back[v]);
    if (all && dZ) load_piece<TAIL, ONCE>(p.in, dZ + row * a.lddz + col, valid[v], back[v]);
    else p.in.clear();
  };
  auto settle_loads = [&](Loads& p, int v) {
    settle<TAIL>(p.y, back[v]);
    settle<TAIL>(p.z, back[v]);
    settle<TAIL>(p.in, back[v]);
  };
  float s[3];  // sums of g, of g (z - m) and, for the mean's rounding error as in the forward pass, of z - m
  float m = 0.f, rstd = 0.f;
  auto add = [&](const Loads& p, int v) {
    float dy[8], x[8];
    p.y.values(dy);
    p.z.values(x);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float g = dy[j] * w[v][j], c = x[j] - m;
      s[0] += g;
      s[1] = fmaf(g, c, s[1]);
      s[2] += j < valid[v] ? c : 0.f;
    }
  };
  float delta, s1, s2;
  auto finish = [&](const Loads& p, int row, int v) {
    const int c = first + v * step;
    float dy[8], x[8], o[8];
    p.y.values(dy);
    p.z.values(x);
    p.in.values(o);
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
      store_piece<TAIL>(out, dR + row * a.lddr + 8 * c, valid[v]);
    }
    if (DROP) {
      const float zero[8] = {};
      drop_piece(a.drop, key, c, row, o, zero);
      out.set(o);
      store_piece<TAIL>(out, dX + row * a.lddx + 8 * c, valid[v]);
    }
  };
  Loads next[V];  // the next row: its loads are under way while the one before is worked on
  float next_m = 0.f, next_rstd = 0.f;
  auto load_row = [&](int row) {
    if (TEAM != kLongTeam) {
#pragma unroll
      for (int v = 0; v < V; v++) load(next[v], row, v, true);
    }
    next_m = a.layer ? a.mean[row] : 0.f;
    next_rstd = a.rstd[row];
  };
  if (team < a.n_rows) load_row(team);
  for (int row = team; row < a.n_rows; row += n_teams) {
    Loads now[V];
    m = next_m;
    rstd = next_rstd;
    if (TEAM != kLongTeam) {
#pragma unroll
      for (int v = 0; v < V; v++) {
        now[v] = next[v];
        settle_loads(now[v], v);
      }
    }
    if (row + n_teams < a.n_rows) load_row(row + n_teams);
    s[0] = s[1] = s[2] = 0.f;
#pragma unroll
    for (int v = 0; v < V; v++) {
      if (TEAM == kLongTeam) {
        Loads p;
        load(p, row, v, false);
        settle_loads(p, v);
        add(p, v);
      } else {
        add(now[v], v);
      }
    }
    if (WIDE) {
      sums.sum(s, wave, n_waves, turn);
    } else {
#pragma unroll
      for (int i = 0; i < 3; i++) s[i] = team_sum<TEAM>(s[i]);
    }
    delta = fabsf(m) * rstd > 1.f ? s[2] * inv_d : 0.f;  // (no mean, no delta)
    s1 = a.layer ? s[0] * inv_d : 0.f;
    s2 = (s[1] - delta * s[0]) * rstd * inv_d;
#pragma unroll
    for (int v = 0; v < V; v++) {
      if (TEAM == kLongTeam) {
        Loads p;
        load(p, row, v, true);
        settle_loads(p, v);
        finish(p, row, v);
      } else {
        finish(now[v], row, v);
      }
    }
  }
  if (!a.partial) return;
  auto store_sums = [&] {
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
  };
  if (WIDE) {
    store_sums();
  } else {  // the teams of a wavefront, then the upper half of the wavefronts to the lower half, until one is left
    if (LANES < 64) {
#pragma unroll
      for (int v = 0; v < V; v++)
#pragma unroll
        for (int j = 0; j < 8; j++) {
          dw[v][j] = add_rows32(LANES == 16 ? add_rows16(dw[v][j]) : dw[v][j]);
          db[v][j] = add_rows32(LANES == 16 ? add_rows16(db[v][j]) : db[v][j]);
        }
    }
    __shared__ float4 all[4][V * 4][64];
    for (int half = n_waves / 2; half > 0; half /= 2) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int v = 0; v < V; v++)
#pragma unroll
          for (int j = 0; j < 8; j += 4) {
            all[wave - half][4 * v + j / 4][lane] = make_float4(dw[v][j], dw[v][j + 1], dw[v][j + 2], dw[v][j + 3]);
            all[wave - half][4 * v + 2 + j / 4][lane] = make_float4(db[v][j], db[v][j + 1], db[v][j + 2], db[v][j + 3]);
          }
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int v = 0; v < V; v++)
#pragma unroll
          for (int j = 0; j < 8; j += 4) {
            const float4 x = all[wave][4 * v + j / 4][lane], y = all[wave][4 * v + 2 + j / 4][lane];
            dw[v][j] += x.x, dw[v][j + 1] += x.y, dw[v][j + 2] += x.z, dw[v][j + 3] += x.w;
            db[v][j] += y.x, db[v][j + 1] += y.y, db[v][j + 2] += y.z, db[v][j + 3] += y.w;
          }
      }
      __syncthreads();
    }
    if (threadIdx.x < LANES) store_sums();
  }
}

// dw (blockIdx.y = 0) and db (1) from the blocks' sums: 32 columns x 32 runs, in a fixed order
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* partial, int blocks, int d, int wf32, void* dw, void* db) {
  __shared__ float part[16][32];
  void* out = blockIdx.y ? db : dw;
  if (!out) return;
  const int lane = threadIdx.x & 31, col = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < d) {
    const float* p = partial + (size_t)blockIdx.y * d + col;
    for (int q = threadIdx.x >> 5; q < blocks; q += 32 * 8) {  // eight loads in flight, the last ones, too
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; u++) v[u] = p[(size_t)min(q + 32 * u, blocks - 1) * 2 * d];
#pragma unroll
      for (int u = 0; u < 8; u++) s += q + 32 * u < blocks ? v[u] : 0.f;
    }
  }
  s = add_rows32(s);
  if ((threadIdx.x & 63) < 32) part[threadIdx.x >> 6][lane] = s;
  __syncthreads();
  if (threadIdx.x < 32 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r++) t += part[r][lane];
    if (wf32) ((float*)out)[col] = t;
    else Elem<bf16_t>::store((bf16_t*)out + col, t);
  }
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
  if (n->n_rows < 0 || n->n_rows > kNormMaxRows || n->d < 1 || n->d > kNormMaxD || !(n->eps >= 0.f) || n->eps > 3.4e38f) {
    set_error("%s: bad sizes: %d rows of %d (1 to %d), eps %g", who, n->n_rows, n->d, kNormMaxD, (double)n->eps);
    return MOE_EINVAL;
  }
  return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_norm_bwd_workspace_bytes(const moe_norm_t* norm) {
  if (check_norm(norm, "moe_norm_bwd_workspace_bytes")) return 0;
  return (size_t)norm_plan(norm, true, true, true).blocks * 2 * (size_t)norm->d * sizeof(float) + 256;  // (no plan of the call has more)
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
  if ((rc = check_places(who, "Z", Z, ldz, "X", X, ldx, n)) || (rc = check_places(who, "Z", Z, ldz, "R", R, ldr, n)) ||
      (rc = check_places(who, "Y", Y, ldy, "X", X, ldx, n)) || (rc = check_places(who, "Y", Y, ldy, "R", R, ldr, n)))
    return rc;
  if (n > 0 && Y == Z) {
    set_error("%s: Y and Z overlap", who);
    return MOE_EINVAL;
  }
  if (Z && !sum) {
    set_error("%s: Z goes with R or drop; without them it would be X", who);
    return MOE_EINVAL;
  }
  if (mean && norm->kind == MOE_NORM_RMS) {
    set_error("%s: an RMS norm has no mean", who);
    return MOE_EINVAL;
  }
  if (n == 0) return MOE_OK;
  const NormPlan p = norm_plan(norm, false, false, false);
  const NormFwd a = {X, R, w, b, Z, Y, mean, rstd, ldx, ldr, ldz, ldy, n, d, norm->kind == MOE_NORM_LAYER, norm->wdtype == MOE_F32, norm->eps, dr};
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid(p.blocks), block(64 * p.waves);
  ProfScope prof("norm_fwd_kernel", st);
// (blocks of two pieces a lane are the plan of bf16 rows alone, and in the backward pass of full pieces)
#define MOE_NORM_FWD_BY_PLAN(T, TAIL, TINY, BY_VALUE)                                         \
  do {                                                                                        \
    if (p.team == kLongTeam) MOE_NORM_FWD(T, BY_VALUE, 2, kLongTeam);                         \
    else if (p.team == kBlockTeam && p.V == 2) MOE_NORM_FWD(bf16_t, BY_VALUE, 2, kBlockTeam); \
    else if (p.team == kBlockTeam) MOE_NORM_FWD(T, TAIL, 1, kBlockTeam);                      \
    else if (p.V == 2) MOE_NORM_FWD(T, BY_VALUE, 2, kWaveTeam);                               \
    else if (p.team == kLanes16Team) MOE_NORM_FWD(T, TINY, 1, kLanes16Team);                  \
    else if (p.team == kLanes32Team) MOE_NORM_FWD(T, TAIL, 1, kLanes32Team);                  \
    else MOE_NORM_FWD(T, TAIL, 1, kWaveTeam);                                                 \
  } while (0)
#define MOE_NORM_FWD(T, TAIL, V, TEAM)                                                                                \
  do {                                                                                                                \
    if (!sum && rstd) hipLaunchKernelGGL((norm_fwd_kernel<T, TAIL, V, TEAM, kPlain>), grid, block, 0, st, a);         \
    else if (!sum) hipLaunchKernelGGL((norm_fwd_kernel<T, TAIL, V, TEAM, kPass>), grid, block, 0, st, a);             \
    else if (dr.threshold == 0) hipLaunchKernelGGL((norm_fwd_kernel<T, TAIL, V, TEAM, kAdd>), grid, block, 0, st, a); \
    else hipLaunchKernelGGL((norm_fwd_kernel<T, TAIL, V, TEAM, kDrop>), grid, block, 0, st, a);                       \
  } while (0)
  if (norm->dtype == MOE_F32) MOE_NORM_FWD_BY_PLAN(float, kByValue, kByValue, kByValue);
  else if (d % 8) MOE_NORM_FWD_BY_PLAN(bf16_t, kTail, kTinyTail, kByValue);
  else MOE_NORM_FWD_BY_PLAN(bf16_t, kNoTail, kNoTail, kNoTail);
#undef MOE_NORM_FWD
#undef MOE_NORM_FWD_BY_PLAN
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
  if ((rc = check_places(who, "dR", dR, lddr, "dY", dY, lddy, n)) || (rc = check_places(who, "dR", dR, lddr, "dZ", dZ, lddz, n)) ||
      (rc = check_places(who, "dR", dR, lddr, "Z", Z, ldz, n)) || (rc = check_places(who, "dX", dX, lddx, "dY", dY, lddy, n)) ||
      (rc = check_places(who, "dX", dX, lddx, "dZ", dZ, lddz, n)) || (rc = check_places(who, "dX", dX, lddx, "Z", Z, ldz, n)))
    return rc;
  if (n > 0 && dR && dR == dX) {
    set_error("%s: dR and dX overlap", who);
    return MOE_EINVAL;
  }
  const bool weights = dw || db;
  const NormPlan p = norm_plan(norm, true, dr.threshold != 0, (dR && (dR == dY || dR == Z)) || (dX && (dX == dY || dX == Z)));
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
    const NormBwd a = {dY, Z, w, dZ, mean, rstd, dR, dX, weights && !p.columns ? (float*)ws : nullptr, dw, db, lddy, ldz, lddz, lddr, lddx, n, d,
                       norm->kind == MOE_NORM_LAYER, norm->wdtype == MOE_F32, p.blocks, dr};
    const dim3 grid(p.blocks + (weights ? p.columns : 0)), block(64 * p.waves);
    const bool once = dZ && !p.columns;
    ProfScope prof("norm_bwd_kernel", st);
#define MOE_NORM_BWD_AS(T, TAIL, V, TEAM, ONCE)                                                           \
  do {                                                                                                    \
    if (drop) hipLaunchKernelGGL((norm_bwd_kernel<T, TAIL, V, TEAM, true, ONCE>), grid, block, 0, st, a); \
    else hipLaunchKernelGGL((norm_bwd_kernel<T, TAIL, V, TEAM, false, ONCE>), grid, block, 0, st, a);     \
  } while (0)
#define MOE_NORM_BWD(T, TAIL, V, TEAM)                 \
  do {                                                 \
    if (once) MOE_NORM_BWD_AS(T, TAIL, V, TEAM, true); \
    else MOE_NORM_BWD_AS(T, TAIL, V, TEAM, false);     \
  } while (0)
#define MOE_NORM_BWD_BY_PLAN(T, TAIL, TINY, BY_VALUE)                                        \
  do {                                                                                       \
    if (p.team == kLongTeam) MOE_NORM_BWD_AS(T, BY_VALUE, 2, kLongTeam, false);              \
    else if (p.team == kBlockTeam && p.V == 2) MOE_NORM_BWD(bf16_t, kNoTail, 2, kBlockTeam); \
    else if (p.team == kBlockTeam) MOE_NORM_BWD(T, TAIL, 1, kBlockTeam);                     \
    else if (p.V == 2) MOE_NORM_BWD(T, TAIL, 2, kWaveTeam);                                  \
    else if (p.team == kLanes16Team) MOE_NORM_BWD(T, TINY, 1, kLanes16Team);                 \
    else if (p.team == kLanes32Team) MOE_NORM_BWD(T, TAIL, 1, kLanes32Team);                 \
    else MOE_NORM_BWD(T, TAIL, 1, kWaveTeam);                                                \
  } while (0)
    if (norm->dtype == MOE_F32) MOE_NORM_BWD_BY_PLAN(float, kByValue, kByValue, kByValue);
    else if (d % 8) MOE_NORM_BWD_BY_PLAN(bf16_t, kTail, kTinyTail, kByValue);
    else MOE_NORM_BWD_BY_PLAN(bf16_t, kNoTail, kNoTail, kNoTail);
#undef MOE_NORM_BWD_BY_PLAN
#undef MOE_NORM_BWD
#undef MOE_NORM_BWD_AS
  }
  if (weights && (n == 0 || !p.columns)) {
    ProfScope prof("norm_weights_kernel", st);
    hipLaunchKernelGGL(norm_weights_kernel, dim3((d + 31) / 32, 2), dim3(1024), 0, st, (const float*)ws, n > 0 ? p.blocks : 0, d, (int)(norm->wdtype == MOE_F32),
                       dw, db);
  }
  return n > 0 || weights ? launch_status(who) : MOE_OK;
}
