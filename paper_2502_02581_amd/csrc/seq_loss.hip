// moe_seq_loss / moe_seq_loss_bwd: balance loss and expert counts of every sequence, z loss of the router, and their gradient.
//
//   sequence s owns tokens [start_s, start_s + len_s); T_s of them; S' sequences have any, T' is their sum
//   p_t = the gate's scores as shares of one;  P_se = (1 / T_s) sum_t p_te;  n_se = how often e was chosen;  f_se = n_se / (k T_s)
//   balance = alpha / S' sum_s E sum_e f_se P_se;   z = beta / T' sum_t lse_t^2, lse_t = log sum_e exp(logit_te)
//   dz_te = coef_s n_s. through the shares (the loads held constant) + coef_z lse_t softmax_te,  coef_s = alpha E / (S' k T_s^2),  coef_z = 2 beta / T'
//
// Tokens are cut into chunks of equal length, one a wavefront, and chunks into the pieces that belong to one sequence.  Sequences ascend, so chunk c's
// piece of sequence s has the number c + s: along the tokens one of the two grows by one at every border, no two pieces share a number, and those of a
// sequence are neighbours.  The sums of a piece, of a sequence's pieces and of the loss are each added in a fixed order.
#include <initializer_list>

#include "rows.h"

namespace moe {

constexpr int kSeqBlocks = 1024;  // blocks of the second launch at most
struct SeqInfo {                  // start of the workspace
  int32_t filled, tokens;         // S', T'
  uint32_t done, pad;             // blocks of the second launch that have ended
  double2 part[kSeqBlocks];       // their sums of the two losses
};
struct SeqArgs {
  const float* logits;
  const int32_t *topk, *start, *len;
  int T, E, k, gate, S, chunk, chunks;
  float* psum;       // [chunks + S][E] sums of shares
  uint16_t* pcount;  // [chunks + S][E]
  float* pz;         // [chunks + S] sums of lse^2
  SeqInfo* info;
};

// The tokens of sequence s, within 0 .. T and not beyond the next one's first: whatever the arrays hold, no index leaves the tensors.
__device__ __forceinline__ int2 seq_range(const int32_t* start, const int32_t* len, int S, int T, int s) {
  if (!start) return make_int2(0, T);
  const int from = min(max(start[s], 0), T);
  const int next = s + 1 < S || !len ? start[s + 1] : T;
  const int64_t end = len ? (int64_t)start[s] + len[s] : next;
  const int to = (int)min(min(end, (int64_t)max(next, 0)), (int64_t)T);
  return make_int2(from, max(to, from));
}

// The last sequence that starts at or before t, at least 0 (uniform): each step asks 64 places at once.
__device__ __forceinline__ int find_seq(const int32_t* start, int S, int t) {
  if (!start) return 0;
  int lo = 0, n = S;  // the answer is in [lo, lo + n) or it is lo
  while (n > 1) {
    const int step = (n + 63) / 64, at = (int)(threadIdx.x & 63) * step;
    const uint64_t ask = __ballot(at < n && start[lo + (at < n ? at : 0)] <= t);
    const int q = ask ? 63 - __clzll(ask) : 0;
    lo += q * step;
    n = min(step, n - q * step);
  }
  return lo;
}

// A row of logits over L lanes: lane l of the group holds experts 4 (l + L q) .. + 3, q < Q.
template <int L> __device__ __forceinline__ float group_sum(float x) {
  if (L >= 2) x = add_dpp(x, 0);
  if (L >= 4) x = add_dpp(x, 1);
  if (L >= 8) x = add_dpp(x, 2);
  if (L >= 16) x = add_dpp(x, 3);
  if (L >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (L >= 64) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  }
  return x;
}
template <int L> __device__ __forceinline__ float group_max(float x) {
#pragma unroll
  for (int m = 1; m < L; m <<= 1) x = fmaxf(x, __shfl_xor(x, m, kWave));
  return x;
}
template <int Q> struct Row {
  float v[Q][4];
};
template <int L, int Q>
__device__ __forceinline__ void load_logits(const float* row, int lane, int E, Row<Q>& x) {
#pragma unroll
  for (int q = 0; q < Q; q++) {
    const int e = 4 * (lane + L * q);
    if (e + 4 <= E) {
      __builtin_memcpy(x.v[q], row + e, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) x.v[q][j] = e + j < E ? row[e + j] : -INFINITY;
    }
  }
}
// soft: softmax; score, share: the gate's; lse.  A row without a finite logit has shares and lse 0, as has one whose sigmoid scores are all 0 in fp32.
template <int L, int Q>
__device__ __forceinline__ void gate_row(const Row<Q>& x, int lane, int E, bool softmax, bool need_soft, Row<Q>& soft, Row<Q>& score, Row<Q>& share, float& lse) {
  lse = 0.f;
  if (softmax || need_soft) {
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) m = fmaxf(m, x.v[q][j]);
    m = group_max<L>(m);
    const bool empty = m == -INFINITY;
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        soft.v[q][j] = empty ? 0.f : expf(x.v[q][j] - m);
        s += soft.v[q][j];
      }
    s = group_sum<L>(s);
    const float inv = empty ? 0.f : 1.f / s;
    lse = empty ? 0.f : m + logf(s);
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) soft.v[q][j] *= inv;
  }
  if (softmax) {
    share = soft;
    return;
  }
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < Q; q++)
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const bool in = 4 * (lane + L * q) + j < E;
      score.v[q][j] = in ? 1.f / (1.f + expf(-x.v[q][j])) : 0.f;
      s += score.v[q][j];
    }
  s = group_sum<L>(s);
#pragma unroll
  for (int q = 0; q < Q; q++)
#pragma unroll
    for (int j = 0; j < 4; j++) share.v[q][j] = s == 0.f ? 0.f : score.v[q][j] / s;  // (divided: a single expert's share is 1)
}

template <int L, int Q>
__global__ __launch_bounds__(256) void seq_sums_kernel(SeqArgs a, int want_z) {
  extern __shared__ int32_t hist_all[];  // [4][E]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x == gridDim.x - 1) {  // the last block: how many sequences have tokens, and how many tokens there are
    int filled = 0, tokens = 0;
    for (int s = threadIdx.x; s < a.S; s += 256) {
      const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
      filled += r.y > r.x;
      tokens += r.y - r.x;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
      filled += __shfl_xor(filled, m, kWave);
      tokens += __shfl_xor(tokens, m, kWave);
    }
    __shared__ int part[2][4];
    if (lane == 0) {
      part[0][wave] = filled;
      part[1][wave] = tokens;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      a.info->filled = part[0][0] + part[0][1] + part[0][2] + part[0][3];
      a.info->tokens = part[1][0] + part[1][1] + part[1][2] + part[1][3];
      a.info->done = 0;
    }
    return;
  }
  const int c = blockIdx.x * 4 + wave;
  if (c >= a.chunks) return;
  int32_t* hist = hist_all + wave * a.E;
  for (int e = lane; e < a.E; e += 64) hist[e] = 0;
  constexpr int G = 64 / L;
  const int group = lane / L, l = lane % L;
  const int t0 = c * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const bool softmax = a.gate == MOE_GATE_SOFTMAX;
  for (int s = find_seq(a.start, a.S, t0); s < a.S; s++) {
    const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
    if (r.x >= t1) break;
    const int from = max(r.x, t0), to = min(r.y, t1);
    if (from >= to) continue;
    // how often each expert was chosen: whole numbers, so the order of the additions plays no part
    for (int64_t i = (int64_t)from * a.k + lane; i < (int64_t)to * a.k; i += 64) {
      const int e = a.topk[i];
      if ((unsigned)e < (unsigned)a.E) atomicAdd(&hist[e], 1);
    }
    Row<Q> acc;
    float z2 = 0.f;
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) acc.v[q][j] = 0.f;
    for (int t = from + group; t < to; t += G) {
      Row<Q> x, soft, score, share;
      float lse;
      load_logits<L, Q>(a.logits + (size_t)t * a.E, l, a.E, x);
      gate_row<L, Q>(x, l, a.E, softmax, want_z, soft, score, share, lse);
      z2 = fmaf(lse, lse, z2);
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc.v[q][j] += share.v[q][j];
    }
#pragma unroll
    for (int m = L; m < 64; m <<= 1) {
      z2 += __shfl_xor(z2, m, kWave);
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc.v[q][j] += __shfl_xor(acc.v[q][j], m, kWave);
    }
    const size_t piece = (size_t)c + s;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane == 0) a.pz[piece] = z2;
    if (group == 0) {
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int e = 4 * (l + L * q) + j;
          if (e < a.E) a.psum[piece * a.E + e] = acc.v[q][j];
        }
    }
    for (int e = lane; e < a.E; e += 64) {
      a.pcount[piece * a.E + e] = (uint16_t)hist[e];
      hist[e] = 0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// P, counts and coef of every sequence, and the losses.  A job is 16 experts of a sequence; the block's threads are 16 columns x runs.
struct SeqFinish {
  SeqArgs a;
  float alpha, beta;
  int32_t* counts;
  float *P, *loss, *coef;
};
__global__ __launch_bounds__(1024) void seq_finish_kernel(SeqFinish f) {
  const SeqArgs& a = f.a;
  __shared__ float psum[64][16];
  __shared__ int32_t pcount[64][16];
  __shared__ double wsum[2][16];
  __shared__ int last;
  const int col = threadIdx.x & 15, run = threadIdx.x >> 4, runs = blockDim.x >> 4;
  const int tiles = (a.E + 15) / 16;
  const int filled = a.info->filled, tokens = a.info->tokens;
  const double per_seq = filled > 0 ? (double)f.alpha * a.E / filled : 0.;
  double balance = 0., z2 = 0.;
  for (int64_t job = blockIdx.x; job < (int64_t)a.S * tiles; job += gridDim.x) {
    const int s = (int)(job / tiles), e = (int)(job - (int64_t)s * tiles) * 16 + col;
    const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
    const int n = r.y - r.x;
    const int64_t p0 = n ? (int64_t)(r.x / a.chunk) + s : 0, p1 = n ? (int64_t)((r.y - 1) / a.chunk) + s + 1 : 0;
    float sum = 0.f;
    int count = 0;
    if (e < a.E) {
#pragma unroll 4
      for (int64_t p = p0 + run; p < p1; p += runs) {
        sum += a.psum[p * a.E + e];
        count += a.pcount[p * a.E + e];
      }
    }
    psum[run][col] = sum;
    pcount[run][col] = count;
    __syncthreads();
    if (run == 0 && e < a.E) {
      for (int q = 1; q < runs; q++) {
        sum += psum[q][col];
        count += pcount[q][col];
      }
      const float share = n ? sum / (float)n : 0.f;
      f.P[(size_t)s * a.E + e] = share;
      f.counts[(size_t)s * a.E + e] = count;
      if (n) balance += per_seq * ((double)count / ((double)a.k * n)) * share;
      if (e == 0) f.coef[s] = n ? (float)(per_seq / ((double)a.k * n * n)) : 0.f;
    }
    if (e < 16 && f.beta != 0.f)  // (the first of the sequence's jobs)
      for (int64_t p = p0 + threadIdx.x; p < p1; p += blockDim.x) z2 += a.pz[p];
    __syncthreads();
  }
  // the block's sums, then, in the block that ends last, those of all blocks
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    balance += __shfl_xor(balance, m, kWave);
    z2 += __shfl_xor(z2, m, kWave);
  }
  const int n_waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    wsum[0][threadIdx.x >> 6] = balance;
    wsum[1][threadIdx.x >> 6] = z2;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double b = 0., z = 0.;
    for (int w = 0; w < n_waves; w++) {
      b += wsum[0][w];
      z += wsum[1][w];
    }
    __hip_atomic_store(&a.info->part[blockIdx.x].x, b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&a.info->part[blockIdx.x].y, z, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(&a.info->done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  double b = 0., z = 0.;
  for (int q = threadIdx.x; q < (int)gridDim.x; q += blockDim.x) {
    b += __hip_atomic_load(&a.info->part[q].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    z += __hip_atomic_load(&a.info->part[q].y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    b += __shfl_xor(b, m, kWave);
    z += __shfl_xor(z, m, kWave);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    wsum[0][threadIdx.x >> 6] = b;
    wsum[1][threadIdx.x >> 6] = z;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    b = z = 0.;
    for (int w = 0; w < n_waves; w++) {
      b += wsum[0][w];
      z += wsum[1][w];
    }
    const double per_token = tokens > 0 ? (double)f.beta / tokens : 0.;
    f.loss[0] = (float)b;
    f.loss[1] = (float)(per_token * z);
    f.coef[a.S] = (float)(2. * per_token);
  }
}

template <int L, int Q>
__global__ __launch_bounds__(256) void seq_bwd_kernel(SeqArgs a, const int32_t* __restrict__ counts, const float* __restrict__ coef, float dloss,
                                                      int accumulate, float* dlogits) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 4 + wave;
  if (c >= a.chunks) return;
  constexpr int G = 64 / L;
  const int group = lane / L, l = lane % L;
  const int t0 = c * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const bool softmax = a.gate == MOE_GATE_SOFTMAX;
  const float cz = dloss * coef[a.S];
  int at = t0;  // tokens before it are done
  auto outside = [&](int to) {  // tokens of no sequence have no gradient
    if (!accumulate)
      for (size_t i = (size_t)at * a.E + lane; i < (size_t)to * a.E; i += 64) dlogits[i] = 0.f;
  };
  for (int s = find_seq(a.start, a.S, t0); s < a.S; s++) {
    const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
    if (r.x >= t1) break;
    const int from = max(r.x, at), to = min(r.y, t1);
    if (from >= to) continue;
    outside(from);
    Row<Q> up;
    const float cs = dloss * coef[s];
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = 4 * (l + L * q) + j;
        up.v[q][j] = e < a.E ? cs * (float)counts[(size_t)s * a.E + e] : 0.f;
      }
    for (int t = from + group; t < to; t += G) {
      Row<Q> x, soft, score, share;
      float lse, dot = 0.f;
      load_logits<L, Q>(a.logits + (size_t)t * a.E, l, a.E, x);
      gate_row<L, Q>(x, l, a.E, softmax, cz != 0.f, soft, score, share, lse);
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) dot = fmaf(share.v[q][j], up.v[q][j], dot);
      dot = group_sum<L>(dot);
      const float zl = cz * lse;
#pragma unroll
      for (int q = 0; q < Q; q++) {
        const int e = 4 * (l + L * q);
        float* o = dlogits + (size_t)t * a.E + e;
        float dz[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
          dz[j] = share.v[q][j] * (up.v[q][j] - dot);
          if (!softmax) dz[j] *= 1.f - score.v[q][j];
          if (cz != 0.f) dz[j] = fmaf(zl, soft.v[q][j], dz[j]);
        }
        if (e + 4 <= a.E) {
          if (accumulate) {
            float old[4];
            __builtin_memcpy(old, o, 16);
#pragma unroll
            for (int j = 0; j < 4; j++) dz[j] += old[j];
          }
          __builtin_memcpy(o, dz, 16);
        } else {
#pragma unroll
          for (int j = 0; j < 4; j++)
            if (e + j < a.E) o[j] = accumulate ? o[j] + dz[j] : dz[j];
        }
      }
    }
    at = to;
  }
  outside(t1);
}

// instances by the lanes that a row of logits takes: CALL(L, Q)
#define MOE_BY_ROW(E, CALL)           \
  do {                                \
    if ((E) <= 4) CALL(1, 1);         \
    else if ((E) <= 8) CALL(2, 1);    \
    else if ((E) <= 16) CALL(4, 1);   \
    else if ((E) <= 32) CALL(8, 1);   \
    else if ((E) <= 64) CALL(16, 1);  \
    else if ((E) <= 128) CALL(32, 1); \
    else if ((E) <= 256) CALL(64, 1); \
    else if ((E) <= 512) CALL(64, 2); \
    else CALL(64, 4);                 \
  } while (0)

// tokens of a wavefront: enough wavefronts for the chip, and in each enough tokens for its groups
static int seq_chunk(int T, int E) {
  const int lanes = E <= 4 ? 1 : E <= 8 ? 2 : E <= 16 ? 4 : E <= 32 ? 8 : E <= 64 ? 16 : E <= 128 ? 32 : 64;
  const int groups = 64 / lanes;
  const int want = (T + 4095) / 4096;
  const int chunk = (want + groups - 1) / groups * groups;
  return chunk < 4 ? 4 : chunk > 256 ? 256 : chunk;
}
struct SeqPlan {
  int chunk, chunks;
  size_t pieces, sums, counts, z, bytes;  // places of the workspace
};
static SeqPlan seq_plan(const moe_shape_t* s, int n_seqs) {
  SeqPlan p;
  p.chunk = seq_chunk(s->T, s->E);
  p.chunks = (s->T + p.chunk - 1) / p.chunk;
  p.pieces = (size_t)p.chunks + n_seqs;
  p.sums = align_up(sizeof(SeqInfo), 256);
  p.counts = p.sums + align_up(p.pieces * s->E * 4, 256);
  p.z = p.counts + align_up(p.pieces * s->E * 2, 256);
  p.bytes = p.z + align_up(p.pieces * 4, 256);
  return p;
}
static int check_seqs(const moe_shape_t* shape, int n_seqs, const int32_t* start, const int32_t* len, const char* who) {
  const int rc = check_shape(shape, who);
  if (rc) return rc;
  if (n_seqs < 1 || n_seqs > 1 << 24 || (!start && (len || n_seqs != 1))) {
    set_error("%s: bad sequences: %d of them (1 to 2^24; without seq_start one, and then no seq_len)", who, n_seqs);
    return MOE_EINVAL;
  }
  return MOE_OK;
}

static bool aligned4(std::initializer_list<const void*> tensors) {
  uintptr_t all = 0;
  for (const void* p : tensors) all |= (uintptr_t)p;
  return (all & 3) == 0;
}

}  // namespace moe

extern "C" size_t moe_seq_loss_workspace_bytes(const moe_shape_t* shape, int32_t n_seqs) {
  if (!shape || shape->T < 0 || shape->E < 1 || shape->E > MOE_MAX_EXPERTS || n_seqs < 1) return 0;
  return moe::seq_plan(shape, n_seqs).bytes;
}

extern "C" int moe_seq_loss(const moe_shape_t* shape, const float* logits, const int32_t* topk_idx, int32_t n_seqs, const int32_t* seq_start,
                            const int32_t* seq_len, float alpha, float beta, int32_t* counts, float* P, float* loss, float* coef, void* ws,
                            size_t ws_bytes, void* stream) {
  using namespace moe;
  int rc = check_seqs(shape, n_seqs, seq_start, seq_len, "moe_seq_loss");
  if (rc) return rc;
  if (!counts || !P || !loss || !coef || !ws || (shape->T > 0 && (!logits || !topk_idx))) {
    set_error("moe_seq_loss: null pointer");
    return MOE_EINVAL;
  }
  if (!aligned16(ws) || !aligned4({logits, topk_idx, seq_start, seq_len, counts, P, loss, coef})) {
    set_error("moe_seq_loss: ws must be 16-byte aligned, every other tensor aligned to its values");
    return MOE_EINVAL;
  }
  const SeqPlan p = seq_plan(shape, n_seqs);
  if (ws_bytes < p.bytes) {
    set_error("moe_seq_loss: workspace of %zu bytes, need %zu", ws_bytes, p.bytes);
    return MOE_EWS;
  }
  hipStream_t st = (hipStream_t)stream;
  char* w = (char*)ws;
  const SeqArgs a = {logits, topk_idx, seq_start, seq_len, shape->T, shape->E, shape->k, shape->gate, n_seqs, p.chunk, p.chunks,
                     (float*)(w + p.sums), (uint16_t*)(w + p.counts), (float*)(w + p.z), (SeqInfo*)w};
  {
    ProfScope prof("seq_sums_kernel", st);
    const dim3 grid((p.chunks + 3) / 4 + 1), block(256);
    const size_t lds = 4 * sizeof(int32_t) * shape->E;
#define MOE_SEQ_SUMS(L, Q) hipLaunchKernelGGL((seq_sums_kernel<L, Q>), grid, block, lds, st, a, (int)(beta != 0.f))
    MOE_BY_ROW(shape->E, MOE_SEQ_SUMS);
#undef MOE_SEQ_SUMS
  }
  {
    ProfScope prof("seq_finish_kernel", st);
    const int64_t jobs = (int64_t)n_seqs * ((shape->E + 15) / 16);
    const int per = p.chunks / n_seqs;  // pieces of an ordinary sequence
    const SeqFinish f = {a, alpha, beta, counts, P, loss, coef};
    hipLaunchKernelGGL(seq_finish_kernel, dim3((unsigned)(jobs < kSeqBlocks ? jobs : kSeqBlocks)), dim3(per > 256 ? 1024 : per > 32 ? 256 : 64), 0, st, f);
  }
  return launch_status("moe_seq_loss");
}

extern "C" int moe_seq_loss_bwd(const moe_shape_t* shape, const float* logits, int32_t n_seqs, const int32_t* seq_start, const int32_t* seq_len,
                                const int32_t* counts, const float* coef, float dloss, int32_t accumulate, float* dlogits, void* stream) {
  using namespace moe;
  int rc = check_seqs(shape, n_seqs, seq_start, seq_len, "moe_seq_loss_bwd");
  if (rc) return rc;
  if (shape->T == 0) return MOE_OK;  // nothing to do (empty tensors may be null)
  if (!logits || !counts || !coef || !dlogits) {
    set_error("moe_seq_loss_bwd: null pointer");
    return MOE_EINVAL;
  }
  if (!aligned4({logits, seq_start, seq_len, counts, coef, dlogits})) {
    set_error("moe_seq_loss_bwd: every tensor must be aligned to its values");
    return MOE_EINVAL;
  }
  const SeqPlan p = seq_plan(shape, n_seqs);
  const SeqArgs a = {logits, nullptr, seq_start, seq_len, shape->T, shape->E, shape->k, shape->gate, n_seqs, p.chunk, p.chunks, nullptr, nullptr, nullptr, nullptr};
  hipStream_t st = (hipStream_t)stream;
  ProfScope prof("seq_bwd_kernel", st);
  const dim3 grid((p.chunks + 3) / 4), block(256);
#define MOE_SEQ_BWD(L, Q) hipLaunchKernelGGL((seq_bwd_kernel<L, Q>), grid, block, 0, st, a, counts, coef, dloss, (int)accumulate, dlogits)
  MOE_BY_ROW(shape->E, MOE_SEQ_BWD);
#undef MOE_SEQ_BWD
  return launch_status("moe_seq_loss_bwd");
}
