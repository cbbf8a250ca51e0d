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

constexpr int kSeqBlocks = 1024, kSeqGroups = kSeqBlocks / 32;  // blocks of the second launch at most
struct SeqInfo {  // start of the workspace
  int32_t filled, tokens;  // S', T'
  uint32_t done[1 + kSeqGroups][16];  // blocks of the second launch that have ended, by groups of 32, and groups that have (a line of the cache each)
  float2 part[kSeqBlocks];            // their sums of the two losses
};
struct SeqArgs {
  const float* logits;
  const int32_t *topk, *start, *len;
  int T, E, k, gate, S, chunk, chunks;
  float* psum;       // [chunks + S][E, in fours] sums of shares
  uint16_t* pcount;  // the same of choices
  float* pz;         // [chunks + S] sums of lse^2
  SeqInfo* info;
};

// The tokens of sequence s, within 0 .. T and not beyond the next one's first: whatever the arrays hold, no index leaves the tensors.
__device__ __forceinline__ int2 seq_range(const int32_t* start, const int32_t* len, int S, int T, int s) {
  if (!start) return make_int2(0, T);
  const int first = start[s], next = s + 1 < S || !len ? start[s + 1] : T;
  const int64_t end = len ? (int64_t)first + len[s] : next;
  const int from = min(max(first, 0), T);
  const int to = (int)min(min(end, (int64_t)max(next, 0)), (int64_t)T);
  return make_int2(from, max(to, from));
}

// The sequences that have tokens in [t0, t1), one after the other.  A lane holds the range of one of 64 neighbouring sequences, so that the next one costs no load, and empty
// ones cost nothing.
struct SeqWalk {
  int2 range;
  uint64_t hits;  // lanes whose sequence has tokens in the chunk and was not visited
  int base;
  __device__ __forceinline__ void window(const SeqArgs& a, int t0, int t1) {
    const int s = base + (int)(threadIdx.x & 63);
    range = s < a.S ? seq_range(a.start, a.len, a.S, a.T, s) : make_int2(a.T, a.T);
    hits = __ballot(range.x < t1 && range.y > t0 && range.y > range.x);
  }
  __device__ __forceinline__ void begin(const SeqArgs& a, int t0, int t1) {
    base = 0;
    int n = a.S;  // the last sequence that starts at or before t0 is in [base, base + n), or it is base: each step asks 64 places at once
    while (n > 64) {
      const int step = (n + 63) / 64, at = (int)(threadIdx.x & 63) * step;
      const uint64_t ask = __ballot(at < n && a.start[base + (at < n ? at : 0)] <= t0);
      const int q = ask ? 63 - __clzll(ask) : 0;
      base += q * step;
      n = min(step, n - q * step);
    }
    window(a, t0, t1);
  }
  // the next one: its number and its tokens within the chunk; false: there is none
  __device__ __forceinline__ bool next(const SeqArgs& a, int t0, int t1, int& s, int& from, int& to) {
    while (!hits) {
      if (base + 64 >= a.S || __builtin_amdgcn_readlane(range.x, 63) >= t1) return false;
      base += 64;
      window(a, t0, t1);
    }
    const int i = __ffsll((unsigned long long)hits) - 1;
    hits &= hits - 1;
    s = base + i;
    from = max(__builtin_amdgcn_readlane(range.x, i), t0);
    to = min(__builtin_amdgcn_readlane(range.y, i), t1);
    return true;
  }
};

// A row of logits over L lanes: lane l of the group holds experts 4 (l + L q) .. + 3, q < Q.
template <int L> __device__ __forceinline__ float group_sum(float x) {
  if (L >= 2) x = add_lanes1(x);
  if (L >= 4) x = add_lanes2(x);
  if (L >= 8) x = add_lanes4(x);
  if (L >= 16) x = add_lanes8(x);
  if (L >= 32) x = add_rows16(x);
  if (L >= 64) x = add_rows32(x);
  return x;
}
template <int L> __device__ __forceinline__ float group_max(float x) {
  if (L >= 2) x = fmaxf(x, dpp<0xB1>(x));
  if (L >= 4) x = fmaxf(x, dpp<0x4E>(x));
  if (L >= 8) x = fmaxf(x, dpp<0x141>(x));
  if (L >= 16) x = fmaxf(x, dpp<0x140>(x));
  if (L >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  if (L >= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  return x;
}
// 1 / x within one rounding or so of it: the instruction's value, improved once
__device__ __forceinline__ float reciprocal(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return fmaf(fmaf(-x, r, 1.f), r, r);
}
template <int Q> struct Row {
  float v[Q][4];
};
template <int L, int Q>
__device__ __forceinline__ void load_logits(const float* row, int l, int E, bool there, Row<Q>& x) {
#pragma unroll
  for (int q = 0; q < Q; q++) {
    const int e = 4 * (l + L * q);
    if (there && e + 4 <= E) {
      __builtin_memcpy(x.v[q], row + e, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) x.v[q][j] = there && e + j < E ? row[e + j] : -INFINITY;
    }
  }
}
// The exponentials are the instruction's, 2^(x log2 e): off by 1.5 |x| + 2 roundings, so a share e^-10 of the row's largest by 17, the largest by none.  (The kernels are bound by
// their instructions before they are by bytes: with expf and divisions 131072 tokens of 64 experts take 14.7 + 18.4 us.)
// soft: softmax; score, share: the gate's; lse.  A row without a finite logit has shares and lse 0, as has one whose sigmoid scores are all 0 in fp32.
template <int L, int Q>
__device__ __forceinline__ void gate_row(const Row<Q>& x, int l, int E, bool softmax, bool need_soft, Row<Q>& soft, Row<Q>& score, Row<Q>& share, float& lse) {
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
        soft.v[q][j] = empty ? 0.f : __expf(x.v[q][j] - m);
        s += soft.v[q][j];
      }
    s = group_sum<L>(s);
    const float inv = empty ? 0.f : reciprocal(s);
    lse = empty ? 0.f : m + __logf(s);
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
      const bool in = 4 * (l + L * q) + j < E;
      score.v[q][j] = in ? __builtin_amdgcn_rcpf(1.f + __expf(-x.v[q][j])) : 0.f;
      s += score.v[q][j];
    }
  s = group_sum<L>(s);
  const float inv = s == 0.f ? 0.f : reciprocal(s);
#pragma unroll
  for (int q = 0; q < Q; q++)
#pragma unroll
    for (int j = 0; j < 4; j++) {  // the quotient, its own error taken out: a single expert's share is 1
      const float p = score.v[q][j] * inv;
      share.v[q][j] = fmaf(fmaf(-p, s, score.v[q][j]), inv, p);
    }
}
// The first row's load goes out before the search for the chunk's sequences, the next row's before this one is used.  (Four rows at once are no faster: there are other
// wavefronts; a chunk of fewer rows is, where tokens are few: 256 tokens of 8 experts 4.9 -> 2.9 us.)
template <int L, int Q>
__global__ __launch_bounds__(256) void seq_sums_kernel(SeqArgs a, int want_z, float alpha_E, float* coef) {
  extern __shared__ int32_t hist_all[];  // [4][Ep]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x == gridDim.x - 1) {  // the last block: how many sequences have tokens, how many tokens there are, and the sequences' factors
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
    filled = part[0][0] + part[0][1] + part[0][2] + part[0][3];
    if (threadIdx.x == 0) {
      a.info->filled = filled;
      a.info->tokens = part[1][0] + part[1][1] + part[1][2] + part[1][3];
    }
    if (threadIdx.x <= kSeqGroups) a.info->done[threadIdx.x][0] = 0;
    for (int s = threadIdx.x; s < a.S; s += 256) {
      const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
      const float n = (float)(r.y - r.x);
      coef[s] = r.y > r.x ? alpha_E / (float)filled / (float)a.k / n / n : 0.f;
    }
    return;
  }
  const int c = blockIdx.x * 4 + wave;
  if (c >= a.chunks) return;
  constexpr int G = 64 / L;
  const int group = lane / L, l = lane % L, Ep = (a.E + 3) & ~3;
  const int t0 = c * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const bool softmax = a.gate == MOE_GATE_SOFTMAX;
  Row<Q> x, share, acc;
  float lse, z2 = 0.f;
  int ids;            // the first 64 choices of the next tokens
  int at = t0;        // first of the G tokens whose shares are at hand
  auto load = [&](int t) {
    load_logits<L, Q>(a.logits + (size_t)(t + group) * a.E, l, a.E, t + group < t1, x);
    const int64_t i = (int64_t)t * a.k + lane;
    ids = i < (int64_t)t1 * a.k ? a.topk[i] : -1;
  };
  int id = -1;
  auto use = [&]() {
    Row<Q> soft, score;
    gate_row<L, Q>(x, l, a.E, softmax, want_z, soft, score, share, lse);
    id = ids;
    if (at + G < t1) load(at + G);
  };
  load(t0);
  int32_t* hist = hist_all + wave * Ep;
  for (int e = lane; e < Ep; e += 64) hist[e] = 0;
  SeqWalk walk;
  walk.begin(a, t0, t1);
  use();
  int s, from, to;
  while (walk.next(a, t0, t1, s, from, to)) {
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) acc.v[q][j] = 0.f;
    z2 = 0.f;
    for (;;) {
      // how often each expert was chosen: whole numbers, so the order of the additions plays no part
      const int64_t lo = (int64_t)max(from, at) * a.k, hi = (int64_t)min(to, at + G) * a.k;
      int64_t i = (int64_t)at * a.k + lane;
      if (i >= lo && i < hi && (unsigned)id < (unsigned)a.E) atomicAdd(&hist[id], 1);
      for (i += 64; i < hi; i += 64)
        if (i >= lo) {
          const int e = a.topk[i];
          if ((unsigned)e < (unsigned)a.E) atomicAdd(&hist[e], 1);
        }
      const int t = at + group;
      if (t >= from && t < to) {
        z2 = fmaf(lse, lse, z2);
#pragma unroll
        for (int q = 0; q < Q; q++)
#pragma unroll
          for (int j = 0; j < 4; j++) acc.v[q][j] += share.v[q][j];
      }
      if (to <= at + G) break;
      at += G;
      use();
    }
#pragma unroll
    for (int m = L; m < 64; m <<= 1) {
      z2 += __shfl_xor(z2, m, kWave);
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc.v[q][j] += __shfl_xor(acc.v[q][j], m, kWave);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const size_t piece = (size_t)c + s;
    if (lane == 0) a.pz[piece] = z2;
    if (group == 0) {
#pragma unroll
      for (int q = 0; q < Q; q++) {
        const int e = 4 * (l + L * q);
        if (e >= Ep) continue;
        *reinterpret_cast<float4*>(a.psum + piece * Ep + e) = make_float4(acc.v[q][0], acc.v[q][1], acc.v[q][2], acc.v[q][3]);
        const int4 n = *reinterpret_cast<const int4*>(hist + e);
        *reinterpret_cast<uint2*>(a.pcount + piece * Ep + e) = make_uint2((uint32_t)n.x | (uint32_t)n.y << 16, (uint32_t)n.z | (uint32_t)n.w << 16);
        *reinterpret_cast<int4*>(hist + e) = make_int4(0, 0, 0, 0);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// P and counts of every sequence, and the losses.  A job is 16 experts of a sequence: four lanes side by side, and as many pieces at once as the team, a wavefront or
// (WIDE) a block, has fours.
struct SeqFinish {
  SeqArgs a;
  float alpha, beta;
  int32_t* counts;
  float *P, *loss, *coef;
};
template <int WAVES>
__global__ __launch_bounds__(256) void seq_finish_kernel(SeqFinish f) {
  const SeqArgs& a = f.a;
  constexpr bool WIDE = WAVES > 1;
  constexpr int kWaves = WIDE ? WAVES : 4, kRuns = 16 * WAVES;
  __shared__ float4 psum[WIDE ? WAVES : 1][4];
  __shared__ int4 pcount[WIDE ? WAVES : 1][4];
  __shared__ float wsum[2][2][kWaves];
  __shared__ int last;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tiles = (a.E + 15) / 16, Ep = (a.E + 3) & ~3;
  const int run = (WIDE ? threadIdx.x : lane) >> 2;
  const int teams = WIDE ? gridDim.x : gridDim.x * 4;
  float balance = 0.f, z2 = 0.f;
  for (int64_t job = WIDE ? blockIdx.x : blockIdx.x * 4 + wave; job < (int64_t)a.S * tiles; job += teams) {
    const int s = (int)(job / tiles), tile = (int)(job - (int64_t)s * tiles), e = tile * 16 + 4 * (lane & 3);
    const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
    const int n = r.y - r.x;
    const int64_t p0 = n ? (int64_t)(r.x / a.chunk) + s : 0, p1 = n ? (int64_t)((r.y - 1) / a.chunk) + s + 1 : 0;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    int count[4] = {0, 0, 0, 0};
    if (e < Ep) {
#pragma unroll 8
      for (int64_t p = p0 + run; p < p1; p += kRuns) {
        const float4 v = *reinterpret_cast<const float4*>(a.psum + p * Ep + e);
        const uint2 m = *reinterpret_cast<const uint2*>(a.pcount + p * Ep + e);
        sum[0] += v.x; sum[1] += v.y; sum[2] += v.z; sum[3] += v.w;
        count[0] += m.x & 0xffff; count[1] += m.x >> 16; count[2] += m.y & 0xffff; count[3] += m.y >> 16;
      }
    }
    if (tile == 0 && f.beta != 0.f)
      for (int64_t p = p0 + (WIDE ? threadIdx.x : lane); p < p1; p += 64 * WAVES) z2 += a.pz[p];
#pragma unroll
    for (int j = 0; j < 4; j++) {  // lanes whose numbers differ by a multiple of four
      sum[j] = add_rows32(add_rows16(add_quads(sum[j])));
      count[j] = add_rows32(add_rows16(add_quads(count[j])));
    }
    if (WIDE) {
      if (lane < 4) {
        psum[wave][lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        pcount[wave][lane] = make_int4(count[0], count[1], count[2], count[3]);
      }
      __syncthreads();
      if (threadIdx.x < 4) {
#pragma unroll
        for (int w = 1; w < WAVES; w++) {
          const float4 v = psum[w][lane];
          const int4 m = pcount[w][lane];
          sum[0] += v.x; sum[1] += v.y; sum[2] += v.z; sum[3] += v.w;
          count[0] += m.x; count[1] += m.y; count[2] += m.z; count[3] += m.w;
        }
      }
      __syncthreads();
    }
    if ((WIDE ? (int)threadIdx.x : lane) < 4) {
      const float per = n ? 1.f / (float)n : 0.f;
      float b = 0.f;
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (e + j < a.E) {
          const float share = n ? sum[j] / (float)n : 0.f;
          f.P[(size_t)s * a.E + e + j] = share;
          f.counts[(size_t)s * a.E + e + j] = count[j];
          b = fmaf(share, (float)count[j], b);
        }
      balance = fmaf(b, per, balance);
    }
  }
  // The block's sums, then, in the block that ends last, those of all blocks.  Sums and counters go past the caches that other dies do not see (atomics of the agent's scope), and
  // a counter only after the sums have arrived (the wait): releasing and acquiring would write back and drop whole caches for these 8 bytes.  (Counters by groups: a
  // thousand additions to one place take 15 us.)
  auto block_sum = [&](int turn, float b, float z) {
    b = lanes_sum(b);
    z = lanes_sum(z);
    if (lane == 0) {
      wsum[turn][0][wave] = b;
      wsum[turn][1][wave] = z;
    }
    __syncthreads();
    double2 t = {0., 0.};
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
      t.x += wsum[turn][0][w];
      t.y += wsum[turn][1][w];
    }
    return t;
  };
  double2 t = block_sum(0, balance, z2);
  if (gridDim.x > 1) {
    if (threadIdx.x == 0) {
      __hip_atomic_store(&a.info->part[blockIdx.x].x, (float)t.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&a.info->part[blockIdx.x].y, (float)t.y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __builtin_amdgcn_s_waitcnt(0);
      const uint32_t groups = (gridDim.x + 31) / 32, group = blockIdx.x % groups, members = (gridDim.x - group + groups - 1) / groups;
      last = __hip_atomic_fetch_add(&a.info->done[1 + group][0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1 &&
             __hip_atomic_fetch_add(&a.info->done[0][0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
    }
    __syncthreads();
    if (!last) return;
    float b = 0.f, z = 0.f;
#pragma unroll 4
    for (int q = threadIdx.x; q < (int)gridDim.x; q += 64 * kWaves) {
      b += __hip_atomic_load(&a.info->part[q].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      z += __hip_atomic_load(&a.info->part[q].y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    t = block_sum(1, b, z);
  }
  if (threadIdx.x == 0) {
    const int filled = a.info->filled, tokens = a.info->tokens;
    const double per_token = tokens > 0 ? (double)f.beta / tokens : 0.;
    f.loss[0] = filled > 0 ? (float)((double)f.alpha * a.E / ((double)filled * a.k) * t.x) : 0.f;
    f.loss[1] = (float)(per_token * t.y);
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
  Row<Q> next;
  int at = t0;  // first of the G tokens at hand
  auto load = [&](int t) { load_logits<L, Q>(a.logits + (size_t)(t + group) * a.E, l, a.E, t + group < t1, next); };
  load(t0);
  const float cz = dloss * coef[a.S];
  SeqWalk walk;
  walk.begin(a, t0, t1);
  int done = t0;  // tokens before it are written
  auto outside = [&](int to) {  // tokens of no sequence have no gradient
    if (!accumulate)
      for (size_t i = (size_t)done * a.E + lane; i < (size_t)to * a.E; i += 64) dlogits[i] = 0.f;
  };
  int s, from, to;
  while (walk.next(a, t0, t1, s, from, to)) {
    Row<Q> up;
    const float cs = dloss * coef[s];
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = 4 * (l + L * q) + j;
        up.v[q][j] = e < a.E ? cs * (float)counts[(size_t)s * a.E + e] : 0.f;
      }
    outside(from);
    for (;;) {
      const int t = at + group;
      const Row<Q> x = next;
      const bool more = to > at + G;  // (otherwise these tokens may be another sequence's, too)
      if (more) load(at + G);
      if (t >= from && t < to) {
        Row<Q> soft, score, share;
        float lse, dot = 0.f;
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
      if (!more) break;
      at += G;
    }
    done = to;
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

// tokens of a wavefront: enough wavefronts for the chip, four tokens or its groups' at least
static int seq_chunk(int T, int E) {
  const int groups = E <= 4 ? 64 : E <= 8 ? 32 : E <= 16 ? 16 : E <= 32 ? 8 : E <= 64 ? 4 : E <= 128 ? 2 : 1;
  const int want = (T + MOE_KNOB("SEQ_WAVES", 4096) - 1) / MOE_KNOB("SEQ_WAVES", 4096), least = groups < 4 ? MOE_KNOB("SEQ_LEAST", 4) : groups;
  const int chunk = (want + groups - 1) / groups * groups;
  return chunk < least ? least : chunk > 256 ? 256 : chunk;
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
  const size_t Ep = align_up(s->E, 4);
  p.sums = align_up(sizeof(SeqInfo), 256);
  p.counts = p.sums + align_up(p.pieces * Ep * 4, 256);
  p.z = p.counts + align_up(p.pieces * Ep * 2, 256);
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
    const size_t lds = 4 * sizeof(int32_t) * align_up(shape->E, 4);
#define MOE_SEQ_SUMS(L, Q) hipLaunchKernelGGL((seq_sums_kernel<L, Q>), grid, block, lds, st, a, (int)(beta != 0.f), alpha * (float)shape->E, coef)
    MOE_BY_ROW(shape->E, MOE_SEQ_SUMS);
#undef MOE_SEQ_SUMS
  }
  {
    ProfScope prof("seq_finish_kernel", st);
    const int pieces = p.chunks / n_seqs;  // of an ordinary sequence
    const int waves = pieces > MOE_KNOB("SEQ_WIDE4", 32) ? 4 : 1;
    const int64_t jobs = (int64_t)n_seqs * ((shape->E + 15) / 16), blocks = waves > 1 ? jobs : (jobs + 3) / 4;
    const SeqFinish f = {a, alpha, beta, counts, P, loss, coef};
    const dim3 grid((unsigned)(blocks < kSeqBlocks ? blocks : kSeqBlocks)), block(256);
    if (waves == 4) hipLaunchKernelGGL(seq_finish_kernel<4>, grid, block, 0, st, f);
    else hipLaunchKernelGGL(seq_finish_kernel<1>, grid, block, 0, st, f);
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
