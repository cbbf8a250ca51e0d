// moe_seq_loss / moe_seq_loss_bwd: balance loss and expert counts of every sequence, z loss of the router, and their gradient.
//
//   sequence s owns tokens [start_s, start_s + len_s); T_s of them; S' sequences have any, T' is their sum
//   p_t = the gate's scores as shares of one;  P_se = (1 / T_s) sum_t p_te;  n_se = how often e was chosen;  f_se = n_se / (k T_s)
//   balance = alpha / S' sum_s E sum_e f_se P_se;   z = beta / T' sum_t lse_t^2, lse_t = log sum_e exp(logit_te)
//   dz_te = coef_s n_s. through the shares (the loads held constant) + coef_z lse_t softmax_te,  coef_s = alpha E / (S' k T_s^2),  coef_z = 2 beta / T'
//
// Tokens are cut into chunks of equal length, each a wavefront's or a block's, and chunks into the pieces that belong to one sequence.  Sequences ascend, so chunk c's
// piece of sequence s has the number c + s: along the tokens one of the two grows by one at every border, no two pieces share a number, and those of a
// sequence are neighbours.  The sums of a piece, of a sequence's pieces and of the loss are each added in a fixed order.
#include <initializer_list>

#include "rows.h"

namespace moe {

constexpr int kSeqBlocks = 1024, kSeqGroups = kSeqBlocks / 32;  // blocks of the second launch at most
constexpr int kSeqTotals = 16;                                  // blocks that count sequences and tokens, at most
struct SeqInfo {                      // start of the workspace
  int2 totals[kSeqTotals];            // S' and T', in parts
  uint32_t done[1 + kSeqGroups][16];  // blocks of the second launch that have ended, by groups of 32, and groups that have (a line of the cache each)
  float2 part[kSeqBlocks];            // their sums of the two losses
};
struct SeqArgs {
  const float* logits;
  const int32_t *topk, *start, *len;
  int T, E, k, gate, S, chunk, chunks, parts;
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
// the same place of all groups
template <int L> __device__ __forceinline__ float across_groups(float x) {
  if (L <= 1) x = add_lanes1(x);
  if (L <= 2) x = add_lanes2(x);
  if (L <= 4) x = add_quads(x);
  if (L == 8) x += dpp<0x128>(x);  // a rotation of sixteen by eight
  if (L <= 16) x = add_rows16(x);
  if (L <= 32) x = add_rows32(x);
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
// The exponentials are the instruction's, 2^(x log2 e): off by 1.5 |x| + 2 roundings, so a share e^-10 of the row's largest by 17, the largest by none.  (With
// expf and divisions 131072 tokens of 64 experts take 14.7 + 18.4 us for 11.1 + 15.0.)
// soft: softmax; share: the gate's; rest: what its sigmoid scores lack to 1; lse.  A row of -inf alone has shares and lse 0, one whose sigmoid scores are all 0 in fp32 shares of 0.  NaN in a row is in all of them.
template <int L, int Q>
__device__ __forceinline__ void gate_row(const Row<Q>& x, int l, int E, bool softmax, bool need_soft, Row<Q>& soft, Row<Q>& rest, Row<Q>& share, float& lse) {
  lse = 0.f;
  if (softmax || need_soft) {
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) m = fmaxf(m, x.v[q][j]);
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.f;  // nothing but -inf, whose sum is 0, and NaN, which the maximum passes over and the sum does not
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        soft.v[q][j] = __expf(x.v[q][j] - m);
        s += soft.v[q][j];
      }
    s = group_sum<L>(s);
    const bool empty = s == 0.f;  // (any other row's largest value adds 1)
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
  Row<Q> score;
#pragma unroll
  for (int q = 0; q < Q; q++)
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const bool in = 4 * (l + L * q) + j < E;
      const float e = __expf(-x.v[q][j]);
      score.v[q][j] = in ? __builtin_amdgcn_rcpf(1.f + e) : 0.f;
      rest.v[q][j] = e < 1.f ? e * score.v[q][j] : 1.f - score.v[q][j];  // (the difference has few bits left where the score is close to 1)
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
// The pieces of chunk c, by a team of W wavefronts, all of which see the same sequences.  lds: the team's, (1 + W) E words, E in fours; W > 1: the team is
// the block.
// The first tokens' loads go out before the search for the chunk's sequences, the next ones' before these are used.  (Four rows of a lane at once are no faster: there are
// other wavefronts; a chunk of fewer rows is, where tokens are few: 256 tokens of 8 experts 4.9 -> 2.9 us.)  Teams of four, because what the second launch has to read is a
// piece a chunk, and its few blocks read slowly (8192 tokens of 256 experts: 9.1 us behind chunks of a wavefront).
template <int L, int Q, int W>
__device__ __forceinline__ void chunk_sums(const SeqArgs& a, int c, int wave, int32_t* lds, bool want_z) {
  constexpr int G = 64 / L, GW = G * W;
  __shared__ float zsum[W];
  const int lane = threadIdx.x & 63, thread = W > 1 ? (int)threadIdx.x : lane;
  const int group = (W > 1 ? wave * G : 0) + lane / L, l = lane % L, Ep = (a.E + 3) & ~3;
  const int t0 = c * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const bool softmax = a.gate == MOE_GATE_SOFTMAX;
  int32_t* hist = lds;
  float* sums = reinterpret_cast<float*>(lds + Ep) + (W > 1 ? wave * Ep : 0);
  Row<Q> x, share, acc;
  float lse, z2 = 0.f;
  int ids;      // the first choices of the next tokens
  int id = -1;  // of these
  int at = t0;  // first of the GW tokens whose shares are at hand
  auto load = [&](int t) {
    load_logits<L, Q>(a.logits + (size_t)(t + group) * a.E, l, a.E, t + group < t1, x);
    const int64_t i = (int64_t)t * a.k + thread;
    ids = i < (int64_t)t1 * a.k ? a.topk[i] : -1;
  };
  auto use = [&]() {
    Row<Q> soft, rest;
    gate_row<L, Q>(x, l, a.E, softmax, want_z, soft, rest, share, lse);
    id = ids;
    if (at + GW < t1) load(at + GW);
  };
  auto together = [&]() {
    if (W > 1) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  load(t0);
  for (int e = thread; e < Ep; e += 64 * W) hist[e] = 0;
  SeqWalk walk;
  walk.begin(a, t0, t1);
  use();
  int s, from, to;
  together();
  while (walk.next(a, t0, t1, s, from, to)) {
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) acc.v[q][j] = 0.f;
    z2 = 0.f;
    for (;;) {
      // how often each expert was chosen: whole numbers, so the order of the additions plays no part
      const int64_t lo = (int64_t)max(from, at) * a.k, hi = (int64_t)min(to, at + GW) * a.k;
      int64_t i = (int64_t)at * a.k + thread;
      if (i >= lo && i < hi && (unsigned)id < (unsigned)a.E) atomicAdd(&hist[id], 1);
      for (i += 64 * W; i < hi; i += 64 * W)
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
      if (to <= at + GW) break;
      at += GW;
      use();
    }
    z2 = across_groups<L>(z2);
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) acc.v[q][j] = across_groups<L>(acc.v[q][j]);
    const size_t piece = (size_t)c + s;
    if (W > 1) {
      if (lane < L) {
#pragma unroll
        for (int q = 0; q < Q; q++)
          if (4 * (l + L * q) < Ep)
            *reinterpret_cast<float4*>(sums + 4 * (l + L * q)) = make_float4(acc.v[q][0], acc.v[q][1], acc.v[q][2], acc.v[q][3]);
        if (lane == 0) zsum[wave] = z2;
      }
      together();
      // the team's sums, wavefront after wavefront
      for (int e = 4 * thread; e < Ep; e += 256 * W) {
        const float* all = reinterpret_cast<const float*>(lds + Ep) + e;
        float4 v = *reinterpret_cast<const float4*>(all);
#pragma unroll
        for (int w = 1; w < W; w++) {
          const float4 o = *reinterpret_cast<const float4*>(all + w * Ep);
          v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        *reinterpret_cast<float4*>(a.psum + piece * Ep + e) = v;
      }
      if (thread == 0) {
        float z = zsum[0];
#pragma unroll
        for (int w = 1; w < W; w++) z += zsum[w];
        a.pz[piece] = z;
      }
    } else {
      together();
      if (lane == 0) a.pz[piece] = z2;
      if (lane < L) {
#pragma unroll
        for (int q = 0; q < Q; q++)
          if (4 * (l + L * q) < Ep)
            *reinterpret_cast<float4*>(a.psum + piece * Ep + 4 * (l + L * q)) = make_float4(acc.v[q][0], acc.v[q][1], acc.v[q][2], acc.v[q][3]);
      }
    }
    for (int e = 4 * thread; e < Ep; e += 256 * W) {
      const int4 n = *reinterpret_cast<const int4*>(hist + e);
      *reinterpret_cast<uint2*>(a.pcount + piece * Ep + e) = make_uint2((uint32_t)n.x | (uint32_t)n.y << 16, (uint32_t)n.z | (uint32_t)n.w << 16);
      *reinterpret_cast<int4*>(hist + e) = make_int4(0, 0, 0, 0);
    }
    together();
  }
}
// How many of the sequences of part `part` of `parts` have tokens, and how many tokens they have (x, y), by a block of W wavefronts; one barrier.
template <int W>
__device__ __forceinline__ int2 seq_totals(const SeqArgs& a, int part, int parts) {
  __shared__ int2 of_wave[W];
  int filled = 0, tokens = 0;
#pragma unroll 8
  for (int s = part * 64 * W + (int)threadIdx.x; s < a.S; s += parts * 64 * W) {
    const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
    filled += r.y > r.x;
    tokens += r.y - r.x;
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    filled += __shfl_xor(filled, m, kWave);
    tokens += __shfl_xor(tokens, m, kWave);
  }
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = make_int2(filled, tokens);
  __syncthreads();
  filled = tokens = 0;
#pragma unroll
  for (int w = 0; w < W; w++) {
    filled += of_wave[w].x;
    tokens += of_wave[w].y;
  }
  return make_int2(filled, tokens);
}

// P and counts of every sequence, and the losses.  A job is 16 experts of a sequence: four lanes side by side.
struct SeqFinish {
  SeqArgs a;
  float alpha, beta;
  int32_t* counts;
  float *P, *loss, *coef;
};
struct Job {
  int s, e, n;     // sequence, the lane's first expert, tokens
  int64_t p0, p1;  // pieces
  float sum[4];
  int count[4];
  __device__ __forceinline__ Job(const SeqArgs& a, int64_t job, int64_t jobs, int lane) {
    const int tiles = (a.E + 15) / 16;
    const bool there = job < jobs;
    s = there ? (int)(job / tiles) : 0;
    e = there ? (int)(job - (int64_t)s * tiles) * 16 + 4 * (lane & 3) : 1 << 30;
    const int2 r = seq_range(a.start, a.len, a.S, a.T, s);
    n = r.y - r.x;
    p0 = there && n ? (int64_t)(r.x / a.chunk) + s : 0;
    p1 = there && n ? (int64_t)((r.y - 1) / a.chunk) + s + 1 : 0;
#pragma unroll
    for (int j = 0; j < 4; j++) sum[j] = 0.f, count[j] = 0;
  }
  // pieces first, first + step, ..: U of a lane in flight
  template <int U>
  __device__ __forceinline__ void add(const SeqArgs& a, int64_t first, int step) {
    const int Ep = (a.E + 3) & ~3;
    if (e >= Ep) return;
    for (int64_t p = first; p < p1; p += U * step) {
      float4 v[U];
      uint2 m[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int64_t at = (p + u * step < p1 ? p + u * step : p) * Ep + e;
        v[u] = *reinterpret_cast<const float4*>(a.psum + at);
        m[u] = *reinterpret_cast<const uint2*>(a.pcount + at);
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (p + u * step >= p1) break;
        sum[0] += v[u].x; sum[1] += v[u].y; sum[2] += v[u].z; sum[3] += v[u].w;
        count[0] += m[u].x & 0xffff; count[1] += m[u].x >> 16; count[2] += m[u].y & 0xffff; count[3] += m[u].y >> 16;
      }
    }
  }
  // over the lanes whose numbers differ by a multiple of four
  __device__ __forceinline__ void over_lanes() {
#pragma unroll
    for (int j = 0; j < 4; j++) {
      sum[j] = add_rows32(add_rows16(add_quads(sum[j])));
      count[j] = add_rows32(add_rows16(add_quads(count[j])));
    }
  }
  // writes P, counts and the sequence's factor; the lane's part of sum_e count * P / tokens
  __device__ __forceinline__ float write(const SeqFinish& f, int filled) const {
    float b = 0.f;
    if (e == 0) f.coef[s] = n ? f.alpha * (float)f.a.E / (float)filled / (float)f.a.k / (float)n / (float)n : 0.f;
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (e + j < f.a.E) {
        const float share = n ? sum[j] / (float)n : 0.f;
        f.P[(size_t)s * f.a.E + e + j] = share;
        f.counts[(size_t)s * f.a.E + e + j] = count[j];
        b = fmaf(share, (float)count[j], b);
      }
    return n ? b / (float)n : 0.f;
  }
};
// The thread's sums over the jobs of wavefront `first` of `step`: of count * P / tokens, and of lse^2.  A job is a wavefront's, or (SHORT) four lanes', but for those of
// many pieces, which then follow one after the other.
template <bool SHORT>
__device__ __forceinline__ float2 finish_jobs(const SeqFinish& f, int filled, int64_t first, int64_t step) {
  const SeqArgs& a = f.a;
  const int lane = threadIdx.x & 63;
  const int64_t jobs = (int64_t)a.S * ((a.E + 15) / 16);
  float balance = 0.f, z2 = 0.f;
  auto by_all = [&](int64_t job) {
    Job all(a, job, jobs, lane);
    all.add<4>(a, all.p0 + (lane >> 2), 16);
    if (all.e < 16 && f.beta != 0.f)
      for (int64_t p = all.p0 + lane; p < all.p1; p += 64) z2 += a.pz[p];
    all.over_lanes();
    if (lane < 4) balance += all.write(f, filled);
  };
  if (!SHORT) {
    for (int64_t job = first; job < jobs; job += step) by_all(job);
    return make_float2(balance, z2);
  }
  for (int64_t w = first; w * 16 < jobs; w += step) {
    Job mine(a, w * 16 + (lane >> 2), jobs, lane);
    const bool many = mine.p1 - mine.p0 > 16;
    if (!many) {
      mine.add<4>(a, mine.p0, 1);
      if (mine.e == 0 && f.beta != 0.f)
        for (int64_t p = mine.p0; p < mine.p1; p++) z2 += a.pz[p];
      if (mine.e < a.E) balance += mine.write(f, filled);
    }
    uint64_t left = __ballot(many && (lane & 3) == 0);
    while (left) {
      const int q = (__ffsll((unsigned long long)left) - 1) >> 2;
      left &= left - 1;
      by_all(w * 16 + q);
    }
  }
  return make_float2(balance, z2);
}
// The same for sequences of many pieces each: a job is a block's, of four wavefronts.
__device__ __forceinline__ float2 finish_long_jobs(const SeqFinish& f, int filled) {
  __shared__ float4 psum[4][4];
  __shared__ int4 pcount[4][4];
  const SeqArgs& a = f.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t jobs = (int64_t)a.S * ((a.E + 15) / 16);
  float balance = 0.f, z2 = 0.f;
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    Job all(a, job, jobs, lane);
    all.add<8>(a, all.p0 + (threadIdx.x >> 2), 64);
    if (all.e < 16 && f.beta != 0.f)
      for (int64_t p = all.p0 + threadIdx.x; p < all.p1; p += 256) z2 += a.pz[p];
    all.over_lanes();
    if (lane < 4) {
      psum[wave][lane] = make_float4(all.sum[0], all.sum[1], all.sum[2], all.sum[3]);
      pcount[wave][lane] = make_int4(all.count[0], all.count[1], all.count[2], all.count[3]);
    }
    __syncthreads();
    if (threadIdx.x < 4) {
#pragma unroll
      for (int w = 1; w < 4; w++) {
        const float4 v = psum[w][lane];
        const int4 m = pcount[w][lane];
        all.sum[0] += v.x; all.sum[1] += v.y; all.sum[2] += v.z; all.sum[3] += v.w;
        all.count[0] += m.x; all.count[1] += m.y; all.count[2] += m.z; all.count[3] += m.w;
      }
      balance += all.write(f, filled);
    }
    __syncthreads();
  }
  return make_float2(balance, z2);
}
// the sum over a block of W wavefronts; one barrier
template <int W>
__device__ __forceinline__ double2 finish_sum(float2 v, float2 (&part)[W]) {
  v.x = lanes_sum(v.x);
  v.y = lanes_sum(v.y);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  double2 t = {0., 0.};
#pragma unroll
  for (int w = 0; w < W; w++) {
    t.x += part[w].x;
    t.y += part[w].y;
  }
  return t;
}
__device__ __forceinline__ void write_losses(const SeqFinish& f, int filled, int tokens, double2 t) {
  const double per_token = tokens > 0 ? (double)f.beta / tokens : 0.;
  f.loss[0] = filled > 0 ? (float)((double)f.alpha * f.a.E / ((double)filled * f.a.k) * t.x) : 0.f;
  f.loss[1] = (float)(per_token * t.y);
  f.coef[f.a.S] = (float)(2. * per_token);
}

template <int L, int Q, int W>
__global__ __launch_bounds__(256) void seq_sums_kernel(SeqArgs a, int want_z) {
  extern __shared__ int32_t lds[];  // [W > 1 ? 1 + W : 4][E, in fours]
  const int part = (int)blockIdx.x - ((int)gridDim.x - a.parts);
  if (part >= 0) {  // the last blocks: what all sequences share
    const int2 t = seq_totals<4>(a, part, a.parts);
    if (threadIdx.x == 0) a.info->totals[part] = t;
    if (part == 0 && threadIdx.x <= kSeqGroups) a.info->done[threadIdx.x][0] = 0;
    return;
  }
  const int wave = threadIdx.x >> 6;
  if (W > 1) {
    chunk_sums<L, Q, 4>(a, blockIdx.x, wave, lds, want_z);
  } else {
    const int c = blockIdx.x * 4 + wave;
    if (c < a.chunks) chunk_sums<L, Q, 1>(a, c, wave, lds + wave * ((a.E + 3) & ~3), want_z);
  }
}

enum { kShort = 0, kOrdinary = 1, kLong = 2 };  // pieces of a sequence
template <int LENGTH>
__global__ __launch_bounds__(256) void seq_finish_kernel(SeqFinish f) {
  const SeqArgs& a = f.a;
  __shared__ float2 part[2][4];
  __shared__ int last;
  int2 totals = {0, 0};
  for (int p = 0; p < a.parts; p++) {
    totals.x += a.info->totals[p].x;
    totals.y += a.info->totals[p].y;
  }
  const float2 mine = LENGTH == kLong ? finish_long_jobs(f, totals.x)
                                      : finish_jobs<LENGTH == kShort>(f, totals.x, (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), (int64_t)gridDim.x * 4);
  // The block's sums, then, in the block that ends last, those of all blocks.  Sums and counters go past the caches that other dies do not see (atomics of the agent's scope), and
  // a counter only after the sums have arrived (the wait): releasing and acquiring would write back and drop whole caches for these 8 bytes.  (Counters by groups: a
  // thousand additions to one place take 15 us.)
  double2 t = finish_sum<4>(mine, part[0]);
  if (gridDim.x > 1) {
    if (threadIdx.x == 0) {
      __hip_atomic_store(&a.info->part[blockIdx.x].x, (float)t.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&a.info->part[blockIdx.x].y, (float)t.y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const uint32_t groups = (gridDim.x + 31) / 32, group = blockIdx.x % groups, members = (gridDim.x - group + groups - 1) / groups;
      last = __hip_atomic_fetch_add(&a.info->done[1 + group][0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1 &&
             __hip_atomic_fetch_add(&a.info->done[0][0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
    }
    __syncthreads();
    if (!last) return;
    float2 v = {0.f, 0.f};
#pragma unroll 4
    for (int q = threadIdx.x; q < (int)gridDim.x; q += 256) {
      v.x += __hip_atomic_load(&a.info->part[q].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      v.y += __hip_atomic_load(&a.info->part[q].y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    t = finish_sum<4>(v, part[1]);
  }
  if (threadIdx.x == 0) write_losses(f, totals.x, totals.y, t);
}

// Both steps in one block, for calls that are over before a second launch would begin.  Its wavefronts leave their pieces in the workspace, too; only their counters of choices
// are in LDS.
template <int L, int Q>
__global__ __launch_bounds__(1024) void seq_small_kernel(SeqFinish f) {
  extern __shared__ int32_t lds[];  // [chunks, up to 16][E, in fours]
  __shared__ float2 part[16];
  const SeqArgs& a = f.a;
  const int wave = threadIdx.x >> 6;
  for (int c = wave; c < a.chunks; c += 16) chunk_sums<L, Q, 1>(a, c, wave, lds + wave * ((a.E + 3) & ~3), f.beta != 0.f);
  const int2 t = seq_totals<16>(a, 0, 1);
  __syncthreads();  // the pieces are there
  const bool few = a.S * ((a.E + 15) / 16) <= 16;  // jobs
  const double2 sums = finish_sum<16>(few ? finish_jobs<false>(f, t.x, wave, 16) : finish_jobs<true>(f, t.x, wave, 16), part);
  if (threadIdx.x == 0) write_losses(f, t.x, t.y, sums);
}

// A wavefront writes down whose each of its tokens is, then goes through them, each lane's group with a token of its own; the loads of the next step's logits, and of its
// sequences' counts where they are others, are under way meanwhile.  (Sequence by sequence, the counts' latency shows at every border: 64 sequences of four tokens 11.5 us.)
template <int L, int Q>
__global__ __launch_bounds__(256) void seq_bwd_kernel(SeqArgs a, const int32_t* __restrict__ counts, const float* __restrict__ coef, float dloss,
                                                      int accumulate, float* dlogits) {
  extern __shared__ int32_t lds[];  // [4][chunk]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 4 + wave;
  if (c >= a.chunks) return;
  constexpr int G = 64 / L;
  const int group = lane / L, l = lane % L;
  const int t0 = c * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const bool softmax = a.gate == MOE_GATE_SOFTMAX;
  Row<Q> next_x;
  auto load = [&](int t) { load_logits<L, Q>(a.logits + (size_t)(t + group) * a.E, l, a.E, t + group < t1, next_x); };
  load(t0);
  const float cz = dloss * coef[a.S];
  SeqWalk walk;
  walk.begin(a, t0, t1);
  int32_t* owner = lds + wave * a.chunk;
  for (int i = lane; i < t1 - t0; i += 64) owner[i] = -1;
  int s, from, to;
  while (walk.next(a, t0, t1, s, from, to))
    for (int t = from + lane; t < to; t += 64) owner[t - t0] = s;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  Row<Q> up;
  int32_t next_up[Q][4];
  float next_c = 0.f;
  int now = -1, next = -1;  // the token's sequence; -1: none
  bool other;               // the next step has another one in some group
  auto load_counts = [&](int t) {
    next = t + group < t1 ? owner[t + group - t0] : -1;
    other = __any(next != now && next >= 0);
    if (!other) return;
    const int at = max(next, 0);
    next_c = coef[at];
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = 4 * (l + L * q) + j;
        next_up[q][j] = e < a.E ? counts[(size_t)at * a.E + e] : 0;
      }
  };
  load_counts(t0);
  for (int t = t0; t < t1; t += G) {
    const Row<Q> x = next_x;
    if (other) {
      const float cs = dloss * next_c;
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) up.v[q][j] = cs * (float)next_up[q][j];
    }
    now = next;
    const int mine = t + group;
    if (t + G < t1) {
      load(t + G);
      load_counts(t + G);
    }
    if (mine >= t1 || (now < 0 && accumulate)) continue;
    Row<Q> dz;  // tokens of no sequence have no gradient
#pragma unroll
    for (int q = 0; q < Q; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) dz.v[q][j] = 0.f;
    if (now >= 0) {
      Row<Q> soft, rest, share;
      float lse, dot = 0.f;
      gate_row<L, Q>(x, l, a.E, softmax, cz != 0.f, soft, rest, share, lse);
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) dot = fmaf(share.v[q][j], up.v[q][j], dot);
      dot = group_sum<L>(dot);
      const float zl = cz * lse;
#pragma unroll
      for (int q = 0; q < Q; q++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
          dz.v[q][j] = share.v[q][j] * (up.v[q][j] - dot);
          if (!softmax) dz.v[q][j] *= rest.v[q][j];
          if (cz != 0.f) dz.v[q][j] = fmaf(zl, soft.v[q][j], dz.v[q][j]);
        }
    }
#pragma unroll
    for (int q = 0; q < Q; q++) {
      const int e = 4 * (l + L * q);
      float* o = dlogits + (size_t)mine * a.E + e;
      if (e + 4 <= a.E) {
        if (accumulate) {
          float old[4];
          __builtin_memcpy(old, o, 16);
#pragma unroll
          for (int j = 0; j < 4; j++) dz.v[q][j] += old[j];
        }
        __builtin_memcpy(o, dz.v[q], 16);
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++)
          if (e + j < a.E) o[j] = accumulate ? o[j] + dz.v[q][j] : dz.v[q][j];
      }
    }
  }
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

// Tokens of a team, whole steps of it (64 lanes of a wavefront over a row's lanes): enough teams for the chip.  Teams that leave pieces for the second launch are half as many where
// they would have less than four steps each (8192 tokens of 256 experts: 512 teams 5.8 + 6.3 us, 1024 5.5 + 7.6).
static int seq_step(int E) { return E <= 4 ? 64 : E <= 8 ? 32 : E <= 16 ? 16 : E <= 32 ? 8 : E <= 64 ? 4 : E <= 128 ? 2 : 1; }
static int seq_chunk(int T, int step, int teams) {
  const int want = (T + teams - 1) / teams, chunk = (want + step - 1) / step * step;
  return chunk < step ? step : chunk > 512 ? 512 : chunk;
}
struct SeqPlan {
  bool small;  // one block, one launch
  bool team;   // chunks are a block's, not a wavefront's
  int chunk, chunks;
  size_t pieces, sums, counts, z, bytes;  // places of the workspace
};
static SeqPlan seq_plan(const moe_shape_t* s, int n_seqs, bool backward) {
  SeqPlan p;
  p.small = !backward && (int64_t)s->T * s->E <= 16384 && (int64_t)n_seqs * ((s->E + 15) / 16) <= 64;
  const int step = seq_step(s->E);
  p.team = !p.small && !backward && s->T >= (int64_t)n_seqs * 8 * step;  // (a team meets at every border of two sequences)
  p.chunk = p.small ? seq_chunk(s->T, step, s->E > 512 ? 8 : 16) : p.team ? seq_chunk(s->T, 4 * step, s->T < 1024 * 16 * step ? 512 : 1024) : seq_chunk(s->T, step, 4096);
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
  if (shape->T > INT32_MAX - (1 << 16)) {  // (the end of the last chunk is an index, too)
    set_error("%s: T=%d overflows the index range", who, shape->T);
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
  if (!shape || shape->T < 0 || shape->T > INT32_MAX - (1 << 16) || shape->E < 1 || shape->E > MOE_MAX_EXPERTS || n_seqs < 1) return 0;
  return moe::seq_plan(shape, n_seqs, false).bytes;
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
  const SeqPlan p = seq_plan(shape, n_seqs, false);
  if (ws_bytes < p.bytes) {
    set_error("moe_seq_loss: workspace of %zu bytes, need %zu", ws_bytes, p.bytes);
    return MOE_EWS;
  }
  hipStream_t st = (hipStream_t)stream;
  char* w = (char*)ws;
  const int parts = n_seqs < 2048 * kSeqTotals ? (n_seqs + 2047) / 2048 : kSeqTotals;
  const SeqArgs a = {logits, topk_idx, seq_start, seq_len, shape->T, shape->E, shape->k, shape->gate, n_seqs, p.chunk, p.chunks, parts,
                     (float*)(w + p.sums), (uint16_t*)(w + p.counts), (float*)(w + p.z), (SeqInfo*)w};
  const SeqFinish f = {a, alpha, beta, counts, P, loss, coef};
  const int64_t jobs = (int64_t)n_seqs * ((shape->E + 15) / 16);
  const size_t hist = sizeof(int32_t) * align_up(shape->E, 4);
  if (p.small) {  // (32 KB of LDS at most)
    ProfScope prof("seq_small_kernel", st);
#define MOE_SEQ_SMALL(L, Q) hipLaunchKernelGGL((seq_small_kernel<L, Q>), dim3(1), dim3(1024), (size_t)(p.chunks < 16 ? p.chunks : 16) * hist, st, f)
    MOE_BY_ROW(shape->E, MOE_SEQ_SMALL);
#undef MOE_SEQ_SMALL
    return launch_status("moe_seq_loss");
  }
  {
    ProfScope prof("seq_sums_kernel", st);
    const dim3 grid((p.team ? p.chunks : (p.chunks + 3) / 4) + parts), block(256);
#define MOE_SEQ_SUMS(L, Q)                                                                                                                        \
  do {                                                                                                                                            \
    if (p.team) hipLaunchKernelGGL((seq_sums_kernel<L, Q, 4>), grid, block, 5 * hist, st, a, (int)(beta != 0.f));                  \
    else hipLaunchKernelGGL((seq_sums_kernel<L, Q, 1>), grid, block, 4 * hist, st, a, (int)(beta != 0.f));                         \
  } while (0)
    MOE_BY_ROW(shape->E, MOE_SEQ_SUMS);
#undef MOE_SEQ_SUMS
  }
  {
    ProfScope prof("seq_finish_kernel", st);
    const int pieces = p.chunks / n_seqs;  // of an ordinary sequence
    const int64_t blocks = pieces > 32 ? jobs : pieces > 4 || jobs <= 256 ? (jobs + 3) / 4 : (jobs + 63) / 64;
    const dim3 grid((unsigned)(blocks < kSeqBlocks ? blocks : kSeqBlocks)), block(256);
    if (pieces > 32) hipLaunchKernelGGL(seq_finish_kernel<kLong>, grid, block, 0, st, f);
    else if (pieces > 4 || jobs <= 256) hipLaunchKernelGGL(seq_finish_kernel<kOrdinary>, grid, block, 0, st, f);
    else hipLaunchKernelGGL(seq_finish_kernel<kShort>, grid, block, 0, st, f);
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
  const SeqPlan p = seq_plan(shape, n_seqs, true);
  const SeqArgs a = {logits, nullptr, seq_start, seq_len, shape->T, shape->E, shape->k, shape->gate, n_seqs, p.chunk, p.chunks, 0, nullptr, nullptr, nullptr, nullptr};
  hipStream_t st = (hipStream_t)stream;
  ProfScope prof("seq_bwd_kernel", st);
  const dim3 grid((p.chunks + 3) / 4), block(256);
#define MOE_SEQ_BWD(L, Q) hipLaunchKernelGGL((seq_bwd_kernel<L, Q>), grid, block, 4 * sizeof(int32_t) * p.chunk, st, a, counts, coef, dloss, (int)accumulate, dlogits)
  MOE_BY_ROW(shape->E, MOE_SEQ_BWD);
#undef MOE_SEQ_BWD
  return launch_status("moe_seq_loss_bwd");
}
