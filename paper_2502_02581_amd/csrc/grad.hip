// moe_grad_norm / moe_grad_clip: the global norm of a layer's (or a model's) gradients and their clipping.
//
// The weight gradients of routed experts are compacted: n_active slots, a number that only the GPU knows.  Both calls read it there, so a
// training step has no synchronisation between its backward pass and its optimiser, and slots that no expert used are
// neither read nor written.
#include <algorithm>
#include <memory>
#include <new>

#include "moe_common.h"

namespace moe {

// Both passes are bound by HBM: two layers of 60 experts, d = 2048, d_ff = 1408, 2.06 GB of gradients: norm 367 + 5 us (5.6 TB/s read), clipping 774 us (5.3 TB/s
// read and written).  Many small tensors cost a launch each way and nothing else: 32 of 4 KB to 1 MB, 7 + 3 + 9 us.
//
// Tensors are cut into chunks of kChunk values, numbered through all tensors of a launch; blocks take them in turn.
constexpr int kChunk = 16384, kGradThreads = 256, kGradBlocks = 2048, kGradsPerLaunch = 48;
struct GradList {
  const void* g[kGradsPerLaunch];
  void* out[kGradsPerLaunch];
  const int32_t* n_active[kGradsPerLaunch];
  int64_t n[kGradsPerLaunch], slot[kGradsPerLaunch];
  uint32_t first[kGradsPerLaunch + 1];  // first chunk of every tensor, then their number
  uint64_t f32;                         // bit i: tensor i is fp32
  int32_t count;
};
// the tensor of chunk c, and the values [from, to) of it that the chunk covers (none: from >= to)
struct Chunk {
  int t;
  int64_t from, to;
};
__device__ __forceinline__ Chunk find_chunk(const GradList& l, uint32_t c) {
  int lo = 0, hi = l.count;  // the last tensor that starts at or before c (uniform over the block)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= c) lo = mid;
    else hi = mid;
  }
  int64_t n = l.n[lo];
  if (l.n_active[lo]) n = min(n, max((int64_t)*l.n_active[lo], (int64_t)0) * l.slot[lo]);
  const int64_t from = (int64_t)(c - l.first[lo]) * kChunk;
  return {lo, from, min(from + kChunk, n)};
}

// Squares are summed in 64 bits: the sum has no overflow or underflow for any finite gradient (its root may be beyond fp32's range), and an error that is far below the result's rounding
// whatever the number of values.  A lane has eight loads of 16 bytes in flight and four sums; its partial sum, the block's and those of the blocks are added in a
// fixed order, so two calls give the same bits.
template <typename T>
__device__ __forceinline__ double chunk_squares(const T* g, int64_t from, int64_t to) {
  constexpr int N = Vec16<T>::N, U = 8;
  double t[4] = {};
  int64_t i = from + (int64_t)threadIdx.x * N;
  for (; i + (int64_t)(U - 1) * kGradThreads * N + N <= to; i += (int64_t)U * kGradThreads * N) {
    float v[U][N];
#pragma unroll
    for (int u = 0; u < U; u++) Vec16<T>::load(g + i + (int64_t)u * kGradThreads * N, v[u]);
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int j = 0; j < N; j++) t[j & 3] = fma((double)v[u][j], (double)v[u][j], t[j & 3]);
  }
  double s = (t[0] + t[1]) + (t[2] + t[3]);
  for (; i < to; i += (int64_t)kGradThreads * N)
    for (int j = 0; j < N && i + j < to; j++) {
      const double x = Elem<T>::load(g + i + j);
      s = fma(x, x, s);
    }
  return s;
}
__device__ __forceinline__ double block_sum(double s, double* part) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, kWave);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}
__global__ __launch_bounds__(kGradThreads) void grad_squares_kernel(GradList l, double* partial, int add) {
  __shared__ double part[4];
  double s = 0;
  for (uint32_t c = blockIdx.x; c < l.first[l.count]; c += gridDim.x) {
    const Chunk k = find_chunk(l, c);
    if (k.from >= k.to) continue;
    if (l.f32 >> k.t & 1) s += chunk_squares((const float*)l.g[k.t], k.from, k.to);
    else s += chunk_squares((const bf16_t*)l.g[k.t], k.from, k.to);
  }
  s = block_sum(s, part);
  if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + s : s;
}
__global__ __launch_bounds__(kGradThreads) void grad_norm_kernel(const double* partial, float* norm) {
  __shared__ double part[4];
  double s = 0;
  for (int i = threadIdx.x; i < kGradBlocks; i += kGradThreads) s += partial[i];
  s = block_sum(s, part);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* out, int64_t from, int64_t to, float f) {
  constexpr int N = Vec16<T>::N, U = 4;
  int64_t i = from + (int64_t)threadIdx.x * N;
  for (; i + (int64_t)(U - 1) * kGradThreads * N + N <= to; i += (int64_t)U * kGradThreads * N) {
    float v[U][N];
#pragma unroll
    for (int u = 0; u < U; u++) Vec16<T>::load(g + i + (int64_t)u * kGradThreads * N, v[u]);
#pragma unroll
    for (int u = 0; u < U; u++) {
#pragma unroll
      for (int j = 0; j < N; j++) v[u][j] *= f;
      Vec16<T>::store(out + i + (int64_t)u * kGradThreads * N, v[u]);
    }
  }
  for (; i < to; i += (int64_t)kGradThreads * N)
    for (int j = 0; j < N && i + j < to; j++) Elem<T>::store(out + i + j, Elem<T>::load(g + i + j) * f);
}
__global__ __launch_bounds__(kGradThreads) void grad_scale_kernel(GradList l, const float* norm, float max_norm) {
  // (a norm that is NaN makes the factor NaN, so that it is seen in the gradients, too)
  const double f0 = (double)max_norm / ((double)*norm + 1e-6);
  const float f = f0 >= 1. ? 1.f : (float)f0;
  // The last chunks first: the norm's pass has left them in the memory-side cache.
  const uint32_t n = l.first[l.count];
  for (uint32_t c = blockIdx.x; c < n; c += gridDim.x) {
    const Chunk k = find_chunk(l, n - 1 - c);
    if (k.from >= k.to || (f == 1.f && l.g[k.t] == l.out[k.t])) continue;
    if (l.f32 >> k.t & 1) chunk_scale((const float*)l.g[k.t], (float*)l.out[k.t], k.from, k.to, f);
    else chunk_scale((const bf16_t*)l.g[k.t], (bf16_t*)l.out[k.t], k.from, k.to, f);
  }
}

static int check_grads(const moe_grad_t* grads, int n, bool out, const char* who) {
  if (n < 0 || (n > 0 && !grads)) {
    set_error("%s: bad list of %d gradients", who, n);
    return MOE_EINVAL;
  }
  uint64_t chunks = 0;
  for (int i = 0; i < n; i++) {
    const moe_grad_t& g = grads[i];
    if (g.dtype != MOE_F32 && g.dtype != MOE_BF16) {
      set_error("%s: gradient %d: unknown dtype %d", who, i, g.dtype);
      return MOE_EDTYPE;
    }
    if (g.n < 0 || g.n >= (int64_t)1 << 40 || (g.n > 0 && (!g.g || (out && !g.out))) || (g.n_active && g.slot < 1) || g.slot >= (int64_t)1 << 31) {
      set_error("%s: gradient %d: null pointer or bad size (%lld values, slots of %lld)", who, i, (long long)g.n, (long long)g.slot);
      return MOE_EINVAL;
    }
    if (!aligned16(g.g) || (out && !aligned16(g.out)) || (uintptr_t)g.n_active % 4) {
      set_error("%s: gradient %d: every tensor must be 16-byte aligned", who, i);
      return MOE_EINVAL;
    }
    chunks += (uint64_t)((g.n + kChunk - 1) / kChunk);
  }
  if (chunks >= (uint64_t)1 << 31) {
    set_error("%s: too many values", who);
    return MOE_EINVAL;
  }
  return MOE_OK;
}
// What is written must not overlap anything else that is read or written: chunks are scaled in no order.  Tensors by address; each against the furthest end of
// those before it (96 tensors and as many outputs: 3 us).
static int check_outputs(const moe_grad_t* grads, int n, const char* who) {
  struct Span {
    uintptr_t from, to;
    int i;
    bool out;
  };
  std::unique_ptr<Span[]> spans(new (std::nothrow) Span[2 * (size_t)n]);
  if (!spans) {
    set_error("%s: no host memory for a list of %d gradients", who, n);
    return MOE_EINVAL;
  }
  size_t m = 0;
  for (int i = 0; i < n; i++) {
    const moe_grad_t& g = grads[i];
    if (g.n == 0) continue;
    const size_t bytes = (size_t)g.n * elem_size(g.dtype);
    spans[m++] = {(uintptr_t)g.out, (uintptr_t)g.out + bytes, i, true};
    if (g.g != g.out) spans[m++] = {(uintptr_t)g.g, (uintptr_t)g.g + bytes, i, false};
  }
  std::sort(spans.get(), spans.get() + m, [](const Span& a, const Span& b) { return a.from < b.from; });
  const Span *in = nullptr, *out = nullptr;  // those that reach furthest so far
  for (size_t k = 0; k < m; k++) {
    const Span& s = spans[k];
    const Span* hit = out && s.from < out->to ? out : s.out && in && s.from < in->to ? in : nullptr;
    if (hit && hit->out && s.out) {
      set_error("%s: outputs %d and %d overlap (a tensor is there twice)", who, hit->i, s.i);
      return MOE_EINVAL;
    }
    if (hit) {
      const Span &o = s.out ? s : *hit, &g = s.out ? *hit : s;
      set_error(o.i == g.i ? "%s: output %d overlaps its gradient (%d) without being it" : "%s: output %d is another gradient (%d), or overlaps it", who, o.i, g.i);
      return MOE_EINVAL;
    }
    const Span*& far = s.out ? out : in;
    if (!far || s.to > far->to) far = &s;
  }
  return MOE_OK;
}
// tensors [from, ..) of a launch; returns the first one behind it
static int fill_list(GradList& l, const moe_grad_t* grads, int n, int from) {
  l = {};
  int i = from;
  for (; i < n && l.count < kGradsPerLaunch; i++) {
    const moe_grad_t& g = grads[i];
    if (g.n == 0) continue;
    const int k = l.count++;
    l.g[k] = g.g; l.out[k] = g.out; l.n[k] = g.n; l.n_active[k] = g.n_active; l.slot[k] = g.slot;
    l.f32 |= (uint64_t)(g.dtype == MOE_F32) << k;
    l.first[k + 1] = l.first[k] + (uint32_t)((g.n + kChunk - 1) / kChunk);
  }
  return i;
}

}  // namespace moe

extern "C" size_t moe_grad_norm_workspace_bytes(void) { return moe::kGradBlocks * sizeof(double); }

extern "C" int moe_grad_norm(const moe_grad_t* grads, int32_t n, float* norm, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  const int rc = check_grads(grads, n, false, "moe_grad_norm");
  if (rc) return rc;
  if (!norm || !ws || !aligned16(ws) || (uintptr_t)norm % 4) {
    set_error("moe_grad_norm: null pointer or workspace not 16-byte aligned");
    return MOE_EINVAL;
  }
  if (ws_bytes < moe_grad_norm_workspace_bytes()) {
    set_error("moe_grad_norm: workspace of %zu bytes, need %zu", ws_bytes, moe_grad_norm_workspace_bytes());
    return MOE_EWS;
  }
  hipStream_t st = (hipStream_t)stream;
  int i = 0, add = 0;
  do {  // (also without gradients: the partial sums are written)
    GradList l;
    i = fill_list(l, grads, n, i);
    ProfScope prof("grad_squares_kernel", st);
    hipLaunchKernelGGL(grad_squares_kernel, dim3(kGradBlocks), dim3(kGradThreads), 0, st, l, (double*)ws, add);
    add = 1;
  } while (i < n);
  {
    ProfScope prof("grad_norm_kernel", st);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kGradThreads), 0, st, (const double*)ws, norm);
  }
  return launch_status("moe_grad_norm");
}

extern "C" int moe_grad_clip(const moe_grad_t* grads, int32_t n, const float* norm, float max_norm, void* stream) {
  using namespace moe;
  int rc = check_grads(grads, n, true, "moe_grad_clip");
  if (!rc) rc = check_outputs(grads, n, "moe_grad_clip");
  if (rc) return rc;
  if (!norm || (uintptr_t)norm % 4 || !(max_norm >= 0.f)) {
    set_error("moe_grad_clip: null pointer, or max_norm not a number from 0 on");
    return MOE_EINVAL;
  }
  hipStream_t st = (hipStream_t)stream;
  bool any = false;
  for (int i = n; i > 0;) {  // (see grad_scale_kernel for the order)
    const int from = std::max(i - kGradsPerLaunch, 0);
    GradList l;
    fill_list(l, grads, i, from);
    i = from;
    if (l.count == 0) continue;
    any = true;
    ProfScope prof("grad_scale_kernel", st);
    hipLaunchKernelGGL(grad_scale_kernel, dim3(std::min<uint32_t>(l.first[l.count], kGradBlocks)), dim3(kGradThreads), 0, st, l, norm, max_norm);
  }
  return any ? launch_status("moe_grad_clip") : MOE_OK;
}
