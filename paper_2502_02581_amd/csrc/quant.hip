// moe_quant_rows / moe_quant_weights: see quant_format.h for the format.
#include <algorithm>

#include "quant_format.h"

namespace moe {

// ------------------------------------------------------------------------------------- rows
// Sixteen lanes per block of 128 values, eight values a lane: 16 (fp32: 32) bytes in, 8 out; the maximum by four exchanges.
// Bound by HBM: it reads every value and writes every code once.  8192 x 7168 values, back to back on buffers that no cache holds: bf16 34.1 us, 5.2 TB/s, of which
// the kernel is 28.2 (with the maximum by exchanges through LDS and the conversion from fp32 36.5); fp32 51.0, 5.8 TB/s (kernel 47.2; 61.3 with the whole and the cut
// pieces of a row loaded by one loop, which kept two of a lane's values in scratch memory).
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    Vec16<T>::load(p, v);
  } else {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* __restrict__ X, int64_t ldx, uint32_t n_blocks, uint32_t per_row, int cols,
                                                         uint8_t* __restrict__ Q, int64_t ldq, uint8_t* __restrict__ S, int64_t lds) {
  const int lane = threadIdx.x & 15;
  for (uint32_t b = blockIdx.x * 16 + (threadIdx.x >> 4); b < n_blocks; b += gridDim.x * 16) {
    const uint32_t row = b / per_row, kb = b - row * per_row, c0 = kb * kQuantBlock + lane * 8;
    const T* x = X + (int64_t)row * ldx + c0;
    uint2 codes;
    int e;
    if constexpr (VEC && sizeof(T) == 2) {
      uint32_t v[1][4] = {};
      if (c0 + 8 <= (uint32_t)cols) {
        const uint4 t = *reinterpret_cast<const uint4*>(x);
        v[0][0] = t.x; v[0][1] = t.y; v[0][2] = t.z; v[0][3] = t.w;
      } else {
        for (int i = 0; i < cols - (int)c0; i++) v[0][i / 2] |= (uint32_t)x[i] << (16 * (i % 2));
      }
      uint2 c[1];
      int b1[1];
      quant_blocks_bf16(v, 0xffffffffu, c, b1);
      codes = c[0];
      e = b1[0];
    } else {
      float v[8] = {};
      if (VEC && c0 + 8 <= (uint32_t)cols) {
        load8(x, v);
      } else {
        const int n = cols - (int)c0;  // how many of the eight there are
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < n ? Elem<T>::load(x + i) : 0.f;
      }
      int m[1] = {0};
#pragma unroll
      for (int i = 0; i < 8; i++) m[0] = max(m[0], (int)finite_bits(v[i]));
      row_max16(m);
      e = quant_exponent((uint32_t)m[0]);
      const float f = quant_factor(e);
      const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
      codes = make_uint2(quant_codes(lo, f), quant_codes(hi, f));
    }
    *reinterpret_cast<uint2*>(Q + (int64_t)row * ldq + c0) = codes;
    if (lane == 0) S[(int64_t)row * lds + kb] = (uint8_t)e;
  }
}

// ---------------------------------------------------------------------------------- matrices
// A block of 256 threads per 128 x 128 values, 8 x 8 of them a thread: the values are read once and both layouts are written from
// registers, the transposed one through LDS, so that all three streams are whole 128-byte pieces.  Bound by HBM: 60 bf16 matrices of 2048 x 1408, both
// layouts, 135 us, 5.1 TB/s, where a plain copy moves 4.8, fp32 ones 189 us, 5.5; 24 bf16 ones of 1000 x 1368, which end in cut blocks and a partial round, 34 us,
// 3.8 TB/s.  (LDS pieces swizzled so that no banks conflict: no change.)
struct QuantMatrix {
  uint8_t *Q, *S;       // [G][K rows of ldq bytes], [G][K / 128 rows of lds bytes]; NULL: not wanted
  int64_t ldq, lds;
  uint8_t *Qt, *St;     // the transposed matrix
  int64_t ldqt, ldst;
};
// 4 x 4 bytes: word i of `r` holds row i, of the result column i
__device__ __forceinline__ void transpose4(const uint32_t (&r)[4], uint32_t (&c)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602);
  const uint32_t x = __builtin_amdgcn_perm(r[3], r[2], 0x05010400), y = __builtin_amdgcn_perm(r[3], r[2], 0x07030602);
  c[0] = __builtin_amdgcn_perm(x, a, 0x05040100);
  c[1] = __builtin_amdgcn_perm(x, a, 0x07060302);
  c[2] = __builtin_amdgcn_perm(y, b, 0x05040100);
  c[3] = __builtin_amdgcn_perm(y, b, 0x07060302);
}
template <typename T>
__global__ __launch_bounds__(256) void quant_matrix_kernel(const T* __restrict__ W, int K, int N, QuantMatrix p) {
  constexpr int LD = 136;  // bytes of a column in LDS: eight more than it has
  __shared__ __align__(16) uint8_t tile[kQuantBlock * LD];
  __shared__ uint32_t part[4];
  const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
  const int k0 = blockIdx.y * kQuantBlock + rg * 8, n0 = blockIdx.x * kQuantBlock + cg * 8;
  const int64_t g = blockIdx.z;
  float v[8][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    // (K and N are multiples of 8: a thread's values are all there or all missing)
    if (k0 < K && n0 < N) {
      load8(W + (g * K + k0 + i) * N + n0, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) v[i][j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; j++) m = max(m, finite_bits(v[i][j]));
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, x, kWave));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(part[0], part[1]), max(part[2], part[3]));
  const int e = quant_exponent(m);
  const float f = quant_factor(e);
  uint32_t lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const float a[4] = {v[i][0], v[i][1], v[i][2], v[i][3]}, b[4] = {v[i][4], v[i][5], v[i][6], v[i][7]};
    lo[i] = quant_codes(a, f);
    hi[i] = quant_codes(b, f);
  }
  if (p.Q && k0 < K)
#pragma unroll
    for (int i = 0; i < 8; i++) *reinterpret_cast<uint2*>(p.Q + (g * K + k0 + i) * p.ldq + n0) = make_uint2(lo[i], hi[i]);
  if (threadIdx.x == 0) {
    if (p.S) p.S[(g * gridDim.y + blockIdx.y) * p.lds + blockIdx.x] = (uint8_t)e;
    if (p.St) p.St[(g * gridDim.x + blockIdx.x) * p.ldst + blockIdx.y] = (uint8_t)e;
  }
  if (!p.Qt) return;
#pragma unroll
  for (int q = 0; q < 2; q++) {  // columns 0..3, 4..7 of the thread
    uint32_t up[4], down[4], a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; i++) { up[i] = q ? hi[i] : lo[i]; down[i] = q ? hi[4 + i] : lo[4 + i]; }
    transpose4(up, a);
    transpose4(down, b);
#pragma unroll
    for (int j = 0; j < 4; j++) *reinterpret_cast<uint2*>(tile + (cg * 8 + q * 4 + j) * LD + rg * 8) = make_uint2(a[j], b[j]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const int n = i * 16 + rg, col = blockIdx.x * kQuantBlock + n;
    if (col < N)
      *reinterpret_cast<uint2*>(p.Qt + (g * N + col) * p.ldqt + blockIdx.y * kQuantBlock + cg * 8) = *reinterpret_cast<const uint2*>(tile + n * LD + cg * 8);
  }
}

static int check_dtype(int dtype, const char* who) {
  if (dtype == MOE_F32 || dtype == MOE_BF16) return MOE_OK;
  set_error("%s: unknown dtype %d", who, dtype);
  return MOE_EDTYPE;
}

// 16-byte loads where every row starts on 16 bytes, else value by value
static void launch_quant_rows(const void* X, int dtype, int n_rows, int cols, int64_t ldx, uint8_t* Q, uint8_t* S, int64_t ldq, int64_t lds,
                              hipStream_t st) {
  const bool vec = aligned16(X) && ldx * elem_size(dtype) % 16 == 0;
  const uint32_t per_row = (uint32_t)quant_blocks(cols), n = (uint32_t)n_rows * per_row;
  const dim3 grid(std::min<uint32_t>((n + 15) / 16, 32768));
  ProfScope prof("quant_rows_kernel", st);
#define MOE_QUANT_ROWS(T, V) hipLaunchKernelGGL((quant_rows_kernel<T, V>), grid, dim3(256), 0, st, (const T*)X, ldx, n, per_row, cols, Q, ldq, S, lds)
  if (dtype == MOE_F32) {
    if (vec) MOE_QUANT_ROWS(float, true);
    else MOE_QUANT_ROWS(float, false);
  } else {
    if (vec) MOE_QUANT_ROWS(bf16_t, true);
    else MOE_QUANT_ROWS(bf16_t, false);
  }
#undef MOE_QUANT_ROWS
}
}  // namespace moe

extern "C" int64_t moe_quant_row_bytes(int64_t cols) { return cols < 1 ? 0 : moe::quant_row(cols); }
extern "C" int64_t moe_quant_scale_bytes(int64_t cols) { return cols < 1 ? 0 : moe::quant_blocks(cols); }

extern "C" int moe_quant_rows(const void* X, int32_t dtype, int32_t n_rows, int32_t cols, int64_t ldx, void* Q, void* S, void* stream) {
  using namespace moe;
  const int rc = check_dtype(dtype, "moe_quant_rows");
  if (rc) return rc;
  if (n_rows < 0 || cols < 1 || ldx < cols || (int64_t)n_rows * quant_blocks(cols) >= (int64_t)1 << 31 || ldx >= (int64_t)1 << 40) {
    set_error("moe_quant_rows: bad n_rows=%d cols=%d ldx=%lld", n_rows, cols, (long long)ldx);
    return MOE_EINVAL;
  }
  if (n_rows == 0) return MOE_OK;
  if (!X || !Q || !S) {
    set_error("moe_quant_rows: null pointer");
    return MOE_EINVAL;
  }
  const size_t es = elem_size(dtype);
  if (!aligned16(Q) || (uintptr_t)X % es) {
    set_error("moe_quant_rows: codes must be 16-byte aligned, values aligned to their size");
    return MOE_EINVAL;
  }
  launch_quant_rows(X, dtype, n_rows, cols, ldx, (uint8_t*)Q, (uint8_t*)S, quant_row(cols), quant_blocks(cols), (hipStream_t)stream);
  return launch_status("moe_quant_rows");
}

extern "C" int moe_quant_weights(const void* W, int32_t dtype, int32_t n_groups, int32_t K, int32_t N, void* Q, int64_t ldq, void* S, int64_t lds,
                                 void* Qt, int64_t ldqt, void* St, int64_t ldst, void* stream) {
  using namespace moe;
  const int rc = check_dtype(dtype, "moe_quant_weights");
  if (rc) return rc;
  if (n_groups < 1 || n_groups > MOE_MAX_EXPERTS || K < 1 || N < 1 || K % 8 || N % 8 || quant_blocks(K) > 65535) {
    set_error("moe_quant_weights: bad n_groups=%d K=%d N=%d (K and N are multiples of 8)", n_groups, K, N);
    return MOE_EINVAL;
  }
  if (!W || (!Q && !Qt) || !Q != !S || !Qt != !St) {
    set_error("moe_quant_weights: null pointer (codes and exponents go together)");
    return MOE_EINVAL;
  }
  if ((Q && (ldq < quant_row(N) || lds < quant_blocks(N) || ldq % 16)) || (Qt && (ldqt < quant_row(K) || ldst < quant_blocks(K) || ldqt % 16))) {
    set_error("moe_quant_weights: rows of codes take moe_quant_row_bytes, a multiple of 16, rows of exponents moe_quant_scale_bytes");
    return MOE_EINVAL;
  }
  if (!aligned16(W) || !aligned16(Q) || !aligned16(Qt)) {
    set_error("moe_quant_weights: every tensor must be 16-byte aligned");
    return MOE_EINVAL;
  }
  const QuantMatrix p = {(uint8_t*)Q, (uint8_t*)S, ldq, lds, (uint8_t*)Qt, (uint8_t*)St, ldqt, ldst};
  const dim3 grid((unsigned)quant_blocks(N), (unsigned)quant_blocks(K), (unsigned)n_groups);
  hipStream_t st = (hipStream_t)stream;
  {
    ProfScope prof("quant_matrix_kernel", st);
    if (dtype == MOE_F32) hipLaunchKernelGGL(quant_matrix_kernel<float>, grid, dim3(256), 0, st, (const float*)W, K, N, p);
    else hipLaunchKernelGGL(quant_matrix_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)W, K, N, p);
  }
  return launch_status("moe_quant_weights");
}
