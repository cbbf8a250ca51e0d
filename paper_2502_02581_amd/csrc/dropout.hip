// moe_dropout: dropout of a branch from a counter-based generator, with the residual stream added on the way; without it, its own adjoint.
//   out = r + (kept ? x * 65536 / (65536 - threshold) : 0)
// The mask is a function of the counter (piece and site, row, step) and of the seed, so nothing about it is stored and any pass over the rows, in any order or layout,
// finds it again.  Sixteen bits a value: one call of the generator serves the eight values of a piece.
#include <math.h>

#include "rows.h"

namespace moe {

struct DropoutArgs {
  const void *X, *R;
  void* out;
  int64_t ldx, ldr, ldo, pieces;  // pieces of all rows
  int32_t cols;
  uint32_t per_row, magic;        // pieces of a row, and 2^32 / per_row rounded up (0: one)
  Dropout drop;
};

// A block takes kDropThreads * U neighbouring pieces, numbered through the rows.  Their rows: the block's first one by a 64-bit division, the others by a product with
// the reciprocal, which is exact for numbers below per_row + kDropThreads * U (per_row up to 2^15: the product's error is below 2^15 * 2^16 / 2^32 of a row's).
constexpr int kDropThreads = 256;
template <typename T, int TAIL, int U>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropoutArgs a) {
  const DropKey key = drop_key(a.drop);
  const int64_t base = (int64_t)blockIdx.x * (kDropThreads * U);
  const uint32_t row0 = (uint32_t)(base / a.per_row), off = (uint32_t)(base - (int64_t)row0 * a.per_row);
  Piece<T> x[U], r[U];
  uint32_t row[U], c[U];
  int valid[U], back[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    const uint32_t i = u * kDropThreads + threadIdx.x, q = off + i;
    const uint32_t over = a.magic ? __umulhi(q, a.magic) : q;
    row[u] = row0 + over;
    c[u] = q - over * a.per_row;
    valid[u] = base + i < a.pieces ? a.cols - 8 * (int)c[u] : 0;
    back[u] = piece_back<TAIL>(8 * (int)c[u], valid[u]);
    load_piece<TAIL, true>(x[u], (const T*)a.X + (int64_t)row[u] * a.ldx + 8 * c[u], valid[u], back[u]);
    r[u].clear();
    if (a.R) load_piece<TAIL, true>(r[u], (const T*)a.R + (int64_t)row[u] * a.ldr + 8 * c[u], valid[u], back[u]);
  }
#pragma unroll
  for (int u = 0; u < U; u++) {
    float v[8], add[8];
    settle<TAIL>(x[u], back[u]);
    settle<TAIL>(r[u], back[u]);
    x[u].values(v);
    r[u].values(add);
    if (a.drop.threshold) {
      drop_piece(a.drop, key, c[u], row[u], v, add);
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) v[j] += add[j];
    }
    x[u].set(v);
    store_piece<TAIL>(x[u], (T*)a.out + (int64_t)row[u] * a.ldo + 8 * c[u], valid[u]);
  }
}

int check_rows(const char* who, const char* what, const void* p, int64_t ld, int64_t n_rows, int64_t cols, size_t elem, bool needed) {
  if (!p) {
    if (!needed || n_rows == 0) return MOE_OK;
    set_error("%s: null pointer: %s", who, what);
    return MOE_EINVAL;
  }
  if ((uintptr_t)p % elem) {
    set_error("%s: %s must be aligned to its values", who, what);
    return MOE_EINVAL;
  }
  if (n_rows > 1 && (ld < cols || ld >= (int64_t)1 << 40)) {
    set_error("%s: %s: a row stride of %lld for rows of %lld", who, what, (long long)ld, (long long)cols);
    return MOE_EINVAL;
  }
  return MOE_OK;
}

int check_places(const char* who, const char* out, const void* p, int64_t ldp, const char* in, const void* q, int64_t ldq, int64_t n_rows) {
  if (!p || p != q || n_rows <= 1 || ldp == ldq) return MOE_OK;
  set_error("%s: %s is %s, but with a row stride of %lld for %lld", who, out, in, (long long)ldp, (long long)ldq);
  return MOE_EINVAL;
}
int make_dropout(const moe_drop_t* drop, Dropout& out, const char* who) {
  out = {nullptr, 0, 0, 1.f};
  if (!drop) return MOE_OK;
  const double t = floor((double)drop->p * 65536. + 0.5);
  if (!(drop->p >= 0.f) || t > 65535.) {
    set_error("%s: a dropout probability of %g (0 or more, less than 1 - 2^-17)", who, (double)drop->p);
    return MOE_EINVAL;
  }
  if (drop->site > 65535u) {
    set_error("%s: dropout site %u (0 to 65535)", who, drop->site);
    return MOE_EINVAL;
  }
  out.threshold = (uint32_t)t;
  out.site = drop->site << 16;
  out.scale = (float)(65536. / (65536. - t));
  out.rng = drop->rng;
  if (out.threshold && (!drop->rng || (uintptr_t)drop->rng % 8)) {
    set_error("%s: null pointer or misaligned: the dropout's rng", who);
    return MOE_EINVAL;
  }
  return MOE_OK;
}

}  // namespace moe

extern "C" int moe_dropout(const void* X, int64_t ldx, const void* R, int64_t ldr, int32_t dtype, int32_t n_rows, int32_t cols, const moe_drop_t* drop,
                           void* out, int64_t ldo, void* stream) {
  using namespace moe;
  const char* who = "moe_dropout";
  if (dtype != MOE_F32 && dtype != MOE_BF16) {
    set_error("%s: unknown dtype %d", who, dtype);
    return MOE_EDTYPE;
  }
  if (!drop) {
    set_error("%s: drop is NULL", who);
    return MOE_EINVAL;
  }
  Dropout d;
  int rc = make_dropout(drop, d, who);
  if (rc) return rc;
  if (n_rows < 0 || cols < 1 || cols > 1 << 18) {
    set_error("%s: bad sizes: %d rows of %d (1 to 2^18)", who, n_rows, cols);
    return MOE_EINVAL;
  }
  if (n_rows == 0) return MOE_OK;
  const size_t e = elem_size(dtype);
  if ((rc = check_rows(who, "X", X, ldx, n_rows, cols, e, true)) || (rc = check_rows(who, "R", R, ldr, n_rows, cols, e, false)) ||
      (rc = check_rows(who, "out", out, ldo, n_rows, cols, e, true)) || (rc = check_places(who, "out", out, ldo, "X", X, ldx, n_rows)) ||
      (rc = check_places(who, "out", out, ldo, "R", R, ldr, n_rows)))
    return rc;
  const uint32_t per_row = (uint32_t)(cols + 7) / 8;
  const int64_t pieces = (int64_t)n_rows * per_row;
  const DropoutArgs a = {X, R, out, ldx, ldr, ldo, pieces, cols, per_row, per_row == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + per_row - 1) / per_row), d};
  hipStream_t st = (hipStream_t)stream;
  constexpr int U = 2;
  const int64_t blocks = (pieces + kDropThreads * U - 1) / (kDropThreads * U);
  if (blocks >= (int64_t)1 << 24) {  // (a launch has less than 2^32 threads)
    set_error("%s: %d rows of %d are too many values for a call (2^36)", who, n_rows, cols);
    return MOE_EINVAL;
  }
  ProfScope prof("dropout_kernel", st);
  if (dtype == MOE_F32) hipLaunchKernelGGL((dropout_kernel<float, kByValue, U>), dim3((unsigned)blocks), dim3(kDropThreads), 0, st, a);
  else if (cols % 8 == 0) hipLaunchKernelGGL((dropout_kernel<bf16_t, kNoTail, U>), dim3((unsigned)blocks), dim3(kDropThreads), 0, st, a);
  else if (cols > 8) hipLaunchKernelGGL((dropout_kernel<bf16_t, kTail, U>), dim3((unsigned)blocks), dim3(kDropThreads), 0, st, a);
  else hipLaunchKernelGGL((dropout_kernel<bf16_t, kTinyTail, U>), dim3((unsigned)blocks), dim3(kDropThreads), 0, st, a);
  return launch_status(who);
}
