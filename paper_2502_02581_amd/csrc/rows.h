// Device helpers of the kernels that stream token rows of any length and alignment: pieces of eight values, sums over a wavefront and
// over the wavefronts of a row, and the counter-based generator of the dropout.
#pragma once

#include "moe_common.h"

namespace moe {

// ---- pieces: eight neighbouring values of a row, 16 bytes in bf16, 32 in fp32.
// Global loads and stores of 16 bytes need no alignment beyond that of a value here, so a row of any length at any address is full pieces and at
// most one short one.  Value by value, two bf16 values make a register, so the wavefront waits where it loads them instead of where it uses them; so a short bf16 piece is
// loaded as the row's last eight values and settled (shifted down) in front of its use (norm's backward pass of 400 x 30: 6.2 us for 11.9; residual of 4000 x 2001 both ways
// 49.8 for 56.1).  Of an output in place it may read values of the piece before that are overwritten already: they are shifted out.  In fp32 a value is a register, and they
// are loaded one by one (777 x 333 backward 8.1 us, settled 9.2).  Stores are value by value.
// Rows that nothing on the chip reads again soon are loaded with the streaming hint (ONCE): what the call writes, and what was written before it, then stays longer in the
// memory-side cache (dropout of 16384 x 2048 and its adjoint 65.0 -> 60.1 us, a norm's step with residual stream, 8192 x 4096, 121 -> 117.5).  The same hint on stores makes the
// call itself faster still (56.7 us) and the one that reads its results slower (the norm's backward pass 61.5 -> 68).
typedef __attribute__((ext_vector_type(4))) uint32_t piece_u32x4;
template <bool ONCE> __device__ __forceinline__ piece_u32x4 load16(const void* p) {
  piece_u32x4 w;
  if (ONCE) {
    typedef piece_u32x4 __attribute__((aligned(2))) anywhere;
    w = __builtin_nontemporal_load(reinterpret_cast<const anywhere*>(p));
  } else {
    __builtin_memcpy(&w, p, 16);
  }
  return w;
}
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
  piece_u32x4 w;
  __device__ __forceinline__ void clear() { w = (piece_u32x4)0; }
  template <bool ONCE> __device__ __forceinline__ void load(const bf16_t* p) { w = load16<ONCE>(p); }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void store(bf16_t* p) const { __builtin_memcpy(p, &w, 16); }
  // without its first n values, 0 to 7
  __device__ __forceinline__ void shift(int n) {
    uint32_t a = w[0], b = w[1], c = w[2], d = w[3];
    a = n & 4 ? c : a, b = n & 4 ? d : b, c = n & 4 ? 0u : c, d = n & 4 ? 0u : d;
    a = n & 2 ? b : a, b = n & 2 ? c : b, c = n & 2 ? d : c, d = n & 2 ? 0u : d;
    a = n & 1 ? a >> 16 | b << 16 : a, b = n & 1 ? b >> 16 | c << 16 : b, c = n & 1 ? c >> 16 | d << 16 : c, d = n & 1 ? d >> 16 : d;
    w = (piece_u32x4){a, b, c, d};
  }
};
template <> struct Piece<float> {
  piece_u32x4 w[2];
  __device__ __forceinline__ void clear() { w[0] = w[1] = (piece_u32x4)0; }
  template <bool ONCE> __device__ __forceinline__ void load(const float* p) {
    w[0] = load16<ONCE>(p);
    w[1] = load16<ONCE>(p + 4);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = __uint_as_float(w[i >> 2][i & 3]);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) w[i >> 2][i & 3] = __float_as_uint(v[i]);
  }
  __device__ __forceinline__ void store(float* p) const {
    __builtin_memcpy(p, &w[0], 16);
    __builtin_memcpy(p + 4, &w[1], 16);
  }
};
// How the short piece is loaded.  kNoTail: there is none.  kTail: settled; kTinyTail: so too, unless the row has less than eight values.
enum { kNoTail = 0, kTail = 1, kTinyTail = 2, kByValue = 3 };
// by how much a piece whose first value is `col` is settled
template <int TAIL>
__device__ __forceinline__ int piece_back(int col, int valid) {
  return (TAIL == kTail || TAIL == kTinyTail) && valid > 0 && valid < 8 && col > 0 ? 8 - valid : 0;
}
// piece at p of which `valid` values (0 to 8, any other number counts as the nearer one) are part of the row; the others are zero, once it is settled
template <int TAIL, bool ONCE = false, typename T>
__device__ __forceinline__ void load_piece(Piece<T>& x, const T* p, int valid, int back) {
  constexpr bool SETTLED = TAIL == kTail || TAIL == kTinyTail;
  if (valid + (SETTLED ? back : 0) >= 8) {
    x.template load<ONCE>(SETTLED ? p - back : p);
  } else {
    x.clear();
    if (TAIL >= kTinyTail && valid > 0) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; j++) v[j] = j < valid ? Elem<T>::load(p + j) : 0.f;
      x.set(v);
    }
  }
}
template <int TAIL, typename T>
__device__ __forceinline__ void settle(Piece<T>& x, int back) {
  if constexpr (TAIL == kTail || TAIL == kTinyTail) x.shift(back);
}
template <int TAIL = kByValue, typename T>
__device__ __forceinline__ void store_piece(const Piece<T>& x, T* p, int valid) {
  if (valid >= 8) {
    x.store(p);
  } else if (TAIL && valid > 0) {
    float v[8];
    x.values(v);
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (j < valid) Elem<T>::store(p + j, v[j]);
  }
}

// ---- sums.  Every lane adds in the same order as its partner, so all lanes end with the same bits.
template <int CONTROL, typename T> __device__ __forceinline__ T dpp(T x) {
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ float add_lanes1(float x) { return x + dpp<0xB1>(x); }   // lane ^ 1
__device__ __forceinline__ float add_lanes2(float x) { return x + dpp<0x4E>(x); }   // lane ^ 2
__device__ __forceinline__ float add_lanes4(float x) { return x + dpp<0x141>(x); }  // the other four of eight, mirrored
__device__ __forceinline__ float add_lanes8(float x) { return x + dpp<0x140>(x); }  // the other eight of sixteen, mirrored
// lanes of sixteen whose numbers differ by 4, 8 or 12 (rotations by 8 and 4)
template <typename T> __device__ __forceinline__ T add_quads(T x) {
  x += dpp<0x128>(x);
  return x + dpp<0x124>(x);
}
// over each sixteen neighbouring lanes
__device__ __forceinline__ float row16_sum(float x) { return add_lanes8(add_lanes4(add_lanes2(add_lanes1(x)))); }
// lane ^ 16, lane ^ 32
template <typename T> __device__ __forceinline__ T add_rows16(T x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return __builtin_bit_cast(T, (uint32_t)a[0]) + __builtin_bit_cast(T, (uint32_t)a[1]);
}
template <typename T> __device__ __forceinline__ T add_rows32(T x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return __builtin_bit_cast(T, (uint32_t)a[0]) + __builtin_bit_cast(T, (uint32_t)a[1]);
}
// over the wavefront, without LDS (wave_sum's exchanges go through it)
__device__ __forceinline__ float lanes_sum(float x) { return add_rows32(add_rows16(row16_sum(x))); }
// N sums over the n_waves (up to 16) wavefronts of a block: one barrier.  `part` holds two sets that calls use in turn: who writes a set again has passed the
// barrier of the call between, which nobody reaches before reading that set.
template <int N>
struct RowSums {
  float part[2][N][16];
  template <int M>
  __device__ __forceinline__ void sum(float (&s)[M], int wave, int n_waves, int& turn) {
    static_assert(M <= N, "sums");
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < M; i++) {
      const float t = lanes_sum(s[i]);
      if (lane == 0) part[turn][i][wave] = t;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; i++) s[i] = row16_sum((lane & 15) < n_waves ? part[turn][i][lane & 15] : 0.f);
    turn ^= 1;
  }
};

// ---- dropout.  Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two 32 x 32 bit products turn a
// counter of four words and a key of two into four random words.  One call decides over a piece: its eight half-words, in order, against a threshold.
struct Dropout {
  const uint64_t* rng;  // device: seed, step
  uint32_t threshold;   // 65536 p, rounded; 0: nothing is dropped, and rng is not read
  uint32_t site;        // shifted: site << 16
  float scale;          // 65536 / (65536 - threshold)
};
struct DropKey {
  uint32_t k0, k1, c2, c3;
};
__device__ __forceinline__ DropKey drop_key(const Dropout& d) {
  if (d.threshold == 0) return {};
  const uint64_t seed = d.rng[0], step = d.rng[1];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
}
__device__ __forceinline__ void drop_words(const DropKey& key, uint32_t c0, uint32_t c1, uint32_t (&out)[4]) {
  uint32_t c2 = key.c2, c3 = key.c3, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; r++) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}
// v[j] = kept ? v[j] * scale + add[j] : add[j], for piece `c` of row `row`
__device__ __forceinline__ void drop_piece(const Dropout& d, const DropKey& key, uint32_t c, uint32_t row, float (&v)[8], const float (&add)[8]) {
  uint32_t bits[4];
  drop_words(key, c + d.site, row, bits);
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const uint32_t h = j & 1 ? bits[j >> 1] >> 16 : bits[j >> 1] & 0xffffu;
    v[j] = h >= d.threshold ? fmaf(v[j], d.scale, add[j]) : add[j];
  }
}

// host: checks and converts the arguments of a dropout (drop may be NULL: none)
int make_dropout(const moe_drop_t* drop, Dropout& out, const char* who);

// host: checks one tensor of rows of a call: its pointer (needed: not NULL), alignment and row stride
int check_rows(const char* who, const char* what, const void* p, int64_t ld, int64_t n_rows, int64_t cols, size_t elem, bool needed);
// host: an output that is an input has to have its rows where that has them
int check_places(const char* who, const char* out, const void* p, int64_t ldp, const char* in, const void* q, int64_t ldq, int64_t n_rows);

}  // namespace moe
