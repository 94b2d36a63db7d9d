// What the attention kernels over the paged cache share.
#pragma once

#include <float.h>

#include "cache.h"

namespace spindle {

constexpr int kRows = 16;                        // query rows of a matrix instruction
constexpr float kLog2e = 1.44269504088896340736f;

// What the matrix instructions are fed.  Codes are exact in f16 and in bf16, and so are 16-bit queries in their own type; f32
// queries are three bf16 (24 bits).  The softmax's weights are bf16 whatever the queries are, two for 16-bit queries (16 bits) and
// three for f32 (24): bf16 has float's range, where no weight falls off, and none loses bits because its page's scale is far
// below another's.  One f16 for f16 queries would hold 11 bits over a factor of 2^38, V's scale included, and leave out half of the
// products with V: 59 and not 66 us for five prompts of up to 1500 tokens with capped scores, 600 and 717 for 2048 queries over
// 16384 tokens, 34.7 and 35.8 for 32 ragged contexts of up to 8192.
struct Bf16Operand {
  typedef b8 frag;
  static __device__ __forceinline__ f4 mma(frag x, frag y, f4 z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }
  static __device__ __forceinline__ f16v mma32(frag x, frag y, f16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }
  // x as the sum of n operands: leading 16 bits, and what is left (exact but for the last one)
  template <int n>
  static __device__ __forceinline__ void split(const float *x, frag *out) {
    float rest[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) rest[j] = x[j];
#pragma unroll
    for (int k = 0; k < n - 1; ++k) {
      u4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * j + 1]), __float_as_uint(rest[2 * j]), 0x07060302u);
#pragma unroll
      for (int j = 0; j < 8; ++j) rest[j] -= __uint_as_float(__float_as_uint(rest[j]) & 0xFFFF0000u);
      out[k] = __builtin_bit_cast(frag, w);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) out[n - 1][j] = (__bf16)rest[j];
  }
  template <int FMT>
  static __device__ __forceinline__ frag codes(uint32_t lo, uint32_t hi, float scale = 1.f) {
    uint32_t p[4];
    Code<FMT>::to_bf16(lo, scale, p);
    Code<FMT>::to_bf16(hi, scale, p + 2);
    const u4 w = {p[0], p[1], p[2], p[3]};
    return __builtin_bit_cast(frag, w);
  }
};

struct F16Operand {
  typedef h8 frag;
  static __device__ __forceinline__ f4 mma(frag x, frag y, f4 z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }
  static __device__ __forceinline__ f16v mma32(frag x, frag y, f16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, z, 0, 0, 0); }
  template <int n>
  static __device__ __forceinline__ void split(const float *x, frag *out) {
    static_assert(n == 1, "f16 queries are one operand");
#pragma unroll
    for (int j = 0; j < 8; ++j) out[0][j] = (_Float16)x[j];
  }
  template <int FMT>
  static __device__ __forceinline__ frag codes(uint32_t lo, uint32_t hi) {
    union {
      h8 v;
      h2 p[4];
    } r;
    Code<FMT>::to_half(lo, &r.p[0], &r.p[1]);
    Code<FMT>::to_half(hi, &r.p[2], &r.p[3]);
    return r.v;
  }
};

template <int DT>
struct Num {
  typedef Bf16Operand Q;                         // of queries and K
  static constexpr int kQ = DT == SPINDLE_F32 ? 3 : 1, kP = DT == SPINDLE_F32 ? 3 : 2;
};
template <>
struct Num<SPINDLE_F16> {
  typedef F16Operand Q;
  static constexpr int kQ = 1, kP = 2;
};
typedef Bf16Operand Weights;                     // of the weights and V

// A row's weights are counted from a logit that its largest one may exceed by so much (log2) before what was gathered is
// scaled down; they are lowered by as much, so that none is above 1 and its product with V is no larger than V.
constexpr float kSlack = 8.f;

struct AttendArgs {
  CacheView c;
  const int32_t *table, *len, *cu, *prefix, *q_pos;
  const float *slopes;
  const char *Q;
  char *out;
  float *lse;
  float *part_o;                                 // [row of all][split][128] outputs of a split, each divided by its own sum
  float2 *part_ml;                               // [row of all][split] largest logit (log2), sum
  long long qst, qsh;                            // bytes
  float scale, softcap, cap_in, cap_out, per_cap;   // 2 log2 e / softcap, softcap log2 e, 1 / softcap
  int width, max_q, total_q, group, heads_q;
  int batch, splits, piece, row_tiles;           // a sequence's pieces go to its chunks in turn: chunk s has s, s + splits, ..
};

// Rows of 4 bytes become columns: out[d] holds byte d of t0, t1, t2, t3.
__device__ __forceinline__ void transpose4(uint32_t t0, uint32_t t1, uint32_t t2, uint32_t t3, uint32_t *out) {
  const uint32_t a = __builtin_amdgcn_perm(t1, t0, 0x05010400u), b = __builtin_amdgcn_perm(t1, t0, 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(t3, t2, 0x05010400u), d = __builtin_amdgcn_perm(t3, t2, 0x07030602u);
  out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// A load whose address is the same for the whole wave, of memory that the kernel does not write: through the scalar cache
// and into a scalar register, so that a page's number is there without a vector load's wait and a lane read.
template <typename T>
__device__ __forceinline__ T uniform_load(const T *p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) T *>(reinterpret_cast<uintptr_t>(p));
}

template <typename T>
__device__ __forceinline__ T uniform_load_at(const T *p, uint32_t index) {   // index * sizeof(T) below 2^32
  return uniform_load(reinterpret_cast<const T *>(reinterpret_cast<const char *>(p) + (uint32_t)(index * (uint32_t)sizeof(T))));
}

// The larger of two numbers, NaN if one is (no instruction is spent on making a NaN quiet, as fmaxf would).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Over the four lanes that hold a row (lane % 16 is the row), without a trip through LDS: the swap of 16 (32) lanes of a
// register with itself gives both halves to everyone.
__device__ __forceinline__ float over_groups_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Over the two lanes that hold a row (lane % 32 is the row).
__device__ __forceinline__ float over_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float over_halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float over_groups_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// log sum exp of a row from its reference logit (log2) and sum; a row that sees nothing has -inf, NaN stays.
__device__ __forceinline__ float lse_of(float top, float sum) {
  return sum > 0.f ? (top + kSlack + __builtin_amdgcn_logf(sum)) / kLog2e : sum == sum ? -INFINITY : sum;
}

// What a row of the tile is, and what it has gathered so far.
struct RowState {
  int limit;                                     // tokens before it are seen
  int q_at;                                      // position, for the bias
  float slope;                                   // in log2 units
  float m, l;                                    // reference logit (log2), sum of the weights
};

// A lane's part of a query row as the operands of kSteps steps, those of step s from dimension offset_of(s) on.
template <int DT, int kSteps, typename Where>
__device__ __forceinline__ void load_query(typename Num<DT>::Q::frag (*q)[Num<DT>::kQ], const char *src, bool on, Where offset_of) {
  typedef typename Elem<DT>::type T;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    T e[8];
    float v[8];
    if (on) __builtin_memcpy(e, __builtin_assume_aligned(src + offset_of(s) * sizeof(T), 16), sizeof(e));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = on ? Elem<DT>::to_float(e[j]) : 0.f;
    Num<DT>::Q::template split<Num<DT>::kQ>(v, q[s]);
  }
}

// What a kernel has to do to the logits, beside their masks.
constexpr int kPlain = 0, kCapped = 1, kBiased = 2;   // kBiased: a bias, positions or a wide cap, and a cap if there is one

// A logit in log2 units is offset + slope z: of a plain product z is the product itself, of a capped one
//   cap tanh(x / cap) = cap - 2 cap / (1 + e^(2 x / cap)),  z = -1 / (1 + e^(2 x / cap))
// so that the largest z is found first and what is left is one multiply-add on the way into the exponential.  The sum is
// off by some 2^-23 of the cap, whatever the logit: too much of a wide cap, most of whose logits are far below it.  Those
// are x (1 - y^2 / 3 + ..) up to y = x / cap = 1/8, where the next term is 2^-29 of x, and the sum's error 2^-20 behind it.
constexpr float kWideCap = 64.f;

__device__ __forceinline__ float wide_capped(float x, const AttendArgs &a) {
  const float y = x * a.per_cap, y2 = y * y;
  const float near = x * (1.f + y2 * (-1.f / 3.f + y2 * (2.f / 15.f - y2 * (17.f / 315.f))));
  const float far = a.softcap * (1.f + 2.f * __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(y * (2.f * kLog2e))));
  return __builtin_fabsf(y) < 0.125f ? near : far;
}

template <int kMode>
__device__ __forceinline__ float raw_logit(float s, float f, const AttendArgs &a, const RowState &st, int k_at) {
  if (kMode == kPlain) return s;
  if (kMode == kCapped) return __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(s * fminf(f * a.cap_in, FLT_MAX)));   // (0 * inf is none)
  float w = s * f;
  if (a.softcap > kWideCap) w = wide_capped(w, a) * kLog2e;
  else if (a.softcap > 0.f) w = a.cap_out + 2.f * a.cap_out * __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(w * a.cap_in));
  else w *= kLog2e;
  w -= st.slope * __builtin_fabsf((float)(int)((uint32_t)st.q_at - (uint32_t)k_at));
  return k_at < 0 ? -INFINITY : w;
}
template <int kMode>
__device__ __forceinline__ float logit_slope(float f, const AttendArgs &a) {
  return kMode == kPlain ? f : kMode == kCapped ? 2.f * a.cap_out : 1.f;
}
template <int kMode>
__device__ __forceinline__ float logit_offset(const AttendArgs &a) {
  return kMode == kCapped ? a.cap_out : 0.f;
}

// Takes the largest logit of a row's step: what was gathered is scaled down (by what is returned) if it has grown by more than
// the slack.
__device__ __forceinline__ float gather(RowState &st, float top, bool *scaled) {
  const bool grown = top > st.m + kSlack;                  // -inf at first: then any logit is more
  *scaled = __any(grown);
  if (!*scaled) return 1.f;
  const float back = grown ? __builtin_amdgcn_exp2f(st.m - top) : 1.f;   // 2^-inf is 0
  if (grown) st.m = top;
  st.l *= back;
  return back;
}

// Positions of four slots in a row, in one load that asks for no more than their own alignment.
__device__ __forceinline__ void load_positions(const int32_t *from, int *to) {
  u4 w;
  __builtin_memcpy(&w, from, sizeof(w));
#pragma unroll
  for (int j = 0; j < 4; ++j) to[j] = (int)w[j];
}

constexpr int kManyRows = 128;                   // query rows of a workgroup of the kernel for many rows

constexpr int kManyStep = 64;                    // tokens of its step

// Launches the kernel for many rows (16-bit queries).
spindle_status launch_attend_rows(const AttendArgs &a, int dtype, int format, int mode, unsigned blocks, hipStream_t st);

}  // namespace spindle
