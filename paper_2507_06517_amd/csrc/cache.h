// The paged cache in 8 bits: what its kernels share (layout, code formats).
#pragma once

#include "common.h"

namespace spindle {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

constexpr float kTinyScale = 0x1p-126f;      // no scale is smaller: 1 / scale stays finite

struct CacheView {
  uint8_t *k, *v;            // [n_pages][H][P][128] codes
  float *ks, *vs;            // [n_pages][H]
  int32_t *pos;              // [n_pages][H][P], or NULL
  int32_t n_pages, H, P, shift;   // P = 1 << shift tokens a page
};

spindle_status check_cache(const spindle_cache *c, CacheView *out);
spindle_status check_table(const void *table, int32_t width, const void *len, int32_t batch, const CacheView &c);

__device__ __forceinline__ size_t page_row(const CacheView &c, int page, int head) {   // first token row of a page of one head
  return ((size_t)page * c.H + head) * c.P;
}

// The same in as few scalar instructions as it takes (an attention step's waves issue one instruction at a time): n_pages x H is
// below 2^30, so that a page of a head has a 32-bit number, and its scale a 32-bit offset.
__device__ __forceinline__ uint32_t page_number(const CacheView &c, int page, int head) { return (uint32_t)page * (uint32_t)c.H + (uint32_t)head; }
__device__ __forceinline__ uint64_t page_bytes(const CacheView &c, uint32_t number, int slot) {
  return ((uint64_t)number << (c.shift + 7)) + ((uint32_t)slot << 7);
}

// What of an E4M3 scale goes into a bf16 operand: the power of two that it is, or that lies below it, and no more than 2^100, where
// no code becomes infinite.
__device__ __forceinline__ float operand_scale(float scale) {
  return __uint_as_float(min(max(__float_as_uint(scale) & 0x7F800000u, 0x00800000u), 0x71800000u));
}

template <int FMT>
struct Code;

// E4M3: scales are powers of two, so that x / scale is exact and a page whose scale grows loses nothing but what falls
// below the smallest code.
template <>
struct Code<SPINDLE_E4M3> {
  static __device__ __forceinline__ float scale_for(float amax) {            // smallest 2^e >= amax / 448
    if (!(amax > 0.f)) return kTinyScale;
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);  // 448 = 1.75 2^8; biased exponent of the scale
    return __uint_as_float((uint32_t)(e < 1 ? 1 : e) << 23);
  }
  static __device__ __forceinline__ float clean(float t) {                    // saturated, NaN is zero
    return t != t ? 0.f : __builtin_amdgcn_fmed3f(t, -448.f, 448.f);
  }
  static __device__ __forceinline__ uint32_t encode4(const float *x, float s, float rs) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(clean(x[0] * rs), clean(x[1] * rs), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clean(x[2] * rs), clean(x[3] * rs), w, true);
  }
  static __device__ __forceinline__ void decode4(uint32_t w, float *x) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  }
  // codes at scale `from` as codes at scale `to`
  static __device__ __forceinline__ uint32_t rescale4(uint32_t w, float from, float to) {
    float x[4];
    decode4(w, x);
    return encode4(x, 1.f, from / to);
  }
  static __device__ __forceinline__ uint32_t largest4(uint32_t w) {            // order key of the largest magnitude of 4 codes
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, (w >> (8 * i)) & 0x7Fu);
    return m;
  }
  static __device__ __forceinline__ float magnitude(uint32_t key) {
    return __builtin_amdgcn_cvt_pk_f32_fp8((int)key, false)[0];
  }
  // four codes as f16, two pairs
  static __device__ __forceinline__ void to_half(uint32_t w, h2 *lo, h2 *hi) {
    *lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
    *hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
  }
  // four codes times a power of two as bf16 (exact within its range), in two words
  static __device__ __forceinline__ void to_bf16(uint32_t w, float scale, uint32_t *out) {
    out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  }
};

// Integers: the scale is amax / 127 rounded to float.  A code is the integer nearest to the true quotient; the float product
// decides unless it comes within 1e-4 of a half (its error is below 4e-5), where the division in doubles does.
template <>
struct Code<SPINDLE_I8> {
  static __device__ __forceinline__ float scale_for(float amax) { return fmaxf(amax / 127.f, kTinyScale); }
  static __device__ __forceinline__ int nearest(float x, double by, float t) {
    if (t != t) return 0;
    float r = __builtin_rintf(t = __builtin_amdgcn_fmed3f(t, -128.f, 128.f));
    if (__builtin_fabsf(__builtin_fabsf(t - r) - 0.5f) < 1e-4f) r = (float)__builtin_rint(fmin(fmax((double)x / by, -127.0), 127.0));
    return (int)__builtin_amdgcn_fmed3f(r, -127.f, 127.f);
  }
  static __device__ __forceinline__ uint32_t encode4(const float *x, float s, float rs) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)nearest(x[i], (double)s, x[i] * rs) & 0xFFu) << (8 * i);
    return w;
  }
  static __device__ __forceinline__ uint32_t rescale4(uint32_t w, float from, float to) {
    const float f = from / to;
    uint32_t o = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = (int8_t)(w >> (8 * i));
      const float t = c ? (float)c * f : 0.f;                         // (f overflows where zeros alone go to the smallest scale)
      float r = __builtin_rintf(t);
      if (__builtin_fabsf(__builtin_fabsf(t - r) - 0.5f) < 1e-4f) r = (float)__builtin_rint((double)c * (double)from / (double)to);
      o |= ((uint32_t)(int)__builtin_amdgcn_fmed3f(r, -127.f, 127.f) & 0xFFu) << (8 * i);
    }
    return o;
  }
  static __device__ __forceinline__ uint32_t largest4(uint32_t w) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = (int8_t)(w >> (8 * i));
      m = max(m, (uint32_t)(c < 0 ? -c : c));
    }
    return m;
  }
  static __device__ __forceinline__ float magnitude(uint32_t key) { return (float)key; }
  // as they are (their scales are no powers of two, a product would be rounded): 0x6400 | (c + 128) is the f16 number
  // 1024 + c + 128
  static __device__ __forceinline__ void to_half(uint32_t w, h2 *lo, h2 *hi) {
    w ^= 0x80808080u;
    const h2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
    *lo = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    *hi = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
  }
  // (the 8 bits of an integer fit bf16: the upper half of its float is all of it)
  static __device__ __forceinline__ void to_bf16(uint32_t w, float, uint32_t *out) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
    out[0] = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u);
    out[1] = __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u);
  }
};

}  // namespace spindle
