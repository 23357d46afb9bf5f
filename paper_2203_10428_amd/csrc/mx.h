// Device helpers of rows in 8 and 4 bits (pgcn.h: blocks of 32 elements, one power of two each).
#pragma once

#include "ops.h"

namespace pgcn {

struct Int8 {
  static constexpr int kFormat = PGCN_MX_INT8, kBytes = 32;      // bytes of a block
};
struct Fp4 {
  static constexpr int kFormat = PGCN_MX_FP4, kBytes = 16;
};

// What a launch over the chunks of many rows needs to find a chunk's row: flat chunk index = row per + chunk.
// A workgroup divides its first index once; its threads' are at most 2^11 further.
struct Chunks {
  int64_t total;
  uint32_t per, magic;      // magic: 2^32 / per rounded up, for per < 2048
};
inline Chunks chunks_of(int64_t rows, int64_t per) {
  Chunks c;
  c.total = rows * per;
  c.per = (uint32_t)per;
  c.magic = per > 1 && per < 2048 ? (uint32_t)(((uint64_t(1) << 32) + per - 1) / per) : 0;
  return c;
}

#ifdef __HIPCC__
// x / per of x < per + 2048: exact by the rounded-up reciprocal while x per < 2^32; a larger per goes in at most once.
__device__ __forceinline__ uint32_t chunk_row(const Chunks &c, uint32_t x) {
  if (c.per >= 2048) return x >= c.per ? 1u : 0u;
  return c.per == 1 ? x : __umulhi(x, c.magic);
}

// The scale's byte of a block whose largest magnitude has the bits m (sign cleared).
// INT8: q = m 2^(133 - s) rounds to 128 from 127.5 on, a mantissa of 1.9921875: adding what is missing to 2
// carries into the exponent there.  Below 2^-126 the scale is the smallest one, or the next from 127.5 2^-133 on.
// FP4: 7 is halfway to 8, which there is not: a mantissa of 1.75.
template <class F>
__device__ __forceinline__ uint32_t scale_byte(uint32_t m) {
  if (m >= 0x7f800000u) return 255u;
  if (F::kFormat == PGCN_MX_INT8) {
    if (m < 0x00800000u) return m >= 0x007f8000u ? 1u : 0u;
    return min(254u, (m + 0x10000u) >> 23);
  }
  const uint32_t t = (m + 0x200000u) >> 23;
  return t < 2u ? 0u : min(252u, t - 2u);
}

// 2^(s - 127) as a float (a subnormal one for s = 0)
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s == 0u ? 0x00400000u : s << 23); }

// What one step of an INT8 block is worth: 2^(s - 133), NaN for 255.
__device__ __forceinline__ float int8_step(uint32_t s) {
  return s == 255u ? __uint_as_float(0x7fc00000u) : __builtin_ldexpf(1.f, (int)s - 133);
}

// Eight elements of a block as bytes.  INT8: x 2^(133 - s) + 1.5 2^23 in one product-sum, rounded once to nearest
// even: its low byte is q.  Scales that are no float, and the one where values are cut off, take the longer way.
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
__device__ __forceinline__ op_u32x2 pack8(Int8, const float (&x)[8], uint32_t s) {
  uint32_t q[8];
  if (s >= 6u && s <= 253u) {
    const float f = __uint_as_float((260u - s) << 23);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = __float_as_uint(__builtin_fmaf(x[e], f, 12582912.f));
  } else if (s != 255u) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      q[e] = (uint32_t)(int)fminf(fmaxf(__builtin_rintf(__builtin_ldexpf(x[e], 133 - (int)s)), -127.f), 127.f);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = 0u;
  }
  return op_u32x2{bytes4(q[0], q[1], q[2], q[3]), bytes4(q[4], q[5], q[6], q[7])};
}
__device__ __forceinline__ uint32_t pack8(Fp4, const float (&x)[8], uint32_t s) {
  if (s == 255u) return 0u;
  const float f = scale_of(s);
  uint32_t v = 0u;       // rounded to nearest even, cut off at 6, signs of zeros kept
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[0], x[1], f, 0);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[2], x[3], f, 1);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[4], x[5], f, 2);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[6], x[7], f, 3);
  return v;
}

// Four elements of a block from their bytes, in the low ones of q.
__device__ __forceinline__ void unpack4(Int8, uint32_t q, uint32_t s, float *v) {
  const float step = int8_step(s);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)(int)(int8_t)(q >> (8 * e)) * step;
}
__device__ __forceinline__ void unpack4(Fp4, uint32_t q, uint32_t s, float *v) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const float f = scale_of(s);
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, f, 1);
  const float w[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = s == 255u ? __uint_as_float(0x7fc00000u) : w[e];
}
// Four or eight of them from memory.
template <int E>
__device__ __forceinline__ void unpack(Int8, const uint8_t *q, uint32_t s, float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < E / 4; ++i) unpack4(Int8{}, reinterpret_cast<const uint32_t *>(q)[i], s, v + 4 * i);
}
template <int E>
__device__ __forceinline__ void unpack(Fp4, const uint8_t *q, uint32_t s, float (&v)[E]) {
  const uint32_t bits = E == 4 ? *reinterpret_cast<const uint16_t *>(q) : *reinterpret_cast<const uint32_t *>(q);
#pragma unroll
  for (int i = 0; i < E / 4; ++i) unpack4(Fp4{}, bits >> (16 * i), s, v + 4 * i);
}
template <class F>
struct Bits8;      // the bytes of eight elements
template <>
struct Bits8<Int8> {
  typedef op_u32x2 type;
};
template <>
struct Bits8<Fp4> {
  typedef uint32_t type;
};

// n (may be <= 0 or > 8) of eight neighbouring elements from a 16-byte aligned place, zeros for the rest; no
// vector is read that holds none of them.  kOnce: the line is read once and need not stay in a cache.
template <bool kOnce, class V>
__device__ __forceinline__ V load_vector(const void *p) {
  if constexpr (kOnce) return __builtin_nontemporal_load((const V *)p);
  else return *(const V *)p;
}
template <bool kOnce>
__device__ __forceinline__ void load8(F32, const float *p, int64_t n, float (&v)[8]) {
  const op_f32x4 none = {0.f, 0.f, 0.f, 0.f};
  const op_f32x4 a = n > 0 ? load_vector<kOnce, op_f32x4>(p) : none;
  const op_f32x4 b = n > 4 ? load_vector<kOnce, op_f32x4>(p + 4) : none;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? (e < 4 ? a[e % 4] : b[e % 4]) : 0.f;
}
template <bool kOnce>
__device__ __forceinline__ void load8(BF16, const uint16_t *p, int64_t n, float (&v)[8]) {
  const op_u32x4 none = {0u, 0u, 0u, 0u};
  const op_u32x4 a = n > 0 ? load_vector<kOnce, op_u32x4>(p) : none;
  BF16::unpack(a, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? v[e] : 0.f;
}
#endif

}  // namespace pgcn
