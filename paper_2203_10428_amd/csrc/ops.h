// Internal declarations of the operators beside the layers: top logits of a row, the
// distillation loss and group normalisation.
#pragma once

#include "internal.h"

namespace pgcn {

// Threads of one launch: grids are counted in 32 bits of threads.
constexpr int64_t kMaxLaunch = int64_t(1) << 31;

// ---- kernel launchers (arguments already checked by the entry points) ------
int launch_top_logits(const pgcn_top_logits_args &a, hipStream_t s);
size_t top_logits_workspace(int32_t dtype, int64_t rows, int32_t classes, int32_t top);
int launch_distill(const pgcn_distill_args &a, hipStream_t s);
size_t distill_workspace(int32_t dtype, int64_t rows, int32_t classes, int32_t top);
int launch_group_norm_fwd(const pgcn_group_norm_fwd_args &a, hipStream_t s);
int launch_group_norm_bwd(const pgcn_group_norm_bwd_args &a, hipStream_t s);
size_t group_norm_workspace(int32_t dtype, int32_t channels, int32_t groups, int64_t samples, int64_t sample_rows);

#ifdef __HIPCC__
// ---- device helpers ---------------------------------------------------------

// A row's elements in 16-byte vectors: 4 floats or 8 bf16 values, computed on as floats.
typedef float op_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t op_u32x4 __attribute__((ext_vector_type(4)));

struct F32 {
  typedef float type;
  typedef op_f32x4 raw;
  static constexpr int E = 4;
  static __device__ __forceinline__ void unpack(const raw &r, float (&v)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = r[e];
  }
  static __device__ __forceinline__ raw pack(const float (&v)[E]) { return raw{v[0], v[1], v[2], v[3]}; }
  static __device__ __forceinline__ float get(const type *p) { return *p; }
  static __device__ __forceinline__ void put(type *p, float x) { *p = x; }
};

// bf16 bits; float -> bf16 rounds to nearest even (one rounding per stored value)
struct BF16 {
  typedef uint16_t type;
  typedef op_u32x4 raw;
  static constexpr int E = 8;
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ uint32_t two(float a, float b) {
    const pair p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
  }
  static __device__ __forceinline__ void unpack(const raw &r, float (&v)[E]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ raw pack(const float (&v)[E]) {
    return raw{two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7])};
  }
  static __device__ __forceinline__ float get(const type *p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ void put(type *p, float x) { *p = (uint16_t)two(x, 0.f); }
};

// Stores the first n (1 .. E) elements of a vector: whole, or one by one at a row's end, so
// that nothing past the row's columns is written.
template <class T>
__device__ __forceinline__ void store_some(typename T::type *p, const float (&v)[T::E], int n) {
  if (n >= T::E) {
    *reinterpret_cast<typename T::raw *>(p) = T::pack(v);
  } else {
#pragma unroll
    for (int e = 0; e < T::E; ++e)
      if (e < n) T::put(p + e, v[e]);
  }
}

// Keeps the packed vectors, and not what one pass over them computed, in registers for the next.
template <class Raw, int kVecs>
__device__ __forceinline__ void keep_packed(Raw (&raw)[kVecs]) {
#pragma unroll
  for (int i = 0; i < kVecs; ++i) asm volatile("" : "+v"(raw[i]));
}

// ---- log-sums ---------------------------------------------------------------

constexpr float kNegInf = -INFINITY;

// sum of e^{(x - m) a} over some x, with m their maximum (s == 0: none but -inf seen)
struct LogSum {
  float m, s;
};

__device__ __forceinline__ float exp_diff(float x, float m, float a) { return x == kNegInf ? 0.f : __expf((x - m) * a); }

__device__ __forceinline__ LogSum merge(const LogSum &x, const LogSum &y, float a) {
  LogSum r;
  r.m = fmaxf(x.m, y.m);
  r.s = x.s * exp_diff(x.m, r.m, a) + y.s * exp_diff(y.m, r.m, a);
  return r;
}

constexpr float kLog2e = 1.44269504088896341f;

// e^{(x - m) T'} with scale = T' log2 e; 0 for x = -inf (m finite)
__device__ __forceinline__ float exp_at(float x, float m, float scale) { return __builtin_amdgcn_exp2f((x - m) * scale); }

// e^{(x - m) T'} for many x: one product-sum each, 2^{x scale - shift} fix, where fix takes up what
// shift = m scale was rounded by: at most 32 below 2^30, so that 2^{m scale - shift}, fix and sums of
// 2^18 such terms are in range.  From 2^30 on (a finite mask value or a far offset at a low temperature)
// a neighbour of m is 2^6 exponents away or more, and any scale that leaves it there gives the same 1
// and 0: the power of two that brings m to [2^30, 2^31), with which m scale is not rounded at all.
struct Exps {
  float scale, shift, fix;
  __device__ __forceinline__ Exps(float m, float scale_) {
    const uint32_t exponent = (__float_as_uint(m) >> 23) & 0xff;
    scale = fabsf(m * scale_) < 0x1p30f ? scale_ : __uint_as_float((2 * 127 + 30 - exponent) << 23);
    shift = m * scale;
    fix = __builtin_amdgcn_exp2f(-__builtin_fmaf(m, scale, -shift));
  }
  __device__ __forceinline__ float raw(float x) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale, -shift)); }
};

// ---- sums and maxima over neighbouring lanes --------------------------------
//
// kLanes (a power of two up to 64) lanes each get the result: the first four steps are register
// moves within rows of 16 lanes (exchange in pairs, in quads, mirrored halves, mirrored row), the
// rest shuffles.  Every lane adds the same pairs, so all hold the same bits.
template <int kCtrl>
__device__ __forceinline__ float lane_move(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), kCtrl, 0xf, 0xf, true));
}

template <int kLanes, class Op>
__device__ __forceinline__ float lanes_all(float v, Op op) {
  if (kLanes >= 2) v = op(v, lane_move<0xB1>(v));
  if (kLanes >= 4) v = op(v, lane_move<0x4E>(v));
  if (kLanes >= 8) v = op(v, lane_move<0x141>(v));
  if (kLanes >= 16) v = op(v, lane_move<0x140>(v));
  if (kLanes >= 32) v = op(v, __shfl_xor(v, 16, 64));
  if (kLanes >= 64) v = op(v, __shfl_xor(v, 32, 64));
  return v;
}

template <int kLanes>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_all<kLanes>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_all<kLanes>(v, [](float a, float b) { return a + b; });
}

// Orders the LDS accesses of a wave's lanes (they are executed in order; this keeps the compiler from moving them).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
#endif

}  // namespace pgcn
