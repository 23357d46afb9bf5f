// Internal declarations of the operators beside the layers: top logits of a row, the
// distillation loss and group normalisation.
#pragma once

#include "internal.h"

namespace pgcn {

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
#endif

}  // namespace pgcn
