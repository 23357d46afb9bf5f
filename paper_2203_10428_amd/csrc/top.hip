// The largest logits of every row with their classes, and the log-sum of the others.
#include <algorithm>

#include "ops.h"

namespace pgcn {

namespace {

// ------------------------------------------------------------ top logits ---

// Order of (value, lowest class first) as whole numbers; -0 counts as +0.  0: never chosen
// (-inf and NaN).
__device__ __forceinline__ uint64_t top_key(float x, int c) {
  if (!(x > kNegInf)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (uint32_t)~c;
}

__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ int key_class(uint64_t k) { return (int)~(uint32_t)k; }

// One workgroup per row; every listed class is found by a pass over the row.
template <class T>
__global__ __launch_bounds__(256) void top_rows_kernel(pgcn_top_logits_args a) {
  __shared__ uint64_t best[4];
  __shared__ LogSum part[4];
  const int64_t r = blockIdx.x;
  const int C = a.classes, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const typename T::type *z = (const typename T::type *)a.Z + r * a.ld;
  uint64_t last = ~(uint64_t)0;
  for (int k = 0; k < a.top; ++k) {
    uint64_t m = 0;
    for (int c = threadIdx.x; c < C; c += 256) {
      const uint64_t key = top_key(T::get(z + c), c);
      if (key < last && key > m) m = key;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t y = __shfl_xor((unsigned long long)m, o, 64);
      m = y > m ? y : m;
    }
    __syncthreads();
    if (lane == 0) best[wave] = m;
    __syncthreads();
    m = best[0];
    for (int w = 1; w < 4; ++w) m = best[w] > m ? best[w] : m;
    if (threadIdx.x == 0) {
      a.top_values[r * a.ld_top + k] = m ? key_value(m) : kNegInf;
      a.top_ids[r * a.ld_top + k] = m ? key_class(m) : -1;
    }
    last = m;
  }
  if (!a.tail_lse) return;
  const float inv_t = 1.0f / a.temperature;
  LogSum l = kNothing;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float x = T::get(z + c);
    if (top_key(x, c) < last || x != x) add(l, x, inv_t);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l = merge(l, LogSum{__shfl_xor(l.m, o, 64), __shfl_xor(l.s, o, 64)}, inv_t);
  if (lane == 0) part[wave] = l;
  __syncthreads();
  l = merge(merge(part[0], part[1], inv_t), merge(part[2], part[3], inv_t), inv_t);
  if (threadIdx.x == 0) a.tail_lse[r] = l.m * inv_t + __logf(l.s);
}

}  // namespace

size_t top_logits_workspace(int32_t, int64_t, int32_t, int32_t) { return 0; }

int launch_top_logits(const pgcn_top_logits_args &a, hipStream_t s) {
  if (a.rows == 0) return PGCN_OK;
  TraceScope ts(PGCN_TK_TOP_LOGITS, s);
  if (a.dtype == PGCN_BF16)
    hipLaunchKernelGGL(top_rows_kernel<BF16>, dim3((unsigned)a.rows), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(top_rows_kernel<F32>, dim3((unsigned)a.rows), dim3(256), 0, s, a);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
