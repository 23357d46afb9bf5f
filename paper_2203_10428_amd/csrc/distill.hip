// Top logits of a row, and the loss of a student's logits against a teacher's top logits
// with its gradient.
//
// With z a row of the student's logits, T the temperature, (y_k, t_k) the teacher's listed
// classes and logits and b the log-sum of its other logits at T:
//     L = log(sum_k e^{t_k / T} + e^b),  p_k = e^{t_k / T - L},  rho = e^{b - L}
//     q = softmax(z / T),  s = sum of q over the classes that are not listed
//     KL = sum_k p_k (log p_k - log q_{y_k}) + rho (log rho - log s)
//     d KL / d z_c = (q_c - p_c) / T            where c is listed
//                    q_c (1 - rho / s) / T      elsewhere
// The sum s is formed from the unlisted classes themselves, with their own maximum: 1 minus
// the listed ones would lose s where the student is sure of its answer.
#include <algorithm>

#include "ops.h"

namespace pgcn {

namespace {

constexpr float kNegInf = -INFINITY;

// ------------------------------------------------------------- log-sums ----

// sum of e^{(x - m) a} over some x, with m their maximum (s == 0: none but -inf seen)
struct LogSum {
  float m, s;
};
constexpr LogSum kNothing = {kNegInf, 0.f};

__device__ __forceinline__ float exp_diff(float x, float m, float a) { return x == kNegInf ? 0.f : __expf((x - m) * a); }

// A NaN leaves m and makes s NaN.
__device__ __forceinline__ void add(LogSum &l, float x, float a) {
  if (x == kNegInf) return;
  const float m = fmaxf(l.m, x);
  l.s = l.s * exp_diff(l.m, m, a) + __expf((x - m) * a);
  l.m = m;
}

__device__ __forceinline__ LogSum merge(const LogSum &x, const LogSum &y, float a) {
  LogSum r;
  r.m = fmaxf(x.m, y.m);
  r.s = x.s * exp_diff(x.m, r.m, a) + y.s * exp_diff(y.m, r.m, a);
  return r;
}

template <int kLanes>
__device__ __forceinline__ LogSum lanes_merge(LogSum l, float a) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    LogSum y;
    y.m = __shfl_xor(l.m, o, 64);
    y.s = __shfl_xor(l.s, o, 64);
    l = merge(l, y, a);
  }
  return l;
}

// Over a workgroup of kThreads: every thread gets the result.  `part` is not reused by the
// next call without a barrier in between.
template <int kThreads>
__device__ __forceinline__ LogSum block_merge(LogSum l, float a, LogSum *part) {
  l = lanes_merge<64>(l, a);
  if (kThreads == 64) return l;
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = l;
  __syncthreads();
  LogSum r = part[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) r = merge(r, part[w], a);
  return r;
}

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
  l = block_merge<256>(l, inv_t, part);
  if (threadIdx.x == 0) a.tail_lse[r] = l.m * inv_t + __logf(l.s);
}

// ---------------------------------------------------------- distillation ---

// What the gradient needs of a row: see the formulas above.  All exponents are taken
// relative to a maximum, in the logits' own units.
struct RowStats {
  float m;          // maximum of the student's row
  float log_all;    // log sum e^{(z - m) / T}
  float m_rest, inv_rest, rest_gain;  // unlisted: e^{(z - m_rest) / T} inv_rest rest_gain = q (1 - rho / s)
  float mt, log_t;  // teacher: p_k = e^{(t_k - mt) / T - log_t}
  float rho, log_rho, log_s;
  float inv_hard;   // 1 / sum e^{z - m}
  float log_hard;
  bool soft;        // the teacher lists something
};

__device__ __forceinline__ RowStats row_stats(const LogSum &rest, const LogSum &top, const LogSum &teacher,
                                              const LogSum &hard, bool has_tail, float tail, float inv_t) {
  RowStats st;
  const LogSum all = merge(rest, top, inv_t);
  st.m = all.m;
  st.log_all = __logf(all.s);
  st.soft = teacher.s != 0.f;                      // NaN counts: it has to show
  st.mt = teacher.m;
  st.log_rho = kNegInf;
  if (has_tail && tail != kNegInf) {
    const float b = tail - teacher.m * inv_t;      // e^b beside the listed ones' sum
    const float top_ = fmaxf(b, 0.f);
    st.log_t = top_ + __logf(teacher.s * __expf(-top_) + __expf(b - top_));
    st.log_rho = b - st.log_t;
    st.rho = __expf(st.log_rho);
  } else {
    st.log_t = __logf(teacher.s);
    st.rho = 0.f * st.log_t;                       // a NaN among the listed values spreads to the row
  }
  st.m_rest = rest.m;
  const bool some = rest.s != 0.f;
  st.log_s = some ? (rest.m - all.m) * inv_t + __logf(rest.s) - st.log_all : kNegInf;
  st.inv_rest = some ? 1.0f / rest.s : 0.f;
  st.rest_gain = __expf(st.log_s) - st.rho;        // s - rho
  st.log_hard = __logf(hard.s);
  st.inv_hard = 1.0f / hard.s;
  return st;
}

__device__ __forceinline__ float kl_term(float p, float log_p, float log_q) { return p > 0.f ? p * (log_p - log_q) : (p == 0.f ? 0.f : p); }

// One workgroup per row, the row read twice.
template <class T>
__global__ __launch_bounds__(256) void distill_rows_kernel(pgcn_distill_args a, float *row_loss) {
  extern __shared__ uint32_t listed[];             // a bit for every class: listed by the teacher
  __shared__ LogSum part[4][4];
  __shared__ int ids[PGCN_MAX_TOP];
  __shared__ float wave_loss[4];
  __shared__ int bad;
  const int64_t r = blockIdx.x;
  const int C = a.classes, K = a.top, k = threadIdx.x, lane = k % 64, wave = k / 64;
  const typename T::type *z = (const typename T::type *)a.Z + r * a.ld;
  typename T::type *j = (typename T::type *)a.J + r * a.ld;
  const float inv_t = 1.0f / a.temperature;

  for (int w = k; w < (C + 31) / 32; w += 256) listed[w] = 0;
  int id = -1;
  float t = kNegInf, zk = kNegInf;
  if (k < K) {
    id = a.top_ids[r * a.ld_top + k];
    t = a.top_values[r * a.ld_top + k];
  }
  if (k == 0) bad = 0;
  if (k < PGCN_MAX_TOP) ids[k] = id;
  __syncthreads();
  if (id >= C) {
    bad = 1;                                       // every writer writes the same value
    id = -1;
  }
  for (int i = 0; i < k && i < K; ++i)
    if (ids[i] == id) id = -1;                     // listed before: the lowest slot counts
  if (id >= 0) {
    atomicOr(&listed[id / 32], 1u << (id % 32));
    zk = T::get(z + id);
  } else {
    t = kNegInf;
  }
  const int y = a.labels ? a.labels[r] : -1;
  const bool has_y = y >= 0 && y < C;
  __syncthreads();

  LogSum rest = kNothing, hard = kNothing, top = kNothing, teacher = kNothing;
  for (int c = k; c < C; c += 256) {
    const float x = T::get(z + c);
    if (!((listed[c / 32] >> (c % 32)) & 1u)) add(rest, x, inv_t);
    add(hard, x, 1.0f);
  }
  add(top, zk, inv_t);
  add(teacher, t, inv_t);
  rest = block_merge<256>(rest, inv_t, part[0]);
  hard = block_merge<256>(hard, 1.0f, part[1]);
  top = block_merge<256>(top, inv_t, part[2]);
  teacher = block_merge<256>(teacher, inv_t, part[3]);
  const RowStats st = row_stats(rest, top, teacher, hard, a.tail_lse != nullptr, a.tail_lse ? a.tail_lse[r] : 0.f, inv_t);

  const float soft = st.soft ? a.soft_scale * inv_t : 0.f, hs = has_y ? a.hard_scale : 0.f;
  for (int c = k; c < C; c += 256) {
    if ((listed[c / 32] >> (c % 32)) & 1u) continue;
    const float x = T::get(z + c);
    float g = 0.f;
    if (st.soft) g = soft * exp_diff(x, st.m_rest, inv_t) * st.inv_rest * st.rest_gain;
    if (has_y) g += hs * (exp_diff(x, st.m, 1.0f) * st.inv_hard - (c == y ? 1.f : 0.f));
    T::put(j + c, g);
  }
  float loss = 0.f;
  if (id >= 0) {
    float g = 0.f;
    if (st.soft) {
      const float log_p = (t - st.mt) * inv_t - st.log_t, p = t == kNegInf ? 0.f : __expf(log_p);
      const float log_q = (zk - st.m) * inv_t - st.log_all;
      loss = a.soft_scale * kl_term(p, log_p, log_q);
      g = soft * (__expf(log_q) - p);
    }
    if (has_y) g += hs * (exp_diff(zk, st.m, 1.0f) * st.inv_hard - (id == y ? 1.f : 0.f));
    T::put(j + id, g);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) loss += __shfl_xor(loss, o, 64);
  if (lane == 0) wave_loss[wave] = loss;
  __syncthreads();
  if (k == 0) {
    loss = wave_loss[0] + wave_loss[1] + wave_loss[2] + wave_loss[3];
    if (st.soft) loss += a.soft_scale * kl_term(st.rho, st.log_rho, st.log_s);
    if (has_y) loss += hs * (st.m + st.log_hard - T::get(z + y));
    if (bad || (y != -1 && !has_y)) loss = __builtin_nanf("");  // an id out of range poisons the loss
    row_loss[r] = loss;
  }
}

// Sum of the rows' losses in a fixed order, fp64.
__global__ __launch_bounds__(1024) void distill_sum_kernel(const float *row_loss, int64_t rows, float *out) {
  __shared__ double part[1024];
  double s = 0.0;
  for (int64_t r = threadIdx.x; r < rows; r += 1024) s += (double)row_loss[r];
  part[threadIdx.x] = s;
  __syncthreads();
  for (int w = 512; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) *out = (float)part[0];
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

size_t distill_workspace(int32_t, int64_t rows, int32_t, int32_t) { return (size_t)rows * sizeof(float); }

int launch_distill(const pgcn_distill_args &a, hipStream_t s) {
  TraceScope ts(PGCN_TK_DISTILL, s);
  float *row_loss = (float *)a.workspace;
  if (a.rows > 0) {
    const size_t lds = (size_t)((a.classes + 31) / 32) * 4;
    if (a.dtype == PGCN_BF16)
      hipLaunchKernelGGL(distill_rows_kernel<BF16>, dim3((unsigned)a.rows), dim3(256), lds, s, a, row_loss);
    else
      hipLaunchKernelGGL(distill_rows_kernel<F32>, dim3((unsigned)a.rows), dim3(256), lds, s, a, row_loss);
    PGCN_HIP(hipGetLastError());
  }
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, row_loss, a.rows, a.loss_out);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
