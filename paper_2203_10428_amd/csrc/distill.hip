// The loss of a student's logits against a teacher's top logits, with its gradient.
//
// With z a row of the student's logits, T the temperature, (y_k, t_k) the teacher's listed
// classes and logits and b the log-sum of its other logits at T:
//     L = log(sum_k e^{t_k / T} + e^b),  p_k = e^{t_k / T - L},  rho = e^{b - L}
//     q = softmax(z / T),  s = sum of q over the classes that are not listed
//     KL = sum_k p_k (log p_k - log q_{y_k}) + rho (log rho - log s)
//     d KL / d z_c = (q_c - p_c) / T            where c is listed
//                    q_c (1 - rho / s) / T      elsewhere
// The sum s is formed from the unlisted classes themselves, with their own maximum: 1 minus
// the listed ones would lose s where the student is sure of its answer.  All sums and the
// loss are fp32 over a row, fp64 over the rows.
//
// Bound by one read of Z and one write of J.  A row stays in registers between its sums and
// its gradient: in a few lanes of a wave (up to 2,048 classes), in a workgroup (up to 32,768
// fp32 or 65,536 bf16 classes).  Longer rows, and few long ones, are cut into parts and read twice.
#include <algorithm>

#include "ops.h"

namespace pgcn {

namespace {

// a maximum to subtract: 0 where there was nothing but -inf
__device__ __forceinline__ float base_of(float m) { return m == kNegInf ? 0.f : m; }

// What the loss and the gradient need of a row: see the formulas above.  Exponents are taken
// relative to a maximum, in the logits' own units.
struct RowStats {
  float m, log_all;       // of the student's row: maximum, log sum e^{(z - m) / T}
  float m_rest, log_s;    // unlisted: maximum, log of their share s
  float gain;             // unlisted: d KL / d z T = e^{(z - m_rest) / T} gain
  float mt, log_t;        // teacher: p_k = e^{(t_k - mt) / T - log_t}
  float rho, log_rho;
  float inv_hard, log_hard;   // sum e^{z - m}: its reciprocal, its logarithm
  bool soft;              // the teacher lists something, and its term counts
  bool some;              // there is an unlisted logit above -inf
};

// `two`: `hard` is the sum of e^{z - m}; else the temperature is 1 (or no row has a label) and the soft sum is it.
__device__ __forceinline__ RowStats row_stats(const LogSum &rest, const LogSum &top, const LogSum &teacher, bool two, float hard, float m,
                                              float tail, float inv_t, float soft_scale) {
  RowStats st;
  const LogSum all = merge(rest, top, inv_t);
  st.m = m;
  st.log_all = __logf(all.s);
  st.soft = teacher.s != 0.f && soft_scale != 0.f; // NaN counts: it has to show
  st.mt = base_of(teacher.m);
  if (tail != kNegInf) {
    const float b = tail - st.mt * inv_t;          // e^b beside the listed ones' sum
    const float big = fmaxf(b, 0.f);
    st.log_t = big + __logf(teacher.s * __expf(-big) + __expf(b - big));
    st.log_rho = b - st.log_t;
    st.rho = __expf(st.log_rho);
  } else {
    st.log_t = __logf(teacher.s);
    st.log_rho = kNegInf;
    st.rho = 0.f * st.log_t;                       // a NaN among the listed values spreads to the row
  }
  st.m_rest = base_of(rest.m);
  st.some = rest.s != 0.f;
  st.log_s = st.some ? (rest.m - all.m) * inv_t + __logf(rest.s) - st.log_all : kNegInf;
  st.gain = st.some ? (__expf(st.log_s) - st.rho) * __builtin_amdgcn_rcpf(rest.s) : 0.f;
  st.log_hard = two ? __logf(hard) : st.log_all;
  st.inv_hard = __builtin_amdgcn_rcpf(two ? hard : all.s);
  return st;
}

__device__ __forceinline__ float kl_term(float p, float log_p, float log_q) {
  return p > 0.f ? p * (log_p - log_q) : (p == 0.f ? 0.f : p);
}

// A listed class: its loss term, and its gradient without the one-hot part.
__device__ __forceinline__ float listed_term(const RowStats &st, float t, float z, float inv_t, float soft, float hard, float soft_scale,
                                             float &loss) {
  float g = 0.f;
  if (st.soft) {
    const float log_p = (t - st.mt) * inv_t - st.log_t, p = t == kNegInf ? 0.f : __expf(log_p);
    const float log_q = (z - st.m) * inv_t - st.log_all;
    loss = soft_scale * kl_term(p, log_p, log_q);
    g = soft * (__expf(log_q) - p);
  }
  if (hard != 0.f) g += hard * (z == kNegInf ? 0.f : __expf(z - st.m)) * st.inv_hard;
  return g;
}

// The row's loss beside its listed terms.
__device__ __forceinline__ float row_loss(const RowStats &st, float listed, float z_label, bool has_label, bool poison, float soft_scale,
                                          float hard) {
  float l = listed;
  if (st.soft) l += soft_scale * kl_term(st.rho, st.log_rho, st.log_s);
  if (has_label && hard != 0.f) l += hard * ((st.m - z_label) + st.log_hard);     // m + log would round the logarithm to m's digits
  return poison ? __builtin_nanf("") : l;          // an id or label out of range
}

// ---- short rows: kLanes lanes of a wave hold a row, kVecs vectors each ---------------------
//
// What a row costs besides its elements (reductions, logarithms) is spent by every lane, so few
// lanes take a row: about 16 elements each, down to 4 lanes.  The row's image in LDS serves the
// listed classes, kSlots to a lane: their logits are read from it, and their gradients written
// into it for the lane that holds the class.
// Bound by instructions, up to about 100 classes by a row's fixed ones: vector instructions are issued in
// 0.80 of all cycles of 306,000 x 47 top 16 bf16, 34 us (2.8 TB/s), 0.60 in fp32, 43.5 us (3.6), and 0.46 of
// 58,000 x 41 top 8 fp32, 11.7 us (2.0), at 3.5 waves to a SIMD.  100,000 x 128 top 8 fp32 24.4 (4.5),
// 10,000 x 2,000 top 64 fp32 40 (4.1), bf16 31 (2.7).

template <class T, int kLanes, int kVecs, int kSlots>
__global__ __launch_bounds__(256) void distill_short_kernel(pgcn_distill_args a, double *part) {
  constexpr int kWide = kLanes * kVecs * T::E, kRows = 256 / kLanes;
  constexpr int kStride = kWide + 4;               // neighbouring rows begin in other banks
  constexpr int kWords = (kWide + 31) / 32;
  __shared__ __align__(16) float image_[kRows * kStride];
  __shared__ uint32_t bits_[kRows * kWords];
  __shared__ double sums[kRows];
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes, C = a.classes, K = a.top;
  float *image = image_ + slot * kStride;
  uint32_t *bits = bits_ + slot * kWords;
  const float inv_t = 1.0f / a.temperature, scale_t = inv_t * kLog2e;
  const bool same = a.temperature == 1.0f;         // the hard term's exponentials are the soft ones
  const bool two = !same && a.labels;
  double total = 0.0;

  for (int64_t r = (int64_t)blockIdx.x * kRows + slot; r < a.rows; r += (int64_t)gridDim.x * kRows) {
    const typename T::type *zr = (const typename T::type *)a.Z + r * a.ld;
    float x[kVecs][T::E];
    typename T::raw raw[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int c0 = (lane + kLanes * i) * T::E;
      raw[i] = c0 < C ? *reinterpret_cast<const typename T::raw *>(zr + c0) : typename T::raw{};
    }
    int id[kSlots];
    float t[kSlots], zk[kSlots];
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int k = lane + kLanes * i;
      id[i] = k < K ? a.top_ids[r * a.ld_top + k] : -1;
      t[i] = k < K ? a.top_values[r * a.ld_top + k] : kNegInf;
    }
    const int y = a.labels ? a.labels[r] : -1;
    const float tail = a.tail_lse ? a.tail_lse[r] : kNegInf;
    const bool has_y = y >= 0 && y < C;
    bool bad = y != -1 && !has_y;

    wave_sync();                                   // the row before is done with its image
#pragma unroll
    for (int w = 0; w < kWords; w += kLanes)
      if (w + lane < kWords) bits[w + lane] = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int c0 = (lane + kLanes * i) * T::E;
      T::unpack(raw[i], x[i]);
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        if (c0 + e >= C) x[i][e] = kNegInf;
        image[c0 + e] = x[i][e];
      }
    }
    wave_sync();
    bool twice = false;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      if (id[i] >= C) {
        bad = true;
        id[i] = -1;
      }
      if (id[i] >= 0) twice |= (atomicOr(&bits[id[i] / 32], 1u << (id[i] % 32)) >> (id[i] % 32)) & 1u;
    }
    if (__any(twice)) {                            // of equal ids the lowest slot counts
      int keep[kSlots];
#pragma unroll
      for (int i = 0; i < kSlots; ++i) keep[i] = id[i];
      for (int o = 0; o < kLanes; ++o)
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
          const int other = __shfl(id[j], o, kLanes);
#pragma unroll
          for (int i = 0; i < kSlots; ++i)
            if (other == id[i] && o + kLanes * j < lane + kLanes * i) keep[i] = -1;
        }
#pragma unroll
      for (int i = 0; i < kSlots; ++i) id[i] = keep[i];
    }
    wave_sync();
    float mt = kNegInf, m_top = kNegInf, m_rest = kNegInf;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      if (id[i] < 0) t[i] = kNegInf;
      zk[i] = id[i] >= 0 ? image[id[i]] : kNegInf;
      mt = fmaxf(mt, t[i]);
      m_top = fmaxf(m_top, zk[i]);
    }
    const float z_label = has_y ? image[y] : 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int c0 = (lane + kLanes * i) * T::E;
      const uint32_t listed = bits[c0 / 32] >> (c0 % 32);
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        x[i][e] = (listed >> e) & 1u ? kNegInf : x[i][e];
        m_rest = fmaxf(m_rest, x[i][e]);
      }
    }
    mt = lanes_max<kLanes>(mt);
    m_top = lanes_max<kLanes>(m_top);
    m_rest = lanes_max<kLanes>(m_rest);
    const float m = fmaxf(m_top, m_rest), bt = base_of(mt), b_top = base_of(m_top), b_rest = base_of(m_rest), b_all = base_of(m);
    float s_t = 0.f, s_top = 0.f, s_rest = 0.f, s_hard = 0.f;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      s_t += exp_at(t[i], bt, scale_t);
      s_top += exp_at(zk[i], b_top, scale_t);
      if (two) s_hard += exp_at(zk[i], b_all, kLog2e);
    }
    if (two) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < T::E; ++e) s_hard += exp_at(x[i][e], b_all, kLog2e);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        x[i][e] = exp_at(x[i][e], b_rest, scale_t);
        s_rest += x[i][e];
      }
    s_t = lanes_sum<kLanes>(s_t);
    s_top = lanes_sum<kLanes>(s_top);
    s_rest = lanes_sum<kLanes>(s_rest);
    const LogSum rest = {m_rest, s_rest}, top = {m_top, s_top};
    if (two) s_hard = lanes_sum<kLanes>(s_hard);
    const RowStats st = row_stats(rest, top, LogSum{mt, s_t}, two, s_hard, m, tail, inv_t, a.soft_scale);
    const float soft = st.soft ? a.soft_scale * inv_t : 0.f, hard = has_y ? a.hard_scale : 0.f;

    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < kSlots; ++i)
      if (id[i] >= 0) {
        float l = 0.f;
        image[id[i]] = listed_term(st, t[i], zk[i], inv_t, soft, hard, a.soft_scale, l);
        loss += l;
      }
    loss = lanes_sum<kLanes>(loss);
    const float any_bad = lanes_max<kLanes>(bad ? 1.f : 0.f);
    wave_sync();
    // unlisted: soft e^{(z - m_rest) / T} gain + hard e^{z - m} / sum
    const float gh = hard != 0.f ? hard * st.inv_hard : 0.f;
    float gs = soft != 0.f ? soft * st.gain : 0.f;
    if (same && gh != 0.f && st.some) gs += gh * exp_at(b_rest, b_all, kLog2e);
    if (has_y && lane == 0) {                      // the label's gradient goes by the image too
      const uint32_t old = atomicOr(&bits[y / 32], 1u << (y % 32));
      float g = image[y];
      if (!((old >> (y % 32)) & 1u)) {
        g = exp_at(z_label, b_rest, scale_t) * gs;
        if (two) g += exp_at(z_label, b_all, kLog2e) * gh;
      }
      image[y] = g - hard;
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int c0 = (lane + kLanes * i) * T::E;
      if (c0 >= C) continue;
      const uint32_t given = bits[c0 / 32] >> (c0 % 32);
      float g[T::E];
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        const float im = image[c0 + e];
        float v = x[i][e] * gs;
        if (two) v += exp_at(im, b_all, kLog2e) * gh;
        g[e] = (given >> e) & 1u ? im : v;
      }
      store_some<T>((typename T::type *)a.J + r * a.ld + c0, g, C - c0);
    }
    if (lane == 0) total += (double)row_loss(st, loss, z_label, has_y, any_bad != 0.f, a.soft_scale, hard);
  }
  if (lane == 0) sums[slot] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kRows; ++i) total += sums[i];
    if (gridDim.x == 1) *a.loss_out = (float)total;
    else part[blockIdx.x] = total;
  }
}

// ---- long rows: a workgroup holds a row, kVecs vectors to a thread --------------------------
//
// The listed classes have a bit each in LDS and are taken out of the threads' vectors (-inf);
// thread k takes slot k, and writes its class's gradient over the one that the vector left.
// Bound by memory: 4,096 x 32,000 top 64 fp32 207 us, 5.1 TB/s, vector instructions in 0.34 of the cycles;
// 1,024 x 32,000 bf16 32 us, 4.1 TB/s, 0.60.
// Without the bound of four waves to a SIMD the scheduler holds more than it has and spills (516 us).

template <int kThreads>
struct ListLds {
  int ids[PGCN_MAX_TOP];
  int twice, bad;
  float m_rest[kThreads / 64], s_rest[kThreads / 64], s_hard[kThreads / 64];
  float m_top[4], m_t[4], s_top[4], s_t[4], s_hard_top[4], loss[4];
};

// Slot threadIdx.x of row r: its class (-1: none, or listed before) in `id`.  Sets a bit for
// every listed class in [first, first + 32 words), seen by all after the call.
template <int kThreads>
__device__ __forceinline__ void list_classes(const pgcn_distill_args &a, int64_t r, uint32_t *bits, int first, int words,
                                             ListLds<kThreads> &l, int &id, float &t) {
  const int k = threadIdx.x, K = a.top;
  id = -1;
  t = kNegInf;
  if (k < K) {
    id = a.top_ids[r * a.ld_top + k];
    t = a.top_values[r * a.ld_top + k];
  }
  for (int w = k; w < words; w += kThreads) bits[w] = 0;
  if (k == 0) l.twice = l.bad = 0;
  __syncthreads();
  if (id >= a.classes) {
    l.bad = 1;                                     // every writer writes the same value
    id = -1;
  }
  if (k < PGCN_MAX_TOP) l.ids[k] = id;
  const int c = id - first;
  if (id >= 0) {
    if (c >= 0 && c < 32 * words) {
      if ((atomicOr(&bits[c / 32], 1u << (c % 32)) >> (c % 32)) & 1u) l.twice = 1;
    } else {
      l.twice = 1;                                 // no bit of its own: compare the ids
    }
  }
  __syncthreads();
  if (l.twice && id >= 0) {                        // of equal ids the lowest slot counts
    bool again = false;
    for (int i = 0; i < k; ++i) again |= l.ids[i] == id;
    if (again) id = -1;
  }
  if (id < 0) t = kNegInf;
}

// -inf for the elements whose bit is set, and from the n-th on.
template <class T>
__device__ __forceinline__ void drop_listed(float (&x)[T::E], uint32_t bits, int n) {
  bits &= (1u << T::E) - 1;
  if (n < T::E) bits |= ~0u << (n > 0 ? n : 0);
  if (bits)                                        // most vectors have none
#pragma unroll
    for (int e = 0; e < T::E; ++e)
      if ((bits >> e) & 1u) x[e] = kNegInf;
}

// The same value, unknown to the compiler: what follows from it is computed anew in each pass over
// a row, and not kept in registers that the row needs.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Maximum and sums over the workgroup, of the listed classes (the first four waves) and the
// others: m_rest is the maximum of the thread's own unlisted logits, rest(base, scale) the sum
// of their e^{(z - base) scale ln 2}, hard(base) of e^{z - base}.
template <int kThreads, class Rest, class Hard>
__device__ __forceinline__ RowStats block_stats(const pgcn_distill_args &a, int64_t r, ListLds<kThreads> &l, float t, float zk,
                                                float m_rest, float inv_t, Rest rest_sum, Hard hard_sum) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const float scale_t = inv_t * kLog2e;
  const bool two = a.labels && a.temperature != 1.0f;      // the hard term has exponentials of its own
  m_rest = lanes_max<64>(m_rest);
  if (lane == 0) l.m_rest[wave] = m_rest;
  if (wave < 4) {
    const float m_top = lanes_max<64>(zk), m_t = lanes_max<64>(t);
    if (lane == 0) {
      l.m_top[wave] = m_top;
      l.m_t[wave] = m_t;
    }
  }
  __syncthreads();
  m_rest = l.m_rest[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m_rest = fmaxf(m_rest, l.m_rest[w]);
  const float m_top = fmaxf(fmaxf(l.m_top[0], l.m_top[1]), fmaxf(l.m_top[2], l.m_top[3]));
  const float m_t = fmaxf(fmaxf(l.m_t[0], l.m_t[1]), fmaxf(l.m_t[2], l.m_t[3]));
  const float m = fmaxf(m_rest, m_top), b_rest = base_of(m_rest), b_all = base_of(m);
  float s_rest = lanes_sum<64>(rest_sum(b_rest, scale_t));
  float s_hard = two ? lanes_sum<64>(hard_sum(b_all)) : 0.f;
  if (lane == 0) {
    l.s_rest[wave] = s_rest;
    l.s_hard[wave] = s_hard;
  }
  if (wave < 4) {
    const float s_top = lanes_sum<64>(exp_at(zk, base_of(m_top), scale_t)), s_t = lanes_sum<64>(exp_at(t, base_of(m_t), scale_t));
    const float s_h = lanes_sum<64>(exp_at(zk, b_all, kLog2e));
    if (lane == 0) {
      l.s_top[wave] = s_top;
      l.s_t[wave] = s_t;
      l.s_hard_top[wave] = s_h;
    }
  }
  __syncthreads();
  s_rest = l.s_rest[0];
  s_hard = l.s_hard[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    s_rest += l.s_rest[w];
    s_hard += l.s_hard[w];
  }
  const LogSum rest = {m_rest, s_rest}, top = {m_top, (l.s_top[0] + l.s_top[1]) + (l.s_top[2] + l.s_top[3])};
  const LogSum teacher = {m_t, (l.s_t[0] + l.s_t[1]) + (l.s_t[2] + l.s_t[3])};
  s_hard += (l.s_hard_top[0] + l.s_hard_top[1]) + (l.s_hard_top[2] + l.s_hard_top[3]);
  return row_stats(rest, top, teacher, two, s_hard, m, a.tail_lse ? a.tail_lse[r] : kNegInf, inv_t, a.soft_scale);
}

template <class T, int kVecs>
__device__ __forceinline__ float vectors_sum(typename T::raw (&raw)[kVecs], float base, float scale) {
  keep_packed(raw);
  const Exps ex(base, scale);
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    float x[T::E];
    T::unpack(raw[i], x);
#pragma unroll
    for (int e = 0; e < T::E; ++e) s[e % 2] += ex.raw(x[e]);
    if (kVecs > 4) __builtin_amdgcn_sched_barrier(0);
  }
  return (s[0] + s[1]) * ex.fix;
}

// Gradient of unlisted logits: soft e^{(z - m_rest) / T} gain + hard e^{z - m} / sum, a factor for
// each exponential, a single one where the temperature is 1.
struct RestGrad {
  Exps rest, all;
  float soft, hard;
  bool two;
  __device__ __forceinline__ RestGrad(const pgcn_distill_args &a, const RowStats &st, float soft_, float hard_, float inv_t)
      : rest(st.m_rest, inv_t * kLog2e), all(base_of(st.m), kLog2e) {
    const float gh = hard_ != 0.f ? hard_ * st.inv_hard : 0.f;
    soft = soft_ != 0.f ? soft_ * st.gain : 0.f;
    two = a.temperature != 1.0f && gh != 0.f;
    hard = two ? gh * all.fix : 0.f;
    if (!two && gh != 0.f && st.some) soft += gh * exp_at(st.m_rest, base_of(st.m), kLog2e);
    soft *= rest.fix;
  }
  template <int N>
  __device__ __forceinline__ void operator()(float (&x)[N]) const {
    if (two) {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = rest.raw(x[e]) * soft + all.raw(x[e]) * hard;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = rest.raw(x[e]) * soft;
    }
  }
  __device__ __forceinline__ float one(float x) const { return rest.raw(x) * soft + (two ? all.raw(x) * hard : 0.f); }
};

// The gradient of a thread's vectors, from class `first` on.
template <class T, int kThreads, int kVecs>
__device__ __forceinline__ void store_vectors(typename T::raw (&raw)[kVecs], const RestGrad &grad, typename T::type *jr, int first,
                                              int C) {
  keep_packed(raw);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c0 = first + ((int)threadIdx.x + kThreads * i) * T::E;
    if (c0 < C) {
      float x[T::E];
      T::unpack(raw[i], x);
      grad(x);
      store_some<T>(jr + c0, x, C - c0);
    }
    __builtin_amdgcn_sched_barrier(0);             // one vector at a time: their temporaries do not add up
  }
}

// What the vectors left out, once they are stored: the listed classes of [first, last), and the label
// if no slot lists it (`bits` begin with class `first`).
template <class T>
__device__ __forceinline__ void store_listed(const RestGrad &grad, typename T::type *jr, int id, float g, int y, float z_label,
                                             float hard, const uint32_t *bits, int first, int last) {
  if (id >= first && id < last) T::put(jr + id, g);
  if (threadIdx.x == 0 && hard != 0.f && y >= first && y < last && !((bits[(y - first) / 32] >> ((y - first) % 32)) & 1u))
    T::put(jr + y, grad.one(z_label) - hard);
}

template <class T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads, 4) void distill_long_kernel(pgcn_distill_args a, double *part) {
  extern __shared__ uint32_t bits[];
  __shared__ ListLds<kThreads> l;
  const int64_t r = blockIdx.x;
  const int C = a.classes, k = threadIdx.x, lane = k % 64, wave = k / 64;
  const typename T::type *zr = (const typename T::type *)a.Z + r * a.ld;
  typename T::type *jr = (typename T::type *)a.J + r * a.ld;
  const float inv_t = 1.0f / a.temperature;
  typename T::raw raw[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c0 = (k + kThreads * i) * T::E;
    raw[i] = c0 < C ? *reinterpret_cast<const typename T::raw *>(zr + c0) : typename T::raw{};
  }
  const int y = a.labels ? a.labels[r] : -1;
  const bool has_y = y >= 0 && y < C;
  int id;
  float t;
  list_classes<kThreads>(a, r, bits, 0, (C + 31) / 32, l, id, t);
  const float zk = id >= 0 ? T::get(zr + id) : kNegInf, z_label = has_y ? T::get(zr + y) : 0.f;
  float m_rest = kNegInf;
  const int n = again(C);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c0 = (k + kThreads * i) * T::E;
    float x[T::E];
    T::unpack(raw[i], x);
    drop_listed<T>(x, (c0 < n ? bits[c0 / 32] : 0u) >> (c0 % 32), n - c0);
#pragma unroll
    for (int e = 0; e < T::E; ++e) m_rest = fmaxf(m_rest, x[e]);
    raw[i] = T::pack(x);                           // exact: values that were read, or -inf
    __builtin_amdgcn_sched_barrier(0);
  }
  auto sum = [&](float base, float scale) { return vectors_sum<T>(raw, base, scale); };
  const RowStats st = block_stats<kThreads>(a, r, l, t, zk, m_rest, inv_t, sum, [&](float base) { return sum(base, kLog2e); });
  const float soft = st.soft ? a.soft_scale * inv_t : 0.f, hard = has_y ? a.hard_scale : 0.f;
  const RestGrad grad(a, st, soft, hard, inv_t);
  store_vectors<T, kThreads>(raw, grad, jr, 0, again(C));
  float loss = 0.f, g = 0.f;
  if (id >= 0) g = listed_term(st, t, zk, inv_t, soft, hard, a.soft_scale, loss) - (id == y ? hard : 0.f);
  if (wave < 4) {
    loss = lanes_sum<64>(loss);
    if (lane == 0) l.loss[wave] = loss;
  }
  __syncthreads();                                 // the vectors' stores come before the listed ones
  store_listed<T>(grad, jr, id, g, y, z_label, hard, bits, 0, C);
  if (k == 0) {
    const float listed = (l.loss[0] + l.loss[1]) + (l.loss[2] + l.loss[3]);
    part[r] = (double)row_loss(st, listed, z_label, has_y, l.bad || (y != -1 && !has_y), a.soft_scale, hard);
  }
}

// ---- parts of a row: few long rows, and rows too long for a workgroup ---------------------------
//
// A first launch leaves every part's maximum and sums, a second one joins a row's parts in each
// of its workgroups and writes the part's gradient.  Bound by the chain of the two launches:
// 16 x 131,071 top 32 bf16 3.9 and 6.5 us, 128 x 131,000 fp32 13 and 26 (5.2 TB/s over both).

constexpr int kPartThreads = 256, kPartVecs = 4;

// The part's own vectors without its listed classes, and slot threadIdx.x of the row.
template <class T>
__device__ __forceinline__ float load_part(const pgcn_distill_args &a, int64_t r, int first, uint32_t *bits, ListLds<kPartThreads> &l,
                                           typename T::raw (&raw)[kPartVecs], int &id, float &t) {
  constexpr int kRange = kPartThreads * kPartVecs * T::E;
  const typename T::type *zr = (const typename T::type *)a.Z + r * a.ld;
#pragma unroll
  for (int i = 0; i < kPartVecs; ++i) {
    const int c0 = first + ((int)threadIdx.x + kPartThreads * i) * T::E;
    raw[i] = c0 < a.classes ? *reinterpret_cast<const typename T::raw *>(zr + c0) : typename T::raw{};
  }
  list_classes<kPartThreads>(a, r, bits, first, kRange / 32, l, id, t);
  float m = kNegInf;
  const int n = again(a.classes - first);
#pragma unroll
  for (int i = 0; i < kPartVecs; ++i) {
    const int c = ((int)threadIdx.x + kPartThreads * i) * T::E;
    float x[T::E];
    T::unpack(raw[i], x);
    drop_listed<T>(x, bits[c / 32] >> (c % 32), n - c);
#pragma unroll
    for (int e = 0; e < T::E; ++e) m = fmaxf(m, x[e]);
    raw[i] = T::pack(x);
  }
  return m;
}

// sums[row][part] = maximum, sum of e^{(z - m) / T}, sum of e^{z - m}
template <class T>
__global__ __launch_bounds__(kPartThreads) void distill_part_sums_kernel(pgcn_distill_args a, int parts, float4 *sums) {
  constexpr int kRange = kPartThreads * kPartVecs * T::E;
  __shared__ uint32_t bits[kRange / 32];
  __shared__ ListLds<kPartThreads> l;
  const int64_t r = blockIdx.x / parts;
  const int part = (int)(blockIdx.x % parts), lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  typename T::raw raw[kPartVecs];
  int id;
  float t;
  float m = lanes_max<64>(load_part<T>(a, r, part * kRange, bits, l, raw, id, t));
  if (lane == 0) l.m_rest[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(l.m_rest[0], l.m_rest[1]), fmaxf(l.m_rest[2], l.m_rest[3]));
  const bool two = a.labels && a.temperature != 1.0f;
  const float s = lanes_sum<64>(vectors_sum<T>(raw, base_of(m), kLog2e / a.temperature));
  const float h = two ? lanes_sum<64>(vectors_sum<T>(raw, base_of(m), kLog2e)) : 0.f;
  if (lane == 0) {
    l.s_rest[wave] = s;
    l.s_hard[wave] = h;
  }
  __syncthreads();
  if (threadIdx.x == 0)
    sums[blockIdx.x] = make_float4(m, (l.s_rest[0] + l.s_rest[1]) + (l.s_rest[2] + l.s_rest[3]),
                                   (l.s_hard[0] + l.s_hard[1]) + (l.s_hard[2] + l.s_hard[3]), 0.f);
}

template <class T>
__global__ __launch_bounds__(kPartThreads) void distill_part_grad_kernel(pgcn_distill_args a, int parts, const float4 *sums,
                                                                         double *losses) {
  constexpr int kRange = kPartThreads * kPartVecs * T::E;
  __shared__ uint32_t bits[kRange / 32];
  __shared__ ListLds<kPartThreads> l;
  const int64_t r = blockIdx.x / parts;
  const int part = (int)(blockIdx.x % parts), first = part * kRange, C = a.classes, k = threadIdx.x, lane = k % 64, wave = k / 64;
  const typename T::type *zr = (const typename T::type *)a.Z + r * a.ld;
  typename T::type *jr = (typename T::type *)a.J + r * a.ld;
  const float inv_t = 1.0f / a.temperature;
  const float4 p = k < parts ? sums[r * parts + k] : make_float4(kNegInf, 0.f, 0.f, 0.f);       // at most 64 parts
  const int y = a.labels ? a.labels[r] : -1;
  const bool has_y = y >= 0 && y < C;
  typename T::raw raw[kPartVecs];
  int id;
  float t;
  load_part<T>(a, r, first, bits, l, raw, id, t);
  const float zk = id >= 0 ? T::get(zr + id) : kNegInf, z_label = has_y ? T::get(zr + y) : 0.f;
  const RowStats st = block_stats<kPartThreads>(a, r, l, t, zk, p.x, inv_t,
                                                [&](float base, float scale) { return p.y == 0.f ? 0.f : p.y * exp_at(p.x, base, scale); },
                                                [&](float base) { return p.z == 0.f ? 0.f : p.z * exp_at(p.x, base, kLog2e); });
  const float soft = st.soft ? a.soft_scale * inv_t : 0.f, hard = has_y ? a.hard_scale : 0.f;
  const RestGrad grad(a, st, soft, hard, inv_t);
  store_vectors<T, kPartThreads>(raw, grad, jr, first, again(C));
  float loss = 0.f, g = 0.f;
  if (id >= 0) g = listed_term(st, t, zk, inv_t, soft, hard, a.soft_scale, loss) - (id == y ? hard : 0.f);
  loss = lanes_sum<64>(loss);
  if (lane == 0) l.loss[wave] = loss;
  __syncthreads();                                 // the vectors' stores come before the listed ones
  store_listed<T>(grad, jr, id, g, y, z_label, hard, bits, first, first + kRange);
  if (part == 0 && k == 0) {
    const float listed = (l.loss[0] + l.loss[1]) + (l.loss[2] + l.loss[3]);
    losses[r] = (double)row_loss(st, listed, z_label, has_y, l.bad || (y != -1 && !has_y), a.soft_scale, hard);
  }
}

// Sum of the parts in a fixed order.
__global__ __launch_bounds__(1024) void distill_sum_kernel(const double *part, int64_t n, float *out) {
  __shared__ double red[16];
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) s += red[i];
    *out = (float)s;
  }
}

constexpr int kShortBlocks = 2048;

// Lanes and vectors of a short row: 16 elements to a lane, 4 to 64 lanes, then more elements.  8 and
// 16 to a lane, us: 100,000 x 128 fp32 30 and 24, 50,000 x 300 53 and 39, 306,000 x 47 bf16 42 and 38.
void short_row(int elems, int vecs, int &lanes, int &per) {
  lanes = 4;
  while (lanes < 64 && lanes * 16 < vecs * elems) lanes *= 2;
  per = 1;
  while (lanes * per < vecs) per *= 2;
}

// Classes that a wave takes: with its list in registers a row needs no barrier.  A workgroup and a
// wave, us: 20,000 x 1,025 fp32 76 and 47, bf16 72 and 45; 10,000 x 2,000 46 and 40, 42 and 31.
constexpr int kShortClasses = 2048;

int vector_elems(int32_t dtype) { return dtype == PGCN_BF16 ? BF16::E : F32::E; }

unsigned short_blocks(int64_t rows, int lanes) {
  const int64_t n = 256 / lanes;
  return (unsigned)std::min<int64_t>((rows + n - 1) / n, kShortBlocks);
}

template <class T, int kLanes, int kVecs>
int short_go(const pgcn_distill_args &a, hipStream_t s) {
  const unsigned blocks = short_blocks(a.rows, kLanes);
  double *part = (double *)a.workspace;
  const int slots = (a.top + kLanes - 1) / kLanes;
  constexpr int kMost = kLanes * kVecs * T::E / kLanes < PGCN_MAX_TOP / kLanes ? kVecs * T::E : PGCN_MAX_TOP / kLanes;
  if (slots <= 1)
    hipLaunchKernelGGL((distill_short_kernel<T, kLanes, kVecs, 1>), dim3(blocks), dim3(256), 0, s, a, part);
  else if (slots <= 2)
    hipLaunchKernelGGL((distill_short_kernel<T, kLanes, kVecs, 2>), dim3(blocks), dim3(256), 0, s, a, part);
  else if (slots <= 4)
    hipLaunchKernelGGL((distill_short_kernel<T, kLanes, kVecs, 4>), dim3(blocks), dim3(256), 0, s, a, part);
  else
    hipLaunchKernelGGL((distill_short_kernel<T, kLanes, kVecs, kMost>), dim3(blocks), dim3(256), 0, s, a, part);
  PGCN_HIP(hipGetLastError());
  if (blocks == 1) return PGCN_OK;
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, part, (int64_t)blocks, a.loss_out);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

template <class T, int kThreads, int kVecs>
int long_go(const pgcn_distill_args &a, hipStream_t s) {
  double *part = (double *)a.workspace;
  const size_t lds = (size_t)((a.classes + 31) / 32) * 4;
  const int64_t most = kMaxLaunch / kThreads;
  for (int64_t row0 = 0; row0 < a.rows; row0 += most) {
    pgcn_distill_args b = a;
    b.rows = std::min(most, a.rows - row0);
    b.Z = (const typename T::type *)a.Z + row0 * a.ld;
    b.J = (typename T::type *)a.J + row0 * a.ld;
    b.top_values += row0 * a.ld_top;
    b.top_ids += row0 * a.ld_top;
    if (b.tail_lse) b.tail_lse += row0;
    if (b.labels) b.labels += row0;
    hipLaunchKernelGGL((distill_long_kernel<T, kThreads, kVecs>), dim3((unsigned)b.rows), dim3(kThreads), lds, s, b, part + row0);
    PGCN_HIP(hipGetLastError());
  }
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, part, a.rows, a.loss_out);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

constexpr int kLongVecs = 8192;                    // vectors of the longest row that a workgroup holds

// Parts of a row, 0: whole rows.  A row that no workgroup's registers hold goes in parts, and so do
// long rows too few to fill the chip.  us of the kernels whole and in parts: 1 x 16,000 fp32 8.5 and
// 10.1, 4 x 32,000 10.6 and 11.1, 16 x 32,000 13.8 and 11.5; bf16 32 x 32,000 11.4 and 12.2,
// 1 x 65,000 15.9 and 11.2, 128 x 65,000 19.7 and 19.3; 512 x 32,000 fp32 28 and 43.
int row_parts(int32_t dtype, int64_t rows, int32_t classes) {
  const int64_t range = kPartThreads * kPartVecs * vector_elems(dtype), parts = (classes + range - 1) / range;
  if (classes <= kShortClasses) return 0;
  const int vecs = (classes + vector_elems(dtype) - 1) / vector_elems(dtype);
  if (parts > kLongVecs / (kPartThreads * kPartVecs) || (rows <= 128 && vecs > 4096)) return (int)parts;
  return 0;
}

template <class T>
int parts_go(const pgcn_distill_args &a, int parts, hipStream_t s) {
  double *losses = (double *)a.workspace;
  float4 *sums = (float4 *)((char *)a.workspace + align_up((size_t)a.rows * sizeof(double), 16));
  const dim3 grid((unsigned)(a.rows * parts));
  hipLaunchKernelGGL(distill_part_sums_kernel<T>, grid, dim3(kPartThreads), 0, s, a, parts, sums);
  PGCN_HIP(hipGetLastError());
  hipLaunchKernelGGL(distill_part_grad_kernel<T>, grid, dim3(kPartThreads), 0, s, a, parts, sums, losses);
  PGCN_HIP(hipGetLastError());
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, losses, a.rows, a.loss_out);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

template <class T>
int distill_go(const pgcn_distill_args &a, hipStream_t s) {
  const int vecs = (a.classes + T::E - 1) / T::E;
  if (a.classes <= kShortClasses) {
    int lanes, per;
    short_row(T::E, vecs, lanes, per);
    constexpr int k16 = 16 / T::E;                 // vectors of 16 elements
    switch (lanes * 100 + per) {
      case 401: return short_go<T, 4, 1>(a, s);
      case 402: return short_go<T, 4, 2>(a, s);
      case 404: return short_go<T, 4, k16>(a, s);
      case 800 + k16: return short_go<T, 8, k16>(a, s);
      case 1600 + k16: return short_go<T, 16, k16>(a, s);
      case 3200 + k16: return short_go<T, 32, k16>(a, s);
      case 6400 + k16: return short_go<T, 64, k16>(a, s);
      default: return short_go<T, 64, 2 * k16>(a, s);
    }
  }
  const int parts = row_parts(a.dtype, a.rows, a.classes);
  if (parts) return parts_go<T>(a, parts, s);
  if constexpr (T::E == 4) {                       // short rows end at 512 vectors
    if (vecs <= 1024) return long_go<T, 256, 4>(a, s);
    if (vecs <= 2048) return long_go<T, 256, 8>(a, s);
    if (vecs <= 4096) return long_go<T, 256, 16>(a, s);
    return long_go<T, 512, 16>(a, s);
  } else {                                         // unpacked bf16 takes more registers: 8 vectors at most
    if (vecs <= 512) return long_go<T, 256, 2>(a, s);
    if (vecs <= 1024) return long_go<T, 256, 4>(a, s);
    if (vecs <= 2048) return long_go<T, 256, 8>(a, s);
    if (vecs <= 4096) return long_go<T, 512, 8>(a, s);
    return long_go<T, 1024, 8>(a, s);
  }
}

}  // namespace

size_t distill_workspace(int32_t dtype, int64_t rows, int32_t classes, int32_t) {
  if (classes > kShortClasses) {
    const size_t parts = (size_t)row_parts(dtype, rows, classes);
    return align_up((size_t)rows * sizeof(double), 16) + parts * (size_t)rows * sizeof(float4);
  }
  int lanes, per;
  const int e = vector_elems(dtype);
  short_row(e, (classes + e - 1) / e, lanes, per);
  return short_blocks(rows, lanes) * sizeof(double);
}

int launch_distill(const pgcn_distill_args &a, hipStream_t s) {
  TraceScope ts(PGCN_TK_DISTILL, s);
  if (a.rows > 0) return a.dtype == PGCN_BF16 ? distill_go<BF16>(a, s) : distill_go<F32>(a, s);
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, (const double *)nullptr, (int64_t)0, a.loss_out);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
