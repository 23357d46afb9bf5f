// Group normalisation of features-last rows with an activation, forward and backward.
//
// Over the n = sample_rows x (channels / groups) elements of a sample's group:
//     xhat = (x - mu) r,  r = 1 / sqrt(var + eps),  u = gamma xhat + beta,  Y = act(u)
//     du = J act'(u);  dbeta = sum du,  dgamma = sum du xhat over all rows
//     dX = r (gamma du - c1 - xhat c2),  c1 = mean(gamma du),  c2 = mean(gamma du xhat) over the group
// The variance is a sum of squared distances from a mean, joined from parts by
//     M2 = M2_a + M2_b + (mu_a - mu_b)^2 n_a n_b / (n_a + n_b)
// (Chan, Golub and LeVeque, 1983), so that a mean far from zero costs no digits.
// u is formed by one rounded fp32 operation after another, (x - mu) r gamma + beta, in both
// directions: the backward's 1[u > 0] is the forward's.
#include <algorithm>

#include "ops.h"

namespace pgcn {

namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------ activations --

template <int kAct>
__device__ __forceinline__ float act(float u) {
  if (kAct == PGCN_ACT_RELU) return u > 0.f || u != u ? u : 0.f;      // a NaN stays one
  if (kAct == PGCN_ACT_SILU) return u / (1.0f + __expf(-u));
  if (kAct == PGCN_ACT_GELU) return 0.5f * u * (1.0f + erff(u * 0.70710678118654752f));
  return u;
}

template <int kAct>
__device__ __forceinline__ float act_slope(float u) {
  if (kAct == PGCN_ACT_RELU) return u > 0.f ? 1.f : 0.f;
  if (kAct == PGCN_ACT_SILU) {
    const float g = 1.0f / (1.0f + __expf(-u));
    return g * (1.0f + u * (1.0f - g));
  }
  if (kAct == PGCN_ACT_GELU)
    return 0.5f * (1.0f + erff(u * 0.70710678118654752f)) + u * __expf(-0.5f * u * u) * 0.39894228040143268f;
  return 1.f;
}

__device__ __forceinline__ float normed(float x, float mu, float r) {
#pragma clang fp contract(off)
  const float d = x - mu;
  return d * r;
}

__device__ __forceinline__ float affine(float xhat, float gamma, float beta) {
#pragma clang fp contract(off)
  const float g = xhat * gamma;
  return g + beta;
}

// -------------------------------------------------------------- statistics --

struct Moments {
  float n = 0.f, mu = 0.f, m2 = 0.f;
};

__device__ __forceinline__ Moments join(const Moments &a, const Moments &b) {
  if (b.n == 0.f) return a;
  if (a.n == 0.f) return b;
  Moments r;
  r.n = a.n + b.n;
  const float d = b.mu - a.mu, w = b.n / r.n;
  r.mu = a.mu + d * w;
  r.m2 = a.m2 + b.m2 + d * d * a.n * w;
  return r;
}

// How a sample's rows are cut: `chunks` ranges of `per` rows (the last may be shorter), so that
// few long samples fill the chip too.
struct Cut {
  int64_t per;
  int chunks;
};

// Column layout of a workgroup: 1 << sh lanes side by side on a row's vectors, the rest on rows.
int column_shift(int vecs) {
  int sh = 0;
  while (sh < 8 && (1 << sh) < vecs) ++sh;
  return sh;
}

constexpr int kMaxChunks = 256;

Cut cut_rows(int64_t samples, int64_t sample_rows, int64_t min_rows) {
  samples = std::max<int64_t>(1, samples);
  int64_t want = std::max<int64_t>(1, 1024 / samples);
  want = std::min<int64_t>(std::min<int64_t>(want, kMaxChunks), (sample_rows + min_rows - 1) / min_rows);
  Cut c;
  c.per = (sample_rows + want - 1) / want;
  c.chunks = (int)((sample_rows + c.per - 1) / c.per);
  return c;
}

__device__ __forceinline__ int64_t chunk_rows(int64_t sample_rows, int64_t per, int chunk) {
  const int64_t left = sample_rows - (int64_t)chunk * per;
  return left < per ? left : per;
}

// Moments of every group over one chunk of one sample.  part[(sample chunks + chunk) groups + g] = (mu, M2).
template <class T>
__global__ __launch_bounds__(kThreads) void moments_kernel(pgcn_group_norm_fwd_args a, Cut cut, int sh, float2 *part) {
  extern __shared__ float lds[];                        // channel mean, channel M2: [2][channels]
  __shared__ float red[2][kThreads * 8];
  const int f = a.channels, vecs = (f + T::E - 1) / T::E, lx = 1 << sh, ty = kThreads >> sh;
  const int tx = threadIdx.x & (lx - 1), slot = threadIdx.x >> sh;
  const int64_t sample = blockIdx.x / cut.chunks;
  const int chunk = (int)(blockIdx.x - sample * cut.chunks);
  const int64_t rows = chunk_rows(a.sample_rows, cut.per, chunk);
  const typename T::type *x0 = (const typename T::type *)a.X + (sample * a.sample_rows + (int64_t)chunk * cut.per) * a.ld_x;

  for (int v0 = 0; v0 < vecs; v0 += lx) {
    const int vec = v0 + tx;
    float mu[T::E] = {}, m2[T::E] = {};
    int n = 0;
    if (vec < vecs) {
      for (int64_t r = slot; r < rows; r += ty) {
        float x[T::E];
        T::unpack(*reinterpret_cast<const typename T::raw *>(x0 + r * a.ld_x + vec * T::E), x);
        ++n;
        const float w = 1.0f / (float)n;
#pragma unroll
        for (int e = 0; e < T::E; ++e) {                // Welford's recurrence
          const float d = x[e] - mu[e];
          mu[e] += d * w;
          m2[e] += d * (x[e] - mu[e]);
        }
      }
    }
    // join the row slots, halving them; slot s has seen ceil((rows - s) / ty) rows
    for (int half = ty / 2; half > 0; half >>= 1) {
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        red[0][threadIdx.x * T::E + e] = mu[e];
        red[1][threadIdx.x * T::E + e] = m2[e];
      }
      __shared__ int cnt[kThreads];
      cnt[threadIdx.x] = n;
      __syncthreads();
      if (slot < half) {
        const int o = threadIdx.x + half * lx;
        const int no = cnt[o];
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          const Moments m = join(Moments{(float)n, mu[e], m2[e]}, Moments{(float)no, red[0][o * T::E + e], red[1][o * T::E + e]});
          mu[e] = m.mu;
          m2[e] = m.m2;
        }
        n += no;
      }
      __syncthreads();
    }
    if (slot == 0 && vec < vecs) {
#pragma unroll
      for (int e = 0; e < T::E; ++e)
        if (vec * T::E + e < f) {
          lds[vec * T::E + e] = mu[e];
          lds[f + vec * T::E + e] = m2[e];
        }
    }
  }
  __syncthreads();
  // a group's channels all have `rows` elements: mu is their average, M2 gains their spread
  const int cg = f / a.groups;
  for (int g = threadIdx.x; g < a.groups; g += kThreads) {
    float s = 0.f;
    for (int c = 0; c < cg; ++c) s += lds[g * cg + c];
    const float mu = s / (float)cg;
    float m2 = 0.f, d2 = 0.f;
    for (int c = 0; c < cg; ++c) {
      const float d = lds[g * cg + c] - mu;
      m2 += lds[f + g * cg + c];
      d2 += d * d;
    }
    part[(int64_t)blockIdx.x * a.groups + g] = make_float2(mu, m2 + d2 * (float)rows);
  }
}

// Joins a sample's chunks, normalises `per` of its rows.
template <class T, int kAct>
__global__ __launch_bounds__(kThreads) void normalise_kernel(pgcn_group_norm_fwd_args a, Cut cut, int64_t per, int blocks,
                                                             int sh, const float2 *part) {
  extern __shared__ float lds[];                        // mean, 1 / deviation: [2][groups]
  const int f = a.channels, cg = f / a.groups, vecs = (f + T::E - 1) / T::E, lx = 1 << sh, ty = kThreads >> sh;
  const int tx = threadIdx.x & (lx - 1), slot = threadIdx.x >> sh;
  const int64_t sample = blockIdx.x / blocks;
  const int block = (int)(blockIdx.x - sample * blocks);
  for (int g = threadIdx.x; g < a.groups; g += kThreads) {
    Moments m;
    for (int c = 0; c < cut.chunks; ++c) {
      const float2 p = part[(sample * cut.chunks + c) * a.groups + g];
      m = join(m, Moments{(float)chunk_rows(a.sample_rows, cut.per, c) * (float)cg, p.x, p.y});
    }
    const float r = 1.0f / sqrtf(m.m2 / m.n + a.eps);
    lds[g] = m.mu;
    lds[a.groups + g] = r;
    if (block == 0) {
      if (a.mean) a.mean[sample * a.groups + g] = m.mu;
      if (a.rstd) a.rstd[sample * a.groups + g] = r;
    }
  }
  __syncthreads();
  const int64_t rows = chunk_rows(a.sample_rows, per, block), row0 = sample * a.sample_rows + (int64_t)block * per;
  for (int vec = tx; vec < vecs; vec += lx) {
    float mu[T::E], rs[T::E], ga[T::E], be[T::E];
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      const int c = vec * T::E + e < f ? vec * T::E + e : f - 1;
      mu[e] = lds[c / cg];
      rs[e] = lds[a.groups + c / cg];
      ga[e] = a.gamma ? a.gamma[c] : 1.f;
      be[e] = a.beta ? a.beta[c] : 0.f;
    }
    for (int64_t r = slot; r < rows; r += ty) {
      float x[T::E];
      T::unpack(*reinterpret_cast<const typename T::raw *>((const typename T::type *)a.X + (row0 + r) * a.ld_x + vec * T::E), x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) x[e] = act<kAct>(affine(normed(x[e], mu[e], rs[e]), ga[e], be[e]));
      store_some<T>((typename T::type *)a.Y + (row0 + r) * a.ld_y + vec * T::E, x, f - vec * T::E);
    }
  }
}

// Sums of du and du xhat for every channel over one chunk of one sample: part[block][2][channels].
template <class T, int kAct>
__global__ __launch_bounds__(kThreads) void grad_sums_kernel(pgcn_group_norm_bwd_args a, Cut cut, int sh, float *part) {
  __shared__ float red[2][kThreads * 8];
  const int f = a.channels, cg = f / a.groups, vecs = (f + T::E - 1) / T::E, lx = 1 << sh, ty = kThreads >> sh;
  const int tx = threadIdx.x & (lx - 1), slot = threadIdx.x >> sh;
  const int64_t sample = blockIdx.x / cut.chunks;
  const int chunk = (int)(blockIdx.x - sample * cut.chunks);
  const int64_t rows = chunk_rows(a.sample_rows, cut.per, chunk), row0 = sample * a.sample_rows + (int64_t)chunk * cut.per;
  for (int v0 = 0; v0 < vecs; v0 += lx) {
    const int vec = v0 + tx;
    float s1[T::E] = {}, s2[T::E] = {};
    if (vec < vecs) {
      float mu[T::E], rs[T::E], ga[T::E], be[T::E];
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        const int c = vec * T::E + e < f ? vec * T::E + e : f - 1;
        mu[e] = a.mean[sample * a.groups + c / cg];
        rs[e] = a.rstd[sample * a.groups + c / cg];
        ga[e] = a.gamma ? a.gamma[c] : 1.f;
        be[e] = a.beta ? a.beta[c] : 0.f;
      }
      for (int64_t r = slot; r < rows; r += ty) {
        float x[T::E], j[T::E];
        T::unpack(*reinterpret_cast<const typename T::raw *>((const typename T::type *)a.X + (row0 + r) * a.ld_x + vec * T::E), x);
        T::unpack(*reinterpret_cast<const typename T::raw *>((const typename T::type *)a.J_out + (row0 + r) * a.ld_j_out + vec * T::E), j);
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          const float xh = normed(x[e], mu[e], rs[e]), du = j[e] * act_slope<kAct>(affine(xh, ga[e], be[e]));
          s1[e] += du;
          s2[e] += du * xh;
        }
      }
    }
    for (int half = ty / 2; half > 0; half >>= 1) {
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        red[0][threadIdx.x * T::E + e] = s1[e];
        red[1][threadIdx.x * T::E + e] = s2[e];
      }
      __syncthreads();
      if (slot < half) {
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          s1[e] += red[0][(threadIdx.x + half * lx) * T::E + e];
          s2[e] += red[1][(threadIdx.x + half * lx) * T::E + e];
        }
      }
      __syncthreads();
    }
    if (slot == 0 && vec < vecs) {
      float *p = part + (int64_t)blockIdx.x * 2 * f + vec * T::E;
#pragma unroll
      for (int e = 0; e < T::E; ++e)
        if (vec * T::E + e < f) {
          p[e] = s1[e];
          p[f + e] = s2[e];
        }
    }
  }
}

// sums[sample][i] = sum over the sample's chunks of part[sample][chunk][i], i < width.
__global__ __launch_bounds__(kThreads) void add_chunks_kernel(const float *part, int chunks, int64_t entries, int width, float *sums) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= entries) return;
  const int64_t b = i / width;
  const float *p = part + b * chunks * width + (i - b * width);
  float s = 0.f;
  for (int c = 0; c < chunks; ++c) s += p[(int64_t)c * width];
  sums[i] = s;
}

// Sums over the samples: dbeta from the first half of sums[sample][2][channels], dgamma from the second.
__global__ __launch_bounds__(kThreads) void param_grads_kernel(const float *sums, int64_t samples, int f, float *dgamma, float *dbeta) {
  __shared__ float red[kThreads];
  const int i = blockIdx.x * 32 + (threadIdx.x & 31), slot = threadIdx.x >> 5;
  float s = 0.f;
  if (i < 2 * f)
    for (int64_t b = slot; b < samples; b += kThreads / 32) s += sums[b * 2 * f + i];
  red[threadIdx.x] = s;
  __syncthreads();
  if (slot == 0 && i < 2 * f) {
    for (int k = 1; k < kThreads / 32; ++k) s += red[threadIdx.x + 32 * k];
    if (i < f) {
      if (dbeta) dbeta[i] = s;
    } else if (dgamma) {
      dgamma[i - f] = s;
    }
  }
}

// dX of `per` rows of a sample, from the sample's channel sums.
template <class T, int kAct>
__global__ __launch_bounds__(kThreads) void grad_rows_kernel(pgcn_group_norm_bwd_args a, int64_t per, int blocks, int sh,
                                                             const float *sums) {
  extern __shared__ float lds[];                        // c1, c2: [2][groups]
  const int f = a.channels, cg = f / a.groups, vecs = (f + T::E - 1) / T::E, lx = 1 << sh, ty = kThreads >> sh;
  const int tx = threadIdx.x & (lx - 1), slot = threadIdx.x >> sh;
  const int64_t sample = blockIdx.x / blocks;
  const int block = (int)(blockIdx.x - sample * blocks);
  const float inv_n = 1.0f / ((float)a.sample_rows * (float)cg);
  for (int g = threadIdx.x; g < a.groups; g += kThreads) {
    const float *p = sums + sample * 2 * f + g * cg;
    float c1 = 0.f, c2 = 0.f;
    for (int c = 0; c < cg; ++c) {
      const float ga = a.gamma ? a.gamma[g * cg + c] : 1.f;
      c1 += ga * p[c];
      c2 += ga * p[f + c];
    }
    lds[g] = c1 * inv_n;
    lds[a.groups + g] = c2 * inv_n;
  }
  __syncthreads();
  const int64_t rows = chunk_rows(a.sample_rows, per, block), row0 = sample * a.sample_rows + (int64_t)block * per;
  for (int vec = tx; vec < vecs; vec += lx) {
    float mu[T::E], rs[T::E], ga[T::E], be[T::E], c1[T::E], c2[T::E];
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      const int c = vec * T::E + e < f ? vec * T::E + e : f - 1;
      mu[e] = a.mean[sample * a.groups + c / cg];
      rs[e] = a.rstd[sample * a.groups + c / cg];
      ga[e] = a.gamma ? a.gamma[c] : 1.f;
      be[e] = a.beta ? a.beta[c] : 0.f;
      c1[e] = lds[c / cg];
      c2[e] = lds[a.groups + c / cg];
    }
    for (int64_t r = slot; r < rows; r += ty) {
      float x[T::E], j[T::E];
      T::unpack(*reinterpret_cast<const typename T::raw *>((const typename T::type *)a.X + (row0 + r) * a.ld_x + vec * T::E), x);
      T::unpack(*reinterpret_cast<const typename T::raw *>((const typename T::type *)a.J_out + (row0 + r) * a.ld_j_out + vec * T::E), j);
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        const float xh = normed(x[e], mu[e], rs[e]), du = j[e] * act_slope<kAct>(affine(xh, ga[e], be[e]));
        x[e] = rs[e] * (ga[e] * du - c1[e] - xh * c2[e]);
      }
      store_some<T>((typename T::type *)a.J_in + (row0 + r) * a.ld_j_in + vec * T::E, x, f - vec * T::E);
    }
  }
}

struct Shape {
  int vecs, sh;
  Cut stat, apply;
};

Shape shape_of(int32_t dtype, int32_t channels, int64_t samples, int64_t sample_rows) {
  const int e = dtype == PGCN_BF16 ? BF16::E : F32::E;
  Shape s;
  s.vecs = (channels + e - 1) / e;
  s.sh = column_shift(s.vecs);
  const int64_t ty = kThreads >> s.sh;
  s.stat = cut_rows(samples, sample_rows, 8 * ty);
  s.apply.per = 8 * ty;
  s.apply.chunks = (int)((sample_rows + s.apply.per - 1) / s.apply.per);
  return s;
}

template <class T, int kAct>
int fwd(const pgcn_group_norm_fwd_args &a, hipStream_t s) {
  const Shape sp = shape_of(a.dtype, a.channels, a.samples, a.sample_rows);
  float2 *part = (float2 *)a.workspace;
  hipLaunchKernelGGL(moments_kernel<T>, dim3((unsigned)(a.samples * sp.stat.chunks)), dim3(kThreads), 8 * (size_t)a.channels, s,
                     a, sp.stat, sp.sh, part);
  PGCN_HIP(hipGetLastError());
  hipLaunchKernelGGL((normalise_kernel<T, kAct>), dim3((unsigned)(a.samples * sp.apply.chunks)), dim3(kThreads), 8 * (size_t)a.groups,
                     s, a, sp.stat, sp.apply.per, sp.apply.chunks, sp.sh, part);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

template <class T, int kAct>
int bwd(const pgcn_group_norm_bwd_args &a, hipStream_t s) {
  const Shape sp = shape_of(a.dtype, a.channels, a.samples, a.sample_rows);
  const int w = 2 * a.channels;
  float *part = (float *)a.workspace, *sums = part;
  if (a.samples > 0) {
    hipLaunchKernelGGL((grad_sums_kernel<T, kAct>), dim3((unsigned)(a.samples * sp.stat.chunks)), dim3(kThreads), 0, s, a, sp.stat,
                       sp.sh, part);
    PGCN_HIP(hipGetLastError());
    if (sp.stat.chunks > 1) {
      sums = part + a.samples * sp.stat.chunks * w;
      const int64_t entries = a.samples * w;
      hipLaunchKernelGGL(add_chunks_kernel, dim3((unsigned)((entries + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, part,
                         sp.stat.chunks, entries, w, sums);
      PGCN_HIP(hipGetLastError());
    }
  }
  if (a.dgamma || a.dbeta) {
    hipLaunchKernelGGL(param_grads_kernel, dim3((unsigned)((w + 31) / 32)), dim3(kThreads), 0, s, sums, a.samples, a.channels,
                       a.dgamma, a.dbeta);
    PGCN_HIP(hipGetLastError());
  }
  if (a.J_in && a.samples > 0) {
    hipLaunchKernelGGL((grad_rows_kernel<T, kAct>), dim3((unsigned)(a.samples * sp.apply.chunks)), dim3(kThreads),
                       8 * (size_t)a.groups, s, a, sp.apply.per, sp.apply.chunks, sp.sh, sums);
    PGCN_HIP(hipGetLastError());
  }
  return PGCN_OK;
}

}  // namespace

size_t group_norm_workspace(int32_t dtype, int32_t channels, int32_t groups, int64_t samples, int64_t sample_rows) {
  if (samples == 0) return 0;
  const Shape sp = shape_of(dtype, channels, samples, sample_rows);
  const size_t f = 8 * (size_t)samples * (size_t)sp.stat.chunks * (size_t)groups;
  const size_t b = 8 * (size_t)channels * (size_t)samples * (size_t)(sp.stat.chunks + 1);
  return std::max(f, b);
}

#define PGCN_BY_TYPE(fn, a, s)                                               \
  switch ((a.dtype == PGCN_BF16 ? 4 : 0) + a.act) {                          \
    case 0: return fn<F32, PGCN_ACT_NONE>(a, s);                             \
    case 1: return fn<F32, PGCN_ACT_RELU>(a, s);                             \
    case 2: return fn<F32, PGCN_ACT_SILU>(a, s);                             \
    case 3: return fn<F32, PGCN_ACT_GELU>(a, s);                             \
    case 4: return fn<BF16, PGCN_ACT_NONE>(a, s);                            \
    case 5: return fn<BF16, PGCN_ACT_RELU>(a, s);                            \
    case 6: return fn<BF16, PGCN_ACT_SILU>(a, s);                            \
    default: return fn<BF16, PGCN_ACT_GELU>(a, s);                           \
  }

int launch_group_norm_fwd(const pgcn_group_norm_fwd_args &a, hipStream_t s) {
  if (a.samples == 0) return PGCN_OK;
  TraceScope ts(PGCN_TK_GROUP_NORM, s);
  PGCN_BY_TYPE(fwd, a, s)
}

int launch_group_norm_bwd(const pgcn_group_norm_bwd_args &a, hipStream_t s) {
  TraceScope ts(PGCN_TK_GROUP_NORM_BWD, s);
  PGCN_BY_TYPE(bwd, a, s)
}

}  // namespace pgcn
