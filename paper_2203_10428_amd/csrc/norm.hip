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

__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.0f + __expf(-u)); }

// GELU, u Phi(u), and its slope Phi(u) + u phi(u), by minimax fits.  With a = |u|, v = u^2 and t = 1 / (1 + k a), the tail
// Phi(-a) is e^{-v / 2} times a smooth function of t (fitted up to a = 14, from where e^{-v / 2} is 0), which keeps the
// digits of its far end.  An 8-bit result needs no more, one form for both directions, within 1.5e-7 of the tail.
// In fp32 t's rounding shows near 0, so for a <= 1.25 Phi - 1/2 is u times a polynomial in v (2e-9), and beyond
// it u Phi = max(u, 0) - a Phi(-a), with a Phi(-a) e^{v / 2} fitted as a whole (2e-7 of itself), and the slope likewise.
// rms error against 64 bits on [-3, -2], [-2, -1.25], [-1.25, -0.6], [0, 1.25]: u Phi 5e-9, 1.6e-8, 1.2e-8, 1.7e-8, the slope
// 7e-9, 1.6e-8, 2.5e-8, 3.2e-8; plain fp32 forms with erf 2.2e-8, 1.7e-8, 1.2e-8, 2.3e-8 and 1e-8, 1.4e-8, 1.5e-8, 3.4e-8.
constexpr float kNear2 = 1.25f * 1.25f, kPhi0 = 0.39894228040143268f;

__device__ __forceinline__ float inv_1p(float k, float a) { return __builtin_amdgcn_rcpf(__builtin_fmaf(k, a, 1.0f)); }
__device__ __forceinline__ float exp_half(float v) { return __builtin_amdgcn_exp2f(v * (-0.5f * kLog2e)); }

__device__ __forceinline__ float normal_cdf(float u, float &e) {
  const float t = inv_1p(0.3f, fabsf(u));
  e = exp_half(u * u);
  const float tail = e * t * (0.119629301f + t * (0.120753959f + t * (0.0999134928f + t * (0.128561616f + t * (-0.0536836162f +
                     t * (0.206353471f + t * (-0.157203063f + t * 0.0356747694f)))))));
  return u < 0.f ? tail : 1.0f - tail;
}

template <class T>
__device__ __forceinline__ float gelu(float u) {
  if (T::E == BF16::E) {
    float e;
    return u * normal_cdf(u, e);
  }
  const float v = u * u, t = inv_1p(0.6f, fabsf(u));
  const float far = fmaxf(u, 0.f) - exp_half(v) * (0.398910642f + t * (0.00111445237f + t * (-0.159502506f + t * (-0.168464243f +
                    t * (-0.775735795f + t * (1.18716598f + t * -0.494058937f))))));
  const float near = 0.5f * u + v * (0.398942262f + v * (-0.0664899871f + v * (0.00997150317f + v * (-0.00118271261f +
                     v * (0.000110329238f + v * -6.64525169e-06f)))));
  return v < kNear2 ? near : far;
}

template <class T>
__device__ __forceinline__ float gelu_slope(float u) {
  if (T::E == BF16::E) {
    float e;
    const float c = normal_cdf(u, e);
    return c + u * e * kPhi0;
  }
  const float a = fabsf(u), v = u * u, t = inv_1p(0.3f, a);
  const float h = exp_half(v) * (t * (0.119705357f + t * (0.119321547f + t * (0.111028418f + t * (0.0824648142f +
                  t * (0.0568446219f + t * (0.052795399f + t * -0.0424533971f)))))) - kPhi0 * a);       // Phi(-a) - a phi(a)
  const float far = u < 0.f ? h : 1.0f - h;
  const float near = 0.5f + u * (0.797884524f + v * (-0.265961289f + v * (0.0598397814f + v * (-0.00949377846f +
                     v * (0.00114656577f + v * (-0.000106548643f + v * 6.19606453e-06f))))));
  return v < kNear2 ? near : far;
}

// y = act(u), the choice once for a whole array
template <class T>
__device__ __forceinline__ void activate(float (&u)[T::E], int act) {
  constexpr int N = T::E;
  if (act == PGCN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = u[i] <= 0.f ? 0.f : u[i];      // a NaN stays one
  } else if (act == PGCN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] *= sigmoid(u[i]);
  } else if (act == PGCN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = gelu<T>(u[i]);
  }
}

// j *= act'(u)
template <class T>
__device__ __forceinline__ void times_slope(float (&j)[T::E], const float (&u)[T::E], int act) {
  constexpr int N = T::E;
  if (act == PGCN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) j[i] = u[i] > 0.f ? j[i] : 0.f;
  } else if (act == PGCN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float g = sigmoid(u[i]);
      j[i] *= g * (1.0f + u[i] * (1.0f - g));
    }
  } else if (act == PGCN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) j[i] *= gelu_slope<T>(u[i]);
  }
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

// The group of a channel, c / cg: c < 2^13 makes the high word of c ceil(2^32 / cg) exact.
uint32_t group_magic(int cg) { return cg > 1 ? (uint32_t)(((uint64_t(1) << 32) + cg - 1) / cg) : 0; }
__device__ __forceinline__ int group_of(uint32_t magic, int c) { return magic ? (int)__umulhi((uint32_t)c, magic) : c; }

// ---------------------------------------------- samples of many rows -------
//
// Two launches: the first leaves each chunk's group statistics, the second joins a sample's
// chunks in every workgroup and writes the rows.  Few long samples are cut into enough chunks
// to fill the chip.
//
// The second launch reads the sample again, all of it from beyond L2 (fetched bytes).  us of the two launches:
// forward 1 x 58,000 x 256 fp32 in 8 groups, GELU, 12.4 (4.8 TB/s) and 25.7 (4.6), backward with SiLU 26.6 (4.5)
// and 33.6 (5.3): memory.  Backward 8 x 4,096 x 320 bf16 in 32 groups, SiLU, 17.4 (2.4) and 20.0 (3.1): neither
// memory nor instructions (issued in 0.37 and 0.40 of the cycles), but the chain of a workgroup at two or
// three waves to a SIMD: its parameters one by one, about 12 rows to a thread, the join.
//
// A workgroup's threads: lx side by side on a row's vectors (all of them where a row has at most
// 256), ty row slots above one another, the rest idle.
struct Cut {
  int vecs, lx, ty;
  int64_t per;           // rows of a chunk (the last may be shorter)
  int chunks;
  int64_t out_per;       // rows of a workgroup of the second launch
  int out_blocks;
  uint32_t magic;        // of groups, see group_of
};

constexpr int kBatch = 4;              // rows that a thread loads together
// Workgroups of the two launches, about.  More chunks are more statistics for every workgroup of
// the second one to join.  us of both launches, 1 x 58,000 x 256 fp32 forward and 8 x 4,096 x 320
// bf16 backward: 512 and 512 39.3, 37.4; 512 and 1,024 37.3, 37.5; 1,024 and 1,024 39.3, 42.6.
constexpr int kStatBlocks = 512, kOutBlocks = 1024;

Cut cut_rows(int32_t dtype, int32_t channels, int32_t groups, int64_t samples, int64_t sample_rows) {
  const int e = dtype == PGCN_BF16 ? BF16::E : F32::E;
  Cut c;
  c.vecs = (channels + e - 1) / e;
  c.magic = group_magic(channels / groups);
  const int tiles = (c.vecs + kThreads - 1) / kThreads;
  c.lx = (c.vecs + tiles - 1) / tiles;
  c.ty = kThreads / c.lx;
  const int64_t least = (int64_t)kBatch * c.ty, n = std::max<int64_t>(1, samples);
  auto cut = [&](int blocks) {           // rows of a part, whole batches
    const int64_t parts = std::min(std::max<int64_t>(1, blocks / n), (sample_rows + least - 1) / least);
    return ((sample_rows + parts - 1) / parts + least - 1) / least * least;
  };
  c.per = cut(kStatBlocks);
  c.chunks = (int)((sample_rows + c.per - 1) / c.per);
  c.out_per = cut(kOutBlocks);
  c.out_blocks = (int)((sample_rows + c.out_per - 1) / c.out_per);
  return c;
}

__device__ __forceinline__ int64_t chunk_rows(int64_t sample_rows, int64_t per, int chunk) {
  const int64_t left = sample_rows - (int64_t)chunk * per;
  return left < per ? left : per;
}

// One value for every group, formed by teams of lanes: value(g, lane of the team, team size)
// gives a lane's part, which the team adds up; done(g, sum) is called once a group.
template <class Value, class Done>
__device__ __forceinline__ void for_groups(int groups, Value value, Done done) {
  int team = 1;
  while (team < 64 && 2 * team * groups <= kThreads) team *= 2;
  const int t = threadIdx.x & (team - 1), teams = kThreads / team;
  for (int g0 = 0; g0 < groups; g0 += teams) {
    const int g = g0 + threadIdx.x / team;
    float s = g < groups ? value(g, t, team) : 0.f;
    for (int o = team / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (g < groups && t == 0) done(g, s);
  }
}

// A group's chunks joined: `total(g, x, y)` gets the sums over the chunks of value(n, part).x and
// .y in fp64, n the elements of the chunk.  Threads side by side take neighbouring groups, the
// others every deep-th chunk.
struct Sum2 {
  double x, y;
};

template <class Value, class Total>
__device__ __forceinline__ void join_chunks(const float2 *part, int chunks, int groups, int64_t sample_rows, int64_t per, int cg,
                                            Sum2 *red, Value value, Total total) {
  const int wide = groups < kThreads ? groups : kThreads, deep = kThreads / wide;
  const int tx = threadIdx.x % wide, slot = threadIdx.x / wide;
  for (int g0 = 0; g0 < groups; g0 += wide) {
    const int g = g0 + tx;
    Sum2 m = {0.0, 0.0};
    if (g < groups && slot < deep) {
#pragma unroll 8
      for (int c = slot; c < chunks; c += deep) {
        const Sum2 v = value((double)chunk_rows(sample_rows, per, c) * (double)cg, part[(int64_t)c * groups + g]);
        m.x += v.x;
        m.y += v.y;
      }
    }
    __syncthreads();
    red[threadIdx.x] = m;
    __syncthreads();
    for (int n = deep; n > 1; n = (n + 1) / 2) {
      const int half = (n + 1) / 2;
      if (slot + half < n) {
        red[threadIdx.x].x += red[threadIdx.x + half * wide].x;
        red[threadIdx.x].y += red[threadIdx.x + half * wide].y;
      }
      __syncthreads();
    }
    if (slot == 0 && g < groups) total(g, red[threadIdx.x]);
  }
}

// Moments of every group over one chunk of one sample: part[(sample chunks + chunk) groups + g] = (mu, M2).
template <class T>
__global__ __launch_bounds__(kThreads) void moments_kernel(pgcn_group_norm_fwd_args a, Cut cut, float2 *part) {
  extern __shared__ float lds[];                        // channel mean, channel M2: [2][channels], then the group means
  __shared__ float red[2][T::E][kThreads];
  __shared__ int cnt[kThreads];
  const int f = a.channels, tx = threadIdx.x % cut.lx, slot = threadIdx.x / cut.lx;
  const int64_t sample = blockIdx.x / cut.chunks;
  const int chunk = (int)(blockIdx.x - sample * cut.chunks);
  const int64_t rows = chunk_rows(a.sample_rows, cut.per, chunk);
  const typename T::type *x0 = (const typename T::type *)a.X + (sample * a.sample_rows + (int64_t)chunk * cut.per) * a.ld_x;

  for (int v0 = 0; v0 < cut.vecs; v0 += cut.lx) {
    const int vec = v0 + tx;
    float mu[T::E] = {}, m2[T::E] = {};
    int n = 0;
    if (vec < cut.vecs && slot < cut.ty) {
      const typename T::type *p = x0 + slot * a.ld_x + vec * T::E;
      const int64_t step = cut.ty * a.ld_x;
      int64_t r = slot;
      for (; r + (kBatch - 1) * cut.ty < rows; r += kBatch * cut.ty, p += kBatch * step) {
        // a batch's own moments first, then one join: fewer steps in the chain
        typename T::raw raw[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) raw[b] = *reinterpret_cast<const typename T::raw *>(p + b * step);
        float x[kBatch][T::E];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) T::unpack(raw[b], x[b]);
        const float w = (float)kBatch * __builtin_amdgcn_rcpf((float)(n + kBatch)), wn = (float)n * w;
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          const float bm = ((x[0][e] + x[1][e]) + (x[2][e] + x[3][e])) * (1.0f / kBatch), d = bm - mu[e];
          float q = 0.f;
#pragma unroll
          for (int b = 0; b < kBatch; ++b) q += (x[b][e] - bm) * (x[b][e] - bm);
          mu[e] += d * w;
          m2[e] += q + d * d * wn;
        }
        n += kBatch;
      }
      if (r < rows) {                                                // what is left, loaded together too
        typename T::raw raw[kBatch - 1];
#pragma unroll
        for (int b = 0; b < kBatch - 1; ++b)
          raw[b] = *reinterpret_cast<const typename T::raw *>(r + b * cut.ty < rows ? p + b * step : p);
#pragma unroll
        for (int b = 0; b < kBatch - 1; ++b) {
          if (r + b * cut.ty >= rows) break;
          float x[T::E];
          T::unpack(raw[b], x);
          const float w = __builtin_amdgcn_rcpf((float)(n + 1)), wn = (float)n * w;
#pragma unroll
          for (int e = 0; e < T::E; ++e) {
            const float d = x[e] - mu[e];
            mu[e] += d * w;
            m2[e] += d * d * wn;
          }
          ++n;
        }
      }
    }
    for (int left = cut.ty; left > 1; left = (left + 1) / 2) {      // join the row slots
      const int half = (left + 1) / 2;
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        red[0][e][threadIdx.x] = mu[e];
        red[1][e][threadIdx.x] = m2[e];
      }
      cnt[threadIdx.x] = n;
      __syncthreads();
      if (slot + half < left) {
        const int o = threadIdx.x + half * cut.lx, no = cnt[o];
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          const Moments m = join(Moments{(float)n, mu[e], m2[e]}, Moments{(float)no, red[0][e][o], red[1][e][o]});
          mu[e] = m.mu;
          m2[e] = m.m2;
        }
        n += no;
      }
      __syncthreads();
    }
    if (slot == 0 && vec < cut.vecs) {
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
  float *mean = lds + 2 * f;
  for_groups(a.groups, [&](int g, int t, int team) {
    float s = 0.f;
    for (int c = t; c < cg; c += team) s += lds[g * cg + c];
    return s;
  }, [&](int g, float s) { mean[g] = s / (float)cg; });
  __syncthreads();
  for_groups(a.groups, [&](int g, int t, int team) {
    float s = 0.f;
    for (int c = t; c < cg; c += team) {
      const float d = lds[g * cg + c] - mean[g];
      s += lds[f + g * cg + c] + d * d * (float)rows;
    }
    return s;
  }, [&](int g, float s) { part[(int64_t)blockIdx.x * a.groups + g] = make_float2(mean[g], s); });
}

// Joins a sample's chunks, normalises `out_per` of its rows.
template <class T>
__global__ __launch_bounds__(kThreads) void normalise_kernel(pgcn_group_norm_fwd_args a, Cut cut, const float2 *part) {
  extern __shared__ float lds[];                        // mean, 1 / deviation: [2][groups]
  __shared__ Sum2 red[kThreads];
  const int f = a.channels, cg = f / a.groups, tx = threadIdx.x % cut.lx, slot = threadIdx.x / cut.lx;
  const int64_t sample = blockIdx.x / cut.out_blocks;
  const int block = (int)(blockIdx.x - sample * cut.out_blocks);
  const double n = (double)a.sample_rows * (double)cg;
  // sums of x and of squares: fp64 leaves 29 bits of the variance where the mean is 4,096 deviations away
  join_chunks(part + sample * cut.chunks * a.groups, cut.chunks, a.groups, a.sample_rows, cut.per, cg, red,
              [](double k, const float2 &p) { return Sum2{k * (double)p.x, (double)p.y + k * (double)p.x * (double)p.x}; },
              [&](int g, const Sum2 &t) {
    const double mu = t.x / n, var = (t.y - t.x * mu) / n;
    const float r = 1.0f / sqrtf((float)(var > 0.0 || var != var ? var : 0.0) + a.eps);
    lds[g] = (float)mu;
    lds[a.groups + g] = r;
    if (block == 0) {
      if (a.mean) a.mean[sample * a.groups + g] = (float)mu;
      if (a.rstd) a.rstd[sample * a.groups + g] = r;
    }
  });
  __syncthreads();
  if (slot >= cut.ty) return;
  const int64_t rows = chunk_rows(a.sample_rows, cut.out_per, block), row0 = sample * a.sample_rows + (int64_t)block * cut.out_per;
  for (int vec = tx; vec < cut.vecs; vec += cut.lx) {
    float mu[T::E], rs[T::E], ga[T::E], be[T::E];
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      const int c = vec * T::E + e < f ? vec * T::E + e : f - 1, g = group_of(cut.magic, c);
      mu[e] = lds[g];
      rs[e] = lds[a.groups + g];
      ga[e] = a.gamma ? a.gamma[c] : 1.f;
      be[e] = a.beta ? a.beta[c] : 0.f;
    }
    const typename T::type *p = (const typename T::type *)a.X + (row0 + slot) * a.ld_x + vec * T::E;
    typename T::type *y = (typename T::type *)a.Y + (row0 + slot) * a.ld_y + vec * T::E;
    const int64_t step = cut.ty * a.ld_x, step_y = cut.ty * a.ld_y;
    const int left = f - vec * T::E;
    auto one = [&](const typename T::raw &raw, typename T::type *to) {
      float x[T::E];
      T::unpack(raw, x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) x[e] = affine(normed(x[e], mu[e], rs[e]), ga[e], be[e]);
      activate<T>(x, a.act);
      store_some<T>(to, x, left);
    };
    int64_t r = slot;
    for (; r + (kBatch - 1) * cut.ty < rows; r += kBatch * cut.ty, p += kBatch * step, y += kBatch * step_y) {
      typename T::raw raw[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) raw[b] = *reinterpret_cast<const typename T::raw *>(p + b * step);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) one(raw[b], y + b * step_y);
    }
    if (r < rows) {
      typename T::raw raw[kBatch - 1];
#pragma unroll
      for (int b = 0; b < kBatch - 1; ++b)
        raw[b] = *reinterpret_cast<const typename T::raw *>(r + b * cut.ty < rows ? p + b * step : p);
#pragma unroll
      for (int b = 0; b < kBatch - 1; ++b)
        if (r + b * cut.ty < rows) one(raw[b], y + b * step_y);
    }
  }
}

// xhat -> x, du -> j of one vector.
template <class T>
__device__ __forceinline__ void grad_vector(const typename T::raw &xr, const typename T::raw &jr, const float (&mu)[T::E],
                                            const float (&rs)[T::E], const float (&ga)[T::E], const float (&be)[T::E], int act,
                                            float (&x)[T::E], float (&j)[T::E]) {
  float u[T::E];
  T::unpack(xr, x);
  T::unpack(jr, j);
#pragma unroll
  for (int e = 0; e < T::E; ++e) {
    x[e] = normed(x[e], mu[e], rs[e]);
    u[e] = affine(x[e], ga[e], be[e]);
  }
  times_slope<T>(j, u, act);
}

// Sums over one chunk of one sample: of gamma du and gamma du xhat for every group,
// part[sample][chunk][groups].  A workgroup walks chunks and adds up du and du xhat for every
// channel over all of its own, channel_part[block][2][channels] (null: not wanted), so that many
// short samples leave few of them.
template <class T>
__global__ __launch_bounds__(kThreads) void grad_sums_kernel(pgcn_group_norm_bwd_args a, Cut cut, float2 *part, float *channel_part) {
  extern __shared__ float lds[];                        // [2][channels]
  __shared__ float red[2][T::E][kThreads];
  const int f = a.channels, cg = f / a.groups, tx = threadIdx.x % cut.lx, slot = threadIdx.x / cut.lx;
  for (int64_t unit = blockIdx.x; unit < a.samples * cut.chunks; unit += gridDim.x) {
    const int64_t sample = unit / cut.chunks;
    const int chunk = (int)(unit - sample * cut.chunks);
    const int64_t rows = chunk_rows(a.sample_rows, cut.per, chunk), row0 = sample * a.sample_rows + (int64_t)chunk * cut.per;
    for (int v0 = 0; v0 < cut.vecs; v0 += cut.lx) {
      const int vec = v0 + tx;
      float s1[T::E] = {}, s2[T::E] = {};
      if (vec < cut.vecs && slot < cut.ty) {
        float mu[T::E], rs[T::E], ga[T::E], be[T::E];
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          const int c = vec * T::E + e < f ? vec * T::E + e : f - 1, g = group_of(cut.magic, c);
          mu[e] = a.mean[sample * a.groups + g];
          rs[e] = a.rstd[sample * a.groups + g];
          ga[e] = a.gamma ? a.gamma[c] : 1.f;
          be[e] = a.beta ? a.beta[c] : 0.f;
        }
        const typename T::type *p = (const typename T::type *)a.X + (row0 + slot) * a.ld_x + vec * T::E;
        const typename T::type *q = (const typename T::type *)a.J_out + (row0 + slot) * a.ld_j_out + vec * T::E;
        const int64_t step = cut.ty * a.ld_x, step_j = cut.ty * a.ld_j_out;
        auto one = [&](const typename T::raw &xr, const typename T::raw &jr) {
          float x[T::E], j[T::E];
          grad_vector<T>(xr, jr, mu, rs, ga, be, a.act, x, j);
#pragma unroll
          for (int e = 0; e < T::E; ++e) {
            s1[e] += j[e];
            s2[e] += j[e] * x[e];
          }
        };
        int64_t r = slot;
        for (; r + (kBatch - 1) * cut.ty < rows; r += kBatch * cut.ty, p += kBatch * step, q += kBatch * step_j) {
          typename T::raw xr[kBatch], jr[kBatch];
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            xr[b] = *reinterpret_cast<const typename T::raw *>(p + b * step);
            jr[b] = *reinterpret_cast<const typename T::raw *>(q + b * step_j);
          }
#pragma unroll
          for (int b = 0; b < kBatch; ++b) one(xr[b], jr[b]);
        }
        if (r < rows) {
          typename T::raw xr[kBatch - 1], jr[kBatch - 1];
#pragma unroll
          for (int b = 0; b < kBatch - 1; ++b) {
            const bool in = r + b * cut.ty < rows;
            xr[b] = *reinterpret_cast<const typename T::raw *>(in ? p + b * step : p);
            jr[b] = *reinterpret_cast<const typename T::raw *>(in ? q + b * step_j : q);
          }
#pragma unroll
          for (int b = 0; b < kBatch - 1; ++b)
            if (r + b * cut.ty < rows) one(xr[b], jr[b]);
        }
      }
      for (int left = cut.ty; left > 1; left = (left + 1) / 2) {
        const int half = (left + 1) / 2;
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          red[0][e][threadIdx.x] = s1[e];
          red[1][e][threadIdx.x] = s2[e];
        }
        __syncthreads();
        if (slot + half < left) {
#pragma unroll
          for (int e = 0; e < T::E; ++e) {
            s1[e] += red[0][e][threadIdx.x + half * cut.lx];
            s2[e] += red[1][e][threadIdx.x + half * cut.lx];
          }
        }
        __syncthreads();
      }
      if (slot == 0 && vec < cut.vecs) {
        float *p = channel_part ? channel_part + (int64_t)blockIdx.x * 2 * f : nullptr;
#pragma unroll
        for (int e = 0; e < T::E; ++e) {
          const int c = vec * T::E + e;
          if (c >= f) break;
          const float ga = a.gamma ? a.gamma[c] : 1.f;
          lds[c] = ga * s1[e];
          lds[f + c] = ga * s2[e];
          if (p) {
            const bool first = unit == blockIdx.x;
            p[c] = first ? s1[e] : p[c] + s1[e];
            p[f + c] = first ? s2[e] : p[f + c] + s2[e];
          }
        }
      }
    }
    __syncthreads();
    for (int h = 0; h < 2; ++h)
      for_groups(a.groups, [&](int g, int t, int team) {
        float s = 0.f;
        for (int c = t; c < cg; c += team) s += lds[h * f + g * cg + c];
        return s;
      }, [&](int g, float s) { (&part[unit * a.groups + g].x)[h] = s; });
    __syncthreads();
  }
}

// Sums over n of part[n][2][channels], 32 of the 2 channels values to a workgroup: the first half
// is dbeta, the second dgamma.
__device__ void param_grads(const float *part, int64_t n, int f, int block, float *dgamma, float *dbeta) {
  __shared__ double red[kThreads];
  const int i = block * 32 + (threadIdx.x & 31), slot = threadIdx.x >> 5;
  double s = 0.0;                                       // thousands of terms in one chain
  if (i < 2 * f) {
#pragma unroll 8
    for (int64_t b = slot; b < n; b += kThreads / 32) s += (double)part[b * 2 * f + i];
  }
  red[threadIdx.x] = s;
  __syncthreads();
  if (slot == 0 && i < 2 * f) {
    for (int k = 1; k < kThreads / 32; ++k) s += red[threadIdx.x + 32 * k];
    if (i < f) {
      if (dbeta) dbeta[i] = (float)s;
    } else if (dgamma) {
      dgamma[i - f] = (float)s;
    }
  }
}

__global__ __launch_bounds__(kThreads) void param_grads_kernel(const float *part, int64_t n, int f, float *dgamma, float *dbeta) {
  param_grads(part, n, f, blockIdx.x, dgamma, dbeta);
}

// dX of `out_per` rows of a sample, from its chunks' group sums; the last `param_blocks`
// workgroups add up the channel sums instead.
template <class T>
__global__ __launch_bounds__(kThreads) void grad_rows_kernel(pgcn_group_norm_bwd_args a, Cut cut, const float2 *part,
                                                             const float *channel_part, int sum_blocks, int row_blocks) {
  extern __shared__ float lds[];                        // c1, c2: [2][groups]
  __shared__ Sum2 red[kThreads];
  if ((int)blockIdx.x >= row_blocks) {
    param_grads(channel_part, sum_blocks, a.channels, blockIdx.x - row_blocks, a.dgamma, a.dbeta);
    return;
  }
  const int f = a.channels, cg = f / a.groups, tx = threadIdx.x % cut.lx, slot = threadIdx.x / cut.lx;
  const int64_t sample = blockIdx.x / cut.out_blocks;
  const int block = (int)(blockIdx.x - sample * cut.out_blocks);
  const double inv_n = 1.0 / ((double)a.sample_rows * (double)cg);
  join_chunks(part + sample * cut.chunks * a.groups, cut.chunks, a.groups, a.sample_rows, cut.per, cg, red,
              [](double, const float2 &p) { return Sum2{(double)p.x, (double)p.y}; },
              [&](int g, const Sum2 &t) {
    lds[g] = (float)(t.x * inv_n);
    lds[a.groups + g] = (float)(t.y * inv_n);
  });
  __syncthreads();
  if (slot >= cut.ty) return;
  const int64_t rows = chunk_rows(a.sample_rows, cut.out_per, block), row0 = sample * a.sample_rows + (int64_t)block * cut.out_per;
  for (int vec = tx; vec < cut.vecs; vec += cut.lx) {
    float mu[T::E], rs[T::E], ga[T::E], be[T::E], c1[T::E], c2[T::E];
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      const int c = vec * T::E + e < f ? vec * T::E + e : f - 1, g = group_of(cut.magic, c);
      mu[e] = a.mean[sample * a.groups + g];
      rs[e] = a.rstd[sample * a.groups + g];
      ga[e] = a.gamma ? a.gamma[c] : 1.f;
      be[e] = a.beta ? a.beta[c] : 0.f;
      c1[e] = lds[g];
      c2[e] = lds[a.groups + g];
    }
    const typename T::type *p = (const typename T::type *)a.X + (row0 + slot) * a.ld_x + vec * T::E;
    const typename T::type *q = (const typename T::type *)a.J_out + (row0 + slot) * a.ld_j_out + vec * T::E;
    typename T::type *y = (typename T::type *)a.J_in + (row0 + slot) * a.ld_j_in + vec * T::E;
    const int64_t step = cut.ty * a.ld_x, step_j = cut.ty * a.ld_j_out, step_y = cut.ty * a.ld_j_in;
    const int left = f - vec * T::E;
    auto one = [&](const typename T::raw &xr, const typename T::raw &jr, typename T::type *to) {
      float x[T::E], j[T::E];
      grad_vector<T>(xr, jr, mu, rs, ga, be, a.act, x, j);
#pragma unroll
      for (int e = 0; e < T::E; ++e) x[e] = rs[e] * (ga[e] * j[e] - c1[e] - x[e] * c2[e]);
      store_some<T>(to, x, left);
    };
    int64_t r = slot;
    for (; r + (kBatch - 1) * cut.ty < rows; r += kBatch * cut.ty, p += kBatch * step, q += kBatch * step_j, y += kBatch * step_y) {
      typename T::raw xr[kBatch], jr[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        xr[b] = *reinterpret_cast<const typename T::raw *>(p + b * step);
        jr[b] = *reinterpret_cast<const typename T::raw *>(q + b * step_j);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) one(xr[b], jr[b], y + b * step_y);
    }
    if (r < rows) {
      typename T::raw xr[kBatch - 1], jr[kBatch - 1];
#pragma unroll
      for (int b = 0; b < kBatch - 1; ++b) {
        const bool in = r + b * cut.ty < rows;
        xr[b] = *reinterpret_cast<const typename T::raw *>(in ? p + b * step : p);
        jr[b] = *reinterpret_cast<const typename T::raw *>(in ? q + b * step_j : q);
      }
#pragma unroll
      for (int b = 0; b < kBatch - 1; ++b)
        if (r + b * cut.ty < rows) one(xr[b], jr[b], y + b * step_y);
    }
  }
}

// -------------------------------------------- samples that fit registers ---
//
// kLanes threads hold a sample, one row or a few, kVecs 16-byte vectors each (vector lane + kLanes i
// of all its rows' vectors), so that X (and J) cross the memory once and both passes over the
// sample stay in registers.  A workgroup walks samples at a fixed stride: gamma, beta and the
// backward's channel sums stay in registers too.  Bound by memory in fp32 (30,000 x 1,024: forward
// 4.97, backward 4.6 TB/s, 2,048 channels 4.6 and 4.8).  In bf16, where a byte carries twice the elements, a
// sample's chain of load, sums and activation is as long again for half the bytes (2.9 and 2.5 TB/s, 3.9 and 3.2):
// 30,000 x 1,024 with SiLU 41.6 and 64 us, instructions in 0.49 and 0.42 of the cycles, at 5 and 3 waves to a SIMD.
// How a group's sum is formed:
enum class Sum {
  ROW,     // one group: all the sample's threads
  LANES    // one row, groups of 2^k neighbouring vectors: shuffles inside them
};           // any other groups: see any_fwd_kernel

struct RowShape {
  int f, groups, cg, vecs;
  int rows, all;       // rows of a sample, vectors of all of them
  int span;            // LANES: vectors of a group
  int team;            // any groups: lanes of a team
  uint32_t magic;      // of groups, see group_of
};

// A thread's vectors: their first channel (from f on: none) and row.
template <class T, int kLanes, int kVecs>
__device__ __forceinline__ void place_vectors(const RowShape &sp, int (&c0)[kVecs], int (&row)[kVecs]) {
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int p = threadIdx.x % kLanes + kLanes * i;
    row[i] = sp.rows > 1 ? p / sp.vecs : 0;
    c0[i] = p < sp.all ? (p - row[i] * sp.vecs) * T::E : 1 << 20;
    if (p >= sp.all) row[i] = 0;
  }
}

template <int kLanes>
__device__ __forceinline__ void row_sync() {
  if (kLanes > 64) {
    __syncthreads();
  } else {                       // the row's threads are lanes of one wave, whose LDS accesses keep their order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Sums of w (0 past the channels) over every vector's group.  `lds`: kThreads / 64 floats (ROW over
// several waves).
template <class T, int kLanes, int kVecs, Sum kSum>
__device__ __forceinline__ void group_sums(const float (&w)[kVecs][T::E], float (&out)[kVecs], const RowShape &sp, float *lds) {
  float s[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    float h[T::E / 2];
#pragma unroll
    for (int e = 0; e < T::E / 2; ++e) h[e] = w[i][e] + w[i][e + T::E / 2];
    s[i] = T::E == 4 ? h[0] + h[1] : (h[0] + h[T::E / 4]) + (h[1] + h[T::E / 2 - 1]);
  }
  if (kSum == Sum::ROW) {
    float r = s[0];
#pragma unroll
    for (int i = 1; i < kVecs; ++i) r += s[i];
#pragma unroll
    for (int o = (kLanes < 64 ? kLanes : 64) / 2; o > 0; o >>= 1) r += __shfl_xor(r, o, 64);
    if (kLanes > 64) {
      __syncthreads();
      if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = r;
      __syncthreads();
      r = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) out[i] = r;
  } else {
    for (int o = 1; o < sp.span; o <<= 1)
#pragma unroll
      for (int i = 0; i < kVecs; ++i) s[i] += __shfl_xor(s[i], o, 64);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) out[i] = s[i];
  }
}

template <class T>
__device__ __forceinline__ void load_vec_params(const float *p, float other, int f, int c, float (&out)[T::E]) {
#pragma unroll
  for (int e = 0; e < T::E; ++e) out[e] = p && c + e < f ? p[c + e] : other;
}
template <class T, int kVecs>
__device__ __forceinline__ void load_params(const float *p, float other, int f, const int (&c0)[kVecs], float (&out)[kVecs][T::E]) {
#pragma unroll
  for (int i = 0; i < kVecs; ++i) load_vec_params<T>(p, other, f, c0[i], out[i]);
}

// The sample whose first row is row0.
template <class T, int kVecs>
__device__ __forceinline__ void load_rows(const void *base, int64_t row0, int64_t ld, int f, const int (&c0)[kVecs], const int (&row)[kVecs],
                                          float (&x)[kVecs][T::E]) {
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    typename T::raw r = {};
    if (c0[i] < f) r = *reinterpret_cast<const typename T::raw *>((const typename T::type *)base + (row0 + row[i]) * ld + c0[i]);
    T::unpack(r, x[i]);
  }
}

// Two fp32 vectors a thread fit eight waves to a SIMD, backward five where shuffles add up the groups: the bounds keep
// GELU's temporaries from taking two registers more, and a wave with them from every activation: 239,000 x 512 in 32
// groups, SiLU, backward at four 300 us, at five 295 to 297.
template <class T, int kLanes, int kVecs, Sum kSum>
__global__ __launch_bounds__(kThreads, T::E == 4 && kVecs == 2 ? 8 : 1) void rows_fwd_kernel(pgcn_group_norm_fwd_args a, RowShape sp) {
  __shared__ float lds[kThreads / 64];
  const int slot = threadIdx.x / kLanes;
  int c0[kVecs], row[kVecs];
  place_vectors<T, kLanes>(sp, c0, row);
  float ga[kVecs][T::E], be[kVecs][T::E];
  load_params<T>(a.gamma, 1.f, sp.f, c0, ga);
  load_params<T>(a.beta, 0.f, sp.f, c0, be);
  const float inv_n = 1.0f / ((float)sp.cg * (float)sp.rows);
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / kLanes) + slot; r < a.samples; r += (int64_t)gridDim.x * (kThreads / kLanes)) {
    float x[kVecs][T::E], w[kVecs][T::E], mu[kVecs], rs[kVecs];
    load_rows<T>(a.X, r * sp.rows, a.ld_x, sp.f, c0, row, x);
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
      for (int e = 0; e < T::E; ++e) w[i][e] = x[i][e] = c0[i] + e < sp.f ? x[i][e] : 0.f;
    group_sums<T, kLanes, kVecs, kSum>(w, mu, sp, lds);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      mu[i] *= inv_n;
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        const float d = x[i][e] - mu[i];
        w[i][e] = c0[i] + e < sp.f ? d * d : 0.f;
      }
    }
    group_sums<T, kLanes, kVecs, kSum>(w, rs, sp, lds);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      rs[i] = 1.0f / sqrtf(rs[i] * inv_n + a.eps);
      if (c0[i] < sp.f) {
        const int g = group_of(sp.magic, c0[i]);
        if (g * sp.cg == c0[i] && row[i] == 0) {   // the thread with a group's first element writes its statistics
          if (a.mean) a.mean[r * sp.groups + g] = mu[i];
          if (a.rstd) a.rstd[r * sp.groups + g] = rs[i];
        }
#pragma unroll
        for (int e = 0; e < T::E; ++e) x[i][e] = affine(normed(x[i][e], mu[i], rs[i]), ga[i][e], be[i][e]);
        activate<T>(x[i], a.act);
        store_some<T>((typename T::type *)a.Y + (r * sp.rows + row[i]) * a.ld_y + c0[i], x[i], sp.f - c0[i]);
      }
    }
  }
}

// A workgroup's channel sums: its slots' and the sample's rows' joined in a fixed order, p[2][channels].
template <class T, int kLanes, int kVecs>
__device__ __forceinline__ void write_channel_sums(const RowShape &sp, const int (&c0)[kVecs], const float (&s1)[kVecs][T::E],
                                                   const float (&s2)[kVecs][T::E], float *p, float *lds_all) {
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (sp.rows == 1) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        float v[T::E];
#pragma unroll
        for (int e = 0; e < T::E; ++e) v[e] = half ? s2[i][e] : s1[i][e];
        constexpr int kSlots = kThreads / kLanes;
        if (kSlots > 1) {
          __syncthreads();
#pragma unroll
          for (int e = 0; e < T::E; ++e) lds_all[e * kThreads + threadIdx.x] = v[e];
          __syncthreads();
          if (slot == 0) {
#pragma unroll 1
            for (int k = 1; k < kSlots; ++k)
#pragma unroll
              for (int e = 0; e < T::E; ++e) v[e] += lds_all[e * kThreads + k * kLanes + lane];
          }
        }
        if (slot == 0)
#pragma unroll
          for (int e = 0; e < T::E; ++e)
            if (c0[i] + e < sp.f) p[half * sp.f + c0[i] + e] = v[e];
      }
    } else {
      // the sums of every slot's vectors side by side, then a thread for every channel
      __syncthreads();
      float *at = lds_all + slot * sp.all * T::E;
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        if (c0[i] < sp.f)
#pragma unroll
          for (int e = 0; e < T::E; ++e) at[(lane + kLanes * i) * T::E + e] = half ? s2[i][e] : s1[i][e];
      __syncthreads();
      const int wide = sp.vecs * T::E, n = kThreads / kLanes * sp.rows;
      for (int c = threadIdx.x; c < sp.f; c += kThreads) {
        float v = 0.f;
        for (int k = 0; k < n; ++k) v += lds_all[k * wide + c];
        p[half * sp.f + c] = v;
      }
    }
  }
}

// The backward of those rows; a workgroup's channel sums go to part[workgroup][2][channels].
template <class T, int kLanes, int kVecs, Sum kSum>
__global__ __launch_bounds__(kThreads, kVecs * T::E <= 4 ? 4 : T::E == 4 && kVecs == 2 && kSum == Sum::LANES ? 5 : kVecs <= 4 ? 2 : 1) void rows_bwd_kernel(pgcn_group_norm_bwd_args a, RowShape sp, float *part) {
  extern __shared__ float lds_all[];
  const int slot = threadIdx.x / kLanes;
  int c0[kVecs], row[kVecs];
  place_vectors<T, kLanes>(sp, c0, row);
  float ga[kVecs][T::E], be[kVecs][T::E], s1[kVecs][T::E] = {}, s2[kVecs][T::E] = {};
  constexpr bool kReread = kVecs * T::E > 16;         // gamma and beta out of L1 for every sample
  if (!kReread) {
    load_params<T>(a.gamma, 1.f, sp.f, c0, ga);
    load_params<T>(a.beta, 0.f, sp.f, c0, be);
  }
  const float inv_n = 1.0f / ((float)sp.cg * (float)sp.rows);
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / kLanes) + slot; r < a.samples; r += (int64_t)gridDim.x * (kThreads / kLanes)) {
    float x[kVecs][T::E], j[kVecs][T::E], w[kVecs][T::E], c1[kVecs], c2[kVecs], rs[kVecs];
    load_rows<T>(a.X, r * sp.rows, a.ld_x, sp.f, c0, row, x);
    load_rows<T>(a.J_out, r * sp.rows, a.ld_j_out, sp.f, c0, row, j);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (kReread) {
        load_vec_params<T>(a.gamma, 1.f, sp.f, c0[i], ga[i]);
        load_vec_params<T>(a.beta, 0.f, sp.f, c0[i], be[i]);
      }
      const int64_t g = r * sp.groups + group_of(sp.magic, c0[i] < sp.f ? c0[i] : 0);
      const float mu = a.mean[g];
      float u[T::E];
      rs[i] = a.rstd[g];
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        x[i][e] = normed(x[i][e], mu, rs[i]);
        u[e] = affine(x[i][e], ga[i][e], be[i][e]);
      }
      times_slope<T>(j[i], u, a.act);
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        const bool in = c0[i] + e < sp.f;
        x[i][e] = in ? x[i][e] : 0.f;
        j[i][e] = in ? j[i][e] : 0.f;
        s1[i][e] += j[i][e];
        s2[i][e] += j[i][e] * x[i][e];
        j[i][e] *= ga[i][e];
        w[i][e] = j[i][e] * x[i][e];
      }
    }
    if (!a.J_in) continue;
    group_sums<T, kLanes, kVecs, kSum>(j, c1, sp, lds_all);
    group_sums<T, kLanes, kVecs, kSum>(w, c2, sp, lds_all);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
#pragma unroll
      for (int e = 0; e < T::E; ++e)
        x[i][e] = rs[i] * (j[i][e] - c1[i] * inv_n - x[i][e] * (c2[i] * inv_n));
      if (c0[i] < sp.f)
        store_some<T>((typename T::type *)a.J_in + (r * sp.rows + row[i]) * a.ld_j_in + c0[i], x[i], sp.f - c0[i]);
    }
  }
  if (part) write_channel_sums<T, kLanes>(sp, c0, s1, s2, part + (int64_t)blockIdx.x * 2 * sp.f, lds_all);
}

// ---- the same for any groups --------------------------------------------------------------
//
// The sample's values go through LDS, where a team of lanes takes each group; what is needed after
// the sums is read from there again and not held in registers.  gamma and beta lie in LDS too.
// An element is written once and read once (forward: twice) as a single float, gamma, beta and the group's
// values come from LDS again, one phase after another: LDS instructions are under way in 0.41 of the cycles
// forward and 0.55 backward, vector instructions issued in half.  30,000 x 1,000 fp32 in 8 groups: forward
// 102 us (2.4 TB/s), backward 114 (3.2); 1,024 channels in 32 groups by shuffles 52 and 80.

// Calls f(offset into the image) for the part of group g that lane t of its team takes.
template <class F>
__device__ __forceinline__ void group_walk(const RowShape &sp, int wide, int g, int t, F f) {
  const int n = sp.rows * sp.cg;
  if (sp.rows == 1) {
#pragma unroll 4
    for (int c = t; c < n; c += sp.team) f(g * sp.cg + c);
  } else {
#pragma unroll 4
    for (int k = t; k < n; k += sp.team) {
      const int r = group_of(sp.magic, k);
      f(r * wide + g * sp.cg + k - r * sp.cg);
    }
  }
}

__device__ __forceinline__ float team_sum(float s, int team) {
  for (int o = team / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  return s;
}

// gamma and beta to LDS: [2][wide].
__device__ __forceinline__ void stage_params(const float *gamma, const float *beta, int f, int wide, float *to) {
  for (int c = threadIdx.x; c < wide; c += kThreads) {
    to[c] = gamma && c < f ? gamma[c] : 1.f;
    to[wide + c] = beta && c < f ? beta[c] : 0.f;
  }
  __syncthreads();
}

template <class T>
__device__ __forceinline__ void from_lds(const float *p, float (&v)[T::E]) {
#pragma unroll
  for (int e = 0; e < T::E; e += 4) {
    const op_f32x4 q = *reinterpret_cast<const op_f32x4 *>(p + e);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[e + k] = q[k];
  }
}
template <class T>
__device__ __forceinline__ void to_lds(float *p, const float (&v)[T::E]) {
#pragma unroll
  for (int e = 0; e < T::E; e += 4) *reinterpret_cast<op_f32x4 *>(p + e) = op_f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
}
// Two values of its group for each element of the vector from channel c on, from a[groups] and b[groups].
template <class T>
__device__ __forceinline__ void of_groups(const RowShape &sp, int c, const float *a, const float *b, float (&x)[T::E], float (&y)[T::E]) {
  if (sp.cg % T::E == 0) {
    const int g = group_of(sp.magic, c);
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      x[e] = a[g];
      y[e] = b[g];
    }
  } else {
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      const int g = group_of(sp.magic, c + e < sp.f ? c + e : sp.f - 1);
      x[e] = a[g];
      y[e] = b[g];
    }
  }
}

// Floats of LDS: the workgroup's gamma and beta, and for each of its samples `images` images and
// 2 images values for every group.
inline int64_t any_lds(const RowShape &sp, int e, int slots, int images) {
  return 2 * (int64_t)sp.vecs * e + slots * images * ((int64_t)sp.all * e + (2 * sp.groups + 3) / 4 * 4);
}

template <class T, int kLanes, int kVecs>
__global__ __launch_bounds__(kThreads, kVecs * T::E <= 16 ? 4 : 2) void any_fwd_kernel(pgcn_group_norm_fwd_args a, RowShape sp) {
  extern __shared__ __align__(16) float lds_any[];
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes, wide = sp.vecs * T::E;
  const float *params = lds_any;
  float *image = lds_any + 2 * wide + slot * (sp.all * T::E + (2 * sp.groups + 3) / 4 * 4), *mu = image + sp.all * T::E, *rs = mu + sp.groups;
  int c0[kVecs], row[kVecs];
  place_vectors<T, kLanes>(sp, c0, row);
  stage_params(a.gamma, a.beta, sp.f, wide, lds_any);
  const float inv_n = 1.0f / ((float)sp.cg * (float)sp.rows);
  const int t = lane & (sp.team - 1), teams = kLanes / sp.team;
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / kLanes) + slot; r < a.samples; r += (int64_t)gridDim.x * (kThreads / kLanes)) {
    float x[kVecs][T::E];
    load_rows<T>(a.X, r * sp.rows, a.ld_x, sp.f, c0, row, x);
    row_sync<kLanes>();                            // the sample before is done with the image
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (c0[i] < sp.f) to_lds<T>(image + (lane + kLanes * i) * T::E, x[i]);
    row_sync<kLanes>();
    for (int g0 = 0; g0 < sp.groups; g0 += teams) {                   // the same rounds for every lane
      const int g = g0 + lane / sp.team;
      const bool in = g < sp.groups;
      float s = 0.f, q = 0.f;
      if (in) group_walk(sp, wide, g, t, [&](int at) { s += image[at]; });
      const float m = team_sum(s, sp.team) * inv_n;
      if (in)
        group_walk(sp, wide, g, t, [&](int at) {
          const float d = image[at] - m;
          q += d * d;
        });
      q = 1.0f / sqrtf(team_sum(q, sp.team) * inv_n + a.eps);
      if (in && t == 0) {
        mu[g] = m;
        rs[g] = q;
        if (a.mean) a.mean[r * sp.groups + g] = m;
        if (a.rstd) a.rstd[r * sp.groups + g] = q;
      }
    }
    row_sync<kLanes>();
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (c0[i] >= sp.f) continue;
      float gm[T::E], gr[T::E], ga[T::E], be[T::E];
      of_groups<T>(sp, c0[i], mu, rs, gm, gr);
      from_lds<T>(params + c0[i], ga);
      from_lds<T>(params + wide + c0[i], be);
#pragma unroll
      for (int e = 0; e < T::E; ++e) x[i][e] = affine(normed(x[i][e], gm[e], gr[e]), ga[e], be[e]);
      activate<T>(x[i], a.act);
      store_some<T>((typename T::type *)a.Y + (r * sp.rows + row[i]) * a.ld_y + c0[i], x[i], sp.f - c0[i]);
    }
  }
}

// Four waves to a SIMD are worth the four registers spilt outside the loop (128 of 136), us at three
// and at four: 100,000 x 300 in 4 groups fp32 189 and 135, bf16 157 and 123; 10,000 x 2 x 1,024 in
// 8 groups 98 and 69, 82 and 61.  A kernel for samples of one row that kept all but the sums in registers
// took 115 for the first.
template <class T, int kLanes, int kVecs>
__global__ __launch_bounds__(kThreads, kVecs * T::E <= 8 ? 4 : kVecs * T::E <= 16 ? 2 : 1) void any_bwd_kernel(
    pgcn_group_norm_bwd_args a, RowShape sp, float *part) {
  extern __shared__ __align__(16) float lds_any[];
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes, wide = sp.vecs * T::E;
  const float *params = lds_any;
  // images of gamma du and xhat; mean and 1 / deviation, then the two sums, for every group
  float *image = lds_any + 2 * wide + slot * 2 * (sp.all * T::E + (2 * sp.groups + 3) / 4 * 4), *xhat = image + sp.all * T::E;
  float *mu = xhat + sp.all * T::E, *rs = mu + sp.groups, *c1 = rs + sp.groups, *c2 = c1 + sp.groups;
  int c0[kVecs], row[kVecs];
  place_vectors<T, kLanes>(sp, c0, row);
  stage_params(a.gamma, a.beta, sp.f, wide, lds_any);
  float s1[kVecs][T::E] = {}, s2[kVecs][T::E] = {};
  const float inv_n = 1.0f / ((float)sp.cg * (float)sp.rows);
  const int t = lane & (sp.team - 1), teams = kLanes / sp.team;
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / kLanes) + slot; r < a.samples; r += (int64_t)gridDim.x * (kThreads / kLanes)) {
    float x[kVecs][T::E], j[kVecs][T::E];
    load_rows<T>(a.X, r * sp.rows, a.ld_x, sp.f, c0, row, x);
    load_rows<T>(a.J_out, r * sp.rows, a.ld_j_out, sp.f, c0, row, j);
    row_sync<kLanes>();                            // the sample before is done with its values
    for (int g = lane; g < sp.groups; g += kLanes) {
      mu[g] = a.mean[r * sp.groups + g];
      rs[g] = a.rstd[r * sp.groups + g];
    }
    row_sync<kLanes>();
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (c0[i] >= sp.f) continue;
      float gm[T::E], gr[T::E], ga[T::E], be[T::E], u[T::E];
      of_groups<T>(sp, c0[i], mu, rs, gm, gr);
      from_lds<T>(params + c0[i], ga);
      from_lds<T>(params + wide + c0[i], be);
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        x[i][e] = normed(x[i][e], gm[e], gr[e]);
        u[e] = affine(x[i][e], ga[e], be[e]);
      }
      times_slope<T>(j[i], u, a.act);
#pragma unroll
      for (int e = 0; e < T::E; ++e) {
        if (c0[i] + e >= sp.f) j[i][e] = x[i][e] = 0.f;
        s1[i][e] += j[i][e];
        s2[i][e] += j[i][e] * x[i][e];
        j[i][e] *= ga[e];
      }
      to_lds<T>(image + (lane + kLanes * i) * T::E, j[i]);
      to_lds<T>(xhat + (lane + kLanes * i) * T::E, x[i]);
    }
    if (!a.J_in) continue;
    row_sync<kLanes>();
    for (int g0 = 0; g0 < sp.groups; g0 += teams) {
      const int g = g0 + lane / sp.team;
      float s = 0.f, q = 0.f;
      if (g < sp.groups)
        group_walk(sp, wide, g, t, [&](int at) {
          const float v = image[at];
          s += v;
          q += v * xhat[at];
        });
      s = team_sum(s, sp.team) * inv_n;
      q = team_sum(q, sp.team) * inv_n;
      if (g < sp.groups && t == 0) {
        c1[g] = s;
        c2[g] = q;
      }
    }
    row_sync<kLanes>();
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (c0[i] >= sp.f) continue;
      float g1[T::E], g2[T::E], gm[T::E], gr[T::E], xv[T::E], jv[T::E];
      of_groups<T>(sp, c0[i], c1, c2, g1, g2);
      of_groups<T>(sp, c0[i], mu, rs, gm, gr);
      from_lds<T>(image + (lane + kLanes * i) * T::E, jv);
      from_lds<T>(xhat + (lane + kLanes * i) * T::E, xv);
#pragma unroll
      for (int e = 0; e < T::E; ++e) xv[e] = gr[e] * (jv[e] - g1[e] - xv[e] * g2[e]);
      store_some<T>((typename T::type *)a.J_in + (r * sp.rows + row[i]) * a.ld_j_in + c0[i], xv, sp.f - c0[i]);
    }
  }
  if (!part) return;
  __syncthreads();
  write_channel_sums<T, kLanes>(sp, c0, s1, s2, part + (int64_t)blockIdx.x * 2 * sp.f, lds_any);
}

// part[n][2][channels] summed over n.
int launch_param_grads(const float *part, int64_t n, int channels, float *dgamma, float *dbeta, hipStream_t s) {
  hipLaunchKernelGGL(param_grads_kernel, dim3((unsigned)((2 * channels + 31) / 32)), dim3(kThreads), 0, s, part, n, channels, dgamma,
                     dbeta);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

// ---- launches: rows --------------------------------------------------------

bool is_pow2(int x) { return (x & (x - 1)) == 0; }

constexpr int kRowElems = 32 * kThreads;          // of the largest sample that fits: 8 fp32 or 4 bf16 vectors to a thread

RowShape row_shape(int32_t dtype, int32_t f, int32_t groups, int64_t sample_rows) {
  const int e = dtype == PGCN_BF16 ? BF16::E : F32::E;
  RowShape sp;
  sp.f = f;
  sp.groups = groups;
  sp.cg = f / groups;
  sp.vecs = (f + e - 1) / e;
  sp.rows = (int)sample_rows;
  sp.all = sp.vecs * sp.rows;
  sp.span = sp.rows == 1 && sp.cg % e == 0 ? sp.cg / e : 0;
  sp.magic = group_magic(sp.cg);
  sp.team = 1;
  return sp;
}

// Whether lanes shuffle a group's sum, or all add up one.
bool plain_groups(const RowShape &sp, int lanes) {
  return sp.groups == 1 || (sp.span > 0 && is_pow2(sp.span) && sp.span <= std::min(lanes, 64));
}

constexpr int kMaxLds = 150 << 10;      // of a compute unit's 160 KB

// Threads and vectors of a sample: the fewest lanes that hold it in one vector each, a wave up to
// two, then a workgroup up to kRowElems.  us of 30,000 rows, a wave of four vectors and a workgroup
// of one: forward / backward of 1,024 fp32 channels 53 / 91 and 50 / 80, of 2,048 bf16 ones
// 94 / 271 and 65 / 111.  A wave of two and a workgroup of one half idle: 100,000 x 300 fp32 in four
// groups 108 / 135 and 249 / 258.
// false: the sample goes in chunks.  us here and in chunks, forward / backward: 100,000 x 4 x 64 in
// 8 groups 80 / 95 and 564 / 1,364; 5,000 x 32 x 100 in 5 groups 39 / 91 and 55 / 129.  Groups of
// several rows pay for LDS by the element and fp32 chunks win from 4,096 elements on: 5,000 x
// 64 x 96 fp32 87 / 207 and 79 / 161, but bf16 68 / 158 and 91 / 203.
bool row_threads(int32_t dtype, int32_t f, int32_t groups, int64_t sample_rows, int images, RowShape &sp, int &lanes, int &per, bool &plain) {
  const int e = dtype == PGCN_BF16 ? BF16::E : F32::E;
  if (sample_rows > kRowElems || (f + e - 1) / e * e * sample_rows > kRowElems) return false;
  sp = row_shape(dtype, f, groups, sample_rows);
  const int vecs = sp.all;
  lanes = vecs <= 4 ? 4 : vecs <= 8 ? 8 : vecs <= 16 ? 16 : vecs <= 32 ? 32 : vecs <= 128 ? 64 : kThreads;
  plain = plain_groups(sp, lanes);
  if (!plain) lanes = std::max(lanes, 8);
  per = 1;
  while (lanes * per < vecs) per *= 2;
  while (sp.team < 64 && 2 * sp.team * sp.groups <= lanes) sp.team *= 2;
  if (plain) return true;
  return (sample_rows == 1 || per <= 4) && 4 * any_lds(sp, e, kThreads / lanes, images) <= kMaxLds;
}

constexpr int kRowBlocksFwd = 2048, kRowBlocksBwd = 1024;

unsigned row_blocks(int64_t rows, int lanes, int most) {
  const int64_t n = kThreads / lanes, b = (rows + n - 1) / n;
  return (unsigned)std::min<int64_t>(b, most);
}

// LDS bytes of a backward: the sums' join, and what the kernel itself takes.
template <class T>
size_t join_lds(const RowShape &sp, int lanes) {
  return 4 * (size_t)(sp.rows > 1 ? kThreads / lanes * sp.all * T::E : kThreads * T::E);
}

template <class T, int kLanes, int kVecs, Sum kSum>
int rows_go(const pgcn_group_norm_fwd_args &a, const RowShape &sp, hipStream_t s) {
  hipLaunchKernelGGL((rows_fwd_kernel<T, kLanes, kVecs, kSum>), dim3(row_blocks(a.samples, kLanes, kRowBlocksFwd)), dim3(kThreads), 0, s, a,
                     sp);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

template <class T, int kLanes, int kVecs, Sum kSum>
int rows_go(const pgcn_group_norm_bwd_args &a, const RowShape &sp, hipStream_t s) {
  const unsigned blocks = row_blocks(a.samples, kLanes, kRowBlocksBwd);
  float *part = a.dgamma || a.dbeta ? (float *)a.workspace : nullptr;
  if (!part && !a.J_in) return PGCN_OK;
  hipLaunchKernelGGL((rows_bwd_kernel<T, kLanes, kVecs, kSum>), dim3(blocks), dim3(kThreads), join_lds<T>(sp, kLanes), s, a, sp, part);
  PGCN_HIP(hipGetLastError());
  return part ? launch_param_grads(part, blocks, a.channels, a.dgamma, a.dbeta, s) : PGCN_OK;
}

template <class T, int kLanes, int kVecs>
int any_go(const pgcn_group_norm_fwd_args &a, const RowShape &sp, hipStream_t s) {
  hipLaunchKernelGGL((any_fwd_kernel<T, kLanes, kVecs>), dim3(row_blocks(a.samples, kLanes, kRowBlocksFwd)), dim3(kThreads),
                     4 * (size_t)any_lds(sp, T::E, kThreads / kLanes, 1), s, a, sp);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

template <class T, int kLanes, int kVecs>
int any_go(const pgcn_group_norm_bwd_args &a, const RowShape &sp, hipStream_t s) {
  const unsigned blocks = row_blocks(a.samples, kLanes, kRowBlocksBwd);
  float *part = a.dgamma || a.dbeta ? (float *)a.workspace : nullptr;
  if (!part && !a.J_in) return PGCN_OK;
  const size_t lds = std::max(4 * (size_t)any_lds(sp, T::E, kThreads / kLanes, 2), join_lds<T>(sp, kLanes));
  hipLaunchKernelGGL((any_bwd_kernel<T, kLanes, kVecs>), dim3(blocks), dim3(kThreads), lds, s, a, sp, part);
  PGCN_HIP(hipGetLastError());
  return part ? launch_param_grads(part, blocks, a.channels, a.dgamma, a.dbeta, s) : PGCN_OK;
}

// The kernel of a sample's shape; `args` forward or backward.
template <class T, class Args>
int rows_of(const Args &a, const RowShape &sp, int lanes, int per, bool plain, hipStream_t s) {
  constexpr int kMost = T::E == 4 ? 8 : 4;
  if (!plain) {
    switch (lanes * 10 + per) {
      case 81: return any_go<T, 8, 1>(a, sp, s);
      case 161: return any_go<T, 16, 1>(a, sp, s);
      case 321: return any_go<T, 32, 1>(a, sp, s);
      case 641: return any_go<T, 64, 1>(a, sp, s);
      case 642: return any_go<T, 64, 2>(a, sp, s);
      case 2561: return any_go<T, 256, 1>(a, sp, s);
      case 2562: return any_go<T, 256, 2>(a, sp, s);
      case 2564: return any_go<T, 256, 4>(a, sp, s);
      default: return any_go<T, 256, kMost>(a, sp, s);
    }
  }
  const bool one = sp.groups == 1;
  switch (lanes * 10 + per) {
    case 41: return one ? rows_go<T, 4, 1, Sum::ROW>(a, sp, s) : rows_go<T, 4, 1, Sum::LANES>(a, sp, s);
    case 81: return one ? rows_go<T, 8, 1, Sum::ROW>(a, sp, s) : rows_go<T, 8, 1, Sum::LANES>(a, sp, s);
    case 161: return one ? rows_go<T, 16, 1, Sum::ROW>(a, sp, s) : rows_go<T, 16, 1, Sum::LANES>(a, sp, s);
    case 321: return one ? rows_go<T, 32, 1, Sum::ROW>(a, sp, s) : rows_go<T, 32, 1, Sum::LANES>(a, sp, s);
    case 641: return one ? rows_go<T, 64, 1, Sum::ROW>(a, sp, s) : rows_go<T, 64, 1, Sum::LANES>(a, sp, s);
    case 642: return one ? rows_go<T, 64, 2, Sum::ROW>(a, sp, s) : rows_go<T, 64, 2, Sum::LANES>(a, sp, s);
    case 2561: return one ? rows_go<T, 256, 1, Sum::ROW>(a, sp, s) : rows_go<T, 256, 1, Sum::LANES>(a, sp, s);
    case 2562: return one ? rows_go<T, 256, 2, Sum::ROW>(a, sp, s) : rows_go<T, 256, 2, Sum::LANES>(a, sp, s);
    case 2564: return one ? rows_go<T, 256, 4, Sum::ROW>(a, sp, s) : rows_go<T, 256, 4, Sum::LANES>(a, sp, s);
    default: return one ? rows_go<T, 256, kMost, Sum::ROW>(a, sp, s) : rows_go<T, 256, kMost, Sum::LANES>(a, sp, s);
  }
}

// ---- launches: samples of many rows ----------------------------------------

template <class T>
int chunks_fwd(const pgcn_group_norm_fwd_args &a, hipStream_t s) {
  const Cut cut = cut_rows(a.dtype, a.channels, a.groups, a.samples, a.sample_rows);
  float2 *part = (float2 *)a.workspace;
  hipLaunchKernelGGL(moments_kernel<T>, dim3((unsigned)(a.samples * cut.chunks)), dim3(kThreads),
                     4 * (2 * (size_t)a.channels + (size_t)a.groups), s, a, cut, part);
  PGCN_HIP(hipGetLastError());
  hipLaunchKernelGGL(normalise_kernel<T>, dim3((unsigned)(a.samples * cut.out_blocks)), dim3(kThreads), 8 * (size_t)a.groups, s, a, cut,
                     part);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

// Bytes of the chunks' group sums, before their channel sums.
size_t group_part_bytes(const Cut &cut, int32_t groups, int64_t samples) {
  return align_up(8 * (size_t)samples * (size_t)cut.chunks * (size_t)groups, 16);
}

int chunk_sum_blocks(const Cut &cut, int64_t samples) { return (int)std::min<int64_t>(samples * cut.chunks, kStatBlocks); }

template <class T>
int chunks_bwd(const pgcn_group_norm_bwd_args &a, hipStream_t s) {
  const Cut cut = cut_rows(a.dtype, a.channels, a.groups, a.samples, a.sample_rows);
  const bool params = a.dgamma || a.dbeta;
  if (a.samples == 0) return params ? launch_param_grads(nullptr, 0, a.channels, a.dgamma, a.dbeta, s) : PGCN_OK;
  if (!params && !a.J_in) return PGCN_OK;
  float2 *part = (float2 *)a.workspace;
  float *channel_part = params ? (float *)((char *)a.workspace + group_part_bytes(cut, a.groups, a.samples)) : nullptr;
  const int sum_blocks = chunk_sum_blocks(cut, a.samples);
  hipLaunchKernelGGL(grad_sums_kernel<T>, dim3((unsigned)sum_blocks), dim3(kThreads), 8 * (size_t)a.channels, s, a, cut,
                     part, channel_part);
  PGCN_HIP(hipGetLastError());
  const unsigned row_blocks = a.J_in ? (unsigned)(a.samples * cut.out_blocks) : 0;
  const unsigned param_blocks = params ? (unsigned)((2 * a.channels + 31) / 32) : 0;
  hipLaunchKernelGGL(grad_rows_kernel<T>, dim3(row_blocks + param_blocks), dim3(kThreads), 8 * (size_t)a.groups, s, a, cut, part,
                     channel_part, sum_blocks, (int)row_blocks);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace

size_t group_norm_workspace(int32_t dtype, int32_t channels, int32_t groups, int64_t samples, int64_t sample_rows) {
  if (samples == 0) return 0;
  RowShape sp;
  int lanes, per;
  bool plain;
  if (row_threads(dtype, channels, groups, sample_rows, 2, sp, lanes, per, plain))
    return 8 * (size_t)channels * row_blocks(samples, lanes, kRowBlocksBwd);
  const Cut cut = cut_rows(dtype, channels, groups, samples, sample_rows);
  return group_part_bytes(cut, groups, samples) + 8 * (size_t)channels * (size_t)chunk_sum_blocks(cut, samples);
}

int launch_group_norm_fwd(const pgcn_group_norm_fwd_args &a, hipStream_t s) {
  if (a.samples == 0) return PGCN_OK;
  TraceScope ts(PGCN_TK_GROUP_NORM, s);
  RowShape sp;
  int lanes, per;
  bool plain;
  if (row_threads(a.dtype, a.channels, a.groups, a.sample_rows, 1, sp, lanes, per, plain))
    return a.dtype == PGCN_BF16 ? rows_of<BF16>(a, sp, lanes, per, plain, s) : rows_of<F32>(a, sp, lanes, per, plain, s);
  return a.dtype == PGCN_BF16 ? chunks_fwd<BF16>(a, s) : chunks_fwd<F32>(a, s);
}

int launch_group_norm_bwd(const pgcn_group_norm_bwd_args &a, hipStream_t s) {
  TraceScope ts(PGCN_TK_GROUP_NORM_BWD, s);
  RowShape sp;
  int lanes, per;
  bool plain;
  if (a.samples > 0 && row_threads(a.dtype, a.channels, a.groups, a.sample_rows, 2, sp, lanes, per, plain))
    return a.dtype == PGCN_BF16 ? rows_of<BF16>(a, sp, lanes, per, plain, s) : rows_of<F32>(a, sp, lanes, per, plain, s);
  return a.dtype == PGCN_BF16 ? chunks_bwd<BF16>(a, s) : chunks_bwd<F32>(a, s);
}

}  // namespace pgcn
