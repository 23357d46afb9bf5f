// The largest logits of every row with their classes, and the log-sum of the others.
//
// Order: (value, lower class first) with -0 equal to +0; -inf and NaN are never listed.  Bound by
// one read of Z.  Three kernels:
//   - many short rows: a thread walks a row and keeps its list in registers (top_lists_kernel);
//   - longer rows: a wave or a workgroup holds a row in registers.  The list lies above a
//     threshold that at least `top` elements reach.  Each wave's r-th largest lane maximum, r =
//     top / waves, is tried, and the largest taken that `top` lane maxima reach.  What reaches it,
//     little more than `top` elements, goes to LDS, where each is ranked by counting.
//     Where too many reach it (ties, sorted rows) the threshold is bisected, and among equal
//     values the class;
//   - rows longer than that: parts of a row first, then the lists of its parts.
// The log-sum is one more pass over the registers, with no test for what is listed: an exponential's
// clamp makes 1 of each listed one, and their number is taken off the sum.
// Bound by the instructions for an element (unpack, maximum, compare, product-sum, exponential, sum) where
// rows fill the chip: vector instructions are issued in 0.8 of all cycles of 2,048 x 65,536 top 64, fp32 148 us
// (3.6 TB/s), bf16 101 us (2.7 TB/s), and of 20,000 x 250 top 128, 56 us, most of it ranking; joining 2,048
// rows' parts takes 17 us.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "ops.h"

namespace pgcn {

namespace {

// Order of (value, lowest class first) as whole numbers.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }

// ---- a row in the registers of a wave or a workgroup ----------------------------------------

struct TopArgs {
  const void *Z;
  int64_t rows, ld, ld_top;
  int classes, top, fill;      // slots from the last listed one to `fill` hold -inf and -1
  int range, parts;            // a unit of work: classes [part range, (part + 1) range) of a row
  float inv_t;
  float *values;               // [units][ld_top]
  int32_t *ids;
  float *tail;                 // [rows], or null
  float2 *part_tail;           // [units]: maximum and sum instead of their logarithm, or null
  const int32_t *listed_ids;   // the row is a list of `classes` entries with these ids, or null
  const float2 *listed_tails;  // and `tails` log-sums for every row
  int tails;
};

// f(x, class, true) for n elements read again from memory, by a unit's threads in the order of the
// registers; f(., ., false) past the end, so that all lanes take the same turns.
template <class T, int kThreads, class F>
__device__ __forceinline__ void each_in_memory(const typename T::type *z, int n, int lane, F f) {
#pragma unroll 1
  for (int c0 = lane * T::E; c0 - lane * T::E < n; c0 += kThreads * T::E) {
    const typename T::raw raw = c0 < n ? *reinterpret_cast<const typename T::raw *>(z + c0) : typename T::raw{};
    float x[T::E];
    T::unpack(raw, x);
#pragma unroll
    for (int e = 0; e < T::E; ++e) f(x[e], c0 + e, c0 + e < n);
  }
}

// Candidates of a wave, and of a unit's waves together.
constexpr int wave_candidates(int waves) { return waves == 1 ? 192 : waves == 4 ? 192 : 96; }

template <int kThreads>
struct TopLds {
  static constexpr int kWaves = kThreads / 64, kEach = wave_candidates(kWaves);
  uint64_t found[kWaves > 1 ? kWaves * kEach : 1];     // by wave
  uint64_t list[kWaves * kEach];                       // one after another
  float wave_f[2][kWaves];
  int wave_n[2][kWaves], reach[kWaves][kWaves];
  int count, ties;
  uint64_t last;               // key of rank top - 1
};

template <int kThreads>
__device__ __forceinline__ void unit_sync() {
  if (kThreads > 64) __syncthreads();
  else wave_sync();
}

// Over the unit's waves, one after another; `turn` alternates the buffers between calls, so that one
// barrier a call is enough.
template <int kThreads>
__device__ __forceinline__ int waves_add(int n, TopLds<kThreads> &l, int &turn) {
  if (kThreads == 64) return n;
  turn ^= 1;
  if (threadIdx.x % 64 == 0) l.wave_n[turn][threadIdx.x / 64] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) n += l.wave_n[turn][w];
  return n;
}
template <int kThreads, class Op>
__device__ __forceinline__ float waves_all(float v, TopLds<kThreads> &l, int &turn, Op op) {
  if (kThreads == 64) return v;
  turn ^= 1;
  if (threadIdx.x % 64 == 0) l.wave_f[turn][threadIdx.x / 64] = v;
  __syncthreads();
  v = l.wave_f[turn][0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v = op(v, l.wave_f[turn][w]);
  return v;
}

// A value that at least r of a wave's 64 reach and few more: their r-th largest, less at most 2^14
// units in the last place.
__device__ __forceinline__ float reached_by(float v, int r) {
  uint32_t lo = __builtin_amdgcn_readfirstlane(order_of(-lanes_max<64>(-v)));
  uint32_t hi = __builtin_amdgcn_readfirstlane(order_of(lanes_max<64>(v))) + 1;
  while (hi - lo > 1u << 14) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (__popcll(__ballot(v >= value_of(mid))) >= r) lo = mid;
    else hi = mid;
  }
  return value_of(lo);
}

// Waves to a SIMD: as many as spill (next to) nothing.  8 vectors of bf16 at five waves, 15 registers
// spilt, and at four: 2,048 x 65,536 top 8 111 and 83 us, 4,096 x 32,768 122 and 90.
template <class T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads < 256 ? 256 : kThreads, kVecs <= 2 ? 8 : T::E == 4 ? 7 : kVecs == 4 ? 6 : 4) void top_unit_kernel(
    TopArgs a) {
  constexpr int kUnits = kThreads < 256 ? 256 / kThreads : 1, kWaves = kThreads / 64;
  __shared__ TopLds<kThreads> lds[kUnits];
  const int lane = threadIdx.x % kThreads, slot = threadIdx.x / kThreads;
  TopLds<kThreads> &l = lds[slot];
  const int64_t unit = (int64_t)blockIdx.x * kUnits + slot;
  if (unit >= a.rows * a.parts) return;            // whole waves; a workgroup of several units has no barrier
  const int64_t row = unit / a.parts;
  const int first = (int)(unit - row * a.parts) * a.range, n_all = a.classes - first < a.range ? a.classes - first : a.range;
  const int K = a.top;
  const typename T::type *z = (const typename T::type *)a.Z + row * a.ld + first;
  typename T::raw raw[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c0 = (lane + kThreads * i) * T::E;
    raw[i] = c0 < n_all ? *reinterpret_cast<const typename T::raw *>(z + c0) : typename T::raw{};
  }
  float top = kNegInf;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c0 = (lane + kThreads * i) * T::E;
    float x[T::E];
    T::unpack(raw[i], x);
    if (c0 + T::E > n_all) {
#pragma unroll
      for (int e = 0; e < T::E; ++e)
        if (c0 + e >= n_all) x[e] = kNegInf;
      raw[i] = T::pack(x);
    }
#pragma unroll
    for (int e = 0; e < T::E; ++e) top = __builtin_elementwise_maximum(top, x[e]);      // a NaN passes on
    __builtin_amdgcn_sched_barrier(0);
  }
  const bool nan = top != top;
  if (__ballot(nan)) {                             // and is no maximum
    top = kNegInf;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float x[T::E];
      T::unpack(raw[i], x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) top = fmaxf(top, x[e]);
    }
  }

  int turn = 0;
  const int most = K + (kWaves > 1 ? 128 : 63);    // candidates to rank
  const int vecs = (n_all + T::E - 1) / T::E, maxima = vecs < kThreads ? vecs : kThreads;
  // The wave's share of K lane maxima.  Above 64 there is no threshold: more slots than maxima, or a short row
  // in one wave, whose idle lanes count in 64 too; its list is found by bisection.
  const int r = (64 * K + maxima - 1) / maxima;
  float v = kNegInf;                               // a short row is its own list of candidates
  if (n_all > most && r <= 64) v = reached_by(top, r);
  if (kWaves > 1 && n_all > most && r <= 64) {
    // every wave's value is a candidate: the largest that K lane maxima of the unit reach (all reach the smallest)
    if (threadIdx.x % 64 == 0) l.wave_f[0][threadIdx.x / 64] = v;
    __syncthreads();
    int reach = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int k = __popcll(__ballot(top >= l.wave_f[0][w]));
      reach = threadIdx.x % 64 == w ? k : reach;
    }
    if (threadIdx.x % 64 < kWaves) l.reach[threadIdx.x / 64][threadIdx.x % 64] = reach;
    __syncthreads();
    v = kNegInf;
    if (threadIdx.x % 64 < kWaves) {
      int k = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) k += l.reach[w][threadIdx.x % 64];
      if (k >= K) v = l.wave_f[0][threadIdx.x % 64];
    }
    v = lanes_max<64>(v);
  }
  v = fmaxf(v, -FLT_MAX);                          // x >= v: every x above -inf
  constexpr int kEach = TopLds<kThreads>::kEach;
  const int wave = kWaves > 1 ? threadIdx.x / 64 : 0, wl = threadIdx.x % 64;
  uint64_t *found = kWaves > 1 ? l.found + wave * kEach : l.list;
  int mine = 0;                                    // of this wave
  keep_packed(raw);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    float x[T::E];
    T::unpack(raw[i], x);
#pragma unroll
    for (int e = 0; e < T::E; ++e) {
      const uint64_t in = __ballot(x[e] >= v);
      if (in) {
        const int at = mine + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0));
        if (x[e] >= v && at < kEach)
          found[at] = ((uint64_t)order_of(x[e]) << 32) | (uint32_t)~((lane + kThreads * i) * T::E + e);
        mine += __popcll(in);
      }
    }
    __builtin_amdgcn_sched_barrier(0);             // one vector at a time: their temporaries do not add up
  }
  int n = mine, ties = 0;                          // ties: equal to the last listed value, not listed and not in the list
  bool over = mine > kEach;
  if (kWaves > 1) {
    turn ^= 1;
    if (wl == 0) l.wave_n[turn][wave] = mine;
    __syncthreads();
    int before = 0;
    n = 0;
    over = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int k = l.wave_n[turn][w];
      before += w < wave ? k : 0;
      n += k;
      over |= k > kEach;
    }
    if (n <= most && !over)
      for (int j = wl; j < mine; j += 64) l.list[before + j] = found[j];
  }
  if (lane == 0) l.count = l.ties = 0;
  unit_sync<kThreads>();
  if (n > most || over) {                          // ties, or a row in some order: bisect
    auto visit = [&](auto f) {                     // few registers are walked again, many would be held twice
      if constexpr (kVecs <= 4) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          float x[T::E];
          T::unpack(raw[i], x);
#pragma unroll
          for (int e = 0; e < T::E; ++e) f(x[e], (lane + kThreads * i) * T::E + e, true);
        }
      } else {
        each_in_memory<T, kThreads>(z, n_all, lane, f);
      }
    };
    auto count = [&](auto in) {
      int k = 0;
      visit([&](float x, int c, bool ok) { k += __popcll(__ballot(ok && in(x, c))); });
      return waves_add<kThreads>(k, l, turn);
    };
    const float m = waves_all<kThreads>(lanes_max<64>(top), l, turn, [](float x, float y) { return fmaxf(x, y); });
    uint32_t lo = order_of(v), hi = order_of(m) + 1;
    int above = 0;                                 // elements from `hi` on
    n = count([&](float x, int) { return x >= v; });
    while (n > most && hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const float y = value_of(mid);
      const int k = count([&](float x, int) { return x >= y; });
      if (k >= K) {
        lo = mid;
        n = k;
      } else {
        hi = mid;
        above = k;
      }
    }
    const float tie = value_of(lo);
    int upto = n_all;
    if (n > most) {                                // all of them equal but for `above` < K: the lowest classes
      int from = -1, to = n_all - 1;
      while (to - from > 1) {
        const int mid = (from + to) / 2;
        if (above + count([&](float x, int c) { return x == tie && c <= mid; }) >= K) to = mid;
        else from = mid;
      }
      upto = to;
      ties = n - K;
      n = K;
    }
    visit([&](float x, int c, bool ok) {
      if (ok && (x > tie || (x == tie && c <= upto)))
        l.list[atomicAdd(&l.count, 1)] = ((uint64_t)order_of(x) << 32) | (uint32_t)~c;     // any order: what follows goes by rank
    });
    unit_sync<kThreads>();
  }
  float *values = a.values + unit * a.ld_top;
  int32_t *ids = a.ids + unit * a.ld_top;
  // A thread's keys together against each key of the list (at most 191 of a wave, 384 of a workgroup), us one
  // after another and together: 127,010 x 116 top 75 fp32 219 and 171, 20,000 x 250 top 128 81 and 57.
  auto ranked = [&](auto keys_) {
    constexpr int kKeys = decltype(keys_)::value;
    uint64_t key[kKeys];
    int rank[kKeys] = {};
#pragma unroll
    for (int q = 0; q < kKeys; ++q) key[q] = lane + q * kThreads < n ? l.list[lane + q * kThreads] : 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const uint64_t other = l.list[i];
#pragma unroll
      for (int q = 0; q < kKeys; ++q) rank[q] += other > key[q] ? 1 : 0;
    }
#pragma unroll
    for (int q = 0; q < kKeys; ++q) {
      if (lane + q * kThreads >= n) continue;
      if (rank[q] < K) {
        const int c = (int)~(uint32_t)key[q];
        values[rank[q]] = value_of((uint32_t)(key[q] >> 32));
        ids[rank[q]] = a.listed_ids ? a.listed_ids[row * a.ld + c] : first + c;
      }
      if (rank[q] == K - 1) l.last = key[q];
    }
  };
  if (n <= kThreads) ranked(std::integral_constant<int, 1>{});
  else if (n <= 2 * kThreads) ranked(std::integral_constant<int, 2>{});
  else if constexpr (kThreads == 64) ranked(std::integral_constant<int, 3>{});
  for (int k = (n < K ? n : K) + lane; k < a.fill; k += kThreads) {
    values[k] = kNegInf;
    ids[k] = -1;
  }
  if (!a.tail && !a.part_tail) return;

  // the others: below the last listed value, and what equals it and is not listed
  unit_sync<kThreads>();
  const float scale = a.inv_t * kLog2e;
  const float last = n >= K ? value_of((uint32_t)(l.last >> 32)) : -FLT_MAX;       // all above -inf are listed
  float m = last;                                  // no exponent of the others is above 0
  float s = 0.f;
  if (last <= FLT_MAX && n_all > 2 * K) {
    // all of them, each at most 1: the listed ones count for 1, which the sum holds exactly.  Where
    // they are not most of it, taking them off again loses no more than a bit.
    const Exps ex(m, scale);
    float s0 = 0.f, s1 = 0.f;
    keep_packed(raw);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float x[T::E];
      T::unpack(raw[i], x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) (e % 2 ? s1 : s0) += __builtin_amdgcn_fmed3f(ex.raw(x[e]), 0.f, 1.f);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (nan) s0 = __builtin_nanf("");
    s = waves_all<kThreads>(lanes_sum<64>(s0 + s1), l, turn, [](float x, float y) { return x + y; });
    const float listed = (float)(n < K ? n : K);
    s = s - listed < listed ? 0.f : (s - listed) * ex.fix;
  }
  if (s == 0.f) {                                  // the others alone, from their own maximum
    if (n >= K) {                                  // those equal to the last listed one
      const uint64_t key = l.last;
      for (int j = lane; j < n; j += kThreads)
        if (l.list[j] < key && (l.list[j] >> 32) == (key >> 32)) atomicAdd(&l.ties, 1);
      unit_sync<kThreads>();
      ties += l.ties;
    }
    m = kNegInf;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float x[T::E];
      T::unpack(raw[i], x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) m = fmaxf(m, x[e] >= last ? kNegInf : x[e]);
    }
    m = waves_all<kThreads>(lanes_max<64>(ties ? last : m), l, turn, [](float x, float y) { return fmaxf(x, y); });
    const Exps ex(fabsf(m) <= FLT_MAX ? m : 0.f, scale);
    float s0 = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float x[T::E];
      T::unpack(raw[i], x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) s0 += ex.raw(x[e] >= last ? kNegInf : x[e]);
    }
    s = waves_all<kThreads>(lanes_sum<64>(s0 * ex.fix), l, turn, [](float x, float y) { return x + y; });
    if (s == s) {
      if (m == INFINITY) s = 1.f;                  // an infinity that is not listed
      else s += (float)ties;
    }
  }
  if (threadIdx.x % kThreads >= 64) return;
  if (a.tails) {                                   // what the row's parts left out (at most 64)
    const float2 p = lane < a.tails ? a.listed_tails[row * a.tails + lane] : make_float2(kNegInf, 0.f);
    const float pm = lanes_max<64>(p.x), all = fmaxf(m, pm), b = all == kNegInf ? 0.f : all;
    const float ps = lanes_sum<64>(p.y == 0.f ? 0.f : p.y * exp_at(p.x, b, scale));
    s = (s == 0.f ? 0.f : s * exp_at(m, b, scale)) + ps;
    m = all;
  }
  if (lane == 0) {
    if (a.part_tail) a.part_tail[unit] = make_float2(m, s);
    else a.tail[row] = s == 0.f ? kNegInf : m * a.inv_t + __logf(s);
  }
}

// ---- a thread to a row ----------------------------------------------------------------------
//
// The list is kept sorted: x > v_i for some i on, and v_i becomes the middle one of v_{i-1}, x and
// v_i, its class the one that goes with it.  Classes come in ascending order, so of equal values the
// one that is there stays in front.  What falls out at the end is no part of the list any more and
// goes into the log-sum.  A wave's rows pass through LDS in tiles of kTile classes.  Bound by the
// list's instructions, 3 kSlots for a class, and their chain: 58,000 x 41 top 8 fp32 10.7 us, at under one wave
// to a SIMD, which issues vector instructions in 0.44 of its cycles; 306,000 x 47 31 us (2.5 TB/s, 0.65 of all
// cycles), bf16 29.

constexpr int kTile = 32, kStep = 4;

// Both are there: a select, and no branch.
template <class V>
__device__ __forceinline__ V pick(bool c, V a, V b) {
  return c ? a : b;
}

template <class T, int kSlots>
__global__ __launch_bounds__(256) void top_lists_kernel(pgcn_top_logits_args a) {
  constexpr int kAcross = kTile / T::E, kDown = 64 / kAcross, kLoads = 64 / kDown;
  __shared__ float tile_[4][64 * (kTile + 1)];
  const int lane = threadIdx.x % 64, C = a.classes, K = a.top;
  float *tile = tile_[threadIdx.x / 64];
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / 64) * 64;
  if (row0 >= a.rows) return;
  const float scale = kLog2e / a.temperature;
  const int tx = lane % kAcross, ty = lane / kAcross;
  typename T::raw raw[kLoads];
  auto load = [&](int c0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int64_t r = row0 + ty + kDown * i;
      const int c = c0 + tx * T::E;
      raw[i] = r < a.rows && c < C ? *reinterpret_cast<const typename T::raw *>((const typename T::type *)a.Z + r * a.ld + c)
                                   : typename T::raw{};
    }
  };
  float v[kSlots];
  int ids[kSlots];
#pragma unroll
  for (int k = 0; k < kSlots; ++k) {
    v[k] = kNegInf;
    ids[k] = -1;
  }
  float m = kNegInf, s = 0.f;
  bool nan = false, inf = false;
  // kStep values that are no part of the list: one rescaling of the sum for all of them
  auto left_out = [&](const float (&x)[kStep]) {
    float big = m;
#pragma unroll
    for (int i = 0; i < kStep; ++i) big = pick(x[i] > big, x[i], big);
    inf |= big > FLT_MAX;                          // an infinity that is not listed
    const float base = pick(big > kNegInf, big, 0.f);
    float add[kStep];
#pragma unroll
    for (int i = 0; i < kStep; ++i) add[i] = exp_at(x[i], base, scale);
    s = __builtin_fmaf(s, exp_at(m, base, scale), (add[0] + add[1]) + (add[2] + add[3]));
    m = big;
  };
  load(0);
  for (int c0 = 0; c0 < C; c0 += kTile) {
    wave_sync();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float x[T::E];
      T::unpack(raw[i], x);
#pragma unroll
      for (int e = 0; e < T::E; ++e)
        tile[(ty + kDown * i) * (kTile + 1) + tx * T::E + e] = c0 + tx * T::E + e < C ? x[e] : kNegInf;
    }
    wave_sync();
    if (c0 + kTile < C) load(c0 + kTile);
    const int n = C - c0 < kTile ? C - c0 : kTile;
    for (int c = 0; c < n; c += kStep) {           // past C the tile holds -inf
      float x[kStep];
#pragma unroll
      for (int j = 0; j < kStep; ++j) x[j] = tile[lane * (kTile + 1) + c + j];
#pragma unroll
      for (int j = 0; j < kStep; ++j) {
        nan |= x[j] != x[j];
        const float y = pick(x[j] == x[j], x[j], kNegInf);
        x[j] = pick(y > v[kSlots - 1], v[kSlots - 1], y);
#pragma unroll
        for (int i = kSlots - 1; i >= 0; --i) {
          ids[i] = pick(y > v[i], c0 + c + j, ids[i]);
          if (i > 0) ids[i] = pick(y > v[i - 1], ids[i - 1], ids[i]);
          v[i] = i > 0 ? __builtin_amdgcn_fmed3f(v[i - 1], y, v[i]) : pick(y > v[0], y, v[0]);
        }
      }
      left_out(x);
    }
  }
#pragma unroll
  for (int k = 0; k < kSlots; k += kStep) {
    float x[kStep];
#pragma unroll
    for (int j = 0; j < kStep; ++j) x[j] = k + j < K ? kNegInf : v[k + j];
    if (k + kStep > K) left_out(x);
  }
  // the lists by way of the tile, so that neighbouring lanes write neighbouring slots
  constexpr int kSide = kSlots < kTile ? kSlots : kTile;
  const int kx = lane % kSide, ky = lane / kSide;
  auto write = [&](auto *out, auto *slots, auto value) {
#pragma unroll
    for (int k0 = 0; k0 < kSlots; k0 += kSide) {
      wave_sync();
#pragma unroll
      for (int k = 0; k < kSide; ++k) slots[lane * (kTile + 1) + k] = value(k0 + k);
      wave_sync();
      if (k0 + kx < K)
#pragma unroll 4
        for (int i = ky; i < 64; i += 64 / kSide)
          if (row0 + i < a.rows) out[(row0 + i) * a.ld_top + k0 + kx] = slots[i * (kTile + 1) + kx];
    }
  };
  write(a.top_values, tile, [&](int k) { return v[k]; });
  write(a.top_ids, (int32_t *)tile, [&](int k) { return ids[k]; });
  const int64_t r = row0 + lane;
  if (r >= a.rows) return;
  if (a.tail_lse) a.tail_lse[r] = nan ? __builtin_nanf("") : inf ? INFINITY : s == 0.f ? kNegInf : m / a.temperature + __logf(s);
}

// ---- launches -------------------------------------------------------------------------------

int vector_elems(int32_t dtype) { return dtype == PGCN_BF16 ? BF16::E : F32::E; }

// Vectors of the longest row that a workgroup holds: the register file's limit in bf16; 4,096 x 32,768
// fp32 top 8 whole 148 us, in parts 129, top 64 both 162.  Few rows are not cut for the sake of more
// workgroups: the second launch costs more, 1 x 16,000 fp32 top 50 7.9 us whole, 7.5 + 9.9 in parts,
// 8 x 32,000 bf16 top 8 9.1 and 7.0 + 5.0.
constexpr int kLongVecs = 4096;
// Vectors of a part of a row: long ones share the cost of a part's threshold.  1,024 and 2,048, us of
// 2,048 x 65,536: fp32 top 8 157 and 126, top 64 206 and 151, top 256 562 and 420; bf16 top 64 131 and
// 109, top 256 365 and 269; 1 x 100,003 fp32 top 50 both 17, 128 x 100,003 bf16 top 64 31 and 28.
constexpr int kPartVecs = 2048;

// Parts of a row, 1: the whole of it at once.
int top_parts(int32_t dtype, int32_t classes) {
  const int e = vector_elems(dtype), range = kPartVecs * e;
  return classes > kLongVecs * e ? (classes + range - 1) / range : 1;
}

// Whether a thread takes a row: fits to both kernels' times, in us.  A thread's walk is a chain, so few
// rows cost its length and many rows their instructions; a unit costs about the same for any row
// that it holds.  Lists and units, us: 1,000 x 41 top 8 9.7, 5; 58,000 x 41 top 8 11.8, 36; 58,000 x
// 100 top 64 75, 90; 306,000 x 64 top 16 56, 180; 306,000 x 200 top 16 154, 270; 306,000 x 500 top 64
// 1,181, 627.
bool lists_taken(int64_t rows, int32_t classes, int32_t top) {
  if (top > 64) return false;
  int slots = 4;
  while (slots < top) slots *= 2;
  const double walk = std::max(0.04 + 0.0085 * slots, (double)rows * (0.8 + 0.105 * slots) * 1e-6);
  return 3.5 + classes * walk < 5.0 + (double)rows * (top <= 16 ? 0.8e-3 : 1.5e-3);
}

template <class T, int kThreads, int kVecs>
int unit_go(const TopArgs &all, hipStream_t s) {
  constexpr int kUnits = kThreads < 256 ? 256 / kThreads : 1, kBlock = kThreads < 256 ? 256 : kThreads;
  const int64_t most = kMaxLaunch / kBlock * kUnits / all.parts;
  for (int64_t row0 = 0; row0 < all.rows; row0 += most) {
    TopArgs a = all;
    a.rows = std::min(most, all.rows - row0);
    a.Z = (const typename T::type *)all.Z + row0 * all.ld;
    a.values += row0 * all.parts * all.ld_top;
    a.ids += row0 * all.parts * all.ld_top;
    if (a.tail) a.tail += row0;
    if (a.part_tail) a.part_tail += row0 * all.parts;
    if (a.listed_ids) a.listed_ids += row0 * all.ld;
    if (a.listed_tails) a.listed_tails += row0 * all.tails;
    const int64_t units = a.rows * a.parts;
    hipLaunchKernelGGL((top_unit_kernel<T, kThreads, kVecs>), dim3((unsigned)((units + kUnits - 1) / kUnits)), dim3(kBlock), 0, s, a);
    PGCN_HIP(hipGetLastError());
  }
  return PGCN_OK;
}

// More lane maxima than slots keep the threshold tight; more threads than that are more to bring together.
// A workgroup and a wave to a row of up to 256 vectors, us of 20,000 rows, fp32 and bf16: 500 classes
// top 65 99 and 47, 150 and 47; 1,000 top 100 114 and 74, 135 and 69; 250 top 128 141 and 57, 152 and 61.
// Lists of parts are joined by a workgroup, which is faster for one row of many entries and slower from some
// hundred rows on, workgroup and wave: 1 x 100,003 top 50 7.7 and 9.6, top 8 5.8 and 5.6; 16 rows top 50 9.6 and
// 10.2; 2,048 x 65,536 top 64 17 and 11, top 8 9.2 and 5.9, beside a first launch of 100 to 150 us.
template <class T>
int units(const TopArgs &a, hipStream_t s) {
  const int vecs = (std::min(a.range, a.classes) + T::E - 1) / T::E;
  if (a.top <= 128 && vecs <= 256 && !a.listed_ids) {
    if (vecs <= 64) return unit_go<T, 64, 1>(a, s);
    if (vecs <= 128) return unit_go<T, 64, 2>(a, s);
    return unit_go<T, 64, 4>(a, s);
  }
  if (vecs <= 1024 || (a.top <= 64 && vecs <= 2048)) {
    if (vecs <= 256) return unit_go<T, 256, 1>(a, s);
    if (vecs <= 512) return unit_go<T, 256, 2>(a, s);
    if (vecs <= 1024) return unit_go<T, 256, 4>(a, s);
    return unit_go<T, 256, 8>(a, s);
  }
  if (vecs <= 2048) return unit_go<T, 512, 4>(a, s);
  return unit_go<T, 512, 8>(a, s);
}

template <class T, int kSlots>
int lists_go(const pgcn_top_logits_args &a, hipStream_t s) {
  hipLaunchKernelGGL((top_lists_kernel<T, kSlots>), dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, a);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

// Workspace of a row in parts: their values, ids and log-sums.
struct PartLists {
  size_t ids, tails, bytes;
};
PartLists part_lists(int64_t rows, int parts, int32_t top) {
  PartLists p;
  p.ids = align_up((size_t)rows * parts * top * 4, 16);
  p.tails = 2 * p.ids;
  p.bytes = p.tails + (size_t)rows * parts * sizeof(float2);
  return p;
}

template <class T>
int top_go(const pgcn_top_logits_args &a, hipStream_t s) {
  if (lists_taken(a.rows, a.classes, a.top)) {
    if (a.top <= 4) return lists_go<T, 4>(a, s);
    if (a.top <= 8) return lists_go<T, 8>(a, s);
    if (a.top <= 16) return lists_go<T, 16>(a, s);
    if (a.top <= 32) return lists_go<T, 32>(a, s);
    return lists_go<T, 64>(a, s);
  }
  const int parts = top_parts(a.dtype, a.classes);
  TopArgs t{};
  t.Z = a.Z;
  t.rows = a.rows;
  t.ld = a.ld;
  t.classes = a.classes;
  t.top = t.fill = a.top;
  t.range = parts > 1 ? kPartVecs * T::E : a.classes;
  t.parts = parts;
  t.inv_t = 1.0f / a.temperature;
  t.values = a.top_values;
  t.ids = a.top_ids;
  t.ld_top = a.ld_top;
  t.tail = a.tail_lse;
  if (parts == 1) return units<T>(t, s);
  const int wide = (a.top + 3) / 4 * 4;            // lists of whole vectors
  const PartLists p = part_lists(a.rows, parts, wide);
  char *ws = (char *)a.workspace;
  t.values = (float *)ws;
  t.ids = (int32_t *)(ws + p.ids);
  t.ld_top = t.fill = wide;
  t.tail = nullptr;
  t.part_tail = a.tail_lse ? (float2 *)(ws + p.tails) : nullptr;
  const int rc = units<T>(t, s);
  if (rc) return rc;
  // The lists of a row's parts, one after another, are a row themselves: equal values stand in the
  // order of their classes in it.
  TopArgs u = t;
  u.Z = t.values;
  u.ld = u.classes = u.range = parts * wide;
  u.fill = a.top;
  u.parts = 1;
  u.values = a.top_values;
  u.ids = a.top_ids;
  u.ld_top = a.ld_top;
  u.tail = a.tail_lse;
  u.part_tail = nullptr;
  u.listed_ids = t.ids;
  u.listed_tails = t.part_tail;
  u.tails = a.tail_lse ? parts : 0;
  return units<F32>(u, s);
}

}  // namespace

size_t top_logits_workspace(int32_t dtype, int64_t rows, int32_t classes, int32_t top) {
  if (lists_taken(rows, classes, top)) return 0;
  const int parts = top_parts(dtype, classes);
  return parts > 1 ? part_lists(rows, parts, (top + 3) / 4 * 4).bytes : 0;
}

int launch_top_logits(const pgcn_top_logits_args &a, hipStream_t s) {
  if (a.rows == 0) return PGCN_OK;
  TraceScope ts(PGCN_TK_TOP_LOGITS, s);
  return a.dtype == PGCN_BF16 ? top_go<BF16>(a, s) : top_go<F32>(a, s);
}

}  // namespace pgcn
