// The largest logits of every row with their classes, and the log-sum of the others.
//
// Order: (value, lower class first) with -0 equal to +0; -inf and NaN are never listed.  Bound by
// one read of Z.  Three kernels:
//   - many short rows: a thread walks a row and keeps its list in registers (top_lists_kernel);
//   - longer rows: a wave or a workgroup holds a row in registers.  The list lies above a
//     threshold that at least `top` elements reach: each wave's r-th largest lane maximum, r =
//     top / waves, has r elements of that wave at or above it.  What reaches the smallest of
//     them, little more than `top` elements, goes to LDS, where each is ranked by counting.
//     Where too many reach it (ties, sorted rows) the threshold is bisected, and among equal
//     values the class;
//   - few rows, and rows longer than that: parts of a row first, then the lists of its parts.
#include <algorithm>
#include <cfloat>

#include "ops.h"

namespace pgcn {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp_at(float x, float m, float scale) { return __builtin_amdgcn_exp2f((x - m) * scale); }

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

constexpr int kCandidates = 512;

// Elements of a row's registers: f(x, class) for each.
template <class T, int kThreads, int kVecs, class F>
__device__ __forceinline__ void each(typename T::raw (&raw)[kVecs], int lane, F f) {
  keep_packed(raw);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    float x[T::E];
    T::unpack(raw[i], x);
    const int c0 = (lane + kThreads * i) * T::E;
#pragma unroll
    for (int e = 0; e < T::E; ++e) f(x[e], c0 + e);
    __builtin_amdgcn_sched_barrier(0);             // one vector at a time: their temporaries do not add up
  }
}

template <int kThreads>
struct TopLds {
  static constexpr int kWaves = kThreads / 64;
  uint64_t list[kCandidates];
  float wave_f[2][kWaves];
  int wave_n[2][kWaves];
  int count;
  uint64_t last, next;         // keys of rank top - 1 and top
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

// The r-th largest of a wave's 64 values (r <= 64).
__device__ __forceinline__ float nth_of_wave(float v, int r) {
  const int lane = threadIdx.x % 64;
  if (r <= 8) {
    float m = v;
    for (int i = 0;; ++i) {
      m = lanes_max<64>(v);
      if (i == r - 1) return m;
      const int first = __ffsll((unsigned long long)__ballot(v == m)) - 1;
      if (lane == first) v = kNegInf;
    }
  }
  int rank = 0;
#pragma unroll 8
  for (int j = 0; j < 64; ++j) {
    const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), j));
    rank += o > v || (o == v && j < lane) ? 1 : 0;
  }
  const int at = __ffsll((unsigned long long)__ballot(rank == r - 1)) - 1;
  return __shfl(v, at, 64);
}

template <class T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads < 256 ? 256 : kThreads) void top_unit_kernel(TopArgs a) {
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
  float top = kNegInf;                             // a NaN is no maximum
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
    for (int e = 0; e < T::E; ++e) top = fmaxf(top, x[e]);
    __builtin_amdgcn_sched_barrier(0);
  }

  int turn = 0;
  const int r = (K + kWaves - 1) / kWaves;
  float v = r <= 64 ? nth_of_wave(top, r) : kNegInf;
  v = waves_all<kThreads>(v, l, turn, [](float x, float y) { return fminf(x, y); });
  v = fmaxf(v, -FLT_MAX);                          // x >= v: every x above -inf
  auto count = [&](auto in) {
    int n = 0;
    each<T, kThreads>(raw, lane, [&](float x, int c) { n += __popcll(__ballot(in(x, c))); });
    return waves_add<kThreads>(n, l, turn);
  };
  int n = count([&](float x, int) { return x >= v; });
  float tie = v;                                   // in the list: x > tie, or x == tie and its class is at most `upto`
  int upto = n_all;
  if (n > kCandidates) {
    float m = waves_all<kThreads>(lanes_max<64>(top), l, turn, [](float x, float y) { return fmaxf(x, y); });
    uint32_t lo = order_of(v), hi = order_of(m) + 1;
    int above = 0;                                 // elements from `hi` on
    while (n > kCandidates && hi - lo > 1) {
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
    tie = value_of(lo);
    if (n > kCandidates) {                         // all of them equal but for `above` < K: the lowest classes
      int from = -1, to = n_all - 1;
      while (to - from > 1) {
        const int mid = (from + to) / 2;
        if (above + count([&](float x, int c) { return x == tie && c <= mid; }) >= K) to = mid;
        else from = mid;
      }
      upto = to;
      n = K;
    }
  }

  if (lane == 0) l.count = 0;
  unit_sync<kThreads>();
  each<T, kThreads>(raw, lane, [&](float x, int c) {
    if (x > tie || (x == tie && c <= upto)) {
      const int at = atomicAdd(&l.count, 1);       // any order: what follows goes by rank
      l.list[at] = ((uint64_t)order_of(x) << 32) | (uint32_t)~c;
    }
  });
  unit_sync<kThreads>();
  float *values = a.values + unit * a.ld_top;
  int32_t *ids = a.ids + unit * a.ld_top;
  for (int j = lane; j < n; j += kThreads) {
    const uint64_t key = l.list[j];
    int rank = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) rank += l.list[i] > key ? 1 : 0;
    if (rank < K) {
      const int c = (int)~(uint32_t)key;
      values[rank] = value_of((uint32_t)(key >> 32));
      ids[rank] = a.listed_ids ? a.listed_ids[row * a.ld + c] : first + c;
    }
    if (rank == K - 1) l.last = key;
    if (rank == K) l.next = key;
  }
  for (int k = (n < K ? n : K) + lane; k < a.fill; k += kThreads) {
    values[k] = kNegInf;
    ids[k] = -1;
  }
  if (!a.tail && !a.part_tail) return;

  unit_sync<kThreads>();
  const float scale = a.inv_t * kLog2e;
  float last = -FLT_MAX;                           // all above -inf are listed
  int last_c = n_all;
  if (n >= K) {
    last = value_of((uint32_t)(l.last >> 32));
    last_c = (int)~(uint32_t)l.last;
  }
  auto other = [&](float x, int c) { return !(x > last || (x == last && c <= last_c)); };
  float m;
  if (n > K) {
    m = value_of((uint32_t)(l.next >> 32));
  } else {
    m = kNegInf;
    each<T, kThreads>(raw, lane, [&](float x, int c) { m = fmaxf(m, other(x, c) ? x : kNegInf); });
    m = waves_all<kThreads>(lanes_max<64>(m), l, turn, [](float x, float y) { return fmaxf(x, y); });
  }
  const float base = m == kNegInf ? 0.f : m;
  float s = 0.f;
  each<T, kThreads>(raw, lane, [&](float x, int c) { s += exp_at(other(x, c) ? x : kNegInf, base, scale); });
  s = waves_all<kThreads>(lanes_sum<64>(s), l, turn, [](float x, float y) { return x + y; });
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
// An element is one fp64 number: its value, with the class in the lowest of the 29 bits that a
// float leaves free, so that of equal values the lower class is larger.  The list is kept sorted by
// one maximum and one minimum a slot; what falls out at its end is no part of it any more and goes
// into the log-sum.  A wave's rows pass through LDS in tiles of kTile classes.

constexpr int kTile = 32;
constexpr uint32_t kClassMask = PGCN_MAX_CLASSES - 1;

__device__ __forceinline__ double list_key(float x, int c) {
  if (!(x > kNegInf)) return -__builtin_inf();
  const double d = x > FLT_MAX ? 0x1p200 : (double)(x + 0.f);         // infinity, in numbers
  const uint64_t b = __builtin_bit_cast(uint64_t, d);
  return __builtin_bit_cast(double, b | ((b >> 63) ? (uint32_t)c : kClassMask - (uint32_t)c));
}

__device__ __forceinline__ int key_class(double k) {
  const uint64_t b = __builtin_bit_cast(uint64_t, k);
  return (b >> 63) ? (int)((uint32_t)b & kClassMask) : (int)(kClassMask - ((uint32_t)b & kClassMask));
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
  double list[kSlots];
#pragma unroll
  for (int k = 0; k < kSlots; ++k) list[k] = -__builtin_inf();
  float m = kNegInf, s = 0.f;
  bool nan = false;
  auto left_out = [&](float x) {
    const float e = __builtin_amdgcn_exp2f(-fabsf(x - m) * scale);
    nan |= x > FLT_MAX;                            // an infinity that is not listed
    if (x > kNegInf) {
      s = x > m ? s * e + 1.0f : s + e;
      m = fmaxf(m, x);
    }
  };
  load(0);
  for (int c0 = 0; c0 < C; c0 += kTile) {
    wave_sync();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float x[T::E];
      T::unpack(raw[i], x);
#pragma unroll
      for (int e = 0; e < T::E; ++e) tile[(ty + kDown * i) * (kTile + 1) + tx * T::E + e] = x[e];
    }
    wave_sync();
    if (c0 + kTile < C) load(c0 + kTile);
    const int n = C - c0 < kTile ? C - c0 : kTile;
    for (int c = 0; c < n; ++c) {
      const float x = tile[lane * (kTile + 1) + c];
      nan |= x != x;
      double k = list_key(x, c0 + c);
#pragma unroll
      for (int i = 0; i < kSlots; ++i) {
        const double hi = __builtin_fmax(list[i], k);
        k = __builtin_fmin(list[i], k);
        list[i] = hi;
      }
      left_out((float)k);
    }
  }
  const int64_t r = row0 + lane;
  if (r >= a.rows) return;
#pragma unroll
  for (int k = 0; k < kSlots; ++k) {
    const bool some = list[k] > -__builtin_inf();
    if (k < K) {
      a.top_values[r * a.ld_top + k] = some ? (float)list[k] : kNegInf;
      a.top_ids[r * a.ld_top + k] = some ? key_class(list[k]) : -1;
    } else if (some) {
      left_out((float)list[k]);
    }
  }
  if (a.tail_lse) a.tail_lse[r] = nan ? __builtin_nanf("") : s == 0.f ? kNegInf : m / a.temperature + __logf(s);
}

// ---- launches -------------------------------------------------------------------------------

int vector_elems(int32_t dtype) { return dtype == PGCN_BF16 ? BF16::E : F32::E; }

constexpr int kPartThreads = 256, kPartVecs = 4, kLongVecs = 8192;

// Parts of a row, 1: the whole of it at once.
int top_parts(int32_t dtype, int64_t rows, int32_t classes) {
  const int64_t range = (int64_t)kPartThreads * kPartVecs * vector_elems(dtype), parts = (classes + range - 1) / range;
  return parts > kLongVecs / (kPartThreads * kPartVecs) || (rows <= 128 && parts >= 4) ? (int)parts : 1;
}

// Whether a thread takes a row.
bool lists_taken(int64_t rows, int32_t classes, int32_t top) {
  if (top > 64) return false;
  int slots = 4;
  while (slots < top) slots *= 2;
  const int64_t walk = (int64_t)classes * (2 * slots + 12);            // instructions of a wave
  return walk <= 2048 || (rows >= 32768 && walk / 64 <= 500);
}

template <class T, int kThreads, int kVecs>
int unit_go(const TopArgs &a, hipStream_t s) {
  constexpr int kUnits = kThreads < 256 ? 256 / kThreads : 1;
  const int64_t units = a.rows * a.parts;
  hipLaunchKernelGGL((top_unit_kernel<T, kThreads, kVecs>), dim3((unsigned)((units + kUnits - 1) / kUnits)),
                     dim3(kThreads < 256 ? 256 : kThreads), 0, s, a);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

template <class T>
int units(const TopArgs &a, hipStream_t s) {
  const int vecs = (std::min(a.range, a.classes) + T::E - 1) / T::E;
  if (vecs <= 64) return unit_go<T, 64, 1>(a, s);
  if (vecs <= 128) return unit_go<T, 64, 2>(a, s);
  if (vecs <= 256) return unit_go<T, 64, 4>(a, s);
  if (vecs <= 512) return unit_go<T, 64, 8>(a, s);
  if (vecs <= 1024) return unit_go<T, 256, 4>(a, s);
  if (vecs <= 2048) return unit_go<T, 256, 8>(a, s);
  if (vecs <= 4096) return unit_go<T, 512, 8>(a, s);
  return unit_go<T, 1024, 8>(a, s);
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
  const int parts = top_parts(a.dtype, a.rows, a.classes);
  TopArgs t{};
  t.Z = a.Z;
  t.rows = a.rows;
  t.ld = a.ld;
  t.classes = a.classes;
  t.top = t.fill = a.top;
  t.range = parts > 1 ? kPartThreads * kPartVecs * T::E : a.classes;
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
  const int parts = top_parts(dtype, rows, classes);
  return parts > 1 ? part_lists(rows, parts, (top + 3) / 4 * 4).bytes : 0;
}

int launch_top_logits(const pgcn_top_logits_args &a, hipStream_t s) {
  if (a.rows == 0) return PGCN_OK;
  TraceScope ts(PGCN_TK_TOP_LOGITS, s);
  return a.dtype == PGCN_BF16 ? top_go<BF16>(a, s) : top_go<F32>(a, s);
}

}  // namespace pgcn
