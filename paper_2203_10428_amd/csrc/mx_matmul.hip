// Product of two matrices of FP4 rows, C = a b^T, on the scaled matrix instructions.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes from each lane a block of 32 elements with its scale: row lane % 32 and
// one of two blocks, lane / 32.  Which two blocks of a row go together is free as long as both operands agree, so
// in a slab of eight blocks (256 elements, 128 bytes a row) lane half h takes block 4 h + t in step t: its four
// scales are one dword, of which the instruction picks byte t.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "mx.h"

namespace pgcn {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t dwords __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatmulArgs {
  const uint8_t *A, *SA, *B, *SB;
  void *C;
  float *parts;           // [splits, m, n4] sums over a part of the blocks each, or null: C is written
  int64_t m, ld_a, ld_sa, ld_b, ld_sb, ld_c, n4;
  int32_t n, blocks, relu, tiles_m, tiles_n;
  int32_t span;           // blocks of one part, a multiple of 8
};

__device__ __forceinline__ i32x8 wide(const op_u32x4 &q) { return i32x8{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0}; }

// 16 bytes or one dword a lane from memory to LDS, place + lane size, without a register between.  Written out, so that
// the compiler does not wait for it before every LDS read: landed() does, once a slab.  No register is written.
template <int kBytes>
__device__ __forceinline__ void to_lds(const void *src, uint32_t place) {
  if constexpr (kBytes == 16)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(place) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(place) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_place(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// Waits until at most n of the wave's loads are under way and its LDS reads are done, then for the workgroup's other waves.
template <int n>
__device__ __forceinline__ void landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | ((n >> 4) << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Four neighbouring results of a row, col a multiple of 4.
template <class T>
__device__ __forceinline__ void finish4(const MatmulArgs &p, int64_t row, int col, op_f32x4 v) {
  typename T::type *out = (typename T::type *)p.C + row * p.ld_c + col;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = p.relu && v[e] < 0.f ? 0.f : v[e];
  if (col + 4 <= p.n) {
    if constexpr (sizeof(typename T::type) == 4) *reinterpret_cast<op_f32x4 *>(out) = v;
    else *reinterpret_cast<op_u32x2 *>(out) = op_u32x2{BF16::two(v[0], v[1]), BF16::two(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < p.n) T::put(out + e, v[e]);
  }
}

// One stage of LDS: a slab's eight blocks of every row, block c at place c ^ (row % 8), so that neighbouring lanes' reads
// of one block touch all banks.
template <int BM, int BN>
struct Stage {
  uint8_t a[BM * 128], b[BN * 128];
};

// BM x BN results to a workgroup of four waves, two by two, in slabs of eight blocks, four steps of two; NS stages.
// 8192 x 8192 x 8192 with bf16 results: 265 us, 4.1 PFLOP/s.  Its matrix instructions alone take 151 us, its loads alone
// 160, of which the scales 23 (16 bytes of a row at a time); without the results' stores 229.  Loads and LDS reads issued
// in one piece instead of between the products: 343; results stored from the accumulators, 16 bytes of a row at a time: 302.
template <class T, int BM, int BN, int NS>
__global__ __launch_bounds__(256) void matmul_tile(MatmulArgs p) {
  constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
  constexpr int kLoadsA = BM / 32, kLoads = (BM + BN) / 32, kScaleLoads = BM / 64, kSlabLoads = kLoads + kScaleLoads;     // of a wave
  typedef Stage<BM, BN> St;
  static_assert(BM == BN && (NS & (NS - 1)) == 0, "halves of the scales are alike; stages in turn");
  __shared__ __attribute__((aligned(1024))) St stages[NS];
  __shared__ __attribute__((aligned(1024))) uint32_t scales[NS][(BM + BN) * 4];         // of two slabs each: four dwords a row
  const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64);

  // tiles of one XCD (workgroups 8 apart) are neighbours: bands of eight tile rows, column by column
  const uint32_t total = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n, part = BM == 64 ? blockIdx.x / total : 0u, g = blockIdx.x - part * total;
  const uint32_t l = total % 8 == 0 ? (g % 8) * (total / 8) + g / 8 : g;
  const uint32_t band = l / (8u * p.tiles_n), in_band = l - band * 8u * p.tiles_n;
  const uint32_t band_rows = min(8u, (uint32_t)p.tiles_m - 8u * band);
  const int64_t i0 = (int64_t)(8u * band + in_band % band_rows) * BM;
  const int j0 = (int)(in_band / band_rows) * BN;
  const int begin = (int)part * p.span, slabs = (min(p.span, p.blocks - begin) + 7) / 8;

  // what this lane brings of a slab: rows past the matrix repeat its last one, blocks past the row its last one
  const int pos = begin + (lane % 8 ^ lane / 8);          // loads are 8 rows apart
  const uint8_t *src[kLoads], *src_sa[kScaleLoads], *src_sb[kScaleLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = 8 * (wave * kLoadsA + i % kLoadsA) + lane / 8;
    src[i] = i < kLoadsA ? p.A + min(p.m - 1, i0 + row) * p.ld_a : p.B + min((int64_t)p.n - 1, (int64_t)j0 + row) * p.ld_b;
  }
#pragma unroll
  for (int i = 0; i < kScaleLoads; ++i) {                 // 16 rows' four dwords
    const int64_t row = 16 * (wave * kScaleLoads + i) + lane / 4;
    src_sa[i] = p.SA + min(p.m - 1, i0 + row) * p.ld_sa;
    src_sb[i] = p.SB + min((int64_t)p.n - 1, j0 + row) * p.ld_sb;
  }
  const int last_dword = (p.blocks - 1) / 4;
  const uint32_t place = lds_place(stages), place_s = lds_place(scales);
  int64_t off = 0;
  auto bring = [&](int i, uint32_t stage) __attribute__((always_inline)) {
    const uint32_t in = (uint32_t)(i < kLoadsA ? offsetof(St, a) : offsetof(St, b)) + (uint32_t)(wave * kLoadsA + i % kLoadsA) * 1024u;
    to_lds<16>(src[i] + off, place + (stage & (NS - 1)) * (uint32_t)sizeof(St) + in);
  };
  auto at_slab = [&](int slab) __attribute__((always_inline)) { off = 16 * (int64_t)min(8 * slab + pos, p.blocks - 1); };
  // of 2 pair, 2 pair + 1: the scales of A's rows or of B's
  auto bring_scales = [&](int i, int pair, int of_b) __attribute__((always_inline)) {
    const int64_t d = 4 * (int64_t)min(begin / 4 + 4 * pair + lane % 4, last_dword);
    const uint8_t *sa = src_sa[i], *sb = src_sb[i];
    to_lds<4>((of_b ? sb : sa) + d,
              place_s + (uint32_t)((pair & (NS - 1)) * (int)sizeof(scales[0]) + (of_b * (BM / 16) + wave * kScaleLoads + i) * 256));
  };
  // with an even slab those of B for it and the next, with an odd one those of A for the next two
  auto scales_with = [&](int i, int slab) __attribute__((always_inline)) { bring_scales(i, (slab + 1) / 2, slab % 2 == 0); };

  f32x16 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = (f32x16){};
  // lane half h takes blocks 4 h + k of a slab in step k: byte k of scale dword h
  const int h = lane / 32, r = lane % 32, wm0 = (wave / 2) * WM, wn0 = (wave % 2) * WN;
  struct Operands {
    op_u32x4 a[TM], b[TN];
  };
  struct Scales {
    uint32_t a[TM], b[TN];
  };
  auto read = [&](Operands &o, int q, int slab, int k) __attribute__((always_inline)) {
    const St &S = stages[slab & (NS - 1)];
    const int at = 16 * ((4 * h + k) ^ (r % 8));
    if (q < TN) o.b[q] = *reinterpret_cast<const op_u32x4 *>(S.b + (wn0 + 32 * q + r) * 128 + at);
    else o.a[q - TN] = *reinterpret_cast<const op_u32x4 *>(S.a + (wm0 + 32 * (q - TN) + r) * 128 + at);
  };
  auto read_scale = [&](Scales &o, int q, int slab) __attribute__((always_inline)) {
    const uint32_t *S = scales[slab / 2 & (NS - 1)] + 2 * (slab % 2) + h;
    if (q < TN) o.b[q] = S[4 * (BM + wn0 + 32 * q + r)];
    else o.a[q - TN] = S[4 * (wm0 + 32 * (q - TN) + r)];
  };
  auto keep_scales = [&](Scales &o, int slab) __attribute__((always_inline)) {
    // blocks past the row's last one count with the smallest scale on both sides: below any float
    const int some = p.blocks - begin - 8 * slab - 4 * h;
    const uint32_t keep = some >= 4 ? 0xffffffffu : some <= 0 ? 0u : (1u << (8 * some)) - 1u;
#pragma unroll
    for (int i = 0; i < TM; ++i) o.a[i] &= keep;
#pragma unroll
    for (int j = 0; j < TN; ++j) o.b[j] &= keep;
  };
  // One step's products, B's rows as the instruction's rows: a lane then holds four neighbouring columns of one row of
  // C.  While the matrix cores work, the wave issues what `between` has for the place behind each product.
  auto multiply = [&](const Operands &o, const Scales &c, auto which, auto between) __attribute__((always_inline)) {
    constexpr int k = decltype(which)::value;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        acc[j][i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(o.b[j]), wide(o.a[i]), acc[j][i], 4, 4, k, (int)c.b[j], k, (int)c.a[i]);
        __builtin_amdgcn_sched_barrier(0);
        between(j * TM + i);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  constexpr int kProducts = TM * TN;
  // the places q of n things that go behind product number m
  auto spread = [&](int m, int n, auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < n; ++q)
      if (q * kProducts / n == m) f(q);
  };
  typedef std::integral_constant<int, 0> Step0;
  typedef std::integral_constant<int, 1> Step1;
  typedef std::integral_constant<int, 2> Step2;
  typedef std::integral_constant<int, 3> Step3;

#pragma unroll
  for (int i = 0; i < kScaleLoads; ++i) bring_scales(i, 0, 0);
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (i < slabs) {
      at_slab(i);
#pragma unroll
      for (int q = 0; q < (i < NS - 1 ? kLoads : kLoadsA); ++q) bring(q, i);
#pragma unroll
      for (int q = 0; q < (i < NS - 1 ? kScaleLoads : 0); ++q) scales_with(q, i);
    }
  if (slabs >= NS) landed<kLoadsA + (NS - 2) * kSlabLoads>();
  else landed<0>();
  Operands x, y;
  Scales c, d;
#pragma unroll
  for (int q = 0; q < TM + TN; ++q) {
    read_scale(c, q, 0);
    read(x, q, 0, 0);
  }
  keep_scales(c, 0);

  // A step's operands are read behind the products of the step before.  Before a slab's last step its stage is read
  // out in every wave and the next slab has landed; behind that step the next slab's first operands are read, and the
  // slab that takes the stage sets out, A's rows behind this step, B's and scales behind the next two.  No branch among them: the
  // compiler would move products past it.
  auto first_three = [&](int s, auto more) __attribute__((always_inline)) {
    multiply(x, c, Step0{}, [&](int m) __attribute__((always_inline)) {
      spread(m, TM + TN, [&](int q) __attribute__((always_inline)) { read(y, q, s, 1); });
      if constexpr (decltype(more)::value) spread(m, kLoads - kLoadsA, [&](int q) __attribute__((always_inline)) { bring(kLoadsA + q, s + NS - 1); });
    });
    multiply(y, c, Step1{}, [&](int m) __attribute__((always_inline)) {
      spread(m, TM + TN, [&](int q) __attribute__((always_inline)) { read(x, q, s, 2); });
      if constexpr (decltype(more)::value) spread(m, kScaleLoads, [&](int q) __attribute__((always_inline)) { scales_with(q, s + NS - 1); });
    });
    multiply(x, c, Step2{}, [&](int m) __attribute__((always_inline)) {
      spread(m, TM + TN, [&](int q) __attribute__((always_inline)) { read(y, q, s, 3); });
    });
  };
  auto last = [&](int s, auto more) __attribute__((always_inline)) {
    constexpr bool kMore = decltype(more)::value;
    landed<kMore ? (NS - 2) * kSlabLoads : 0>();
    if constexpr (kMore) at_slab(s + NS);
    multiply(y, c, Step3{}, [&](int m) __attribute__((always_inline)) {
      spread(m, TM + TN, [&](int q) __attribute__((always_inline)) { read(x, q, s + 1, 0); });
      spread(m, TM + TN, [&](int q) __attribute__((always_inline)) { read_scale(d, q, s + 1); });
      if constexpr (kMore) spread(m, kLoadsA, [&](int q) __attribute__((always_inline)) { bring(q, s + NS); });
    });
    keep_scales(d, s + 1);
    c = d;
  };
  int s = 0;
  if (slabs >= NS) {
    for (; s + NS < slabs; ++s) {
      first_three(s, std::true_type{});
      last(s, std::true_type{});
    }
    first_three(s, std::true_type{});
    last(s, std::false_type{});
    ++s;
  }
  for (; s + 1 < slabs; ++s) {
    first_three(s, std::false_type{});
    last(s, std::false_type{});
  }
  first_three(s, std::false_type{});
  multiply(y, c, Step3{}, [](int) {});

  // 32 rows of a wave at a time through LDS, so that whole lines are written
  __syncthreads();
  auto write = [&](auto type, typename decltype(type)::type *C, int64_t ld, int cols, bool relu) __attribute__((always_inline)) {
    typedef decltype(type) O;
    constexpr int kElem = sizeof(typename O::type), kRow = WN * kElem + 16, kChunks = WN * kElem / 16;
    static_assert(4 * 32 * kRow <= sizeof(stages), "fits the stages");
    uint8_t *buf = (uint8_t *)stages + wave * 32 * kRow;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = relu && acc[j][i][4 * q + e] < 0.f ? 0.f : acc[j][i][4 * q + e];
          uint8_t *to = buf + r * kRow + (32 * j + 8 * q + 4 * h) * kElem;
          if constexpr (kElem == 4) *reinterpret_cast<op_f32x4 *>(to) = op_f32x4{v[0], v[1], v[2], v[3]};
          else *reinterpret_cast<op_u32x2 *>(to) = op_u32x2{BF16::two(v[0], v[1]), BF16::two(v[2], v[3])};
        }
      wave_sync();                                        // lanes read what others wrote
#pragma unroll
      for (int pass = 0; pass < kChunks / 2; ++pass) {
        const int down = pass * (64 / kChunks) + lane / kChunks, col = j0 + wn0 + lane % kChunks * O::E;
        const int64_t row = i0 + wm0 + 32 * i + down;
        const op_u32x4 w = *reinterpret_cast<const op_u32x4 *>(buf + down * kRow + lane % kChunks * 16);
        if (row >= p.m || col >= cols) continue;
        typename O::type *to = C + row * ld + col;
        if (col + O::E <= cols) {
          *reinterpret_cast<op_u32x4 *>(to) = w;
        } else {
#pragma unroll
          for (int e = 0; e < O::E; ++e)
            if (col + e < cols) {
              if constexpr (kElem == 4) to[e] = __uint_as_float(w[e]);
              else to[e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
            }
        }
      }
      wave_sync();                                        // the next rows are written after these reads
    }
  };
  if (BM == 64 && p.parts) write(F32{}, p.parts + (int64_t)part * p.m * p.n4, p.n4, (int)p.n4, false);
  else write(T{}, (typename T::type *)p.C, p.ld_c, p.n, p.relu);
}

// Up to 16 rows: what counts is how fast B arrives.  v_mfma_scale_f32_16x16x128_f8f6f4: a lane holds a block of row
// lane % 16, one of four neighbouring ones, straight from memory.  A wave takes 16 blocks in turn, 256 bytes of each of
// its 16 rows, whose scales are one 16-byte load; the eight waves' sums are added in LDS, in order.
constexpr int kRowWaves = 8, kGroup = 16, kGroups = 2;
template <class T>
__global__ __launch_bounds__(64 * kRowWaves) void matmul_rows(MatmulArgs p) {
  __shared__ __attribute__((aligned(16))) float sums[kRowWaves][64][4];
  const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64), r = lane % 16, q = lane / 16;
  const uint32_t part = blockIdx.x / (uint32_t)p.tiles_n;
  const int j0 = 16 * (int)(blockIdx.x - part * (uint32_t)p.tiles_n);
  const int begin = (int)part * p.span, end = min(p.blocks, begin + p.span), last_dword = (p.blocks - 1) / 4;
  const int64_t row_a = min(p.m - 1, (int64_t)r), row_b = min(p.n - 1, j0 + r);
  const uint8_t *a = p.A + row_a * p.ld_a, *sa = p.SA + row_a * p.ld_sa, *b = p.B + row_b * p.ld_b, *sb = p.SB + row_b * p.ld_sb;
  struct Group {
    op_u32x4 a[4], b[4];
    dwords sa, sb;
  };
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int b0 = begin + kGroup * wave; b0 < end; b0 += kGroup * kRowWaves * kGroups) {
    Group x[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {                   // past the last group: the last one again, not counted
      const int at = min(b0 + u * kGroup * kRowWaves, (end - 1) / kGroup * kGroup);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t off = 16 * (int64_t)min(at + 4 * k + q, p.blocks - 1);
        x[u].b[k] = *reinterpret_cast<const op_u32x4 *>(b + off);
        x[u].a[k] = *reinterpret_cast<const op_u32x4 *>(a + off);
      }
      if (at / 4 + 3 <= last_dword) {
        x[u].sb = *reinterpret_cast<const dwords *>(sb + at);
        x[u].sa = *reinterpret_cast<const dwords *>(sa + at);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int d = 4 * min(at / 4 + k, last_dword);
          x[u].sb[k] = *reinterpret_cast<const uint32_t *>(sb + d);
          x[u].sa[k] = *reinterpret_cast<const uint32_t *>(sa + d);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kGroups; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) {                       // a block that is none counts with the smallest scales: below any float
        const bool in = b0 + u * kGroup * kRowWaves + 4 * k + q < end;
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(x[u].b[k]), wide(x[u].a[k]), acc, 4, 4, 0,
                                                               (int)(in ? x[u].sb[k] >> (8 * q) : 0u), 0, (int)(in ? x[u].sa[k] >> (8 * q) : 0u));
      }
  }
  *reinterpret_cast<f32x4 *>(sums[wave][lane]) = acc;
  __syncthreads();
  if (wave > 0 || r >= p.m) return;
  op_f32x4 v = *reinterpret_cast<const op_f32x4 *>(sums[0][lane]);
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) v += *reinterpret_cast<const op_f32x4 *>(sums[w][lane]);
  if (!p.parts) finish4<T>(p, r, j0 + 4 * q, v);
  else if (j0 + 4 * q < p.n) *reinterpret_cast<op_f32x4 *>(p.parts + (part * p.m + r) * p.n4 + j0 + 4 * q) = v;
}

// C from the parts' sums, added in order.
template <class T>
__global__ __launch_bounds__(256) void join(MatmulArgs p, int splits) {
  const int64_t at = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x), size = p.m * p.n4;
  if (at >= size) return;
  const int64_t row = at / p.n4;
  op_f32x4 v = *reinterpret_cast<const op_f32x4 *>(p.parts + at);
  for (int z = 1; z < splits; ++z) v += *reinterpret_cast<const op_f32x4 *>(p.parts + z * size + at);
  finish4<T>(p, row, (int)(at - row * p.n4), v);
}

struct Shape {
  int tile, splits, span;         // tile: 16 rows, or BM = BN
};

// Up to 16 rows on their own: 16 x 8192 x 8192 13 us, in 64 x 64 tiles 14 and 3 to join them.  Otherwise the largest tile
// of which there is one for every compute unit: it brings the fewest bytes to a product (8192 x 8192 x 8192: 268 us in
// tiles of 256; 3500 x 3000 x 4096, half as many of them as units: 37 in tiles of 128).  The count does not see tiles that
// are mostly filled up, where one side is short: 306,000 x 47 x 128 takes 88 us, 32 x 65,536 x 4096 39.  More stages than two help where a
// compute unit has one small tile (777 x 1000 x 5000: 11.4 us with four, 15.8 with two), not where others fill it
// (58,000 x 256 x 602 in tiles of 128: 21.6 with two, 31.7 with four).
// Where units are left without a tile, the blocks are split among as many workgroups as there are units (two a unit for
// few rows), at least four slabs or a group for every wave each (128 x 1000 x 8192: 5.9 us and 3.8 to join them, whole
// 13.5); no more, for joining costs 4 us.
Shape shape_of(int64_t m, int32_t n, int32_t k) {
  Shape c;
  const auto tiles = [&](int64_t b) { return ((m + b - 1) / b) * ((n + b - 1) / b); };
  c.tile = m <= 16 ? 16 : tiles(256) >= 256 ? 256 : tiles(128) >= 256 ? 128 : 64;
  const int64_t unit = c.tile == 16 ? kGroup : 8, units = (mx_blocks(k) + unit - 1) / unit;
  int64_t s = 1;
  if (c.tile == 16) s = std::min<int64_t>(512 / tiles(16), units / kRowWaves);
  if (c.tile == 64) s = std::min<int64_t>(256 / tiles(64), units / 4);
  s = std::max<int64_t>(1, std::min(s, ((int64_t)64 << 20) / (m * ((n + 3) / 4 * 4) * 4)));    // parts of 64 MB together
  const int64_t each = (units + s - 1) / s;
  c.span = (int)(unit * each);
  c.splits = (int)((units + each - 1) / each);
  return c;
}

template <class T>
void launch(MatmulArgs &a, const Shape &c, hipStream_t s) {
  const int bm = c.tile;
  a.tiles_m = (int)((a.m + bm - 1) / bm);
  a.tiles_n = (a.n + bm - 1) / bm;
  a.span = c.span;
  const dim3 grid((unsigned)((int64_t)a.tiles_m * a.tiles_n * c.splits)), block(256);
  if (bm == 16) hipLaunchKernelGGL((matmul_rows<T>), grid, dim3(64 * kRowWaves), 0, s, a);
  else if (bm == 256) hipLaunchKernelGGL((matmul_tile<T, 256, 256, 2>), grid, block, 0, s, a);
  else if (bm == 128) hipLaunchKernelGGL((matmul_tile<T, 128, 128, 2>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((matmul_tile<T, 64, 64, 4>), grid, block, 0, s, a);
  if (c.splits > 1)
    hipLaunchKernelGGL((join<T>), dim3((unsigned)((a.m * a.n4 / 4 + 255) / 256)), block, 0, s, a, c.splits);
}

}  // namespace

size_t mx_matmul_workspace(int32_t, int64_t m, int32_t n, int32_t k) {
  if (m == 0) return 0;
  const Shape c = shape_of(m, n, k);
  return c.splits > 1 ? (size_t)c.splits * (size_t)m * (size_t)((n + 3) / 4 * 4) * sizeof(float) : 0;
}

int launch_mx_matmul(const pgcn_mx_matmul_args &x, hipStream_t s) {
  const Shape c = shape_of(x.m, x.n, x.k);
  MatmulArgs a{};
  a.A = x.A, a.SA = x.A_scales, a.B = x.B, a.SB = x.B_scales, a.C = x.C;
  a.parts = c.splits > 1 ? (float *)x.workspace : nullptr;
  a.m = x.m, a.ld_a = x.ld_a, a.ld_sa = x.ld_a_scales, a.ld_b = x.ld_b, a.ld_sb = x.ld_b_scales, a.ld_c = x.ld_c;
  a.n = x.n, a.n4 = (x.n + 3) / 4 * 4, a.blocks = (int32_t)mx_blocks(x.k), a.relu = x.relu;
  TraceScope ts(PGCN_TK_MX_MATMUL, s);
  if (c.splits > 1) ts.set_launches(2);
  if (x.dtype == PGCN_BF16) launch<BF16>(a, c, s);
  else launch<F32>(a, c, s);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
