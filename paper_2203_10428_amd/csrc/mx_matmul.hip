// Product of two matrices of FP4 rows, C = a b^T, on the scaled matrix instructions.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes from each lane a block of 32 elements with its scale: row lane % 32 and
// one of two blocks, lane / 32.  Which two blocks of a row go together is free as long as both operands agree, so
// in a slab of eight blocks (256 elements, 128 bytes a row) lane half h takes block 4 h + t in step t: its four
// scales are one dword, of which the instruction picks byte t.
#include <algorithm>

#include "mx.h"

namespace pgcn {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatmulArgs {
  const uint8_t *A, *SA, *B, *SB;
  void *C;
  int64_t m, ld_a, ld_sa, ld_b, ld_sb, ld_c;
  int32_t n, blocks, relu, tiles_m, tiles_n;
};

__device__ __forceinline__ i32x8 wide(const op_u32x4 &q) { return i32x8{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0}; }

// 16 bytes or one dword a lane from memory to LDS, base + lane size, without a register between.
template <int kBytes>
__device__ __forceinline__ void to_lds(const void *src, void *dst) {
  typedef const __attribute__((address_space(1))) void *from;
  typedef __attribute__((address_space(3))) void *to;
  if constexpr (kBytes == 16) __builtin_amdgcn_global_load_lds((from)src, (to)dst, 16, 0, 0);
  else __builtin_amdgcn_global_load_lds((from)src, (to)dst, 4, 0, 0);
}

// Waits until at most n of the wave's loads are under way, then for the workgroup's other waves.
template <int n>
__device__ __forceinline__ void landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

constexpr int kSlabBytes = 128, kSlabBlocks = 8;

// One stage of LDS: rows of 128 bytes, whose 16-byte block c is kept at place c ^ (row % 8), so that neighbouring
// lanes' reads of one block touch all banks; a slab's two scale dwords of every row apart.
template <int BM, int BN>
struct Stage {
  uint8_t a[BM * kSlabBytes], b[BN * kSlabBytes];
  uint32_t sa[2][BM], sb[2][BN];
};

// BM x BN results to a workgroup of four waves, two by two.
template <class T, int BM, int BN>
__global__ __launch_bounds__(256) void matmul_tile(MatmulArgs p) {
  constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
  constexpr int kLoadsA = BM / 32, kLoadsB = BN / 32, kScaleLoads = (BM + BN) / 128, kLoads = kLoadsA + kLoadsB + kScaleLoads;
  __shared__ __attribute__((aligned(1024))) Stage<BM, BN> S0, S1;
  const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64);

  // tiles of one XCD (workgroups 8 apart) are neighbours: bands of eight tile rows, column by column
  const uint32_t total = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n, g = blockIdx.x;
  const uint32_t l = total % 8 == 0 ? (g % 8) * (total / 8) + g / 8 : g;
  const uint32_t band = l / (8u * p.tiles_n), in_band = l - band * 8u * p.tiles_n;
  const uint32_t band_rows = min(8u, (uint32_t)p.tiles_m - 8u * band);
  const int64_t i0 = (int64_t)(8u * band + in_band % band_rows) * BM;
  const int j0 = (int)(in_band / band_rows) * BN;

  // what this lane brings of a slab: rows past the matrix repeat its last one, blocks past the row its last one
  const int pos = (lane % 8) ^ (lane / 8);
  const uint8_t *src_a[kLoadsA], *src_b[kLoadsB], *src_s[kScaleLoads];
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) src_a[i] = p.A + min(p.m - 1, i0 + 8 * (wave * kLoadsA + i) + lane / 8) * p.ld_a;
#pragma unroll
  for (int i = 0; i < kLoadsB; ++i) src_b[i] = p.B + min((int64_t)p.n - 1, (int64_t)j0 + 8 * (wave * kLoadsB + i) + lane / 8) * p.ld_b;
#pragma unroll
  for (int i = 0; i < kScaleLoads; ++i) {
    const int part = 4 * i + wave;                        // 64 rows' dwords: A's first, A's second, B's
    const bool of_a = part < BM / 32;
    const int q = of_a ? part : part - BM / 32, rows = (of_a ? BM : BN) / 64;
    const int64_t row = (of_a ? i0 : (int64_t)j0) + 64 * (q % rows) + lane;
    src_s[i] = of_a ? p.SA + min(p.m - 1, row) * p.ld_sa : p.SB + min((int64_t)p.n - 1, row) * p.ld_sb;
  }
  const int last_dword = (p.blocks - 1) / 4;
  auto bring = [&](Stage<BM, BN> &S, int slab) __attribute__((always_inline)) {
    const int64_t off = 16 * (int64_t)min(kSlabBlocks * slab + pos, p.blocks - 1);
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) to_lds<16>(src_a[i] + off, S.a + (wave * kLoadsA + i) * 1024);
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i) to_lds<16>(src_b[i] + off, S.b + (wave * kLoadsB + i) * 1024);
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
      const int part = 4 * i + wave;
      const bool of_a = part < BM / 32;
      const int q = of_a ? part : part - BM / 32, rows = (of_a ? BM : BN) / 64;
      const int d = q / rows;
      to_lds<4>(src_s[i] + 4 * (int64_t)min(2 * slab + d, last_dword), (of_a ? S.sa[d] : S.sb[d]) + 64 * (q % rows));
    }
  };

  f32x16 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = (f32x16){};
  const int h = lane / 32, r = lane % 32, wm0 = (wave / 2) * WM, wn0 = (wave % 2) * WN;
  auto compute = [&](Stage<BM, BN> &S, int slab) __attribute__((always_inline)) {
    // blocks past the row's last one count with the smallest scale on both sides: below any float
    const int some = p.blocks - kSlabBlocks * slab - 4 * h;
    const uint32_t keep = some >= 4 ? 0xffffffffu : some <= 0 ? 0u : (1u << (8 * some)) - 1u;
    uint32_t sa[TM], sb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = S.sa[h][wm0 + 32 * i + r] & keep;
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = S.sb[h][wn0 + 32 * j + r] & keep;
    struct Operands {
      op_u32x4 a[TM], b[TN];
    };
    auto read = [&](Operands &o, int k) __attribute__((always_inline)) {
      const int at = 16 * ((4 * h + k) ^ (r % 8));
#pragma unroll
      for (int i = 0; i < TM; ++i) o.a[i] = *reinterpret_cast<const op_u32x4 *>(S.a + (wm0 + 32 * i + r) * kSlabBytes + at);
#pragma unroll
      for (int j = 0; j < TN; ++j) o.b[j] = *reinterpret_cast<const op_u32x4 *>(S.b + (wn0 + 32 * j + r) * kSlabBytes + at);
      __builtin_amdgcn_sched_barrier(0);
    };
    // B's rows as the instruction's rows: a lane then holds four neighbouring columns of one row of C
    auto multiply = [&](const Operands &o, auto which) __attribute__((always_inline)) {
      constexpr int k = decltype(which)::value;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i)
          acc[j][i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(o.b[j]), wide(o.a[i]), acc[j][i], 4, 4, k, (int)sb[j], k, (int)sa[i]);
      __builtin_amdgcn_sched_barrier(0);
    };
    Operands x, y;                                        // a step's operands are read while the step before is multiplied
    read(x, 0);
    read(y, 1);
    multiply(x, std::integral_constant<int, 0>{});
    read(x, 2);
    multiply(y, std::integral_constant<int, 1>{});
    read(y, 3);
    multiply(x, std::integral_constant<int, 2>{});
    multiply(y, std::integral_constant<int, 3>{});
  };

  const int slabs = (p.blocks + kSlabBlocks - 1) / kSlabBlocks;
  bring(S0, 0);
  int s = 0;
  for (; s + 1 < slabs; s += 2) {
    bring(S1, s + 1);
    landed<kLoads>();
    compute(S0, s);
    __builtin_amdgcn_s_barrier();
    bring(S0, min(s + 2, slabs - 1));                     // past the last slab: brought again, not used
    landed<kLoads>();
    compute(S1, s + 1);
    __builtin_amdgcn_s_barrier();
  }
  landed<0>();
  if (s < slabs) compute(S0, s);

#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t row = i0 + wm0 + 32 * i + r;
    if (row >= p.m) continue;
    typename T::type *out = (typename T::type *)p.C + row * p.ld_c;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = j0 + wn0 + 32 * j + 8 * q + 4 * h;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = acc[j][i][4 * q + e];
          v[e] = p.relu && x < 0.f ? 0.f : x;
        }
        if (col + 4 <= p.n) {
          if constexpr (sizeof(typename T::type) == 4) *reinterpret_cast<op_f32x4 *>(out + col) = op_f32x4{v[0], v[1], v[2], v[3]};
          else *reinterpret_cast<op_u32x2 *>(out + col) = op_u32x2{BF16::two(v[0], v[1]), BF16::two(v[2], v[3])};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < p.n) T::put(out + col + e, v[e]);
        }
      }
  }
}

template <class T>
void launch_tile(MatmulArgs &a, int bm, int bn, hipStream_t s) {
  a.tiles_m = (int)((a.m + bm - 1) / bm);
  a.tiles_n = (a.n + bn - 1) / bn;
  const dim3 grid((unsigned)((int64_t)a.tiles_m * a.tiles_n)), block(256);
  if (bm == 256) hipLaunchKernelGGL((matmul_tile<T, 256, 256>), grid, block, 0, s, a);
  else if (bm == 128) hipLaunchKernelGGL((matmul_tile<T, 128, 128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((matmul_tile<T, 64, 64>), grid, block, 0, s, a);
}

}  // namespace

size_t mx_matmul_workspace(int32_t, int64_t, int32_t, int32_t) { return 0; }

int launch_mx_matmul(const pgcn_mx_matmul_args &x, hipStream_t s) {
  MatmulArgs a{x.A, x.A_scales, x.B, x.B_scales, x.C, x.m, x.ld_a, x.ld_a_scales, x.ld_b, x.ld_b_scales, x.ld_c, x.n,
               (int32_t)mx_blocks(x.k), x.relu, 0, 0};
  TraceScope ts(PGCN_TK_MX_MATMUL, s);
  const auto tiles = [&](int64_t b) { return ((x.m + b - 1) / b) * ((x.n + b - 1) / b); };
  const int b = tiles(256) >= 256 ? 256 : tiles(128) >= 256 ? 128 : 64;
  if (x.dtype == PGCN_BF16) launch_tile<BF16>(a, b, b, s);
  else launch_tile<F32>(a, b, b, s);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
