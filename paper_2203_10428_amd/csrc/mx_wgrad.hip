// Weight gradient from a layer's input held in 8 bits: dW = v^T (J o 1[H > 0]), a sum over the rows (nodes).
//
// Every v is exact in bf16, so the product runs on the bf16 matrix cores: with J o mask in three exact bf16 parts
// (fp32 arithmetic: three products where two fp32 operands take six), or rounded to bf16 once.
// The rows are cut into splits; a workgroup adds one BM x BN tile over one split in slabs of 16 rows, and a second
// launch adds the splits' partial tiles in a fixed order.  A slab goes through registers into LDS as it lies in
// memory, a row of features after another, and the transposing LDS reads give each lane the four rows' values of one
// feature that the matrix instruction wants.  Two LDS stages and two register sets: loads have two slabs of
// products to arrive.
#include <algorithm>

#include "mx.h"

namespace pgcn {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kSlab = 16, kPad = 32;       // rows; bf16 elements behind a row in LDS: four rows read together are on other banks

struct WgradArgs {
  const uint8_t *Q, *S;
  const float *J, *H;
  float *out;             // [splits, f_in, f_out]
  int64_t rows, ld_q, ld_s, ld_j, ld_h, chunk;
  int32_t f_in, f_out, tiles_n, tiles;
};

// Eight INT8 elements as bf16: (u - 128) step, u = q + 128, is exact, so its high half is the value.  One product-sum,
// but for the largest scale, with which 128 step is no float.
__device__ __forceinline__ op_u32x4 bf16_of(const op_u32x2 &q, float step) {
  op_u32x4 w;
  if (step > 0x1p120f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = q[i / 2] >> (16 * (i % 2));
      w[i] = __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(u >> 8) * step), __float_as_uint((float)(int8_t)u * step), 0x07060302u);
    }
    return w;
  }
  const float off = -128.f * step;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t u = q[i] ^ 0x80808080u;
    const float a = __builtin_fmaf((float)(u & 0xffu), step, off), b = __builtin_fmaf((float)((u >> 8) & 0xffu), step, off);
    const float c = __builtin_fmaf((float)((u >> 16) & 0xffu), step, off), d = __builtin_fmaf((float)(u >> 24), step, off);
    w[2 * i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    w[2 * i + 1] = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x07060302u);
  }
  return w;
}

// Two floats in three bf16 parts each: the high half, what is left rounded to nearest, and the rest.
__device__ __forceinline__ void parts2(float x, float y, uint32_t (&p)[3]) {
  const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
  p[0] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  const float r = x - __uint_as_float(a & 0xffff0000u), s = y - __uint_as_float(b & 0xffff0000u);
  p[1] = BF16::two(r, s);
  p[2] = BF16::two(r - __uint_as_float(p[1] << 16), s - __uint_as_float(p[1] & 0xffff0000u));
}

// Four rows' values of this lane's feature, from a place of its own in four rows of 16 neighbouring features.
__device__ __forceinline__ bf16x8 transposed(const uint16_t *lo, const uint16_t *hi) {
  typedef __attribute__((address_space(3))) i16x4 *lds;
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)lo), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)hi);
  typedef short i16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf16x8, (i16x8){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

template <int BM, int BN, int kParts, bool kMasked>
__global__ __launch_bounds__(256, 2) void wgrad(WgradArgs p) {
  constexpr int LA = BM + kPad, LB = BN + kPad;
  constexpr int CA = BM / 8, CB = BN / 4, RB = 256 / CB, VA = (kSlab * CA + 255) / 256, VB = kSlab / RB;
  constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
  static_assert(kSlab * CA % 64 == 0 && VB >= 1, "whole waves have an item");
  __shared__ __attribute__((aligned(16))) uint16_t As[2][kSlab * LA];
  __shared__ __attribute__((aligned(16))) uint16_t Bs[2][kParts][kSlab * LB];

  const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64);
  // a split's tiles are neighbours on one XCD: its rows are read there several times
  const uint32_t g = blockIdx.x, l = gridDim.x % 8 == 0 ? (g % 8) * (gridDim.x / 8) + g / 8 : g;
  const uint32_t split = l / (uint32_t)p.tiles, tile = l - split * (uint32_t)p.tiles;
  const int m0 = (int)(tile / p.tiles_n) * BM, n0 = (int)(tile % p.tiles_n) * BN;
  const int64_t begin = split * p.chunk, end = min(p.rows, begin + p.chunk);

  // staging: items t + 256 i of v, a row's eight features, the last for some waves alone; row rb + RB i and four of J
  const int cb = 4 * (t % CB), rb = t / CB;
  int ca[VA], ra[VA];
#pragma unroll
  for (int i = 0; i < VA; ++i) ca[i] = 8 * ((t + 256 * i) % CA), ra[i] = (t + 256 * i) / CA;
  auto has = [&](int i) __attribute__((always_inline)) { return (i + 1) * 256 <= kSlab * CA || 64 * wave + 256 * i < kSlab * CA; };
  struct Regs {
    op_u32x2 q[VA];
    uint32_t s[VA];
    op_f32x4 j[VB], h[VB];
  };
  // Columns past the matrix read its first ones: their products are not stored.
  const int64_t col_j = n0 + cb < p.f_out ? n0 + cb : 0, off_j = rb * p.ld_j + col_j, off_h = rb * p.ld_h + col_j;
  int64_t off_q[VA], off_s[VA];
#pragma unroll
  for (int i = 0; i < VA; ++i) {
    const int64_t col = m0 + ca[i] < p.f_in ? m0 + ca[i] : 0;
    off_q[i] = ra[i] * p.ld_q + col;
    off_s[i] = ra[i] * p.ld_s + col / 32;
  }
  auto load = [&](Regs &R, int64_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VA; ++i)
      if (has(i)) {
        R.q[i] = *reinterpret_cast<const op_u32x2 *>(p.Q + k * p.ld_q + off_q[i]);
        R.s[i] = (p.S + k * p.ld_s)[off_s[i]];
      }
#pragma unroll
    for (int i = 0; i < VB; ++i) {
      R.j[i] = *reinterpret_cast<const op_f32x4 *>(p.J + (k + RB * i) * p.ld_j + off_j);
      if (kMasked) R.h[i] = *reinterpret_cast<const op_f32x4 *>(p.H + (k + RB * i) * p.ld_h + off_h);
    }
  };
  auto load_last = [&](Regs &R, int64_t k) __attribute__((always_inline)) {      // zeros for rows past the last one
#pragma unroll
    for (int i = 0; i < VA; ++i) {
      const bool in = has(i) && k + ra[i] < p.rows;
      R.q[i] = in ? *reinterpret_cast<const op_u32x2 *>(p.Q + k * p.ld_q + off_q[i]) : op_u32x2{0u, 0u};
      R.s[i] = in ? (p.S + k * p.ld_s)[off_s[i]] : 0u;
    }
#pragma unroll
    for (int i = 0; i < VB; ++i) {
      const int64_t row = k + rb + RB * i;
      const bool in = row < p.rows;
      R.j[i] = in ? *reinterpret_cast<const op_f32x4 *>(p.J + row * p.ld_j + col_j) : op_f32x4{0.f, 0.f, 0.f, 0.f};
      if (kMasked) R.h[i] = in ? *reinterpret_cast<const op_f32x4 *>(p.H + row * p.ld_h + col_j) : op_f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  auto store = [&](const Regs &R, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VA; ++i)
      if (has(i)) *reinterpret_cast<op_u32x4 *>(&As[buf][ra[i] * LA + ca[i]]) = bf16_of(R.q[i], int8_step(R.s[i]));
#pragma unroll
    for (int i = 0; i < VB; ++i) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = !kMasked || R.h[i][e] > 0.f ? R.j[i][e] : 0.f;
      const int at = (rb + RB * i) * LB + cb;
      if constexpr (kParts == 1) {
        *reinterpret_cast<op_u32x2 *>(&Bs[buf][0][at]) = op_u32x2{BF16::two(x[0], x[1]), BF16::two(x[2], x[3])};
      } else {
        uint32_t u[3], v[3];
        parts2(x[0], x[1], u);
        parts2(x[2], x[3], v);
#pragma unroll
        for (int part = 0; part < 3; ++part) *reinterpret_cast<op_u32x2 *>(&Bs[buf][part][at]) = op_u32x2{u[part], v[part]};
      }
    }
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = (f32x16){};
  // operand of the matrix instruction: feature lane % 32, rows 8 (lane / 32) + 0 .. 7 of the slab; 16 lanes read
  // rows 0 .. 3 and then 4 .. 7 of those, four lanes to a row
  const int h = lane / 32, wm0 = (wave / 2) * WM, wn0 = (wave % 2) * WN;
  const int tr = 8 * h + (lane % 16) / 4, tc = 16 * ((lane / 16) % 2) + 4 * (lane % 4);
  auto compute = [&](int buf) __attribute__((always_inline)) {
    bf16x8 a[TM], b[2][TN];
    auto read = [&](int part) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const uint16_t *at = &Bs[buf][part][tr * LB + wn0 + 32 * j + tc];
        b[part & 1][j] = transposed(at, at + 4 * LB);
      }
    };
    read(kParts - 1);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const uint16_t *at = &As[buf][tr * LA + wm0 + 32 * i + tc];
      a[i] = transposed(at, at + 4 * LA);
    }
#pragma unroll
    for (int part = kParts - 1; part >= 0; --part) {      // smallest first; the next part is read meanwhile
      if (part > 0) read(part - 1);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[part & 1][j], acc[i][j], 0, 0, 0);
    }
  };

  const int64_t full = begin < end ? (end - begin) / kSlab : 0, last = begin + (full - 1) * kSlab;
  Regs R0, R1;
  if (full > 0) {
    load(R0, begin);
    load(R1, min(begin + kSlab, last));                   // past the last full slab: it again, not used
    store(R0, 0);
    __syncthreads();
    int64_t k = begin;
    for (; k < last; k += 2 * kSlab) {
      load(R0, min(k + 2 * kSlab, last));
      compute(0);
      store(R1, 1);
      __syncthreads();
      load(R1, min(k + 3 * kSlab, last));
      compute(1);
      store(R0, 0);
      __syncthreads();
    }
    if (k == last) compute(0);
  }
  if (begin + full * kSlab < end) {                       // the rows that are left, fewer than a slab
    load_last(R0, begin + full * kSlab);
    store(R0, 1);
    __syncthreads();
    compute(1);
  }

  float *out = p.out + (int64_t)split * p.f_in * p.f_out;
  const bool whole = m0 + BM <= p.f_in && n0 + BN <= p.f_out;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = m0 + wm0 + 32 * i + 8 * (e / 4) + 4 * h + e % 4, n = n0 + wn0 + 32 * j + lane % 32;
        if (whole || (m < p.f_in && n < p.f_out)) out[(int64_t)m * p.f_out + n] = acc[i][j][e];
      }
}

struct Shape {
  int bm, bn, splits;
  int64_t chunk;
};

// Tile: 256 or 192 features of v where that fills up no more than 128 do, since a slab's J is split into its parts by
// every tile row (fp32: 239,000 x 512 x 512 347 us with 256, 455 with 128; 239,000 x 300 x 512 284 with 192, 348 with 128;
// 58,000 x 602 x 256, which 256 would fill up to 768: 81 against 76).
// Splits: as many workgroups as are resident at once, or fewer where their partial tiles cost more than they bring.  fp32
// 128-row tiles three to a compute unit (58,000 x 602 x 256: 76 us and 8 for adding the partial tiles, at two 83 and 6), with
// two tiles two, with one one (306,000 x 128 x 128: 75 us with the adding, at three 93; 306,000 x 128 x 256: 135 at two, 148 at
// three); larger tiles two.  bf16, which waits for memory, two, with up to two tiles one (306,000 x 128 x 256: 126, at two
// 135; 100,000 x 400 x 128: 55 and 71).  Tiles of 64 columns two (306,000 x 100 x 47 fp32: 39, at one 49, at three 47).
// At least 64 rows to a split; where that leaves compute units idle down to 32, as a workgroup's slabs are a chain.
// The partial matrices stay below 64 MB together.
Shape shape_of(int32_t dtype, int64_t rows, int32_t f_in, int32_t f_out) {
  Shape c;
  c.bn = f_out <= 64 ? 64 : 128;
  const auto filled = [&](int bm) { return (f_in + bm - 1) / bm * bm; };
  c.bm = f_in <= 128 || c.bn == 64 ? 128 : filled(256) <= filled(128) ? 256 : filled(192) <= filled(128) ? 192 : 128;
  const int64_t tiles = (int64_t)((f_in + c.bm - 1) / c.bm) * ((f_out + c.bn - 1) / c.bn);
  int64_t slots = 512;
  if (c.bn == 128 && dtype == PGCN_BF16 && tiles <= 2) slots = 256;
  if (c.bn == 128 && dtype == PGCN_F32 && c.bm == 128) slots = std::min<int64_t>(256 * tiles, 768);
  // no more than the fp32 and bf16 forms take, whose scratch a layer's backward has
  const int64_t tile_bytes = (int64_t)f_in * f_out * 4;
  const int64_t by_bytes =
      std::max<int64_t>(1, std::min<int64_t>((int64_t)64 << 20, gemm_workspace(Gemm::TN_MASK_SPLITK, f_in, f_out, (int32_t)rows)) / tile_bytes);
  int64_t s = std::max<int64_t>(1, std::min({slots / tiles, (rows + 63) / 64, by_bytes}));
  if (tiles * s < 256) s = std::max(s, std::min({(rows + 31) / 32, (256 + tiles - 1) / tiles, by_bytes}));
  int64_t e = s;                                          // a multiple of 8 workgroups: see the order of tiles
  while (e > 1 && tiles * e % 8 != 0) --e;
  if (tiles * e % 8 == 0 && 2 * e >= s) s = e;
  c.chunk = std::max<int64_t>(kSlab, ((rows + s - 1) / s + kSlab - 1) / kSlab * kSlab);
  c.splits = (int)std::max<int64_t>(1, (rows + c.chunk - 1) / c.chunk);
  return c;
}

template <int BM, int BN>
void launch_tile(const WgradArgs &a, int splits, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.tiles * splits));
  if (a.H) {
    if (bf16) hipLaunchKernelGGL((wgrad<BM, BN, 1, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((wgrad<BM, BN, 3, true>), grid, dim3(256), 0, s, a);
  } else {
    if (bf16) hipLaunchKernelGGL((wgrad<BM, BN, 1, false>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((wgrad<BM, BN, 3, false>), grid, dim3(256), 0, s, a);
  }
}

}  // namespace

size_t mx_wgrad_workspace(int32_t dtype, int64_t rows, int32_t f_in, int32_t f_out) {
  const Shape c = shape_of(dtype, rows, f_in, f_out);
  return c.splits > 1 ? (size_t)c.splits * f_in * f_out * sizeof(float) : 0;
}

int launch_mx_wgrad(const pgcn_mx_wgrad_args &x, hipStream_t s) {
  const Shape c = shape_of(x.dtype, x.rows, x.f_in, x.f_out);
  WgradArgs a{x.Q, x.S, x.J, x.H, c.splits > 1 ? (float *)x.workspace : x.dW, x.rows, x.ld_q, x.ld_s, x.ld_j, x.ld_h, c.chunk,
              x.f_in, x.f_out, (x.f_out + c.bn - 1) / c.bn, 0};
  a.tiles = (x.f_in + c.bm - 1) / c.bm * a.tiles_n;
  {
    TraceScope ts(PGCN_TK_MX_WGRAD, s);
    const bool bf16 = x.dtype == PGCN_BF16;
    if (c.bn == 64) launch_tile<128, 64>(a, c.splits, bf16, s);
    else if (c.bm == 128) launch_tile<128, 128>(a, c.splits, bf16, s);
    else if (c.bm == 192) launch_tile<192, 128>(a, c.splits, bf16, s);
    else launch_tile<256, 128>(a, c.splits, bf16, s);
    PGCN_HIP(hipGetLastError());
  }
  if (c.splits == 1) return PGCN_OK;
  return launch_splitk_reduce((const float *)x.workspace, c.splits, (int64_t)x.f_in * x.f_out, x.dW, s);
}

}  // namespace pgcn
