// Rows in 8 and 4 bits: quantised as they are written (gathered or transposed), and read back with a moving
// average.  Per block of 32 elements: s from the largest magnitude, q = round(x / 2^(s - 127) 64) or the nearest
// of the 4-bit magnitudes.  All of it is exact but the one rounding of an element.
#include "mx.h"

namespace pgcn {

namespace {

constexpr int kThreads = 256;

// One launch counts its threads along x in 32 bits: the workgroups go along y too.
inline dim3 grid_of(int64_t workgroups) {
  const int64_t x = workgroups < (int64_t(1) << 22) ? workgroups : int64_t(1) << 22;
  return dim3((unsigned)x, (unsigned)((workgroups + x - 1) / x));
}
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

struct QuantArgs {
  const void *X;
  const int32_t *index;
  uint8_t *Q, *S;
  int64_t rows, src_rows, ld_x, ld_q, ld_s;
  int32_t cols;
  Chunks chunks;        // of 8 elements, four to a block
};

// Four neighbouring lanes to a block, eight elements each.  Bound by memory: 239,000 x 512 fp32 to INT8 110 us, 5.6 TB/s,
// with loads past the caches (127 through them); gathered rows, which several peers are sent, go through them
// (462,000 rows of 239,000: 199 us against 212).  More than one chunk to a thread changes nothing.
template <class T, class F, bool kGather>
__global__ __launch_bounds__(kThreads) void quantize_rows(QuantArgs a) {
  const int64_t first = workgroup() * kThreads;
  const int64_t row0 = first / a.chunks.per;
  const uint32_t at = (uint32_t)(first - row0 * a.chunks.per) + threadIdx.x;
  if (first + threadIdx.x >= a.chunks.total) return;     // whole blocks: a row's chunks are a multiple of four
  const uint32_t down = chunk_row(a.chunks, at), c = at - down * a.chunks.per;
  const int64_t row = row0 + down;
  const int64_t src = kGather ? a.index[row] : row;
  float x[8];
  const bool some = src >= 0 && src < a.src_rows;
  const typename T::type *X = (const typename T::type *)a.X + (some ? src * a.ld_x + 8 * (int64_t)c : 0);
  load8<!kGather>(T{}, X, some ? a.cols - 8 * (int64_t)c : 0, x);
  uint32_t m = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
  m = max(m, __float_as_uint(lane_move<0xB1>(__uint_as_float(m))));
  m = max(m, __float_as_uint(lane_move<0x4E>(__uint_as_float(m))));
  const uint32_t s = src >= a.src_rows ? 255u : scale_byte<F>(m);
  *reinterpret_cast<typename Bits8<F>::type *>(a.Q + row * a.ld_q + (int64_t)c * (F::kBytes / 4)) = pack8(F{}, x, s);
  if (c % 4 == 0) a.S[row * a.ld_s + c / 4] = (uint8_t)s;
}

// The transpose of rows that are not aligned to 16 bytes, a layer's compact weights: a thread to a block, 32 rows of
// one column.
__global__ __launch_bounds__(kThreads) void quantize_unaligned_cols(QuantArgs a, uint32_t col_groups) {
  const int64_t block = workgroup() / col_groups;
  const int64_t col = (workgroup() - block * col_groups) * kThreads + threadIdx.x;
  if (col >= a.cols || 32 * block >= a.rows) return;
  const float *X = (const float *)a.X + col;
  uint32_t m = 0u;
  for (int64_t r = 32 * block; r < min(a.rows, 32 * block + 32); ++r) m = max(m, __float_as_uint(X[r * a.ld_x]) & 0x7fffffffu);
  const uint32_t s = scale_byte<Fp4>(m);
  for (int i = 0; i < 4; ++i) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t r = 32 * block + 8 * i + e;
      x[e] = r < a.rows ? X[r * a.ld_x] : 0.f;
    }
    *reinterpret_cast<uint32_t *>(a.Q + col * a.ld_q + (4 * block + i) * (Fp4::kBytes / 4)) = pack8(Fp4{}, x, s);
  }
  a.S[col * a.ld_s + block] = (uint8_t)s;
}

// The transpose: a thread holds 32 rows of 4 (fp32) or 8 (bf16) columns in registers, whole blocks of its columns, so
// nothing is exchanged.  Eight lanes read 128 bytes of a row, and the eight blocks of a wave are neighbours in Q.
template <class T, class F>
__global__ __launch_bounds__(kThreads) void quantize_cols(QuantArgs a, uint32_t col_groups) {
  const int64_t bands = workgroup() / col_groups;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t block = 8 * bands + lane / 8;
  const int64_t col = T::E * ((workgroup() - bands * col_groups) * 32 + 8 * wave + lane % 8);
  if (col >= a.cols || 32 * block >= a.rows) return;
  const typename T::type *X = (const typename T::type *)a.X + 32 * block * a.ld_x + col;
  const int64_t rows = a.rows - 32 * block;
  op_u32x4 x[32];
#pragma unroll
  for (int r = 0; r < 32; ++r) x[r] = r < rows ? load_vector<true, op_u32x4>(X + r * a.ld_x) : op_u32x4{0u, 0u, 0u, 0u};
  const int cols = (int)min((int64_t)T::E, a.cols - col);
#pragma unroll
  for (int c = 0; c < T::E; ++c) {
    auto bits = [&](int r) __attribute__((always_inline)) {          // as a float's
      if constexpr (T::E == 4) return x[r][c];
      else return c % 2 ? x[r][c / 2] & 0xffff0000u : x[r][c / 2] << 16;
    };
    uint32_t m = 0u;
#pragma unroll
    for (int r = 0; r < 32; ++r) m = max(m, bits(r) & 0x7fffffffu);
    const uint32_t s = scale_byte<F>(m);
    typename Bits8<F>::type q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(bits(8 * i + e));
      q[i] = pack8(F{}, v, s);
    }
    if (c < cols) {
      op_u32x4 *out = reinterpret_cast<op_u32x4 *>(a.Q + (col + c) * a.ld_q + block * F::kBytes);
      if constexpr (F::kBytes == 16) {
        out[0] = op_u32x4{q[0], q[1], q[2], q[3]};
      } else {
        out[0] = op_u32x4{q[0][0], q[0][1], q[1][0], q[1][1]};
        out[1] = op_u32x4{q[2][0], q[2][1], q[3][0], q[3][1]};
      }
      a.S[(col + c) * a.ld_s + block] = (uint8_t)s;
    }
  }
}

struct ReadArgs {
  const uint8_t *Q, *S;
  void *out;
  int64_t ld_q, ld_s, ld_out;
  int32_t cols;
  float gamma, rest;       // rest = 1 - gamma
  Chunks chunks;           // of 16 bytes of out that hold some of a row's
};

// A thread to 16 bytes of out, so that a wave writes whole lines (32 bytes to a thread: 462,000 x 512 with the moving average
// 368 us against 341, 6.4 TB/s), past the caches where it has not read them (239,000 x 256 fp32: 44 us, through them 52; the
// step that gathers them next takes no longer, 16.3 ms on 239,000 nodes against 16.4).
template <class T, class F, bool kAverage>
__global__ __launch_bounds__(kThreads) void read_rows(ReadArgs a) {
  constexpr int E = T::E;
  const int64_t first = workgroup() * kThreads;
  const int64_t row0 = first / a.chunks.per;
  const uint32_t at = (uint32_t)(first - row0 * a.chunks.per) + threadIdx.x;
  if (first + threadIdx.x >= a.chunks.total) return;
  const uint32_t down = chunk_row(a.chunks, at), c = at - down * a.chunks.per;
  const int64_t row = row0 + down;
  float v[E];
  unpack<E>(F{}, a.Q + row * a.ld_q + (int64_t)c * (F::kBytes * E / 32), a.S[row * a.ld_s + c / (32 / E)], v);
  typename T::type *out = (typename T::type *)a.out + row * a.ld_out + E * (int64_t)c;
  const int n = a.cols - E * (int)c;
  if constexpr (kAverage) {
    const typename T::raw x = *reinterpret_cast<const typename T::raw *>(out);
    static_assert(E == 4, "a moving average is kept in fp32");
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = __builtin_fmaf(a.gamma, x[e], a.rest * v[e]);
  }
  if (!kAverage && n >= E) __builtin_nontemporal_store(T::pack(v), (typename T::raw *)out);
  else store_some<T>(out, v, n);
}

template <class T, class F>
void quantize(const QuantArgs &a, bool transpose, hipStream_t s) {
  if (transpose) {
    const int64_t groups = (a.cols + 32 * T::E - 1) / (32 * T::E), bands = (mx_blocks(a.rows) + 7) / 8;
    hipLaunchKernelGGL((quantize_cols<T, F>), grid_of(groups * bands), dim3(kThreads), 0, s, a, (uint32_t)groups);
  } else {
    const dim3 grid = grid_of((a.chunks.total + kThreads - 1) / kThreads);
    if (a.index) hipLaunchKernelGGL((quantize_rows<T, F, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((quantize_rows<T, F, false>), grid, dim3(kThreads), 0, s, a);
  }
}

}  // namespace

int launch_mx_quantize(const pgcn_mx_quantize_args &x, hipStream_t s) {
  QuantArgs a{x.X, x.index, x.Q, x.S, x.rows, x.src_rows, x.ld_x, x.ld_q, x.ld_s, x.cols, chunks_of(x.rows, 4 * mx_blocks(x.cols))};
  TraceScope ts(PGCN_TK_MX_QUANTIZE, s);
  const bool int8 = x.format == PGCN_MX_INT8;
  if (x.transpose && x.ld_x % 4 != 0) {           // only a layer's own call: fp32 weights in 4 bits
    const int64_t groups = (a.cols + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(quantize_unaligned_cols, grid_of(groups * mx_blocks(a.rows)), dim3(kThreads), 0, s, a, (uint32_t)groups);
    PGCN_HIP(hipGetLastError());
    return PGCN_OK;
  }
  if (x.dtype == PGCN_BF16) int8 ? quantize<BF16, Int8>(a, x.transpose, s) : quantize<BF16, Fp4>(a, x.transpose, s);
  else int8 ? quantize<F32, Int8>(a, x.transpose, s) : quantize<F32, Fp4>(a, x.transpose, s);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

int launch_mx_dequantize(const pgcn_mx_dequantize_args &x, hipStream_t s) {
  const ReadArgs a{x.Q, x.S, x.out, x.ld_q, x.ld_s, x.ld_out, x.cols, x.gamma, 1.f - x.gamma, chunks_of(x.rows, x.dtype == PGCN_BF16 ? (x.cols + 7) / 8 : (x.cols + 3) / 4)};
  const dim3 grid = grid_of((a.chunks.total + kThreads - 1) / kThreads), block(kThreads);
  TraceScope ts(PGCN_TK_MX_DEQUANTIZE, s);
  const bool int8 = x.format == PGCN_MX_INT8;
  if (x.dtype == PGCN_BF16) {
    if (int8) hipLaunchKernelGGL((read_rows<BF16, Int8, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_rows<BF16, Fp4, false>), grid, block, 0, s, a);
  } else if (x.gamma > 0.f) {
    if (int8) hipLaunchKernelGGL((read_rows<F32, Int8, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_rows<F32, Fp4, true>), grid, block, 0, s, a);
  } else {
    if (int8) hipLaunchKernelGGL((read_rows<F32, Int8, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_rows<F32, Fp4, false>), grid, block, 0, s, a);
  }
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
