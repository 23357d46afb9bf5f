// Product of two matrices of FP4 rows, C = a b^T, on the scaled matrix instructions: v_mfma_scale_f32_16x16x128_f8f6f4
// takes a block of 32 elements with its scale from each lane (lane: row lane % 16, block lane / 16 of four).
#include "mx.h"

namespace pgcn {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct MatmulArgs {
  const uint8_t *A, *SA, *B, *SB;
  void *C;
  int64_t m, ld_a, ld_sa, ld_b, ld_sb, ld_c;
  int32_t n, blocks, relu, groups_n;
};

// A block and its scale; zeros past the matrix.
__device__ __forceinline__ i32x8 block_of(const uint8_t *Q, const uint8_t *S, int64_t row, int block, bool there, int64_t ld_q, int64_t ld_s, int &scale) {
  op_u32x4 q = {0u, 0u, 0u, 0u};
  scale = 0;
  if (there) {
    q = *reinterpret_cast<const op_u32x4 *>(Q + row * ld_q + 16 * (int64_t)block);
    scale = S[row * ld_s + block];
  }
  return i32x8{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0};
}

// A wave to 16 x 16 results.
template <class T>
__global__ __launch_bounds__(256) void matmul(MatmulArgs a) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t i = (int64_t)(blockIdx.x / a.groups_n) * 16;
  const int64_t j = (int64_t)(blockIdx.x % a.groups_n) * 64 + 16 * wave;
  if (j >= a.n) return;
  const int64_t ra = i + lane % 16, rb = j + lane % 16;
  op_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int b = 0; b < a.blocks; b += 4) {
    int sa, sb;
    const int mine = b + lane / 16;
    const i32x8 x = block_of(a.A, a.SA, ra, mine, ra < a.m && mine < a.blocks, a.ld_a, a.ld_sa, sa);
    const i32x8 y = block_of(a.B, a.SB, rb, mine, rb < a.n && mine < a.blocks, a.ld_b, a.ld_sb, sb);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, 0, sa, 0, sb);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t row = i + 4 * (lane / 16) + e;
    if (row < a.m && rb < a.n)
      T::put((typename T::type *)a.C + row * a.ld_c + rb, a.relu && acc[e] < 0.f ? 0.f : acc[e]);
  }
}

}  // namespace

size_t mx_matmul_workspace(int32_t, int64_t, int32_t, int32_t) { return 0; }

int launch_mx_matmul(const pgcn_mx_matmul_args &x, hipStream_t s) {
  const MatmulArgs a{x.A, x.A_scales, x.B, x.B_scales, x.C, x.m, x.ld_a, x.ld_a_scales, x.ld_b, x.ld_b_scales, x.ld_c, x.n,
                     (int32_t)mx_blocks(x.k), x.relu, (x.n + 63) / 64};
  TraceScope ts(PGCN_TK_MX_MATMUL, s);
  const dim3 grid((unsigned)((x.m + 15) / 16 * a.groups_n));
  if (x.dtype == PGCN_BF16) hipLaunchKernelGGL((matmul<BF16>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((matmul<F32>), grid, dim3(256), 0, s, a);
  PGCN_HIP(hipGetLastError());
  return PGCN_OK;
}

}  // namespace pgcn
