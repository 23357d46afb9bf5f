// Weight gradient from a layer's input held in 8 bits: dW = v^T (J o 1[H > 0]), a sum over the rows.  The rows
// are cut into splits; a workgroup adds one tile over one split, and a second launch adds the splits' partial
// tiles in a fixed order.
#include <algorithm>

#include "mx.h"

namespace pgcn {

namespace {

constexpr int kTile = 64, kSlab = 16;

struct WgradArgs {
  const uint8_t *Q, *S;
  const float *J, *H;
  float *out;             // [splits, f_in, f_out]
  int64_t rows, ld_q, ld_s, ld_j, ld_h, chunk;
  int32_t f_in, f_out, tiles_n, tiles;
};

struct Split {
  int64_t chunk;
  int splits;
};
Split wgrad_split(int64_t rows, int32_t f_in, int32_t f_out) {
  const int64_t tiles = (int64_t)((f_in + kTile - 1) / kTile) * ((f_out + kTile - 1) / kTile);
  int64_t s = std::max<int64_t>(1, std::min<int64_t>(1024 / tiles, (rows + 63) / 64));
  const int64_t chunk = std::max<int64_t>(kSlab, ((rows + s - 1) / s + kSlab - 1) / kSlab * kSlab);
  return Split{chunk, (int)std::max<int64_t>(1, (rows + chunk - 1) / chunk)};
}

template <bool kBf16>
__global__ __launch_bounds__(256) void wgrad(WgradArgs a) {
  __shared__ float As[kSlab][kTile + 4], Bs[kSlab][kTile + 4];
  const int t = threadIdx.x, tile = blockIdx.x % a.tiles;
  const int64_t split = blockIdx.x / a.tiles;
  const int m0 = tile / a.tiles_n * kTile, n0 = tile % a.tiles_n * kTile;
  const int64_t begin = split * a.chunk, end = min(a.rows, begin + a.chunk);
  const int r = t / 16, c = 4 * (t % 16);               // staging: a row of the slab, four columns
  float acc[4][4] = {};
  for (int64_t k = begin; k < end; k += kSlab) {
    const int64_t row = k + r;
    float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
    if (row < end && m0 + c < a.f_in) {
      const uint32_t q = *reinterpret_cast<const uint32_t *>(a.Q + row * a.ld_q + m0 + c);
      const float step = int8_step(a.S[row * a.ld_s + (m0 + c) / 32]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (float)(int)(int8_t)(q >> (8 * e)) * step;
    }
    if (row < end && n0 + c < a.f_out) {
      const op_f32x4 j = *reinterpret_cast<const op_f32x4 *>(a.J + row * a.ld_j + n0 + c);
      op_f32x4 h = {1.f, 1.f, 1.f, 1.f};
      if (a.H) h = *reinterpret_cast<const op_f32x4 *>(a.H + row * a.ld_h + n0 + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = h[e] > 0.f ? j[e] : 0.f;
        if (kBf16) y[e] = (float)(__bf16)y[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      As[r][c + e] = x[e];
      Bs[r][c + e] = y[e];
    }
    __syncthreads();
    for (int i = 0; i < kSlab; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] = __builtin_fmaf(As[i][4 * (t / 16) + u], Bs[i][4 * (t % 16) + v], acc[u][v]);
  }
  float *out = a.out + split * a.f_in * a.f_out;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int m = m0 + 4 * (t / 16) + u, n = n0 + 4 * (t % 16) + v;
      if (m < a.f_in && n < a.f_out) out[(int64_t)m * a.f_out + n] = acc[u][v];
    }
}

}  // namespace

size_t mx_wgrad_workspace(int32_t, int64_t rows, int32_t f_in, int32_t f_out) {
  const Split sp = wgrad_split(rows, f_in, f_out);
  return sp.splits > 1 ? (size_t)sp.splits * f_in * f_out * sizeof(float) : 0;
}

int launch_mx_wgrad(const pgcn_mx_wgrad_args &x, hipStream_t s) {
  const Split sp = wgrad_split(x.rows, x.f_in, x.f_out);
  WgradArgs a{x.Q, x.S, x.J, x.H, sp.splits > 1 ? (float *)x.workspace : x.dW, x.rows, x.ld_q, x.ld_s, x.ld_j, x.ld_h, sp.chunk,
              x.f_in, x.f_out, (x.f_out + kTile - 1) / kTile, 0};
  a.tiles = (x.f_in + kTile - 1) / kTile * a.tiles_n;
  {
    TraceScope ts(PGCN_TK_MX_WGRAD, s);
    const dim3 grid((unsigned)(a.tiles * sp.splits));
    if (x.dtype == PGCN_BF16) hipLaunchKernelGGL((wgrad<true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((wgrad<false>), grid, dim3(256), 0, s, a);
    PGCN_HIP(hipGetLastError());
  }
  if (sp.splits == 1) return PGCN_OK;
  return launch_splitk_reduce((const float *)x.workspace, sp.splits, (int64_t)x.f_in * x.f_out, x.dW, s);
}

}  // namespace pgcn
