// The backward of the norms around a block (norm_bwd.hpp) on bf16 rows, its launches, and the
// sum of the workgroups' parts.
#include "norm_bwd.hpp"

namespace mapl {

namespace {

// out[j][c] (+)= sum over the workgroups' parts in a fixed order; 1024 / COLS runs of them
// side by side for COLS columns.
constexpr int COLS = 64;
__global__ __launch_bounds__(1024) void k_norm_sum(const float* __restrict__ part, int n, int d, NormSums o, int add) {
  constexpr int RUNS = 1024 / COLS;
  __shared__ float red[RUNS][COLS];
  const int j = blockIdx.y, c = blockIdx.x * COLS + threadIdx.x % COLS, k = threadIdx.x / COLS;
  float* out = j == 0 ? o.dw_post : j == 1 ? o.dscale : o.dw_pre;
  if (!out) return;
  float s = 0.f;
  const float* p = part + (int64_t)j * d + c;
#pragma unroll 8
  for (int i = k; i < n; i += RUNS) s += p[(int64_t)i * 3 * d];
  red[k][threadIdx.x % COLS] = s;
  __syncthreads();
  if (k == 0) {
#pragma unroll
    for (int i = 1; i < RUNS; ++i) s += red[i][threadIdx.x];
    out[c] = add ? out[c] + s : s;
  }
}

}  // namespace

// Workgroups: two a CU (three where y is all there is, which takes fewer registers, and of the 192
// lanes for up to 1536 values; one past 4096 values, as many as fit), but one where each would see less than four rows in turn,
// since each leaves 3 d sums to be read again.  In us with 256, 512 and 768, T = 32768 and d = 2048
// in bf16: with a gated branch 289, 205, 211; y alone 162, 98, 93; T = 1021, d = 1024 13.0, 14.1, 14.1; T = 2048,
// d = 8192 71.5, 81.0; T = 8000, d = 1536 with 512 and 768 53.1, 49.7.
int norm_bwd_parts(int64_t T, int d, int parts) {
  const int rows = (d <= 64 ? 32 : d <= 128 ? 16 : d <= 256 ? 8 : d <= 512 ? 4 : d <= 1024 ? 2 : 1) * (norm_bwd_wide(T, d) ? 2 : 1);
  const int64_t n = (T + rows - 1) / rows;
  const int most = d > 4096 ? 256 : parts == NORM_PRE || (d > 1024 && d <= 1536) ? 768 : 512;
  const int64_t w = n / 4 > 256 ? n / 4 : 256;
  return (int)(n < w ? n : w < most ? w : most);
}

hipError_t launch_norm_bwd_f32(const NormArgs& g, hipStream_t s);  // fp32 x (k_norm_bwd_f32.hip)

hipError_t launch_norm_bwd(const NormArgs& g, hipStream_t s) {
  if (g.x_f32) return launch_norm_bwd_f32(g, s);
  return g.once ? pick<bf16_t, bf16_t, true>(g, s) : pick<bf16_t, bf16_t, false>(g, s);
}

hipError_t launch_norm_sum(const float* part, int n, int d, const NormSums& o, int add, hipStream_t s) {
  hipLaunchKernelGGL(k_norm_sum, dim3(d / COLS, 3), dim3(1024), 0, s, part, n, d, o, add);
  return hipGetLastError();
}

}  // namespace mapl
