// The norms around a block of a stage, with the block's gate and residual
// scale: for every token (row of d values)
//   n  = h r_h w_post, r_h = (mean h^2 + eps)^-1/2       (with NORM_POST; else n = h)
//   x' = x + alpha s (n act(G))                          (with NORM_BRANCH; else x' = x)
//   y  = x' r_x w_pre, r_x = (mean x'^2 + eps)^-1/2      (with NORM_PRE)
// in one pass, x' rounded to its type before y is computed from it.  Sums,
// statistics and everything in between are fp32.
//
// Bound by HBM: 10 bytes a value where everything is bf16.  T = 32768, d = 2048 with a gated
// branch whose two arrays are halves of one product's output 116 us, 5.8 TB/s (a large copy
// here 4.9); T = 8192, d = 1024 14.1 us, 5.9 TB/s; the residual add and
// y alone (no norm of h, no gate) 101 us and 11.5, an fp32 stream with the gated bf16 block 163 and 26.6.  What carried it: one row a wave or a workgroup with all of
// its loads first and no branch before them (143 us with one around each), rows by a scalar
// base and 32-bit offsets, one-shot workgroups (with 2048 of them in a loop 150 and 129),
// fp32 rows in runs of 1 KiB a wave and access, rows past 8192 on 512 lanes (T = 4096, d = 8256 with
// 1024 lanes 92 us, 71; d = 12288 113, 90; d = 16384 128, 121).
#include "norm_rows.hpp"

namespace mapl {

namespace {

// A row is held by LANES lanes, eight values NV times each; a workgroup of THREADS
// takes THREADS / LANES rows.
template <typename X, typename H, int LANES, int NV, int THREADS, bool BRANCH, bool PRE, int GATE, bool ONCE>
__global__ __launch_bounds__(THREADS) void k_norm_fwd(const NormArgs g) {
  constexpr int ROWS = THREADS / LANES;
  constexpr bool SPLIT = sizeof(X) == 4, FINE = sizeof(X) == 4;
  __shared__ float lds[sums_floats(LANES, ROWS)];
  int turn = 0;
  const Cols<LANES, SPLIT, ONCE> c{(int)threadIdx.x % LANES, g.d};
  const float inv_d = 1.f / (float)g.d;
  const int64_t d = g.d;
  const bool ragged = g.d != LANES * NV * 8;
  const int64_t row = (int64_t)blockIdx.x * ROWS + sub_row<LANES, ROWS>();
  const bool live = ROWS == 1 || row < g.T;  // (past the last row: the last one again, not written)
  const int64_t t = live ? row : g.T - 1;
  Oct<X> x[NV];
  Oct<H> h[NV], u[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (BRANCH) h[v].load((const H*)g.h + t * g.ld_h, c, v);
    x[v].load((const X*)g.x + t * d, c, v);
    if constexpr (GATE != 0) u[v].load((const H*)g.gate + t * g.ld_g, c, v);
  }
  if (ragged) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (BRANCH) h[v].zero_past(c, v);
      x[v].zero_past(c, v);
    }
  }
  float z[NV][8];
  if constexpr (BRANCH) {
    const float *w_post = or_ones(g.w_post), *scale = or_ones(g.scale);
    float r = 1.f;
    if (g.parts & NORM_POST) {
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(h[v].get(i), h[v].get(i), s[0]);
      const uint32_t over = row_sums<LANES, ROWS, 1>(s, lds, turn);
      r = row_scale<LANES, ROWS, NV>(s[0], over, [&](int v, int i) { return h[v].get(i); }, inv_d, g.eps, lds, turn);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], sc[8];
      vec8(w_post, c, v, w);
      vec8(scale, c, v, sc);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        z[v][i] = h[v].get(i) * r * w[i];
        if constexpr (GATE != 0) {
          float f, df;
          act_both<GATE, FINE>(u[v].get(i), f, df);
          z[v][i] *= f;
        }
        z[v][i] = fmaf(g.alpha * sc[i], z[v][i], x[v].get(i));
      }
      put8((X*)g.xo + t * d, c, v, z[v], live);
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) z[v][i] = x[v].get(i);
  }
  if constexpr (PRE) {
    const float* w_pre = or_ones(g.w_pre);
    if (BRANCH && ragged)  // (a gate or a weight that is no number may have made one of the zeros past the end)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[v][i] = c.in(v, i >> 2) ? z[v][i] : 0.f;
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] = fmaf(z[v][i], z[v][i], s[0]);
    const uint32_t over = row_sums<LANES, ROWS, 1>(s, lds, turn);
    const float r = row_scale<LANES, ROWS, NV>(s[0], over, [&](int v, int i) { return z[v][i]; }, inv_d, g.eps, lds, turn);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8];
      vec8(w_pre, c, v, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[v][i] = z[v][i] * r * w[i];
      put8((H*)g.y + t * d, c, v, z[v], live);
    }
  }
}

template <typename X, typename H, int LANES, int NV, int THREADS, bool ONCE>
hipError_t run(const NormArgs& g, hipStream_t s) {
  constexpr int ROWS = THREADS / LANES;
  const bool br = g.parts & NORM_BRANCH, pre = g.parts & NORM_PRE;
  void (*f)(NormArgs) = k_norm_fwd<X, H, LANES, NV, THREADS, false, true, 0, ONCE>;
  if (br && pre)
    f = g.act == 0 ? k_norm_fwd<X, H, LANES, NV, THREADS, true, true, 0, ONCE>
        : g.act == NORM_SILU ? k_norm_fwd<X, H, LANES, NV, THREADS, true, true, NORM_SILU, ONCE>
                             : k_norm_fwd<X, H, LANES, NV, THREADS, true, true, NORM_SIGMOID, ONCE>;
  else if (br)
    f = g.act == 0 ? k_norm_fwd<X, H, LANES, NV, THREADS, true, false, 0, ONCE>
        : g.act == NORM_SILU ? k_norm_fwd<X, H, LANES, NV, THREADS, true, false, NORM_SILU, ONCE>
                             : k_norm_fwd<X, H, LANES, NV, THREADS, true, false, NORM_SIGMOID, ONCE>;
  // (a launch holds fewer than 2^32 threads)
  constexpr int64_t MOST = (int64_t)1 << 21;
  for (int64_t t = 0; t < g.T; t += MOST * ROWS) {
    NormArgs a = g;
    a.T = g.T - t < MOST * ROWS ? g.T - t : MOST * ROWS;
    a.x = (const X*)g.x + t * g.d;
    if (br) {
      a.h = (const H*)g.h + t * g.ld_h;
      a.xo = (X*)g.xo + t * g.d;
      if (g.act) a.gate = (const H*)g.gate + t * g.ld_g;
    }
    if (pre) a.y = (H*)g.y + t * g.d;
    hipLaunchKernelGGL(f, dim3((unsigned)((a.T + ROWS - 1) / ROWS)), dim3(THREADS), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The lanes of a row: few enough idle ones, and few enough variants (T = 4096, d = 4160 with 512 lanes 42 us,
// with 320 37; d = 6144 the same with 384 as with 512).
template <typename X, typename H, bool ONCE>
hipError_t pick(const NormArgs& g, hipStream_t s) {
  if (g.d <= 64) return run<X, H, 8, 1, 256, ONCE>(g, s);
  if (g.d <= 128) return run<X, H, 16, 1, 256, ONCE>(g, s);
  if (g.d <= 256) return run<X, H, 32, 1, 256, ONCE>(g, s);
  if (g.d <= 512) return run<X, H, 64, 1, 256, ONCE>(g, s);
  if (g.d <= 1024) return run<X, H, 64, 2, 256, ONCE>(g, s);
  if (g.d <= 1536) return run<X, H, 192, 1, 192, ONCE>(g, s);
  if (g.d <= 2048) return run<X, H, 256, 1, 256, ONCE>(g, s);
  if (g.d <= 2560) return run<X, H, 320, 1, 320, ONCE>(g, s);
  if (g.d <= 4096) return run<X, H, 256, 2, 256, ONCE>(g, s);
  if (g.d <= 5120) return run<X, H, 320, 2, 320, ONCE>(g, s);
  if (g.d <= 8192) return run<X, H, 512, 2, 512, ONCE>(g, s);
  if (g.d <= 12288) return run<X, H, 512, 3, 512, ONCE>(g, s);
  return run<X, H, 512, 4, 512, ONCE>(g, s);
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs& g, hipStream_t s) {
  if (g.x_f32 && g.h_f32) return g.once ? pick<float, float, true>(g, s) : pick<float, float, false>(g, s);
  if (g.x_f32) return g.once ? pick<float, bf16_t, true>(g, s) : pick<float, bf16_t, false>(g, s);
  return g.once ? pick<bf16_t, bf16_t, true>(g, s) : pick<bf16_t, bf16_t, false>(g, s);
}

}  // namespace mapl
