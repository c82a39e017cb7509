// The norms around a block of a stage, with the block's gate and residual
// scale: for every token (row of d values)
//   n  = h r_h w_post, r_h = (mean h^2 + eps)^-1/2       (with NORM_POST; else n = h)
//   x' = x + alpha s (n act(G))                          (with NORM_BRANCH; else x' = x)
//   y  = x' r_x w_pre, r_x = (mean x'^2 + eps)^-1/2      (with NORM_PRE)
// in one pass, x' rounded to its type before y is computed from it, and the
// gradient with respect to x, h, G and the three vectors, in one pass and a sum
// over the workgroups' parts of the vectors' gradients.  The backward computes
// r_h and r_x again from the rows that it reads anyway: nothing is kept for it.
// Sums, statistics and everything in between are fp32.
//
// Bound by HBM: 10 bytes a value forward, 16 backward where everything is bf16.
#include "common.hpp"
#include "kernels.hpp"

namespace mapl {

namespace {

// eight consecutive values as they lie in memory
template <typename X>
struct Oct;
template <>
struct Oct<bf16_t> {
  u32x4 w;
  __device__ void load(const bf16_t* p) { w = *(const u32x4*)p; }
  __device__ void zero() { w = u32x4{0, 0, 0, 0}; }
  __device__ float get(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
};
template <>
struct Oct<float> {
  f32x4_t a, b;
  __device__ void load(const float* p) { a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 4); }
  __device__ void zero() { a = b = f32x4_t{0, 0, 0, 0}; }
  __device__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};
// (rounds v to what memory holds)
__device__ __forceinline__ void store8(bf16_t* p, float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = pack_bf2(v[2 * i], v[2 * i + 1]);
    v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  *(u32x4*)p = w;
}
__device__ __forceinline__ void store8(float* p, float (&v)[8]) {
  *(f32x4_t*)p = f32x4_t{v[0], v[1], v[2], v[3]};
  *(f32x4_t*)(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); }

// The sums of v over the LANES lanes of a row, in every one of them.  A row of
// more than a wave meets in LDS: two areas in turn, so that one barrier a sum
// does (the one of the next sum lies between an area's reads and its next writes).
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* lds, int& turn) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    v[n] = dpp_add<0xB1>(v[n]);   // lane ^ 1
    v[n] = dpp_add<0x4E>(v[n]);   // lane ^ 2
    v[n] = dpp_add<0x141>(v[n]);  // the other half of 8
    v[n] = dpp_add<0x140>(v[n]);  // the other half of 16
    if constexpr (LANES == 32) v[n] += __shfl_xor(v[n], 16, WAVE);
    if constexpr (LANES >= 64) v[n] = (lane_of(v[n], 0) + lane_of(v[n], 16)) + (lane_of(v[n], 32) + lane_of(v[n], 48));
  }
  if constexpr (LANES > 64) {
    constexpr int W = LANES / 64;
    float* a = lds + turn * 4 * W;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) a[n * W + (threadIdx.x >> 6)] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += a[n * W + w];
      v[n] = s;
    }
    turn ^= 1;
  }
}

// (mean z^2 + eps)^-1/2 from ss = sum z^2.  Where that overflows (a row whose size
// is past 1e18) the sum is taken again 2^-80 times smaller: no term is then past
// 2^96, and what falls out at the low end is 2^-40 of the largest.
template <int LANES, int NV>
__device__ __forceinline__ float row_scale(float ss, const float (&z)[NV][8], float inv_d, float eps, float* lds, int& turn) {
  if (!(ss < 1e38f)) {
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = z[v][i] * 0x1p-80f;
        s[0] = fmaf(q, q, s[0]);
      }
    row_sums<LANES, 1>(s, lds, turn);
    return 0x1p-80f / sqrtf(s[0] * inv_d);
  }
  return 1.f / sqrtf(fmaf(ss, inv_d, eps));
}

// sigmoid(g) and 1 - sigmoid(g), both to the last digits at either end
__device__ __forceinline__ void sigmoid2(float g, float& a, float& b) {
  const float e = expf(-fabsf(g)), r = 1.f / (1.f + e), q = e * r;
  a = g >= 0.f ? r : q;
  b = g >= 0.f ? q : r;
  if (g != g) a = b = g;
}
__device__ __forceinline__ float act_of(float g, int kind) {
  float a, b;
  sigmoid2(g, a, b);
  return kind == NORM_SILU ? g * a : a;
}
__device__ __forceinline__ void act_both(float g, int kind, float& f, float& df) {
  float a, b;
  sigmoid2(g, a, b);
  f = kind == NORM_SILU ? g * a : a;
  df = kind == NORM_SILU ? a * fmaf(g, b, 1.f) : a * b;
}

// column of the lane's v-th run of eight
template <int LANES>
__device__ __forceinline__ int col(int lane, int v) { return (v * LANES + lane) * 8; }

__device__ __forceinline__ void load_vec(const float* w, int c, float (&f)[8]) {
  const f32x4_t a = *(const f32x4_t*)(w + c), b = *(const f32x4_t*)(w + c + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
}

// A row is held by LANES lanes, eight consecutive values NV times each; a workgroup
// of THREADS takes THREADS / LANES rows at a time.
template <typename X, typename H, int LANES, int NV, bool BRANCH, bool PRE>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_norm_fwd(const NormArgs g) {
  constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
  __shared__ float lds[2 * 4 * (LANES > 64 ? LANES / 64 : 1)];
  int turn = 0;
  const int lane = threadIdx.x % LANES, d = g.d;
  const float inv_d = 1.f / (float)d;
  const bool post = g.parts & NORM_POST;
  for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; t < g.T; t += (int64_t)gridDim.x * ROWS) {
    Oct<X> x[NV];
    Oct<H> h[NV], u[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = col<LANES>(lane, v);
      if (c < d) {
        x[v].load((const X*)g.x + t * d + c);
        if constexpr (BRANCH) {
          h[v].load((const H*)g.h + t * g.ld_h + c);
          if (g.gate) u[v].load((const H*)g.gate + t * g.ld_g + c);
        }
      } else {
        x[v].zero(), h[v].zero(), u[v].zero();
      }
    }
    float z[NV][8];
    if constexpr (BRANCH) {
      float r = 1.f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[v][i] = h[v].get(i);
      if (post) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) s[0] = fmaf(z[v][i], z[v][i], s[0]);
        row_sums<LANES, 1>(s, lds, turn);
        r = row_scale<LANES, NV>(s[0], z, inv_d, g.eps, lds, turn);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
        if (c < d) {
          float w[8];
          if (post && g.w_post) {
            load_vec(g.w_post, c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] = z[v][i] * r * w[i];
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] *= r;
          }
          if (g.gate)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] *= act_of(u[v].get(i), g.act);
          if (g.scale) {
            load_vec(g.scale, c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] = fmaf(g.alpha * w[i], z[v][i], x[v].get(i));
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] = fmaf(g.alpha, z[v][i], x[v].get(i));
          }
          store8((X*)g.xo + t * d + c, z[v]);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[v][i] = x[v].get(i);
    }
    if constexpr (PRE) {
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(z[v][i], z[v][i], s[0]);
      row_sums<LANES, 1>(s, lds, turn);
      const float r = row_scale<LANES, NV>(s[0], z, inv_d, g.eps, lds, turn);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
        if (c < d) {
          if (g.w_pre) {
            float w[8];
            load_vec(g.w_pre, c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] = z[v][i] * r * w[i];
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] *= r;
          }
          store8((H*)g.y + t * d + c, z[v]);
        }
      }
    }
  }
}

// dX = dx' + r_x (dy w_pre - x' r_x^2 mean(dy w_pre x')), then with dX
//   dn = alpha s dX act, dh = r_h (dn w_post - h r_h^2 mean(dn w_post h)), dG = alpha s dX n act'
// and the lane's columns of dw_pre = sum dy x' r_x, ds = sum alpha dX n act,
// dw_post = sum dn h r_h over the workgroup's rows, summed over its groups of
// lanes in LDS and left in part[workgroup][3][d] (dw_post, ds, dw_pre).
template <typename X, typename H, int LANES, int NV, bool BRANCH, bool PRE>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_norm_bwd(const NormArgs g) {
  constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
  constexpr int NS = (BRANCH ? 2 : 0) + (PRE ? 1 : 0), S0 = BRANCH ? 0 : 2;  // sums: dw_post, ds, dw_pre
  __shared__ float lds[2 * 4 * (LANES > 64 ? LANES / 64 : 1)];
  __shared__ float red[ROWS > 1 ? NS * LANES * NV * 8 : 1];
  int turn = 0;
  const int lane = threadIdx.x % LANES, d = g.d;
  const float inv_d = 1.f / (float)d;
  const bool post = g.parts & NORM_POST;
  float acc[NS][NV][8];
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[j][v][i] = 0.f;

  for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; t < g.T; t += (int64_t)gridDim.x * ROWS) {
    Oct<X> x[NV], dxo[NV];
    Oct<H> dy[NV], h[NV], u[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = col<LANES>(lane, v);
      x[v].zero(), dxo[v].zero(), dy[v].zero(), h[v].zero(), u[v].zero();
      if (c < d) {
        if constexpr (PRE) {
          x[v].load((const X*)g.x + t * d + c);
          dy[v].load((const H*)g.dy + t * d + c);
        }
        if (g.dxo) dxo[v].load((const X*)g.dxo + t * d + c);
        if constexpr (BRANCH) {
          h[v].load((const H*)g.h + t * g.ld_h + c);
          if (g.gate) u[v].load((const H*)g.gate + t * g.ld_g + c);
        }
      }
    }
    // the sums that need nothing but the inputs, at once
    float s[3] = {0.f, 0.f, 0.f};
    float z[NV][8], q[NV][8];
    if constexpr (PRE) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
        float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (c < d && g.w_pre) load_vec(g.w_pre, c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          z[v][i] = x[v].get(i);
          q[v][i] = dy[v].get(i) * w[i];
          s[0] = fmaf(z[v][i], z[v][i], s[0]);
          s[1] = fmaf(q[v][i], z[v][i], s[1]);
        }
      }
    }
    float y[NV][8];
    if constexpr (BRANCH) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[v][i] = h[v].get(i);
          s[2] = fmaf(y[v][i], y[v][i], s[2]);
        }
    }
    row_sums<LANES, 3>(s, lds, turn);
    // dX in q
    if constexpr (PRE) {
      const float r = row_scale<LANES, NV>(s[0], z, inv_d, g.eps, lds, turn);
      const float k = r * (r * (s[1] * inv_d));
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          acc[2 - S0][v][i] = fmaf(dy[v].get(i) * r, z[v][i], acc[2 - S0][v][i]);
          q[v][i] = fmaf(r, fmaf(-z[v][i], k, q[v][i]), dxo[v].get(i));
        }
        if (c < d) {
          float o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = q[v][i];
          store8((X*)g.dx + t * d + c, o);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) q[v][i] = dxo[v].get(i);
    }
    if constexpr (BRANCH) {
      const float r = post ? row_scale<LANES, NV>(s[2], y, inv_d, g.eps, lds, turn) : 1.f;
      float sh[1] = {0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
        float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, sc[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (c < d && post && g.w_post) load_vec(g.w_post, c, w);
        if (c < d && g.scale) load_vec(g.scale, c, sc);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float n0 = y[v][i] * r, n = n0 * w[i], e = g.alpha * q[v][i];
          float f = 1.f, df = 0.f;
          if (g.gate) act_both(u[v].get(i), g.act, f, df);
          acc[1][v][i] = fmaf(e, n * f, acc[1][v][i]);
          const float dt = e * sc[i];
          o[i] = dt * n * df;
          const float dn = dt * f;
          acc[0][v][i] = fmaf(dn, n0, acc[0][v][i]);
          q[v][i] = dn * w[i];
          sh[0] = fmaf(q[v][i], y[v][i], sh[0]);
        }
        if (c < d && g.gate) store8((H*)g.dgate + t * g.ld_g + c, o);
      }
      if (post) {
        row_sums<LANES, 1>(sh, lds, turn);
        const float k = r * (r * (sh[0] * inv_d));
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) q[v][i] = r * fmaf(-y[v][i], k, q[v][i]);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
        if (c < d) store8((H*)g.dh + t * g.ld_h + c, q[v]);
      }
    }
  }
  if (!g.part) return;
  float* part = g.part + (int64_t)blockIdx.x * 3 * d;
  if constexpr (ROWS > 1) {
    for (int k = 0; k < ROWS; ++k) {
      __syncthreads();
      if ((int)threadIdx.x / LANES == k)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            float* p = red + j * LANES * NV * 8 + col<LANES>(lane, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = k ? p[i] + acc[j][v][i] : acc[j][v][i];
          }
    }
    __syncthreads();
    for (int j = 0; j < NS; ++j)
      for (int c = threadIdx.x; c < d; c += THREADS) part[(j + S0) * d + c] = red[j * LANES * NV * 8 + c];
  } else {
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = col<LANES>(lane, v);
        if (c < d) store8(part + (j + S0) * d + c, acc[j][v]);
      }
  }
}

// out[j][c] (+)= sum over the workgroups' parts in a fixed order; 16 runs of them
// side by side for 64 columns.
__global__ __launch_bounds__(1024) void k_norm_sum(const float* __restrict__ part, int n, int d, NormSums o, int add) {
  __shared__ float red[16][64];
  const int j = blockIdx.y, c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
  float* out = j == 0 ? o.dw_post : j == 1 ? o.dscale : o.dw_pre;
  if (!out) return;
  float s = 0.f;
  const float* p = part + (int64_t)j * d + c;
#pragma unroll 8
  for (int i = k; i < n; i += 16) s += p[(int64_t)i * 3 * d];
  red[k][threadIdx.x & 63] = s;
  __syncthreads();
  if (k == 0) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i][threadIdx.x];
    out[c] = add ? out[c] + s : s;
  }
}

// (no output of T rows, but sums to give: zeros unless they are added to)
template <typename X, typename H, int LANES, int NV>
hipError_t run(const NormArgs& g, bool bwd, int wgs, hipStream_t s) {
  constexpr int THREADS = LANES > 256 ? LANES : 256;
  const bool br = g.parts & NORM_BRANCH, pre = g.parts & NORM_PRE;
  void (*f)(NormArgs);
  if (bwd)
    f = br ? pre ? k_norm_bwd<X, H, LANES, NV, true, true> : k_norm_bwd<X, H, LANES, NV, true, false> : k_norm_bwd<X, H, LANES, NV, false, true>;
  else
    f = br ? pre ? k_norm_fwd<X, H, LANES, NV, true, true> : k_norm_fwd<X, H, LANES, NV, true, false> : k_norm_fwd<X, H, LANES, NV, false, true>;
  hipLaunchKernelGGL(f, dim3(wgs), dim3(THREADS), 0, s, g);
  return hipGetLastError();
}

template <typename X, typename H>
hipError_t pick(const NormArgs& g, bool bwd, int wgs, hipStream_t s) {
  if (g.d <= 128) return run<X, H, 16, 1>(g, bwd, wgs, s);
  if (g.d <= 256) return run<X, H, 32, 1>(g, bwd, wgs, s);
  if (g.d <= 512) return run<X, H, 64, 1>(g, bwd, wgs, s);
  if (g.d <= 1024) return run<X, H, 64, 2>(g, bwd, wgs, s);
  if (g.d <= 2048) return run<X, H, 256, 1>(g, bwd, wgs, s);
  if (g.d <= 4096) return run<X, H, 256, 2>(g, bwd, wgs, s);
  if (g.d <= 8192) return run<X, H, 512, 2>(g, bwd, wgs, s);
  return run<X, H, 1024, 2>(g, bwd, wgs, s);
}

int rows_per_wg(int d) { return d <= 128 ? 16 : d <= 256 ? 8 : d <= 1024 ? 4 : 1; }

hipError_t launch(const NormArgs& g, bool bwd, int wgs, hipStream_t s) {
  if (g.x_f32) return g.h_f32 ? pick<float, float>(g, bwd, wgs, s) : pick<float, bf16_t>(g, bwd, wgs, s);
  return pick<bf16_t, bf16_t>(g, bwd, wgs, s);
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs& g, hipStream_t s) {
  const int64_t w = (g.T + rows_per_wg(g.d) - 1) / rows_per_wg(g.d);
  return launch(g, false, (int)(w < 2048 ? w : 2048), s);
}

int norm_bwd_parts(int64_t T, int d) {
  const int64_t w = (T + rows_per_wg(d) - 1) / rows_per_wg(d);
  return (int)(w < 512 ? w : 512);
}

hipError_t launch_norm_bwd(const NormArgs& g, hipStream_t s) { return launch(g, true, norm_bwd_parts(g.T, g.d), s); }

hipError_t launch_norm_sum(const float* part, int n, int d, const NormSums& o, int add, hipStream_t s) {
  hipLaunchKernelGGL(k_norm_sum, dim3(d / 64, 3), dim3(1024), 0, s, part, n, d, o, add);
  return hipGetLastError();
}

}  // namespace mapl
