// Softmax cross entropy over the vocabulary, l[t][v] = H[t] . W[v], without
// keeping the logits:
//   forward   lse[t] = log sum_v exp l[t][v], loss[t] = lse[t] - l[t][y_t]
//   backward  dl[t][v] = w_t (exp(l[t][v] - lse[t]) - [v = y_t]),
//             dH = scale dl W, dW (+)= scale dl^T H
// bf16: the products run in big_gemm.hpp's tiles.  The forward's epilogue
// reduces a tile's logits to a maximum and a sum of exponentials per token
// (k_xent_lse), k_xent_join merges them over the vocabulary.  The backward
// takes the vocabulary in pieces: logits again with the epilogue turning them
// into dl (bf16, k_xent_dl), then dl's two products (k_xent_out).  fp32: the
// same steps with the fp32 products' kernels and the logits of one piece in
// the workspace (k_xent_*_f32).
#include "big_gemm.hpp"

namespace mapl {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_inff();

template <class Cfg>
struct XentGrid {
  static constexpr int PER_CU = 2 * 2 * Cfg::STAGE <= 160 * 1024 ? 2 : 1;
};

// reference point of a row's exponentials: its maximum, or 0 where that is
// not finite (exp2(l - 0) then gives 0 for l = -inf, inf for l = inf)
__device__ __forceinline__ float xent_ref(float m) { return __builtin_isfinite(m) ? m : 0.f; }

// C(m, n) = logit of vocabulary entry m, token n.
template <class Cfg>
__global__ __launch_bounds__(Cfg::THREADS) __attribute__((amdgpu_waves_per_eu(Cfg::NW / 4 * XentGrid<Cfg>::PER_CU))) void
k_xent_lse(BgShape g, XentTok a, float2* part, float* tgt) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[2 * Cfg::STAGE];
  bg_run<Cfg>(g, smem, [&](f32x16_t (&acc)[Cfg::FM][Cfg::FN], const BgTile& t, int wm, int wn, int lane) {
    const int m0 = t.m * Cfg::BM + wm * Cfg::FM * 32, half = lane >> 5;
    if (m0 + Cfg::FM * 32 > g.M) {  // past the vocabulary: no logit
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (m0 + 32 * i + acc_row(e, lane) >= g.M)
#pragma unroll
            for (int j = 0; j < Cfg::FN; ++j) acc[i][j][e] = NEG_INF;
    }
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j) {
      const int n = t.n * Cfg::BN + (wn * Cfg::FN + j) * 32 + (lane & 31);
      float mx = NEG_INF;
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, acc[i][j][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, WAVE));
      const float r = -xent_ref(mx) * LOG2E;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, r));
      sum += __shfl_xor(sum, 32, WAVE);
      const int y = n < g.N ? (int)((unsigned)a.y[n] - (unsigned)m0) : -1;
      if (__any((unsigned)y < (unsigned)(Cfg::FM * 32))) {  // a target's logit is here
#pragma unroll
        for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (y == 32 * i + acc_row(e, lane)) tgt[n] = acc[i][j][e];
      }
      if (half == 0 && n < g.N) part[(int64_t)(t.m * Cfg::WVM + wm) * g.N + n] = make_float2(mx, sum);
    }
  });
#endif
}

// lse and loss from `np` partial (maximum, sum) pairs per token; sixteen
// tokens and sixteen runs of partials per workgroup.
__global__ __launch_bounds__(256) void k_xent_join(const float2* __restrict__ part, int np, int T, XentTok a,
                                                   const float* __restrict__ tgt, float* __restrict__ loss,
                                                   float* __restrict__ lse) {
  __shared__ float2 sh[16][17];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int t = blockIdx.x * 16 + tx;
  float m = NEG_INF, s = 0.f;
  if (t < T)
    for (int p = ty; p < np; p += 16) {
      const float2 v = part[(int64_t)p * T + t];
      const float mn = fmaxf(m, v.x), r = xent_ref(mn);
      s = s * __builtin_amdgcn_exp2f((xent_ref(m) - r) * LOG2E) + v.y * __builtin_amdgcn_exp2f((xent_ref(v.x) - r) * LOG2E);
      m = mn;
    }
  sh[ty][tx] = make_float2(m, s);
  __syncthreads();
  if (ty == 0 && t < T) {
    for (int q = 1; q < 16; ++q) m = fmaxf(m, sh[q][tx].x);
    const float r = xent_ref(m);
    s = 0.f;
    for (int q = 0; q < 16; ++q)
      s += sh[q][tx].y * __builtin_amdgcn_exp2f((xent_ref(sh[q][tx].x) - r) * LOG2E);
    const float L = r + logf(s);
    lse[t] = L;
    loss[t] = a.y[t] < 0 ? 0.f : L - tgt[t];
  }
}

// what the backward needs of a token: {lse log2 e, w_t (0 where masked), y, 0};
// and H with the masked tokens' rows as zeros (their values may be anything,
// and 0 times an infinity is no zero).
template <typename V>
__global__ __launch_bounds__(256) void k_xent_prep(const V* __restrict__ H, int T, int cpr, XentTok a,
                                                   const float* __restrict__ lse, float4* __restrict__ tok,
                                                   V* __restrict__ Hm) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t = i / cpr;
  if (t >= T) return;
  const int c = (int)(i - t * cpr);
  const int y = a.y[t];
  const float w = y < 0 ? 0.f : a.weight ? a.weight[t] : 1.f;
  if (c == 0) tok[t] = make_float4(lse[t] * LOG2E, w, __int_as_float(y), 0.f);
  if (Hm) Hm[i] = w != 0.f ? H[i] : V{};
}

// dl (bf16 [T][ld], columns past the piece zero) of the vocabulary piece that
// starts at v0.  C(m, n) as in k_xent_lse.
template <class Cfg>
__global__ __launch_bounds__(Cfg::THREADS) __attribute__((amdgpu_waves_per_eu(Cfg::NW / 4 * XentGrid<Cfg>::PER_CU))) void
k_xent_dl(BgShape g, const float4* __restrict__ tok, int v0, bf16_t* __restrict__ dl, int64_t ld) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[2 * Cfg::STAGE];
  bg_run<Cfg>(g, smem, [&](f32x16_t (&acc)[Cfg::FM][Cfg::FN], const BgTile& t, int wm, int wn, int lane) {
    const int m0 = t.m * Cfg::BM + wm * Cfg::FM * 32, half = lane >> 5;
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j) {
      const int n = t.n * Cfg::BN + (wn * Cfg::FN + j) * 32 + (lane & 31);
      const float4 k = n < g.N ? tok[n] : make_float4(0.f, 0.f, __int_as_float(-1), 0.f);
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, -k.x));
      const int y = (int)((unsigned)__float_as_int(k.z) - (unsigned)(v0 + m0));
      if (__any((unsigned)y < (unsigned)(Cfg::FM * 32))) {
#pragma unroll
        for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (y == 32 * i + acc_row(e, lane)) acc[i][j][e] -= 1.f;
      }
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          acc[i][j][e] = k.y != 0.f && m0 + 32 * i + acc_row(e, lane) < g.M ? acc[i][j][e] * k.y : 0.f;
      if (n < g.N) {
        bf16_t* o = dl + (int64_t)n * ld + m0 + 4 * half;
#pragma unroll
        for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (m0 + 32 * i + 8 * q < ld)
              *(uint2*)(o + 32 * i + 8 * q) = make_uint2(pack_bf2(acc[i][j][4 * q], acc[i][j][4 * q + 1]),
                                                         pack_bf2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
      }
    }
  });
#endif
}

// out[n][m] (+)= scale C(m, n); rows of masked tokens are zeros (tok given).
template <class Cfg>
__global__ __launch_bounds__(Cfg::THREADS) __attribute__((amdgpu_waves_per_eu(Cfg::NW / 4 * XentGrid<Cfg>::PER_CU))) void
k_xent_out(BgShape g, XentOut o) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[2 * Cfg::STAGE];
  bg_run<Cfg>(g, smem, [&](f32x16_t (&acc)[Cfg::FM][Cfg::FN], const BgTile& t, int wm, int wn, int lane) {
    const int m0 = t.m * Cfg::BM + wm * Cfg::FM * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j) {
      const int n = t.n * Cfg::BN + (wn * Cfg::FN + j) * 32 + (lane & 31);
      if (n >= g.N) continue;
      const bool zero = o.tok && o.tok[n].y == 0.f;
      const int64_t at = (int64_t)n * o.ld + m0;
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (m0 + 32 * i + 8 * q >= g.M) continue;
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = zero ? 0.f : o.scale * acc[i][j][4 * q + e];
          const int64_t x = at + 32 * i + 8 * q;
          if (o.f32) {
            float4* p = (float4*)((float*)o.out + t.split * o.split_stride + x);
            if (o.add) {
              const float4 b = *p;
              v[0] += b.x; v[1] += b.y; v[2] += b.z; v[3] += b.w;
            }
            *p = make_float4(v[0], v[1], v[2], v[3]);
          } else {
            uint2* p = (uint2*)((bf16_t*)o.out + x);
            if (o.add) {
              const uint2 b = *p;
              v[0] += bf2f(b.x & 0xFFFFu); v[1] += bf2f(b.x >> 16);
              v[2] += bf2f(b.y & 0xFFFFu); v[3] += bf2f(b.y >> 16);
            }
            *p = make_uint2(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]));
          }
        }
    }
  });
#endif
}

// dH[t] = bf16(scale sum_s part[s][t]) in the order of s, zeros for masked tokens.
__global__ __launch_bounds__(256) void k_xent_sum(const float4* __restrict__ part, int splits, int64_t n4, int cpr,
                                                  const float4* __restrict__ tok, float scale,
                                                  uint2* __restrict__ dH) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n4) return;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (tok[i / cpr].y != 0.f) {
    for (int s = 0; s < splits; ++s) {
      const float4 p = part[s * n4 + i];
      v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
    }
  }
  dH[i] = make_uint2(pack_bf2(scale * v.x, scale * v.y), pack_bf2(scale * v.z, scale * v.w));
}

// ------------------------------------------------------------------- fp32
// One token per workgroup, the logits of a vocabulary piece in a row of `ld`.
__device__ __forceinline__ float block_max(float v, float* sh) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* sh) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (sh[0] + sh[1]) + (sh[2] + sh[3]);
  __syncthreads();
  return v;
}

__global__ __launch_bounds__(256) void k_xent_lse_f32(const float* __restrict__ l, int64_t ld, int n, int v0, XentTok a,
                                                      float2* __restrict__ part, float* __restrict__ tgt) {
  __shared__ float sh[4];
  const int t = blockIdx.x;
  const float* row = l + t * ld;
  float m = NEG_INF;
  for (int v = threadIdx.x; v < n; v += 256) m = fmaxf(m, row[v]);
  m = block_max(m, sh);
  const float r = xent_ref(m);
  float s = 0.f;
  for (int v = threadIdx.x; v < n; v += 256) s += expf(row[v] - r);
  s = block_sum(s, sh);
  if (threadIdx.x == 0) {
    part[t] = make_float2(m, s);
    const int y = a.y[t];
    if (y >= v0 && y - v0 < n) tgt[t] = row[y - v0];
  }
}

__global__ __launch_bounds__(256) void k_xent_dl_f32(float* __restrict__ l, int64_t ld, int n, int v0,
                                                     const float* __restrict__ lse, XentTok a, float scale) {
  const int t = blockIdx.x;
  float* row = l + t * ld;
  const int y = a.y[t];
  const float w = y < 0 ? 0.f : a.weight ? a.weight[t] : 1.f;
  const float L = lse[t];
  for (int v = threadIdx.x; v < ld; v += 256) {
    const float p = v < n ? expf(row[v] - L) - (y >= v0 && v == y - v0 ? 1.f : 0.f) : 0.f;
    row[v] = w != 0.f && v < n ? scale * (w * p) : 0.f;
  }
}

// the rows of masked tokens set to zero (0 times an infinite weight row is no zero)
__global__ __launch_bounds__(256) void k_xent_zero_rows(float4* __restrict__ X, int64_t n4, int cpr, XentTok a) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n4) return;
  const int64_t t = i / cpr;
  if (a.y[t] < 0 || (a.weight && a.weight[t] == 0.f)) X[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}

// bit 0 of flag: a target at or past V
__global__ void k_xent_check(const int32_t* __restrict__ y, int T, int64_t V, int* flag) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t < T && y[t] >= V) *flag = 1;
}

using Big_cc = BgCfg<2, 4, 4, 2, false, false>;
using Big_tc = BgCfg<2, 4, 4, 2, true, false>;
using Big_tt = BgCfg<2, 4, 4, 2, true, true>;
using Mid_cc = BgCfg<2, 2, 2, 2, false, false>;
using Mid_tc = BgCfg<2, 2, 2, 2, true, false>;
using Mid_tt = BgCfg<2, 2, 2, 2, true, true>;

template <class Cfg>
BgShape shape(const XentGemm& q) {
  BgShape g{};
  g.P = {q.P, q.ldp};
  g.Q = {q.Q, q.ldq};
  g.M = q.M;
  g.N = q.N;
  g.K = q.K;
  g.kper = q.kper > 0 ? q.kper : (q.K + 63) / 64 * 64;
  g.splits = (int)((q.K + g.kper - 1) / g.kper);
  g.mt = (q.M + Cfg::BM - 1) / Cfg::BM;
  g.nt = (q.N + Cfg::BN - 1) / Cfg::BN;
  return g;
}
template <class Cfg>
dim3 grid(const BgShape& g) {
  const int items = g.mt * g.nt * g.splits, most = 256 * XentGrid<Cfg>::PER_CU;
  return dim3(items < most ? (items + 7) / 8 * 8 : most);
}
bool fits(const XentGemm& q) {
  return q.M > 0 && q.N > 0 && q.K > 0 && q.ldp % 8 == 0 && q.ldq % 8 == 0 && q.ldp <= (1 << 21) && q.ldq <= (1 << 21) &&
         q.kper % 64 == 0;
}

}  // namespace

bool xent_big_tiles(int64_t M, int64_t N, int64_t splits) {
  return (M + 255) / 256 * ((N + 255) / 256) * splits >= 256;
}

int xent_partials(int64_t V, int64_t T) { return (int)(xent_big_tiles(V, T, 1) ? 2 * ((V + 255) / 256) : 2 * ((V + 127) / 128)); }

hipError_t launch_xent_lse(const XentGemm& q, const XentTok& a, float* part, float* tgt, hipStream_t s) {
  if (!fits(q) || q.K % 64) return hipErrorInvalidValue;
  if (xent_big_tiles(q.M, q.N, 1)) {
    const BgShape g = shape<Big_cc>(q);
    hipLaunchKernelGGL(k_xent_lse<Big_cc>, grid<Big_cc>(g), dim3(Big_cc::THREADS), 0, s, g, a, (float2*)part, tgt);
  } else {
    const BgShape g = shape<Mid_cc>(q);
    hipLaunchKernelGGL(k_xent_lse<Mid_cc>, grid<Mid_cc>(g), dim3(Mid_cc::THREADS), 0, s, g, a, (float2*)part, tgt);
  }
  return hipGetLastError();
}

hipError_t launch_xent_join(const float* part, int np, int T, const XentTok& a, const float* tgt, float* loss, float* lse,
                            hipStream_t s) {
  hipLaunchKernelGGL(k_xent_join, dim3((T + 15) / 16), dim3(256), 0, s, (const float2*)part, np, T, a, tgt, loss, lse);
  return hipGetLastError();
}

hipError_t launch_xent_prep(const void* H, int esize, int T, int d, const XentTok& a, const float* lse, float* tok, void* Hm,
                            hipStream_t s) {
  const int cpr = d * esize / 16;
  const int64_t n = (int64_t)T * cpr;
  hipLaunchKernelGGL(k_xent_prep<uint4>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, (const uint4*)H, T, cpr, a,
                     lse, (float4*)tok, (uint4*)Hm);
  return hipGetLastError();
}

hipError_t launch_xent_dl(const XentGemm& q, const float* tok, int v0, bf16_t* dl, int64_t ld, hipStream_t s) {
  if (!fits(q) || q.K % 64) return hipErrorInvalidValue;
  if (xent_big_tiles(q.M, q.N, 1)) {
    const BgShape g = shape<Big_cc>(q);
    hipLaunchKernelGGL(k_xent_dl<Big_cc>, grid<Big_cc>(g), dim3(Big_cc::THREADS), 0, s, g, (const float4*)tok, v0, dl, ld);
  } else {
    const BgShape g = shape<Mid_cc>(q);
    hipLaunchKernelGGL(k_xent_dl<Mid_cc>, grid<Mid_cc>(g), dim3(Mid_cc::THREADS), 0, s, g, (const float4*)tok, v0, dl, ld);
  }
  return hipGetLastError();
}

hipError_t launch_xent_out(const XentGemm& q, int q_along_rows, const XentOut& o, hipStream_t s) {
  if (!fits(q) || q.M % 64) return hipErrorInvalidValue;
  const int64_t splits = q.kper > 0 ? (q.K + q.kper - 1) / q.kper : 1;
  if (splits > 1 && !o.f32) return hipErrorInvalidValue;
  const bool big = xent_big_tiles(q.M, q.N, splits);
#define MAPL_XENT_OUT(C)                                                                          \
  do {                                                                                            \
    const BgShape g = shape<C>(q);                                                                \
    hipLaunchKernelGGL(k_xent_out<C>, grid<C>(g), dim3(C::THREADS), 0, s, g, o);                  \
  } while (0)
  if (q_along_rows) {
    if (big) MAPL_XENT_OUT(Big_tt); else MAPL_XENT_OUT(Mid_tt);
  } else {
    if (big) MAPL_XENT_OUT(Big_tc); else MAPL_XENT_OUT(Mid_tc);
  }
#undef MAPL_XENT_OUT
  return hipGetLastError();
}

hipError_t launch_xent_sum(const float* part, int splits, int T, int d, const float* tok, float scale, bf16_t* dH,
                           hipStream_t s) {
  const int64_t n4 = (int64_t)T * d / 4;
  hipLaunchKernelGGL(k_xent_sum, dim3((unsigned)((n4 + 255) / 256)), dim3(256), 0, s, (const float4*)part, splits, n4, d / 4,
                     (const float4*)tok, scale, (uint2*)dH);
  return hipGetLastError();
}

hipError_t launch_xent_lse_f32(const float* l, int64_t ld, int T, int n, int v0, const XentTok& a, float* part, float* tgt,
                               hipStream_t s) {
  hipLaunchKernelGGL(k_xent_lse_f32, dim3(T), dim3(256), 0, s, l, ld, n, v0, a, (float2*)part, tgt);
  return hipGetLastError();
}

hipError_t launch_xent_dl_f32(float* l, int64_t ld, int T, int n, int v0, const float* lse, const XentTok& a, float scale,
                              hipStream_t s) {
  hipLaunchKernelGGL(k_xent_dl_f32, dim3(T), dim3(256), 0, s, l, ld, n, v0, lse, a, scale);
  return hipGetLastError();
}

hipError_t launch_xent_zero_rows(float* X, int T, int d, const XentTok& a, hipStream_t s) {
  const int64_t n4 = (int64_t)T * d / 4;
  hipLaunchKernelGGL(k_xent_zero_rows, dim3((unsigned)((n4 + 255) / 256)), dim3(256), 0, s, (float4*)X, n4, d / 4, a);
  return hipGetLastError();
}

hipError_t launch_xent_check(const int32_t* y, int T, int64_t V, int* flag, hipStream_t s) {
  hipLaunchKernelGGL(k_xent_check, dim3((T + 255) / 256), dim3(256), 0, s, y, T, V, flag);
  return hipGetLastError();
}

}  // namespace mapl
