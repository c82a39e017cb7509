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
  static constexpr int PER_CU = 2 * Cfg::SMEM <= 160 * 1024 ? 2 : 1;
};
#define XENT_KERNEL(C) \
  __global__ __launch_bounds__(C::THREADS) __attribute__((amdgpu_waves_per_eu(C::NW / 4 * XentGrid<C>::PER_CU))) void

// reference point of a row's exponentials: its maximum, or 0 where that is
// not finite (exp2(l - 0) then gives 0 for l = -inf, inf for l = inf)
__device__ __forceinline__ float xent_ref(float m) { return __builtin_isfinite(m) ? m : 0.f; }

// exp(x - ref) is one fma and an exp2, exp2(x log2 e - ref log2 e), whose rounded
// product ref log2 e is off by up to |ref| 2^-24 (and overflows at the type's end).  Up
// to this |ref| that is 2^-14 at most, as much as the rounding of a log-sum-exp of that
// size; past it the difference x - ref is taken first.
constexpr float XENT_FAR = 1024.f;

// what a sum of exponentials relative to its maximum m counts for relative to
// r: nothing if there was no logit above -inf (exp(0 - r) may be infinite, and 0
// times that is no zero)
__device__ __forceinline__ float xent_rel(float m, float r) {
  return m == NEG_INF ? 0.f : __builtin_amdgcn_exp2f((xent_ref(m) - r) * LOG2E);
}

// The lane's number as the epilogues take it: opaque, so that what follows from
// it is computed there and not held in registers through the K loop.
__device__ __forceinline__ int xent_lane() {
  int l = threadIdx.x & 63;
  asm volatile("" : "+v"(l));
  return l;
}

// Every accumulator (i, e) of a lane, m = m0 + 16 i + 4 (lane / 16) + e, by
// compile-time numbers.  (The target and the end of the vocabulary are compared
// with 16 i + e, the lane's part on their side: those are immediates, the sums would be a
// register each.)
template <int FM, typename F>
__device__ __forceinline__ void xent_each(F&& f) {
  static_for<0, 4 * FM>([&](auto xc) {
    constexpr int X = decltype(xc)::value;
    f(std::integral_constant<int, X / 4>{}, std::integral_constant<int, X % 4>{});
  });
}
// f(i, e, it lies at or past m0 + end)
template <int FM, typename F>
__device__ __forceinline__ void xent_from(int end, int lane, F&& f) {
  end -= 4 * (lane >> 4);
  xent_each<FM>([&](auto i, auto e) { f(i, e, 16 * i + e >= end); });
}

// C(m, n) = logit of vocabulary entry m, token n.  A wave reduces its 16 FM
// vocabulary entries of each token in registers (the four lanes that share a
// token meet by shuffles); the pair goes to part.  Bound by the products
// (T = 32768, d = 2048, V = 32003 2.89 to 3.03 ms by the card, 1.49 to 1.42 PFLOP/s), with
// few tokens by W's bytes (T = 37, V = 32000 24 us, 5.5 TB/s).
template <class Cfg>
XENT_KERNEL(Cfg) k_xent_lse(BgShape g, XentTok a, float2* part, float* tgt) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[Cfg::SMEM];
  constexpr int FM = Cfg::FM, FN = Cfg::FN;
  bg_run<Cfg>(
      g, smem, [](const BgTile&, int, int) {},
      [&](f32x4_t (&acc)[FM][FN], const BgTile& t, int wm, int wn) {
        const int lane = xent_lane();
        const int m0 = t.m * Cfg::BM + 16 * wm * FM;
        int ys[FN];  // used after a j's sums: the loads' time is theirs
#pragma unroll
        for (int j = 0; j < FN; ++j)
          ys[j] = a.y[min(t.n * Cfg::BN + 16 * (wn * FN + j) + (lane & 15), g.N - 1)];
        const bool edge = m0 + 16 * FM > g.M;  // past the vocabulary: no logit
        static_for<0, FN>([&](auto j) {
          const int n = t.n * Cfg::BN + 16 * (wn * FN + j) + (lane & 15);
          float x[4 * FM];
          xent_each<FM>([&](auto i, auto e) {
            float& v = x[4 * i + e];
            v = acc[i][j][decltype(e)::value];
            // taken from the accumulators here: two uses of them below would
            // have the compiler move them between register files in the K loop
            asm volatile("" : "+v"(v));
          });
          if (edge) xent_from<FM>(g.M - m0, lane, [&](auto i, auto e, bool past) { x[4 * i + e] = past ? NEG_INF : x[4 * i + e]; });
          float mx = NEG_INF;
          xent_each<FM>([&](auto i, auto e) {
            if constexpr (decltype(e)::value % 2 == 0) mx = fmaxf(fmaxf(x[4 * i + e], x[4 * i + e + 1]), mx);
          });
          mx = fmaxf(mx, __shfl_xor(mx, 16, WAVE));
          mx = fmaxf(mx, __shfl_xor(mx, 32, WAVE));
          const float ref = xent_ref(mx);
          const bool far = fabsf(ref) > XENT_FAR;
          const float r = far ? 0.f : -ref * LOG2E;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
          if (__any(far)) {  // (masked runs of the vocabulary; a near token's values are those of the other branch)
            const float c = far ? ref : 0.f;
            xent_each<FM>([&](auto i, auto e) { sum[e] += __builtin_amdgcn_exp2f(fmaf(x[4 * i + e] - c, LOG2E, r)); });
          } else {
            xent_each<FM>([&](auto i, auto e) { sum[e] += __builtin_amdgcn_exp2f(fmaf(x[4 * i + e], LOG2E, r)); });
          }
          float s = (sum[0] + sum[1]) + (sum[2] + sum[3]);
          s += __shfl_xor(s, 16, WAVE);
          s += __shfl_xor(s, 32, WAVE);
          const int y = (int)((unsigned)ys[j] - (unsigned)m0);
          if (__any((unsigned)y < 16u * FM)) {  // a target's logit is here
            float v = 0.f;
            xent_each<FM>([&](auto i, auto e) { v = y - 4 * (lane >> 4) == 16 * i + e ? x[4 * i + e] : v; });
            if (n < g.N && (unsigned)y < 16u * FM && ((y >> 2) & 3) == lane >> 4) tgt[n] = v;
          }
          if (lane < 16 && n < g.N) part[(int64_t)(t.m * Cfg::WVM + wm) * g.N + n] = make_float2(mx, s);
          __builtin_amdgcn_sched_barrier(0);  // one j's values at a time in registers
        });
      });
#endif
}

// lse and loss from `np` partial (maximum, sum) pairs per token: TX tokens and
// 256 / TX runs of partials per workgroup, four pairs requested at a time.
// TX = 16 reads whole lines; with few tokens TX = 4 has four times the loads in
// flight (V = 32000, by events around the launch: 37 tokens 14 -> 7 us, 1021 tokens 10.5 -> 7.0;
// 2047 tokens 6.6 with TX = 16, 9.7 with 4).
template <int TX>
__global__ __launch_bounds__(256) void k_xent_join(const float2* __restrict__ part, int np, int T, XentTok a,
                                                   const float* __restrict__ tgt, float* __restrict__ loss,
                                                   float* __restrict__ lse) {
  constexpr int RUNS = 256 / TX, U = 4;
  __shared__ float2 sh[RUNS][TX + 1];
  const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
  const int t = blockIdx.x * TX + tx;
  float m = NEG_INF, s = 0.f;
  for (int p0 = ty; p0 < np; p0 += RUNS * U) {
    float2 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + u * RUNS;
      v[u] = t < T && p < np ? part[(int64_t)p * T + t] : make_float2(NEG_INF, 0.f);
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, v[u].x);
    const float r = xent_ref(mn);
    s *= xent_rel(m, r);
#pragma unroll
    for (int u = 0; u < U; ++u) s += v[u].y * xent_rel(v[u].x, r);
    m = mn;
  }
  sh[ty][tx] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x < TX && t < T) {
    for (int q = 1; q < RUNS; ++q) m = fmaxf(m, sh[q][tx].x);
    const float r = xent_ref(m);
    s = 0.f;
    for (int q = 0; q < RUNS; ++q) s += sh[q][tx].y * xent_rel(sh[q][tx].x, r);
    const float L = r + logf(s);
    lse[t] = L;
    loss[t] = a.y[t] < 0 ? 0.f : L - tgt[t];
  }
}

constexpr int XENT_NEG = 1 << 24;  // above any vocabulary entry
constexpr int XENT_RAW = 1 << 25;

// What the backward needs of a token: tok = {lse log2 e - log2 w, y}, so that
// exp2(l log2 e - .x) is w exp(l - lse); y is -1 where the token is masked (or
// w is 0), and where w is negative (.x without w) XENT_NEG is added to it.  A
// token with |lse| past XENT_FAR has .x = lse, and XENT_RAW + XENT_NEG added to y.  And
// H with the masked tokens' rows as zeros (their values may be anything, and 0 times an
// infinity is no zero).  Bound by HBM: [32768, 2048] 268 MB in 45 us, 6 TB/s.
__global__ __launch_bounds__(256) void k_xent_prep(const uint4* __restrict__ H, int T, int cpr, XentTok a,
                                                   const float* __restrict__ lse, float2* __restrict__ tok,
                                                   uint4* __restrict__ Hm) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)T * cpr; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / cpr;
    const int c = (int)(i - t * cpr);
    const int y = a.y[t];
    const float w = y < 0 ? 0.f : a.weight ? a.weight[t] : 1.f;
    if (c == 0) {  // (a target past any vocabulary stays below XENT_NEG)
      const float L = lse[t];
      const bool far = fabsf(L) > XENT_FAR;
      tok[t] = make_float2(far ? L : L * LOG2E - (w > 0.f ? log2f(w) : 0.f),
                           __int_as_float(w == 0.f ? -1 : min(y, XENT_NEG - 1) + (far ? XENT_RAW + XENT_NEG : w > 0.f ? 0 : XENT_NEG)));
    }
    if (Hm) Hm[i] = w != 0.f ? H[i] : make_uint4(0, 0, 0, 0);
  }
}

// dl (bf16 [T][ld], columns past the piece zero) of the vocabulary piece that
// starts at v0.  C(m, n) as in k_xent_lse.  Bound by the products and, after
// them, by the exponentials (one a logit at a quarter of the vector rate: at T = 8192,
// d = 1024, V = 32000 a tenth of a launch, 453 us where dW's product of the same size takes 400).
// T = 32768, d = 2048, V = 32000 3.2 ms, 1.35 PFLOP/s.
template <class Cfg>
XENT_KERNEL(Cfg) k_xent_dl(BgShape g, XentTok a, const float2* __restrict__ tok, int v0, bf16_t* __restrict__ dl, int64_t ld) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[Cfg::SMEM];
  constexpr int FM = Cfg::FM, FN = Cfg::FN;
  float2 ks[FN];
  bg_run<Cfg>(
      g, smem,
      [&](const BgTile& t, int wm, int wn) {
        const int lane = xent_lane();
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int n = t.n * Cfg::BN + 16 * (wn * FN + j) + (lane & 15);
          ks[j] = tok[min(n, g.N - 1)];
        }
      },
      [&](f32x4_t (&acc)[FM][FN], const BgTile& t, int wm, int wn) {
        const int lane = xent_lane();
        const int m0 = t.m * Cfg::BM + 16 * wm * FM;
        const bool edge = m0 + 16 * FM > g.M;  // past the vocabulary: zeros
        static_for<0, FN>([&](auto j) {
          const int n = t.n * Cfg::BN + 16 * (wn * FN + j) + (lane & 15);
          const float2 k = ks[j];
          const int yk = __float_as_int(k.y), yt = yk >= XENT_NEG ? yk & (XENT_NEG - 1) : yk;
          if (__any(yk >= XENT_RAW)) {
            const float c = yk >= XENT_RAW ? k.x : 0.f, r = yk >= XENT_RAW ? 0.f : -k.x;
            xent_each<FM>([&](auto i, auto e) {
              constexpr int E = decltype(e)::value;
              acc[i][j][E] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][E] - c, LOG2E, r));
            });
          } else {
            xent_each<FM>([&](auto i, auto e) {
              constexpr int E = decltype(e)::value;
              acc[i][j][E] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][E], LOG2E, -k.x));
            });
          }
          if (__any(yk < 0 || yk >= XENT_NEG)) {  // masked tokens; a weight that is not in k.x
            const float f = yk >= XENT_NEG && a.weight && n < g.N ? a.weight[n] : 1.f;
            xent_each<FM>([&](auto i, auto e) {
              constexpr int E = decltype(e)::value;
              acc[i][j][E] = yk < 0 ? 0.f : acc[i][j][E] * f;
            });
          }
          const int y = (int)((unsigned)yt - (unsigned)(v0 + m0));
          if (__any((unsigned)y < 16u * FM)) {
            const float w = a.weight && n < g.N ? a.weight[n] : 1.f;
            xent_each<FM>([&](auto i, auto e) { acc[i][j][decltype(e)::value] -= y - 4 * (lane >> 4) == 16 * i + e ? w : 0.f; });
          }
          if (edge) xent_from<FM>(g.M - m0, lane, [&](auto i, auto e, bool past) { acc[i][j][decltype(e)::value] = past ? 0.f : acc[i][j][decltype(e)::value]; });
          bf16_t* o = dl + (int64_t)n * ld + m0 + bg_pack8_m(lane);
          static_for<0, FM / 2>([&](auto h) {
            constexpr int I = 2 * decltype(h)::value;
            const u32x4 v = bg_pack8(acc[I][j], acc[I + 1][j]);
            // ld % 64 == 0: a whole pair of blocks or none of it
            if (n < g.N && m0 + 16 * I < ld) *(u32x4*)(o + 16 * I) = v;
          });
          __builtin_amdgcn_sched_barrier(0);  // one j's values at a time in registers
        });
      });
#endif
}

// out[n][m] (+)= scale C(m, n); rows of masked tokens are zeros (tok given).
// Bound by the products; T = 32768, d = 2048, V = 32000 in four pieces: dW 2.9 ms, 1.49
// PFLOP/s, dH, whose fp32 sums are read and written by every piece, 3.2 ms, 1.33.
template <class Cfg>
XENT_KERNEL(Cfg) k_xent_out(BgShape g, XentOut o) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[Cfg::SMEM];
  constexpr int FM = Cfg::FM, FN = Cfg::FN;
  const float2* const tok = o.tok;
  int ys[FN];
  bg_run<Cfg>(
      g, smem,
      [&](const BgTile& t, int wm, int wn) {
        const int lane = xent_lane();
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int n = t.n * Cfg::BN + 16 * (wn * FN + j) + (lane & 15);
          ys[j] = tok ? __float_as_int(tok[min(n, g.N - 1)].y) : 0;
        }
      },
      [&](f32x4_t (&acc)[FM][FN], const BgTile& t, int wm, int wn) {
        const int lane = xent_lane();
        const int m0 = t.m * Cfg::BM + 16 * wm * FM;  // M % 64 == 0: pairs of blocks are whole or not there
        static_for<0, FN>([&](auto j) {
          const int n = t.n * Cfg::BN + 16 * (wn * FN + j) + (lane & 15);
          const bool zero = ys[j] < 0;
          static_for<0, FM / 2>([&](auto h) {
            constexpr int I = 2 * decltype(h)::value;
            const bool here = n < g.N && m0 + 16 * I < g.M;
            f32x4_t v[2] = {o.scale * acc[I][j], o.scale * acc[I + 1][j]};
            if (zero) v[0] = v[1] = f32x4_t{};
            const int64_t at = (int64_t)n * o.ld + m0 + 16 * I;
            if (o.f32) {
              float* p = (float*)o.out + t.split * o.split_stride + at + 4 * (lane >> 4);
              if (here) {
                if (o.add) {
                  v[0] += *(const f32x4_t*)p;
                  v[1] += *(const f32x4_t*)(p + 16);
                }
                *(f32x4_t*)p = v[0];
                *(f32x4_t*)(p + 16) = v[1];
              }
            } else {
              if (o.add && here) {
                const bf16_t* p = (const bf16_t*)o.out + at + 4 * (lane >> 4);
                const uint2 a = *(const uint2*)p, b = *(const uint2*)(p + 16);
                v[0] += f32x4_t{bf2f(a.x & 0xFFFFu), bf2f(a.x >> 16), bf2f(a.y & 0xFFFFu), bf2f(a.y >> 16)};
                v[1] += f32x4_t{bf2f(b.x & 0xFFFFu), bf2f(b.x >> 16), bf2f(b.y & 0xFFFFu), bf2f(b.y >> 16)};
              }
              const u32x4 w = bg_pack8(v[0], v[1]);
              if (here) *(u32x4*)((bf16_t*)o.out + at + bg_pack8_m(lane)) = w;
            }
          });
          __builtin_amdgcn_sched_barrier(0);
        });
      });
#endif
}

// sum_s part[s][i] in the order of s, eight terms requested at a time
__device__ __forceinline__ float4 xent_runs_sum(const float4* __restrict__ part, int splits, int64_t n4, int64_t i) {
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  int s = 0;
  for (; s + 8 <= splits; s += 8) {
    float4 p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) p[u] = part[(s + u) * n4 + i];
#pragma unroll
    for (int u = 0; u < 8; ++u) { v.x += p[u].x; v.y += p[u].y; v.z += p[u].z; v.w += p[u].w; }
  }
  for (; s < splits; ++s) {
    const float4 p = part[s * n4 + i];
    v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
  }
  return v;
}

// dH[t] = bf16(scale sum_s part[s][t]), zeros for masked tokens (us, against one
// term requested at a time: T = 37, d = 2048, 32 runs 7.0, 14.6; T = 100,
// d = 1024, 64 runs 10.3, 21.5; T = 8192, two runs, 84 MB 20 either way).
__global__ __launch_bounds__(256) void k_xent_sum(const float4* __restrict__ part, int splits, int64_t n4, int cpr,
                                                  const float2* __restrict__ tok, float scale,
                                                  uint2* __restrict__ dH) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (__float_as_int(tok[i / cpr].y) >= 0) v = xent_runs_sum(part, splits, n4, i);
    dH[i] = make_uint2(pack_bf2(scale * v.x, scale * v.y), pack_bf2(scale * v.z, scale * v.w));
  }
}

// dW (+)= scale sum_s part[s] over the runs of tokens.  Bound by the launch and the
// partial sums' bytes, at most 64 MB and mostly in the last-level cache.
__global__ __launch_bounds__(256) void k_xent_sum_dW(const float4* __restrict__ part, int splits, int64_t n4, float scale,
                                                     void* __restrict__ out, int f32, int add) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    float4 v = xent_runs_sum(part, splits, n4, i);
    v = make_float4(scale * v.x, scale * v.y, scale * v.z, scale * v.w);
    if (f32) {
      float4* p = (float4*)out + i;
      if (add) {
        const float4 a = *p;
        v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
      }
      *p = v;
    } else {
      uint2* p = (uint2*)out + i;
      if (add) {
        const uint2 a = *p;
        v.x += bf2f(a.x & 0xFFFFu); v.y += bf2f(a.x >> 16); v.z += bf2f(a.y & 0xFFFFu); v.w += bf2f(a.y >> 16);
      }
      *p = make_uint2(pack_bf2(v.x, v.y), pack_bf2(v.z, v.w));
    }
  }
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

// Of a token's exponentials exp(l - lse), the target's own and the sum of the
// others: what all of them are multiplied by and the target's entry of dl.  Where lse
// is this vocabulary's own log-sum-exp up to rounding (its error as a logarithm within
// 256 units of 2^-24, and 16 of lse's own), they are divided by their sum and the entry is minus
// the others' sum, so that a token whose target has nearly all of the probability keeps its
// gradient's digits: exp(l - lse) - 1 would leave the rounding errors of l and lse there, which are
// as large (lse from another fp32 product: dH is off by 1.9e-6 of its norm that way at T = 512, d = 256,
// V = 1000 and by 2.2e-7 this way, at V = 3 by 9.1e-6 and 8.7e-8).  Any other lse counts as it is given.
__device__ __forceinline__ float2 xent_norm(float others, float own, float lse) {
  const float s = others + own;
  if (fabsf(logf(s)) < 0x1p-24f * (256.f + 16.f * fabsf(lse))) return make_float2(1.f / s, -(others * (1.f / s)));
  return make_float2(1.f, own - 1.f);
}

// sums[t] (+)= {the others' exponentials, the target's own} of the piece at v0, for
// xent_norm over a vocabulary of several pieces.
__global__ __launch_bounds__(256) void k_xent_sums_f32(const float* __restrict__ l, int64_t ld, int n, int v0,
                                                       const float* __restrict__ lse, XentTok a, float2* __restrict__ sums) {
  __shared__ float sh[4];
  const int t = blockIdx.x;
  const float* row = l + t * ld;
  const int y = a.y[t], at = y >= v0 && y - v0 < n ? y - v0 : -1;
  const float L = lse[t];
  float others = 0.f, own = 0.f;
  for (int v = threadIdx.x; v < n; v += 256) {
    const float p = expf(row[v] - L);
    if (v == at) own = p; else others += p;
  }
  others = block_sum(others, sh);
  own = block_sum(own, sh);
  if (threadIdx.x == 0) {
    const float2 before = v0 > 0 ? sums[t] : make_float2(0.f, 0.f);
    sums[t] = make_float2(before.x + others, before.y + own);
  }
}

// dl in place; with Hm also the token's row of H, zeros where it is masked.
// WHOLE: the piece is all of the vocabulary, whose sums are taken here (T = 512,
// V = 1000: 8.0 us, without them 6.7); else they are in `sums`.
template <bool WHOLE>
__global__ __launch_bounds__(256) void k_xent_dl_f32(float* __restrict__ l, int64_t ld, int n, int v0,
                                                     const float* __restrict__ lse, const float2* __restrict__ sums, XentTok a,
                                                     float scale, const float4* __restrict__ H, float4* __restrict__ Hm, int cpr) {
  __shared__ float sh[4];
  const int t = blockIdx.x;
  float* row = l + t * ld;
  const int y = a.y[t], at = y >= v0 && y - v0 < n ? y - v0 : -1;
  const float w = y < 0 ? 0.f : a.weight ? a.weight[t] : 1.f;
  if (Hm)
    for (int c = threadIdx.x; c < cpr; c += 256)
      Hm[(int64_t)t * cpr + c] = w != 0.f ? H[(int64_t)t * cpr + c] : make_float4(0.f, 0.f, 0.f, 0.f);
  const float L = lse[t];
  float2 f;  // what the exponentials are multiplied by, the target's entry
  if constexpr (WHOLE) {
    float others = 0.f, own = 0.f;
    for (int v = threadIdx.x; v < n; v += 256) {
      const float p = expf(row[v] - L);
      row[v] = p;
      if (v == at) own = p; else others += p;
    }
    others = block_sum(others, sh);
    f = xent_norm(others, block_sum(own, sh), L);
  } else {
    f = xent_norm(sums[t].x, sums[t].y, L);
  }
  for (int v = threadIdx.x; v < ld; v += 256) {
    float p = 0.f;
    if (v < n) p = v == at ? f.y : (WHOLE ? row[v] : expf(row[v] - L)) * f.x;
    row[v] = w != 0.f && v < n ? scale * (w * p) : 0.f;
  }
}

// the rows of masked tokens set to zero (0 times an infinite weight row is no zero)
__global__ __launch_bounds__(256) void k_xent_zero_rows(float4* __restrict__ X, int64_t n4, int cpr, XentTok a) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / cpr;
    if (a.y[t] < 0 || (a.weight && a.weight[t] == 0.f)) X[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}

// bit 0 of flag: a target at or past V
__global__ void k_xent_check(const int32_t* __restrict__ y, int T, int64_t V, int* flag) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t < T && y[t] >= V) *flag = 1;
}

using Big_cc = BgCfg<2, 2, 8, 8, false, false>;
using Big_tc = BgCfg<2, 2, 8, 8, true, false>;
using Big_tt = BgCfg<2, 2, 8, 8, true, true>;
using Mid_cc = BgCfg<2, 2, 4, 4, false, false>;
using Mid_tc = BgCfg<2, 2, 4, 4, true, false>;
using Mid_tt = BgCfg<2, 2, 4, 4, true, true>;

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
// workgroups of 256 for n values (a launch holds fewer than 2^32 threads: the rest in turns)
dim3 blocks_of(int64_t n) {
  const int64_t b = (n + 255) / 256;
  return dim3((unsigned)(b < (1 << 23) ? b : 1 << 23));
}
bool fits(const XentGemm& q) {
  return q.M > 0 && q.N > 0 && q.K > 0 && q.ldp % 8 == 0 && q.ldq % 8 == 0 && q.ldp <= (1 << 21) && q.ldq <= (1 << 21) &&
         q.kper % 64 == 0;
}

}  // namespace

// 256 x 256 tiles, one workgroup per CU, against 128 x 128 ones, two: the time
// of a launch is its rounds over the 256 CUs times a round's, and a round of
// 128-tiles (half the outputs of the other) takes 5/8 of one of 256-tiles, 3/4
// where K is deep (the same work from twice the LDS and L2 reads, at less
// power while K is short).  Measured, us, 256 and 128 tiles, d = 1024:
//   lse  T = 1024: V = 8192 30, 21; V = 9216 29, 34; V = 14336 31, 36;
//        V = 19200 56, 51; V = 27648 58, 67; T = 8192, V = 24576 338, 380
//   dW   T = 8192: V = 8192 168, 126; V = 9216 172, 222; V = 19200 366, 391
//   dl   T = 37, V = 128000 57, 43; dW there 100, 130
bool xent_big_tiles(int64_t M, int64_t N, int64_t K, int64_t splits) {
  const int64_t big = (M + 255) / 256 * ((N + 255) / 256) * splits, mid = (M + 127) / 128 * ((N + 127) / 128) * splits;
  return 8 * ((big + 255) / 256) <= (K > 2048 ? 6 : 5) * ((mid + 511) / 512);
}

int xent_partials(int64_t V, int64_t T, int64_t d) {
  return (int)(xent_big_tiles(V, T, d, 1) ? 2 * ((V + 255) / 256) : 2 * ((V + 127) / 128));
}

hipError_t launch_xent_lse(const XentGemm& q, const XentTok& a, float* part, float* tgt, hipStream_t s) {
  if (!fits(q) || q.K % 64) return hipErrorInvalidValue;
  if (xent_big_tiles(q.M, q.N, q.K, 1)) {
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
  if (T > 1024)
    hipLaunchKernelGGL(k_xent_join<16>, dim3((T + 15) / 16), dim3(256), 0, s, (const float2*)part, np, T, a, tgt, loss, lse);
  else
    hipLaunchKernelGGL(k_xent_join<4>, dim3((T + 3) / 4), dim3(256), 0, s, (const float2*)part, np, T, a, tgt, loss, lse);
  return hipGetLastError();
}

hipError_t launch_xent_prep(const bf16_t* H, int T, int d, const XentTok& a, const float* lse, float* tok, bf16_t* Hm,
                            hipStream_t s) {
  const int cpr = d / 8;
  const int64_t n = (int64_t)T * cpr;
  hipLaunchKernelGGL(k_xent_prep, blocks_of(n), dim3(256), 0, s, (const uint4*)H, T, cpr, a,
                     lse, (float2*)tok, (uint4*)Hm);
  return hipGetLastError();
}

hipError_t launch_xent_dl(const XentGemm& q, const XentTok& a, const float* tok, int v0, bf16_t* dl, int64_t ld, hipStream_t s) {
  if (!fits(q) || q.K % 64) return hipErrorInvalidValue;
  if (xent_big_tiles(q.M, q.N, q.K, 1)) {
    const BgShape g = shape<Big_cc>(q);
    hipLaunchKernelGGL(k_xent_dl<Big_cc>, grid<Big_cc>(g), dim3(Big_cc::THREADS), 0, s, g, a, (const float2*)tok, v0, dl, ld);
  } else {
    const BgShape g = shape<Mid_cc>(q);
    hipLaunchKernelGGL(k_xent_dl<Mid_cc>, grid<Mid_cc>(g), dim3(Mid_cc::THREADS), 0, s, g, a, (const float2*)tok, v0, dl, ld);
  }
  return hipGetLastError();
}

hipError_t launch_xent_out(const XentGemm& q, int q_along_rows, const XentOut& o, hipStream_t s) {
  if (!fits(q) || q.M % 64) return hipErrorInvalidValue;
  const int64_t splits = q.kper > 0 ? (q.K + q.kper - 1) / q.kper : 1;
  if (splits > 1 && !o.f32) return hipErrorInvalidValue;
  const bool big = xent_big_tiles(q.M, q.N, splits > 1 ? q.kper : q.K, splits);
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
  hipLaunchKernelGGL(k_xent_sum, blocks_of(n4), dim3(256), 0, s, (const float4*)part, splits, n4, d / 4,
                     (const float2*)tok, scale, (uint2*)dH);
  return hipGetLastError();
}

hipError_t launch_xent_sum_dW(const float* part, int splits, int64_t n, float scale, void* out, int f32, int add,
                              hipStream_t s) {
  hipLaunchKernelGGL(k_xent_sum_dW, blocks_of(n / 4), dim3(256), 0, s, (const float4*)part, splits, n / 4, scale, out, f32,
                     add);
  return hipGetLastError();
}

hipError_t launch_xent_lse_f32(const float* l, int64_t ld, int T, int n, int v0, const XentTok& a, float* part, float* tgt,
                               hipStream_t s) {
  hipLaunchKernelGGL(k_xent_lse_f32, dim3(T), dim3(256), 0, s, l, ld, n, v0, a, (float2*)part, tgt);
  return hipGetLastError();
}

hipError_t launch_xent_sums_f32(const float* l, int64_t ld, int T, int n, int v0, const float* lse, const XentTok& a,
                                float* sums, hipStream_t s) {
  hipLaunchKernelGGL(k_xent_sums_f32, dim3(T), dim3(256), 0, s, l, ld, n, v0, lse, a, (float2*)sums);
  return hipGetLastError();
}

hipError_t launch_xent_dl_f32(float* l, int64_t ld, int T, int n, int v0, const float* sums, const float* lse,
                              const XentTok& a, float scale, const void* H, void* Hm, int d, hipStream_t s) {
  if (sums)
    hipLaunchKernelGGL(k_xent_dl_f32<false>, dim3(T), dim3(256), 0, s, l, ld, n, v0, lse, (const float2*)sums, a, scale,
                       (const float4*)H, (float4*)Hm, d / 4);
  else
    hipLaunchKernelGGL(k_xent_dl_f32<true>, dim3(T), dim3(256), 0, s, l, ld, n, v0, lse, nullptr, a, scale,
                       (const float4*)H, (float4*)Hm, d / 4);
  return hipGetLastError();
}

hipError_t launch_xent_zero_rows(float* X, int T, int d, const XentTok& a, hipStream_t s) {
  const int64_t n4 = (int64_t)T * d / 4;
  hipLaunchKernelGGL(k_xent_zero_rows, blocks_of(n4), dim3(256), 0, s, (float4*)X, n4, d / 4, a);
  return hipGetLastError();
}

hipError_t launch_xent_check(const int32_t* y, int T, int64_t V, int* flag, hipStream_t s) {
  hipLaunchKernelGGL(k_xent_check, dim3((T + 255) / 256), dim3(256), 0, s, y, T, V, flag);
  return hipGetLastError();
}

}  // namespace mapl
