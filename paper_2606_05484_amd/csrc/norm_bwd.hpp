// The gradient of the norms around a block (k_norm_fwd.hip) with respect to x, h,
// G and the three vectors, in one pass over the rows and a sum over the
// workgroups' parts of the vectors' gradients:
//   dX = dx' + r_x (dy w_pre - x' r_x^2 mean(dy w_pre x')), then with dX
//   dn = alpha s dX act, dh = r_h (dn w_post - h r_h^2 mean(dn w_post h)), dG = alpha s dX n act'
//   dw_pre = sum dy x' r_x, ds = sum alpha dX n act, dw_post = sum dn h r_h
// r_h and r_x are computed again from the rows that are read anyway: the forward
// keeps nothing for it.  Sums and everything in between are fp32.
//
// Bound by HBM (16 bytes a value where everything is bf16) and nearly as much by the vector
// unit, about 45 operations a value: T = 32768, d = 2048 with a gated branch 200 us, 5.4 TB/s, and 4.5
// for the parts' sum; with 110 operations a value (a gate's kind decided for each, IEEE divisions, the
// vectors loaded for every row) 237.  The next row's loads issued ahead cost a third of
// the occupancy and gained nothing (224).
#pragma once
#include "norm_rows.hpp"

namespace mapl {

namespace {

// A row is held by LANES lanes, eight values NV times each; a workgroup of THREADS takes
// THREADS / LANES rows at a time, adds its rows' shares of the vectors' gradients in
// registers and then over its groups of lanes in LDS, and leaves them in
// part[workgroup][3][d] (dw_post, ds, dw_pre).
template <typename X, typename H, int LANES, int NV, int THREADS, bool BRANCH, bool PRE, int GATE, bool ONCE>
__global__ __launch_bounds__(THREADS) void k_norm_bwd(const NormArgs g) {
  constexpr int ROWS = THREADS / LANES;
  constexpr bool SPLIT = sizeof(X) == 4, FINE = sizeof(X) == 4;
  constexpr int NS = (BRANCH ? 2 : 0) + (PRE ? 1 : 0), S0 = BRANCH ? 0 : 2;  // sums: dw_post, ds, dw_pre
  __shared__ float lds[sums_floats(LANES, ROWS)];
  __shared__ float red[ROWS > 1 ? NS * LANES * NV * 8 : 1];
  int turn = 0;
  const Cols<LANES, SPLIT, ONCE> c{(int)threadIdx.x % LANES, g.d};
  const int sub = sub_row<LANES, ROWS>();
  const int64_t d = g.d;
  const float inv_d = 1.f / (float)g.d;
  const bool post = g.parts & NORM_POST, ragged = g.d != LANES * NV * 8;
  const float *w_post = or_ones(g.w_post), *scale = or_ones(g.scale), *w_pre = or_ones(g.w_pre);
  // Rows past 8192 values do not stay in registers: what a step needs is loaded again (from the
  // caches) a run of eight at a time.  d = 16384, T = 1024 in bf16: 106 us and 7 for the sum (held, with
  // more spills, 165 to 234).  Up to 12288 on 768 lanes, T = 4096, d = 8256 160 us, d = 12288 210 (on 512 lanes
  // 172 and 212, 253 and 301 with room for 16384; past 12288 1024 lanes spill more).
  // That spares most spills, not all, since the first pass's rows live beside the sums until both scales
  // are known.  Registers spilled a lane: bf16 none up to 12288, past it 22 to 26 with branch and y; all fp32 16 or
  // 17, past it 78 or 79; an fp32 stream with a bf16 block 39, past it 89; past 12288 without y up to 12 and 19; y
  // alone none.  T = 4096 gated, d = 8256, 12288 and 16384: all fp32 281, 371, 759 us, an fp32 stream
  // with a bf16 block 307, 376, 637, bf16 159, 209, 350.
  constexpr bool AGAIN = LANES * NV * 8 > 8192;
  float acc[NS][NV][8];
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[j][v][i] = 0.f;
  // one run of eight: the vectors stay in registers; two would not leave room
  constexpr bool HELD = NV == 1;
  float wp[8], wq[8], sc[8];
  if constexpr (HELD) {
    vec8(w_pre, c, 0, wp);
    vec8(w_post, c, 0, wq);
    vec8(scale, c, 0, sc);
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] *= g.alpha;
  }

  for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < g.T; t0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = t0 + sub;
    const bool live = ROWS == 1 || row < g.T;  // (past the last row: that one again with no gradient, not written)
    const int64_t t = live ? row : g.T - 1;
    Oct<X> x[NV], dxo[NV];
    Oct<H> dy[NV], h[NV], u[NV];
    auto load_y = [&](int v, auto&& c) {
      if constexpr (PRE) {
        x[v].load((const X*)g.x + t * d, c, v);
        dy[v].load((const H*)g.dy + t * d, c, v);
      }
    };
    auto load_h = [&](int v, auto&& c) {
      if constexpr (BRANCH) h[v].load((const H*)g.h + t * g.ld_h, c, v);
    };
    auto load_rest = [&](int v) {
      if (!PRE || g.dxo)
        dxo[v].load((const X*)g.dxo + t * d, c, v);
      else
        dxo[v].zero();
      if constexpr (GATE != 0 && !AGAIN) u[v].load((const H*)g.gate + t * g.ld_g, c, v);
    };
    auto clear_y = [&](int v) {
      if constexpr (PRE) {
        if (ragged) x[v].zero_past(c, v), dy[v].zero_past(c, v);
        if (ROWS > 1 && !live) dy[v].zero();
      }
    };
    auto clear_h = [&](int v) {
      if constexpr (BRANCH)
        if (ragged) h[v].zero_past(c, v);
    };
    const Cols<LANES, SPLIT, ONCE && !AGAIN> first{c.lane, c.d};
#pragma unroll
    for (int v = 0; v < NV; ++v) load_y(v, first), load_h(v, first);
    if constexpr (!AGAIN) {
#pragma unroll
      for (int v = 0; v < NV; ++v) load_rest(v);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) clear_y(v), clear_h(v);
    if (!AGAIN && ROWS > 1 && !live) {
#pragma unroll
      for (int v = 0; v < NV; ++v) dxo[v].zero();
    }
    // the sums that need nothing but the inputs, at once
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (PRE) {
        if constexpr (!HELD) vec8(w_pre, c, v, wp);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float z = x[v].get(i);
          s[0] = fmaf(z, z, s[0]);
          s[1] = fmaf(dy[v].get(i) * wp[i], z, s[1]);
        }
      }
      if constexpr (BRANCH) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[2] = fmaf(h[v].get(i), h[v].get(i), s[2]);
      }
    }
    const uint32_t over = row_sums<LANES, ROWS, 3>(s, lds, turn);
    float q[NV][8];  // dX
    if constexpr (PRE) {
      const float r = row_scale<LANES, ROWS, NV>(s[0], over & 1, [&](int v, int i) { return x[v].get(i); }, inv_d, g.eps, lds, turn);
      const float k = r * (r * (s[1] * inv_d));
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float o[8];
        if constexpr (!HELD) vec8(w_pre, c, v, wp);
        if constexpr (AGAIN) {
          load_y(v, first);
          load_rest(v);
          clear_y(v);
        }
        x[v].forget(), dy[v].forget();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float z = x[v].get(i), y = dy[v].get(i);
          acc[2 - S0][v][i] = fmaf(z * r, y, acc[2 - S0][v][i]);  // (y r may underflow where z is large)
          q[v][i] = fmaf(r, fmaf(-z, k, y * wp[i]), dxo[v].get(i));
          o[i] = q[v][i];
        }
        if constexpr (!HELD) pin8(acc[2 - S0][v]), pin8(q[v]), pin8(o);
        put8((X*)g.dx + t * d, c, v, o, live);
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if constexpr (AGAIN) load_rest(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) q[v][i] = dxo[v].get(i);
      }
    }
    if constexpr (BRANCH) {
      const float r = post ? row_scale<LANES, ROWS, NV>(s[2], over & 4, [&](int v, int i) { return h[v].get(i); }, inv_d, g.eps, lds, turn) : 1.f;
      float sh[1] = {0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float o[8];
        if constexpr (!HELD) {
          vec8(w_post, c, v, wq);
          vec8(scale, c, v, sc);
#pragma unroll
          for (int i = 0; i < 8; ++i) sc[i] *= g.alpha;
        }
        if constexpr (AGAIN) {
          load_h(v, first);
          if constexpr (GATE != 0) u[v].load((const H*)g.gate + t * g.ld_g, c, v);
          clear_h(v);
        }
        h[v].forget();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float hi = h[v].get(i), n0 = hi * r, n = n0 * wq[i], dt = q[v][i] * sc[i];
          float f = 1.f, df = 0.f;
          if constexpr (GATE != 0) act_both<GATE, FINE>(u[v].get(i), f, df);
          acc[1][v][i] = fmaf(q[v][i], GATE ? n * f : n, acc[1][v][i]);
          const float dn = GATE ? dt * f : dt;
          if constexpr (GATE != 0) o[i] = dt * n * df;
          acc[0][v][i] = fmaf(dn, n0, acc[0][v][i]);
          q[v][i] = dn * wq[i];
          sh[0] = fmaf(q[v][i], hi, sh[0]);
        }
        if constexpr (!HELD) pin8(acc[0][v]), pin8(acc[1][v]), pin8(q[v]);
        if constexpr (!HELD && GATE != 0) pin8(o);
        if constexpr (GATE != 0) put8((H*)g.dgate + t * g.ld_g, c, v, o, live);
      }
      float k = 0.f;
      if (post) {
        row_sums<LANES, ROWS, 1>(sh, lds, turn);
        k = r * (r * (sh[0] * inv_d));
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if constexpr (AGAIN) {
          load_h(v, c);
          clear_h(v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) q[v][i] = r * fmaf(-h[v].get(i), k, q[v][i]);
        put8((H*)g.dh + t * g.ld_h, c, v, q[v], live);
      }
    }
  }
  if (!g.part) return;
  float* part = g.part + (int64_t)blockIdx.x * 3 * d;
  if constexpr (BRANCH) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[1][v][i] *= g.alpha;
  }
  if constexpr (ROWS > 1) {
    for (int k = 0; k < ROWS; ++k) {
      __syncthreads();
      if ((int)threadIdx.x / LANES == k)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              float* p = red + j * LANES * NV * 8 + c.at(v, q);
#pragma unroll
              for (int i = 0; i < 4; ++i) p[i] = k ? p[i] + acc[j][v][4 * q + i] : acc[j][v][4 * q + i];
            }
    }
    __syncthreads();
    for (int j = 0; j < NS; ++j)
      for (int k = threadIdx.x; k < d; k += THREADS) part[(j + S0) * d + k] = red[j * LANES * NV * 8 + k];
  } else {
    const Cols<LANES, SPLIT, false> kept{c.lane, c.d};  // (read by the next launch)
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int v = 0; v < NV; ++v) put8(part + (j + S0) * d, kept, v, acc[j][v]);
  }
}

// Some thousand rows of this width: workgroups of twice as many, so that more are under way at once
// with no more parts to sum.  d = 1024, us with and without: T = 1021 12.4, 13.1; T = 3000 18.5,
// 20.6; d = 2048: T = 1024 15.4, 16.2; T = 1500 18.6, 21.0.  (Fewer leave CUs idle: T = 64 10.1, 9.6.)
inline bool norm_bwd_wide(int64_t T, int d) {
  const int rows = d <= 1024 ? 2 : 1;
  return ((d > 512 && d <= 1024) || (d > 1536 && d <= 2048)) && T > 256 * rows && T <= 2048 * rows;
}

template <typename X, typename H, int LANES, int NV, int THREADS, bool ONCE>
hipError_t run(const NormArgs& g, hipStream_t s) {
  const bool br = g.parts & NORM_BRANCH, pre = g.parts & NORM_PRE;
  void (*f)(NormArgs) = k_norm_bwd<X, H, LANES, NV, THREADS, false, true, 0, ONCE>;
  if (br && pre)
    f = g.act == 0 ? k_norm_bwd<X, H, LANES, NV, THREADS, true, true, 0, ONCE>
        : g.act == NORM_SILU ? k_norm_bwd<X, H, LANES, NV, THREADS, true, true, NORM_SILU, ONCE>
                             : k_norm_bwd<X, H, LANES, NV, THREADS, true, true, NORM_SIGMOID, ONCE>;
  else if (br)
    f = g.act == 0 ? k_norm_bwd<X, H, LANES, NV, THREADS, true, false, 0, ONCE>
        : g.act == NORM_SILU ? k_norm_bwd<X, H, LANES, NV, THREADS, true, false, NORM_SILU, ONCE>
                             : k_norm_bwd<X, H, LANES, NV, THREADS, true, false, NORM_SIGMOID, ONCE>;
  hipLaunchKernelGGL(f, dim3(norm_bwd_parts(g.T, g.d, g.parts)), dim3(THREADS), 0, s, g);
  return hipGetLastError();
}

// The lanes of a row: few enough idle ones, and few enough variants.  With the next power of two in
// their place, T = 8000, us: d = 2112, y alone 38 (320 lanes: 28), d = 1536 gated 54 (192: 50); T = 4096: d = 4160 gated
// 92 (320 twice: 87), d = 6144 the same with 384 as with 512.
template <typename X, typename H, bool ONCE>
hipError_t pick(const NormArgs& g, hipStream_t s) {
  if constexpr (!ONCE) {
    if (norm_bwd_wide(g.T, g.d)) return g.d <= 1024 ? run<X, H, 128, 1, 512, false>(g, s) : run<X, H, 256, 1, 512, false>(g, s);
  }
  if (g.d <= 64) return run<X, H, 8, 1, 256, ONCE>(g, s);
  if (g.d <= 128) return run<X, H, 16, 1, 256, ONCE>(g, s);
  if (g.d <= 256) return run<X, H, 32, 1, 256, ONCE>(g, s);
  if (g.d <= 512) return run<X, H, 64, 1, 256, ONCE>(g, s);
  if (g.d <= 1024) return run<X, H, 128, 1, 256, ONCE>(g, s);
  if (g.d <= 1536) return run<X, H, 192, 1, 192, ONCE>(g, s);
  if (g.d <= 2048) return run<X, H, 256, 1, 256, ONCE>(g, s);
  if (g.d <= 2560) return run<X, H, 320, 1, 320, ONCE>(g, s);
  if (g.d <= 4096) return run<X, H, 256, 2, 256, ONCE>(g, s);
  if (g.d <= 5120) return run<X, H, 320, 2, 320, ONCE>(g, s);
  if (g.d <= 8192) return run<X, H, 512, 2, 512, ONCE>(g, s);
  if (g.d <= 12288) return run<X, H, 768, 2, 768, ONCE>(g, s);
  return run<X, H, 512, 4, 512, ONCE>(g, s);
}

}  // namespace

}  // namespace mapl
