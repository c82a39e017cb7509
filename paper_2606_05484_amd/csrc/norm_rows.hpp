// What the forward and the backward of the norms around a block (k_norm_fwd.hip,
// norm_bwd.hpp) share: how a row of d values lies over lanes, its sums, and the gate.
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace mapl {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Rows are read and written past the caches' keeping (ONCE) where a call's arrays are more
// than those hold.
template <bool ONCE, typename V>
__device__ __forceinline__ V row_load(const V* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool ONCE, typename V>
__device__ __forceinline__ void row_store(V* p, V v) {
  if constexpr (ONCE)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}

// Where a lane's v-th eight values of a row lie: two fours.  Side by side, or with
// SPLIT (fp32 rows) LANES fours apart, so that a wave's 16-byte accesses are whole
// runs of 1 KiB (side by side each would touch half of every line).  Lanes past the row's
// end load its last values (no branch around a load: they leave together).
template <int LANES, bool SPLIT, bool ONCE_>
struct Cols {
  static constexpr bool ONCE = ONCE_;
  int lane, d;
  __device__ __forceinline__ int at(int v, int q) const {
    return SPLIT ? (v * 2 + q) * LANES * 4 + lane * 4 : (v * LANES + lane) * 8 + 4 * q;
  }
  __device__ __forceinline__ bool in(int v, int q) const { return at(v, SPLIT ? q : 0) < d; }
  __device__ __forceinline__ uint32_t from(int v, int q) const {
    return SPLIT ? min(at(v, q), d - 4) : min(at(v, 0), d - 8) + 4 * q;
  }
};

// a row's value i (uniform base, 32-bit offset: a scalar and a vector register address it)
template <typename V, typename X>
__device__ __forceinline__ V* at_value(X* row, uint32_t i) {
  typedef typename std::conditional<std::is_const<V>::value, const char, char>::type C;
  return (V*)((C*)row + i * (uint32_t)sizeof(X));
}

// eight values of a row as they lie in memory
template <typename X>
struct Oct;
template <>
struct Oct<bf16_t> {
  u32x4 w;
  template <int L, bool S, bool O>
  __device__ __forceinline__ void load(const bf16_t* row, const Cols<L, S, O>& c, int v) {
    if constexpr (S) {
      const u32x2 a = row_load<O>(at_value<const u32x2>(row, c.from(v, 0))), b = row_load<O>(at_value<const u32x2>(row, c.from(v, 1)));
      w = u32x4{a.x, a.y, b.x, b.y};
    } else {
      w = row_load<O>(at_value<const u32x4>(row, c.from(v, 0)));
    }
  }
  template <int L, bool S, bool O>
  __device__ __forceinline__ void zero_past(const Cols<L, S, O>& c, int v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = c.in(v, i >> 1) ? w[i] : 0u;
  }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ void zero() { w = u32x4{0, 0, 0, 0}; }
  // what was made of the values is made again where it is used next, not kept in registers
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
};
template <>
struct Oct<float> {
  f32x4_t a, b;
  template <int L, bool S, bool O>
  __device__ __forceinline__ void load(const float* row, const Cols<L, S, O>& c, int v) {
    a = row_load<O>(at_value<const f32x4_t>(row, c.from(v, 0))), b = row_load<O>(at_value<const f32x4_t>(row, c.from(v, 1)));
  }
  template <int L, bool S, bool O>
  __device__ __forceinline__ void zero_past(const Cols<L, S, O>& c, int v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = c.in(v, 0) ? a[i] : 0.f, b[i] = c.in(v, 1) ? b[i] : 0.f;
  }
  __device__ __forceinline__ void zero() { a = b = f32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void forget() {}
};
// Makes f here and now: what it is made of would else be carried past the next branches (sums to
// the loop's end, stored values to their store), in several times the registers.  For rows that fill them;
// where there is room the compiler's order is the faster one.
__device__ __forceinline__ void pin8(float (&f)[8]) {
  asm volatile("" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]), "+v"(f[4]), "+v"(f[5]), "+v"(f[6]), "+v"(f[7]));
}
// (rounds f to what memory holds)
template <int L, bool S, bool O>
__device__ __forceinline__ void put8(bf16_t* row, const Cols<L, S, O>& c, int v, float (&f)[8], bool live = true) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = pack_bf2(f[2 * i], f[2 * i + 1]);
    f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  if constexpr (S) {
    if (live && c.in(v, 0)) row_store<O>(at_value<u32x2>(row, c.at(v, 0)), u32x2{w.x, w.y});
    if (live && c.in(v, 1)) row_store<O>(at_value<u32x2>(row, c.at(v, 1)), u32x2{w.z, w.w});
  } else if (live && c.in(v, 0)) {
    row_store<O>(at_value<u32x4>(row, c.at(v, 0)), w);
  }
}
template <int L, bool S, bool O>
__device__ __forceinline__ void put8(float* row, const Cols<L, S, O>& c, int v, float (&f)[8], bool live = true) {
  const f32x4_t a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
  if (live && c.in(v, 0)) row_store<O>(at_value<f32x4_t>(row, c.at(v, 0)), a);
  if (live && c.in(v, 1)) row_store<O>(at_value<f32x4_t>(row, c.at(v, 1)), b);
}

// what a vector that is not given reads as
static __device__ const struct Ones {
  float v[16384];
  constexpr Ones() : v() {
    for (float& x : v) x = 1.f;
  }
} ones;
__device__ __forceinline__ const float* or_ones(const float* w) { return w ? w : ones.v; }
template <int L, bool S, bool O>
__device__ __forceinline__ void vec8(const float* w, const Cols<L, S, O>& c, int v, float (&f)[8]) {
  typedef const __attribute__((address_space(1))) char* Global;  // (the ones' or the caller's: global memory either way)
  typedef const __attribute__((address_space(1))) f32x4_t* Four;
  const Global p = (Global)(const char*)w;
  const f32x4_t a = *(Four)(p + 4u * c.from(v, 0)), b = *(Four)(p + 4u * c.from(v, 1));
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); }

// The sums of v over the LANES lanes of a row, in every one of them, and a bit for each
// that is past 1e38 or no number (in any of the workgroup's rows that share its barriers).
// A row of more than a wave meets in LDS: two areas in turn, so that one barrier a sum does
// (the one of the next sum lies between an area's reads and its next writes).
constexpr float SUM_LIMIT = 1e38f;
template <int LANES, int ROWS, int N>
__device__ __forceinline__ uint32_t row_sums(float (&v)[N], float* lds, int& turn) {
  uint32_t over = 0;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    v[n] = dpp_add<0xB1>(v[n]);   // lane ^ 1
    v[n] = dpp_add<0x4E>(v[n]);   // lane ^ 2
    v[n] = dpp_add<0x141>(v[n]);  // the other half of 8
    if constexpr (LANES >= 16) v[n] = dpp_add<0x140>(v[n]);  // the other half of 16
    if constexpr (LANES == 32) v[n] += __shfl_xor(v[n], 16, WAVE);
    if constexpr (LANES >= 64) v[n] = (lane_of(v[n], 0) + lane_of(v[n], 16)) + (lane_of(v[n], 32) + lane_of(v[n], 48));
    if constexpr (LANES <= 64) over |= v[n] < SUM_LIMIT ? 0u : 1u << n;
  }
  if constexpr (LANES > 64) {
    constexpr int W = LANES / 64, WAVES = W * ROWS;
    float* a = lds + turn * 4 * WAVES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) a[n * WAVES + wave] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += a[n * WAVES + k * W + w];
        if (ROWS == 1 || wave / W == k) v[n] = s;
        over |= s < SUM_LIMIT ? 0u : 1u << n;
      }
    }
    turn ^= 1;
  }
  return over;
}
constexpr int sums_floats(int lanes, int rows) { return lanes > 64 ? 2 * 4 * (lanes / 64) * rows : 1; }

// (mean z^2 + eps)^-1/2 from ss = sum z^2: the instruction's and a Newton step.  Where the
// sum overflows (a row whose size is past 1e17; `over`, as row_sums has it) it is taken again 2^-80
// times smaller: no term is then past 2^96, and what falls out at the low end is 2^-40 of
// the largest.
__device__ __forceinline__ float inv_root(float x) {
  const float r = __builtin_amdgcn_rsqf(x);
  return fmaf(r * fmaf(-x * r, r, 1.f), 0.5f, r);
}
template <int LANES, int ROWS, int NV, typename Z>
__device__ __forceinline__ float row_scale(float ss, uint32_t over, Z z, float inv_d, float eps, float* lds, int& turn) {
  if (over) {
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = z(v, i) * 0x1p-80f;
        s[0] = fmaf(q, q, s[0]);
      }
    row_sums<LANES, ROWS, 1>(s, lds, turn);
    if (!(ss < SUM_LIMIT)) return 0x1p-80f / sqrtf(s[0] * inv_d);
  }
  return inv_root(fmaf(ss, inv_d, eps));
}

// sigmoid(g) = 1 / (1 + e) and 1 - sigmoid(g) = e / (1 + e) with e = exp(-g), each to a few of
// its last digits at either end (and 1 where e overflows).  FINE (an fp32 stream): the
// rounding of -g log2(e), which is |g| units of e's last digit, put right to first order,
// and the reciprocal with a Newton step.  A bf16 stream goes without: its values' own rounding is 2^16
// of those units, and the vectors' gradients are off by up to 1.3 |g| of them a term.  It would cost,
// T = 32768, d = 2048 gated, 230 us in place of 201 backward and 119 in place of 117 forward; an fp32 stream
// with a bf16 block, T = 16384: backward 136 with it and 142 without, forward 83 and 82.
template <bool FINE>
__device__ __forceinline__ void sigmoid2(float g, float& a, float& b) {
  constexpr float L = -1.44269504088896341f;
  const float t = g * L;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (FINE) {
    const float lo = fmaf(g, -1.92596299e-8f, fmaf(g, L, -t));  // (and what L itself is short of)
    e = fabsf(g) < 87.f ? fmaf(e, lo * 0.693147180559945309f, e) : e;
  }
  const float n = 1.f + e;
  a = __builtin_amdgcn_rcpf(n);
  if constexpr (FINE) a = t > 126.f ? a : fmaf(fmaf(-n, a, 1.f), a, a);
  b = t > 126.f ? 1.f : e * a;  // (NaN stays)
}
// act(g) and its derivative; KIND: NORM_SIGMOID or NORM_SILU
template <int KIND, bool FINE>
__device__ __forceinline__ void act_both(float g, float& f, float& df) {
  float a, b;
  sigmoid2<FINE>(g, a, b);
  f = KIND == NORM_SILU ? g * a : a;
  df = KIND == NORM_SILU ? a * fmaf(g, b, 1.f) : a * b;
}

// which of the workgroup's rows (uniform where a wave has one: addresses are then scalar)
template <int LANES, int ROWS>
__device__ __forceinline__ int sub_row() {
  if constexpr (ROWS == 1) return 0;
  if constexpr (LANES >= 64) return __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
  return threadIdx.x / LANES;
}

}  // namespace mapl
