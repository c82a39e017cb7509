// The optimizer's step over all tensors of a stage: the norm of their gradients
// with the factor that clips it, and AdamW with states in fp32 or in 8 bits:
//   g' = factor g,  m <- m + (1 - b1)(g' - m),  v <- v + (1 - b2)(g'^2 - v)
//   p <- p - (lr wd p + lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps))
// A launch takes up to 52 tensors (the norm 176) from its arguments and cuts them in
// pieces of OPTIM_PIECE values, one a workgroup, so that many small tensors and a
// large one fill the chip alike.
//
// 8-bit states.  Blocks of 128 values of a tensor have an exponent byte each for m
// and for s = sqrt(v).  m: sign, 4 exponent and 3 mantissa bits (the values of
// float8_e4m3fn); s: 4 and 4 bits, no sign.  Both grids end in equal steps down to
// 0.  With k the least number for which 1.75 2^k (m) or 1.9375 2^k (s) holds the
// block's largest magnitude, byte k + 127 (at least 24; 255: NaNs), a value is
// m = code 2^(k - 8) or s = code 2^k.
// The rounding is stochastic, up with the probability that makes its mean the
// value, by 16 bits of a hash of (seed, t, tensor, place): rounding to nearest
// would leave s where it is, since a step moves it by about (1 - b2) / 2 of itself
// and its codes lie 1/32 to 1/16 of s apart.  At random such a move x of a distance D
// has a variance of x D, deviations fade at 1 - b2 = 2 x / s a step, so s is spread
// around its right mean by sqrt(D s) / 2, 9 to 12 % of s, whatever b2 is.  An s above 0
// never becomes 0 (m / s would be huge).
// What is rounded to 8 bits are fp32 numbers whose every operation is rounded to
// nearest (no contraction in state_update): the same bits wherever they are computed.
//
// Bound by HBM: fp32 states 28 bytes a value (bf16 gradients and copy), 8 bits 16.03.  266 M
// values: 1.30 ms, 5.7 TB/s, and 0.75 ms, 5.7 TB/s (a large copy here 4.9 TB/s); their states unpacked 0.45
// ms, 5.9 TB/s, packed 0.47, 5.6.  All of a piece's loads first (four runs of four values a lane; two 1407 and 825 us, before
// the caches were passed by: 1390 and 799 with four), pieces of 4096 (of 2048 1421 and 801).
#include "common.hpp"
#include "kernels.hpp"

namespace mapl {

namespace {

constexpr int OPTIM_PIECE = 4096, OB = 128;

__device__ __forceinline__ uint32_t hash32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x9E3779B9u;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 16);
}

// the tensor that a piece belongs to (uniform): every lane looks at one or a few (a search would
// wait for its loads in turn)
template <typename Table>
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t piece) {
  const int l = threadIdx.x & 63;
  int i = -1;
#pragma unroll
  for (int k = 0; k < Table::MOST; k += WAVE) {
    const bool below = k + l < t.count && t.first[k + l] <= piece;
    i += __builtin_popcountll(__ballot(below));
  }
  return __builtin_amdgcn_readfirstlane(i);
}

// Values i .. i + 3 of n, a lane's share: a wave's 16-byte accesses are whole runs of
// 1 KiB (with eight fp32 values a lane every store would write half of each line: the unpacking of
// 266 M values 644 us, 473 with four).  ALL: none lies past n; else those that do read as
// zeros and are not written.  ONCE: nothing reads the line soon (a hint to the caches).
template <bool ONCE, typename V>
__device__ __forceinline__ V fetch(const V* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool ONCE, typename V>
__device__ __forceinline__ void keep(V* p, V v) {
  if constexpr (ONCE)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

template <bool ALL, bool ONCE = false>
__device__ __forceinline__ f32x4_t get4(const float* p, int64_t i, int64_t n) {
  if (ALL || i + 4 <= n) return fetch<ONCE>((const f32x4_t*)(p + i));
  f32x4_t f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = i + j < n ? p[i + j] : 0.f;
  return f;
}
template <bool ALL, bool ONCE = false>
__device__ __forceinline__ f32x4_t get4(const bf16_t* p, int64_t i, int64_t n) {
  uint32_t w[2] = {0, 0};
  if (ALL || i + 4 <= n) {
    const u32x2 v = fetch<ONCE>((const u32x2*)(p + i));
    w[0] = v.x, w[1] = v.y;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < n) w[j >> 1] |= (uint32_t)p[i + j] << (16 * (j & 1));
  }
  return f32x4_t{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
                 __uint_as_float(w[1] & 0xffff0000u)};
}
template <bool ALL, bool ONCE = false>
__device__ __forceinline__ uint32_t get4(const uint8_t* p, int64_t i, int64_t n) {
  if (ALL || i + 4 <= n) return fetch<ONCE>((const uint32_t*)(p + i));
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < n) w |= (uint32_t)p[i + j] << (8 * j);
  return w;
}
template <bool ALL, bool ONCE = false>
__device__ __forceinline__ void put4(float* p, int64_t i, int64_t n, const f32x4_t& f) {
  if (ALL || i + 4 <= n) {
    keep<ONCE>((f32x4_t*)(p + i), f);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < n) p[i + j] = f[j];
  }
}
template <bool ALL, bool ONCE = false>
__device__ __forceinline__ void put4(bf16_t* p, int64_t i, int64_t n, const f32x4_t& f) {
  if (ALL || i + 4 <= n) {
    keep<ONCE>((u32x2*)(p + i), u32x2{pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3])});
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < n) p[i + j] = (bf16_t)f2bf(f[j]);
  }
}
template <bool ALL, bool ONCE = false>
__device__ __forceinline__ void put4(uint8_t* p, int64_t i, int64_t n, uint32_t w) {
  if (ALL || i + 4 <= n) {
    keep<ONCE>((uint32_t*)(p + i), w);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < n) p[i + j] = (uint8_t)(w >> (8 * j));
  }
}

// ------------------------------------------------------------------ 8-bit states
__device__ __forceinline__ float pow2_byte(int b) { return __uint_as_float((uint32_t)b << 23); }  // 2^(b - 127)

// m and s of four codes; 255 stands for NaNs, and bytes below 24 are not made (0 before the first step)
__device__ __forceinline__ void decode4(uint32_t qm, uint32_t qs, uint32_t e, f32x4_t& m, f32x4_t& s) {
  const uint32_t em = e & 255u, es = e >> 8;
  const float um = em == 255 ? __builtin_nanf("") : em < 24 ? 0.f : pow2_byte(em - 8);
  const float us = es == 255 ? __builtin_nanf("") : es < 24 ? 0.f : pow2_byte(es);
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(qm, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(qm, true);
  m = f32x4_t{a[0] * um, a[1] * um, b[0] * um, b[1] * um};
#pragma unroll
  for (int j = 0; j < 4; ++j)  // a code's bits are those of a number 2^112 times smaller (subnormal below 16)
    s[j] = __uint_as_float(((qs >> (8 * j)) & 255u) << 19) * 0x1p112f * us;
}

// the largest of the 32 lanes that hold a block of 128
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true));   // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true));   // lane ^ 2
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true));  // the other half of 8
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true));  // the other half of 16
  const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));  // rows 0 0 2 2 and 1 1 3 3
  return max(w.x, w.y);
}
__device__ __forceinline__ uint32_t exponent_byte(uint32_t amax, uint32_t room) {
  const uint32_t b = (amax + room) >> 23;
  return b < 24 ? 24u : b > 255 ? 255u : b;
}
// the code of y in [0, top]: its bits above the least normal number 2^LOW, whole
// steps below it, and `noise` (16 bits) added behind the last bit that is kept
template <int BITS, int LOW>
__device__ __forceinline__ uint32_t code_of(float y, uint32_t noise) {
  constexpr int DROP = 23 - BITS;
  constexpr float least = LOW == -6 ? 0x1p-6f : 0x1p-14f, whole = LOW == -6 ? 0x1p29f : 0x1p37f;
  static_assert(LOW == -6 || LOW == -14, "m and s");
  const uint32_t t = y >= least ? __float_as_uint(y) - ((126 + LOW) << 23) : (uint32_t)(y * whole);
  return (t + (noise << (DROP - 16))) >> DROP;
}

// codes and exponent bytes of a lane's four values of m and s (s >= 0, or NaN)
template <typename Noise>
__device__ __forceinline__ uint32_t encode4(const f32x4_t& m, const f32x4_t& s, Noise noise, uint32_t& qm, uint32_t& qs) {
  uint32_t am = 0, as = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    am = max(am, __float_as_uint(m[j]) & 0x7fffffffu);
    as = max(as, __float_as_uint(s[j]) & 0x7fffffffu);
  }
  const uint32_t em = exponent_byte(block_max(am), 0x1fffff), es = exponent_byte(block_max(as), 0x7ffff);
  const float um = em == 255 ? 0.f : pow2_byte(262 - em), us = es >= 254 ? es == 255 ? 0.f : 0x1p-127f : pow2_byte(254 - es);
  qm = qs = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t r = noise(j);
    const float a = em == 255 ? 0.f : fabsf(m[j]), b = es == 255 ? 0.f : s[j];
    uint32_t cm = code_of<3, -6>(a * um, r & 0xffffu), cs = code_of<4, -14>(b * us, r >> 16);
    cm |= (__float_as_uint(m[j]) >> 24) & 128u;
    cs = max(cs, b > 0.f ? 1u : 0u);
    qm |= cm << (8 * j);
    qs |= cs << (8 * j);
  }
  return em | es << 8;
}

// ------------------------------------------------------------------ AdamW
// the states' step, every operation rounded on its own; g is the clipped gradient
__device__ __forceinline__ void state_update(float g, float c1, float c2, float& m, float& v) {
#pragma clang fp contract(off)
  m = m + (g - m) * c1;
  v = v + (g * g - v) * c2;
}

// a step's numbers for one tensor
struct Step {
  float factor, c1, c2, up, rs, eps, decay;  // up = lr / (1 - b1^t), rs = (1 - b2^t)^-1/2, decay = lr wd
  uint32_t key;
};

// A lane's four values `at` .. at + 3 of a tensor, its loads and what is made of them.
template <typename G, bool LOW, bool ALL, bool ONCE>
struct Four {
  f32x4_t p, g, m, v;
  uint32_t qm, qs, e;
  __device__ __forceinline__ void load(const OptimTensor& x, int64_t at) {
    p = get4<ALL, ONCE>(x.p, at, x.n);
    g = get4<ALL, ONCE>((const G*)x.g, at, x.n);
    if constexpr (LOW) {
      qm = get4<ALL, ONCE>((const uint8_t*)x.m, at, x.n);
      qs = get4<ALL, ONCE>((const uint8_t*)x.v, at, x.n);
      e = *(const uint16_t*)(x.e + at / OB * 2);
    } else {
      m = get4<ALL, ONCE>((const float*)x.m, at, x.n);
      v = get4<ALL, ONCE>((const float*)x.v, at, x.n);
    }
  }
  __device__ __forceinline__ void step(const OptimTensor& x, int64_t at, const Step& a) {
    f32x4_t s;
    if constexpr (LOW) {
      decode4(qm, qs, e, m, s);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = s[j] * s[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float mj = m[j], vj = v[j];
      state_update(g[j] * a.factor, a.c1, a.c2, mj, vj);
      m[j] = mj, v[j] = vj;
      s[j] = sqrtf(vj);  // (v may be subnormal: g past 1e-19 and an eps as small)
      p[j] -= fmaf(a.decay, p[j], a.up * (mj / fmaf(s[j], a.rs, a.eps)));
    }
    put4<ALL, ONCE>(x.p, at, x.n, p);
    if (x.p16) put4<ALL, ONCE>(x.p16, at, x.n, p);
    if constexpr (LOW) {
      e = encode4(m, s, [&](int j) { return hash32(a.key + (uint32_t)at + j); }, qm, qs);
      put4<ALL, ONCE>((uint8_t*)x.m, at, x.n, qm);
      put4<ALL, ONCE>((uint8_t*)x.v, at, x.n, qs);
      if ((threadIdx.x & 31) == 0) *(uint16_t*)(x.e + at / OB * 2) = (uint16_t)e;
    } else {
      put4<ALL, ONCE>((float*)x.m, at, x.n, m);
      put4<ALL, ONCE>((float*)x.v, at, x.n, v);
    }
  }
};

template <typename G, bool LOW, bool ONCE>
__global__ __launch_bounds__(256) void k_adamw(const OptimTable t, const AdamwArgs a) {
  Step q{1.f, a.c1, a.c2, 0.f, 0.f, a.eps, 0.f, 0u};
  if (a.stats) {
    if (!(fabsf(a.stats[0]) <= 3.4028234663852886e38f)) return;  // not a finite norm: no step
    q.factor = a.stats[1];
  }
  const int i = tensor_of(t, blockIdx.x);
  const OptimTensor x = t.t[i];
  const int n_step = a.step_at ? max(*a.step_at, 1) : a.step;
  const float lr = (a.lr_at ? *a.lr_at : a.lr) * x.lr_scale;
  q.up = lr / -expm1f((float)n_step * a.ln_b1);
  q.rs = 1.f / sqrtf(-expm1f((float)n_step * a.ln_b2));
  q.decay = lr * x.weight_decay;
  q.key = hash32(hash32(hash32(a.seed) + (uint32_t)n_step) ^ (t.index + i));
  const int64_t base = (int64_t)(blockIdx.x - t.first[i]) * OPTIM_PIECE + threadIdx.x * 4;
  constexpr int K = OPTIM_PIECE / 1024;
  if (base - threadIdx.x * 4 + OPTIM_PIECE <= x.n) {
    Four<G, LOW, true, ONCE> f[K];
#pragma unroll
    for (int k = 0; k < K; ++k) f[k].load(x, base + k * 1024);
#pragma unroll
    for (int k = 0; k < K; ++k) f[k].step(x, base + k * 1024, q);
  } else {  // (a block's lanes go on together: its maximum is theirs)
    for (int k = 0; k < K; ++k) {
      const int64_t at = base + k * 1024;
      if (at - (threadIdx.x & 31) * 4 >= x.n) break;
      Four<G, LOW, false, false> f;
      f.load(x, at);
      f.step(x, at, q);
    }
  }
}

// 8-bit states to fp32 (p: m's values, g: v's), and back, rounded to nearest
template <bool ALL>
struct Unpack4 {
  uint32_t qm, qs, e;
  __device__ __forceinline__ void load(const OptimTensor& x, int64_t at) {
    qm = get4<ALL>((const uint8_t*)x.m, at, x.n);
    qs = get4<ALL>((const uint8_t*)x.v, at, x.n);
    e = *(const uint16_t*)(x.e + at / OB * 2);
  }
  __device__ __forceinline__ void store(const OptimTensor& x, int64_t at) {
    f32x4_t m, s;
    decode4(qm, qs, e, m, s);
    put4<ALL>(x.p, at, x.n, m);
    put4<ALL>((float*)x.g, at, x.n, s * s);
  }
};
template <bool ALL>
struct Pack4 {
  f32x4_t m, s;
  __device__ __forceinline__ void load(const OptimTensor& x, int64_t at) {
    m = get4<ALL>(x.p, at, x.n);
    s = get4<ALL>((const float*)x.g, at, x.n);
  }
  __device__ __forceinline__ void store(const OptimTensor& x, int64_t at) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = sqrtf(s[j]);
    uint32_t qm, qs;
    const uint32_t e = encode4(m, s, [](int) { return 0x80008000u; }, qm, qs);
    put4<ALL>((uint8_t*)x.m, at, x.n, qm);
    put4<ALL>((uint8_t*)x.v, at, x.n, qs);
    if ((threadIdx.x & 31) == 0) *(uint16_t*)(x.e + at / OB * 2) = (uint16_t)e;
  }
};
// (two workgroups a piece: unpacking 266 M values takes 473 us with one, 451 with two)
template <template <bool> class F>
__global__ __launch_bounds__(256) void k_adamw_convert(const OptimTable t) {
  const uint32_t piece = blockIdx.x >> 1;
  const int i = tensor_of(t, piece);
  const OptimTensor x = t.t[i];
  constexpr int HALF = OPTIM_PIECE / 2, K = HALF / 1024;
  const int64_t start = (int64_t)(piece - t.first[i]) * OPTIM_PIECE + (blockIdx.x & 1) * HALF, base = start + threadIdx.x * 4;
  if (start + HALF <= x.n) {
    F<true> f[K];
#pragma unroll
    for (int k = 0; k < K; ++k) f[k].load(x, base + k * 1024);
#pragma unroll
    for (int k = 0; k < K; ++k) f[k].store(x, base + k * 1024);
  } else {  // (a block's lanes go on together: its maximum is theirs)
    for (int k = 0; k < K; ++k) {
      const int64_t at = base + k * 1024;
      if (at - (threadIdx.x & 31) * 4 >= x.n) break;
      F<false> f;
      f.load(x, at);
      f.store(x, at);
    }
  }
}

// ------------------------------------------------------------------ the gradients' norm
constexpr int GRAD_WGS = 2048;

template <int CTRL>
__device__ __forceinline__ double dpp_add64(double v) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  const u32x2 o = {(uint32_t)__builtin_amdgcn_update_dpp(0, w.x, CTRL, 0xf, 0xf, true),
                   (uint32_t)__builtin_amdgcn_update_dpp(0, w.y, CTRL, 0xf, 0xf, true)};
  return v + __builtin_bit_cast(double, o);
}
__device__ __forceinline__ double lane64(double v, int l) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  const u32x2 o = {(uint32_t)__builtin_amdgcn_readlane(w.x, l), (uint32_t)__builtin_amdgcn_readlane(w.y, l)};
  return __builtin_bit_cast(double, o);
}
__device__ __forceinline__ double wave_sum64(double v) {
  v = dpp_add64<0xB1>(v);   // lane ^ 1
  v = dpp_add64<0x4E>(v);   // lane ^ 2
  v = dpp_add64<0x141>(v);  // the other half of 8
  v = dpp_add64<0x140>(v);  // the other half of 16
  return (lane64(v, 0) + lane64(v, 16)) + (lane64(v, 32) + lane64(v, 48));
}

// Sums of squares in 64 bits: no gradient that fp32 holds overflows them, and the
// order, which the launch fixes, shows in no digit of the norm.  266 M bf16 values 79 us, 6.7 TB/s
// (with 1024 workgroups 103).
template <typename G, bool ONCE>
__global__ __launch_bounds__(256) void k_grad_squares(const GradTable t, double* __restrict__ part) {
  __shared__ double w[4];
  double s = 0.0;
  for (uint32_t piece = blockIdx.x; piece < t.first[t.count]; piece += gridDim.x) {
    const int i = tensor_of(t, piece);
    const int64_t n = t.t[i].n, base = (int64_t)(piece - t.first[i]) * OPTIM_PIECE;
    const G* p = (const G*)t.t[i].g;
    f32x4_t g[OPTIM_PIECE / 1024];
    if (base + OPTIM_PIECE <= n) {
#pragma unroll
      for (int k = 0; k < OPTIM_PIECE / 1024; ++k) g[k] = get4<true, ONCE>(p, base + k * 1024 + threadIdx.x * 4, n);
    } else {
#pragma unroll
      for (int k = 0; k < OPTIM_PIECE / 1024; ++k) g[k] = get4<false>(p, base + k * 1024 + threadIdx.x * 4, n);
    }
#pragma unroll
    for (int k = 0; k < OPTIM_PIECE / 1024; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = fma((double)g[k][j], (double)g[k][j], s);
  }
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (w[0] + w[1]) + (w[2] + w[3]);
}

// norm = scale sqrt(sum), factor = scale min(1, most / norm); the step counts if the norm is a number
__global__ __launch_bounds__(512) void k_grad_norm(const double* __restrict__ part, int n, float grad_scale, float most,
                                                   float* __restrict__ stats, int32_t* __restrict__ step) {
  __shared__ double w[8];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 4 * 512) {
    double v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + k * 512 < n ? part[i + k * 512] : 0.0;
    s += (v[0] + v[1]) + (v[2] + v[3]);
  }
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
  const double norm = fabs((double)grad_scale) * sqrt(s);
  stats[0] = (float)norm;
  stats[1] = (float)(norm > (double)most ? (double)grad_scale * ((double)most / norm) : (double)grad_scale);
  if (step && (float)norm <= 3.4028234663852886e38f) *step += 1;
}

}  // namespace

int64_t optim_pieces(int64_t n) { return (n + OPTIM_PIECE - 1) / OPTIM_PIECE; }
int grad_norm_parts(int64_t pieces) { return (int)(pieces < GRAD_WGS ? pieces : GRAD_WGS); }

hipError_t launch_grad_squares(const GradTable& t, int g_f32, int once, double* part, hipStream_t s) {
  void (*f)(GradTable, double*) = g_f32 ? once ? k_grad_squares<float, true> : k_grad_squares<float, false>
                                         : once ? k_grad_squares<bf16_t, true> : k_grad_squares<bf16_t, false>;
  hipLaunchKernelGGL(f, dim3(grad_norm_parts(t.first[t.count])), dim3(256), 0, s, t, part);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const double* part, int n, float grad_scale, float max_norm, float* stats, int32_t* step,
                            hipStream_t s) {
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(512), 0, s, part, n, grad_scale, max_norm, stats, step);
  return hipGetLastError();
}

template <typename G, bool LOW>
static hipError_t run_adamw(const OptimTable& t, const AdamwArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((a.once ? k_adamw<G, LOW, true> : k_adamw<G, LOW, false>), dim3(t.first[t.count]), dim3(256), 0, s, t, a);
  return hipGetLastError();
}
hipError_t launch_adamw(const OptimTable& t, const AdamwArgs& a, hipStream_t s) {
  if (a.low) return a.g_f32 ? run_adamw<float, true>(t, a, s) : run_adamw<bf16_t, true>(t, a, s);
  return a.g_f32 ? run_adamw<float, false>(t, a, s) : run_adamw<bf16_t, false>(t, a, s);
}

hipError_t launch_adamw_unpack(const OptimTable& t, hipStream_t s) {
  hipLaunchKernelGGL(k_adamw_convert<Unpack4>, dim3(2 * t.first[t.count]), dim3(256), 0, s, t);
  return hipGetLastError();
}

hipError_t launch_adamw_pack(const OptimTable& t, hipStream_t s) {
  hipLaunchKernelGGL(k_adamw_convert<Pack4>, dim3(2 * t.first[t.count]), dim3(256), 0, s, t);
  return hipGetLastError();
}

}  // namespace mapl
