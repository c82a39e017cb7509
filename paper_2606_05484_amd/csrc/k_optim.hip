// The optimizer's step over all tensors of a stage: the norm of their gradients
// with the factor that clips it, and AdamW with states in fp32 or in 8 bits:
//   g' = factor g,  m <- m + (1 - b1)(g' - m),  v <- v + (1 - b2)(g'^2 - v)
//   p <- p - (lr wd p + lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps))
// A launch takes up to OPTIM_TENSORS tensors from its arguments and cuts them in
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
// Bound by HBM: fp32 states 30 bytes a value (bf16 gradients and copy), 8 bits 16.06.
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

// the tensor that a piece belongs to (uniform)
__device__ __forceinline__ int tensor_of(const OptimTable& t, uint32_t piece) {
  int at = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1)
    if (at + step < t.count && t.first[at + step] <= piece) at += step;
  return at;
}

// values i .. i + 7 of n (those past n are zeros), and back
__device__ __forceinline__ void get8(const float* p, int64_t i, int64_t n, float (&f)[8]) {
  if (i + 8 <= n) {
    const f32x4_t a = *(const f32x4_t*)(p + i), b = *(const f32x4_t*)(p + i + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = a[j], f[4 + j] = b[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = i + j < n ? p[i + j] : 0.f;
  }
}
__device__ __forceinline__ void get8(const bf16_t* p, int64_t i, int64_t n, float (&f)[8]) {
  if (i + 8 <= n) {
    const u32x4 w = *(const u32x4*)(p + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(w[j] << 16), f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = i + j < n ? bf2f(p[i + j]) : 0.f;
  }
}
__device__ __forceinline__ uint2 get8b(const uint8_t* p, int64_t i, int64_t n) {
  if (i + 8 <= n) return *(const uint2*)(p + i);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (i + j < n) w[j >> 2] |= (uint32_t)p[i + j] << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void put8(float* p, int64_t i, int64_t n, const float (&f)[8]) {
  if (i + 8 <= n) {
    *(f32x4_t*)(p + i) = f32x4_t{f[0], f[1], f[2], f[3]};
    *(f32x4_t*)(p + i + 4) = f32x4_t{f[4], f[5], f[6], f[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < n) p[i + j] = f[j];
  }
}
__device__ __forceinline__ void put8(bf16_t* p, int64_t i, int64_t n, const float (&f)[8]) {
  if (i + 8 <= n) {
    *(u32x4*)(p + i) = u32x4{pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]), pack_bf2(f[4], f[5]), pack_bf2(f[6], f[7])};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < n) p[i + j] = (bf16_t)f2bf(f[j]);
  }
}
__device__ __forceinline__ void put8b(uint8_t* p, int64_t i, int64_t n, uint2 w) {
  if (i + 8 <= n) {
    *(uint2*)(p + i) = w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < n) p[i + j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
  }
}

// ------------------------------------------------------------------ 8-bit states
__device__ __forceinline__ float pow2_byte(int b) { return __uint_as_float((uint32_t)b << 23); }  // 2^(b - 127)

// m and s of eight codes; 255 stands for NaNs, and bytes below 24 are not made (0 before the first step)
__device__ __forceinline__ void decode8(uint2 qm, uint2 qs, uint32_t e, float (&m)[8], float (&s)[8]) {
  const uint32_t em = e & 255u, es = e >> 8;
  const float um = em == 255 ? __builtin_nanf("") : em < 24 ? 0.f : pow2_byte(em - 8);
  const float us = es == 255 ? __builtin_nanf("") : es < 24 ? 0.f : pow2_byte(es);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t w = h ? qm.y : qm.x, z = h ? qs.y : qs.x;
    const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    m[4 * h] = a[0] * um, m[4 * h + 1] = a[1] * um, m[4 * h + 2] = b[0] * um, m[4 * h + 3] = b[1] * um;
#pragma unroll
    for (int j = 0; j < 4; ++j)  // a code's bits are those of a number 2^112 times smaller (subnormal below 16)
      s[4 * h + j] = __uint_as_float(((z >> (8 * j)) & 255u) << 19) * 0x1p112f * us;
  }
}

// the largest of the 16 lanes that hold a block of 128
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true));
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

// codes and exponent bytes of a lane's eight values of m and s (s >= 0, or NaN)
template <typename Noise>
__device__ __forceinline__ uint32_t encode8(const float (&m)[8], const float (&s)[8], Noise noise, uint2& qm, uint2& qs) {
  uint32_t am = 0, as = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    am = max(am, __float_as_uint(m[j]) & 0x7fffffffu);
    as = max(as, __float_as_uint(s[j]) & 0x7fffffffu);
  }
  const uint32_t em = exponent_byte(block_max(am), 0x1fffff), es = exponent_byte(block_max(as), 0x7ffff);
  const float um = em == 255 ? 0.f : pow2_byte(262 - em), us = es >= 254 ? es == 255 ? 0.f : 0x1p-127f : pow2_byte(254 - es);
  uint32_t wm[2] = {0, 0}, ws[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t r = noise(j);
    const float a = em == 255 ? 0.f : fabsf(m[j]), b = es == 255 ? 0.f : s[j];
    uint32_t cm = code_of<3, -6>(a * um, r & 0xffffu), cs = code_of<4, -14>(b * us, r >> 16);
    cm |= (__float_as_uint(m[j]) >> 24) & 128u;
    cs = max(cs, b > 0.f ? 1u : 0u);
    wm[j >> 2] |= cm << (8 * (j & 3));
    ws[j >> 2] |= cs << (8 * (j & 3));
  }
  qm = make_uint2(wm[0], wm[1]), qs = make_uint2(ws[0], ws[1]);
  return em | es << 8;
}

// ------------------------------------------------------------------ AdamW
// the states' step, every operation rounded on its own; g is the clipped gradient
__device__ __forceinline__ void state_update(float g, float c1, float c2, float& m, float& v) {
#pragma clang fp contract(off)
  m = m + (g - m) * c1;
  v = v + (g * g - v) * c2;
}

struct Step {
  float factor, a, rs, decay, eps;  // lr / (1 - b1^t), (1 - b2^t)^-1/2, lr wd
};

template <typename G, bool LOW>
__global__ __launch_bounds__(256) void k_adamw(const OptimTable t, const AdamwArgs a) {
  float factor = 1.f;
  if (a.stats) {
    if (!(fabsf(a.stats[0]) <= 3.4028234663852886e38f)) return;  // not a finite norm: no step
    factor = a.stats[1];
  }
  const int i = tensor_of(t, blockIdx.x);
  const OptimTensor& x = t.t[i];
  const int n_step = a.step_at ? max(*a.step_at, 1) : a.step;
  const float lr = (a.lr_at ? *a.lr_at : a.lr) * x.lr_scale;
  const float up = lr / -expm1f((float)n_step * a.ln_b1), rs = 1.f / sqrtf(-expm1f((float)n_step * a.ln_b2));
  const float decay = lr * x.weight_decay;
  const uint32_t key = hash32(hash32(hash32(a.seed) + (uint32_t)n_step) ^ (t.index + i));
  const int64_t n = x.n, base = (int64_t)(blockIdx.x - t.first[i]) * OPTIM_PIECE;
  for (int64_t at = base + threadIdx.x * 8; at < base + OPTIM_PIECE && at - (threadIdx.x & 15) * 8 < n; at += 256 * 8) {
    float p[8], g[8], m[8], v[8], s[8];
    get8(x.p, at, n, p);
    get8((const G*)x.g, at, n, g);
    if constexpr (LOW) {
      const uint2 qm = get8b((const uint8_t*)x.m, at, n), qs = get8b((const uint8_t*)x.v, at, n);
      decode8(qm, qs, *(const uint16_t*)(x.e + at / OB * 2), m, s);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = s[j] * s[j];
    } else {
      get8((const float*)x.m, at, n, m);
      get8((const float*)x.v, at, n, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      state_update(g[j] * factor, a.c1, a.c2, m[j], v[j]);
      s[j] = LOW ? sqrtf(v[j]) : __builtin_amdgcn_sqrtf(v[j]);
      p[j] -= fmaf(decay, p[j], up * (m[j] / fmaf(s[j], rs, a.eps)));
    }
    put8(x.p, at, n, p);
    if (x.p16) put8(x.p16, at, n, p);
    if constexpr (LOW) {
      uint2 qm, qs;
      const uint32_t e = encode8(m, s, [&](int j) { return hash32(key + (uint32_t)at + j); }, qm, qs);
      put8b((uint8_t*)x.m, at, n, qm);
      put8b((uint8_t*)x.v, at, n, qs);
      if ((threadIdx.x & 15) == 0) *(uint16_t*)(x.e + at / OB * 2) = (uint16_t)e;
    } else {
      put8((float*)x.m, at, n, m);
      put8((float*)x.v, at, n, v);
    }
  }
}

// 8-bit states to fp32 (p: m's values, g: v's), and back, rounded to nearest
template <bool PACK>
__global__ __launch_bounds__(256) void k_adamw_convert(const OptimTable t) {
  const int i = tensor_of(t, blockIdx.x);
  const OptimTensor& x = t.t[i];
  const int64_t n = x.n, base = (int64_t)(blockIdx.x - t.first[i]) * OPTIM_PIECE;
  for (int64_t at = base + threadIdx.x * 8; at < base + OPTIM_PIECE && at - (threadIdx.x & 15) * 8 < n; at += 256 * 8) {
    float m[8], s[8];
    if constexpr (PACK) {
      get8(x.p, at, n, m);
      get8((const float*)x.g, at, n, s);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = sqrtf(s[j]);
      uint2 qm, qs;
      const uint32_t e = encode8(m, s, [](int) { return 0x80008000u; }, qm, qs);
      put8b((uint8_t*)x.m, at, n, qm);
      put8b((uint8_t*)x.v, at, n, qs);
      if ((threadIdx.x & 15) == 0) *(uint16_t*)(x.e + at / OB * 2) = (uint16_t)e;
    } else {
      decode8(get8b((const uint8_t*)x.m, at, n), get8b((const uint8_t*)x.v, at, n), *(const uint16_t*)(x.e + at / OB * 2), m, s);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] *= s[j];
      put8(x.p, at, n, m);
      put8((float*)x.g, at, n, s);
    }
  }
}

// ------------------------------------------------------------------ the gradients' norm
constexpr int GRAD_WGS = 1024;

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
  return v;
}

// Sums of squares in 64 bits: no gradient that fp32 holds overflows them, and the
// order, which the launch fixes, shows in no digit of the norm.
template <typename G>
__global__ __launch_bounds__(256) void k_grad_squares(const OptimTable t, double* __restrict__ part) {
  __shared__ double w[4];
  double s = 0.0;
  for (uint32_t piece = blockIdx.x; piece < t.first[t.count]; piece += gridDim.x) {
    const int i = tensor_of(t, piece);
    const int64_t n = t.t[i].n, base = (int64_t)(piece - t.first[i]) * OPTIM_PIECE;
#pragma unroll
    for (int k = 0; k < OPTIM_PIECE / 2048; ++k) {
      float g[8];
      get8((const G*)t.t[i].g, base + k * 2048 + threadIdx.x * 8, n, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fma((double)g[j], (double)g[j], s);
    }
  }
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (w[0] + w[1]) + (w[2] + w[3]);
}

// norm = scale sqrt(sum), factor = scale min(1, most / norm); the step counts if the norm is a number
__global__ __launch_bounds__(1024) void k_grad_norm(const double* __restrict__ part, int n, float grad_scale, float most,
                                                    float* __restrict__ stats, int32_t* __restrict__ step) {
  __shared__ double w[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < 16; ++i) s += w[i];
  const double norm = fabs((double)grad_scale) * sqrt(s);
  stats[0] = (float)norm;
  stats[1] = (float)(norm > (double)most ? (double)grad_scale * ((double)most / norm) : (double)grad_scale);
  if (step && (float)norm <= 3.4028234663852886e38f) *step += 1;
}

}  // namespace

int64_t optim_pieces(int64_t n) { return (n + OPTIM_PIECE - 1) / OPTIM_PIECE; }
int grad_norm_parts(int64_t pieces) { return (int)(pieces < GRAD_WGS ? pieces : GRAD_WGS); }

hipError_t launch_grad_squares(const OptimTable& t, int g_f32, double* part, hipStream_t s) {
  const dim3 grid(grad_norm_parts(t.first[t.count]));
  if (g_f32)
    hipLaunchKernelGGL(k_grad_squares<float>, grid, dim3(256), 0, s, t, part);
  else
    hipLaunchKernelGGL(k_grad_squares<bf16_t>, grid, dim3(256), 0, s, t, part);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const double* part, int n, float grad_scale, float max_norm, float* stats, int32_t* step,
                            hipStream_t s) {
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(1024), 0, s, part, n, grad_scale, max_norm, stats, step);
  return hipGetLastError();
}

hipError_t launch_adamw(const OptimTable& t, const AdamwArgs& a, hipStream_t s) {
  void (*f)(OptimTable, AdamwArgs) = a.g_f32 ? a.low ? k_adamw<float, true> : k_adamw<float, false>
                                             : a.low ? k_adamw<bf16_t, true> : k_adamw<bf16_t, false>;
  hipLaunchKernelGGL(f, dim3(t.first[t.count]), dim3(256), 0, s, t, a);
  return hipGetLastError();
}

hipError_t launch_adamw_unpack(const OptimTable& t, hipStream_t s) {
  hipLaunchKernelGGL(k_adamw_convert<false>, dim3(t.first[t.count]), dim3(256), 0, s, t);
  return hipGetLastError();
}

hipError_t launch_adamw_pack(const OptimTable& t, hipStream_t s) {
  hipLaunchKernelGGL(k_adamw_convert<true>, dim3(t.first[t.count]), dim3(256), 0, s, t);
  return hipGetLastError();
}

}  // namespace mapl
