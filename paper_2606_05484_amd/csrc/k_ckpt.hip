// Activations kept in 8 bits between forward and backward.  Blocks of 32
// tokens of one channel share a power-of-two scale: with a the block's largest
// magnitude and e = floor(log2 a) (at least -120), the exponent byte is
// e + 127 and the values are q = rne(X 2^(6 - e)) in [-127, 127], standing for
// q 2^(e - 6); a block with a NaN or an infinity has the byte 255 and stands
// for NaNs.  Layout q [ceil(T / 32)][d][32], exponents [ceil(T / 32)][d];
// tokens past T are zeros.  A power of two makes q exact to define (no
// reciprocal's rounding decides a value) and q 2^(e - 6) exact in bf16; the
// run of 32 tokens is the contraction's direction in the backward's dU.
#include "common.hpp"
#include "kernels.hpp"

namespace mapl {

namespace {

constexpr int CK_B = 32;

// exponent byte of a block from the largest magnitude's bits (fp32, sign off;
// NaN and infinity are the largest of all)
__device__ __forceinline__ uint32_t ck_byte(uint32_t amax) {
  const uint32_t e = amax >> 23;
  return e < 7 ? 7u : e;  // 255 for NaN and infinity
}
__device__ __forceinline__ float ck_unit(uint32_t byte) { return __uint_as_float((byte - 6) << 23); }       // 2^(e-6)
__device__ __forceinline__ float ck_inverse(uint32_t byte) { return __uint_as_float((260 - byte) << 23); }  // 2^(6-e)

__device__ __forceinline__ float ck_load(const float* p) { return *p; }
__device__ __forceinline__ float ck_load(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void ck_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void ck_store(bf16_t* p, float v) { *p = (bf16_t)f2bf(v); }

// one thread per block of 32 tokens
template <typename X>
__global__ __launch_bounds__(256) void k_ckpt_pack(const X* __restrict__ x, int64_t T, int d, uint4* __restrict__ q,
                                                   uint8_t* __restrict__ e) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t b = i / d;
  const int c = (int)(i - b * d);
  if (b * CK_B >= T) return;
  float v[CK_B];
  uint32_t amax = 0;
#pragma unroll
  for (int t = 0; t < CK_B; ++t) {
    v[t] = b * CK_B + t < T ? ck_load(x + (b * CK_B + t) * d + c) : 0.f;
    amax = max(amax, __float_as_uint(v[t]) & 0x7fffffffu);
  }
  const uint32_t byte = ck_byte(amax);
  const float inv = byte == 255 ? 0.f : ck_inverse(byte);
  uint32_t w[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    w[g] = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float f = byte == 255 ? 0.f : fminf(fmaxf(rintf(v[4 * g + k] * inv), -127.f), 127.f);
      w[g] |= ((uint32_t)(int)f & 255u) << (8 * k);
    }
  }
  q[2 * i] = make_uint4(w[0], w[1], w[2], w[3]);
  q[2 * i + 1] = make_uint4(w[4], w[5], w[6], w[7]);
  e[i] = (uint8_t)byte;
}

template <typename X>
__global__ __launch_bounds__(256) void k_ckpt_unpack(const uint4* __restrict__ q, const uint8_t* __restrict__ e, int64_t T,
                                                     int d, X* __restrict__ x) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t b = i / d;
  const int c = (int)(i - b * d);
  if (b * CK_B >= T) return;
  const uint4 a0 = q[2 * i], a1 = q[2 * i + 1];
  const uint32_t w[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
  const uint32_t byte = e[i];
  const float unit = byte == 255 ? __builtin_nanf("") : ck_unit(byte);
#pragma unroll
  for (int t = 0; t < CK_B; ++t)
    if (b * CK_B + t < T) ck_store(x + (b * CK_B + t) * d + c, (float)(int8_t)(w[t >> 2] >> (8 * (t & 3))) * unit);
}

}  // namespace

hipError_t launch_ckpt_pack(const void* X, int f32, int64_t T, int d, void* q, uint8_t* e, hipStream_t s) {
  const int64_t n = (T + CK_B - 1) / CK_B * d;
  const dim3 grid((unsigned)((n + 255) / 256));
  if (f32)
    hipLaunchKernelGGL(k_ckpt_pack<float>, grid, dim3(256), 0, s, (const float*)X, T, d, (uint4*)q, e);
  else
    hipLaunchKernelGGL(k_ckpt_pack<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)X, T, d, (uint4*)q, e);
  return hipGetLastError();
}

hipError_t launch_ckpt_unpack(const void* q, const uint8_t* e, int64_t T, int d, void* X, int f32, hipStream_t s) {
  const int64_t n = (T + CK_B - 1) / CK_B * d;
  const dim3 grid((unsigned)((n + 255) / 256));
  if (f32)
    hipLaunchKernelGGL(k_ckpt_unpack<float>, grid, dim3(256), 0, s, (const uint4*)q, e, T, d, (float*)X);
  else
    hipLaunchKernelGGL(k_ckpt_unpack<bf16_t>, grid, dim3(256), 0, s, (const uint4*)q, e, T, d, (bf16_t*)X);
  return hipGetLastError();
}

}  // namespace mapl
