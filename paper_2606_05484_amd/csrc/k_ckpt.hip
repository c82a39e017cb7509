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

__device__ __forceinline__ void ck_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void ck_store(bf16_t* p, float v) { *p = (bf16_t)f2bf(v); }

// The 32 bytes of a block from its values (fp32 bits): |v| 2^(6-e) is below
// 128, and adding 1.5 2^23 rounds it to an integer (ties to even) whose two's
// complement is the sum's low byte; 128 itself is held at 127 before the byte
// is taken.
__device__ __forceinline__ void ck_block(const uint32_t (&v)[CK_B], uint32_t amax, uint4* q, uint32_t& byte) {
  byte = ck_byte(amax);
  const float inv = ck_inverse(byte == 255 ? 127u : byte), magic = 12582912.f;
  uint32_t w[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      r[k] = __float_as_uint(__builtin_amdgcn_fmed3f(fmaf(__uint_as_float(v[4 * g + k]), inv, magic), magic - 127.f,
                                                     magic + 127.f));
    const uint32_t lo = __builtin_amdgcn_perm(r[1], r[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(r[3], r[2], 0x0c0c0400u);
    w[g] = byte == 255 ? 0u : lo | (hi << 16);
  }
  q[0] = make_uint4(w[0], w[1], w[2], w[3]);
  q[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// One lane per 4 bytes of a token's row (two bf16 channels, or one fp32), its
// 32 tokens loaded at once: 256 bytes of a row per wave and load, 32 loads in
// flight.  PAIR: bf16.
template <bool PAIR>
__global__ __launch_bounds__(128) void k_ckpt_pack(const uint32_t* __restrict__ x, int64_t T, int cols, uint4* __restrict__ q,
                                                   uint8_t* __restrict__ e) {
  const int64_t i = (int64_t)blockIdx.x * 128 + threadIdx.x;
  const int64_t b = i / cols;
  const int c = (int)(i - b * cols);
  if (b * CK_B >= T) return;
  const uint32_t* p = x + b * CK_B * cols + c;
  uint32_t v[CK_B];
  if ((b + 1) * CK_B <= T) {
#pragma unroll
    for (int t = 0; t < CK_B; ++t) v[t] = p[(int64_t)t * cols];
  } else {
#pragma unroll
    for (int t = 0; t < CK_B; ++t) v[t] = b * CK_B + t < T ? p[(int64_t)t * cols] : 0u;
  }
  uint32_t byte;
  if constexpr (PAIR) {
    uint32_t lo[CK_B], a0 = 0, a1 = 0;
#pragma unroll
    for (int t = 0; t < CK_B; ++t) {
      lo[t] = v[t] << 16;
      v[t] &= 0xffff0000u;
      a0 = max(a0, lo[t] & 0x7fffffffu);
      a1 = max(a1, v[t] & 0x7fffffffu);
    }
    uint32_t byte1;
    ck_block(lo, a0, q + 4 * i, byte);
    ck_block(v, a1, q + 4 * i + 2, byte1);
    ((uint16_t*)e)[i] = (uint16_t)(byte | byte1 << 8);
  } else {
    uint32_t a = 0;
#pragma unroll
    for (int t = 0; t < CK_B; ++t) a = max(a, v[t] & 0x7fffffffu);
    ck_block(v, a, q + 2 * i, byte);
    e[i] = (uint8_t)byte;
  }
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
  const int cols = f32 ? d : d / 2;
  const int64_t n = (T + CK_B - 1) / CK_B * cols;
  const dim3 grid((unsigned)((n + 127) / 128));
  if (f32)
    hipLaunchKernelGGL(k_ckpt_pack<false>, grid, dim3(128), 0, s, (const uint32_t*)X, T, cols, (uint4*)q, e);
  else
    hipLaunchKernelGGL(k_ckpt_pack<true>, grid, dim3(128), 0, s, (const uint32_t*)X, T, cols, (uint4*)q, e);
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
