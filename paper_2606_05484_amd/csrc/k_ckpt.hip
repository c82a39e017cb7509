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
// 2^(e-6); NaN for 255.  (Bytes below 7 are not made by the packing and count as 0.)
__device__ __forceinline__ float ck_unit(uint32_t byte) {
  return byte == 255 ? __builtin_nanf("") : byte < 7 ? 0.f : __uint_as_float((byte - 6) << 23);
}
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
// flight.  PAIR: bf16.  Bound by HBM: [32768, 2048] bf16, 203 MB, 45 us, 4.5 TB/s.
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

// One lane per block: 32 bytes and an exponent in, a channel of 32 tokens out
// (a wave's stores are runs of 64 channels).  Bound by HBM: [32768, 2048] to bf16, 203 MB, 32 us, 6.4
// TB/s right after the pack (a part of q still lies in the last-level cache).
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
  const float unit = ck_unit(byte);
#pragma unroll
  for (int t = 0; t < CK_B; ++t)
    if (b * CK_B + t < T) ck_store(x + (b * CK_B + t) * d + c, (float)(int8_t)(w[t >> 2] >> (8 * (t & 3))) * unit);
}

// ------------------------------------------------- weight gradient from a checkpoint
// part[s][m][n] = sum over the tokens t of split s of Xq[t][m] Q[t][n], Xq
// from its checkpoint.  A lane's fragment of the matrix instruction is eight
// consecutive tokens of one channel, so the checkpoint's bytes go straight
// from memory to registers in operand order: 16 bytes are a lane's tokens of
// two k-steps (tokens 16 h + 8 step .. +7 of the block, h = lane / 32; Q's
// fragments take the same tokens), one exponent byte scales them, and
// byte -> fp32 -> fma -> bf16 is exact; the operand is half of Xq so that the
// fma's 255 2^121 and 128 2^121 stay finite, and the sums are doubled at the
// end.  The anchor rows come as bf16 in the same order (k_prep.hip).  Q's
// 64-token stages are copied into LDS as they are and read transposed
// (tr_frag).
// A workgroup owns 128 rows x BN columns with two groups of four waves
// (2 x 2 waves of 64 x BN / 2): group g takes the g-th 32-token block of every
// stage, so two waves per SIMD hide each other's waits with no more operand
// traffic; the groups' sums meet in LDS at the end.  T = 32768, d = 2048, r = 256, 128
// anchors: 47 us, 0.78 PFLOP/s; of these about 35 are its stages (1.1 us each, no
// one of conversion, products, LDS reads or loads alone: without any one of them 4-8 us
// less), the rest the partial sums (33 MB) and the start.  A wave converts the next
// stage's bytes under the first k-step's products and reads the next stage's first
// fragments under the second's.
constexpr int W8_BM = 128, W8_KT = 64, W8_THREADS = 512, W8_NS = 4;
typedef __attribute__((address_space(3))) void* w8_lds_ptr;

// bf16 pairs of the four values of w (biased bytes, q + 128): q unit, off = -128 unit
__device__ __forceinline__ void w8_convert(uint32_t w, float unit, float off, uint32_t& lo, uint32_t& hi) {
  const float f0 = (float)(w & 255u), f1 = (float)((w >> 8) & 255u), f2 = (float)((w >> 16) & 255u), f3 = (float)(w >> 24);
  lo = pack_bf2(fmaf(f0, unit, off), fmaf(f1, unit, off));
  hi = pack_bf2(fmaf(f2, unit, off), fmaf(f3, unit, off));
}

// What a lane loads of a stage for one 32-row block: 16 bytes and the four
// exponents that its own is among, or (ANCH) 16 bf16 values.
template <bool ANCH>
struct W8Raw {
  u32x4 v;
  uint32_t e;
};
template <>
struct W8Raw<true> {
  u32x4 v, w;
};

template <int BN, bool ANCH>
__device__ __forceinline__ void w8_run(const Wgrad8Args& g, char* smem, int split, int m0, int n0, int wave, int lane) {
  constexpr int FM = 2, FN = BN / 64;
  constexpr int QCPR = BN / 8, QBYTES = W8_KT * BN * 2;
  constexpr int QBLK = QBYTES / 1024 / 8;  // 1 KiB DMA blocks per wave per stage
  const int grp = wave >> 2, wm = (wave >> 1) & 1, wn = wave & 1, half = lane >> 5;
  const int64_t t0 = (int64_t)split * g.tokens_per_split;
  const int nt = (int)min((int64_t)g.tokens_per_split, g.T - t0);  // >= 1
  const int KS = (nt + W8_KT - 1) / W8_KT, nb = (nt + CK_B - 1) / CK_B;
  const int rows = ANCH ? g.ka : g.d;  // of P

  // Q: lane i of block b writes row b (64 / QCPR) + i / QCPR, chunk i % QCPR (swizzled)
  uint32_t q_off[QBLK];
#pragma unroll
  for (int j = 0; j < QBLK; ++j) {
    const int row = (wave * QBLK + j) * (64 / QCPR) + lane / QCPR;
    q_off[j] = (uint32_t)row * (uint32_t)g.ldq * 2u + (uint32_t)(n0 + 8 * ((lane % QCPR) ^ wg_sw(row, QCPR))) * 2u;
  }
  const bf16_t* qp = g.Q + t0 * g.ldq;
  // (past the last stage zeros: a load under a condition would have the
  // compiler's waits for P's loads, which count what was issued after them,
  // drain these as well)
  auto issue = [&](int s) {
    const int n = max(0, min(W8_KT, nt - s * W8_KT));
    const __amdgpu_buffer_rsrc_t rq = uniform_rsrc(qp + (int64_t)s * W8_KT * g.ldq, (uint32_t)n * (uint32_t)g.ldq * 2u);
    char* dst = smem + (s % W8_NS) * QBYTES + wave * QBLK * 1024;
#pragma unroll
    for (int j = 0; j < QBLK; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (w8_lds_ptr)(dst + j * 1024), 16, q_off[j], 0, 0, 0);
    asm volatile("" ::: "memory");
  };

  // the wave's part of P in stage s: rows m0 + 64 wm + 32 i + lane % 32 (zeros
  // past P's rows and past the split's blocks).  Every call issues 2 FM
  // loads: the waits below count on it.
  const uint32_t ch = m0 + wm * 64 + (lane & 31);
  const int64_t b0 = t0 / CK_B + grp;
  auto fetch = [&](int s, W8Raw<ANCH> (&r)[FM]) {
    const bool any = 2 * s + grp < nb;
    constexpr int B = ANCH ? 2 * CK_B : CK_B;  // bytes of a row's block
    const char* base = (ANCH ? (const char*)g.ga : (const char*)g.q) + (b0 + 2 * s) * rows * B;
    const __amdgpu_buffer_rsrc_t rv = uniform_rsrc(base, any ? (uint32_t)rows * B : 0u);
    if constexpr (ANCH) {
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        r[i].v = __builtin_amdgcn_raw_buffer_load_b128(rv, (ch + 32 * i) * B + 32 * half, 0, 0);
        r[i].w = __builtin_amdgcn_raw_buffer_load_b128(rv, (ch + 32 * i) * B + 32 * half + 16, 0, 0);
      }
    } else {
      const __amdgpu_buffer_rsrc_t re = uniform_rsrc(g.e + (b0 + 2 * s) * rows, any ? (uint32_t)rows : 0u);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        r[i].v = __builtin_amdgcn_raw_buffer_load_b128(rv, (ch + 32 * i) * B + 16 * half, 0, 0);
        r[i].e = __builtin_amdgcn_raw_buffer_load_b32(re, (ch + 32 * i) & ~3u, 0, 0);
      }
    }
    asm volatile("" ::: "memory");
  };
  // dword w of a row block's bytes: half a fragment of k-step w / 2
  auto convert = [&](const W8Raw<ANCH>& r, auto wc, u32x4& f0, u32x4& f1) {
    constexpr int W = decltype(wc)::value;
    if constexpr (ANCH) {
      // a copy made here (v_mov by hand: left to itself the compiler renames
      // and copies at the loop's top, waiting for the newest loads there)
#pragma unroll
      for (int c = 2 * (W & 1); c < 2 * (W & 1) + 2; ++c) {
        uint32_t x;
        asm volatile("v_mov_b32 %0, %1" : "=v"(x) : "v"(W < 2 ? r.v[c] : r.w[c]));
        (W < 2 ? f0 : f1)[c] = x;
      }
    } else {
      const float unit = 0.5f * ck_unit(__builtin_amdgcn_ubfe(r.e, 8 * (lane & 3), 8));
      uint32_t lo, hi;
      w8_convert(r.v[W] ^ 0x80808080u, unit, -128.f * unit, lo, hi);
      u32x4& f = W < 2 ? f0 : f1;
      f[2 * (W & 1)] = lo;
      f[2 * (W & 1) + 1] = hi;
    }
  };

  // transposed reads of Q: token 32 grp + 16 (lane / 32) + 8 step + 4 h + j, column group as in tr_frag
  const int g4 = lane >> 4, j4 = (lane & 15) >> 2, q4 = lane & 3;
  uint32_t qb[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int row = 32 * grp + 16 * (g4 >> 1) + j4, col = wn * (BN / 2) + 32 * j + 16 * (g4 & 1) + 4 * q4;
    qb[j] = lds_addr(smem) + (uint32_t)(row * BN * 2 + 16 * ((col >> 3) ^ wg_sw(row, QCPR)) + 2 * (col & 7));
  }
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  u32x4 fb[2][FN];
  auto frags = [&](int s, auto stepc) {
    constexpr int STEP = decltype(stepc)::value;
    const uint32_t base = (uint32_t)(s % W8_NS * QBYTES);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      u32x2 a, b;
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(a) : "v"(qb[j] + base), "i"(8 * STEP * BN * 2) : "memory");
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(b) : "v"(qb[j] + base), "i"((8 * STEP + 4) * BN * 2) : "memory");
      fb[STEP][j] = u32x4{a.x, a.y, b.x, b.y};
    }
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;

  f32x16_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x16_t{};

  // Issue order: Q 0, Q 1, P 0, Q 2, P 1, Q 3, P 2, then in stage s Q s + 4, P s + 3.
  constexpr int PLOADS = 2 * FM;
  W8Raw<ANCH> raw[2][FM];
  u32x4 fa[2][2][FM];  // [stage parity][k-step][i]
  issue(0);
  issue(1);
  fetch(0, raw[0]);
  issue(2);
  fetch(1, raw[1]);
  issue(3);
#pragma unroll
  for (int i = 0; i < FM; ++i)
    static_for<0, 4>([&](auto wc) { convert(raw[0][i], wc, fa[0][0][i], fa[0][1][i]); });
  fetch(2, raw[0]);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * QBLK + 3 * PLOADS) : "memory");
  __builtin_amdgcn_s_barrier();
  frags(0, S0{});
  lds_wait0();
  reg_pin(fb[0]);

  // One k-step's products, a quarter of the next stage's conversion of row
  // block H after each quarter of them: a wave issues in order, and the
  // matrix unit works on while the vector unit converts.
  auto products = [&](auto hc, const u32x4 (&a)[FM], const W8Raw<ANCH>& r, u32x4& f0, u32x4& f1) {
    constexpr int H = decltype(hc)::value, NM = FM * FN, PER = NM / 4 > 0 ? NM / 4 : 1;
    static_for<0, NM>([&](auto xc) {
      constexpr int X = decltype(xc)::value;
      acc[X / FN][X % FN] = mfma32x32x16(as_uint4(a[X / FN]), as_uint4(fb[H][X % FN]), acc[X / FN][X % FN]);
      if constexpr (X % PER == PER - 1) {
        constexpr int W = X / PER;
        convert(r, std::integral_constant<int, W>{}, f0, f1);
        if constexpr (NM == 2) convert(r, std::integral_constant<int, W + 2>{}, f0, f1);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto stage = [&](int s, auto parc) {
    constexpr int C = decltype(parc)::value, N = C ^ 1;
    frags(s, S1{});
    products(S0{}, fa[C][0], raw[N][0], fa[N][0][0], fa[N][1][0]);
    lds_wait0();
    reg_pin(fb[1]);
    // this wave's loads of Q's stage s + 1 have returned: after them came three
    // of P and two of Q; past the barrier every wave's have, and every
    // wave has read stage s
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * QBLK + 3 * PLOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    issue(s + 4);
    frags(s + 1, S0{});
    products(S1{}, fa[C][1], raw[N][1], fa[N][0][1], fa[N][1][1]);
    fetch(s + 3, raw[N]);
    lds_wait0();
    reg_pin(fb[0]);
  };
  int s = 0;
  for (; s + 1 < KS; s += 2) {
    stage(s, S0{});
    stage(s + 1, S1{});
  }
  if (s < KS) stage(s, S0{});

  // each group hands the other its sums of one row block through LDS, adds
  // the other's to its own block and stores it
  static_assert(FM == 2, "a row block for each group");
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  f32x4_t* sh = (f32x4_t*)smem + (wave & 3) * (FM * FN * 4 * 64) + lane;
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      f32x4_t v;
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = grp ? acc[0][j][4 * h + u] : acc[1][j][4 * h + u];
      sh[((grp * FN + j) * 4 + h) * 64] = v;
    }
  __syncthreads();
  // the rows of the tile in a resource: those past P's end are not stored
  const int all = g.d + g.ka;
  const float* out = g.part + ((int64_t)split * all + (ANCH ? g.d : 0) + m0) * g.N;
  const __amdgpu_buffer_rsrc_t ro = uniform_rsrc(out, (uint32_t)(min(W8_BM, rows - m0) * g.N) * 4u);
  const uint32_t o0 = 4u * (uint32_t)((wm * 64 + grp * 32 + 4 * (lane >> 5)) * g.N + n0 + wn * (BN / 2) + (lane & 31));
#pragma unroll
  for (int j = 0; j < FN; ++j) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const f32x4_t o = sh[(((grp ^ 1) * FN + j) * 4 + h) * 64];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float v = (grp ? acc[1][j][4 * h + u] : acc[0][j][4 * h + u]) + o[u];
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(ANCH ? v : 2.f * v), ro, o0 + 4u * (uint32_t)((8 * h + u) * g.N), 128 * j, 0);
      }
    }
  }
}

template <int BN>
__global__ __launch_bounds__(W8_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_wgrad8(Wgrad8Args g) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int QBYTES = W8_KT * BN * 2, SUM = W8_BM * BN * 4;
  __shared__ __attribute__((aligned(1024))) char smem[W8_NS * QBYTES > SUM ? W8_NS * QBYTES : SUM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // consecutive items (n fastest, then m: the workgroups of a token split) on one XCD
  const int NY = g.N / BN, Gt = gridDim.x;
  const int mtiles = (g.d + W8_BM - 1) / W8_BM, all = mtiles + (g.ka + W8_BM - 1) / W8_BM;
  int item = blockIdx.x;
  {
    const int xcd = item % 8, k = item / 8, q = Gt / 8, rem = Gt % 8;
    item = xcd < rem ? xcd * (q + 1) + k : rem * (q + 1) + (xcd - rem) * q + k;
  }
  const int idx = __builtin_amdgcn_readfirstlane(item / NY), ny = item - idx * NY;
  const int split = __builtin_amdgcn_readfirstlane(idx / all), mt = idx - split * all;
  if (mt < mtiles)
    w8_run<BN, false>(g, smem, split, mt * W8_BM, ny * BN, wave, lane);
  else
    w8_run<BN, true>(g, smem, split, (mt - mtiles) * W8_BM, ny * BN, wave, lane);
#endif
}

}  // namespace

hipError_t launch_wgrad8(const Wgrad8Args& g, hipStream_t s) {
  if (g.T <= 0) return hipSuccess;
  if (g.d % 64 || g.ka % 16 || g.ldq % 8 || g.tokens_per_split % W8_KT || g.splits < 1 ||
      (int64_t)(g.splits - 1) * g.tokens_per_split >= g.T)
    return hipErrorInvalidValue;
  const int tiles = ((g.d + W8_BM - 1) / W8_BM + (g.ka + W8_BM - 1) / W8_BM) * g.splits;
  if (g.N % 256 == 0)
    hipLaunchKernelGGL(k_wgrad8<256>, dim3(tiles * (g.N / 256)), dim3(W8_THREADS), 0, s, g);
  else if (g.N % 128 == 0)
    hipLaunchKernelGGL(k_wgrad8<128>, dim3(tiles * (g.N / 128)), dim3(W8_THREADS), 0, s, g);
  else if (g.N % 64 == 0)
    hipLaunchKernelGGL(k_wgrad8<64>, dim3(tiles * (g.N / 64)), dim3(W8_THREADS), 0, s, g);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

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
