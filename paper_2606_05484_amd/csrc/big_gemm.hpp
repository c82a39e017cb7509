// The products of the vocabulary's cross entropy: C(m, n) = sum_k P(m, k) Q(n, k)
// on bf16 operands with fp32 accumulation, in tiles of one workgroup per CU.
// Device code; included by the kernel sources only.
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace mapl {

namespace {

typedef __attribute__((address_space(3))) void* bg_lds_ptr;

// One operand X(row, k): rows contiguous along k (X + row ld + k), or (TR)
// along the rows (X + k ld + row).  `rows` counts the valid rows where they
// are k-contiguous; in either form what lies past the last valid row or past
// k's end reads as zero, and under TR columns past the matrix read whatever
// follows in memory (never past the last k-row): they reach only outputs
// that the caller does not store.
struct BgMat {
  const bf16_t* p;
  int64_t ld;
};

// m x n output, k-range K in `splits` runs of `kper` (a multiple of 64).
struct BgShape {
  BgMat P, Q;
  int M, N;
  int64_t K, kper;
  int splits;
  int mt, nt;  // tiles
};

template <int WVM_, int WVN_, int FM_, int FN_, bool PT_, bool QT_>
struct BgCfg {
  static constexpr int WVM = WVM_, WVN = WVN_, FM = FM_, FN = FN_;
  static constexpr bool PT = PT_, QT = QT_;
  static constexpr int NW = WVM * WVN, THREADS = 64 * NW;
  static constexpr int BM = 32 * FM * WVM, BN = 32 * FN * WVN, BK = 64;
  static constexpr int PBYTES = BM * BK * 2, QBYTES = BN * BK * 2, STAGE = PBYTES + QBYTES;
  static constexpr int PL = PBYTES / 1024 / NW, QL = QBYTES / 1024 / NW, LOADS = PL + QL;
};

template <int OFF>
__device__ __forceinline__ void bg_read(u32x4& r, uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "ds offset is 16 bits");
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "i"(OFF) : "memory");
}
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
template <int OFF>
__device__ __forceinline__ u32x2 bg_read_tr(uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "ds offset is 16 bits");
  u32x2 r;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "i"(OFF) : "memory");
  return r;
}

// A panel of ROWS operand rows x 64 k in LDS and its fragments.
//   k-contiguous: 128 B per row, 16 B chunk c of row r at c ^ ((r >> 1) & 7);
//   TR: ROWS 2 B per k-row, chunk c of k-row r at c ^ (4 (r & 3)) (wg_sw).
// base[]: the lane's fragment addresses (k-contiguous: one per 16-deep
// k-step; TR: one per i & 3, the XOR acting on the fragment's number).
template <int ROWS, int F, bool TR>
struct BgPanel {
  static constexpr int NB = 4;
  uint32_t base[NB];
  __device__ __forceinline__ void init(uint32_t lds, int row0, int lane) {
    if constexpr (!TR) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        base[kk] = lds + (uint32_t)((row0 + (lane & 31)) * 128 + 16 * ((2 * kk + (lane >> 5)) ^ (((lane & 31) >> 1) & 7)));
    } else {
      const int g = lane >> 4, sidx = lane & 15, j = sidx >> 2, q = sidx & 3;
      const int k = 8 * (g >> 1) + j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = row0 + 16 * (g & 1) + 4 * q;
        base[i] = lds + (uint32_t)(k * (ROWS * 2) + 16 * (((col >> 3) + 4 * i) ^ (4 * j)) + 2 * (col & 7));
      }
    }
  }
  __device__ __forceinline__ void shift(int bytes) {
#pragma unroll
    for (int i = 0; i < NB; ++i) base[i] += (uint32_t)bytes;
  }
  template <int KK, int I>
  __device__ __forceinline__ void read(u32x4& r) const {
    if constexpr (!TR) {
      bg_read<I * 32 * 128>(r, base[KK]);
    } else {
      const u32x2 a = bg_read_tr<KK * 16 * ROWS * 2 + (I >> 2) * 256>(base[I & 3]);
      const u32x2 b = bg_read_tr<(KK * 16 + 4) * ROWS * 2 + (I >> 2) * 256>(base[I & 3]);
      r = u32x4{a.x, a.y, b.x, b.y};
    }
  }
};

// Byte offset, from a panel's first element, that lane i of 1 KiB block b
// loads (direct-to-LDS blocks are written in lane order).
template <int ROWS, bool TR>
__device__ __forceinline__ uint32_t bg_lane_off(int b, int lane, int64_t ld) {
  if constexpr (!TR) {
    const int row = 8 * b + (lane >> 3);
    return (uint32_t)row * (uint32_t)ld * 2u + 16u * (uint32_t)((lane & 7) ^ ((row >> 1) & 7));
  } else {
    constexpr int CPR = ROWS / 8;
    const int row = b * (64 / CPR) + lane / CPR;
    return (uint32_t)row * (uint32_t)ld * 2u + 16u * (uint32_t)((lane % CPR) ^ (4 * (row & 3)));
  }
}

// Tile `item` of the launch: splits outermost, then groups of eight n-tiles,
// within a group n fastest, so that the 32 items an XCD's CUs take together
// are 4 x 8 tiles (12 panels for 32 tiles in its L2).
struct BgTile {
  int split, m, n;
};
__device__ __forceinline__ BgTile bg_tile(const BgShape& g, int item) {
  constexpr int GN = 8;
  const int per = g.mt * g.nt;
  BgTile t;
  t.split = item / per;
  int i = item - t.split * per;
  const int full = g.nt / GN * GN * g.mt;  // items in whole groups
  if (i < full) {
    const int grp = i / (GN * g.mt), j = i - grp * GN * g.mt;
    t.m = j / GN;
    t.n = grp * GN + j % GN;
  } else {
    const int w = g.nt % GN, j = i - full;
    t.m = j / w;
    t.n = g.nt / GN * GN + j % w;
  }
  return t;
}

// Every tile of this workgroup in turn: item = round gridDim + place, places
// dealt so that each XCD's workgroups hold consecutive items (gridDim a
// multiple of 8).  epi(acc, tile) takes a finished tile's accumulators:
// acc[i][j] element e of lane l is C(m, n) at m = tile.m BM + wave's first row +
// 32 i + acc_row(e, l), n = tile.n BN + wave's first column + 32 j + l % 32.
// smem: 2 Cfg::STAGE bytes.
//
// Two stages of 64 k.  A stage's products run in four k-steps of 16 whose
// fragments are read one k-step ahead; before the last k-step of stage s every
// wave has its last fragments of s, so one barrier there both frees s's buffer for stage s + 2
// and publishes s + 1, whose first fragments are read under the last
// k-step's products.  The stage sequence runs on over tile ends: the next
// tile's first two stages load during an epilogue.
template <class Cfg, typename Epi>
__device__ __forceinline__ void bg_run(const BgShape& g, char* smem, Epi&& epi) {
  constexpr int FM = Cfg::FM, FN = Cfg::FN, BK = Cfg::BK;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / Cfg::WVN, wn = wave % Cfg::WVN;
  const int G = gridDim.x, place = (blockIdx.x & 7) * (G >> 3) + (blockIdx.x >> 3);
  const int items = g.mt * g.nt * g.splits;
  if (place >= items) return;

  uint32_t offP[Cfg::PL], offQ[Cfg::QL];
#pragma unroll
  for (int j = 0; j < Cfg::PL; ++j) offP[j] = bg_lane_off<Cfg::BM, Cfg::PT>(wave * Cfg::PL + j, lane, g.P.ld);
#pragma unroll
  for (int j = 0; j < Cfg::QL; ++j) offQ[j] = bg_lane_off<Cfg::BN, Cfg::QT>(wave * Cfg::QL + j, lane, g.Q.ld);
  char* const ldsP = smem + wave * Cfg::PL * 1024;
  char* const ldsQ = smem + Cfg::PBYTES + wave * Cfg::QL * 1024;

  // the loader's place in the stage sequence
  int l_item = place, l_buf = 0;
  int64_t l_left = 0;  // k still to load of the tile
  const bf16_t *l_p = nullptr, *l_q = nullptr;
  uint32_t l_np = 0, l_nq = 0;  // bytes of a k-contiguous panel's resource; TR: of a row before the panel
  auto open = [&]() {
    const BgTile t = bg_tile(g, l_item);
    const int64_t k0 = t.split * g.kper;
    l_left = min(g.kper, g.K - k0);
    const int64_t m0 = (int64_t)t.m * Cfg::BM, n0 = (int64_t)t.n * Cfg::BN;
    l_p = g.P.p + (Cfg::PT ? k0 * g.P.ld + m0 : m0 * g.P.ld + k0);
    l_q = g.Q.p + (Cfg::QT ? k0 * g.Q.ld + n0 : n0 * g.Q.ld + k0);
    l_np = Cfg::PT ? (uint32_t)(2 * m0) : (uint32_t)((min((int64_t)Cfg::BM, g.M - m0) - 1) * g.P.ld * 2 + 2 * BK);
    l_nq = Cfg::QT ? (uint32_t)(2 * n0) : (uint32_t)((min((int64_t)Cfg::BN, g.N - n0) - 1) * g.Q.ld * 2 + 2 * BK);
  };
  __amdgpu_buffer_rsrc_t rp, rq;
  auto stage_open = [&]() {  // resources of the next stage to load
    uint32_t np = l_np, nq = l_nq;
    if constexpr (Cfg::PT || Cfg::QT) {
      const int rows = (int)min(l_left, (int64_t)BK);
      if constexpr (Cfg::PT) np = (uint32_t)rows * (uint32_t)g.P.ld * 2u - l_np;
      if constexpr (Cfg::QT) nq = (uint32_t)rows * (uint32_t)g.Q.ld * 2u - l_nq;
    }
    rp = uniform_rsrc(l_p, np);
    rq = uniform_rsrc(l_q, nq);
  };
  auto issue = [&](auto b0c, auto b1c) {
    constexpr int B0 = decltype(b0c)::value, B1 = decltype(b1c)::value;
    static_for<B0, B1>([&](auto ic) {
      constexpr int I = decltype(ic)::value;
      if constexpr (I < Cfg::PL)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rp, (bg_lds_ptr)(ldsP + l_buf + I * 1024), 16, offP[I], 0, 0, 0);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (bg_lds_ptr)(ldsQ + l_buf + (I - Cfg::PL) * 1024), 16,
                                                 offQ[I - Cfg::PL], 0, 0, 0);
    });
  };
  auto stage_next = [&]() {  // past the stage just issued
    l_buf ^= Cfg::STAGE;
    l_left -= BK;
    if (l_left > 0) {
      l_p += Cfg::PT ? BK * g.P.ld : BK;
      l_q += Cfg::QT ? BK * g.Q.ld : BK;
    } else {
      l_item += G;
      if (l_item < items) open();
    }
  };
  using C0 = std::integral_constant<int, 0>;
  using CALL = std::integral_constant<int, Cfg::LOADS>;

  open();
  stage_open();
  issue(C0{}, CALL{});
  stage_next();
  if (l_item < items) {
    stage_open();
    issue(C0{}, CALL{});
    stage_next();
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Cfg::LOADS) : "memory");
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __builtin_amdgcn_s_barrier();

  BgPanel<Cfg::BM, FM, Cfg::PT> pp;
  BgPanel<Cfg::BN, FN, Cfg::QT> pq;
  pp.init(lds_addr(smem), wm * FM * 32, lane);
  pq.init(lds_addr(smem) + Cfg::PBYTES, wn * FN * 32, lane);

  u32x4 fp[2][FM], fq[2][FN];
  auto read = [&](auto kkc, auto setc, auto ic) {  // fragment IC of k-step KK into set SET: P's, then Q's
    constexpr int KK = decltype(kkc)::value, SET = decltype(setc)::value, I = decltype(ic)::value;
    if constexpr (I < FM)
      pp.template read<KK, I>(fp[SET][I]);
    else if constexpr (I < FM + FN)
      pq.template read<KK, I - FM>(fq[SET][I - FM]);
  };
  static_for<0, FM + FN>([&](auto ic) { read(C0{}, C0{}, ic); });
  lds_wait0();
  reg_pin(fp[0]);
  reg_pin(fq[0]);

  f32x16_t acc[FM][FN];
  int step = Cfg::STAGE;  // to the other buffer
  for (int item = place; item < items; item += G) {
    const BgTile t = bg_tile(g, item);
    const int KS = (int)((min(g.kper, g.K - t.split * g.kper) + BK - 1) / BK);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x16_t{};
    for (int s = 0; s < KS; ++s) {
      const bool more = s + 1 < KS || item + G < items;  // another stage follows
      static_for<0, 4>([&](auto kkc) {
        constexpr int KK = decltype(kkc)::value, CB = KK & 1, NB = CB ^ 1, NK = (KK + 1) & 3;
        bool load = false;
        if constexpr (KK == 3) {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          pp.shift(step);
          pq.shift(step);
          step = -step;
          load = l_item < items;
          if (load) stage_open();
        }
        constexpr int NM = FM * FN;
        static_for<0, NM>([&](auto xc) {
          constexpr int X = decltype(xc)::value, I = X / FN, J = X % FN;
          acc[I][J] = mfma32x32x16(as_uint4(fp[CB][I]), as_uint4(fq[CB][J]), acc[I][J]);
          // the next k-step's fragments over the first half of the products
          constexpr int R = FM + FN, H = NM / 2 > 0 ? NM / 2 : 1;
          constexpr int R0 = X < H ? X * R / H : R, R1 = X < H ? (X + 1) * R / H : R;
          if (KK < 3 || more)
            static_for<R0, R1>([&](auto ic) {
              read(std::integral_constant<int, NK>{}, std::integral_constant<int, NB>{}, ic);
            });
          if constexpr (KK == 3) {
            constexpr int L0 = X * Cfg::LOADS / NM, L1 = (X + 1) * Cfg::LOADS / NM;
            if (load) issue(std::integral_constant<int, L0>{}, std::integral_constant<int, L1>{});
          }
          __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (KK == 3) {
          if (load) stage_next();
        }
        lds_wait0();
        reg_pin(fp[NB]);
        reg_pin(fq[NB]);
      });
    }
    epi(acc, t, wm, wn, lane);
  }
}

}  // namespace

}  // namespace mapl
