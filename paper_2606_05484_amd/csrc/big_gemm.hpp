// The products of the vocabulary's cross entropy: C(m, n) = sum_k P(m, k) Q(n, k)
// on bf16 operands with fp32 accumulation, in tiles of one workgroup per CU.
// Device code; included by the kernel sources only.
//
// What bounds it: with 256 x 256 tiles the matrix units are busy 65-75 % of a
// launch, its epilogues included, and the clock has fallen to 1.82-1.90 GHz,
// i.e. the card's power.  Hence the 16 x 16 x 32 instruction (half of the 32 x
// 32 x 16 one's accumulator traffic per product: 2048 x 32000 x 8192 942 -> 895
// us when it came), four waves of 128 x 128 outputs (a fragment from LDS feeds
// eight products), the XCD-blocked tile order and no operand copied twice.
// 32000 x 32768 outputs, K = 2048: 1.45 PFLOP/s with the softmax's epilogue,
// 1.35 with the gradient's (a library's plain product of these sizes reaches
// 1.37-1.48 on the same card).
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace mapl {

namespace {

typedef __attribute__((address_space(3))) void* bg_lds_ptr;

// One operand X(row, k): rows contiguous along k (X + row ld + k), or (TR)
// along the rows (X + k ld + row).  What lies past the last valid row of a
// k-contiguous operand, or past k's end under TR, reads as zero; a k-contiguous operand has
// k's range up to a multiple of 64 readable.  Under TR the columns past
// the matrix are whatever follows in memory (never past the last k-row):
// they reach only outputs that the caller does not store.
struct BgMat {
  const bf16_t* p;
  int64_t ld;
};

// M x N output, k-range K in `splits` runs of `kper` (a multiple of 64).
struct BgShape {
  BgMat P, Q;
  int M, N;
  int64_t K, kper;
  int splits;
  int mt, nt;  // tiles
};

// WVM x WVN waves of 16 FM x 16 FN outputs each; square tiles.
template <int WVM_, int WVN_, int FM_, int FN_, bool PT_, bool QT_>
struct BgCfg {
  static constexpr int WVM = WVM_, WVN = WVN_, FM = FM_, FN = FN_;
  static constexpr bool PT = PT_, QT = QT_;
  static constexpr int NW = WVM * WVN, THREADS = 64 * NW;
  static constexpr int BM = 16 * FM * WVM, BN = 16 * FN * WVN, BK = 64;
  static constexpr int PANEL = BM * BK * 2, SMEM = 5 * PANEL;
  static constexpr int LOADS = PANEL / 1024 / NW;  // 1 KiB direct-to-LDS blocks per wave and panel
  static_assert(BM == BN, "P and Q panels share a ring of slots");
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

// A panel of ROWS operand rows x 64 k in LDS and its fragments (16 rows x 32
// k: lane l row l % 16, k 8 (l / 16) .. +7).
//   k-contiguous: 128 B per row, 16 B chunk c of row r at c ^ ((r >> 1) & 7);
//   TR: ROWS 2 B per k-row, chunk c of k-row r at c ^ (4 (r & 3)) (wg_sw), read
//   transposed (see tr_frag).
// base[]: the lane's fragment addresses (k-contiguous: one per 32-deep
// k-step; TR: one per fragment number (i / 2) & 3, which the XOR acts on).
template <int ROWS, bool TR>
struct BgPanel {
  static constexpr int NB = TR ? 4 : 2;
  uint32_t base[NB];
  __device__ __forceinline__ void init(uint32_t lds, int row0, int lane) {
    if constexpr (!TR) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        base[kk] = lds + (uint32_t)((row0 + (lane & 15)) * 128 + 16 * ((4 * kk + (lane >> 4)) ^ ((lane & 15) >> 1)));
    } else {
      const int j = (lane & 15) >> 2, q = lane & 3, k = 8 * (lane >> 4) + j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = row0 + 32 * i + 4 * q;
        base[i] = lds + (uint32_t)(k * (ROWS * 2) + 16 * ((col >> 3) ^ (4 * j)) + 2 * (col & 7));
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
      bg_read<I * 16 * 128>(r, base[KK]);
    } else {
      constexpr int X = KK * 32 * ROWS * 2 + (I >> 3) * 256 + (I & 1) * 32;
      const u32x2 a = bg_read_tr<X>(base[(I >> 1) & 3]);
      const u32x2 b = bg_read_tr<X + 4 * ROWS * 2>(base[(I >> 1) & 3]);
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
// multiple of 8).  Before a tile's products pre(tile, wm, wn) may request what
// its epilogue reads; epi(acc, tile, wm, wn) takes the finished
// accumulators: acc[i][j][e] of lane l is C(m, n) at m = tile.m BM + 16 (wm FM + i)
// + 4 (l / 16) + e, n = tile.n BN + 16 (wn FN + j) + l % 16.
// smem: Cfg::SMEM bytes.
//
// P's and Q's panels of 64 k take turns in a ring of five slots.  A stage's
// products run in two k-steps of 32 whose fragments are read one k-step
// ahead; before the second every wave has its last fragments of the
// stage, so one barrier there both frees the stage's slots and publishes the
// next stage.  Under the first k-step's products P's panel of the stage after
// next is loaded, under the second's Q's.  The sequence runs on over tile
// ends: the next tile's first panels load, and its first fragments are
// read, before an epilogue.
// With one wave per SIMD nothing hides a stall, so the products' stream holds no branch: past
// the last stage the loads go on with empty resources (zeros into free slots).
template <class Cfg, typename Pre, typename Epi>
__device__ __forceinline__ void bg_run(const BgShape& g, char* smem, Pre&& pre, Epi&& epi) {
  constexpr int FM = Cfg::FM, FN = Cfg::FN, BK = Cfg::BK, PANEL = Cfg::PANEL, RING = 5 * PANEL, LOADS = Cfg::LOADS;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / Cfg::WVN, wn = wave % Cfg::WVN;
  const int G = gridDim.x, place = (blockIdx.x & 7) * (G >> 3) + (blockIdx.x >> 3);
  const int items = g.mt * g.nt * g.splits;
  if (place >= items) return;

  uint32_t offP[LOADS], offQ[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    offP[j] = bg_lane_off<Cfg::BM, Cfg::PT>(wave * LOADS + j, lane, g.P.ld);
    offQ[j] = bg_lane_off<Cfg::BN, Cfg::QT>(wave * LOADS + j, lane, g.Q.ld);
  }
  char* const lds0 = smem + wave * LOADS * 1024;

  // the loader's place in the panel sequence
  int l_item = place, l_slot = 0;  // l_slot: byte offset of the next panel's slot
  int64_t l_left = 0;              // k still to load of the tile; 0: past the last tile
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
  __amdgpu_buffer_rsrc_t rsP, rsQ;  // of the panels being issued
  auto open_p = [&]() {
    const uint32_t n = Cfg::PT ? (uint32_t)min(l_left, (int64_t)BK) * (uint32_t)g.P.ld * 2u - l_np : l_np;
    rsP = uniform_rsrc(l_p, l_left > 0 ? n : 0u);
  };
  auto open_q = [&]() {
    const uint32_t n = Cfg::QT ? (uint32_t)min(l_left, (int64_t)BK) * (uint32_t)g.Q.ld * 2u - l_nq : l_nq;
    rsQ = uniform_rsrc(l_q, l_left > 0 ? n : 0u);
  };
  auto issue = [&](auto qc, auto b0c, auto b1c) {
    constexpr bool Q = decltype(qc)::value;
    static_for<decltype(b0c)::value, decltype(b1c)::value>([&](auto ic) {
      constexpr int I = decltype(ic)::value;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(Q ? rsQ : rsP, (bg_lds_ptr)(lds0 + l_slot + I * 1024), 16,
                                               Q ? offQ[I] : offP[I], 0, 0, 0);
    });
  };
  auto bump = [&]() { l_slot = l_slot + PANEL == RING ? 0 : l_slot + PANEL; };
  auto stage_next = [&]() {  // past a stage whose P and Q resources are made
    l_left -= BK;
    l_p += Cfg::PT ? BK * g.P.ld : BK;
    l_q += Cfg::QT ? BK * g.Q.ld : BK;
    if (l_left <= 0) {
      l_item += G;
      l_left = 0;
      if (l_item < items) open();
    }
  };
  using C0 = std::integral_constant<int, 0>;
  using CL = std::integral_constant<int, LOADS>;

  open();
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    open_p();
    open_q();
    issue(std::false_type{}, C0{}, CL{});
    bump();
    issue(std::true_type{}, C0{}, CL{});
    bump();
    stage_next();
  }
  open_p();
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
  __builtin_amdgcn_s_barrier();

  BgPanel<Cfg::BM, Cfg::PT> pp;
  BgPanel<Cfg::BN, Cfg::QT> pq;
  pp.init(lds_addr(smem), wm * FM * 16, lane);
  pq.init(lds_addr(smem) + PANEL, wn * FN * 16, lane);

  u32x4 fp[2][FM], fq[2][FN];
  auto read = [&](auto kkc, auto ic) {  // fragment IC of k-step KK into its set: Q's, then P's
    constexpr int KK = decltype(kkc)::value, I = decltype(ic)::value;
    if constexpr (I < FN)
      pq.template read<KK, I>(fq[KK][I]);
    else if constexpr (I < FM + FN)
      pp.template read<KK, I - FN>(fp[KK][I - FN]);
  };
  static_for<0, FM + FN>([&](auto ic) { read(C0{}, ic); });
  lds_wait0();
  reg_pin(fp[0]);
  reg_pin(fq[0]);

  f32x4_t acc[FM][FN];
  int slot_p = 0, slot_q = PANEL;
  // One k-step's products (FIRST: the tile's first, on zeros), the next k-step's
  // fragments read over their first three quarters, and a panel's loads spread
  // over all of them.  What the next k-step needs besides is computed between
  // products too, a few scalar operations at a time.
  auto kstep = [&](auto kkc, auto firstc) {
    constexpr int KK = decltype(kkc)::value;
    constexpr bool FIRST = decltype(firstc)::value;
    constexpr int NM = FM * FN, R = FM + FN, H = NM * 3 / 4;
    if constexpr (KK == 1) {
      // the next stage's P and Q have landed; the P after them may still fly
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
      __builtin_amdgcn_s_barrier();
    }
    static_for<0, NM>([&](auto xc) {
      constexpr int X = decltype(xc)::value, I = X / FN, J = X % FN;
      acc[I][J] = mfma16x16x32(as_uint4(fp[KK][I]), as_uint4(fq[KK][J]), FIRST ? f32x4_t{} : acc[I][J]);
      constexpr int R0 = X < H ? X * R / H : R, R1 = X < H ? (X + 1) * R / H : R;
      static_for<R0, R1>([&](auto ic) { read(std::integral_constant<int, KK ^ 1>{}, ic); });
      constexpr int L0 = X * LOADS / NM, L1 = (X + 1) * LOADS / NM;
      issue(std::integral_constant<bool, KK == 1>{}, std::integral_constant<int, L0>{}, std::integral_constant<int, L1>{});
      if constexpr (KK == 0) {
        if constexpr (X == NM / 4) open_q();
        if constexpr (X == H + 1) {  // this stage's fragments are all requested: on to the next one's slots
          const int np = slot_p + 2 * PANEL >= RING ? slot_p + 2 * PANEL - RING : slot_p + 2 * PANEL;
          pp.shift(np - slot_p);
          slot_p = np;
        }
        if constexpr (X == H + 2) {
          const int nq = slot_q + 2 * PANEL >= RING ? slot_q + 2 * PANEL - RING : slot_q + 2 * PANEL;
          pq.shift(nq - slot_q);
          slot_q = nq;
        }
      } else {
        if constexpr (X == NM / 4) stage_next();
        if constexpr (X == NM / 2) open_p();
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    bump();
    lds_wait0();
    reg_pin(fp[KK ^ 1]);
    reg_pin(fq[KK ^ 1]);
  };
  using C1 = std::integral_constant<int, 1>;
  for (int item = place; item < items; item += G) {
    const BgTile t = bg_tile(g, item);
    const int KS = __builtin_amdgcn_readfirstlane((int)((min(g.kper, g.K - t.split * g.kper) + BK - 1) / BK));
    pre(t, wm, wn);
    kstep(C0{}, std::true_type{});
    kstep(C1{}, std::false_type{});
    for (int s = 1; s < KS; ++s) {
      kstep(C0{}, std::false_type{});
      kstep(C1{}, std::false_type{});
    }
    epi(acc, t, wm, wn);
  }
  // nothing may still be written into the LDS of a workgroup that has ended
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// The 4 x 4 outputs of two blocks (i, i + 1) as bf16, eight consecutive m per
// lane: after the swap of neighbouring 16-lane groups lane l holds m = 16 (i + g % 2)
// + 8 (g / 2) .. + 7, g = l / 16, of its n.
__device__ __forceinline__ u32x4 bg_pack8(const f32x4_t& a, const f32x4_t& b) {
  uint32_t p[4] = {pack_bf2(a[0], a[1]), pack_bf2(a[2], a[3]), pack_bf2(b[0], b[1]), pack_bf2(b[2], b[3])};
  const auto s0 = __builtin_amdgcn_permlane16_swap(p[0], p[2], false, false);
  const auto s1 = __builtin_amdgcn_permlane16_swap(p[1], p[3], false, false);
  return u32x4{s0[0], s1[0], s0[1], s1[1]};
}
// The m of bg_pack8's first value relative to block i's first.
__device__ __forceinline__ int bg_pack8_m(int lane) { return 16 * ((lane >> 4) & 1) + 8 * (lane >> 5); }

}  // namespace

}  // namespace mapl
