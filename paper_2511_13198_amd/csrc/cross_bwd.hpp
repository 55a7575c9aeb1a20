// Cross attention, backward.  With P = exp(scale Q K^T - LSE), D_i = <dO_i, O_i>:
//   dV = P^T dO,  dS = P (dO V^T - D),  dK = scale dS^T Q,  dQ = scale dS K,
// over the visible pairs; the shared keys' dK and dV sum all rows of the batch.
//
// As in the self-attention backward P is recomputed from LSE in two kernels without
// atomics, whose products, copies and registers are those:
//   * cross_dq_kernel    tiles of packed rows over their keys (shared, then own), as
//                        the forward; also writes D for the next kernel;
//   * cross_dkdv_kernel  tiles of keys over the rows that see them: a shared tile
//                        over all rows of the batch, an own tile over its
//                        sequence's, all in one launch, so that they fill the chip
//                        together and the shared tiles' long loops are cut into
//                        parts of about the own tiles' length.
// P and dS enter the products as bf16 (off by at most 2^-8 of each), which is the matrix
// cores' full rate, and D of rows with more than 64 keys comes from the rounded O, which
// is what the forward keeps; sums are 32 bits, gradients are written in 32 bits or rounded
// to bf16 once (off by 2.4e-3 of their norm, 1.7e-3 of which that rounding is).
//
// dK/dV row steps.  A step is BQ rows: `pack` heads of the group (the largest power
// of two that divides it, at most 32) by BQ / pack tokens, so that a sequence of few
// tokens still fills a step, and a step's rows have one address pattern.
//
// Bound by the products: 8 sequences of 256-2,048 rows over 1,024-8,192 keys, 32/8 heads,
// dQ 343 us (3 products, 1,071 TFLOP/s), dK/dV 490 us (4 products, 1,001 TFLOP/s) in a
// running loop (381 and 565 in a profiled dozen passes, matrix cores busy 53 % and 47 % of
// the time at 1.9 GHz).  Short rows over many keys are bound by reading keys and writing
// gradients: 32 x 8-200 rows over 577-1,024 keys, 16 heads, d = 64, bf16 gradients, 33 and
// 58 us (dK/dV moves 0.24 GB), 32-bit ones 33 and 71.
#pragma once
#include "cross.hpp"

namespace pdy {

struct CrossBwdArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* kp;
  const uint16_t* vp;
  const uint16_t* o;
  const uint16_t* dout;
  const float* lse;  // [hq][tq]
  float* dd;         // D, [hq][tq]: written by the dQ kernel
  void* dq;          // float, or bf16 with out_bf16
  void* dk;
  void* dv;
  void* dkp;
  void* dvp;
  int out_bf16;
  CrossBatch b;
  CrossCut cut;
  float scale;
  float scale_log2;
  int pack_log2;
  // partial gradients (fp32, scaled): part [slice][rows][D] -- rows are tq * hq pairs
  // for dQ, (prefix + tk) * hkv for dK (part) and dV (part2), the shared keys first --
  // and how many slices a row of dQ (a key) has at part_n; dQ with CROSS_APART as the
  // forward
  float* part;
  float* part2;
  int32_t* part_n;
};

// Rows that see so many keys at most have D from P and dP (cross_dq_kernel); no more than
// a tile of the smallest.
constexpr int kCrossFewKeys = 64;

template <int D, int NW, int KG = 1>
struct CrossDqCfg {
  static constexpr int RG = NW / KG;
  static constexpr int BQ = 32 * RG;
  // 4-wave workgroups keep 64 so that two of them fit a CU's LDS
  static constexpr int BK = NW == 8 ? 128 : 64;
  static_assert(kCrossFewKeys <= BK, "few keys are in one tile");
  static constexpr int WK = BK / KG;
  static constexpr int NT = NW * 64;
  using KL = DualLayout<D>;  // K is read as rows (S^T) and transposed (dQ^T)
  // V is read as rows (dP^T)
  using VL = std::conditional_t<D == 64, DualLayout<D>, RowsLayout<D>>;
  static constexpr int KTILE = KL::elems(BK);
  static constexpr int VTILE = VL::elems(BK);
  static constexpr int LDS_BYTES = 2 * (KTILE + VTILE) * 2;
  static constexpr int F32_PASS = NW * (D / 32) * kF32Block * 4 <= LDS_BYTES ? D / 32 : 1;
  static_assert(NW * (KG > 1 ? D / 32 : F32_PASS) * kF32Block * 4 <= LDS_BYTES &&
                    NW * 32 * kBf16Pitch<D> * 2 <= LDS_BYTES,
                "dQ is turned in the tile buffers");
};

template <int D, int NW, int KG>
__global__ void __launch_bounds__(NW * 64, D == 64 && NW == 8 && KG == 1 ? 4 : NW == 4 ? 2 : 1)
    cross_dq_kernel(CrossBwdArgs a) {
  using C = CrossDqCfg<D, NW, KG>;
  using KL = typename C::KL;
  using VL = typename C::VL;
  constexpr int BQ = C::BQ, BK = C::BK;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];

  int hk, entry;
  xcd_order(blockIdx.x, gridDim.x, a.b.hkv, hk, entry);
  CrossPlace at;
  if (!cross_place_rows<KG <= 2>(a.b, a.cut, entry, at)) return;
  const int g = a.b.g;
  const CrossSeq sq = at.s;
  const int row_end = (sq.q_lo + sq.nq) * g;
  const int row0 = sq.q_lo * g + at.tile * BQ;

  const int l = __lane_id();
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // wave-uniform
  const int hh = l >> 5;
  const int rg = KG == 1 ? w : w % C::RG;
  const int kg = KG == 1 ? 0 : w / C::RG;
  const int wrow0 = row0 + rg * 32;
  const int row = wrow0 + (l & 31);
  const int wk0 = kg * C::WK;
  const int late = sq.nk - sq.nq - sq.q_lo + 1;  // as in the forward
  auto key_end = [&](int r) __attribute__((always_inline)) {
    return a.b.causal ? min(sq.nk, cross_token(a.b, max(min(r, row_end - 1), 0)) + late) : sq.nk;
  };
  const int lane_end = key_end(row);
  const int wave_first = __builtin_amdgcn_readfirstlane(key_end(wrow0));
  const int wave_end = __builtin_amdgcn_readfirstlane(key_end(wrow0 + 31));
  const int wg_end = __builtin_amdgcn_readfirstlane(max(0, key_end(row0 + BQ - 1)));
  const size_t kvstride = (size_t)a.b.hkv * D;
  auto row_off = [&](int r) __attribute__((always_inline)) {
    const int tok = cross_token(a.b, r);
    return ((size_t)tok * a.b.hq + hk * g + (r - tok * g)) * D;
  };

  const bool apart = a.cut.keys == CROSS_APART;
  const bool shared = apart && at.index == 0;  // this workgroup: shared keys alone
  const bool second = apart && !shared;
  const int npre = shared || a.cut.keys == CROSS_FUSED ? cross_tiles(a.b.prefix, BK) : 0;
  const int nown = shared ? 0 : cross_tiles(wg_end, BK);
  const int ntiles = npre + nown;
  const int t_begin = (int)((int64_t)at.part * ntiles / at.nparts);
  const int t_end = (int)((int64_t)(at.part + 1) * ntiles / at.nparts);
  auto kbuf = [&](int t) __attribute__((always_inline)) { return smem + (t & 1) * C::KTILE; };
  auto vbuf = [&](int t) __attribute__((always_inline)) {
    return smem + 2 * C::KTILE + (t & 1) * C::VTILE;
  };
  const int k_row = row_lane_base<KL>();
  const int k_tr = tr_lane_base<KL>();
  const int v_row = row_lane_base<VL>();

  using KD = TileDma<KL, BK, NW>;
  using VD = TileDma<VL, BK, NW>;
  constexpr int PK = KD::PER_WAVE, NCOPY = PK + VD::PER_WAVE;
  constexpr int STEPS = (C::WK / 32) * (D / 16);
  constexpr int GAP = STEPS / NCOPY > 1 ? STEPS / NCOPY : 1;
  // (at d = 64 both layouts are the same, and so are the copies' offsets)
  constexpr bool kSame = std::is_same_v<KL, VL>;
  KD kd;
  VD vd_own;
  VD& vd = [&]() -> VD& {
    if constexpr (kSame) return kd;
    else return vd_own;
  }();
  kd.init(kvstride);
  if constexpr (!kSame) vd.init(kvstride);
  struct Tile {
    const uint16_t *k, *v;
    int keys;
  };
  auto tile_at = [&](int t) __attribute__((always_inline)) {
    const bool pre = t < npre;
    const int k0 = (pre ? t : t - npre) * BK;
    const size_t off = (size_t)(pre ? k0 : sq.k_lo + k0) * kvstride + (size_t)hk * D;
    return Tile{(pre ? a.kp : a.k) + off, (pre ? a.vp : a.v) + off,
                (pre ? a.b.prefix : sq.nk) - k0};
  };
  auto issue = [&](int t) __attribute__((always_inline)) {
    const Tile x = tile_at(t);
    kd.issue(x.k, kvstride, x.keys, kbuf(t));
    vd.issue(x.v, kvstride, x.keys, vbuf(t));
  };
  // some row sees few keys (the first has the fewest): its D is summed from P and dP, below
  const bool few = ntiles > 0 && a.b.prefix + max(0, __builtin_amdgcn_readfirstlane(key_end(row0))) <=
                                     kCrossFewKeys;
  if (few) {
    issue(0);
    if (npre > 0) issue(1);
  } else if (t_begin < t_end) {
    issue(t_begin);
  }
  bf16x8 qf[D / 16], gf[D / 16];
  float lse2 = 0.f, ddv = 0.f;
  {
    const bool ok = row < row_end;
    const int r = ok ? row : row0;
    const size_t roff = row_off(r) + hh * 8;
    bf16x8 of[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) gf[ks] = load_bf16x8(a.dout + roff + ks * 16, ok);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) of[ks] = load_bf16x8(a.o + roff + ks * 16, ok);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = load_bf16x8(a.q + roff + ks * 16, ok);
    const int tok = cross_token(a.b, r);
    const size_t li = (size_t)(hk * g + (r - tok * g)) * a.b.tq + tok;
    if (ok) lse2 = a.lse[li];
    float dsum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        dsum[j & 3] = __builtin_fmaf((float)of[ks][j], (float)gf[ks][j], dsum[j & 3]);
    ddv = (dsum[0] + dsum[1]) + (dsum[2] + dsum[3]);
    ddv += partner32(ddv);
    if (ok) {
      lse2 *= kLog2e;
      // a row without any visible key has LSE = -inf and no gradient
      if (lse2 == -INFINITY) lse2 = INFINITY;
      if (hh == 0 && at.part == 0 && kg == 0) {
        if (!second && !few) a.dd[li] = ddv;
        if (a.part_n)
          a.part_n[(second ? (size_t)a.b.tq * a.b.hq : 0) + (size_t)tok * a.b.hq + hk * g +
                   (r - tok * g)] = at.nparts;
      }
    }
  }

  // S^T and dP^T of 32 keys of tile `it`, from key kb * 32 of this wave's on; hook(N) runs
  // after the products of the N-th K-step
  auto products = [&](auto KB, int it, f32x16& s, f32x16& dp, auto&& hook)
                      __attribute__((always_inline)) {
    constexpr int kb = decltype(KB)::value;
    constexpr int NKS = D / 16, PIPE = D == 64 && NW == 8 && KG == 1 ? 1 : 2;
    const uint32_t kra = lds_addr(kbuf(it)) + (k_row + wk0 * KL::ROW) * 2;
    const uint32_t vra = lds_addr(vbuf(it)) + (v_row + wk0 * VL::ROW) * 2;
    s = zero16();
    dp = zero16();
    u32x4 rk[PIPE + 1], rv[PIPE + 1];
    auto rd = [&](auto KS) __attribute__((always_inline)) {
      constexpr int ks = decltype(KS)::value, sl = ks % (PIPE + 1);
      row_issue<KL, kb * 32, ks * 16>(kra, rk[sl]);
      row_issue<VL, kb * 32, ks * 16>(vra, rv[sl]);
    };
    static_for<PIPE>([&](auto KS) { rd(KS); });
    static_for<NKS>([&](auto KS) {
      constexpr int ks = decltype(KS)::value, sl = ks % (PIPE + 1);
      if constexpr (ks + PIPE < NKS) {
        rd(std::integral_constant<int, ks + PIPE>{});
        row_wait<2 * PIPE>(rk[sl], rv[sl]);
      } else {
        row_wait<2 * (NKS - 1 - ks)>(rk[sl], rv[sl]);
      }
      s = mfma32(as_bf16x8(rk[sl]), qf[ks], s);
      dp = mfma32(as_bf16x8(rv[sl]), gf[ks], dp);
      hook(std::integral_constant<int, kb * NKS + ks>{});
    });
  };
  auto mask = [&](f32x16& s, int lim) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (acc_row_off(r) >= lim) s[r] = -INFINITY;
  };

  if (few) {
    // D = sum_j P_ij dP_ij in 32 bits over the first tile of the shared and of the own
    // keys, for the rows that see no others.  D from O carries O's rounding into
    // dS = P (dP - D): of a row with one key, whose dS is 0, that is all there is, and up
    // to some ten keys it shows beside dS's own rounding (dQ of 50 sequences of 21-338
    // causal rows off by 2.7e-3 of its norm, 2.4e-3 so).
    float dot = 0.f;
    wait_dma();
    __syncthreads();
    for (int it = 0; it <= npre; ++it) {
      const int end = (it < npre ? a.b.prefix : lane_end) - wk0;
      // keys of the tile that such a row of this wave sees end here
      const int some = (it < npre ? a.b.prefix : min(wave_end, kCrossFewKeys - a.b.prefix)) - wk0;
      static_for<(C::WK < kCrossFewKeys ? C::WK : kCrossFewKeys) / 32>([&](auto KB) {
        if (decltype(KB)::value * 32 >= some) return;
        f32x16 s, dp;
        products(KB, it, s, dp, [](auto) {});
        mask(s, end - (decltype(KB)::value * 32 + hh * 4));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          dot = __builtin_fmaf(fast_exp2(__builtin_fmaf(s[r], a.scale_log2, -lse2)), dp[r], dot);
      });
    }
    dot += partner32(dot);
    if constexpr (KG > 1) {
      // (in the second buffer: the first tile is the one that the loop begins with)
      __syncthreads();
      float* sums = reinterpret_cast<float*>(kbuf(1)) + rg * KG * 32;
      if (l < 32) sums[kg * 32 + l] = dot;
      __syncthreads();
      dot = 0.f;
#pragma unroll
      for (int j = 0; j < KG; ++j) dot += sums[j * 32 + (l & 31)];
    }
    if (a.b.prefix + max(0, lane_end) <= kCrossFewKeys) ddv = dot;
    // (no workgroup of apart lists: few keys are fused)
    if (hh == 0 && at.part == 0 && kg == 0 && row < row_end) {
      const int tok = cross_token(a.b, row);
      a.dd[(size_t)(hk * g + (row - tok * g)) * a.b.tq + tok] = ddv;
    }
    if (t_begin > 0) {
      __syncthreads();
      if (t_begin < t_end) issue(t_begin);
    }
  }
  f32x16 dqa[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dqa[i] = zero16();

  // keys of tile `it` for this wave (returns false where it has none)
  auto compute = [&](int it, auto&& hook) __attribute__((always_inline)) {
    const bool pre = it < npre;
    const int k0 = (pre ? it : it - npre) * BK + wk0;
    const int some = pre ? a.b.prefix : wave_end, every = pre ? a.b.prefix : wave_first;
    if (wrow0 >= row_end || k0 >= some) return false;
    const int end = pre ? a.b.prefix : lane_end;
    const uint32_t ka = lds_addr(kbuf(it)) + (k_tr + wk0 * KL::ROW) * 2;
    const bool need_mask = k0 + C::WK > every;
    static_for<C::WK / 32>([&](auto KB) {
      constexpr int kb = decltype(KB)::value;
      f32x16 s, dp;
      products(KB, it, s, dp, hook);
      if (need_mask) mask(s, end - (k0 + kb * 32 + hh * 4));
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float pv = fast_exp2(__builtin_fmaf(s[r], a.scale_log2, -lse2));
        s[r] = pv * (dp[r] - ddv);  // dS^T
      }
      constexpr int NDB = D / 32;
      TrRegs kt0[NDB], kt1[NDB];
      __builtin_amdgcn_s_setprio(1);
      const uint32_t kab = ka + kb * 32 * KL::ROW * 2;
      static_for<NDB>([&](auto DB) { tr_issue<KL, 0, DB * 32>(kab, kt0[DB]); });
      static_for<NDB>([&](auto DB) { tr_issue<KL, 16, DB * 32>(kab, kt1[DB]); });
      tr_wait<2 * NDB>(kt0);
      const bf16x8 sb0 = pack8(s, 0);
#pragma unroll
      for (int db = 0; db < NDB; ++db) dqa[db] = mfma32(kt0[db].operand(), sb0, dqa[db]);
      tr_wait<0>(kt1);
      const bf16x8 sb1 = pack8(s, 8);
#pragma unroll
      for (int db = 0; db < NDB; ++db) dqa[db] = mfma32(kt1[db].operand(), sb1, dqa[db]);
      __builtin_amdgcn_s_setprio(0);
    });
    return true;
  };

  for (int it = t_begin; it < t_end; ++it) {
    const bool more = it + 1 < t_end;
    wait_dma();
    __syncthreads();
    // past the last tile the copies get an empty range, so that no branch surrounds
    // them; a wave's last V copy may lie past the tile (a branch)
    const Tile x = tile_at(it + 1);
    const int keys_next = more ? x.keys : 0;
    const typename KD::Src rsk = KD::src(x.k, kvstride, keys_next);
    const typename VD::Src rsv = VD::src(x.v, kvstride, keys_next);
    const int bn = (it + 1) & 1;
    const bool ran = compute(it, [&](auto N) __attribute__((always_inline)) {
      constexpr int n = decltype(N)::value;
      auto copy = [&](auto CI) __attribute__((always_inline)) {
        constexpr int c = decltype(CI)::value;
        if constexpr (c < PK) kd.issue_one(c, rsk, kbuf(bn));
        else vd.issue_one(c - PK, rsv, vbuf(bn));
      };
      if constexpr (n % GAP == 0 && n / GAP < NCOPY - 1)
        copy(std::integral_constant<int, n / GAP>{});
      if constexpr (n == STEPS - 1)
        static_for<NCOPY>([&](auto CI) {
          if constexpr (decltype(CI)::value * GAP >= STEPS || decltype(CI)::value == NCOPY - 1)
            copy(CI);
        });
    });
    if (!ran && more) issue(it + 1);
  }
  wait_dma();
  if (wrow0 >= row_end) return;
  __syncthreads();

  const bool partial = apart || at.nparts > 1;
  const size_t slice =
      (size_t)(second ? a.cut.max_parts + at.part : at.part) * a.b.tq * a.b.hq * D;
  if constexpr (KG > 1) {
    float* slots = reinterpret_cast<float*>(smem) + rg * KG * (D / 32) * kF32Block;
    const int lane_off = acc_slot_lane();
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      acc_to_lds(dqa[db], a.scale, slots + (kg * (D / 32) + db) * kF32Block, lane_off);
    __syncthreads();
    combine_groups<D, KG>(
        slots, kg,
        [](int, float (&wt)[KG]) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < KG; ++j) wt[j] = 1.f;
        },
        [&](int r, int c, const float (&x)[8]) __attribute__((always_inline)) {
          if (wrow0 + r >= row_end) return;
          const size_t off = row_off(wrow0 + r) + c;
          if (partial) cross_put8(x, a.part + slice + off);
          else if (a.out_bf16) cross_put8(x, (uint16_t*)a.dq + off);
          else cross_put8(x, (float*)a.dq + off);
        });
    return;
  }
  if (!partial && a.out_bf16) {
    cross_store_bf16<D>(dqa, a.scale, row_end - wrow0, smem + w * 32 * kBf16Pitch<D>,
                        [&](int r) { return (uint16_t*)a.dq + row_off(wrow0 + r); });
  } else {
    float* dst = partial ? a.part + slice : (float*)a.dq;
    cross_store_f32<D, C::F32_PASS>(dqa, a.scale, row_end - wrow0,
                                    reinterpret_cast<float*>(smem) + w * C::F32_PASS * kF32Block,
                                    [&](int r) { return dst + row_off(wrow0 + r); });
  }
}

// Copies of a step's rows: packed row r of the step is token r >> pack_log2, head
// r % pack from the step's first on.
template <class L, int ROWS, int NW>
struct PackedDma : TileDma<L, ROWS, NW> {
  using Base = TileDma<L, ROWS, NW>;
  __device__ __forceinline__ void init_packed(size_t token_stride, int d, int pack_log2) {
    const int l = __lane_id();
    this->wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < Base::PER_WAVE; ++i) {
      const int slot = (this->wave + NW * i) * 64 + l;
      const int r = slot / L::SLOTS_PER_ROW;
      const int c = L::chunk_at(r, slot % L::SLOTS_PER_ROW);
      const size_t off =
          (r >> pack_log2) * token_stride + (size_t)(r & ((1 << pack_log2) - 1)) * d + c * 8;
      this->voff[i] = c < 0 ? Base::kPadOffset : (uint32_t)(off * 2);
    }
  }
};

// QG, NW: as in the self-attention dK/dV kernel (two query groups over 128 keys, or
// 8 or 4 waves over 256 or 128).
template <int D, int QG = 1, int NW_ = 8>
struct CrossDkdvCfg {
  static constexpr int NW = NW_;
  static constexpr int KW = NW / QG;
  static constexpr int BK = 32 * KW;
  static constexpr int BQ = NW == 4 && D == 128 ? 32 : 64;
  static constexpr int NT = NW * 64;
  using QL = DualLayout<D>;
  using KL = RowsLayout<D>;
  static constexpr int QTILE = QL::elems(BQ);
  static constexpr int KTILE = KL::elems(BK);
  static constexpr int STAGE = 2 * QTILE * 2 + 2 * BQ * 4;
  static constexpr int TILE_BYTES = 2 * STAGE + KTILE * 2;
  static constexpr int OUT_BYTES = NW * (D / 32) * kF32Block * 4;
  static constexpr int LDS_BYTES = QG > 1 && OUT_BYTES > TILE_BYTES ? OUT_BYTES : TILE_BYTES;
  static constexpr int F32_PASS = D / 32;
  static_assert(NW * F32_PASS * kF32Block * 4 <= LDS_BYTES,
                "the gradients are turned in the tile buffers");
  static_assert(LDS_BYTES <= 160 * 1024, "LDS of one CU");
};

template <int D, int QG, int NWAVES>
__global__ void __launch_bounds__(NWAVES * 64, NWAVES == 4 ? 2 : D == 64 ? 3 : 1)
    cross_dkdv_kernel(CrossBwdArgs a) {
  using C = CrossDkdvCfg<D, QG, NWAVES>;
  using QL = typename C::QL;
  using KL = typename C::KL;
  constexpr int BK = C::BK, BQ = C::BQ, NW = C::NW;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];

  int hk, entry;
  xcd_order(blockIdx.x, gridDim.x, a.b.hkv, hk, entry);
  const int g = a.b.g;
  const int sh = a.pack_log2, sweeps = g >> sh;  // head groups of `pack` heads
  // the list: the shared keys over the whole batch (if any), then the sequences
  const bool pre = a.b.prefix > 0;
  CrossPlace at;
  if (!cross_place<false>(
          a.b, a.cut, pre, entry,
          [&](const CrossSeq& s, bool, int& tiles, int& units) __attribute__((always_inline)) {
            cross_key_units(a.b, a.cut, sh, s, tiles, units);
          },
          at))
    return;
  const bool shared = pre && at.index == 0;
  const CrossSeq sq = at.s;
  const uint16_t* const kin = shared ? a.kp : a.k;
  const uint16_t* const vin = shared ? a.vp : a.v;
  const bool causal = a.b.causal && !shared;
  const int kt0 = at.tile * BK;  // first key of the tile, within the sequence
  const int q_hi = sq.q_lo + sq.nq;
  // first token that sees key j of the sequence: j + early (causal)
  const int early = sq.q_lo + sq.nq - sq.nk;

  const int l = __lane_id();
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // wave-uniform
  const int hh = l >> 5;
  const int kw = QG == 1 ? w : w % C::KW;
  const int qg = QG == 1 ? 0 : w / C::KW;
  const int kw0 = kt0 + kw * 32;
  const int key = kw0 + (l & 31);  // this lane's key
  const size_t qstride = (size_t)a.b.hq * D;
  const size_t kvstride = (size_t)a.b.hkv * D;

  if (a.part_n && hk == 0 && at.part == 0 && qg == 0 && hh == 0 && key < sq.room)
    a.part_n[(shared ? 0 : a.b.prefix) + sq.k_lo + key] = at.nparts;

  f32x16 dka[D / 32], dva[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    dka[i] = zero16();
    dva[i] = zero16();
  }
  bf16x8 vf[D / 16];
  {
    const bool ok = key < sq.nk;
    const uint16_t* vp = vin + (size_t)(sq.k_lo + (ok ? key : 0)) * kvstride + (size_t)hk * D + hh * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) vf[ks] = load_bf16x8(vp + ks * 16, ok);
  }

  uint8_t* const base = reinterpret_cast<uint8_t*>(smem);
  uint16_t* const ktile_s = reinterpret_cast<uint16_t*>(base + 2 * C::STAGE);
  auto qbuf = [&](int b) __attribute__((always_inline)) {
    return reinterpret_cast<uint16_t*>(base + b * C::STAGE);
  };
  auto gbuf = [&](int b) __attribute__((always_inline)) { return qbuf(b) + C::QTILE; };
  auto stats = [&](int b) __attribute__((always_inline)) {
    return reinterpret_cast<float*>(base + b * C::STAGE + 2 * C::QTILE * 2);
  };

  // tokens that can see this tile, in steps of BQ >> sh, for each head group, from the
  // last down
  const int step_tokens = BQ >> sh;
  const int qstart = causal ? max(sq.q_lo, kt0 + early) : sq.q_lo;
  const int nqt = kt0 < sq.nk ? max(0, cross_tiles(q_hi - qstart, step_tokens)) : 0;
  const int64_t all = (int64_t)nqt * sweeps;
  const int s_begin = (int)(at.part * all / at.nparts);
  const int nsteps = (int)((at.part + 1) * all / at.nparts) - s_begin;
  struct StepPos {
    int h;   // first query head
    int t0;  // first token
  };
  const int t_last = qstart + (nqt - 1) * step_tokens;
  const StepPos first =
      nqt > 0 ? StepPos{hk * g + ((s_begin / nqt) << sh), t_last - (s_begin % nqt) * step_tokens}
              : StepPos{hk * g, qstart};
  auto advance = [&](const StepPos& p) __attribute__((always_inline)) {
    return p.t0 > qstart ? StepPos{p.h, p.t0 - step_tokens} : StepPos{p.h + (1 << sh), t_last};
  };

  float stat = 0.f;
  auto load_stat = [&](const StepPos& p) __attribute__((always_inline)) {
    // (the lane computed anew: nothing of this holds a register over the products)
    const int t = w * 64 + fresh_lane_id();
    if (t < 2 * BQ) {
      const int r = t % BQ;
      const int tok = r >> sh;
      // (hq * tq is below 2^31)
      const int idx = p.h * a.b.tq + p.t0 + (r & ((1 << sh) - 1)) * a.b.tq + tok;
      stat = tok < q_hi - p.t0 ? (t < BQ ? a.lse[idx] : a.dd[idx]) : 0.f;
    }
  };
  auto store_stat = [&](int b) __attribute__((always_inline)) {
    const int t = w * 64 + fresh_lane_id();
    // a row without any visible key (LSE = -inf) must contribute nothing
    if (t < 2 * BQ) stats(b)[t] = t < BQ ? (stat == -INFINITY ? INFINITY : stat * kLog2e) : stat;
  };

  const int q_row = row_lane_base<QL>();
  const int q_tr = tr_lane_base<QL>();
  const int k_row = row_lane_base<KL>();

  auto compute = [&](int step, const StepPos& p, int hf, auto&& hook) __attribute__((always_inline)) {
    const int b = step & 1;
    const uint16_t* qs = qbuf(b);
    const uint16_t* gs = gbuf(b);
    const float* lse_s = stats(b);
    const float* dd_s = lse_s + BQ;
    const int tok_first = p.t0 + ((hf * 32) >> sh), tok_last = p.t0 + ((hf * 32 + 31) >> sh);
    const bool active = kw0 < sq.nk && tok_first < q_hi && (!causal || tok_last >= kw0 + early);
    if (!active) return false;
    const bool need_mask = (causal && tok_first < kw0 + 31 + early) || tok_last >= q_hi;
    f32x16 s = zero16(), dp = zero16();
    {
      constexpr int NKS = D / 16, PIPE = 2;
      const uint32_t qa = lds_addr(qs) + (q_row + hf * 32 * QL::ROW) * 2;
      const uint32_t ga = lds_addr(gs) + (q_row + hf * 32 * QL::ROW) * 2;
      const uint32_t ka = lds_addr(ktile_s) + (k_row + kw * 32 * KL::ROW) * 2;
      u32x4 rq[PIPE + 1], rk[PIPE + 1], rg[PIPE + 1];
      auto rd = [&](auto KS) __attribute__((always_inline)) {
        constexpr int ks = decltype(KS)::value, sl = ks % (PIPE + 1);
        row_issue<QL, 0, ks * 16>(qa, rq[sl]);
        row_issue<KL, 0, ks * 16>(ka, rk[sl]);
        row_issue<QL, 0, ks * 16>(ga, rg[sl]);
      };
      static_for<PIPE>([&](auto KS) { rd(KS); });
      static_for<NKS>([&](auto KS) {
        constexpr int ks = decltype(KS)::value, sl = ks % (PIPE + 1);
        if constexpr (ks + PIPE < NKS) {
          rd(std::integral_constant<int, ks + PIPE>{});
          row_wait<3 * PIPE>(rq[sl], rk[sl], rg[sl]);
        } else {
          row_wait<3 * (NKS - 1 - ks)>(rq[sl], rk[sl], rg[sl]);
        }
        s = mfma32(as_bf16x8(rq[sl]), as_bf16x8(rk[sl]), s);
        dp = mfma32(as_bf16x8(rg[sl]), vf[ks], dp);
        hook(KS);
      });
    }
    if (need_mask) {
      // accumulator row r is packed row hf 32 + hh 4 + acc_row_off(r) of the step; the
      // lane's key is visible from token `lo` on
      const int ml = fresh_lane_id(), here = hf * 32 + (ml >> 5) * 4;
      const int lo = (causal ? kw0 + (ml & 31) + early : sq.q_lo) - p.t0;
      const int rel = (min(max(lo, 0), BQ) << sh) - here;
      const int rows_left = (min(q_hi - p.t0, BQ) << sh) - here;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (acc_row_off(r) < rel || acc_row_off(r) >= rows_left) s[r] = -INFINITY;
    }
#pragma unroll
    for (int grp = 0; grp < 4; ++grp) {
      const int rl = hf * 32 + grp * 8 + hh * 4;
      const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse_s + rl);
      const f32x4 d4 = *reinterpret_cast<const f32x4*>(dd_s + rl);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = grp * 4 + e;
        const float pv = fast_exp2(__builtin_fmaf(s[r], a.scale_log2, -l4[e]));
        s[r] = pv;
        dp[r] = pv * (dp[r] - d4[e]);  // dS
      }
    }
    constexpr int NDB = D / 32;
    const uint32_t ga = lds_addr(gs) + (q_tr + hf * 32 * QL::ROW) * 2;
    const uint32_t qa = lds_addr(qs) + (q_tr + hf * 32 * QL::ROW) * 2;
    TrRegs ra[NDB], rb[NDB];
    __builtin_amdgcn_s_setprio(1);
    static_for<NDB>([&](auto DB) { tr_issue<QL, 0, DB * 32>(ga, ra[DB]); });
    static_for<NDB>([&](auto DB) { tr_issue<QL, 0, DB * 32>(qa, rb[DB]); });
    const bf16x8 pb0 = pack8(s, 0), sb0 = pack8(dp, 0);
    tr_wait<2 * NDB>(ra);
#pragma unroll
    for (int db = 0; db < NDB; ++db) dva[db] = mfma32(ra[db].operand(), pb0, dva[db]);
    static_for<NDB>([&](auto DB) { tr_issue<QL, 16, DB * 32>(ga, ra[DB]); });
    tr_wait<2 * NDB>(rb);
#pragma unroll
    for (int db = 0; db < NDB; ++db) dka[db] = mfma32(rb[db].operand(), sb0, dka[db]);
    static_for<NDB>([&](auto DB) { tr_issue<QL, 16, DB * 32>(qa, rb[DB]); });
    const bf16x8 pb1 = pack8(s, 8), sb1 = pack8(dp, 8);
    tr_wait<2 * NDB>(ra);
#pragma unroll
    for (int db = 0; db < NDB; ++db) dva[db] = mfma32(ra[db].operand(), pb1, dva[db]);
    tr_wait<0>(rb);
#pragma unroll
    for (int db = 0; db < NDB; ++db) dka[db] = mfma32(rb[db].operand(), sb1, dka[db]);
    __builtin_amdgcn_s_setprio(0);
    return true;
  };

  auto row_ptr = [&](const uint16_t* t, const StepPos& p) __attribute__((always_inline)) {
    return t + (size_t)p.t0 * qstride + (size_t)p.h * D;
  };
  auto tokens_valid = [&](const StepPos& p) __attribute__((always_inline)) { return q_hi - p.t0; };

  if (nsteps > 0) {
    // (keys not in use and rows past the sequence read as zeros; the keys' sums are
    // dropped below, the rows masked)
    {
      TileDma<KL, BK, NW> kd;
      kd.init(kvstride);
      kd.issue(kin + (size_t)(sq.k_lo + kt0) * kvstride + (size_t)hk * D, kvstride, sq.nk - kt0,
               ktile_s);
    }
    using QD = PackedDma<QL, BQ, NW>;
    constexpr int PQ = QD::PER_WAVE;
    constexpr int NKS = D / 16;
    static_assert(2 * (PQ - 1) <= NKS, "one copy per K-step of S/dP, and the last ones");
    QD qd;
    qd.init_packed(qstride, D, sh);
    auto issue = [&](int step, const StepPos& p) __attribute__((always_inline)) {
      qd.issue(row_ptr(a.q, p), qstride, tokens_valid(p), qbuf(step & 1));
      qd.issue(row_ptr(a.dout, p), qstride, tokens_valid(p), gbuf(step & 1));
    };
    StepPos cur = first;
    issue(0, cur);
    load_stat(cur);
    for (int step = 0; step < nsteps; ++step) {
      const bool more = step + 1 < nsteps;
      // (past the last step `nxt` is only used for address arithmetic)
      const StepPos nxt = advance(cur);
      wait_dma();
      store_stat(step & 1);
      __syncthreads();
      if (more) load_stat(nxt);
      const int rvn = more ? tokens_valid(nxt) : 0;
      const typename QD::Src rsq = QD::src(row_ptr(a.q, nxt), qstride, rvn);
      const typename QD::Src rsg = QD::src(row_ptr(a.dout, nxt), qstride, rvn);
      const int bn = (step + 1) & 1;
      const bool ran = compute(step, cur, QG > 1 ? qg : 0, [&](auto KS) __attribute__((always_inline)) {
        constexpr int c = decltype(KS)::value;
        if constexpr (c < PQ - 1) {
          qd.issue_one(c, rsq, qbuf(bn));
        } else if constexpr (c < 2 * (PQ - 1)) {
          qd.issue_one(c - (PQ - 1), rsg, gbuf(bn));
        }
        if constexpr (c == NKS - 1) {
          qd.issue_one(PQ - 1, rsq, qbuf(bn));
          qd.issue_one(PQ - 1, rsg, gbuf(bn));
        }
      });
      if (!ran && more) issue(step + 1, nxt);
      if constexpr (QG == 1 && BQ == 64) compute(step, cur, 1, [](auto) {});
      cur = nxt;
    }
  }

  wait_dma();
  if (kw0 >= sq.room) return;
  __syncthreads();
  // keys not in use get no gradient
  const int el = fresh_lane_id();
  const bool in_use = kw0 + (el & 31) < sq.nk;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dka[db][r] = in_use ? dka[db][r] : 0.f;
      dva[db][r] = in_use ? dva[db][r] : 0.f;
    }
  const bool partial = at.nparts > 1;
  const int nrows = sq.room - kw0;
  const size_t off = (size_t)(sq.k_lo + kw0) * kvstride + (size_t)hk * D;
  const size_t poff = ((size_t)at.part * (a.b.prefix + a.b.tk) +
                       (shared ? 0 : a.b.prefix)) * kvstride + off;
  void* const dkout = shared ? a.dkp : a.dk;
  void* const dvout = shared ? a.dvp : a.dv;
  float* lds = reinterpret_cast<float*>(smem) + w * C::F32_PASS * kF32Block;
  auto put = [&](const f32x16 (&x)[D / 32], float mul, void* dst, float* part, float* slot)
                 __attribute__((always_inline)) {
    if (partial)
      store_rows_f32<D, C::F32_PASS>(x, mul, part + poff, kvstride, nrows, false, slot, el);
    else if (a.out_bf16)
      store_rows_bf16<D>(x, mul, (uint16_t*)dst + off, kvstride, nrows,
                         reinterpret_cast<uint16_t*>(slot));
    else
      store_rows_f32<D, C::F32_PASS>(x, mul, (float*)dst + off, kvstride, nrows, false, slot, el);
    wave_lds_fence();
  };
  if constexpr (QG == 2) {
    // the groups exchange halves: group 0 keeps dK and hands over its dV, group 1
    // the other way round
    const int lane_off = acc_slot_lane();
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      acc_to_lds(qg ? dka[db] : dva[db], 1.f, lds + db * kF32Block, lane_off);
    __syncthreads();
    lds = reinterpret_cast<float*>(smem) + (w ^ C::KW) * C::F32_PASS * kF32Block;
    f32x16 sum[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(lds + db * kF32Block + lane_off + i * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sum[db][i * 4 + e] = (qg ? dva[db] : dka[db])[i * 4 + e] + x[e];
      }
    put(sum, qg ? 1.f : a.scale, qg ? dvout : dkout, qg ? a.part2 : a.part, lds);
  } else {
    put(dka, a.scale, dkout, a.part, lds);
    put(dva, 1.f, dvout, a.part2, lds);
  }
}

// Sums of partial gradients: row i (a head's D floats; `heads` of them to a token or
// key) has n[i / each] slices from 0 on, and n1[i / each] from max_parts on where the
// shared and the own keys were apart.  Rows with one slice are written already.
struct CrossSumJob {
  const float* part;
  const int32_t* n;
  const int32_t* n1;   // or NULL
  int max_parts;
  int heads;
  int each;            // rows to a count
  int64_t rows;        // rows of a slice
  int64_t first;       // first row to sum, and how many
  int64_t count;
  const int32_t* end;  // tokens (keys) from *end on stay as they are; or NULL
  void* dst;           // row `first`
  int blocks;
};
struct CrossSumArgs {
  CrossSumJob job[5];
  int njobs;
  int out_bf16;
};

template <int D>
__global__ void __launch_bounds__(256) cross_sum_kernel(CrossSumArgs a) {
  constexpr int LANES = D / 8;
  int block = blockIdx.x, j = 0;
  while (j + 1 < a.njobs && block >= a.job[j].blocks) block -= a.job[j++].blocks;
  const CrossSumJob& b = a.job[j];
  const int64_t gid = (int64_t)block * 256 + threadIdx.x;
  const int64_t i = gid / LANES;
  const int c = (int)(gid % LANES) * 8;
  if (i >= b.count) return;
  const int64_t row = b.first + i;
  const int64_t count = row / b.each;
  if (b.end && (int)(i / b.heads) >= *b.end) return;
  const int n0 = min(max(b.n[count], 0), b.max_parts);
  const int n1 = b.n1 ? min(max(b.n1[count], 0), b.max_parts) : 0;
  if (!b.n1 && n0 <= 1) return;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto add = [&](int64_t slice) __attribute__((always_inline)) {
    const float* p = b.part + (slice * b.rows + row) * D + c;
    const f32x4 x0 = *reinterpret_cast<const f32x4*>(p), x1 = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] += x0[e];
      x[4 + e] += x1[e];
    }
  };
  for (int p = 0; p < n0; ++p) add(p);
  for (int p = 0; p < n1; ++p) add(b.max_parts + p);
  if (a.out_bf16) cross_put8(x, (uint16_t*)b.dst + i * D + c);
  else cross_put8(x, (float*)b.dst + i * D + c);
}

}  // namespace pdy
