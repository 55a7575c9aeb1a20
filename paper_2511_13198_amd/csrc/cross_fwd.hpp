// Cross attention, forward: every row over its own sequence's keys and the keys
// that the batch shares.
//   S_ij = scale <q_i, k_j>,  LSE_i = log sum_j exp(S_ij),  O_i = sum_j exp(S_ij - LSE_i) v_j
// over the visible keys j; a row that sees none gets O = 0, LSE = -inf.
//
// The products, the online softmax and the copies are those of the self-attention
// forward: S^T = K Q^T on 32x32x16 matrix instructions with a row per lane, P
// rounded to bf16 and fed back as an operand, K/V tiles copied to LDS a tile or
// more ahead.  P in bf16 is the matrix cores' full rate (two halves of it would be twice
// the products): O is off by 2.3e-3 of its norm, 1.7e-3 of which its own rounding is;
// sums, maxima and LSE are 32 bits.
//
// What differs is where rows and keys come from: packed rows (all heads of a group side
// by side), keys with offsets of their own, shared key tiles before a sequence's own, and
// parts of the keys where rows are few (CrossCut).
//
// KG key groups: the waves are NW / KG row blocks times KG groups that take 1 / KG
// of every key tile; few rows per workgroup, as a token or some of a sequence
// give, still use every wave.
//
// Few rows are bound by reading keys: one token for each of 64 sequences over caches of
// 256-16,384 keys, 32/8 heads, 183 us, 4.9 TB/s.  Many are bound by the products and
// the softmax beside them: 8 sequences of 256-2,048 rows over 1,024-8,192 keys, 32/8
// heads, 250 us in a running loop, 982 TFLOP/s (283 in a profiled dozen passes, matrix
// cores busy 46 % of the time at 2.0 GHz).
#pragma once
#include "cross.hpp"

namespace pdy {

template <int D, int NW, int KG = 1>
struct CrossFwdCfg {
  static constexpr int RG = NW / KG;
  static constexpr int BQ = 32 * RG;
  static constexpr int BK = NW == 4 ? (KG == 4 ? 128 : 64)
                            : KG > 1 || D == 128 ? 128 : 64;
  static constexpr int WK = BK / KG;
  static constexpr int BKS = WK < 64 ? WK : 64;
  static constexpr int NT = NW * 64;
  using KL = RowsLayout<D>;
  using VL = DualLayout<D>;
  static constexpr int KTILE = KL::elems(BK);
  static constexpr int VTILE = VL::elems(BK);
  static constexpr int STAGES = NW == 4 && KG == 4 && D == 128 ? 1 : 2;
  static constexpr int F32_PASS = D == 128 ? 4 : 1;
  // the output tile is turned in the tile buffers; key groups' partial O, then their
  // row statistics
  static constexpr int STAT_OFF = NW * (D / 32) * kF32Block * 4;
  static constexpr int OUT_BYTES = KG > 1 ? STAT_OFF + NW * 32 * 8 : NW * F32_PASS * kF32Block * 4;
  static constexpr int TILE_BYTES = STAGES * (KTILE + VTILE) * 2;
  static constexpr int LDS_BYTES = TILE_BYTES > OUT_BYTES ? TILE_BYTES : OUT_BYTES;
  static_assert(NW * 32 * kBf16Pitch<D> * 2 <= LDS_BYTES && LDS_BYTES <= 160 * 1024, "LDS");
};

struct CrossFwdArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* kp;
  const uint16_t* vp;
  uint16_t* o;
  float* lse;
  CrossBatch b;
  CrossCut cut;
  float scale_log2;
  // partial results: O (fp32, normalised by the part's own sums) and LSE of slice s
  // at part_o [s][tq * hq][D], part_lse [s][tq * hq] (NaN: a NaN or +inf logit), and
  // how many slices a row has at part_n [tq * hq].  CROSS_APART: part_n is of the shared
  // keys, part_n + tq * hq of a sequence's own, whose slices start at max_parts
  float* part_o;
  float* part_lse;
  int32_t* part_n;
};

template <int D, int NW, int KG>
__global__ void __launch_bounds__(NW * 64, NW == 4 ? 2 : 1)
    cross_fwd_kernel(CrossFwdArgs a) {
  using C = CrossFwdCfg<D, NW, KG>;
  using KL = typename C::KL;
  using VL = typename C::VL;
  constexpr int BQ = C::BQ, BK = C::BK, BKS = C::BKS;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];

  int hk, entry;
  xcd_order(blockIdx.x, gridDim.x, a.b.hkv, hk, entry);
  CrossPlace at;
  if (!cross_place_rows<KG <= 2>(a.b, a.cut, entry, at)) return;
  const int g = a.b.g;
  const CrossSeq sq = at.s;
  const int row_end = (sq.q_lo + sq.nq) * g;  // packed rows of the sequence end
  const int row0 = sq.q_lo * g + at.tile * BQ;

  const int l = __lane_id();
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // wave-uniform
  const int hh = l >> 5;
  const int rg = KG == 1 ? w : w % C::RG;
  const int kg = KG == 1 ? 0 : w / C::RG;
  const int wrow0 = row0 + rg * 32;
  const int row = wrow0 + (l & 31);
  const int wk0 = kg * C::WK;
  // first own key that a row's token does not see
  const int late = sq.nk - sq.nq - sq.q_lo + 1;  // key_end = token + late (causal)
  auto key_end = [&](int r) __attribute__((always_inline)) {
    return a.b.causal ? min(sq.nk, cross_token(a.b, max(min(r, row_end - 1), 0)) + late) : sq.nk;
  };
  const int lane_end = key_end(row);
  const int wave_first = __builtin_amdgcn_readfirstlane(key_end(wrow0));
  const int wave_end = __builtin_amdgcn_readfirstlane(key_end(wrow0 + 31));
  const int wg_end = __builtin_amdgcn_readfirstlane(max(0, key_end(row0 + BQ - 1)));

  const size_t kvstride = (size_t)a.b.hkv * D;
  // element offset of packed row r
  auto row_off = [&](int r) __attribute__((always_inline)) {
    const int tok = cross_token(a.b, r);
    return ((size_t)tok * a.b.hq + hk * g + (r - tok * g)) * D;
  };

  bf16x8 qf[D / 16];
  {
    const bool ok = row < row_end;
    const uint16_t* qp = a.q + row_off(ok ? row : row0) + hh * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = load_bf16x8(qp + ks * 16, ok);
  }

  f32x16 oacc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) oacc[i] = zero16();
  float m = -INFINITY;
  float lsum = 0.f;
  f32x16 s[BKS / 32];

  // key tiles: npre of the shared keys, then the sequence's own
  const bool apart = a.cut.keys == CROSS_APART;
  const bool shared = apart && at.index == 0;  // this workgroup: shared keys alone
  const int npre = shared || a.cut.keys == CROSS_FUSED ? cross_tiles(a.b.prefix, BK) : 0;
  const int nown = shared ? 0 : cross_tiles(wg_end, BK);
  const int ntiles = npre + nown;
  const int t_begin = (int)((int64_t)at.part * ntiles / at.nparts);
  const int t_end = (int)((int64_t)(at.part + 1) * ntiles / at.nparts);

  auto kbuf = [&](int t) __attribute__((always_inline)) {
    return smem + (t % C::STAGES) * (C::KTILE + C::VTILE);
  };
  auto vbuf = [&](int t) __attribute__((always_inline)) { return kbuf(t) + C::KTILE; };
  const int k_lane = row_lane_base<KL>();
  const int v_lane = tr_lane_base<VL>();

  auto compute_s = [&](const uint16_t* ktile, auto&& hook) __attribute__((always_inline)) {
    constexpr int NKS = D / 16, NKB = BKS / 32;
    static_assert(NKB == 1 || NKB == 2, "one or two 32-key blocks per step");
    constexpr int PIPE = 3;
    const uint32_t ka = lds_addr(ktile) + k_lane * 2;
    u32x4 kr[PIPE + 1][NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) s[kb] = zero16();
    auto rd = [&](auto KS) __attribute__((always_inline)) {
      constexpr int ks = decltype(KS)::value, sl = ks % (PIPE + 1);
      static_for<NKB>([&](auto KB) {
        row_issue<KL, decltype(KB)::value * 32, ks * 16>(ka, kr[sl][KB]);
      });
    };
    auto wt = [&](auto KS, auto N) __attribute__((always_inline)) {
      constexpr int sl = decltype(KS)::value % (PIPE + 1);
      if constexpr (NKB == 1) row_wait<decltype(N)::value>(kr[sl][0]);
      else row_wait<decltype(N)::value>(kr[sl][0], kr[sl][1]);
    };
    static_for<PIPE>([&](auto KS) { rd(KS); });
    static_for<NKS>([&](auto KS) {
      constexpr int ks = decltype(KS)::value, slot = ks % (PIPE + 1);
      if constexpr (ks + PIPE < NKS) {
        rd(std::integral_constant<int, ks + PIPE>{});
        wt(KS, std::integral_constant<int, NKB * PIPE>{});
      } else {
        wt(KS, std::integral_constant<int, NKB * (NKS - 1 - ks)>{});
      }
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) s[kb] = mfma32(as_bf16x8(kr[slot][kb]), qf[ks], s[kb]);
      hook(KS);
    });
  };

  // Mask (keys from `end` on are not visible to the lane's row; `masked`: some key of
  // the step is not, to some row of the wave), online softmax, O^T += V^T P^T.
  auto softmax_pv = [&](int k0, int end, bool masked, const uint16_t* vtile)
                        __attribute__((always_inline)) {
    if (masked) {
#pragma unroll
      for (int kb = 0; kb < BKS / 32; ++kb) {
        const int lim = end - (k0 + kb * 32 + hh * 4);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (acc_row_off(r) >= lim) s[kb][r] = -INFINITY;
      }
    }
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int kb = 0; kb < BKS / 32; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx[r & 3] = fmaxf(mx[r & 3], s[kb][r]);
    float tmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
    tmax = fmaxf(tmax, partner32(tmax));
    const float mt = tmax * a.scale_log2;
    const bool grow = mt > m + kRescaleSlack;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      const float alpha = grow ? fast_exp2(m - mt) : 1.f;
      m = grow ? mt : m;
      lsum *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
    }
    const float muse = (m == -INFINITY) ? 0.f : m;
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < BKS / 32; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = fast_exp2(__builtin_fmaf(s[kb][r], a.scale_log2, -muse));
        s[kb][r] = p;
        ps[r & 3] += p;
      }
    lsum += (ps[0] + ps[1]) + (ps[2] + ps[3]);
    constexpr int NDB = D / 32, NT16 = BKS / 16;
    const uint32_t va = lds_addr(vtile) + v_lane * 2;
    TrRegs vr[2][NDB];
    if (D == 64 || NW == 4 || w >= 4) __builtin_amdgcn_s_setprio(1);
    static_for<NDB>([&](auto DB) { tr_issue<VL, 0, DB * 32>(va, vr[0][DB]); });
    static_for<NT16>([&](auto T) {
      constexpr int cur = T & 1;
      if constexpr (T + 1 < NT16) {
        static_for<NDB>([&](auto DB) { tr_issue<VL, (T + 1) * 16, DB * 32>(va, vr[cur ^ 1][DB]); });
        tr_wait<2 * NDB>(vr[cur]);
      } else {
        tr_wait<0>(vr[cur]);
      }
      const bf16x8 pf = pack8(s[T >> 1], (T & 1) * 8);
#pragma unroll
      for (int db = 0; db < NDB; ++db) oacc[db] = mfma32(vr[cur][db].operand(), pf, oacc[db]);
    });
    __builtin_amdgcn_s_setprio(0);
  };

  {
    // (keys past the end of a tile's range read as zeros and are masked)
    TileDma<KL, BK, NW> kd;
    TileDma<VL, BK, NW> vd;
    kd.init(kvstride);
    vd.init(kvstride);
    struct Tile {
      const uint16_t *k, *v;
      int keys;  // keys from the tile's first on (0: none)
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
    constexpr int S = C::STAGES;  // 1: a tile's copies begin when its products have ended
    constexpr int PK = TileDma<KL, BK, NW>::PER_WAVE, PV = TileDma<VL, BK, NW>::PER_WAVE;
    if (t_begin < t_end) issue(t_begin);
    for (int it = t_begin; it < t_end; ++it) {
      wait_dma();
      __syncthreads();
      const int tn = it + 1;
      const bool more = tn < t_end;
      const bool pre = it < npre;
      const int k0t = (pre ? it : it - npre) * BK + wk0;  // this wave's first key
      // keys that some row, that every row of this wave sees end here
      const int some = pre ? a.b.prefix : wave_end, every = pre ? a.b.prefix : wave_first;
      if (wrow0 < row_end && k0t < some) {
        // past the last tile the copies get an empty range, so that no branch
        // surrounds them
        const Tile x = tile_at(tn);
        const int keys_next = more ? x.keys : 0;
        const auto rsk = TileDma<KL, BK, NW>::src(x.k, kvstride, keys_next);
        const auto rsv = TileDma<VL, BK, NW>::src(x.v, kvstride, keys_next);
        uint16_t* kl = kbuf(tn);
        uint16_t* vl = vbuf(tn);
        auto copy = [&](auto CI) __attribute__((always_inline)) {
          constexpr int c = decltype(CI)::value;
          if constexpr (c < PV) {
            vd.issue_one(c, rsv, vl);
          } else if constexpr (c < PV + PK) {
            kd.issue_one(c - PV, rsk, kl);
          }
        };
        static_for<C::WK / BKS>([&](auto SUB) {
          constexpr int sub = decltype(SUB)::value;
          const int k0s = k0t + sub * BKS;
          if (sub == 0 || k0s < some) {
            compute_s(kbuf(it) + (wk0 + sub * BKS) * KL::ROW,
                      [&](auto KS) __attribute__((always_inline)) {
                        if constexpr (S > 1 && sub == 0) {
                          constexpr int ks = decltype(KS)::value;
                          if constexpr (ks < PK + PV - 1) copy(KS);
                          if constexpr (ks == D / 16 - 1)
                            static_for<PK + PV - 1>([&](auto CI) {
                              if constexpr (decltype(CI)::value >= D / 16) copy(CI);
                            });
                        }
                      });
            softmax_pv(k0s, pre ? a.b.prefix : lane_end, k0s + BKS > every,
                       vbuf(it) + (wk0 + sub * BKS) * VL::ROW);
          }
        });
        if constexpr (S > 1) copy(std::integral_constant<int, PK + PV - 1>{});
      } else if (S > 1 && more) {
        issue(tn);
      }
      if constexpr (S == 1) {
        __syncthreads();
        if (more) issue(tn);
      }
    }
    wait_dma();
    if (wrow0 >= row_end) return;
    __syncthreads();
  }

  const bool partial = apart || at.nparts > 1;
  const bool second = apart && !shared;
  const size_t pairs = (size_t)a.b.tq * a.b.hq;
  const size_t slice = (size_t)(second ? a.cut.max_parts + at.part : at.part) * pairs;
  if (a.part_n && at.part == 0 && kg == 0 && hh == 0 && row < row_end) {
    const int tok = cross_token(a.b, row);
    a.part_n[(second ? pairs : 0) + (size_t)tok * a.b.hq + hk * g + (row - tok * g)] = at.nparts;
  }
  // LSE of a row from its offset m (base 2) and sum; a part hands a NaN sum on as NaN
  auto lse_of = [&](float m2, float tot) __attribute__((always_inline)) {
    return tot > 0.f ? (m2 + __builtin_log2f(tot)) * kLn2 : partial ? tot - INFINITY : -INFINITY;
  };
  auto put_lse = [&](int r, float x) __attribute__((always_inline)) {
    const int tok = cross_token(a.b, r), h = hk * g + (r - tok * g);
    if (partial) a.part_lse[slice + (size_t)tok * a.b.hq + h] = x;
    else a.lse[(size_t)h * a.b.tq + tok] = x;
  };
  if constexpr (KG == 1) {
    const float ltot = lsum + partner32(lsum);
    const float inv = ltot > 0.f ? 1.f / ltot : 0.f;
    if (partial)
      cross_store_f32<D, C::F32_PASS>(
          oacc, inv, row_end - wrow0,
          reinterpret_cast<float*>(smem) + w * C::F32_PASS * kF32Block,
          [&](int r) { return a.part_o + slice * D + row_off(wrow0 + r); });
    else
      cross_store_bf16<D>(oacc, inv, row_end - wrow0, smem + w * 32 * kBf16Pitch<D>,
                          [&](int r) { return a.o + row_off(wrow0 + r); });
    if (l < 32 && row < row_end) put_lse(row, lse_of(m, ltot));
  } else {
    float* slots = reinterpret_cast<float*>(smem) + rg * KG * (D / 32) * kF32Block;
    f32x2* stat = reinterpret_cast<f32x2*>(reinterpret_cast<uint8_t*>(smem) + C::STAT_OFF) +
                  rg * KG * 32;
    const float ltot = lsum + partner32(lsum);
    const int lane_off = acc_slot_lane();
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      acc_to_lds(oacc[db], 1.f, slots + (kg * (D / 32) + db) * kF32Block, lane_off);
    if (l < 32) stat[kg * 32 + l] = f32x2{m, ltot};
    __syncthreads();
    float lse = 0.f;  // of the row at hand
    combine_groups<D, KG>(
        slots, kg,
        [&](int r, float (&wt)[KG]) __attribute__((always_inline)) {
          f32x2 st[KG];
          float mx = -INFINITY, tot = 0.f;
#pragma unroll
          for (int j = 0; j < KG; ++j) {
            st[j] = stat[j * 32 + r];
            mx = fmaxf(mx, st[j][0]);
          }
#pragma unroll
          for (int j = 0; j < KG; ++j) {
            // (a NaN sum makes the row's)
            wt[j] = st[j][1] > 0.f || st[j][1] != st[j][1] ? fast_exp2(st[j][0] - mx) : 0.f;
            tot += wt[j] * st[j][1];
          }
          const float inv = tot > 0.f || tot != tot ? 1.f / tot : 0.f;
#pragma unroll
          for (int j = 0; j < KG; ++j) wt[j] *= inv;
          lse = lse_of(mx, tot);
        },
        [&](int r, int c, const float (&x)[8]) __attribute__((always_inline)) {
          const int pr = wrow0 + r;
          if (pr >= row_end) return;
          if (partial) cross_put8(x, a.part_o + slice * D + row_off(pr) + c);
          else cross_put8(x, a.o + row_off(pr) + c);
          if (c == 0) put_lse(pr, lse);
        });
  }
}

// Combine the partial results of the rows that have any: part_n[row] slices from 0 on,
// and, where shared and own keys were apart, part_n[tq * hq + row] from slice max_parts
// on.
//   LSE = log sum_p exp(LSE_p),  O = sum_p exp(LSE_p - LSE) O_p;
// a part with LSE = -inf weighs nothing, one with NaN makes the row O = NaN, LSE =
// -inf.  A wave per (token, head) pair: a lane per slice for the weights (64 at a
// time), then 64 / LANES slices at a time, 8 elements a lane, so that the reads of
// many slices are in flight together.  Bound by its launch where rows are few (64 tokens
// of 32 heads, 30 slices 8 us), by reading them where many (24 MB 17 us).
struct CrossMergeArgs {
  const float* part_o;
  const float* part_lse;
  const int32_t* part_n;
  int max_parts;
  int apart;
  const int32_t* cu_q;  // rows end at cu_q[n]
  int n;
  int tq, hq;
  uint16_t* o;
  float* lse;
};

template <int D>
__global__ void __launch_bounds__(256) cross_merge_kernel(CrossMergeArgs a) {
  constexpr int LANES = D / 8, GROUPS = 64 / LANES;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = __lane_id();
  const uint32_t pair = blockIdx.x * 4 + w;  // token * hq + head
  const uint32_t pairs = (uint32_t)a.tq * a.hq;
  if (pair >= pairs) return;
  const int tok = (int)(pair / (uint32_t)a.hq), h = (int)(pair - (uint32_t)tok * a.hq);
  const int c = (l % LANES) * 8, grp = l / LANES;
  const int end = a.cu_q[a.n];
  const int n0 = min(max(a.part_n[pair], 0), a.max_parts);
  const int n1 = a.apart ? min(max(a.part_n[(size_t)pairs + pair], 0), a.max_parts) : 0;
  if (tok >= end) return;  // rows behind the last sequence stay
  if (!a.apart && n0 == 1) return;  // written by its one part
  const int parts = n0 + n1, gap = a.max_parts - n0;
  float mx = -INFINITY, tot = 0.f;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // (more than 64 slices: the sums so far are rescaled by each further 64)
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const int p = p0 + l;
    const float x = p < parts ? a.part_lse[(size_t)(p < n0 ? p : p + gap) * pairs + pair]
                              : -INFINITY;
    float top = x;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    top = fmaxf(top, mx);
    const float keep = mx == -INFINITY ? 0.f : fast_exp2((mx - top) * kLog2e);
    // (NaN where x is NaN: fmaxf passes it over)
    const float wt = x == -INFINITY ? 0.f : fast_exp2((x - top) * kLog2e);
    mx = top;
    float sum = wt;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    tot = tot * keep + sum;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= keep;
    const int m = min(64, parts - p0);
#pragma unroll 4
    for (int j0 = 0; j0 < m; j0 += GROUPS) {
      // (every lane takes part in the exchange; past the last slice the weight is 0)
      const float wj = __shfl(wt, j0 + grp);
      const int pj = p0 + min(j0 + grp, m - 1);
      const float* src = a.part_o + ((size_t)(pj < n0 ? pj : pj + gap) * pairs + pair) * D + c;
      const f32x4 x0 = *reinterpret_cast<const f32x4*>(src);
      const f32x4 x1 = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] += wj * x0[e];
        acc[4 + e] += wj * x1[e];
      }
    }
  }
#pragma unroll
  for (int off = LANES; off < 64; off <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], off);
  const float inv = tot > 0.f ? 1.f / tot : tot != tot ? NAN : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] *= inv;
  if (grp == 0) cross_put8(acc, a.o + (size_t)pair * D + c);
  if (l == 0)
    a.lse[(size_t)h * a.tq + tok] = tot > 0.f ? mx + __builtin_log2f(tot) * kLn2 : -INFINITY;
}

}  // namespace pdy
