// What the cross-attention kernels share: the packed batch they work on, the
// placement of their workgroups, and the output tiles of packed rows.
//
// A batch has n sequences.  Sequence i has the queries cu_q[i] .. cu_q[i + 1] and
// the keys cu_k[i] .. cu_k[i + 1], of which the first len_k[i] are in use (all
// where len_k is NULL); every row also sees the `prefix` keys that the batch
// shares.  causal: the last query of a sequence sees all its keys in use, the one
// before all but the last, ...
//
// Packed rows.  The g query heads of a key/value head read the same keys, so a
// tile's rows are (token, head of the group) pairs: packed row R of kv head hk is
// head hk g + R % g of token R / g.  A tile of 32 NW rows then holds 32 NW / g
// tokens, each K/V tile is read once for the whole group, and one token of a
// sequence still fills g rows of the matrix product.
//
// Offsets read from cu_q, cu_k and len_k are clamped to the tensors, so that no
// value in them makes a kernel leave its tensors.  Tiles end at the lengths that the
// host sized the grid for: a sequence that is longer than it was said to be loses its
// own last tiles, not those of the sequences behind it.
#pragma once
#include "common.hpp"

namespace pdy {

struct CrossBatch {
  const int32_t* cu_q;   // [n + 1]
  const int32_t* cu_k;   // [n + 1]
  const int32_t* len_k;  // [n] or NULL
  int n;
  int tq;      // rows of q
  int tk;      // rows of k, v
  int prefix;  // shared keys
  int hq, hkv;
  int g;           // hq / hkv
  uint32_t g_inv;  // 2^32 / g, rounded down (g > 1)
  int causal;
  int max_k;  // keys of a sequence (in use or not) that get a gradient
};

// One sequence: rows of q and k, keys in use, and rows of k that get a gradient (those
// not in use too).
struct CrossSeq {
  int q_lo, nq, k_lo, nk, room;
};

__device__ __forceinline__ CrossSeq cross_seq(const CrossBatch& b, int i) {
  CrossSeq s;
  s.q_lo = min(max(b.cu_q[i], 0), b.tq);
  s.nq = min(max(b.cu_q[i + 1], s.q_lo), b.tq) - s.q_lo;
  s.k_lo = min(max(b.cu_k[i], 0), b.tk);
  s.nk = s.room = min(max(b.cu_k[i + 1], s.k_lo), b.tk) - s.k_lo;
  if (b.len_k) s.nk = min(max(b.len_k[i], 0), s.nk);
  s.room = min(s.room, b.max_k);
  return s;
}
// The whole batch as one sequence over the shared keys.
__device__ __forceinline__ CrossSeq cross_shared_seq(const CrossBatch& b) {
  return CrossSeq{0, min(max(b.cu_q[b.n], 0), b.tq), 0, b.prefix, b.prefix};
}

// Which rows and keys a launch covers.
enum CrossKeys : int {
  CROSS_OWN = 0,    // a sequence's rows over its own keys
  CROSS_FUSED = 1,  // over the shared keys, then its own
  CROSS_APART = 2,  // all rows of the batch, as one sequence, over the shared keys, and
                    // beside it every sequence's rows over its own: partial results of
                    // both, for few rows a sequence
};

// How a launch's rows and keys are cut.  An item is a tile of `rows` packed rows of
// a sequence and kv head (dK/dV: a tile of keys); its inner work, key tiles (row
// tiles), is cut into parts, one workgroup each, whose partial results another
// kernel combines:
//   a part has at most C = max(least, units / entries) inner tiles, the units being all
//   items' of a kv head: about `entries` parts, alike whatever the lengths, and up to
//   one an item more.
// EVEN and `even` (tiles of many rows, up to kListLanes sequences): under a causal mask
// a sequence's last tiles come first, and C is the least from there on with which the
// parts are no more than `entries`, so that they fit the rounds on the chip that the
// host planned for (6 sequences of 500-2,000 rows behind 16,384 keys, 4 heads: 648 parts
// where 512 fit, 299 us, 432 of them 264).
//   round > 0 (workgroups of a kv head at a time): the sequences of most keys come first,
// their items whole, as many rounds of them as end before an even share of all work
// would, and the others' parts fill the rest of the chip.  16 sequences of 69-759 rows
// behind 4,096 keys, 32/8 heads, 2.2 rounds of 256 rows: forward 342 us whole, 297 and 18
// for the sums with the last 0.2 in parts; dQ 458 with tiles of 64 rows, 405 and 7 (in a
// running loop; a profiled dozen passes 324 and 434).
// C follows from the offsets on the GPU, so that nothing waits for the host: every
// workgroup computes it, and its place in the list, with a lane per sequence; of more
// sequences than lanes cross_list_kernel writes the list once and a workgroup searches
// it, 64 starts at a time (fwd + bwd of sequences of 1-32 rows over 1-64 keys, 8 heads,
// d = 64, us with every workgroup passing over all sequences / with the list: 128 of
// them 38 / 43, 256 71 / 72, 1,024 331 / 240, 16,384 31,600 / 3,880).
constexpr int kListLanes = 64;
struct CrossCut {
  int keys;       // CrossKeys
  int rows_log2;  // packed rows per tile (dK/dV: per step)
  int key_log2;   // keys per tile
  int max_tiles;  // of a sequence's rows
  int max_parts;  // of an item; 1: not cut
  int least;      // fewest inner tiles of a part
  int entries;    // parts of a kv head
  int even;       // parts to `entries` (EVEN)
  int round;      // whole items, then parts (EVEN; 0: all in parts)
  // more than kListLanes sequences: entries of a kv head before each sequence's (after
  // the shared keys') [n], their number, and C; else NULL
  int32_t* list;
};

struct CrossPlace {
  CrossSeq s;
  int index;  // the sequence's place in the list
  int tile;   // tile of the sequence
  int part, nparts;
};

__device__ __forceinline__ int cross_tiles(int x, int tile) { return (x + tile - 1) / tile; }
__device__ __forceinline__ int cross_tiles_log2(int x, int log2) {
  return (x + (1 << log2) - 1) >> log2;
}

// Tiles of a sequence and the units of inner work of each: tiles of packed rows over
// keys (forward, dQ), and tiles of keys over steps of rows (dK/dV; 2^pack_log2 heads of
// the group to a step).
__device__ __forceinline__ void cross_row_units(const CrossBatch& b, const CrossCut& c,
                                                const CrossSeq& s, bool whole_batch, int& tiles,
                                                int& units) {
  const int pre = c.keys == CROSS_FUSED ? cross_tiles_log2(b.prefix, c.key_log2) : 0;
  tiles = cross_tiles_log2(s.nq * b.g, c.rows_log2);
  if (!whole_batch) tiles = min(tiles, c.max_tiles);
  units = cross_tiles_log2(s.nk, c.key_log2) + pre;
}
__device__ __forceinline__ void cross_key_units(const CrossBatch& b, const CrossCut& c,
                                                int pack_log2, const CrossSeq& s, int& tiles,
                                                int& units) {
  tiles = cross_tiles_log2(s.room, c.key_log2);
  units = s.nk > 0 ? cross_tiles_log2(s.nq << pack_log2, c.rows_log2) * (b.g >> pack_log2) : 0;
}

// C for items of so many units of inner work.
__device__ __forceinline__ int cross_cap(const CrossCut& c, float units) {
  return c.max_parts > 1 ? max(c.least, (int)fminf(units / (float)c.entries + 1.f, 1e9f)) : 1 << 30;
}
// Parts of an item of `units`: ceil(units / cap) as a float product (any whole number
// near it does).
__device__ __forceinline__ int cross_parts(const CrossCut& c, float inv_cap, int units) {
  return max(1, min(c.max_parts, (int)ceilf((float)units * inv_cap)));
}

// Sequence, tile and part of entry `entry` of a kv head's list; false past its end.
// of(s, whole_batch, tiles, units): as above.  The list has the shared keys over the whole
// batch first where `shared` is set (index 0), then the n sequences (index i, or i + 1).
// The results are wave-uniform.
template <bool EVEN, class F>
__device__ __forceinline__ bool cross_place(const CrossBatch& b, const CrossCut& c, bool shared,
                                            int entry, F&& of, CrossPlace& out) {
  const int l = __lane_id(), n = b.n;
  CrossSeq s0 = {0, 0, 0, 0, 0};
  int t0 = 0, u0 = 0;
  if (shared) {
    s0 = cross_shared_seq(b);
    of(s0, true, t0, u0);
  }
  // a part's tiles one after another: workgroups that run at a time then stream the
  // same keys (rows), which L2 holds once
  auto place = [&](int at, int tiles, int parts) __attribute__((always_inline)) {
    out.nparts = parts;
    out.part = parts == 1 ? 0 : at / tiles;
    out.tile = at - out.part * tiles;
  };
  auto in_shared = [&](float inv) __attribute__((always_inline)) {
    const int parts = __builtin_amdgcn_readfirstlane(cross_parts(c, inv, u0));
    if (entry < t0 * parts) {
      out.s = s0;
      out.index = 0;
      place(entry, t0, parts);
    }
    return t0 * parts;
  };
  if (c.list) {
    const float inv = 1.f / (float)c.list[n + 1];
    int rel = entry;
    if (shared) {
      const int base = in_shared(inv);
      if (entry < base) return true;
      rel -= base;
    }
    if (rel >= c.list[n]) return false;
    // the last sequence that starts at `rel` or before: of 64 evenly spaced ones, of
    // the 64th part behind the one found, ...
    int lo = 0, span = n, start = 0;
    while (true) {
      const int step = (span + 63) >> 6;
      const int x = l * step < span ? c.list[lo + l * step] : 0x7fffffff;
      const int k = max(0, __builtin_popcountll(__builtin_amdgcn_ballot_w64(x <= rel)) - 1);
      start = __builtin_amdgcn_readlane(x, k);
      lo += k * step;
      span = min(step, span - k * step);
      if (step == 1) break;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const CrossSeq s = cross_seq(b, lo);
    int t, u;
    of(s, false, t, u);
    const int parts = cross_parts(c, inv, u);
    // (always, unless the offsets are wrong)
    if ((uint32_t)(rel - start) >= (uint32_t)(t * parts)) return false;
    out.s = CrossSeq{s.q_lo, s.nq, s.k_lo, s.nk, s.room};
    out.index = lo + (shared ? 1 : 0);
    place(rel - start, __builtin_amdgcn_readfirstlane(t), __builtin_amdgcn_readfirstlane(parts));
    return true;
  }
  CrossSeq s = {0, 0, 0, 0, 0};
  int t = 0, u = 0;
  if (l < n) {
    s = cross_seq(b, l);
    of(s, false, t, u);
  }
  auto get = [&](int v, int src) __attribute__((always_inline)) {
    return __builtin_amdgcn_readlane(v, src);
  };
  auto found = [&](int src) __attribute__((always_inline)) {
    out.s = CrossSeq{get(s.q_lo, src), get(s.nq, src), get(s.k_lo, src), get(s.nk, src),
                     get(s.room, src)};
    out.index = src + (shared ? 1 : 0);
  };
  if constexpr (EVEN) {
    if (c.even) {
      int first = wave_scan(t) - t;  // items before this sequence's
      const int total = get(first + t, 63);
      if (c.max_parts > 1 && c.round) {
        // (6 bits order equal ones; u is below 2^25)
        const int key = (u << 6) | (63 - l);
        first = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) first += get(key, j) > key ? get(t, j) : 0;
      }
      auto holds = [&](int item) __attribute__((always_inline)) {
        return __builtin_amdgcn_ballot_w64(first <= item && item < first + t);
      };
      int whole = c.max_parts > 1 ? 0 : total, entries = c.entries;
      if (c.max_parts > 1 && c.round) {
        // (a workgroup's start and end cost what 320 keys do)
        const float start = (float)(320 >> c.key_log2);
        const float share = wave_sum((float)t * ((float)u + start)) / (float)c.round;
        float end = 0.f;
        while (whole < total) {
          end += (float)get(u, __builtin_ctzll(holds(whole))) + start;
          if (end > share) break;
          whole += c.round;
        }
        whole = min(whole, total);
        entries = c.round * ((total - whole + c.round - 1) / c.round);
      }
      const int cut = min(t, max(0, first + t - whole));  // the sequence's items in parts
      int cap = 1 << 30;
      if (whole < total) {
        cap = max(c.least, (int)fminf(wave_sum((float)cut * (float)u) / (float)entries + 1.f, 1e9f));
        // by bisection, at most up to the largest item (the parts get fewer as C grows)
        int hi = wave_max(cut > 0 ? u : 0);
        while (cap < hi) {
          const int mid = (cap + hi) >> 1;
          const float inv = 1.f / (float)mid;
          const int e = get(wave_scan(cut * max(1, (int)ceilf((float)u * inv))), 63);
          if (e <= entries) hi = mid;
          else cap = mid + 1;
        }
      }
      const int parts = cross_parts(c, 1.f / (float)cap, u);
      int rel = entry, before = first, mine = t - cut;
      if (entry >= whole) {
        rel -= whole;
        mine = cut * parts;
        before = wave_scan(mine) - mine;
      }
      const uint64_t hit = __builtin_amdgcn_ballot_w64(rel >= before && rel < before + mine);
      if (!hit) return false;
      const int src = __builtin_ctzll(hit);
      found(src);
      const int tiles = get(t, src), cuts = get(cut, src), at = rel - get(before, src);
      if (entry < whole) {
        out.nparts = 1;
        out.part = 0;
        out.tile = at;
      } else {
        place(at, cuts, get(parts, src));
        out.tile += tiles - cuts;
      }
      if (b.causal) out.tile = tiles - 1 - out.tile;
      return true;
    }
  }
  const float units = wave_sum((float)t * (float)u) + (float)t0 * (float)u0;
  const float inv = 1.f / (float)cross_cap(c, units);
  int rel = entry;
  if (shared) {
    const int base = in_shared(inv);
    if (entry < base) return true;
    rel -= base;
  }
  const int parts = cross_parts(c, inv, u);
  const int mine = t * parts;
  const int incl = wave_scan(mine);
  const uint64_t hit = __builtin_amdgcn_ballot_w64(rel >= incl - mine && rel < incl);
  if (!hit) return false;
  const int src = __builtin_ctzll(hit);
  found(src);
  place(rel - get(incl - mine, src), get(t, src), get(parts, src));
  return true;
}

// The same for tiles of packed rows (forward, dQ).
template <bool EVEN>
__device__ __forceinline__ bool cross_place_rows(const CrossBatch& b, const CrossCut& c, int entry,
                                                 CrossPlace& out) {
  return cross_place<EVEN>(
      b, c, c.keys == CROSS_APART, entry,
      [&](const CrossSeq& s, bool whole_batch, int& tiles, int& units)
          __attribute__((always_inline)) {
        cross_row_units(b, c, s, whole_batch, tiles, units);
      },
      out);
}

// The lists of one or two launches (a workgroup each): a thread per run of consecutive
// sequences, their units summed for C, then their entries scanned.
struct CrossListArgs {
  CrossBatch b;
  CrossCut cut[2];
  int kv[2];  // dK/dV
  int pack_log2;
};
constexpr int kListThreads = 1024;
__global__ void __launch_bounds__(kListThreads) cross_list_kernel(CrossListArgs a) {
  constexpr int kWaves = kListThreads / 64;
  __shared__ float wave_units[kWaves];
  __shared__ int64_t wave_entries[kWaves];
  const CrossBatch& b = a.b;
  const CrossCut& c = a.cut[blockIdx.x];
  const int kv = a.kv[blockIdx.x], t = threadIdx.x, w = t >> 6;
  const int run = (b.n + kListThreads - 1) / kListThreads;
  const int first = min(b.n, t * run), last = min(b.n, first + run);
  auto of = [&](const CrossSeq& s, bool whole_batch, int& tiles, int& units)
                __attribute__((always_inline)) {
    if (kv) cross_key_units(b, c, a.pack_log2, s, tiles, units);
    else cross_row_units(b, c, s, whole_batch, tiles, units);
  };
  int tiles, units, cap = cross_cap(c, 0.f);
  if (c.max_parts > 1) {
    float sum = 0.f;
    for (int i = first; i < last; ++i) {
      of(cross_seq(b, i), false, tiles, units);
      sum += (float)tiles * (float)units;
    }
    sum = wave_sum(sum);
    if ((t & 63) == 0) wave_units[w] = sum;
    __syncthreads();
    sum = 0.f;
    for (int i = 0; i < kWaves; ++i) sum += wave_units[i];
    if (kv ? b.prefix > 0 : c.keys == CROSS_APART) {
      of(cross_shared_seq(b), true, tiles, units);
      sum += (float)tiles * (float)units;
    }
    cap = cross_cap(c, sum);
  }
  const float inv = 1.f / (float)cap;
  auto entries = [&](int i) __attribute__((always_inline)) {
    of(cross_seq(b, i), false, tiles, units);
    return (int64_t)tiles * cross_parts(c, inv, units);
  };
  int64_t mine = 0;
  for (int i = first; i < last; ++i) mine += entries(i);
  int64_t at = mine;  // inclusive sum over the wave's lanes
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(at, off, 64);
    if ((t & 63) >= off) at += y;
  }
  if ((t & 63) == 63) wave_entries[w] = at;
  __syncthreads();
  at -= mine;
  for (int i = 0; i < w; ++i) at += wave_entries[i];
  // (past 31 bits, with wrong offsets alone, the list ends)
  auto put = [&](int i) __attribute__((always_inline)) {
    c.list[i] = (int)min(at, (int64_t)0x7fffffff);
  };
  for (int i = first; i < last; ++i) {
    put(i);
    at += entries(i);
  }
  if (t == kListThreads - 1) {
    put(b.n);
    c.list[b.n + 1] = cap;
  }
}

// Token of packed row r (r >= 0): r / g by the reciprocal, off by at most one.
__device__ __forceinline__ int cross_token(const CrossBatch& b, int r) {
  if (b.g == 1) return r;  // uniform
  const int t = (int)__umulhi((uint32_t)r, b.g_inv);
  return r - t * b.g >= b.g ? t + 1 : t;
}

// ---------------------------------------------------------------------------
// Output tiles of packed rows: as store_rows_bf16 and store_rows_f32, with the
// address of a row (0 .. 31 of the wave's tile) from `at`.
// ---------------------------------------------------------------------------
template <int D, class At>
__device__ __forceinline__ void cross_store_bf16(const f32x16 (&acc)[D / 32], float mul, int nrows,
                                                 uint16_t* lds, At&& at) {
  constexpr int P = kBf16Pitch<D>, LANES = D / 8, ROWS = 64 / LANES;
  if (nrows <= 0) return;  // wave-uniform
  const int l = fresh_lane_id();
  const int wr = (l & 31) * P + (l >> 5) * 4;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x16& x = acc[db];
      const f32x2 v01 = {x[g * 4] * mul, x[g * 4 + 1] * mul};
      const f32x2 v23 = {x[g * 4 + 2] * mul, x[g * 4 + 3] * mul};
      *reinterpret_cast<u32x2*>(lds + wr + db * 32 + g * 8) =
          u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(v01, bf16x2)),
                __builtin_bit_cast(uint32_t, __builtin_convertvector(v23, bf16x2))};
    }
  wave_lds_fence();
  const int rr = l / LANES, c = (l % LANES) * 8;
  const uint32_t rd = lds_addr(lds) + (rr * P + c) * 2;
  static_for<32 / ROWS / 4>([&](auto I) {
    constexpr int i0 = decltype(I)::value * 4;
    u32x4 v[4];
    constexpr int o = i0 * ROWS * P * 2, st = ROWS * P * 2;
    lds_read4<o, o + st, o + 2 * st, o + 3 * st>(rd, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (i0 + i) * ROWS + rr;
      if (r < nrows) *reinterpret_cast<u32x4*>((uint16_t*)at(r) + c) = v[i];
    }
  });
  wave_lds_fence();
}

template <int D, int PASS, class At>
__device__ __forceinline__ void cross_store_f32(const f32x16 (&acc)[D / 32], float mul, int nrows,
                                                float* lds, At&& at) {
  static_assert((D / 32) % PASS == 0, "whole passes");
  if (nrows <= 0) return;  // wave-uniform
  const int l = fresh_lane_id();
  const int wr = acc_slot_lane(l);
  const int rr = l >> 3, c = (l & 7) * 4;  // read: 8 lanes a row
  const uint32_t rd = lds_addr(lds) + (rr * kF32Pitch + c) * 4;
  static_for<D / 32 / PASS>([&](auto Pass) {
    constexpr int p = decltype(Pass)::value * PASS;
#pragma unroll
    for (int b = 0; b < PASS; ++b) acc_to_lds(acc[p + b], mul, lds + b * kF32Block, wr);
    wave_lds_fence();
    static_for<PASS>([&](auto B) {
      constexpr int b = decltype(B)::value;
      u32x4 raw[4];
      constexpr int o = b * kF32Block * 4, st = 8 * kF32Pitch * 4;
      lds_read4<o, o + st, o + 2 * st, o + 3 * st>(rd, raw);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i * 8 + rr < nrows)
          *reinterpret_cast<f32x4*>((float*)at(i * 8 + rr) + (p + b) * 32 + c) =
              __builtin_bit_cast(f32x4, raw[i]);
    });
    wave_lds_fence();
  });
}

}  // namespace pdy
