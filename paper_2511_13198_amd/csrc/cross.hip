// C-ABI of the attention over keys of another length and over shared keys:
// argument checks, launch shapes, workspace and launches.  The contract is in
// include/pdyattn.h.
#include "../../include/pdyattn.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "cross_bwd.hpp"
#include "cross_fwd.hpp"
#include "host.hpp"

using namespace pdy_host;

namespace {

struct CrossSizes {
  int64_t tq, tk, n, max_q, max_k, prefix, hq, hkv, d;
  int64_t g() const { return hq / hkv; }
  int64_t seq_rows() const { return max_q * g(); }  // packed rows of the longest sequence
};

pdy_status check_cross_sizes(int32_t prefix, int32_t tq, int32_t tk, int32_t n, int32_t max_q,
                             int32_t max_k, int32_t hq, int32_t hkv, int32_t d, CrossSizes* out) {
  if (tq < 0 || tk < 0)
    return fail(PDY_ERR_INVALID_ARG, "total_q and total_k must be >= 0 (got %d, %d)", tq, tk);
  if (prefix < 0) return fail(PDY_ERR_INVALID_ARG, "prefix_len must be >= 0 (got %d)", prefix);
  if (n < 1) return fail(PDY_ERR_INVALID_ARG, "num_seqs must be >= 1 (got %d)", n);
  if (max_q < 0 || max_q > tq || (tq > 0 && max_q < 1))
    return fail(PDY_ERR_INVALID_ARG, "max_seqlen_q must be in [1, total_q] (got %d, total_q=%d)",
                max_q, tq);
  if (max_k < 0 || max_k > tk)
    return fail(PDY_ERR_INVALID_ARG, "max_seqlen_k must be in [0, total_k] (got %d, total_k=%d)",
                max_k, tk);
  if (hq < 1 || hkv < 1)
    return fail(PDY_ERR_INVALID_ARG, "head counts must be >= 1 (got Hq=%d, Hkv=%d)", hq, hkv);
  if (hq % hkv != 0)
    return fail(PDY_ERR_INVALID_ARG, "num_heads_q (%d) must be a multiple of num_heads_kv (%d)",
                hq, hkv);
  if (d != 64 && d != 128)
    return fail(PDY_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", d);
  // packed rows and workgroups are counted in 32 bits (a tile has 32 rows or more, a
  // sequence an unfilled tile at most)
  if (((int64_t)tq + n) * hq >= (int64_t)1 << 31 || ((int64_t)tk + prefix) * hkv >= (int64_t)1 << 31)
    return fail(PDY_ERR_INVALID_ARG, "problem too large for one launch");
  // (a tile's copies address its 64 tokens of q or 256 keys by bytes in 31 bits)
  if ((int64_t)hq * d >= 1 << 24 || (int64_t)hkv * d >= 1 << 22)
    return fail(PDY_ERR_INVALID_ARG, "too many heads for one launch (Hq=%d, Hkv=%d)", hq, hkv);
  *out = CrossSizes{tq, tk, n, max_q, max_k, prefix, hq, hkv, d};
  return PDY_OK;
}

constexpr int64_t kCUs = 256;

// A launch's workgroups: nw waves in `groups` key groups, 32 * nw / groups rows.
struct CrossShape {
  int nw, groups;
  int rows() const { return 32 * nw / groups; }
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Row tiles of a kv head at most: `rows` packed rows of each of `n` sequences of at
// most max_q of the tq queries.
int64_t most_items(const CrossSizes& s, int64_t n, int64_t max_q, int rows) {
  return std::min(s.tq * s.g() / rows + n, n * ceil_div(max_q * s.g(), rows));
}

// ---- tiles of rows: forward and dQ ----

// Workgroup shapes: 32 rows in 4 key groups, 64 in 2, 128, and 8 waves over 256.  4-wave
// workgroups share a CU by two, so that one's start, end and products overlap the
// other's copies; 8 waves over 256 rows read K and V least often.  Up to 64 rows a
// sequence the smallest tile that holds them is taken.  us with tiles of 32, 64, 128
// and 256 rows, forward, d = 128:
//   17 x 1-5 tokens, 24/8 heads, 900-9,000 keys (15 rows) 64 with 32-row tiles and two
//   workgroups a CU, 80 with one; 32 x 8 tokens, 32/4 heads, 256-8,192 keys (64 rows)
//   52 / 52 / 58 with 64, 128, 256 rows; 32 x 32, 32/8 heads (128 rows) 97 / 82 / 91.
CrossShape few_rows_shape(int64_t rows) {
  if (rows <= 32) return {4, 4};
  return rows <= 64 ? CrossShape{4, 2} : CrossShape{4, 1};
}

// What the forward and the dQ kernel differ in.
struct RowKernel {
  bool dq;
  int key_tile(const CrossSizes& s, const CrossShape& sh) const {
    if (dq) return sh.nw == 8 ? 128 : 64;
    if (sh.nw == 4) return sh.groups == 4 ? 128 : 64;
    return s.d == 128 ? 128 : 64;
  }
  // workgroups of a shape on the chip at a time (d = 64: by registers and LDS)
  int64_t slots(const CrossSizes& s, const CrossShape& sh) const {
    if (sh.nw == 8) return s.d == 64 ? 2 * kCUs : kCUs;
    return s.d == 64 && !dq ? 3 * kCUs : 2 * kCUs;
  }
  // a workgroup's time on 64 keys, alone on its CU or beside others: d = 128, 200 rows x
  // 30,810 keys x 16 heads (64 x 484 such units) and 8 x 256-2,048 rows over 1,024-8,192
  // keys, 32/8 heads (a full chip); d = 64, 4 x 281-1,127 rows behind 24,028 keys
  double unit_us(const CrossSizes& s, const CrossShape& sh, bool full) const {
    if (s.d == 64) {
      if (sh.nw == 8) return full ? 1.9 : 1.2;
      return sh.groups == 1 ? (full ? 1.9 : 1.1) : full ? 0.95 : 0.85;
    }
    if (sh.nw == 8) return dq ? 1.75 : 1.48;
    if (sh.groups == 1) return dq ? (full ? 2.0 : 1.4) : full ? 1.6 : 1.46;
    return dq ? (full ? 1.1 : 0.85) : 1.1;
  }
};
constexpr RowKernel kFwd{false}, kDq{true};

// One launch over tiles of rows.
struct CrossRows {
  CrossShape sh;
  pdy::CrossCut cut;
  int64_t wgs;  // per kv head
};

constexpr int kMaxParts = 64;
// Sequences that every workgroup puts in order for whole rounds, at about 0.1 us each: 51
// sequences' forward 47 us unsorted, 55 sorted.
constexpr int64_t kSorted = 32;
constexpr int64_t kPartBytes = (int64_t)256 << 20;  // partial results at most
constexpr double kMoveBytesPerUs = 4.0e6;           // partial results written and read back

// Few rows a sequence behind many shared keys: these once for the rows of all
// sequences, apart from the sequences' own keys, with partial results of both.  Fused,
// every sequence's tile of 32 rows or more streams them; us apart / fused, d = 128:
//   64 sequences of 1 token, 32/8 heads, behind 32,768 keys 97 / 662; 32 of 8 tokens (32
//   rows) behind 8,000 64 / 78, of 16 (64 rows) 99 / 138, of 32 (128 rows, 40 sequences,
//   a step) 853 / 858.
// Where the (sequence, kv head) pairs are more than 4 a CU, fused takes rounds that apart
// does not.  Apart saves what a tile has beyond a sequence's R rows and costs partial
// results a row, so the keys from which it pays grow with R / (tile - R).  us fused / apart
// (or their ratio) behind so many shared keys, 1,280-4,096 pairs:
//   d = 128: R = 1, 512 sequences of 8/8 heads over 100 own keys: 128 79 / 79, 256 91 / 79;
//   R = 4, 32/8 heads: 128 80 / 88, 256 93 / 89; R = 8, 2,048 of 16/2 over 400: 256 0.94,
//   512 of 32/4 over 1,000-2,000: 250 317 / 338;
//   R = 16, 256 of 8/8 over 400: 200 97 / 113, 700 123 / 119; R = 32, 160 of 32/8 over 30:
//   1,000 66 / 80, 2,000 101 / 98; R = 64, 256 of 16/8 over 100: 1,000 124 / 191, 3,500
//   312 / 346
//   d = 64: R = 1: 128 55 / 42; R = 4: 128 57 / 51, 256 64 / 52; R = 8: 128 0.95, 192 1.02,
//   over 1,000-2,000 120 168 / 182;
//   R = 16: 200 62 / 72, 400 71 / 75, 700 80 / 76; R = 32: 1,000 49 / 54, 2,000 69 / 63;
//   R = 64: 1,000 67 / 131, 3,500 176 / 217
// Up to 6 pairs a CU fused keeps 256 keys, which long own keys want: 140 sequences of 8/8
// heads over 3,000-6,000 keys, d = 64, behind 16-120 286 / 331, d = 128, behind 160-250 481 /
// 515 (over up to 2,000 35 / 34 and 63 / 62; 130 over 30 keys of d = 64 behind 128 1.14).
constexpr int64_t kApartRows = 64, kApartPrefix = 512, kApartPrefixMany = 256;
int64_t fused_keys(const CrossSizes& s) {
  const int64_t pairs = s.n * s.hkv, rows = s.seq_rows();  // (rows: at most kApartRows)
  if (pairs <= 4 * kCUs) return kApartPrefix;
  const int64_t line = (s.d == 64 ? 0 : 128) +
                       (rows <= 32 ? 800 * rows / (54 - rows) : 500 * rows / (72 - rows));
  return pairs <= 6 * kCUs ? std::max(kApartPrefixMany, line) : line;
}

// Few rows over so many keys at most, shared ones among them, are one whole item a tile:
// the launch that combines partial results takes longer than these save.  us with parts /
// whole, a token for each of 1-60 sequences over 400, 800, 1,500 keys: d = 64 10.6 / 7.8,
// 11.0 / 9.9, 10.7 / 14.0; d = 128 11.6 / 10.2, 12.5 / 13.9, 11.8 / 20.5.  Parts / whole behind
// 256 shared and 400 own keys, 32/8 heads of 128, 64 sequences 28.7 / 24.0, 512 167 / 167.
// Apart / whole, up to a pair a CU, over 100 own and 520, 700 shared keys: 8 sequences of 32/8
// heads of 128 13.2 / 13.4, 12.0 / 14.9, of 64 11.1 / 9.9, 10.4 / 10.7; 32 of them 17.1 / 16.2,
// 17.1 / 18.0 and d = 64 whole / apart 0.82, 0.89.
// From one to two pairs a CU the line grows with a sequence's rows R, as above.  Time whole
// over time apart, 384 and 512 pairs over 100 and 400 own keys:
//   d = 128, R = 1: behind 520 keys 0.98-1.14, 600 0.98-1.21; R = 4: 520 0.88-1.00, 700
//   0.90-1.09, 800 0.95-1.16; R = 8: 700 0.79-1.00, 900 0.89-0.97; R = 16: 700 0.79; R = 64:
//   700 0.50
//   d = 64, R = 1: 520 0.96-1.06, 600 0.96-1.05; R = 4: 700 0.91-1.04, 800 0.96-1.07; R = 8:
//   900 0.92-0.98; R = 16: 700 0.78; R = 64: 700 0.56
bool short_keys(const CrossSizes& s) {
  const int64_t pairs = s.n * s.hkv;
  if (s.prefix > kApartPrefix && pairs > kCUs && pairs <= 2 * kCUs)
    return s.prefix <= 500 + 60 * s.seq_rows() && s.max_k <= 512;
  const int64_t most = s.prefix > kApartPrefix ? (s.d == 64 ? 800 : 640)
                       : s.d == 64 || (s.prefix > 0 && pairs >= 2 * kCUs) ? 1024 : 512;
  return s.max_k + s.prefix <= most;
}

// Shape and parts of a launch over sequences of more than 64 rows: the ones of least
// estimated time, from the average rows and keys of a sequence.  With I items of u
// units, on `slots` workgroups at a time,
//   whole: ceil(I / slots) (start + u unit), and no less than the longest item's;
//   in p parts: ceil(I p / slots) (start + u / p unit) + partial results;
//   whole rounds, the rest in parts: I (start + u unit) / slots + start + partial results.
// us measured, 256-row tiles / 128 whole / 128 in parts (their sums included): 9 x 427
// rows x 4 heads 56 / 59 / 57, 51 x 79 x 16 64 / 49 / 57, 2,000 x 8 over 3,000 keys 79 / 76
// / 54, 4 x 1,041 x 8 causal 37 / 38 / 44; 21 x 208 rows over 1-5,792 keys, one head, whole
// 67, in parts 26.
struct RowsChoice {
  CrossShape sh;
  int parts;        // 1: whole
  int64_t entries;  // of all heads: whole rounds
  int64_t round;    // of all heads: whole rounds, then parts (0: all alike)
};
RowsChoice choose_rows(const CrossSizes& s, const RowKernel& k, bool causal) {
  const double own = std::min<double>((double)s.max_k, (double)s.tk / s.n);
  const double seen = causal ? std::max(own - 0.5 * s.tq / s.n, 0.5 * own) : own;
  const double keys = seen + s.prefix, rows = (double)s.tq * s.g();
  const double longest = std::max(1.0, (double)(s.max_k + s.prefix) / 64);
  const double alike = std::min(1.0, (own + s.prefix) / (64 * longest));
  RowsChoice best{{8, 1}, 1, 0, 0};
  double least = 1e30;
  constexpr double kStart = 7.0, kMerge = 5.0;
  for (const CrossShape& sh : {CrossShape{8, 1}, CrossShape{4, 1}, CrossShape{4, 2}}) {
    if (sh.rows() >= 2 * s.seq_rows()) continue;
    const int64_t slots = k.slots(s, sh);
    const double items = std::min(rows / sh.rows() + 0.5 * s.n,
                                  (double)most_items(s, s.n, s.max_q, sh.rows())) * s.hkv;
    const double units = std::max(1.0, keys / 64);
    for (int p = 1; p <= kMaxParts && p <= std::max(1.0, units / 4); ++p) {
      const double bytes = (double)p * rows * s.hkv * s.d * 4;
      if (p > 1 && bytes > kPartBytes) break;
      const double rounds = std::ceil(items * p / slots);
      const double unit = k.unit_us(s, sh, items * p > kCUs);
      // (items that differ in length do not end in rounds)
      const double lasts = p > 1 ? rounds : alike * rounds + (1 - alike) * (items / slots + 0.5);
      double t = lasts * (kStart + units / p * unit);
      // (parts have to be better by 5%, whole rounds and parts by 8%: the estimates are
      // that wrong)
      if (p > 1) t = (t + kMerge + 2.0 * bytes / kMoveBytesPerUs) / 0.95;
      else t = std::max(t, kStart + longest * unit);
      if (t < least) {
        least = t;
        best = {sh, p, (int64_t)rounds * slots, 0};
      }
    }
    // (more than a round, or parts would do as well)
    const double bytes = std::min<double>((double)slots * sh.rows(), kMaxParts * rows * s.hkv) *
                         s.d * 4;
    const double t = (items * (kStart + units * k.unit_us(s, sh, true)) / slots + kStart + kMerge +
                      2.0 * bytes / kMoveBytesPerUs) / 0.92;
    if (items > slots && s.n <= kSorted && t < least) {
      least = t;
      best = {sh, 2, slots, slots};
    }
  }
  return best;
}

// Whether the longest of `items` whole items takes longer than all of them side by side, by
// more than the launch that combines parts (16 units of 64 keys): one long sequence among
// short ones.  us whole / in parts: 512 x 1 token, 32/8 heads of 128, over 1,000 keys and one
// of 131,072 2,826 / 497, of 32,768 985 / 469, of 8,192 520 / 457, of 4,096 444 / 447; 32 x 64,
// 16/16 heads, over 300 keys and one of 16,384 275 / 60, of 2,048 49 / 38, of 1,024 34 / 38.
// Even lengths behind too large a bound pay for it: the 512 over 300 keys, 16,384 said, 144 /
// 148; 64 x 64 over 300, 4,096 said, 40 / 47.
bool outlasts(const CrossSizes& s, const RowKernel& k, const CrossShape& sh, int64_t items) {
  const double mean = std::min<double>((double)s.max_k, (double)s.tk / s.n) + s.prefix;
  const double longest = (double)(s.max_k + s.prefix);
  return longest > 0.8 * (double)items * mean / (double)k.slots(s, sh) + 16 * 64;
}

CrossRows rows_launch(const CrossSizes& s, const RowKernel& k, bool causal) {
  CrossRows f;
  pdy::CrossCut& c = f.cut;
  // bytes of one slice of partial results (no queries: nothing is launched)
  const int64_t slice = std::max<int64_t>(1, s.tq) * s.hq * (s.d + 1) * 4;
  const int64_t pairs = s.n * s.hkv;
  c.keys = s.prefix == 0 ? pdy::CROSS_OWN
           : s.seq_rows() > kApartRows || 2 * slice > kPartBytes || s.prefix <= fused_keys(s) ||
                   (pairs <= 2 * kCUs && short_keys(s))
               ? pdy::CROSS_FUSED
               : pdy::CROSS_APART;
  const bool apart = c.keys == pdy::CROSS_APART;
  int64_t most = kMaxParts, entries, round = 0;  // parts of an item, and of all
  if (s.seq_rows() > 64) {
    const RowsChoice r = choose_rows(s, k, causal);
    f.sh = r.sh;
    entries = r.entries;
    round = r.round;
    if (r.parts == 1) most = 1;
  } else {
    f.sh = few_rows_shape(apart ? s.tq * s.g() : s.seq_rows());
    // (few rows are bound by reading keys, of lengths that the host does not know:
    // more parts than fit at a time even them out)
    const bool few = f.sh.groups == 4;
    if (k.dq && few) f.sh = {4, 2};
    entries = (few ? 4 : 2) * kCUs;
    const int64_t items = most_items(s, s.n, s.max_q, f.sh.rows()) * s.hkv;
    if (!apart && (items >= (few ? 16 : 2) * kCUs || short_keys(s)) &&
        !outlasts(s, k, f.sh, items))
      most = 1;
  }
  const int rows = f.sh.rows(), keys_tile = k.key_tile(s, f.sh);
  c.rows_log2 = __builtin_ctz((unsigned)rows);
  c.key_log2 = __builtin_ctz((unsigned)keys_tile);
  c.max_tiles = (int)ceil_div(s.seq_rows(), rows);
  c.least = 2;
  const int64_t items =
      most_items(s, s.n, s.max_q, rows) + (apart ? ceil_div(s.tq * s.g(), rows) : 0);
  c.entries = (int)ceil_div(entries, s.hkv);
  c.even = s.seq_rows() > 64;
  c.round = (int)ceil_div(round, s.hkv);
  c.list = nullptr;
  const int64_t own = ceil_div(s.max_k, keys_tile), pre = ceil_div(s.prefix, keys_tile);
  const int64_t tiles = apart ? std::max(own, pre) : own + pre;
  most = std::min<int64_t>({most, tiles / c.least, kPartBytes / (slice * (apart ? 2 : 1))});
  c.max_parts = (int)std::max<int64_t>(1, most);
  f.wgs = items + (c.max_parts > 1 ? c.entries + 2 : 0);
  return f;
}

// Whether a grid's threads can be counted in 32 bits, as a launch's are.
bool fits_grid(int64_t wgs, int threads) { return wgs * threads < (int64_t)1 << 32; }

// Partial results that a launch writes at most (0: none).
int slices_of(const CrossRows& f) {
  return f.cut.keys == pdy::CROSS_APART ? 2 * f.cut.max_parts
                                        : f.cut.max_parts > 1 ? f.cut.max_parts : 0;
}

// The list of a launch over more sequences than lanes.
size_t list_bytes(const CrossSizes& s) {
  return s.n > pdy::kListLanes ? align256((size_t)(s.n + 2) * 4) : 0;
}
size_t part_n_bytes(const CrossSizes& s) { return align256((size_t)s.tq * s.hq * 2 * 4); }
size_t part_o_bytes(const CrossSizes& s, int slices) {
  return align256((size_t)slices * s.tq * s.hq * s.d * 4);
}
size_t part_lse_bytes(const CrossSizes& s, int slices) {
  return align256((size_t)slices * s.tq * s.hq * 4);
}

size_t fwd_bytes(const CrossSizes& s, const CrossRows& f) {
  const int n = slices_of(f);
  return list_bytes(s) +
         (n == 0 ? 256 : part_n_bytes(s) + part_o_bytes(s, n) + part_lse_bytes(s, n));
}

// ---- tiles of keys: dK, dV ----
struct CrossKv {
  CrossShape sh;  // groups: query groups; 32 * nw / groups keys
  pdy::CrossCut cut;
  int64_t wgs;    // per kv head
};

int pack_log2(const CrossSizes& s) {
  int n = 0;
  while (n < 5 && s.g() % (2 << n) == 0) ++n;
  return n;
}

// rooms: max_k may bound the keys in use alone, and tiles cover those not in use too.
CrossKv kv_launch(const CrossSizes& s, bool rooms) {
  CrossKv k;
  auto items = [&](int tile) {
    return std::min(s.tk / tile + s.n, s.n * ceil_div(s.max_k, tile)) + ceil_div(s.prefix, tile);
  };
  // Few rows a sequence, so few steps a tile, or d = 64: two 4-wave workgroups a CU; else
  // 256-key tiles where they fill the chip four times over, two query groups over 128
  // where not.  us with 4 waves, 8, and 8 in groups: 16 sequences of 64-1,024 rows behind
  // 4,096 keys, 32/8 heads 616 / 607 / 580; 9 x 427 rows x 273-2,190 keys, 16/4 heads 84 /
  // 93 / 76; 51 x 79 behind 385, 16 heads 70 / 77 / 84; d = 64, 32 x 8-200 rows over
  // 577-1,024 keys, 16 heads 60 / 63 / 110, 4 x 281-1,127 behind 24,028, 16/8 heads 419 /
  // 438 / 487.
  if (items(128) * s.hkv >= 2 * kCUs && (s.d == 64 || s.tq * s.g() <= 512 * s.n)) k.sh = {4, 1};
  else k.sh = {8, items(256) * s.hkv >= 4 * kCUs ? 1 : 2};
  pdy::CrossCut& c = k.cut;
  c.keys = pdy::CROSS_FUSED;
  c.key_log2 = __builtin_ctz((unsigned)k.sh.rows());
  c.rows_log2 = k.sh.nw == 4 && s.d == 128 ? 5 : 6;  // CrossDkdvCfg::BQ
  c.max_tiles = 0;  // (of rows)
  c.list = nullptr;
  c.least = 4;
  const int64_t n = items(k.sh.rows()), target = kCUs;
  c.entries = (int)ceil_div(target, s.hkv);
  c.even = c.round = 0;
  const int64_t slice = (s.prefix + s.tk) * s.hkv * s.d * 8;
  int64_t parts = std::min<int64_t>(16, slice ? kPartBytes / slice : 1);
  // Items alike in their rows need no cut once they fill the chip; a shared tile has
  // the rows of all sequences, and one sequence may have many more rows than the others:
  // its items' steps against an even share of all, as for rows above.  us of a backward with
  // parts / whole: 300 x 16 tokens over 60 keys, 8/1 heads of 128, one of 8,192 tokens 173 /
  // 1,439, of 512 60 / 129, of 128 55 / 65; 256 x 16 of 32/8 over as many keys, one of 512 134 /
  // 169, of 128 110 / 105; even lengths, 2,048 said, 215 / 213.
  const int64_t steps_of = (int64_t)1 << c.rows_log2;
  const double slots = (k.sh.nw == 4 ? 2.0 : 1.0) * kCUs;
  const double share = std::max(1.0, (double)(s.tq * s.g()) / (s.n * steps_of)) * n * s.hkv / slots;
  const bool alike = s.prefix == 0 && (double)(s.max_q * s.g()) / steps_of <= share + 8;
  if (n * s.hkv >= target && (alike || s.n == 1)) parts = 1;
  // Items of few steps are not cut: the launch that sums parts takes longer than they
  // save.  us of a backward with parts / whole, longest items of 1, 4, 8 and 16 steps: 4
  // sequences over 300 keys, 8 heads, d = 64 18.6 / 16.1, 23.5 / 21.0, 28.9 / 22.4, 36.2 /
  // 24.7; 8 query heads to one of 128 28.7 / 25.7 (2), 35.6 / 34.9 (8), 36.9 / 47.8 (16).
  const int sh = pack_log2(s);
  const int64_t rows = s.prefix > 0 ? s.tq : s.max_q;  // that see the longest
  if (ceil_div(rows << sh, 1 << c.rows_log2) * (s.g() >> sh) <= 8) parts = 1;
  c.max_parts = (int)std::max<int64_t>(1, parts);
  const int64_t tiles = rooms ? s.tk / k.sh.rows() + s.n + ceil_div(s.prefix, k.sh.rows()) : n;
  k.wgs = tiles + (c.max_parts > 1 ? c.entries + 2 : 0);
  return k;
}

// Workspace of a backward: the lists, D, the counts of parts, the partial dQ, and dK and
// dV.
struct CrossBwdSpace {
  size_t list, dd, counts_q, counts_k, part_q, part_kv, total;
};
CrossBwdSpace bwd_space(const CrossSizes& s, const CrossRows& q, const CrossKv& kv) {
  CrossBwdSpace x;
  x.list = list_bytes(s);
  x.dd = align256((size_t)s.hq * s.tq * 4);
  x.counts_q = slices_of(q) ? part_n_bytes(s) : 0;
  x.counts_k = kv.cut.max_parts > 1 ? align256((size_t)(s.prefix + s.tk) * 4) : 0;
  x.part_q = part_o_bytes(s, slices_of(q));
  x.part_kv = kv.cut.max_parts > 1 ? align256((size_t)kv.cut.max_parts * (s.prefix + s.tk) *
                                              s.hkv * s.d * 4)
                                   : 0;
  x.total = std::max<size_t>(256, 2 * x.list + x.dd + x.counts_q + x.counts_k + x.part_q + 2 * x.part_kv);
  return x;
}

// ---- kernels by shape; called without arguments they set their attributes ----
template <int D, int NW, int KG>
hipError_t launch_fwd(const pdy::CrossFwdArgs* a, dim3 grid, hipStream_t st) {
  using C = pdy::CrossFwdCfg<D, NW, KG>;
  if (a == nullptr) return set_lds(pdy::cross_fwd_kernel<D, NW, KG>, C::LDS_BYTES);
  hipLaunchKernelGGL((pdy::cross_fwd_kernel<D, NW, KG>), grid, dim3(C::NT), C::LDS_BYTES, st, *a);
  return hipSuccess;
}
template <int D, int NW, int KG>
hipError_t launch_dq(const pdy::CrossBwdArgs* a, dim3 grid, hipStream_t st) {
  using C = pdy::CrossDqCfg<D, NW, KG>;
  if (a == nullptr) return set_lds(pdy::cross_dq_kernel<D, NW, KG>, C::LDS_BYTES);
  hipLaunchKernelGGL((pdy::cross_dq_kernel<D, NW, KG>), grid, dim3(C::NT), C::LDS_BYTES, st, *a);
  return hipSuccess;
}
template <int D, int NW, int QG>
hipError_t launch_dkdv(const pdy::CrossBwdArgs* a, dim3 grid, hipStream_t st) {
  using C = pdy::CrossDkdvCfg<D, QG, NW>;
  if (a == nullptr) return set_lds(pdy::cross_dkdv_kernel<D, QG, NW>, C::LDS_BYTES);
  hipLaunchKernelGGL((pdy::cross_dkdv_kernel<D, QG, NW>), grid, dim3(C::NT), C::LDS_BYTES, st, *a);
  return hipSuccess;
}

struct CrossKernels {
  int nw, groups;
  hipError_t (*fwd[2])(const pdy::CrossFwdArgs*, dim3, hipStream_t);  // d = 64, 128
  hipError_t (*dq[2])(const pdy::CrossBwdArgs*, dim3, hipStream_t);
  hipError_t (*dkdv[2])(const pdy::CrossBwdArgs*, dim3, hipStream_t);
};
template <int NW, int G>
constexpr CrossKernels row_kernels() {
  return {NW, G, {launch_fwd<64, NW, G>, launch_fwd<128, NW, G>},
          {launch_dq<64, NW, G>, launch_dq<128, NW, G>}, {nullptr, nullptr}};
}
// (dK/dV of d = 64 has no 256-key tiles: no launch takes them)
template <int NW, int G>
constexpr CrossKernels with_dkdv(CrossKernels k) {
  k.nw = NW;
  k.groups = G;
  if constexpr (NW == 4 || G > 1) k.dkdv[0] = launch_dkdv<64, NW, G>;
  k.dkdv[1] = launch_dkdv<128, NW, G>;
  return k;
}
constexpr CrossKernels kCrossKernels[] = {
    with_dkdv<8, 1>(row_kernels<8, 1>()), with_dkdv<4, 1>(row_kernels<4, 1>()),
    row_kernels<4, 2>(), with_dkdv<8, 2>(CrossKernels{}),
    CrossKernels{4, 4, {launch_fwd<64, 4, 4>, launch_fwd<128, 4, 4>}, {}, {}}};
const CrossKernels& cross_kernels(const CrossShape& sh) {
  for (const CrossKernels& k : kCrossKernels)
    if (k.nw == sh.nw && k.groups == sh.groups) return k;
  return kCrossKernels[0];  // (not reached: every shape the launches use is listed)
}

hipError_t init_cross_kernels() {
  static hipError_t status = [] {
    for (const CrossKernels& k : kCrossKernels)
      for (int d = 0; d < 2; ++d) {
        hipError_t e = hipSuccess;
        if (k.fwd[d]) e = k.fwd[d](nullptr, dim3(), nullptr);
        if (e == hipSuccess && k.dq[d]) e = k.dq[d](nullptr, dim3(), nullptr);
        if (e == hipSuccess && k.dkdv[d]) e = k.dkdv[d](nullptr, dim3(), nullptr);
        if (e != hipSuccess) return e;
      }
    return hipSuccess;
  }();
  return status;
}

pdy_status check_offsets(const int32_t* p, const char* name) {
  if (p == nullptr) return fail(PDY_ERR_INVALID_ARG, "%s is NULL", name);
  if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0)
    return fail(PDY_ERR_INVALID_ARG, "%s is not 4-byte aligned", name);
  return PDY_OK;
}

struct CrossIn {
  const void *q, *k, *v, *kp, *vp;
  const int32_t *cu_q, *cu_k, *len_k;
};

pdy_status check_cross_in(const CrossIn& x, const CrossSizes& s) {
  pdy_status st;
  if ((st = check_offsets(x.cu_q, "cu_seqlens_q")) || (st = check_offsets(x.cu_k, "cu_seqlens_k")))
    return st;
  if (s.tq > 0 && (st = check_ptr(x.q, "q"))) return st;
  if (s.tk > 0 && ((st = check_ptr(x.k, "k")) || (st = check_ptr(x.v, "v")))) return st;
  if (s.prefix > 0 && ((st = check_ptr(x.kp, "k_prefix")) || (st = check_ptr(x.vp, "v_prefix"))))
    return st;
  if (x.len_k && (reinterpret_cast<uintptr_t>(x.len_k) & 3u) != 0)
    return fail(PDY_ERR_INVALID_ARG, "seqlens_k is not 4-byte aligned");
  return PDY_OK;
}

pdy::CrossBatch batch_of(const CrossIn& x, const CrossSizes& s, int32_t causal) {
  return pdy::CrossBatch{x.cu_q, x.cu_k, x.len_k, (int)s.n, (int)s.tq, (int)s.tk, (int)s.prefix,
                         (int)s.hq, (int)s.hkv, (int)s.g(), (uint32_t)((1ull << 32) / s.g()),
                         causal, (int)(x.len_k ? s.tk : s.max_k)};
}

// The lists of a launch over rows, over keys (NULL: none), or both.
hipError_t launch_lists(const pdy::CrossBatch& b, const pdy::CrossCut* q, const pdy::CrossCut* kv,
                        int pack_log2, hipStream_t hs) {
  pdy::CrossListArgs l{b, {}, {}, pack_log2};
  int n = 0;
  if (q) l.cut[n++] = *q;
  if (kv) {
    l.kv[n] = 1;
    l.cut[n++] = *kv;
  }
  return launch_timed(K_CROSS_LIST, hs, [&] {
    hipLaunchKernelGGL(pdy::cross_list_kernel, dim3(n), dim3(pdy::kListThreads), 0, hs, l);
  });
}

pdy_status cross_fwd_impl(const CrossIn& x, const CrossSizes& s, int32_t causal, float scale,
                          void* o, float* lse, void* workspace, size_t workspace_bytes,
                          void* stream, const char* who) {
  pdy_status st;
  if ((st = check_scale(scale, causal)) != PDY_OK) return st;
  if (s.tq == 0) return PDY_OK;
  if ((st = check_cross_in(x, s)) || (st = check_ptr(o, "o")) || (st = check_ptr(lse, "lse")) ||
      (st = check_ptr(workspace, "workspace")))
    return st;
  CrossRows f = rows_launch(s, kFwd, causal != 0);
  const size_t need = fwd_bytes(s, f);
  if (workspace_bytes < need)
    return fail(PDY_ERR_WORKSPACE, "workspace has %zu bytes, %s needs %zu", workspace_bytes, who,
                need);
  if (!fits_grid(f.wgs * s.hkv, f.sh.nw * 64))
    return fail(PDY_ERR_INVALID_ARG, "problem too large for one launch");
  hipError_t e = init_cross_kernels();
  if (e != hipSuccess) return hip_fail(e, "kernel attribute setup");
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);

  const int slices = slices_of(f);
  uint8_t* const lists = reinterpret_cast<uint8_t*>(workspace);
  uint8_t* const w = lists + list_bytes(s);
  pdy::CrossFwdArgs a;
  a.q = static_cast<const uint16_t*>(x.q);
  a.k = static_cast<const uint16_t*>(x.k);
  a.v = static_cast<const uint16_t*>(x.v);
  a.kp = static_cast<const uint16_t*>(x.kp);
  a.vp = static_cast<const uint16_t*>(x.vp);
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.b = batch_of(x, s, causal);
  if (list_bytes(s)) {
    f.cut.list = reinterpret_cast<int32_t*>(lists);
    e = launch_lists(a.b, &f.cut, nullptr, 0, hs);
    if (e != hipSuccess) return hip_fail(e, "cross_list_kernel launch");
  }
  a.cut = f.cut;
  a.scale_log2 = scale * pdy::kLog2e;
  a.part_n = slices ? reinterpret_cast<int32_t*>(w) : nullptr;
  a.part_o = reinterpret_cast<float*>(w + part_n_bytes(s));
  a.part_lse = reinterpret_cast<float*>(w + part_n_bytes(s) + part_o_bytes(s, slices));
  const dim3 grid((unsigned)(f.wgs * s.hkv));
  e = launch_timed(K_CROSS_FWD, hs,
                   [&] { (void)cross_kernels(f.sh).fwd[s.d == 128](&a, grid, hs); });
  if (e != hipSuccess) return hip_fail(e, "cross_fwd_kernel launch");
  if (slices == 0) return PDY_OK;
  const pdy::CrossMergeArgs m{a.part_o, a.part_lse, a.part_n, f.cut.max_parts,
                              f.cut.keys == pdy::CROSS_APART, x.cu_q, (int)s.n, (int)s.tq,
                              (int)s.hq, a.o, lse};
  const dim3 blocks((unsigned)ceil_div(s.tq * s.hq, 4));
  e = launch_timed(K_CROSS_MERGE, hs, [&] {
    if (s.d == 64) hipLaunchKernelGGL(pdy::cross_merge_kernel<64>, blocks, dim3(256), 0, hs, m);
    else hipLaunchKernelGGL(pdy::cross_merge_kernel<128>, blocks, dim3(256), 0, hs, m);
  });
  if (e != hipSuccess) return hip_fail(e, "cross_merge_kernel launch");
  return PDY_OK;
}

struct CrossGrads {
  void *dq, *dk, *dv, *dkp, *dvp;
};

pdy_status cross_bwd_impl(const CrossIn& x, const void* o, const float* lse, const void* dout,
                          const CrossSizes& s, int32_t causal, float scale, int32_t grad_bf16,
                          const CrossGrads& g, void* workspace, size_t workspace_bytes,
                          void* stream, const char* who) {
  pdy_status st;
  if ((st = check_scale(scale, causal)) != PDY_OK) return st;
  if (grad_bf16 != 0 && grad_bf16 != 1)
    return fail(PDY_ERR_INVALID_ARG, "grad_bf16 must be 0 or 1 (got %d)", grad_bf16);
  if (s.tq == 0 && s.tk == 0 && s.prefix == 0) return PDY_OK;
  if ((st = check_cross_in(x, s)) != PDY_OK) return st;
  if (s.tq > 0 && ((st = check_ptr(o, "o")) || (st = check_ptr(lse, "lse")) ||
                   (st = check_ptr(dout, "dout")) || (st = check_ptr(g.dq, "dq"))))
    return st;
  if (s.tk > 0 && ((st = check_ptr(g.dk, "dk")) || (st = check_ptr(g.dv, "dv")))) return st;
  if (s.prefix > 0 &&
      ((st = check_ptr(g.dkp, "dk_prefix")) || (st = check_ptr(g.dvp, "dv_prefix"))))
    return st;
  if ((st = check_ptr(workspace, "workspace")) != PDY_OK) return st;
  CrossRows f = rows_launch(s, kDq, causal != 0);
  CrossKv kv = kv_launch(s, x.len_k != nullptr);
  const CrossBwdSpace sp = bwd_space(s, f, kv);
  if (workspace_bytes < sp.total)
    return fail(PDY_ERR_WORKSPACE, "workspace has %zu bytes, %s needs %zu", workspace_bytes, who,
                sp.total);
  if (!fits_grid(f.wgs * s.hkv, f.sh.nw * 64) || !fits_grid(kv.wgs * s.hkv, kv.sh.nw * 64))
    return fail(PDY_ERR_INVALID_ARG, "problem too large for one launch");
  hipError_t e = init_cross_kernels();
  if (e != hipSuccess) return hip_fail(e, "kernel attribute setup");
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);

  uint8_t* w = reinterpret_cast<uint8_t*>(workspace);
  auto take = [&](size_t bytes) {
    uint8_t* r = w;
    w += bytes;
    return r;
  };
  uint8_t* const lists = take(2 * sp.list);
  float* dd = reinterpret_cast<float*>(take(sp.dd));
  int32_t* counts_q = reinterpret_cast<int32_t*>(take(sp.counts_q));
  int32_t* counts_k = reinterpret_cast<int32_t*>(take(sp.counts_k));
  float* part_q = reinterpret_cast<float*>(take(sp.part_q));
  float* part_k = reinterpret_cast<float*>(take(sp.part_kv));
  float* part_v = reinterpret_cast<float*>(take(sp.part_kv));

  pdy::CrossBwdArgs a;
  a.q = static_cast<const uint16_t*>(x.q);
  a.k = static_cast<const uint16_t*>(x.k);
  a.v = static_cast<const uint16_t*>(x.v);
  a.kp = static_cast<const uint16_t*>(x.kp);
  a.vp = static_cast<const uint16_t*>(x.vp);
  a.o = static_cast<const uint16_t*>(o);
  a.dout = static_cast<const uint16_t*>(dout);
  a.lse = lse;
  a.dd = dd;
  a.dq = g.dq;
  a.dk = g.dk;
  a.dv = g.dv;
  a.dkp = g.dkp;
  a.dvp = g.dvp;
  a.out_bf16 = grad_bf16;
  a.b = batch_of(x, s, causal);
  a.scale = scale;
  a.scale_log2 = scale * pdy::kLog2e;
  a.pack_log2 = pack_log2(s);
  // (keys of no sequence alone: no tile of keys)
  const bool rows = s.tq > 0, keys = kv.wgs > 0;
  if (sp.list && (rows || keys)) {
    f.cut.list = reinterpret_cast<int32_t*>(lists);
    kv.cut.list = reinterpret_cast<int32_t*>(lists + sp.list);
    e = launch_lists(a.b, rows ? &f.cut : nullptr, keys ? &kv.cut : nullptr, a.pack_log2, hs);
    if (e != hipSuccess) return hip_fail(e, "cross_list_kernel launch");
  }

  // dQ first: it also writes D, which dK/dV reads
  if (rows) {
    a.cut = f.cut;
    a.part = part_q;
    a.part2 = nullptr;
    a.part_n = slices_of(f) ? counts_q : nullptr;
    const dim3 grid((unsigned)(f.wgs * s.hkv));
    e = launch_timed(K_CROSS_DQ, hs,
                     [&] { (void)cross_kernels(f.sh).dq[s.d == 128](&a, grid, hs); });
    if (e != hipSuccess) return hip_fail(e, "cross_dq_kernel launch");
  }
  if (keys) {
    a.cut = kv.cut;
    a.part = part_k;
    a.part2 = part_v;
    a.part_n = kv.cut.max_parts > 1 ? counts_k : nullptr;
    const dim3 grid((unsigned)(kv.wgs * s.hkv));
    e = launch_timed(K_CROSS_DKDV, hs,
                     [&] { (void)cross_kernels(kv.sh).dkdv[s.d == 128](&a, grid, hs); });
    if (e != hipSuccess) return hip_fail(e, "cross_dkdv_kernel launch");
  }
  // the parts' sums, all in one launch
  pdy::CrossSumArgs sum{};
  sum.njobs = 0;
  sum.out_bf16 = grad_bf16;
  int64_t blocks = 0;
  auto add = [&](const float* part, const int32_t* n, const int32_t* n1, int max_parts,
                 int64_t heads, int64_t each, int64_t rows, int64_t first, int64_t count, const int32_t* end,
                 void* dst) {
    if (count == 0) return;
    const int b = (int)ceil_div(count * (s.d / 8), 256);
    sum.job[sum.njobs++] = pdy::CrossSumJob{part, n, n1, max_parts, (int)heads, (int)each, rows, first, count,
                                            end, dst, b};
    blocks += b;
  };
  if (rows && slices_of(f) > 0)
    add(part_q, counts_q, f.cut.keys == pdy::CROSS_APART ? counts_q + s.tq * s.hq : nullptr,
        f.cut.max_parts, s.hq, 1, s.tq * s.hq, 0, s.tq * s.hq, x.cu_q + s.n, g.dq);
  if (kv.cut.max_parts > 1) {
    const int64_t rows = (s.prefix + s.tk) * s.hkv, pre = s.prefix * s.hkv;
    for (int i = 0; i < 2; ++i) {
      const float* part = i ? part_v : part_k;
      add(part, counts_k, nullptr, kv.cut.max_parts, s.hkv, s.hkv, rows, 0, pre, nullptr,
          i ? g.dvp : g.dkp);
      add(part, counts_k, nullptr, kv.cut.max_parts, s.hkv, s.hkv, rows, pre, s.tk * s.hkv, x.cu_k + s.n,
          i ? g.dv : g.dk);
    }
  }
  if (sum.njobs > 0) {
    const dim3 grid((unsigned)blocks);
    e = launch_timed(K_CROSS_SUM, hs, [&] {
      if (s.d == 64) hipLaunchKernelGGL(pdy::cross_sum_kernel<64>, grid, dim3(256), 0, hs, sum);
      else hipLaunchKernelGGL(pdy::cross_sum_kernel<128>, grid, dim3(256), 0, hs, sum);
    });
    if (e != hipSuccess) return hip_fail(e, "cross_sum_kernel launch");
  }
  return PDY_OK;
}

}  // namespace

extern "C" {

pdy_status pdy_cross_launch_shapes(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                   int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                   int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                                   int32_t causal, int32_t* shapes) {
  g_err[0] = 0;
  CrossSizes s;
  const pdy_status st = check_cross_sizes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q,
                                          max_seqlen_k, num_heads_q, num_heads_kv, head_dim, &s);
  if (st != PDY_OK) return st;
  if (causal != 0 && causal != 1) return fail(PDY_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (shapes == nullptr) return fail(PDY_ERR_INVALID_ARG, "shapes is NULL");
  std::fill(shapes, shapes + 12, 0);
  auto put = [&](int i, const CrossShape& sh, const pdy::CrossCut& c) {
    shapes[3 * i] = sh.nw;
    shapes[3 * i + 1] = sh.groups;
    shapes[3 * i + 2] = c.max_parts;
  };
  if (s.tq > 0) {
    const CrossRows f = rows_launch(s, kFwd, causal != 0), q = rows_launch(s, kDq, causal != 0);
    put(0, f.sh, f.cut);
    put(1, q.sh, q.cut);
    shapes[9] = f.cut.keys == pdy::CROSS_APART;
    shapes[10] = f.cut.round > 0;
    shapes[11] = q.cut.round > 0;
  }
  if (s.tk + s.prefix > 0) {
    const CrossKv kv = kv_launch(s, false);
    put(2, kv.sh, kv.cut);
  }
  return PDY_OK;
}

size_t attn_prefix_fwd_workspace_size(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                      int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                      int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim) {
  CrossSizes s;
  if (check_cross_sizes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                        num_heads_q, num_heads_kv, head_dim, &s) != PDY_OK)
    return 0;
  // (enough for both masks)
  return s.tq == 0 ? 256
                   : std::max(fwd_bytes(s, rows_launch(s, kFwd, false)),
                              fwd_bytes(s, rows_launch(s, kFwd, true)));
}

size_t attn_cross_fwd_workspace_size(int32_t total_q, int32_t total_k, int32_t num_seqs,
                                     int32_t max_seqlen_q, int32_t max_seqlen_k,
                                     int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim) {
  return attn_prefix_fwd_workspace_size(0, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                                        num_heads_q, num_heads_kv, head_dim);
}

pdy_status attn_prefix_fwd(const void* q, const void* k, const void* v, const void* k_prefix,
                           const void* v_prefix, const int32_t* cu_seqlens_q,
                           const int32_t* cu_seqlens_k, const int32_t* seqlens_k,
                           int32_t prefix_len, int32_t num_seqs, int32_t total_q, int32_t total_k,
                           int32_t max_seqlen_q, int32_t max_seqlen_k, int32_t num_heads_q,
                           int32_t num_heads_kv, int32_t head_dim, int32_t causal, float scale,
                           void* o, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream) {
  g_err[0] = 0;
  CrossSizes s;
  const pdy_status st = check_cross_sizes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q,
                                          max_seqlen_k, num_heads_q, num_heads_kv, head_dim, &s);
  if (st != PDY_OK) return st;
  return cross_fwd_impl({q, k, v, k_prefix, v_prefix, cu_seqlens_q, cu_seqlens_k, seqlens_k}, s,
                        causal, scale, o, lse, workspace, workspace_bytes, stream,
                        "attn_prefix_fwd");
}

pdy_status attn_cross_fwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens_q,
                          const int32_t* cu_seqlens_k, const int32_t* seqlens_k, int32_t num_seqs,
                          int32_t total_q, int32_t total_k, int32_t max_seqlen_q,
                          int32_t max_seqlen_k, int32_t num_heads_q, int32_t num_heads_kv,
                          int32_t head_dim, int32_t causal, float scale, void* o, float* lse,
                          void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  CrossSizes s;
  const pdy_status st = check_cross_sizes(0, total_q, total_k, num_seqs, max_seqlen_q,
                                          max_seqlen_k, num_heads_q, num_heads_kv, head_dim, &s);
  if (st != PDY_OK) return st;
  return cross_fwd_impl({q, k, v, nullptr, nullptr, cu_seqlens_q, cu_seqlens_k, seqlens_k}, s,
                        causal, scale, o, lse, workspace, workspace_bytes, stream,
                        "attn_cross_fwd");
}

size_t attn_prefix_bwd_workspace_size(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                      int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                      int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim) {
  CrossSizes s;
  if (check_cross_sizes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                        num_heads_q, num_heads_kv, head_dim, &s) != PDY_OK)
    return 0;
  const CrossKv kv = kv_launch(s, false);  // (its parts, whatever max_k bounds)
  return std::max(bwd_space(s, rows_launch(s, kDq, false), kv).total,
                  bwd_space(s, rows_launch(s, kDq, true), kv).total);
}

size_t attn_cross_bwd_workspace_size(int32_t total_q, int32_t total_k, int32_t num_seqs,
                                     int32_t max_seqlen_q, int32_t max_seqlen_k,
                                     int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim) {
  return attn_prefix_bwd_workspace_size(0, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                                        num_heads_q, num_heads_kv, head_dim);
}

pdy_status attn_prefix_bwd(const void* q, const void* k, const void* v, const void* k_prefix,
                           const void* v_prefix, const void* o, const float* lse, const void* dout,
                           const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                           const int32_t* seqlens_k, int32_t prefix_len, int32_t num_seqs,
                           int32_t total_q, int32_t total_k, int32_t max_seqlen_q,
                           int32_t max_seqlen_k, int32_t num_heads_q, int32_t num_heads_kv,
                           int32_t head_dim, int32_t causal, float scale, int32_t grad_bf16,
                           void* dq, void* dk, void* dv, void* dk_prefix, void* dv_prefix,
                           void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  CrossSizes s;
  const pdy_status st = check_cross_sizes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q,
                                          max_seqlen_k, num_heads_q, num_heads_kv, head_dim, &s);
  if (st != PDY_OK) return st;
  return cross_bwd_impl({q, k, v, k_prefix, v_prefix, cu_seqlens_q, cu_seqlens_k, seqlens_k}, o,
                        lse, dout, s, causal, scale, grad_bf16, {dq, dk, dv, dk_prefix, dv_prefix},
                        workspace, workspace_bytes, stream, "attn_prefix_bwd");
}

pdy_status attn_cross_bwd(const void* q, const void* k, const void* v, const void* o,
                          const float* lse, const void* dout, const int32_t* cu_seqlens_q,
                          const int32_t* cu_seqlens_k, const int32_t* seqlens_k, int32_t num_seqs,
                          int32_t total_q, int32_t total_k, int32_t max_seqlen_q,
                          int32_t max_seqlen_k, int32_t num_heads_q, int32_t num_heads_kv,
                          int32_t head_dim, int32_t causal, float scale, int32_t grad_bf16,
                          void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                          void* stream) {
  g_err[0] = 0;
  CrossSizes s;
  const pdy_status st = check_cross_sizes(0, total_q, total_k, num_seqs, max_seqlen_q,
                                          max_seqlen_k, num_heads_q, num_heads_kv, head_dim, &s);
  if (st != PDY_OK) return st;
  return cross_bwd_impl({q, k, v, nullptr, nullptr, cu_seqlens_q, cu_seqlens_k, seqlens_k}, o, lse,
                        dout, s, causal, scale, grad_bf16, {dq, dk, dv, nullptr, nullptr},
                        workspace, workspace_bytes, stream, "attn_cross_bwd");
}

}  // extern "C"
