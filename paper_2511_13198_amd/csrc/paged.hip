// C-ABI of the paged key/value cache: argument checks, launch shapes, workspace and
// launches.  The contract is in include/pdyattn.h.
#include "../../include/pdyattn.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "host.hpp"
#include "paged.hpp"

using namespace pdy_host;

namespace {

constexpr int64_t kCUs = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The pool and its tables, checked.
struct PagedSizes {
  int64_t n, num_pages, page, max_pages, max_k, hkv, d;
  bool e4m3;
  int64_t row_bytes() const { return d * (e4m3 ? 1 : 2); }
};

pdy_status check_ints(const int32_t* p, const char* name) {
  if (p == nullptr) return fail(PDY_ERR_INVALID_ARG, "%s is NULL", name);
  if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0)
    return fail(PDY_ERR_INVALID_ARG, "%s is not 4-byte aligned", name);
  return PDY_OK;
}

pdy_status check_heads(int32_t n, int32_t hkv, int32_t d) {
  if (n < 1) return fail(PDY_ERR_INVALID_ARG, "num_seqs must be >= 1 (got %d)", n);
  if (hkv < 1) return fail(PDY_ERR_INVALID_ARG, "head counts must be >= 1 (got Hkv=%d)", hkv);
  if (d != 64 && d != 128)
    return fail(PDY_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", d);
  if ((int64_t)hkv * d >= 1 << 22)
    return fail(PDY_ERR_INVALID_ARG, "too many heads for one launch (Hkv=%d)", hkv);
  return PDY_OK;
}

pdy_status check_pool(const void* k, const void* v, const float* k_scale, const float* v_scale,
                      const int32_t* table, const int32_t* len, int32_t n, int32_t num_pages,
                      int32_t page, int32_t max_pages, int32_t max_k, int32_t hkv, int32_t d,
                      int32_t e4m3, bool scales, PagedSizes* out) {
  pdy_status st = check_heads(n, hkv, d);
  if (st != PDY_OK) return st;
  if (page < 16 || page % 16 != 0)
    return fail(PDY_ERR_INVALID_ARG, "page_size must be a multiple of 16 (got %d)", page);
  if (num_pages < 0 || max_pages < 0)
    return fail(PDY_ERR_INVALID_ARG, "num_pages and max_pages must be >= 0 (got %d, %d)",
                num_pages, max_pages);
  // runs of 16 keys are counted in 32 bits over the pool, keys over a sequence (and a little
  // past its end)
  if ((int64_t)num_pages * hkv * (page / 16) >= (int64_t)1 << 31 ||
      (int64_t)max_pages * page >= (int64_t)1 << 30)
    return fail(PDY_ERR_INVALID_ARG, "too many pages (num_pages=%d, max_pages=%d)", num_pages,
                max_pages);
  if (max_k < 0 || max_k > (int64_t)max_pages * page)
    return fail(PDY_ERR_INVALID_ARG,
                "max_seqlen_k must be in [0, max_pages * page_size] (got %d, %d * %d)", max_k,
                max_pages, page);
  if (e4m3 & ~1) return fail(PDY_ERR_INVALID_ARG, "cache_e4m3 must be 0 or 1");
  if ((st = check_ints(len, "seqlens_k")) != PDY_OK) return st;
  if (max_pages > 0 && (st = check_ints(table, "page_table"))) return st;
  if (num_pages > 0 && ((st = check_ptr(k, "k_pages")) || (st = check_ptr(v, "v_pages"))))
    return st;
  if (scales && e4m3) {
    if ((st = check_ints(reinterpret_cast<const int32_t*>(k_scale), "k_scale")) ||
        (st = check_ints(reinterpret_cast<const int32_t*>(v_scale), "v_scale")))
      return st;
  } else if (scales && (k_scale || v_scale)) {
    return fail(PDY_ERR_INVALID_ARG,
                "k_scale and v_scale are of an e4m3 cache (a bf16 one has none)");
  }
  *out = PagedSizes{n, num_pages, page, max_pages, max_k, hkv, d, e4m3 != 0};
  return PDY_OK;
}

pdy::PagedCache cache_of(const PagedSizes& s, const int32_t* table, const int32_t* len) {
  const int64_t runs = s.page / 16;
  return pdy::PagedCache{table, len, (int)s.n, (int)s.num_pages, (int)s.page, (int)s.max_pages,
                         (int)s.max_k, (int)s.hkv, (int)runs, (uint32_t)((1ull << 32) / runs)};
}

// K of a head that an eviction keeps, up to which (and a workgroup a CU) one launch selects
// and copies: us of two launches / one, 8 kv heads, d = 128, bf16: 300 keys to 100 of 1
// sequence 10.2 / 9.0, of 4 10.9 / 9.3, of 16 13.2 / 10.7, of 64 22.2 / 22.8; 1,000 to 250
// 10.4 / 10.4, 11.8 / 11.5, 14.7 / 15.3; to 500 10.6 / 13.5, 13.2 / 16.8, 20.3 / 22.8.
constexpr int64_t kFusedBytes = 48 << 10;

// Whether a grid's threads can be counted in 32 bits, as a launch's are.
bool fits_grid(int64_t wgs, int threads) { return wgs * threads < (int64_t)1 << 32; }

// ---- attention ----
struct PagedRows {
  int64_t tq, max_q, hq;
};

pdy_status check_rows(int32_t tq, int32_t n, int32_t max_q, int32_t hq, int32_t hkv, int32_t d,
                      PagedRows* out) {
  if (tq < 0) return fail(PDY_ERR_INVALID_ARG, "total_q must be >= 0 (got %d)", tq);
  if (max_q < 0 || max_q > tq || (tq > 0 && max_q < 1))
    return fail(PDY_ERR_INVALID_ARG, "max_seqlen_q must be in [1, total_q] (got %d, total_q=%d)",
                max_q, tq);
  if (hq < 1 || hq % hkv != 0)
    return fail(PDY_ERR_INVALID_ARG, "num_heads_q (%d) must be a multiple of num_heads_kv (%d)",
                hq, hkv);
  if (((int64_t)tq + n) * hq >= (int64_t)1 << 31)
    return fail(PDY_ERR_INVALID_ARG, "problem too large for one launch");
  if ((int64_t)hq * d >= 1 << 24)
    return fail(PDY_ERR_INVALID_ARG, "too many heads for one launch (Hq=%d)", hq);
  *out = PagedRows{tq, max_q, hq};
  return PDY_OK;
}

// Keys and values of more bytes do not stay in the 256 MB last-level cache until they are
// read again, and are faster read past it.  us through / past it: 64 sequences over 256-16,384
// keys of 8 heads, 888 MB 167 / 149, e4m3 444 MB 91 / 80; 17 over 900-9,000, 278 MB 61 / 56; 256
// over up to 2,048 of 2 heads, 75 MB, three such caches in turn 22 / 34.
constexpr int64_t kCachedBytes = (int64_t)128 << 20;
constexpr int kMaxParts = 256;
constexpr int64_t kPartBytes = (int64_t)64 << 20;   // partial results at most

constexpr int64_t kLogitBytes = (int64_t)1 << 30;   // logits left for the weights at most

// A launch's row tiles (16 << shape rows) and parts.
struct PagedPlan {
  int shape;
  int max_tiles;
  bool whole;  // items are not cut
  int waves;   // of a workgroup
  pdy::PagedCut cut;
  int64_t wgs;  // a kv head
  int64_t logit_rows, logit_keys;   // (rows 0: no logits are left)
  size_t part_o, part_lse, part_n, logits;  // bytes of the workspace
  size_t bytes() const { return std::max<size_t>(256, part_o + part_lse + part_n + logits); }
};

// Sequences of so many keys at most stay whole: the launch that joins parts takes longer than
// they save.  us cut / whole for a token of 32/8 heads, n sequences of equal lengths and of
// 1 .. max (evenly over the logarithm), d = 128, bf16:
//   n = 1: 1,024 8.9 / 8.7, 2,048 9.1 / 12.4;  n = 8: 2,048 18.2 / 15.8 and 9.6 / 8.7, 4,096
//   34.6 / 45.7 and 10.5 / 12.7;  n = 32: 2,048 55.0 / 49.4 and 13.4 / 12.7, 4,096 99.1 / 96.4 and
//   15.7 / 19.3;  n = 256: 1,024 (1 ..) 51.6 / 46.5, 2,048 73.6 / 74.9, 4,096 118 / 132
// e4m3: n = 1: 1,024 9.0 / 8.3, 2,048 9.3 / 11.7;  n = 64: 2,048 56.7 / 51.9 and 17.4 / 16.7,
//   4,096 (1 ..) 22.6 / 26.7
// d = 64: n = 1: 2,048 8.6 / 9.0, 4,096 8.9 / 13.4;  n = 8 .. 32: 4,096 20.8 / 17.2 and 9.1 / 8.5,
//   54.7 / 50.1 and 13.5 / 13.0;  n = 64: 2,048 16.3 / 13.7 (1 ..), 4,096 20.5 / 21.5
int64_t whole_keys(int64_t pairs, int64_t d) {
  if (d == 64) return pairs >= 64 && pairs <= kCUs ? 4096 : 2048;
  return pairs < 64 ? 1024 : 2048;
}

PagedPlan plan_fwd(const PagedRows& r, int64_t n, int64_t max_k, int64_t hkv, int64_t d,
                   int64_t row_bytes, bool weigh) {
  PagedPlan p;
  const int64_t g = r.hq / hkv, rows = std::max<int64_t>(1, r.max_q * g);
  p.shape = rows <= 16 ? 0 : rows <= 32 ? 1 : 2;
  const int64_t tile = 16 << p.shape;
  p.max_tiles = (int)ceil_div(rows, tile);
  const int64_t items = std::min(r.tq * g / tile + n, n * p.max_tiles);
  const int64_t slice = std::max<int64_t>(1, r.tq) * r.hq * (d + 1) * 4;
  p.cut.least = 8;
  // Two rounds of two workgroups a CU, which even out lengths that the host does not know.  Of
  // 64 rows of 128 a CU holds one, and one round with the items' last parts is the fastest: us
  // with 4 / 2 / 1 parts a CU, and with 1 less the items, for 16 tokens of each of 12 sequences
  // over 1,000-8,000 keys, 32/8 heads 77 / 61 / 54 / 42 (their bytes take 25), e4m3 68 / 52 /
  // 48 / 37 (13), of one over 50,000 81 / 61 / 48 / 47; 12 tokens of each of 40 sequences over
  // 500-4,000 (320 items) 93 / 76 / 67 (51).
  int64_t entries = 4 * kCUs;
  if (p.shape == 2 && d == 128) entries = 8 * items * hkv <= 5 * kCUs ? kCUs - items * hkv : kCUs;
  p.cut.entries = (int)ceil_div(entries, hkv);
  p.cut.max_parts = (int)std::max<int64_t>(
      1, std::min<int64_t>({kMaxParts, p.cut.entries + 1, ceil_div(max_k, 32) / p.cut.least,
                            kPartBytes / slice}));
  p.whole = max_k <= whole_keys(n * hkv, d);
  if (p.whole) p.cut.max_parts = 1;
  // a workgroup a CU at most: 8 waves, where a step is short (us with 4 / 8 for a token of 8
  // kv heads over 1,024 keys: bf16 of 128 8.7 / 8.7, e4m3 9.2 / 8.3, of 64 7.7 / 6.9; 64 tokens
  // 49.8 / 51.6, 28.1 / 32.0, 26.7 / 29.4)
  p.waves = p.shape == 0 && p.whole && n * hkv <= kCUs && row_bytes < 256 ? 8 : 4;
  const bool cut = p.cut.max_parts > 1;
  p.wgs = cut ? items + p.cut.entries + 1 : n * p.max_tiles;
  p.part_o = cut ? align256((size_t)p.cut.max_parts * r.tq * r.hq * d * 4) : 0;
  p.part_lse = cut ? align256((size_t)p.cut.max_parts * r.tq * r.hq * 4) : 0;
  p.part_n = cut ? align256((size_t)r.tq * r.hq * 4) : 0;
  p.logit_keys = ceil_div(std::max<int64_t>(max_k, 1), 32) * 32;
  const bool leave = weigh && p.shape == 0 && n * hkv * rows <= kLogitBytes / 4 / p.logit_keys;
  p.logit_rows = leave ? rows : 0;
  p.logits = align256((size_t)(n * hkv * p.logit_rows * p.logit_keys * 4));
  return p;
}

template <int D, bool F8, int RB, int NW, bool LOGITS = false, bool WHOLE = false>
hipError_t launch_fwd(const pdy::PagedFwdArgs* a, dim3 grid, hipStream_t st) {
  using C = pdy::PagedFwdCfg<D, F8, RB, NW>;
  constexpr auto kernel = pdy::paged_fwd_kernel<D, F8, RB, NW, LOGITS, WHOLE>;
  if (a == nullptr) return set_lds(kernel, C::LDS_BYTES);
  hipLaunchKernelGGL(kernel, grid, dim3(C::NT), C::LDS_BYTES, st, *a);
  return hipSuccess;
}
using LaunchFwd = hipError_t (*)(const pdy::PagedFwdArgs*, dim3, hipStream_t);
// [d = 64, 128][bf16, e4m3][16, 32, 64 rows; 16: leaving their logits; whole items by 4 waves,
// by 8; both leaving their logits]
constexpr int kShapes = 8;
template <int D, bool F8>
constexpr LaunchFwd kFwdOf[kShapes] = {launch_fwd<D, F8, 1, 4>, launch_fwd<D, F8, 2, 4>,
                                       launch_fwd<D, F8, 4, 4>, launch_fwd<D, F8, 1, 4, true>,
                                       launch_fwd<D, F8, 1, 4, false, true>,
                                       launch_fwd<D, F8, 1, 8, false, true>,
                                       launch_fwd<D, F8, 1, 4, true, true>,
                                       launch_fwd<D, F8, 1, 8, true, true>};
const LaunchFwd* const kFwd[2][2] = {{kFwdOf<64, false>, kFwdOf<64, true>},
                                     {kFwdOf<128, false>, kFwdOf<128, true>}};

template <int D, bool F8, int RB>
void launch_weigh(const pdy::PagedWeighArgs& a, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL((pdy::paged_weigh_kernel<D, F8, RB>), grid, dim3(256), 0, st, a);
}
using LaunchWeigh = void (*)(const pdy::PagedWeighArgs&, dim3, hipStream_t);
template <int D, bool F8>
constexpr LaunchWeigh kWeighOf[3] = {launch_weigh<D, F8, 1>, launch_weigh<D, F8, 2>,
                                     launch_weigh<D, F8, 4>};
const LaunchWeigh* const kWeigh[2][2] = {{kWeighOf<64, false>, kWeighOf<64, true>},
                                         {kWeighOf<128, false>, kWeighOf<128, true>}};

hipError_t init_paged_kernels() {
  static hipError_t status = [] {
    for (const auto& d : kFwd)
      for (const LaunchFwd* f : d)
        for (int i = 0; i < kShapes; ++i) {
          const hipError_t e = f[i](nullptr, dim3(), nullptr);
          if (e != hipSuccess) return e;
        }
    return hipSuccess;
  }();
  return status;
}

}  // namespace

extern "C" {

pdy_status attn_paged_write(const void* k, const void* v, const int32_t* cu_seqlens,
                            const int32_t* page_table, const int32_t* seqlens_k,
                            const float* k_scale, const float* v_scale, int32_t num_seqs,
                            int32_t total_tokens, int32_t num_pages, int32_t page_size,
                            int32_t max_pages, int32_t num_heads_kv, int32_t head_dim,
                            int32_t cache_e4m3, void* k_pages, void* v_pages, float* scores,
                            void* stream) {
  g_err[0] = 0;
  PagedSizes s;
  pdy_status st;
  if (total_tokens < 0 || total_tokens >= (1 << 26) - 4)
    return fail(PDY_ERR_INVALID_ARG, "total_tokens must be >= 0 and below 2^26 - 4 (got %d)",
                total_tokens);
  const int64_t room = std::min<int64_t>((int64_t)std::max(max_pages, 0) * std::max(page_size, 0),
                                         0x7fffffff);
  if ((st = check_pool(k_pages, v_pages, k_scale, v_scale, page_table, seqlens_k, num_seqs,
                       num_pages, page_size, max_pages, (int32_t)room, num_heads_kv, head_dim,
                       cache_e4m3, true, &s)))
    return st;
  if (total_tokens == 0) return PDY_OK;
  if ((st = check_ints(cu_seqlens, "cu_seqlens")) || (st = check_ptr(k, "k")) ||
      (st = check_ptr(v, "v")))
    return st;
  if (scores && (st = check_ptr(scores, "scores"))) return st;
  pdy::PagedWriteArgs a;
  a.c = cache_of(s, page_table, seqlens_k);
  a.in[0] = static_cast<const uint16_t*>(k);
  a.in[1] = static_cast<const uint16_t*>(v);
  a.pages[0] = k_pages;
  a.pages[1] = v_pages;
  a.scale[0] = k_scale;
  a.scale[1] = v_scale;
  a.scores = scores;
  a.cu = cu_seqlens;
  a.tokens = total_tokens;
  // tokens of a workgroup: as many as leave 4 of these a CU
  a.each_log2 = 0;
  while (a.each_log2 < pdy::kWriteLog2 && total_tokens >> (a.each_log2 + 1) >= 4 * kCUs)
    ++a.each_log2;
  const int64_t units = (int64_t)num_heads_kv * head_dim / 8;
  a.units_inv = (uint32_t)((1ull << 32) / units);
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)ceil_div(total_tokens, 1 << a.each_log2));
  const hipError_t e = launch_timed(K_PAGED_WRITE, hs, [&] {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, hs, a); };
    if (head_dim == 64)
      s.e4m3 ? go(pdy::paged_write_kernel<64, true>) : go(pdy::paged_write_kernel<64, false>);
    else
      s.e4m3 ? go(pdy::paged_write_kernel<128, true>) : go(pdy::paged_write_kernel<128, false>);
  });
  if (e != hipSuccess) return hip_fail(e, "paged_write_kernel launch");
  return PDY_OK;
}

size_t attn_paged_fwd_workspace_size(int32_t total_q, int32_t num_seqs, int32_t max_seqlen_q,
                                     int32_t max_seqlen_k, int32_t num_heads_q,
                                     int32_t num_heads_kv, int32_t head_dim, int32_t with_scores) {
  g_err[0] = 0;
  PagedRows r;
  if (check_heads(num_seqs, num_heads_kv, head_dim) != PDY_OK || max_seqlen_k < 0 ||
      (with_scores & ~1) ||
      check_rows(total_q, num_seqs, max_seqlen_q, num_heads_q, num_heads_kv, head_dim, &r) !=
          PDY_OK)
    return 0;
  return plan_fwd(r, num_seqs, max_seqlen_k, num_heads_kv, head_dim, 0, with_scores).bytes();
}

pdy_status attn_paged_fwd(const void* q, const void* k_pages, const void* v_pages,
                          const int32_t* page_table, const int32_t* cu_seqlens_q,
                          const int32_t* seqlens_k, const float* k_scale, const float* v_scale,
                          int32_t num_seqs, int32_t total_q, int32_t num_pages, int32_t page_size,
                          int32_t max_pages, int32_t max_seqlen_q, int32_t max_seqlen_k,
                          int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                          int32_t cache_e4m3, int32_t causal, float scale, void* o, float* lse,
                          float* scores, void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  PagedSizes s;
  PagedRows r;
  pdy_status st;
  if ((st = check_pool(k_pages, v_pages, k_scale, v_scale, page_table, seqlens_k, num_seqs,
                       num_pages, page_size, max_pages, max_seqlen_k, num_heads_kv, head_dim,
                       cache_e4m3, true, &s)) ||
      (st = check_rows(total_q, num_seqs, max_seqlen_q, num_heads_q, num_heads_kv, head_dim, &r)) ||
      (st = check_scale(scale, causal)))
    return st;
  if (total_q == 0) return PDY_OK;
  if ((st = check_ints(cu_seqlens_q, "cu_seqlens_q")) || (st = check_ptr(q, "q")) ||
      (st = check_ptr(o, "o")) || (st = check_ptr(lse, "lse")) ||
      (st = check_ptr(workspace, "workspace")))
    return st;
  if (scores && (st = check_ptr(scores, "scores"))) return st;
  const PagedPlan p = plan_fwd(r, s.n, s.max_k, s.hkv, s.d, s.row_bytes(), scores != nullptr);
  if (workspace_bytes < p.bytes())
    return fail(PDY_ERR_WORKSPACE, "workspace has %zu bytes, attn_paged_fwd needs %zu",
                workspace_bytes, p.bytes());
  const int64_t g = r.hq / s.hkv;
  pdy::PagedFwdArgs a;
  a.c = cache_of(s, page_table, seqlens_k);
  a.q = static_cast<const uint16_t*>(q);
  a.k = k_pages;
  a.v = v_pages;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.cu_q = cu_seqlens_q;
  a.tq = total_q;
  a.hq = num_heads_q;
  a.g = (int)g;
  a.g_inv = (uint32_t)((1ull << 32) / g);
  a.causal = causal;
  a.max_tiles = p.max_tiles;
  // (tiles of one sequence share its keys through the caches)
  const int64_t fit = kCachedBytes / (s.hkv * 64 * s.row_bytes());
  a.stream_steps = p.max_tiles == 1 && s.n * ceil_div(s.max_k, 32) > fit ? (int)fit : -1;
  // (weights from the keys read K again: us past the caches / through them with V past, for 32
  // tokens of 16 heads, d = 64, over 4,000-16,384 keys of 6 sequences (K 100 MB) 72 / 67, of 16
  // (250 MB) 164 / 150, of 24 (390 MB) 244 / 232)
  a.keep_k = scores != nullptr;
  a.cut = p.cut;
  a.scale_log2 = scale * pdy::kLog2e;
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_lse = reinterpret_cast<float*>(ws + p.part_o);
  a.part_n = reinterpret_cast<int32_t*>(ws + p.part_o + p.part_lse);
  a.logits = reinterpret_cast<float*>(ws + p.part_o + p.part_lse + p.part_n);
  a.logit_rows = (int)p.logit_rows;
  a.logit_keys = (int)p.logit_keys;
  const int64_t wgs = p.wgs * s.hkv;
  const bool weighs = fits_grid(s.n * s.hkv * ceil_div(s.max_k, 512), 256) && s.n <= 65535 &&
                      s.hkv <= 65535;
  if (!fits_grid(wgs, 64 * p.waves) || (scores && !weighs))
    return fail(PDY_ERR_INVALID_ARG, "problem too large for one launch");
  hipError_t e = init_paged_kernels();
  if (e != hipSuccess) return hip_fail(e, "kernel attribute setup");
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  int kernel = p.shape;
  if (p.shape == 0 && p.whole) kernel = (p.logit_rows > 0 ? 6 : 4) + (p.waves == 8);
  else if (p.logit_rows > 0) kernel = 3;
  e = launch_timed(K_PAGED_FWD, hs, [&] {
    (void)kFwd[s.d == 128][s.e4m3][kernel](&a, dim3((unsigned)wgs), hs);
  });
  if (e != hipSuccess) return hip_fail(e, "paged_fwd_kernel launch");
  // a workgroup a (token, head) pair where few have many parts: us with a wave / a workgroup
  // for 32 pairs of 128 parts 17.5 / 6.6
  const bool wide = r.tq * r.hq <= 2 * kCUs && p.cut.max_parts > 16;
  const pdy::PagedMergeArgs m{a.part_o, a.part_lse, a.part_n, p.cut.max_parts, a.cu_q, a.c.n, a.tq,
                              a.hq, a.o, a.lse, wide};
  const int64_t merge_blocks =
      p.cut.max_parts == 1 ? 0 : wide ? r.tq * r.hq : ceil_div(r.tq * r.hq, 4);
  if (p.logit_rows > 0) {
    const int64_t key_blocks = ceil_div(std::max<int64_t>(s.max_k, 1), pdy::kWeighKeys);
    const pdy::PagedJoinArgs b{m, (int)merge_blocks, a.c, a.g, (int)key_blocks, a.logits,
                               a.logit_rows, a.logit_keys, a.scale_log2, a.k_scale, scores};
    const int64_t blocks = merge_blocks + s.n * s.hkv * key_blocks;
    const dim3 grid((unsigned)blocks);
    e = launch_timed(K_PAGED_JOIN, hs, [&] {
      if (s.d == 64) hipLaunchKernelGGL(pdy::paged_join_kernel<64>, grid, dim3(256), 0, hs, b);
      else hipLaunchKernelGGL(pdy::paged_join_kernel<128>, grid, dim3(256), 0, hs, b);
    });
    if (e != hipSuccess) return hip_fail(e, "paged_join_kernel launch");
    return PDY_OK;
  }
  if (merge_blocks > 0) {
    const dim3 grid((unsigned)merge_blocks);
    e = launch_timed(K_PAGED_MERGE, hs, [&] {
      if (s.d == 64) hipLaunchKernelGGL(pdy::paged_merge_kernel<64>, grid, dim3(256), 0, hs, m);
      else hipLaunchKernelGGL(pdy::paged_merge_kernel<128>, grid, dim3(256), 0, hs, m);
    });
    if (e != hipSuccess) return hip_fail(e, "paged_merge_kernel launch");
  }
  if (scores) {
    const pdy::PagedWeighArgs b{a.c, a.q, a.k, a.k_scale, a.cu_q, a.lse, a.tq, a.hq, a.g, a.g_inv,
                                a.causal, a.scale_log2, scores};
    const dim3 grid((unsigned)ceil_div(ceil_div(std::max<int64_t>(s.max_k, 1), 16),
                                       4 * pdy::kWeighRuns), (unsigned)s.hkv, (unsigned)s.n);
    e = launch_timed(K_PAGED_WEIGH, hs, [&] {
      kWeigh[s.d == 128][s.e4m3][p.shape](b, grid, hs);
    });
    if (e != hipSuccess) return hip_fail(e, "paged_weigh_kernel launch");
  }
  return PDY_OK;
}

// (As of every call that may come to need scratch memory; no kernel takes it now.)
size_t attn_paged_evict_workspace_size(int32_t num_seqs, int32_t max_seqlen_k,
                                       int32_t num_heads_kv, int32_t budget) {
  g_err[0] = 0;
  if (num_seqs < 1 || max_seqlen_k < 0 || num_heads_kv < 1 || budget < 1) return 0;
  return 256;
}

pdy_status attn_paged_evict(void* k_pages, void* v_pages, float* scores, const int32_t* page_table,
                            const int32_t* seqlens_k, const int32_t* new_table, int32_t num_seqs,
                            int32_t num_pages, int32_t page_size, int32_t max_pages,
                            int32_t new_max_pages, int32_t max_seqlen_k, int32_t num_heads_kv,
                            int32_t head_dim, int32_t cache_e4m3, int32_t budget, int32_t recent,
                            int32_t first, int32_t* kept, int32_t* new_lens, void* workspace,
                            size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  PagedSizes s;
  pdy_status st;
  if ((st = check_pool(k_pages, v_pages, nullptr, nullptr, page_table, seqlens_k, num_seqs,
                       num_pages, page_size, max_pages, max_seqlen_k, num_heads_kv, head_dim,
                       cache_e4m3, false, &s)))
    return st;
  if (budget < 1) return fail(PDY_ERR_INVALID_ARG, "budget must be >= 1 (got %d)", budget);
  if (recent < 0 || first < 0 || (int64_t)recent + first > budget)
    return fail(PDY_ERR_INVALID_ARG,
                "recent and first must be >= 0 and together at most the budget (got %d, %d, %d)",
                recent, first, budget);
  const int64_t most = std::min<int64_t>(budget, s.max_k);
  if (new_max_pages < 0 || (int64_t)new_max_pages * page_size < most)
    return fail(PDY_ERR_INVALID_ARG, "new_table has room for %d pages of %d keys, %d may stay",
                new_max_pages, page_size, (int)most);
  if (s.n * s.hkv * budget >= (int64_t)1 << 31 || !fits_grid(s.n * s.hkv, pdy::kSelectThreads))
    return fail(PDY_ERR_INVALID_ARG, "problem too large for one launch");
  if (s.hkv > 65535 || s.n > 65535)
    return fail(PDY_ERR_INVALID_ARG, "too many sequences or heads for one launch");
  if (num_pages > 0 && (st = check_ptr(scores, "scores"))) return st;
  if (new_max_pages > 0 && (st = check_ints(new_table, "new_table"))) return st;
  if (new_table != nullptr && new_table == page_table)
    return fail(PDY_ERR_INVALID_ARG, "new_table must name other pages than page_table");
  if ((st = check_ints(kept, "kept")) || (st = check_ints(new_lens, "new_lens")) ||
      (st = check_ptr(workspace, "workspace")))
    return st;
  // (in bytes: some workgroups read a length when others have written the new ones)
  const int64_t gap = (int64_t)(reinterpret_cast<uintptr_t>(new_lens) -
                                reinterpret_cast<uintptr_t>(seqlens_k));
  if (gap != 0 && gap < 4 * s.n && -gap < 4 * s.n)
    return fail(PDY_ERR_INVALID_ARG, "new_lens overlaps seqlens_k without being it");
  if (workspace_bytes < 256)
    return fail(PDY_ERR_WORKSPACE, "workspace has %zu bytes, attn_paged_evict needs %zu",
                workspace_bytes, (size_t)256);
  pdy::PagedEvictArgs a;
  a.c = cache_of(s, page_table, seqlens_k);
  a.new_table = new_table;
  a.new_pages = new_max_pages;
  a.budget = budget;
  a.recent = recent;
  a.first = first;
  a.scores = scores;
  a.k = static_cast<uint8_t*>(k_pages);
  a.v = static_cast<uint8_t*>(v_pages);
  a.kept = kept;
  a.new_len = new_lens;
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  // the smallest number of keys a thread that holds those of the longest sequence that may go
  // (and up to 15 in front of them)
  const int64_t quads = ceil_div(s.max_k - recent - (first & ~15), 4 * pdy::kSelectThreads);
  const int per = quads <= 1 ? 0 : quads <= 4 ? 1 : quads <= 8 ? 2 : 3;
  // Few rows are copied by the workgroups that selected them, not in a launch of its own.
  // (Where the new lengths are written over the old, these are read until the end.)
  const bool fused = per <= 1 && most * s.row_bytes() <= kFusedBytes && s.n * s.hkv <= kCUs &&
                     gap != 0;
  const int lanes = s.row_bytes() == 64 ? 0 : s.row_bytes() == 128 ? 1 : 2;
  hipError_t e = launch_timed(K_PAGED_SELECT, hs, [&] {
    const dim3 grid((unsigned)(s.n * s.hkv)), block(pdy::kSelectThreads);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, hs, a); };
    if (fused && per == 0)
      lanes == 0   ? go(pdy::paged_select_kernel<1, 4>)
      : lanes == 1 ? go(pdy::paged_select_kernel<1, 8>)
                   : go(pdy::paged_select_kernel<1, 16>);
    else if (fused)
      lanes == 0   ? go(pdy::paged_select_kernel<4, 4>)
      : lanes == 1 ? go(pdy::paged_select_kernel<4, 8>)
                   : go(pdy::paged_select_kernel<4, 16>);
    else if (per == 0) go(pdy::paged_select_kernel<1, 0>);
    else if (per == 1) go(pdy::paged_select_kernel<4, 0>);
    else if (per == 2) go(pdy::paged_select_kernel<8, 0>);
    else go(pdy::paged_select_kernel<0, 0>);
  });
  if (e != hipSuccess) return hip_fail(e, "paged_select_kernel launch");
  if (fused) return PDY_OK;
  e = launch_timed(K_PAGED_GATHER, hs, [&] {
    auto go = [&](auto kernel, int rows) {
      const dim3 grid((unsigned)std::max<int64_t>(1, ceil_div(most, rows)), (unsigned)s.hkv,
                      (unsigned)s.n);
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, hs, a);
    };
    if (lanes == 0) go(pdy::paged_gather_kernel<4>, pdy::kGatherRows<4, 256>);
    else if (lanes == 1) go(pdy::paged_gather_kernel<8>, pdy::kGatherRows<8, 256>);
    else go(pdy::paged_gather_kernel<16>, pdy::kGatherRows<16, 256>);
  });
  if (e != hipSuccess) return hip_fail(e, "paged_gather_kernel launch");
  return PDY_OK;
}

pdy_status pdy_paged_launch_shapes(int32_t total_q, int32_t num_seqs, int32_t max_seqlen_q,
                                   int32_t max_seqlen_k, int32_t num_heads_q,
                                   int32_t num_heads_kv, int32_t head_dim, int32_t cache_e4m3,
                                   int32_t with_scores, int32_t* shapes) {
  g_err[0] = 0;
  PagedRows r;
  pdy_status st;
  if ((st = check_heads(num_seqs, num_heads_kv, head_dim)) ||
      (st = check_rows(total_q, num_seqs, max_seqlen_q, num_heads_q, num_heads_kv, head_dim, &r)))
    return st;
  if (max_seqlen_k < 0)
    return fail(PDY_ERR_INVALID_ARG, "max_seqlen_k must be >= 0 (got %d)", max_seqlen_k);
  if ((cache_e4m3 & ~1) || (with_scores & ~1))
    return fail(PDY_ERR_INVALID_ARG, "cache_e4m3 and with_scores must be 0 or 1");
  if (shapes == nullptr) return fail(PDY_ERR_INVALID_ARG, "shapes is NULL");
  const PagedPlan p = plan_fwd(r, num_seqs, max_seqlen_k, num_heads_kv, head_dim,
                               head_dim * (cache_e4m3 ? 1 : 2), with_scores);
  shapes[0] = p.waves;
  shapes[1] = 16 << p.shape;
  shapes[2] = p.cut.max_parts;
  shapes[3] = p.logit_rows > 0;
  return PDY_OK;
}

}  // extern "C"
