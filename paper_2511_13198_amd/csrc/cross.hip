// C-ABI of the attention over keys of another length and over shared keys:
// argument checks, launch shapes, workspace and launches.  The contract is in
// include/pdyattn.h.
#include "../../include/pdyattn.h"

#include <hip/hip_runtime.h>

#include <algorithm>

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

// ---- forward ----

// Rows of a sequence decide the workgroups' shape: the smallest tile that holds
// them; few rows leave the waves to key groups.
CrossShape fwd_shape(int64_t rows) {
  if (rows <= 32) return {4, 4};
  if (rows <= 64) return {8, 4};
  if (rows <= 128) return {8, 2};
  return {8, 1};
}

int fwd_key_tile(const CrossSizes& s, const CrossShape& sh) {
  return sh.groups > 1 || s.d == 128 ? 128 : 64;
}

// One launch of the forward kernel.
struct CrossFwd {
  CrossShape sh;
  pdy::CrossCut cut;
  int64_t wgs;  // per kv head
};

constexpr int kMaxParts = 64;
constexpr int64_t kPartBytes = (int64_t)256 << 20;  // partial results at most

CrossFwd fwd_launch(const CrossSizes& s, pdy::CrossKeys keys, int max_parts_of = kMaxParts) {
  const bool shared = keys == pdy::CROSS_SHARED;
  const int64_t n = shared ? 1 : s.n, max_q = shared ? s.tq : s.max_q;
  CrossFwd f;
  f.sh = fwd_shape(max_q * s.g());
  pdy::CrossCut& c = f.cut;
  c.keys = keys;
  c.rows = f.sh.rows();
  c.key_tile = fwd_key_tile(s, f.sh);
  c.least = 2;
  c.slice = 0;
  c.always_part = 0;
  const int64_t items = most_items(s, n, max_q, c.rows);
  const int64_t target = 2 * kCUs;
  c.per_head = (float)((double)target / s.hkv);
  const int64_t tiles = (shared ? 0 : ceil_div(s.max_k, c.key_tile)) +
                        (keys == pdy::CROSS_OWN ? 0 : ceil_div(s.prefix, c.key_tile));
  const int64_t slice = s.tq * s.hq * (s.d + 1) * 4;
  int64_t parts = std::min<int64_t>({max_parts_of, tiles / c.least, kPartBytes / slice});
  if (items * s.hkv >= target) parts = 1;
  c.max_parts = (int)std::max<int64_t>(1, parts);
  f.wgs = items + (c.max_parts > 1 ? ceil_div(target, s.hkv) + 2 : 0);
  return f;
}

// The launches of a forward: own keys, or shared and own keys in one, or one each.
struct CrossFwdPlan {
  int launches;
  CrossFwd l[2];
  bool merge() const { return launches > 1 || l[0].cut.max_parts > 1; }
  int slices() const {
    return merge() ? l[0].cut.max_parts + (launches > 1 ? l[1].cut.max_parts : 0) : 0;
  }
};

CrossFwdPlan fwd_plan(const CrossSizes& s) {
  CrossFwdPlan p;
  if (s.prefix == 0) {
    p.launches = 1;
    p.l[0] = fwd_launch(s, pdy::CROSS_OWN);
  } else if (s.seq_rows() > 64) {
    p.launches = 1;
    p.l[0] = fwd_launch(s, pdy::CROSS_FUSED);
  } else {
    // few rows a sequence: the shared keys once for the rows of all of them
    p.launches = 2;
    p.l[0] = fwd_launch(s, pdy::CROSS_SHARED);
    p.l[1] = fwd_launch(s, pdy::CROSS_OWN);
    p.l[0].cut.always_part = p.l[1].cut.always_part = 1;
    p.l[1].cut.slice = p.l[0].cut.max_parts;
  }
  return p;
}

size_t part_n_bytes(const CrossSizes& s) { return align256((size_t)s.tq * 4); }
size_t part_o_bytes(const CrossSizes& s, int slices) {
  return align256((size_t)slices * s.tq * s.hq * s.d * 4);
}
size_t part_lse_bytes(const CrossSizes& s, int slices) {
  return align256((size_t)slices * s.tq * s.hq * 4);
}

size_t fwd_bytes(const CrossSizes& s, const CrossFwdPlan& p) {
  if (!p.merge()) return 256;
  return 2 * part_n_bytes(s) + part_o_bytes(s, p.slices()) + part_lse_bytes(s, p.slices());
}

template <int D, int NW, int KG>
hipError_t launch_fwd(const pdy::CrossFwdArgs* a, dim3 grid, hipStream_t st) {
  using C = pdy::CrossFwdCfg<D, NW, KG>;
  if (a == nullptr) return set_lds(pdy::cross_fwd_kernel<D, NW, KG>, C::LDS_BYTES);
  hipLaunchKernelGGL((pdy::cross_fwd_kernel<D, NW, KG>), grid, dim3(C::NT), C::LDS_BYTES, st, *a);
  return hipSuccess;
}

struct CrossKernels {
  int nw, groups;
  hipError_t (*fwd[2])(const pdy::CrossFwdArgs*, dim3, hipStream_t);  // d = 64, 128
};
template <int NW, int G>
constexpr CrossKernels cross_kernels_of() {
  return CrossKernels{NW, G, {launch_fwd<64, NW, G>, launch_fwd<128, NW, G>}};
}
constexpr CrossKernels kCrossKernels[] = {cross_kernels_of<8, 1>(), cross_kernels_of<8, 2>(),
                                          cross_kernels_of<8, 4>(), cross_kernels_of<4, 4>()};
const CrossKernels& cross_kernels(const CrossShape& sh) {
  for (const CrossKernels& k : kCrossKernels)
    if (k.nw == sh.nw && k.groups == sh.groups) return k;
  return kCrossKernels[0];  // (not reached: every shape the launches use is listed)
}

hipError_t init_cross_kernels() {
  static hipError_t status = [] {
    for (const CrossKernels& k : kCrossKernels)
      for (int d = 0; d < 2; ++d) {
        hipError_t e = k.fwd[d](nullptr, dim3(), nullptr);
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
  if ((st = check_ptr(x.q, "q")) || (st = check_offsets(x.cu_q, "cu_seqlens_q")) ||
      (st = check_offsets(x.cu_k, "cu_seqlens_k")))
    return st;
  if (s.tk > 0 && ((st = check_ptr(x.k, "k")) || (st = check_ptr(x.v, "v")))) return st;
  if (s.prefix > 0 && ((st = check_ptr(x.kp, "k_prefix")) || (st = check_ptr(x.vp, "v_prefix"))))
    return st;
  if (x.len_k && (reinterpret_cast<uintptr_t>(x.len_k) & 3u) != 0)
    return fail(PDY_ERR_INVALID_ARG, "seqlens_k is not 4-byte aligned");
  return PDY_OK;
}

pdy::CrossBatch batch_of(const CrossIn& x, const CrossSizes& s, int32_t causal) {
  return pdy::CrossBatch{x.cu_q, x.cu_k, x.len_k, (int)s.n, (int)s.tq, (int)s.tk, (int)s.prefix,
                         (int)s.hq, (int)s.hkv, causal};
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
  const CrossFwdPlan p = fwd_plan(s);
  const size_t need = fwd_bytes(s, p);
  if (workspace_bytes < need)
    return fail(PDY_ERR_WORKSPACE, "workspace has %zu bytes, %s needs %zu", workspace_bytes, who,
                need);
  hipError_t e = init_cross_kernels();
  if (e != hipSuccess) return hip_fail(e, "kernel attribute setup");
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);

  pdy::CrossFwdArgs a;
  a.q = static_cast<const uint16_t*>(x.q);
  a.k = static_cast<const uint16_t*>(x.k);
  a.v = static_cast<const uint16_t*>(x.v);
  a.kp = static_cast<const uint16_t*>(x.kp);
  a.vp = static_cast<const uint16_t*>(x.vp);
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.b = batch_of(x, s, causal);
  a.scale_log2 = scale * pdy::kLog2e;
  a.part_o = a.part_lse = nullptr;
  a.part_n = nullptr;
  int32_t* counts = reinterpret_cast<int32_t*>(workspace);
  if (p.merge()) {
    uint8_t* w = reinterpret_cast<uint8_t*>(workspace) + 2 * part_n_bytes(s);
    a.part_o = reinterpret_cast<float*>(w);
    a.part_lse = reinterpret_cast<float*>(w + part_o_bytes(s, p.slices()));
  }
  for (int i = 0; i < p.launches; ++i) {
    const CrossFwd& f = p.l[i];
    a.cut = f.cut;
    if (p.merge()) a.part_n = counts + i * (part_n_bytes(s) / 4);
    const dim3 grid((unsigned)(f.wgs * s.hkv));
    e = launch_timed(K_CROSS_FWD, hs,
                     [&] { (void)cross_kernels(f.sh).fwd[s.d == 128](&a, grid, hs); });
    if (e != hipSuccess) return hip_fail(e, "cross_fwd_kernel launch");
  }
  if (p.merge()) {
    pdy::CrossMergeArgs m;
    m.part_o = a.part_o;
    m.part_lse = a.part_lse;
    m.part_n = counts;
    m.part_n1 = p.launches > 1 ? counts + part_n_bytes(s) / 4 : nullptr;
    m.max0 = p.l[0].cut.max_parts;
    m.max1 = p.launches > 1 ? p.l[1].cut.max_parts : 0;
    m.cu_q = x.cu_q;
    m.n = (int)s.n;
    m.tq = (int)s.tq;
    m.hq = (int)s.hq;
    m.o = a.o;
    m.lse = lse;
    const dim3 blocks((unsigned)ceil_div(s.tq * s.hq * (s.d / 8), 256));
    e = launch_timed(K_CROSS_MERGE, hs, [&] {
      if (s.d == 64) hipLaunchKernelGGL(pdy::cross_merge_kernel<64>, blocks, dim3(256), 0, hs, m);
      else hipLaunchKernelGGL(pdy::cross_merge_kernel<128>, blocks, dim3(256), 0, hs, m);
    });
    if (e != hipSuccess) return hip_fail(e, "cross_merge_kernel launch");
  }
  return PDY_OK;
}

}  // namespace

extern "C" {

size_t attn_prefix_fwd_workspace_size(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                      int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                      int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim) {
  CrossSizes s;
  if (check_cross_sizes(prefix_len, total_q, total_k, num_seqs, max_seqlen_q, max_seqlen_k,
                        num_heads_q, num_heads_kv, head_dim, &s) != PDY_OK)
    return 0;
  return s.tq == 0 ? 256 : fwd_bytes(s, fwd_plan(s));
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

}  // extern "C"
