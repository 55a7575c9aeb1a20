// A paged key/value cache: new keys into their pages, attention of few rows a sequence
// over the pages, the keys' sums of attention weight, and eviction by them.
//
// k and v are [num_pages][hkv][page][D], bf16 or e4m3 (value = byte * the head's scale);
// key j of sequence i and head h is row j % page of page table[i][j / page].  A head's rows
// of a page lie together, so that a run of 16 keys (pages are multiples of it) is one
// piece of memory.  Such runs are numbered over the whole pool: run u starts at u * 16 * D
// elements (scores: u * 16).
//
// Lengths and page numbers read from memory are clamped, so that no value in them makes a
// kernel leave its tensors.
#pragma once
#include "common.hpp"

namespace pdy {

constexpr float kE4m3Max = 448.f;

struct PagedCache {
  const int32_t* table;  // [n][max_pages]
  const int32_t* len;    // [n]
  int n;
  int num_pages;
  int page;             // keys a page
  int max_pages;        // of a sequence
  int max_k;            // most keys of a sequence (at most max_pages * page)
  int hkv;
  int runs;             // page / 16
  uint32_t runs_inv;    // 2^32 / runs, rounded down (runs > 1)
};

// Keys in use of sequence i.
__device__ __forceinline__ int paged_len(const PagedCache& c, int i) {
  return c.num_pages > 0 ? min(max(c.len[i], 0), c.max_k) : 0;
}
// x / runs by the reciprocal, off by at most one (x >= 0).
__device__ __forceinline__ int paged_div(const PagedCache& c, int x) {
  if (c.runs == 1) return x;  // uniform
  const int t = (int)__umulhi((uint32_t)x, c.runs_inv);
  return x - t * c.runs >= c.runs ? t + 1 : t;
}
// The run that holds keys 16 x .. 16 x + 15 of sequence i and head h (x in use); -1: its page
// is none of the pool's.
__device__ __forceinline__ int paged_run(const PagedCache& c, int i, int h, int x) {
  const int p = paged_div(c, x);
  const int id = c.table[(size_t)i * c.max_pages + p];
  return (uint32_t)id < (uint32_t)c.num_pages ? (id * c.hkv + h) * c.runs + (x - p * c.runs) : -1;
}

// The sequence of packed token t: the last one that starts at t or before, of 64 evenly
// spaced offsets, of the 64th part behind the one found, ...; n where t is behind the last.
// (wave-uniform)
__device__ __forceinline__ int paged_seq_of(const int32_t* cu, int n, int t) {
  int lo = 0, span = n + 1;
  while (true) {
    const int step = (span + 63) >> 6, l = __lane_id();
    const bool at = l * step < span && cu[lo + l * step] <= t;
    const int k = max(0, __builtin_popcountll(__builtin_amdgcn_ballot_w64(at)) - 1);
    lo += k * step;
    span = min(step, span - k * step);
    if (step == 1) break;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// ---------------------------------------------------------------------------
// New keys and values into their pages.  Token t of a sequence with nq new tokens and nk
// keys in use (the new ones among them) is its key nk - nq + t.  A workgroup takes 2^each_log2
// tokens, 8 elements a thread: it loads them, finds the tokens' places, and stores.  e4m3
// rounds the 32-bit quotient x / scale to the nearest (beyond the largest number to it).
//
// Bound by memory, one token a sequence by the launch (3.3 us on the GPU).  All is read and
// written once, so past the caches: 8 prompts of 1,024-8,192 tokens to e4m3, 154 MB, 39.3 us
// through them, 35.4 past them, and 33.3 with two rounds' loads in flight (4.6 TB/s).
// ---------------------------------------------------------------------------
struct PagedWriteArgs {
  PagedCache c;
  const uint16_t* in[2];  // k, v [tokens][hkv][D]
  void* pages[2];
  const float* scale[2];  // [hkv]; NULL: bf16
  float* scores;          // NULL: none
  const int32_t* cu;
  int tokens;
  int each_log2;
  uint32_t units_inv;  // 2^32 / (hkv D / 8), rounded down
};
constexpr int kWriteLog2 = 4;

// 8 bf16 of one 16-byte word as 8 e4m3 of x / s.  The quotient is x inv and a correction by
// its remainder, which is as exact as the division (a quotient that a rounding to e4m3 could
// tell from it is hit), in 3 instructions where the division takes 10 and more.  (Beside the
// traffic of prompts either is hidden: 38.0 and 39.2 us.)  512 stands for all that is larger.
// A remainder under 2^-126 would lose bits, so a scale below 2^-64 is taken 2^64 times, and x
// with it.
__device__ __forceinline__ u32x2 paged_e4m3(const u32x4& x, float scale) {
  const float up = scale < 0x1p-64f ? 0x1p64f : 1.f, s = scale * up, inv = 1.f / s;
  uint32_t out[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[2] = {__uint_as_float(x[i] << 16) * up, __uint_as_float(x[i] & 0xffff0000u) * up};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float q = fminf(fmaxf(y[j] * inv, -512.f), 512.f);
      const float z = copysignf(__builtin_fmaf(__builtin_fmaf(-q, s, y[j]), inv, q), q);  // (-0)
      y[j] = z == z ? fminf(fmaxf(z, -kE4m3Max), kE4m3Max) : z;  // (a NaN stays one)
    }
    if (i & 1) out[i >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], out[i >> 1], true);
    else out[i >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], out[i >> 1], false);
  }
  return u32x2{out[0], out[1]};
}

template <int D, bool F8>
__global__ void __launch_bounds__(256) paged_write_kernel(PagedWriteArgs a) {
  constexpr int LANES = D / 8;  // of a row
  constexpr int AHEAD = 2;      // rounds of 256 threads loaded at a time
  __shared__ int64_t row_of[1 << kWriteLog2];  // row of kv head 0 in the pool; -1: none
  const PagedCache& c = a.c;
  const int t0 = blockIdx.x << a.each_log2, count = min(1 << a.each_log2, a.tokens - t0);
  const int units = c.hkv * LANES, total = count * units;
  const size_t from = (size_t)t0 * units * 8;
  for (int u0 = 0; u0 < total; u0 += 256 * AHEAD) {
    u32x4 x[AHEAD][2];
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) {
      const int u = u0 + r * 256 + threadIdx.x;
      if (u < total)
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
          x[r][kv] = __builtin_nontemporal_load(
              reinterpret_cast<const u32x4*>(a.in[kv] + from + (size_t)u * 8));
    }
    if (u0 == 0) {  // (behind the loads: neither waits for the other)
      if (threadIdx.x < 64) {
        int i = paged_seq_of(a.cu, c.n, t0);
        const int t = t0 + threadIdx.x;
        if ((int)threadIdx.x < count) {
          if (i < c.n && a.cu[i + 1] <= t) {  // of a later sequence: by bisection
            int hi = c.n;  // cu[i] <= t, and t < cu[hi + 1] or hi = n
            while (i < hi) {
              const int mid = (i + hi + 1) >> 1;
              if (a.cu[mid] <= t) i = mid;
              else hi = mid - 1;
            }
          }
          int64_t row = -1;
          if (i < c.n) {
            const int j = paged_len(c, i) - (a.cu[i + 1] - t);
            const int run = j >= 0 && j < c.max_k ? paged_run(c, i, 0, j >> 4) : -1;
            if (run >= 0) row = (int64_t)run * 16 + (j & 15);
          }
          row_of[threadIdx.x] = row;
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) {
      const int u = u0 + r * 256 + threadIdx.x;
      if (u >= total) continue;
      int k = (int)__umulhi((uint32_t)u, a.units_inv);  // u / units, off by at most one
      if (u - k * units >= units) ++k;
      const int h = (u - k * units) / LANES, e = (u % LANES) * 8;
      if (row_of[k] < 0) continue;
      const size_t row = (size_t)row_of[k] + (size_t)h * c.page;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        if constexpr (F8) {
          __builtin_nontemporal_store(
              paged_e4m3(x[r][kv], a.scale[kv][h]),
              reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.pages[kv]) + row * D + e));
        } else {
          __builtin_nontemporal_store(
              x[r][kv],
              reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.pages[kv]) + row * D + e));
        }
      }
      if (a.scores && e == 0) a.scores[row] = 0.f;
    }
  }
}

// ---------------------------------------------------------------------------
// Attention of few rows a sequence over its pages.
//   S_ij = scale <q_i, k_j>,  LSE_i = log sum_j exp(S_ij),  O_i = sum_j exp(S_ij - LSE_i) v_j
// over the visible keys j (causal: the last query sees every key, the one before all but
// the last, ...); a row that sees none gets O = 0, LSE = -inf.
//
// Rows are packed: the g heads of a group side by side, row R of a sequence and kv head hk
// being head hk g + R % g of token R / g, so that a key is read once for its group.  A
// workgroup has a tile of 16 RB packed rows of a sequence and a kv head; its waves take steps
// of 32 keys in turn, each on its own: S^T = K Q^T and O^T += V^T P^T on 16x16x32 matrix
// instructions (a row per lane of 16, its keys over the four groups of lanes), K and V copied
// to the wave's own LDS, so that no barrier stands in the loop.  At the end the waves' O,
// maxima and sums are combined.
//
// Bound by the bytes of K and V (d flops a byte and row of a group at most): what counts is
// that copies never pause.  A wave's 16 KB of LDS hold K and V of one step (d = 128, bf16) to
// four; K of a later step is issued as soon as the registers have the K in its place, V
// likewise, and waits are for a count of copies, so that a tile and more is always in flight:
// with each step waiting for its own copies a token for each of 64 sequences over 256-16,384
// keys of 8 heads (888 MB) took 410 us, so 266, with the keys in parts 166, past the caches 148
// (6.0 TB/s; a kernel that only reads reaches 6.3); e4m3 318, 152, 92, 79.  32 KB: no gain.
//
// P is rounded to bf16, as in the other attention kernels (O is off by 2.3e-3 of its norm,
// 1.7e-3 of which its own rounding is); logits, sums, maxima and LSE are 32 bits.  e4m3
// keys and values are widened to bf16, exactly, on their way to the matrix instructions;
// the scales go into the logits' and the output's.
// ---------------------------------------------------------------------------
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// The largest (the sum) of the values that lanes l, l ^ 16, l ^ 32, l ^ 48 hold.
__device__ __forceinline__ float quad_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The logits' factor, the head's scale in it.  Never 0 or infinite, where the product rounds to
// that: a masked logit (-inf) times 0, and a logit of 0 times infinity, would be NaN.
__device__ __forceinline__ float paged_scale(float scale_log2, const float* k_scale, int hk) {
  const float x = k_scale ? scale_log2 * k_scale[hk] : scale_log2;
  return x == 0.f ? __uint_as_float(1u) : fminf(x, 3.4028235e38f);
}
// 8 e4m3 as 8 bf16.
__device__ __forceinline__ bf16x8 widen8(const u32x2& x) {
  bf16x8 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 y = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i >> 1], 1.f, true)
                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i >> 1], 1.f, false);
    out[2 * i] = y[0];
    out[2 * i + 1] = y[1];
  }
  return out;
}

// LDS reads of the tiles, to be waited for: 16 bytes of K; 8 keys of a column of V (of 16
// bits 4 of a run and 4 of the next).
template <int OFF>
__device__ __forceinline__ void paged_read16(uint32_t addr, u32x4& x) {
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(x) : "v"(addr), "i"(OFF));
}
// (early clobber: the second read needs the address after the first was issued)
template <int RUN>
__device__ __forceinline__ void paged_read_tr16(uint32_t addr, u32x2& x, u32x2& y) {
  asm volatile("ds_read_b64_tr_b16 %0, %2\n\tds_read_b64_tr_b16 %1, %2 offset:%3"
               : "=&v"(x), "=&v"(y) : "v"(addr), "i"(RUN));
}
__device__ __forceinline__ void paged_read_tr8(uint32_t addr, u32x2& x) {
  asm volatile("ds_read_b64_tr_b8 %0, %1" : "=v"(x) : "v"(addr));
}
// Waits until at most N LDS operations are outstanding; the registers are tied to it.
template <int N>
__device__ __forceinline__ void paged_wait(u32x2& x) {
  asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(x) : "i"(N));
}
template <int N>
__device__ __forceinline__ void paged_wait(u32x2& x, u32x2& y) {
  asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(x), "+v"(y) : "i"(N));
}

// A wave's tile of 32 keys (two runs) in LDS: rows of D elements as they are in memory, the
// 16-byte chunks of row r exchanged by exclusive or, so that the reads of K (a chunk of 16
// rows a quarter-wave) and the transposing reads of V (8 rows of 32 bytes, or 16 of 16,
// a half-wave) meet no bank twice.
template <int D, bool F8>
struct PagedTile {
  static constexpr int ROW = D * (F8 ? 1 : 2);  // bytes
  static constexpr int CHUNKS = ROW / 16;
  static constexpr int RUN = 16 * ROW;          // bytes of a run
  static constexpr int COPIES = RUN / 1024;     // instructions that copy it
  static constexpr int BYTES = 2 * RUN;
  __device__ __forceinline__ static int swz_k(int r) {
    return ROW == 256 ? r & 15 : ROW == 128 ? (r >> 1) & 7 : (r >> 2) & 3;
  }
  __device__ __forceinline__ static int swz_v(int r) {
    if constexpr (!F8) return ROW == 256 ? (2 * r) & 15 : 2 * ((r >> 1) & 3);
    return ROW == 128 ? ((r >> 1) & 3) + 4 * ((r >> 4) & 1) : ((r >> 2) & 1) + 2 * ((r >> 4) & 1);
  }
};

template <int D, bool F8, int RB, int NW>
struct PagedFwdCfg {
  using T = PagedTile<D, F8>;
  static constexpr int NT = NW * 64;
  static constexpr int ROWS = 16 * RB;
  static constexpr int SLOTS = 16384 / (2 * T::BYTES);  // tiles of K and V: 16 KB a wave
  static constexpr int WAVE = SLOTS * 2 * T::BYTES;
  // waves a SIMD at least: 2 leave 256 registers, without a need for accumulation registers
  // (and copies to and from them); 64 rows of 128 need more (478, e4m3 459: one wave a SIMD)
  static constexpr int WAVES = RB * D >= 512 ? 1 : 2;
  static constexpr int PITCH = D + 4;        // floats of a combined row
  static constexpr int STAT = NW * ROWS * PITCH * 4;
  static constexpr int END = STAT + NW * ROWS * 8;
  static constexpr int LDS_BYTES = NW * WAVE > END ? NW * WAVE : END;
  static_assert(LDS_BYTES <= 160 * 1024, "LDS");
};

// How a launch is cut.  An item is a row tile of a sequence and a kv head; its steps of 32
// keys are cut into parts of at most C = max(least, steps of all items / entries), a
// workgroup each: about `entries` parts a kv head, alike whatever the lengths, and up to
// one an item more.  C follows from the lengths on the GPU, so that nothing waits for the
// host: every workgroup computes it and its own place, with a lane per sequence, or a thread
// where there are more.
struct PagedCut {
  int max_parts;  // of an item; 1: not cut
  int least;      // fewest steps of a part
  int entries;    // parts of a kv head
};
// A sequence as the kernels see it: its rows in q, and its keys.
struct PagedSeq {
  int q_lo, nq, nk;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedCache& c, const int32_t* cu_q, int tq,
                                              int i) {
  const int lo = cu_q[i], hi = cu_q[i + 1], len = c.len[i];
  PagedSeq s;
  s.q_lo = min(max(lo, 0), tq);
  s.nq = min(max(hi, s.q_lo), tq) - s.q_lo;
  s.nk = c.num_pages > 0 ? min(max(len, 0), c.max_k) : 0;
  return s;
}

struct PagedPlace {
  PagedSeq s;
  int seq, tile, part, nparts;
  float steps;  // of all items
};

// Steps of 32 keys of all sequences, by every wave on its own (of more than 1,024 sequences
// by the first).
__device__ __forceinline__ float paged_all_steps(const PagedCache& c) {
  const int n = min(c.n, 1024);
  float sum = 0.f;
  for (int i = __lane_id(); i < n; i += 64) sum += (float)((paged_len(c, i) + 31) >> 5);
  return wave_sum(sum) * ((float)c.n / (float)n);
}

// Entry `entry` of a kv head's list; false past its end.  get(i): sequence i; of(s, tiles,
// steps): its row tiles, and steps of each.  (wave-uniform)
template <int NT, class G, class F>
__device__ __forceinline__ bool paged_place(const PagedCut& c, int n, int entry, G&& get, F&& of,
                                            PagedPlace& out) {
  __shared__ float sum_of[NT / 64];
  __shared__ int entries_of[NT / 64], found[6];
  const bool wide = n > 64;  // uniform
  const int id = wide ? threadIdx.x : __lane_id(), stride = wide ? NT : 64;
  const int w = threadIdx.x >> 6, l = __lane_id();
  // (the first sequence of a lane is kept: more than one has a lane beyond 256 alone)
  PagedSeq s0 = {0, 0, 0};
  int tiles0 = 0, steps0 = 0, tiles, steps;
  if (id < n) {
    s0 = get(id);
    of(s0, tiles0, steps0);
  }
  float sum = (float)tiles0 * (float)steps0;
  for (int i = id + stride; i < n; i += stride) {
    of(get(i), tiles, steps);
    sum += (float)tiles * (float)steps;
  }
  sum = wave_sum(sum);
  if (wide) {
    if (l == 0) sum_of[w] = sum;
    __syncthreads();
    sum = 0.f;
    for (int i = 0; i < NT / 64; ++i) sum += sum_of[i];
  }
  const int cap = max(c.least, (int)fminf(sum / (float)c.entries + 1.f, 1e9f));
  const float inv = 1.f / (float)cap;
  // ceil(steps / cap) as a float product (any whole number near it does)
  auto parts = [&](int steps) __attribute__((always_inline)) {
    return max(1, min(c.max_parts, (int)ceilf((float)steps * inv)));
  };
  int np = parts(steps0), mine = tiles0 * np;
  for (int i = id + stride; i < n; i += stride) {
    of(get(i), tiles, steps);
    mine += tiles * parts(steps);
  }
  int before = wave_scan(mine) - mine;
  if (wide) {
    if (l == 63) entries_of[w] = before + mine;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    for (int i = 0; i < w; ++i) before += entries_of[i];
  }
  const bool hit = entry >= before && entry < before + mine;
  int seq = id, rel = entry - before;
  if (hit && rel >= tiles0 * np) {
    rel -= tiles0 * np;
    for (int i = id + stride; i < n; i += stride) {
      seq = i;
      s0 = get(i);
      of(s0, tiles, steps);
      np = parts(steps);
      if (rel < tiles * np) break;
      rel -= tiles * np;
    }
  }
  if (wide) {
    if (hit) {
      found[0] = seq;
      found[1] = rel;
      found[2] = np;
      found[3] = s0.q_lo;
      found[4] = s0.nq;
      found[5] = s0.nk;
    }
    __syncthreads();
    seq = found[0];
    rel = found[1];
    np = found[2];
    s0 = PagedSeq{found[3], found[4], found[5]};
    if (seq < 0) return false;
  } else {
    const uint64_t any = __builtin_amdgcn_ballot_w64(hit);
    if (!any) return false;
    const int src = __builtin_ctzll(any);
    auto lane = [&](int& x) __attribute__((always_inline)) {
      x = __builtin_amdgcn_readlane(x, src);
    };
    lane(seq);
    lane(rel);
    lane(np);
    lane(s0.q_lo);
    lane(s0.nq);
    lane(s0.nk);
  }
  auto uni = [](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(x); };
  out.s = PagedSeq{uni(s0.q_lo), uni(s0.nq), uni(s0.nk)};
  out.steps = sum;
  out.seq = uni(seq);
  out.nparts = uni(np);
  rel = uni(rel);
  out.tile = rel / out.nparts;
  out.part = rel - out.tile * out.nparts;
  return true;
}

struct PagedFwdArgs {
  PagedCache c;
  const uint16_t* q;
  const void* k;
  const void* v;
  const float* k_scale;  // [hkv]; NULL: 1
  const float* v_scale;
  const int32_t* cu_q;
  int tq, hq, g;
  uint32_t g_inv;
  int causal;
  int max_tiles;  // row tiles of a sequence
  PagedCut cut;
  // steps of 32 keys of a kv head beyond which K and V do not fit the last-level cache, and
  // are read past it; -1: they are read through it without a look
  int stream_steps;
  int keep_k;  // (more than 16 rows) K through the caches all the same
  float scale_log2;
  uint16_t* o;
  float* lse;
  // partial results (max_parts > 1): O (fp32, normalised by the part's own sums) and LSE of
  // part p at part_o [p][tq * hq][D], part_lse [p][tq * hq] (NaN: a NaN or +inf logit), and
  // how many parts a row has at part_n [tq * hq]
  float* part_o;
  float* part_lse;
  int32_t* part_n;
  // logits <q_i, k_j> of row r of sequence i and kv head h at [(i hkv + h) rows + r][keys],
  // -inf where not visible (LOGITS)
  float* logits;
  int logit_rows, logit_keys;
};

// One copy of 1 KB into LDS: lane l's 16 bytes at base + voff, zeros from `bytes` on; STREAM:
// past the caches (non-temporal).
template <bool STREAM>
__device__ __forceinline__ void paged_copy(uint64_t base, int bytes, uint32_t voff, uint8_t* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto rs =
      __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, bytes, kBufferFlags);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds, 16,
                                           voff, 0, 0, STREAM ? 2 : 0);
#endif
}

// 16 bytes to base + voff, nowhere from `bytes` on: one store, whatever the lanes.
__device__ __forceinline__ void paged_store(uint64_t base, int bytes, uint32_t voff, f32x4 x) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto rs =
      __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, bytes, kBufferFlags);
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), rs, voff, 0, 0);
#endif
}

template <int D, bool F8, int RB, int NW, bool LOGITS, bool WHOLE>
__global__ void __launch_bounds__(NW * 64, (PagedFwdCfg<D, F8, RB, NW>::WAVES))
    paged_fwd_kernel(PagedFwdArgs a) {
  using C = PagedFwdCfg<D, F8, RB, NW>;
  using T = typename C::T;
  constexpr int KS = D / 32, DB = D / 16;
  extern __shared__ __attribute__((aligned(1024))) uint8_t paged_smem[];
  const PagedCache& c = a.c;
  const int hk = blockIdx.x % (unsigned)c.hkv, entry = blockIdx.x / (unsigned)c.hkv;
  const int l = __lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Lane 2 i + s knows where run s of the wave's step i (mod 32) is: the 32 keys of its step
  // j are those from (first + NW j) 32 on.  (A run past the last key in use may be any.)
  int runs_of = 0;
  auto find_runs = [&](int seq, int first, int j) __attribute__((always_inline)) {
    const int x = 2 * (first + NW * (j + (l >> 1))) + (l & 1);
    runs_of = x * 16 < c.max_k && c.num_pages > 0 ? max(0, paged_run(c, seq, hk, x)) : 0;
  };
  PagedPlace at;
  if (WHOLE || a.cut.max_parts == 1) {
    at.seq = WHOLE ? entry : entry / a.max_tiles;
    at.tile = entry - at.seq * (WHOLE ? 1 : a.max_tiles);
    at.part = 0;
    at.nparts = 1;
    if constexpr (WHOLE) find_runs(at.seq, w, 0);  // (without waiting for the lengths)
    at.s = paged_seq(c, a.cu_q, a.tq, at.seq);
    at.steps = a.stream_steps >= 0 ? paged_all_steps(c) : 0.f;
  } else if (!paged_place<C::NT>(
                 a.cut, c.n, entry,
                 [&](int i) __attribute__((always_inline)) {
                   return paged_seq(c, a.cu_q, a.tq, i);
                 },
                 [&](const PagedSeq& s, int& tiles, int& steps) __attribute__((always_inline)) {
                   tiles = min((s.nq * a.g + C::ROWS - 1) / C::ROWS, a.max_tiles);
                   steps = (s.nk + 31) >> 5;
                 },
                 at)) {
    return;
  }
  const int seq = at.seq, tile = at.tile, q_lo = at.s.q_lo, nq = at.s.nq, nk = at.s.nk;
  const int row_end = nq * a.g;  // packed rows, from the sequence's first on
  const int row0 = tile * C::ROWS;
  if (row0 >= row_end) return;
  const int i16 = l & 15, grp = l >> 4;
  auto token = [&](int r) __attribute__((always_inline)) {
    if (a.g == 1) return r;
    const int t = (int)__umulhi((uint32_t)r, a.g_inv);
    return r - t * a.g >= a.g ? t + 1 : t;
  };
  auto key_end = [&](int r) __attribute__((always_inline)) {
    return a.causal ? max(0, min(nk, token(min(r, row_end - 1)) + nk - nq + 1)) : nk;
  };
  // (token, head) pair of a packed row, counted over the batch
  auto pair_of = [&](int r) __attribute__((always_inline)) {
    const int t = token(r);
    return (size_t)(q_lo + t) * a.hq + hk * a.g + (r - t * a.g);
  };
  int end[RB];
  bf16x8 qf[RB][KS];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int r = row0 + b * 16 + i16;
    end[b] = key_end(r);
    const bool ok = r < row_end;
    const uint16_t* qp = a.q + pair_of(ok ? r : row0) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[b][ks] = load_bf16x8(qp + (F8 ? ((ks >> 1) * 4 + grp) * 16 + (ks & 1) * 8
                                       : ks * 32 + grp * 8), ok);
  }
  const int all_end = __builtin_amdgcn_readfirstlane(key_end(row0));            // seen by every row
  const int some_end = __builtin_amdgcn_readfirstlane(key_end(row0 + C::ROWS - 1));  // by some
  const float scale2 = paged_scale(a.scale_log2, F8 ? a.k_scale : nullptr, hk);

  f32x4 oacc[RB][DB];
  float m[RB], lsum[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    m[b] = -INFINITY;
    lsum[b] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[b][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  uint8_t* const mine = paged_smem + w * C::WAVE;  // SLOTS times K, V
  uint32_t kv_off[2][T::COPIES][2];  // this lane's bytes of a run: [k, v][copy][run]
#pragma unroll
  for (int i = 0; i < T::COPIES; ++i) {
    const int at = i * 1024 + l * 16, r = at / T::ROW, slot = (at % T::ROW) / 16;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      kv_off[0][i][s] = r * T::ROW + (slot ^ T::swz_k(r + 16 * s)) * 16;
      kv_off[1][i][s] = r * T::ROW + (slot ^ T::swz_v(r + 16 * s)) * 16;
    }
  }
  const uint32_t ka = lds_addr(mine) + i16 * T::ROW + (grp ^ T::swz_k(i16)) * 16;
  uint32_t va;
  if constexpr (F8) {
    const int e = i16 >> 1, r = e < 4 ? 4 * grp + e : 16 + 4 * grp + e - 4;
    va = lds_addr(mine) + T::BYTES + r * T::ROW + T::swz_v(r) * 16 + (i16 & 1) * 8;
  } else {
    const int r = 4 * grp + (i16 >> 2);
    va = lds_addr(mine) + T::BYTES + r * T::ROW + T::swz_v(r) * 16 + ((i16 & 3) >> 1) * 16 +
         (i16 & 1) * 8;
  }

  // the part's steps, and this wave's
  const int all_steps = (some_end + 31) >> 5;
  const int first = (WHOLE ? 0 : (int)((int64_t)at.part * all_steps / at.nparts)) + w;
  const int last = WHOLE ? all_steps : (int)((int64_t)(at.part + 1) * all_steps / at.nparts);
  const int steps = max(0, last - first + NW - 1) / NW;
  // copies of step j's K (kv = 0) or V; past the last step of an empty range, so that
  // every step has as many copies
  auto issue = [&](auto Stream, auto Kv, int j) __attribute__((always_inline)) {
    constexpr int kv = decltype(Kv)::value;
    uint8_t* const to = mine + ((j % C::SLOTS) * 2 + kv) * T::BYTES;
    const uint64_t base = (uint64_t)(kv ? a.v : a.k);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int run = __builtin_amdgcn_readlane(runs_of, ((j & 31) * 2) | s);
      const int valid = j < steps ? min(16, nk - (first + NW * j) * 32 - s * 16) : 0;
      const int bytes = __builtin_amdgcn_readfirstlane(max(0, valid) * T::ROW);
      const uint64_t from = base + (uint64_t)run * T::RUN;
      uint8_t* const dst = to + s * T::RUN;
#pragma unroll
      for (int i = 0; i < T::COPIES; ++i)
        paged_copy<((decltype(Stream)::value >> kv) & 1) != 0>(from, bytes, kv_off[kv][i][s],
                                                                dst + i * 1024);
    }
  };
  // What is in flight behind a step's K when its products begin, and behind its V when these
  // are read: (2 SLOTS - 1) tiles' copies, and the stores of logits since the step's K were
  // issued (in front of those of their step) or its V (behind them); before step SLOTS
  // these are fewer, and not counted.
  constexpr int FLIGHT = (2 * C::SLOTS - 1) * 2 * T::COPIES;
  auto wait_step = [&](auto V, int j) __attribute__((always_inline)) {
    constexpr int stores = LOGITS ? 2 * (decltype(V)::value ? C::SLOTS - 1 : C::SLOTS) : 0;
    if (stores > 0 && j >= C::SLOTS) wait_dma_n<FLIGHT + stores>();
    else wait_dma_n<FLIGHT>();
  };
  // (rows that are none lie behind the end of the buffer)
  uint32_t logit_off = 0;
  uint64_t logit_at = 0;
  if constexpr (LOGITS) {
    static_assert(RB == 1, "one row a lane");
    logit_off = i16 < row_end - row0 ? (uint32_t)(i16 * a.logit_keys + grp * 4) * 4 : 0x80000000u;
    logit_at = (uint64_t)(a.logits + (size_t)(seq * c.hkv + hk) * a.logit_rows * a.logit_keys);
  }
  constexpr std::integral_constant<int, 0> K;
  constexpr std::integral_constant<int, 1> V;
  auto all_of = [&](auto Stream) __attribute__((always_inline)) {
    if (steps <= 0) return;
    if (!WHOLE) find_runs(seq, first, 0);
    wait_dma();
#pragma unroll
    for (int j = 0; j < C::SLOTS; ++j) {
      issue(Stream, K, j);
      issue(Stream, V, j);
    }
    for (int j = 0; j < steps; ++j) {
      const int k0 = (first + NW * j) * 32;
      const uint32_t slot = (j % C::SLOTS) * 2 * T::BYTES;
      wait_step(std::false_type{}, j);

      // S^T = K Q^T, two runs of 16 keys, all reads ahead of the products
      f32x4 s[RB][2];
      constexpr int N = F8 ? KS / 2 : KS;
      u32x4 kr[N][2];
      static_for<N>([&](auto I) {
        constexpr int i = decltype(I)::value;
        paged_read16<0>((ka ^ (i * 64)) + slot, kr[i][0]);
        paged_read16<T::RUN>((ka ^ (i * 64)) + slot, kr[i][1]);
      });
#pragma unroll
      for (int b = 0; b < RB; ++b) s[b][0] = s[b][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      static_for<N>([&](auto I) {
        constexpr int i = decltype(I)::value;
        row_wait<2 * (N - 1 - i)>(kr[i][0], kr[i][1]);
#pragma unroll
        for (int h = 0; h < KS / N; ++h) {
          const int ks = i * (KS / N) + h;
#pragma unroll
          for (int run = 0; run < 2; ++run) {
            bf16x8 x;
            if constexpr (F8) x = widen8(u32x2{kr[i][run][h * 2], kr[i][run][h * 2 + 1]});
            else x = as_bf16x8(kr[i][run]);
#pragma unroll
            for (int b = 0; b < RB; ++b) s[b][run] = mfma16(x, qf[b][ks], s[b][run]);
          }
        }
      });
      const int next = j + C::SLOTS;
      if ((next & 31) == 0) {  // (the last use of the ones before was V's)
        find_runs(seq, first, next);
        wait_dma();
      }
      wave_lds_fence();
      issue(Stream, K, next);

      // V's reads run beside the softmax
      wait_step(std::true_type{}, j);
      constexpr int VR = F8 ? 1 : 2;  // reads of 16 columns
      u32x2 vr[DB][VR];
      static_for<DB>([&](auto I) {
        constexpr int db = decltype(I)::value;
        if constexpr (F8) paged_read_tr8((va ^ (db * 16)) + slot, vr[db][0]);
        else paged_read_tr16<T::RUN>((va ^ (db * 32)) + slot, vr[db][0], vr[db][VR - 1]);
      });

      bf16x8 pf[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        if (k0 + 32 > all_end) {
#pragma unroll
          for (int run = 0; run < 2; ++run)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (k0 + run * 16 + grp * 4 + r >= end[b]) s[b][run][r] = -INFINITY;
        }
        if constexpr (LOGITS)
#pragma unroll
          for (int run = 0; run < 2; ++run)
            paged_store(logit_at, a.logit_rows * a.logit_keys * 4,
                        logit_off + (uint32_t)(k0 + run * 16) * 4, s[b][run]);
        float top = -INFINITY;
#pragma unroll
        for (int run = 0; run < 2; ++run)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, s[b][run][r]);
        top = quad_max(top) * scale2;
        const bool grow = top > m[b] + kRescaleSlack;
        if (__builtin_amdgcn_ballot_w64(grow) != 0) {
          const float alpha = grow ? fast_exp2(m[b] - top) : 1.f;
          m[b] = grow ? top : m[b];
          lsum[b] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[b][db] *= alpha;
        }
        const float muse = m[b] == -INFINITY ? 0.f : m[b];
#pragma unroll
        for (int run = 0; run < 2; ++run)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = fast_exp2(__builtin_fmaf(s[b][run][r], scale2, -muse));
            lsum[b] += p;
            pf[b][run * 4 + r] = (__bf16)p;
          }
      }

      // O^T += V^T P^T, 16 columns at a time
      static_for<DB>([&](auto I) {
        constexpr int db = decltype(I)::value;
        bf16x8 x;
        if constexpr (F8) {
          paged_wait<DB - 1 - db>(vr[db][0]);
          x = widen8(vr[db][0]);
        } else {
          paged_wait<2 * (DB - 1 - db)>(vr[db][0], vr[db][VR - 1]);
          x = TrRegs{vr[db][0], vr[db][VR - 1]}.operand();
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) oacc[b][db] = mfma16(x, pf[b], oacc[b][db]);
      });
      wave_lds_fence();
      issue(Stream, V, next);
    }
  };
  const bool stream = a.stream_steps >= 0 && at.steps > (float)a.stream_steps;
  if (RB > 1 && stream && a.keep_k) all_of(std::integral_constant<int, 2>{});
  else if (stream) all_of(std::integral_constant<int, 3>{});
  else all_of(std::integral_constant<int, 0>{});

  // combine the waves: O, offset and sum of every row through LDS
  wait_dma();
  __syncthreads();
  float* const slots = reinterpret_cast<float*>(paged_smem);
  f32x2* const stat = reinterpret_cast<f32x2*>(paged_smem + C::STAT);
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float tot = quad_sum(lsum[b]);
    float* const to = slots + ((size_t)w * C::ROWS + b * 16 + i16) * C::PITCH + grp * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(to + db * 16) = oacc[b][db];
    if (grp == 0) stat[w * C::ROWS + b * 16 + i16] = f32x2{m[b], tot};
  }
  __syncthreads();
  const float out_scale = F8 ? a.v_scale[hk] : 1.f;
  for (int u = threadIdx.x; u < C::ROWS * (D / 8); u += C::NT) {
    const int r = u / (D / 8), e = (u % (D / 8)) * 8;
    if (row0 + r >= row_end) continue;
    float mx = -INFINITY, tot = 0.f;
#pragma unroll
    for (int j = 0; j < NW; ++j) mx = fmaxf(mx, stat[j * C::ROWS + r][0]);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const f32x2 st = stat[j * C::ROWS + r];
      // (a NaN sum makes the row's)
      const float wt = st[1] > 0.f || st[1] != st[1] ? fast_exp2(st[0] - mx) : 0.f;
      tot += wt * st[1];
      const float* const src = slots + ((size_t)j * C::ROWS + r) * C::PITCH + e;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] += wt * src[k];
    }
    const float inv = tot > 0.f || tot != tot ? out_scale / tot : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] *= inv;
    const size_t pair = pair_of(row0 + r), pairs = (size_t)a.tq * a.hq;
    // (a part hands a NaN sum on as NaN)
    const float lse = tot > 0.f ? (mx + __builtin_log2f(tot)) * kLn2
                      : !WHOLE && at.nparts > 1 ? tot - INFINITY : -INFINITY;
    if (!WHOLE && e == 0 && at.part == 0 && a.cut.max_parts > 1) a.part_n[pair] = at.nparts;
    if (!WHOLE && at.nparts > 1) {
      cross_put8(x, a.part_o + (at.part * pairs + pair) * D + e);
      if (e == 0) a.part_lse[at.part * pairs + pair] = lse;
    } else {
      cross_put8(x, a.o + pair * D + e);
      const int t = token(row0 + r);
      if (e == 0) a.lse[(size_t)(hk * a.g + (row0 + r - t * a.g)) * a.tq + q_lo + t] = lse;
    }
  }
}

// Combine the partial results of the rows that have more than one:
//   LSE = log sum_p exp(LSE_p),  O = sum_p exp(LSE_p - LSE) O_p;
// a part with LSE = -inf weighs nothing, one with NaN makes the row O = NaN, LSE = -inf.  A
// wave per (token, head) pair, or a workgroup where parts are many: a lane per part for the
// weights (64 at a time), then 512 / D parts at a time, 8 elements a lane.  Bound by the
// launch and two rounds of loads: 5 us, 32 rows of 128 parts 6.6 (a wave each: 17.5).
struct PagedMergeArgs {
  const float* part_o;
  const float* part_lse;
  const int32_t* part_n;
  int max_parts;
  const int32_t* cu_q;  // rows end at cu_q[n]
  int n;
  int tq, hq;
  uint16_t* o;
  float* lse;
  int wide;  // a workgroup a pair
};

// One pair by W waves of a workgroup (1, or all 4, a share of the parts each).
template <int D, int W>
__device__ __forceinline__ void paged_merge(const PagedMergeArgs& a, uint32_t pair) {
  constexpr int LANES = D / 8, GROUPS = 64 / LANES;
  __shared__ float acc_of[W][D];
  __shared__ float stat_of[W][2];
  const int l = __lane_id();
  const int w = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t pairs = (uint32_t)a.tq * a.hq;
  if (pair >= pairs) return;
  const int tok = (int)(pair / (uint32_t)a.hq), h = (int)(pair - (uint32_t)tok * a.hq);
  // (one wave: read before it is known how many there are)
  const float x0 = W == 1 && l < a.max_parts ? a.part_lse[(size_t)l * pairs + pair] : 0.f;
  const int parts = min(max(a.part_n[pair], 0), a.max_parts);
  // rows behind the last sequence stay, and those written by their one part
  if (tok >= a.cu_q[a.n] || parts <= 1) return;
  const int c = (l % LANES) * 8, grp = l / LANES;
  float mx = -INFINITY, tot = 0.f;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int share = (parts + W - 1) / W, last = min(parts, (w + 1) * share);  // this wave's
  // (more than 64 parts: the sums so far are rescaled by each further 64)
  for (int p0 = w * share; p0 < last; p0 += 64) {
    const float x = p0 + l >= last ? -INFINITY
                    : W == 1 && p0 == 0 ? x0 : a.part_lse[(size_t)(p0 + l) * pairs + pair];
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
    const int m = min(64, last - p0);
#pragma unroll 4
    for (int j0 = 0; j0 < m; j0 += GROUPS) {
      // (every lane takes part in the exchange; past the last part the weight is 0)
      const float wj = __shfl(wt, j0 + grp);
      const int pj = p0 + min(j0 + grp, m - 1);
      const float* src = a.part_o + ((size_t)pj * pairs + pair) * D + c;
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
  if constexpr (W > 1) {
    if (grp == 0) cross_put8(acc, &acc_of[w][c]);
    if (l == 0) {
      stat_of[w][0] = mx;
      stat_of[w][1] = tot;
    }
    __syncthreads();
    if (w != 0) return;
    mx = stat_of[0][0];
#pragma unroll
    for (int i = 1; i < W; ++i) mx = fmaxf(mx, stat_of[i][0]);
    tot = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float t = stat_of[i][1];
      const float wt = t > 0.f || t != t ? fast_exp2((stat_of[i][0] - mx) * kLog2e) : 0.f;
      tot += wt * t;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += wt * acc_of[i][c + e];
    }
  }
  const float inv = tot > 0.f ? 1.f / tot : tot != tot ? NAN : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] *= inv;
  if (grp == 0) cross_put8(acc, a.o + (size_t)pair * D + c);
  if (l == 0)
    a.lse[(size_t)h * a.tq + tok] = tot > 0.f ? mx + __builtin_log2f(tot) * kLn2 : -INFINITY;
}

template <int D>
__global__ void __launch_bounds__(256) paged_merge_kernel(PagedMergeArgs a) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // token * hq + head
  if (a.wide) paged_merge<D, 4>(a, blockIdx.x);
  else paged_merge<D, 1>(a, blockIdx.x * 4 + w);
}

// ---------------------------------------------------------------------------
// The keys' weights: scores_j += sum over the sequence's rows i (of all heads of the group)
// of exp(S_ij - LSE_i), for the visible keys.  A key's rows are summed in a fixed order, by one
// lane from the logits, by four from the keys, whose sums are joined, and added once, without
// atomics: the same call gives the same bits.  (LSE differs in rounding with the parts that a
// launch is cut into, and the weights with it.)  Rows with LSE = -inf (no key, or a NaN or
// +inf logit) add nothing.
// ---------------------------------------------------------------------------

// From the logits that the attention kernel left (up to 16 rows a sequence and kv head), in
// one launch with the joining of parts: a workgroup past those that join takes 4,096 keys
// of a sequence and kv head, and joins the parts' LSE of its rows itself.  (Workgroups start
// at about 440 a microsecond: with 1,024 keys each, the 4,608 of 64 sequences of up to 8,192
// keys and 8 kv heads had all started after 10.5 us, of 14.)  The logits cost 4 bytes a row
// and key written and read, the keys again 2 D: a token of those sequences, 32/8 heads, 306 us
// from the keys, 140 so (the attention 128, without logits 110; this kernel 13).
struct PagedJoinArgs {
  PagedMergeArgs m;
  int merge_blocks;
  PagedCache c;
  int g, key_blocks;
  const float* logits;
  int logit_rows, logit_keys;
  float scale_log2;
  const float* k_scale;
  float* scores;
};

constexpr int kWeighKeys = 4096;  // of a workgroup, 4 a thread at a time

template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedJoinArgs a) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = __lane_id();
  if ((int)blockIdx.x < a.merge_blocks) {
    if (a.m.wide) paged_merge<D, 4>(a.m, blockIdx.x);
    else paged_merge<D, 1>(a.m, blockIdx.x * 4 + w);
    return;
  }
  __shared__ float lse2[16];  // base 2
  const PagedCache& c = a.c;
  const int block = blockIdx.x - a.merge_blocks;
  const int item = block / a.key_blocks, seq = item / c.hkv, hk = item - seq * c.hkv;
  const int nk = paged_len(c, seq), j0 = (block - item * a.key_blocks) * kWeighKeys;
  const int q_lo = min(max(a.m.cu_q[seq], 0), a.m.tq);
  const int nq = min(max(a.m.cu_q[seq + 1], q_lo), a.m.tq) - q_lo;
  const int rows = min(nq * a.g, a.logit_rows);
  if (j0 >= nk || rows == 0) return;
  constexpr int AHEAD = 4;  // rows
  struct Keys {  // 4 of this thread
    int j, run;
    f32x4 x[AHEAD], old;
  };
  const float* const item_logits = a.logits + (size_t)item * a.logit_rows * a.logit_keys;
  auto load = [&](int i, Keys& k) __attribute__((always_inline)) {
    k.j = j0 + i * 1024 + threadIdx.x * 4;
    k.run = -1;
    if (k.j < nk) {
#pragma unroll
      for (int r = 0; r < AHEAD; ++r)
        k.x[r] = *reinterpret_cast<const f32x4*>(
            item_logits + (size_t)min(r, rows - 1) * a.logit_keys + k.j);
      k.run = paged_run(c, seq, hk, k.j >> 4);
    }
    if (k.run >= 0)
      k.old = *reinterpret_cast<const f32x4*>(a.scores + (size_t)k.run * 16 + (k.j & 15));
  };
  Keys keys[2];
  load(0, keys[0]);  // (while the rows' LSE are joined)
  const size_t pairs = (size_t)a.m.tq * a.m.hq;
  for (int r = w; r < rows; r += 4) {
    const int t = q_lo + r / a.g, h = hk * a.g + r % a.g;
    const size_t pair = (size_t)t * a.m.hq + h;
    const float y0 = l < a.m.max_parts && a.m.max_parts > 1 ? a.m.part_lse[l * pairs + pair] : 0.f;
    const int parts = a.m.max_parts > 1 ? min(max(a.m.part_n[pair], 0), a.m.max_parts) : 1;
    float z = -INFINITY;
    if (parts <= 1) {
      z = a.m.lse[(size_t)h * a.m.tq + t] * kLog2e;
    } else {
      float top = -INFINITY, sum = 0.f;
      for (int p = l; p < parts; p += 64)
        top = fmaxf(top, p == l ? y0 : a.m.part_lse[p * pairs + pair]);
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
      for (int p = l; p < parts; p += 64) {
        const float y = p == l ? y0 : a.m.part_lse[p * pairs + pair];
        sum += y == -INFINITY ? 0.f : fast_exp2((y - top) * kLog2e);
      }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
      if (sum > 0.f) z = top * kLog2e + __builtin_log2f(sum);  // (a NaN sum: nothing)
    }
    if (l == 0) lse2[r] = z;
  }
  __syncthreads();
  const float scale2 = paged_scale(a.scale_log2, a.k_scale, hk);
  static_for<kWeighKeys / 1024>([&](auto I) {
    constexpr int i = decltype(I)::value;
    if (j0 + i * 1024 >= nk) return;  // uniform
    if constexpr ((i + 1) * 1024 < kWeighKeys) load(i + 1, keys[(i + 1) & 1]);
    Keys& k = keys[i & 1];
    if (k.run < 0) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < rows; r0 += AHEAD) {
#pragma unroll
      for (int r = 0; r < AHEAD; ++r) {
        const float z = r0 + r < rows ? lse2[r0 + r] : -INFINITY;
        if (z > -INFINITY)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += fast_exp2(__builtin_fmaf(k.x[r][e], scale2, -z));
      }
      if (r0 + AHEAD < rows)
#pragma unroll
        for (int r = 0; r < AHEAD; ++r)
          k.x[r] = *reinterpret_cast<const f32x4*>(
              item_logits + (size_t)min(r0 + AHEAD + r, rows - 1) * a.logit_keys + k.j);
    }
    float* const to = a.scores + (size_t)k.run * 16 + (k.j & 15);
    if (k.j + 4 <= nk) {
      *reinterpret_cast<f32x4*>(to) = k.old + sum;
    } else {
      for (int e = 0; e < nk - k.j; ++e) to[e] = k.old[e] + sum[e];
    }
  });
}

// From the keys again, where rows are many: a wave holds 16 RB rows, and takes runs of 16
// keys, some loaded while one is worked on.  S = Q K^T here, a key per lane of 16, so that a
// key's rows are in its four lanes' registers, and the sum over them is joined once.  Bound
// by K's bytes, where the attention left them in the last-level cache: 32 tokens of 6
// sequences over 4,000-16,384 keys of 16 heads, d = 64 (K 100 MB), 23 us, from memory 27.
struct PagedWeighArgs {
  PagedCache c;
  const uint16_t* q;
  const void* k;
  const float* k_scale;
  const int32_t* cu_q;
  const float* lse;
  int tq, hq, g;
  uint32_t g_inv;
  int causal;
  float scale_log2;
  float* scores;
};

constexpr int kWeighRuns = 8;  // of a wave

template <int D, bool F8, int RB>
__global__ void __launch_bounds__(256) paged_weigh_kernel(PagedWeighArgs a) {
  constexpr int KS = D / 32;
  using T = PagedTile<D, F8>;
  const PagedCache& c = a.c;
  const int hk = blockIdx.y, seq = blockIdx.z;
  const int q_lo = min(max(a.cu_q[seq], 0), a.tq);
  const int nq = min(max(a.cu_q[seq + 1], q_lo), a.tq) - q_lo;
  const int nk = paged_len(c, seq);
  const int l = __lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = l & 15, grp = l >> 4;
  const int rows = nq * a.g;
  const float scale2 = paged_scale(a.scale_log2, F8 ? a.k_scale : nullptr, hk);
  const int first = (blockIdx.x * 4 + w) * kWeighRuns;
  const int count = min(kWeighRuns, ((nk + 15) >> 4) - first);
  if (count <= 0) return;
  // lane i knows where run first + i is
  int runs_of = -1;
  if (l < count) runs_of = paged_run(c, seq, hk, first + l);
  using Raw = std::conditional_t<F8, u32x2, u32x4>;
  auto load = [&](int x, Raw (&k)[KS]) __attribute__((always_inline)) {
    const int run = max(0, __builtin_amdgcn_readlane(runs_of, min(x, count - 1)));
    const uint8_t* const kp =
        static_cast<const uint8_t*>(a.k) + (size_t)run * T::RUN + i16 * T::ROW;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      k[ks] = __builtin_nontemporal_load(
          reinterpret_cast<const Raw*>(kp + (ks * 32 + grp * 8) * (F8 ? 1 : 2)));
  };
  float sum[kWeighRuns], old[kWeighRuns];  // (lanes of a key: the same)
#pragma unroll
  for (int x = 0; x < kWeighRuns; ++x) {
    sum[x] = 0.f;
    old[x] = a.scores[(size_t)max(0, __builtin_amdgcn_readlane(runs_of, x)) * 16 + i16];
  }
  for (int r0 = 0; r0 < rows; r0 += 16 * RB) {
    constexpr int AHEAD = 4;  // runs in flight
    Raw kr[AHEAD][KS];
#pragma unroll
    for (int x = 0; x < AHEAD - 1; ++x) load(x, kr[x]);
    bf16x8 qf[RB][KS];
    float lse2[RB][4];
    int end[RB][4], all_end = 0x7fffffff;  // of the lane's rows, and seen by all of them
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      auto place = [&](int r, int& t, int& h) __attribute__((always_inline)) {
        t = r;
        if (a.g > 1) {
          t = (int)__umulhi((uint32_t)r, a.g_inv);
          t = r - t * a.g >= a.g ? t + 1 : t;
        }
        h = hk * a.g + (r - t * a.g);
      };
      int t, h;
      place(min(r0 + b * 16 + i16, rows - 1), t, h);
      const uint16_t* const qp = a.q + ((size_t)(q_lo + t) * a.hq + h) * D + grp * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[b][ks] = load_bf16x8(qp + ks * 32, true);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = r0 + b * 16 + grp * 4 + e;
        place(min(r, rows - 1), t, h);
        const float lse = a.lse[(size_t)h * a.tq + q_lo + t];
        const bool ok = r < rows && lse > -INFINITY;
        end[b][e] = ok ? (a.causal ? min(nk, t + nk - nq + 1) : nk) : 0;
        lse2[b][e] = ok ? lse * kLog2e : 0.f;
        all_end = min(all_end, end[b][e]);
      }
    }
    static_for<kWeighRuns>([&](auto I) {
      // (runs past the last are the last again, and masked: no branch parts the loads)
      constexpr int x = decltype(I)::value, cur = x % AHEAD;
      if constexpr (x + AHEAD - 1 < kWeighRuns) load(x + AHEAD - 1, kr[(x + AHEAD - 1) % AHEAD]);
      bf16x8 kf[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if constexpr (F8) kf[ks] = widen8(kr[cur][ks]);
        else kf[ks] = as_bf16x8(kr[cur][ks]);
      }
      const int j = (first + x) * 16 + i16;
      const bool masked = __builtin_amdgcn_ballot_w64((first + x + 1) * 16 > all_end) != 0;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mfma16(qf[b][ks], kf[ks], s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = fast_exp2(__builtin_fmaf(s[e], scale2, -lse2[b][e]));
          sum[x] += !masked || j < end[b][e] ? p : 0.f;
        }
      }
    });
  }
#pragma unroll
  for (int x = 0; x < kWeighRuns; ++x) {
    const float all = quad_sum(sum[x]);
    const int run = __builtin_amdgcn_readlane(runs_of, x);
    if (run >= 0 && grp == 0 && (first + x) * 16 + i16 < nk)
      a.scores[(size_t)run * 16 + i16] = old[x] + all;
  }
}

// ---------------------------------------------------------------------------
// Eviction.  Of a head's L keys the first `first`, the last `recent` and, of those between,
// the ones of the highest scores stay, `budget` together; equal scores: the earlier key.
// Scores are ordered as numbers, a NaN below all.
//
// paged_select_kernel, a workgroup per sequence and head, finds the smallest score that
// stays: its 32 bits from the highest on, 11 at a time, each by the counts of the keys that
// share the bits found so far; then writes the numbers of the keys that stay, in order.
// Scores are read once, into registers.  Over up to 32,768 keys the time is that of one
// workgroup's steps one after the other, while those of 4 sequences and 8 heads leave most CUs
// idle: 18 us with the sums over waves in a loop and a page looked up for every 4 keys, 14 with
// them in one scan, passes with constant shifts and a page's place found once for its run.  Its
// waves wait (for LDS, barriers and the scores) 58 % of that, and issue VALU work in 12 %.
// paged_gather_kernel copies them to their new places, bound by memory: 64 sequences of 2,304
// keys to 2,048, 8 heads, d = 128, 1.07 GB, 207 us (5.2 TB/s; through the caches 217).
// ---------------------------------------------------------------------------
struct PagedEvictArgs {
  PagedCache c;
  const int32_t* new_table;  // [n][new_pages]
  int new_pages;
  int budget, recent, first;
  float* scores;
  uint8_t* k;
  uint8_t* v;
  int32_t* kept;  // [n][hkv][budget]
  int32_t* new_len;
};

// Scores as unsigned numbers of the same order, a NaN as 1; 0 is no key.
__device__ __forceinline__ uint32_t paged_order(float x) {
  const uint32_t b = __float_as_uint(x);
  return x != x ? 1u : b == 0x80000000u ? 0x80000000u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048;

// Rows j0 .. of sequence and head to their new places, by THREADS threads, LANES lanes of 16
// bytes a row: the workgroup finds the places of 4 THREADS / LANES rows, then every thread
// copies 4 rows' chunks of K and V, all loaded before the first is stored.
template <int LANES, int THREADS>
constexpr int kGatherRows = 4 * THREADS / LANES;

template <int LANES, int THREADS>
__device__ __forceinline__ void paged_gather(const PagedEvictArgs& a, int seq, int hk, int j0,
                                             int n) {
  constexpr int ROWS = kGatherRows<LANES, THREADS>, STEP = THREADS / LANES;
  static_assert(ROWS <= THREADS, "a thread a row");
  __shared__ int64_t src_of[ROWS], dst_of[ROWS];  // -1: none
  const PagedCache& c = a.c;
  const int t = threadIdx.x, j = j0 + t;
  if (t < ROWS) {
    int64_t src = -1, dst = -1;
    if (j < n) {
      const int from = a.kept[((size_t)seq * c.hkv + hk) * a.budget + j];
      const int p = paged_div(c, j >> 4);
      const int id = a.new_table[(size_t)seq * a.new_pages + p];
      const int run = from >= 0 ? paged_run(c, seq, hk, from >> 4) : -1;
      if (run >= 0 && (uint32_t)id < (uint32_t)c.num_pages) {
        src = (int64_t)run * 16 + (from & 15);
        dst = ((int64_t)(id * c.hkv + hk) * c.runs + ((j >> 4) - p * c.runs)) * 16 + (j & 15);
      }
    }
    src_of[t] = src;
    dst_of[t] = dst;
  }
  __syncthreads();
  const int e = (t % LANES) * 16;
  u32x4 x[4][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t src = src_of[t / LANES + i * STEP];
    if (src >= 0) {
      x[i][0] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(a.k + src * (LANES * 16) + e));
      x[i][1] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(a.v + src * (LANES * 16) + e));
    }
  }
  float score = 0.f;
  const bool mine = t < ROWS && src_of[t] >= 0;
  if (mine) score = a.scores[src_of[t]];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t dst = dst_of[t / LANES + i * STEP];
    if (dst >= 0) {
      __builtin_nontemporal_store(x[i][0],
                                  reinterpret_cast<u32x4*>(a.k + dst * (LANES * 16) + e));
      __builtin_nontemporal_store(x[i][1],
                                  reinterpret_cast<u32x4*>(a.v + dst * (LANES * 16) + e));
    }
  }
  if (mine) a.scores[dst_of[t]] = score;
}

// QUADS: groups of 4 keys that a thread holds in registers; 0: every pass reads them again.
template <int QUADS>
__device__ __forceinline__ void paged_select(const PagedEvictArgs& a, int seq, int hk) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t wave_more[kSelectWaves], wave_tie[kSelectWaves], found[2];
  const PagedCache& c = a.c;
  const int t = threadIdx.x, l = __lane_id();
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int n = paged_len(c, seq);
  int32_t* const kept = a.kept + ((size_t)seq * c.hkv + hk) * a.budget;
  if (n <= a.budget) {
    for (int j = t; j < a.budget; j += kSelectThreads) kept[j] = j < n ? j : -1;
    return;
  }
  // (first + recent <= budget < n)
  const int lo = a.first, hi = n - a.recent;
  const int stay = a.budget - a.first - a.recent;  // of the keys lo .. hi
  // this wave's keys: `per` rounds of 256 from `from` on, 4 a lane
  const int start = lo & ~15;
  const int per = ((hi - start + kSelectWaves - 1) / kSelectWaves + 255) >> 8;
  const int from = start + w * per * 256 + l * 4;
  struct Quad {
    uint32_t x[4];
  };
  auto order = [&](int j, int run) __attribute__((always_inline)) {
    Quad q = {{0u, 0u, 0u, 0u}};
    if (j < hi) {
      const f32x4* const at =
          reinterpret_cast<const f32x4*>(a.scores + (size_t)max(run, 0) * 16 + (j & 15));
      const f32x4 y = run < 0 ? f32x4{NAN, NAN, NAN, NAN} : *at;
#pragma unroll
      for (int e = 0; e < 4; ++e) q.x[e] = j + e >= lo && j + e < hi ? paged_order(y[e]) : 0u;
    }
    return q;
  };
  Quad key[QUADS > 0 ? QUADS : 1];
  if constexpr (QUADS > 0) {
    // lane i knows where run i of every 64 of them is
    constexpr int BATCHES = (QUADS + 3) / 4;
    int runs_of[BATCHES];
#pragma unroll
    for (int b = 0; b < BATCHES; ++b)
      runs_of[b] = paged_run(c, seq, hk, min(((from - l * 4) >> 4) + b * 64 + l, (hi - 1) >> 4));
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      const int run = __shfl(runs_of[u / 4], u % 4 * 16 + (l >> 2));
      key[u] = u < per ? order(from + u * 256, run) : Quad{{0u, 0u, 0u, 0u}};
    }
  }
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (QUADS > 0) {
#pragma unroll
      for (int u = 0; u < QUADS; ++u)
        if (u < per) f(from + u * 256, key[u]);  // uniform
    } else {
#pragma unroll 2
      for (int u = 0; u < per; ++u) {
        const int j = from + u * 256;
        f(j, order(j, j < hi ? paged_run(c, seq, hk, j >> 4) : -1));
      }
    }
  };
  // the sum over the waves in front of this one
  auto in_front = [&](const uint32_t* of) __attribute__((always_inline)) {
    const int x = wave_scan(l < w ? (int)of[l] : 0);
    return (uint32_t)__builtin_amdgcn_readlane(x, 63);
  };
  // the stay-th largest: bits 31..21, 20..10, 9..0; `need`: how many stay of those that
  // share its bits
  uint32_t bits = 0u, need = (uint32_t)stay;
  if (stay > 0)
    static_for<3>([&](auto Pass) __attribute__((always_inline)) {
      constexpr int pass = decltype(Pass)::value;
      constexpr int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
      constexpr uint32_t bins = 1u << width;
      hist[t] = hist[t + kSelectThreads] = 0u;
      __syncthreads();
      each([&](int, const Quad& q) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
        {
          // (what is no key counts as the smallest, and `stay` are keys)
          const uint32_t x = pass == 0 ? q.x[e] : q.x[e] - bits;
          if (pass == 0 ? x != 0u : x >> shift < bins) atomicAdd(&hist[x >> shift], 1u);
        }
      });
      __syncthreads();
      // counts from the highest bin down: two bins a thread
      const uint32_t b1 = bins - 1 - 2 * t, h1 = 2 * t < (int)bins ? hist[b1] : 0u,
                     h0 = 2 * t < (int)bins ? hist[b1 - 1] : 0u;
      const uint32_t incl = (uint32_t)wave_scan((int)(h1 + h0));
      if (l == 63) wave_more[w] = incl;
      __syncthreads();
      const uint32_t above = incl - h1 - h0 + in_front(wave_more);
      if (above < need && need <= above + h1 + h0) {
        const bool second = need > above + h1;
        found[0] = second ? b1 - 1 : b1;
        found[1] = need - above - (second ? h1 : 0u);
      }
      __syncthreads();
      bits |= found[0] << shift;
      need = found[1];
    });
  // each wave's keys in order: those above, and the first `need` equal ones
  uint32_t more = 0u, ties = 0u;
  each([&](int, const Quad& q) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      more += __builtin_popcountll(__builtin_amdgcn_ballot_w64(q.x[e] > bits));
      ties += __builtin_popcountll(__builtin_amdgcn_ballot_w64(q.x[e] == bits));
    }
  });
  __syncthreads();  // (the last reads of wave_more)
  if (l == 0) {
    wave_more[w] = more;
    wave_tie[w] = ties;
  }
  __syncthreads();
  uint32_t tie = in_front(wave_tie), at = in_front(wave_more) + a.first + min(tie, need);
  // lanes below this one that a ballot has
  auto below = [&](uint64_t m) __attribute__((always_inline)) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  };
  if (stay > 0)
    each([&](int j, const Quad& q) __attribute__((always_inline)) {
      bool mine[4];
      uint64_t eq[4], any = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mine[e] = q.x[e] > bits;
        eq[e] = __builtin_amdgcn_ballot_w64(q.x[e] == bits);
        any |= eq[e];
      }
      if (any) {  // uniform
        uint32_t before = tie;
#pragma unroll
        for (int e = 0; e < 4; ++e) before += below(eq[e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (q.x[e] == bits) {
            mine[e] = before < need;
            ++before;
          }
          tie += __builtin_popcountll(eq[e]);
        }
      }
      uint32_t to = at;
      uint64_t in[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        in[e] = __builtin_amdgcn_ballot_w64(mine[e]);
        to += below(in[e]);
        at += __builtin_popcountll(in[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (mine[e]) kept[to++] = j + e;
    });
  for (int j = t; j < a.first; j += kSelectThreads) kept[j] = j;
  for (int j = t; j < a.recent; j += kSelectThreads) kept[a.budget - a.recent + j] = hi + j;
}

// A workgroup a sequence and head.  LANES > 0: it copies the rows as well.
template <int QUADS, int LANES>
__global__ void __launch_bounds__(kSelectThreads) paged_select_kernel(PagedEvictArgs a) {
  const int hk = blockIdx.x % (unsigned)a.c.hkv, seq = blockIdx.x / (unsigned)a.c.hkv;
  paged_select<QUADS>(a, seq, hk);
  if constexpr (LANES > 0) {
    const int n = min(paged_len(a.c, seq), a.budget);
    for (int j0 = 0; j0 < n; j0 += kGatherRows<LANES, kSelectThreads>) {
      __syncthreads();  // (kept, and the places of the rows before, are read)
      paged_gather<LANES, kSelectThreads>(a, seq, hk, j0, n);
    }
    if (hk == 0 && threadIdx.x == 0) a.new_len[seq] = n;
  }
}

template <int LANES>
__global__ void __launch_bounds__(256) paged_gather_kernel(PagedEvictArgs a) {
  const int hk = blockIdx.y, seq = blockIdx.z;
  const int n = min(paged_len(a.c, seq), a.budget);
  if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) a.new_len[seq] = n;
  const int j0 = blockIdx.x * kGatherRows<LANES, 256>;
  if (j0 < n) paged_gather<LANES, 256>(a, seq, hk, j0, n);
}

}  // namespace pdy
