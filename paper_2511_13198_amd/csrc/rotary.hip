// C-ABI of the rotary positions: argument checks, the frequencies as fractions of a
// turn, and the launch.  The contract is in include/pdyattn.h.
#include "../../include/pdyattn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host.hpp"
#include "rotary.hpp"

using namespace pdy_host;

namespace {

constexpr int64_t kFill = 1024;  // workgroups

// 1 / (2 pi) as a binary fraction, the first 64 bits first: enough that the largest
// double's whole turns are known.
constexpr uint64_t kInvTwoPi[] = {
    0x28be60db9391054a, 0x7f09d5f47d4d3770, 0x36d8a5664f10e410, 0x7f9458eaf7aef158,
    0x6dc91b8e909374b8, 0x01924bba82746487, 0x3f877ac72c4a69cf, 0xba208d7d4baed121,
    0x3a671c09ad17df90, 0x4e64758e60d4ce7d, 0x272117e2ef7e4a0e, 0xc7fe25fff7816603,
    0xfbcbc462d6829b47, 0xdb4d9fb3c9f2c26d, 0xd3d18fd9a797fa8b, 0x5d49eeb1faf97c5e,
    0xcf41ce7de294a4ba, 0x9afed7ec47e35742, 0x1580cc11bf1edaea};

// w / 2 pi modulo 1 as a fraction of 2^64, to the nearest.  With w = m 2^e, m of 53 bits,
// the bits of 1 / (2 pi) up to weight 2^-e give whole turns, and of those behind 192 leave
// the product off by less than 2^-138.
uint64_t turn_of(double w) {
  int e;
  const uint64_t m = (uint64_t)std::ldexp(std::frexp(std::fabs(w), &e), 53);
  e -= 53;
  // 64 bits from weight 2^-(at + 1) on (those in front of the point are 0)
  auto bits = [](int at) -> uint64_t {
    if (at <= -64) return 0;
    if (at < 0) return kInvTwoPi[0] >> -at;
    const int j = at / 64, s = at % 64;
    return s == 0 ? kInvTwoPi[j] : kInvTwoPi[j] << s | kInvTwoPi[j + 1] >> (64 - s);
  };
  typedef unsigned __int128 u128;
  const u128 low = (u128)m * bits(e + 128), mid = (u128)m * bits(e + 64) + (uint64_t)(low >> 64);
  const uint64_t turn = m * bits(e) + (uint64_t)(mid >> 64) + ((uint64_t)mid >> 63);
  return w < 0 ? -turn : turn;
}

template <class In, class Out, int D>
void launch_rotary(pdy::RotaryArgs& a, bool inter, int64_t heads, hipStream_t st) {
  constexpr int kHeads = 64 * 2 * (16 / (int)sizeof(In)) / D;  // of a wave's round
  // a wave takes its token's heads all, so that the angles are computed once, unless
  // that leaves the chip idle: then a part of the rounds each
  const int64_t rounds = (heads + kHeads - 1) / kHeads, blocks = ((int64_t)a.tokens + 3) / 4;
  const int64_t cuts = std::min(rounds, std::max<int64_t>(1, kFill / blocks));
  a.rounds = (int)((rounds + cuts - 1) / cuts);
  const dim3 grid((unsigned)blocks, (unsigned)((rounds + a.rounds - 1) / a.rounds));
  if (inter)
    hipLaunchKernelGGL((pdy::rotary_kernel<In, Out, D, true>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((pdy::rotary_kernel<In, Out, D, false>), grid, dim3(256), 0, st, a);
}

template <class In, class Out>
void launch_rotary(pdy::RotaryArgs& a, int d, bool inter, int64_t heads, hipStream_t st) {
  if (d == 64) launch_rotary<In, Out, 64>(a, inter, heads, st);
  else launch_rotary<In, Out, 128>(a, inter, heads, st);
}

}  // namespace

extern "C" {

pdy_status attn_rotary_turns(const double* freqs, int32_t num_pairs, uint64_t* turns) {
  g_err[0] = 0;
  if (num_pairs < 0 || (num_pairs > 0 && (freqs == nullptr || turns == nullptr)))
    return fail(PDY_ERR_INVALID_ARG, "attn_rotary_turns: bad arrays");
  for (int p = 0; p < num_pairs; ++p) {
    if (!std::isfinite(freqs[p])) return fail(PDY_ERR_INVALID_ARG, "freqs[%d] is not finite", p);
    turns[p] = turn_of(freqs[p]);
  }
  return PDY_OK;
}

pdy_status attn_rotary(const void* q, const void* k, const int32_t* positions,
                       int32_t total_tokens, int32_t num_axes, int32_t num_heads_q,
                       int32_t num_heads_kv, int32_t head_dim, int32_t num_pairs,
                       const uint64_t* turns, const int32_t* pair_axes, int32_t interleaved,
                       int32_t inverse, int32_t in_fp32, int32_t out_fp32, void* q_out,
                       void* k_out, void* stream) {
  g_err[0] = 0;
  pdy_status st;
  // (a launch's threads, 64 a token, are counted in 32 bits)
  if (total_tokens < 0 || total_tokens >= (1 << 26) - 4)
    return fail(PDY_ERR_INVALID_ARG, "total_tokens must be >= 0 and below 2^26 - 4 (got %d)",
                total_tokens);
  if (num_axes < 1 || num_axes > pdy::kMaxAxes)
    return fail(PDY_ERR_INVALID_ARG, "num_axes must be in [1, %d] (got %d)", pdy::kMaxAxes,
                num_axes);
  if (num_heads_q < 0 || num_heads_kv < 0 || (int64_t)num_heads_q + num_heads_kv < 1 ||
      (int64_t)num_heads_q + num_heads_kv > 65535)
    return fail(PDY_ERR_INVALID_ARG, "head counts must be >= 0 and 1 to 65,535 together (got %d, %d)",
                num_heads_q, num_heads_kv);
  if (head_dim != 64 && head_dim != 128)
    return fail(PDY_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", head_dim);
  if (num_pairs < 8 || num_pairs > head_dim / 2 || num_pairs % 8 != 0)
    return fail(PDY_ERR_INVALID_ARG,
                "num_pairs must be a multiple of 8 up to head_dim / 2 = %d (got %d)", head_dim / 2,
                num_pairs);
  if ((interleaved & ~1) || (inverse & ~1) || (in_fp32 & ~1) || (out_fp32 & ~1))
    return fail(PDY_ERR_INVALID_ARG, "interleaved, inverse, in_fp32 and out_fp32 must be 0 or 1");
  if (out_fp32 && !in_fp32)
    return fail(PDY_ERR_UNSUPPORTED, "bf16 to fp32 is not supported (bf16, fp32, or fp32 to bf16)");
  if (turns == nullptr || pair_axes == nullptr)
    return fail(PDY_ERR_INVALID_ARG, "turns and pair_axes (host arrays) must not be NULL");
  pdy::RotaryArgs a;
  for (int p = 0; p < num_pairs; ++p) {
    if (pair_axes[p] < 0 || pair_axes[p] >= num_axes)
      return fail(PDY_ERR_INVALID_ARG, "pair_axes[%d] must be in [0, %d) (got %d)", p, num_axes,
                  pair_axes[p]);
    a.freq[p] = turns[p];
    a.axis[p] = (uint8_t)pair_axes[p];
  }
  if (total_tokens == 0) return PDY_OK;
  if (num_heads_q > 0 && ((st = check_ptr(q, "q")) || (st = check_ptr(q_out, "q_out")))) return st;
  if (num_heads_kv > 0 && ((st = check_ptr(k, "k")) || (st = check_ptr(k_out, "k_out")))) return st;
  if (positions == nullptr || (reinterpret_cast<uintptr_t>(positions) & 3u) != 0)
    return fail(PDY_ERR_INVALID_ARG, "positions is NULL or not 4-byte aligned");
  if (in_fp32 != out_fp32 && ((num_heads_q > 0 && q == q_out) || (num_heads_kv > 0 && k == k_out)))
    return fail(PDY_ERR_INVALID_ARG, "in place needs one type for input and output");
  a.in[0] = q;
  a.in[1] = k;
  a.out[0] = q_out;
  a.out[1] = k_out;
  a.heads[0] = num_heads_q;
  a.heads[1] = num_heads_kv;
  a.pos = positions;
  a.tokens = total_tokens;
  a.axes = num_axes;
  a.pairs = num_pairs;
  a.inverse = inverse;
  const int64_t heads = (int64_t)num_heads_q + num_heads_kv;
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  const hipError_t e = launch_timed(K_ROTARY, hs, [&] {
    if (!in_fp32) launch_rotary<uint16_t, uint16_t>(a, head_dim, interleaved, heads, hs);
    else if (out_fp32) launch_rotary<float, float>(a, head_dim, interleaved, heads, hs);
    else launch_rotary<float, uint16_t>(a, head_dim, interleaved, heads, hs);
  });
  if (e != hipSuccess) return hip_fail(e, "rotary_kernel launch");
  return PDY_OK;
}

}  // extern "C"
