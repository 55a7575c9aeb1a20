// Rotary positions with several axes.
//
// The first 2 `pairs` elements of a head are rotated in pairs: pair p, with the axis
// of its section and the frequency w_p (radians a position), by the angle
// positions[t][axis_p] w_p:
//   (x, y) -> (x cos - y sin, x sin + y cos),
// (x, y) being elements p and p + pairs, or 2 p and 2 p + 1 (interleaved); the
// inverse, which is also the gradient's rotation, takes the negative angle.  The rest
// of a head is copied.
//
// Angles.  A position of 10^5 and more times w in 32-bit floats would leave the angle
// off by 10^-2.  The caller gives w_p / 2 pi as a 64-bit fraction F of a turn; pos * F
// mod 2^64 is then the angle in turns with whole turns gone, exact to pos * 2^-65.
// Its upper 32 bits are split into the nearest eighth ... quarter turn and a
// remainder of at most an eighth, whose sine and cosine are the Taylor sums to x^9
// and x^10: the first terms left out are below 1.8e-9 and 1.2e-10 (x <= pi / 4), less
// than a 32-bit rounding.
//
// Bound by memory: each element is read and written once.  A lane keeps the sines and
// cosines of its 8 (4 of 32-bit elements) pairs of a token in registers and takes them
// through the token's heads, so that they are computed once per token and lane.
#pragma once
#include "common.hpp"

namespace pdy {

constexpr int kMaxAxes = 4;
constexpr int kMaxPairs = 64;

struct RotaryArgs {
  const void* in[2];  // q, k: [tokens][heads][d]
  void* out[2];
  int heads[2];
  const int32_t* pos;  // [tokens][axes]
  int tokens, axes;
  int pairs;
  int heads_per_block;  // of q and k together; gridDim.y blocks of them
  int inverse;
  uint64_t freq[kMaxPairs];  // turns a position, as a fraction of 2^64
  uint8_t axis[kMaxPairs];
};

// sin and cos of turn / 2^32 turns.
__device__ __forceinline__ void sincos_turn(uint32_t turn, float& sn, float& cs) {
  const uint32_t quarter = (turn + 0x20000000u) >> 30;  // the nearest quarter turn
  const float x = (float)(int32_t)(turn - (quarter << 30)) * (6.283185307179586f / 4294967296.f);
  const float x2 = x * x;
  float s = 2.7557319224e-6f;  // 1 / 9!
  s = __builtin_fmaf(s, x2, -1.9841269841e-4f);
  s = __builtin_fmaf(s, x2, 8.3333333333e-3f);
  s = __builtin_fmaf(s, x2, -1.6666666667e-1f);
  s = __builtin_fmaf(s * x2, x, x);
  float c = -2.7557319224e-7f;  // -1 / 10!
  c = __builtin_fmaf(c, x2, 2.4801587302e-5f);
  c = __builtin_fmaf(c, x2, -1.3888888889e-3f);
  c = __builtin_fmaf(c, x2, 4.1666666667e-2f);
  c = __builtin_fmaf(c, x2, -0.5f);
  c = __builtin_fmaf(c, x2, 1.f);
  const bool odd = quarter & 1;
  const float a = odd ? c : s, b = odd ? s : c;
  sn = quarter & 2 ? -a : a;
  cs = (quarter + 1) & 2 ? -b : b;
}

// N consecutive elements as floats, and back.
template <int N>
__device__ __forceinline__ void rot_load(const uint16_t* p, float (&x)[N]) {
  static_assert(N == 8, "16 bytes");
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
template <int N>
__device__ __forceinline__ void rot_load(const float* p, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i + e] = v[e];
  }
}
template <int N>
__device__ __forceinline__ void rot_store(uint16_t* p, const float (&x)[N]) {
  uint32_t v[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i)
    v[i] = __builtin_bit_cast(uint32_t,
                              __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
  if constexpr (N == 8) *reinterpret_cast<u32x4*>(p) = u32x4{v[0], v[1], v[2], v[3]};
  else *reinterpret_cast<u32x2*>(p) = u32x2{v[0], v[1]};
}
template <int N>
__device__ __forceinline__ void rot_store(float* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4)
    *reinterpret_cast<f32x4*>(p + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
}

// A lane has the units u and u + d / (2 N) of every head, of N elements each (16
// bytes of input): as pairs p = u N + i, one element of each from either unit
// (halves), or the N / 2 pairs of either unit (interleaved).  D / (2 N) lanes a
// token; a workgroup takes 256 / that many tokens and heads_per_block heads of them.
// Where `pairs` is below d / 2 the halves' second element is in unit (p + pairs) / N.
template <class In, class Out, int D, bool INTER>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a) {
  constexpr int N = 16 / sizeof(In);
  constexpr int LANES = D / (2 * N);
  constexpr int TOKENS = 256 / LANES;
  const int tok = blockIdx.x * TOKENS + threadIdx.x / LANES;
  const int u = threadIdx.x % LANES;
  if (tok >= a.tokens) return;
  // first elements of the lane's two units, and their first pairs (negative: copied)
  int e0, e1, p0, p1;
  const int rot = a.pairs / N;  // units of a half of the rotated part
  if (INTER) {
    e0 = u * N;
    e1 = D / 2 + u * N;
    p0 = e0 < 2 * a.pairs ? e0 / 2 : -1;
    p1 = e1 < 2 * a.pairs ? e1 / 2 : -1;
  } else if (u < rot) {
    e0 = u * N;
    e1 = a.pairs + u * N;
    p0 = p1 = e0;
  } else {  // units behind the rotated part, two a lane
    e0 = 2 * a.pairs + (u - rot) * N;
    e1 = e0 + (D / 2 - a.pairs);
    p0 = p1 = -1;
  }
  float sn[N], cs[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = INTER ? (i < N / 2 ? p0 : p1) : p0;
    sn[i] = 0.f;
    cs[i] = 1.f;
    if (p >= 0) {
      const int q = p + (INTER ? i % (N / 2) : i);
      const int64_t at = a.pos[(size_t)tok * a.axes + a.axis[q]];
      sincos_turn((uint32_t)(((uint64_t)at * a.freq[q]) >> 32), sn[i], cs[i]);
      if (a.inverse) sn[i] = -sn[i];
    }
  }
  const int all = a.heads[0] + a.heads[1];
  const int h_end = min(all, (int)(blockIdx.y + 1) * a.heads_per_block);
  for (int h = blockIdx.y * a.heads_per_block; h < h_end; ++h) {
    const int t = h >= a.heads[0];
    const size_t off = ((size_t)tok * a.heads[t] + (t ? h - a.heads[0] : h)) * D;
    const In* in = static_cast<const In*>(a.in[t]) + off;
    Out* out = static_cast<Out*>(a.out[t]) + off;
    float x[N], y[N], ox[N], oy[N];
    rot_load(in + e0, x);
    rot_load(in + e1, y);
    if (INTER) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const int j = N / 2 + i;
        ox[2 * i] = x[2 * i] * cs[i] - x[2 * i + 1] * sn[i];
        ox[2 * i + 1] = x[2 * i] * sn[i] + x[2 * i + 1] * cs[i];
        oy[2 * i] = y[2 * i] * cs[j] - y[2 * i + 1] * sn[j];
        oy[2 * i + 1] = y[2 * i] * sn[j] + y[2 * i + 1] * cs[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        ox[i] = x[i] * cs[i] - y[i] * sn[i];
        oy[i] = x[i] * sn[i] + y[i] * cs[i];
      }
    }
    if (!INTER && p0 < 0) {  // (copied as it is: a rotation by 0 would turn 0 * inf to NaN)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        ox[i] = x[i];
        oy[i] = y[i];
      }
    }
    if (INTER && p0 < 0)
#pragma unroll
      for (int i = 0; i < N; ++i) ox[i] = x[i];
    if (INTER && p1 < 0)
#pragma unroll
      for (int i = 0; i < N; ++i) oy[i] = y[i];
    rot_store(out + e0, ox);
    rot_store(out + e1, oy);
  }
}

}  // namespace pdy
