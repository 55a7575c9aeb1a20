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
// off by 10^-2.  The caller gives w_p / 2 pi as a 64-bit fraction F of a turn, rounded to
// the nearest; pos * F mod 2^64 is then the angle in turns with whole turns gone, off by
// at most |pos| 2^-65 of a turn, 2^-34.  Its upper 32 bits (off by 2^-32) are split into the nearest eighth ... quarter turn and a
// remainder of at most an eighth, whose sine and cosine are the Taylor sums to x^9
// and x^10: the first terms left out are below 1.8e-9 and 1.2e-10 (x <= pi / 4), less
// than a 32-bit rounding.
//
// Bound by memory: each element is read and written once.  A wave has one token: its
// lanes compute the token's sines and cosines once, a pair each, and exchange them
// through LDS; then D / (2 N) lanes take a head (16 bytes of input a lane and half), so
// that the wave streams neighbouring heads, up to 2 KB at a time, with the next heads'
// loads in flight.  65,536 tokens of 32/8 heads, bf16: 249 us (5.4 TB/s); with a lane's pairs
// kept over one head after another of 8 tokens, 8 KB apart, 295 us.  131,072 of 4/4 in
// 32 bits: 186 us (5.8).
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
  int rounds;  // of a wave over its token's heads; gridDim.y blocks of them
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

__device__ __forceinline__ float rot_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float rot_float(float x) { return x; }

// N consecutive outputs, rounded to nearest even.
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

// A lane has the units u and u + d / (2 N) of a head, of N elements each (16 bytes of
// input): as pairs p = u N + i, one element of each from either unit (halves), or the
// N / 2 pairs of either unit (interleaved).  Where `pairs` is below d / 2 the halves'
// second elements are in unit (p + pairs) / N, and the lanes behind have the units that
// are copied.
template <class In, class Out, int D, bool INTER>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a) {
  constexpr int N = 16 / sizeof(In);
  constexpr int LANES = D / (2 * N);
  constexpr int HEADS = 64 / LANES;  // a round
  __shared__ f32x2 turn[4][kMaxPairs];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = __lane_id();
  const int tok = blockIdx.x * 4 + w;
  if (tok >= a.tokens) return;
  const int u = l % LANES;
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
  const int all = a.heads[0] + a.heads[1];
  const int h_end = min(all, (int)(blockIdx.y + 1) * a.rounds * HEADS);
  int h = blockIdx.y * a.rounds * HEADS + l / LANES;
  // element offset of the lane's head, in q or k
  auto at = [&](int head, int& t) __attribute__((always_inline)) {
    t = head >= a.heads[0];
    return ((size_t)tok * a.heads[t] + (t ? head - a.heads[0] : head)) * D;
  };
  In x[N], y[N];
  auto load = [&](int head) __attribute__((always_inline)) {
    int t;
    const In* in = static_cast<const In*>(a.in[t = head >= a.heads[0]]) + at(head, t);
    *reinterpret_cast<u32x4*>(x) = *reinterpret_cast<const u32x4*>(in + e0);
    *reinterpret_cast<u32x4*>(y) = *reinterpret_cast<const u32x4*>(in + e1);
  };
  if (h < h_end) load(h);  // (on its way while the angles are computed)
  if (l < a.pairs) {
    const int64_t pos = a.pos[(size_t)tok * a.axes + a.axis[l]];
    float sn, cs;
    sincos_turn((uint32_t)(((uint64_t)pos * a.freq[l]) >> 32), sn, cs);
    turn[w][l] = f32x2{a.inverse ? -sn : sn, cs};
  }
  wave_lds_fence();  // (a wave's own LDS operations complete in order)
  float sn[N], cs[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = INTER ? (i < N / 2 ? p0 : p1) : p0;
    const f32x2 v = turn[w][max(p, 0) + (INTER ? i % (N / 2) : i)];
    sn[i] = v[0];
    cs[i] = v[1];
  }
  for (; h < h_end; h += HEADS) {
    float fx[N], fy[N], ox[N], oy[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      fx[i] = rot_float(x[i]);
      fy[i] = rot_float(y[i]);
    }
    if (h + HEADS < h_end) load(h + HEADS);
    if (INTER) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const int j = N / 2 + i;
        ox[2 * i] = fx[2 * i] * cs[i] - fx[2 * i + 1] * sn[i];
        ox[2 * i + 1] = fx[2 * i] * sn[i] + fx[2 * i + 1] * cs[i];
        oy[2 * i] = fy[2 * i] * cs[j] - fy[2 * i + 1] * sn[j];
        oy[2 * i + 1] = fy[2 * i] * sn[j] + fy[2 * i + 1] * cs[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        ox[i] = fx[i] * cs[i] - fy[i] * sn[i];
        oy[i] = fx[i] * sn[i] + fy[i] * cs[i];
      }
    }
    // (copied as it is: a rotation by 0 would turn infinities into NaN)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      ox[i] = p0 < 0 ? fx[i] : ox[i];
      oy[i] = p1 < 0 ? fy[i] : oy[i];
    }
    int t;
    const size_t off = at(h, t);
    Out* out = static_cast<Out*>(a.out[t]) + off;
    rot_store(out + e0, ox);
    rot_store(out + e1, oy);
  }
}

}  // namespace pdy
