// Per-head norm and position rotation of rows of queries and keys.
//
// A row is one head of one token, D 16-bit numbers.  Its D / 8 lanes hold eight channels each, as two
// chunks of four whose places depend on how the channels are paired, so that both numbers of a pair lie in
// the same lane and nothing crosses lanes but the sum of squares:
//   halves:    lane i < rot / 8 holds channels 4i .. 4i + 3 and rot / 2 + 4i .. + 3,
//   adjacent:  lane i holds 8i .. 8i + 7;  lanes behind rot / 8 hold 8i .. 8i + 7 and pass them through.
// Either way a lane's four pairs are 4i .. 4i + 3 of the rotation's rot / 2.
//
//   y = x * (1 / sqrt(mean x^2 + eps)) * w;   a' = a cos - b sin,  b' = b cos + a sin
//
// The sum of squares and its root are taken in fp64: the squares of 16-bit numbers are exact there and sums
// of up to 128 of them all but exact, so the factor does not depend on the order of the additions.  The
// rest is fp32, every product and sum rounded by itself (no contraction), and the row is rounded to 16 bits
// once, at the end.  So a row has the same bits whatever kernel works it out, and what the append kernels
// quantise is what rotate_rows_kernel would have written.
#pragma once
#include "ts_device.h"

namespace ts {

constexpr int kRotaryThreads = 256;
constexpr int kMaxAxes = 4;

struct RotaryParams {
  const float* table;         // [n_pos][rot]: rot / 2 cosines, rot / 2 sines (null: no rotation)
  const int32_t* positions;   // [axes][T] (null: the place in the sequence)
  const float* q_norm;        // [D] (null: no norm)
  const float* k_norm;
  int rot, adjacent, axes, n_pos, T;
  float eps;
  uint32_t axis_bits[4];      // two bits a pair: the axis it turns by
};

template <int N>
__device__ __forceinline__ float group_max_f32(float v) {
  static_assert(N == 8 || N == 16, "group of 8 or 16 lanes");
  auto take = [](float x, float y) { return fmaxf(x, y); };
  auto move = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if (N == 16) v = take(v, move(v, std::integral_constant<int, kDppMirror>{}));
  v = take(v, move(v, std::integral_constant<int, kDppHalfMirror>{}));
  v = take(v, move(v, std::integral_constant<int, kDppXor2>{}));
  v = take(v, move(v, std::integral_constant<int, kDppXor1>{}));
  return v;
}

// Where a lane's channels lie in a row, and the angles of its pairs for one token.
template <int D>
struct RowLanes {
  static constexpr int kLanes = D / 8;
  int c0, c1;     // first channel of either chunk of four
  bool turns;
  __device__ __forceinline__ RowLanes(const RotaryParams& p, int lane_in_row) {
    turns = lane_in_row < p.rot / 8;
    const bool halves = turns && !p.adjacent;
    c0 = halves ? 4 * lane_in_row : 8 * lane_in_row;
    c1 = halves ? p.rot / 2 + 4 * lane_in_row : 8 * lane_in_row + 4;
  }
};

struct Angles {
  float c[4], s[4];
};

// position_of(axis): the token's position on an axis.  Rows of the table are never read past its ends.
template <typename PositionOf>
__device__ __forceinline__ void load_angles(const RotaryParams& p, int lane_in_row, bool turns,
                                            PositionOf position_of, Angles& a) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { a.c[i] = 1.f; a.s[i] = 0.f; }
  if (!turns) return;
  const int pair = 4 * lane_in_row, half = p.rot / 2;
  if (p.axes == 1) {
    const int pos = min(max(position_of(0), 0), p.n_pos - 1);
    const float* row = p.table + (size_t)pos * p.rot + pair;
    const float4 c = *reinterpret_cast<const float4*>(row), s = *reinterpret_cast<const float4*>(row + half);
    a.c[0] = c.x; a.c[1] = c.y; a.c[2] = c.z; a.c[3] = c.w;
    a.s[0] = s.x; a.s[1] = s.y; a.s[2] = s.z; a.s[3] = s.w;
    return;
  }
  const uint32_t w = p.axis_bits[0] * (pair < 16) + p.axis_bits[1] * (pair >= 16 && pair < 32) +
                     p.axis_bits[2] * (pair >= 32 && pair < 48) + p.axis_bits[3] * (pair >= 48);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int axis = (w >> (2 * ((pair + i) & 15))) & 3;
    const int pos = min(max(position_of(axis), 0), p.n_pos - 1);
    const float* row = p.table + (size_t)pos * p.rot + pair + i;
    a.c[i] = row[0];
    a.s[i] = row[half];
  }
}

struct Norm {
  float w[8];
  bool on;
};

__device__ __forceinline__ void load_norm(const float* w, int c0, int c1, Norm& n) {
  n.on = w != nullptr;
#pragma unroll
  for (int i = 0; i < 8; ++i) n.w[i] = 1.f;
  if (!n.on) return;
  const float4 a = *reinterpret_cast<const float4*>(w + c0), b = *reinterpret_cast<const float4*>(w + c1);
  n.w[0] = a.x; n.w[1] = a.y; n.w[2] = a.z; n.w[3] = a.w;
  n.w[4] = b.x; n.w[5] = b.y; n.w[6] = b.z; n.w[7] = b.w;
}

// Two fp32 numbers as 16-bit ones, to nearest even.
template <bool kHalf>
__device__ __forceinline__ uint32_t pack_elems(float x, float y) {
  if (kHalf) return (uint32_t)f32_to_half(x) | (uint32_t)f32_to_half(y) << 16;
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// 1 / sqrt(m): the instruction's estimate y (good to 2^-22 or better), and with e = 1 - m y^2 the series
// y (1 + e / 2 + 3 e^2 / 8), which leaves the last bits of fp64.  (m infinite or 0: y itself, and e is no number.)
__device__ __forceinline__ double inverse_root(double m) {
  const double y = __builtin_amdgcn_rsq(m), e = fma(-m * y, y, 1.0);
  return e == e ? fma(y * e, fma(0.375, e, 0.5), y) : y;
}

// One row, eight channels a lane: normed, rotated and rounded to 16 bits.  All lanes of the row take part.
template <int D, bool kHalf>
__device__ __forceinline__ void rotate_row(const RotaryParams& p, bool turns, const Norm& n, const Angles& t,
                                           uint2& a, uint2& b) {
#pragma clang fp contract(off)
  float y[8] = {elem_lo<kHalf>(a.x), elem_hi<kHalf>(a.x), elem_lo<kHalf>(a.y), elem_hi<kHalf>(a.y),
                elem_lo<kHalf>(b.x), elem_hi<kHalf>(b.x), elem_lo<kHalf>(b.y), elem_hi<kHalf>(b.y)};
  if (n.on) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma((double)y[i], (double)y[i], sum);
    sum = group_sum1_f64<D / 8>(sum);
    const float r = (float)inverse_root(sum * (1.0 / D) + (double)p.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (y[i] * r) * n.w[i];
  }
  if (turns) {
    float z[8];
    if (p.adjacent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[2 * i] = y[2 * i] * t.c[i] - y[2 * i + 1] * t.s[i];
        z[2 * i + 1] = y[2 * i + 1] * t.c[i] + y[2 * i] * t.s[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[i] = y[i] * t.c[i] - y[4 + i] * t.s[i];
        z[4 + i] = y[4 + i] * t.c[i] + y[i] * t.s[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = z[i];
  }
  if (n.on || turns) {   // (what neither norm nor rotation touches keeps its bits)
    a = make_uint2(pack_elems<kHalf>(y[0], y[1]), pack_elems<kHalf>(y[2], y[3]));
    b = make_uint2(pack_elems<kHalf>(y[4], y[5]), pack_elems<kHalf>(y[6], y[7]));
  }
}

// Half of a lane's part of a result row, as a store that the caches need not keep.  The rows of a long prompt
// are read back, if at all, after they have left the caches, and plain stores push out what is still being
// read: 16.5 -> 14.9 us (64 channels, 77.6 MB), 26.4 -> 21.8 (128, 104.4 MB); in the append of prompts to a 4-bit
// cache (145.4 MB) 42.5 -> 37.5.  Loads of that kind lose as much again.
__device__ __forceinline__ void stream_row(uint16_t* dst, uint2 v) {
  __builtin_nontemporal_store(__builtin_bit_cast(stream_u2, v), reinterpret_cast<stream_u2*>(dst));
}

struct RotateParams {
  RotaryParams r;
  const uint16_t *q, *k;         // either may be null
  uint16_t *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;   // elements between tokens
  int Hq, Hkv, T;
  int tokens_per_wg, rows_per_wg;   // a workgroup's tokens (a power of two) and heads
};

// grid (tokens / tokens_per_wg, heads / rows_per_wg).  A row's lanes stay with their token, whose angles
// they hold, and take its heads in turn, kRowsAhead rows on their way at a time (two: 22.4 us where four take
// 21.6).  Memory-bound: every element is read and written once.  8191 tokens of 36 heads, 64 channels, 77.6 MB: 15.0
// to 15.5 us, 5.1 TB/s; 5003 of 40, 128 channels, three axes, 104.4 MB: 21.6 us, 4.8 TB/s; a copy of 2 GiB reaches 4.9.
// One token: 2.8 us, a launch.
constexpr int kRowsAhead = 4;
template <int D, bool kHalf>
__global__ __launch_bounds__(kRotaryThreads) void rotate_rows_kernel(RotateParams p) {
  constexpr int LPR = D / 8, NG = kRotaryThreads / LPR;
  const int group = threadIdx.x / LPR, li = threadIdx.x % LPR;
  const int t = blockIdx.x * p.tokens_per_wg + group % p.tokens_per_wg, step = NG / p.tokens_per_wg;
  if (t >= p.T) return;      // (whole groups of lanes; there is no barrier)
  const RowLanes<D> lanes(p.r, li);
  const int rows = p.Hq + p.Hkv, end = min(rows, (int)(blockIdx.y + 1) * p.rows_per_wg);
  const int first = blockIdx.y * p.rows_per_wg + group / p.tokens_per_wg;
  const uint16_t *q = p.q + t * p.q_stride, *k = p.k + t * p.k_stride - p.Hq * D;
  uint16_t *q_out = p.q_out + t * p.q_out_stride, *k_out = p.k_out + t * p.k_out_stride - p.Hq * D;
  uint2 a[kRowsAhead], b[kRowsAhead];
  auto fetch = [&](int row0) {
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int row = row0 + i * step;
      if (row < end) {
        const uint16_t* src = (row < p.Hq ? q : k) + row * D;
        a[i] = *reinterpret_cast<const uint2*>(src + lanes.c0);
        b[i] = *reinterpret_cast<const uint2*>(src + lanes.c1);
      }
    }
  };
  fetch(first);
  Angles ang;
  load_angles(p.r, li, lanes.turns, [&](int axis) { return p.r.positions[(size_t)axis * p.r.T + t]; }, ang);
  Norm qn, kn;
  load_norm(p.r.q_norm, lanes.c0, lanes.c1, qn);
  load_norm(p.r.k_norm, lanes.c0, lanes.c1, kn);
  for (int row0 = first; row0 < end;) {
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int row = row0 + i * step;
      if (row < end) {
        Norm n;
        n.on = row < p.Hq ? qn.on : kn.on;
#pragma unroll
        for (int c = 0; c < 8; ++c) n.w[c] = row < p.Hq ? qn.w[c] : kn.w[c];
        rotate_row<D, kHalf>(p.r, lanes.turns, n, ang, a[i], b[i]);
        uint16_t* dst = (row < p.Hq ? q_out : k_out) + row * D;
        stream_row(dst + lanes.c0, a[i]);
        stream_row(dst + lanes.c1, b[i]);
      }
    }
    row0 += kRowsAhead * step;
    fetch(row0);
  }
}

}  // namespace ts
