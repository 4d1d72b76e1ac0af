// Appending tokens to the paged cache: any number of tokens for each sequence, keys normed and rotated on
// the way (ts_rotary.h), values transposed into their channel-major tiles, page boxes opened or widened, the
// queries of the same tokens rotated in the same launch.
//
// With offsets a workgroup takes the tokens that fall into ONE page of one sequence, for one KV head and the
// query heads that share it.  So a page's tile and its box have one writer, what the page held already needs
// no atomics, and the box of a new page is worked out from the tokens in hand.  Keys go from registers to
// their slots, the values through LDS.  One token for each sequence goes row by row instead.
#pragma once
#include <float.h>

#include "ts_meta.h"
#include "ts_rotary.h"

namespace ts {

// Formats of the pool as the kernels here tell them apart (TS_KV_*; the values are the interface's).
constexpr int kPoolBf16 = 0, kPoolInt8 = 1, kPoolFp16 = 2, kPoolFp4 = 3;

// ---------------------------------------------------------------------------
// The 4-bit number: e2m1, magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6 for the codes 0 to 7, sign in bit 3.  A
// row's scale is max |x| / 6 rounded up to bf16 (1 for a zero row), so nothing saturates and code * scale
// has at most ten significant bits: exact in fp32.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float fp4_row_scale(float amax) {
  const uint32_t b = __float_as_uint(__fdiv_rn(amax, 6.0f));
  return amax > 0.f ? __uint_as_float((b + 0xffffu) & 0xffff0000u) : 1.0f;
}
typedef float float2_t __attribute__((ext_vector_type(2)));
// The codes of eight numbers of a row, four bits each: the nearest, ties to the even code, no negative zero.  The
// quotient is the reciprocal's product corrected by its remainder: exact where x / scale is a number's border
// (a tie), and elsewhere off by far less than the 2^-11 that eight-bit numbers keep away from one.  kFar: rows of
// very small or large scale are moved to the middle of the range first (exactly).
template <bool kFar>
__device__ __forceinline__ uint32_t fp4_codes(const float (&x)[8], float scale) {
  const float f = !kFar ? 1.0f : scale < 0x1p-60f ? 0x1p100f : scale > 0x1p60f ? 0x1p-100f : 1.0f;
  const float s = kFar ? scale * f : scale, r = __builtin_amdgcn_rcpf(s);
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = kFar ? x[i] * f : x[i], q = y * r;
    z[i] = fmaf(fmaf(-q, s, y), r, q);
  }
  uint32_t w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, z[0], z[1], 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, z[2], z[3], 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, z[4], z[5], 1.0f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, z[6], z[7], 1.0f, 3);
  const uint32_t m = w & 0x77777777u;
  return m | (w & (m + 0x77777777u) & 0x88888888u);   // signs of the numbers that are not zero
}
// The numbers of eight codes, times a factor.
__device__ __forceinline__ void fp4_numbers(uint32_t w, float scale, float (&x)[8]) {
  const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
  const float2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
  x[0] = a[0] * scale; x[1] = a[1] * scale; x[2] = b[0] * scale; x[3] = b[1] * scale;
  x[4] = c[0] * scale; x[5] = c[1] * scale; x[6] = d[0] * scale; x[7] = d[1] * scale;
}
// An exactly known fp32 value rounded to bf16 on one side of it.
__device__ __forceinline__ uint32_t bf16_outwards(float f, bool up) {
  const uint32_t b = __float_as_uint(f);
  return (b >> 16) + (((b & 0xffffu) != 0u && ((b >> 31) != 0u) != up) ? 1u : 0u);
}

// Where a (page, head) block of the 4-bit cache keeps what: offsets in bytes, S tokens of D channels.
//   keys    [S][D / 2]                  two channels a byte, the even one in the low half
//   values  [S / 8][D / 64][16][4][4]   eight tokens of a channel in four bytes, the even token in the low
//                                       half; channel 16 * cb + r is word [cb / 4][r][cb % 4]
//   scales  bf16 [S] of the keys, then [S] of the values
// The lane that multiplies tokens 8o .. 8o + 7 of the channels r, 16 + r, ... finds them in 16-byte pieces,
// and sixteen such lanes take 256 contiguous bytes in one load.
template <int D>
struct Fp4Block {
  __host__ __device__ static constexpr int bytes(int S) { return S * (D + 4); }
  __host__ __device__ static constexpr int values(int S) { return S * (D / 2); }
  __host__ __device__ static constexpr int key_scales(int S) { return S * D; }
  __host__ __device__ static constexpr int value_scales(int S) { return S * D + 2 * S; }
  // word of channel c within its octet of tokens
  __device__ __forceinline__ static int word(int c) { return ((c >> 6) * 16 + (c & 15)) * 4 + ((c >> 4) & 3); }
  __device__ __forceinline__ static int channel(int word) { return (word >> 6) * 64 + (word & 3) * 16 + ((word >> 2) & 15); }
};

struct AppendParams {
  RotaryParams r;
  const uint16_t *q, *k, *v;          // q may be null
  uint16_t* q_out;
  long long q_stride, k_stride, v_stride, q_out_stride;   // elements between tokens
  const int32_t* cu;                  // [B + 1] first token of each sequence (append_rows_kernel)
  const int32_t* seq_lens;
  const int32_t* block_table;
  unsigned char *k_pool, *v_pool;     // 4 bits: the blocks; v_pool null: boxes only
  float *k_scale, *v_scale;           // INT8
  uint16_t *page_min, *page_max;
  int T, B, Hq, Hkv, G, S, Pmax, n_phys;
  long long tile_stride;              // bytes between consecutive (page, head) tiles
  int lens_after;                     // seq_lens count the new tokens already
};

template <int FMT, int D>
struct AppendLds {
  typedef typename std::conditional<FMT == kPoolInt8 || FMT == kPoolFp4, uint8_t, uint16_t>::type Elem;
  static constexpr bool kWide = sizeof(Elem) == 2;
  static constexpr int kRow = D + 8;   // elements of a staged row
  // partial boxes: of each wave, or with 16 bits of as many threads as there are for each pair of channels
  static constexpr int kParts = kWide ? 2 * kRotaryThreads / D : kRotaryThreads / kWave;
  __host__ __device__ static constexpr size_t bytes(int S) {
    return (kWide ? 2 : 1) * (size_t)S * kRow * sizeof(Elem) + 2 * (size_t)kParts * D * 4;
  }
};

// Minimum and maximum as the instruction has them: a NaN gives way to the other number.  (fminf and fmaxf
// quieten their operands with an instruction each first.)
__device__ __forceinline__ float raw_min(float a, float b) {
  float r;
  asm("v_min_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float raw_max(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// A row as the cache stores it: 16 bits (two chunks of four), eight int8 codes, or eight 4-bit codes.
struct StoredRow {
  uint2 a, b;
  float scale;
};
template <int FMT, int D>
__device__ __forceinline__ StoredRow store_form(uint2 x, uint2 y) {
  StoredRow s;
  s.a = x;
  s.b = y;
  s.scale = 1.f;
  if constexpr (FMT == kPoolInt8 || FMT == kPoolFp4) {
    float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y),
                  bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = raw_max(amax, fabsf(f[i]));
    amax = group_max_f32<D / 8>(amax);
    if constexpr (FMT == kPoolInt8) {
      s.scale = i8_row_scale(amax);
      uint32_t c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = (uint32_t)i8_code(f[i], s.scale) & 0xffu;
      s.a.x = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
      s.b.x = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
    } else {
      bool odd = false;      // (a NaN is no maximum: it is looked for by itself)
#pragma unroll
      for (int i = 0; i < 8; ++i) odd |= !(fabsf(f[i]) <= FLT_MAX);
      if (__any(odd)) {      // infinities are the largest number of their row's scale, NaN is 0
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] == f[i] ? fminf(fmaxf(f[i], -FLT_MAX), FLT_MAX) : 0.f;
        amax = fminf(amax, FLT_MAX);
      }
      s.scale = fp4_row_scale(amax);
      s.a.x = __any(s.scale < 0x1p-60f || s.scale > 0x1p60f) ? fp4_codes<true>(f, s.scale) : fp4_codes<false>(f, s.scale);
    }
  }
  return s;
}
// Its numbers as fp32, the smaller and the larger bf16 neighbour where fp32 does not hold them (INT8).
template <int FMT>
__device__ __forceinline__ void stored_numbers(const StoredRow& s, float (&lo)[8], float (&hi)[8]) {
  if constexpr (FMT == kPoolFp4) {
    fp4_numbers(s.a.x, s.scale, lo);
#pragma unroll
    for (int i = 0; i < 8; ++i) hi[i] = lo[i];
  } else if constexpr (FMT == kPoolInt8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double x = (double)(int8_t)((i < 4 ? s.a.x : s.b.x) >> (8 * (i & 3))) * (double)s.scale;
      lo[i] = bf16_to_f32(bf16_directed(x, false));
      hi[i] = bf16_to_f32(bf16_directed(x, true));
    }
  } else {
    constexpr bool kHalf = FMT == kPoolFp16;
    const uint32_t w[4] = {s.a.x, s.a.y, s.b.x, s.b.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[2 * i] = hi[2 * i] = elem_lo<kHalf>(w[i]);
      lo[2 * i + 1] = hi[2 * i + 1] = elem_hi<kHalf>(w[i]);
    }
  }
}
// A key's chunks (channels c0 and c1 on) into its slot of the tile, and its scale.
template <int FMT, int D>
__device__ __forceinline__ void store_key(const AppendParams& p, unsigned char* tile, size_t scale_row, int slot, int c0, int c1,
                                          int li, const StoredRow& s) {
  if constexpr (FMT == kPoolFp4) {
    unsigned char* dst = tile + slot * (D / 2);
    *reinterpret_cast<uint16_t*>(dst + c0 / 2) = (uint16_t)s.a.x;
    *reinterpret_cast<uint16_t*>(dst + c1 / 2) = (uint16_t)(s.a.x >> 16);
    if (li == 0)
      *reinterpret_cast<uint16_t*>(tile + Fp4Block<D>::key_scales(p.S) + 2 * slot) = (uint16_t)(__float_as_uint(s.scale) >> 16);
  } else if constexpr (FMT == kPoolInt8) {
    *reinterpret_cast<uint32_t*>(tile + slot * D + c0) = s.a.x;
    *reinterpret_cast<uint32_t*>(tile + slot * D + c1) = s.b.x;
    if (li == 0) p.k_scale[scale_row + slot] = s.scale;
  } else {
    uint16_t* dst = reinterpret_cast<uint16_t*>(tile) + slot * D;
    *reinterpret_cast<uint2*>(dst + c0) = s.a;
    *reinterpret_cast<uint2*>(dst + c1) = s.b;
  }
}
template <int FMT, int D>
__device__ __forceinline__ void store_value_scale(const AppendParams& p, unsigned char* block, size_t scale_row, int slot, float scale) {
  if constexpr (FMT == kPoolFp4)
    *reinterpret_cast<uint16_t*>(block + Fp4Block<D>::value_scales(p.S) + 2 * slot) = (uint16_t)(__float_as_uint(scale) >> 16);
  else if constexpr (FMT == kPoolInt8) p.v_scale[scale_row + slot] = scale;
}
// fp32 numbers known exactly, or (16 bits, INT8) 16-bit numbers already, as the box holds them.
template <int FMT>
__device__ __forceinline__ uint16_t box_number(float f, bool up) {
  if constexpr (FMT == kPoolFp4) return (uint16_t)bf16_outwards(f, up);
  else if constexpr (FMT == kPoolFp16) return f32_to_half(f);
  else return (uint16_t)(__float_as_uint(f) >> 16);
}
// Where the page `phys` keeps the head's keys (4 bits: the block), its values and its scales.
template <int FMT, int D>
struct PageTiles {
  unsigned char *k, *v;
  size_t scale_row;
  __device__ __forceinline__ PageTiles(const AppendParams& p, int phys, int h) {
    const size_t id = (size_t)phys * p.Hkv + h;
    k = p.k_pool + id * (size_t)p.tile_stride;
    v = FMT == kPoolFp4 ? k + Fp4Block<D>::values(p.S) : p.v_pool + id * (size_t)p.tile_stride;
    scale_row = id * (size_t)p.S;
  }
};

// One token for each sequence: every row by itself, eight or sixteen lanes for each, no LDS and no barrier.
// A key's lanes widen or open its page's box in the channels they hold; a value's lanes put its eight
// numbers into their places in the channel-major tile.  Bound by a chain of trips to memory (length,
// block-table entry and angles, box); the row itself is asked for ahead of them.  64 sequences, 32 KV and 32
// query heads of 128 channels in bf16, 4.2 MB: 5.8 us; one sequence, 4 bits: 4.3.
// grid (sequences, row groups): rows 0 .. Hkv - 1 keys, then values, then queries.
template <int FMT, int D>
__global__ __launch_bounds__(kRotaryThreads) void append_token_rows_kernel(AppendParams p) {
  constexpr bool kHalf = FMT == kPoolFp16;
  constexpr int LPR = D / 8, NG = kRotaryThreads / LPR;
  const int b = blockIdx.x, li = threadIdx.x % LPR, row = blockIdx.y * NG + threadIdx.x / LPR;
  const int rows = 2 * p.Hkv + (p.q != nullptr ? p.Hq : 0);
  if (row >= rows) return;
  const bool is_k = row < p.Hkv, is_v = !is_k && row < 2 * p.Hkv, is_q = row >= 2 * p.Hkv;
  const int h = is_q ? row - 2 * p.Hkv : is_v ? row - p.Hkv : row;
  const RowLanes<D> lanes(p.r, li);
  const int c0 = is_v ? 8 * li : lanes.c0, c1 = is_v ? 8 * li + 4 : lanes.c1;
  if (is_v && p.v_pool == nullptr) return;       // boxes only: there are no values
  const uint16_t* src = (is_k ? p.k + b * p.k_stride : is_v ? p.v + b * p.v_stride : p.q + b * p.q_stride) + h * D;
  uint2 x = *reinterpret_cast<const uint2*>(src + c0), y = *reinterpret_cast<const uint2*>(src + c1);
  const int sh = __builtin_ctz(p.S);
  const int len = p.seq_lens[b] - p.lens_after;
  if (len < 0) return;
  const int j = len >> sh, slot = len & (p.S - 1);
  const bool fits = j < p.Pmax;
  const int phys = fits ? p.block_table[(size_t)b * p.Pmax + j] : -1;
  if (!is_v) {
    Angles ang;
    load_angles(p.r, li, lanes.turns, [&](int axis) { return p.r.positions ? p.r.positions[(size_t)axis * p.r.T + b] : len; },
                ang);
    Norm n;
    load_norm(is_q ? p.r.q_norm : p.r.k_norm, lanes.c0, lanes.c1, n);
    rotate_row<D, kHalf>(p.r, lanes.turns, n, ang, x, y);
  }
  if (is_q) {
    uint16_t* dst = p.q_out + b * p.q_out_stride + h * D;
    *reinterpret_cast<uint2*>(dst + c0) = x;
    *reinterpret_cast<uint2*>(dst + c1) = y;
    return;
  }
  const bool store = p.v_pool != nullptr && phys >= 0 && phys < p.n_phys;
  if (!fits || (p.v_pool != nullptr && !store)) return;
  const StoredRow s = store_form<FMT, D>(x, y);
  const PageTiles<FMT, D> tile(p, store ? phys : 0, h);
  if (is_v) {
    if constexpr (FMT == kPoolFp4) {
      unsigned char* oct = tile.v + (slot >> 3) * (4 * D) + ((slot & 7) >> 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        unsigned char* dst = oct + 4 * Fp4Block<D>::word(8 * li + i);
        const uint32_t code = (s.a.x >> (4 * i)) & 15u, was = *dst;
        *dst = (unsigned char)((slot & 1) ? (was & 15u) | code << 4 : (was & 0xf0u) | code);
      }
    } else if constexpr (FMT == kPoolInt8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        tile.v[(size_t)(8 * li + i) * p.S + slot] = (uint8_t)((i < 4 ? s.a.x : s.b.x) >> (8 * (i & 3)));
    } else {
      const uint32_t w[4] = {s.a.x, s.a.y, s.b.x, s.b.y};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        reinterpret_cast<uint16_t*>(tile.v)[(size_t)(8 * li + i) * p.S + slot] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
    if (li == 0) store_value_scale<FMT, D>(p, tile.k, tile.scale_row, slot, s.scale);
    return;
  }
  if (p.v_pool != nullptr) store_key<FMT, D>(p, tile.k, tile.scale_row, slot, c0, c1, li, s);
  float lo[8], hi[8];
  stored_numbers<FMT>(s, lo, hi);
  const size_t at = (((size_t)b * p.Hkv + h) * p.Pmax + j) * D;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int c = half ? c1 : c0;
    uint2* lo_at = reinterpret_cast<uint2*>(p.page_min + at + c);
    uint2* hi_at = reinterpret_cast<uint2*>(p.page_max + at + c);
    if (slot != 0) {
      const uint2 l = *lo_at, u = *hi_at;
      const uint32_t lw[2] = {l.x, l.y}, uw[2] = {u.x, u.y};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lb = lw[i >> 1], ub = uw[i >> 1];
        lo[4 * half + i] = fminf(lo[4 * half + i], i & 1 ? elem_hi<kHalf>(lb) : elem_lo<kHalf>(lb));
        hi[4 * half + i] = fmaxf(hi[4 * half + i], i & 1 ? elem_hi<kHalf>(ub) : elem_lo<kHalf>(ub));
      }
    }
    uint32_t l[4], u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      l[i] = box_number<FMT>(lo[4 * half + i], false);
      u[i] = box_number<FMT>(hi[4 * half + i], true);
    }
    *lo_at = make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
    *hi_at = make_uint2(u[0] | u[1] << 16, u[2] | u[3] << 16);
  }
}

// Sequence b's new tokens begin at row first_row(b), and its pages are the tasks from first_task(b) on: n tokens touch at most
// n / S + 2 pages (rounded down), so the sequences' tasks do not overlap whatever their lengths.
__device__ __forceinline__ int first_row(const AppendParams& p, int b) { return min(max(p.cu[b], 0), p.T); }
__device__ __forceinline__ int first_task(int row, int sh, int b) { return (row >> sh) + 2 * b; }
// The last sequence whose tasks begin at or before `task`, sixty-four looked at at a time: one trip to memory for up to
// 64 sequences, two for 4096.  (Their pages counted and numbered through took a trip for every 64: 1024 sequences of
// one token 93 us.)
__device__ __forceinline__ int sequence_of(const AppendParams& p, int sh, int task) {
  int b = 0;
  for (int n = p.B; n > 1;) {
    const int step = (n + kWave - 1) / kWave, i = lane_id() * step;
    const uint64_t begun = __ballot(i < n && first_task(first_row(p, b + min(i, n - 1)), sh, b + i) <= task);
    const int skip = max((int)__builtin_popcountll(begun) - 1, 0) * step;
    b += skip;
    n = min(step, n - skip);
  }
  return uniform(b);
}

// Minimum or maximum of a value over the lanes of the wave that hold the same channels.
template <int LPR, bool kMax>
__device__ __forceinline__ float over_groups(float v) {
  auto take = [](float x, float y) { return kMax ? raw_max(x, y) : raw_min(x, y); };
  if (LPR == 8)
    v = take(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), kDppRowRor8, 0xf, 0xf, true)));
  uint2s_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = take(__uint_as_float(r.x), __uint_as_float(r.y));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return take(__uint_as_float(r.x), __uint_as_float(r.y));
}

// grid (Hkv, touched pages or more): the heads of a page one behind the other, as they lie in the projection's rows
// and in the pool (bf16 prompts 73.5 us; the pages of a head one behind the other 81.5).  A token's key, value and queries are dealt to as many groups of
// lanes as the workgroup has for each token, the rows asked for ahead of the lookups.  Half of the time goes to
// the vector unit (some hundred instructions a row), so the box is worked out where that takes the fewest: with
// 16 bits from the keys in LDS, two channels a thread; quantised, from the numbers that the lanes hold anyway, over
// the wave's groups and then, in LDS, over the waves.
// Four waves on a SIMD: five and six spill (twice and three times the time).  Two query rows on their way at a time:
// one and three take 8 % longer; the queries in workgroups of their own 15 %.
// Seven prompts of 14 400 tokens in all, 32 and 8 heads of 128 channels, bf16, 354.9 MB: 73.5 us, 4.8 TB/s; five of
// 6 700, into 4 bits, 145.4 MB: 37.4 us, 3.9 TB/s, the quantiser's instructions on top.
template <int FMT, int D>
__global__ __launch_bounds__(kRotaryThreads, 4) void append_rows_kernel(AppendParams p) {
  constexpr bool kHalf = FMT == kPoolFp16;
  constexpr int LPR = D / 8, NG = kRotaryThreads / LPR;
  typedef AppendLds<FMT, D> Lds;
  typedef typename Lds::Elem Elem;
  extern __shared__ __align__(16) unsigned char smem[];
  Elem* vs = reinterpret_cast<Elem*>(smem);                                                  // [S][kRow]
  Elem* ks = Lds::kWide ? vs + (size_t)p.S * Lds::kRow : vs;                                 // 16 bits: [S][kRow]
  float* box = reinterpret_cast<float*>(ks + (size_t)p.S * Lds::kRow);                       // [2][parts][D]
  const int sh = __builtin_ctz(p.S), h = blockIdx.x, tid = threadIdx.x;
  const int task = blockIdx.z * gridDim.y + blockIdx.y, b = sequence_of(p, sh, task);
  const int c0 = first_row(p, b), n = uniform(first_row(p, b + 1) - c0);
  const int len = uniform(p.seq_lens[b] - (p.lens_after ? p.cu[b + 1] - p.cu[b] : 0));
  const int page = uniform(task - first_task(c0, sh, b)), j = (len >> sh) + page;
  if (n <= 0 || len < 0 || page < 0 || j > (len + n - 1) >> sh) return;      // (a task without a page, or no such length)
  const int p0 = max(j << sh, len), p1 = min((j + 1) << sh, len + n);   // positions of this page's new tokens
  const int ntok = uniform(p1 - p0), slot0 = p0 - (j << sh), tok0 = c0 + p0 - len;
  const bool fits = (long long)len + n <= (long long)p.Pmax << sh;
  const int phys = uniform(fits ? p.block_table[(size_t)b * p.Pmax + j] : -1);
  const bool store = phys >= 0 && phys < p.n_phys;
  const PageTiles<FMT, D> tile(p, store ? phys : 0, h);
  int tp = 1;
  while (tp < ntok && tp < NG) tp <<= 1;
  const int group = tid / LPR, li = tid % LPR, part = group / tp, step = NG / tp;
  const RowLanes<D> lanes(p.r, li);
  Norm qn, kn;
  load_norm(p.r.q_norm, lanes.c0, lanes.c1, qn);
  load_norm(p.r.k_norm, lanes.c0, lanes.c1, kn);
  const bool has_k = store && part == 0, has_v = store && part == (step > 1 ? 1 : 0);
  const int G = p.q != nullptr ? p.G : 0, rounds = (G + step - 1) / step;
  const int g0 = step > 2 ? (part + step - 2) % step : part;          // queries go to the groups behind first
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
  for (int i0 = group % tp; i0 < ntok; i0 += tp) {
    const int tok = tok0 + i0, slot = slot0 + i0;
    constexpr int kAhead = 2;
    const uint16_t* q_src = p.q + tok * p.q_stride + (size_t)h * p.G * D;
    uint2 qa[kAhead], qb[kAhead], ka, kb, va, vb;
    // (the number of rounds is the same for all: a group without a row in the last one fetches another's)
    auto fetch = [&](int round) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (round + i < rounds) {
          const uint16_t* src = q_src + min(g0 + (round + i) * step, G - 1) * D;
          qa[i] = *reinterpret_cast<const uint2*>(src + lanes.c0);
          qb[i] = *reinterpret_cast<const uint2*>(src + lanes.c1);
        }
    };
    if (has_k) {
      const uint16_t* src = p.k + tok * p.k_stride + h * D;
      ka = *reinterpret_cast<const uint2*>(src + lanes.c0);
      kb = *reinterpret_cast<const uint2*>(src + lanes.c1);
    }
    if (has_v) {
      const uint16_t* src = p.v + tok * p.v_stride + h * D + 8 * li;
      va = *reinterpret_cast<const uint2*>(src);
      vb = *reinterpret_cast<const uint2*>(src + 4);
    }
    fetch(0);
    Angles ang;
    load_angles(p.r, li, lanes.turns,
                [&](int axis) { return p.r.positions ? p.r.positions[(size_t)axis * p.r.T + tok] : p0 + i0; }, ang);
    if (has_k) {
      rotate_row<D, kHalf>(p.r, lanes.turns, kn, ang, ka, kb);
      const StoredRow s = store_form<FMT, D>(ka, kb);
      store_key<FMT, D>(p, tile.k, tile.scale_row, slot, lanes.c0, lanes.c1, li, s);
      if constexpr (Lds::kWide) {
        *reinterpret_cast<uint2*>(ks + slot * Lds::kRow + lanes.c0) = s.a;
        *reinterpret_cast<uint2*>(ks + slot * Lds::kRow + lanes.c1) = s.b;
      } else {
        float l[8], u[8];
        stored_numbers<FMT>(s, l, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          lo[i] = raw_min(lo[i], l[i]);
          hi[i] = raw_max(hi[i], u[i]);
        }
      }
    }
    if (has_v) {
      const StoredRow s = store_form<FMT, D>(va, vb);
      Elem* stage = vs + slot * Lds::kRow + 8 * li;
      if constexpr (FMT == kPoolFp4) {
        const uint32_t even = s.a.x & 0x0f0f0f0fu, odd = (s.a.x >> 4) & 0x0f0f0f0fu;     // a byte a code, in order
        *reinterpret_cast<uint2*>(stage) = make_uint2(__builtin_amdgcn_perm(odd, even, 0x05010400u),
                                                      __builtin_amdgcn_perm(odd, even, 0x07030602u));
      } else if constexpr (FMT == kPoolInt8) {
        *reinterpret_cast<uint2*>(stage) = make_uint2(s.a.x, s.b.x);
      } else {
        *reinterpret_cast<uint2*>(stage) = s.a;
        *reinterpret_cast<uint2*>(stage + 4) = s.b;
      }
      if (li == 0) store_value_scale<FMT, D>(p, tile.k, tile.scale_row, slot, s.scale);
    }
    uint16_t* q_dst = p.q_out + tok * p.q_out_stride + (size_t)h * p.G * D;
    for (int round = 0; round < rounds;) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (round + i < rounds) {
          rotate_row<D, kHalf>(p.r, lanes.turns, qn, ang, qa[i], qb[i]);
          const int g = g0 + (round + i) * step;
          if (g < G) {
            stream_row(q_dst + g * D + lanes.c0, qa[i]);
            stream_row(q_dst + g * D + lanes.c1, qb[i]);
          }
        }
      round += kAhead;
      fetch(round);
    }
  }
  if (!store) return;
  const int slot1 = slot0 + ntok;
  if constexpr (Lds::kWide) {
    __syncthreads();
    const int pair = tid % (D / 2), part = tid / (D / 2);
    float l0 = INFINITY, l1 = INFINITY, u0 = -INFINITY, u1 = -INFINITY;
    for (int s = slot0 + part; s < slot1; s += Lds::kParts) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(ks + s * Lds::kRow + 2 * pair);
      const float x = elem_lo<kHalf>(w), y = elem_hi<kHalf>(w);
      l0 = raw_min(l0, x); u0 = raw_max(u0, x);
      l1 = raw_min(l1, y); u1 = raw_max(u1, y);
    }
    *reinterpret_cast<float2*>(box + part * D + 2 * pair) = make_float2(l0, l1);
    *reinterpret_cast<float2*>(box + (Lds::kParts + part) * D + 2 * pair) = make_float2(u0, u1);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = over_groups<LPR, false>(lo[i]);
      hi[i] = over_groups<LPR, true>(hi[i]);
    }
    if (lane_id() < LPR) {
      float* mine = box + wave_id() * D;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mine[lanes.c0 + i] = lo[i];
        mine[lanes.c1 + i] = lo[4 + i];
        mine[Lds::kParts * D + lanes.c0 + i] = hi[i];
        mine[Lds::kParts * D + lanes.c1 + i] = hi[4 + i];
      }
    }
  }
  __syncthreads();
  if (tid < D) {
    float l = box[tid], u = box[Lds::kParts * D + tid];
#pragma unroll
    for (int i = 1; i < Lds::kParts; ++i) {
      l = raw_min(l, box[i * D + tid]);
      u = raw_max(u, box[(Lds::kParts + i) * D + tid]);
    }
    const size_t at = (((size_t)b * p.Hkv + h) * p.Pmax + j) * D + tid;
    if (slot0 != 0) {
      l = raw_min(l, elem_to_f32<kHalf>(p.page_min[at]));
      u = raw_max(u, elem_to_f32<kHalf>(p.page_max[at]));
    }
    p.page_min[at] = box_number<FMT>(l, false);
    p.page_max[at] = box_number<FMT>(u, true);
  }
  // the values: channel-major, the tokens of a channel together
  if constexpr (FMT == kPoolFp4) {
    const int oct0 = slot0 >> 3, octs = ((slot1 + 7) >> 3) - oct0;
    for (int i = tid; i < octs * D; i += kRotaryThreads) {
      const int o = oct0 + i / D, w = i % D, ch = Fp4Block<D>::channel(w);
      uint32_t* dst = reinterpret_cast<uint32_t*>(tile.v) + (size_t)o * D + w;
      // (slots without a new token hold anything: their codes are masked)
      uint32_t word = 0u;
#pragma unroll
      for (int t = 0; t < 8; ++t) word |= (uint32_t)(vs[(8 * o + t) * Lds::kRow + ch] & 15u) << (4 * t);
      const int from = max(slot0 - 8 * o, 0), upto = min(slot1 - 8 * o, 8);
      const uint32_t mask = (upto == 8 ? 0xffffffffu : (1u << (4 * upto)) - 1u) & ~((1u << (4 * from)) - 1u);
      *dst = mask == 0xffffffffu ? word : (*dst & ~mask) | (word & mask);
    }
  } else {
    constexpr int kMost = 16 / (int)sizeof(Elem);      // tokens in 16 bytes
    const int chunk = min(kMost, p.S), csh = __builtin_ctz(chunk);
    const int first = slot0 >> csh, chunks = ((slot1 + chunk - 1) >> csh) - first;
    Elem* dst_tile = reinterpret_cast<Elem*>(tile.v);
    for (int i = tid; i < chunks * D; i += kRotaryThreads) {
      const int ch = i / chunks, s0 = (first + i % chunks) << csh;
      Elem* dst = dst_tile + (size_t)ch * p.S + s0;
      if (s0 >= slot0 && s0 + chunk <= slot1 && chunk == kMost) {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int t = 0; t < kMost; ++t)
          w[t * (int)sizeof(Elem) / 4] |= (uint32_t)vs[(s0 + t) * Lds::kRow + ch]
                                          << (8 * sizeof(Elem) * (t % (4 / (int)sizeof(Elem))));
        *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        for (int t = max(s0, slot0); t < min(s0 + chunk, slot1); ++t) dst[t - s0] = vs[t * Lds::kRow + ch];
      }
    }
  }
}

// The lengths after an append, in a launch of its own: the workgroups of the append read them.
// block_table: a sequence whose one new token has no valid page is left alone (null: not looked at).
static __global__ void advance_lens_kernel(int32_t* seq_lens, const int32_t* cu, const int32_t* block_table, int B,
                                           int T, int sh, int Pmax, int n_phys) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= B) return;
  const int n = cu ? max(min(max(cu[b + 1], 0), T) - min(max(cu[b], 0), T), 0) : 1;
  const int len = seq_lens[b];
  if (len < 0 || (long long)len + n > (long long)Pmax << sh) return;
  if (block_table) {
    const int phys = block_table[(size_t)b * Pmax + (len >> sh)];
    if (phys < 0 || phys >= n_phys) return;
  }
  seq_lens[b] = len + n;
}

}  // namespace ts
