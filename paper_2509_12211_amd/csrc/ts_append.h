// Appending tokens to the paged cache: any number of tokens for each sequence, keys normed and rotated on
// the way (ts_rotary.h), values transposed into their channel-major tiles, page boxes opened or widened, the
// queries of the same tokens rotated in the same launch.
//
// A workgroup takes the tokens that fall into ONE page of one sequence, for one KV head and the query
// heads that share it.  So a page's tile and its box have one writer, what the page held already needs no
// atomics, and the box of a new page is worked out from the tokens in hand.  Keys go from registers to
// their slots; the values, and the keys' stored form for the box, pass through LDS.
#pragma once
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
  if (!(amax > 0.f)) return 1.0f;
  const uint32_t b = __float_as_uint(__fdiv_rn(fminf(amax, 3.3e38f), 6.0f));
  return __uint_as_float((b + 0xffffu) & 0xffff0000u);
}
// Nearest code, ties to the even one; no negative zero; NaN is 0.
__device__ __forceinline__ uint32_t fp4_code(float x, float scale) {
  const float r = __fdiv_rn(x, scale), m = fabsf(r);
  const uint32_t c = (uint32_t)(m > 0.25f) + (uint32_t)(m >= 0.75f) + (uint32_t)(m > 1.25f) + (uint32_t)(m >= 1.75f) +
                     (uint32_t)(m > 2.5f) + (uint32_t)(m >= 3.5f) + (uint32_t)(m > 5.0f);
  return c != 0u && r < 0.f ? c | 8u : c;
}
__device__ __forceinline__ float fp4_value(uint32_t code) {
  const uint32_t m = code & 7u;
  // twice the magnitudes, a nibble each but the last: 0 1 2 3 4 6 8 12
  const float v = 0.5f * (float)((0xc8643210u >> (4 * m)) & 15u);
  return (code & 8u) != 0u ? -v : v;
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
  const int32_t* cu;                  // [B + 1] first token of each sequence (null: one token each)
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
  static constexpr int kRow = D + 8;   // elements of a staged row
  static constexpr int kParts = kRotaryThreads / D;
  __host__ __device__ static constexpr size_t bytes(int S) {
    return 2 * (size_t)S * kRow * sizeof(Elem) + (size_t)S * 4 + 2 * (size_t)kParts * D * 4;
  }
};

// Which page of which sequence workgroup `task` has.  The sequences' touched pages are numbered through;
// every wave works the same answer out.  False: there are fewer.
__device__ __forceinline__ bool find_page(const AppendParams& p, int sh, int task, int& b, int& j) {
  int before = 0;
  for (int base = 0; base < p.B; base += kWave) {
    const int i = base + lane_id();
    int pages = 0, first = 0;
    if (i < p.B) {
      const int c0 = min(max(p.cu[i], 0), p.T), c1 = min(max(p.cu[i + 1], 0), p.T), n = c1 - c0;
      if (n > 0) {
        const int len = p.seq_lens[i] - (p.lens_after ? p.cu[i + 1] - p.cu[i] : 0);
        first = len >> sh;
        pages = ((len + n - 1) >> sh) - first + 1;
      }
    }
    const int upto = before + wave_inclusive_sum(pages);
    const uint64_t mine = __ballot(task < upto && task >= upto - pages);
    if (mine != 0) {
      const int src = __builtin_ctzll(mine);
      b = base + src;
      j = __builtin_amdgcn_readlane(first, src) + task - __builtin_amdgcn_readlane(upto - pages, src);
      b = uniform(b);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return false;
}

// grid (touched pages or more, Hkv)
template <int FMT, int D>
__global__ __launch_bounds__(kRotaryThreads) void append_rows_kernel(AppendParams p) {
  constexpr bool kHalf = FMT == kPoolFp16;
  constexpr bool kQuant = FMT == kPoolInt8 || FMT == kPoolFp4;
  constexpr int LPR = D / 8, NG = kRotaryThreads / LPR;
  typedef AppendLds<FMT, D> Lds;
  typedef typename Lds::Elem Elem;
  extern __shared__ __align__(16) unsigned char smem[];
  Elem* ks = reinterpret_cast<Elem*>(smem);
  Elem* vs = ks + (size_t)p.S * Lds::kRow;
  float* ksc = reinterpret_cast<float*>(vs + (size_t)p.S * Lds::kRow);   // scales of the slots
  float* box = ksc + p.S;                                                // [2][parts][D]
  const int sh = __builtin_ctz(p.S), h = blockIdx.y, tid = threadIdx.x;
  int b, j, c0, n;
  if (p.cu == nullptr) {
    b = blockIdx.x;
    c0 = b;
    n = 1;
    j = -1;
  } else {
    if (!find_page(p, sh, blockIdx.x, b, j)) return;
    c0 = min(max(p.cu[b], 0), p.T);
    n = min(max(p.cu[b + 1], 0), p.T) - c0;
  }
  n = uniform(n);
  const int len = uniform(p.seq_lens[b] - (p.lens_after ? (p.cu ? p.cu[b + 1] - p.cu[b] : 1) : 0));
  if (j < 0) j = len >> sh;
  if (len < 0) return;                                   // (no such length)
  const int p0 = max(j << sh, len), p1 = min((j + 1) << sh, len + n);   // positions of this page's new tokens
  const int ntok = p1 - p0, slot0 = p0 - (j << sh), tok0 = c0 + p0 - len;
  const bool fits = (long long)len + n <= (long long)p.Pmax << sh;
  const int phys = uniform(fits ? p.block_table[(size_t)b * p.Pmax + j] : -1);
  const bool store = fits && p.v_pool != nullptr && phys >= 0 && phys < p.n_phys;
  const bool keep = store || (fits && p.v_pool == nullptr);     // the box follows the keys
  unsigned char* ktile = p.k_pool + ((size_t)(store ? phys : 0) * p.Hkv + h) * (size_t)p.tile_stride;
  unsigned char* vtile = FMT == kPoolFp4 ? ktile + Fp4Block<D>::values(p.S)
                                         : p.v_pool + ((size_t)(store ? phys : 0) * p.Hkv + h) * (size_t)p.tile_stride;
  const size_t scale_row = ((size_t)(store ? phys : 0) * p.Hkv + h) * (size_t)p.S;
  // the rows of a token are dealt to as many of the workgroup's groups of lanes as there are for each token
  int tp = 1;
  while (tp < ntok && tp < NG) tp <<= 1;
  const int group = tid / LPR, li = tid % LPR, first_row = group / tp, step = NG / tp;
  const RowLanes<D> lanes(p.r, li);
  Norm qn, kn;
  load_norm(p.r.q_norm, lanes.c0, lanes.c1, qn);
  load_norm(p.r.k_norm, lanes.c0, lanes.c1, kn);
  // rows of a token: its key, its value, its query heads
  const int rows = 2 + (p.q != nullptr ? p.G : 0);
  for (int i0 = group % tp; i0 < ntok; i0 += tp) {   // (whole rows of lanes go round together)
    const int tok = tok0 + i0, slot = slot0 + i0;
    Angles ang;
    load_angles(p.r, li, lanes.turns,
                [&](int axis) { return p.r.positions ? p.r.positions[(size_t)axis * p.r.T + tok] : p0 + i0; }, ang);
    for (int row = first_row; row < rows; row += step) {
      if (row < 2 && !keep) continue;
      if (row == 1 && !store) continue;
      const uint16_t* src = row == 0   ? p.k + tok * p.k_stride + h * D
                            : row == 1 ? p.v + tok * p.v_stride + h * D
                                       : p.q + tok * p.q_stride + (h * p.G + row - 2) * D;
      const int a0 = row == 1 ? 8 * li : lanes.c0, a1 = row == 1 ? 8 * li + 4 : lanes.c1;
      uint2 x = *reinterpret_cast<const uint2*>(src + a0), y = *reinterpret_cast<const uint2*>(src + a1);
      if (row >= 2) {
        rotate_row<D, kHalf>(p.r, lanes.turns, qn, ang, x, y);
        uint16_t* dst = p.q_out + tok * p.q_out_stride + (h * p.G + row - 2) * D;
        *reinterpret_cast<uint2*>(dst + a0) = x;
        *reinterpret_cast<uint2*>(dst + a1) = y;
        continue;
      }
      if (row == 0) rotate_row<D, kHalf>(p.r, lanes.turns, kn, ang, x, y);
      Elem* stage = (row == 0 ? ks : vs) + slot * Lds::kRow;
      if constexpr (!kQuant) {
        if (row == 0 && store) {
          uint16_t* dst = reinterpret_cast<uint16_t*>(ktile) + slot * D;
          *reinterpret_cast<uint2*>(dst + a0) = x;
          *reinterpret_cast<uint2*>(dst + a1) = y;
        }
        *reinterpret_cast<uint2*>(stage + a0) = x;
        *reinterpret_cast<uint2*>(stage + a1) = y;
      } else {
        const float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y),
                            bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(f[i]));
        amax = group_max_f32<LPR>(amax);
        const float scale = FMT == kPoolInt8 ? i8_row_scale(amax) : fp4_row_scale(amax);
        uint32_t c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          c[i] = FMT == kPoolInt8 ? (uint32_t)i8_code(f[i], scale) & 0xffu : fp4_code(f[i], scale);
        const uint32_t w0 = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, w1 = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
        *reinterpret_cast<uint32_t*>(stage + a0) = w0;
        *reinterpret_cast<uint32_t*>(stage + a1) = w1;
        if (row == 0 && li == 0) ksc[slot] = scale;
        if (store) {
          if constexpr (FMT == kPoolInt8) {
            if (row == 0) {
              *reinterpret_cast<uint32_t*>(ktile + slot * D + a0) = w0;
              *reinterpret_cast<uint32_t*>(ktile + slot * D + a1) = w1;
            }
            if (li == 0) (row == 0 ? p.k_scale : p.v_scale)[scale_row + slot] = scale;
          } else {
            if (row == 0) {
              unsigned char* dst = ktile + slot * (D / 2);
              *reinterpret_cast<uint16_t*>(dst + a0 / 2) = (uint16_t)(c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12);
              *reinterpret_cast<uint16_t*>(dst + a1 / 2) = (uint16_t)(c[4] | c[5] << 4 | c[6] << 8 | c[7] << 12);
            }
            if (li == 0) {
              const int at = row == 0 ? Fp4Block<D>::key_scales(p.S) : Fp4Block<D>::value_scales(p.S);
              *reinterpret_cast<uint16_t*>(ktile + at + 2 * slot) = (uint16_t)(__float_as_uint(scale) >> 16);
            }
          }
        }
      }
    }
  }
  if (!keep) return;
  __syncthreads();
  const int slot1 = slot0 + ntok;
  // the box: a thread takes a channel, and every kParts-th token of it
  const int c = tid % D, part = tid / D;
  float lo = INFINITY, hi = -INFINITY;
  for (int s = slot0 + part; s < slot1; s += Lds::kParts) {
    const Elem e = ks[s * Lds::kRow + c];
    float l, u;
    if constexpr (FMT == kPoolInt8) {
      const double x = (double)(int8_t)e * (double)ksc[s];
      l = bf16_to_f32(bf16_directed(x, false));
      u = bf16_to_f32(bf16_directed(x, true));
    } else if constexpr (FMT == kPoolFp4) {
      l = u = fp4_value(e) * ksc[s];
    } else {
      l = u = elem_to_f32<kHalf>(e);
    }
    lo = fminf(lo, l);
    hi = fmaxf(hi, u);
  }
  box[part * D + c] = lo;
  box[(Lds::kParts + part) * D + c] = hi;
  // the values: channel-major, the tokens of a channel together
  if (store) {
    if constexpr (FMT == kPoolFp4) {
      const int oct0 = slot0 >> 3, octs = ((slot1 + 7) >> 3) - oct0;
      for (int i = tid; i < octs * D; i += kRotaryThreads) {
        const int o = oct0 + i / D, w = i % D, ch = Fp4Block<D>::channel(w);
        uint32_t word = 0u, mask = 0u;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const int s = 8 * o + t;
          if (s >= slot0 && s < slot1) {
            word |= (uint32_t)vs[s * Lds::kRow + ch] << (4 * t);
            mask |= 15u << (4 * t);
          }
        }
        uint32_t* dst = reinterpret_cast<uint32_t*>(vtile) + (size_t)o * D + w;
        *dst = mask == 0xffffffffu ? word : (*dst & ~mask) | word;
      }
    } else {
      constexpr int kMost = 16 / (int)sizeof(Elem);      // tokens in 16 bytes
      const int chunk = min(kMost, p.S), csh = __builtin_ctz(chunk);
      const int first = slot0 >> csh, chunks = ((slot1 + chunk - 1) >> csh) - first;
      Elem* tile = reinterpret_cast<Elem*>(vtile);
      for (int i = tid; i < chunks * D; i += kRotaryThreads) {
        const int ch = i / chunks, s0 = (first + i % chunks) << csh;
        Elem* dst = tile + (size_t)ch * p.S + s0;
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
  __syncthreads();
  if (tid < D) {
#pragma unroll
    for (int i = 1; i < Lds::kParts; ++i) {
      lo = fminf(lo, box[i * D + c]);
      hi = fmaxf(hi, box[(Lds::kParts + i) * D + c]);
    }
    const size_t at = (((size_t)b * p.Hkv + h) * p.Pmax + j) * D + c;
    if (slot0 != 0) {
      lo = fminf(lo, elem_to_f32<kHalf>(p.page_min[at]));
      hi = fmaxf(hi, elem_to_f32<kHalf>(p.page_max[at]));
    }
    if constexpr (FMT == kPoolFp4) {
      p.page_min[at] = (uint16_t)bf16_outwards(lo, false);
      p.page_max[at] = (uint16_t)bf16_outwards(hi, true);
    } else {
      p.page_min[at] = kHalf ? f32_to_half(lo) : (uint16_t)(__float_as_uint(lo) >> 16);
      p.page_max[at] = kHalf ? f32_to_half(hi) : (uint16_t)(__float_as_uint(hi) >> 16);
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
