// Attention over the 4-bit cache, and the rebuild of its page boxes.
//
// Single-query softmax attention over every cached token (dense) or over the pages of a list (sparse), one
// launch.  Fragments of 32 tokens: K (16 tokens x 32 channels a product) and V (16 channels x 32 tokens) are
// expanded to bf16 in registers, one instruction for two codes, and go through v_mfma_f32_16x16x32_bf16;
// the scales of 32 tokens multiply the logits (K) and the softmax weights (V) afterwards.  e2m1 numbers and
// bf16 queries are exact operands; the weights go in as three bf16 numbers (the nearest, the remainder's
// nearest, and what is left: 2^-27 relative; with two an fp32 output was 2e-6 off, twice what the sums
// cost), so nothing but the fp32 sums rounds.
//   logits  St[token][head] = K[token][:] . Q^T[:][head]      row = token, column = head
//   output  Ot[chan][head] += V^T[chan][token] . P^T[token][head]
// Row 4 kb + i of logit tile t is token 8 kb + 4 t + i of the fragment (kb: quarter of the wave), so the eight
// weights a lane has are the eight tokens its quarter contracts in the second product.
//
// Work: the units' fragments are numbered through, unit after unit, and every workgroup takes an equal
// contiguous share, whatever the lengths; each works out from the lengths which.  A workgroup's waves take
// the fragments of a unit in turn and merge in LDS.  A unit that several workgroups share is merged by the
// last of them to arrive (an atomic count in the workspace, set back to zero); nobody waits.
#pragma once
#include "ts_append.h"
#include "ts_attend.h"

namespace ts {

constexpr int kFp4Frag = 32;            // tokens of a fragment
constexpr int kFp4List = 1024;          // list entries held in LDS at a time
constexpr int kFp4Parts = 64;           // about how many workgroups share a unit at the most

// Workgroups of eight waves, two on each compute unit, for 64 channels; with 128 a wave needs more than the
// 128 registers that leaves it (165), so four waves, three on each (1.1 GB of ragged sequences 276 -> 237 us).
template <int D>
struct Fp4Shape {
  static constexpr int kWavesPer = D == 64 ? 8 : 4, kThreadsPer = kWavesPer * kWave;
  static constexpr int kOccupancy = D == 64 ? 4 : 3;          // waves a SIMD
  static constexpr int kResident = 256 * kOccupancy * 4 / kWavesPer;
  static constexpr int kMinShare = 2 * kWavesPer;             // fragments a workgroup has at the least
};

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct Fp4Params {
  const uint16_t* q;
  const unsigned char* pool;
  const int32_t *block_table, *seq_lens;
  const int32_t *sel, *sel_count;   // sparse: [B][Hkv][Kmax], [B]
  float* out;                       // [B][Hq][D] fp32 or bf16
  float* lse;                       // nullable [B][Hq]
  float* part;                      // [workgroups][2][G][D + 2]: what a unit's workgroups hand over
  int32_t* done;                    // [units] workgroups that have; zero between launches
  int B, Hq, Hkv, G, Pmax, Kmax, n_phys, out_bf16;
  long long tile_stride;
  float scale_log2;
};

// Eight codes, two a byte, as an operand of eight bf16 numbers.
__device__ __forceinline__ bf16x8_t fp4_operand(uint32_t w) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int D>
struct Fp4Frag {
  uint32_t k[2][D / 32];   // this lane's D / 4 channels of its two tokens
  uint4 v[D / 64];         // this lane's eight tokens of D / 16 channels
  uint4 ks, vs;            // the eight tokens' scales
  int valid;               // how many of the eight tokens exist
};

// One entry of the list: where a page's block of the unit's head begins, in units of 16 bytes, and in the low
// eight bits how many of its tokens count.
typedef uint64_t Fp4Entry;
__device__ __forceinline__ Fp4Entry fp4_entry(const Fp4Params& p, int phys, int h, int tokens) {
  return ((uint64_t)phys * p.Hkv + h) * (uint64_t)(p.tile_stride >> 4) << 8 | (uint64_t)tokens;
}

// Where fragment `frag` of the list keeps the eight tokens `oct`: the page's block and the first token's slot.
template <int S>
__device__ __forceinline__ const unsigned char* fp4_octet(const Fp4Params& p, const Fp4Entry* list, int frag, int oct,
                                                          int& slot, int& tokens) {
  constexpr int PPF = S < kFp4Frag ? kFp4Frag / S : 1, FPP = S > kFp4Frag ? S / kFp4Frag : 1;
  const Fp4Entry e = list[frag / FPP * PPF + (PPF > 1 ? 8 * oct / S : 0)];
  slot = (FPP > 1 ? kFp4Frag * (frag % FPP) : 0) + (8 * oct) % (S < kFp4Frag ? S : kFp4Frag);
  uint32_t lo = (uint32_t)e, hi = (uint32_t)(e >> 32);
  if (PPF == 1) {      // the same page for all lanes
    lo = (uint32_t)uniform((int)lo);
    hi = (uint32_t)uniform((int)hi);
  }
  tokens = (int)(lo & 0xffu);
  return p.pool + ((((uint64_t)hi << 32 | (lo & ~0xffu)) >> 4));
}

// The keys: rows of tokens 8 (r / 4) + r % 4 and 4 on, r = lane % 16; the scales of this quarter's tokens.
template <int D, int S>
__device__ __forceinline__ void load_fp4_keys(Fp4Frag<D>& f, const Fp4Params& p, const Fp4Entry* list, int frag) {
  const int lane = lane_id(), r = lane & 15, kb = lane >> 4;
  int slot, tokens;
  const unsigned char* row = fp4_octet<S>(p, list, frag, r >> 2, slot, tokens);
  row += (slot + (r & 3)) * (D / 2) + kb * (D / 8);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if constexpr (D == 128) {
      const uint4 w = *reinterpret_cast<const uint4*>(row + 4 * t * (D / 2));
      f.k[t][0] = w.x; f.k[t][1] = w.y; f.k[t][2] = w.z; f.k[t][3] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(row + 4 * t * (D / 2));
      f.k[t][0] = w.x; f.k[t][1] = w.y;
    }
  }
  const unsigned char* tile = fp4_octet<S>(p, list, frag, kb, slot, tokens);
  f.ks = *reinterpret_cast<const uint4*>(tile + Fp4Block<D>::key_scales(S) + 2 * slot);
  f.valid = tokens - slot;
}

// The values of this quarter's tokens and their scales.
template <int D, int S>
__device__ __forceinline__ void load_fp4_values(Fp4Frag<D>& f, const Fp4Params& p, const Fp4Entry* list, int frag) {
  const int lane = lane_id(), r = lane & 15, kb = lane >> 4;
  int slot, tokens;
  const unsigned char* tile = fp4_octet<S>(p, list, frag, kb, slot, tokens);
  const unsigned char* row = tile + Fp4Block<D>::values(S) + (slot / 8) * (4 * D) + r * 16;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) f.v[i] = *reinterpret_cast<const uint4*>(row + 256 * i);
  f.vs = *reinterpret_cast<const uint4*>(tile + Fp4Block<D>::value_scales(S) + 2 * slot);
}

// Running softmax state of a wave: per lane the head lane % 16.
template <int D>
struct Fp4State {
  float4_t acc[D / 16];   // channels 16 cb + 4 kb .. + 3
  float m, l;             // running maximum (log2 units, the same in the four quarters), this quarter's sum
};

// One fragment; with kMore the one behind it (next) is fetched piece by piece into the registers that this
// one leaves: its keys go out behind the first product, its values behind the second.
template <int D, int S, bool kMore>
__device__ __forceinline__ void attend_fp4(Fp4State<D>& st, Fp4Frag<D>& f, const bf16x8_t (&q)[D / 32], const Fp4Params& p,
                                           const Fp4Entry* list, int next) {
  float s[8];
  {
    float ks[8];
    unpack8(f.ks, ks);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < D / 32; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp4_operand(f.k[t][i]), q[i], c, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * t + i] = c[i] * (ks[4 * t + i] * p.scale_log2);
    }
  }
  const int valid = f.valid;
  __builtin_amdgcn_sched_barrier(0);
  if (kMore) load_fp4_keys<D, S>(f, p, list, next);
  __builtin_amdgcn_sched_barrier(0);
  float vs[8];
  unpack8(f.vs, vs);
  if (__any(valid < 8)) {   // slots without a token may hold anything, scales included
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[i] = i < valid ? s[i] : -INFINITY;
      vs[i] = i < valid ? vs[i] : 0.f;
    }
  }
  float m = s[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, s[i]);
  m = fmaxf(rows_max_f32(m), st.m);
  const float ref = m == -INFINITY ? 0.f : m;
  if (__any(m > st.m)) {
    const float a = __builtin_amdgcn_exp2f(st.m - ref);
    st.l *= a;
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) st.acc[cb] *= a;
    st.m = m;
  }
  bf16x8_t hi, lo, rest;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float w = __builtin_amdgcn_exp2f(s[i] - ref);
    st.l += w;
    const float x = w * vs[i];
    hi[i] = (__bf16)x;
    const float y = x - (float)hi[i];
    lo[i] = (__bf16)y;
    rest[i] = (__bf16)(y - (float)lo[i]);
  }
  auto word = [&](int cb) {
    const uint4 w = f.v[cb / 4];
    return cb % 4 == 0 ? w.x : cb % 4 == 1 ? w.y : cb % 4 == 2 ? w.z : w.w;
  };
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) {
    const bf16x8_t v = fp4_operand(word(cb));
    st.acc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, rest, st.acc[cb], 0, 0, 0);
    st.acc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo, st.acc[cb], 0, 0, 0);
    st.acc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, st.acc[cb], 0, 0, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
  if (kMore) load_fp4_values<D, S>(f, p, list, next);
  __builtin_amdgcn_sched_barrier(0);
}

template <int S, bool kSparse>
__device__ __forceinline__ int fp4_frags(const Fp4Params& p, int b) {
  if (kSparse) {
    const int n = min(max(p.sel_count[b], 0), p.Kmax);
    return S <= kFp4Frag ? (n * S + kFp4Frag - 1) / kFp4Frag : n * (S / kFp4Frag);
  }
  const int len = min(max(p.seq_lens[b], 0), p.Pmax * S);
  return (len + kFp4Frag - 1) / kFp4Frag;
}

__device__ __forceinline__ void store_fp4_out(const Fp4Params& p, size_t idx, float v) {
  if (p.out_bf16) reinterpret_cast<uint16_t*>(p.out)[idx] = f32_to_bf16_rn(v);
  else p.out[idx] = v;
}

template <int D, int S, bool kSparse>
__global__ __launch_bounds__(Fp4Shape<D>::kThreadsPer, Fp4Shape<D>::kOccupancy) void fp4_attention_kernel(Fp4Params p) {
  constexpr int kFp4Waves = Fp4Shape<D>::kWavesPer, kFp4Threads = Fp4Shape<D>::kThreadsPer;
  constexpr int PPF = S < kFp4Frag ? kFp4Frag / S : 1, FPP = S > kFp4Frag ? S / kFp4Frag : 1;
  constexpr int kFrags = (kFp4List + 1 - FPP) * FPP / PPF;   // fragments the list in LDS covers, begun within a page too
  constexpr int kRow = D + 4;                        // a head's merged row: channels, maximum, sum
  extern __shared__ __align__(16) unsigned char smem[];
  Fp4Entry* list = reinterpret_cast<Fp4Entry*>(smem);
  float* merge = reinterpret_cast<float*>(list + kFp4List);       // [waves][G][kRow]
  __shared__ int last_one;
  const int tid = threadIdx.x, lane = lane_id(), wave = wave_id(), r = lane & 15, kb = lane >> 4;

  // all fragments of the launch, and where this workgroup's begin
  uint32_t total = 0;
  int longest = 0, mine = 0, upto = 0;     // of a wave's last 64 sequences: this lane's fragments, up to here
  for (int base = 0; base < p.B; base += kWave) {
    const int i = base + lane, f = i < p.B ? fp4_frags<S, kSparse>(p, i) : 0;
    mine = f;
    upto = wave_inclusive_sum(f);
    total += (uint32_t)__builtin_amdgcn_readlane(upto, kWave - 1);
    longest = max(longest, (int)wave_max_u32((uint32_t)f));
    // a sequence without tokens has zeros
    if (blockIdx.x == 0 && wave == 0) {
      uint64_t none = __ballot(i < p.B && f == 0);
      while (none != 0) {
        const int e = base + __builtin_ctzll(none);
        none &= none - 1;
        for (int x = lane; x < p.Hq * D; x += kWave) store_fp4_out(p, (size_t)e * p.Hq * D + x, 0.f);
        if (p.lse)
          for (int x = lane; x < p.Hq; x += kWave) p.lse[(size_t)e * p.Hq + x] = -INFINITY;
      }
    }
  }
  total *= (uint32_t)p.Hkv;
  const uint32_t share = max(max((uint32_t)Fp4Shape<D>::kMinShare, (total + gridDim.x - 1) / gridDim.x),
                             (uint32_t)((longest + kFp4Parts - 1) / kFp4Parts));
  uint32_t at = blockIdx.x * share;
  const uint32_t end = min(total, at + share);
  if (at >= end) return;
  int b = 0, nf = 0;
  uint32_t ustart = 0;    // first fragment of the unit
  for (int base = 0, before = 0; base < p.B; base += kWave) {
    if (p.B > kWave) {      // (up to 64 sequences the lanes have them still)
      mine = base + lane < p.B ? fp4_frags<S, kSparse>(p, base + lane) : 0;
      upto = before + wave_inclusive_sum(mine);
    }
    const uint32_t first = (uint32_t)(upto - mine) * p.Hkv;
    const uint64_t here = __ballot(at >= first && at < (uint32_t)upto * p.Hkv);
    if (here != 0) {
      const int src = __builtin_ctzll(here);
      b = uniform(base + src);
      nf = __builtin_amdgcn_readlane(mine, src);
      ustart = (uint32_t)__builtin_amdgcn_readlane((int)first, src);
      break;
    }
    before = __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  int h = (int)((at - ustart) / (uint32_t)nf);
  ustart += (uint32_t)h * (uint32_t)nf;

  while (at < end) {
    const int f0 = (int)(at - ustart), f1 = (int)min((uint32_t)nf, end - ustart);
    const int u = b * p.Hkv + h;
    const int len = min(max(p.seq_lens[b], 0), p.Pmax * S), count = kSparse ? min(max(p.sel_count[b], 0), p.Kmax) : 0;
    bf16x8_t q[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint16_t* src = p.q + ((size_t)b * p.Hq + h * p.G + min(r, p.G - 1)) * D + kb * (D / 4) + 8 * i;
      uint4 w = *reinterpret_cast<const uint4*>(src);
      if (r >= p.G) w = make_uint4(0u, 0u, 0u, 0u);
      q[i] = __builtin_bit_cast(bf16x8_t, w);
    }
    Fp4State<D> st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) st.acc[cb] = float4_t{0.f, 0.f, 0.f, 0.f};
    for (int c0 = f0; c0 < f1; c0 += kFrags) {
      const int c1 = min(f1, c0 + kFrags), e0 = c0 / FPP * PPF, entries = ((c1 - 1) / FPP + 1) * PPF - e0;
      __syncthreads();    // the list before is read, and so is the merge area
      for (int i = tid; i < entries; i += kFp4Threads) {
        int page = e0 + i;
        bool on = true;
        if (kSparse) {
          on = page < count;
          page = p.sel[(size_t)u * p.Kmax + min(page, p.Kmax - 1)];
        }
        on = on && page >= 0 && page < p.Pmax;
        const int phys = p.block_table[(size_t)b * p.Pmax + (on ? page : 0)];
        on = on && phys >= 0 && phys < p.n_phys;
        list[i] = on ? fp4_entry(p, phys, h, min(max(len - page * S, 0), S)) : fp4_entry(p, 0, h, 0);
      }
      __syncthreads();
      const int shift = c0 % FPP - c0;      // fragments as the list has them
      if (c0 + wave < c1) {
        Fp4Frag<D> fr;
        int f = c0 + wave + shift;
        load_fp4_keys<D, S>(fr, p, list, f);
        load_fp4_values<D, S>(fr, p, list, f);
        for (; f + kFp4Waves < c1 + shift; f += kFp4Waves) attend_fp4<D, S, true>(st, fr, q, p, list, f + kFp4Waves);
        attend_fp4<D, S, false>(st, fr, q, p, list, 0);
      }
    }
    // the waves' results: head rows of channels, maximum, sum
    const float l = rows_sum_f32(st.l);
    if (r < p.G) {
      float* row = merge + (wave * p.G + r) * kRow;
#pragma unroll
      for (int cb = 0; cb < D / 16; ++cb) *reinterpret_cast<float4_t*>(row + 16 * cb + 4 * kb) = st.acc[cb];
      if (kb == 0) {
        row[D] = st.m;
        row[D + 1] = l;
      }
    }
    __syncthreads();
    const uint32_t uend = ustart + (uint32_t)nf;
    const uint32_t w0 = ustart / share, w1 = (uend - 1) / share;
    const bool whole = w0 == w1;
    float* mine = p.part + ((size_t)blockIdx.x * 2 + (at > ustart ? 0 : 1)) * p.G * (D + 2);
    for (int i = tid; i < p.G * D; i += kFp4Threads) {
      const int g = i / D, c = i % D;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kFp4Waves; ++w) M = fmaxf(M, merge[(w * p.G + g) * kRow + D]);
      float o = 0.f, sum = 0.f;
      if (M != -INFINITY) {
#pragma unroll
        for (int w = 0; w < kFp4Waves; ++w) {
          const float* row = merge + (w * p.G + g) * kRow;
          const float a = __builtin_amdgcn_exp2f(row[D] - M);
          o += a * row[c];
          sum += a * row[D + 1];
        }
      }
      if (whole) {
        const size_t head = (size_t)b * p.Hq + h * p.G + g;
        store_fp4_out(p, head * D + c, sum > 0.f ? o / sum : 0.f);
        if (p.lse && c == 0) p.lse[head] = sum > 0.f ? (M + __log2f(sum)) * 0.6931471805599453f : -INFINITY;
      } else {
        store_agent(mine + g * (D + 2) + c, o);
        if (c == 0) {
          store_agent(mine + g * (D + 2) + D, M);
          store_agent(mine + g * (D + 2) + D + 1, sum);
        }
      }
    }
    if (!whole) {
      stores_complete();
      __syncthreads();
      if (tid == 0) {
        const int before = atomic_add_agent(p.done + u, 1);
        last_one = before == (int)(w1 - w0);
        if (last_one) atomic_store_agent(p.done + u, 0);
      }
      __syncthreads();
      if (uniform(last_one)) {
        // maxima and sums of all parts into LDS, their weights over the common maximum from there
        const int parts = (int)(w1 - w0) + 1;
        auto part_of = [&](int e) {
          const uint32_t w = w0 + (uint32_t)e;
          return p.part + ((size_t)w * 2 + (w * share > ustart ? 0 : 1)) * p.G * (D + 2);
        };
        float* tops = merge;                        // [parts][G]
        float* sums = merge + parts * p.G;          // [parts][G]
        constexpr int kAhead = 8;                   // parts asked for together
        float x[kAhead];
        auto fetch = [&](int i, int e0) {
#pragma unroll
          for (int e = 0; e < kAhead; ++e) x[e] = load_agent(part_of(min(e0 + e, parts - 1)) + i / D * (D + 2) + i % D);
        };
        if (tid < p.G * D) fetch(tid, 0);
        for (int i = tid; i < parts * p.G; i += kFp4Threads) {
          const float* row = part_of(i / p.G) + (i % p.G) * (D + 2) + D;
          tops[i] = load_agent(row);
          sums[i] = load_agent(row + 1);
        }
        __syncthreads();
        for (int i = tid; i < p.G * D; i += kFp4Threads) {
          const int g = i / D, c = i % D;
          float M = -INFINITY, o = 0.f, sum = 0.f;
          for (int e = 0; e < parts; ++e) M = fmaxf(M, tops[e * p.G + g]);
          const float ref = M == -INFINITY ? 0.f : M;
          for (int e0 = 0; e0 < parts; e0 += kAhead) {
            if (e0 != 0 || i != tid) fetch(i, e0);
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
              if (e0 + e < parts) {
                const float a = __builtin_amdgcn_exp2f(tops[(e0 + e) * p.G + g] - ref);
                o += x[e] * a;
                sum += sums[(e0 + e) * p.G + g] * a;
              }
            }
          }
          const size_t head = (size_t)b * p.Hq + h * p.G + g;
          store_fp4_out(p, head * D + c, sum > 0.f ? o / sum : 0.f);
          if (p.lse && c == 0) p.lse[head] = sum > 0.f ? (M + __log2f(sum)) * 0.6931471805599453f : -INFINITY;
        }
      }
    }
    // the next unit
    at = uend;
    ustart = uend;
    if (++h == p.Hkv) {
      h = 0;
      if (at < end) {
        do { ++b; nf = uniform(fp4_frags<S, kSparse>(p, b)); } while (nf == 0 && b + 1 < p.B);
      }
    }
  }
}

// Rebuild of the boxes: a page's D / 32 lanes own 32 channels each (16 bytes of a token's row) and walk
// down its tokens.  code * scale is exact in fp32, so the extremes are, and are rounded outwards to bf16.
template <int D>
__global__ __launch_bounds__(kThreads) void build_page_meta_fp4_kernel(MetaParams p) {
  constexpr int LPP = D / 32, PPW = kWave / LPP;    // lanes a page, pages a wave
  const int lane = lane_id(), cg = lane % LPP;
  const int first = (blockIdx.y * kWaves + wave_id()) * PPW, j = first + lane / LPP;
  const int h = blockIdx.x, b = blockIdx.z;
  const int L = p.seq_lens[b];
  const int Pb = min((L + p.S - 1) / p.S, p.Pmax);
  if (uniform(first) >= Pb) return;
  const int phys = p.block_table[(size_t)b * p.Pmax + min(j, Pb - 1)];
  const bool on = j < Pb && phys >= 0 && phys < p.n_phys;
  const int tokens = on ? min(p.S, L - j * p.S) : 0;
  const unsigned char* tile = reinterpret_cast<const unsigned char*>(p.k_pool) +
                              ((size_t)(on ? phys : 0) * p.Hkv + h) * (size_t)p.tile_stride;
  const uint16_t* scales = reinterpret_cast<const uint16_t*>(tile + Fp4Block<D>::key_scales(p.S));
  float lo[32], hi[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
  for (int t = 0; t < tokens; ++t) {
    const uint4 w4 = *reinterpret_cast<const uint4*>(tile + t * (D / 2) + cg * 16);
    const float s = bf16_to_f32(scales[t]);
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x8_t v = fp4_operand(w[i]);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float x = (float)v[c] * s;
        lo[8 * i + c] = fminf(lo[8 * i + c], x);
        hi[8 * i + c] = fmaxf(hi[8 * i + c], x);
      }
    }
  }
  if (!on) return;
  const size_t row = (((size_t)b * p.Hkv + h) * p.Pmax + j) * D + cg * 32;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t a[4], z[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      a[c] = bf16_outwards(lo[8 * i + 2 * c], false) | bf16_outwards(lo[8 * i + 2 * c + 1], false) << 16;
      z[c] = bf16_outwards(hi[8 * i + 2 * c], true) | bf16_outwards(hi[8 * i + 2 * c + 1], true) << 16;
    }
    *reinterpret_cast<uint4*>(p.page_min + row + 8 * i) = make_uint4(a[0], a[1], a[2], a[3]);
    *reinterpret_cast<uint4*>(p.page_max + row + 8 * i) = make_uint4(z[0], z[1], z[2], z[3]);
  }
}

}  // namespace ts
