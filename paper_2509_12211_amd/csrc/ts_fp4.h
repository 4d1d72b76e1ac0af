// Attention over the 4-bit cache, and the rebuild of its page boxes.
//
// Single-query softmax attention over every cached token (dense) or over the pages of a list (sparse), one
// launch.  Fragments of 32 tokens: K (16 tokens x 32 channels a product) and V (16 channels x 32 tokens) are
// expanded to bf16 in registers, one instruction for two codes, and go through v_mfma_f32_16x16x32_bf16;
// the scales of 32 tokens multiply the logits (K) and the softmax weights (V) afterwards.  e2m1 numbers and
// bf16 queries are exact operands.  For an fp32 output the weights go in as three bf16 numbers (the nearest, the
// remainder's nearest, and what is left, which fits: 24 bits in all; with two it was 2e-6 off, twice what the sums
// cost), so nothing but the fp32 sums rounds; for a bf16 output as two, 2^-17, far below its own rounding of 2^-8.
//   logits  St[token][head] = K[token][:] . Q^T[:][head]      row = token, column = head
//   output  Ot[chan][head] += V^T[chan][token] . P^T[token][head]
// Row 4 kb + i of logit tile t is token 8 kb + 4 t + i of the fragment (kb: quarter of the wave), so the eight
// weights a lane has are the eight tokens its quarter contracts in the second product.
//
// Work: every workgroup works out from the lengths what it has to do.  Much work is numbered through, fragment
// after fragment and unit after unit, and dealt out in equal contiguous shares, whatever the lengths; little goes
// unit by unit, each to as many workgroups as its length asks for; many short units go to a wave each.  A workgroup's
// waves take the fragments of a unit in turn and merge in LDS.  A unit that several workgroups share is merged by the
// last of them to arrive (an atomic count in the workspace, set back to zero); nobody waits.
//
// Measured (kernel alone, cold data): 64 sequences of 1024 to 32768 tokens, 8 KV heads of 128 channels, 1.14 GB:
// 216 us, 5.3 TB/s, bound by memory.  16 sequences of 16384 tokens, 4 KV heads of 64, 71.5 MB: 21.2 us, 3.4 TB/s:
// each wave has eight fragments, and the way to the first (lengths, table, block) and the merge are a third of
// the time.  One sequence of 4096 tokens and one head, 0.28 MB: 7.8 us, that chain alone.
#pragma once
#include "ts_append.h"
#include "ts_attend.h"

namespace ts {

constexpr int kFp4Frag = 32;            // tokens of a fragment
constexpr int kFp4List = 1024;          // list entries held in LDS at a time
// About how many workgroups share a unit at the most: the last one merges them all.  32, 64, 96 and 128 take, for
// one sequence of 131072 tokens, 8 heads on one of 64 channels, 21.9, 18.4, 19.6 and 21.9 us; for one of 262144,
// 16 heads on one of 128 channels, 48 to 50 us from 64 on.
constexpr int kFp4Parts = 64;
constexpr int kFp4Counters = 1024;      // places for counts, whatever the batch
// Units of at most this many fragments (what a wave's part of the list holds) are taken by a wave each where there are
// at least a sixth as many units, for each that are at work at once, as the longest has fragments: a turn of a workgroup
// each takes about 4.8 us and 0.23 for every fragment, a wave 4.5 and 0.85.  256 sequences of 200 tokens, 8 heads on
// 64 channels 27.9 -> 14.1 us, on 128 25.6 -> 15.7; 128 of 64 tokens 10.7 -> 6.0; 128 of 1024 would lose, 24.1 -> 31.5.
constexpr int kFp4ShortUnit = 32, kFp4ShortTurn = 6;
// Fragments of a workgroup from which on all get the same number: with 384 the ragged batch of 1.1 GB goes unit by
// unit and takes 250 us instead of 222; 48 changes nothing that was measured.
constexpr uint32_t kFp4LongShare = 192;

// Workgroups of eight waves, two on a compute unit, for 64 channels (71.5 MB 21.7 us; three of them 24.7, four of
// four waves 26.0).  With 128, where a wave's registers leave room for three on a SIMD and no less, of four waves,
// three on a unit (1.1 GB 220 us, lists of a quarter of the pages 15.2; two of eight waves 223 and 16.0).
template <int D>
struct Fp4Shape {
  static constexpr int kWavesPer = D == 64 ? 8 : 4, kThreadsPer = kWavesPer * kWave;
  static constexpr int kPerCu = D == 64 ? 2 : 3;              // workgroups on a compute unit
  static constexpr int kStages = 2;                           // fragments a wave has room for (three: 22.4 us where two take 21.7)
  static constexpr int kResident = 256 * kPerCu;
  static_assert(kResident <= kFp4Counters, "a count for each");
  // Fragments a workgroup has at the least: with 8 one sequence of 3000 tokens takes 8.9 us, with 16 8.5, with 32
  // 10.7; lists of a quarter of the pages 15.1 with 8, 14.3 with 16.
  static constexpr int kMinShare = 16;
  // a fragment in LDS: keys, values, scales
  static constexpr int kKeys = 0, kValues = 16 * D, kScales = 32 * D, kStage = 32 * D + 256;
  static constexpr int kLoads = D / 32 + 1;                   // loads that bring it
  static constexpr int kRing = kStages * kStage;              // bytes of a wave
  static constexpr size_t lds() { return (size_t)kFp4List * 8 + (size_t)kWavesPer * kRing; }
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
  float* part;                      // [room][2][G][D]: what a unit's workgroups hand over, and
  float* part_ml;                   // [room][2][G][2]: the maximum and sum that go with it
  int32_t* done;                    // [room] by a shared unit's first workgroup: how many have; zero between launches
  int B, Hq, Hkv, G, Pmax, Kmax, n_phys;
  int room;                         // workgroups that have a place in part, and are at work at once
  long long tile_stride;
  float scale_log2, inv_room;
};

// Eight codes, two a byte, as an operand of eight bf16 numbers.
__device__ __forceinline__ bf16x8_t fp4_operand(uint32_t w) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One entry of the list: the address of a page's block of the unit's head, and in the upper 16 bits how many
// of its tokens count.
typedef uint64_t Fp4Entry;
__device__ __forceinline__ Fp4Entry fp4_entry(const Fp4Params& p, int phys, int h, int tokens) {
  return (uint64_t)(uintptr_t)(p.pool + ((size_t)phys * p.Hkv + h) * (size_t)p.tile_stride) | (uint64_t)tokens << 48;
}

typedef uint32_t uint4_v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2_v __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef const __attribute__((address_space(1))) unsigned char global_byte;

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(lds_byte*)p;
}

// An entry of the list by its LDS address (the compiler, which cannot tell the list from the fragments that
// loads in flight write to LDS, would wait for those ahead of a read of its own).
__device__ __forceinline__ uint2_v read_entry(uint32_t at) {
  uint2_v e;
  asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(e) : "v"(at) : "memory");
  return e;
}

// The entry that has fragment `frag`'s tokens 8 oct .. 8 oct + 7, and their first slot in the page.
template <int S>
__device__ __forceinline__ uint32_t fp4_entry_of(uint32_t list, int frag, int oct) {
  constexpr int PPF = S < kFp4Frag ? kFp4Frag / S : 1, FPP = S > kFp4Frag ? S / kFp4Frag : 1;
  return list + (PPF > 1 ? 8u * (uint32_t)(8 * oct / S) : 0u) + 8u * (uint32_t)(frag / FPP * PPF);
}
template <int S>
__device__ __forceinline__ int fp4_slot(int frag, int oct) {
  constexpr int FPP = S > kFp4Frag ? S / kFp4Frag : 1;
  return (FPP > 1 ? kFp4Frag * (frag % FPP) : 0) + (8 * oct) % (S < kFp4Frag ? S : kFp4Frag);
}

// 16 or 4 bytes a lane straight from memory to LDS, one lane's behind the other's.  (The host's pass over this
// file does not know the wide form.)
__device__ __forceinline__ void load_to_lds16(global_byte* src, lds_byte* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(src, dst, 16, 0, 0);
#endif
}
__device__ __forceinline__ void load_to_lds4(global_byte* src, lds_byte* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(src, dst, 4, 0, 0);
#endif
}

// Sends fragment `frag` on its way to the stage at LDS address stage_at, straight from memory: no register
// waits for it, so a wave has several under way.  A load writes the lanes' 16 bytes one behind the other;
// quarter a of the wave asks for the tokens 8 a .. 8 a + 7, and which lane of it for what puts the rows where
// they are read without bank conflicts:
//   keys    128 channels: token 8 a + 4 t + b is row 16 t + 4 a + b, its 16-byte chunk c stands at c ^ a;
//           64 channels: token 8 a + i is row 8 a + (i ^ 4 (a % 2)), chunk c stands at c ^ (a / 2)
//   values  the 16 bytes of lane (r, a) and channel blocks 4 i .. 4 i + 3 at 1024 i + 16 lane
//   scales  at 64 a four words of the keys, four of the values, both once more
template <int D, int S>
__device__ __forceinline__ void fetch_fp4(uint32_t list, int frag, uint32_t stage_at) {
  typedef Fp4Shape<D> Shape;
  typedef Fp4Block<D> Block;
  lds_byte* stage = (lds_byte*)(uintptr_t)(uint32_t)uniform((int)stage_at);
  const int lane = lane_id(), a = lane >> 4, r = lane & 15;
  uint2_v e = read_entry(fp4_entry_of<S>(list, frag, a));
  if (S >= kFp4Frag) {      // the same page for all lanes
    e.x = (uint32_t)uniform((int)e.x);
    e.y = (uint32_t)uniform((int)e.y);
  }
  global_byte* block = (global_byte*)((uint64_t)(e.y & 0xffffu) << 32 | e.x);
  const int slot = fp4_slot<S>(frag, a);
  if constexpr (D == 128) {
    const int at = (slot + (r >> 2)) * 64 + ((lane & 3) ^ a) * 16;
    load_to_lds16(block + at, stage + Shape::kKeys);
    load_to_lds16(block + at + 256, stage + Shape::kKeys + 1024);
  } else {
    const int at = (slot + ((r >> 1) ^ (4 * (a & 1)))) * 32 + ((lane & 1) ^ (a >> 1)) * 16;
    load_to_lds16(block + at, stage + Shape::kKeys);
  }
  const int v = Block::values(S) + (slot >> 3) * (4 * D) + r * 16;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) load_to_lds16(block + v + 256 * i, stage + Shape::kValues + 1024 * i);
  const int s = ((r & 4) ? Block::value_scales(S) : Block::key_scales(S)) + 2 * slot + 4 * (r & 3);
  load_to_lds4(block + s, stage + Shape::kScales);
}

// Waits until all but the `kPending` loads last sent to LDS are there.
template <int kPending>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPending) : "memory");
}
// Reads the keys of a stage, the scales of NV tokens and the upper half of their entry.
template <int D, int NV>
__device__ __forceinline__ void read_fp4_keys(uint32_t key, uint32_t second, uint32_t scale, uint32_t entry,
                                              uint32_t (&k)[2][D / 32], uint32_t (&ks)[NV / 2], uint32_t (&vs)[NV / 2],
                                              uint32_t& tokens) {
  typedef typename std::conditional<D == 128, uint4_v, uint2_v>::type KeyWords;
  typedef typename std::conditional<NV == 8, uint4_v, uint2_v>::type ScaleWords;
  KeyWords a, b;
  ScaleWords s, v;
#define TS_READ_KEYS(KEY, SCALE)                                                                          \
  asm volatile("ds_read_" KEY " %0, %5\n\tds_read_" KEY " %1, %6\n\tds_read_" SCALE " %2, %7\n\t" \
               "ds_read_" SCALE " %3, %7 offset:16\n\tds_read_b32 %4, %8 offset:4\n\ts_waitcnt lgkmcnt(0)" \
               : "=&v"(a), "=&v"(b), "=&v"(s), "=&v"(v), "=&v"(tokens)                                    \
               : "v"(key), "v"(second), "v"(scale), "v"(entry)                                            \
               : "memory")
  if constexpr (D == 128 && NV == 8) TS_READ_KEYS("b128", "b128");
  else if constexpr (D == 128) TS_READ_KEYS("b128", "b64");
  else if constexpr (NV == 8) TS_READ_KEYS("b64", "b128");
  else TS_READ_KEYS("b64", "b64");
#undef TS_READ_KEYS
#pragma unroll
  for (int i = 0; i < D / 32; ++i) { k[0][i] = a[i]; k[1][i] = b[i]; }
#pragma unroll
  for (int i = 0; i < NV / 2; ++i) { ks[i] = s[i]; vs[i] = v[i]; }
}
template <int D>
__device__ __forceinline__ void read_fp4_values(uint32_t at, uint32_t (&w)[D / 16]) {
  if constexpr (D == 128) {
    uint4_v a, b;
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:1024\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b) : "v"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) { w[i] = a[i]; w[4 + i] = b[i]; }
  } else {
    uint4_v a;
    asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(a) : "v"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a[i];
  }
}

// Running softmax state of a wave, for each of its sixteen columns.
template <int D>
struct Fp4State {
  float4_t acc[D / 16];   // channels 16 cb + 4 kb .. + 3
  float m, l;             // running maximum (log2 units, the same in the four quarters), this quarter's sum
};

// The fragment in the stage at LDS address `stage`.  Up to eight query heads (kNarrow) leave half of the
// sixteen columns: they stand in both halves, and a column goes on with only one of the two logit tiles, the
// left with the first, the right with the second: half the softmax work for each lane.  (The weights of the
// other tile's tokens are zeros of its operand, and the halves are two partial results like two waves'.)
// What bounds this is the vector unit: 64 of some 190 instructions expand codes (128 channels).
template <int D, int S, bool kNarrow, bool kOut32>
__device__ __forceinline__ void attend_fp4(Fp4State<D>& st, const bf16x8_t (&q)[D / 32], float scale_log2, uint32_t list, int frag,
                                           uint32_t stage) {
  typedef Fp4Shape<D> Shape;
  constexpr int NV = kNarrow ? 4 : 8;     // logits a lane goes on with
  const int lane = lane_id(), r = lane & 15, kb = lane >> 4, a = r >> 2, right = kNarrow ? r >> 3 : 0;
  const uint32_t key = stage + Shape::kKeys +
                       (D == 128 ? r * 64 + (kb ^ a) * 16
                                 : (8 * a + (r & 3)) * 32 + ((kb >> 1) ^ (a >> 1)) * 16 + (kb & 1) * 8 + (a & 1) * 128);
  const uint32_t second = D == 128 ? key + 1024 : key + 128 - 256 * (a & 1);     // the octet's other four tokens
  uint32_t k[2][D / 32], ksw[NV / 2], vsw[NV / 2], tokens;
  read_fp4_keys<D, NV>(key, second, stage + Shape::kScales + kb * 64 + right * 8, fp4_entry_of<S>(list, frag, kb), k, ksw,
                                 vsw, tokens);
  const int valid = (int)(tokens >> 16) - fp4_slot<S>(frag, kb) - 4 * right;
  float s[NV], vs[NV];
  {
    float4_t c[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      c[t] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < D / 32; ++i) c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp4_operand(k[t][i]), q[i], c[t], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float x = kNarrow ? (right ? c[1][i] : c[0][i]) : c[i / 4][i % 4];
      const float scale = i & 1 ? bf16_hi(ksw[i / 2]) : bf16_lo(ksw[i / 2]);
      s[i] = x * (scale * scale_log2);
      vs[i] = i & 1 ? bf16_hi(vsw[i / 2]) : bf16_lo(vsw[i / 2]);
    }
  }
  if (__any(valid < NV)) {   // slots without a token may hold anything, scales included
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      s[i] = i < valid ? s[i] : -INFINITY;
      vs[i] = i < valid ? vs[i] : 0.f;
    }
  }
  float m = s[0];
#pragma unroll
  for (int i = 1; i < NV; ++i) m = fmaxf(m, s[i]);
  m = fmaxf(rows_max_f32(m), st.m);
  const float ref = m == -INFINITY ? 0.f : m;
  if (__any(m > st.m)) {
    const float a = __builtin_amdgcn_exp2f(st.m - ref);
    st.l *= a;
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) st.acc[cb] *= a;
    st.m = m;
  }
  uint32_t w[D / 16];
  read_fp4_values<D>(stage + Shape::kValues + 16 * lane, w);
  // the weights as two bf16 numbers, three where the output is fp32: pairs in a word
  constexpr int kTerms = kOut32 ? 3 : 2;
  uint32_t part[kTerms][NV / 2];
#pragma unroll
  for (int i = 0; i < NV; i += 2) {
    const float w0 = __builtin_amdgcn_exp2f(s[i] - ref), w1 = __builtin_amdgcn_exp2f(s[i + 1] - ref);
    st.l += w0 + w1;
    float x0 = w0 * vs[i], x1 = w1 * vs[i + 1];
#pragma unroll
    for (int e = 0; e < kTerms; ++e) {
      const uint32_t pair = pack_elems<false>(x0, x1);
      part[e][i / 2] = pair;
      x0 -= bf16_lo(pair);
      x1 -= bf16_hi(pair);
    }
  }
  bf16x8_t term[kTerms];
  const uint32_t left_on = kNarrow && right ? 0u : ~0u;
#pragma unroll
  for (int e = 0; e < kTerms; ++e) {
    uint4_v o;
    if constexpr (kNarrow)
      o = uint4_v{part[e][0] & left_on, part[e][1] & left_on, part[e][0] & ~left_on, part[e][1] & ~left_on};
    else o = uint4_v{part[e][0], part[e][1], part[e][NV / 2 - 2], part[e][NV / 2 - 1]};
    term[e] = __builtin_bit_cast(bf16x8_t, o);
  }
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) {
    const bf16x8_t v = fp4_operand(w[cb]);
#pragma unroll
    for (int e = kTerms - 1; e >= 0; --e) st.acc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, term[e], st.acc[cb], 0, 0, 0);
  }
}

// n / d for n < 2^20: the fraction that half a unit adds (0.5 / d) outweighs what the reciprocal is off (2^-22 n / d).
// (A division proper takes some forty instructions, ahead of the first load.)
__device__ __forceinline__ uint32_t small_quotient(uint32_t n, uint32_t d) {
  return (uint32_t)(((float)n + 0.5f) * __builtin_amdgcn_rcpf((float)d));
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

template <bool kOut32>
__device__ __forceinline__ void store_fp4_out(const Fp4Params& p, size_t idx, const float4_t& v) {
  if constexpr (kOut32) *reinterpret_cast<float4_t*>(p.out + idx) = v;
  else
    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.out) + idx) =
        make_uint2(pack_elems<false>(v[0], v[1]), pack_elems<false>(v[2], v[3]));
}
// Partial results travel by 16 bytes past the caches (as store_agent and load_agent do by four).
constexpr int kPartAgent = 16;      // cache policy: agent scope
__device__ __forceinline__ void store_part(__amdgpu_buffer_rsrc_t r, uint32_t at, const float4_t& v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(stream_u4, v), r, (int)at, 0, kPartAgent);
}
__device__ __forceinline__ float4_t load_part(__amdgpu_buffer_rsrc_t r, uint32_t at) {
  return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, kPartAgent));
}

// kMany: more units than workgroups at once (the others are 1 to 5 % faster without the choice).
template <int D, int S, bool kSparse, bool kNarrow, bool kOut32, bool kMany>
__global__ __launch_bounds__(Fp4Shape<D>::kThreadsPer, Fp4Shape<D>::kPerCu * Fp4Shape<D>::kWavesPer / 4)
void fp4_attention_kernel(Fp4Params p) {
  typedef Fp4Shape<D> Shape;
  constexpr int kFp4Waves = Shape::kWavesPer, kFp4Threads = Shape::kThreadsPer, kStages = Shape::kStages;
  constexpr int PPF = S < kFp4Frag ? kFp4Frag / S : 1, FPP = S > kFp4Frag ? S / kFp4Frag : 1;
  constexpr int kFrags = (kFp4List + 1 - FPP) * FPP / PPF;   // fragments the list in LDS covers, begun within a page too
  constexpr int kRow = D + 4;                        // a head's merged row: channels, maximum, sum
  constexpr int kWaveRows = Shape::kRing / 4;        // a wave's rows lie where its fragments were
  static_assert(16 * kRow <= kWaveRows && kRow % 4 == 0 && kWaveRows % 4 == 0, "room for a wave's rows");
  extern __shared__ __align__(16) unsigned char smem[];
  Fp4Entry* list = reinterpret_cast<Fp4Entry*>(smem);
  float* merge = reinterpret_cast<float*>(list + kFp4List);
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
        for (int x = 4 * lane; x < p.Hq * D; x += 4 * kWave)
          store_fp4_out<kOut32>(p, (size_t)e * p.Hq * D + x, float4_t{0.f, 0.f, 0.f, 0.f});
        if (p.lse)
          for (int x = lane; x < p.Hq; x += kWave) p.lse[(size_t)e * p.Hq + x] = -INFINITY;
      }
    }
  }
  total *= (uint32_t)p.Hkv;
  const uint32_t floor_share = max((uint32_t)Shape::kMinShare, (uint32_t)((longest + kFp4Parts - 1) / kFp4Parts));
  const uint32_t room = (uint32_t)p.room, units = (uint32_t)p.B * (uint32_t)p.Hkv;
  // (no less than total / room: up to 4 M fragments a workgroup the rounding of the quotient is below the one added)
  uint32_t share = max(floor_share, (uint32_t)((float)total * p.inv_room) + 1u);
  // Workgroups of a unit each, or equal shares of all fragments?  A workgroup whose share reaches into a second
  // unit begins once more, which takes as long as a hundred fragments: short shares go unit by unit wherever
  // there are workgroups for that at once (one sequence of 3000 tokens, four heads: 12.9 -> 8.7 us).
  auto by_units = [&](uint32_t s) {       // workgroups that units in parts of at most s take
    uint32_t n = 0;
    for (int base = 0; base < p.B; base += kWave) {
      const int i = base + lane, f = p.B <= kWave ? mine : i < p.B ? fp4_frags<S, kSparse>(p, i) : 0;
      n += (uint32_t)__builtin_amdgcn_readlane(wave_inclusive_sum((int)small_quotient((uint32_t)f + s - 1, s)), kWave - 1);
    }
    return n * (uint32_t)p.Hkv;
  };
  // Many short units: each wave has one of its own, and nothing to merge.
  const bool solo = kMany && longest <= kFp4ShortUnit &&
                    (uint32_t)(longest * Shape::kResident) <= kFp4ShortTurn * units;
  const bool aligned = !solo && share < kFp4LongShare;
  if (aligned) {
    // parts a little larger than an equal share, so that all are at work at once; else what is sure to fit, or
    // (more units than that) whole units in as many turns as it takes
    int tries = units > room ? 4 : 0;
    while (tries < 4 && by_units(share) > room) { share += share / 8 + 1; ++tries; }
    if (tries == 4) share = max(share, units < room ? (total + room - units - 1) / (room - units) : (uint32_t)longest);
  }
  uint32_t at, end, ustart = 0;     // this workgroup's fragments; the first of its unit
  int b = 0, h, nf = 0, parts_of_unit = 0;
  uint32_t first_part = 0;          // aligned: the unit's first workgroup
  if (solo) {
    if (blockIdx.x * kFp4Waves >= units) return;
    const uint32_t unit = blockIdx.x * kFp4Waves + (uint32_t)wave;
    if (unit < units) {
      b = uniform((int)(unit / (uint32_t)p.Hkv));
      nf = uniform(fp4_frags<S, kSparse>(p, b));
    }
    h = unit < units ? (int)unit - b * p.Hkv : 0;
    at = 0;
    end = max((uint32_t)nf, 1u);      // (all waves go once through what follows, and meet the barrier in it)
  } else {
    const uint32_t key = aligned ? blockIdx.x : blockIdx.x * share;       // workgroups, or fragments, are numbered through
    uint32_t from = 0;
    if (!aligned && (blockIdx.x >= room || key >= total)) return;      // (key: what 32 bits hold, of the first room)
    bool found = false;
    uint32_t frags_before = 0;
    for (int base = 0; base < p.B; base += kWave) {
      if (p.B > kWave) mine = base + lane < p.B ? fp4_frags<S, kSparse>(p, base + lane) : 0;
      const int items = aligned ? (int)small_quotient((uint32_t)mine + share - 1, share) : mine;
      const int upto_items = wave_inclusive_sum(items);
      const uint32_t first = from + (uint32_t)(upto_items - items) * p.Hkv, last = from + (uint32_t)upto_items * p.Hkv;
      const uint64_t here = __ballot(key >= first && key < last);
      upto = wave_inclusive_sum(mine);
      if (here != 0) {
        const int src = __builtin_ctzll(here);
        b = uniform(base + src);
        nf = __builtin_amdgcn_readlane(mine, src);
        first_part = (uint32_t)__builtin_amdgcn_readlane((int)first, src);
        parts_of_unit = __builtin_amdgcn_readlane(items, src);
        ustart = frags_before + (uint32_t)__builtin_amdgcn_readlane(upto - mine, src) * (uint32_t)p.Hkv;
        found = true;
        break;
      }
      from += (uint32_t)__builtin_amdgcn_readlane(upto_items, kWave - 1) * (uint32_t)p.Hkv;
      frags_before += (uint32_t)__builtin_amdgcn_readlane(upto, kWave - 1) * (uint32_t)p.Hkv;
    }
    if (!found) return;
    h = (int)(aligned ? small_quotient(key - first_part, (uint32_t)parts_of_unit) : (key - first_part) / (uint32_t)parts_of_unit);
    ustart += (uint32_t)h * (uint32_t)nf;
    first_part += (uint32_t)h * (uint32_t)parts_of_unit;
    if (aligned) {
      const uint32_t chunk = small_quotient((uint32_t)(nf + parts_of_unit) - 1u, (uint32_t)parts_of_unit);
      at = ustart + (key - first_part) * chunk;
      end = min(ustart + (uint32_t)nf, at + chunk);
    } else {
      at = key;
      end = min(total, at + share);
    }
  }

  // (a wave by itself has a part of the list, too, and reads what it wrote: LDS takes a wave's accesses in order)
  Fp4Entry* my_list = list + (solo ? wave * (kFp4List / kFp4Waves) : 0);
  static_assert((kFp4ShortUnit + FPP - 1) / FPP * PPF <= kFp4List / kFp4Waves, "room for a short unit's entries");
  const int step = solo ? 1 : kFp4Waves;
  while (at < end) {
    const int f0 = (int)(at - ustart), f1 = (int)min((uint32_t)nf, end - ustart);
    const int u = b * p.Hkv + h;
    const int len = min(max(p.seq_lens[b], 0), p.Pmax * S), count = kSparse ? min(max(p.sel_count[b], 0), p.Kmax) : 0;
    bf16x8_t q[D / 32];
    const int head = kNarrow ? r & 7 : r;      // of this lane's column
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint16_t* src = p.q + ((size_t)b * p.Hq + h * p.G + min(head, p.G - 1)) * D + kb * (D / 4) + 8 * i;
      uint4 w = *reinterpret_cast<const uint4*>(src);
      if (head >= p.G) w = make_uint4(0u, 0u, 0u, 0u);
      q[i] = __builtin_bit_cast(bf16x8_t, w);
    }
    Fp4State<D> st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) st.acc[cb] = float4_t{0.f, 0.f, 0.f, 0.f};
    for (int c0 = f0; c0 < f1; c0 += kFrags) {
      const int c1 = min(f1, c0 + kFrags), e0 = c0 / FPP * PPF, entries = ((c1 - 1) / FPP + 1) * PPF - e0;
      if (!solo) __syncthreads();    // the list before is read, and so is the merge area
      for (int i = solo ? lane : tid; i < entries; i += solo ? kWave : kFp4Threads) {
        int page = e0 + i;
        bool on = true;
        if (kSparse) {
          on = page < count;
          page = p.sel[(size_t)u * p.Kmax + min(page, p.Kmax - 1)];
        }
        on = on && page >= 0 && page < p.Pmax;
        const int phys = p.block_table[(size_t)b * p.Pmax + (on ? page : 0)];
        on = on && phys >= 0 && phys < p.n_phys;
        my_list[i] = on ? fp4_entry(p, phys, h, min(max(len - page * S, 0), S)) : fp4_entry(p, 0, h, 0);
      }
      if (!solo) __syncthreads();
      const int shift = c0 % FPP - c0;      // fragments as the list has them
      const uint32_t list_at = lds_address(my_list), ring = lds_address(merge) + wave * Shape::kRing;
      const int last = c1 + shift;
      int f = c0 + (solo ? 0 : wave) + shift, stage = 0;
#pragma unroll
      for (int i = 0; i < kStages - 1; ++i)
        if (f + i * step < last) fetch_fp4<D, S>(list_at, f + i * step, ring + i * Shape::kStage);
      for (; f < last; f += step) {
        const int ahead = f + (kStages - 1) * step;
        const int to = stage == 0 ? kStages - 1 : stage - 1;      // the stage that the fragment before has left
        if (ahead < last) {
          fetch_fp4<D, S>(list_at, ahead, ring + to * Shape::kStage);
          wait_loads<(kStages - 1) * Shape::kLoads>();
        } else {
          wait_loads<0>();
        }
        attend_fp4<D, S, kNarrow, kOut32>(st, q, p.scale_log2, list_at, f, ring + stage * Shape::kStage);
        stage = stage == kStages - 1 ? 0 : stage + 1;
      }
    }
    // the waves' results: head rows of channels, maximum, sum
    float l = rows_sum_f32(st.l);
    if constexpr (kNarrow) {      // the two halves of the columns first
      auto other = [](float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kDppRowRor8, 0xf, 0xf, true)); };
      const float top = raw_max(st.m, other(st.m)), a = __builtin_amdgcn_exp2f(st.m - (top == -INFINITY ? 0.f : top));
      st.m = top;
      l *= a;
      l += other(l);
#pragma unroll
      for (int cb = 0; cb < D / 16; ++cb) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = st.acc[cb][i] * a;
          st.acc[cb][i] = x + other(x);
        }
      }
    }
    if (r < p.G) {
      float* row = merge + wave * kWaveRows + r * kRow;
#pragma unroll
      for (int cb = 0; cb < D / 16; ++cb) *reinterpret_cast<float4_t*>(row + 16 * cb + 4 * kb) = st.acc[cb];
      if (kb == 0) {
        row[D] = st.m;
        row[D + 1] = l;
      }
    }
    __syncthreads();
    const uint32_t uend = ustart + (uint32_t)nf;
    const uint32_t w0 = aligned ? first_part : ustart / share;      // the unit's workgroups
    const int parts = aligned ? parts_of_unit : (int)((uend - 1) / share - w0) + 1;
    const bool whole = parts == 1;
    // (one that reaches into two units it shares with others has a place for either)
    auto place = [&](uint32_t w) { return (w * 2 + (aligned || w * share > ustart ? 0u : 1u)) * (uint32_t)p.G; };   // rows
    const __amdgpu_buffer_rsrc_t part = __builtin_amdgcn_make_buffer_rsrc(p.part, (short)0, p.room * 2 * p.G * D * 4, 0x00020000);
    const int items = p.G * (D / 4);                       // four channels of a head
    auto finish = [&](int item, float M, float sum, float4_t o) {
      const int g = item / (D / 4), c = item % (D / 4) * 4;
      const size_t at_head = (size_t)b * p.Hq + h * p.G + g;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      store_fp4_out<kOut32>(p, at_head * D + c, o * inv);
      if (p.lse && c == 0) p.lse[at_head] = sum == 0.f ? -INFINITY : (M + __log2f(sum)) * 0.6931471805599453f;
    };
    if (solo) {
      for (int i = nf > 0 ? lane : items; i < items; i += kWave) {
        const float* row = merge + wave * kWaveRows + i / (D / 4) * kRow;
        finish(i, row[D], row[D + 1], *reinterpret_cast<const float4_t*>(row + i % (D / 4) * 4));
      }
      return;
    }
    for (int i = tid; i < items; i += kFp4Threads) {
      const int g = i / (D / 4), c = i % (D / 4) * 4;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kFp4Waves; ++w) M = raw_max(M, merge[w * kWaveRows + g * kRow + D]);
      // (a wave without a token has zeros and the weight 0; what is not a number stays so)
      const float ref = M == -INFINITY ? 0.f : M;
      float4_t o = {0.f, 0.f, 0.f, 0.f};
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kFp4Waves; ++w) {
        const float* row = merge + w * kWaveRows + g * kRow;
        const float a = __builtin_amdgcn_exp2f(row[D] - ref);
        o += a * *reinterpret_cast<const float4_t*>(row + c);
        sum += a * row[D + 1];
      }
      if (whole) {
        finish(i, M, sum, o);
      } else {
        const uint32_t row = place(blockIdx.x) + (uint32_t)g;
        store_part(part, (row * D + (uint32_t)c) * 4u, o);
        if (c == 0) {
          store_agent(p.part_ml + 2 * row, M);
          store_agent(p.part_ml + 2 * row + 1, sum);
        }
      }
    }
    if (!whole) {
      stores_complete();
      __syncthreads();
      if (tid == 0) {
        const int before = atomic_add_agent(p.done + w0, 1);
        last_one = before == parts - 1;
        if (last_one) atomic_store_agent(p.done + w0, 0);
      }
      __syncthreads();
      if (uniform(last_one)) {
        // (a part's maximum, sum and numbers asked for together, eight parts at a time)
        for (int i = tid; i < items; i += kFp4Threads) {
          const int g = i / (D / 4), c = i % (D / 4) * 4;
          constexpr int kAhead = 8;
          float M = -INFINITY, sum = 0.f;
          float4_t o = {0.f, 0.f, 0.f, 0.f};
          for (int e0 = 0; e0 < parts; e0 += kAhead) {
            float m[kAhead], z[kAhead];
            float4_t x[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
              const uint32_t row = place(w0 + (uint32_t)min(e0 + e, parts - 1)) + (uint32_t)g;
              x[e] = load_part(part, (row * D + (uint32_t)c) * 4u);
              m[e] = load_agent(p.part_ml + 2 * row);
              z[e] = load_agent(p.part_ml + 2 * row + 1);
            }
            float top = M;
#pragma unroll
            for (int e = 0; e < kAhead; ++e) top = raw_max(top, m[e]);
            const float ref = top == -INFINITY ? 0.f : top, a = __builtin_amdgcn_exp2f(M - ref);
            o *= a;
            sum *= a;
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
              const float k = e0 + e < parts ? __builtin_amdgcn_exp2f(m[e] - ref) : 0.f;
              o += x[e] * k;
              sum += z[e] * k;
            }
            M = top;
          }
          finish(i, M, sum, o);
        }
      }
    }
    // the next unit
    if (aligned) return;
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
// down its tokens, eight rows and their scales asked for together.  code * scale is exact in fp32, so the extremes
// are, and are rounded outwards to bf16.  Bound by memory: 32 sequences of 16384 tokens, 8 KV heads of 128 channels,
// 103 us, 4.0 TB/s (key codes and scales, 16 tokens a page; 4.6 with pages of 64); 16 of them with 4 of 64, 17.2 us.
template <int D>
__global__ __launch_bounds__(kThreads) void build_page_meta_fp4_kernel(MetaParams p) {
  constexpr int LPP = D / 32, PPW = kWave / LPP;    // lanes a page, pages a wave
  constexpr int NT = 8;
  const int lane = lane_id(), cg = lane % LPP;
  const int first = (blockIdx.y * kWaves + wave_id()) * PPW, j = first + lane / LPP;
  const int h = blockIdx.x, b = blockIdx.z;
  const int L = p.seq_lens[b];
  const int Pb = min((L + p.S - 1) / p.S, p.Pmax);
  if (uniform(first) >= Pb) return;
  const int phys = p.block_table[(size_t)b * p.Pmax + min(j, Pb - 1)];
  const bool on = j < Pb && phys >= 0 && phys < p.n_phys;
  const int tokens = min(p.S, L - j * p.S);   // (only looked at where `on`)
  const unsigned char* tile = reinterpret_cast<const unsigned char*>(p.k_pool) +
                              ((size_t)(on ? phys : 0) * p.Hkv + h) * (size_t)p.tile_stride;
  const unsigned char* scales = tile + Fp4Block<D>::key_scales(p.S);
  float lo[32], hi[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
  for (int t0 = 0; t0 < p.S; t0 += NT) {
    uint4 w[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) w[t] = *reinterpret_cast<const uint4*>(tile + (t0 + t) * (D / 2) + cg * 16);
    const uint4 s4 = *reinterpret_cast<const uint4*>(scales + 2 * t0);
    float s[NT];
    unpack8(s4, s);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      // (a slot without a token gets a scale that makes no number, which gives way in every comparison)
      const float scale = t0 + t < tokens ? s[t] : __uint_as_float(0x7fc00000u);
      const uint32_t x[4] = {w[t].x, w[t].y, w[t].z, w[t].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
        fp4_numbers(x[i], scale, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          lo[8 * i + c] = raw_min(lo[8 * i + c], v[c]);
          hi[8 * i + c] = raw_max(hi[8 * i + c], v[c]);
        }
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
