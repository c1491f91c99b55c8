// Attention over the 4-bit paged cache (lilicorr_window_attention4) and the attention weight that its keys have got
// (lilicorr_key_weights).
//
// A row is one query head of one token; the query heads of a key head are neighbours, so the rows of a request and key
// head are its tokens' groups one after the other. A wave holds RT blocks of 16 rows and goes through tiles of 32
// keys. Tiles come by way of LDS, in rings of copies that go on while a tile is used, where widths are powers of two and
// pages multiples of 16 keys (Ring4, Shared4); elsewhere loads go to registers, a tile ahead.
//
// 16 x 16 x 32 matrix instructions. The order of the summed index is free as long as both operands have the same, so
// each operand is what a lane can load at once. Lane l is c = l % 16 and g = l / 16.
//   Scores S^T[key][row] = K . Q^T. Lane (c, g) has of key c (and 16 + c) the g-th quarter of the head: with heads of
//   128 that is one 16-byte load and one scale, eight conversions a product. The result leaves lane (c, g) with row c
//   and the keys 4 g .. 4 g + 3 (and 16 more).
//   Output O^T[dim][row] = V^T . P^T sums over keys, of which lane (c, g) has just those eight probabilities. So it
//   loads of the same eight keys the c-th sixteenth of the head, 4 bytes with heads of 128: after conversion a pair of
//   neighbouring elements of one key, two v_perm bring two keys' elements together. Product i of D / 16
//   has element i of every sixteenth, so a lane ends with whole runs of its row's output: D / 4 elements at D / 4 g.
// Converted elements are exact in bf16, scale and all.
//
// Softmax: running maximum and sum in fp32, as in the 16-bit cache's attention: powers of two against a reference that
// is a whole number and follows the maximum only when that has grown by more than 2^8. Probabilities go to the second product
// rounded to bf16, and with fp16 outputs as two bf16 terms (with one, a ragged batch was 0.001 off, five times what the
// output's own rounding is). The output's sum is that of the rounded probabilities (weights add up to one), the
// logarithm's that of the unrounded ones.
//
// NaN blocks of values: 0 * NaN is NaN, so where not all rows see a key, its NaN blocks become zeros for the product
// and the rows that do see it are marked, block by block, and get their NaN at the end.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache4.hpp"
#include "common.hpp"
#include "paged.hpp"

namespace lilicorr {
namespace {

typedef __attribute__((address_space(3))) f32x4_t* lds_f32x4_t;

// the largest of three, NaN if one of them is (a row that sees one is NaN anyway). As operations that the compiler
// knows: it puts no wait between a matrix instruction and inline assembly that reads its result.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

struct Attn4Args {
  const uint16_t* q;
  const unsigned char *k, *v, *ks, *vs;
  uint16_t* out;
  float* lse;
  float* part_o;     // [slots][tokens * heads][d], where the keys are split
  f32x4_t* part_ml;  // [slots][tokens * heads]: maximum (powers of two), sums of rounded and unrounded powers
  const int32_t *table, *starts, *totals;
  int64_t q_stride, rows;  // rows = tokens * heads
  int64_t head_stride;     // bytes
  int N, pages, table_width;
  uint32_t group_mul, group_shift;           // n / group, likewise
  uint32_t page_mul, page_shift, page_size;  // n / page_size = (n * page_mul) >> page_shift
  int tokens, heads, kv_heads, group, d;
  int64_t page_stride, token_stride;  // bytes
  int tiles, chunk, most, items;      // row tiles; 32-key tiles of a chunk, and of all; tiles * heads * chunks
  int spread, split;
  int max_tokens, max_length, window, sinks, causal;
  float scale2;  // scale * log2 e
  // lilicorr_key_weights
  const float* lse_in;
  float* weights;
  float decay;
};

template <typename T_, int D_, int RT_, int WH_, int WR_, int WK_, bool RING_>
struct Attn4Config {
  typedef T_ T;
  static constexpr int D = D_;    // heads of D elements or fewer
  static constexpr int RT = RT_;  // blocks of 16 rows of a wave
  static constexpr int WH = WH_, WR = WR_, WK = WK_;  // waves of key heads by waves of rows by waves of keys
  static constexpr bool RING = RING_;  // tiles by way of LDS
  // Several key heads in a workgroup: one ring for all. Rows of one head (prefill) do better each with their own copies than
  // with a barrier a tile: 1966 us against 2095.
  static constexpr bool kShared = WK == 1 && WH > 1;
  // Stages of a ring. Two are enough where a compute unit has two workgroups or three (256 tokens 445 us, 463 with three; 64
  // blocks 306, 311 with three).
  static constexpr int NS = D <= 64 ? 4 : 2;
  static constexpr int kWaves = WH * WR * WK, kThreads = kWaves * kWave;
  static constexpr int BM = 16 * RT * WR;
  static constexpr int ND = D / 16;  // output products
  static constexpr int KW = D / 32;  // 32-bit words that a lane has of a key
  static constexpr int KS = D <= 128 ? 1 : 2;  // scales of them
  static constexpr int VB = D / 32;  // bytes that a lane has of a value
  static constexpr int kTerms = Query<T>::kTerms;
  // the waves' partial outputs, in the order of their lanes, and sums
  static constexpr uint32_t kOut = kWaves * RT * ND * kWave * 16, kSums = kWaves * RT * kWave * 16;
  static constexpr uint32_t kJoin = WK > 1 ? kOut + kSums : 0;
  // Waves of a SIMD that the registers are given out for: two or more keep the accumulators where the vector unit reaches
  // them. Tiles by way of registers need more of those: with three waves they spill (64 requests of one token, heads of
  // 96: 463 us, 98 with two).
  static constexpr int kSimdWaves = D > 128 || (RT == 2 && D > 64 && kTerms > 1)         ? 1
                                    : RT == 1 && kTerms == 1 && (RING || D <= 64) ? 3
                                                                                         : 2;
};

// What a wave has under way of a tile of 32 keys
template <typename C>
struct Raw4 {
  uint32_t k[2][C::KW], ks[2][C::KS];
  uint32_t v[8][C::VB > 4 ? 2 : 1], vs[8];
};

__device__ __forceinline__ int entry4(const Attn4Args& a, int j) {
  return (int)(((uint64_t)(uint32_t)j * a.page_mul) >> a.page_shift);
}

// What a lane has of a key and a value, where loads go straight to registers
template <typename C>
struct Places4 {
  uint32_t k_lane, v_lane;              // bytes of the lane's part within a key's, a value's codes
  uint32_t k_scale, k_scale2, v_scale;  // and within its scales
  uint32_t k_more;                      // from there to the second 16 bytes of a wide head's key

  __device__ __forceinline__ void set(const Attn4Args& a) {
    const int lane = lane_id(), c = lane & 15, g = lane >> 4;
    // past the width of the head: its first part, which meets zeros of the queries, or goes to no output
    const int ke = g * (C::D / 4), ve = c * (C::D / 16);
    k_lane = ke < a.d ? ke / 2 : 0;
    k_scale = ke < a.d ? ke / kBlock4 : 0;
    k_more = C::D > 128 && ke + kBlock4 < a.d ? 16 : 0;
    k_scale2 = k_scale + k_more / 16;
    v_lane = ve < a.d ? ve / 2 : 0;
    v_scale = ve < a.d ? ve / kBlock4 : 0;
  }
};

template <int BYTES>
__device__ __forceinline__ void load_bytes(const unsigned char* p, uint32_t* to) {
  if constexpr (BYTES == 2) {
    to[0] = *reinterpret_cast<const uint16_t*>(p);
  } else if constexpr (BYTES == 4) {
    to[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (BYTES == 8) {
    const u32x2_t w = *reinterpret_cast<const u32x2_t*>(p);
    to[0] = w[0];
    to[1] = w[1];
  } else {
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = w[i];
  }
}

// Asks for the keys (and with VALUES the values) of a tile of 32, any pages and widths. `page` (one register) is the page
// of key lane % 32. The second half of a wide head's part of a key lies 16 bytes on, or is its first where the head
// ends.
template <typename C, bool VALUES>
__device__ __forceinline__ void load4(const Attn4Args& a, const Places4<C>& pl, const unsigned char* k,
                                      const unsigned char* v, const unsigned char* ks, const unsigned char* vs,
                                      int tile, int page, Raw4<C>& r) {
  const int lane = lane_id(), c = lane & 15, g = lane >> 4;
  const int j = tile * 32 + (lane & 31);
  const uint64_t mine = (uint64_t)(uint32_t)page * (uint64_t)a.page_stride +
                        (uint64_t)((uint32_t)j - (uint32_t)entry4(a, j) * a.page_size) * (uint64_t)a.token_stride;
  const uint32_t lo = (uint32_t)(mine >> 4), hi = (uint32_t)(mine >> 36);  // in 16 bytes
  auto of = [&](int key) {
    const uint32_t x = (uint32_t)__builtin_amdgcn_ds_bpermute(key * 4, (int)lo);
    const uint32_t y = (uint32_t)__builtin_amdgcn_ds_bpermute(key * 4, (int)hi);
    return (uint64_t)y << 32 | x;
  };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint64_t at = of(16 * h + c);
    load_bytes<C::D <= 128 ? C::D / 8 : 16>(k + (at << 4) + pl.k_lane, r.k[h]);
    if constexpr (C::D > 128) load_bytes<16>(k + (at << 4) + pl.k_lane + pl.k_more, r.k[h] + 4);
    r.ks[h][0] = ks[at + pl.k_scale];
    if constexpr (C::KS > 1) r.ks[h][1] = ks[at + pl.k_scale2];
    if constexpr (VALUES) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint64_t to = of(16 * h + 4 * g + e);
        load_bytes<C::VB>(v + (to << 4) + pl.v_lane, r.v[4 * h + e]);
        r.vs[4 * h + e] = vs[to + pl.v_scale];
      }
    }
  }
}

// ---- the ring ------------------------------------------------------------------------------------
// The rule (pages of a multiple of 16 tokens, heads of 64, 128 or 256): a wave copies its tiles to LDS, 16 bytes a lane
// and neighbouring lanes neighbouring bytes, NS of them in turn. Loads straight to registers in the operands' layout take four
// times as long: a load instruction costs the address unit 16 steps and more however little it brings, and lanes
// that are neighbours there have different keys (counted: 336 cache accesses a tile; 256 requests of one token 603 us).
// 16 keys lie in one page, so a copy has a uniform base; pieces of 16 bytes are permuted, and values' rows too, so that
// the operands' reads meet no bank conflicts.
typedef __attribute__((address_space(3))) unsigned char* lds_t;
typedef __attribute__((address_space(3))) uint32_t* lds_u32_t;
typedef __attribute__((address_space(3))) float* lds_float_t;
typedef __attribute__((address_space(3))) u32x4_t* lds_u32x4_t;

// Copies to LDS at `dst` in lane order, counted by vmcnt alone; no register is loaded, so none is in flight. WIDE: 16
// bytes a lane from a uniform base and the lane's offset. Else 4 bytes, or with SHORT 2 in 4, from the lane's address.
__device__ __forceinline__ void copy16(lds_t dst, const unsigned char* base, uint32_t lane) {
  const uint32_t at = uniform32((uint32_t)(uintptr_t)dst);
  __asm__ volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(at), "v"(lane), "s"(base) : "memory");
}
__device__ __forceinline__ void copy16(lds_t dst, const unsigned char* from) {
  const uint32_t at = uniform32((uint32_t)(uintptr_t)dst);
  __asm__ volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(at), "v"(from) : "memory");
}
template <bool SHORT>
__device__ __forceinline__ void copy4(lds_t dst, const unsigned char* from) {
  const uint32_t at = uniform32((uint32_t)(uintptr_t)dst);
  if constexpr (SHORT)
    __asm__ volatile("s_nop 0\n\tglobal_load_lds_ushort %1, off" ::"{m0}"(at), "v"(from) : "memory");
  else
    __asm__ volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(at), "v"(from) : "memory");
}

// (by value: a choice between two members would put the structure into memory)
template <typename X>
__device__ __forceinline__ X pick(bool first, X a, X b) {
  return first ? a : b;
}

// Where tiles lie. Offsets are bytes of codes from the head's first one on.
template <bool VALUES>
struct Where4 {
  static constexpr int kBatch = kWave / 2;  // tiles whose places the lanes have, a half each
  const int32_t* trow;
  int e_last;      // last entry that there is
  int base;        // first tile of the batch
  uint64_t off;    // of this lane's half
  int64_t w;       // and its first key's weight, without values
  uint64_t valid;  // the halves whose page is there
  uint32_t ahead;  // page of the next batch's half
  uint64_t seen;   // two bits a tile that was found, the last one's lowest

  struct At {  // a tile's two halves
    uint64_t off0, off1;
    int64_t w0, w1;  // without values
  };
  // The s-th of `tiles` tiles, the number of which in the sequence tile_of gives; one after the other. 64 lanes work the
  // places of 32 tiles out at once, which costs a tile four v_readlane (a tile's places by scalar instructions
  // were 70 of them, one after the other).
  template <typename F>
  __device__ __forceinline__ int entry_at(const Attn4Args& a, int first, int tiles, const F& tile_of, int& j) const {
    j = tile_of(min(first + lane_id() / 2, tiles - 1)) * 32 + 16 * (lane_id() & 1);
    return min(entry4(a, j), e_last);
  }
  template <typename F>
  __device__ __forceinline__ void batch(const Attn4Args& a, int first, int tiles, const F& tile_of, int head) {
    base = first;
    int j;
    entry_at(a, base, tiles, tile_of, j);
    uint32_t page = ahead;
    valid = __ballot(page < (uint32_t)a.pages);
    if (page >= (uint32_t)a.pages) page = 0;
    const uint32_t o = (uint32_t)j - (uint32_t)entry4(a, j) * a.page_size;
    off = (uint64_t)page * (uint64_t)a.page_stride + (uint64_t)o * (uint64_t)a.token_stride;
    if constexpr (!VALUES) w = ((int64_t)page * a.kv_heads + head) * a.page_size + o;
    if (base + kBatch < tiles) ahead = (uint32_t)trow[entry_at(a, base + kBatch, tiles, tile_of, j)];
  }
  // before the first find(): everything that has been asked for so far is there afterwards, so that the compiler puts no
  // wait for it among the copies, which it does not see
  template <typename F>
  __device__ __forceinline__ void begin(const Attn4Args& a, const int32_t* row, int keys, int tiles, const F& tile_of,
                                        int head = 0) {
    int j;
    trow = row;
    e_last = entry4(a, keys - 1);
    ahead = (uint32_t)trow[entry_at(a, 0, tiles, tile_of, j)];
    seen = 0;
    batch(a, 0, tiles, tile_of, head);
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0) alone
  }
  template <typename F>
  __device__ __forceinline__ At find(const Attn4Args& a, int s, int tiles, const F& tile_of, int head = 0) {
    s = min(s, tiles - 1);
    if (__builtin_expect(s >= base + kBatch, 0)) batch(a, base + kBatch, tiles, tile_of, head);
    const int q = 2 * (s - base);
    At r;
    r.off0 = readlane64(off, q);
    r.off1 = readlane64(off, q + 1);
    if constexpr (!VALUES) {
      r.w0 = (int64_t)readlane64((uint64_t)w, q);
      r.w1 = (int64_t)readlane64((uint64_t)w, q + 1);
    }
    seen = seen << 2 | (valid >> q & 3);
    return r;
  }
  // which of the 32 keys of the tile that was found `back` tiles before the last one lie on pages that are there
  __device__ __forceinline__ uint32_t there(int back) const {
    const uint32_t b = (uint32_t)(seen >> (2 * back));
    return ((b & 1) ? 0xffffu : 0u) | ((b & 2) ? 0xffff0000u : 0u);
  }
};

template <typename C, bool VALUES>
struct Ring4 {
  static constexpr int D = C::D, RB = D / 2;      // bytes of a key's codes
  static constexpr int CPR = D / 32;              // 16-byte pieces of them
  static constexpr int KI = 32 * CPR / kWave;     // copies of a tile's keys, D = 64, 128, 256: 1, 2, 4
  static constexpr int SB = D <= 128 ? 4 : 8;     // bytes of a key's scales, in LDS
  static constexpr uint32_t kV = 32 * RB, kS = VALUES ? 2 * kV : kV;
  static constexpr uint32_t kW = kS + 256;  // without values: the keys' weights
  static constexpr uint32_t kStage = kS + (D <= 128 && VALUES ? 256 : 512);
  static constexpr int IPS = KI * (VALUES ? 2 : 1) + (D <= 128 && VALUES ? 1 : 2);  // copies of a stage
  static constexpr int NS = C::NS;
    static constexpr uint32_t kBytes = NS * kStage;

  const unsigned char *k, *v, *ks, *vs;
  lds_t lds;
  uint32_t k_off[2], v_off[2];  // of a lane's piece: bytes
  uint32_t s_off;
  uint32_t k_at, k_x, v_at, ks_at, vs_at;  // LDS offsets of its reads

  __device__ __forceinline__ void set(const Attn4Args& a, const unsigned char* k_, const unsigned char* v_,
                                      const unsigned char* ks_, const unsigned char* vs_, lds_t lds_) {
    k = k_; v = v_; ks = ks_; vs = vs_; lds = lds_;
    const int lane = lane_id(), c = lane & 15, g = lane >> 4;
    const uint32_t ts = (uint32_t)a.token_stride;
    // LDS row r of a half has key r, piece x at place x ^ swizzle(r), or of values key 4 (r % 4) + r / 4 as it is
    const int per = D == 64 ? 32 : kWave;  // lanes that a half's (or with 256 a quarter's) rows take
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int r = (lane % per) / CPR + (D == 256 ? 8 * y : 0), x = lane % CPR;
      k_off[y] = r * ts + (x ^ swizzle(r)) * 16;
      v_off[y] = (4 * (r % 4) + r / 4) * ts + x * 16;
    }
    s_off = (D <= 128 ? lane % 16 : lane / 2 % 16) * (ts / 16) + (D <= 128 ? 0 : lane % 2 * 4);
    k_at = c * RB + (D == 64 ? (uint32_t)((g / 2 ^ swizzle(c)) * 16 + g % 2 * 8) : 0u);
    k_x = swizzle(c);
    v_at = kV + g * RB + c * C::VB;
    ks_at = kS + c * SB + (D == 64 ? g / 2 : D == 128 ? g : 2 * g);
    vs_at = kS + 32 * SB + 4 * g * SB + (D > 128 ? c / 2 : 0);
  }
  static __device__ __forceinline__ uint32_t swizzle(int r) {
    return D == 64 ? (r >> 3) & 1 : D == 128 ? (r >> 2) & 3 : (r >> 1) & 7;
  }

  __device__ __forceinline__ void copy(const Attn4Args& a, const typename Where4<VALUES>::At& at, int stage) const {
    const lds_t to = lds + (uint32_t)stage * kStage;
    if constexpr (D == 64) {
      const uint64_t off = pick(lane_id() < 32, at.off0, at.off1);
      copy16(to, k + off + k_off[0]);
      if constexpr (VALUES) copy16(to + kV, v + off + v_off[0]);
    } else {
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const uint64_t off = pick(i < KI / 2, at.off0, at.off1);
        copy16(to + i * 1024, k + off, k_off[D == 256 ? i % 2 : 0]);
        if constexpr (VALUES) copy16(to + kV + i * 1024, v + off, v_off[D == 256 ? i % 2 : 0]);
      }
    }
    if constexpr (D <= 128) {  // keys' scales and values' at once
      const uint64_t off = pick((lane_id() & 16) == 0, at.off0, at.off1) / 16 + s_off;
      copy4<D == 64>(to + kS, pick(VALUES && lane_id() >= 32, vs, ks) + off);
    } else {
      const uint64_t off = pick(lane_id() < 32, at.off0, at.off1) / 16 + s_off;
      copy4<false>(to + kS, ks + off);
      if constexpr (VALUES) copy4<false>(to + kS + 256, vs + off);
    }
    if constexpr (!VALUES)
      copy4<false>(to + kW, (const unsigned char*)(a.weights + pick((lane_id() & 16) == 0, at.w0, at.w1) + lane_id() % 16));
  }
  // a stage's operands
  __device__ __forceinline__ void read(int stage, Raw4<C>& r) const {
    typedef __attribute__((address_space(3))) uint16_t* lds_u16_t;
    typedef __attribute__((address_space(3))) u32x2_t* lds_u32x2_t;
    const lds_t at = lds + (uint32_t)stage * kStage;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (D == 64) {
        const u32x2_t w = *(lds_u32x2_t)(at + h * 16 * RB + k_at);
        r.k[h][0] = w[0];
        r.k[h][1] = w[1];
      } else {
#pragma unroll
        for (int y = 0; y < C::KW / 4; ++y) {
          const int g = lane_id() >> 4;
          const u32x4_t w = *(lds_u32x4_t)(at + h * 16 * RB + k_at + ((g * (C::KW / 4) + y) ^ k_x) * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) r.k[h][4 * y + i] = w[i];
        }
      }
      if constexpr (C::KS > 1) {
        const uint32_t w = *(lds_u16_t)(at + ks_at + h * 16 * SB);
        r.ks[h][0] = w & 0xff;
        r.ks[h][1] = w >> 8;
      } else {
        r.ks[h][0] = *(at + ks_at + h * 16 * SB);
      }
    }
    if constexpr (VALUES) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const lds_t from = at + v_at + ((e / 4) * 16 + (e % 4) * 4) * RB;
        if constexpr (C::VB == 2) {
          r.v[e][0] = *(lds_u16_t)from;
        } else if constexpr (C::VB == 4) {
          r.v[e][0] = *(lds_u32_t)from;
        } else {
          const u32x2_t w = *(lds_u32x2_t)from;
          r.v[e][0] = w[0];
          r.v[e][1] = w[1];
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (D <= 128) {
          const u32x4_t w = *(lds_u32x4_t)(at + vs_at + h * 16 * SB);
          const uint32_t sh = (lane_id() & 15) / (D == 64 ? 8 : 4) * 8;
#pragma unroll
          for (int e = 0; e < 4; ++e) r.vs[4 * h + e] = w[e] >> sh & 0xff;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) r.vs[4 * h + e] = *(at + vs_at + (16 * h + e) * SB);
        }
      }
    }
  }
};

// The ring of a workgroup whose waves go through the same keys: WH neighbouring key heads (side by side in every token) and
// WR shares of the rows. Its waves share the copies, so that a copy takes whole lines: with a ring for each wave the same
// line was asked for by two waves at once, for which the L1 waits (256 tokens 559 us, 547 with nothing but the
// copies). Rows of WH heads lie in LDS as they do in the cache, keys in their order and values as in Ring4,
// pieces permuted so that reads meet no bank conflicts.
template <typename C, bool VALUES>
struct Shared4 {
  static constexpr int D = C::D, RB = D / 2, HB = C::WH, W = HB * RB;  // bytes of a token's codes
  static constexpr int CPR = D / 32, P = W / 16;          // 16-byte pieces of a head, of a token
  static constexpr int RPI = kWave / P;                   // tokens that a copy moves
  static constexpr int KI = 32 / RPI;                     // copies of a tile's keys
  static constexpr int SB = D / 32;                       // bytes of a head's scales of a key, in LDS
  static constexpr int SW = HB * SB;                      // and of the token's
  static constexpr bool kBoth = 32 * SW <= 128;           // one copy has keys' scales and values'
  static constexpr int SI = kBoth ? 1 : 32 * SW / 256;    // copies of the keys' scales
  static constexpr uint32_t kV = 32 * W, kS = VALUES ? 2 * kV : kV, kVS = kBoth ? 128 : 32 * SW;
  static constexpr uint32_t kW = kS + (kBoth ? 256 : 32 * SW);  // without values: the keys' weights, 256 bytes a head
  static constexpr uint32_t kStage = VALUES ? kS + (kBoth ? 256 : 64 * SW) : kW + HB * 256;
  static constexpr int kCodes = VALUES ? 2 * KI : KI, kAll = kCodes + (VALUES && !kBoth ? 2 * SI : SI);
  static constexpr int CW = (kCodes + 3) / 4, SCW = (kAll - kCodes + 3) / 4;  // a wave's copies of codes, of scales
  static constexpr int IPS = CW + SCW + (VALUES ? 0 : 1);
  static constexpr int NS = C::NS;
  static constexpr uint32_t kBytes = NS * kStage;
  static_assert(C::kWaves == 4 && C::WK == 1, "four waves, the same keys");
  static_assert(HB >= 2 && RPI <= 16, "heads to share, and a copy's tokens lie in one half");

  const unsigned char *k, *v, *ks, *vs;  // of the workgroup's first head
  lds_t lds;
  int wave;
  uint32_t c_off[CW];  // of the lane's piece in the wave's copies of codes, within the half: bytes
  uint32_t s_off[SCW];
  uint32_t k_at, k_x, k_p, v_at, ks_at, vs_at;

  static __device__ __forceinline__ uint32_t swizzle(int r) { return W >= 256 ? r & 15 : (r / (256 / W)) & (P - 1); }
  // (which copy a wave's i-th one is; those past the last are the last one again)
  __device__ __forceinline__ int code_copy(int i) const { return min(wave + 4 * i, kCodes - 1); }
  __device__ __forceinline__ int scale_copy(int i) const { return min(wave + 4 * i, kAll - kCodes - 1); }

  __device__ __forceinline__ void set(const Attn4Args& a, const unsigned char* k_, const unsigned char* v_,
                                      const unsigned char* ks_, const unsigned char* vs_, lds_t lds_, int wave_, int hh) {
    k = k_; v = v_; ks = ks_; vs = vs_; lds = lds_; wave = wave_;
    const int lane = lane_id(), c = lane & 15, g = lane >> 4;
    const uint32_t ts = (uint32_t)a.token_stride;
#pragma unroll
    for (int i = 0; i < CW; ++i) {
      const int n = code_copy(i);
      const int r = (n % KI * RPI + lane / P) % 16, x = lane % P;
      c_off[i] = n < KI ? r * ts + (x ^ swizzle(n % KI * RPI + lane / P)) * 16
                        : (4 * (r % 4) + r / 4) * ts + (x ^ (uint32_t)(CPR * ((r & 3) * HB / 4))) * 16;
    }
#pragma unroll
    for (int i = 0; i < SCW; ++i) {
      // dword `at` of the tile's keys' (or values') scales
      const int at = kBoth ? lane % 32 : (scale_copy(i) % SI) * 64 + lane, key = at * 4 / SW;
      s_off[i] = key % 16 * (ts / 16) + at * 4 % SW;
    }
    k_at = c * W;
    k_x = swizzle(c);
    k_p = hh * CPR;
    // (the lane's keys have R = 4 e + g: the permutation depends on g alone)
    const uint32_t piece = (uint32_t)(hh * CPR + c * C::VB / 16) ^ (uint32_t)(CPR * (g * HB / 4));
    v_at = kV + g * W + piece * 16 + c * C::VB % 16;
    ks_at = kS + c * SW + hh * SB + (D == 64 ? g / 2 : D == 128 ? g : 2 * g);
    vs_at = kS + kVS + 4 * g * SW + hh * SB + c / (512 / D);
  }
  __device__ __forceinline__ void copy(const Attn4Args& a, const typename Where4<VALUES>::At& at, int stage, int hh) const {
    const lds_t to = lds + (uint32_t)stage * kStage;
#pragma unroll
    for (int i = 0; i < CW; ++i) {
      const int n = code_copy(i);
      const bool is_k = n < KI;
      const unsigned char* from = pick(is_k, k, v);
      const lds_t dst = to + n * 1024;
      copy16(dst, from + pick(n % KI < KI / 2, at.off0, at.off1), c_off[i]);
    }
#pragma unroll
    for (int i = 0; i < SCW; ++i) {
      const int n = scale_copy(i);
      const lds_t dst = to + kS + n * 256;
      if constexpr (kBoth) {
        const int key = lane_id() % 32 * 4 / SW;
        copy4<false>(dst, pick(VALUES && lane_id() >= 32, vs, ks) + pick(key < 16, at.off0, at.off1) / 16 + s_off[i]);
      } else {
        const int key = ((n % SI) * 64 + lane_id()) * 4 / SW;
        copy4<false>(dst, pick(n < SI, ks, vs) + pick(key < 16, at.off0, at.off1) / 16 + s_off[i]);
      }
    }
    if constexpr (!VALUES)  // each wave its own head's weights
      copy4<false>(to + kW + hh * 256,
                   (const unsigned char*)(a.weights + pick((lane_id() & 16) == 0, at.w0, at.w1) + lane_id() % 16));
  }
  __device__ __forceinline__ void read(int stage, Raw4<C>& r) const {
    typedef __attribute__((address_space(3))) uint16_t* lds_u16_t;
    typedef __attribute__((address_space(3))) u32x2_t* lds_u32x2_t;
    const lds_t at = lds + (uint32_t)stage * kStage;
    const int g = lane_id() >> 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // (keys 16 apart differ in the permutation where a half is not a whole number of its turns)
      const uint32_t x = k_x ^ (h ? swizzle(16) : 0);
      if constexpr (D == 64) {
        const u32x2_t w = *(lds_u32x2_t)(at + h * 16 * W + k_at + ((k_p + g / 2) ^ x) * 16 + g % 2 * 8);
        r.k[h][0] = w[0];
        r.k[h][1] = w[1];
      } else {
#pragma unroll
        for (int y = 0; y < C::KW / 4; ++y) {
          const u32x4_t w = *(lds_u32x4_t)(at + h * 16 * W + k_at + ((k_p + g * (C::KW / 4) + y) ^ x) * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) r.k[h][4 * y + i] = w[i];
        }
      }
      if constexpr (C::KS > 1) {
        const uint32_t w = *(lds_u16_t)(at + ks_at + h * 16 * SW);
        r.ks[h][0] = w & 0xff;
        r.ks[h][1] = w >> 8;
      } else {
        r.ks[h][0] = *(at + ks_at + h * 16 * SW);
      }
    }
    if constexpr (VALUES) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const lds_t from = at + v_at + ((e / 4) * 16 + (e % 4) * 4) * W;
        if constexpr (C::VB == 2) {
          r.v[e][0] = *(lds_u16_t)from;
        } else if constexpr (C::VB == 4) {
          r.v[e][0] = *(lds_u32_t)from;
        } else {
          const u32x2_t w = *(lds_u32x2_t)from;
          r.v[e][0] = w[0];
          r.v[e][1] = w[1];
        }
        r.vs[e] = *(at + vs_at + ((e / 4) * 16 + e % 4) * SW);
      }
    }
  }
};

// the h-th half's 16 keys as operands of the D / 32 score products
template <typename C>
__device__ __forceinline__ void keys4(const Raw4<C>& r, int h, u32x4_t (&to)[C::KW]) {
#pragma unroll
  for (int w = 0; w < C::KW; ++w) {
    const uint32_t b = r.ks[h][C::KS > 1 ? w / 4 : 0];
    const float s = scale_of(b);
    const uint32_t x = r.k[h][w];
    to[w] = u32x4_t{from4<0>(x, s), from4<1>(x, s), from4<2>(x, s), from4<3>(x, s)};
  }
}

// elements 2 B and 2 B + 1 of the lane's part of its eight values, as operands
template <typename C, int B>
__device__ __forceinline__ void values4(const Raw4<C>& r, const float (&s)[8], u32x4_t& even, u32x4_t& odd) {
  uint32_t p[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = from4<B % 4>(r.v[e][B / 4], s[e]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    even[i] = __builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], 0x05040100u);
    odd[i] = __builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], 0x07060302u);
  }
}

// A wave's row of queries as operands of the score products: elements D / 4 g .. of row `at`, zeros past the width
template <typename C>
__device__ __forceinline__ void queries4(const uint16_t* at, int d, u32x4_t (&q)[C::kTerms][C::KW]) {
  const int g = lane_id() >> 4;
#pragma unroll
  for (int w = 0; w < C::KW; ++w) {
    const int x = g * (C::D / 4) + w * 8;
    const u32x4_t in = x < d ? *reinterpret_cast<const u32x4_t*>(at + x) : u32x4_t{0, 0, 0, 0};
    u32x4_t t[C::kTerms];
    Query<typename C::T>::split(in, t);
#pragma unroll
    for (int i = 0; i < C::kTerms; ++i) q[i][w] = t[i];
  }
}

// The row tile of item group `rest`, where each request has one tile: shifted from chunk to chunk, so that a request's
// chunks go round the XCDs too. With their number even and no shift all of a request is one XCD's, and the XCD
// with the longest ones takes the time: 64 blocks 313 us against 378, 256 tokens 446 against 465, their weights 270
// against 283.
__device__ __forceinline__ int shifted(int rest, int chunk_no, int tiles) {
  return (rest % tiles + (tiles % 2 ? 0 : chunk_no % tiles)) % tiles;
}

// Which rows a tile of BM has: request n, its first row r0 and the end r1 of them, first token, position of the first
// query. False where there are none.
struct Rows4 {
  int n, r0, r1, start, T, total, pos0;
};
template <int BM>
__device__ __forceinline__ bool rows4(const Attn4Args& a, int tile, Rows4& r) {
  auto starts_at = [&](int i) { return min(max(a.starts[i], 0), a.tokens); };
  int n = 0;
  if ((int64_t)a.max_tokens * a.group <= BM) {
    n = tile;
    r.r0 = 0;
  } else {
    // request n's tiles have the numbers floor(starts[n] * group / BM) + n and on, which is at least as many as it
    // has; 64 candidates at a time
    auto first_tile = [&](int i) { return (int)((int64_t)starts_at(i) * a.group / BM) + i; };
    int end = a.N;
    while (end - n > 1) {
      const int step = (end - n + kWave - 1) / kWave, i = n + lane_id() * step;
      const uint64_t le = __ballot(i < end && first_tile(i) <= tile);
      const int last = 63 - __builtin_clzll(le | 1);
      n += last * step;
      end = min(end, n + step);
    }
    n = (int)uniform32(n);
    r.r0 = (tile - first_tile(n)) * BM;
  }
  r.n = n;
  r.start = starts_at(n);
  r.T = starts_at(n + 1) - r.start;
  r.total = max(a.totals[n], 0);
  r.pos0 = r.total - r.T;
  const int T = min(r.T, a.max_tokens);
  if (r.r0 < 0 || r.r0 >= (int64_t)T * a.group) return false;
  r.r1 = (int)min((int64_t)T * a.group, (int64_t)r.r0 + BM);
  return true;
}

// What bounds it, with 32 heads over 8 of 128: 256 tokens (100 to 16100 keys each) 445 us with the join, 5.1 TB/s: HBM, 0.76 of a
// plain read. 64 blocks of 16 tokens 308 us, 8192 tokens of prefill 1930 (855 TFLOP/s, 0.64 of a library
// product): a tile of 32 rows and keys is 512 cycles of matrix instructions and 150 to 190 others, most of them
// conversions, powers and sums, and two waves of a SIMD overlap a third of them. One token over 32768 keys 18.5 us:
// latency, 14 of it here (lengths, pages, first tiles, output) and 4.6 in the join.
template <typename C>
__global__ __launch_bounds__(C::kThreads) __attribute__((amdgpu_waves_per_eu(C::kSimdWaves, C::kSimdWaves)))
void attention4_kernel(Attn4Args a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char attn4_smem[];
  typedef typename C::T T;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = (int)uniform32(tid >> 6);
  const int wh = wave % C::WH, wr = wave / C::WH % C::WR, wk = wave / (C::WH * C::WR);

  // ---- which rows ------------------------------------------------------------------------------
  const int head_groups = a.kv_heads / C::WH;
  const int it = a.spread ? beside((int)blockIdx.x, a.items, head_groups) : (int)blockIdx.x;
  const int head = it % head_groups * C::WH + wh;
  const int rest = it / head_groups;
  const int chunk_no = rest / a.tiles;
  Rows4 rw;
  // long rows first: with a causal mask and no window the last tiles of a request see most
  if (!rows4<C::BM>(a, a.spread ? shifted(rest, chunk_no, a.tiles) : a.tiles - 1 - rest % a.tiles, rw)) return;
  const int r0 = rw.r0, r1 = rw.r1;

  // ---- which keys ------------------------------------------------------------------------------
  const int p_lo = rw.pos0 + r0 / a.group, p_hi = rw.pos0 + (r1 - 1) / a.group;
  int hi = a.causal ? min(rw.total, p_hi + 1) : rw.total;
  hi = max((int)min((int64_t)min(hi, a.max_length), a.table_width * (int64_t)a.page_size), 0);
  const int lo = a.window ? min(max(p_lo - a.window + 1, 0), hi) : 0;
  const int ns = min(a.sinks, lo);
  // tiles of 32 keys: those of the sinks, then those of the window, as one list
  const int t_lo = lo / 32, s_t = min((ns + 31) / 32, t_lo);
  const int nt = min(s_t + (hi + 31) / 32 - t_lo, a.most);
  const int t_begin = chunk_no * a.chunk, t_end = min(nt, t_begin + a.chunk);

  int row[C::RT], p[C::RT];
  int64_t orow[C::RT];
  u32x4_t q[C::RT][C::kTerms][C::KW];
#pragma unroll
  for (int t = 0; t < C::RT; ++t) {
    row[t] = r0 + (wr * C::RT + t) * 16 + c;
    const int rc = min(row[t], r1 - 1), tok = rc / a.group, hq = head * a.group + (rc - tok * a.group);
    orow[t] = ((int64_t)rw.start + tok) * a.heads + hq;
    p[t] = rw.pos0 + tok;
    if (t_begin < t_end) queries4<C>(a.q + ((int64_t)rw.start + tok) * a.q_stride + (int64_t)hq * a.d, a.d, q[t]);
  }
  if (t_begin >= t_end && chunk_no > 0) {  // (chunk 0 of a tile without keys writes its zeros below)
    if (wk == 0 && g == 0)
#pragma unroll
      for (int t = 0; t < C::RT; ++t)
        if (row[t] < r1) a.part_ml[(int64_t)chunk_no * a.rows + orow[t]] = f32x4_t{-__builtin_inff(), 0.f, 0.f, 0.f};
    return;
  }
  // the wave's rows: positions of its first and last
  const int wrow0 = r0 + wr * C::RT * 16;
  const int wp_lo = rw.pos0 + min(wrow0, r1 - 1) / a.group;
  const int wp_hi = rw.pos0 + min(wrow0 + C::RT * 16 - 1, r1 - 1) / a.group;
  // all of the wave's rows see all keys of the tiles below whole_to, from whole_from on or below whole_sinks
  const int whole_to = max(a.causal ? min(hi, wp_lo + 1) : hi, 0) / 32;
  const int whole_from = a.window ? max(wp_hi - a.window + 32, 0) / 32 : 0, whole_sinks = a.window ? a.sinks / 32 : 0;

  const int64_t ho = (int64_t)head * a.head_stride;
  const unsigned char *k = a.k + ho, *v = a.v + ho, *ks = a.ks + ho / 16, *vs = a.vs + ho / 16;
  const int32_t* trow = a.table + (int64_t)rw.n * a.table_width;
  auto tile_at = [&](int i) { return i < s_t ? i : i - s_t + t_lo; };

  f32x4_t o[C::RT][C::ND];
  float m[C::RT], l[C::RT], lu[C::RT];
  f32x4_t ls[C::RT];
  uint32_t poison[C::RT];
#pragma unroll
  for (int t = 0; t < C::RT; ++t) {
#pragma unroll
    for (int i = 0; i < C::ND; ++i) o[t][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m[t] = -__builtin_inff();
    lu[t] = 0.f;
    ls[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    poison[t] = 0;
  }

  // One tile, whose keys all rows see (`whole`) or not: `here` are those that there are. False, and nothing accumulated,
  // where a maximum has grown too far over its reference: then grow(), and again, twice at most (where one
  // row's reference goes far, the others' products are rounded too, which may find another a little grown). The accumulators change outside the loop over the tiles, since the compiler copies them
  // at every join of paths inside it (38 moves a tile with two blocks of rows, 144 with four).
  float mx[C::RT];
  uint64_t far = 0;  // which lanes' references are far
  auto step = [&](Raw4<C>& r, int j0, uint32_t here, bool whole) __attribute__((always_inline)) -> bool {
    uint32_t vis[C::RT];
    if (!whole) {
#pragma unroll
      for (int t = 0; t < C::RT; ++t) {
        vis[t] = here;
        if (a.causal) vis[t] &= bits32_below(p[t] + 1 - j0);
        if (a.window) vis[t] &= bits32_from(p[t] - a.window + 1 - j0) | bits32_below(a.sinks - j0);
      }
    }
    f32x4_t sc[C::RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4_t kk[C::KW];
      keys4<C>(r, h, kk);
#pragma unroll
      for (int t = 0; t < C::RT; ++t) {
        sc[t][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < C::KW; ++w)
#pragma unroll
          for (int u = 0; u < C::kTerms; ++u) sc[t][h] = mfma16(kk[w], q[t][u][w], sc[t][h]);
      }
    }
    bool up = false;
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
      if (!whole) {
        const uint32_t mine = vis[t] >> (4 * g);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          sc[t][e / 4][e % 4] = mine & (1u << (16 * (e / 4) + e % 4)) ? sc[t][e / 4][e % 4] : -__builtin_inff();
      }
      mx[t] = max3(sc[t][0][0], sc[t][0][1], sc[t][0][2]);
      mx[t] = max3(mx[t], sc[t][0][3], sc[t][1][0]);
      mx[t] = max3(mx[t], sc[t][1][1], sc[t][1][2]);
      mx[t] = max3(mx[t], sc[t][1][3], mx[t]);
    }
    const float s2 = far ? 1.f : a.scale2;  // what scores have still to be multiplied by
    if (__builtin_expect(far != 0, 0)) {
#pragma unroll
      for (int t = 0; t < C::RT; ++t) {
        mx[t] = scaled4(mx[t], a.scale2);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[t][e / 4][e % 4] = scaled4(sc[t][e / 4][e % 4], a.scale2);
      }
    }
#pragma unroll
    for (int t = 0; t < C::RT; ++t) up |= grown4(mx[t], s2, m[t]);
    if (__builtin_expect(__ballot(up) != 0, 0)) return false;
    u32x4_t pf[C::RT][C::kTerms];
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
      const float ms = m[t] == -__builtin_inff() ? 0.f : m[t];
      float e[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        e[x] = __builtin_amdgcn_exp2f(fmaf(sc[t][x / 4][x % 4], s2, -ms));
        lu[t] += e[x];
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t w = Bf16::pack(e[2 * x], e[2 * x + 1]);
        pf[t][0][x] = w;
        if constexpr (C::kTerms > 1) {
          const f32x2_t hi = Bf16::unpack(w);
          pf[t][1][x] = Bf16::pack(e[2 * x] - hi[0], e[2 * x + 1] - hi[1]);
        }
      }
    }
    if constexpr (C::kTerms == 1) {
      // sums of the rounded probabilities, in every register of a lane (prefill 1933 us, 1985 with vector instructions)
      const u32x4_t ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
      for (int t = 0; t < C::RT; ++t) ls[t] = mfma16(ones, pf[t][0], ls[t]);
    }
    if (!whole) {  // NaN blocks of values
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, r.vs[e]);
      if (__builtin_expect(__ballot(top > kMostScale) != 0, 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint64_t bad = __ballot(r.vs[e] > kMostScale);
#pragma unroll
          for (int b = 0; b < C::D / kBlock4; ++b) {
            // the first lane of each quarter that has elements of block b
            const uint64_t of = bad >> (b * (512 / C::D));
            const uint32_t keys = ((uint32_t)(of & 1) | ((uint32_t)(of >> 16 & 1) << 4) | ((uint32_t)(of >> 32 & 1) << 8) |
                                   ((uint32_t)(of >> 48 & 1) << 12)) << (e < 4 ? e : 16 + e - 4);
#pragma unroll
            for (int t = 0; t < C::RT; ++t) poison[t] |= vis[t] & keys ? 1u << b : 0u;
          }
          if (r.vs[e] > kMostScale) {
            r.vs[e] = 127;
            r.v[e][0] = 0;
            if constexpr (C::VB > 4) r.v[e][1] = 0;
          }
        }
      }
    }
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = scale_of(r.vs[e]);
    auto product = [&](auto b) __attribute__((always_inline)) {
      constexpr int B = decltype(b)::value;
      u32x4_t even, odd;
      values4<C, B>(r, s, even, odd);
#pragma unroll
      for (int t = 0; t < C::RT; ++t) {
#pragma unroll
        for (int u = 0; u < C::kTerms; ++u) {
          o[t][2 * B] = mfma16(even, pf[t][u], o[t][2 * B]);
          o[t][2 * B + 1] = mfma16(odd, pf[t][u], o[t][2 * B + 1]);
        }
      }
    };
    product(std::integral_constant<int, 0>{});
    product(std::integral_constant<int, 1>{});
    if constexpr (C::VB > 2) {
      product(std::integral_constant<int, 2>{});
      product(std::integral_constant<int, 3>{});
    }
    if constexpr (C::VB > 4) {
      product(std::integral_constant<int, 4>{});
      product(std::integral_constant<int, 5>{});
      product(std::integral_constant<int, 6>{});
      product(std::integral_constant<int, 7>{});
    }
    return true;
  };
  auto grow = [&]() __attribute__((always_inline)) {
    const float s2 = far ? 1.f : a.scale2;
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
      const float top = quad_max(mx[t]);
      const bool grows = grown4(top, s2, m[t]);
      const float to = reference4(top, s2);
      // nothing is accumulated while m is -inf
      const float f = grows ? __builtin_amdgcn_ldexpf(1.f, (int)fmaxf(m[t] - to, -300.f)) : 1.f;
      m[t] = grows ? to : m[t];
      far |= __ballot(far4(m[t]));
      lu[t] *= f;
      ls[t] *= f;
#pragma unroll
      for (int i = 0; i < C::ND; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][i][e] *= f;
    }
  };
  // one tile; of its keys those in `there` are on pages that are there
  auto use = [&](Raw4<C>& r, int i, uint32_t there) __attribute__((always_inline)) -> bool {
    const int tile = tile_at(i), j0 = tile * 32;
    const bool whole = there == ~0u && tile < whole_to && (tile >= whole_from || tile < whole_sinks);
    return step(r, j0, there & bits32_below(hi - j0), whole);
  };
  int i = t_begin + wk;
  if constexpr (C::RING) {
    constexpr bool kShared = C::kShared;
    typedef std::conditional_t<kShared, Shared4<C, true>, Ring4<C, true>> Ring;
    Ring ring;
    Where4<true> where;
    if (i < t_end) {
      if constexpr (kShared) {
        const int64_t first = (int64_t)(head - wh) * a.head_stride;
        ring.set(a, a.k + first, a.v + first, a.ks + first / 16, a.vs + first / 16, (lds_t)attn4_smem, wave, wh);
      } else {
        ring.set(a, k, v, ks, vs, (lds_t)attn4_smem + (uint32_t)wave * Ring::kBytes);
      }
      const int tiles = (t_end - i + C::WK - 1) / C::WK;  // of this wave
      auto tile_of = [&](int s) { return tile_at(i + s * C::WK); };
      auto find = [&](int s) { return where.find(a, s, tiles, tile_of); };
      auto copy = [&](const typename Where4<true>::At& from, int stage) __attribute__((always_inline)) {
        if constexpr (kShared) ring.copy(a, from, stage, wh);
        else ring.copy(a, from, stage);
      };
      // A wave with a ring of its own has NS tiles under way, and copies the next one when it is done with one. Shared, NS - 1:
      // the barrier says that everyone's copies have landed, and that all are done with the tile before, whose place
      // the next copies take.
      constexpr int kAhead = kShared ? C::NS - 1 : C::NS;
      where.begin(a, trow, hi, tiles, tile_of);
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        const auto first = find(s);
        if (s < tiles) copy(first, s);
      }
      auto next = find(kAhead);
      int at = 0, s = 0;
      bool begun = false;  // this tile has been waited for
      while (true) {
        for (; s < tiles; ++s) {
          if (!begun) {
            if (s + kAhead - 1 < tiles)
              __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"((kAhead - 1) * Ring::IPS) : "memory");
            else
              __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if constexpr (kShared) {
              __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
              if (s + kAhead < tiles) copy(next, at == 0 ? C::NS - 1 : at - 1);
              next = find(s + kAhead + 1);
            }
          }
          Raw4<C> r;
          ring.read(at, r);
          const int x = i + s * C::WK;
          begun = true;
          if (!use(r, x, where.there(kShared ? kAhead + 1 : kAhead))) break;
          begun = false;
          if constexpr (!kShared) {
            __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this tile's reads
            if (s + kAhead < tiles) copy(next, at);
            next = find(s + kAhead + 1);
          }
          at = at + 1 == C::NS ? 0 : at + 1;
        }
        if (s >= tiles) break;
        grow();
      }
    }
    if constexpr (C::WK > 1) __syncthreads();  // the rings' memory is used again below
  } else if (i < t_end) {
    Places4<C> pl;
    pl.set(a);
    auto page_of = [&](int i) {  // of key lane % 32 of the list's tile i, or of the last one's last key
      const int j = min(tile_at(min(i, t_end - 1)) * 32 + (lane & 31), hi - 1);
      return trow[entry4(a, j)];
    };
    auto there = [&](int page) { return (uint32_t)__ballot(page >= 0 && page < a.pages); };
    auto load = [&](int i, int page, Raw4<C>& r) __attribute__((always_inline)) {
      load4<C, true>(a, pl, k, v, ks, vs, tile_at(min(i, t_end - 1)), page >= 0 && page < a.pages ? page : 0, r);
    };
    // two sets of registers in turn: a tile is asked for while the one before it is used, its pages a tile earlier
    Raw4<C> ra, rb;
    int pa = page_of(i), pb = page_of(i + C::WK);
    load(i, pa, ra);
    while (true) {
      int next = page_of(i + 2 * C::WK);
      load(i + C::WK, pb, rb);
      while (!use(ra, i, there(pa))) grow();
      pa = next;
      i += C::WK;
      if (i >= t_end) break;
      next = page_of(i + 2 * C::WK);
      load(i + C::WK, pa, ra);
      while (!use(rb, i, there(pb))) grow();
      pb = next;
      i += C::WK;
      if (i >= t_end) break;
    }
  }

  // ---- join the waves that shared the keys ---------------------------------------------------------
#pragma unroll
  for (int t = 0; t < C::RT; ++t) {
    lu[t] = quad_sum(lu[t]);
    l[t] = C::kTerms > 1 ? lu[t] : ls[t][0];  // two terms of a probability round next to nothing
    if (__ballot(poison[t] != 0)) {
      // lane (c, g) has the elements D / 4 g + D / 16 r + i of its row, in o[t][i][r]
#pragma unroll
      for (int i = 0; i < C::ND; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (poison[t] >> ((g * (C::D / 4) + r * (C::D / 16)) / kBlock4) & 1) o[t][i][r] = __builtin_nanf("");
    }
  }
  if constexpr (C::WK > 1) {
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
#pragma unroll
      for (int i = 0; i < C::ND; ++i)
        *(lds_f32x4_t)(attn4_smem + (((wave * C::RT + t) * C::ND + i) * kWave + lane) * 16) = o[t][i];
      *(lds_f32x4_t)(attn4_smem + C::kOut + ((wave * C::RT + t) * kWave + lane) * 16) = f32x4_t{m[t], l[t], lu[t], 0.f};
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
      f32x4_t ml[C::WK];
      float f[C::WK], top = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < C::WK; ++w) {
        ml[w] = *(lds_f32x4_t)(attn4_smem + C::kOut + ((((w * C::WR + wr) * C::WH + wh) * C::RT + t) * kWave + lane) * 16);
        top = fmaxf(top, ml[w][0]);
      }
      l[t] = lu[t] = 0.f;
#pragma unroll
      for (int w = 0; w < C::WK; ++w) {
        f[w] = ml[w][0] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ml[w][0] - top);
        l[t] += f[w] * ml[w][1];
        lu[t] += f[w] * ml[w][2];
      }
      m[t] = top;
#pragma unroll
      for (int i = 0; i < C::ND; ++i) {
        if (i / (C::ND / C::WK) != wk) continue;  // each of the waves joins its share of the products
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < C::WK; ++w)
          sum += f[w] * *(lds_f32x4_t)(attn4_smem + (((((w * C::WR + wr) * C::WH + wh) * C::RT + t) * C::ND + i) * kWave + lane) * 16);
        o[t][i] = sum;
      }
    }
  }

  // ---- write ---------------------------------------------------------------------------------------
  constexpr int kMine = C::ND / C::WK;  // products that this wave writes: elements kMine wk .. of each run of ND
#pragma unroll
  for (int t = 0; t < C::RT; ++t) {
    if (row[t] >= r1) continue;
    const float inv = l[t] == 0.f ? 0.f : 1.f / l[t];  // a row that sees nothing gives zeros
    if (wk == 0 && g == 0) {
      if (a.split) a.part_ml[(int64_t)chunk_no * a.rows + orow[t]] = f32x4_t{m[t], l[t], lu[t], 0.f};
      else if (a.lse)
        a.lse[orow[t]] = lu[t] == 0.f ? -__builtin_inff() : (m[t] + __builtin_amdgcn_logf(lu[t])) * 0.6931471805599453f;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int x = g * (C::D / 4) + r * C::ND + wk * kMine;
      if (x >= a.d) continue;
      float f[kMine];
#pragma unroll
      for (int i = 0; i < C::ND; ++i)
        if (i / kMine == wk) f[i % kMine] = o[t][i][r];
      if (a.split) {
        float* to = a.part_o + ((int64_t)chunk_no * a.rows + orow[t]) * a.d + x;
#pragma unroll
        for (int i = 0; i < kMine; ++i) to[i] = f[i];
      } else {
        uint16_t* to = a.out + orow[t] * a.d + x;
        if constexpr (kMine == 1) {
          to[0] = (uint16_t)T::pack(f[0] * inv, 0.f);
        } else {
#pragma unroll
          for (int i = 0; i < kMine; i += 2)
            *reinterpret_cast<uint32_t*>(to + i) = T::pack(f[i] * inv, f[i + 1] * inv);
        }
      }
    }
  }
}

// Joins the slots of every row in their order, a wave a row: maxima and sums one lane a slot, then the partial outputs
// in 16 bytes a lane, LPR lanes a slot and 64 / LPR slots at once. A slot that saw nothing holds no output. FEW rows:
// all slots are read at once, beside the sums and without them; else only those that count.
constexpr int kJoin4Threads = 256;
template <typename T, int LPR, bool FEW>
__global__ __launch_bounds__(kJoin4Threads) void attention4_join_kernel(Attn4Args a, int slots) {
  constexpr int kAtOnce = kWave / LPR;
  const int lane = lane_id();
  const int64_t row = (int64_t)blockIdx.x * (kJoin4Threads / kWave) + threadIdx.x / kWave;
  const int x = (lane % LPR) * 4;
  if (row >= a.rows) return;
  const int64_t used = (int64_t)min(max(a.starts[a.N], 0), a.tokens) * a.heads;
  // Whether this lane's slot of turn (b, u) saw anything. The uniform part of its number is shifted by the scalar unit: a
  // 64-bit vector shift by a lane's own amount went wrong where the amount lay in the wave's last register.
  auto saw_of = [&](uint64_t which, int b, int u) {
    return (uint32_t)(which >> (b + u * kAtOnce)) >> (lane / LPR) & 1;
  };
  float top = -__builtin_inff(), l = 0.f, lu = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < slots; s0 += kWave) {
    const int here = min(slots - s0, kWave);
    constexpr int kBatch = FEW ? 64 / kAtOnce : 8;
    f32x4_t v[kBatch];
    auto load = [&](int b, uint64_t which) {
      const float* at = a.part_o + ((s0 + b + lane / LPR) * a.rows + row) * a.d + x;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int s = b + u * kAtOnce + lane / LPR;
        v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (s < here && x < a.d && (FEW || saw_of(which, b, u)))
          v[u] = *reinterpret_cast<const f32x4_t*>(at + u * (kAtOnce * a.rows * a.d));
      }
    };
    f32x4_t ml = {-__builtin_inff(), 0.f, 0.f, 0.f};
    if (lane < here) ml = a.part_ml[(s0 + lane) * a.rows + row];
    if constexpr (FEW) load(0, 0);
    const float grown = fmaxf(top, wave_max_dpp(ml[0]));
    const float f0 = top == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(top - grown);
    // the sum of a slot that saw nothing is 0; a NaN stays one
    const float f = ml[0] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ml[0] - grown);
    const bool saw = ml[1] != 0.f;
    const float seen = saw ? f : -1.f;
    top = grown;
    l = l * f0 + wave_sum_dpp(saw ? f * ml[1] : 0.f);
    lu = lu * f0 + wave_sum_dpp(saw ? f * ml[2] : 0.f);
    o *= f0;
    const uint64_t which = __ballot(saw);
    for (int b = 0; b < here; b += kBatch * kAtOnce) {
      if (!FEW || b) load(b, which);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int s = b + u * kAtOnce + lane / LPR;
        const float w = __shfl(seen, s & 63, kWave);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += w < 0.f ? 0.f : w * v[u][e];
      }
    }
  }
  if (row >= used) return;
#pragma unroll
  for (int m = LPR; m < kWave; m <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m, kWave);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lane < LPR && x < a.d)
    *reinterpret_cast<u32x2_t*>(a.out + row * a.d + x) =
        u32x2_t{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
  if (lane == 0 && a.lse)
    a.lse[row] = lu == 0.f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(lu)) * 0.6931471805599453f;
}

// ---- accumulated weights ---------------------------------------------------------------------------

// place of a key's weight
__device__ __forceinline__ int64_t weight_at(const Attn4Args& a, int page, int head, int j) {
  return ((int64_t)page * a.kv_heads + head) * a.page_size + (j - entry4(a, j) * (int)a.page_size);
}

// Requests with at most 16 rows: a wave goes through tiles of 32 keys as in the attention. The scores stand the
// other way round, S[row][key], so that a lane has four rows of one key and the sum over rows is three
// additions and two exchanges. 256 requests of one token (32 heads over 8 of 128) 270 us: HBM, 4.7 TB/s.
template <typename C>
__global__ __launch_bounds__(C::kThreads) void key_weights_few_kernel(Attn4Args a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char attn4_smem[];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = (int)uniform32(tid >> 6), wh = wave % C::WH, wk = wave / C::WH;
  const int head_groups = a.kv_heads / C::WH;
  const int it = a.spread ? beside((int)blockIdx.x, a.items, head_groups) : (int)blockIdx.x;
  const int head = it % head_groups * C::WH + wh;
  const int rest = it / head_groups;
  const int chunk_no = rest / a.tiles;
  Rows4 rw;
  if (!rows4<16>(a, shifted(rest, chunk_no, a.tiles), rw) || rw.T > a.max_tokens) return;
  const int hi = max((int)min((int64_t)min(rw.total, a.max_length), a.table_width * (int64_t)a.page_size), 0);
  const int t_begin = chunk_no * a.chunk, t_end = min((hi + 31) / 32, t_begin + a.chunk);
  int i = t_begin + wk;
  if (i >= t_end) return;

  u32x4_t q[C::kTerms][C::KW];
  {
    const int rc = min(c, rw.r1 - 1), tok = rc / a.group, hq = head * a.group + (rc - tok * a.group);
    queries4<C>(a.q + ((int64_t)rw.start + tok) * a.q_stride + (int64_t)hq * a.d, a.d, q);
  }
  float ls[4];  // of row 4 g + r; no row, or one that sees nothing: its powers are 0
  int p[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int x = 4 * g + r, rc = min(x, rw.r1 - 1), tok = rc / a.group, hq = head * a.group + (rc - tok * a.group);
    const float v = a.lse_in[((int64_t)rw.start + tok) * a.heads + hq];
    ls[r] = x >= rw.r1 || v == -__builtin_inff() ? __builtin_inff() : v * 1.4426950408889634f;
    p[r] = rw.pos0 + tok;
  }
  const int64_t ho = (int64_t)head * a.head_stride;
  const unsigned char *k = a.k + ho, *ks = a.ks + ho / 16;
  const int32_t* trow = a.table + (int64_t)rw.n * a.table_width;
  // the new weight of key lane % 32 of tile x
  auto use = [&](const Raw4<C>& r, float before, int x) __attribute__((always_inline)) {
    const int j0 = x * 32;
    const bool all = !a.causal || j0 + 31 <= rw.pos0;
    float got[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4_t kk[C::KW];
      keys4<C>(r, h, kk);
      f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < C::KW; ++w)
#pragma unroll
        for (int u = 0; u < C::kTerms; ++u) sc = mfma16(q[u][w], kk[w], sc);
      float e[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        e[y] = __builtin_amdgcn_exp2f(ls[y] == __builtin_inff() ? -__builtin_inff() : fmaf(sc[y], a.scale2, -ls[y]));
        if (!all) e[y] = j0 + 16 * h + c <= p[y] ? e[y] : 0.f;
      }
      got[h] = quad_sum((e[0] + e[1]) + (e[2] + e[3]));
    }
    return (j0 + (lane & 31) < rw.pos0 ? a.decay * before : 0.f) + ((lane & 16) ? got[1] : got[0]);
  };
  auto page_of = [&](int x) {
    const int j = min(min(x, t_end - 1) * 32 + (lane & 31), hi - 1);
    return trow[entry4(a, j)];
  };
  auto place = [&](int page) { return page >= 0 && page < a.pages ? page : 0; };
  auto old = [&](int x, int page) {
    return a.weights[weight_at(a, place(page), head, min(x, t_end - 1) * 32 + (lane & 31))];
  };
  if constexpr (C::RING) {
    constexpr bool kShared = C::kShared;
    typedef std::conditional_t<kShared, Shared4<C, false>, Ring4<C, false>> Ring;
    typedef Where4<false> Where;
    Ring ring;
    Where places;
    if constexpr (kShared) {
      const int64_t first = (int64_t)(head - wh) * a.head_stride;
      ring.set(a, a.k + first, a.k, a.ks + first / 16, a.ks, (lds_t)attn4_smem, wave, wh);
    } else {
      ring.set(a, k, k, ks, ks, (lds_t)attn4_smem + (uint32_t)wave * Ring::kBytes);
    }
    const int tiles = (t_end - i + C::WK - 1) / C::WK;
    auto tile_of = [&](int s) { return i + s * C::WK; };
    auto find = [&](int s) { return places.find(a, s, tiles, tile_of, head); };
    auto copy = [&](const typename Where::At& from, int stage) __attribute__((always_inline)) {
      if constexpr (kShared) ring.copy(a, from, stage, wh);
      else ring.copy(a, from, stage);
    };
    places.begin(a, trow, hi, tiles, tile_of, head);
    typename Where::At where[C::NS + 1];  // of the tiles under way, this one first
#pragma unroll
    for (int s = 0; s <= C::NS - 1; ++s) {
      where[s] = find(s);
      if (s < C::NS - 1 && s < tiles) copy(where[s], s);
    }
    int at = 0, to = C::NS - 1;
    constexpr int kAhead = kShared ? C::NS - 2 : C::NS - 1;  // tiles under way while this one is waited for
    for (int s = 0; s < tiles; ++s) {
      __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if constexpr (!kShared) {
        if (s + C::NS - 1 < tiles) copy(where[C::NS - 1], to);
      }
      if (s + kAhead < tiles)
        __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead * Ring::IPS) : "memory");
      else
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if constexpr (kShared) {
        __asm__ volatile("s_barrier" ::: "memory");
        if (s + C::NS - 1 < tiles) copy(where[C::NS - 1], to);
      }
      Raw4<C> r;
      ring.read(at, r);
      const float before = *(lds_float_t)(ring.lds + (uint32_t)at * Ring::kStage + Ring::kW + (kShared ? wh * 256 : 0) + (lane & 31) * 4);
      where[C::NS] = find(s + C::NS);
      const uint32_t there = places.there(C::NS);
      const int x = i + s * C::WK;
      const float w = use(r, before, x);
      if (lane < 32 && x * 32 + lane < hi && (there >> lane & 1))
        a.weights[pick((lane & 16) == 0, where[0].w0, where[0].w1) + (lane & 15)] = w;
#pragma unroll
      for (int y = 0; y < C::NS; ++y) where[y] = where[y + 1];
      at = at + 1 == C::NS ? 0 : at + 1;
      to = to + 1 == C::NS ? 0 : to + 1;
    }
  } else {
    Places4<C> pl;
    pl.set(a);
    auto load = [&](int x, int page, Raw4<C>& r, float& w) __attribute__((always_inline)) {
      load4<C, false>(a, pl, k, k, ks, ks, min(x, t_end - 1), place(page), r);
      w = old(x, page);
    };
    auto store = [&](int x, int page, float w) {
      const int j = x * 32 + lane;
      if (lane < 32 && j < hi && page >= 0 && page < a.pages) a.weights[weight_at(a, page, head, j)] = w;
    };
    Raw4<C> ra, rb;
    float wa, wb;
    int pa = page_of(i), pb = page_of(i + C::WK);
    load(i, pa, ra, wa);
    while (true) {
      int next = page_of(i + 2 * C::WK);
      load(i + C::WK, pb, rb, wb);
      store(i, pa, use(ra, wa, i));
      pa = next;
      i += C::WK;
      if (i >= t_end) break;
      next = page_of(i + 2 * C::WK);
      load(i + C::WK, pa, ra, wa);
      store(i, pb, use(rb, wb, i));
      pb = next;
      i += C::WK;
      if (i >= t_end) break;
    }
  }
}

// More rows: a wave keeps 64 keys as operands and goes through the rows that see them, 16 at a time; the
// scores stand as in the attention, S^T[key][row], so that a row's logarithm is one register and the sum over rows waits for
// the end. The workgroup's waves have the keys of WK neighbouring groups and WR shares of the rows. Rows and their
// logarithms come 64 at a time by way of LDS: loads in the operands' layout have neighbouring lanes in different rows
// and kept the address unit busy four times as long as the matrix cores (a prompt's last 1024 tokens 525 us, 345 now:
// 784 TFLOP/s, matrix instructions 31% of the cycles and 20% of them beside the powers that the rest goes to).
__device__ const uint32_t kZeros4[4] = {0, 0, 0, 0};  // what is copied past the width of the head

template <typename C>
struct Rows4Ring {
  static constexpr int kRows = 64, RB = C::D * 2, P = RB / 16;  // bytes of a row, 16-byte pieces
  static constexpr int RPI = kWave / P, CW = 16 / RPI;          // rows that a copy moves, a wave's copies
  static constexpr int NS = C::D <= 128 ? 3 : 2;
  static constexpr uint32_t kLse = kRows * RB, kStage = kLse + 4 * 256, kBytes = NS * kStage;
  static constexpr int IPS = CW + 1;
  static __device__ __forceinline__ int swizzle(int r) { return RB >= 256 ? r & 15 : (r >> 1) & (P - 1); }
};

template <typename C>
__global__ __launch_bounds__(C::kThreads) void key_weights_many_kernel(Attn4Args a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char attn4_smem[];
  typedef Rows4Ring<C> Ring;
  static_assert(C::kWaves == 4, "four waves copy 16 rows each");
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = (int)uniform32(tid >> 6), wr = wave % C::WR, wk = wave / C::WR;
  const int head = (int)blockIdx.x % a.kv_heads;
  const int rest = (int)blockIdx.x / a.kv_heads;
  const int n = rest / a.tiles;
  auto starts_at = [&](int i) { return min(max(a.starts[i], 0), a.tokens); };
  const int start = starts_at(n), T = starts_at(n + 1) - start, total = max(a.totals[n], 0), pos0 = total - T;
  const int hi = max((int)min((int64_t)min(total, a.max_length), a.table_width * (int64_t)a.page_size), 0);
  const int jg = (rest % a.tiles) * C::WK * 64;  // the workgroup's first key, and the wave's
  const int j0 = jg + wk * 64;
  if (T <= 0 || T > a.max_tokens || jg >= hi) return;
  float acc[4][4];
#pragma unroll
  for (int h = 0; h < 4; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[h][r] = 0.f;
  const int j = j0 + 16 * (c >> 2) + 4 * g + (c & 3);  // the key whose weight this lane writes
  const int32_t* trow = a.table + (int64_t)n * a.table_width;
  u32x4_t kk[4][C::KW];
  {
    Places4<C> pl;
    pl.set(a);
    const int64_t ho = (int64_t)head * a.head_stride;
    const unsigned char *k = a.k + ho, *ks = a.ks + ho / 16;
    Raw4<C> r[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int key = min(j0 + 32 * x + (lane & 31), hi - 1);
      const int page = trow[entry4(a, key)];
      load4<C, false>(a, pl, k, k, ks, ks, min(j0 / 32 + x, (hi - 1) / 32), page >= 0 && page < a.pages ? page : 0, r[x]);
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) keys4<C>(r[h >> 1], h & 1, kk[h]);
  }
  const int my_page = j < hi ? trow[entry4(a, j)] : -1;
  const int rows = T * a.group;
  // the first row that sees the workgroup's first key
  const int first = a.causal ? max(jg - pos0, 0) * a.group / 64 * 64 : 0;
  const int stages = rows > first ? (rows - first + 63) / 64 : 0;
  auto token_of = [&](int row) { return (int)(((uint64_t)(uint32_t)row * a.group_mul) >> a.group_shift); };
  auto copy = [&](int s) __attribute__((always_inline)) {
    const lds_t to = (lds_t)attn4_smem + (uint32_t)(s % Ring::NS) * Ring::kStage;
    const uint16_t* q = a.q + (int64_t)start * a.q_stride + (int64_t)head * a.group * a.d;
#pragma unroll
    for (int i = 0; i < Ring::CW; ++i) {
      const int r = wave * 16 + i * Ring::RPI + lane / Ring::P;
      const int piece = (lane % Ring::P) ^ Ring::swizzle(r), row = min(first + s * 64 + r, rows - 1), tok = token_of(row);
      const uint16_t* at = q + (int64_t)tok * a.q_stride + (int64_t)(row - tok * a.group) * a.d + piece * 8;
      copy16(to + (wave * 16 + i * Ring::RPI) * Ring::RB,
             (const unsigned char*)(piece * 8 < a.d ? at : (const uint16_t*)kZeros4));
    }
    const int row = min(first + s * 64 + wave * 16 + c, rows - 1), tok = token_of(row);
    copy4<false>(to + Ring::kLse + wave * 256,
                 (const unsigned char*)(a.lse_in + ((int64_t)start + tok) * a.heads + head * a.group + (row - tok * a.group)));
  };
  __builtin_amdgcn_s_waitcnt(0x0f70);  // the compiler's own loads, so that it waits for none among the copies
#pragma unroll
  for (int s = 0; s < Ring::NS - 1; ++s)
    if (s < stages) copy(s);
  for (int s = 0; s < stages; ++s) {
    constexpr int kAhead = Ring::NS - 2;
    if (s + kAhead < stages)
      __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead * Ring::IPS) : "memory");
    else
      __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (s + Ring::NS - 1 < stages) copy(s + Ring::NS - 1);
    const lds_t from = (lds_t)attn4_smem + (uint32_t)(s % Ring::NS) * Ring::kStage;
#pragma unroll 1
    for (int u = wr; u < 4; u += C::WR) {
      const int row = first + s * 64 + u * 16 + c;
      if (first + s * 64 + u * 16 >= rows) break;
      u32x4_t q[C::KW][C::kTerms];
#pragma unroll
      for (int w = 0; w < C::KW; ++w) {
        const u32x4_t in = *(lds_u32x4_t)(from + (u * 16 + c) * Ring::RB + ((g * C::KW + w) ^ Ring::swizzle(u * 16 + c)) * 16);
        Query<typename C::T>::split(in, q[w]);
      }
      const float v = *(lds_float_t)(from + Ring::kLse + u * 256 + c * 4);
      // no row, or one that sees nothing: its powers are 0
      const bool none = row >= rows || v == -__builtin_inff();
      const float ls = v * 1.4426950408889634f;
      const int p = pos0 + token_of(min(row, rows - 1));
      const bool all = !__ballot(none || (a.causal && p < j0 + 63));
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < C::KW; ++w)
#pragma unroll
          for (int t = 0; t < C::kTerms; ++t) sc = mfma16(kk[h][w], q[w][t], sc);
        if (!all) {
          const int last = none ? -1 : a.causal ? p - (j0 + 16 * h + 4 * g) : 4;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale2, -ls));
            acc[h][r] += r <= last ? e : 0.f;
          }
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[h][r] += __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale2, -ls));
        }
      }
    }
  }
  // the sum over the 16 lanes' rows; lane (c, g) takes key 16 (c / 4) + 4 g + c % 4
  float got = 0.f;
#pragma unroll
  for (int h = 0; h < 4; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float v = dpp_allreduce16(acc[h][r], [](float x, float y) { return x + y; });
      got = c == 4 * h + r ? v : got;
    }
  if constexpr (C::WR > 1) {
    __syncthreads();  // the last rows have been read
    *(lds_float_t)(attn4_smem + wave * 256 + lane * 4) = got;
    __syncthreads();
    if (wr != 0) return;
    got = 0.f;
#pragma unroll
    for (int w = 0; w < C::WR; ++w) got += *(lds_float_t)(attn4_smem + (wk * C::WR + w) * 256 + lane * 4);
  }
  if (my_page >= 0 && my_page < a.pages) {
    float* w = a.weights + weight_at(a, my_page, head, j);
    *w = (j < pos0 ? a.decay * *w : 0.f) + got;
  }
}

}  // namespace
}  // namespace lilicorr
