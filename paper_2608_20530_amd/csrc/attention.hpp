// The attention kernel over the paged cache (lilicorr_window_attention, lilicorr_prefix_attention).
//
// A row is one query head of one token; the heads / cache heads query heads of a key head are
// neighbours, so the rows of a request and key head are its tokens' groups one after the other, and
// all of them read the same keys and values. A workgroup takes a tile of 32 * WR rows of one key head
// and a chunk of its keys; its WR x WK waves are WR blocks of 32 rows by WK shares of the keys.
//
// Everything is transposed so that a row stays in one lane pair from the scores to the output.
// 32 x 32 x 16 matrix instructions: scores S^T[key][row] = K . Q^T leave lane l with row l % 32 and
// the keys 8 a + 4 (l / 32) + b (a, b < 4) of a block of 32. That is, up to the order of the keys, what the
// second product O^T[dim][row] = V^T . P^T wants of P^T as its second operand, so the
// probabilities go from one product to the next without leaving their lane: only the maximum crosses
// to the other half of the wave, and the sum does once at the end. V^T comes from V as it lies by
// transposing LDS reads, in the same order of keys.
//
// The keys that a tile sees are the first few (sinks) and a run (the window): one list, in which
// position i is key i below the number of sinks and key i + shift above. Stages of 32 KB WK keys
// of that list go to LDS by DMA, 16 bytes a lane from wherever the page table says, into a ring of
// NS stages. Sixteen-byte pieces are permuted within each row as they are copied so that the reads
// meet no bank conflicts (counted: none with heads of 128; with heads of 64 about one cycle a read is left).
// Where WR is 1 each wave copies just what it uses and meets no barrier.
//
// Softmax: running maximum and sum in fp32. The accumulated output is rescaled only when a
// row's maximum has grown by more than 2^8 over the power of two that its powers are taken against (they
// are then at most 2^8; fp32 sums and bf16 hold that, and fp16 holds them times 2^7, which it is given).
// Probabilities are rounded to the cache's type, once, because the matrix cores multiply 16-bit operands (two
// terms of a probability would double the second product); the sum (fp32) is of the rounded ones, as the
// output is, so that weights add up to one. A rescaling is by a power of two and rounds none of them again.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "paged.hpp"

namespace lilicorr {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;
typedef __attribute__((address_space(3))) u32x4_t* lds_u32x4_t;
typedef __attribute__((address_space(3))) f32x4_t* lds_f32x4_t;
typedef __attribute__((address_space(3))) float* lds_float_t;
typedef __attribute__((address_space(3))) int* lds_int_t;
typedef __attribute__((address_space(3))) unsigned char* lds_t;

constexpr int kWaitLoads = 0x0f70;  // s_waitcnt vmcnt(0) alone
constexpr float kRescale = 8.f;  // growth of the maximum, in powers of two, that is let pass
// The power of two that the powers' reference is given (the maximum's lies at most 2^8 above it): fp16 ends at
// 2^16, and its steps of 2^-24 would lose a long run of small probabilities beside one of 1
template <typename T>
constexpr float kLift = 0.f;
template <>
constexpr float kLift<F16> = 7.f;

template <typename T>
__device__ __forceinline__ f32x16_t mfma(const u32x4_t& a, const u32x4_t& b, const f32x16_t& c);
template <>
__device__ __forceinline__ f32x16_t mfma<Bf16>(const u32x4_t& a, const u32x4_t& b,
                                               const f32x16_t& c) {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a),
                                                 __builtin_bit_cast(x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16_t mfma<F16>(const u32x4_t& a, const u32x4_t& b,
                                              const f32x16_t& c) {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a),
                                                __builtin_bit_cast(x8, b), c, 0, 0, 0);
}

// c + a + b for the packed pair, in fp32
template <typename T>
__device__ __forceinline__ float add_pair(uint32_t w, float c);
template <>
__device__ __forceinline__ float add_pair<Bf16>(uint32_t w, float c) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, w), __builtin_bit_cast(pair, 0x3f803f80u), c,
                                         false);
}
template <>
__device__ __forceinline__ float add_pair<F16>(uint32_t w, float c) {
  typedef _Float16 pair __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2(__builtin_bit_cast(pair, w), __builtin_bit_cast(pair, 0x3c003c00u), c, false);
}

// the largest of three; a NaN counts only beside NaNs
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  __asm__("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// bits at and above n, and below it, of 64 (any n)
__device__ __forceinline__ uint64_t bits_from(int n) { return n <= 0 ? ~0ull : n >= 64 ? 0 : ~0ull << n; }
__device__ __forceinline__ uint64_t bits_below(int n) { return ~bits_from(n); }

// both halves of the wave see the larger of their value and the other half's
__device__ __forceinline__ float cross_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max3(__uint_as_float(r[0]), __uint_as_float(r[1]), -__builtin_inff());
}
__device__ __forceinline__ float cross_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16 bytes a lane from where each lane says to 1 KB of LDS in lane order, counted by vmcnt alone. Written
// out because the compiler takes this instruction for one that LDS reads must wait for too: it made
// every read of the loops wait for all that were under way (prefill 608 us with the builtin). No register
// is loaded, so none is in flight.
__device__ __forceinline__ void copy_to_lds(lds_t dst, const unsigned char* src) {
  const uint32_t at = uniform32((uint32_t)(uintptr_t)dst);
  __asm__ volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(at), "v"(src) : "memory");
}

// One pass over keys: over the requests' own ones, or over the shared ones for every query
struct AttnPass {
  const int32_t* table;
  int table_width;
  int shared;          // 0, or the length of the shared keys, which this pass is for
  int tiles, chunk;    // row tiles; keys of a chunk
  int most;            // keys of all chunks
  int items;           // tiles * heads * chunks
  int spread;          // XCDs take runs of items instead of every eighth
  int slot0;           // slot of chunk 0
  int max_tokens, max_length;
  int window, sinks, causal;
};

struct AttnArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  float* part_o;     // [slots][tokens * heads][d], where the keys are split
  f32x2_t* part_ml;  // [slots][tokens * heads]: maximum (powers of two) and sum
  const int32_t *starts, *totals;
  int64_t q_stride, rows;  // rows = tokens * heads
  int64_t head_stride;
  int N, pages, page_size;
  uint32_t page_mul, page_shift;  // n / page_size = (n * page_mul) >> page_shift
  int tokens, heads, kv_heads, group, d;
  uint32_t page_units, token_units, unit_bytes;  // page and token strides in a common unit
  int split;     // whether partial results are written, which attention_join_kernel joins
  float scale2;  // scale * log2 e
  AttnPass shared, own;
};

// heads of D elements (FULL) or fewer, in LDS rows of 64, 128 or 256
template <typename T_, bool FULL_, int D_, int WR_, int WK_, int KB_, int NS_>
struct AttnConfig {
  static constexpr bool FULL = FULL_;
  static constexpr int D = D_, DP = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  typedef T_ T;
  static constexpr int WR = WR_, WK = WK_, KB = KB_, NS = NS_;
  static constexpr int kWaves = WR * WK, kThreads = kWaves * kWave;
  static constexpr int BM = 32 * WR;               // rows of a tile
  static constexpr int SK = 32 * KB * WK;          // keys of a stage
  static constexpr int RB = DP * 2;                // bytes of a row in LDS
  static constexpr int CPR = DP / 8;               // 16-byte pieces of it
  static constexpr int RPI = kWave / CPR;          // rows that one copy instruction moves
  static constexpr int WROWS = SK / kWaves;        // rows of a stage that a wave copies
  static constexpr int IPW = WROWS / RPI;          // copy instructions for them, keys or values
  static constexpr int ND = D / 32;                // output tiles
  static constexpr int LOOK = SK < kWave ? SK : kWave;  // keys whose page a wave looks up
  static constexpr bool kOwn = WR == 1;            // a wave copies just the keys that it uses
  static constexpr uint32_t kTile = SK * RB, kStage = 2 * kTile, kRing = NS * kStage;
  static constexpr uint32_t kMerge = kWaves * 32 * D * 4 + kWaves * kWave * 8;
  // the ring, which the join of the waves uses again; each wave's part of the page table; the word
  // that calls for another try
  static constexpr uint32_t kPages = WK > 1 && kMerge > kRing ? kMerge : kRing;
  static constexpr int kEntries = 256;
  static constexpr uint32_t kFlag = kPages + kWaves * kEntries * 4;
  static constexpr size_t kLds = kFlag + 16;
  // waves of a SIMD, which the kernel's registers are given out for, and workgroups that a compute unit
  // holds with them and its 160 KB of LDS
  static constexpr int kSimdWaves = DP > 128 ? 1 : 2;
  static constexpr int kByWaves = 4 * kSimdWaves / kWaves, kByLds = 160 * 1024 / (int)kLds;
  static constexpr int kAtOnce = kByWaves < kByLds ? kByWaves : kByLds;
  static_assert(kAtOnce >= 1, "a workgroup fits");
  static_assert(KB <= 2, "blocks of a stage and wave");
  static_assert(WROWS % RPI == 0 && WROWS <= kWave, "whole copy instructions");
};

// Piece c of row r of a stage lies at place c ^ swizzle(r) of the row. The keys' reads take one piece of 32
// rows, eight lanes a cycle: eight consecutive rows differ modulo 8, sixteen modulo 16. The values'
// transposing reads take two neighbouring pieces of four consecutive rows with 16 lanes: those rows
// differ in bits 1-2 (and the four pieces that 32 lanes take, in bits 2-3).
template <int CPR>
__device__ __forceinline__ uint32_t swizzle(uint32_t row) {
  const uint32_t r = row & 3, k = row >> 2;
  if (CPR < 16) return (r << 1) ^ (k & 1);
  return (r << 2) ^ (((r ^ (r >> 1)) & 1) << 1) ^ (k & 1) ^ ((k & 2) << 2);
}

// what is copied past the width of heads that are narrower than DP
__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};

// A chunk of the list of keys that a tile sees
struct Keys {
  const int32_t* table;
  int end, begin, ns, shift;
};

// One row by one wave, key by key, in fp32: what a tile falls back to when a value among the keys that
// not all of its rows see is infinite or NaN. A lane has four elements of the head. A last resort, half a
// microsecond a row and key: one infinite value at the edge of one request's mask makes a call of 64 blocks of 16
// behind 4000 keys take 36 ms instead of 0.2.
template <typename T>
__device__ __forceinline__ void attention_row(const AttnArgs& a, const AttnPass& ps, const Keys keys,
                                             int start, int pos0, int head, int r, int64_t part_row,
                                             const uint16_t* kbase, const uint16_t* vbase) {
  const int x = lane_id() * 4;
  const bool mine = x < a.d;
  const int tok = r / a.group, p = pos0 + tok, h = head * a.group + (r - tok * a.group);
  const int64_t orow = ((int64_t)start + tok) * a.heads + h;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -__builtin_inff(), l = 0.f;
  auto load = [&](const uint16_t* at, float(&f)[4]) {
    u32x2_t w = {0, 0};
    if (mine) w = *reinterpret_cast<const u32x2_t*>(at + x);
    const f32x2_t lo = T::unpack(w[0]), hi = T::unpack(w[1]);
    f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
  };
  load(a.q + ((int64_t)start + tok) * a.q_stride + (int64_t)h * a.d, q);
  for (int i = keys.begin; i < keys.end; ++i) {
    const int j = i < keys.ns ? i : i + keys.shift;
    if ((ps.causal && j > p) || (ps.window && j <= p - ps.window && j >= ps.sinks)) continue;
    const int e = j / a.page_size, page = keys.table[e];
    if (page < 0 || page >= a.pages) continue;
    const int64_t at = ((int64_t)((uint32_t)page * a.page_units +
                                  (uint32_t)(j - e * a.page_size) * a.token_units) * a.unit_bytes) >> 1;
    float k[4], v[4];
    load(kbase + at, k);
    load(vbase + at, v);
    const float s = wave_sum(q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3]) * a.scale2;
    const float top = fmaxf(m, s);
    const float f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - top);
    const float w = s == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(s - top);
    m = top;
    l = l * f + w;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = o[c] * f + w * v[c];
  }
  if (part_row >= 0) {
    const int64_t at = part_row + orow;
    if (lane_id() == 0) a.part_ml[at] = f32x2_t{m, l};
    if (mine) *reinterpret_cast<f32x4_t*>(a.part_o + at * a.d + x) = f32x4_t{o[0], o[1], o[2], o[3]};
  } else if (mine) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<u32x2_t*>(a.out + orow * a.d + x) =
        u32x2_t{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
  }
}

template <typename C>
__device__ __forceinline__ void attention_tile(const AttnArgs& a, const AttnPass& ps, const int item,
                                               unsigned char* smem) {
  typedef typename C::T T;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = (int)__builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % C::WR, wk = wave / C::WR;
  const int col = lane & 31, half = lane >> 5;

  // ---- which rows ------------------------------------------------------------------------------
  int it = item;
  if (ps.spread) {
    const int per = ps.items / 8;
    if (it < per * 8) it = (it % 8) * per + it / 8;
  }
  const int head = it % a.kv_heads;
  const int rest = it / a.kv_heads;
  const int chunk_no = rest / ps.tiles;
  // long rows first: with a causal mask and no window the last tiles of a request see most
  const int tile = ps.tiles - 1 - rest % ps.tiles;
  int n = 0, r0, start = 0, T_all, total;
  auto starts_at = [&](int i) { return min(max(a.starts[i], 0), a.tokens); };
  if (ps.shared) {  // every query, against the shared keys
    r0 = tile * C::BM;
    T_all = starts_at(a.N);
    total = ps.shared;
  } else {
    if ((int64_t)ps.max_tokens * a.group <= C::BM) {
      n = tile;
      r0 = 0;
    } else {
      // request n's tiles have the numbers floor(starts[n] * group / BM) + n and on, which is at
      // least as many as it has; 64 candidates at a time
      auto first_tile = [&](int i) {
        return (int)((int64_t)starts_at(i) * a.group / C::BM) + i;
      };
      int end = a.N;
      while (end - n > 1) {
        const int step = (end - n + kWave - 1) / kWave, i = n + lane * step;
        const uint64_t le = __ballot(i < end && first_tile(i) <= tile);
        const int last = 63 - __builtin_clzll(le | 1);
        n += last * step;
        end = min(end, n + step);
      }
      n = (int)uniform32(n);
      r0 = (tile - first_tile(n)) * C::BM;
    }
    start = starts_at(n);
    T_all = starts_at(n + 1) - start;
    total = max(a.totals[n], 0);
  }
  const int T_n = min(T_all, ps.max_tokens);
  if (r0 < 0) return;
  if (r0 >= (int64_t)T_n * a.group) return;
  const int r1 = (int)min((int64_t)T_n * a.group, (int64_t)r0 + C::BM);
  const int pos0 = total - T_all;  // position of the request's first query

  // ---- which keys ------------------------------------------------------------------------------
  const int p_lo = pos0 + r0 / a.group, p_hi = pos0 + (r1 - 1) / a.group;
  int hi = ps.causal ? min(total, p_hi + 1) : total;
  hi = max(min(min(hi, ps.max_length), (int)(ps.table_width * (int64_t)a.page_size)), 0);
  const int lo = ps.window ? min(max(p_lo - ps.window + 1, 0), hi) : 0;
  const int ns = min(ps.sinks, lo);
  const int shift = lo - ns;
  const int nv = min(ns + hi - lo, ps.most);
  const int v_begin = chunk_no * ps.chunk;
  const int v_end = (int)min((int64_t)nv, (int64_t)v_begin + ps.chunk);

  const int row = r0 + wr * 32 + col;  // this lane's row
  const int rowc = min(row, r1 - 1);
  const int tok = rowc / a.group;
  const int64_t orow = ((int64_t)start + tok) * a.heads + head * a.group + (rowc - tok * a.group);
  const int p = pos0 + tok;  // its position: it sees the keys from j_least to j_most, and the sinks
  const int j_most = ps.causal ? p : 0x3fffffff, j_least = ps.window ? p - ps.window + 1 : -0x3fffffff;
  if (v_begin >= nv && chunk_no > 0) {  // (chunk 0 of a tile without keys writes its zeros below)
    if (wk == 0 && half == 0 && row < r1)
      a.part_ml[(int64_t)(ps.slot0 + chunk_no) * a.rows + orow] = f32x2_t{-__builtin_inff(), 0.f};
    return;
  }
  // where the chunk's partial results go
  const int64_t part_row = a.split ? (int64_t)(ps.slot0 + chunk_no) * a.rows : -1;
  // the wave's rows, for the whole block's sake: positions of its first and last
  const int wrow0 = r0 + wr * 32;
  const int wp_lo = pos0 + min(wrow0, r1 - 1) / a.group;
  const int wp_hi = pos0 + min(wrow0 + 31, r1 - 1) / a.group;

  // ---- queries: the second operand of the scores' product ---------------------------------------
  u32x4_t q[C::D / 16];
  {
    const uint16_t* qp = a.q + ((int64_t)start + tok) * a.q_stride +
                         (int64_t)(head * a.group + (rowc - tok * a.group)) * a.d;
#pragma unroll
    for (int i = 0; i < C::D / 16; ++i) {
      const int c = (2 * i + half) * 8;
      q[i] = c < a.d ? *reinterpret_cast<const u32x4_t*>(qp + c) : u32x4_t{0, 0, 0, 0};
    }
  }

  // ---- copies ------------------------------------------------------------------------------------
  const uint16_t* kbase = a.k + (int64_t)head * a.head_stride;
  const uint16_t* vbase = a.v + (int64_t)head * a.head_stride;
  const unsigned char *kbytes = (const unsigned char*)kbase, *vbytes = (const unsigned char*)vbase;
  const int32_t* trow = ps.table + (int64_t)n * ps.table_width;
  // The page numbers of the list's positions, in LDS: the entries of the sinks, then those of the
  // window. A wave keeps kEntries of them, from number x0 on, and fetches the next ones when a stage
  // runs out of them, so that page numbers are not waited for among the copies.
  const int look0 = C::SK <= kWave ? 0 : wave * C::WROWS;
  const int xs = (ns + a.page_size - 1) / a.page_size;
  auto entry_of = [&](int j) { return (int)(((uint64_t)(uint32_t)j * a.page_mul) >> a.page_shift); };
  const int e_lo = entry_of(lo);
  auto number_of = [&](int i, int e) { return i < ns ? e : e - e_lo + xs; };
  const uint32_t tab = C::kPages + wave * (C::kEntries * 4);
  int x0 = 0;
  bool absent = false;  // a page among those so far is not there
  auto fetch = [&](int x, int x_last) {
    x0 = x;
    int page[C::kEntries / kWave];
    bool gone = false;
#pragma unroll
    for (int u = 0; u < C::kEntries / kWave; ++u) {
      const int y = min(x + u * kWave + lane, x_last);
      page[u] = trow[y < xs ? y : y - xs + e_lo];
    }
#pragma unroll
    for (int u = 0; u < C::kEntries / kWave; ++u) {
      gone |= page[u] < 0 || page[u] >= a.pages;
      *(lds_int_t)(smem + tab + (u * kWave + lane) * 4) = page[u];
    }
    absent |= __ballot(gone) != 0;
  };
  const int x_last = v_end > 0 ? number_of(v_end - 1, entry_of(v_end - 1 < ns ? v_end - 1 : v_end - 1 + shift)) : 0;
  const int my_row = lane / C::CPR, my_pos = lane % C::CPR;
  // Where the rows of the stage whose first position is v0 lie, for the copies of this wave; positions
  // past the end take the last key. It is asked for a stage ahead of the copies, among the products.
  typedef uint32_t places_t __attribute__((ext_vector_type(C::IPW)));
  auto prepare = [&](int v0) __attribute__((always_inline)) {
    auto key_at = [&](int i) { return i < ns ? i : i + shift; };
    const int first = min(v0 + look0, v_end - 1), last = min(v0 + look0 + C::LOOK - 1, v_end - 1);
    if (number_of(last, entry_of(key_at(last))) >= x0 + C::kEntries)
      fetch(number_of(first, entry_of(key_at(first))), x_last);
    const int i = min(v0 + look0 + (C::LOOK < kWave && lane >= C::LOOK ? 0 : lane), v_end - 1);
    const int j = key_at(i), e = entry_of(j);
    int page = *(lds_int_t)(smem + tab + (number_of(i, e) - x0) * 4);
    if (absent && (page < 0 || page >= a.pages)) page = 0;
    const uint32_t at = (uint32_t)page * a.page_units + (uint32_t)(j - e * a.page_size) * a.token_units;
    places_t to;
#pragma unroll
    for (int i = 0; i < C::IPW; ++i)
      to[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(
          (wave * C::WROWS + i * C::RPI + my_row - look0) * 4, (int)at);
    return to;
  };
  // and their copies, to the place at `ring`
  auto copy = [&](const places_t from, lds_t ring) __attribute__((always_inline)) {
    const lds_t dst = ring + (uint32_t)(wave * C::WROWS) * C::RB;
#pragma unroll
    for (int i = 0; i < C::IPW; ++i) {
      const int r = wave * C::WROWS + i * C::RPI + my_row;  // row of the stage
      const uint32_t piece = my_pos ^ swizzle<C::CPR>(r);
      const unsigned char* ks = kbytes + piece * 16 + (uint64_t)from[i] * a.unit_bytes;
      const unsigned char* vs = ks + (vbytes - kbytes);
      if constexpr (!C::FULL) {
        if ((int)piece * 8 >= a.d) ks = vs = (const unsigned char*)kZeros;
      }
      copy_to_lds(dst + i * 1024, ks);
      copy_to_lds(dst + C::kTile + i * 1024, vs);
    }
  };

  const auto again = (lds_int_t)(smem + C::kFlag);
  if (tid == 0) *again = 0;  // before the first stage's barrier; read after the last one's
  f32x16_t o[C::ND];
#pragma unroll
  for (int i = 0; i < C::ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  // the power of two that the powers are taken against; this half's share of the sum
  float m = -__builtin_inff(), l = 0.f;

  // LDS offsets of this lane's reads, without the stage
  const uint32_t sub = (uint32_t)wk * (C::KB * 32);  // first key of the wave's share of a stage
  const uint32_t k_at = (sub + col) * C::RB;
  const uint32_t k_x = half ^ swizzle<C::CPR>(col);
  const uint32_t v_row = 4 * half + ((lane & 15) >> 2);
  const uint32_t v_at = C::kTile + (sub + v_row) * C::RB + (lane & 1) * 8;
  const uint32_t v_c = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  const uint32_t v_x = swizzle<C::CPR>(v_row);

  const int stages = v_end > v_begin ? (v_end - v_begin + C::SK - 1) / C::SK : 0;
  // The first page numbers, and with them everything asked for so far: the products below find their
  // operands there and wait for nothing but the copies.
  if (stages) {
    const int first = min(v_begin + look0, v_end - 1);
    fetch(number_of(first, entry_of(first < ns ? first : first + shift)), x_last);
  }
  __builtin_amdgcn_s_waitcnt(kWaitLoads);
  if constexpr (C::kOwn) __syncthreads();  // `again` is 0 before any wave sets it
#pragma unroll
  for (int s = 0; s < C::NS - 1; ++s)
    if (s < stages) {
      copy(prepare(v_begin + s * C::SK), (lds_t)smem + s * C::kStage);
    }
  places_t from = {};
  if (C::NS - 1 < stages) from = prepare(v_begin + (C::NS - 1) * C::SK);
  constexpr int kAhead = C::kOwn ? C::NS - 1 : C::NS - 2;  // stages under way while this one is waited for
  // stage s, which lies at st, while a later one is copied to nx
  auto stage = [&](const lds_t st, const lds_t nx, int s) __attribute__((always_inline)) {
    const bool more = s + C::NS - 1 < stages;
    // a wave that uses its own copies alone begins the next one and waits for its oldest; otherwise
    // the barrier says that everyone's copies have landed and that all are done with the place that the
    // next ones overwrite
    __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the last stage's reads
    if constexpr (C::kOwn) {
      if (more) copy(from, nx);
    }
    if (C::kOwn ? more : s + C::NS - 2 < stages)
      __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead * 2 * C::IPW) : "memory");
    else
      __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (!C::kOwn) {
      __asm__ volatile("s_barrier" ::: "memory");
      if (more) copy(from, nx);
    }
    const bool later = s + C::NS < stages;
    const int v0 = v_begin + s * C::SK + (int)sub;
    constexpr int kKeys = C::KB * 32;
    const int j_lo = v0 < ns ? v0 : v0 + shift, j_hi = v0 + kKeys - 1 + shift;
    constexpr uint64_t kAll = kKeys == 64 ? ~0ull : ((1ull << kKeys) - 1);
    uint64_t here = kAll;  // list positions with a key
    if (absent) {
      const int i = min(v0 + (lane < kKeys ? lane : 0), v_end - 1);
      const int page = trow[entry_of(i < ns ? i : i + shift)];
      here &= __ballot(page >= 0 && page < a.pages);
    }
    here &= bits_below(v_end - v0);
    const bool whole = here == kAll && (v0 >= ns || shift == 0) &&
                       (!ps.causal || j_hi <= wp_lo) && (!ps.window || j_lo > wp_hi - ps.window);
    // the list's positions v0 .. that this lane's row sees: of the sinks' part keys up to its own, of
    // the window's part its window, and sinks that lie in it
    uint64_t vis = 0;
    if (!whole) {
      const uint64_t part = bits_below(ns - v0);
      const int w0 = v0 + shift;
      vis = here & ((part & bits_below(j_most + 1 - v0)) |
                    (~part & bits_below(j_most + 1 - w0) & (bits_from(j_least - w0) | bits_below(ps.sinks - w0))));
      vis >>= 4 * half;
    }
    // Blocks of 32 keys. While one block's powers are taken, the matrix cores have the next block's
    // scores or the last one's output to do: the two are laid out in steps of one matrix instruction
    // each, with operands read three steps ahead, and the scheduler is held to that.
    constexpr int kQK = C::D / 16, kPV = 2 * C::ND;  // steps of a block
    f32x16_t sc[C::KB];
    u32x4_t pf[C::KB * 2], kf[4], vf[4];
    auto load_k = [&](int x) {  // operand x % kQK of block x / kQK
      if (x < kQK * C::KB)
        kf[x & 3] = *(lds_u32x4_t)(st + k_at + (x / kQK) * 32 * C::RB + ((k_x ^ (2 * (x % kQK))) * 16));
    };
    auto load_v = [&](int x) {  // operand of 16 keys x / ND and output tile x % ND
      if (x >= kPV * C::KB) return;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        // rows eight apart differ in bit 3 of the swizzle, rows sixteen apart not at all
        const uint32_t place = (4 * (x % C::ND) + v_c) ^ v_x ^ (C::CPR < 16 ? 0 : 8 * y);
        const uint32_t at = v_at + (16 * (x / C::ND) + 8 * y) * C::RB + place * 16;
        const u32x2_t w = __builtin_bit_cast(
            u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(st + at)));
        vf[x & 3][2 * y] = w[0];
        vf[x & 3][2 * y + 1] = w[1];
      }
    };
    auto score_step = [&](int b, int i) {
      load_k(b * kQK + i + 3);
      if (i == 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
      }
      sc[b] = mfma<T>(kf[(b * kQK + i) & 3], q[i], sc[b]);
    };
    auto output_step = [&](int b, int i) {
      load_v(b * kPV + i + 3);
      o[i % C::ND] = mfma<T>(vf[(b * kPV + i) & 3], pf[2 * b + i / C::ND], o[i % C::ND]);
    };
    float ms = 0.f;
    auto power_step = [&](int b, int e0, int e1) {
#pragma unroll
      for (int e = e0; e < e1; ++e) {
        sc[b][e] = __builtin_amdgcn_exp2f(fmaf(sc[b][e], a.scale2, -ms));
        if (e & 1) {
          uint32_t w = T::pack(sc[b][e - 1], sc[b][e]);
          l = add_pair<T>(w, l);
          __asm__ volatile("" : "+v"(w), "+v"(l));  // here and not later
          pf[b * 2 + (e >> 3)][(e & 7) >> 1] = w;
        }
      }
    };
    // masks the block's scores and brings the maximum up to it: to a whole power of two, so that what is
    // there already changes by an exact factor
    auto maximum = [&](int b) {
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sc[b][e] = (uint32_t)(vis >> (b * 32)) & (1u << (8 * (e >> 2) + (e & 3))) ? sc[b][e] : -__builtin_inff();
      }
      float mx = sc[b][0];
#pragma unroll
      for (int e = 1; e < 15; e += 2) mx = max3(mx, sc[b][e], sc[b][e + 1]);
      mx = cross_max(max3(mx, sc[b][15], mx));
      const bool grows = fmaf(mx, a.scale2, -m) > kRescale;  // -inf - -inf is NaN and does not count
      if (__ballot(grows)) {
        // nothing is accumulated while m is -inf
        const float up = __builtin_floorf(mx * a.scale2);
        const float f = grows ? __builtin_amdgcn_ldexpf(1.f, (int)fmaxf(m - up, -300.f)) : 1.f;
        m = grows ? up : m;
        l *= f;
#pragma unroll
        for (int i = 0; i < C::ND; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[i][e] *= f;
        if (b > 0) {  // the block before has its powers but is not in the output yet
#pragma unroll
          for (int w = 0; w < 8; ++w) {
            const f32x2_t v = T::unpack(pf[(b - 1) * 2 + (w >> 2)][w & 3]);
            pf[(b - 1) * 2 + (w >> 2)][w & 3] = T::pack(v[0] * f, v[1] * f);
          }
        }
      }
    };
    load_k(0);
    load_k(1);
    load_k(2);
#pragma unroll
    for (int i = 0; i < kQK; ++i) {
      score_step(0, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (later) from = prepare(v_begin + (s + C::NS) * C::SK);
#pragma unroll
    for (int b = 0; b < C::KB; ++b) {
      if (b == C::KB - 1) {
        load_v(0);
        load_v(1);
        load_v(2);
      }
      maximum(b);
      ms = m == -__builtin_inff() ? 0.f : m - kLift<T>;
      if (b + 1 < C::KB) {
#pragma unroll
        for (int i = 0; i < kQK; ++i) {
          score_step(b + 1, i);
          power_step(b, i * 16 / kQK, (i + 1) * 16 / kQK);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else if (b > 0) {
#pragma unroll
        for (int i = 0; i < kPV; ++i) {
          output_step(b - 1, i);
          power_step(b, i * 16 / kPV, (i + 1) * 16 / kPV);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        power_step(b, 0, 16);
      }
    }
    // A value that is not finite, in a key that some row does not see, must not reach that row, but
    // 0 * inf is NaN. Rare enough for the whole tile to be done again another way.
    if (!whole) {
      constexpr int kReads = kKeys / C::RPI;
      uint32_t any = 0;
#pragma unroll 1
      for (int i = 0; i < kReads; ++i) {
        const u32x4_t w = *(lds_u32x4_t)(st + C::kTile + sub * C::RB + i * 1024 + lane * 16);
        any |= T::nonfinite(w[0]) | T::nonfinite(w[1]) | T::nonfinite(w[2]) | T::nonfinite(w[3]);
      }
      if (any) *again = 1;
    }
#pragma unroll
    for (int i = 0; i < kPV; ++i) {
      output_step(C::KB - 1, i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if constexpr (C::NS == 2 && C::kRing <= 65536) {  // places that fit the reads' immediate offsets
    for (int s = 0; s < stages; s += 2) {
      stage((lds_t)smem, (lds_t)smem + C::kStage, s);
      if (s + 1 < stages) stage((lds_t)smem + C::kStage, (lds_t)smem, s + 1);
    }
  } else {
    uint32_t ring = 0, ring_new = (C::NS - 1) * C::kStage;
    for (int s = 0; s < stages; ++s) {
      stage((lds_t)smem + ring, (lds_t)smem + ring_new, s);
      ring = ring + C::kStage == C::kRing ? 0 : ring + C::kStage;
      ring_new = ring_new + C::kStage == C::kRing ? 0 : ring_new + C::kStage;
    }
  }

  __syncthreads();  // the last stage has been read, and `again` written
  if (*again) {
    const Keys keys = {trow, v_end, v_begin, ns, shift};
    for (int r = r0 + wave; r < r1; r += C::kWaves)
      attention_row<T>(a, ps, keys, start, pos0, head, r, part_row, kbase, vbase);
    return;
  }

  // ---- join the waves that shared the keys ---------------------------------------------------------
  l = cross_sum(l);
  float mp = m - kLift<T>;
  if constexpr (C::WK > 1) {
    constexpr uint32_t kMl = C::kWaves * 32 * C::D * 4;
#pragma unroll
    for (int t = 0; t < C::ND; ++t)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *(lds_f32x4_t)(smem + (((wave * C::ND + t) * 4 + y) * kWave + lane) * 16) =
            f32x4_t{o[t][4 * y], o[t][4 * y + 1], o[t][4 * y + 2], o[t][4 * y + 3]};
    *(lds_float_t)(smem + kMl + (wave * 2) * kWave * 4 + lane * 4) = mp;
    *(lds_float_t)(smem + kMl + (wave * 2 + 1) * kWave * 4 + lane * 4) = l;
    __syncthreads();
    float f[C::WK], top = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < C::WK; ++w) {
      f[w] = *(lds_float_t)(smem + kMl + ((w * C::WR + wr) * 2) * kWave * 4 + lane * 4);
      top = fmaxf(top, f[w]);
    }
    l = 0.f;
#pragma unroll
    for (int w = 0; w < C::WK; ++w) {
      f[w] = f[w] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(f[w] - top);
      l += f[w] * *(lds_float_t)(smem + kMl + ((w * C::WR + wr) * 2 + 1) * kWave * 4 + lane * 4);
    }
    mp = top;
#pragma unroll
    for (int t = 0; t < C::ND; ++t) {
      if (t % C::WK != wk) continue;  // each of the WK waves joins its share of the output tiles
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < C::WK; ++w)
          sum += f[w] * *(lds_f32x4_t)(smem + ((((w * C::WR + wr) * C::ND + t) * 4 + y) * kWave + lane) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][4 * y + e] = sum[e];
      }
    }
  }

  // ---- write ---------------------------------------------------------------------------------------
  if (row >= r1) return;
  if (part_row >= 0) {
    const int64_t at = part_row + orow;
    if (wk == 0 && half == 0) a.part_ml[at] = f32x2_t{mp, l};
    float* po = a.part_o + at * a.d;
#pragma unroll
    for (int t = 0; t < C::ND; ++t) {
      if (t % C::WK != wk) continue;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int x = t * 32 + 8 * y + 4 * half;
        if (x < a.d)
          *reinterpret_cast<f32x4_t*>(po + x) =
              f32x4_t{o[t][4 * y], o[t][4 * y + 1], o[t][4 * y + 2], o[t][4 * y + 3]};
      }
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing gives zeros
  uint16_t* out = a.out + orow * a.d;
#pragma unroll
  for (int t = 0; t < C::ND; ++t) {
    if (t % C::WK != wk) continue;
#pragma unroll
    for (int y = 0; y < 4; y += 2) {
      // the halves exchange so that each lane has eight neighbours
      u32x4_t w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto r = __builtin_amdgcn_permlane32_swap(
            T::pack(o[t][4 * y + 2 * e] * inv, o[t][4 * y + 2 * e + 1] * inv),
            T::pack(o[t][4 * y + 4 + 2 * e] * inv, o[t][4 * y + 5 + 2 * e] * inv), false, false);
        w[e] = r[0];
        w[2 + e] = r[1];
      }
      const int x = t * 32 + 8 * y + 8 * half;
      if (x < a.d) *reinterpret_cast<u32x4_t*>(out + x) = w;
    }
  }
}

// The shared keys' items come first, where there are any, then the requests' own.
//
// What bounds it (32 heads over 8 key heads of 128, bf16). Few rows a request: reading the cache, once 256
// workgroups are there to read it; 765 us for 256 requests of one token and 100 to 8100 keys (5.65 TB/s),
// 195 us for 64 blocks of 16 behind windows of 4096 (5.2 TB/s). One request: a chain of dependent loads
// (lengths, page numbers, first keys: 2.9, 1.4 and 2 to 5 us cold), 10 us for one token behind a window of
// 4096. Many rows: how far the two waves of a SIMD overlap; 585 to 615 us (895 to 941 TFLOP/s) for 8192 tokens
// behind windows of 4096. Of the SIMDs' cycles 43% have a matrix instruction running and 38% another vector
// instruction, 16% both and about a third neither (counted; waves spend 29% of their time at waits and barriers).
// What 64 keys of a wave cost there, found by leaving a part out: powers 65 us, copies 87, edges of masks 26, the
// test of the maximum 17, page numbers 10. Two waves a SIMD need at most
// 256 registers; tiles of 256 rows in eight waves take 650 us, deeper operand rings and wave priorities
// gain nothing.
template <typename C>
__global__ __launch_bounds__(C::kThreads) __attribute__((amdgpu_waves_per_eu(C::kSimdWaves, C::kSimdWaves)))
void attention_kernel(AttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char attn_smem[];
  const int item = (int)blockIdx.x - a.shared.items;
  attention_tile<C>(a, item < 0 ? a.shared : a.own, item < 0 ? (int)blockIdx.x : item, attn_smem);
}

// Joins the slots of every row in their order, a wave a row: maxima and sums one lane a slot, then the
// partial outputs in 16 bytes a lane, LPR lanes a slot and 64 / LPR slots at once.
// Its first outputs are asked for beside the sums, so that it takes one round trip: 3.5 us for one token behind
// a window of 4096, 20 us (bytes) for 32768 rows. A kernel of its own: joined by the last workgroup to arrive, one
// token took 25 us against 16 (the counter's round trips come after the outputs').
constexpr int kJoinThreads = 256;
template <typename T, int LPR>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(
    const float* __restrict__ part_o, const f32x2_t* __restrict__ part_ml, int64_t rows, int slots,
    int d, const int32_t* __restrict__ starts, int N, int tokens, int heads,
    uint16_t* __restrict__ out) {
  constexpr int kAtOnce = kWave / LPR;
  const int lane = lane_id();
  const int64_t row = (int64_t)blockIdx.x * (kJoinThreads / kWave) + threadIdx.x / kWave;
  const int x = (lane % LPR) * 4;
  if (row >= rows) return;
  const int64_t used = (int64_t)min(max(starts[N], 0), tokens) * heads;
  float top = -__builtin_inff(), l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < slots; s0 += kWave) {
    const int here = min(slots - s0, kWave);
    constexpr int kBatch = 8;
    f32x4_t v[kBatch];
    // a slot that saw nothing holds no output: read all the same, beside its sum, and not used
    auto load = [&](int b) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int s = b + u * kAtOnce + lane / LPR;
        v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (s < here && x < d)
          v[u] = *reinterpret_cast<const f32x4_t*>(part_o + ((s0 + s) * rows + row) * d + x);
      }
    };
    f32x2_t ml = {-__builtin_inff(), 0.f};
    if (lane < here) ml = part_ml[(s0 + lane) * rows + row];
    load(0);
    const float grown = fmaxf(top, wave_max_dpp(ml[0]));
    const float f0 = top == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(top - grown);
    // the sum of a slot that saw nothing is 0; a NaN stays one
    const float f = ml[0] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ml[0] - grown);
    const bool saw = ml[1] != 0.f;
    top = grown;
    l = l * f0 + wave_sum_dpp(saw ? f * ml[1] : 0.f);
    o *= f0;
    const uint64_t which = __ballot(saw);
    for (int b = 0; b < here; b += kBatch * kAtOnce) {
      if (b) load(b);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int s = b + u * kAtOnce + lane / LPR;
        const bool on = s < here && ((which >> (s & 63)) & 1);
        const float w = __shfl(f, s & 63, kWave);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += on ? w * v[u][e] : 0.f;
      }
    }
  }
  if (row >= used) return;
#pragma unroll
  for (int m = LPR; m < kWave; m <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m, kWave);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lane < LPR && x < d)
    *reinterpret_cast<u32x2_t*>(out + row * d + x) =
        u32x2_t{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
}

}  // namespace
}  // namespace lilicorr
