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
// of that list go to LDS by DMA, 16 bytes a lane from wherever the page table says, one stage
// ahead of the products (page numbers one more), with one barrier a stage. Sixteen-byte pieces are
// permuted within each row as they are copied so that the reads meet no bank conflicts.
//
// Softmax: running maximum and sum in fp32. The accumulated output is rescaled only when a
// row's maximum has grown by more than 2^8 over the one that its powers are taken against (they
// are then at most 2^8; fp32 sums and either 16-bit type hold that). Probabilities are rounded to
// the cache's type for the matrix cores, the sum is of the unrounded ones.
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
typedef __attribute__((address_space(3))) void* lds_void_t;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;
typedef __attribute__((address_space(3))) u32x4_t* lds_u32x4_t;
typedef __attribute__((address_space(3))) u32x2_t* lds_u32x2_t;
typedef __attribute__((address_space(3))) f32x4_t* lds_f32x4_t;
typedef __attribute__((address_space(3))) float* lds_float_t;
typedef __attribute__((address_space(3))) int* lds_int_t;

constexpr float kRescale = 8.f;  // growth of the maximum, in powers of two, that is let pass

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

// both halves of the wave see the larger of their value and the other half's
__device__ __forceinline__ float cross_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float cross_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

struct AttnArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  float* part_o;   // [slots][tokens * heads][d], where the keys are split
  f32x2_t* part_ml;  // [slots][tokens * heads]: maximum (powers of two) and sum
  const int32_t *table, *starts, *totals;
  int64_t q_stride, page_stride, token_stride, head_stride, rows;  // rows = tokens * heads
  int N, table_width, pages, page_size;
  uint32_t page_mul, page_shift;  // n / page_size = (n * page_mul) >> page_shift
  int tokens, heads, kv_heads, group, d;
  int window, sinks, causal;
  int max_tokens, max_length;
  int shared;            // 0, or the length of the shared keys, which this pass is for
  int tiles, chunk, slot0;  // keys of a chunk; slot of chunk 0
  int split;                        // whether partial results are written
  float scale2;                     // scale * log2 e
};

template <typename T_, int DP_, int WR_, int WK_, int KB_>
struct AttnConfig {
  typedef T_ T;
  static constexpr int DP = DP_, WR = WR_, WK = WK_, KB = KB_;
  static constexpr int kWaves = WR * WK, kThreads = kWaves * kWave;
  static constexpr int BM = 32 * WR;               // rows of a tile
  static constexpr int SK = 32 * KB * WK;          // keys of a stage
  static constexpr int RB = DP * 2;                // bytes of a row in LDS
  static constexpr int CPR = DP / 8;               // 16-byte pieces of it
  static constexpr int RPI = kWave / CPR;          // rows that one copy instruction moves
  static constexpr int WROWS = SK / kWaves;        // rows of a stage that a wave copies
  static constexpr int IPW = WROWS / RPI;          // copy instructions for them, keys or values
  static constexpr int ND = DP / 32;               // output tiles
  static constexpr int LOOK = SK < kWave ? SK : kWave;  // keys whose page a wave looks up
  static constexpr uint32_t kTile = SK * RB, kStage = 2 * kTile;
  static constexpr uint32_t kMerge = kWaves * 32 * DP * 4 + kWaves * kWave * 8;
  static constexpr uint32_t kFlag = WK > 1 && kMerge > 2 * kStage ? kMerge : 2 * kStage;
  static constexpr size_t kLds = kFlag + 16;       // and the word that calls for another try
  static_assert(WROWS % RPI == 0 && WROWS <= kWave, "whole copy instructions");
  static_assert(SK <= kWave || WR == 1, "a wave looks up the pages of what it copies and uses");
};

// which 16-byte piece of a row lies where: the keys' reads take one piece of 32 rows, the values'
// transposing reads four pieces of four rows
template <int CPR>
__device__ __forceinline__ uint32_t swizzle_k(uint32_t row) {
  return row & (CPR < 16 ? CPR - 1 : 15);
}
template <int CPR>
__device__ __forceinline__ uint32_t swizzle_v(uint32_t row) {
  const uint32_t r = row & 3;
  return CPR >= 16 ? (r << 2) | ((r ^ (r >> 1)) & 1) << 1 : r << 1;
}

// A chunk of the list of keys that a tile sees
struct Keys {
  const int32_t* table;
  int end, begin, ns, shift;
};

// One row by one wave, key by key, in fp32: what a tile falls back to when a value among the keys that
// not all of its rows see is infinite or NaN. A lane has four elements of the head.
template <typename T>
__device__ __forceinline__ void attention_row(const AttnArgs& a, const Keys keys, int start,
                                                        int pos0, int head, int r, int chunk_no,
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
    if ((a.causal && j > p) || (a.window && j <= p - a.window && j >= a.sinks)) continue;
    const int e = j / a.page_size, page = keys.table[e];
    if (page < 0 || page >= a.pages) continue;
    const int64_t at = (int64_t)page * a.page_stride + (int64_t)(j - e * a.page_size) * a.token_stride;
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
  if (a.split) {
    const int64_t at = (int64_t)(a.slot0 + chunk_no) * a.rows + orow;
    if (lane_id() == 0) a.part_ml[at] = f32x2_t{m, l};
    if (mine) *reinterpret_cast<f32x4_t*>(a.part_o + at * a.d + x) = f32x4_t{o[0], o[1], o[2], o[3]};
  } else if (mine) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<u32x2_t*>(a.out + orow * a.d + x) =
        u32x2_t{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
  }
}

template <typename C>
__device__ __forceinline__ void attention_tile(const AttnArgs& a, const int item, unsigned char* smem) {
  typedef typename C::T T;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = (int)__builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % C::WR, wk = wave / C::WR;
  const int col = lane & 31, half = lane >> 5;

  // ---- which rows ------------------------------------------------------------------------------
  const int head = item % a.kv_heads;
  const int rest = item / a.kv_heads;
  const int chunk_no = rest / a.tiles;
  // long rows first: with a causal mask and no window the last tiles of a request see most
  const int tile = a.tiles - 1 - rest % a.tiles;
  int n = 0, r0, start = 0, T_all, total;
  auto starts_at = [&](int i) { return min(max(a.starts[i], 0), a.tokens); };
  if (a.shared) {  // every query, against the shared keys
    r0 = tile * C::BM;
    T_all = starts_at(a.N);
    total = a.shared;
  } else {
    if ((int64_t)a.max_tokens * a.group <= C::BM) {
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
  const int T_n = min(T_all, a.max_tokens);
  if (r0 < 0) return;
  if (r0 >= (int64_t)T_n * a.group) return;
  const int r1 = (int)min((int64_t)T_n * a.group, (int64_t)r0 + C::BM);
  const int pos0 = total - T_all;  // position of the request's first query

  // ---- which keys ------------------------------------------------------------------------------
  const int p_lo = pos0 + r0 / a.group, p_hi = pos0 + (r1 - 1) / a.group;
  int hi = a.causal ? min(total, p_hi + 1) : total;
  hi = max(min(min(hi, a.max_length), (int)(a.table_width * (int64_t)a.page_size)), 0);
  const int lo = a.window ? min(max(p_lo - a.window + 1, 0), hi) : 0;
  const int ns = min(a.sinks, lo);
  const int shift = lo - ns;
  const int nv = ns + hi - lo;
  const int v_begin = chunk_no * a.chunk;
  const int v_end = (int)min((int64_t)nv, (int64_t)v_begin + a.chunk);

  const int row = r0 + wr * 32 + col;  // this lane's row
  const int rowc = min(row, r1 - 1);
  const int tok = rowc / a.group;
  const int64_t orow = ((int64_t)start + tok) * a.heads + head * a.group + (rowc - tok * a.group);
  const int p = pos0 + tok;  // its position: it sees the keys from j_least to j_most, and the sinks
  const int j_most = a.causal ? p : 0x7fffffff, j_least = a.window ? p - a.window + 1 : -0x7fffffff;
  if (v_begin >= nv && chunk_no > 0) {  // (chunk 0 of a tile without keys writes its zeros below)
    if (wk == 0 && half == 0 && row < r1)
      a.part_ml[(int64_t)(a.slot0 + chunk_no) * a.rows + orow] = f32x2_t{-__builtin_inff(), 0.f};
    return;
  }
  // the wave's rows, for the whole block's sake: positions of its first and last
  const int wrow0 = r0 + wr * 32;
  const bool has_rows = wrow0 < r1;
  const int wp_lo = pos0 + min(wrow0, r1 - 1) / a.group;
  const int wp_hi = pos0 + min(wrow0 + 31, r1 - 1) / a.group;

  // ---- queries: the second operand of the scores' product ---------------------------------------
  u32x4_t q[C::DP / 16];
  {
    const uint16_t* qp = a.q + ((int64_t)start + tok) * a.q_stride +
                         (int64_t)(head * a.group + (rowc - tok * a.group)) * a.d;
#pragma unroll
    for (int i = 0; i < C::DP / 16; ++i) {
      const int c = (2 * i + half) * 8;
      q[i] = c < a.d ? *reinterpret_cast<const u32x4_t*>(qp + c) : u32x4_t{0, 0, 0, 0};
    }
  }

  // ---- copies ------------------------------------------------------------------------------------
  const uint16_t* kbase = a.k + (int64_t)head * a.head_stride;
  const uint16_t* vbase = a.v + (int64_t)head * a.head_stride;
  const int32_t* trow = a.table + (int64_t)n * a.table_width;
  constexpr int kLookBase = C::SK <= kWave ? 0 : 1;  // stages wider than a wave: each its own part
  const int look0 = kLookBase ? wave * C::WROWS : 0;
  // pages of the list's positions v0 + look0 + lane; positions past the end take the last key
  struct Look { int page, off; };
  auto look = [&](int v0) {
    const int i = min(v0 + look0 + (lane < C::LOOK ? lane : 0), v_end - 1);
    const int j = i < ns ? i : i + shift;
    const int e = (int)(((uint64_t)(uint32_t)j * a.page_mul) >> a.page_shift);
    return Look{trow[e], j - e * a.page_size};
  };
  auto present = [&](const Look& w) { return w.page >= 0 && w.page < a.pages; };
  const int my_row = lane / C::CPR, my_pos = lane % C::CPR;
  auto copy = [&](const Look& w, int s) {
    const int64_t at = present(w) ? (int64_t)w.page * a.page_stride + (int64_t)w.off * a.token_stride : 0;
    unsigned char* dst = smem + (uint32_t)(s & 1) * C::kStage + (uint32_t)(wave * C::WROWS) * C::RB;
#pragma unroll
    for (int i = 0; i < C::IPW; ++i) {
      const int r = wave * C::WROWS + i * C::RPI + my_row;  // row of the stage
      const int64_t src = (int64_t)shfl64((uint64_t)at, r - look0);
      const uint32_t ck = my_pos ^ swizzle_k<C::CPR>(r), cv = my_pos ^ swizzle_v<C::CPR>(r);
      // past the head's width nothing is copied: the zeros put there before stay
      if ((int)ck * 8 < a.d)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(kbase + src + ck * 8),
                                         (lds_void_t)(dst + i * 1024), 16, 0, 0);
      if ((int)cv * 8 < a.d)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(vbase + src + cv * 8),
                                         (lds_void_t)(dst + C::kTile + i * 1024), 16, 0, 0);
    }
  };

  if (a.d < C::DP) {
    for (uint32_t i = tid * 16; i < 2 * C::kStage; i += C::kThreads * 16)
      *(lds_u32x4_t)(smem + i) = u32x4_t{0, 0, 0, 0};
    __syncthreads();
  }

  const auto again = (lds_int_t)(smem + C::kFlag);
  if (tid == 0) *again = 0;  // before the first stage's barrier; read after the last one's
  f32x16_t o[C::ND];
#pragma unroll
  for (int i = 0; i < C::ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -__builtin_inff(), l = 0.f;  // the maximum in score units; this half's share of the sum

  // LDS offsets of this lane's reads, without the stage
  const uint32_t sub = (uint32_t)wk * (C::KB * 32);  // first key of the wave's share of a stage
  const uint32_t k_at = (sub + col) * C::RB;
  const uint32_t k_x = half ^ swizzle_k<C::CPR>(col);
  const uint32_t v_row = 4 * half + ((lane & 15) >> 2);
  const uint32_t v_at = C::kTile + (sub + v_row) * C::RB + (lane & 1) * 8;
  const uint32_t v_c = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  const uint32_t v_x = swizzle_v<C::CPR>(v_row);

  const int stages = v_end > v_begin ? (v_end - v_begin + C::SK - 1) / C::SK : 0;
  Look next = {0, 0}, cur = {0, 0};
  if (stages) {
    cur = look(v_begin);
    copy(cur, 0);
    next = look(v_begin + C::SK);
  }
  for (int s = 0; s < stages; ++s) {
    const uint64_t have = __ballot(present(cur) || lane >= C::LOOK);
    // this wave's copies have landed, then everyone's; and all waves are done with the other buffer
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (s + 1 < stages) {
      copy(next, s + 1);
      cur = next;
      next = look(v_begin + (s + 2) * C::SK);
    }
    const int v0 = v_begin + s * C::SK + (int)sub;
    if (!has_rows || v0 >= v_end) continue;
    constexpr int kKeys = C::KB * 32;
    const int j_lo = v0 < ns ? v0 : v0 + shift, j_hi = v0 + kKeys - 1 + shift;
    if (v0 >= ns && ((a.causal && j_lo > wp_hi) || (a.window && j_hi <= wp_lo - a.window && j_lo >= a.sinks)))
      continue;  // no row of the wave sees any of it
    constexpr uint64_t kAll = kKeys == 64 ? ~0ull : ((1ull << kKeys) - 1);
    uint64_t here = (have >> (C::SK <= kWave ? (int)sub : 0)) & kAll;  // list positions with a key
    if (v_end - v0 < kKeys) here &= (1ull << (v_end - v0)) - 1;
    const bool whole = here == kAll && (v0 >= ns || shift == 0) &&
                       (!a.causal || j_hi <= wp_lo) && (!a.window || j_lo > wp_hi - a.window);
    unsigned char* st = smem + (uint32_t)(s & 1) * C::kStage;

    // scores
    f32x16_t sc[C::KB];
#pragma unroll
    for (int b = 0; b < C::KB; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
#pragma unroll
      for (int i = 0; i < C::DP / 16; ++i) {
        const u32x4_t kf = *(lds_u32x4_t)(st + k_at + b * 32 * C::RB + ((k_x ^ (2 * i)) * 16));
        sc[b] = mfma<T>(kf, q[i], sc[b]);
      }
    }
    auto key_of = [&](int b, int e) { return v0 + b * 32 + 8 * (e >> 2) + 4 * half + (e & 3); };
    auto sees = [&](int v) {  // this lane's row and the list's position v
      const int j = v < ns ? v : v + shift;
      return ((here >> (v - v0)) & 1) && j <= j_most && (j >= j_least || j < a.sinks);
    };
    if (!whole) {
#pragma unroll
      for (int b = 0; b < C::KB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sc[b][e] = sees(key_of(b, e)) ? sc[b][e] : -__builtin_inff();
    }
    // maximum
    float mx = sc[0][0];
#pragma unroll
    for (int b = 0; b < C::KB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[b][e]);
    mx = cross_max(mx);
    if (__ballot((mx - m) * a.scale2 > kRescale)) {  // -inf - -inf is NaN and does not count
      const float grown = fmaxf(m, mx);
      // nothing is accumulated while m is -inf
      const float f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m - grown) * a.scale2);
      m = grown;
      l *= f;
#pragma unroll
      for (int i = 0; i < C::ND; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= f;
    }
    const float ms = m == -__builtin_inff() ? 0.f : m * a.scale2;
    u32x4_t pf[C::KB * 2];
#pragma unroll
    for (int b = 0; b < C::KB; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        sc[b][e] = __builtin_amdgcn_exp2f(fmaf(sc[b][e], a.scale2, -ms));
        l += sc[b][e];
      }
#pragma unroll
      for (int e = 0; e < 16; e += 2) pf[b * 2 + (e >> 3)][(e & 7) >> 1] = T::pack(sc[b][e], sc[b][e + 1]);
    }
    // A value that is not finite, in a key that some row does not see, must not reach that row, but
    // 0 * inf is NaN. Rare enough for the whole tile to be done again another way.
    if (!whole) {
      constexpr int kReads = kKeys / C::RPI;
      uint32_t any = 0;
#pragma unroll 4
      for (int i = 0; i < kReads; ++i) {
        const u32x4_t w = *(lds_u32x4_t)(st + C::kTile + sub * C::RB + i * 1024 + lane * 16);
        any |= T::nonfinite(w[0]) | T::nonfinite(w[1]) | T::nonfinite(w[2]) | T::nonfinite(w[3]);
      }
      if (any) *again = 1;
    }
    // output
    auto v_frag = [&](int g, int t) {
      const uint32_t at = v_at + 16 * g * C::RB + (((4 * t + v_c) ^ v_x) * 16);
      u32x4_t vf;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const u32x2_t w = __builtin_bit_cast(
            u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(st + at + 8 * y * C::RB)));
        vf[2 * y] = w[0];
        vf[2 * y + 1] = w[1];
      }
      return vf;
    };
#pragma unroll
    for (int g = 0; g < C::KB * 2; ++g)
#pragma unroll
      for (int t = 0; t < C::ND; ++t) o[t] = mfma<T>(v_frag(g, t), pf[g], o[t]);
  }

  __syncthreads();  // the last stage has been read, and `again` written
  if (*again) {
    const Keys keys = {trow, v_end, v_begin, ns, shift};
    for (int r = r0 + wave; r < r1; r += C::kWaves)
      attention_row<T>(a, keys, start, pos0, head, r, chunk_no, kbase, vbase);
    return;
  }

  // ---- join the waves that shared the keys ---------------------------------------------------------
  l = cross_sum(l);
  float mp = m * a.scale2;  // in powers of two
  if constexpr (C::WK > 1) {
    constexpr uint32_t kMl = C::kWaves * 32 * C::DP * 4;
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
  if (a.split) {
    const int64_t at = (int64_t)(a.slot0 + chunk_no) * a.rows + orow;
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

template <typename C>
__global__ __launch_bounds__(C::kThreads) __attribute__((amdgpu_waves_per_eu(C::DP > 128 ? 1 : 2)))
void attention_kernel(AttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char attn_smem[];
  attention_tile<C>(a, (int)blockIdx.x, attn_smem);
}

// Joins the slots of every row in their order: one row for d / 4 lanes.
constexpr int kJoinThreads = 256;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(
    const float* __restrict__ part_o, const f32x2_t* __restrict__ part_ml, int64_t rows, int slots,
    int d, int lanes, const int32_t* __restrict__ starts, int N, int heads, uint16_t* out) {
  const int64_t per = kJoinThreads / lanes;
  const int64_t row = blockIdx.x * per + threadIdx.x / lanes;
  const int x = (threadIdx.x % lanes) * 4;
  const int64_t used = (int64_t)starts[N] * heads;
  if (row >= rows || row >= used || x >= d) return;
  float top = -__builtin_inff(), l = 0.f;
  for (int s = 0; s < slots; ++s) top = fmaxf(top, part_ml[s * rows + row][0]);
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < slots; ++s) {
    const f32x2_t ml = part_ml[s * rows + row];
    if (ml[1] == 0.f) continue;  // saw nothing; a NaN stays one
    const float f = ml[0] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ml[0] - top);
    l += f * ml[1];
    o += f * *reinterpret_cast<const f32x4_t*>(part_o + (s * rows + row) * d + x);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2_t*>(out + row * d + x) =
      u32x2_t{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
}

}  // namespace
}  // namespace lilicorr
