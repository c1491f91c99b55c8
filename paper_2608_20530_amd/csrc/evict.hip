// lilicorr_evict: which tokens of a request a cache head keeps, and their move to the front.
//
// Two kernels. The first one (a workgroup for a request and head) finds the weight of the last token that is kept, bit
// by bit from the top (a radix selection: three histograms of 11, 11 and 10 bits of the weights' order), and
// lists the kept tokens in order. The second one moves them in place: kept token i goes to place i, which is never
// behind where it comes from, so a workgroup that has a stretch of tokens in registers may overwrite everything up to
// where they came from. It goes from stretch to stretch, in order; different 16-byte columns of the cache's rows do not
// meet, so the columns are shared out over workgroups where requests and heads are few.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache4.hpp"
#include "common.hpp"
#include "lilicorr.h"
#include "paged.hpp"

namespace lilicorr {
namespace {

constexpr int kEvictMaxN = 4096;
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave;
constexpr int kBins = 2048;
constexpr int kMoveThreads = 512;

struct EvictArgs {
  unsigned char *k, *v, *ks, *vs;
  float* weights;
  const int32_t *table, *totals, *pages;
  int32_t* queue;
  const int64_t* cursor;
  int32_t *totals_out, *pages_out, *evicted;
  int64_t* cursor_out;
  int32_t* list;  // [N][heads][budget]: slots of the kept tokens, -1 for one without a page
  int64_t page_stride, token_stride, head_stride;
  int N, M, P, C, heads, d, n_pages;
  uint32_t page_mul, page_shift;
  int budget, limit, sinks, recent, max_length;
  // workgroups of the move that share a request and head's wide columns (2, or one for each), and the narrow ones
  int wides, narrows;
  bool words;  // whether scales can be moved 4 at a time
};

struct EvictRow {
  int length, end, left;  // tokens, pages before and after
  bool cut;
};
__device__ __forceinline__ EvictRow evict_row(const EvictArgs& a, int n) {
  EvictRow r;
  r.end = min(max(a.pages[2 * n], 0), a.M);
  r.length = max(min(min(a.totals[n], a.max_length), r.end * a.P), 0);  // P * M < 2^31
  r.cut = r.length > a.limit;
  r.left = r.cut ? (int)(((int64_t)a.budget + a.P - 1) / a.P) : r.end;
  return r;
}

__device__ __forceinline__ int evict_entry(const EvictArgs& a, int j) {
  return (int)(((uint64_t)(uint32_t)j * a.page_mul) >> a.page_shift);
}

// What the calls of this step make of request n besides its keys: its numbers, and its pages to the queue. One workgroup.
__device__ __forceinline__ void evict_numbers(const EvictArgs& a, int n) {
  __shared__ int s_sum[2][kSelectWaves];
  const int tid = threadIdx.x;
  const EvictRow row = evict_row(a, n);
  int before = 0, all = 0;
  for (int i = tid; i < a.N; i += kSelectThreads) {
    const EvictRow r = evict_row(a, i);
    all += r.end - r.left;
    if (i < n) before += r.end - r.left;
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    before += __shfl_xor(before, m, kWave);
    all += __shfl_xor(all, m, kWave);
  }
  if (lane_id() == 0) {
    s_sum[0][tid / kWave] = before;
    s_sum[1][tid / kWave] = all;
  }
  __syncthreads();
  before = all = 0;
  for (int w = 0; w < kSelectWaves; ++w) {
    before += s_sum[0][w];
    all += s_sum[1][w];
  }
  const int64_t tail = a.cursor[1];
  if (tid == 0) {
    const int after = row.cut ? a.budget : row.length;
    a.totals_out[n] = after;
    a.evicted[n] = row.length - after;
    a.pages_out[2 * n] = row.left;
    a.pages_out[2 * n + 1] = a.pages[2 * n + 1];
    if (n == 0) {
      a.cursor_out[0] = a.cursor[0];
      a.cursor_out[1] = tail + all;
      a.cursor_out[2] = a.cursor[2];
    }
  }
  for (int i = tid; i < row.end - row.left; i += kSelectThreads) {
    const int64_t at = (tail + before + i) % a.C;
    a.queue[at < 0 ? at + a.C : at] = a.table[(int64_t)n * a.M + row.left + i];
  }
}

// Bound by instructions and by the round trips of one workgroup: 32768 tokens of 8 heads take 26 us, 64 requests of 500 to
// 16000 tokens and 8 heads 27. A thread has KEYS neighbouring tokens or fewer, so that G of them (4, or 1 where pages
// are no multiple of it) share a page number and a load, and the order of the kept ones is a sum over threads: 48 us
// and 58 with tokens 1024 apart, where each needs a page number, ballots and counts of its own.
template <int G, int KEYS>
__global__ __launch_bounds__(kSelectThreads, G == 4 && KEYS == 16 ? 8 : 4) void evict_select_kernel(EvictArgs a) {
  constexpr int kKeys = KEYS;  // weights that a thread keeps
  // four counts a bin, for a quarter of the lanes each: many weights share a few bins (4096 that no query has met
  // all have 0), and additions of one instruction to one address come one after the other
  __shared__ __attribute__((aligned(16))) int s_bins[kBins * 4];
  __shared__ uint32_t s_wave[4][kSelectWaves];
  __shared__ int s_found[3][2];
  const int tid = threadIdx.x, lane = lane_id(), wave = (int)uniform32(tid / kWave);
  if ((int)blockIdx.x >= a.N * a.heads) return evict_numbers(a, (int)blockIdx.x - a.N * a.heads);
  const int n = (int)blockIdx.x / a.heads, head = (int)blockIdx.x % a.heads;
  const EvictRow row = evict_row(a, n);
  if (!row.cut) return;

  const int32_t* trow = a.table + (int64_t)n * a.M;
  int need = a.budget - a.sinks - a.recent;
  const bool none = need <= 0;  // weights decide about nothing
  // Tokens in stretches of kSelectThreads * kKeys. One stretch is the rule, and its keys are read once.
  constexpr int kStretch = kSelectThreads * kKeys;
  const int stretches = (int)uniform32((row.length + kStretch - 1) / kStretch);
  const int per = stretches > 1 ? kKeys : ((row.length + kSelectThreads - 1) / kSelectThreads + 3) / 4 * 4;
  // The weights' order, greater for the heavier (a token without a page comes last), and slots of the first of G tokens.
  constexpr int kSlots = kKeys / G, kAtOnce = loads_at_once(kSlots);
  static_assert(kKeys % G == 0 && kSlots % kAtOnce == 0, "batches fill the arrays");
  uint32_t key[kKeys] = {};
  int slot[kSlots];
  auto read = [&](int jt) {
#pragma unroll
    for (int x0 = 0; x0 < kSlots; x0 += kAtOnce) {
      if (x0 * G >= per) break;
      int page[kAtOnce], o[kAtOnce];
#pragma unroll
      for (int x = 0; x < kAtOnce; ++x) {
        const int j = min(jt + (x0 + x) * G, (row.length - 1) / G * G), e = evict_entry(a, j);
        page[x] = trow[e];
        o[x] = j - e * a.P;
      }
      float w[kAtOnce][G];
#pragma unroll
      for (int x = 0; x < kAtOnce; ++x) {
        const bool there = page[x] >= 0 && page[x] < a.n_pages;
        slot[x0 + x] = there ? page[x] * a.P + o[x] : -1;
        const float* at = a.weights + ((int64_t)(there ? page[x] : 0) * a.heads + head) * a.P + o[x];
        if constexpr (G == 4) {
          const f32x4_t v = *reinterpret_cast<const f32x4_t*>(at);
#pragma unroll
          for (int y = 0; y < G; ++y) w[x][y] = v[y];
        } else {
          w[x][0] = *at;
        }
      }
#pragma unroll
      for (int x = 0; x < kAtOnce; ++x)
#pragma unroll
        for (int y = 0; y < G; ++y) key[(x0 + x) * G + y] = slot[x0 + x] < 0 ? 0 : order_bits(w[x][y]);
    }
  };
  // bit i: whether it holds for key i
  auto bits = [&](auto holds) {
    uint32_t m = 0;
#pragma unroll
    for (int i = kKeys - 1; i >= 0; --i) m = m + m + (holds(key[i]) ? 1u : 0u);
    return m;
  };
  struct Tokens {
    uint32_t valid, mid;  // of a thread's tokens, those that there are, and those that weights decide about
  };
  auto tokens = [&](int jt) {
    Tokens t;
    t.valid = bits32_below(min(row.length - jt, per));
    t.mid = bits32_from(a.sinks - jt) & bits32_below(row.length - a.recent - jt) & t.valid;
    return t;
  };
  for (int i = tid; i < kBins * 4; i += kSelectThreads) s_bins[i] = 0;
  if (stretches == 1) read(tid * per);
  __syncthreads();

  uint32_t prefix = 0, known = 0;  // the bits of the border that are known, and where
  constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
#pragma unroll 1
  for (int pass = 0; pass < 3 && !none; ++pass) {
    const int shift = kShift[pass];
    const uint32_t mask = (1u << kBits[pass]) - 1;
    for (int s = 0; s < stretches; ++s) {
      const int jt = s * kStretch + tid * per;
      if (stretches > 1) read(jt);
      const uint32_t in = tokens(jt).mid & bits([&](uint32_t k) { return (k & known) == prefix; });
#pragma unroll
      for (int i = 0; i < kKeys; ++i)
        if (in >> i & 1) atomicAdd(&s_bins[(key[i] >> shift & mask) * 4 + (lane & 3)], 1);
    }
    __syncthreads();
    // the bin, from the top, in which the need-th key lies: each thread has the bins 2 x and 2 x + 1 from the top
    u32x4_t* own = reinterpret_cast<u32x4_t*>(s_bins) + kBins - 2 - 2 * tid;
    const u32x4_t l = own[0], h = own[1];
    const int top = (int)(h[0] + h[1] + h[2] + h[3]), low = (int)(l[0] + l[1] + l[2] + l[3]);
    own[0] = own[1] = u32x4_t{0, 0, 0, 0};  // for the next pass
    int sum = top + low;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
      const int o = __shfl_up(sum, m, kWave);
      if (lane >= m) sum += o;
    }
    if (lane == kWave - 1) s_wave[pass][wave] = (uint32_t)sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) sum += (int)s_wave[pass][w];
    const int above = sum - top - low;  // keys in the bins above this thread's
    if (above < need && need <= sum) {
      const bool upper = above + top >= need;
      s_found[pass][0] = upper ? kBins - 1 - 2 * tid : kBins - 2 - 2 * tid;
      s_found[pass][1] = upper ? above : above + top;
    }
    __syncthreads();
    prefix |= ((uint32_t)s_found[pass][0] & mask) << shift;
    known |= mask << shift;
    need -= s_found[pass][1];  // of the keys that share the known bits
  }

  int base_more = 0, base_equal = 0;
  int32_t* list = a.list + ((int64_t)n * a.heads + head) * a.budget;
  for (int s = 0; s < stretches; ++s) {
    const int jt = s * kStretch + tid * per;
    if (stretches > 1) read(jt);
    const Tokens t = tokens(jt);
    // one bit for a token: kept, kept if it is among the first `need` of its kind
    const uint32_t more = t.valid & ~t.mid | (none ? 0 : t.mid & bits([&](uint32_t k) { return k > prefix; }));
    const uint32_t equal = none ? 0 : t.mid & bits([&](uint32_t k) { return k == prefix; });
    // both counts of the threads before, in 16 bits each (a stretch has at most 2^15 tokens)
    const uint32_t own = (uint32_t)__popc(more) | (uint32_t)__popc(equal) << 16;
    uint32_t sum = own;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
      const uint32_t o = (uint32_t)__shfl_up((int)sum, m, kWave);
      if (lane >= m) sum += o;
    }
    if (lane == kWave - 1) s_wave[3][wave] = sum;
    __syncthreads();
    uint32_t all = 0;
    sum -= own;
    for (int w = 0; w < kSelectWaves; ++w) {
      all += s_wave[3][w];
      if (w < wave) sum += s_wave[3][w];
    }
    int e0 = base_equal + (int)(sum >> 16);
    int at = base_more + (int)(sum & 0xffff) + min(e0, need);
#pragma unroll
    for (int x = 0; x < kSlots; ++x)
#pragma unroll
      for (int y = 0; y < G; ++y) {
        const int i = x * G + y;
        const bool eq = equal >> i & 1;
        if ((more >> i & 1) || (eq && e0 < need)) list[at++] = slot[x] < 0 ? -1 : slot[x] + y;
        e0 += eq;
      }
    base_more += (int)(all & 0xffff);
    base_equal += (int)(all >> 16);
    __syncthreads();
  }
}

// A row of a head is columns of 16 bytes, d / 32 of the key and d / 32 of the value, and three narrow ones: the keys' scales,
// the values' scales and the weight. A workgroup moves the keys' columns of a request and head, or the values', or one,
// or narrow ones. A thread holds kHold columns of a stretch, or kNarrow narrow ones, and all loads of a kind are under way
// together (64 requests of 8 heads: the call 86 us, 107 with 8 columns, 90 with 2). A request's heads, which share
// cache lines, go to one XCD (139 us against 161 when they did not).
//
// While a stretch is written the next one is read: what it writes lies at places below its end, and later tokens come
// from places behind that. The wait before the barrier says that every wave has read the stretch that is written.
constexpr int kHold = 4, kNarrow = 4;
__global__ __launch_bounds__(kMoveThreads, 4) void evict_move_kernel(EvictArgs a) {
  const int tid = threadIdx.x, parts = a.wides + a.narrows;
  const int it = beside((int)blockIdx.x, a.N * a.heads * parts, a.heads * parts);  // (neighbouring heads share lines)
  const int part = it % parts, nh = it / parts;
  const int n = nh / a.heads, head = nh % a.heads;
  if (!evict_row(a, n).cut) return;
  const int wide = a.d / kBlock4;  // 16-byte columns of a key; also scale bytes
  const int32_t* list = a.list + (int64_t)nh * a.budget;
  const int32_t* trow = a.table + (int64_t)n * a.M;
  const int64_t ho = (int64_t)head * a.head_stride;
  auto offset = [&](int slot) {  // bytes of codes
    const int page = evict_entry(a, slot);  // slot / P
    return (int64_t)page * a.page_stride + (int64_t)(slot - page * a.P) * a.token_stride + ho;
  };
  auto weight = [&](int slot) {
    const int page = evict_entry(a, slot);
    return a.weights + ((int64_t)page * a.heads + head) * a.P + (slot - page * a.P);
  };
  // Item `item` of a stretch from i0 on with `count` items, `per` of a token: first its slot and its place's page, and when
  // they are there the slot of the place, -1 where there is nothing to do
  auto places = [&](int i0, int item, int count, int per, int& src, int& dst) {
    const int i = i0 + min(item, count - 1) / per;
    src = list[i];
    dst = trow[evict_entry(a, i)];
  };
  auto settle = [&](int i0, int item, int count, int per, int& src, int& dst) {
    const int i = i0 + min(item, count - 1) / per, e = evict_entry(a, i);
    const int slot = dst >= 0 && dst < a.n_pages ? dst * a.P + (i - e * a.P) : -1;
    dst = item >= count || src < 0 || src == slot ? -1 : slot;
    src = max(src, 0);
  };
  if (part < a.wides) {
    const int cs = 2 * wide / a.wides, c0 = part * cs, rows = kMoveThreads * kHold / cs;
    auto count = [&](int i0) { return min(rows, a.budget - i0) * cs; };
    auto column = [&](int x, int slot) {
      const int c = c0 + (x * kMoveThreads + tid) % cs;
      return reinterpret_cast<u32x4_t*>((c < wide ? a.k : a.v) + offset(slot) + (c % wide) * 16);
    };
    auto ask = [&](int i0, int (&src)[kHold], int (&dst)[kHold]) {
      if (i0 >= a.budget) return;
#pragma unroll
      for (int x = 0; x < kHold; ++x) places(i0, x * kMoveThreads + tid, count(i0), cs, src[x], dst[x]);
    };
    auto take = [&](int i0, int (&src)[kHold], int (&dst)[kHold], u32x4_t (&held)[kHold]) {
      if (i0 >= a.budget) return;
#pragma unroll
      for (int x = 0; x < kHold; ++x) {
        settle(i0, x * kMoveThreads + tid, count(i0), cs, src[x], dst[x]);
        held[x] = *column(x, src[x]);
      }
    };
    int src[kHold] = {}, to[kHold] = {}, next[kHold] = {};
    u32x4_t held[kHold] = {}, more[kHold] = {};
    ask(0, src, to);
    take(0, src, to, held);
    ask(rows, src, next);
    for (int i0 = 0; i0 < a.budget; i0 += rows) {
      __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      take(i0 + rows, src, next, more);
      int then[kHold] = {};
      ask(i0 + 2 * rows, src, then);
#pragma unroll
      for (int x = 0; x < kHold; ++x) {
        if (to[x] >= 0) *column(x, to[x]) = held[x];
        to[x] = next[x];
        next[x] = then[x];
        held[x] = more[x];
      }
    }
  } else {
    const int kinds = 3 / a.narrows, k0 = (part - a.wides) * kinds, rows = kMoveThreads * kNarrow / kinds;
    for (int i0 = 0; i0 < a.budget; i0 += rows) {
      const int items = min(rows, a.budget - i0) * kinds;
      int from[kNarrow], to[kNarrow];
      uint32_t held[kNarrow][8];
#pragma unroll
      for (int x = 0; x < kNarrow; ++x) places(i0, x * kMoveThreads + tid, items, kinds, from[x], to[x]);
#pragma unroll
      for (int x = 0; x < kNarrow; ++x) {
        const int kind = k0 + (x * kMoveThreads + tid) % kinds;
        settle(i0, x * kMoveThreads + tid, items, kinds, from[x], to[x]);
        if (kind == 2) {
          held[x][0] = __float_as_uint(*weight(from[x]));
        } else {
          const unsigned char* at = (kind == 0 ? a.ks : a.vs) + offset(from[x]) / 16;
          if (a.words) {
#pragma unroll
            for (int b = 0; b < 2; ++b) held[x][b] = reinterpret_cast<const uint32_t*>(at)[min(b, wide / 4 - 1)];
          } else {
#pragma unroll
            for (int b = 0; b < 8; ++b) held[x][b] = at[min(b, wide - 1)];
          }
        }
      }
      __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kNarrow; ++x) {
        if (to[x] < 0) continue;
        const int kind = k0 + (x * kMoveThreads + tid) % kinds;
        if (kind == 2) {
          *weight(to[x]) = __uint_as_float(held[x][0]);
        } else {
          unsigned char* at = (kind == 0 ? a.ks : a.vs) + offset(to[x]) / 16;
          if (a.words) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
              if (b < wide / 4) reinterpret_cast<uint32_t*>(at)[b] = held[x][b];
          } else {
#pragma unroll
            for (int b = 0; b < 8; ++b)
              if (b < wide) at[b] = (unsigned char)held[x][b];
          }
        }
      }
    }
  }
}

constexpr int64_t kMostTokens = (int64_t)1 << 30;

lilicorr_status evict_sizes(const lilicorr_evict_args& x) {
  if (const lilicorr_status s = cache4_sizes(x.cache)) return s;
  if (x.N < 1 || x.table_width < 1 || x.queue_size < 1 || x.max_length < 0 || x.budget < 1 || x.limit < x.budget ||
      x.sinks < 0 || x.recent < 0 || x.sinks > x.budget || x.recent > x.budget - x.sinks)
    return LILICORR_ERR_INVALID_ARG;
  if (x.N > kEvictMaxN || x.table_width > kMostTokens / x.cache.page_size || x.queue_size > 0x7fffffffll ||
      x.budget > kMostTokens || x.N * x.cache.heads > 0x7fffffffll / 32)
    return LILICORR_ERR_UNSUPPORTED;
  return LILICORR_OK;
}

size_t evict_bytes(const lilicorr_evict_args& x) {
  // requests are cut to the budget only if they can be longer
  const int64_t most = x.table_width * x.cache.page_size;
  const size_t list = most > x.budget ? (size_t)x.N * x.cache.heads * (size_t)x.budget * 4 : 0;
  return list < 256 ? 256 : list;
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" size_t lilicorr_evict_workspace_bytes(const lilicorr_evict_args* args) {
  return args && evict_sizes(*args) == LILICORR_OK ? evict_bytes(*args) : 0;
}

extern "C" lilicorr_status lilicorr_evict(const lilicorr_evict_args* args, hipStream_t stream) {
  if (!args) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_evict_args& x = *args;
  if (const lilicorr_status s = evict_sizes(x)) return s;
  const lilicorr_cache4& c = x.cache;
  if (!c.k || !c.v || !c.k_scales || !c.v_scales || !x.weights || !x.table || !x.totals || !x.pages || !x.queue ||
      !x.cursor || !x.totals_out || !x.pages_out || !x.evicted || !x.cursor_out)
    return LILICORR_ERR_INVALID_ARG;
  if (!aligned16(c.k) || !aligned16(c.v) || !aligned4(c.k_scales) || !aligned4(c.v_scales) ||
      !aligned16(x.weights) || !aligned16(x.workspace) || !aligned4(x.table) ||
      !aligned4(x.totals) || !aligned4(x.pages) || !aligned4(x.queue) || !aligned8(x.cursor) ||
      !aligned4(x.totals_out) || !aligned4(x.pages_out) || !aligned4(x.evicted) || !aligned8(x.cursor_out))
    return LILICORR_ERR_ALIGNMENT;
  if (!x.workspace || x.workspace_bytes < evict_bytes(x)) return LILICORR_ERR_WORKSPACE;
  // only the arrays that are not written may share memory
  constexpr int kRead = 4;
  const size_t n4 = (size_t)x.N * 4, span = cache4_span(c);
  const struct { const void* at; size_t bytes; } parts[] = {
      {x.totals, n4}, {x.pages, 2 * n4}, {x.cursor, 24}, {x.table, n4 * (size_t)x.table_width},
      {x.queue, (size_t)x.queue_size * 4}, {x.totals_out, n4}, {x.pages_out, 2 * n4}, {x.evicted, n4},
      {x.cursor_out, 24}, {x.weights, (size_t)c.pages * c.page_size * c.heads * 4}, {x.workspace, evict_bytes(x)}};
  constexpr int kParts = sizeof(parts) / sizeof(parts[0]);
  for (int i = kRead; i < kParts; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(parts[i].at, parts[i].bytes, parts[j].at, parts[j].bytes)) return LILICORR_ERR_INVALID_ARG;
  const size_t scales = cache4_scales(span);
  for (const auto& p : parts)  // (keys and values may lie side by side in one buffer)
    if (overlap(c.k, span, p.at, p.bytes) || overlap(c.v, span, p.at, p.bytes) ||
        overlap(c.k_scales, scales, p.at, p.bytes) || overlap(c.v_scales, scales, p.at, p.bytes))
      return LILICORR_ERR_INVALID_ARG;
  EvictArgs a = {};
  a.k = (unsigned char*)c.k; a.v = (unsigned char*)c.v;
  a.ks = (unsigned char*)c.k_scales; a.vs = (unsigned char*)c.v_scales;
  a.weights = x.weights;
  a.table = x.table; a.totals = x.totals; a.pages = x.pages; a.queue = x.queue; a.cursor = x.cursor;
  a.totals_out = x.totals_out; a.pages_out = x.pages_out; a.evicted = x.evicted; a.cursor_out = x.cursor_out;
  a.list = (int32_t*)x.workspace;
  a.page_stride = c.page_stride; a.token_stride = c.token_stride; a.head_stride = c.head_stride;
  a.N = (int)x.N; a.M = (int)x.table_width; a.P = c.page_size; a.C = (int)x.queue_size;
  a.heads = c.heads; a.d = c.d; a.n_pages = (int)c.pages;
  divide_by(c.page_size, a.page_mul, a.page_shift);
  const int64_t held = x.table_width * c.page_size;
  a.max_length = (int)(x.max_length < held ? x.max_length : held);
  a.budget = (int)x.budget;
  a.limit = (int)(x.limit < kMostTokens ? x.limit : kMostTokens);
  a.sinks = (int)x.sinks; a.recent = (int)x.recent;
  const int64_t groups = x.N * c.heads;
  const dim3 select((unsigned)(groups + x.N));
  auto choose = [&](auto kernel) { hipLaunchKernelGGL(kernel, select, dim3(kSelectThreads), 0, stream, a); };
  // with 16 weights a thread a compute unit has two workgroups (64 requests of up to 16000 tokens: 27 us against 45)
  if (c.page_size % 4) choose(evict_select_kernel<1, 16>);
  else if (a.max_length <= 16 * kSelectThreads) choose(evict_select_kernel<4, 16>);
  else choose(evict_select_kernel<4, 32>);
  if (a.max_length > x.limit) {
    // Keys and values each to a workgroup where requests and heads are many (64 requests of 8 heads: the call 86 us, 108 with
    // both in one, 132 with two more), and each column to one where they are few (24 us to 17 for one request's move)
    const bool many = groups >= 128;
    a.wides = many ? 2 : 2 * (c.d / kBlock4);
    a.narrows = many ? 1 : 3;
    a.words = c.d % 128 == 0 && (c.page_stride | c.token_stride | c.head_stride) % 64 == 0;
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(groups * (a.wides + a.narrows))), dim3(kMoveThreads), 0, stream, a);
  }
  return launch_status();
}
