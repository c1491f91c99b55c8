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
constexpr int kKeys = 32;  // weights that a thread keeps
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
  int parts;  // workgroups that share a request and head's columns: 1, or one for each
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

// sum of v over the threads of the workgroup; every thread gets it
__device__ __forceinline__ int group_sum(int v, int* s) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, kWave);
  __syncthreads();
  if (lane_id() == 0) s[threadIdx.x / kWave] = v;
  __syncthreads();
  int all = 0;
  for (int w = 0; w < kSelectWaves; ++w) all += s[w];
  return all;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ int s_bins[kBins];
  __shared__ int s_wave[2][kSelectWaves];
  __shared__ int s_count[2][kKeys][kSelectWaves];
  __shared__ int s_found[2];
  const int tid = threadIdx.x, lane = lane_id(), wave = (int)uniform32(tid / kWave);
  const int n = (int)blockIdx.x / a.heads, head = (int)blockIdx.x % a.heads;
  const EvictRow row = evict_row(a, n);

  if (head == 0) {  // the request's numbers, and its pages to the queue
    int before = 0, all = 0;
    for (int i = tid; i < a.N; i += kSelectThreads) {
      const EvictRow r = evict_row(a, i);
      all += r.end - r.left;
      if (i < n) before += r.end - r.left;
    }
    before = group_sum(before, s_wave[0]);
    const int64_t tail = a.cursor[1];
    if (n == 0) {
      all = group_sum(all, s_wave[0]);
      if (tid == 0) {
        a.cursor_out[0] = a.cursor[0];
        a.cursor_out[1] = tail + all;
        a.cursor_out[2] = a.cursor[2];
      }
    }
    if (tid == 0) {
      const int after = row.cut ? a.budget : row.length;
      a.totals_out[n] = after;
      a.evicted[n] = row.length - after;
      a.pages_out[2 * n] = row.left;
      a.pages_out[2 * n + 1] = a.pages[2 * n + 1];
    }
    for (int i = tid; i < row.end - row.left; i += kSelectThreads) {
      const int64_t at = (tail + before + i) % a.C;
      a.queue[at < 0 ? at + a.C : at] = a.table[(int64_t)n * a.M + row.left + i];
    }
  }
  if (!row.cut) return;

  const int32_t* trow = a.table + (int64_t)n * a.M;
  const int first = a.sinks, last = row.length - a.recent;  // the tokens that weights decide about
  int need = a.budget - a.sinks - a.recent;
  // Tokens in stretches of kSelectThreads * kKeys. One stretch is the rule, and its keys are read once.
  constexpr int kStretch = kSelectThreads * kKeys;
  const int stretches = (row.length + kStretch - 1) / kStretch;
  // The weights' order, greater for the heavier (a token without a page comes last), and slots. Eight loads at a time
  // under way, pages and then weights: one by one they are 64 round trips (62 us for 32768 tokens).
  uint32_t key[kKeys];
  int slot[kKeys];
  auto read = [&](int j0) {
    constexpr int kAtOnce = 8;
#pragma unroll
    for (int i0 = 0; i0 < kKeys; i0 += kAtOnce) {
      if (j0 + i0 * kSelectThreads >= row.length) break;
      int page[kAtOnce], o[kAtOnce];
      float w[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int j = min(j0 + (i0 + i) * kSelectThreads + tid, row.length - 1), e = evict_entry(a, j);
        page[i] = trow[e];
        o[i] = j - e * a.P;
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const bool there = page[i] >= 0 && page[i] < a.n_pages;
        slot[i0 + i] = there ? page[i] * a.P + o[i] : -1;
        w[i] = a.weights[((int64_t)(there ? page[i] : 0) * a.heads + head) * a.P + o[i]];
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) key[i0 + i] = slot[i0 + i] < 0 ? 0 : order_bits(w[i]);
    }
  };
  if (stretches == 1) read(0);

  uint32_t prefix = 0, known = 0;  // the bits of the border that are known, and where
  constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = kShift[pass];
    const uint32_t mask = (1u << kBits[pass]) - 1;
    for (int i = tid; i < kBins; i += kSelectThreads) s_bins[i] = 0;
    __syncthreads();
    for (int s = 0; s < stretches; ++s) {
      const int j0 = s * kStretch;
      if (stretches > 1) read(j0);
#pragma unroll
      for (int i = 0; i < kKeys; ++i) {
        if (j0 + i * kSelectThreads >= row.length) break;
        const int j = j0 + i * kSelectThreads + tid;
        const bool in = j >= first && j < last && (key[i] & known) == prefix;
        const uint32_t bin = key[i] >> shift & mask;
        // one addition for a wave whose keys share a bin (keys that no query has met all have 0)
        const uint64_t on = __ballot(in);
        if (!on) continue;
        const uint32_t b0 = readlane32(bin, __builtin_ctzll(on));
        if (__ballot(in && bin == b0) == on) {
          if (lane == 0) atomicAdd(&s_bins[b0], (int)__popcll(on));
        } else if (in) {
          atomicAdd(&s_bins[bin], 1);
        }
      }
    }
    __syncthreads();
    // the bin, from the top, in which the need-th key lies: each thread has the bins 2 x and 2 x + 1 from the top
    const int hi = s_bins[kBins - 1 - 2 * tid], lo = s_bins[kBins - 2 - 2 * tid];
    int sum = hi + lo;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
      const int o = __shfl_up(sum, m, kWave);
      if (lane >= m) sum += o;
    }
    if (lane == kWave - 1) s_wave[1][wave] = sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) sum += s_wave[1][w];
    const int above = sum - hi - lo;  // keys in the bins above this thread's
    if (above < need && need <= sum) {
      const bool upper = above + hi >= need;
      s_found[0] = upper ? kBins - 1 - 2 * tid : kBins - 2 - 2 * tid;
      s_found[1] = upper ? above : above + hi;
    }
    if (tid == 0 && need <= 0) {
      s_found[0] = kBins - 1;
      s_found[1] = 0;
    }
    __syncthreads();
    prefix |= ((uint32_t)s_found[0] & mask) << shift;
    known |= mask << shift;
    need -= s_found[1];  // of the keys that share the known bits
    __syncthreads();
  }
  // need <= 0 from the start: the border lies above every key
  const bool none = a.budget - a.sinks - a.recent <= 0;

  int base_more = 0, base_equal = 0;
  int32_t* list = a.list + ((int64_t)n * a.heads + head) * a.budget;
  for (int s = 0; s < stretches; ++s) {
    const int j0 = s * kStretch;
    if (stretches > 1) read(j0);
    auto kind = [&](int i, bool& more, bool& equal) {
      const int j = j0 + i * kSelectThreads + tid;
      const bool mid = j >= first && j < last;
      more = j < row.length && (!mid || (!none && key[i] > prefix));
      equal = mid && !none && key[i] == prefix;
    };
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      bool more = false, equal = false;
      if (j0 + i * kSelectThreads < row.length) kind(i, more, equal);
      const uint64_t bm = __ballot(more), be = __ballot(equal);
      if (lane == 0) {
        s_count[0][i][wave] = (int)__popcll(bm);
        s_count[1][i][wave] = (int)__popcll(be);
      }
    }
    __syncthreads();
    if (wave < 2) {  // counts before each of the kKeys * kSelectWaves stretches of 64
      int* c = &s_count[wave][0][0];
      int carry = 0;
      for (int x = 0; x < kKeys * kSelectWaves; x += kWave) {
        const int v = c[x + lane];
        int sum = v;
#pragma unroll
        for (int m = 1; m < kWave; m <<= 1) {
          const int o = __shfl_up(sum, m, kWave);
          if (lane >= m) sum += o;
        }
        c[x + lane] = carry + sum - v;
        carry += __shfl(sum, kWave - 1, kWave);
      }
      if (lane == 0) s_found[wave] = carry;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      if (j0 + i * kSelectThreads >= row.length) break;
      bool more, equal;
      kind(i, more, equal);
      const uint64_t below = (1ull << lane) - 1;
      const int m0 = base_more + s_count[0][i][wave] + (int)__popcll(__ballot(more) & below);
      const int e0 = base_equal + s_count[1][i][wave] + (int)__popcll(__ballot(equal) & below);
      if (more || (equal && e0 < need)) list[m0 + min(e0, need)] = slot[i];
    }
    base_more += s_found[0];
    base_equal += s_found[1];
    __syncthreads();
  }
}

// A row of a head is columns of 16 bytes, d / 32 of the key and d / 32 of the value, and three narrow ones: the keys' scales,
// the values' scales and the weight. One workgroup moves all of a request and head, or each column has its own. A thread
// holds kHold columns of a stretch and kNarrow narrow ones. All loads of a kind are under way together.
constexpr int kHold = 8, kNarrow = 4;
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a) {
  const int tid = threadIdx.x;
  const int part = (int)blockIdx.x % a.parts, nh = (int)blockIdx.x / a.parts;
  const int n = nh / a.heads, head = nh % a.heads;
  if (!evict_row(a, n).cut) return;
  const int wide = a.d / kBlock4;  // 16-byte columns of a key; also scale bytes
  const bool alone = a.parts == 1;
  const int c0 = alone ? 0 : part, cs = alone ? 2 * wide : part < 2 * wide ? 1 : 0;  // wide columns, and narrow ones
  const int k0 = alone ? 0 : part - 2 * wide, kinds = alone ? 3 : part < 2 * wide ? 0 : 1;
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
  // tokens of a stretch
  const int rows = min(cs ? kMoveThreads * kHold / cs : 1 << 30, kinds ? kMoveThreads * kNarrow / kinds : 1 << 30);
  for (int i0 = 0; i0 < a.budget; i0 += rows) {
    const int here = min(rows, a.budget - i0), items = here * cs, narrows = here * kinds;
    int from[kHold], to[kHold], nfrom[kNarrow], nto[kNarrow];  // slots; `to` is -1 where there is nothing to do
    auto places = [&](int item, int count, int per, int& src, int& dst) {
      const int i = i0 + min(item, count - 1) / per, e = evict_entry(a, i);
      src = list[i];
      dst = trow[e];  // its page
    };
    auto settle = [&](int item, int count, int per, int& src, int& dst) {
      const int i = i0 + min(item, count - 1) / per, e = evict_entry(a, i);
      const int slot = dst >= 0 && dst < a.n_pages ? dst * a.P + (i - e * a.P) : -1;
      dst = item >= count || src < 0 || src == slot ? -1 : slot;
      src = max(src, 0);
    };
    if (cs) {
#pragma unroll
      for (int x = 0; x < kHold; ++x) places(x * kMoveThreads + tid, items, cs, from[x], to[x]);
    }
    if (kinds) {
#pragma unroll
      for (int x = 0; x < kNarrow; ++x) places(x * kMoveThreads + tid, narrows, kinds, nfrom[x], nto[x]);
    }
    u32x4_t held[kHold];
    if (cs) {
#pragma unroll
      for (int x = 0; x < kHold; ++x) {
        settle(x * kMoveThreads + tid, items, cs, from[x], to[x]);
        const int c = c0 + (x * kMoveThreads + tid) % cs;
        held[x] = *reinterpret_cast<const u32x4_t*>((c < wide ? a.k : a.v) + offset(from[x]) + (c % wide) * 16);
      }
    }
    uint32_t small[kNarrow][8];
    if (kinds) {
#pragma unroll
      for (int x = 0; x < kNarrow; ++x) {
        const int kind = k0 + (x * kMoveThreads + tid) % kinds;
        settle(x * kMoveThreads + tid, narrows, kinds, nfrom[x], nto[x]);
        if (kind < 2) {
          const unsigned char* at = (kind == 0 ? a.ks : a.vs) + offset(nfrom[x]) / 16;
#pragma unroll
          for (int b = 0; b < 8; ++b) small[x][b] = at[min(b, wide - 1)];
        } else {
          small[x][0] = __float_as_uint(*weight(nfrom[x]));
        }
      }
    }
    // everything that this stretch overwrites has been read, by every wave
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (cs) {
#pragma unroll
      for (int x = 0; x < kHold; ++x) {
        if (to[x] < 0) continue;
        const int c = c0 + (x * kMoveThreads + tid) % cs;
        *reinterpret_cast<u32x4_t*>((c < wide ? a.k : a.v) + offset(to[x]) + (c % wide) * 16) = held[x];
      }
    }
    if (kinds) {
#pragma unroll
      for (int x = 0; x < kNarrow; ++x) {
        if (nto[x] < 0) continue;
        const int kind = k0 + (x * kMoveThreads + tid) % kinds;
        if (kind < 2) {
          unsigned char* at = (kind == 0 ? a.ks : a.vs) + offset(nto[x]) / 16;
#pragma unroll
          for (int b = 0; b < 8; ++b)
            if (b < wide) at[b] = (unsigned char)small[x][b];
        } else {
          *weight(nto[x]) = __uint_as_float(small[x][0]);
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
  if (!aligned16(c.k) || !aligned16(c.v) || !aligned4(c.k_scales) || !aligned4(c.v_scales) || !aligned16(x.weights) || !aligned16(x.workspace) || !aligned4(x.table) ||
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
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)groups), dim3(kSelectThreads), 0, stream, a);
  if (a.max_length > x.limit) {
    // few requests and heads: a workgroup for each column (one conversation with 8 heads 24 us, 57 with four columns each)
    a.parts = groups >= 256 ? 1 : 2 * (c.d / kBlock4) + 3;
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(groups * a.parts)), dim3(kMoveThreads), 0, stream, a);
  }
  return launch_status();
}
