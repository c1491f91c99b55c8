// lilicorr_window_attention and lilicorr_prefix_attention: checks, tiles and chunks, launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "attention.hpp"
#include "common.hpp"
#include "lilicorr.h"
#include "paged.hpp"

namespace lilicorr {
namespace {

constexpr size_t kLeastBytes = 256;  // of a workspace
// The longest sequences have so many tokens: lengths, windows and sinks past it say "without end"
constexpr int64_t kMost = (int64_t)1 << 30;
int64_t bounded(int64_t n) { return n < kMost ? n : kMost; }

// One pass over keys: which tile height, how many tiles and chunks
struct Pass {
  int tiles, chunk, chunks;
  bool spread;
};

struct Plan {
  bool shared;
  int BM;
  Pass first, tail;  // the shared keys' pass and the requests' own
  int slots;
  int64_t rows;
  size_t bytes;  // of the workspace
};

// The least height that holds a request's rows: fewer rows than a tile has are computed all the same. Single tokens
// in 32-row tiles share the keys among the four waves (two waves a tile: 822 us and more against 762 for 256 tokens);
// the 64 rows of a block of 16 with four query heads a key head as 2 x 2 waves take 196 us, as 2 x 4 202; 256-row
// tiles of eight waves 650 us against 629 with 128 for a prefill of 8192 tokens (both on an earlier version).
int tile_rows(int64_t rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

// Calls `use` with the kernel of a width and tile height: waves of rows x waves of keys, 32-key blocks a wave and
// stage, stages of the ring. Few rows: four waves share the keys and each keeps its own ring; more: barriers,
// 64 keys a stage, and a ring of two so that two workgroups share a compute unit (a ring of four with one: 302
// against 188 us for 64 blocks of 16 tokens behind 4096 keys).
template <typename T, bool FULL, int D, typename F>
auto with_rows(int BM, const F& use) {
  if constexpr (D <= 64) {
    if (BM == 32) return use(AttnConfig<T, FULL, D, 1, 4, 1, 4>());
    if (BM == 64) return use(AttnConfig<T, FULL, D, 2, 2, 1, 4>());
    return use(AttnConfig<T, FULL, D, 4, 1, 2, 2>());
  } else if constexpr (D <= 128) {
    if (BM == 32) return use(AttnConfig<T, FULL, D, 1, 4, 1, 2>());
    if (BM == 64) return use(AttnConfig<T, FULL, D, 2, 2, 1, 2>());
    return use(AttnConfig<T, FULL, D, 4, 1, 2, 2>());
  } else {
    if (BM == 32) return use(AttnConfig<T, FULL, D, 1, 2, 1, 2>());
    if (BM == 64) return use(AttnConfig<T, FULL, D, 2, 2, 1, 2>());
    return use(AttnConfig<T, FULL, D, 4, 1, 1, 2>());
  }
}

// Heads between the powers of two lie in LDS rows of the next one, and elements past their width are copied from
// zeros. Heads of 65 to 96 leave out the empty quarter of the products (a ragged prefill with heads of 80: 175 us
// against 196).
template <typename T, typename F>
auto with_kernel(int d, int BM, const F& use) {
  if (d == 64) return with_rows<T, true, 64>(BM, use);
  if (d < 64) return with_rows<T, false, 64>(BM, use);
  if (d <= 96) return with_rows<T, false, 96>(BM, use);
  if (d == 128) return with_rows<T, true, 128>(BM, use);
  if (d < 128) return with_rows<T, false, 128>(BM, use);
  if (d == 256) return with_rows<T, true, 256>(BM, use);
  return with_rows<T, false, 256>(BM, use);
}

// Keys of a kernel's stage, and its workgroups that run at once on 256 compute units
struct Fit {
  int stage, slots;
};
Fit kernel_fit(int d, int BM) {
  return with_kernel<Bf16>(d, BM, [](auto c) { return Fit{decltype(c)::SK, 256 * decltype(c)::kAtOnce}; });
}

// A pass's row tiles (of all heads) and the stages of keys that a tile sees at most
struct Work {
  int64_t items, stages;
};

// How many stages a chunk has, for both passes: the least of an estimate in stages' times. A workgroup
// begins and ends for about three (page numbers, queries, first copies; output). As long as all run at
// once the longest one counts, else also the work of all over the workgroups that run at once, and half
// of a last one. Split keys add the join's launch (two and a half) and fp32 partial outputs that are written
// and read again, at 5 TB/s against 1.5 us a stage. The times in stages were fitted to heads of 128, where the
// chosen length is the best one for one token (13.5 us) and 32 tokens behind a prefix (30.4), and within 3% for 64
// blocks behind one (357 against 347). Narrower heads have shorter stages: 4% for a ragged batch with heads of 64
// (23.1 against 22.1) and 10% for a prefix with heads of 80 (21.2 against 19.2).
int64_t chunk_stages(const Work& shared, const Work& own, int slots, int64_t out_elements) {
  const int64_t longest = shared.stages > own.stages ? shared.stages : own.stages;
  int64_t best = longest, last = 0;
  double least = 0;
  for (int64_t k = 1; k <= 64; ++k) {
    const int64_t s = (longest + k - 1) / k;
    if (s == last) continue;
    last = s;
    const int64_t cs = (shared.stages + s - 1) / s, co = (own.stages + s - 1) / s;
    const double groups = (double)shared.items * cs + (double)own.items * co;
    double t = s + 3;
    if (groups > slots) {
      const double all =
          ((double)shared.items * shared.stages + (double)own.items * own.stages + 3 * groups) / slots;
      t = (all > t ? all : t) + 0.5 * (s < own.stages ? s : own.stages) + 3;
    }
    if (cs + co > 1) t += 2.5 + (double)(cs + co) * out_elements * 8 / 5e6 / 1.5;
    if (k == 1 || t < least) {
      least = t;
      best = s;
    }
    if (s == 1) break;
  }
  return best;
}

Pass make_pass(int64_t tiles, int64_t stages, int64_t chunk, int stage, bool spread) {
  const int64_t chunks = (stages + chunk - 1) / chunk;
  return {(int)tiles, (int)(chunk * stage), (int)(chunks < 1 ? 1 : chunks), spread};
}

// the largest unit that page and token strides are whole multiples of: the kernels count offsets in it
// in 32 bits, and a head's width or more is usual
int64_t stride_unit(const lilicorr_cache& c) {
  int64_t x = c.page_stride, y = c.token_stride;
  while (y) {
    const int64_t r = x % y;
    x = y;
    y = r;
  }
  return x ? x < (1 << 30) ? x : 8 : 8;
}

lilicorr_status make_plan(const lilicorr_attention_args& a, bool shared, Plan& p) {
  if (const lilicorr_status s = cache_sizes(a.cache)) return s;
  if (a.tokens < 0 || a.N < 1 || a.table_width < 1 || a.heads < 1 || a.window < 0 || a.sinks < 0 ||
      a.max_tokens < 0 || a.max_length < 0 || a.q_stride < 0)
    return LILICORR_ERR_INVALID_ARG;
  if (a.heads % a.cache.heads) return LILICORR_ERR_INVALID_ARG;
  if (!(a.scale > 0.f) || !isfinite(a.scale)) return LILICORR_ERR_INVALID_ARG;
  if (a.sinks > 0 && a.window == 0) return LILICORR_ERR_INVALID_ARG;
  if (shared ? (a.shared_length < 1 || a.window != 0) : a.shared_length != 0)
    return LILICORR_ERR_INVALID_ARG;
  if (a.heads > 65535 || a.N > (1 << 20) || a.tokens > kMost / a.heads ||
      a.table_width > kMost / a.cache.page_size || a.shared_length > kMost)
    return LILICORR_ERR_UNSUPPORTED;
  if (!stride_ok(a.q_stride)) return LILICORR_ERR_ALIGNMENT;
  if ((double)a.cache.page_stride * (double)(a.cache.pages - 1) +
          (double)a.cache.token_stride * (a.cache.page_size - 1) >=
      4294967296.0 * (double)stride_unit(a.cache))
    return LILICORR_ERR_UNSUPPORTED;

  const int64_t group = a.heads / a.cache.heads;
  const int64_t max_tokens = a.max_tokens < a.tokens ? a.max_tokens : a.tokens;
  p.shared = shared;
  p.rows = a.tokens * a.heads;
  const int64_t own = max_tokens * group, all = a.tokens * group;
  // one launch has one tile height; where the shared keys are read for all rows together, theirs
  const int BM = tile_rows(shared ? all : own);
  const int64_t tiles = own <= BM ? a.N : a.tokens * group / BM + a.N;
  int64_t keys = a.table_width * a.cache.page_size;
  if (a.max_length < keys) keys = a.max_length;
  if (a.window) {
    // a tile's queries see at most this many: from the first one's window to the last one itself, or
    // to the request's last token
    const int64_t tile_tokens = BM / group + 1;
    const int64_t seen = bounded(a.window) + bounded(a.sinks) +
                         (a.causal && tile_tokens < max_tokens ? tile_tokens : max_tokens);
    if (seen < keys) keys = seen;
  }
  const int64_t shared_tiles = shared ? (all + BM - 1) / BM : 0;
  const Fit fit = kernel_fit(a.cache.d, BM);
  const auto stages = [&](int64_t k) { return k > 0 ? (k + fit.stage - 1) / fit.stage : 1; };
  const Work shared_work = {shared_tiles * a.cache.heads, shared ? stages(a.shared_length) : 0};
  const Work own_work = {tiles * a.cache.heads, stages(keys)};
  const int64_t chunk = chunk_stages(shared_work, own_work, fit.slots, p.rows * a.cache.d);
  p.BM = BM;
  // where every key is read once, runs of items keep a request's heads on one XCD (their tokens lie side
  // by side, and eight XCDs with a head each would use an eighth of every L2: 825 against 1068 us for 256
  // tokens); tiles that share keys find them in the L2 of their head's XCD (prefill 664 against 772 us;
  // these figures too are of an earlier version)
  p.tail = make_pass(tiles, own_work.stages, chunk, fit.stage, own <= BM);
  p.slots = p.tail.chunks;
  if (shared) {
    p.first = make_pass(shared_tiles, shared_work.stages, chunk, fit.stage, false);
    p.slots += p.first.chunks;
  }
  const int64_t most_items = 0x7fffffffll / a.cache.heads;
  if ((int64_t)p.tail.tiles * p.tail.chunks +
          (shared ? (int64_t)p.first.tiles * p.first.chunks : 0) > most_items)
    return LILICORR_ERR_UNSUPPORTED;
  p.bytes = kLeastBytes;
  if (p.slots > 1) p.bytes += (size_t)p.slots * p.rows * (8 + (size_t)a.cache.d * 4);
  return LILICORR_OK;
}

template <typename C>
void launch(const AttnArgs& a, hipStream_t stream) {
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(attention_kernel<C>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::kLds);
  (void)attr;
  hipLaunchKernelGGL(attention_kernel<C>, dim3((unsigned)(a.shared.items + a.own.items)),
                     dim3(C::kThreads), C::kLds, stream, a);
}

AttnPass attn_pass(const Pass& p, int kv_heads, int slot0) {
  AttnPass r = {};
  r.tiles = p.tiles;
  r.chunk = p.chunk;
  r.most = p.chunk * p.chunks;
  r.items = p.tiles * p.chunks * kv_heads;
  r.spread = p.spread;
  r.slot0 = slot0;
  return r;
}

template <typename T, int LPR>
void launch_join(const AttnArgs& a, const Plan& p, hipStream_t stream) {
  constexpr int64_t per = kJoinThreads / kWave;
  hipLaunchKernelGGL((attention_join_kernel<T, LPR>), dim3((unsigned)((p.rows + per - 1) / per)),
                     dim3(kJoinThreads), 0, stream, a.part_o, a.part_ml, p.rows, p.slots, a.d,
                     a.starts, a.N, a.tokens, a.heads, a.out);
}

template <typename T>
lilicorr_status run(const lilicorr_attention_args& x, const Plan& p, hipStream_t stream) {
  AttnArgs a = {};
  const lilicorr_cache& c = x.cache;
  a.q = (const uint16_t*)x.q; a.k = (const uint16_t*)c.k; a.v = (const uint16_t*)c.v;
  a.out = (uint16_t*)x.out;
  a.starts = x.starts; a.totals = x.totals;
  a.q_stride = x.q_stride; a.head_stride = c.head_stride;
  a.rows = p.rows;
  a.N = (int)x.N; a.pages = (int)c.pages; a.page_size = c.page_size;
  // n / P = (n * mul) >> shift for n < 2^31, mul = floor(2^shift / P) + 1 below 2^32
  int bits = 0;
  while ((1 << bits) < c.page_size) ++bits;
  a.page_shift = 31 + bits;
  a.page_mul = (uint32_t)((((uint64_t)1 << a.page_shift) / c.page_size) + 1);
  a.tokens = (int)x.tokens; a.heads = x.heads; a.kv_heads = c.heads; a.group = x.heads / c.heads;
  a.d = c.d;
  const int64_t unit = stride_unit(c);
  a.page_units = (uint32_t)(c.page_stride / unit);
  a.token_units = (uint32_t)(c.token_stride / unit);
  a.unit_bytes = (uint32_t)(unit * 2);
  a.scale2 = x.scale * 1.4426950408889634f;
  a.own = attn_pass(p.tail, c.heads, p.shared ? p.first.chunks : 0);
  a.own.table = x.table;
  a.own.table_width = (int)x.table_width;
  a.own.max_tokens = (int)(x.max_tokens < x.tokens ? x.max_tokens : x.tokens);
  a.own.max_length = (int)bounded(x.max_length);
  a.own.window = (int)bounded(x.window);
  a.own.sinks = (int)bounded(x.sinks);
  a.own.causal = x.causal != 0;
  if (p.shared) {
    a.shared = attn_pass(p.first, c.heads, 0);
    a.shared.table = x.shared_table;
    a.shared.table_width = (int)((x.shared_length + c.page_size - 1) / c.page_size);
    a.shared.shared = a.shared.max_length = (int)x.shared_length;
    a.shared.max_tokens = a.tokens;
  }
  unsigned char* w = (unsigned char*)x.workspace;
  a.split = p.slots > 1;
  a.part_o = (float*)w;
  a.part_ml = (f32x2_t*)(w + (size_t)p.slots * p.rows * c.d * 4);
  with_kernel<T>(a.d, p.BM, [&](auto c) { launch<decltype(c)>(a, stream); });
  if (a.split) {
    if (c.d <= 64) launch_join<T, 16>(a, p, stream);
    else if (c.d <= 128) launch_join<T, 32>(a, p, stream);
    else launch_join<T, 64>(a, p, stream);
  }
  return launch_status();
}

size_t workspace_bytes(const lilicorr_attention_args* a, bool shared) {
  Plan p;
  return a && make_plan(*a, shared, p) == LILICORR_OK ? p.bytes : 0;
}

lilicorr_status attention(const lilicorr_attention_args* a, bool shared, hipStream_t stream) {
  if (!a) return LILICORR_ERR_INVALID_ARG;
  Plan p;
  if (const lilicorr_status s = make_plan(*a, shared, p)) return s;
  if (a->tokens == 0) return LILICORR_OK;
  if (!a->q || !a->out || !a->cache.k || !a->cache.v || !a->table || !a->starts || !a->totals)
    return LILICORR_ERR_INVALID_ARG;
  if (shared != (a->shared_table != nullptr) || a->q == a->out) return LILICORR_ERR_INVALID_ARG;
  if (!aligned16(a->q) || !aligned16(a->out) || !aligned16(a->cache.k) || !aligned16(a->cache.v) ||
      !aligned16(a->workspace) || !aligned4(a->table) || !aligned4(a->starts) ||
      !aligned4(a->totals) || !aligned4(a->shared_table))
    return LILICORR_ERR_ALIGNMENT;
  if (!a->workspace || a->workspace_bytes < p.bytes) return LILICORR_ERR_WORKSPACE;
  if (a->max_tokens == 0) return LILICORR_OK;
  const size_t row = (size_t)a->heads * a->cache.d * 2;
  if (rows_overlap(a->q, a->q_stride * 2, row, a->tokens, a->out, row * (size_t)a->tokens))
    return LILICORR_ERR_INVALID_ARG;
  return a->cache.dtype == LILICORR_BF16 ? run<Bf16>(*a, p, stream) : run<F16>(*a, p, stream);
}

}  // namespace
}  // namespace lilicorr

extern "C" size_t lilicorr_window_attention_workspace_bytes(const lilicorr_attention_args* args) {
  return lilicorr::workspace_bytes(args, false);
}

extern "C" size_t lilicorr_prefix_attention_workspace_bytes(const lilicorr_attention_args* args) {
  return lilicorr::workspace_bytes(args, true);
}

extern "C" lilicorr_status lilicorr_window_attention(const lilicorr_attention_args* args,
                                                     hipStream_t stream) {
  return lilicorr::attention(args, false, stream);
}

extern "C" lilicorr_status lilicorr_prefix_attention(const lilicorr_attention_args* args,
                                                     hipStream_t stream) {
  return lilicorr::attention(args, true, stream);
}
