// lilicorr_window_attention4 and lilicorr_key_weights: checks, tiles and chunks, launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "attention4.hpp"
#include "cache4.hpp"
#include "common.hpp"
#include "lilicorr.h"
#include "paged.hpp"

namespace lilicorr {
namespace {

// Many keys in all (cache heads times tiles of 32 keys): a workgroup's waves share key heads rather than keys, and copies of
// whole lines. 256 requests of one token, a million such tiles: 445 us against 548 with shared keys, their weights 270
// against 362; 64 blocks 307 against 318. With fewer the workgroups do not fill the chip: a call of some ten thousand 139 us
// with shared keys, 185 with shared heads.
constexpr int64_t kManyTiles = 65536;
constexpr size_t kLeastBytes4 = 256;  // of a workspace
// The longest sequences have so many tokens: lengths, windows and sinks past it say "without end"
constexpr int64_t kMost4 = (int64_t)1 << 30;
int64_t bounded4(int64_t n) { return n < kMost4 ? n : kMost4; }

struct Plan4 {
  int BM, tiles, chunk, chunks;  // rows of a tile; row tiles; 32-key tiles of a chunk; chunks
  int heads;  // key heads that a workgroup's waves share
  bool ring, spread;
  int64_t rows;
  size_t bytes;  // of the workspace
};

// Whether a wave has registers for two blocks of 16 rows: tiles by way of registers leave wider heads none (2048 tokens behind
// 2048, heads of 96: 606 us with two blocks, whose registers spill, 285 with one).
constexpr bool two_blocks4(int d, bool ring) { return d <= (ring ? 128 : 64); }

// Calls `use` with the kernel of a width, a tile height and what the workgroup's waves share: key heads (`heads`: a token's
// heads lie side by side, and so share cache lines) or keys.
template <typename T, int D, bool RING, typename F>
void with_rows4(int BM, bool heads, const F& use) {
  if constexpr (RING) {
    if (heads) {
      if (BM == 16) return use(Attn4Config<T, D, 1, 4, 1, 1, RING>());
      if constexpr (D <= 128) {
        if (BM == 32) return use(Attn4Config<T, D, 2, 4, 1, 1, RING>());
        if (BM == 64) return use(Attn4Config<T, D, 2, 2, 2, 1, RING>());
      } else {
        if (BM == 32) return use(Attn4Config<T, D, 1, 2, 2, 1, RING>());
      }
    }
  }
  if (BM == 16) return use(Attn4Config<T, D, 1, 1, 1, 4, RING>());
  if constexpr (!two_blocks4(D, RING)) {
    if (BM == 32) return use(Attn4Config<T, D, 1, 1, 2, 2, RING>());
    return use(Attn4Config<T, D, 1, 1, 4, 1, RING>());
  } else {
    if (BM == 32) return use(Attn4Config<T, D, 2, 1, 1, 4, RING>());
    if (BM == 64) return use(Attn4Config<T, D, 2, 1, 2, 2, RING>());
    return use(Attn4Config<T, D, 2, 1, 4, 1, RING>());
  }
}
int tile_rows4(int64_t rows, bool two) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 || !two ? 64 : 128; }

template <typename T, typename F>
void with_kernel4(int d, bool ring, int BM, bool heads, const F& use) {
  auto width = [&](auto f) {
    constexpr bool RING = decltype(f)::value;
    if (d <= 64) with_rows4<T, 64, RING>(BM, heads, use);
    else if (d <= 128) with_rows4<T, 128, RING>(BM, heads, use);
    else with_rows4<T, 256, RING>(BM, heads, use);
  };
  if (ring) width(std::true_type());
  else width(std::false_type());
}

// What both calls check: sizes, then (without a workspace's query) the strides' reach
template <typename A>
lilicorr_status sizes4(const A& a) {
  if (const lilicorr_status s = cache4_sizes(a.cache)) return s;
  if (a.dtype != LILICORR_BF16 && a.dtype != LILICORR_F16) return LILICORR_ERR_INVALID_ARG;
  if (a.tokens < 0 || a.N < 1 || a.table_width < 1 || a.heads < 1 || a.max_tokens < 0 || a.max_length < 0 ||
      a.q_stride < 0)
    return LILICORR_ERR_INVALID_ARG;
  if (a.heads % a.cache.heads) return LILICORR_ERR_INVALID_ARG;
  if (!(a.scale > 0.f) || !isfinite(a.scale)) return LILICORR_ERR_INVALID_ARG;
  if (a.heads > 65535 || a.N > (1 << 20) || a.tokens > kMost4 / a.heads || a.table_width > kMost4 / a.cache.page_size)
    return LILICORR_ERR_UNSUPPORTED;
  if (!stride_ok(a.q_stride)) return LILICORR_ERR_ALIGNMENT;
  // 16 keys of a page are reached with 32-bit offsets
  if (a.cache.token_stride >= (int64_t)1 << 27) return LILICORR_ERR_UNSUPPORTED;
  return LILICORR_OK;
}

// whether tiles can go by way of LDS: 16 keys in a page, whole rows of 64, 128 or 256, scales where the copies' 4 bytes (2
// with heads of 64) want them
bool ring_fits(const lilicorr_cache4& c) {
  if (c.page_size % 16 || (c.d != 64 && c.d != 128 && c.d != 256)) return false;
  const int64_t unit = c.d == 64 ? 2 : 4;
  auto even = [&](int64_t s) { return s % (16 * unit) == 0; };
  return even(c.page_stride) && even(c.token_stride) && even(c.head_stride);
}

// whether a token's heads lie side by side, with scales where 4-byte copies want them
bool heads_together(const lilicorr_cache4& c) {
  return c.head_stride == c.d / 2 && c.page_stride % 64 == 0 && c.token_stride % 64 == 0;
}

lilicorr_status make_plan4(const lilicorr_attention4_args& a, Plan4& p) {
  if (const lilicorr_status s = sizes4(a)) return s;
  if (a.window < 0 || a.sinks < 0 || (a.sinks > 0 && a.window == 0)) return LILICORR_ERR_INVALID_ARG;
  const int64_t group = a.heads / a.cache.heads;
  const int64_t max_tokens = a.max_tokens < a.tokens ? a.max_tokens : a.tokens;
  p.rows = a.tokens * a.heads;
  const int64_t own = max_tokens * group;
  p.ring = ring_fits(a.cache);
  const bool two = two_blocks4(a.cache.d, p.ring);
  p.BM = tile_rows4(own, two);
  const int64_t tiles = own <= p.BM ? a.N : a.tokens * group / p.BM + a.N;
  int64_t keys = a.table_width * a.cache.page_size;
  if (a.max_length < keys) keys = a.max_length;
  int64_t most = (keys + 31) / 32;
  if (a.window) {
    // a tile's queries see at most this many: from the first one's window to the last one itself, or to the request's
    // last token; each of the two runs may begin and end inside a tile of 32
    const int64_t tile_tokens = p.BM / group + 1;
    const int64_t seen = bounded4(a.window) + (a.causal && tile_tokens < max_tokens ? tile_tokens : max_tokens);
    const int64_t tiles32 = (seen + 31) / 32 + 1 + (bounded4(a.sinks) + 31) / 32;
    if (tiles32 < most) most = tiles32;
  }
  if (most < 1) most = 1;
  p.spread = own <= p.BM;
  // key heads over the waves, where that still leaves every compute unit work
  const int wide = p.BM == 16 || (p.BM == 32 && two) ? 4 : p.BM == 32 || (p.BM == 64 && two) ? 2 : 1;
  const int64_t pairs = tiles * a.cache.heads;
  const bool together = p.ring && wide > 1 && a.cache.heads % wide == 0 && heads_together(a.cache);
  p.heads = together && pairs * most >= kManyTiles ? wide : 1;
  const int64_t items = pairs / p.heads;
  const int wk = p.heads > 1 ? 1 : wide;  // (waves that share keys are as many)
  int64_t chunk, chunks;
  if (p.heads > 1) {
    // A workgroup's share of the time should be small, the partial results' too, which with more rows weigh more: 256 tokens
    // 446 us with 64 tiles a chunk, 449 with 48, 480 with 84; 64 blocks 310 with 84, 319 with 64, 346 with 128
    chunk = (most * items + 1535) / 1536;
    const int64_t cap = p.BM <= 16 ? 64 : 84;
    chunk = chunk < 8 ? 8 : chunk > cap ? cap : chunk;
    chunks = (most + chunk - 1) / chunk;
  } else {
    // workgroups that all run at once; more of them only make more to join (37 requests of up to 33 tokens behind a window 34.7
    // us, 36.2 with 768, 42.2 with 384; one token 18.4 with 512 and 768, 19.6 with 384)
    const int64_t want = 512;
    chunks = items >= want ? 1 : want / items;
    const int64_t fit = (most + 2 * wk - 1) / (2 * wk);
    if (chunks > fit) chunks = fit;
  }
  if (chunks > 64) chunks = 64;
  chunk = (most + chunks - 1) / chunks;
  chunks = (most + chunk - 1) / chunk;
  if (tiles * chunks > 0x7fffffffll / a.cache.heads) return LILICORR_ERR_UNSUPPORTED;
  p.tiles = (int)tiles;
  p.chunk = (int)chunk;
  p.chunks = (int)chunks;
  p.bytes = kLeastBytes4;
  if (chunks > 1) p.bytes += (size_t)chunks * p.rows * (16 + (size_t)a.cache.d * 4);
  return LILICORR_OK;
}

template <typename A>
Attn4Args common4(const A& x) {
  Attn4Args a = {};
  const lilicorr_cache4& c = x.cache;
  a.q = (const uint16_t*)x.q;
  a.k = (const unsigned char*)c.k; a.v = (const unsigned char*)c.v;
  a.ks = (const unsigned char*)c.k_scales; a.vs = (const unsigned char*)c.v_scales;
  a.table = x.table; a.starts = x.starts; a.totals = x.totals;
  a.q_stride = x.q_stride;
  a.head_stride = c.head_stride; a.page_stride = c.page_stride; a.token_stride = c.token_stride;
  a.rows = x.tokens * x.heads;
  a.N = (int)x.N; a.pages = (int)c.pages; a.page_size = (uint32_t)c.page_size; a.table_width = (int)x.table_width;
  divide_by(c.page_size, a.page_mul, a.page_shift);
  divide_by(x.heads / c.heads, a.group_mul, a.group_shift);
  a.tokens = (int)x.tokens; a.heads = x.heads; a.kv_heads = c.heads; a.group = x.heads / c.heads; a.d = c.d;
  a.max_tokens = (int)(x.max_tokens < x.tokens ? x.max_tokens : x.tokens);
  a.max_length = (int)bounded4(x.max_length);
  a.causal = x.causal != 0;
  a.scale2 = x.scale * 1.4426950408889634f;
  return a;
}

// LDS of a workgroup's tiles
template <typename C, bool VALUES>
constexpr uint32_t ring_bytes() {
  if constexpr (!C::RING) return 0;
  else if constexpr (C::kShared) return Shared4<C, VALUES>::kBytes;
  else return C::kWaves * Ring4<C, VALUES>::kBytes;
}

template <typename C>
void launch4(const Attn4Args& a, hipStream_t stream) {
  constexpr uint32_t kRing = ring_bytes<C, true>();
  constexpr uint32_t kLds = kRing > C::kJoin ? kRing : C::kJoin;
  static_assert(kLds <= 160 * 1024, "a workgroup fits");
  if constexpr (kLds > 65536) {
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(attention4_kernel<C>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    (void)attr;
  }
  hipLaunchKernelGGL(attention4_kernel<C>, dim3((unsigned)a.items), dim3(C::kThreads), kLds, stream, a);
}

template <typename T, int LPR>
void launch_join4(const Attn4Args& a, int slots, hipStream_t stream) {
  constexpr int64_t per = kJoin4Threads / kWave;
  const dim3 grid((unsigned)((a.rows + per - 1) / per));
  if (a.rows <= 1024)
    hipLaunchKernelGGL((attention4_join_kernel<T, LPR, true>), grid, dim3(kJoin4Threads), 0, stream, a, slots);
  else
    hipLaunchKernelGGL((attention4_join_kernel<T, LPR, false>), grid, dim3(kJoin4Threads), 0, stream, a, slots);
}

template <typename T>
lilicorr_status run4(const lilicorr_attention4_args& x, const Plan4& p, hipStream_t stream) {
  Attn4Args a = common4(x);
  a.out = (uint16_t*)x.out;
  a.lse = x.lse;
  a.window = (int)bounded4(x.window);
  a.sinks = (int)bounded4(x.sinks);
  a.tiles = p.tiles; a.chunk = p.chunk; a.most = p.chunk * p.chunks;
  a.items = p.tiles * p.chunks * (a.kv_heads / p.heads);
  a.spread = p.spread;
  a.split = p.chunks > 1;
  a.part_o = (float*)x.workspace;
  a.part_ml = (f32x4_t*)((unsigned char*)x.workspace + (size_t)p.chunks * p.rows * a.d * 4);
  with_kernel4<T>(a.d, p.ring, p.BM, p.heads > 1, [&](auto c) { launch4<decltype(c)>(a, stream); });
  if (a.split) {
    if (a.d <= 64) launch_join4<T, 16>(a, p.chunks, stream);
    else if (a.d <= 128) launch_join4<T, 32>(a, p.chunks, stream);
    else launch_join4<T, 64>(a, p.chunks, stream);
  }
  return launch_status();
}

template <typename C>
void launch_many(const Attn4Args& a, hipStream_t stream) {
  constexpr uint32_t kLds = Rows4Ring<C>::kBytes;
  if constexpr (kLds > 65536) {
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(key_weights_many_kernel<C>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    (void)attr;
  }
  hipLaunchKernelGGL(key_weights_many_kernel<C>, dim3((unsigned)((int64_t)a.tiles * a.N * a.kv_heads)),
                     dim3(C::kThreads), kLds, stream, a);
}

template <typename T, bool RING>
void launch_weights(Attn4Args a, int d, bool heads_together, hipStream_t stream) {
  const bool few = (int64_t)a.max_tokens * a.group <= 16;
  int64_t keys = (int64_t)a.table_width * a.page_size;
  if (a.max_length < keys) keys = a.max_length;
  if (keys < 1) return;
  auto run = [&](auto width) {
    constexpr int D = decltype(width)::value;
    if (few) {
      const int64_t most = (keys + 31) / 32;
      auto launch = [&](auto c, int64_t items, int64_t chunk) {
        typedef decltype(c) C;
        a.tiles = a.N;
        a.chunk = (int)chunk;
        a.items = (int)(items * ((most + chunk - 1) / chunk));
        a.spread = 1;
        constexpr uint32_t kLds = ring_bytes<C, false>();
        static_assert(kLds <= 65536, "no attribute is asked for");
        hipLaunchKernelGGL(key_weights_few_kernel<C>, dim3((unsigned)a.items), dim3(C::kThreads), kLds, stream, a);
      };
      const int64_t pairs = (int64_t)a.N * a.kv_heads;
      if constexpr (RING) {
        // (nothing is joined, so chunks are short: 256 tokens 270 us with 16 tiles, 272 with 24, 275 with 32)
        if (a.kv_heads % 4 == 0 && heads_together && pairs * most >= kManyTiles)
          return launch(Attn4Config<T, D, 1, 4, 1, 1, RING>(), pairs / 4, 16);
      }
      const int64_t want = 1024, fit = (most + 7) / 8;
      int64_t chunks = pairs >= want ? 1 : want / pairs;
      if (chunks > fit) chunks = fit;
      launch(Attn4Config<T, D, 1, 1, 1, 4, RING>(), pairs, (most + chunks - 1) / chunks);
    } else {
      const int64_t groups = (keys + 63) / 64;
      // enough key groups: neighbouring ones share the rows that they read; else the waves share the rows
      if (groups * a.N * a.kv_heads >= 2048) {
        typedef Attn4Config<T, D, 1, 1, 1, 4, false> C;
        a.tiles = (int)((groups + 3) / 4);
        launch_many<C>(a, stream);
      } else {
        typedef Attn4Config<T, D, 1, 1, 4, 1, false> C;
        a.tiles = (int)groups;
        launch_many<C>(a, stream);
      }
    }
  };
  if (d <= 64) run(std::integral_constant<int, 64>());
  else if (d <= 128) run(std::integral_constant<int, 128>());
  else run(std::integral_constant<int, 256>());
}

template <typename T>
lilicorr_status run_weights(const lilicorr_key_weights_args& x, hipStream_t stream) {
  Attn4Args a = common4(x);
  a.lse_in = x.lse;
  a.weights = x.weights;
  a.decay = x.decay;
  if (ring_fits(x.cache)) launch_weights<T, true>(a, a.d, heads_together(x.cache), stream);
  else launch_weights<T, false>(a, a.d, false, stream);
  return launch_status();
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" size_t lilicorr_window_attention4_workspace_bytes(const lilicorr_attention4_args* args) {
  Plan4 p;
  return args && make_plan4(*args, p) == LILICORR_OK ? p.bytes : 0;
}

extern "C" lilicorr_status lilicorr_window_attention4(const lilicorr_attention4_args* args, hipStream_t stream) {
  if (!args) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_attention4_args& x = *args;
  Plan4 p;
  if (const lilicorr_status s = make_plan4(x, p)) return s;
  if (x.tokens == 0) return LILICORR_OK;
  const lilicorr_cache4& c = x.cache;
  if (!x.q || !x.out || !c.k || !c.v || !c.k_scales || !c.v_scales || !x.table || !x.starts || !x.totals || x.q == x.out)
    return LILICORR_ERR_INVALID_ARG;
  if (!aligned16(x.q) || !aligned16(x.out) || !aligned16(c.k) || !aligned16(c.v) || !aligned16(x.workspace) ||
      !aligned4(x.lse) || !aligned4(c.k_scales) || !aligned4(c.v_scales) || !aligned4(x.table) ||
      !aligned4(x.starts) || !aligned4(x.totals))
    return LILICORR_ERR_ALIGNMENT;
  if (!x.workspace || x.workspace_bytes < p.bytes) return LILICORR_ERR_WORKSPACE;
  if (x.max_tokens == 0) return LILICORR_OK;
  // what is written must not lie on what other waves still read or write
  const size_t row = (size_t)x.heads * c.d * 2, span = cache4_span(c);
  const struct { const void* at; size_t bytes; } parts[] = {
      {x.out, row * (size_t)x.tokens}, {x.lse, x.lse ? (size_t)x.heads * (size_t)x.tokens * 4 : 0}, {x.workspace, p.bytes},
      {c.k, span}, {c.v, span}, {c.k_scales, cache4_scales(span)}, {c.v_scales, cache4_scales(span)},
      {x.table, (size_t)x.N * x.table_width * 4}, {x.starts, ((size_t)x.N + 1) * 4}, {x.totals, (size_t)x.N * 4}};
  constexpr int kWritten = 3, kParts = sizeof(parts) / sizeof(parts[0]);
  for (int i = 0; i < kWritten; ++i) {
    if (rows_overlap(x.q, x.q_stride * 2, row, x.tokens, parts[i].at, parts[i].bytes)) return LILICORR_ERR_INVALID_ARG;
    for (int j = i + 1; j < kParts; ++j)
      if (overlap(parts[i].at, parts[i].bytes, parts[j].at, parts[j].bytes)) return LILICORR_ERR_INVALID_ARG;
  }
  return x.dtype == LILICORR_BF16 ? run4<Bf16>(x, p, stream) : run4<F16>(x, p, stream);
}

extern "C" lilicorr_status lilicorr_key_weights(const lilicorr_key_weights_args* args, hipStream_t stream) {
  if (!args) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_key_weights_args& x = *args;
  if (const lilicorr_status s = sizes4(x)) return s;
  if (!(x.decay >= 0.f) || !isfinite(x.decay)) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_cache4& c = x.cache;
  const int64_t keys = x.table_width * c.page_size < x.max_length ? x.table_width * c.page_size : x.max_length;
  if ((keys + 63) / 64 * x.N > 0x7fffffffll / c.heads) return LILICORR_ERR_UNSUPPORTED;
  if (x.tokens == 0) return LILICORR_OK;
  if (!x.q || !x.lse || !x.weights || !c.k || !c.k_scales || !x.table || !x.starts || !x.totals)
    return LILICORR_ERR_INVALID_ARG;
  if (!aligned16(x.q) || !aligned16(c.k) || !aligned16(x.weights) || !aligned4(x.lse) || !aligned4(c.k_scales) ||
      !aligned4(x.table) || !aligned4(x.starts) || !aligned4(x.totals))
    return LILICORR_ERR_ALIGNMENT;
  if (x.max_tokens == 0) return LILICORR_OK;
  // what other waves still read must not lie where the weights do
  const size_t row = (size_t)x.heads * c.d * 2, w = (size_t)c.pages * c.page_size * c.heads * 4;
  const size_t span = cache4_span(c);
  if (rows_overlap(x.q, x.q_stride * 2, row, x.tokens, x.weights, w) ||
      overlap(x.lse, (size_t)x.heads * (size_t)x.tokens * 4, x.weights, w) || overlap(c.k, span, x.weights, w) ||
      overlap(c.k_scales, cache4_scales(span), x.weights, w) ||
      overlap(x.table, (size_t)x.N * x.table_width * 4, x.weights, w) ||
      overlap(x.starts, ((size_t)x.N + 1) * 4, x.weights, w) || overlap(x.totals, (size_t)x.N * 4, x.weights, w))
    return LILICORR_ERR_INVALID_ARG;
  return x.dtype == LILICORR_BF16 ? run_weights<Bf16>(x, stream) : run_weights<F16>(x, stream);
}
