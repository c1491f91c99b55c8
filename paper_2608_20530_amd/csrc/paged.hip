// The paged cache's bookkeeping and its writers: lilicorr_page_plan (places for one step's tokens),
// lilicorr_qk_norm_rope (head norms, rotation and cache write in one pass) and lilicorr_qk_norm_rope4 (the same into
// a 4-bit cache).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cache4.hpp"
#include "common.hpp"
#include "lilicorr.h"
#include "paged.hpp"

namespace lilicorr {
namespace {

// ---- page plan ---------------------------------------------------------------------------------
// Everything a request needs follows from four prefix sums over the requests before it: new tokens,
// pages taken, pages given back (and the head of the queue). The requests are few (a step's batch),
// so every workgroup makes the sums for itself, 16 bytes a request from the L2, and takes its share
// of the items: tokens, then taken pages, then given-back pages, each found by a binary search in the
// sums. No workgroup waits for another and one launch does it all. Nothing that is read is written in
// the same call: entries [end, end + take) of a table row and ring places from the tail on are
// written, entries below end and places from the head on are read. Bound by latency: one round trip
// for the lengths, the sums in LDS, a search of log2 N LDS reads, one round trip for the page.
// 4.3 us for one request and a block of 16, 6.6 us for 256 requests and 16384 tokens.
constexpr int kPlanThreads = 256;
constexpr int kPlanMaxN = 4096;

struct PlanArgs {
  const int32_t *lengths, *incoming, *pages;
  int32_t *table, *queue;
  const int64_t* cursor;
  int N, P, M, C;
  int64_t tokens, window;
  int first;  // table entries that hold the first `sinks` tokens
  int32_t* pages_out;
  int64_t* cursor_out;
  int32_t *starts, *totals, *slots, *positions;
};

// entries of a request's table row that are filled
__device__ __forceinline__ int row_end(const PlanArgs& a, int n) { return min(max(a.pages[2 * n], 0), a.M); }

// The tokens that a request holds: those that there were no pages for were never stored, and the pages
// that it gets now hold something else where they would be.
__device__ __forceinline__ int row_length(const PlanArgs& a, int n, int end) {
  return min(max(a.lengths[n], 0), end * a.P);  // P * M < 2^31
}

struct PlanRow {
  int64_t total;
  int fresh, take, give, end, since, kept;
  bool ended;
};

__device__ __forceinline__ PlanRow plan_row(const PlanArgs& a, int n) {
  PlanRow r;
  const int I = a.incoming[n];
  r.end = row_end(a, n);
  const int L = row_length(a, n, r.end);
  r.since = max(max(a.pages[2 * n + 1], 0), a.first);
  r.kept = min(a.first, r.end);
  r.ended = I < 0;
  if (r.ended) {
    r.fresh = r.take = 0;
    r.total = 0;
    r.give = r.kept + max(r.end - r.since, 0);
  } else {
    r.fresh = I;
    r.total = (int64_t)L + I;
    const int64_t need = (r.total + a.P - 1) / a.P;
    r.take = max((int)(need < a.M ? need : a.M) - r.end, 0);
    int upto = 0;
    if (a.window) {
      const int64_t behind = (int64_t)L - a.window + 1;  // tokens that no query sees any more
      if (behind > 0) upto = (int)(behind / a.P < r.end ? behind / a.P : r.end);
    }
    r.give = max(upto - r.since, 0);
  }
  return r;
}

__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  const int lane = lane_id();
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int64_t o = (int64_t)shfl64((uint64_t)v, lane - m < 0 ? lane : lane - m);
    if (lane >= m) v += o;
  }
  return v;
}

__device__ __forceinline__ int clamp32(int64_t v) {
  return v < 0x7fffffff ? (int)v : 0x7fffffff;
}

// the last n in [0, N) with sums[n] <= at, for sums[0] = 0 and at < sums[N]
__device__ __forceinline__ int find_row(const int* sums, int N, int at) {
  int lo = 0, hi = N;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (sums[mid] <= at) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PlanArgs a) {
  extern __shared__ int plan_smem[];
  int* const s_tok = plan_smem;              // [N + 1] sums before each request
  int* const s_take = s_tok + a.N + 1;
  int* const s_give = s_take + a.N + 1;
  __shared__ int64_t s_part[3][kPlanThreads / kWave];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;

  const int64_t head = a.cursor[0], tail = a.cursor[1];
  int64_t base[3] = {0, 0, 0};
  for (int n0 = 0; n0 < a.N; n0 += kPlanThreads) {
    const int n = n0 + tid;
    PlanRow r = {};
    if (n < a.N) r = plan_row(a, n);
    int64_t v[3] = {r.fresh, r.take, r.give}, in[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      in[i] = wave_scan(v[i]);
      if (lane == kWave - 1) s_part[i][wave] = in[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int64_t before = base[i], all = 0;
#pragma unroll
      for (int w = 0; w < kPlanThreads / kWave; ++w) {
        if (w < wave) before += s_part[i][w];
        all += s_part[i][w];
      }
      if (n < a.N) plan_smem[i * (a.N + 1) + n] = clamp32(before + in[i] - v[i]);
      base[i] += all;
    }
    __syncthreads();
  }
  if (tid < 3) plan_smem[tid * (a.N + 1) + a.N] = clamp32(base[tid]);
  __syncthreads();

  // free pages, and where the queue's head and tail lie in the ring
  const int64_t free64 = tail - head;
  const int avail = free64 < 0 ? 0 : (int)(free64 < a.C ? free64 : a.C);
  const int at_head = (int)(((head % a.C) + a.C) % a.C), at_tail = (int)(((tail % a.C) + a.C) % a.C);
  auto ring = [&](int at, int i) {  // i < C
    const uint32_t x = (uint32_t)at + (uint32_t)i;
    return (int)(x < (uint32_t)a.C ? x : x - (uint32_t)a.C);
  };

  if (blockIdx.x == 0) {
    for (int n = tid; n < a.N; n += kPlanThreads) {
      const PlanRow r = plan_row(a, n);
      const int granted = max(min(r.take, avail - min(s_take[n], avail)), 0);
      a.pages_out[2 * n] = r.ended ? 0 : r.end + granted;
      a.pages_out[2 * n + 1] = r.ended ? 0 : r.since + r.give;
      // a token past the last row is not taken: it counts neither here nor in starts
      const int64_t rows = a.tokens > s_tok[n] ? a.tokens - s_tok[n] : 0;
      a.totals[n] = clamp32(r.total - (r.fresh > rows ? r.fresh - rows : 0));
    }
    for (int n = tid; n <= a.N; n += kPlanThreads)
      a.starts[n] = s_tok[n] < a.tokens ? s_tok[n] : (int)a.tokens;
    if (tid == 0) {
      a.cursor_out[0] = head + (base[1] < avail ? base[1] : avail);
      a.cursor_out[1] = tail + base[2];
      a.cursor_out[2] = base[1] > avail ? base[1] - avail : 0;
    }
  }

  const int fresh = s_tok[a.N], take = s_take[a.N], give = min(s_give[a.N], a.C);
  const int64_t items = a.tokens + take + give;
  for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + tid; i < items;
       i += (int64_t)gridDim.x * kPlanThreads) {
    if (i < a.tokens) {  // a token's slot and position
      int slot = -1, pos = -1;
      if (i < fresh) {
        const int n = find_row(s_tok, a.N, (int)i);
        const int end = row_end(a, n);
        pos = clamp32((int64_t)row_length(a, n, end) + ((int)i - s_tok[n]));
        const int e = pos / a.P;
        int page = -1;
        if (e < end) {
          page = a.table[(int64_t)n * a.M + e];
        } else if (e < a.M) {
          const int64_t g = (int64_t)s_take[n] + (e - end);
          if (g < avail) page = a.queue[ring(at_head, (int)g)];
        }
        if (page >= 0) slot = clamp32((int64_t)page * a.P + pos % a.P);
      }
      a.slots[i] = slot;
      a.positions[i] = pos;
    } else if (i < a.tokens + take) {  // a taken page into its table row
      const int g = (int)(i - a.tokens);
      const int n = find_row(s_take, a.N, g);
      const int e = row_end(a, n) + (g - s_take[n]);
      if (e < a.M) a.table[(int64_t)n * a.M + e] = g < avail ? a.queue[ring(at_head, g)] : -1;
    } else {  // a page that goes back to the queue
      const int g = (int)(i - a.tokens - take);
      const int n = find_row(s_give, a.N, g);
      const PlanRow r = plan_row(a, n);
      const int k = g - s_give[n];
      const int e = r.ended ? (k < r.kept ? k : r.since + k - r.kept) : r.since + k;
      if (e < a.M) a.queue[ring(at_tail, g)] = a.table[(int64_t)n * a.M + e];
    }
  }
}

// ---- head norms, rotation, cache write ---------------------------------------------------------
// A head is held by LPH lanes, eight elements (16 bytes) each, so a wave has 64 / LPH heads at once
// and a load or store instruction moves whole heads. The wave stays with one token for all of its
// share of heads: the token's cosines and sines, its slot and the norm weights stay in registers. A
// lane needs its partner's elements of the pairs (i, i + rot / 2): rot is a multiple of 16, so the
// partner holds them at the same place and four 32-bit shuffles bring them. Bound by HBM: each
// element read once and written once (85 us for 16381 tokens of 32 + 2 x 8 heads of 128, 4.8 TB/s; a large
// copy reaches 5.06). One token is bound by latency, 3.3 us: everything that it needs is asked for in wide
// loads that do not wait for one another (5.9 with the weights and angles loaded one by one).
constexpr int kRopeThreads = 256;

struct RopeArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  int64_t tokens;
  int parts;  // waves that share a token
  int heads, kv_heads, d, rot, interleaved;
  const int32_t *slots, *positions;
  const float* cos_sin;
  int64_t max_positions;
  const float *q_weight, *k_weight;
  float eps;
  uint16_t *k_cache, *v_cache, *q_out;
  int64_t pages, page_stride, token_stride, head_stride;  // elements; bytes of codes with 4 bits
  int page_size;
  unsigned char *k_scales, *v_scales;  // 4 bits
};

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value,
                                                      0xf, 0xf, false));
  };
  v += dpp(v, std::integral_constant<int, 0xB1>{});   // quad_perm 1,0,3,2
  v += dpp(v, std::integral_constant<int, 0x4E>{});   // quad_perm 2,3,0,1
  v += dpp(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
  if (LPH >= 16) v += dpp(v, std::integral_constant<int, 0x140>{});  // row_mirror
  if (LPH >= 32) v += __shfl_xor(v, 16, kWave);
  return v;
}

// COUNT floats from a 16-byte aligned place
template <int COUNT>
__device__ __forceinline__ void load_floats(const float* from, float (&to)[8]) {
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < COUNT; i += 4) {
    const f32x4_t t = *reinterpret_cast<const f32x4_t*>(from + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) to[i + e] = t[e];
  }
}

// one lane's part of a head: weights of its own elements and of its partner's, cosines and sines of
// its pairs
struct RopeLane {
  float cs[8], sn[8];   // interleaved: four pairs, in [0, 4)
  int partner;          // lane that holds the other halves of the pairs
  bool turned, upper;   // whether this lane's elements turn; whether they are the pairs' b
};

// y: the lane's eight elements. BOUND: `size` for each the sum of the magnitudes that it was made from, `sound` whether
// the mean of squares lies where fp32 neither overflows nor gets coarse
template <typename T, int LPH, bool BOUND>
__device__ __forceinline__ void norm_turn32(const u32x4_t& w, bool norm, const float (&wt)[8],
                                            const float (&wp)[8], const RopeLane& r, int d, float eps, int rot,
                                            int interleaved, float (&y)[8], float (&size)[8], bool& sound) {
  float x[8];
  sound = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2_t t = T::unpack(w[i]);
    x[2 * i] = t[0];
    x[2 * i + 1] = t[1];
  }
  float inv = 1.f;
  if (norm) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
    s = head_sum<LPH>(s);
    const float mean = s * (1.f / (float)d) + eps;
    if constexpr (BOUND) sound = mean > 0x1p-60f && mean < 0x1p60f;
    inv = rsqrtf(mean);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = norm ? x[i] * inv * wt[i] : x[i];
  if constexpr (BOUND) {
#pragma unroll
    for (int i = 0; i < 8; ++i) size[i] = fabsf(y[i]);
  }
  if (rot) {
    if (interleaved) {
      if (r.turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = y[2 * i], b = y[2 * i + 1];
          if constexpr (BOUND) {
            size[2 * i] = fabsf(a * r.cs[i]) + fabsf(b * r.sn[i]);
            size[2 * i + 1] = fabsf(a * r.sn[i]) + fabsf(b * r.cs[i]);
          }
          y[2 * i] = a * r.cs[i] - b * r.sn[i];
          y[2 * i + 1] = a * r.sn[i] + b * r.cs[i];
        }
      }
    } else {
      u32x4_t o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = (uint32_t)__shfl((int)w[i], r.partner, kWave);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2_t t = T::unpack(o[i]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int j = 2 * i + e;
          const float z = norm ? t[e] * inv * wp[j] : t[e];
          if constexpr (BOUND) size[j] = r.turned ? fabsf(y[j] * r.cs[j]) + fabsf(z * r.sn[j]) : size[j];
          // a c - b s for the lower half, b c + a s for the upper one
          const float turn = r.upper ? y[j] * r.cs[j] + z * r.sn[j] : y[j] * r.cs[j] - z * r.sn[j];
          y[j] = r.turned ? turn : y[j];
        }
      }
    }
  }
}

template <typename T, int LPH>
__device__ __forceinline__ u32x4_t norm_turn(const u32x4_t& w, bool norm, const float (&wt)[8],
                                             const float (&wp)[8], const RopeLane& r, int d,
                                             float eps, int rot, int interleaved) {
  float y[8], size[8];
  bool sound;
  norm_turn32<T, LPH, false>(w, norm, wt, wp, r, d, eps, rot, interleaved, y, size, sound);
  u32x4_t out;
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = T::pack(y[2 * i], y[2 * i + 1]);
  return out;
}

// ---- the same in 4 bits ------------------------------------------------------------------------
// A block of 32 elements lies in four neighbouring lanes. With the block's largest magnitude m 2^e, 1 <= m < 2, its
// scale is 2^(e - 2) if m <= 7 / 4 and 2^(e - 1) if not; adding 2^21 - 1 to the mantissa's 23 bits carries into the
// exponent in just the second case.
__device__ __forceinline__ uint32_t scale4(float most) {
  const int e = (int)((__float_as_uint(most) + 0x1fffffu) >> 23) - 2;  // of a biased exponent
  return (uint32_t)min(max(e, (int)kLeastScale), (int)kMostScale);
}

// codes of eight elements: nearest, ties to the even code, saturating (the conversion's own rounding)
__device__ __forceinline__ uint32_t codes4(const float (&y)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  return w;
}

// the largest over four neighbouring lanes, NaN if one is
__device__ __forceinline__ float block_max(float v) {
  v = __builtin_elementwise_maximum(
      v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, false)));
  return __builtin_elementwise_maximum(
      v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, false)));
}

struct Code4 {
  uint32_t w, scale;
};

// Values that are what they are: v as it comes.
template <typename T>
__device__ __forceinline__ Code4 quantise(const u32x4_t& w) {
  float y[8], most = 0.f;
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i];
    const f32x2_t t = T::unpack(x);
    y[2 * i] = t[0];
    y[2 * i + 1] = t[1];
    bad |= T::nonfinite(x);
    most = fmaxf(most, fmaxf(fabsf(t[0]), fabsf(t[1])));
  }
  most = block_max(bad ? __builtin_inff() : most);
  if (most == __builtin_inff()) return {0, kNanScale};
  const uint32_t s = scale4(most);
  return {codes4(y, scale_of(s)), s};
}

// A key in 64 bits, from its elements on: sums, norm, rotation, scale and codes. No contraction: each operation is
// rounded as it stands in the formula. `weight` and `weight_p` at the lane's and its partner's elements, or NULL; `angles`
// at its pairs' cosines.
template <typename T, int LPH>
__device__ __forceinline__ Code4 quantise64(const u32x4_t& w, const float* weight, const float* weight_p, const float* angles,
                                            int partner, bool turned, bool upper, int d, float eps, int rot,
                                            int interleaved) {
#pragma clang fp contract(off)
  const bool norm = weight != nullptr;
  float wt[8], wp[8];
  RopeLane r;
  r.partner = partner;
  r.turned = turned;
  r.upper = upper;
  if (norm) {
    load_floats<8>(weight, wt);
    load_floats<8>(weight_p, wp);
  }
  if (rot && interleaved) {
    load_floats<4>(angles, r.cs);
    load_floats<4>(angles + rot / 2, r.sn);
  } else if (rot) {
    load_floats<8>(angles, r.cs);
    load_floats<8>(angles + rot / 2, r.sn);
  }
  double x[8], s = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = w[i];
    const f32x2_t t = T::unpack(u);
    x[2 * i] = t[0];
    x[2 * i + 1] = t[1];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) s += x[i] * x[i];
#pragma unroll
  for (int m = 1; m < LPH; m <<= 1)
    s += __longlong_as_double((long long)shfl_xor64((uint64_t)__double_as_longlong(s), m));
  const double root = norm ? sqrt(s / d + (double)eps) : 1.0;
  double y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = norm ? x[i] / root * (double)wt[i] : x[i];
  if (rot && interleaved) {
    if (r.turned) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double a = y[2 * i], b = y[2 * i + 1], c = r.cs[i], n = r.sn[i];
        y[2 * i] = a * c - b * n;
        y[2 * i + 1] = a * n + b * c;
      }
    }
  } else if (rot) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = (uint32_t)__shfl((int)w[i], r.partner, kWave);
      const f32x2_t t = T::unpack(u);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = 2 * i + e;
        const double z = norm ? (double)t[e] / root * (double)wp[j] : (double)t[e], c = r.cs[j], n = r.sn[j];
        const double turn = r.upper ? z * n + y[j] * c : y[j] * c - z * n;
        y[j] = r.turned ? turn : y[j];
      }
    }
  }
  double most = 0;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    bad |= !(fabs(y[i]) < __builtin_inf());
    most = fmax(most, fabs(y[i]));
  }
  if (bad) most = __builtin_inf();
#pragma unroll
  for (int m = 1; m < 4; m <<= 1)
    most = fmax(most, __longlong_as_double((long long)shfl_xor64((uint64_t)__double_as_longlong(most), m)));
  if (most == __builtin_inf()) return {0, kNanScale};
  int e;
  const double f = frexp(most, &e);  // most = f 2^e, 0.5 <= f < 1
  e = most == 0 ? -200 : e - (f <= 0.875 ? 3 : 2);
  const int b = min(max(e + 127, (int)kLeastScale), (int)kMostScale);
  const double back = ldexp(1.0, 127 - b);
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double v = fabs(y[i]) * back;  // exact
    const uint32_t c = (v > 0.25) + (v >= 0.75) + (v > 1.25) + (v >= 1.75) + (v > 2.5) + (v >= 3.5) + (v > 5.0);
    out |= (c | ((uint64_t)__double_as_longlong(y[i]) >> 63 ? 8u : 0u)) << (4 * i);
  }
  return {out, (uint32_t)b};
}

// A key in fp32, and whether some element's scale, code or sign is not certain: then it is done again in 64 bits. An
// element is at most 2^-20 of the magnitudes that it was made from off (sum of squares 13 roundings, halved by the
// root; mean, root, two factors, two products and a sum: 16 in all of 2^-24), so it is certain where four times that
// up or down changes nothing. That holds where nothing overflows (the size is infinite or the mean too large then) and
// where what underflows does not count: with a mean of 2^-60 .. 2^60 and weights up to kWild a product that fp32 rounds more
// coarsely than 2^-24 makes an error of 2^-129 in the end and a pair below 2^-105. An element that is not over kSmall is done
// again unless its own x is 0 (the other of its pair sees to what that one makes). With normal values one step of a wave
// in 400 is done again.
constexpr float kUncertain = 0x1p-18f, kSmall = 0x1p-100f, kWild = 0x1p20f;
template <typename T, int LPH>
__device__ __forceinline__ Code4 quantise_key(const u32x4_t& w, bool norm, const float (&wt)[8], const float (&wp)[8],
                                              const RopeLane& r, int d, float eps, int rot, int interleaved,
                                              bool& unsure) {
  float y[8], size[8], lo[8], hi[8], most_lo = 0.f, most_hi = 0.f;
  bool sound;
  norm_turn32<T, LPH, true>(w, norm, wt, wp, r, d, eps, rot, interleaved, y, size, sound);
  unsure = !sound;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float off = size[i] * kUncertain, v = fabsf(y[i]);
    lo[i] = v - off;
    hi[i] = v + off;
    const uint32_t word = w[i / 2];
    unsure |= !(lo[i] > kSmall) && T::unpack(word)[i % 2] != 0.f;  // the sign
    most_lo = fmaxf(most_lo, lo[i]);
    most_hi = __builtin_elementwise_maximum(most_hi, hi[i]);  // NaN if one is
  }
  most_lo = block_max(most_lo);
  most_hi = block_max(most_hi);
  const uint32_t s = scale4(most_lo);
  unsure |= !(most_hi < 0x1p126f) || s != scale4(most_hi);
  const float scale = scale_of(s);
  unsure |= codes4(lo, scale) != codes4(hi, scale);
  return {codes4(y, scale), s};
}

template <typename T, int LPH, bool FOUR>
__global__ __launch_bounds__(kRopeThreads, FOUR ? 4 : 1) void qk_norm_rope_kernel(RopeArgs a) {
  constexpr int kHeads = kWave / LPH;  // heads a wave holds
  const int lane = lane_id(), l = lane % LPH, g = lane / LPH;
  const int e0 = l * 8;
  const bool mine = e0 < a.d;  // lanes past the head's width hold nothing

  RopeLane r;
  const int half = a.rot / 2;
  r.turned = mine && e0 < a.rot;
  r.upper = e0 >= half;
  const int po = a.interleaved || !r.turned ? e0 : (r.upper ? e0 - half : e0 + half);
  r.partner = g * LPH + po / 8;
  const bool norm_q = a.q_weight != nullptr, norm_k = a.k_weight != nullptr;
  // (lanes that hold nothing read the first ones)
  float qw[8], qp[8], kw[8], kp[8];
  if (norm_q) {
    load_floats<8>(a.q_weight + (mine ? e0 : 0), qw);
    load_floats<8>(a.q_weight + (mine ? po : 0), qp);
  }
  if (norm_k) {
    load_floats<8>(a.k_weight + (mine ? e0 : 0), kw);
    load_floats<8>(a.k_weight + (mine ? po : 0), kp);
  }
  bool wild = false;
  if (FOUR && norm_k)
#pragma unroll
    for (int i = 0; i < 8; ++i) wild |= !(fabsf(kw[i]) <= kWild);

  const int qs = (a.heads + kHeads - 1) / kHeads, ks = (a.kv_heads + kHeads - 1) / kHeads;
  const int steps = qs + 2 * ks;
  constexpr int kBatch = 4;  // steps whose loads are under way together
  const int wave = (int)uniform32(threadIdx.x / kWave);
  const int waves = (int)gridDim.x * (kRopeThreads / kWave);
  const int64_t items = a.tokens * a.parts;
  // 4 bits: the wave's steps whose keys have to be done again in 64 bits, as (turn, step); with more than kAgain of them
  // all keys are. They are done after the rest, so that they cost the rest no registers (within it: 229 of them, and
  // 119 us for 16381 tokens).
  constexpr int kAgain = 64;
  __shared__ uint32_t s_again[FOUR ? kRopeThreads / kWave : 1][FOUR ? kAgain : 1];
  uint32_t again = __ballot(wild) ? kAgain + 1 : 0, turn = 0;
  for (int64_t it = (int64_t)blockIdx.x * (kRopeThreads / kWave) + wave; it < items; it += waves, ++turn) {
    const int64_t t = it / a.parts;
    const int part = (int)(it - t * a.parts);
    const int s0 = steps * part / a.parts, s1 = steps * (part + 1) / a.parts;
    u32x4_t w[kBatch];
    auto load = [&](int s, u32x4_t& x) {  // this lane's piece of step s
      const int kind = s < qs ? 0 : s < qs + ks ? 1 : 2;
      const int h = (s - (kind == 0 ? 0 : kind == 1 ? qs : qs + ks)) * kHeads + g;
      const uint16_t* src = kind == 0 ? a.q + t * a.q_stride
                                      : kind == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride;
      x = u32x4_t{0, 0, 0, 0};
      if (s < s1 && mine && h < (kind == 0 ? a.heads : a.kv_heads))
        x = *reinterpret_cast<const u32x4_t*>(src + (int64_t)h * a.d + e0);
    };
#pragma unroll
    for (int u = 0; u < kBatch; ++u) load(s0 + u, w[u]);
    const int pos = a.positions[t], slot = a.slots[t];
    const bool live = a.rot ? pos >= 0 && pos < a.max_positions : pos >= 0;
    const int page = slot < 0 ? -1 : slot / a.page_size;
    const bool stored = live && page >= 0 && page < a.pages;
    const int64_t at =
        stored ? page * a.page_stride + (int64_t)(slot - page * a.page_size) * a.token_stride : 0;
    if (live && a.rot) {
      const float* cs = a.cos_sin + (int64_t)pos * a.rot;
      if (a.interleaved) {
        const int p0 = r.turned ? e0 / 2 : 0;
        load_floats<4>(cs + p0, r.cs);
        load_floats<4>(cs + half + p0, r.sn);
      } else {
        const int p0 = !r.turned ? 0 : r.upper ? e0 - half : e0;
        load_floats<8>(cs + p0, r.cs);
        load_floats<8>(cs + half + p0, r.sn);
      }
    }
    for (int s = s0; s < s1; s += kBatch) {
      u32x4_t x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) x[u] = w[u];
      if (s + kBatch < s1) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) load(s + kBatch + u, w[u]);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (s + u >= s1) break;
        if (s + u < qs) {
          const int h = (s + u) * kHeads + g;
          const u32x4_t y = live ? norm_turn<T, LPH>(x[u], norm_q, qw, qp, r, a.d, a.eps, a.rot, a.interleaved)
                                 : u32x4_t{0, 0, 0, 0};
          if (mine && h < a.heads)
            *reinterpret_cast<u32x4_t*>(a.q_out + (t * a.heads + h) * a.d + e0) = y;
        } else {
          if (!stored) break;
          const bool is_k = s + u < qs + ks;
          const int h = (is_k ? s + u - qs : s + u - qs - ks) * kHeads + g;
          if constexpr (FOUR) {
            bool unsure = false;
            const Code4 y = is_k ? quantise_key<T, LPH>(x[u], norm_k, kw, kp, r, a.d, a.eps, a.rot, a.interleaved, unsure)
                                 : quantise<T>(x[u]);
            if (__ballot(unsure)) {
              if (again < kAgain) s_again[wave][again] = turn * steps + (s + u);
              ++again;
            }
            const int64_t to = at + (int64_t)h * a.head_stride;
            if (mine && h < a.kv_heads) {
              *reinterpret_cast<uint32_t*>((unsigned char*)(is_k ? a.k_cache : a.v_cache) + to + l * 4) = y.w;
              if (l % 4 == 0) (is_k ? a.k_scales : a.v_scales)[to / 16 + l / 4] = (unsigned char)y.scale;
            }
            continue;
          }
          const u32x4_t y =
              is_k ? norm_turn<T, LPH>(x[u], norm_k, kw, kp, r, a.d, a.eps, a.rot, a.interleaved) : x[u];
          uint16_t* dst = (is_k ? a.k_cache : a.v_cache) + at + (int64_t)h * a.head_stride;
          if (mine && h < a.kv_heads) *reinterpret_cast<u32x4_t*>(dst + e0) = y;
        }
      }
    }
  }
  if constexpr (FOUR) {
    const int64_t first = (int64_t)blockIdx.x * (kRopeThreads / kWave) + wave;
    const uint32_t all = turn * (uint32_t)steps;  // (turn, step) of all of the wave's turns
    const bool listed = again <= kAgain;
    for (uint32_t i = 0; i < (listed ? again : all); ++i) {
      const uint32_t which = uniform32(listed ? s_again[wave][i] : i);
      const int64_t it = first + (int64_t)(which / steps) * waves, t = it / a.parts;
      const int s = (int)(which % steps), part = (int)(it - t * a.parts);
      if (s < qs || s >= qs + ks || s < steps * part / a.parts || s >= steps * (part + 1) / a.parts) continue;
      const int pos = a.positions[t], slot = a.slots[t];
      const int page = slot < 0 ? -1 : slot / a.page_size;
      if (pos < 0 || (a.rot && pos >= a.max_positions) || page < 0 || page >= a.pages) continue;
      const int h = (s - qs) * kHeads + g;
      u32x4_t x = {0, 0, 0, 0};
      if (mine && h < a.kv_heads) x = *reinterpret_cast<const u32x4_t*>(a.k + t * a.k_stride + (int64_t)h * a.d + e0);
      const int p0 = !r.turned ? 0 : a.interleaved ? e0 / 2 : r.upper ? e0 - half : e0;
      const Code4 y = quantise64<T, LPH>(x, norm_k ? a.k_weight + (mine ? e0 : 0) : nullptr,
                                         norm_k ? a.k_weight + (mine ? po : 0) : nullptr,
                                         a.rot ? a.cos_sin + (int64_t)pos * a.rot + p0 : nullptr, r.partner, r.turned,
                                         r.upper, a.d, a.eps, a.rot, a.interleaved);
      const int64_t to = page * a.page_stride + (int64_t)(slot - page * a.page_size) * a.token_stride +
                         (int64_t)h * a.head_stride;
      if (mine && h < a.kv_heads) {
        *reinterpret_cast<uint32_t*>((unsigned char*)a.k_cache + to + l * 4) = y.w;
        if (l % 4 == 0) a.k_scales[to / 16 + l / 4] = (unsigned char)y.scale;
      }
    }
  }
}

template <typename T, bool FOUR>
void launch_rope(const RopeArgs& a, hipStream_t stream) {
  const int64_t items = a.tokens * a.parts, per = kRopeThreads / kWave;
  const int64_t want = (items + per - 1) / per;
  // four workgroups a compute unit, which stay (16381 tokens of 32 + 2 x 8 heads of 128: 86 us; 114 with 512
  // workgroups, 86 to 88 with 2048 and more)
  const dim3 grid((unsigned)(want < 1024 ? want : 1024));
  if (a.d <= 64)
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, 8, FOUR>), grid, dim3(kRopeThreads), 0, stream, a);
  else if (a.d <= 128)
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, 16, FOUR>), grid, dim3(kRopeThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, 32, FOUR>), grid, dim3(kRopeThreads), 0, stream, a);
}

// waves that share a token
int rope_parts(int64_t tokens, int heads, int kv_heads, int d) {
  // Few tokens: their steps spread over more waves, one each, or about three each while the waves have
  // work at once anyway. With 12 steps a token (32 + 2 x 8 heads of 128): 16 tokens 3.6 us as 12 waves, 4.7
  // as 4, 9.8 as 1; 256 tokens 5.5, 5.1, 10.3; 1024 tokens 12.9, 9.1, 11.8; 2048 tokens 13.3 as 4, 13.0 as
  // 2, 14.6 as 1; 4096 tokens 22.0, 20.5, 20.1. The two limits were chosen there, for all widths.
  const int each = d <= 64 ? 8 : d <= 128 ? 4 : 2;  // heads of a step
  const int64_t steps = (heads + each - 1) / each + 2 * ((kv_heads + each - 1) / each);
  const int64_t fit = 6144 / tokens, third = (steps + 2) / 3;
  return (int)(tokens * steps <= 2400 ? steps : fit < 1 ? 1 : fit < third ? fit : third);
}

}  // namespace
}  // namespace lilicorr

using namespace lilicorr;

extern "C" lilicorr_status lilicorr_page_plan(const lilicorr_page_plan_args* args,
                                              hipStream_t stream) {
  if (!args) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_page_plan_args& x = *args;
  if (!x.lengths || !x.incoming || !x.pages || !x.table || !x.queue || !x.cursor || !x.pages_out ||
      !x.cursor_out || !x.starts || !x.totals)
    return LILICORR_ERR_INVALID_ARG;
  if (x.N < 1 || x.page_size < 1 || x.table_width < 1 || x.queue_size < 1 || x.tokens < 0 ||
      x.window < 0 || x.sinks < 0 || (x.sinks > 0 && x.window == 0))
    return LILICORR_ERR_INVALID_ARG;
  if (x.tokens > 0 && (!x.slots || !x.positions)) return LILICORR_ERR_INVALID_ARG;
  if (x.pages_out == x.pages || x.cursor_out == x.cursor) return LILICORR_ERR_INVALID_ARG;
  if (x.N > kPlanMaxN || x.page_size > 65536 || x.table_width > 0x7fffffffll / x.page_size ||
      x.queue_size > 0x7fffffffll || x.tokens > 0x7fffffffll || x.window > 0x7fffffffll ||
      x.sinks > 0x7fffffffll - x.page_size)
    return LILICORR_ERR_UNSUPPORTED;
  if (!aligned4(x.lengths) || !aligned4(x.incoming) || !aligned4(x.pages) || !aligned4(x.table) ||
      !aligned4(x.queue) || !aligned8(x.cursor) || !aligned4(x.pages_out) ||
      !aligned8(x.cursor_out) || !aligned4(x.starts) || !aligned4(x.totals) || !aligned4(x.slots) ||
      !aligned4(x.positions))
    return LILICORR_ERR_ALIGNMENT;
  // workgroups read what others' outputs would lie on: only the arrays that are not written may share memory
  constexpr int kRead = 4;
  const size_t n4 = (size_t)x.N * 4, t4 = (size_t)x.tokens * 4;
  const struct { const void* at; size_t bytes; } parts[] = {
      {x.lengths, n4}, {x.incoming, n4}, {x.pages, 2 * n4}, {x.cursor, 24},
      {x.table, n4 * (size_t)x.table_width}, {x.queue, (size_t)x.queue_size * 4}, {x.pages_out, 2 * n4},
      {x.cursor_out, 24}, {x.starts, n4 + 4}, {x.totals, n4}, {x.slots, t4}, {x.positions, t4}};
  constexpr int kParts = sizeof(parts) / sizeof(parts[0]);
  for (int i = kRead; i < kParts; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(parts[i].at, parts[i].bytes, parts[j].at, parts[j].bytes)) return LILICORR_ERR_INVALID_ARG;
  PlanArgs a;
  a.lengths = x.lengths; a.incoming = x.incoming; a.pages = x.pages;
  a.table = x.table; a.queue = x.queue; a.cursor = x.cursor;
  a.N = (int)x.N; a.P = (int)x.page_size; a.M = (int)x.table_width; a.C = (int)x.queue_size;
  a.tokens = x.tokens; a.window = x.window;
  a.first = (int)((x.sinks + x.page_size - 1) / x.page_size);
  a.pages_out = x.pages_out; a.cursor_out = x.cursor_out;
  a.starts = x.starts; a.totals = x.totals; a.slots = x.slots; a.positions = x.positions;
  // a workgroup for 256 tokens; a batch without new tokens still has pages to give back
  int64_t grid = (x.tokens + kPlanThreads - 1) / kPlanThreads;
  if (grid < (x.N + 63) / 64) grid = (x.N + 63) / 64;
  if (grid > 1024) grid = 1024;
  hipLaunchKernelGGL(page_plan_kernel, dim3((unsigned)grid), dim3(kPlanThreads),
                     3 * ((size_t)x.N + 1) * sizeof(int), stream, a);
  return launch_status();
}

extern "C" lilicorr_status lilicorr_qk_norm_rope(const lilicorr_qk_norm_rope_args* args,
                                                 hipStream_t stream) {
  if (!args) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_qk_norm_rope_args& x = *args;
  const lilicorr_cache& c = x.cache;
  if (const lilicorr_status s = cache_sizes(c)) return s;
  if (x.heads < 1 || x.tokens < 0 || x.rot < 0 || x.rot > c.d || x.max_positions < 0)
    return LILICORR_ERR_INVALID_ARG;
  if (!(x.eps >= 0.f) || !isfinite(x.eps)) return LILICORR_ERR_INVALID_ARG;
  if (x.q_stride < 0 || x.k_stride < 0 || x.v_stride < 0) return LILICORR_ERR_INVALID_ARG;
  if (x.rot % 16 || x.heads > 65535 || x.tokens > 0x7fffffffll) return LILICORR_ERR_UNSUPPORTED;
  if (!stride_ok(x.q_stride) || !stride_ok(x.k_stride) || !stride_ok(x.v_stride))
    return LILICORR_ERR_ALIGNMENT;
  if (x.tokens == 0) return LILICORR_OK;
  if (!x.q || !x.k || !x.v || !x.slots || !x.positions || !x.q_out || !c.k || !c.v ||
      (x.rot > 0 && !x.cos_sin))
    return LILICORR_ERR_INVALID_ARG;
  // q rows that are turned in place must be laid out as the output is
  if (x.q_out == x.q && x.tokens > 1 && x.q_stride != (int64_t)x.heads * c.d)
    return LILICORR_ERR_INVALID_ARG;
  if (!aligned16(x.q) || !aligned16(x.k) || !aligned16(x.v) || !aligned16(x.q_out) ||
      !aligned16(c.k) || !aligned16(c.v) || !aligned16(x.cos_sin) || !aligned16(x.q_weight) ||
      !aligned16(x.k_weight) || !aligned4(x.slots) || !aligned4(x.positions))
    return LILICORR_ERR_ALIGNMENT;
  // what other waves still read must not lie where q_out does
  const size_t q_row = (size_t)x.heads * c.d * 2, k_row = (size_t)c.heads * c.d * 2, out_bytes = q_row * (size_t)x.tokens;
  if ((x.q_out != x.q && rows_overlap(x.q, x.q_stride * 2, q_row, x.tokens, x.q_out, out_bytes)) ||
      rows_overlap(x.k, x.k_stride * 2, k_row, x.tokens, x.q_out, out_bytes) ||
      rows_overlap(x.v, x.v_stride * 2, k_row, x.tokens, x.q_out, out_bytes))
    return LILICORR_ERR_INVALID_ARG;
  RopeArgs a = {};
  a.q = (const uint16_t*)x.q; a.k = (const uint16_t*)x.k; a.v = (const uint16_t*)x.v;
  a.q_stride = x.q_stride; a.k_stride = x.k_stride; a.v_stride = x.v_stride;
  a.tokens = x.tokens;
  a.heads = x.heads; a.kv_heads = c.heads; a.d = c.d; a.rot = x.rot;
  a.interleaved = x.interleaved != 0;
  a.slots = x.slots; a.positions = x.positions; a.cos_sin = x.cos_sin;
  a.max_positions = x.max_positions;
  a.q_weight = x.q_weight; a.k_weight = x.k_weight; a.eps = x.eps;
  a.k_cache = (uint16_t*)c.k; a.v_cache = (uint16_t*)c.v; a.q_out = (uint16_t*)x.q_out;
  a.pages = c.pages; a.page_stride = c.page_stride; a.token_stride = c.token_stride;
  a.head_stride = c.head_stride;
  a.page_size = c.page_size;
  a.parts = rope_parts(x.tokens, x.heads, c.heads, c.d);
  if (c.dtype == LILICORR_BF16) launch_rope<Bf16, false>(a, stream);
  else launch_rope<F16, false>(a, stream);
  return launch_status();
}

extern "C" lilicorr_status lilicorr_qk_norm_rope4(const lilicorr_qk_norm_rope4_args* args, hipStream_t stream) {
  if (!args) return LILICORR_ERR_INVALID_ARG;
  const lilicorr_qk_norm_rope4_args& x = *args;
  const lilicorr_cache4& c = x.cache;
  if (const lilicorr_status s = cache4_sizes(c)) return s;
  if (x.dtype != LILICORR_BF16 && x.dtype != LILICORR_F16) return LILICORR_ERR_INVALID_ARG;
  if (x.heads < 1 || x.tokens < 0 || x.rot < 0 || x.rot > c.d || x.max_positions < 0)
    return LILICORR_ERR_INVALID_ARG;
  if (!(x.eps >= 0.f) || !isfinite(x.eps)) return LILICORR_ERR_INVALID_ARG;
  if (x.q_stride < 0 || x.k_stride < 0 || x.v_stride < 0) return LILICORR_ERR_INVALID_ARG;
  if (x.rot % 16 || x.heads > 65535 || x.tokens > 0x7fffffffll) return LILICORR_ERR_UNSUPPORTED;
  if (!stride_ok(x.q_stride) || !stride_ok(x.k_stride) || !stride_ok(x.v_stride))
    return LILICORR_ERR_ALIGNMENT;
  if (x.tokens == 0) return LILICORR_OK;
  if (!x.q || !x.k || !x.v || !x.slots || !x.positions || !x.q_out || !c.k || !c.v || !c.k_scales || !c.v_scales ||
      (x.rot > 0 && !x.cos_sin))
    return LILICORR_ERR_INVALID_ARG;
  // q rows that are turned in place must be laid out as the output is
  if (x.q_out == x.q && x.tokens > 1 && x.q_stride != (int64_t)x.heads * c.d) return LILICORR_ERR_INVALID_ARG;
  if (!aligned16(x.q) || !aligned16(x.k) || !aligned16(x.v) || !aligned16(x.q_out) || !aligned16(c.k) ||
      !aligned16(c.v) || !aligned4(c.k_scales) || !aligned4(c.v_scales) || !aligned16(x.cos_sin) ||
      !aligned16(x.q_weight) || !aligned16(x.k_weight) ||
      !aligned4(x.slots) || !aligned4(x.positions))
    return LILICORR_ERR_ALIGNMENT;
  // what other waves still read must not lie where q_out does, nor q_out in the cache
  const size_t q_row = (size_t)x.heads * c.d * 2, k_row = (size_t)c.heads * c.d * 2, out = q_row * (size_t)x.tokens;
  const size_t span = cache4_span(c);
  if ((x.q_out != x.q && rows_overlap(x.q, x.q_stride * 2, q_row, x.tokens, x.q_out, out)) ||
      rows_overlap(x.k, x.k_stride * 2, k_row, x.tokens, x.q_out, out) ||
      rows_overlap(x.v, x.v_stride * 2, k_row, x.tokens, x.q_out, out))
    return LILICORR_ERR_INVALID_ARG;
  const struct { const void* at; size_t bytes; } parts[] = {
      {c.k, span}, {c.v, span}, {c.k_scales, cache4_scales(span)}, {c.v_scales, cache4_scales(span)}};
  for (const auto& p : parts)
    if (overlap(x.q_out, out, p.at, p.bytes) || rows_overlap(x.q, x.q_stride * 2, q_row, x.tokens, p.at, p.bytes) ||
        rows_overlap(x.k, x.k_stride * 2, k_row, x.tokens, p.at, p.bytes) ||
        rows_overlap(x.v, x.v_stride * 2, k_row, x.tokens, p.at, p.bytes))
      return LILICORR_ERR_INVALID_ARG;
  RopeArgs a = {};
  a.q = (const uint16_t*)x.q; a.k = (const uint16_t*)x.k; a.v = (const uint16_t*)x.v;
  a.q_stride = x.q_stride; a.k_stride = x.k_stride; a.v_stride = x.v_stride;
  a.tokens = x.tokens;
  a.heads = x.heads; a.kv_heads = c.heads; a.d = c.d; a.rot = x.rot;
  a.interleaved = x.interleaved != 0;
  a.slots = x.slots; a.positions = x.positions; a.cos_sin = x.cos_sin;
  a.max_positions = x.max_positions;
  a.q_weight = x.q_weight; a.k_weight = x.k_weight; a.eps = x.eps;
  a.k_cache = (uint16_t*)c.k; a.v_cache = (uint16_t*)c.v; a.q_out = (uint16_t*)x.q_out;
  a.k_scales = (unsigned char*)c.k_scales; a.v_scales = (unsigned char*)c.v_scales;
  a.pages = c.pages; a.page_stride = c.page_stride; a.token_stride = c.token_stride;
  a.head_stride = c.head_stride;
  a.page_size = c.page_size;
  a.parts = rope_parts(x.tokens, x.heads, c.heads, c.d);
  if (x.dtype == LILICORR_BF16) launch_rope<Bf16, true>(a, stream);
  else launch_rope<F16, true>(a, stream);
  return launch_status();
}
