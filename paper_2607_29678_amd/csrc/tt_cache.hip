// tt_cache_append: keys and values of a step's tokens into the slots of a paged
// cache, with the position rotation applied on the way, to the queries too.
//
// The work is a copy with one rotation: a block takes a few tokens, computes the
// cosine and sine of each of their pairs once (all heads of a token share them),
// and then moves 16 bytes a thread (32 where the two halves of a pair lie apart).
// Angles: position * frequency is exact in 64 bits but for its last place, and so
// is what is left of it after whole turns; in 32 bits a position of 10^6 would
// have an angle that is off by 0.03.
//
// What bounds it: reads and writes; 30,001 tokens of 20 + 4 + 4 heads of 96 elements in
// f16, half of each rotated, take 69 us, 4.7 TB/s of a plain copy's 4.9.  96 tokens: the
// host call and the chain of slot, angles and store.
#include "tt_cache.h"

namespace tt {
namespace {

constexpr int APP_THREADS = 256;
constexpr int APP_TOKENS = 3;  // most tokens of a block

// u / d for u < 2^16 and d < 2^16, as a product
struct Division {
  uint32_t d = 1, m = 0;
  Division() = default;
  explicit Division(uint32_t by) : d(by), m(by > 1 ? 0xFFFFFFFFu / by + 1 : 0) {}
  __device__ __forceinline__ uint32_t of(uint32_t u) const { return d > 1 ? __umulhi(u, m) : u; }
};

template <class T>
struct AppendArgs {
  tt_cache cache;
  int64_t tokens;
  const int64_t* slots;
  const int32_t* positions;
  const float* frequencies;
  const T *keys, *values, *queries;
  T* rotated;
  int64_t key_stride, value_stride, query_stride, rotated_stride;
  int pairs;
  int each;              // tokens of a block
  int turned, straight;  // units of a rotated head and of one that is copied
  uint32_t q_units, k_units, units;  // units of a token: queries, then keys, then values
  Division by_units, by_turned, by_straight;
};

enum AppendMode { HALVES, NEIGHBOURS, ELEMENTS };

// MODE says what a unit of work is.  HALVES: 8 elements and the 8 that are pairs
// behind them (or 8 that are not rotated); NEIGHBOURS: 8 elements; ELEMENTS: one
// pair or one element that is not rotated, for rows off their alignment and for
// pairs that do not come in vectors (INTERLEAVED there).
template <class T, AppendMode MODE, bool INTERLEAVED>
__global__ __launch_bounds__(APP_THREADS) void append_kernel(AppendArgs<T> a) {
  __shared__ float2 turn[APP_TOKENS * TT_MAX_HEAD_DIM / 2];  // (cos, sin) of [token][pair]
  __shared__ int64_t place[APP_TOKENS];                      // of the token's slot in the caches; -1: none
  using V8 = Vec8<T>;
  const int tid = threadIdx.x, pairs = a.pairs, dim = a.cache.dim;
  const int64_t first = (int64_t)blockIdx.x * a.each;
  const int here = a.tokens - first < a.each ? (int)(a.tokens - first) : a.each;
  const uint32_t total = (uint32_t)here * a.units;

  struct Unit {
    const T* in;
    int token, head, part, at, apart;  // at: first element; apart: distance of the second half, 0: none
    V8 x, y;
    T p, q;
  };
  // A unit's place in its token, and its elements
  auto fetch = [&](uint32_t i) {
    Unit n;
    n.token = (int)a.by_units.of(i);
    uint32_t u = i - (uint32_t)n.token * a.units;
    const int64_t t = first + n.token;
    n.part = u < a.q_units ? 0 : u < a.q_units + a.k_units ? 1 : 2;
    n.in = n.part == 0 ? a.queries + t * a.query_stride : n.part == 1 ? a.keys + t * a.key_stride : a.values + t * a.value_stride;
    u -= n.part == 0 ? 0 : n.part == 1 ? a.q_units : a.q_units + a.k_units;
    const uint32_t size = n.part == 2 ? a.straight : a.turned;
    n.head = (int)(n.part == 2 ? a.by_straight.of(u) : a.by_turned.of(u));
    const int w = (int)(u - (uint32_t)n.head * size);
    const int rotated = n.part == 2 ? 0 : pairs;  // pairs of this head
    n.apart = 0;
    if (MODE == ELEMENTS) {
      const bool turns = w < rotated;
      n.at = !turns ? w + rotated : INTERLEAVED ? 2 * w : w;
      if (turns) n.apart = INTERLEAVED ? 1 : pairs;
    } else if (MODE == HALVES) {
      const bool turns = 8 * w < rotated;
      n.at = turns ? 8 * w : 8 * w + rotated;
      if (turns) n.apart = pairs;
    } else {
      n.at = 8 * w;
    }
    const T* p = n.in + n.head * dim + n.at;
    if (MODE == ELEMENTS) {
      n.p = *p;
      if (n.apart) n.q = p[n.apart];
    } else {
      n.x = *reinterpret_cast<const V8*>(p);
      if (n.apart) n.y = *reinterpret_cast<const V8*>(p + n.apart);
    }
    return n;
  };
  auto finish = [&](Unit n) {
    const int64_t at = place[n.token];
    if (at < 0) return;
    const float2* cs = turn + n.token * pairs;
    if (MODE == ELEMENTS) {
      if (n.apart) {
        const float2 c = cs[INTERLEAVED ? n.at >> 1 : n.at];
        const float x = (float)n.p, y = (float)n.q;
        n.p = (T)fmaf(x, c.x, -(y * c.y));
        n.q = (T)fmaf(x, c.y, y * c.x);
      }
    } else if (MODE == HALVES) {
      if (n.apart) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float2 c = cs[n.at + i];
          const float x = (float)n.x[i], y = (float)n.y[i];
          n.x[i] = (T)fmaf(x, c.x, -(y * c.y));
          n.y[i] = (T)fmaf(x, c.y, y * c.x);
        }
      }
    } else if (n.part != 2 && n.at < 2 * pairs) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float2 c = cs[n.at / 2 + i];
        const float x = (float)n.x[2 * i], y = (float)n.x[2 * i + 1];
        n.x[2 * i] = (T)fmaf(x, c.x, -(y * c.y));
        n.x[2 * i + 1] = (T)fmaf(x, c.y, y * c.x);
      }
    }
    T* out = n.part == 0 ? a.rotated + (first + n.token) * a.rotated_stride + n.head * dim
                         : static_cast<T*>(n.part == 1 ? a.cache.keys : a.cache.values) + at + n.head * a.cache.head_stride;
    out += n.at;
    if (MODE == ELEMENTS) {
      *out = n.p;
      if (n.apart) out[n.apart] = n.q;
    } else {
      *reinterpret_cast<V8*>(out) = n.x;
      if (n.apart) *reinterpret_cast<V8*>(out + n.apart) = n.y;
    }
  };

  Unit next;
  if ((uint32_t)tid < total) next = fetch(tid);  // (under way while the angles are computed)
  if (tid < here) {
    const int64_t slot = a.slots[first + tid], page = slot < 0 ? -1 : slot / a.cache.page_size;
    place[tid] = page < 0 || page >= a.cache.pages
                     ? -1
                     : page * a.cache.page_stride + (slot - page * a.cache.page_size) * a.cache.slot_stride;
  }
  for (int i = tid; i < here * pairs; i += APP_THREADS) {
    const int t = i / pairs;
    const double turns = (double)a.positions[first + t] * (double)a.frequencies[i - t * pairs] * 0.15915494309189535;
    float c, s;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    turn[i] = {c, s};
  }
  __syncthreads();
  for (uint32_t i = tid; i < total; i += APP_THREADS) {
    const Unit now = next;
    if (i + APP_THREADS < total) next = fetch(i + APP_THREADS);
    finish(now);
  }
}

template <class T>
int run_append(AppendArgs<T> a, int q_heads, bool interleaved, hipStream_t st) {
  const tt_cache& c = a.cache;
  auto vectors = [](const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; };
  const bool aligned = vectors(a.keys, a.key_stride) && vectors(a.values, a.value_stride) &&
                       (q_heads == 0 || (vectors(a.queries, a.query_stride) && vectors(a.rotated, a.rotated_stride)));
  const AppendMode mode = !aligned || a.pairs % (interleaved ? 4 : 8) ? ELEMENTS : interleaved ? NEIGHBOURS : HALVES;
  a.straight = mode == ELEMENTS ? c.dim : c.dim / 8;
  a.turned = mode == ELEMENTS ? c.dim - a.pairs : mode == HALVES ? (c.dim - a.pairs) / 8 : c.dim / 8;
  const int64_t q = (int64_t)q_heads * a.turned, k = (int64_t)c.kv_heads * a.turned, v = (int64_t)c.kv_heads * a.straight;
  a.q_units = (uint32_t)q;
  a.k_units = (uint32_t)k;
  a.units = (uint32_t)(q + k + v);
  // Tokens of a block, once there are blocks enough: of one to three, the number that
  // keeps most of its threads busy.  us with 1, 2, 3 and 8: 30,001 tokens of 336 units
  // 93, 76, 71 and 68 (66, 88, 98 and 95% busy); 20,000 of 448 units 91, -, 98 and 109 (88%).
  auto busy = [&](int64_t n) { return n * a.units * 1000 / ((n * a.units + APP_THREADS - 1) / APP_THREADS * APP_THREADS); };
  int64_t each = 1;
  for (int64_t n = 2; n <= APP_TOKENS && n <= a.tokens / 1024; n++)
    if (busy(n) > busy(each)) each = n;
  if (each * a.units > 65535) each = 65535 / a.units;  // (Division)
  a.each = (int)(each < 1 ? 1 : each);
  a.by_units = Division(a.units);
  a.by_turned = Division(a.turned);
  a.by_straight = Division(a.straight);
  const int64_t blocks = (a.tokens + a.each - 1) / a.each;
  if (blocks > (int64_t)UINT32_MAX / APP_THREADS) return TT_ERR_TOO_LARGE;
  auto* kernel = mode == HALVES       ? append_kernel<T, HALVES, false>
                 : mode == NEIGHBOURS ? append_kernel<T, NEIGHBOURS, true>
                 : interleaved        ? append_kernel<T, ELEMENTS, true>
                                      : append_kernel<T, ELEMENTS, false>;
  return launch(kernel, dim3((uint32_t)blocks), dim3(APP_THREADS), st, a) == hipSuccess ? TT_OK : TT_ERR_HIP;
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int tt_cache_append(const tt_cache* cache, int64_t tokens, const int64_t* slots, const int32_t* positions,
                               const float* frequencies, int32_t pairs, int32_t interleaved, const void* keys,
                               int64_t key_stride, const void* values, int64_t value_stride, int32_t q_heads,
                               const void* queries, int64_t query_stride, void* rotated, int64_t rotated_stride,
                               void* stream) {
  if (!cache) return TT_ERR_NULL_ARG;
  const int bad = check_cache(*cache);
  if (bad == TT_ERR_BAD_ARG) return bad;
  const int64_t width = (int64_t)cache->kv_heads * cache->dim, q_width = (int64_t)q_heads * cache->dim;
  if (tokens < 0 || tokens > INT32_MAX || pairs < 0 || 2 * (int64_t)pairs > cache->dim || key_stride < width ||
      value_stride < width || q_heads < 0 || (q_heads > 0 && (query_stride < q_width || rotated_stride < q_width)) ||
      (q_heads > 0 && rotated == queries && query_stride != rotated_stride))
    return TT_ERR_BAD_ARG;
  if ((q_heads + 2 * (int64_t)cache->kv_heads) * cache->dim > 65535) return TT_ERR_TOO_LARGE;
  if (tokens == 0) return TT_OK;
  if (bad) return bad;
  if (!slots || (pairs > 0 && (!positions || !frequencies)) || !keys || !values || (q_heads > 0 && (!queries || !rotated)))
    return TT_ERR_NULL_ARG;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    AppendArgs<T> a{};
    a.cache = *cache;
    a.tokens = tokens;
    a.slots = slots;
    a.positions = positions;
    a.frequencies = frequencies;
    a.keys = static_cast<const T*>(keys);
    a.values = static_cast<const T*>(values);
    a.queries = static_cast<const T*>(queries);
    a.rotated = static_cast<T*>(rotated);
    a.key_stride = key_stride;
    a.value_stride = value_stride;
    a.query_stride = query_stride;
    a.rotated_stride = rotated_stride;
    a.pairs = pairs;
    return run_append(a, q_heads, interleaved != 0, static_cast<hipStream_t>(stream));
  };
  return cache->type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}
