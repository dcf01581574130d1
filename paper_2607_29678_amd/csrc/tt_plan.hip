// tt_step_plan: offsets, positions, cache slots, page tables and next-token
// targets of a serving step, from the requests' lengths.
//
// The work is a pair of running sums over the requests (new tokens, new pages)
// and then one independent item per token, per new page and per request.  One
// launch does all of it: every block sums the lengths again for itself (8-12
// bytes a request out of the L2) and takes its share of the items, so that no
// block waits for another and nothing has to be cleared between calls.  A
// second launch, or a wait between blocks, would cost more than the repeated
// sums up to the few thousand requests that a step has.
//
// What bounds it is latency: a chain of two loads, the sums and a search in LDS.
// 96 requests of one token take 6.6 us, 2,048 of them 9.2, 301 of
// 16,381 tokens 7.9, 64 of 420,000 tokens 8.7: 24 bytes written and 4 read a
// token, 11.8 MB, at 1.3 TB/s.
//
// Page numbers of new pages are read from the stack of free pages, not from
// the table that some other block may or may not have written yet.
#include "../../include/toktier_model.h"
#include "tt_internal.h"

namespace tt {
namespace {

constexpr int PLAN_THREADS = 512;
constexpr int PLAN_EACH = 4;                              // requests summed by a thread
constexpr int PLAN_CHUNK = PLAN_THREADS * PLAN_EACH;      // requests whose sums are in LDS at once
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int64_t PLAN_TOKENS = 4 * PLAN_THREADS;         // tokens of a block
constexpr int64_t PLAN_MAX_BLOCKS = 1024;

struct PlanShared {
  int32_t tok[PLAN_CHUNK + 1];  // first token of each request, from the chunk's first
  int32_t page[PLAN_CHUNK + 1]; // first new page of each request, from the chunk's first
  int32_t cached[PLAN_CHUNK], held[PLAN_CHUNK];
  int64_t sums[PLAN_WAVES][2];
  int32_t bad;
};

struct Request {
  int64_t fresh, take;  // new tokens, new pages
  int32_t held;         // pages before the step
  bool bad;
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int32_t page_size) {
  // lengths below 2^32: one 32-bit division
  return tokens <= 0 ? 0 : (int64_t)(((uint32_t)tokens - 1u) / (uint32_t)page_size) + 1;
}

__device__ __forceinline__ Request request_of(const tt_step& s, int64_t c, int64_t n, int64_t h) {
  Request q;
  const int64_t held = s.held ? h : pages_of(c, s.page_size);
  const int64_t need = pages_of(c + n, s.page_size);
  q.bad = c < 0 || n < 0 || held < 0 || c + n > INT32_MAX || need > s.table_width || held > s.table_width;
  q.fresh = q.bad ? 0 : n;
  q.take = q.bad || need <= held ? 0 : need - held;
  q.held = held < 0 ? 0 : (int32_t)(held > INT32_MAX ? INT32_MAX : held);
  return q;
}

// Running sums of one chunk of requests into LDS (they are used only once the
// totals are known to fit 32 bits); returns the chunk's totals.
__device__ void sum_chunk(const tt_step& s, int64_t first, int n, PlanShared& sh, int64_t& toks, int64_t& pages) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t a = 0, b = 0;
  int32_t fresh[PLAN_EACH], take[PLAN_EACH];
  bool bad = false;
  // every length is asked for before the first is used
  int32_t lc[PLAN_EACH], ln[PLAN_EACH], lh[PLAN_EACH];
#pragma unroll
  for (int i = 0; i < PLAN_EACH; i++) {
    const int r = tid * PLAN_EACH + i;
    lc[i] = ln[i] = lh[i] = 0;
    if (r < n) {
      lc[i] = s.cached[first + r];
      ln[i] = s.fresh[first + r];
      if (s.held) lh[i] = s.held[first + r];
    }
  }
#pragma unroll
  for (int i = 0; i < PLAN_EACH; i++) {
    const int r = tid * PLAN_EACH + i;
    fresh[i] = take[i] = 0;
    if (r < n) {
      const Request q = request_of(s, lc[i], ln[i], lh[i]);
      bad |= q.bad;
      fresh[i] = (int32_t)q.fresh;
      take[i] = (int32_t)q.take;
      sh.cached[r] = lc[i];
      sh.held[r] = q.held;
    }
    a += fresh[i];
    b += take[i];
  }
  int64_t ia = a, ib = b;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t pa = __shfl_up(ia, d), pb = __shfl_up(ib, d);
    if (lane >= d) {
      ia += pa;
      ib += pb;
    }
  }
  if (lane == 63) {
    sh.sums[wave][0] = ia;
    sh.sums[wave][1] = ib;
  }
  if (bad) sh.bad = 1;
  __syncthreads();
  int64_t ba = 0, bb = 0;
  toks = pages = 0;
#pragma unroll
  for (int w = 0; w < PLAN_WAVES; w++) {
    if (w < wave) {
      ba += sh.sums[w][0];
      bb += sh.sums[w][1];
    }
    toks += sh.sums[w][0];
    pages += sh.sums[w][1];
  }
  ba += ia - a;
  bb += ib - b;
#pragma unroll
  for (int i = 0; i < PLAN_EACH; i++) {
    const int r = tid * PLAN_EACH + i;
    if (r < n) {
      sh.tok[r] = (int32_t)ba;
      sh.page[r] = (int32_t)bb;
    }
    ba += fresh[i];
    bb += take[i];
  }
  if (tid == 0) {
    sh.tok[n] = (int32_t)toks;
    sh.page[n] = (int32_t)pages;
  }
  __syncthreads();
}

// The last request of the chunk whose sum is <= x, where x < sums[n]: requests
// without items share their sum with the next one and are passed over.
__device__ __forceinline__ int owner_of(const int32_t* sums, int n, int32_t x) {
  int lo = 0, hi = n;  // sums[lo] <= x < sums[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Token x of the chunk, which is request r's.
struct Token {
  int64_t slot;
  int32_t pos;
};
__device__ __forceinline__ Token token_of(const tt_step& s, const PlanShared& sh, int64_t first, int64_t base_p,
                                          int64_t count, int r, int32_t x) {
  const int32_t pos = sh.cached[r] + (x - sh.tok[r]), entry = (int32_t)((uint32_t)pos / (uint32_t)s.page_size);
  const int32_t held = sh.held[r];
  // (one load either way: of the table, or of the stack where the page is new)
  const int32_t* from = entry < held ? s.tables + (first + r) * s.table_stride + entry
                                     : s.free_pages + (count - 1 - (base_p + sh.page[r] + (entry - held)));
  return {(int64_t)*from * s.page_size + (pos - entry * s.page_size), pos};
}

// ONE: all requests are in one chunk, and the per-token arrays are aligned to 16
// bytes; a thread then stores four tokens at a time.  Without it lengths are summed
// twice and tokens searched for and stored one by one: 2,049 requests of one
// token take 17.3 us, 4,000 21.5; with one array off its alignment 301 requests of
// 16,381 tokens take 12.0, 64 of 420,000 12.0.
template <bool ONE>
__global__ __launch_bounds__(PLAN_THREADS) void plan_kernel(tt_step s) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x;
  const int64_t n = s.n_requests, blocks = gridDim.x, block = blockIdx.x;
  const int64_t count = *s.free_count;
  if (tid == 0) sh.bad = 0;
  __syncthreads();

  int64_t toks = 0, pages = 0, ct = 0, cp = 0;
  for (int64_t first = 0; first < n; first += PLAN_CHUNK) {
    const int m = (int)(n - first < PLAN_CHUNK ? n - first : PLAN_CHUNK);
    sum_chunk(s, first, m, sh, ct, cp);
    toks += ct;
    pages += cp;
    if (!ONE) __syncthreads();
  }
  const bool bad = sh.bad || toks > s.max_tokens || count < 0 || count > s.n_free;
  const bool fail = bad || pages > count;
  const int64_t end = fail ? 0 : toks;
  if (block == 0 && tid == 0) {
    s.result[0] = bad ? TT_ERR_BAD_ARG : pages > count ? TT_ERR_OOM : toks;
    s.result[1] = fail ? count : count - pages;
    s.offsets[n] = (int32_t)end;
  }

  // this block's shares of the tokens and of the new pages
  const int64_t t0 = PLAN_TOKENS * block, t1 = s.max_tokens;
  const int64_t p0 = fail ? 0 : pages * block / blocks, p1 = fail ? 0 : pages * (block + 1) / blocks;

  int64_t base_t = 0, base_p = 0;
  for (int64_t first = 0; first < n; first += PLAN_CHUNK) {
    const int m = (int)(n - first < PLAN_CHUNK ? n - first : PLAN_CHUNK);
    if (!ONE) sum_chunk(s, first, m, sh, ct, cp);  // (a single chunk's sums are still in LDS)
    if (!ONE && !fail) {
      for (int64_t u = t0; u < t1; u += PLAN_TOKENS * blocks) {
        const int64_t a = u > base_t ? u : base_t, stop = u + PLAN_TOKENS < base_t + ct ? u + PLAN_TOKENS : base_t + ct;
        for (int64_t t = a + tid; t < stop; t += PLAN_THREADS) {
          const int32_t x = (int32_t)(t - base_t);
          const int r = owner_of(sh.tok, m, x);
          const Token y = token_of(s, sh, first, base_p, count, r, x);
          s.slots[t] = y.slot;
          s.positions[t] = y.pos;
          s.requests[t] = (int32_t)(first + r);
          if (s.targets) s.targets[t] = x + 1 < sh.tok[r + 1] ? s.ids[t + 1] : -1;
        }
      }
    }
    if (!fail) {
      const int64_t pa = p0 > base_p ? p0 : base_p, pb = p1 < base_p + cp ? p1 : base_p + cp;
      for (int64_t p = pa + tid; p < pb; p += PLAN_THREADS) {
        const int32_t x = (int32_t)(p - base_p);
        const int r = owner_of(sh.page, m, x);
        s.tables[(first + r) * s.table_stride + sh.held[r] + (x - sh.page[r])] = s.free_pages[count - 1 - p];
      }
    }
    for (int64_t r = block * PLAN_THREADS + tid; r < m; r += blocks * PLAN_THREADS) {
      const int32_t news = sh.tok[r + 1] - sh.tok[r], taken = sh.page[r + 1] - sh.page[r];
      s.offsets[first + r] = fail ? 0 : (int32_t)(base_t + sh.tok[r]);
      s.lengths[first + r] = fail ? 0 : sh.cached[r] + news;
      s.pages[first + r] = sh.held[r] + (fail ? 0 : taken);
    }
    base_t += ct;
    base_p += cp;
    if (!ONE) __syncthreads();
  }
  if (ONE) {
    using I4 = __attribute__((ext_vector_type(4))) int32_t;
    using L2 = __attribute__((ext_vector_type(2))) int64_t;
    for (int64_t u = t0 + 4 * tid; u < t1; u += PLAN_TOKENS * blocks) {
      I4 pos = {0, 0, 0, 0}, req = {-1, -1, -1, -1}, target = {-1, -1, -1, -1};
      int64_t slot[4] = {-1, -1, -1, -1};
      if (u < end) {
        int r = owner_of(sh.tok, (int)n, (int32_t)u);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int32_t x = (int32_t)u + i;
          if (x >= end) break;
          while (x >= sh.tok[r + 1]) r++;  // (ends: x is below the last sum)
          const Token y = token_of(s, sh, 0, 0, count, r, x);
          slot[i] = y.slot;
          pos[i] = y.pos;
          req[i] = r;
          if (s.targets && x + 1 < sh.tok[r + 1]) target[i] = s.ids[x + 1];
        }
      }
      if (u + 4 <= t1) {
        *reinterpret_cast<L2*>(s.slots + u) = L2{slot[0], slot[1]};
        *reinterpret_cast<L2*>(s.slots + u + 2) = L2{slot[2], slot[3]};
        *reinterpret_cast<I4*>(s.positions + u) = pos;
        *reinterpret_cast<I4*>(s.requests + u) = req;
        if (s.targets) *reinterpret_cast<I4*>(s.targets + u) = target;
      } else {
        for (int i = 0; u + i < t1; i++) {
          s.slots[u + i] = i == 0 ? slot[0] : i == 1 ? slot[1] : slot[2];
          s.positions[u + i] = i == 0 ? pos[0] : i == 1 ? pos[1] : pos[2];
          s.requests[u + i] = i == 0 ? req[0] : i == 1 ? req[1] : req[2];
          if (s.targets) s.targets[u + i] = i == 0 ? target[0] : i == 1 ? target[1] : target[2];
        }
      }
    }
  } else {
    for (int64_t u = t0; u < t1; u += PLAN_TOKENS * blocks)
      for (int64_t t = (u > end ? u : end) + tid; t < u + PLAN_TOKENS && t < t1; t += PLAN_THREADS) {
        s.slots[t] = -1;
        s.positions[t] = 0;
        s.requests[t] = -1;
        if (s.targets) s.targets[t] = -1;
      }
  }
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int32_t tt_current_device(void) {
  int device = 0;
  return hipGetDevice(&device) == hipSuccess ? device : TT_ERR_HIP;
}

extern "C" int tt_step_plan(const tt_step* step, void* stream) {
  if (!step) return TT_ERR_NULL_ARG;
  const tt_step& s = *step;
  if (s.n_requests < 0 || s.page_size < 1 || s.table_width < 0 || s.table_stride < s.table_width || s.max_tokens < 0 ||
      s.max_tokens > INT32_MAX || s.n_free < 0 || s.n_free > INT32_MAX || !s.ids != !s.targets)
    return TT_ERR_BAD_ARG;
  if (!s.offsets || !s.result || !s.free_count || (s.n_free > 0 && !s.free_pages) ||
      (s.n_requests > 0 && (!s.cached || !s.fresh || !s.lengths || !s.pages || (s.table_width > 0 && !s.tables))) ||
      (s.max_tokens > 0 && (!s.slots || !s.positions || !s.requests)))
    return TT_ERR_NULL_ARG;
  // blocks read these while others already write the outputs
  if (s.result == s.free_count || s.result + 1 == s.free_count ||
      (s.n_requests > 0 && (s.pages == s.held || s.lengths == s.cached || s.lengths == s.fresh)) ||
      (s.max_tokens > 0 && s.ids && s.targets == s.ids))
    return TT_ERR_BAD_ARG;
  int64_t blocks = (s.max_tokens + PLAN_TOKENS - 1) / PLAN_TOKENS;
  if (blocks > PLAN_MAX_BLOCKS) blocks = PLAN_MAX_BLOCKS;
  if (blocks < 1) blocks = 1;
  auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
  const bool one = s.n_requests <= PLAN_CHUNK && aligned(s.slots) && aligned(s.positions) && aligned(s.requests) &&
                   aligned(s.targets);
  return launch(one ? plan_kernel<true> : plan_kernel<false>, dim3((uint32_t)blocks), dim3(PLAN_THREADS),
                static_cast<hipStream_t>(stream), s) == hipSuccess
             ? TT_OK
             : TT_ERR_HIP;
}
