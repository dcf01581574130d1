// tt_cache_attention: attention of a step's tokens over a paged cache, with an
// optional sliding window and first tokens that stay visible.
#include "tt_cache.h"

namespace tt {
namespace {

struct AttentionArgs {
  tt_cache c;
  tt_attention s;
  int64_t capacity;  // tokens that a request's table has room for
};

// A wave for each token and head: 64 keys at a time, one a lane, a running
// maximum and sum, then the values with a lane's dims.
template <class T>
__global__ __launch_bounds__(64) void attention_kernel(AttentionArgs a) {
  __shared__ float query[TT_MAX_HEAD_DIM];
  const tt_attention& s = a.s;
  const int lane = threadIdx.x, dim = a.c.dim;
  const int64_t t = blockIdx.x / (uint32_t)s.q_heads;
  const int h = (int)(blockIdx.x % (uint32_t)s.q_heads), kv = h / (s.q_heads / a.c.kv_heads);
  // the last request whose first token is at or before t
  int lo = 0, hi = s.n_requests;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (s.offsets[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  if (lo >= s.n_requests || s.offsets[lo] > t) return;
  const int64_t p = (int64_t)s.lengths[lo] - s.offsets[lo + 1] + t;
  const int64_t last = p < a.capacity ? p : a.capacity;
  int64_t begin = s.window ? p - s.window + 1 : 0;
  begin = begin < 0 ? 0 : begin > a.capacity ? a.capacity : begin;
  const T* q = static_cast<const T*>(s.queries) + t * s.query_stride + h * dim;
  for (int d = lane; d < dim; d += 64) query[d] = (float)q[d];
  __syncthreads();
  float m = NEG_INF, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  const float c = s.scale * LOG2E;
  const int32_t* table = s.tables + lo * s.table_stride;
  auto run = [&](int64_t j0, int64_t end) {
    for (; j0 < end; j0 += 64) {
      const int64_t j = j0 + lane;
      const T* value = nullptr;
      float x = NEG_INF;
      if (j < end) {
        const int64_t entry = j / a.c.page_size;
        const int32_t page = entry < s.table_width ? table[entry] : -1;
        if (page < 0 || page >= a.c.pages) {
          x = __builtin_nanf("");
        } else {
          const int64_t at = page * a.c.page_stride + (j - entry * a.c.page_size) * a.c.slot_stride + kv * a.c.head_stride;
          const T* key = static_cast<const T*>(a.c.keys) + at;
          value = static_cast<const T*>(a.c.values) + at;
          x = 0.f;
          for (int d = 0; d < dim; d++) x = fmaf(query[d], (float)key[d], x);
        }
      }
      float top = larger(m, x);
      for (int d = 32; d; d >>= 1) top = larger(top, __shfl_xor(top, d));
      const float base = top == NEG_INF ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f((m - base) * c);
      const float e = __builtin_amdgcn_exp2f((x - base) * c);
      float all = e;
      for (int d = 32; d; d >>= 1) all += __shfl_xor(all, d);
      sum = fmaf(sum, f, all);
      m = top;
      for (int i = 0; i < 4; i++) acc[i] *= f;
      const int n = (int)(end - j0 < 64 ? end - j0 : 64);
      for (int k = 0; k < n; k++) {
        const float pk = __shfl(e, k);
        const T* v = reinterpret_cast<const T*>(__shfl((unsigned long long)value, k));
        for (int i = 0; i < 4; i++)
          if (v && lane + 64 * i < dim) acc[i] = fmaf(pk, (float)v[lane + 64 * i], acc[i]);
      }
    }
  };
  const int64_t front = s.sinks < begin ? s.sinks : begin;
  run(0, front < last + 1 ? front : last + 1);
  run(begin, last + 1);
  T* out = static_cast<T*>(s.out) + t * s.out_stride + h * dim;
  const bool none = m == NEG_INF;
  for (int i = 0; i < 4; i++)
    if (lane + 64 * i < dim) out[lane + 64 * i] = (T)(none ? 0.f : acc[i] / sum);
  if (s.logsums && lane == 0) s.logsums[t * s.q_heads + h] = none ? NEG_INF : fmaf(m, s.scale, logf(sum));
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int64_t tt_cache_attention_workspace(int64_t tokens, int32_t n_requests, int32_t q_heads, int32_t kv_heads,
                                                int32_t dim) {
  if (tokens < 0 || tokens > INT32_MAX || n_requests < 0 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || dim < 8 ||
      dim > TT_MAX_HEAD_DIM || dim % 8)
    return TT_ERR_BAD_ARG;
  return 0;
}

extern "C" int tt_cache_attention(const tt_cache* cache, const tt_attention* step, void* workspace, int64_t workspace_bytes,
                                  void* stream) {
  if (!cache || !step) return TT_ERR_NULL_ARG;
  const tt_attention& s = *step;
  const int bad = check_cache(*cache);
  if (bad == TT_ERR_BAD_ARG) return bad;
  const int64_t need = tt_cache_attention_workspace(s.tokens, s.n_requests, s.q_heads, cache->kv_heads, cache->dim);
  const int64_t width = (int64_t)s.q_heads * cache->dim;
  if (need < 0 || s.table_width < 0 || s.table_stride < s.table_width || s.window < 0 || s.sinks < 0 || !good_scale(s.scale) ||
      s.query_stride < width || s.out_stride < width || (s.out && s.out == s.queries) || workspace_bytes < need ||
      reinterpret_cast<uintptr_t>(workspace) % 256)
    return TT_ERR_BAD_ARG;
  if (s.tokens == 0 || s.n_requests == 0) return TT_OK;
  if (bad) return bad;
  if (!s.offsets || !s.lengths || (s.table_width > 0 && !s.tables) || !s.queries || !s.out || (need && !workspace))
    return TT_ERR_NULL_ARG;
  if (s.tokens > (int64_t)UINT32_MAX / 64 / s.q_heads) return TT_ERR_TOO_LARGE;
  AttentionArgs a{*cache, s, (int64_t)s.table_width * cache->page_size};
  return launch(cache->type == TT_BF16 ? attention_kernel<bf16_t> : attention_kernel<f16_t>,
                dim3((uint32_t)(s.tokens * s.q_heads)), dim3(64), static_cast<hipStream_t>(stream), a) == hipSuccess
             ? TT_OK
             : TT_ERR_HIP;
}
