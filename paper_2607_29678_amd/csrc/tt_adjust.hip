// tt_adjust_logits and its gradient: penalties for repeated tokens, biases and
// masks on rows of stored logits.
//
// One pass: a block takes a run of a row's columns, counts in LDS which of them the
// row's history names (integers: the order does not matter) and which entry of the
// bias list names them last, and then streams the columns through.
#include "tt_scores.h"

namespace tt {
namespace {

constexpr int ADJ_THREADS = 256;

template <class T>
struct AdjustArgs {
  tt_adjustment a;
  const T* in;  // logits, or the gradient with respect to the result
  T* out;
  int64_t in_stride, out_stride;
  int chunks;  // blocks of a row
};

template <class T>
struct Vec16 {
  static constexpr int N = 16 / (int)sizeof(T);
  T v[N];
};

__device__ __forceinline__ int64_t held(int64_t x, int64_t most) { return x < 0 ? 0 : x > most ? most : x; }

template <class T, int COLS, bool GRAD, bool HISTORY, bool BIAS>
__global__ __launch_bounds__(ADJ_THREADS) void adjust_kernel(AdjustArgs<T> g) {
  __shared__ __align__(16) uint32_t counts[HISTORY ? COLS : 4];
  __shared__ __align__(16) uint32_t entries[BIAS ? COLS : 4];  // place in the bias list, from 1
  const tt_adjustment& a = g.a;
  const int tid = threadIdx.x;
  const uint32_t row32 = blockIdx.x / (uint32_t)g.chunks, chunk = blockIdx.x - row32 * (uint32_t)g.chunks;
  const int64_t row = row32, c0 = (int64_t)chunk * COLS;
  const int cols = (int)(a.vocab - c0 < COLS ? a.vocab - c0 : COLS);
  for (int i = tid * 4; i < COLS; i += ADJ_THREADS * 4) {
    if (HISTORY) *reinterpret_cast<uint4*>(counts + i) = uint4{0, 0, 0, 0};
    if (BIAS) *reinterpret_cast<uint4*>(entries + i) = uint4{0, 0, 0, 0};
  }
  if (HISTORY || BIAS) __syncthreads();
  if (HISTORY) {
    const int64_t h0 = held(a.history_offsets[row], a.n_history), h1 = held(a.history_offsets[row + 1], a.n_history);
    for (int64_t i = h0 + tid; i < h1; i += ADJ_THREADS) {
      const int64_t j = a.history[i] - c0;
      if (j >= 0 && j < cols) atomicAdd(&counts[j], 1u);
    }
  }
  int64_t b0 = 0;
  if (BIAS) {
    b0 = held(a.bias_offsets[row], a.n_biases);
    const int64_t b1 = held(a.bias_offsets[row + 1], a.n_biases);
    for (int64_t i = b0 + tid; i < b1; i += ADJ_THREADS) {
      const int64_t j = a.bias_ids[i] - c0;
      if (j >= 0 && j < cols) atomicMax(&entries[j], (uint32_t)(i - b0 + 1));
    }
  }
  const float rep = HISTORY && a.repetition ? a.repetition[row] : 1.f;
  const float presence = HISTORY && !GRAD && a.presence ? a.presence[row] : 0.f;
  const float frequency = HISTORY && !GRAD && a.frequency ? a.frequency[row] : 0.f;
  const int32_t mask = a.mask_rows ? a.mask_rows[row] : -1;
  const bool no_mask = mask >= a.n_masks;
  const uint32_t* words = mask < 0 || no_mask ? nullptr : a.masks + mask * a.mask_stride;
  if (HISTORY || BIAS) __syncthreads();
  const T* in = g.in + row * g.in_stride + c0;
  const T* logits = static_cast<const T*>(a.logits) + row * a.stride + c0;
  T* out = g.out + row * g.out_stride + c0;
  for (int i = tid; i < cols; i += ADJ_THREADS) {
    float y = (float)in[i];
    if (HISTORY) {
      const uint32_t n = counts[i];
      if (n) {
        const float x = GRAD ? (float)logits[i] : y;
        y = x > 0.f ? y / rep : y * rep;
        if (!GRAD) y = y - presence - frequency * (float)n;
      }
    }
    if (BIAS) {
      const uint32_t e = entries[i];
      if (e) y += a.bias_values[b0 + e - 1];
    }
    const int64_t j = c0 + i;
    if (words && !(words[j >> 5] >> (j & 31) & 1)) y = GRAD ? 0.f : NEG_INF;
    if (no_mask) y = __builtin_nanf("");
    out[i] = (T)y;
  }
}

template <class T, bool GRAD>
int run_adjust(AdjustArgs<T> g, hipStream_t st) {
  constexpr int COLS = 4096;
  g.chunks = (int)((g.a.vocab + COLS - 1) / COLS);
  if (g.a.rows > (int64_t)UINT32_MAX / ADJ_THREADS / g.chunks) return TT_ERR_TOO_LARGE;
  const bool history = g.a.history != nullptr && g.a.n_history > 0, bias = !GRAD && g.a.bias_ids != nullptr && g.a.n_biases > 0;
  auto* kernel = history ? bias ? adjust_kernel<T, COLS, GRAD, true, !GRAD> : adjust_kernel<T, COLS, GRAD, true, false>
                         : bias ? adjust_kernel<T, COLS, GRAD, false, !GRAD> : adjust_kernel<T, COLS, GRAD, false, false>;
  return launch(kernel, dim3((uint32_t)(g.a.rows * g.chunks)), dim3(ADJ_THREADS), st, g) == hipSuccess ? TT_OK : TT_ERR_HIP;
}

// What both calls refuse; 1: nothing to do.
int check_adjustment(const tt_adjustment& a, bool gradient) {
  if (a.rows < 0 || a.vocab < 1 || a.vocab > INT32_MAX || !score_type(a.type) || a.stride < a.vocab || a.n_history < 0 ||
      a.n_biases < 0 || a.n_masks < 0 || (a.n_history > 0 && !a.history != !a.history_offsets) ||
      (!a.history_offsets && (a.repetition || a.presence || a.frequency)) ||
      (a.n_biases > 0 && (!a.bias_ids != !a.bias_values || !a.bias_ids != !a.bias_offsets)) ||
      (a.n_masks > 0 && (!a.masks != !a.mask_rows || (a.masks && a.mask_stride < (a.vocab + 31) / 32))))
    return TT_ERR_BAD_ARG;
  if (a.n_biases >= INT64_C(0xFFFFFFFF) || a.n_history >= INT64_C(0xFFFFFFFF)) return TT_ERR_TOO_LARGE;
  if (a.rows == 0) return 1;
  return a.logits || gradient ? TT_OK : TT_ERR_NULL_ARG;
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int tt_adjust_logits(const tt_adjustment* a, void* out, int64_t out_stride, void* stream) {
  if (!a) return TT_ERR_NULL_ARG;
  const int status = check_adjustment(*a, false);
  if (status < 0) return status;
  if (out_stride < a->vocab || (out == a->logits && a->rows && out_stride != a->stride)) return TT_ERR_BAD_ARG;
  if (status == 1) return TT_OK;
  if (!out) return TT_ERR_NULL_ARG;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    return run_adjust<T, false>(AdjustArgs<T>{*a, static_cast<const T*>(a->logits), static_cast<T*>(out), a->stride, out_stride, 0},
                                static_cast<hipStream_t>(stream));
  };
  return a->type == TT_F32 ? go(float{}) : a->type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}

extern "C" int tt_adjust_logits_grad(const tt_adjustment* a, const void* grad_out, int64_t grad_out_stride, void* grad_logits,
                                     int64_t grad_logits_stride, void* stream) {
  if (!a) return TT_ERR_NULL_ARG;
  const int status = check_adjustment(*a, true);
  if (status < 0) return status;
  if (grad_out_stride < a->vocab || grad_logits_stride < a->vocab ||
      (a->rows && ((grad_logits == grad_out && grad_logits_stride != grad_out_stride) || (grad_logits && grad_logits == a->logits))))
    return TT_ERR_BAD_ARG;
  if (status == 1) return TT_OK;
  if (!grad_out || !grad_logits || (a->repetition && !a->logits)) return TT_ERR_NULL_ARG;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    tt_adjustment b = *a;
    if (!b.repetition) b.history = nullptr;  // (the only part of it that the gradient looks at)
    return run_adjust<T, true>(AdjustArgs<T>{b, static_cast<const T*>(grad_out), static_cast<T*>(grad_logits), grad_out_stride,
                                             grad_logits_stride, 0},
                               static_cast<hipStream_t>(stream));
  };
  return a->type == TT_F32 ? go(float{}) : a->type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}
