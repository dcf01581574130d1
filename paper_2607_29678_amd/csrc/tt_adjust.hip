// tt_adjust_logits and its gradient: penalties for repeated tokens, biases and
// masks on rows of stored logits.
//
// One pass: a block takes a run of a row's columns, counts in LDS which of them the
// row's history names (integers: the order does not matter) and which entry of the
// bias list names them last, and then streams the columns through: 16 bytes a load,
// all of a thread's loads under way before the lists are read.
//
// What bounds it: reading and writing the rows.  512 rows of 100,257 in f32 with 2,000
// tokens of history and masks take 83 us, 5.0 TB/s (70 without lists and masks); in bf16
// 72, where the rows alone take 42: every block of 4,096 columns reads the row's whole
// history, and its stores wait for that.  The gradient of 1,536 rows in bf16 takes 108 us
// without a history and 206 with one of 1,000 tokens a row.  Its traffic, with scattered
// reads of the logits of repeated tokens, whose sign the slope depends on, is 745 MB, 150 us
// at a copy's rate.  The rest is the order of a block's work: lists, barrier, vectors and
// logits, stores, with nothing of the next columns under way.  32 rows of 50,257: the host
// call.
#include "tt_scores.h"

namespace tt {
namespace {

constexpr int ADJ_THREADS = 256;
// Vectors of a thread: four, but two where LDS holds a count or a place for each
// column of 16 bits, so that more blocks fit a compute unit (512 rows of 100,257 in
// bf16 with histories of 2,000 tokens 73 us, with four 89; with 100 and biases 76 and 112)
template <class T, bool LISTS>
constexpr int adj_vecs() { return LISTS && sizeof(T) == 2 ? 2 : 4; }

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
// Past the caches, as in the gradient of token scores: loads of any alignment, aligned stores
template <class T>
__device__ __forceinline__ Vec16<T> load_once(const T* p) {
  using U4 = __attribute__((ext_vector_type(4), aligned(2))) uint32_t;
  return __builtin_bit_cast(Vec16<T>, (__attribute__((ext_vector_type(4))) uint32_t)__builtin_nontemporal_load(reinterpret_cast<const U4*>(p)));
}
template <class T>
__device__ __forceinline__ void store_once(T* p, const Vec16<T>& v) {
  using U4 = __attribute__((ext_vector_type(4))) uint32_t;
  __builtin_nontemporal_store(__builtin_bit_cast(U4, v), reinterpret_cast<U4*>(p));
}

__device__ __forceinline__ int64_t held(int64_t x, int64_t most) { return x < 0 ? 0 : x > most ? most : x; }

// A barrier for LDS alone: loads from memory stay under way across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Columns of a block: vectors that are aligned in the output, chunk * ADJ_THREADS *
// VECS being the first; the first block also has the row's columns before them,
// the last one those behind.  LDS holds column j at j - base + N: a count, for the gradient a bit.
template <class T, bool GRAD, bool HISTORY, bool BIAS>
__global__ __launch_bounds__(ADJ_THREADS) void adjust_kernel(AdjustArgs<T> g) {
  constexpr int N = Vec16<T>::N, VECS = adj_vecs<T, !GRAD && (HISTORY || BIAS)>(), COLS = ADJ_THREADS * VECS * N, ROOM = COLS + 2 * N;
  constexpr int WORDS = GRAD ? (ROOM + 31) / 32 + 1 : ROOM;
  __shared__ __align__(16) uint32_t counts[HISTORY ? (WORDS + 3) / 4 * 4 : 4];
  __shared__ __align__(16) uint32_t entries[BIAS ? ROOM : 4];  // place in the bias list, from 1
  __shared__ int named;                                        // whether a list names a column of the block
  const tt_adjustment& a = g.a;
  const int tid = threadIdx.x;
  const uint32_t row32 = blockIdx.x / (uint32_t)g.chunks, chunk = blockIdx.x - row32 * (uint32_t)g.chunks;
  const int64_t row = row32;
  const T* in = g.in + row * g.in_stride;
  const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
  T* out = g.out + row * g.out_stride;
  int head = (int)((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / (int)sizeof(T);
  if (head > a.vocab) head = (int)a.vocab;
  const int vecs = (int)((a.vocab - head) / N), tail = head + vecs * N, v0 = (int)chunk * ADJ_THREADS * VECS;
  const int64_t base = head + (int64_t)v0 * N;
  const bool last = chunk + 1 == (uint32_t)g.chunks;
  // the block's columns (the last block may have none but the tail, which begins up to N before its base)
  const int64_t lo = !chunk ? 0 : last && tail < base ? tail : base, hi = last ? a.vocab : base + COLS;
  // What does not depend on the lists is asked for first; but the gradient asks for
  // its vectors when it knows which logits it needs, so that both come at once.
  Vec16<T> x[VECS];
  auto fetch = [&] {
#pragma unroll
    for (int k = 0; k < VECS; k++)
      if (v0 + k * ADJ_THREADS + tid < vecs) x[k] = load_once(in + base + (int64_t)(k * ADJ_THREADS + tid) * N);
  };
  if (!GRAD || !HISTORY) fetch();
  int64_t h0 = 0, h1 = 0, b0 = 0, b1 = 0;
  if (HISTORY) {
    h0 = held(a.history_offsets[row], a.n_history);
    h1 = held(a.history_offsets[row + 1], a.n_history);
  }
  if (BIAS) {
    b0 = held(a.bias_offsets[row], a.n_biases);
    b1 = held(a.bias_offsets[row + 1], a.n_biases);
  }
  const float rep = HISTORY && a.repetition ? a.repetition[row] : 1.f;
  const float presence = HISTORY && !GRAD && a.presence ? a.presence[row] : 0.f;
  const float frequency = HISTORY && !GRAD && a.frequency ? a.frequency[row] : 0.f;
  const int32_t mask = a.mask_rows ? a.mask_rows[row] : -1;
  const bool no_mask = mask >= a.n_masks;
  const uint32_t* words = mask < 0 || no_mask ? nullptr : a.masks + mask * a.mask_stride;
  uint32_t allowed[VECS];  // bits of each vector
#pragma unroll
  for (int k = 0; k < VECS; k++) {
    const int64_t v = v0 + k * ADJ_THREADS + tid, j = head + v * N;
    allowed[k] = ~0u;
    if (words && v < vecs) {
      const int shift = (int)(j & 31);
      allowed[k] = words[j >> 5] >> shift;
      if (shift > 32 - N) allowed[k] |= words[(j >> 5) + 1] << (32 - shift);
    }
  }
  if (HISTORY || BIAS) {
    if (HISTORY)
      for (int i = tid * 4; i < WORDS; i += ADJ_THREADS * 4) *reinterpret_cast<uint4*>(counts + i) = uint4{0, 0, 0, 0};
    if (BIAS)
      for (int i = tid * 4; i < ROOM; i += ADJ_THREADS * 4) *reinterpret_cast<uint4*>(entries + i) = uint4{0, 0, 0, 0};
    if (tid == 0) named = 0;
    lds_barrier();
    bool mine = false;
    if (HISTORY) {
#pragma unroll 4
      for (int64_t i = h0 + tid; i < h1; i += ADJ_THREADS) {
        const int64_t j = a.history[i];
        if (j >= lo && j < hi) {
          const int at = (int)(j - base) + N;
          if (GRAD) atomicOr(&counts[at >> 5], 1u << (at & 31));
          else atomicAdd(&counts[at], 1u);
          mine = true;
        }
      }
    }
    if (BIAS) {
      for (int64_t i = b0 + tid; i < b1; i += ADJ_THREADS) {
        const int64_t j = a.bias_ids[i];
        if (j >= lo && j < hi) {
          atomicMax(&entries[j - base + N], (uint32_t)(i - b0 + 1));
          mine = true;
        }
      }
    }
    if (mine) named = 1;
    lds_barrier();
  }
  if (GRAD && HISTORY) fetch();
  const bool lists = (HISTORY || BIAS) && named;
  auto penalised = [&](float y, float z, uint32_t n) {
    y = z > 0.f ? y / rep : y * rep;
    return GRAD ? y : y - presence - frequency * (float)n;
  };
  const float nan = __builtin_nanf(""), banned = GRAD ? 0.f : no_mask ? nan : NEG_INF;
  // Vectors that the history names a column of: the gradient needs their logits, all under way at once
  uint32_t hit[VECS];
  Vec16<T> z[VECS];
#pragma unroll
  for (int k = 0; k < VECS; k++) {
    const int v = k * ADJ_THREADS + tid;
    hit[k] = 0;
    if (!HISTORY || !lists || v0 + v >= vecs) continue;
    if (GRAD) {
      hit[k] = counts[(v * N + N) >> 5] >> ((v * N + N) & 31) & ((1u << N) - 1);  // (a vector's bits are in one word)
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const uint4 n = *reinterpret_cast<const uint4*>(counts + v * N + i + N);
        hit[k] |= ((n.x ? 1u : 0u) | (n.y ? 2u : 0u) | (n.z ? 4u : 0u) | (n.w ? 8u : 0u)) << i;
      }
    }
    if (GRAD) hit[k] &= allowed[k];
    if (GRAD && hit[k]) z[k] = load_once(logits + base + (int64_t)v * N);
  }
#pragma unroll
  for (int k = 0; k < VECS; k++) {
    const int v = k * ADJ_THREADS + tid;
    if (v0 + v >= vecs) continue;
    const int64_t j = base + (int64_t)v * N;
    float y[N];
#pragma unroll
    for (int i = 0; i < N; i++) y[i] = (float)x[k].v[i];
    if (HISTORY && hit[k]) {
#pragma unroll
      for (int i = 0; i < N; i++) {
        const float f = penalised(y[i], GRAD ? (float)z[k].v[i] : y[i], GRAD ? 1u : counts[v * N + i + N]);
        y[i] = hit[k] >> i & 1 ? f : y[i];
      }
    }
    if (BIAS && lists) {
#pragma unroll
      for (int i = 0; i < N; i++) {
        const uint32_t e = entries[v * N + i + N];
        if (e) y[i] += a.bias_values[b0 + e - 1];
      }
    }
    Vec16<T> w;
#pragma unroll
    for (int i = 0; i < N; i++) w.v[i] = (T)(allowed[k] >> i & 1 ? no_mask ? nan : y[i] : banned);
    store_once(out + j, w);
  }
  auto edge = [&](int64_t j) {
    const int i = (int)(j - base) + N;
    float y = (float)in[j];
    const uint32_t n = !HISTORY || !lists ? 0 : GRAD ? counts[i >> 5] >> (i & 31) & 1 : counts[i], e = BIAS && lists ? entries[i] : 0;
    if (n) y = penalised(y, GRAD ? (float)logits[j] : y, n);
    if (e) y += a.bias_values[b0 + e - 1];
    out[j] = (T)(words && !(words[j >> 5] >> (j & 31) & 1) ? banned : no_mask ? nan : y);
  };
  if (chunk == 0 && tid < head) edge(tid);
  if (last && tid < (int)(a.vocab - tail)) edge((int64_t)tail + tid);  // (tail + tid may pass 32 bits)
}

template <class T, bool GRAD>
int run_adjust(AdjustArgs<T> g, hipStream_t st) {
  const bool history = g.a.history != nullptr && g.a.n_history > 0, bias = !GRAD && g.a.bias_ids != nullptr && g.a.n_biases > 0;
  const int64_t cols = ADJ_THREADS * Vec16<T>::N * (!GRAD && (history || bias) ? adj_vecs<T, true>() : adj_vecs<T, false>());
  g.chunks = (int)((g.a.vocab + cols - 1) / cols);
  if (g.a.rows > (int64_t)UINT32_MAX / ADJ_THREADS / g.chunks) return TT_ERR_TOO_LARGE;
  auto* kernel = history ? bias ? adjust_kernel<T, GRAD, true, !GRAD> : adjust_kernel<T, GRAD, true, false>
                         : bias ? adjust_kernel<T, GRAD, false, !GRAD> : adjust_kernel<T, GRAD, false, false>;
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
