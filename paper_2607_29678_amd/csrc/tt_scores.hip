// tt_token_scores and its gradient: log probabilities of given tokens, entropy
// and the top alternatives of rows of stored logits.
//
// Forward: one pass over the logits.  Every thread keeps a running maximum and
// the two sums of a softmax (sum e and sum e d, which gives the entropy) of the
// entries that it strides over.  The running maxima also find the alternatives:
// the n_alt-th largest of 128 groups' maxima is a lower bound of the n_alt-th
// largest logit, so entries below it are passed over, one comparison for each
// 16-byte vector, and the few vectors that reach it are kept in LDS; what they
// hold above the last bound is ordered at the end.
#include "tt_scores.h"

namespace tt {
namespace {

constexpr int SC_THREADS = 256;
constexpr int SC_VECS = 192;       // 16-byte vectors with a possible alternative that a wave keeps in LDS
constexpr int SC_CANDS = 512;      // candidates that are ordered there
// Many short rows: a wave takes a row, and the reductions at a row's end are one
// wave's.  us with a wave and with a block a row, bf16, without and with 20
// alternatives: 8,192 rows of 8,449 30 / 47 and 46 / 65, of 16,384 48 / 59 and
// 68 / 80, 4,096 of 32,000 44 / 51 and 60 / 65 (the bound leaves that to blocks).
constexpr int64_t WAVE_ROWS = 2048, WAVE_VOCAB = 16384;

// Parts of a row that several blocks take.  A part has a block's start and end
// again and the parts are joined by a second launch, some 4 us in all, so that
// only long rows gain, and the longer they are the more rows there are to fill
// the chip without; finding alternatives takes longer and gains earlier.  us whole
// and in parts (bf16 unless said):
//   rows x vocab     scores alone       with 8 alternatives
//      8 x  32,000     7.5 /  8.0          13.3 / 11.4 (11 parts)
//      8 x 100,257    13.9 /  7.9          24.3 / 12.4 (32)
//     64 x 100,257    14.2 / 10.7          24.5 / 15.9 (16)
//    200 x 100,257    15.6 / 17.1          25.4 / 20.6 (5; f32 37.3 / 23.4)
//    400 x 100,257    21.7 / 25.8          31.6 / 31.0 (2; f32 44.4 / 36.9)
//    501 x   8,449     7.7 / 12.0          10.6 / 15.4 (2)
//    700 x 100,257    30.3 / 35.6          38.0 / 40.8 (2)
// 64 parts cost more to join than they save (8 rows of 256,000: 18.1 against 12.6).
constexpr int SC_MAX_SPLITS = 32;
constexpr int64_t SC_SPLIT_COLS = 2800;   // fewest columns of a part
constexpr int64_t SC_BLOCKS = 1024;       // blocks that fill the chip (4 per compute unit)
int scores_splits(int64_t rows, int64_t vocab, int32_t n_alt) {
  const int64_t full = rows < 100 ? 100 : rows;
  if (rows <= 0 || rows > (n_alt ? 512 : 256) || vocab < (n_alt ? 24576 : 40960) * full / 100) return 1;
  int64_t n = SC_BLOCKS / rows;
  if (n > vocab / SC_SPLIT_COLS) n = vocab / SC_SPLIT_COLS;
  return (int)(n > SC_MAX_SPLITS ? SC_MAX_SPLITS : n);
}
// Parts that a workspace has room for: a bound of the above that does not follow
// its figures, so that callers' sizes stay right when those change.
int64_t scores_room(int64_t rows, int64_t vocab) {
  if (rows <= 0 || rows >= SC_BLOCKS) return 0;
  int64_t n = SC_BLOCKS / rows < 64 ? SC_BLOCKS / rows : 64;
  if (n > vocab / 2048) n = vocab / 2048;
  return n > 1 ? rows * n : 0;
}
static_assert(SC_MAX_SPLITS <= 64 && SC_SPLIT_COLS >= 2048, "scores_room");

// A part's statistics and its alternatives in descending order (0: none)
struct PartHead {
  Stats st;
  float given;  // logit of the given token, in the part that holds it
};
__host__ __device__ inline int64_t part_bytes(int n_alt) { return (int64_t)sizeof(PartHead) + 8 * (int64_t)n_alt; }

// Order of alternatives: the larger logit, then the lower ID.  Never 0.
__device__ __forceinline__ uint64_t alt_key(float x, uint32_t id) {
  const uint32_t b = __float_as_uint(x + 0.f);  // (-0 equals 0)
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (0xFFFFFFFFu - id);
}
__device__ __forceinline__ float alt_value(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ int32_t alt_id(uint64_t key) { return (int32_t)(0xFFFFFFFFu - (uint32_t)key); }

template <class T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  T v[N];
};
template <class T>
__device__ __forceinline__ Vec<T> load_vec(const T* p) {  // of any alignment
  using U4 = __attribute__((ext_vector_type(4), aligned(2))) uint32_t;
  return __builtin_bit_cast(Vec<T>, (__attribute__((ext_vector_type(4))) uint32_t)__builtin_nontemporal_load(reinterpret_cast<const U4*>(p)));
}
template <class T>
__device__ __forceinline__ void store_vec_once(T* p, const Vec<T>& v) {
  using U4 = __attribute__((ext_vector_type(4))) uint32_t;
  __builtin_nontemporal_store(__builtin_bit_cast(U4, v), reinterpret_cast<U4*>(p));
}
// Aligned, and not kept in the caches: a row is read once (7.1 TB/s on reads of
// 4 GiB against 6.3 with ordinary loads).
template <class T>
__device__ __forceinline__ Vec<T> load_vec_once(const T* p) {
  using U4 = __attribute__((ext_vector_type(4))) uint32_t;
  return __builtin_bit_cast(Vec<T>, __builtin_nontemporal_load(reinterpret_cast<const U4*>(p)));
}

// A thread's entries of columns [0, n) of p: 16-byte vectors of the aligned
// middle, strided over the block, and one entry of the head or the tail each.
template <class T>
struct Span {
  const T* p;
  int64_t n, head, vecs, tail;
  __device__ Span(const T* p_, int64_t n_) : p(p_), n(n_) {
    constexpr int N = Vec<T>::N;
    head = (int64_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int64_t)sizeof(T);
    if (head > n) head = n;
    vecs = (n - head) / N;
    tail = head + vecs * N;
  }
};

template <class T>
struct ScoreArgs {
  const T* logits;
  int64_t rows, vocab, stride;
  float scale;
  const int32_t* targets;
  float *logprobs, *stats, *entropy;
  int n_alt;
  int32_t* alt_ids;
  float* alt_logprobs;
  uint8_t* parts;  // workspace: rows * splits parts
  int splits;
  int64_t per_part;  // columns of a part
};

template <int THREADS>
struct SumShared {
  Stats st[THREADS / 64];
};
template <int THREADS>
struct ScoreShared : SumShared<THREADS> {
  float maxima[THREADS];
  alignas(16) uint8_t vec[THREADS / 64][SC_VECS][16];
  uint32_t vec_at[THREADS / 64][SC_VECS];
  alignas(16) uint64_t cands[SC_CANDS];
  uint64_t best[TT_MAX_ALTERNATIVES];
  float bound;
  int n_vecs[THREADS / 64], n_cands;
};

__device__ __forceinline__ uint32_t ordered(float x) { return (uint32_t)(alt_key(x, 0) >> 32); }

// A value that at least n_alt entries seen so far reach, from the threads'
// running maxima: the n_alt-th largest of 128 maxima of two threads each (of 64
// threads: of their own), found bit by bit (in order of values, down to LOWEST) in one wave.  -inf where fewer
// than n_alt of them are larger.
template <uint32_t LOWEST, int THREADS>
__device__ __forceinline__ float bound_of(float mine, int n_alt, ScoreShared<THREADS>& sh) {
  const int tid = threadIdx.x;
  sh.maxima[tid] = mine;
  __syncthreads();
  if (tid < 64) {
    static_assert(THREADS == 64 || THREADS == 256, "one or four maxima a lane");
    uint32_t a = ordered(sh.maxima[tid]), b = 0;
    if constexpr (THREADS == 256) {
      a = ordered(fmaxf(sh.maxima[tid], sh.maxima[tid + 64]));
      b = ordered(fmaxf(sh.maxima[tid + 128], sh.maxima[tid + 192]));
    }
    uint32_t key = 0;
#pragma unroll
    for (uint32_t bit = 0x80000000u; bit >= LOWEST; bit >>= 1) {
      const uint32_t want = key | bit;
      const int n = __popcll(__ballot(a >= want)) + __popcll(__ballot(b >= want));
      if (n >= n_alt) key = want;
    }
    if (tid == 0) sh.bound = key <= 0x007FFFFFu ? NEG_INF : alt_value((uint64_t)key << 32);
  }
  __syncthreads();
  return sh.bound;
}

// How many of the n keys are better; zeros up to a multiple of 8 follow them.
__device__ __forceinline__ int better(const uint64_t* keys, int n, uint64_t key) {
  using U64x2 = __attribute__((ext_vector_type(2))) uint64_t;
  int count = 0;
  for (int j = 0; j < n; j += 8) {
    U64x2 q[4];
#pragma unroll
    for (int i = 0; i < 4; i++) q[i] = *reinterpret_cast<const U64x2*>(keys + j + 2 * i);
#pragma unroll
    for (int i = 0; i < 4; i++) count += (q[i][0] > key) + (q[i][1] > key);
  }
  return count;
}

// Orders the n candidates by counting the better ones (keys are distinct).
template <int THREADS>
__device__ __forceinline__ void order_candidates(int n, int n_alt, ScoreShared<THREADS>& sh) {
  if (threadIdx.x < 8 && n + threadIdx.x < SC_CANDS) sh.cands[n + threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const uint64_t k = sh.cands[i];
    const int place = better(sh.cands, n, k);
    if (place < n_alt) sh.best[place] = k;
  }
}

// The alternatives of a span whose candidates did not fit: `mine` is the
// thread's largest entry, and bound_of() now speaks for the whole span.
//  - Entries above the bound are collected again; if that falls short of n_alt,
//    equal entries (masks of a finite value) follow in order of their IDs.
//  - Should even the entries above it not fit, places are filled one by one.
template <class T, int THREADS>
__device__ __forceinline__ void find_again(const Span<T>& sp, uint32_t first, int n_alt, float mine,
                                           ScoreShared<THREADS>& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float bound = bound_of<1u, THREADS>(mine, n_alt, sh);
  if (tid == 0) sh.n_cands = 0;
  __syncthreads();
  for (int64_t j = tid; j < sp.n; j += THREADS) {
    const float x = (float)sp.p[j];
    if (x > bound) {
      const int at = atomicAdd(&sh.n_cands, 1);
      if (at < SC_CANDS) sh.cands[at] = alt_key(x, first + (uint32_t)j);
    }
  }
  __syncthreads();
  const int n = sh.n_cands;
  if (n <= SC_CANDS) {
    order_candidates(n, n_alt, sh);
    int have = n;
    for (int64_t j0 = 0; j0 < sp.n && have < n_alt && bound > NEG_INF; j0 += THREADS) {
      const int64_t j = j0 + tid;
      const bool tie = j < sp.n && (float)sp.p[j] == bound;
      const uint64_t votes = __ballot(tie);
      __syncthreads();
      if (lane == 0) sh.maxima[wave] = (float)__popcll(votes);
      __syncthreads();
      int at = have + __popcll(votes & ((1ull << lane) - 1ull));
      for (int w = 0; w < THREADS / 64; w++) {
        if (w < wave) at += (int)sh.maxima[w];
        have += (int)sh.maxima[w];
      }
      if (tie && at < n_alt) sh.best[at] = alt_key(bound, first + (uint32_t)j);
    }
    __syncthreads();
    return;
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < n_alt; r++) {
    uint64_t k = 0;  // the thread's best key below the last one
    for (int64_t j = tid; j < sp.n; j += THREADS) {
      const uint64_t q = alt_key((float)sp.p[j], first + (uint32_t)j);
      if (q < last && q > k) k = q;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
      const uint64_t o = __shfl_xor(k, d);
      k = o > k ? o : k;
    }
    __syncthreads();
    if (lane == 0) sh.cands[wave] = k;
    __syncthreads();
    last = sh.cands[0];
    for (int w = 1; w < THREADS / 64; w++) last = sh.cands[w] > last ? sh.cands[w] : last;
    if (tid == 0) sh.best[r] = last;
  }
  __syncthreads();
}

// One part of one row per block (or wave).  2,048 rows of 100,257 in bf16 take
// 70-73 us, 5.7 TB/s, and in f32 135, 6.1: bound by reading the logits.  With 20
// alternatives they take 82-87, 4.9 TB/s: a wave's candidates come on top.  8 rows
// with 5 alternatives in 17 parts take 7 us and 4-5 to join them: latency.  Without
// alternatives eight waves a SIMD keep more loads under way (76 us with the 71
// registers that the compiler takes of its own accord).
template <class T, bool ALT, int THREADS>
__global__ __launch_bounds__(THREADS, ALT ? 1 : 8) void scores_kernel(ScoreArgs<T> a) {
  __shared__ std::conditional_t<ALT, ScoreShared<THREADS>, SumShared<THREADS>> sh;
  constexpr int N = Vec<T>::N, U = ALT ? 2 : 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t row32 = blockIdx.x / (uint32_t)a.splits, part = blockIdx.x - row32 * (uint32_t)a.splits;
  const int64_t row = row32;
  const int64_t c0 = a.per_part * part, c1 = c0 + a.per_part < a.vocab ? c0 + a.per_part : a.vocab;
  const T* p = a.logits + row * a.stride + c0;
  const Span<T> sp(p, c1 - c0);
  const float c = a.scale * LOG2E;
  const uint32_t first = (uint32_t)c0;
  if constexpr (ALT) {
    if (tid < a.n_alt) sh.best[tid] = 0;
    if (tid == 0) sh.n_cands = 0;
  }

  // the given token's logit (loaded ahead of the sums)
  const int32_t target = a.targets ? a.targets[row] : -1;
  const bool holds_given = target >= c0 && target < c1;
  float x_given = holds_given ? (float)p[target - c0] : 0.f;

  // The row's largest entry stays out of the sums (Stats).  That is looked after
  // only in the steps in which the wave's largest entry, `most`, rises, some log of
  // their number: each lane then leaves out its largest so far.
  Stats st = empty_stats();
  float held = NEG_INF, most = NEG_INF, bound = NEG_INF;
  // U vectors at a time share one move of the maximum.  The loop runs equally
  // often in every thread: it holds barriers.  The vectors of the next step are
  // under way while the last ones are summed; in the last step a thread repeats
  // the last vector where it has none, and takes it for -inf.
  constexpr int STEP = U * THREADS;
  const int vecs = (int)sp.vecs, steps = (vecs + STEP - 1) / STEP;
  const T* body = p + sp.head;
  Vec<T> y[U];
  auto fetch = [&](int step) {
#pragma unroll
    for (int k = 0; k < U; k++) {
      const int v = step * STEP + k * THREADS + tid;
      y[k] = load_vec_once(body + (int64_t)(v < vecs ? v : vecs - 1) * N);
    }
  };
  int n_vecs = 0;  // vectors that this wave has kept
  auto take = [&](int step, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int v = step * STEP + tid, here = vecs - step * STEP;  // vectors of this step
    float x[U][N], top[U], m = st.m;
#pragma unroll
    for (int k = 0; k < U; k++)
#pragma unroll
      for (int i = 0; i < N; i++) x[k][i] = (float)y[k].v[i];
    if (step + 1 < steps) fetch(step + 1);
#pragma unroll
    for (int k = 0; k < U; k++) {
      top[k] = NEG_INF;
      if (!WHOLE && k * THREADS >= here) continue;  // (the same for every thread)
      if (!WHOLE && k * THREADS + tid >= here) {
#pragma unroll
        for (int i = 0; i < N; i++) x[k][i] = NEG_INF;
      }
      top[k] = x[k][0];
#pragma unroll
      for (int i = 1; i < N; i++) top[k] = larger(top[k], x[k][i]);
      m = larger(m, top[k]);
    }
    lower(st, m, c);
    const Reference ref = reference(m, c);
    auto sums = [&](auto plain, auto rises) {
#pragma unroll
      for (int k = 0; k < U; k++) {
        if (!WHOLE && k * THREADS >= here) continue;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          if (decltype(rises)::value) {
            add_two<decltype(plain)::value>(st, held, x[k][i], x[k][i + 1], ref, c);
          } else {
            add_entry<decltype(plain)::value>(st, x[k][i], ref, c);
            add_entry<decltype(plain)::value>(st, x[k][i + 1], ref, c);
          }
        }
      }
    };
    const uint64_t above = __ballot(m > most);
    for (uint64_t v = above; v; v = __ballot(m > most))
      most = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m), __builtin_ctzll(v)));
    if (__ballot(!is_plain(m, c))) sums(std::false_type{}, std::true_type{});
    else if (above) sums(std::true_type{}, std::true_type{});
    else sums(std::true_type{}, std::false_type{});
    if constexpr (ALT) {
      if ((step & (step + 1)) == 0) bound = bound_of<0x10000u, THREADS>(st.m, a.n_alt, sh);  // after 1, 2, 4, 8 ... steps
#pragma unroll
      for (int k = 0; k < U; k++) {
        const bool mine = top[k] >= bound && top[k] > NEG_INF;
        const uint64_t votes = __ballot(mine);
        if (votes == 0) continue;
        const int at = n_vecs + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(votes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)votes, 0));
        if (mine && at < SC_VECS) {
          Vec<T> z;
#pragma unroll
          for (int i = 0; i < N; i++) z.v[i] = (T)x[k][i];
          __builtin_memcpy(sh.vec[wave][at], &z, 16);
          sh.vec_at[wave][at] = (uint32_t)(sp.head + (int64_t)(v + k * THREADS) * N);
        }
        n_vecs += __popcll(votes);
      }
    }
  };
  if (steps > 0) fetch(0);
  x_given = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x_given)));  // (no vector register in the loop)
  for (int step = 0; step + 1 < steps; step++) take(step, std::true_type{});
  if (steps > 0) take(steps - 1, std::false_type{});
  auto edge = [&](int64_t j) {
    const float x = (float)p[j], m = larger(st.m, x), less = smaller(held, x);
    lower(st, m, c);
    add_entry<false>(st, less, reference(m, c), c);
    held = larger(held, x);
  };
  if (tid < sp.head) edge(tid);
  if (sp.tail + tid < sp.n) edge(sp.tail + tid);
  const float mine = st.m;
  st = wave_join(st, held, c);
  if constexpr (THREADS > 64) {
    if (lane == 0) sh.st[wave] = st;
    __syncthreads();
    st = sh.st[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; w++) st = join(st, sh.st[w], c);
  }

  if constexpr (ALT) {
    if (steps == 0) bound = bound_of<0x10000u, THREADS>(mine, a.n_alt, sh);
    auto keep = [&](float x, uint32_t j) {
      if (x >= bound && x > NEG_INF) {
        const int at = atomicAdd(&sh.n_cands, 1);
        if (at < SC_CANDS) sh.cands[at] = alt_key(x, first + j);
      }
    };
    // every wave looks through what it kept itself
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const bool all_kept = n_vecs <= SC_VECS;
    for (int i = lane; all_kept && i < n_vecs * N; i += 64)
      keep((float)reinterpret_cast<const T*>(sh.vec[wave])[i], sh.vec_at[wave][i / N] + i % N);
    if (lane == 0) sh.n_vecs[wave] = n_vecs;
    if (tid < sp.head) keep((float)p[tid], tid);
    if (sp.tail + tid < sp.n) keep((float)p[sp.tail + tid], (uint32_t)sp.tail + tid);
    __syncthreads();
    const int n = sh.n_cands;
    bool fits = n <= SC_CANDS;
#pragma unroll
    for (int w = 0; w < THREADS / 64; w++) fits &= sh.n_vecs[w] <= SC_VECS;
    if (fits) {
      order_candidates(n, a.n_alt, sh);
      __syncthreads();
    } else {
      __syncthreads();
      find_again(sp, first, a.n_alt, mine, sh);
    }
  }
  if (a.splits > 1) {
    uint8_t* out = a.parts + (row * a.splits + part) * part_bytes(a.n_alt);
    if (tid == 0) *reinterpret_cast<PartHead*>(out) = {st, x_given};
    if constexpr (ALT)
      if (tid < a.n_alt) reinterpret_cast<uint64_t*>(out + sizeof(PartHead))[tid] = sh.best[tid];
    return;
  }
  const RowScores r = row_scores(st, c);
  if (tid == 0) {
    if (a.logprobs) a.logprobs[row] = given_log_prob(target, a.vocab, x_given, r, a.scale);
    if (a.stats) {
      a.stats[2 * row] = r.m;
      a.stats[2 * row + 1] = r.log_s;
    }
    if (a.entropy) a.entropy[row] = r.entropy;
  }
  if constexpr (ALT) {
    if (tid < a.n_alt) {
      const uint64_t k = sh.best[tid];
      const bool nan = r.log_s != r.log_s;
      a.alt_ids[row * a.n_alt + tid] = k && !nan ? alt_id(k) : -1;
      a.alt_logprobs[row * a.n_alt + tid] = nan ? r.log_s : k ? log_prob(alt_value(k), r, a.scale) : NEG_INF;
    }
  }
}

// Joins the parts of a row.  The parts' lists are in order, so that n_alt
// entries reach the least of their entries of one place; those are ordered.
template <class T>
__global__ __launch_bounds__(SC_THREADS) void scores_join_kernel(ScoreArgs<T> a) {
  __shared__ __align__(16) uint64_t lists[SC_MAX_SPLITS * TT_MAX_ALTERNATIVES];  // [splits][n_alt]
  __shared__ __align__(16) uint64_t cands[SC_CANDS];
  __shared__ uint64_t least;
  __shared__ int found;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, k = a.n_alt, n = a.splits * k;
  const float c = a.scale * LOG2E;
  const uint8_t* in = a.parts + row * a.splits * part_bytes(k);
  PartHead head = {empty_stats(), 0.f};
  if (lane < a.splits) head = *reinterpret_cast<const PartHead*>(in + lane * part_bytes(k));
  const int32_t t = a.targets ? a.targets[row] : -1;
  if (tid == 0) found = 0;
  for (int i = tid; i < ((n + 7) & ~7); i += SC_THREADS) {
    const int part = i / (k ? k : 1);
    lists[i] = i < n ? reinterpret_cast<const uint64_t*>(in + part * part_bytes(k) + sizeof(PartHead))[i - part * k] : 0;
  }
  const float x_given = __shfl(head.given, t >= 0 && t < a.vocab ? (int)(t / a.per_part) : 0);
  const Stats st = wave_join(head.st, head.st.m, c);  // (every wave for itself)
  const RowScores r = row_scores(st, c);
  const bool nan = r.log_s != r.log_s;
  if (tid == 0) {
    if (a.logprobs) a.logprobs[row] = given_log_prob(t, a.vocab, x_given, r, a.scale);
    if (a.stats) {
      a.stats[2 * row] = r.m;
      a.stats[2 * row + 1] = r.log_s;
    }
    if (a.entropy) a.entropy[row] = r.entropy;
  }
  if (!k) return;
  __syncthreads();
  if (tid < 64) {
    const int level = (k + a.splits - 1) / a.splits - 1;  // every list's entry of this place: n_alt entries reach the least
    uint64_t low = lane < a.splits ? lists[lane * k + level] : ~0ull;
#pragma unroll
    for (int d = 32; d; d >>= 1) {
      const uint64_t o = __shfl_xor(low, d);
      low = o < low ? o : low;
    }
    if (tid == 0) least = low;
  }
  __syncthreads();
  for (int i = tid; i < n; i += SC_THREADS) {
    const uint64_t key = lists[i];
    if (key && key >= least) {
      const int at = atomicAdd(&found, 1);
      if (at < SC_CANDS) cands[at] = key;
    }
  }
  __syncthreads();
  // places by counting the better candidates; where there are too many to keep
  // (rows that are masked in some parts), among all lists
  const bool fits = found <= SC_CANDS;
  const int total = fits ? found : n;
  if (fits && tid < 8 && found + tid < SC_CANDS) cands[found + tid] = 0;
  __syncthreads();
  for (int i = tid; i < total; i += SC_THREADS) {
    const uint64_t key = fits ? cands[i] : lists[i];
    if (key < least || key == 0) continue;
    const int place = fits ? better(cands, total, key) : better(lists, total, key);
    if (place >= k) continue;
    a.alt_ids[row * k + place] = nan ? -1 : alt_id(key);
    a.alt_logprobs[row * k + place] = nan ? r.log_s : log_prob(alt_value(key), r, a.scale);
  }
  if (tid >= found && tid < k) {
    a.alt_ids[row * k + tid] = -1;
    a.alt_logprobs[row * k + tid] = nan ? r.log_s : NEG_INF;
  }
}

// Gradient: every entry is read once and written once, by loads and stores that
// the caches do not keep.  A block takes THREADS * U vectors of a row: neighbouring
// blocks write neighbouring addresses (1,536 rows of 100,257 in bf16: 100 us, 6.2
// TB/s; a run of seven steps of one row in a block: 138 us; with ordinary loads and
// stores 107 us).  The stores are aligned, the loads may not be.
template <class T>
struct GradArgs {
  const T* logits;
  T* grad;
  int64_t rows, vocab, stride, grad_stride;
  float scale;
  const int32_t* targets;
  const float *stats, *entropy, *grad_logprobs, *grad_entropy;
  int chunks;  // blocks of a row
};

template <class T, int THREADS, int U>
__global__ __launch_bounds__(THREADS) void scores_grad_kernel(GradArgs<T> a) {
  constexpr int N = Vec<T>::N;
  const int tid = threadIdx.x;
  const uint32_t row32 = blockIdx.x / (uint32_t)a.chunks, chunk = blockIdx.x - row32 * (uint32_t)a.chunks;
  const int64_t row = row32;
  const T* in = a.logits + row * a.stride;
  T* out = a.grad + row * a.grad_stride;
  const Span<T> sp(out, a.vocab);
  const int vecs = (int)sp.vecs, v = (int)chunk * THREADS * U + tid;
  Vec<T> x[U];
#pragma unroll
  for (int k = 0; k < U; k++)
    if (v + k * THREADS < vecs) x[k] = load_vec(in + sp.head + (int64_t)(v + k * THREADS) * N);
  const RowGrad g = row_grad(a.targets, a.stats, a.entropy, a.grad_logprobs, a.grad_entropy, row, a.vocab, a.scale);
  const float c = a.scale * LOG2E;
  auto one = [&](float x) { return (T)(g.zero ? 0.f : grad_of(x, c, g)); };
  auto edge = [&](float x, bool given) { return given && !g.zero ? (T)grad_of_given(x, c, g) : one(x); };
#pragma unroll
  for (int k = 0; k < U; k++) {
    const int w = v + k * THREADS;
    if (w >= vecs) continue;
    Vec<T> z;
    const int64_t at = g.target - (sp.head + (int64_t)w * N);  // place of the given token in this vector
#pragma unroll
    for (int i = 0; i < N; i++) z.v[i] = one((float)x[k].v[i]);
    if (at >= 0 && at < N) {
      float given = 0.f;
#pragma unroll
      for (int i = 0; i < N; i++) given = i == (int)at ? (float)x[k].v[i] : given;
      const T y = edge(given, true);
#pragma unroll
      for (int i = 0; i < N; i++) z.v[i] = i == (int)at ? y : z.v[i];
    }
    store_vec_once(out + sp.head + (int64_t)w * N, z);
  }
  if (chunk == 0 && tid < sp.head) out[tid] = edge((float)in[tid], tid == g.target);
  if (chunk + 1 == (uint32_t)a.chunks && sp.tail + tid < a.vocab)
    out[sp.tail + tid] = edge((float)in[sp.tail + tid], sp.tail + tid == g.target);
}

template <class T>
int run_scores(ScoreArgs<T> a, hipStream_t st) {
  const bool wave = a.rows >= WAVE_ROWS && a.vocab <= WAVE_VOCAB;
  auto* kernel = wave ? a.n_alt ? scores_kernel<T, true, 64> : scores_kernel<T, false, 64>
                      : a.n_alt ? scores_kernel<T, true, SC_THREADS> : scores_kernel<T, false, SC_THREADS>;
  if (launch(kernel, dim3((uint32_t)(a.rows * a.splits)), dim3(wave ? 64 : SC_THREADS), st, a) != hipSuccess)
    return TT_ERR_HIP;
  if (a.splits > 1 && launch(scores_join_kernel<T>, dim3((uint32_t)a.rows), dim3(SC_THREADS), st, a) != hipSuccess)
    return TT_ERR_HIP;
  return TT_OK;
}

template <class T>
int run_grad(GradArgs<T> a, hipStream_t st) {
  // short rows: a wave each, its vectors all under way at once
  const bool wave = a.vocab <= 64 * 4 * Vec<T>::N;
  const int threads = wave ? 64 : SC_THREADS;
  const int64_t cols = (int64_t)Vec<T>::N * (wave ? 64 * 4 : SC_THREADS * 2);
  a.chunks = (int)((a.vocab + cols - 1) / cols);
  if (a.rows > (int64_t)UINT32_MAX / threads / a.chunks) return TT_ERR_TOO_LARGE;
  return launch(wave ? scores_grad_kernel<T, 64, 4> : scores_grad_kernel<T, SC_THREADS, 2>, dim3((uint32_t)(a.rows * a.chunks)),
                dim3(threads), st, a) == hipSuccess
             ? TT_OK
             : TT_ERR_HIP;
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int64_t tt_token_scores_workspace(int64_t rows, int64_t vocab, int32_t n_alt) {
  if (rows < 0 || vocab < 1 || vocab > INT32_MAX || n_alt < 0 || n_alt > TT_MAX_ALTERNATIVES) return TT_ERR_BAD_ARG;
  return scores_room(rows, vocab) * part_bytes(n_alt);
}

extern "C" int tt_token_scores(const void* logits, int32_t type, int64_t rows, int64_t vocab, int64_t stride, float scale,
                               const int32_t* targets, float* logprobs, float* stats, float* entropy, int32_t n_alt,
                               int32_t* alt_ids, float* alt_logprobs, void* workspace, int64_t workspace_bytes,
                               void* stream) {
  const int64_t need = tt_token_scores_workspace(rows, vocab, n_alt);
  if (need < 0 || !score_type(type) || stride < vocab || !good_scale(scale) || workspace_bytes < need ||
      reinterpret_cast<uintptr_t>(workspace) % 256)
    return TT_ERR_BAD_ARG;
  if (rows > (int64_t)UINT32_MAX / SC_THREADS) return TT_ERR_TOO_LARGE;
  if (rows == 0) return TT_OK;
  if (!logits || (need && !workspace) || (n_alt && (!alt_ids || !alt_logprobs))) return TT_ERR_NULL_ARG;
  const int splits = scores_splits(rows, vocab, n_alt);
  auto go = [&](auto zero) {
    using T = decltype(zero);
    return run_scores(ScoreArgs<T>{static_cast<const T*>(logits), rows, vocab, stride, scale, targets, logprobs, stats,
                                   entropy, n_alt, alt_ids, alt_logprobs, static_cast<uint8_t*>(workspace),
                                   splits, (vocab + splits - 1) / splits},
                      static_cast<hipStream_t>(stream));
  };
  return type == TT_F32 ? go(float{}) : type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}

extern "C" int tt_token_scores_grad(const void* logits, int32_t type, int64_t rows, int64_t vocab, int64_t stride,
                                    float scale, const int32_t* targets, const float* stats, const float* entropy,
                                    const float* grad_logprobs, const float* grad_entropy, void* grad_logits,
                                    int64_t grad_stride, void* stream) {
  if (rows < 0 || vocab < 1 || vocab > INT32_MAX || !score_type(type) || stride < vocab || grad_stride < vocab ||
      !good_scale(scale) || (grad_logits == logits && rows && grad_stride != stride))
    return TT_ERR_BAD_ARG;
  if (rows == 0) return TT_OK;
  if (!logits || !grad_logits || !stats || (grad_entropy && !entropy)) return TT_ERR_NULL_ARG;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    return run_grad(GradArgs<T>{static_cast<const T*>(logits), static_cast<T*>(grad_logits), rows, vocab, stride,
                                grad_stride, scale, targets, stats, entropy, grad_logprobs, grad_entropy, 0},
                    static_cast<hipStream_t>(stream));
  };
  return type == TT_F32 ? go(float{}) : type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}
