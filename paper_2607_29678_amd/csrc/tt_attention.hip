// tt_cache_attention: attention of a step's tokens over a paged cache, with an
// optional sliding window and first tokens that stay visible.
//
// Work is cut into items: a tile of a request's tokens with the query heads that
// share a key head (their products share the loads of keys and values), and every
// item into units, tiles of keys that some of its tokens see.  The units of a key head
// stand in one line, and the head's workers take equal parts of it: a step of long and
// short requests, of single tokens and prompts, is even by construction, and a
// graph's launches need no lengths on the host.  Every block finds its part by
// summing the items' units for itself.  Where an item's units fall to several
// workers, each leaves its sums in the workspace, and a second launch joins them.
//
// Products are of transposed tiles: S^T = K Q^T puts a query's scores into the
// lanes of one column, so that the running maximum and sum are a lane's own and the
// exponentials are, as they stand, the operand of O^T = V^T P^T.  Values are
// transposed by the loads from LDS.  An online softmax keeps the sums of a row as of
// a maximum that goes up only by more than a factor of 2^8, so that most tiles move
// nothing.
//
// What bounds it: single tokens, reads of keys and values (96 requests of 4,000 tokens,
// 32 heads over 8 of 128 elements: 1.63 GB in 317 us, 5.1 TB/s, the rate of a plain
// copy being 4.9); prompts, the matrix cores and the vector instructions beside them
// (14,001 tokens, the same heads: 1,150 to 1,240 us on several cards, 720 to 780
// TFLOP/s; a plain library product 1,160 to 1,490); a few short requests, the search of
// every block's part, cold, 6 us of 13, and the join, 4 to 9.
#include "tt_cache.h"

namespace tt {
namespace {

// n / d for 0 <= n < 2^31, as a product: with 2^s <= d < 2^(s + 1) and
// m = floor(2^(32 + s) / d) + 1, m d exceeds 2^(32 + s) by at most d, and n times
// that stays below 2^(32 + s).
struct Quotient {
  uint32_t d, m;
  int s;
  explicit Quotient(uint32_t by = 1) : d(by), m(0), s(0) {
    while ((by >> s) > 1) s++;
    if (by & (by - 1)) m = (uint32_t)(((uint64_t)1 << (32 + s)) / by) + 1;
  }
  __device__ __forceinline__ int of(int n) const { return (int)((m ? __umulhi((uint32_t)n, m) : (uint32_t)n) >> s); }
};

constexpr int ATT_THREADS = 256;
constexpr int ATT_WAVES = 4;
constexpr int STAGED = 1024;  // requests whose offsets and lengths are held in LDS for the search
// Rows (tokens times query heads of a key head) of a request up to which, on average,
// the small path takes a step.  us by the small and by the large path, heads of 128 but
// where 64 is said: 300 requests of 2,000 tokens, 1 row of 64 471 / 524; 4 of 700, 4 rows
// 21.8 / 24.8; 64 of 4,000, 4 rows 213 / 204, 16 rows 227 / 204, 20 rows 337 / 205, 40 rows
// 611 / 210 (the small path reads the keys once for every 16 rows); 2 of 120,000, 7 rows
// 126 / 114; 64 of 20,000 in a window of 4,096, 16 rows of 64 128 / 122, 40 rows 328 / 127.
// (So long requests of 4 to 16 rows would be 5 to 10% faster by the large path.)  The mean
// speaks for all of a step: 256 single tokens behind 4,000 and a prompt of 700 840 / 845, of
// 900 834 / 954; 32 single tokens with 8 rows each and 60 more of one request 184 / 138.
constexpr int SMALL_ROWS = 16;
constexpr int EACH = 4;       // items counted by a thread at a time

// What the small path (16 rows a wave, 32 keys a unit) and the large one (128 rows a
// block, 64 keys a unit) make of a step.
struct Plan {
  int rows;        // of an item
  int keys;        // of a unit
  int workers;
  int heads;       // query heads of an item
  int tokens;      // of an item
  int groups;      // items that the query heads of a key head take
  int least;       // fewest units of a worker
  // Head units each have workers / stride workers, who take equal parts of its units:
  // worker w is with head unit w % stride, so that neighbours read neighbouring heads
  // of the same tokens.  More head units than workers: stride is 1 and all units stand
  // in one line, head after head.
  int stride, parts;
  Quotient by_tokens;
};

struct AttentionArgs {
  tt_cache c;
  tt_attention s;
  int capacity;  // tokens that a request's table has room for (at most 2^31 - 65)
  Plan small, large;
  Quotient by_page;
  uint32_t page_step, slot_step;  // strides in vectors of 8 elements
  int per_kv;      // query heads of a key head
  bool vectors;    // queries and out are aligned to 16 bytes
  bool wide;       // sums of units may pass 32 bits, or there are more requests than LDS holds
  uint8_t* parts;  // workspace
};

// What a worker leaves for the join.
struct Leaf {
  int32_t pieces;              // of the item that its last piece begins and others go on; 0: none
  int32_t row0, tokens, head;  // that item's first row of queries, its tokens and its head unit
  int32_t low;                 // position of its first token
};

// The workspace: which path ran (256 bytes), a leaf for each worker, two pieces for each
__host__ __device__ inline int64_t piece_floats(int rows, int dim) { return (int64_t)rows * (dim + 2); }
__host__ __device__ inline int64_t leaves_bytes(int workers) { return 256 + (((int64_t)workers * (int64_t)sizeof(Leaf) + 255) & ~255); }
__device__ __forceinline__ Leaf* leaves_of(const AttentionArgs& a) { return reinterpret_cast<Leaf*>(a.parts + 256); }
__device__ __forceinline__ float* piece_of(const AttentionArgs& a, const Plan& p, int worker, int which) {
  return reinterpret_cast<float*>(a.parts + leaves_bytes(p.workers)) + (2 * (int64_t)worker + which) * piece_floats(p.rows, a.c.dim);
}

// One request's place in the step, and an item of it.
struct Item {
  int row0, tokens;        // rows of queries
  int low;                 // position of the first token
  int front, begin, last;  // some token sees key j if j <= last and (j < front or j >= begin)
  int front_units, begin_unit, units;
};

__device__ __forceinline__ int clamped(int64_t x, int64_t least, int64_t most) { return (int)(x < least ? least : x > most ? most : x); }
__device__ __forceinline__ int offset_of(const tt_attention& s, int r) { return clamped(s.offsets[r], 0, s.tokens); }

// Slot `slot` of the step's items: request r's begin at slot offsets[r] / tokens + r,
// which leaves each one room enough.  (Slots without tokens have no units.)
__device__ __forceinline__ Item item_of(const AttentionArgs& a, const Plan& p, int slot, int r, int off0, int off1, int raw1, int length) {
  Item t;
  const int64_t at = (int64_t)slot - (p.by_tokens.of(off0) + (int64_t)r);
  const int64_t row0 = off0 + at * p.tokens;
  t.row0 = (int)row0;
  t.tokens = 0;
  t.units = 0;
  if (at < 0 || row0 >= off1) return t;
  t.tokens = off1 - row0 < p.tokens ? (int)(off1 - row0) : p.tokens;
  const int64_t low = (int64_t)length - raw1 + row0, high = low + t.tokens - 1;
  t.low = clamped(low, INT32_MIN / 2, INT32_MAX - 256);  // (positions of an item's tokens do not overflow)
  t.last = clamped(high, -1, a.capacity);
  t.begin = a.s.window ? clamped(low - a.s.window + 1, 0, a.capacity) : 0;
  t.front = a.s.sinks < t.begin ? a.s.sinks : t.begin;
  const int keys = p.keys;
  t.front_units = (t.front + keys - 1) / keys;
  t.begin_unit = t.begin / keys;
  if (t.begin_unit < t.front_units) t.begin_unit = t.front_units;
  t.units = t.last < 0 ? 1 : t.front_units + t.last / keys - t.begin_unit + 1;
  if (t.units < t.front_units) t.units = t.front_units;
  if (t.units < 1) t.units = 1;
  return t;
}

struct Search {
  int32_t offsets[STAGED + 1], lengths[STAGED];
  int64_t sums[ATT_WAVES];
  int live[ATT_WAVES];
};
// Where a worker begins
struct Start {
  int slot, request, head, unit, slots;
  int64_t count;  // units
  int64_t size;   // units of every worker but the last ones
  Item item;
};

// Offsets and lengths to LDS (of as many requests as it holds), and whether the
// step's requests have few rows a key head, so that the small path takes it.
__device__ __forceinline__ bool few_rows(const AttentionArgs& a, Search& sh) {
  const tt_attention& s = a.s;
  const int tid = threadIdx.x, n = s.n_requests;
  const bool staged = n <= STAGED;
  int live = 0;
  for (int i = tid; i <= n; i += ATT_THREADS) {
    const int x = s.offsets[i], length = i < n ? s.lengths[i] : 0;
    live += i < n && s.offsets[i + 1] > x;
    if (staged) {
      sh.offsets[i] = x;
      if (i < n) sh.lengths[i] = length;
    }
  }
  const int tokens = clamped(s.offsets[n], 0, s.tokens);
#pragma unroll
  for (int d = 32; d; d >>= 1) live += __shfl_xor(live, d);
  if ((tid & 63) == 0) sh.live[tid >> 6] = live;
  __syncthreads();
  live = 0;
#pragma unroll
  for (int w = 0; w < ATT_WAVES; w++) live += sh.live[w];
  return (int64_t)tokens * a.per_kv <= (int64_t)live * SMALL_ROWS;
}

// n / d; 64-bit divisions take hundreds of instructions
__device__ __forceinline__ int64_t divided(int64_t n, int64_t d) {
  return n <= INT32_MAX && d <= INT32_MAX ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}
__device__ __forceinline__ int32_t divided(int32_t n, int32_t d) { return (int32_t)((uint32_t)n / (uint32_t)d); }

// Sum of the lanes up to and with this one
__device__ __forceinline__ int32_t wave_scan(int32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // within rows of 16: 1, 2, 4, 8 lanes back
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // a row's last lane to the next row
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
  return x;
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up((long long)x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Finds the parts of the block's COUNT workers (first, first + 1, ...), with 32-bit sums
// from LDS (SHORT) or with 64-bit sums from memory, where the sizes that the host sees
// do not keep them below 2^31 or there are more requests than LDS holds.
template <int COUNT, bool SHORT, class I = std::conditional_t<SHORT, int32_t, int64_t>>
__device__ __forceinline__ void find_starts_by(const AttentionArgs& a, const Plan& p, int first, Search& sh, Start* starts) {
  const tt_attention& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = s.n_requests;
  if (tid < COUNT) starts[tid].count = 0;
  auto raw = [&](int r) {
    if constexpr (SHORT) return sh.offsets[r];
    else return s.offsets[r];
  };
  auto length = [&](int r) {
    if constexpr (SHORT) return sh.lengths[r];
    else return s.lengths[r];
  };
  auto offset = [&](int r) { return clamped(raw(r), 0, s.tokens); };
  auto begin = [&](int r) { return p.by_tokens.of(offset(r)) + r; };
  const int slots = begin(n);
  // threads take one slot each, or EACH
  const int each = slots <= ATT_THREADS ? 1 : EACH;
  auto item = [&](int slot, int r) {
    return item_of(a, p, slot, r, offset(r), offset(r + 1), raw(r + 1), length(r));
  };
  auto request_of = [&](int slot) {
    int lo = 0, hi = n;  // requests [0, lo) begin at or before the slot
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (begin(mid) <= slot) lo = mid + 1;
      else hi = mid;
    }
    return lo > 0 ? lo - 1 : 0;
  };
  // units of the thread's slots from slot0 on, the first of them of request r
  auto count = [&](int slot0, int r) {
    I sum = 0;
#pragma unroll 1
    for (int slot = slot0; slot < slot0 + each && slot < slots; slot++) {
      while (r + 1 < n && begin(r + 1) <= slot) r++;
      sum += item(slot, r).units;
    }
    return sum;
  };
  // sums of the threads before this one, and of all
  auto scan = [&](I mine, I& before) {
    const I x = wave_scan(mine);
    __syncthreads();
    if (lane == 63) sh.sums[wave] = x;
    __syncthreads();
    before = x - mine;
    I all = 0;
#pragma unroll
    for (int w = 0; w < ATT_WAVES; w++) {
      if (w < wave) before += (I)sh.sums[w];
      all += (I)sh.sums[w];
    }
    return all;
  };
  const int at_once = ATT_THREADS * each;
  I total = 0, before = 0, mine = 0;
  int request = 0;
  for (int64_t slot0 = 0; slot0 < slots; slot0 += at_once) {
    const int slot = (int)slot0 + tid * each;
    request = slot < slots ? request_of(slot) : 0;
    mine = slot < slots ? count(slot, request) : 0;
    total += scan(mine, before);
  }
  if (total == 0) return;
  const I line = p.stride > 1 ? total : total * (I)(a.c.kv_heads * p.groups);
  I size = divided(line + p.parts - 1, (I)p.parts);
  if (size < p.least) size = p.least;
  I base = 0;
  for (int64_t slot0 = 0; slot0 < slots; slot0 += at_once) {
    const int slot_mine = (int)slot0 + tid * each;
    I here = total;
    if (slots > at_once) {
      request = slot_mine < slots ? request_of(slot_mine) : 0;
      mine = slot_mine < slots ? count(slot_mine, request) : 0;
      here = scan(mine, before);
    }
    int part = p.stride > 1 ? divided(first, p.stride) : first, head_unit = p.stride > 1 ? first - part * p.stride : 0;
    for (int w = 0; w < COUNT; w++) {
      const I from = part * size;
      if (part >= p.parts || from >= line) break;
      const I over = p.stride > 1 ? 0 : divided(from, total);
      I x = from - over * total - base - before;
      if (x >= 0 && x < mine) {
        int r = request;
        for (int slot = slot_mine; slot < slot_mine + each && slot < slots; slot++) {
          while (r + 1 < n && begin(r + 1) <= slot) r++;
          const Item t = item(slot, r);
          if (x < t.units) {
            starts[w] = {slot, r, p.stride > 1 ? head_unit : (int)over, (int)x, slots, from + size < line ? size : line - from, size, t};
            break;
          }
          x -= t.units;
        }
      }
      if (p.stride == 1 || ++head_unit == p.stride) {
        part++;
        head_unit = 0;
      }
    }
    base += here;
  }
  __syncthreads();
}
template <int COUNT>
__device__ __forceinline__ void find_starts(const AttentionArgs& a, const Plan& p, int first, Search& sh, Start* starts) {
  if (a.wide) find_starts_by<COUNT, false>(a, p, first, sh, starts);
  else find_starts_by<COUNT, true>(a, p, first, sh, starts);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) { return ((int64_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x); }

// A worker's walk through the items
struct Walk {
  int slot, request, head, unit, slots;
  int64_t left, size;
  Item item;
  __device__ __forceinline__ void read(const AttentionArgs& a, const Plan& p) {
    const int raw1 = a.s.offsets[request + 1];
    take(item_of(a, p, slot, request, offset_of(a.s, request), offset_of(a.s, request + 1), raw1, a.s.lengths[request]));
  }
  __device__ __forceinline__ void take(const Item& t) {
    item = {uniform(t.row0),  uniform(t.tokens),      uniform(t.low),        uniform(t.front), uniform(t.begin),
            uniform(t.last),  uniform(t.front_units), uniform(t.begin_unit), uniform(t.units)};
  }
  __device__ __forceinline__ explicit Walk(const Start& st)
      : slot(uniform(st.slot)), request(uniform(st.request)), head(uniform(st.head)), unit(uniform(st.unit)),
        slots(uniform(st.slots)),
        left(uniform(st.count)), size(uniform(st.size)) {
    take(st.item);
  }
  // to the next item that has units (there is one: left > 0; offsets that are not
  // in order may have none, and the walk ends there)
  __device__ __forceinline__ void next(const AttentionArgs& a, const Plan& p) {
    unit = 0;
    do {
      slot++;
      if (slot >= slots) {
        slot = 0;
        request = 0;
        head++;
      }
      while (request + 1 < a.s.n_requests &&
             (int64_t)p.by_tokens.of(offset_of(a.s, request + 1)) + request + 1 <= slot)
        request++;
      request = uniform(request);
      read(a, p);
    } while (item.units == 0 && head < a.c.kv_heads * p.groups);
    if (item.units == 0) left = 0;
  }
};

template <class T>
__device__ __forceinline__ Vec8<T> zero8() {
  Vec8<T> z;
#pragma unroll
  for (int i = 0; i < 8; i++) z[i] = (T)0.f;
  return z;
}
template <class T>
__device__ __forceinline__ Vec8<T> nan8() {
  Vec8<T> z;
#pragma unroll
  for (int i = 0; i < 8; i++) z[i] = (T)__builtin_nanf("");
  return z;
}
// Elements that are not finite, as bits
template <class T>
__device__ __forceinline__ uint32_t not_finite(const Vec8<T>& v) {
  constexpr uint32_t TOP = std::is_same<T, bf16_t>::value ? 0x7F80u : 0x7C00u;
  using U8 = __attribute__((ext_vector_type(8))) uint16_t;
  const U8 u = __builtin_bit_cast(U8, v);
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) bits |= ((u[i] & TOP) == TOP ? 1u : 0u) << i;
  return bits;
}
template <class T>
__device__ __forceinline__ Vec8<T> load8(const T* p, bool vectors) {
  if (vectors) return *reinterpret_cast<const Vec8<T>*>(p);
  Vec8<T> z;
#pragma unroll
  for (int i = 0; i < 8; i++) z[i] = p[i];
  return z;
}
// A result lies between its values, but the weights' roundings may carry it past the
// largest one that f16 has (65,504; infinite from 65,520 on).  What is not finite stays.
template <class T>
__device__ __forceinline__ T result(float x) {
  constexpr float MOST = 65504.f;
  if (std::is_same<T, f16_t>::value && fabsf(x) < __builtin_inff()) x = __builtin_amdgcn_fmed3f(x, -MOST, MOST);
  return (T)x;
}
template <class T>
__device__ __forceinline__ void store4(T* p, const float* x, float f, bool vectors) {
  using T4 = T __attribute__((ext_vector_type(4)));
  T4 z;
#pragma unroll
  for (int i = 0; i < 4; i++) z[i] = result<T>(x[i] * f);
  if (vectors) {
    *reinterpret_cast<T4*>(p) = z;
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) p[i] = z[i];
  }
}

// Adds what is not finite of four values to o[at], ... (the empty statement keeps the
// loads of several calls apart: registers are for the products)
template <class T, class F>
__device__ __forceinline__ void add_not_finite(const T* value, bool there, F* o, int at) {
  using T4 = T __attribute__((ext_vector_type(4)));
  if (there) {
    const T4 x = *reinterpret_cast<const T4*>(value);
#pragma unroll
    for (int i = 0; i < 4; i++) (*o)[at + i] += fabsf((float)x[i]) < __builtin_inff() ? 0.f : (float)x[i];
  }
  asm volatile("" ::: "memory");
}
using F4 = float __attribute__((ext_vector_type(4)));
using F16 = float __attribute__((ext_vector_type(16)));
__device__ __forceinline__ F4 product16(Vec8<bf16_t> a, Vec8<bf16_t> b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F4 product16(Vec8<f16_t> a, Vec8<f16_t> b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F16 product32(Vec8<bf16_t> a, Vec8<bf16_t> b, F16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F16 product32(Vec8<f16_t> a, Vec8<f16_t> b, F16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// Four rows of 16 columns, transposed: of 16 lanes, lane i gives the address of
// columns 4 (i % 4) to 4 (i % 4) + 3 of row i / 4 and receives column i.
using S4 = short __attribute__((ext_vector_type(4)));
template <class T>
__device__ __forceinline__ S4 transposed(const T* p) {
  using P = __attribute__((address_space(3))) S4*;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p));
}
template <class T>
__device__ __forceinline__ Vec8<T> both(S4 a, S4 b) {
  using S8 = short __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(Vec8<T>, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Whether every token of the item sees every key of [k0, k0 + keys)
__device__ __forceinline__ bool all_seen(const AttentionArgs& a, const Item& t, int k0, int keys) {
  const int end = k0 + keys;
  const int64_t begin = a.s.window ? (int64_t)t.low + t.tokens - a.s.window : 0;  // of the last token
  return end <= t.last + 1 && end - 1 <= t.low && (k0 >= begin || end <= a.s.sinks);
}
__device__ __forceinline__ bool sees(const AttentionArgs& a, int position, int key) {
  int64_t begin = a.s.window ? (int64_t)position - a.s.window + 1 : 0;
  if (begin > a.capacity) begin = a.capacity;
  return key <= position && key <= a.capacity && (key >= begin || key < a.s.sinks);
}
// Bit j: whether the token at `position` sees key k0 + j (j < keys <= 64)
__device__ __forceinline__ uint64_t seen_bits(const AttentionArgs& a, int position, int k0, int keys) {
  auto below = [&](int64_t n) {  // bits [0, n - k0)
    const int x = clamped(n - k0, 0, keys);
    return x >= 64 ? ~0ull : (1ull << x) - 1ull;
  };
  const int last = position < a.capacity ? position : a.capacity;
  int64_t begin = a.s.window ? (int64_t)position - a.s.window + 1 : 0;
  if (begin > a.capacity) begin = a.capacity;
  return below((int64_t)last + 1) & (~below(begin) | below(a.s.sinks));
}
__device__ __forceinline__ bool needed(const Item& t, int key) { return key <= t.last && (key < t.front || key >= t.begin); }
__device__ __forceinline__ int first_key(const Item& t, int unit, int keys) {
  return (unit < t.front_units ? unit : t.begin_unit + unit - t.front_units) * keys;
}
// Where a key's token is: its page (-1: there is none, -2: no token of the item sees
// it), and its place in the page
struct Place {
  int page, slot;
};
__device__ __forceinline__ Place place_of(const AttentionArgs& a, const Item& t, const int32_t* table, int key) {
  const int entry = a.by_page.of(key);
  Place x = {-2, key - entry * (int)a.by_page.d};
  if (needed(t, key)) x.page = entry < a.s.table_width ? table[entry] : -1;
  return x;
}
__device__ __forceinline__ bool is_page(const AttentionArgs& a, int page) { return (uint32_t)page < (uint32_t)a.c.pages; }
// (strides in vectors of 8 elements: products of 32 bits by 32)
__device__ __forceinline__ int64_t vector_at(const AttentionArgs& a, const Place& x, int64_t head) {
  return (int64_t)(((uint64_t)(uint32_t)x.page * a.page_step + (uint64_t)(uint32_t)x.slot * a.slot_step) * 8) + head;
}

// The weights 2^(score - m) are rounded to the type for the second product, their sum is
// of 32 bits.  (One rounding a weight, half a place: the matrix cores take operands of the
// type, and the result is rounded by as much again; errors come to 1.4 times those of
// weights of 32 bits.  A second product, of what the rounding leaves, takes no time on the
// small path up to 128 elements, but what it leaves of a weight may be 0 or negative, and an
// infinite value would come out as NaN.)  m goes up only where a score is more than SLACK
// powers of two above the largest it is of.
// A weight of f16 has full places from 2^-14 on and none below 2^-25, while the sum holds
// them all: many small ones would be missing above and there below, 16% of a result with
// one key 17.4 above 20,000 others.  So m lies HEAD below that largest score: weights go up
// to 2^15, and n keys lose at most n 2^-32 of their largest value.
constexpr float SLACK = 8.f;
template <class T>
constexpr float HEAD = std::is_same<T, f16_t>::value ? 7.f : 0.f;
// A product that no addition may be joined to: differences of such from a maximum of such
// are not above 0, however large they are
__device__ __forceinline__ float rounded(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}
// Whether m goes up to top - HEAD (the difference: far from zero a sum rounds to either side)
template <class T>
__device__ __forceinline__ bool rises(float m, float top) { return top - m > SLACK + HEAD<T>; }

// ---- 16 rows a wave: single tokens -----------------------------------------------

// A wave takes its units by itself: 32 keys and values go from memory to registers,
// the keys straight into the product, the values through LDS that is the wave's own.
// The next unit's are under way during the exponentials and the second product: 16 KB
// a wave, 128 KB a compute unit.  Loads that do not stay in the caches were slower
// (96 requests of 4,000 tokens 385 us against 367: a row comes in two requests of 64
// bytes a cache line), and so were workers that follow each other within a head (367
// against 334: neighbours then read rows 2 KB apart).
template <class T, int KK>  // KK: 32 elements of a head
struct SmallShared {
  static constexpr int PITCH = KK * 32 + 16;  // (rows 32 bytes apart in the banks)
  T values[ATT_WAVES][32][PITCH];
};
template <class T, int KK>
__device__ __forceinline__ void small_path(const AttentionArgs& a, Search& search, SmallShared<T, KK>& sh, Start* starts) {
  constexpr int DT = 2 * KK, KEYS = 32, PITCH = SmallShared<T, KK>::PITCH;
  const Plan& p = a.small;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, quad = lane >> 4;
  const int dim = a.c.dim;
  // (pairs of neighbouring blocks on one XCD: blocks go to the XCDs in turn)
  const int block = (int)((blockIdx.x & ~15u) | (blockIdx.x & 7u) << 1 | (blockIdx.x >> 3 & 1u)), first = block * ATT_WAVES, worker = first + wave;
  find_starts<ATT_WAVES>(a, p, first, search, starts);
  Walk w(starts[wave]);
  __syncthreads();  // (the search's LDS is the values' from here on)
  T(*values)[PITCH] = sh.values[wave];
  Leaf leaf = {0, 0, 0, 0, 0};
  const float c = a.s.scale * LOG2E;
  bool chunk[KK];
#pragma unroll
  for (int kk = 0; kk < KK; kk++) chunk[kk] = kk * 32 + quad * 8 < dim;

  while (w.left > 0) {
    const Item& t = w.item;
    const int take = (int64_t)(t.units - w.unit) < w.left ? t.units - w.unit : (int)w.left;
    const int kv = w.head / p.groups, h0 = (w.head - kv * p.groups) * p.heads;
    const int heads = a.per_kv - h0 < p.heads ? a.per_kv - h0 : p.heads;
    const int rows = t.tokens * p.heads;  // (rows of heads past the last one are not used)
    const int my_token = col / p.heads, my_head = col - my_token * p.heads;
    const bool live = col < rows && my_head < heads;
    const int position = t.low + my_token;
    const int64_t q_row = t.row0 + my_token, q_head = (int64_t)kv * a.per_kv + h0 + my_head;
    Vec8<T> q[KK];
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
      q[kk] = zero8<T>();
      if (live && chunk[kk])
        q[kk] = load8(static_cast<const T*>(a.s.queries) + q_row * a.s.query_stride + q_head * dim + kk * 32 + quad * 8, a.vectors);
    }
    const int32_t* table = a.s.tables + w.request * a.s.table_stride;
    const int64_t head = (int64_t)kv * a.c.head_stride + quad * 8;
    const T *K = static_cast<const T*>(a.c.keys), *V = static_cast<const T*>(a.c.values);
    Vec8<T> k[2][KK], v[2][KK];
    Place places[2];
    auto fetch_places = [&](int unit) {
      const int k0 = first_key(t, unit, KEYS);
#pragma unroll
      for (int i = 0; i < 2; i++) places[i] = place_of(a, t, table, k0 + 16 * i + col);
    };
    auto fetch = [&] {
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const int64_t at = vector_at(a, places[i], head);
        const bool there = is_page(a, places[i].page);
#pragma unroll
        for (int kk = 0; kk < KK; kk++) {
          if (there && chunk[kk]) {
            k[i][kk] = *reinterpret_cast<const Vec8<T>*>(K + at + kk * 32);
            v[i][kk] = *reinterpret_cast<const Vec8<T>*>(V + at + kk * 32);
          } else {
            k[i][kk] = !there && places[i].page != -2 ? nan8<T>() : zero8<T>();
            v[i][kk] = zero8<T>();
          }
        }
      }
    };
    F4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; d++) o[d] = F4{0.f, 0.f, 0.f, 0.f};
    float m = NEG_INF, sum = 0.f;
    const int end = w.unit + take;
    fetch_places(w.unit);
    fetch();
    if (w.unit + 1 < end) fetch_places(w.unit + 1);
    for (int unit = w.unit; unit < end; unit++) {
      const int k0 = first_key(t, unit, KEYS);
      const bool edge = !all_seen(a, t, k0, KEYS);
      // values of keys that only some tokens see must not reach the others through 0 * NaN
      uint64_t spoiled[2] = {0, 0};
      if (edge && t.tokens > 1) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
          uint32_t any = 0;
#pragma unroll
          for (int kk = 0; kk < KK; kk++) {
            const uint32_t bad = not_finite(v[i][kk]);
            any |= bad;
#pragma unroll
            for (int e = 0; e < 8; e++)
              if (bad >> e & 1) v[i][kk][e] = (T)0.f;
          }
          uint64_t votes = __ballot(any != 0);
          votes |= votes >> 32;
          spoiled[i] = (votes | votes >> 16) & 0xFFFF;
        }
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int kk = 0; kk < KK; kk++) *reinterpret_cast<Vec8<T>*>(&values[16 * i + col][kk * 32 + quad * 8]) = v[i][kk];
      F4 s[2];
#pragma unroll
      for (int i = 0; i < 2; i++) {
        s[i] = F4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; kk++) s[i] = product16(k[i][kk], q[kk], s[i]);
      }
      if (unit + 1 < end) {
        fetch();
        if (unit + 2 < end) fetch_places(unit + 2);
      }
      if (edge) {
        const uint32_t seen = (uint32_t)seen_bits(a, position, k0, KEYS) >> (quad * 4);
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[i][e] = seen & 1u << (16 * i + e) ? s[i][e] : NEG_INF;
      }
      float top = NEG_INF;
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          s[i][e] = rounded(s[i][e], c);
          top = fmaxf(top, s[i][e]);
        }
      if (__ballot(rises<T>(m, top))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        top = rises<T>(m, top) ? top - HEAD<T> : m;  // (a row's own choice: its result does not depend on its neighbours)
        const float f = top == m ? 1.f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        sum *= f;
#pragma unroll
        for (int d = 0; d < DT; d++) o[d] *= f;
      }
      const float base = m == NEG_INF ? 0.f : m;
      Vec8<T> weights;
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float x = __builtin_amdgcn_exp2f(s[i][e] - base);
          sum += x;
          weights[4 * i + e] = (T)x;
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int d = 0; d < DT; d++) {
        const T* from = &values[quad * 4 + (col >> 2)][d * 16 + (col & 3) * 4];
        o[d] = product16(both<T>(transposed(from), transposed(from + 16 * PITCH)), weights, o[d]);
      }
      __builtin_amdgcn_wave_barrier();
      if (spoiled[0] | spoiled[1]) {
        for (int j = 0; j < 32; j++) {
          if (!(spoiled[j >> 4] >> (j & 15) & 1)) continue;
          const Place x = place_of(a, t, table, k0 + j);
          if (!is_page(a, x.page) || !sees(a, position, k0 + j)) continue;
          const T* value = V + vector_at(a, x, (int64_t)kv * a.c.head_stride);
#pragma unroll
          for (int d = 0; d < DT; d++) add_not_finite(value + d * 16 + quad * 4, d * 16 + quad * 4 < dim, &o[d], 0);
        }
      }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const bool began = w.unit > 0, ends = end == t.units;
    if (!began && ends) {
      const bool none = position < 0;
      if (live) {
        const float f = none ? 0.f : 1.f / sum;
        T* out = static_cast<T*>(a.s.out) + q_row * a.s.out_stride + q_head * dim + quad * 4;
#pragma unroll
        for (int d = 0; d < DT; d++) {
          const float x[4] = {o[d][0], o[d][1], o[d][2], o[d][3]};
          if (d * 16 + quad * 4 < dim) store4(out + d * 16, x, f, a.vectors);
        }
        if (a.s.logsums && quad == 0) a.s.logsums[q_row * a.s.q_heads + q_head] = none ? NEG_INF : (m == NEG_INF ? 0.f : m) * LN2 + logf(sum);
      }
    } else {
      float* piece = piece_of(a, p, worker, began ? 0 : 1);
      if (live) {
#pragma unroll
        for (int d = 0; d < DT; d++)
          if (d * 16 + quad * 4 < dim) {
            float* x = piece + (int64_t)col * dim + d * 16 + quad * 4;
            *reinterpret_cast<F4*>(x) = o[d];
          }
        if (quad == 0) *reinterpret_cast<float2*>(piece + (int64_t)p.rows * dim + 2 * col) = float2{m, sum};
      }
      if (!began) {
        leaf.pieces = 1 + (int)divided(t.units - end + w.size - 1, w.size);
        leaf.row0 = t.row0;
        leaf.tokens = t.tokens;
        leaf.head = w.head;
        leaf.low = t.low;
      }
    }
    w.left -= take;
    if (w.left > 0) w.next(a, p);
  }
  if (lane == 0) leaves_of(a)[worker] = leaf;
}

// ---- 128 rows a block: prompts ---------------------------------------------------

// Four waves of 32 rows share tiles of 64 keys and values in LDS, two of each: the
// next unit's come straight from memory during a unit's products, so that one barrier
// a unit is enough and no registers wait for them (a prefill of 14,001 tokens 1,390 us,
// through registers 1,834).  A load writes 1 KB as it comes,
// so rows stand without gaps, and the vectors of 16 bytes trade places in their row
// instead (key_place, value_place): rows that are read at once lie in other banks.
template <class T, int DP>  // DP: elements of a head, with zeros behind its own
struct LargeShared {
  static constexpr int KEYS = 64, PER_ROW = DP == 64 ? 8 : DP == 256 ? 32 : 16;  // vectors of a row
  Vec8<T> keys[2][KEYS][PER_ROW];
  Vec8<T> values[2][KEYS][PER_ROW];
  // a read of keys takes one vector of 16 rows at a time, one of values four of 4 rows
  static __device__ __forceinline__ int key_place(int row) { return PER_ROW == 8 ? row >> 1 & 7 : PER_ROW == 16 ? row & 15 : row & 7; }
  static __device__ __forceinline__ int value_place(int row) { return PER_ROW == 8 ? (row >> 1 & 1) << 2 : (row & 3) << 2; }
};
// 16 bytes a lane from memory to LDS, at `to` + 16 lane.  Written as assembly, since
// for the builtin the compiler makes every later read of LDS wait for the load; there
// is no result register.  It takes a wait state from the write of m0 to its use.
template <class T>
__device__ __forceinline__ void load_to_lds(const T* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "m0", "memory");
}
// Waits for this wave's loads and LDS accesses, then for the block's other waves.
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
template <class T, int DP>
__device__ __forceinline__ void large_path(const AttentionArgs& a, Search& search, LargeShared<T, DP>& sh, Start* starts,
                                           unsigned long long* spoiled) {
  using Shared = LargeShared<T, DP>;
  constexpr int KEYS = 64, KK = DP / 16, DT = DP / 32, PER_ROW = Shared::PER_ROW;
  constexpr int PASS = ATT_THREADS / PER_ROW, PASSES = KEYS / PASS;
  const Plan& p = a.large;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
  const int dim = a.c.dim, worker = blockIdx.x;
  find_starts<1>(a, p, worker, search, starts);
  Walk w(starts[0]);
  __syncthreads();  // (the search's LDS is the tiles' from here on)
  // what lies behind a head's elements is not loaded: zeros, once
  for (int i = tid; i < (int)(sizeof(sh.keys) / 16); i += ATT_THREADS) (&sh.keys[0][0][0])[i] = zero8<T>();
  __syncthreads();
  Leaf leaf = {0, 0, 0, 0, 0};
  const float c = a.s.scale * LOG2E;
  // the vector that this thread loads: its place in LDS, and which one of keys and values comes there
  const int place = tid % PER_ROW, row_in = tid / PER_ROW;
  const int k_vec = place ^ Shared::key_place(row_in), v_vec = place ^ Shared::value_place(row_in);
  const bool k_loads = k_vec * 8 < dim, v_loads = v_vec * 8 < dim;
  const uint32_t wave_at = uniform((int)((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&sh.keys[0][0][0])) + wave * 1024;
  constexpr uint32_t STAGE = KEYS * PER_ROW * 16;  // bytes of a tile; the values' two follow the keys' two
  // a lane's places in the tiles
  const int k_in = half ^ Shared::key_place(col), v_row = 4 * half + ((lane & 15) >> 2);
  const int v_in = ((lane >> 4 & 1) * 2 + ((lane & 3) >> 1)) ^ Shared::value_place(v_row);
  const T *K = static_cast<const T*>(a.c.keys), *V = static_cast<const T*>(a.c.values);
  int turn = 0;  // tiles of the present unit

  while (w.left > 0) {
    const Item& t = w.item;
    const int take = (int64_t)(t.units - w.unit) < w.left ? t.units - w.unit : (int)w.left;
    const int kv = w.head / p.groups, h0 = (w.head - kv * p.groups) * p.heads;
    const int heads = a.per_kv - h0 < p.heads ? a.per_kv - h0 : p.heads;
    const int row = wave * 32 + col, rows = t.tokens * p.heads;
    const int my_token = row / p.heads, my_head = row - my_token * p.heads;
    const bool live = row < rows && my_head < heads;
    const int position = t.low + my_token;
    const int64_t q_row = t.row0 + my_token, q_head = (int64_t)kv * a.per_kv + h0 + my_head;
    // the wave's tokens
    const int wave_rows = rows - wave * 32 < 32 ? rows - wave * 32 : 32;
    const int low = t.low + uniform(wave * 32 / p.heads), high = t.low + uniform((wave * 32 + wave_rows - 1) / p.heads);
    Vec8<T> q[KK];
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
      q[kk] = zero8<T>();
      if (live && kk * 16 + half * 8 < dim)
        q[kk] = load8(static_cast<const T*>(a.s.queries) + q_row * a.s.query_stride + q_head * dim + kk * 16 + half * 8, a.vectors);
    }
    const int32_t* table = a.s.tables + w.request * a.s.table_stride;
    const int64_t head = (int64_t)kv * a.c.head_stride;
    Place mine;  // of the key whose number in the unit is the lane's
    auto fetch_places = [&](int unit) { mine = place_of(a, t, table, first_key(t, unit, KEYS) + lane); };
    auto fetch = [&](int to) {
      const int64_t at_mine = is_page(a, mine.page) ? vector_at(a, mine, head) : mine.page == -2 ? -2 : -1;
#pragma unroll
      for (int i = 0; i < PASSES; i++) {
        const int64_t at = __shfl((long long)at_mine, PASS * i + row_in);
        const uint32_t lds = wave_at + to * STAGE + i * (PASS * PER_ROW * 16);
        if (at >= 0 && k_loads) load_to_lds(K + at + k_vec * 8, lds);
        if (at >= 0 && v_loads) load_to_lds(V + at + v_vec * 8, lds + 2 * STAGE);
        if (at < 0) {
          if (k_loads) sh.keys[to][PASS * i + row_in][place] = at == -1 ? nan8<T>() : zero8<T>();
          if (v_loads) sh.values[to][PASS * i + row_in][place] = zero8<T>();
        }
      }
    };
    F16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 16; e++) o[d][e] = 0.f;
    float m = NEG_INF, sum = 0.f;
    const int end = w.unit + take;
    fetch_places(w.unit);
    fetch(turn);
    if (w.unit + 1 < end) fetch_places(w.unit + 1);
    for (int unit = w.unit; unit < end; unit++) {
      loads_done();
      if (unit + 1 < end) {
        fetch(turn ^ 1);
        if (unit + 2 < end) fetch_places(unit + 2);
      }
      const int k0 = first_key(t, unit, KEYS);
      const int64_t begin_low = a.s.window ? (int64_t)low - a.s.window + 1 : 0, begin_high = a.s.window ? (int64_t)high - a.s.window + 1 : 0;
      // values of keys that only some tokens see must not reach the others through 0 * NaN:
      // they are 0 in the product and added to those who see them
      uint64_t bad = 0;
      if (t.tokens > 1 && !all_seen(a, t, k0, KEYS)) {
        if (tid == 0) *spoiled = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PASSES; i++) {
          Vec8<T> v = sh.values[turn][PASS * i + row_in][place];
          const uint32_t bits = v_loads ? not_finite(v) : 0;
          if (bits) {
            atomicOr(spoiled, 1ull << (PASS * i + row_in));
#pragma unroll
            for (int e = 0; e < 8; e++)
              if (bits >> e & 1) v[e] = (T)0.f;
            sh.values[turn][PASS * i + row_in][place] = v;
          }
        }
        __syncthreads();
        bad = (uint64_t)uniform((int64_t)*spoiled);
      }
      const bool any = wave_rows > 0 && k0 <= high && (k0 + KEYS > begin_low || k0 < a.s.sinks || begin_low > a.capacity);
      if (any) {
        F16 s[2];
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 16; e++) s[i][e] = 0.f;
        // Reads stay a group of products ahead (of its own accord the compiler reads
        // right before each product and waits: 1,390 us for 1,258): two steps of keys,
        // then four tiles of values.
        Vec8<T> k[2][4], v[2][DT];
        auto read_keys = [&](int kk, Vec8<T>* to) {
#pragma unroll
          for (int i = 0; i < 4; i++) to[i] = sh.keys[turn][32 * (i & 1) + col][(2 * (kk + (i >> 1))) ^ k_in];
        };
        auto read_values = [&](int i, Vec8<T>* to) {
#pragma unroll
          for (int d = 0; d < DT; d++) {
            const T* from = reinterpret_cast<const T*>(&sh.values[turn][16 * i + v_row][(4 * d) ^ v_in]) + (lane & 1) * 4;
            to[d] = both<T>(transposed(from), transposed(from + 8 * PER_ROW * 8));
          }
        };
        read_keys(0, k[0]);
#pragma unroll
        for (int kk = 0; kk < KK; kk += 2) {
          if (kk + 2 < KK) read_keys(kk + 2, k[(kk / 2 + 1) & 1]);
          else read_values(0, v[0]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < 4; i++) s[i & 1] = product32(k[kk / 2 & 1][i], q[kk + (i >> 1)], s[i & 1]);
          __builtin_amdgcn_sched_barrier(0);
        }
        const bool whole = k0 + KEYS <= t.last + 1 && k0 + KEYS - 1 <= low && (k0 >= begin_high || k0 + KEYS <= a.s.sinks);
        if (!whole) {
          const uint64_t seen = seen_bits(a, position, k0, KEYS) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 2; i++) {
            const uint32_t word = (uint32_t)(seen >> (32 * i));
#pragma unroll
            for (int e = 0; e < 16; e++) s[i][e] = word & 1u << (8 * (e / 4) + e % 4) ? s[i][e] : NEG_INF;
          }
        }
        float top = NEG_INF;
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 16; e++) top = fmaxf(top, s[i][e]);
        top *= c;
        float base = m == NEG_INF ? 0.f : m;
        if (__ballot(rises<T>(m, top) || fabsf(m) >= PLAIN_MOST)) {
          top = fmaxf(top, __shfl_xor(top, 32));
          top = rises<T>(m, top) ? top - HEAD<T> : m;  // (a row's own choice: its result does not depend on its neighbours)
          const float f = top == m ? 1.f : __builtin_amdgcn_exp2f(m - top);
          m = top;
          sum *= f;
#pragma unroll
          for (int d = 0; d < DT; d++) o[d] *= f;
          base = m == NEG_INF ? 0.f : m;
          // One multiply-add gives an exponent, by the exact product of score and scale.  m is
          // rounded, and half its last place is what the largest weight would be off by, to
          // overflow: far maxima's exponents are the difference of rounded products, brought
          // to the form that the multiply-add takes.
          if (fabsf(base) >= PLAIN_MOST) {
            const float back = 1.f / c;
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
              for (int e = 0; e < 16; e++) s[i][e] = (rounded(s[i][e], c) - base) * back;
            base = 0.f;
          }
        }
        // (the exponentials of a step's weights are between the products of the last one:
        // with one place found by a lane instead of a row's by 16, 1,258 us -> 1,204.  The
        // additions to the row's sum are not: the compiler puts a tile's 32 behind its last
        // product, in one chain)
        Vec8<T> weights[2];
        auto weigh = [&](int i) {
#pragma unroll
          for (int e = 0; e < 8; e++) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i / 2][i % 2 * 8 + e], c, -base));
            sum += x;
            weights[i & 1][e] = (T)x;
          }
        };
        weigh(0);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          if (i < 3) read_values(i + 1, v[(i + 1) & 1]);
          __builtin_amdgcn_sched_barrier(0);
          if (i < 3) weigh(i + 1);
#pragma unroll
          for (int d = 0; d < DT; d++) o[d] = product32(v[i & 1][d], weights[i & 1], o[d]);
#pragma unroll
          for (int d = 0; d < DT; d++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, 28 / DT, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        for (; bad; bad &= bad - 1) {
          const int key = k0 + __builtin_ctzll(bad);
          const Place x = place_of(a, t, table, key);
          if (!is_page(a, x.page) || !sees(a, position, key)) continue;
          const T* value = V + vector_at(a, x, head) + 4 * half;
#pragma unroll
          for (int d = 0; d < DT; d++)
#pragma unroll
            for (int e = 0; e < 16; e += 4) add_not_finite(value + d * 32 + 2 * e, d * 32 + 2 * e + 4 * half < dim, &o[d], e);
        }
      }
      turn ^= 1;
    }
    sum += __shfl_xor(sum, 32);
    const bool began = w.unit > 0, ends = end == t.units;
    if (!began && ends) {
      const bool none = position < 0;
      if (live) {
        const float f = none ? 0.f : 1.f / sum;
        T* out = static_cast<T*>(a.s.out) + q_row * a.s.out_stride + q_head * dim + half * 4;
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float x[4] = {o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
            if (d * 32 + 2 * e + half * 4 < dim) store4(out + d * 32 + 2 * e, x, f, a.vectors);
          }
        if (a.s.logsums && half == 0) a.s.logsums[q_row * a.s.q_heads + q_head] = none ? NEG_INF : (m == NEG_INF ? 0.f : m) * LN2 + logf(sum);
      }
    } else {
      float* piece = piece_of(a, p, worker, began ? 0 : 1);
      if (live) {
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const int at = d * 32 + 2 * e + half * 4;
            if (at < dim) *reinterpret_cast<F4*>(piece + (int64_t)row * dim + at) = F4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
          }
        if (half == 0) *reinterpret_cast<float2*>(piece + (int64_t)p.rows * dim + 2 * row) = float2{m, sum};
      }
      if (!began) {
        leaf.pieces = 1 + (int)divided(t.units - end + w.size - 1, w.size);
        leaf.row0 = t.row0;
        leaf.tokens = t.tokens;
        leaf.head = w.head;
        leaf.low = t.low;
      }
    }
    w.left -= take;
    if (w.left > 0) w.next(a, p);
  }
  if (tid == 0) leaves_of(a)[worker] = leaf;
}

template <class T, int DP>
__global__ __launch_bounds__(ATT_THREADS, DP <= 128 ? 2 : 1) void attention_kernel(AttentionArgs a) {
  __shared__ __align__(16) union {
    Search search;
    SmallShared<T, DP / 32> small;
    LargeShared<T, DP> large;
  } sh;
  __shared__ Start starts[ATT_WAVES];
  __shared__ unsigned long long spoiled;
  const bool small = few_rows(a, sh.search);
  if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<int32_t*>(a.parts) = small;
  if (small) small_path<T, DP / 32>(a, sh.search, sh.small, starts);
  else large_path<T, DP>(a, sh.search, sh.large, starts, &spoiled);
}

// ---- joins the pieces of items that several workers have ----------------------------

// A block looks after every 256th worker (neighbours begin items together); the blocks of one x share the rows of the
// items that these begin and others go on.  Groups of lanes take a row each, or, where
// an item has many pieces, all of them one row, each every n-th piece.
constexpr int JOIN_X = 256, JOIN_Y = 4, JOIN_MOST = 2048 / JOIN_X;
template <class T>
__global__ __launch_bounds__(ATT_THREADS) void join_kernel(AttentionArgs a, int lanes) {
  __shared__ F4 sums[ATT_THREADS];
  __shared__ float2 heads[ATT_THREADS];
  // (a dependent load takes a microsecond or two here: the leaves come with the word
  // that says how many there are)
  int32_t counts[JOIN_MOST];
#pragma unroll
  for (int i = 0; i < JOIN_MOST; i++) counts[i] = leaves_of(a)[min((int)blockIdx.x + i * JOIN_X, a.small.workers - 1)].pieces;
  const bool small = *reinterpret_cast<const int32_t*>(a.parts) != 0;
  const Plan& p = small ? a.small : a.large;
  const int tid = threadIdx.x, dim = a.c.dim, each = p.workers / JOIN_X;
  const int groups = ATT_THREADS / lanes, group = tid / lanes, at = (tid - group * lanes) * 4;
  int turn = 0;  // tasks before this item's
  // (a piece that is all NaN has no maximum: its sums count as they are)
  auto weight = [](float x, float y, float top) { return x == NEG_INF ? (y != y ? 1.f : 0.f) : __builtin_amdgcn_exp2f(x - top); };
  for (int k = 0; k < each; k++) {
    int pieces = counts[0];
#pragma unroll
    for (int i = 1; i < JOIN_MOST; i++) pieces = i == k ? counts[i] : pieces;
    if (!pieces) continue;
    const int worker = blockIdx.x + k * JOIN_X, most = (p.workers - 1 - worker) / p.stride + 1;
    if (pieces > most) pieces = most;
    const Leaf leaf = leaves_of(a)[worker];
    const int kv = leaf.head / p.groups, h0 = (leaf.head - kv * p.groups) * p.heads;
    const bool many = pieces > 2 * groups;
    const int rows = leaf.tokens * p.heads, share = many ? 1 : groups;  // rows at a time
    const int tasks = (rows + share - 1) / share;
    for (int task = (int)((blockIdx.y + JOIN_Y - turn % JOIN_Y) % JOIN_Y); task < tasks; task += JOIN_Y) {
      const int row = many ? task : task * share + group;
      const int token = row / p.heads, head = row - token * p.heads;
      const bool mine = row < rows && head < a.per_kv - h0 && at < dim;
      float m = NEG_INF, sum = 0.f;
      F4 o = {0.f, 0.f, 0.f, 0.f};
      auto add = [&](auto ahead, int begin, int step) {
        constexpr int AHEAD = decltype(ahead)::value;  // pieces under way at once
        for (int i0 = begin; i0 < pieces; i0 += AHEAD * step) {
          float2 h[AHEAD];
          F4 x[AHEAD];
#pragma unroll
          for (int u = 0; u < AHEAD; u++) {
            const int i = i0 + u * step;
            h[u] = float2{NEG_INF, 0.f};
            x[u] = F4{0.f, 0.f, 0.f, 0.f};
            if (i < pieces) {
              const float* piece = piece_of(a, p, worker + i * p.stride, i ? 0 : 1);
              h[u] = *reinterpret_cast<const float2*>(piece + (int64_t)p.rows * dim + 2 * row);
              x[u] = *reinterpret_cast<const F4*>(piece + (int64_t)row * dim + at);
            }
          }
          float top = m;
#pragma unroll
          for (int u = 0; u < AHEAD; u++) top = fmaxf(top, h[u].x);
          const float f = weight(m, sum, top);
          sum *= f;
          o *= f;
#pragma unroll
          for (int u = 0; u < AHEAD; u++) {
            const float g = weight(h[u].x, h[u].y, top);
            sum += h[u].y * g;
            o += x[u] * g;
          }
          m = top;
        }
      };
      if (mine) {
        if (many) add(std::integral_constant<int, 8>{}, group, groups);
        else add(std::integral_constant<int, 4>{}, 0, 1);
      }
      if (many) {
        __syncthreads();
        sums[tid] = o;
        heads[tid] = float2{m, sum};
        __syncthreads();
        if (group != 0 || !mine) continue;
        float top = m;
        for (int g = 1; g < groups; g++) top = fmaxf(top, heads[g * lanes + tid].x);
        o = F4{0.f, 0.f, 0.f, 0.f};
        sum = 0.f;
        for (int g = 0; g < groups; g++) {
          const float2 h = heads[g * lanes + tid];
          const float f = weight(h.x, h.y, top);
          sum += h.y * f;
          o += sums[g * lanes + tid] * f;
        }
        m = top;
      }
      if (!mine) continue;
      const bool none = leaf.low + token < 0;
      const int64_t q_row = leaf.row0 + token, q_head = (int64_t)kv * a.per_kv + h0 + head;
      const float x[4] = {o[0], o[1], o[2], o[3]};
      store4(static_cast<T*>(a.s.out) + q_row * a.s.out_stride + q_head * dim + at, x, none ? 0.f : 1.f / sum, a.vectors);
      if (a.s.logsums && at == 0) a.s.logsums[q_row * a.s.q_heads + q_head] = none ? NEG_INF : (m == NEG_INF ? 0.f : m) * LN2 + logf(sum);
    }
    turn += tasks;
  }
}

// ---- the calls ----------------------------------------------------------------------

constexpr int BLOCKS = 512;  // two a compute unit; heads of more than 128 elements: one

Plan plan_of(bool small, int32_t q_heads, int32_t kv_heads, int32_t dim) {
  const int per_kv = q_heads / kv_heads;
  Plan p;
  p.rows = small ? SMALL_ROWS : 128;
  p.keys = small ? 32 : 64;
  p.workers = BLOCKS / (dim > 128 ? 2 : 1) * (small ? ATT_WAVES : 1);
  p.least = small ? 1 : 4;  // (a prompt of 700 tokens 46 us, with 1 unit 53; 4 requests of 700, 5 tokens each 24.4 and 21.8)
  p.heads = per_kv < p.rows ? per_kv : p.rows;
  p.groups = (per_kv + p.heads - 1) / p.heads;
  p.tokens = p.rows / p.heads;
  p.by_tokens = Quotient((uint32_t)p.tokens);
  const int heads = kv_heads * p.groups;
  p.stride = heads <= p.workers ? heads : 1;
  p.parts = p.workers / p.stride;
  return p;
}

int64_t room_of(const Plan& p, int dim) { return leaves_bytes(p.workers) + 2 * (int64_t)p.workers * piece_floats(p.rows, dim) * 4; }

template <class T>
int run_attention(const AttentionArgs& a, hipStream_t st) {
  const int kk = (a.c.dim + 31) / 32;
  int lanes = 8;  // of a row in the join
  while (lanes * 4 < a.c.dim) lanes *= 2;
  auto* kernel = kk <= 2 ? attention_kernel<T, 64> : kk == 3 ? attention_kernel<T, 96> : kk == 4 ? attention_kernel<T, 128> : attention_kernel<T, 256>;
  if (launch(kernel, dim3(a.large.workers), dim3(ATT_THREADS), st, a) != hipSuccess) return TT_ERR_HIP;
  return launch(join_kernel<T>, dim3(JOIN_X, JOIN_Y), dim3(ATT_THREADS), st, a, lanes) == hipSuccess ? TT_OK : TT_ERR_HIP;
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int64_t tt_cache_attention_workspace(int64_t tokens, int32_t n_requests, int32_t q_heads, int32_t kv_heads,
                                                int32_t dim) {
  if (tokens < 0 || tokens > INT32_MAX || n_requests < 0 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || dim < 8 ||
      dim > TT_MAX_HEAD_DIM || dim % 8)
    return TT_ERR_BAD_ARG;
  if (tokens == 0 || n_requests == 0) return 0;
  const int64_t small = room_of(plan_of(true, q_heads, kv_heads, dim), dim), large = room_of(plan_of(false, q_heads, kv_heads, dim), dim);
  return small > large ? small : large;
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
      s.query_stride < width || s.out_stride < width || (s.out && s.out == s.queries) || (workspace && workspace_bytes < need) ||
      reinterpret_cast<uintptr_t>(workspace) % 256)
    return TT_ERR_BAD_ARG;
  if (s.tokens == 0 || s.n_requests == 0) return TT_OK;
  if (bad) return bad;
  if (!s.offsets || !s.lengths || (s.table_width > 0 && !s.tables) || !s.queries || !s.out || !workspace) return TT_ERR_NULL_ARG;
  // slots of items are numbered in 32 bits
  if (s.tokens + s.n_requests > INT32_MAX || cache->page_stride / 8 > UINT32_MAX || cache->slot_stride / 8 > UINT32_MAX)
    return TT_ERR_TOO_LARGE;
  auto in_vectors = [](const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; };
  const int64_t capacity = (int64_t)s.table_width * cache->page_size;
  const AttentionArgs a{*cache,
                  s,
                  (int)(capacity < INT32_MAX - 64 ? capacity : INT32_MAX - 64),
                  plan_of(true, s.q_heads, cache->kv_heads, cache->dim),
                  plan_of(false, s.q_heads, cache->kv_heads, cache->dim),
                  Quotient((uint32_t)cache->page_size),
                  (uint32_t)(cache->page_stride / 8),
                  (uint32_t)(cache->slot_stride / 8),
                  s.q_heads / cache->kv_heads,
                  in_vectors(s.queries, s.query_stride) && in_vectors(s.out, s.out_stride),
                  // at most this many items of a head unit, units of an item and head units (8,192 tokens
                  // of 1,000 requests, tables of 131,072: 160 us, found with short sums 153; of 4 prompts 303 both)
                  s.n_requests > STAGED || (double)(s.tokens + s.n_requests) * ((double)capacity / 32 + 3) * s.q_heads * 2 >= INT32_MAX,
                  static_cast<uint8_t*>(workspace)};
  return cache->type == TT_BF16 ? run_attention<bf16_t>(a, static_cast<hipStream_t>(stream))
                                : run_attention<f16_t>(a, static_cast<hipStream_t>(stream));
}
