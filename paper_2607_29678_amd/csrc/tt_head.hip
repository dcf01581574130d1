// tt_head_scores and its gradients: scores of logits = hidden weight^T that are
// never stored, on the matrix cores.
//
// Every product here is C[m][n] = sum_k A[m][k] B[n][k] in tiles of BM x BN that
// four (or eight) waves share.  m runs over the vocabulary in the scores, so a
// lane's accumulators hold entries of one token's row and the softmax statistics
// are sums within the lane.  The gradients take the gradient of the logits G as
// it stands and hidden or weight as it stands: an operand may be contiguous in k
// or in m (or n), and LDS transposes the latter on the way to the registers.
#include "tt_scores.h"

namespace tt {
namespace {

using f32x16 = __attribute__((ext_vector_type(16))) float;

template <class T>
struct Mfma;
template <>
struct Mfma<bf16_t> {
  using V8 = __attribute__((ext_vector_type(8))) bf16_t;
  using V4 = __attribute__((ext_vector_type(4))) bf16_t;
  static __device__ __forceinline__ f32x16 mul(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<f16_t> {
  using V8 = __attribute__((ext_vector_type(8))) f16_t;
  using V4 = __attribute__((ext_vector_type(4))) f16_t;
  static __device__ __forceinline__ f32x16 mul(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// An operand: `rows` rows of k entries, or (by columns) k rows of `rows` entries.
template <class T>
struct Operand {
  const T* p;
  int64_t stride, rows;
};

constexpr int CUS = 256;  // compute units
constexpr int BK = 64;  // entries of k that are staged at once: rows of 128 bytes in LDS

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// A buffer of 2 GiB from p on: what lies past it reads as 0.
using Buffer = __attribute__((ext_vector_type(4))) uint32_t;
constexpr uint32_t BUFFER_BYTES = 0x80000000u;
__device__ __forceinline__ Buffer buffer_at(const void* p) {
  const uint64_t at = (uint64_t)(uintptr_t)p;
  return Buffer{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, BUFFER_BYTES, 0x00020000u};
}
// 16 bytes a lane from the buffer's byte `offset` to LDS, at `to` + 16 lane.
// Written as assembly, since for the builtin the compiler makes every later
// read of LDS wait for the load; there is no result register.  It takes a wait
// state from the write of m0 to its use, and five from a vector instruction's
// write of a scalar register to a load's use of it, which the compiler does not
// look after in here.
// ONCE: what is read once does not stay in the caches.
template <bool ONCE = false>
__device__ __forceinline__ void load_to_lds(Buffer from, uint32_t offset, uint32_t to) {
  if (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to), "v"(offset), "s"(from) : "m0", "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(from) : "m0", "memory");
}
// Waits for all but the last N of this wave's loads and for its LDS reads, then
// for the block's other waves.
template <int N>
__device__ __forceinline__ void loads_done_but() {
  static_assert(N < 64, "field of s_waitcnt");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Four entries of one column each lane: within 16 lanes, lane l reads four
// entries of row l / 4 and receives column l of the 4 x 16 block.
template <class V4>
__device__ __forceinline__ V4 read_transposed(const void* p) {
  using S4 = __attribute__((ext_vector_type(4))) short;
  return __builtin_bit_cast(V4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4*)p));
}

// AC, BC: the operand is contiguous in m (n) instead of in k
template <class T, int BM_, int BN_, int WM_, int WN_, bool VEC_, bool AC = false, bool BC = false>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr bool VEC = VEC_;  // rows are aligned to 16 bytes and k is a multiple of 8
  static constexpr bool DIRECT = VEC && BM == 256 && BN >= 128;
  static constexpr int THREADS = 64 * WM * WN;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // 32 x 32 products of a wave
  using Elem = T;
  using V8 = typename Mfma<T>::V8;
  using V4 = typename Mfma<T>::V4;
  static constexpr int NA = BM * 8 / THREADS, NB = BN * 8 / THREADS;  // 16-byte pieces a thread stages
  static_assert(NA * THREADS == BM * 8 && NB * THREADS == BN * 8, "whole pieces");
  struct Shared {
    T a[2][BM * BK], b[2][BN * BK];
  };

  // Piece q of a stage: row q / 8, entries 8 (q % 8) and on.  In LDS the pieces
  // of a row are permuted by the row's number, so that the 16 rows that are read
  // at a time (two of them fill the 64 banks) lie in different banks.
  static __device__ __forceinline__ int twist(int row) { return row >> 1 & 7; }
  static __device__ __forceinline__ int place(int row, int piece) { return row * BK + ((piece ^ twist(row)) << 3); }

  // An operand by columns is staged as 64 rows of BM (BN) entries; blocks of 32
  // entries are permuted by this, so that the four rows that half a wave reads
  // at a time lie in different banks.
  static __device__ __forceinline__ int spread(int row) { return row & 3; }

  static __device__ __forceinline__ V8 load(const Operand<T>& o, int64_t row, int64_t k, int64_t k_end) {
    V8 v = {};
    if (VEC) {
      if (row < o.rows && k < k_end) v = *reinterpret_cast<const V8*>(o.p + row * o.stride + k);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (row < o.rows && k + i < k_end) v[i] = o.p[row * o.stride + k + i];
    }
    return v;
  }

  static __device__ __forceinline__ void multiply(const Operand<T>& a, const Operand<T>& b, int64_t m0, int64_t n0,
                                                  int64_t k0, int64_t k1, Shared& sh, f32x16 (&acc)[TM][TN]) {
    if constexpr (DIRECT) multiply_direct(a, b, m0, n0, k0, k1, sh, acc);
    else multiply_staged(a, b, m0, n0, k0, k1, sh, acc);
  }

  // acc = A[m0 ..][k0, k1) B[n0 ..][k0, k1); ends with every wave past its last read of sh
  static __device__ __forceinline__ void multiply_staged(const Operand<T>& a, const Operand<T>& b, int64_t m0, int64_t n0,
                                                  int64_t k0, int64_t k1, Shared& sh, f32x16 (&acc)[TM][TN]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
      for (int j = 0; j < TN; j++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    V8 ra[NA], rb[NB];
    auto fetch = [&](int64_t k) {
#pragma unroll
      for (int i = 0; i < NA; i++) {
        const int q = tid + i * THREADS;
        ra[i] = load(a, m0 + (q >> 3), k + (q & 7) * 8, k1);
      }
#pragma unroll
      for (int i = 0; i < NB; i++) {
        const int q = tid + i * THREADS;
        rb[i] = load(b, n0 + (q >> 3), k + (q & 7) * 8, k1);
      }
    };
    auto stage = [&](int buf) {
#pragma unroll
      for (int i = 0; i < NA; i++) {
        const int q = tid + i * THREADS;
        *reinterpret_cast<V8*>(&sh.a[buf][place(q >> 3, q & 7)]) = ra[i];
      }
#pragma unroll
      for (int i = 0; i < NB; i++) {
        const int q = tid + i * THREADS;
        *reinterpret_cast<V8*>(&sh.b[buf][place(q >> 3, q & 7)]) = rb[i];
      }
    };
    const int steps = (int)((k1 - k0 + BK - 1) / BK);
    fetch(k0);
    stage(0);
    __syncthreads();
    for (int s = 0; s < steps; s++) {
      if (s + 1 < steps) fetch(k0 + (int64_t)(s + 1) * BK);
      const T *la = sh.a[s & 1], *lb = sh.b[s & 1];
#pragma unroll
      for (int kk = 0; kk < BK / 16; kk++) {
        V8 fa[TM], fb[TN];
#pragma unroll
        for (int i = 0; i < TM; i++)
          fa[i] = *reinterpret_cast<const V8*>(&la[place(wm * TM * 32 + i * 32 + (lane & 31), kk * 2 + (lane >> 5))]);
#pragma unroll
        for (int j = 0; j < TN; j++)
          fb[j] = *reinterpret_cast<const V8*>(&lb[place(wn * TN * 32 + j * 32 + (lane & 31), kk * 2 + (lane >> 5))]);
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int j = 0; j < TN; j++) acc[i][j] = Mfma<T>::mul(fa[i], fb[j], acc[i][j]);
      }
      if (s + 1 < steps) stage((s + 1) & 1);
      __syncthreads();
    }
  }

  // The same for aligned operands, with the pieces loaded straight into LDS.
  // The rows of a fragment for the next 16 entries of k are read while the
  // matrix cores work on the last ones, across the change of stages too: the
  // barrier stands before the last products of a stage, when its fragments are
  // in registers, and the stage's buffer is then filled for the stage after the
  // next.  Rows past an operand's last and entries past k1 are read as zeros;
  // so are the two stages past the last, which keeps the loop free of branches.
  static constexpr int WAVES = WM * WN, DA = BM / 8 / WAVES, DB = BN / 8 / WAVES;  // loads of 8 rows by a wave
  static __device__ __forceinline__ void multiply_direct(const Operand<T>& a, const Operand<T>& b, int64_t m0, int64_t n0,
                                                         int64_t k0, int64_t k1, Shared& sh, f32x16 (&acc)[TM][TN]) {
    static_assert(VEC && DA * WAVES * 8 == BM && DB * WAVES * 8 == BN, "whole loads");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // Byte offsets of this lane's pieces from the tile's first entry, and the
    // entries of k that a piece has left at stage 0.
    uint32_t oa[DA], ob[DB];
    // (by columns a load holds 512 / BM rows: row_in() of its first row on)
    auto row_in = [&](int load, int columns) { return load * (512 / columns) + lane / (columns / 8); };
    auto offset = [&](const Operand<T>& o, int64_t first, int load, int columns, auto by_columns) {
      if (decltype(by_columns)::value) {
        const int64_t row = row_in(load, columns);
        const int64_t col = (((lane % (columns / 8) >> 2) ^ spread((int)row)) << 5) + (lane & 3) * 8;
        return first + col < o.rows ? (uint32_t)(row * o.stride + col) * 2 : BUFFER_BYTES;
      }
      const int64_t row = load * 8 + (lane >> 3);  // eight rows of 64 entries
      return first + row < o.rows ? (uint32_t)(row * o.stride + ((lane & 7) ^ twist((int)row)) * 8) * 2 : BUFFER_BYTES;
    };
    using A = std::integral_constant<bool, AC>;
    using B = std::integral_constant<bool, BC>;
#pragma unroll
    for (int i = 0; i < DA; i++) oa[i] = offset(a, m0, wave * DA + i, BM, A{});
#pragma unroll
    for (int i = 0; i < DB; i++) ob[i] = offset(b, n0, wave * DB + i, BN, B{});
    const T* pa = AC ? a.p + k0 * a.stride + m0 : a.p + m0 * a.stride + k0;
    const T* pb = BC ? b.p + k0 * b.stride + n0 : b.p + n0 * b.stride + k0;
    const int64_t next_a = AC ? BK * a.stride : BK, next_b = BC ? BK * b.stride : BK;
    const uint32_t la = __builtin_amdgcn_readfirstlane(lds_address(sh.a) + wave * DA * 1024);
    const uint32_t lb = __builtin_amdgcn_readfirstlane(lds_address(sh.b) + wave * DB * 1024);
    // From the stage on that is not full, pieces past k1 are moved out of the buffer.
    const int full_stages = (int)((k1 - k0) / BK), rest = (int)((k1 - k0) % BK);
    auto cut = [&](int stage) {
      const int here = stage > full_stages ? 0 : rest;
      auto past = [&](int load, int columns, auto by_columns) {
        const int row = decltype(by_columns)::value ? row_in(load, columns) : load * 8 + (lane >> 3);
        return (decltype(by_columns)::value ? row : ((lane & 7) ^ twist(row)) * 8) >= here;
      };
#pragma unroll
      for (int i = 0; i < DA; i++)
        if (past(wave * DA + i, BM, A{})) oa[i] = BUFFER_BYTES;
#pragma unroll
      for (int i = 0; i < DB; i++)
        if (past(wave * DB + i, BN, B{})) ob[i] = BUFFER_BYTES;
    };
    Buffer ba = buffer_at(pa), bb = buffer_at(pb);
    auto load_piece = [&](int stage, int i) {  // loads 0 .. DA + DB - 1 of a stage
      const uint32_t at = stage & 1;
      if (i < DA) load_to_lds(ba, oa[i < DA ? i : 0], la + at * (BM * BK * 2) + i * 1024);
      else load_to_lds(bb, ob[i < DA ? 0 : i - DA], lb + at * (BN * BK * 2) + (i - DA) * 1024);
    };
    // the buffers and offsets of a stage; stages are loaded in order
    auto begin_stage = [&](int stage) {
      ba = buffer_at(pa + stage * next_a);
      bb = buffer_at(pb + stage * next_b);
      if (stage >= full_stages) cut(stage);
    };
    V8 fa[2][TM], fb[2][TN];
    // fragment of rows (columns) 32 i .. 32 i + 31 from `first` on, 16 entries of k from 16 kk on
    auto fragment = [&](const T* p, int first, int kk, int columns, auto by_columns) {
      if (decltype(by_columns)::value) {
        const int row = kk * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
        const T* q = p + row * columns + ((((first >> 5) ^ spread(row)) << 5) | ((lane >> 4 & 1) << 4) | ((lane & 3) << 2));
        const V4 x = read_transposed<V4>(q), y = read_transposed<V4>(q + 4 * columns);
        return (V8)__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      }
      return *reinterpret_cast<const V8*>(&p[place(first + (lane & 31), kk * 2 + (lane >> 5))]);
    };
    // fragment n of the next products, in the order in which those need them
    constexpr int FRAGMENTS = TM + TN;
    auto read_one = [&](int buf, int kk, int to, int n) {
      if (n == 0 || n > TN) {
        const int i = n == 0 ? 0 : n - TN;
        fa[to][i] = fragment(sh.a[buf], wm * TM * 32 + i * 32, kk, BM, A{});
      } else {
        fb[to][n - 1] = fragment(sh.b[buf], wn * TN * 32 + (n - 1) * 32, kk, BN, B{});
      }
    };
    auto one = [&](int from, int ij) {
      const int i = ij / TN, j = ij % TN;
      acc[i][j] = Mfma<T>::mul(fa[from][i], fb[from][j], acc[i][j]);
    };
    begin_stage(0);
#pragma unroll
    for (int i = 0; i < DA + DB; i++) load_piece(0, i);
    begin_stage(1);
#pragma unroll
    for (int i = 0; i < DA + DB; i++) load_piece(1, i);
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
      for (int j = 0; j < TN; j++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    loads_done_but<DA + DB>();
#pragma unroll
    for (int n = 0; n < FRAGMENTS; n++) read_one(0, 0, 0, n);
    const int steps = (int)((k1 - k0 + BK - 1) / BK);
    int s = 0;
    // Reads and loads are issued between the products: a wave issues in order,
    // and a row of reads would leave its matrix core idle until LDS took them.
    constexpr int P = TM * TN;
    do {
#pragma unroll
      for (int kk = 0; kk < BK / 16; kk++) {
        const bool last = kk == BK / 16 - 1;
        if (last) {
          begin_stage(s + 2);
          loads_done_but<0>();
        }
#pragma unroll
        for (int ij = 0; ij < P; ij++) {
          one(kk & 1, ij);
#pragma unroll
          for (int n = ij * FRAGMENTS / P; n < (ij + 1) * FRAGMENTS / P; n++)
            read_one((last ? s + 1 : s) & 1, last ? 0 : kk + 1, (kk + 1) & 1, n);
          if (last) {
#pragma unroll
            for (int i = ij * (DA + DB) / P; i < (ij + 1) * (DA + DB) / P; i++) load_piece(s + 2, i);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } while (++s < steps);
    loads_done_but<0>();
    // What reads the accumulators by assembly has to wait for the last products
    // itself: the accumulators go through the wait, so that no product is behind
    // it and no read ahead of it.
    auto pass = [&] {
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) asm volatile("" : "+a"(acc[i][j]));
    };
    pass();
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
    pass();
  }

  // One value of an accumulator, out of an accumulation register where the
  // accumulators fill those: they stay there until each is used.
  static __device__ __forceinline__ float value(const f32x16 (&acc)[TM][TN], int i, int j, int r) {
    if (!DIRECT) return acc[i][j][r];
    float x;
    asm("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[i][j][r]));
    return x;
  }

  // Where accumulator r of product (i, j) lies: row m (four consecutive rows for
  // r = 4 g .. 4 g + 3) and column n of the tile.
  static __device__ __forceinline__ int row_of(int i, int group) {
    const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / WN;
    return wm * TM * 32 + i * 32 + group * 8 + (lane >> 5) * 4;
  }
  static __device__ __forceinline__ int col_of(int j) {
    const int lane = threadIdx.x & 63, wn = (threadIdx.x >> 6) % WN;
    return wn * TN * 32 + j * 32 + (lane & 31);
  }
};

// Tiles in an order that keeps each of the eight dies (blocks are dealt to them
// in turn) on a run of neighbouring tiles: its L2 then holds the rows of A that
// the run's tiles share.
__device__ __forceinline__ uint32_t die_order(uint32_t b, uint32_t n) {
  const uint32_t per = n / 8, rest = n % 8, die = b % 8, i = b / 8;
  return die * per + (die < rest ? die : rest) + i;
}

// (m tile, n tile) of the id-th tile: groups of eight n tiles, all m tiles of a
// group before the next, so that tiles that run together share rows of both.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t m_tiles, uint32_t n_tiles, int64_t& mt, int64_t& nt) {
  const uint32_t group = id / (m_tiles * 8), first = group * 8, width = n_tiles - first < 8 ? n_tiles - first : 8;
  const uint32_t in = id - group * m_tiles * 8;
  mt = in / width;
  nt = first + in % width;
}

// ---- forward ---------------------------------------------------------------

struct Part {
  float m, s, u, pad;
};

template <class T>
struct HeadArgs {
  Operand<T> weight, hidden;
  int64_t width;
  float scale;
  const int32_t* targets;
  Part* parts;    // [rows][vocabulary tiles]
  float* given;   // [rows] logit of the given token
  int32_t m_tiles, n_tiles;
};

// Bound by the matrix cores: 4,001 rows of 2,048 at 100,257 entries in bf16 take
// 1.47-1.52 ms with the join, 1.08-1.12 PFLOP/s (the library's plain product of 4,096 rows
// takes 1.46 and writes 0.8 GB of logits that would be read again).  Four
// waves share a tile of 256 x 256, so that each keeps 128 x 128 sums in half of its
// registers: the fewest LDS reads a product that fit.
template <class Tl>
__global__ __launch_bounds__(Tl::THREADS, Tl::DIRECT ? 1 : 2) void head_scores_kernel(HeadArgs<typename Tl::Elem> a) {
  __shared__ typename Tl::Shared sh;
  const uint32_t tile = die_order(blockIdx.x, gridDim.x);
  int64_t mt, nt;
  tile_of(tile, (uint32_t)a.m_tiles, (uint32_t)a.n_tiles, mt, nt);
  const int64_t m0 = mt * Tl::BM, n0 = nt * Tl::BN;
  const int64_t rows = a.hidden.rows;
  int targets[Tl::TN];  // (loaded ahead of the products)
#pragma unroll
  for (int j = 0; j < Tl::TN; j++) {
    const int64_t t = n0 + Tl::col_of(j);
    targets[j] = a.targets && t < rows ? a.targets[t] : -1;
  }
  f32x16 acc[Tl::TM][Tl::TN];
  Tl::multiply(a.weight, a.hidden, m0, n0, 0, a.width, sh, acc);

  const float c = a.scale * LOG2E;
  const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / Tl::WN;
  Part* joined = reinterpret_cast<Part*>(&sh);  // [WM][BN]
  const int left = a.weight.rows - m0 < Tl::BM ? (int)(a.weight.rows - m0) : Tl::BM;  // entries of this tile
  auto columns = [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      const int col = Tl::col_of(j);
      const int64_t t = n0 + col;
      // an entry's place is 32 i + 8 (r / 4) + r % 4 from the lane's first one
      int last = left - Tl::row_of(0, 0);
      const int64_t in_tile = targets[j] - m0;
      const int given = targets[j] >= 0 && in_tile >= 0 && in_tile < left ? (int)in_tile - Tl::row_of(0, 0) : -1;
      auto entry = [&](int i, int r) {
        const float x = Tl::value(acc, i, j, r);
        return WHOLE || 32 * i + 8 * (r >> 2) + (r & 3) < last ? x : NEG_INF;
      };
      // (opaque, so that the comparisons of all entries are not made ahead and kept)
      if (!WHOLE) asm volatile("" : "+v"(last));
      float m = NEG_INF;
#pragma unroll
      for (int i = 0; i < Tl::TM; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) m = larger(m, entry(i, r));
      __builtin_amdgcn_sched_barrier(0);
      const bool mine = given >= 0 && given < Tl::TM * 32 && !(given & 4);
      if (__ballot(mine)) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < Tl::TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (32 * i + 8 * (r >> 2) + (r & 3) == given) x = Tl::value(acc, i, j, r);
        if (mine) a.given[t] = x;
      }
      const float less = smaller(m, __shfl_xor(m, 32));
      m = larger(m, __shfl_xor(m, 32));
      const Reference ref = reference(m, c);
      Stats st = {m, 0.f, 0.f};
      float left_out = NEG_INF;  // (ends as the lane's largest entry)
      if (!WHOLE) asm volatile("" : "+v"(last));
      auto sums = [&](auto plain) {
#pragma unroll
        for (int i = 0; i < Tl::TM; i++) {
#pragma unroll
          for (int r = 0; r < 16; r += 2)
            add_two<decltype(plain)::value>(st, left_out, entry(i, r), entry(i, r + 1), ref, c);
          __builtin_amdgcn_sched_barrier(0);  // (the accumulators do not fit the other registers all at once)
        }
      };
      if (__ballot(!is_plain(m, c)) == 0) sums(std::true_type{});
      else sums(std::false_type{});
      st.s += __shfl_xor(st.s, 32);
      st.u += __shfl_xor(st.u, 32);
      add_entry<false>(st, less, ref, c);  // (of the two lanes' largest entries only the larger one is left out)
      if (lane < 32) joined[wm * Tl::BN + col] = {m, st.s, st.u, 0.f};
    }
  };
  if (left == Tl::BM) columns(std::true_type{});
  else columns(std::false_type{});
  __syncthreads();
  for (int col = threadIdx.x; col < Tl::BN; col += Tl::THREADS) {
    if (n0 + col >= rows) break;
    Stats st = empty_stats();
#pragma unroll
    for (int w = 0; w < Tl::WM; w++) {
      const Part& q = joined[w * Tl::BN + col];
      st = join(st, Stats{q.m, q.s, q.u}, c);
    }
    a.parts[(n0 + col) * a.m_tiles + mt] = {st.m, st.s, st.u, 0.f};
  }
}

// The same for up to 64 rows, where the weights stream through once and nothing
// else counts.  Small blocks of two waves, as many as LDS holds, take every
// so-many-th tile of 64 vocabulary entries; their stages follow each other across
// tiles, so that two of them are always under way, past the caches.
// Blocks begin at different k: rows are often a power of two apart, and blocks in
// step would ask the same few memory channels.
// Every lane keeps the statistics of its own entries of a column to the end.
// 4 rows of 2,048 at 50,257 entries: 45-47 us, 206 MB of weights at 4.5 TB/s; of
// 4,096 at 100,257, where start and end weigh less: 5.9 TB/s.  64 rows: 59 us
// (65 rows by tiles of 256 x 128: 45).
template <class T, int BN_>
struct Stream {
  using Elem = T;
  using Tl = Tile<T, 64, BN_, 2, 1, true>;
  static constexpr int BN = BN_, STAGES = 3, DA = 4, DB = BN / 16;  // loads of a wave in a stage
  static constexpr int BLOCKS = CUS * (BN == 32 ? 4 : 3);  // as many as LDS holds at once
  struct Shared {
    T a[STAGES][64 * BK], b[STAGES][BN * BK];
    Part joined[2][BN];
  };
};

template <class S>
__global__ __launch_bounds__(128, 1) void head_stream_kernel(HeadArgs<typename S::Elem> a) {
  using T = typename S::Elem;
  using Tl = typename S::Tl;
  using V8 = typename Tl::V8;
  constexpr int DA = S::DA, DB = S::DB, STAGES = S::STAGES, BN = S::BN;
  __shared__ typename S::Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int blocks = gridDim.x, steps = (int)((a.width + BK - 1) / BK);
  const int64_t vocab = a.weight.rows, rows = a.hidden.rows;
  int targets[Tl::TN];
#pragma unroll
  for (int j = 0; j < Tl::TN; j++) {
    const int64_t t = j * 32 + (lane & 31);
    targets[j] = a.targets && t < rows ? a.targets[t] : -1;
  }
  uint32_t oa[DA], ob[DB];
  auto place_of = [&](int row, int64_t stride) { return (uint32_t)(row * stride + ((lane & 7) ^ Tl::twist(row)) * 8) * 2; };
#pragma unroll
  for (int i = 0; i < DA; i++) oa[i] = place_of((wave * DA + i) * 8 + (lane >> 3), a.weight.stride);
#pragma unroll
  for (int i = 0; i < DB; i++) {
    const int row = (wave * DB + i) * 8 + (lane >> 3);
    ob[i] = row < rows ? place_of(row, a.hidden.stride) : BUFFER_BYTES;
  }
  const uint32_t la = __builtin_amdgcn_readfirstlane(lds_address(sh.a) + wave * DA * 1024);
  const uint32_t lb = __builtin_amdgcn_readfirstlane(lds_address(sh.b) + wave * DB * 1024);

  // the next stage to load
  int64_t load_m0 = (int64_t)blockIdx.x * 64;
  const int phase = blockIdx.x % steps, whole = (int)(a.width / BK);
  int load_i = 0, load_k = phase, load_buf = 0;
  const T* load_tile = a.weight.p + load_m0 * a.weight.stride;
  auto load_stage = [&] {
    const Buffer ba = buffer_at(load_tile + load_k * BK), bb = buffer_at(a.hidden.p + load_k * BK);
    const uint32_t ta = la + load_buf * (64 * BK * 2), tb = lb + load_buf * (BN * BK * 2);
    if (load_m0 + 64 <= vocab && load_k < whole) {
#pragma unroll
      for (int i = 0; i < DA; i++) load_to_lds<true>(ba, oa[i], ta + i * 1024);
#pragma unroll
      for (int i = 0; i < DB; i++) load_to_lds(bb, ob[i], tb + i * 1024);
    } else {  // the last entries of k or of the vocabulary, and the stages past the last tile: zeros behind them
      const int64_t k_left = a.width - (int64_t)load_k * BK, rows_left = vocab - load_m0;
#pragma unroll
      for (int i = 0; i < DA; i++) {
        const int row = (wave * DA + i) * 8 + (lane >> 3);
        const bool real = ((lane & 7) ^ Tl::twist(row)) * 8 < k_left && row < rows_left;
        load_to_lds<true>(ba, real ? oa[i] : BUFFER_BYTES, ta + i * 1024);
      }
#pragma unroll
      for (int i = 0; i < DB; i++) {
        const int row = (wave * DB + i) * 8 + (lane >> 3);
        const bool real = ((lane & 7) ^ Tl::twist(row)) * 8 < k_left && rows_left > 0;
        load_to_lds(bb, real ? ob[i] : BUFFER_BYTES, tb + i * 1024);
      }
    }
    load_buf = load_buf == STAGES - 1 ? 0 : load_buf + 1;
    if (++load_k == steps) load_k = 0;
    if (++load_i == steps) {
      load_i = 0;
      load_m0 += (int64_t)blocks * 64;
      load_tile += (int64_t)blocks * 64 * a.weight.stride;
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; i++) load_stage();

  const float c = a.scale * LOG2E;
  Stats st[Tl::TN];
#pragma unroll
  for (int j = 0; j < Tl::TN; j++) st[j] = empty_stats();
  int buf = 0;
  for (int64_t m0 = (int64_t)blockIdx.x * 64; m0 < vocab; m0 += (int64_t)blocks * 64) {
    f32x16 acc[Tl::TN], odd[Tl::TN];  // (two sums: a product need not wait for the last one)
#pragma unroll
    for (int j = 0; j < Tl::TN; j++)
#pragma unroll
      for (int r = 0; r < 16; r++) acc[j][r] = odd[j][r] = 0.f;
    for (int k = 0; k < steps; k++) {
      loads_done_but<(STAGES - 2) * (DA + DB)>();  // this stage is here, and both waves are past the last one
      V8 fa[BK / 16], fb[Tl::TN][BK / 16];
#pragma unroll
      for (int kk = 0; kk < BK / 16; kk++) {
        fa[kk] = *reinterpret_cast<const V8*>(&sh.a[buf][Tl::place(wave * 32 + (lane & 31), kk * 2 + (lane >> 5))]);
#pragma unroll
        for (int j = 0; j < Tl::TN; j++)
          fb[j][kk] = *reinterpret_cast<const V8*>(&sh.b[buf][Tl::place(j * 32 + (lane & 31), kk * 2 + (lane >> 5))]);
      }
      load_stage();
#pragma unroll
      for (int kk = 0; kk < BK / 16; kk += 2)
#pragma unroll
        for (int j = 0; j < Tl::TN; j++) {
          acc[j] = Mfma<T>::mul(fa[kk], fb[j][kk], acc[j]);
          odd[j] = Mfma<T>::mul(fa[kk + 1], fb[j][kk + 1], odd[j]);
        }
      buf = buf == STAGES - 1 ? 0 : buf + 1;
    }
#pragma unroll
    for (int j = 0; j < Tl::TN; j++)
#pragma unroll
      for (int r = 0; r < 16; r++) acc[j][r] += odd[j][r];
    const int64_t mine = m0 + wave * 32 + (lane >> 5) * 4;  // entry 8 (r / 4) + r % 4 from here on
    const int last = vocab - mine < 32 ? (int)(vocab - mine) : 32;
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      const int64_t given = targets[j] - mine;
      float m = st[j].m;
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const int at = 8 * (r >> 2) + (r & 3);
        if (at == given) a.given[j * 32 + (lane & 31)] = acc[j][r];
        if (at >= last) acc[j][r] = NEG_INF;
        m = larger(m, acc[j][r]);
      }
      float left_out = st[j].m;
      lower(st[j], m, c);
      const Reference ref = reference(m, c);
#pragma unroll
      for (int r = 0; r < 16; r += 2) add_two<false>(st[j], left_out, acc[j][r], acc[j][r + 1], ref, c);
    }
  }
  loads_done_but<0>();
#pragma unroll
  for (int j = 0; j < Tl::TN; j++) {
    const Stats o = {__shfl_xor(st[j].m, 32), __shfl_xor(st[j].s, 32), __shfl_xor(st[j].u, 32)};
    st[j] = join(st[j], o, c);
    if (lane < 32) sh.joined[wave][j * 32 + lane] = {st[j].m, st[j].s, st[j].u, 0.f};
  }
  __syncthreads();
  if (tid < BN && tid < rows) {
    const Part &p = sh.joined[0][tid], &q = sh.joined[1][tid];
    const Stats all = join(Stats{p.m, p.s, p.u}, Stats{q.m, q.s, q.u}, c);
    a.parts[tid * blocks + blockIdx.x] = {all.m, all.s, all.u, 0.f};
  }
}

// Joins a row's parts: one wave per row.
__global__ __launch_bounds__(256) void head_join_kernel(const Part* parts, const float* given, int32_t n_parts,
                                                        int64_t rows, int64_t vocab, float scale, const int32_t* targets,
                                                        float* logprobs, float* stats, float* entropy) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  const float c = scale * LOG2E;
  const int32_t t = targets ? targets[row] : -1;
  const float x_given = t >= 0 && t < vocab ? given[row] : 0.f;
  Stats st = empty_stats();
  constexpr int U = 8;
  for (int i = lane; i - lane < n_parts; i += 64 * U) {
    Part q[U];
#pragma unroll
    for (int k = 0; k < U; k++) q[k] = i + 64 * k < n_parts ? parts[row * n_parts + i + 64 * k] : Part{NEG_INF, 0.f, 0.f, 0.f};
    float m = st.m;
#pragma unroll
    for (int k = 0; k < U; k++) m = larger(m, q[k].m);
    float left_out = st.m;
    lower(st, m, c);
    const Reference ref = reference(m, c);
#pragma unroll
    for (int k = 0; k < U; k++) {
      Stats o = {q[k].m, q[k].s, q[k].u};
      lower(o, m, c);
      st.s += o.s;
      st.u += o.u;
      add_entry<false>(st, smaller(left_out, q[k].m), ref, c);
      left_out = larger(left_out, q[k].m);
    }
  }
  st = wave_join(st, st.m, c);
  if (lane) return;
  const RowScores r = row_scores(st, c);
  if (logprobs) logprobs[row] = given_log_prob(t, vocab, x_given, r, scale);
  if (stats) {
    stats[2 * row] = r.m;
    stats[2 * row + 1] = r.log_s;
  }
  if (entropy) entropy[row] = r.entropy;
}

// ---- gradients -------------------------------------------------------------

// What G is multiplied by before it is rounded, and its inverse.  The largest
// gradient of a log probability becomes a power of two: where all rows have the
// same one (a mean over rows), its rounding would be in every entry of G alike and
// not average out (2.2 times the results' own rounding at 1 / 510 in bf16).  And
// the largest possible entry comes to 2^12 to 2^13, as 16-bit floats hold up to 65,504
// and lose small entries below 2^-14.
// Only gradients that row_grad() passes on count: what stands at a row without a
// token, or in a row whose G is 0 or no number, must not take the others' bits.
// One block, which has little to do but wait for its loads: those of four rows a
// thread are under way at once (2,048 rows 5.3 us, 16,384 18.7).
constexpr int SCALE_THREADS = 1024;
__global__ __launch_bounds__(SCALE_THREADS) void grad_scale_kernel(int64_t rows, int64_t vocab, float most_entropy,
                                                                   float scale, const int32_t* targets,
                                                                   const float* stats, const float* grad_logprobs,
                                                                   const float* grad_entropy, float* out) {
  constexpr int U = 4, WAVES = SCALE_THREADS / 64;
  __shared__ float part[2][WAVES];
  const int tid = threadIdx.x;
  float m = 0.f, ml = 0.f;  // the largest possible entry, the largest gradient of a log probability
  for (int64_t first = tid; first < rows; first += U * SCALE_THREADS) {
    int32_t t[U];
    float log_s[U], gl[U], ge[U];
#pragma unroll
    for (int k = 0; k < U; k++) {
      const int64_t i = first + k * SCALE_THREADS < rows ? first + k * SCALE_THREADS : first;
      t[k] = targets ? targets[i] : -1;
      log_s[k] = stats[2 * i + 1];
      gl[k] = grad_logprobs ? grad_logprobs[i] : 0.f;
      ge[k] = grad_entropy ? grad_entropy[i] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < U; k++) {
      const float l = t[k] >= 0 ? fabsf(gl[k]) * scale : 0.f, g = l + fabsf(ge[k]) * most_entropy * scale;
      // (log s: -inf where there is no distribution, or NaN)
      if (t[k] < vocab && log_s[k] > NEG_INF && g < __builtin_inff()) {
        m = fmaxf(m, g);
        ml = fmaxf(ml, l);
      }
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    m = fmaxf(m, __shfl_xor(m, d));
    ml = fmaxf(ml, __shfl_xor(ml, d));
  }
  if ((tid & 63) == 0) {
    part[0][tid >> 6] = m;
    part[1][tid >> 6] = ml;
  }
  __syncthreads();
  if (tid) return;
#pragma unroll
  for (int w = 1; w < WAVES; w++) {
    m = fmaxf(m, part[0][w]);
    ml = fmaxf(ml, part[1][w]);
  }
  int e = 0, el = 0;
  if (m > 0.f) {
    frexpf(m, &e);  // m < 2^e
    e = 13 - e;
    e = e > 100 ? 100 : e < -100 ? -100 : e;
  }
  const float x = ml > 0.f ? 2.f * frexpf(ml, &el) : 1.f;  // in [1, 2)
  out[0] = ldexpf(1.f / x, e);
  out[1] = ldexpf(x, -e);
}

// Copies rows of any alignment into aligned ones with zeros behind them, and all
// rows again behind those where they are wanted twice.  Entry by entry: 50,257
// rows of 1,024 take 95 us, 2.2 TB/s.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(Operand<T> in, int64_t width, T* out, int64_t stride, bool twice) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < in.rows * stride; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / stride, col = i - row * stride;
    const T x = col < width ? in.p[row * in.stride + col] : (T)0.f;
    out[i] = x;
    if (twice) out[i + in.rows * stride] = x;
  }
}

template <class T>
struct GradLogitsArgs {
  Operand<T> weight, hidden;  // weight: the rows of this piece of the vocabulary
  int64_t width, first, vocab;  // the piece's first entry, the whole vocabulary
  float scale;
  const int32_t* targets;
  const float *stats, *entropy, *grad_logprobs, *grad_entropy;
  const float* factor;  // NULL: 1
  T* g;                 // [g_rows][g_stride], both multiples of 64; SPLIT: [2][rows][g_stride]
  int64_t g_stride, g_rows;
  int32_t m_tiles, n_tiles;
};

// A wave's share of a tile, rounded, through LDS: n runs over its TN * 32 rows,
// each of TM * 32 entries, so that 16 lanes store a row's 256 bytes.  The wave's
// part of LDS is its own; 16-byte pieces of a row are permuted against bank
// conflicts.
template <class Tl, class V4>
__device__ __forceinline__ void keep_four(typename Tl::Shared& sh, int i, int j, int q, V4 x) {
  static_assert(Tl::TM == 4, "rows of 256 bytes");
  const int lane = threadIdx.x & 63, row = j * 32 + (lane & 31);
  char* p = reinterpret_cast<char*>(&sh) + ((threadIdx.x >> 6) * Tl::TN * 32 + row) * 256;
  *reinterpret_cast<V4*>(p + (((i * 4 + q) ^ (row & 15)) << 4) + (lane >> 5) * 8) = x;
}
// put(row, first entry, 8 entries) for every row of the wave's share
template <class Tl, class F>
__device__ __forceinline__ void for_rows(typename Tl::Shared& sh, F put) {
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / Tl::WN, wn = wave % Tl::WN;
  const char* p = reinterpret_cast<const char*>(&sh) + wave * Tl::TN * 32 * 256;
#pragma unroll 8
  for (int k = 0; k < Tl::TN * 8; k++) {
    const int row = k * 4 + (lane >> 4), piece = lane & 15;
    const auto x = *reinterpret_cast<const typename Tl::V8*>(p + row * 256 + ((piece ^ (row & 15)) << 4));
    put(wn * Tl::TN * 32 + row, wm * 128 + piece * 8, x);
  }
}

// G, zero past the last row and the piece's last entry.  SPLIT: G rounded, and
// behind it what the rounding took off, rounded.  The three products of 2,048 rows
// of 2,048 at 100,257 entries in bf16 take 2.36 ms, 1.07 PFLOP/s; this one, with
// an exponential an entry behind it, 0.90 ms of them, grad_weight's 0.74 (1.13
// PFLOP/s) and grad_hidden's 0.69 (1.22).
template <class Tl, bool SPLIT>
__global__ __launch_bounds__(Tl::THREADS, 1) void grad_logits_kernel(GradLogitsArgs<typename Tl::Elem> a) {
  using T = typename Tl::Elem;
  __shared__ typename Tl::Shared sh;
  const uint32_t tile = die_order(blockIdx.x, gridDim.x);
  int64_t mt, nt;
  tile_of(tile, (uint32_t)a.m_tiles, (uint32_t)a.n_tiles, mt, nt);
  const int64_t m0 = mt * Tl::BM, n0 = nt * Tl::BN;
  RowGrad grads[Tl::TN];  // (loaded ahead of the products)
#pragma unroll
  for (int j = 0; j < Tl::TN; j++) {
    const int64_t t = n0 + Tl::col_of(j);
    grads[j] = {};
    grads[j].zero = true;
    grads[j].target = -1;
    if (t < a.hidden.rows)
      grads[j] = row_grad(a.targets, a.stats, a.entropy, a.grad_logprobs, a.grad_entropy, t, a.vocab, a.scale);
  }
  const float c = a.scale * LOG2E;
  if (a.factor) {
    const float factor = a.factor[0];
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      grads[j].a *= factor;
      grads[j].b *= factor;
      grads[j].g *= factor;
      grads[j].h *= factor;
    }
  }
  f32x16 acc[Tl::TM][Tl::TN];
  Tl::multiply(a.weight, a.hidden, m0, n0, 0, a.width, sh, acc);
  const int lane = threadIdx.x & 63, left = a.weight.rows - m0 < Tl::BM ? (int)(a.weight.rows - m0) : Tl::BM;
  auto columns = [&](auto whole, bool rest) {
    constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      if (SPLIT && n0 + Tl::col_of(j) - (lane & 31) >= a.hidden.rows) continue;  // (the same for the wave)
      const RowGrad& g = grads[j];
      // an entry's place is 32 i + 8 (r / 4) + r % 4 from the lane's first one
      const int64_t at = g.target - a.first - m0 - Tl::row_of(0, 0);
      const int given = g.target >= 0 && at >= 0 && at < Tl::TM * 32 ? (int)at : -1;
      int last = left - Tl::row_of(0, 0);
      if (!WHOLE) asm volatile("" : "+v"(last));  // (opaque: comparisons are not made ahead and kept)
      __builtin_amdgcn_sched_barrier(0);
      float at_given = 0.f;
      auto four = [&](int i, int q, auto with_given, auto some_zero) {
        using zeros = decltype(some_zero);
        typename Tl::V4 out;
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const int place = 32 * i + 8 * q + r;
          float y = grad_of(Tl::value(acc, i, j, 4 * q + r), c, g);
          if (decltype(with_given)::value && place == given) y = at_given;
          if ((zeros::value && g.zero) || (!WHOLE && place >= last)) y = 0.f;
          out[r] = (T)(SPLIT && rest ? y - (float)(T)y : y);
        }
        keep_four<Tl>(sh, i, j, q, out);
      };
      // rows without a gradient, and given tokens, are in few tiles
      const bool any = __ballot(given >= 0 || g.zero);
      if (any) {
#pragma unroll
        for (int i = 0; i < Tl::TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (32 * i + 8 * (r >> 2) + (r & 3) == given) at_given = Tl::value(acc, i, j, r);
        at_given = grad_of_given(at_given, c, g);
      }
#pragma unroll
      for (int i = 0; i < Tl::TM; i++) {
#pragma unroll
        for (int q = 0; q < 4; q++) {
          if (any) four(i, q, std::true_type{}, std::true_type{});
          else four(i, q, std::false_type{}, std::false_type{});
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  for (int plane = 0; plane < (SPLIT ? 2 : 1); plane++) {
    if (plane) __syncthreads();
    if (left == Tl::BM) columns(std::true_type{}, plane);
    else columns(std::false_type{}, plane);
    T* to = a.g + plane * a.g_rows * a.g_stride;
    for_rows<Tl>(sh, [&](int row, int m, typename Tl::V8 x) {
      if (n0 + row < a.g_rows && m0 + m < a.g_stride)
        *reinterpret_cast<typename Tl::V8*>(to + (n0 + row) * a.g_stride + m0 + m) = x;
    });
  }
}

template <class T>
struct ProductArgs {
  Operand<T> a, b;
  int64_t k, k_part;  // k and the part of it that a block takes
  int32_t m_tiles, n_tiles;
  const float* factor;  // [1]: inverse of G's factor; NULL: 1
  T* out;               // [b.rows][out_stride]: the product, rounded (k_part >= k)
  int64_t out_stride;
  int64_t out_width;    // entries of a row that are written, at most a.rows
  float* sums;          // or parts [k parts][b.rows][a.rows] in 32 bits,
  bool add;             // added to what is there
};

// out[n][m] = sum_k A[m][k] B[n][k]
template <class Tl>
__global__ __launch_bounds__(Tl::THREADS, 1) void product_kernel(ProductArgs<typename Tl::Elem> a) {
  using T = typename Tl::Elem;
  using F4 = __attribute__((ext_vector_type(4))) float;
  __shared__ typename Tl::Shared sh;
  const uint32_t tile = die_order(blockIdx.x, gridDim.x), tiles = (uint32_t)(a.m_tiles * a.n_tiles);
  const uint32_t part = tile / tiles;
  int64_t mt, nt;
  tile_of(tile % tiles, (uint32_t)a.m_tiles, (uint32_t)a.n_tiles, mt, nt);
  const int64_t m0 = mt * Tl::BM, n0 = nt * Tl::BN;
  const int64_t k0 = part * a.k_part, k1 = k0 + a.k_part < a.k ? k0 + a.k_part : a.k;
  f32x16 acc[Tl::TM][Tl::TN];
  Tl::multiply(a.a, a.b, m0, n0, k0, k1, sh, acc);
  if (!a.out) {
    const int left = a.a.rows - m0 < Tl::BM ? (int)(a.a.rows - m0) : Tl::BM;  // (a multiple of 8)
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      const int64_t n = n0 + Tl::col_of(j);
      if (n >= a.b.rows) continue;
      float* sums = a.sums + ((int64_t)part * a.b.rows + n) * a.a.rows + m0;
#pragma unroll
      for (int i = 0; i < Tl::TM; i++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int m = Tl::row_of(i, q);
          if (m >= left) continue;
          F4 y;
#pragma unroll
          for (int r = 0; r < 4; r++) y[r] = Tl::value(acc, i, j, 4 * q + r);
          if (a.add) y += *reinterpret_cast<F4*>(sums + m);
          *reinterpret_cast<F4*>(sums + m) = y;
        }
    }
    return;
  }
  const float factor = a.factor ? a.factor[1] : 1.f;
#pragma unroll
  for (int j = 0; j < Tl::TN; j++)
#pragma unroll
    for (int i = 0; i < Tl::TM; i++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        typename Tl::V4 z;
#pragma unroll
        for (int r = 0; r < 4; r++) z[r] = (T)(Tl::value(acc, i, j, 4 * q + r) * factor);
        keep_four<Tl>(sh, i, j, q, z);
      }
  // whole pieces of 16 bytes, or entry by entry
  const bool whole = a.out_width % 8 == 0 && a.out_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
  for_rows<Tl>(sh, [&](int row, int m, typename Tl::V8 x) {
    if (n0 + row >= a.b.rows || m0 + m >= a.out_width) return;
    T* p = a.out + (n0 + row) * a.out_stride + m0 + m;
    if (whole) {
      *reinterpret_cast<typename Tl::V8*>(p) = x;
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (m0 + m + i < a.out_width) p[i] = x[i];
    }
  });
}

// out[row][col] = factor * the sum of the parts, for the first `cols` of their rows of `width`
template <class T>
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* sums, int32_t parts, int64_t rows, int64_t width,
                                                        int64_t cols, const float* factor, T* out, int64_t stride) {
  const float f = factor ? factor[1] : 1.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) {
    float y = 0.f;
    const int64_t row = i / cols, col = i - row * cols;
    for (int p0 = 0; p0 < parts; p0 += 8) {  // (eight parts under way: with few rows there is nothing else to wait on)
      float x[8];
#pragma unroll
      for (int p = 0; p < 8; p++) x[p] = p0 + p < parts ? sums[((p0 + p) * rows + row) * width + col] : 0.f;
#pragma unroll
      for (int p = 0; p < 8; p++) y += x[p];
    }
    out[row * stride + col] = (T)(y * f);
  }
}

// ---- host ------------------------------------------------------------------

constexpr int64_t up(int64_t x, int64_t n) { return (x + n - 1) / n * n; }
constexpr int64_t div_up(int64_t x, int64_t n) { return (x + n - 1) / n; }
constexpr int64_t PIECE = 256;    // the vocabulary is taken in multiples of this
constexpr int64_t MOST_PIECE = 1 << 21;  // (256 rows of G, and of hidden and weight, lie in one buffer)

constexpr int FEW_TILE = 64;  // vocabulary entries of a tile for up to 64 rows
int64_t forward_tile_rows(int64_t rows) { return rows <= 64 ? FEW_TILE : 256; }

bool head_sizes(int64_t rows, int64_t vocab, int64_t width) {
  return rows >= 0 && rows <= INT32_MAX && vocab >= 1 && vocab <= INT32_MAX && width >= 1 && width <= INT32_MAX;
}

template <class T>
bool vectors(const Operand<T>& o, int64_t k) {
  return k % 8 == 0 && o.stride % 8 == 0 && reinterpret_cast<uintptr_t>(o.p) % 16 == 0 &&
         o.stride <= ((int64_t)BUFFER_BYTES / 2 - 64) / 256;  // the tile's rows in one buffer
}

// Both set the number of a row's parts.
template <class Tl>
int run_forward(HeadArgs<typename Tl::Elem>& a, hipStream_t st) {
  const int64_t m = div_up(a.weight.rows, Tl::BM), n = div_up(a.hidden.rows, Tl::BN);
  if (m * n > (int64_t)UINT32_MAX / Tl::THREADS) return TT_ERR_TOO_LARGE;
  a.m_tiles = (int32_t)m;
  a.n_tiles = (int32_t)n;
  return launch(head_scores_kernel<Tl>, dim3((uint32_t)(m * n)), dim3(Tl::THREADS), st, a) == hipSuccess ? TT_OK : TT_ERR_HIP;
}
template <class S>
int run_stream(HeadArgs<typename S::Elem>& a, hipStream_t st) {
  const int64_t tiles = div_up(a.weight.rows, 64);
  a.m_tiles = (int32_t)(tiles < S::BLOCKS ? tiles : S::BLOCKS);
  return launch(head_stream_kernel<S>, dim3((uint32_t)a.m_tiles), dim3(128), st, a) == hipSuccess ? TT_OK : TT_ERR_HIP;
}

// Whether tiles of 256 x 128 finish before tiles of 256 x 256: the tiles run in
// rounds of one per compute unit, and a round of the narrow ones takes NARROW of
// a round of the wide ones.
constexpr double NARROW = 0.6;
bool narrow(int64_t m, int64_t n, int64_t parts) {
  const int64_t wide = div_up(div_up(m, 256) * div_up(n, 256) * parts, CUS);
  return (double)div_up(div_up(m, 256) * div_up(n, 128) * parts, CUS) * NARROW < (double)wide;
}

template <class T, bool VEC>
int forward_by_rows(HeadArgs<T>& a, hipStream_t st) {
  const int64_t rows = a.hidden.rows;
  if (VEC && rows <= 32) return run_stream<Stream<T, 32>>(a, st);
  if (VEC && rows <= 64) return run_stream<Stream<T, 64>>(a, st);
  if (rows <= 64) return run_forward<Tile<T, FEW_TILE, 64, 2, 1, false>>(a, st);
  // (entry by entry through registers.  At 2,048 x 50,257 with weights off their
  // alignment: 4 rows 217 us, aligned 47; 300 rows 939 and 97; 2,048 rows 4,406 and 413)
  if (!VEC) return run_forward<Tile<T, 256, 128, 4, 2, false>>(a, st);
  if (narrow(a.weight.rows, rows, 1)) return run_forward<Tile<T, 256, 128, 2, 2, true>>(a, st);
  return run_forward<Tile<T, 256, 256, 2, 2, true>>(a, st);
}

// Up to so many rows G is kept in two parts, rounded and what that took off, and
// the products sum both.  With G rounded alone the results are off by 1.4 times
// their own rounding, as the errors of many entries average out; those of the
// given tokens of a few rows do not (2.5 times for one row, 1.6 for 128).  us with
// G rounded alone and in two parts, bf16: one row of 1,024 at a vocabulary of
// 50,257 89 / 97, 64 98 / 126, 128 110 / 151, 256 159 / 227; 256 of 2,048 at
// 100,257 514 / 731.  More rows would pay up to two thirds for what averages out.
constexpr int64_t SPLIT_ROWS = 256;

// Layout of the gradients' workspace for pieces of `piece` vocabulary entries.
struct GradPlan {
  bool split;             // G in two parts, one after the other
  int64_t padded;         // rows, up to a multiple of 64
  int64_t g_rows;         // rows of G that count, those of both parts
  int64_t wide;           // width, up to a multiple of 8
  int64_t k_part, parts;  // parts of k in grad_hidden (of every piece alike, so that their sums can go on)
  int64_t factor, sums, g, hidden, weight, bytes;
};
// Parts of k, by what they cost: rounds of tiles, each as long as a part, and
// the parts' sums, written and read again.  SUM is the time of one of these sums
// in units of one entry of k of a 256 x 256 tile (30 ns).  grad_hidden alone, us:
// 640 rows of 1,024 at a vocabulary of 50,257: 12 parts 187, the 21 that fill the
// chip with wide tiles 214, one 684; 2,048 of 2,048 at 100,257: 4 parts 1,590, 8
// 1,635, one 2,539; 1,500 of 4,096: 8 parts 2,307, 2 2,335, one 2,745.
constexpr double SUM = 8.0 / 5e12 / 30e-9;
int64_t parts_of_k(int64_t rows, int64_t width, int64_t piece) {
  const int64_t m = div_up(width, 256), wide = m * div_up(rows, 256), slim = m * div_up(rows, 128);
  int64_t most = div_up(piece, 1024), best = 1;  // more than 512 entries of k each (nine steps)
  if (most > 64) most = 64;
  double least = 0;
  for (int64_t n = 1; n <= most; n++) {
    const double w = (double)div_up(wide * n, CUS), s = (double)div_up(slim * n, CUS) * NARROW;
    const double time = (w < s ? w : s) * (double)up(div_up(piece, n), 64) + (n > 1 ? SUM * (double)(n * rows * width) : 0);
    if (n == 1 || time < least) {
      least = time;
      best = n;
    }
    if (wide * n >= 8 * CUS) break;  // the last round no longer counts
  }
  return best;
}
// pack: hidden and weight are copied to aligned rows
GradPlan grad_plan(int64_t rows, int64_t width, int64_t piece, bool pack) {
  GradPlan p;
  p.split = rows <= SPLIT_ROWS;
  p.padded = up(rows, 64);
  p.g_rows = p.split ? 2 * rows : rows;
  p.wide = up(width, 8);
  p.parts = parts_of_k(p.g_rows, width, piece);
  p.k_part = up(div_up(piece, p.parts), 64);
  p.parts = div_up(piece, p.k_part);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t was = at;
    at += up(bytes, 256);
    return was;
  };
  p.factor = take(8);
  p.sums = take(4 * p.parts * p.g_rows * p.wide);
  p.g = take(2 * (p.split ? p.g_rows : p.padded) * piece);
  p.hidden = take(p.split ? 2 * p.g_rows * p.wide : pack ? 2 * rows * p.wide : 0);
  p.weight = take(pack ? 2 * piece * p.wide : 0);
  p.bytes = at;
  return p;
}

template <class T>
struct GradCall {
  Operand<T> hidden, weight;
  int64_t width;
  float scale;
  const int32_t* targets;
  const float *stats, *entropy, *grad_logprobs, *grad_entropy;
  T *grad_hidden, *grad_weight;
  int64_t grad_hidden_stride, grad_weight_stride;
  uint8_t* work;
  int64_t work_bytes;
};

template <class T>
hipError_t pack(const Operand<T>& in, int64_t width, T* out, int64_t stride, hipStream_t st, bool twice = false) {
  const int64_t blocks = div_up(in.rows * stride, 1024);
  return launch(pack_kernel<T>, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), dim3(256), st, in, width, out, stride,
                twice);
}

template <class Tl>
hipError_t product(ProductArgs<typename Tl::Elem> a, hipStream_t st) {
  a.m_tiles = (int32_t)div_up(a.a.rows, Tl::BM);
  a.n_tiles = (int32_t)div_up(a.b.rows, Tl::BN);
  return launch(product_kernel<Tl>, dim3((uint32_t)((int64_t)a.m_tiles * a.n_tiles * (a.k ? div_up(a.k, a.k_part) : 1))),
                dim3(Tl::THREADS), st, a);
}

// The products' tiles: grad_weight sums over rows, grad_hidden over the vocabulary.
template <class T, int BN>
using ByHidden = Tile<T, 256, BN, 2, 2, true, true, true>;
template <class T, int BN>
using ByWeight = Tile<T, 256, BN, 2, 2, true, true, false>;

template <class T>
hipError_t grad_weight_product(const ProductArgs<T>& a, hipStream_t st) {
  return narrow(a.a.rows, a.b.rows, 1) ? product<ByHidden<T, 128>>(a, st) : product<ByHidden<T, 256>>(a, st);
}
template <class T>
hipError_t grad_hidden_product(const ProductArgs<T>& a, hipStream_t st) {
  return narrow(a.a.rows, a.b.rows, div_up(a.k, a.k_part)) ? product<ByWeight<T, 128>>(a, st)
                                                          : product<ByWeight<T, 256>>(a, st);
}
template <class Tl, bool SPLIT = false>
hipError_t grad_logits(GradLogitsArgs<typename Tl::Elem> a, hipStream_t st) {
  a.m_tiles = (int32_t)div_up(a.weight.rows, Tl::BM);
  a.n_tiles = (int32_t)div_up(a.hidden.rows, Tl::BN);
  return launch(grad_logits_kernel<Tl, SPLIT>, dim3((uint32_t)((int64_t)a.m_tiles * a.n_tiles)), dim3(Tl::THREADS), st, a);
}

template <class T>
int run_gradients(const GradCall<T>& c, hipStream_t st) {
  auto bad = [](hipError_t e) { return e != hipSuccess; };
  const int64_t rows = c.hidden.rows, vocab = c.weight.rows;
  if (rows == 0) {  // grad_weight is the empty sum
    const ProductArgs<T> pa{{nullptr, 0, up(c.width, 8)}, {nullptr, 0, vocab}, 0, 1, 0, 0, nullptr, c.grad_weight,
                            c.grad_weight_stride, c.width, nullptr, false};
    return !c.grad_weight || !bad(grad_weight_product(pa, st)) ? TT_OK : TT_ERR_HIP;
  }
  const bool aligned = vectors(c.hidden, c.width) && vectors(c.weight, c.width);
  // The largest piece of the vocabulary that the workspace holds.  640 rows of 1,024
  // at 50,257 in bf16: 277 us with the ample size and half way to it, 583 with a tenth of
  // the way from the least one, 2,940 with the least (three launches for 256 entries).
  int64_t piece = PIECE, most = up(vocab < MOST_PIECE ? vocab : MOST_PIECE, PIECE);
  if (grad_plan(rows, c.width, most, !aligned).bytes <= c.work_bytes) piece = most;
  while (piece < most) {
    const int64_t mid = up((piece + most) / 2, PIECE);
    if (grad_plan(rows, c.width, mid, !aligned).bytes <= c.work_bytes) piece = mid;
    else most = mid - PIECE;
  }
  const GradPlan p = grad_plan(rows, c.width, piece, !aligned);
  const int64_t width = aligned ? c.width : p.wide;
  T* g = reinterpret_cast<T*>(c.work + p.g);
  float* sums = reinterpret_cast<float*>(c.work + p.sums);
  const float* factor = nullptr;
  if (std::is_same<T, f16_t>::value || !p.split) {
    float* f = reinterpret_cast<float*>(c.work + p.factor);
    const float entropy = logf((float)vocab) + 0.5f;  // |p (log p + H)| <= 1/e + log(vocab)
    if (bad(launch(grad_scale_kernel, dim3(1), dim3(SCALE_THREADS), st, rows, vocab, entropy, c.scale, c.targets, c.stats, c.grad_logprobs,
                   c.grad_entropy, f)))
      return TT_ERR_HIP;
    factor = f;
  }
  Operand<T> hidden = c.hidden;
  if (!aligned || p.split) {
    T* to = reinterpret_cast<T*>(c.work + p.hidden);
    if (bad(pack(c.hidden, c.width, to, p.wide, st, p.split))) return TT_ERR_HIP;
    hidden = {to, p.wide, rows};
  }
  const bool direct = p.parts == 1 && piece >= vocab && !p.split;  // grad_hidden needs no sums in between
  for (int64_t first = 0; first < vocab; first += piece) {
    const int64_t n = vocab - first < piece ? vocab - first : piece, g_stride = up(n, 64);
    Operand<T> weight{c.weight.p + first * c.weight.stride, c.weight.stride, n};
    if (!aligned) {
      T* to = reinterpret_cast<T*>(c.work + p.weight);
      if (bad(pack(weight, c.width, to, p.wide, st))) return TT_ERR_HIP;
      weight = {to, p.wide, n};
    }
    const GradLogitsArgs<T> ga{weight,    hidden,          width,          first,  vocab, c.scale,  c.targets, c.stats,
                               c.entropy, c.grad_logprobs, c.grad_entropy, factor, g,     g_stride, p.split ? rows : p.padded, 0, 0};
    if (bad(p.split              ? grad_logits<Tile<T, 256, 128, 2, 2, true>, true>(ga, st)
            : narrow(n, rows, 1) ? grad_logits<Tile<T, 256, 128, 2, 2, true>>(ga, st)
                                 : grad_logits<Tile<T, 256, 256, 2, 2, true>>(ga, st)))
      return TT_ERR_HIP;
    if (c.grad_weight) {
      const ProductArgs<T> pa{{hidden.p, hidden.stride, width}, {g, g_stride, n}, p.g_rows, p.g_rows, 0, 0, factor,
                              c.grad_weight + first * c.grad_weight_stride, c.grad_weight_stride, c.width, nullptr, false};
      if (bad(grad_weight_product(pa, st))) return TT_ERR_HIP;
    }
    if (c.grad_hidden) {
      const ProductArgs<T> pa{{weight.p, weight.stride, width}, {g, g_stride, p.g_rows}, n, direct ? n : p.k_part, 0, 0,
                              direct ? factor : nullptr, direct ? c.grad_hidden : nullptr, c.grad_hidden_stride, c.width,
                              sums, first > 0};
      if (bad(grad_hidden_product(pa, st))) return TT_ERR_HIP;
    }
  }
  if (c.grad_hidden && !direct) {
    const int64_t blocks = div_up(rows * c.width, 256);
    const int32_t used = (int32_t)div_up(vocab < piece ? vocab : piece, p.k_part);  // parts of the first piece
    if (bad(launch(sum_parts_kernel<T>, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), dim3(256), st,
                   static_cast<const float*>(sums), used * (p.split ? 2 : 1), rows, width, c.width, factor, c.grad_hidden,
                   c.grad_hidden_stride)))
      return TT_ERR_HIP;
  }
  return TT_OK;
}

}  // namespace
}  // namespace tt

using namespace tt;

extern "C" int64_t tt_head_scores_workspace(int64_t rows, int64_t vocab, int64_t width) {
  if (!head_sizes(rows, vocab, width)) return TT_ERR_BAD_ARG;
  return up(rows * 4, 256) + rows * div_up(vocab, forward_tile_rows(rows)) * (int64_t)sizeof(Part);
}

extern "C" int tt_head_scores(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                              int32_t type, int64_t rows, int64_t vocab, int64_t width, float scale,
                              const int32_t* targets, float* logprobs, float* stats, float* entropy, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  const int64_t need = tt_head_scores_workspace(rows, vocab, width);
  if (need < 0 || (type != TT_BF16 && type != TT_F16) || hidden_stride < width || weight_stride < width ||
      !good_scale(scale) || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 256)
    return TT_ERR_BAD_ARG;
  if (rows == 0) return TT_OK;
  if (!hidden || !weight || !workspace) return TT_ERR_NULL_ARG;
  if (div_up(rows, 4) > (int64_t)UINT32_MAX / 256) return TT_ERR_TOO_LARGE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* given = static_cast<float*>(workspace);
  Part* parts = reinterpret_cast<Part*>(static_cast<uint8_t*>(workspace) + up(rows * 4, 256));
  int32_t n_parts = 0;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    HeadArgs<T> a{{static_cast<const T*>(weight), weight_stride, vocab},
                  {static_cast<const T*>(hidden), hidden_stride, rows},
                  width, scale, targets, parts, given, 0, 0};
    const int s = vectors(a.weight, width) && vectors(a.hidden, width) ? forward_by_rows<T, true>(a, st)
                                                                       : forward_by_rows<T, false>(a, st);
    n_parts = a.m_tiles;
    return s;
  };
  const int s = type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
  if (s != TT_OK) return s;
  return launch(head_join_kernel, dim3((uint32_t)div_up(rows, 4)), dim3(256), st, static_cast<const Part*>(parts),
                static_cast<const float*>(given), n_parts, rows, vocab, scale, targets, logprobs, stats, entropy) == hipSuccess
             ? TT_OK
             : TT_ERR_HIP;
}

extern "C" int64_t tt_head_scores_grad_workspace(int64_t rows, int64_t vocab, int64_t width, int32_t ample) {
  if (!head_sizes(rows, vocab, width)) return TT_ERR_BAD_ARG;
  if (width > MOST_PIECE) return TT_ERR_TOO_LARGE;
  if (rows == 0) return 0;
  return grad_plan(rows, width, ample ? up(vocab < MOST_PIECE ? vocab : MOST_PIECE, PIECE) : PIECE, true).bytes;
}

extern "C" int tt_head_scores_grad(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                                   int32_t type, int64_t rows, int64_t vocab, int64_t width, float scale,
                                   const int32_t* targets, const float* stats, const float* entropy,
                                   const float* grad_logprobs, const float* grad_entropy, void* grad_hidden,
                                   int64_t grad_hidden_stride, void* grad_weight, int64_t grad_weight_stride,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
  const int64_t need = tt_head_scores_grad_workspace(rows, vocab, width, 0);
  if (need < 0) return (int)need;
  if ((type != TT_BF16 && type != TT_F16) || hidden_stride < width || weight_stride < width ||
      (grad_hidden && grad_hidden_stride < width) || (grad_weight && grad_weight_stride < width) || !good_scale(scale) ||
      workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 256)
    return TT_ERR_BAD_ARG;
  if (!grad_hidden && !grad_weight) return TT_OK;
  if (!weight || (rows > 0 && (!hidden || !stats || !workspace || (grad_entropy && !entropy)))) return TT_ERR_NULL_ARG;
  // launches of at most 2^32 threads
  if (div_up(vocab, 128) * (div_up(rows, 128) + div_up(width, 128)) > (int64_t)UINT32_MAX / 256 ||
      div_up(rows, 128) * div_up(width, 256) * 256 > (int64_t)UINT32_MAX / 256)
    return TT_ERR_TOO_LARGE;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    return run_gradients(GradCall<T>{{static_cast<const T*>(hidden), hidden_stride, rows},
                                     {static_cast<const T*>(weight), weight_stride, vocab},
                                     width, scale, targets, stats, entropy, grad_logprobs, grad_entropy,
                                     static_cast<T*>(grad_hidden), static_cast<T*>(grad_weight), grad_hidden_stride,
                                     grad_weight_stride, static_cast<uint8_t*>(workspace), workspace_bytes},
                         static_cast<hipStream_t>(stream));
  };
  return type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}
