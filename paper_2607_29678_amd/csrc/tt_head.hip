// tt_head_scores and its gradients: scores of logits = hidden weight^T that are
// never stored, on the matrix cores.
//
// Every product here is C[m][n] = sum_k A[m][k] B[n][k] with both operands
// contiguous in k, in tiles of BM x BN that eight (or four) waves share.  m runs
// over the vocabulary in the scores, so a lane's accumulators hold entries of
// one token's row and the softmax statistics are sums within the lane.
#include "tt_scores.h"

namespace tt {
namespace {

using f32x16 = __attribute__((ext_vector_type(16))) float;

template <class T>
struct Mfma;
template <>
struct Mfma<bf16_t> {
  using V8 = __attribute__((ext_vector_type(8))) bf16_t;
  static __device__ __forceinline__ f32x16 mul(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<f16_t> {
  using V8 = __attribute__((ext_vector_type(8))) f16_t;
  static __device__ __forceinline__ f32x16 mul(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// An operand: rows of k entries.
template <class T>
struct Operand {
  const T* p;
  int64_t stride, rows;
};

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
// read of LDS wait for the load; there is no result register.  (m0 is the
// compiler's to set before each use of its own; a write of it needs one wait
// state before its use.)
__device__ __forceinline__ void load_to_lds(Buffer from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(from));
}
// Waits for all but the last N of this wave's loads and for its LDS reads, then
// for the block's other waves.
template <int N>
__device__ __forceinline__ void loads_done_but() {
  static_assert(N < 64, "field of s_waitcnt");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <class T, int BM_, int BN_, int WM_, int WN_, bool VEC_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr bool VEC = VEC_;  // rows are aligned to 16 bytes and k is a multiple of 8
  static constexpr bool DIRECT = VEC && BM == 256 && BN == 256;
  static constexpr int THREADS = 64 * WM * WN;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // 32 x 32 products of a wave
  using Elem = T;
  using V8 = typename Mfma<T>::V8;
  static constexpr int NA = BM * 8 / THREADS, NB = BN * 8 / THREADS;  // 16-byte pieces a thread stages
  static_assert(NA * THREADS == BM * 8 && NB * THREADS == BN * 8, "whole pieces");
  struct Shared {
    T a[2][BM * BK], b[2][BN * BK];
  };

  // Piece q of a stage: row q / 8, entries 8 (q % 8) and on.  In LDS the pieces
  // of a row are permuted by the row's low bits, so that the 32 rows that a wave
  // reads at one k lie in different banks.
  static __device__ __forceinline__ int place(int row, int piece) { return row * BK + ((piece ^ (row & 7)) << 3); }

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
    uint32_t oa[DA], ob[DB];  // byte offsets from the tile's first row
    const int piece = (lane & 7) ^ (lane >> 3);  // (a load starts at a row that is a multiple of 8)
#pragma unroll
    for (int i = 0; i < DA; i++) {
      const int64_t row = (wave * DA + i) * 8 + (lane >> 3);
      oa[i] = m0 + row < a.rows ? (uint32_t)(row * a.stride + piece * 8) * 2 : BUFFER_BYTES;
    }
#pragma unroll
    for (int i = 0; i < DB; i++) {
      const int64_t row = (wave * DB + i) * 8 + (lane >> 3);
      ob[i] = n0 + row < b.rows ? (uint32_t)(row * b.stride + piece * 8) * 2 : BUFFER_BYTES;
    }
    const T *pa = a.p + m0 * a.stride + k0, *pb = b.p + n0 * b.stride + k0;
    const uint32_t la = __builtin_amdgcn_readfirstlane(lds_address(sh.a) + wave * DA * 1024);
    const uint32_t lb = __builtin_amdgcn_readfirstlane(lds_address(sh.b) + wave * DB * 1024);
    const int64_t mine = k1 - k0 - piece * 8;  // entries of k from this lane's piece on
    const int stages_here = mine <= 0 ? 0 : (int)((mine + BK - 1) / BK);  // stages in which the lane has any
    auto load_piece = [&](int stage, int i) {  // loads 0 .. DA + DB - 1 of a stage
      const uint32_t at = stage & 1;
      const bool real = stage < stages_here;
      if (i < DA)
        load_to_lds(buffer_at(pa + (int64_t)stage * BK), real ? oa[i < DA ? i : 0] : BUFFER_BYTES,
                    la + at * (BM * BK * 2) + i * 1024);
      else
        load_to_lds(buffer_at(pb + (int64_t)stage * BK), real ? ob[i < DA ? 0 : i - DA] : BUFFER_BYTES,
                    lb + at * (BN * BK * 2) + (i - DA) * 1024);
    };
    V8 fa[2][TM], fb[2][TN];
    auto read = [&](int buf, int kk, int to) {
#pragma unroll
      for (int i = 0; i < TM; i++)
        fa[to][i] = *reinterpret_cast<const V8*>(&sh.a[buf][place(wm * TM * 32 + i * 32 + (lane & 31), kk * 2 + (lane >> 5))]);
#pragma unroll
      for (int j = 0; j < TN; j++)
        fb[to][j] = *reinterpret_cast<const V8*>(&sh.b[buf][place(wn * TN * 32 + j * 32 + (lane & 31), kk * 2 + (lane >> 5))]);
    };
    auto one = [&](int from, int ij) {
      const int i = ij / TN, j = ij % TN;
      acc[i][j] = Mfma<T>::mul(fa[from][i], fb[from][j], acc[i][j]);
    };
#pragma unroll
    for (int i = 0; i < DA + DB; i++) load_piece(0, i);
#pragma unroll
    for (int i = 0; i < DA + DB; i++) load_piece(1, i);
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
      for (int j = 0; j < TN; j++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    loads_done_but<DA + DB>();
    read(0, 0, 0);
    const int steps = (int)((k1 - k0 + BK - 1) / BK);
    int s = 0;
    do {
#pragma unroll
      for (int kk = 0; kk < BK / 16 - 1; kk++) {
        read(s & 1, kk + 1, (kk + 1) & 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ij = 0; ij < TM * TN; ij++) one(kk & 1, ij);
        __builtin_amdgcn_sched_barrier(0);
      }
      loads_done_but<0>();
      read((s + 1) & 1, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ij = 0; ij < TM * TN; ij++) {  // the loads are issued between the products
        one(1, ij);
#pragma unroll
        for (int i = ij * (DA + DB) / (TM * TN); i < (ij + 1) * (DA + DB) / (TM * TN); i++) load_piece(s + 2, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    } while (++s < steps);
    loads_done_but<0>();
    // (what reads the accumulators by assembly has to wait for the last products itself)
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
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

template <class Tl>
__global__ __launch_bounds__(Tl::THREADS, Tl::BM == 256 && Tl::BN == 256 ? Tl::THREADS / 256 : 2) void head_scores_kernel(HeadArgs<typename Tl::Elem> a) {
  __shared__ typename Tl::Shared sh;
  const uint32_t tile = die_order(blockIdx.x, gridDim.x);
  int64_t mt, nt;
  tile_of(tile, (uint32_t)a.m_tiles, (uint32_t)a.n_tiles, mt, nt);
  const int64_t m0 = mt * Tl::BM, n0 = nt * Tl::BN;
  f32x16 acc[Tl::TM][Tl::TN];
  Tl::multiply(a.weight, a.hidden, m0, n0, 0, a.width, sh, acc);

  const float c = a.scale * LOG2E;
  const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / Tl::WN;
  Part* joined = reinterpret_cast<Part*>(&sh);  // [WM][BN]
  const int64_t rows = a.hidden.rows;
  const int left = a.weight.rows - m0 < Tl::BM ? (int)(a.weight.rows - m0) : Tl::BM;  // entries of this tile
  auto columns = [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      const int col = Tl::col_of(j);
      const int64_t t = n0 + col;
      // an entry's place is 32 i + 8 (r / 4) + r % 4 from the lane's first one
      int last = left - Tl::row_of(0, 0), given = -1;
      if (a.targets && t < rows) {
        const int64_t g = a.targets[t] - m0;
        if (g >= 0 && g < left) given = (int)g - Tl::row_of(0, 0);
      }
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
        for (int r = 0; r < 16; r++) m = fmaxf(m, entry(i, r));
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
      m = fmaxf(m, __shfl_xor(m, 32));
      const float ref = reference(m);
      float s0 = 0.f, u0 = 0.f;
      if (!WHOLE) asm volatile("" : "+v"(last));
#pragma unroll
      for (int i = 0; i < Tl::TM; i++) {
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const float d = (entry(i, r) - ref) * c, e = __builtin_amdgcn_exp2f(d);
          s0 += e;
          u0 += weigh(e, d);
        }
        __builtin_amdgcn_sched_barrier(0);  // (the accumulators do not fit the other registers all at once)
      }
      s0 += __shfl_xor(s0, 32);
      u0 += __shfl_xor(u0, 32);
      if (lane < 32) joined[wm * Tl::BN + col] = {m, s0, u0, 0.f};
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

// Joins a row's parts: one wave per row.
__global__ __launch_bounds__(256) void head_join_kernel(const Part* parts, const float* given, int32_t n_parts,
                                                        int64_t rows, int64_t vocab, float scale, const int32_t* targets,
                                                        float* logprobs, float* stats, float* entropy) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  const float c = scale * LOG2E;
  Stats st = empty_stats();
  for (int i = lane; i < n_parts; i += 64) {
    const Part q = parts[row * n_parts + i];
    st = join(st, Stats{q.m, q.s, q.u}, c);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) st = join(st, shuffled_xor(st, d), c);
  if (lane) return;
  const RowScores r = row_scores(st);
  const int32_t t = targets ? targets[row] : -1;
  if (logprobs) logprobs[row] = given_log_prob(t, vocab, t >= 0 && t < vocab ? given[row] : 0.f, r, scale);
  if (stats) {
    stats[2 * row] = r.m;
    stats[2 * row + 1] = r.log_s;
  }
  if (entropy) entropy[row] = r.entropy;
}

// ---- gradients -------------------------------------------------------------

// A power of two that brings the largest possible entry of G near 2^13 (16-bit
// floats hold up to 65,504, and lose small entries below 2^-14), and its inverse.
__global__ __launch_bounds__(256) void grad_scale_kernel(int64_t rows, float most_entropy, float scale,
                                                         const float* grad_logprobs, const float* grad_entropy,
                                                         float* out) {
  __shared__ float part[4];
  float m = 0.f;
  for (int64_t i = threadIdx.x; i < rows; i += 256) {
    const float g = (grad_logprobs ? fabsf(grad_logprobs[i]) : 0.f) + (grad_entropy ? fabsf(grad_entropy[i]) * most_entropy : 0.f);
    m = fmaxf(m, g * scale);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x) return;
  m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  int e = 0;
  if (m > 0.f && m < __builtin_inff()) {
    frexpf(m, &e);  // m < 2^e
    e = 13 - e;
    e = e > 100 ? 100 : e < -100 ? -100 : e;
  }
  out[0] = ldexpf(1.f, e);
  out[1] = ldexpf(1.f, -e);
}

// out[c][r] = in[r][c] for r < rows, 0 for rows <= r < padded; 64 x 64 tiles.
template <class T>
__global__ __launch_bounds__(256) void transpose_kernel(const T* in, int64_t stride, int64_t rows, int64_t cols, T* out,
                                                        int64_t padded) {
  __shared__ T tile[64][66];
  const int64_t tiles_r = padded / 64;
  const int64_t r0 = (blockIdx.x % tiles_r) * 64, c0 = (blockIdx.x / tiles_r) * 64;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll 4
  for (int i = y; i < 64; i += 4) tile[i][x] = r0 + i < rows && c0 + x < cols ? in[(r0 + i) * stride + c0 + x] : (T)0.f;
  __syncthreads();
#pragma unroll 4
  for (int i = y; i < 64; i += 4)
    if (c0 + i < cols) out[(c0 + i) * padded + r0 + x] = tile[x][i];
}

template <class T>
struct GradLogitsArgs {
  Operand<T> weight, hidden;  // weight: the rows of this piece of the vocabulary
  int64_t width, first, vocab;  // the piece's first entry, the whole vocabulary
  float scale;
  const int32_t* targets;
  const float *stats, *entropy, *grad_logprobs, *grad_entropy;
  const float* factor;  // NULL: 1
  T* g;    // [padded rows][g_stride] or NULL
  T* gt;   // [piece][gt_stride] or NULL
  int64_t g_stride, gt_stride;
  int32_t m_tiles, n_tiles;
};

// G and its transpose, zero past the last row and the piece's last entry.
template <class Tl>
__global__ __launch_bounds__(Tl::THREADS, Tl::BM == 256 && Tl::BN == 256 ? Tl::THREADS / 256 : 2) void grad_logits_kernel(GradLogitsArgs<typename Tl::Elem> a) {
  using T = typename Tl::Elem;
  using T4 = __attribute__((ext_vector_type(4))) T;
  __shared__ typename Tl::Shared sh;
  const uint32_t tile = die_order(blockIdx.x, gridDim.x);
  int64_t mt, nt;
  tile_of(tile, (uint32_t)a.m_tiles, (uint32_t)a.n_tiles, mt, nt);
  const int64_t m0 = mt * Tl::BM, n0 = nt * Tl::BN;
  f32x16 acc[Tl::TM][Tl::TN];
  Tl::multiply(a.weight, a.hidden, m0, n0, 0, a.width, sh, acc);
  const float c = a.scale * LOG2E, factor = a.factor ? a.factor[0] : 1.f;
#pragma unroll
  for (int j = 0; j < Tl::TN; j++) {
    const int64_t t = n0 + Tl::col_of(j);
    RowGrad g = {};
    g.zero = true;
    if (t < a.hidden.rows)
      g = row_grad(a.targets, a.stats, a.entropy, a.grad_logprobs, a.grad_entropy, t, a.vocab, a.scale);
    const int64_t given = g.target - a.first;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < Tl::TM; i++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int64_t v = m0 + Tl::row_of(i, q);
        T4 out;
#pragma unroll
        for (int r = 0; r < 4; r++) {
          float y = 0.f;
          if (!g.zero && v + r < a.weight.rows) {
            y = grad_of(Tl::value(acc, i, j, 4 * q + r), c, g);
            if (v + r == given) y += g.g;
          }
          out[r] = (T)(y * factor);
        }
        if (a.g && v < a.g_stride && t < a.gt_stride) *reinterpret_cast<T4*>(a.g + t * a.g_stride + v) = out;
        if (a.gt && t < a.gt_stride) {
#pragma unroll
          for (int r = 0; r < 4; r++)
            if (v + r < a.weight.rows) a.gt[(v + r) * a.gt_stride + t] = out[r];
        }
      }
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
  float* sums;          // or parts [k parts][b.rows][a.rows] in 32 bits,
  bool add;             // added to what is there
};

// out[n][m] = sum_k A[m][k] B[n][k]
template <class Tl>
__global__ __launch_bounds__(Tl::THREADS, Tl::BM == 256 && Tl::BN == 256 ? Tl::THREADS / 256 : 2) void product_kernel(ProductArgs<typename Tl::Elem> a) {
  using T = typename Tl::Elem;
  using T4 = __attribute__((ext_vector_type(4))) T;
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
  const float factor = a.factor ? a.factor[1] : 1.f;
  const int left = a.a.rows - m0 < Tl::BM ? (int)(a.a.rows - m0) : Tl::BM;
  // whole groups of four entries, aligned to their size, or entry by entry
  const bool fours = a.a.rows % 4 == 0 && (a.out ? a.out_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 7) == 0 : true);
  auto put = [&](auto whole) {
#pragma unroll
    for (int j = 0; j < Tl::TN; j++) {
      const int64_t n = n0 + Tl::col_of(j);
      if (n >= a.b.rows) continue;
      T* out = a.out + n * a.out_stride + m0;
      float* sums = a.sums + ((int64_t)part * a.b.rows + n) * a.a.rows + m0;
#pragma unroll
      for (int i = 0; i < Tl::TM; i++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int m = Tl::row_of(i, q);
          if (m >= left) continue;
          F4 y;
          T4 z;
#pragma unroll
          for (int r = 0; r < 4; r++) {
            y[r] = Tl::value(acc, i, j, 4 * q + r);
            z[r] = (T)(y[r] * factor);
          }
          if (decltype(whole)::value) {
            if (a.out) {
              *reinterpret_cast<T4*>(out + m) = z;
            } else {
              if (a.add) y += *reinterpret_cast<F4*>(sums + m);
              *reinterpret_cast<F4*>(sums + m) = y;
            }
          } else {
#pragma unroll 1
            for (int r = 0; r < 4; r++)
              if (m + r < left) {
                if (a.out) out[m + r] = z[r];
                else sums[m + r] = a.add ? sums[m + r] + y[r] : y[r];
              }
          }
        }
    }
  };
  if (fours) put(std::true_type{});
  else put(std::false_type{});
}

// out[row][col] = factor * the sum of the parts
template <class T>
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* sums, int32_t parts, int64_t rows, int64_t cols,
                                                        const float* factor, T* out, int64_t stride) {
  const float f = factor ? factor[1] : 1.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) {
    float y = 0.f;
    for (int p = 0; p < parts; p++) y += sums[p * rows * cols + i];
    out[i / cols * stride + i % cols] = (T)(y * f);
  }
}

// ---- host ------------------------------------------------------------------

constexpr int64_t up(int64_t x, int64_t n) { return (x + n - 1) / n * n; }
constexpr int64_t div_up(int64_t x, int64_t n) { return (x + n - 1) / n; }
constexpr int64_t PIECE = 256;    // the vocabulary is taken in multiples of this
constexpr int64_t CUS = 256;      // compute units

int64_t forward_tile_rows(int64_t rows) { return rows <= 64 ? 128 : 256; }

bool head_sizes(int64_t rows, int64_t vocab, int64_t width) {
  return rows >= 0 && rows <= INT32_MAX && vocab >= 1 && vocab <= INT32_MAX && width >= 1 && width <= INT32_MAX;
}

template <class T>
bool vectors(const Operand<T>& o, int64_t k) {
  return k % 8 == 0 && o.stride % 8 == 0 && reinterpret_cast<uintptr_t>(o.p) % 16 == 0 &&
         o.stride <= ((int64_t)BUFFER_BYTES / 2 - 64) / 256;  // the tile's rows in one buffer
}

template <class Tl>
int run_forward(HeadArgs<typename Tl::Elem> a, hipStream_t st) {
  const int64_t m = div_up(a.weight.rows, Tl::BM), n = div_up(a.hidden.rows, Tl::BN);
  if (m * n > (int64_t)UINT32_MAX / Tl::THREADS) return TT_ERR_TOO_LARGE;
  a.m_tiles = (int32_t)m;
  a.n_tiles = (int32_t)n;
  return launch(head_scores_kernel<Tl>, dim3((uint32_t)(m * n)), dim3(Tl::THREADS), st, a) == hipSuccess ? TT_OK : TT_ERR_HIP;
}

template <class T, bool VEC>
int forward_by_rows(const HeadArgs<T>& a, hipStream_t st) {
  const int64_t rows = a.hidden.rows;
  if (rows <= 32) return run_forward<Tile<T, 128, 32, 4, 1, VEC>>(a, st);
  if (rows <= 64) return run_forward<Tile<T, 128, 64, 4, 1, VEC>>(a, st);
  if (rows <= 128) return run_forward<Tile<T, 256, 128, 4, 2, VEC>>(a, st);
  return run_forward<Tile<T, 256, 256, VEC ? 2 : 4, 2, VEC>>(a, st);
}

// Layout of the gradients' workspace for pieces of `piece` vocabulary entries.
struct GradPlan {
  int64_t padded;         // rows, up to a multiple of 64
  int64_t k_part, parts;  // parts of k in grad_hidden (of every piece alike, so that their sums can go on)
  int64_t factor, hidden_t, sums, g, gt, weight_t, bytes;
};
GradPlan grad_plan(int64_t rows, int64_t width, int64_t piece) {
  GradPlan p;
  p.padded = up(rows, 64);
  p.parts = CUS / (div_up(width, 256) * div_up(rows, 256));
  const int64_t most = div_up(piece, 1024);  // at least 16 steps of k each
  if (p.parts > most) p.parts = most;
  if (p.parts < 1) p.parts = 1;
  p.k_part = up(div_up(piece, p.parts), 64);
  p.parts = div_up(piece, p.k_part);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t was = at;
    at += up(bytes, 256);
    return was;
  };
  p.factor = take(8);
  p.hidden_t = take(2 * width * p.padded);
  p.sums = take(4 * p.parts * rows * width);
  p.g = take(2 * p.padded * piece);
  p.gt = take(2 * p.padded * piece);
  p.weight_t = take(2 * width * piece);
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
  int64_t piece;
};

template <class T>
hipError_t transpose(const Operand<T>& in, int64_t cols, T* out, int64_t padded, hipStream_t st) {
  return launch(transpose_kernel<T>, dim3((uint32_t)(padded / 64 * div_up(cols, 64))), dim3(256), st, in.p, in.stride,
                in.rows, cols, out, padded);
}

template <class Tl>
hipError_t grad_logits(GradLogitsArgs<typename Tl::Elem> a, hipStream_t st) {
  a.m_tiles = (int32_t)div_up(a.weight.rows, Tl::BM);
  a.n_tiles = (int32_t)div_up(a.hidden.rows, Tl::BN);
  return launch(grad_logits_kernel<Tl>, dim3((uint32_t)((int64_t)a.m_tiles * a.n_tiles)), dim3(Tl::THREADS), st, a);
}

template <class Tl>
hipError_t product(ProductArgs<typename Tl::Elem> a, hipStream_t st) {
  a.m_tiles = (int32_t)div_up(a.a.rows, Tl::BM);
  a.n_tiles = (int32_t)div_up(a.b.rows, Tl::BN);
  return launch(product_kernel<Tl>, dim3((uint32_t)((int64_t)a.m_tiles * a.n_tiles * (a.k ? div_up(a.k, a.k_part) : 1))),
                dim3(Tl::THREADS), st, a);
}

template <class T>
int run_gradients(const GradCall<T>& c, hipStream_t st) {
  const int64_t rows = c.hidden.rows, vocab = c.weight.rows;
  if (rows == 0) {  // grad_weight is the empty sum
    using Whole = Tile<T, 256, 256, 2, 2, true>;
    const ProductArgs<T> pa{{c.hidden.p, 0, c.width}, {c.hidden.p, 0, vocab}, 0, 1, 0, 0, nullptr, c.grad_weight,
                            c.grad_weight_stride, nullptr, false};
    return !c.grad_weight || product<Whole>(pa, st) == hipSuccess ? TT_OK : TT_ERR_HIP;
  }
  const GradPlan p = grad_plan(rows, c.width, c.piece);
  float* factor = nullptr;
  T* hidden_t = reinterpret_cast<T*>(c.work + p.hidden_t);
  T* weight_t = reinterpret_cast<T*>(c.work + p.weight_t);
  T* g = reinterpret_cast<T*>(c.work + p.g);
  T* gt = reinterpret_cast<T*>(c.work + p.gt);
  float* sums = reinterpret_cast<float*>(c.work + p.sums);
  const bool vec = vectors(c.hidden, c.width) && vectors(c.weight, c.width);
  auto bad = [](hipError_t e) { return e != hipSuccess; };
  if (std::is_same<T, f16_t>::value) {
    factor = reinterpret_cast<float*>(c.work + p.factor);
    const float most = logf((float)vocab) + 0.5f;  // |p (log p + H)| <= 1/e + log(vocab)
    if (bad(launch(grad_scale_kernel, dim3(1), dim3(256), st, rows, most, c.scale, c.grad_logprobs, c.grad_entropy, factor)))
      return TT_ERR_HIP;
  }
  if (c.grad_weight && bad(transpose(c.hidden, c.width, hidden_t, p.padded, st))) return TT_ERR_HIP;
  for (int64_t first = 0; first < vocab; first += c.piece) {
    const int64_t n = vocab - first < c.piece ? vocab - first : c.piece, n_padded = up(n, 64);
    const Operand<T> weight{c.weight.p + first * c.weight.stride, c.weight.stride, n};
    const GradLogitsArgs<T> ga{weight,  c.hidden,        c.width,        first, vocab,    c.scale, c.targets, c.stats,
                               c.entropy, c.grad_logprobs, c.grad_entropy, factor,
                               c.grad_hidden ? g : nullptr, c.grad_weight ? gt : nullptr, n_padded, p.padded, 0, 0};
    if (bad(vec ? grad_logits<Tile<T, 256, 256, 2, 2, true>>(ga, st) : grad_logits<Tile<T, 256, 256, 4, 2, false>>(ga, st)))
      return TT_ERR_HIP;
    using Whole = Tile<T, 256, 256, 2, 2, true>;
    if (c.grad_weight) {
      const ProductArgs<T> pa{{hidden_t, p.padded, c.width}, {gt, p.padded, n}, p.padded, p.padded, 0, 0, factor,
                              c.grad_weight + first * c.grad_weight_stride, c.grad_weight_stride, nullptr, false};
      if (bad(product<Whole>(pa, st))) return TT_ERR_HIP;
    }
    if (c.grad_hidden) {
      if (bad(transpose(weight, c.width, weight_t, n_padded, st))) return TT_ERR_HIP;
      const ProductArgs<T> pa{{weight_t, n_padded, c.width}, {g, n_padded, rows}, n_padded, p.k_part, 0, 0, nullptr,
                              nullptr, 0, sums, first > 0};
      if (bad(product<Whole>(pa, st))) return TT_ERR_HIP;
    }
  }
  if (c.grad_hidden) {
    const int64_t blocks = div_up(rows * c.width, 256);
    const int32_t used = (int32_t)div_up(up(vocab < c.piece ? vocab : c.piece, 64), p.k_part);  // parts of the first piece
    if (bad(launch(sum_parts_kernel<T>, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), dim3(256), st,
                   static_cast<const float*>(sums), used, rows, c.width, static_cast<const float*>(factor), c.grad_hidden,
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
      !good_scale(scale) || workspace_bytes < need)
    return TT_ERR_BAD_ARG;
  if (rows == 0) return TT_OK;
  if (!hidden || !weight || !workspace) return TT_ERR_NULL_ARG;
  if (div_up(rows, 4) > (int64_t)UINT32_MAX / 256) return TT_ERR_TOO_LARGE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  float* given = static_cast<float*>(workspace);
  Part* parts = reinterpret_cast<Part*>(static_cast<uint8_t*>(workspace) + up(rows * 4, 256));
  auto go = [&](auto zero) {
    using T = decltype(zero);
    const HeadArgs<T> a{{static_cast<const T*>(weight), weight_stride, vocab},
                        {static_cast<const T*>(hidden), hidden_stride, rows},
                        width, scale, targets, parts, given, 0, 0};
    return vectors(a.weight, width) && vectors(a.hidden, width) ? forward_by_rows<T, true>(a, st)
                                                                : forward_by_rows<T, false>(a, st);
  };
  const int s = type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
  if (s != TT_OK) return s;
  return launch(head_join_kernel, dim3((uint32_t)div_up(rows, 4)), dim3(256), st, static_cast<const Part*>(parts),
                static_cast<const float*>(given), (int32_t)div_up(vocab, forward_tile_rows(rows)), rows, vocab, scale,
                targets, logprobs, stats, entropy) == hipSuccess
             ? TT_OK
             : TT_ERR_HIP;
}

extern "C" int64_t tt_head_scores_grad_workspace(int64_t rows, int64_t vocab, int64_t width, int32_t ample) {
  if (!head_sizes(rows, vocab, width)) return TT_ERR_BAD_ARG;
  if (rows == 0) return 0;
  return grad_plan(rows, width, ample ? up(vocab, PIECE) : PIECE).bytes;
}

extern "C" int tt_head_scores_grad(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                                   int32_t type, int64_t rows, int64_t vocab, int64_t width, float scale,
                                   const int32_t* targets, const float* stats, const float* entropy,
                                   const float* grad_logprobs, const float* grad_entropy, void* grad_hidden,
                                   int64_t grad_hidden_stride, void* grad_weight, int64_t grad_weight_stride,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
  const int64_t need = tt_head_scores_grad_workspace(rows, vocab, width, 0);
  if (need < 0 || (type != TT_BF16 && type != TT_F16) || hidden_stride < width || weight_stride < width ||
      (grad_hidden && grad_hidden_stride < width) || (grad_weight && grad_weight_stride < width) || !good_scale(scale) ||
      workspace_bytes < need)
    return TT_ERR_BAD_ARG;
  if (!grad_hidden && !grad_weight) return TT_OK;
  if (!weight || (rows > 0 && (!hidden || !stats || !workspace || (grad_entropy && !entropy)))) return TT_ERR_NULL_ARG;
  // launches of at most 2^32 threads
  if (div_up(vocab, 256) * (div_up(rows, 256) + div_up(width, 256)) > (int64_t)UINT32_MAX / 512 ||
      up(rows, 64) / 64 * div_up(width, 64) > (int64_t)UINT32_MAX / 256 ||
      div_up(vocab, 64) * div_up(width, 64) > (int64_t)UINT32_MAX / 256)
    return TT_ERR_TOO_LARGE;
  // the largest piece of the vocabulary that the workspace holds
  int64_t lo = 1, hi = div_up(vocab, PIECE);
  while (lo < hi) {
    const int64_t mid = (lo + hi + 1) / 2;
    if (rows == 0 || grad_plan(rows, width, mid * PIECE).bytes <= workspace_bytes) lo = mid;
    else hi = mid - 1;
  }
  auto go = [&](auto zero) {
    using T = decltype(zero);
    return run_gradients(GradCall<T>{{static_cast<const T*>(hidden), hidden_stride, rows},
                                     {static_cast<const T*>(weight), weight_stride, vocab},
                                     width, scale, targets, stats, entropy, grad_logprobs, grad_entropy,
                                     static_cast<T*>(grad_hidden), static_cast<T*>(grad_weight), grad_hidden_stride,
                                     grad_weight_stride, static_cast<uint8_t*>(workspace), lo * PIECE},
                         static_cast<hipStream_t>(stream));
  };
  return type == TT_BF16 ? go(bf16_t{}) : go(f16_t{});
}
