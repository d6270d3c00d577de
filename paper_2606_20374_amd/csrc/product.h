// Matrix products on bfloat16 or float16 tiles, with 32-bit sums: the part
// that the feed-forward block and the cross entropy share.
//
//   C[m][n] = sum over k of A(m, k) B(n, k)
//
// Either operand is stored with k innermost ("rows": x, weights in a forward
// product) or with k as the outer dimension ("columns": weights and inputs in
// gradients). A workgroup owns TM x TN of C and takes k in steps of 64 through
// two pairs of LDS tiles, loaded straight from memory.
//
// All products are v_mfma_f32_16x16x32 with B's rows as the instruction's
// first operand, so that a lane holds one m (its column) and four consecutive
// n: with c = lane % 16 and q = lane / 16, register e of a block is n = 4 q + e,
// m = c, and of both operands a lane holds k = 8 q + j, j = 0 .. 7.
//
// Bound by power: products of 8,192^3 run at 1,484 TFLOP/s (both operands with k
// innermost), 1,469 and 1,461 (one, none), at 1.6 to 1.9 GHz; in the operators'
// large calls the matrix units are busy 74 to 79% of the cycles. The 32x32x16 instruction, which moves
// twice as much through the accumulators, took 6 to 8% longer in the same loop;
// steps of 32 k, which ask for half lines, 13% (k innermost) and 4%.
#pragma once

#include <cmath>
#include <type_traits>
#include <utility>

#include "ops_internal.h"

namespace argus {
namespace product {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 64;  // k of a tile

__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c, bf16_t) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c, f16_t) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Past every buffer's end: reads as zeros. A lane's offset is compared with what
// the scalar offset leaves of the buffer, so that one has to lie inside.
constexpr int kNowhere = 0x7ffffff0;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int64_t bytes) {
  bytes = bytes < 0 ? 0 : bytes;
  bytes = bytes > kNowhere ? kNowhere : bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}

__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, void* lds, int off, int more) {
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass has no 16-byte form and drops kernels that name it
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, off, more, 0, 0);
#endif
}

// An operand in memory. Rows: `rows` rows of `k` elements; columns: `k` rows of
// `rows` elements. Strides and the inner extents are multiples of 8 elements.
struct Operand {
  const void* p;
  int64_t rows, k, stride;
};

// Loads of both halves of tiles of 2 ROWS rows by 64 k with k innermost: 128
// bytes a row (requests of 64 bytes leave half of each L2 line unused), eight
// pieces of 16 bytes. Piece c of row r lies at place c ^ (r >> 1 & 7), so that
// the 16 rows of one cycle's read take all 64 banks; a wavefront's lanes write
// consecutive places, so the exchange is made on the global side.
template <int ROWS, int THREADS>
struct LoadRows {
  static constexpr int N = ROWS * 8 / THREADS;
  static_assert(N >= 1 && ROWS * 8 % THREADS == 0 && THREADS % 128 == 0);
  __amdgpu_buffer_rsrc_t r[2];
  int off[2][N], at;  // the same in both halves where they are of one operand
  __device__ __forceinline__ LoadRows(const Operand& o, int64_t row0) : LoadRows(o, row0, o, row0 + ROWS) {}
  // halves of their own
  __device__ __forceinline__ LoadRows(const Operand& o, int64_t row0, const Operand& p, int64_t row1) {
    const int row = threadIdx.x >> 3;
    at = ((threadIdx.x & 7) ^ ((threadIdx.x >> 4) & 7)) * 8;
    row1 = row1 < p.rows ? row1 : p.rows - 1;  // a half past the end: of one row, and dropped
    r[0] = buffer((const char*)o.p + row0 * o.stride * 2, ((o.rows - row0 - 1) * o.stride + o.k) * 2);
    r[1] = buffer((const char*)p.p + row1 * p.stride * 2, ((p.rows - row1 - 1) * p.stride + p.k) * 2);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      off[0][i] = (int)(((row + i * (THREADS / 8)) * o.stride + at) * 2);
      off[1][i] = (int)(((row + i * (THREADS / 8)) * p.stride + at) * 2);
    }
  }
  // Half of the tile of k = k0 .. k0 + 63, zeros from k_end on.
  template <class T>
  __device__ __forceinline__ void load(int half, int k0, int k_end, T* tile) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), from = k0 < k_end ? k0 * 2 : 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      load_lds(r[half], tile + (i * THREADS + wave * 64) * 8, k0 + at < k_end ? off[half][i] : kNowhere, from);
  }
};

// Place of piece c of row k of a half tile with k as the outer dimension, as an
// exchange c ^ swap: a transposed read takes, of 32 lanes at a time, two
// neighbouring pieces of rows k .. k + 3 and k + 8 .. k + 11, which are then all
// 64 banks. Rows of eight pieces lie two to the banks' width.
template <int PIECES>
__device__ __forceinline__ constexpr int swap_cols(int k) {
  static_assert(PIECES == 8 || PIECES == 16);
  return PIECES == 16 ? ((k & 3) << 2) ^ ((k >> 2) & 2) : ((k & 2) << 1) ^ ((k >> 2) & 2);
}

// The same with k as the outer dimension: 64 k by COLS columns.
template <int COLS, int THREADS>
struct LoadCols {
  static constexpr int PIECES = COLS / 8, N = kStep * PIECES / THREADS;
  static_assert(N >= 1 && kStep * PIECES % THREADS == 0);
  const char* p;
  int64_t k, stride;
  int off[2][N], cols;
  __device__ __forceinline__ LoadCols(const Operand& o, int64_t col0) {
    p = (const char*)o.p + col0 * 2;
    k = o.k;
    stride = o.stride;
    cols = (int)(o.rows - col0 < 2 * COLS ? o.rows - col0 : 2 * COLS);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = i * THREADS + threadIdx.x, row = at / PIECES;
        const int c = h * COLS + ((at % PIECES) ^ swap_cols<PIECES>(row)) * 8;
        off[h][i] = c < cols ? (int)((row * stride + c) * 2) : kNowhere;
      }
  }
  template <class T>
  __device__ __forceinline__ void load(int half, int k0, int k_end, T* tile) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int left = (int)(k < k_end ? k : k_end) - k0;
    const auto r = buffer(p + k0 * stride * 2, ((int64_t)(left - 1) * stride + cols) * 2);
#pragma unroll
    for (int i = 0; i < N; ++i) load_lds(r, tile + (i * THREADS + wave * 64) * 8, off[half][i], 0);
  }
};

// Reads of blocks of 16 rows (or columns) by 32 k as operands, from row
// `first` of a half tile on.
template <bool ROWS, int WIDTH, int BLOCKS>
struct Read;
template <int WIDTH, int BLOCKS>
struct Read<true, WIDTH, BLOCKS> {
  uint32_t at[2];
  __device__ __forceinline__ explicit Read(int first) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < 2; ++s) at[s] = (first + (lane & 15)) * 128 + ((4 * s + (lane >> 4)) ^ ((lane >> 1) & 7)) * 16;
  }
  template <class T>
  __device__ __forceinline__ s16x8 get(const T* tile, int b, int s) const {
    typedef __attribute__((address_space(3))) const char* lds_ptr;
    const lds_ptr p = (lds_ptr)(__attribute__((address_space(3))) const void*)tile;
    return *(__attribute__((address_space(3))) const s16x8*)(p + at[s] + b * 16 * 128);
  }
};
template <int WIDTH, int BLOCKS>
struct Read<false, WIDTH, BLOCKS> {
  uint32_t at[BLOCKS];
  __device__ __forceinline__ explicit Read(int first) {
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
      at[b] = (8 * q + (i >> 2)) * WIDTH * 2 +
              (((first + 16 * b) / 8 + (i & 3) / 2) ^ swap_cols<WIDTH / 8>(8 * q + (i >> 2))) * 16 + (i & 1) * 8;
  }
  // Sixteen lanes read four rows of sixteen columns and each gets one column.
  template <class T>
  __device__ __forceinline__ s16x8 get(const T* tile, int b, int s) const {
    typedef __attribute__((address_space(3))) const char* lds_ptr;
    typedef __attribute__((address_space(3))) s16x4* tr_ptr;
    const lds_ptr p = (lds_ptr)(__attribute__((address_space(3))) const void*)tile;
    const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + at[b] + (32 * s) * WIDTH * 2));
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + at[b] + (32 * s + 4) * WIDTH * 2));
    return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// At most n of the loads that this wavefront issued are still under way, and
// none of its reads from LDS.
template <int n>
__device__ __forceinline__ void wait_loads() {
  static_assert(n < 64);
  __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | ((n >> 4) << 14));
}
// All wavefronts are here; nothing is waited for.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Arrays of a workgroup's LDS. Kernels that hold tiles of several layouts use
// the same ones for all.
template <class T, int SIZE>
struct Lds {
  template <int WHICH>
  static __device__ __forceinline__ T* array() {
    __shared__ __align__(16) T a[SIZE];
    return a;
  }
  template <int N, int... I>
  static __device__ __forceinline__ void all(T* (&p)[N], std::integer_sequence<int, I...>) {
    ((p[I] = array<I>()), ...);
  }
};

// The tile of a workgroup, in two halves of its rows and two of its columns.
// Wavefronts lie WM by WN over it, each with the same share of both halves, so
// that it takes the tile's quarters one after the other; a feed-forward tile
// holds gate columns in one half and up columns in the other.
template <class T_, int TM_, int TN_, int WM_, int WN_, bool ROWS_A, bool ROWS_B, int STAGES = 2>
struct Tile {
  static_assert(STAGES == 2 || STAGES == 4);
  using T = T_;
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, THREADS = 64 * WM * WN;
  static constexpr int FM = TM / WM / 16, FN = TN / WN / 16, HM = FM / 2, HN = FN / 2;
  static_assert(HM >= 1 && HN >= 1 && FM % 2 == 0 && FN % 2 == 0);
  using LoadA = std::conditional_t<ROWS_A, LoadRows<TM / 2, THREADS>, LoadCols<TM / 2, THREADS>>;
  using LoadB = std::conditional_t<ROWS_B, LoadRows<TN / 2, THREADS>, LoadCols<TN / 2, THREADS>>;
  static constexpr int kLoads = LoadA::N + LoadB::N;  // of one half of each

  f32x4 acc[FM][FN];

  static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
  static __device__ __forceinline__ int row_of(int b) { return b / HM * (TM / 2) + wave() / WN * (HM * 16) + b % HM * 16; }
  static __device__ __forceinline__ int col_of(int b) { return b / HN * (TN / 2) + wave() % WN * (HN * 16) + b % HN * 16; }

  // What is loaded together, the same half of A and of B (with four stages both
  // halves), is an array of its own: the compiler, too, waits before a read for
  // the loads into its array, and tells only a few arrays apart.
  static constexpr int kArrays = 4, kA = TM / 2 * kStep, kB = TN / 2 * kStep;
  static constexpr int kArray = (kA + kB) * (STAGES / 2);
  using Shared = Lds<T, kArray>;

  // Order of a quarter's instructions: its reads from LDS and its loads one by
  // one between the products.
  template <int LOADS, int READS, int PRODUCTS = 2 * HM * HN>
  static __device__ __forceinline__ void interleave() {
    constexpr int kProducts = PRODUCTS, kAll = READS + LOADS;
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
      for (int j = i * kAll / kProducts; j < (i + 1) * kAll / kProducts; ++j) {
        if (j < READS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        else __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // Rounds the values v(j, e) of row block i and of the columns of halves H .. H +
  // NH - 1 to T and writes them by way of LDS: 64 bytes of a row together, where
  // a lane of the result holds 8. row(r) is the tile's row r in memory, or null;
  // columns from `cols` on (a multiple of 8) are left out.
  template <int H, int NH, class V, class R>
  __device__ __forceinline__ void write(int i, int64_t cols, V v, R row) {
    constexpr int W = HN * 16 + 8, kEach = kArray / (WM * WN / 2);  // 16 bytes more: rows in other banks
    static_assert(HN == 2 && 2 * 16 * W <= kEach);
    const int lane = threadIdx.x & 63;
    T* s = (wave() & 1 ? Shared::template array<1>() : Shared::template array<0>()) + (wave() >> 1) * kEach;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int j = 0; j < HN; ++j) {
        Vec<T, 4> o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o.e[e] = (T)v((H + h) * HN + j, e);
        *(uint2*)(s + (h * 16 + (lane & 15)) * W + j * 16 + 4 * (lane >> 4)) = __builtin_bit_cast(uint2, o);
      }
    asm volatile("" ::: "memory");  // one wavefront: LDS takes its instructions in order
    const int c = (lane & 3) * 8;
    T* to = row(row_of(i) + (lane >> 2));
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const uint4 x = *(const uint4*)(s + (h * 16 + (lane >> 2)) * W + c);
      const int64_t col = col_of((H + h) * HN) + c;
      if (to && col < cols) *(uint4*)(to + col) = x;
    }
    asm volatile("" ::: "memory");
  }

  // Adds the products of k = k_begin .. k_end - 1 (k_begin a multiple of kStep).
  //
  // Two stages: tiles are taken by halves. A step of 64 k takes the quarters (A0,
  // B0), (A0, B1), (A1, B1), (A1, B0), and during each reads the half that the
  // next one but one (A0, B0: of the next step) needs. At its first barrier the
  // step's A0 and B0 have been read by all, and their places get those of the
  // step after the next; at the second, before (A1, B1), A1 and B1. So each load
  // has one and a half steps, and two barriers a step are enough.
  //
  // Four stages, for workgroups that are alone on their CU: a step reads all
  // operands of the next one, so that a wavefront with few products does not
  // wait for LDS at each of them, and a load has three steps.
  template <bool MORE = false>  // to what is there
  __device__ __forceinline__ void run(const LoadA& la, const LoadB& lb, int k_begin, int k_end) {
    T *arrays[kArrays], *A[2 * STAGES], *B[2 * STAGES];
    Shared::all(arrays, std::make_integer_sequence<int, kArrays>{});
#pragma unroll
    for (int i = 0; i < 2 * STAGES; ++i) {
      A[i] = STAGES == 2 ? arrays[i] : arrays[i / 2] + i % 2 * (kA + kB);
      B[i] = A[i] + kA;
    }
    const Read<ROWS_A, TM / 2, HM> ra(wave() / WN * (HM * 16));
    const Read<ROWS_B, TN / 2, HN> rb(wave() % WN * (HN * 16));
    if constexpr (!MORE)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    if (k_begin >= k_end) return;
    constexpr int RA = 2 * HM * (ROWS_A ? 1 : 2), RB = 2 * HN * (ROWS_B ? 1 : 2);
    s16x8 fa[STAGES][2][HM], fb[STAGES][2][HN];
    auto read_a = [&](int to, const T* A) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < HM; ++i) fa[to][s][i] = ra.get(A, i, s);
    };
    auto read_b = [&](int to, const T* B) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < HN; ++j) fb[to][s][j] = rb.get(B, j, s);
    };
    // quarter (hi, hj), with the operands fa[x] and fb[y]
    auto multiply = [&](int hi, int hj, int x, int y) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < HM; ++i)
#pragma unroll
          for (int j = 0; j < HN; ++j)
            acc[hi * HM + i][hj * HN + j] = mfma(fb[y][s][j], fa[x][s][i], acc[hi * HM + i][hj * HN + j], T{});
    };
    auto load = [&](int half, int k0, T* A, T* B) __attribute__((always_inline)) {
      la.load(half, k0, k_end, A);
      lb.load(half, k0, k_end, B);
    };
    int k = k_begin;
    // The loops below have one way in and one out: with a way out in the middle
    // the compiler allows for paths that leave steps out, on which loads would
    // still be under way, and waits for all of them in every round.
    const int steps = (k_end - k_begin + kStep - 1) / kStep;
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) load(h, k + s * kStep, A[2 * s + h], B[2 * s + h]);
    if constexpr (STAGES == 2) {
      wait_loads<3 * kLoads>();
      meet();
      read_a(0, A[0]);
      read_b(0, B[0]);
      auto step = [&](int x) __attribute__((always_inline)) {
        const int next = 2 * (x ^ 1);
        wait_loads<2 * kLoads>();
        meet();
        load(0, k + 2 * kStep, A[2 * x], B[2 * x]);
        read_b(x ^ 1, B[2 * x + 1]);
        multiply(0, 0, 0, x);
        interleave<kLoads, RB>();
        read_a(1, A[2 * x + 1]);
        multiply(0, 1, 0, x ^ 1);
        interleave<0, RA>();
        wait_loads<2 * kLoads>();
        meet();
        load(1, k + 2 * kStep, A[2 * x + 1], B[2 * x + 1]);
        read_a(0, A[next]);
        multiply(1, 1, 1, x ^ 1);
        interleave<kLoads, RA>();
        read_b(x ^ 1, B[next]);
        multiply(1, 0, 1, x);
        interleave<0, RB>();
        k += kStep;
      };
      for (int n = steps / 2; n > 0; --n) {
        step(0);
        step(1);
      }
      if (steps & 1) step(0);
    } else {
      auto read = [&](int to, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          read_a(2 * to + h, A[2 * s + h]);
          read_b(2 * to + h, B[2 * s + h]);
        }
      };
      wait_loads<6 * kLoads>();
      meet();
      read(0, 0);
      auto step = [&](int s) __attribute__((always_inline)) {
        const int x = s & 1;
        wait_loads<4 * kLoads>();
        meet();
#pragma unroll
        for (int h = 0; h < 2; ++h) load(h, k + 4 * kStep, A[2 * s + h], B[2 * s + h]);
        read(x ^ 1, (s + 1) % 4);
#pragma unroll
        for (int h = 0; h < 4; ++h) multiply(h >> 1, h & 1, 2 * x + (h >> 1), 2 * x + (h & 1));
        interleave<2 * kLoads, 2 * (RA + RB), 2 * FM * FN>();
        k += kStep;
      };
      for (int n = steps / 4; n > 0; --n) {
        step(0);
        step(1);
        step(2);
        step(3);
      }
      if (steps & 3) step(0);
      if ((steps & 3) > 1) step(1);
      if ((steps & 3) > 2) step(2);
    }
    wait_loads<0>();  // none may write into LDS that another use has taken
    meet();
  }
};

// Tile (m, n) and part of k of workgroup `at` of S by mt by nt. Workgroups go to
// the eight XCDs in turn; each XCD takes a consecutive piece of the order, which
// runs through the parts and in each through bands of kBand rows of tiles, so
// that tiles which share operands are in the same L2 at the same time.
constexpr int kBand = 8;
__device__ __forceinline__ int tile_at(int at, int mt, int nt, int& m, int& n, int S = 1) {
  int id = (int)xcd_item(at, (int64_t)S * mt * nt);
  const int part = id / (mt * nt);
  id -= part * (mt * nt);
  const int band = id / (kBand * nt), in = id - band * (kBand * nt);
  const int high = mt - band * kBand < kBand ? mt - band * kBand : kBand;
  n = in / high;
  m = band * kBand + in - n * high;
  return part;
}

// Part s of S of k steps: multiples of kStep.
__device__ __forceinline__ void my_part(int64_t k, int s, int S, int& begin, int& end) {
  const int64_t steps = (k + kStep - 1) / kStep;
  begin = (int)(steps * s / S) * kStep;
  end = (int)(steps * (s + 1) / S) * kStep;
  if (end > k) end = (int)k;
}

// Where the rows of a product go: the first n0 to out0, those from at1 on to
// out1, n1 of them. Rows between are not kept.
struct Rows {
  void *out0, *out1;
  int64_t n0, at1, n1;
};
template <class T>
__device__ __forceinline__ T* row_at(const Rows& r, int64_t m, int64_t cols) {
  if (m < r.n0) return (T*)r.out0 + m * cols;
  if (m >= r.at1 && m < r.at1 + r.n1) return (T*)r.out1 + (m - r.at1) * cols;
  return nullptr;
}

// Products of few tokens, bound by the bytes of the weights: a workgroup takes NB
// blocks of 16 weight rows, each read once, straight into registers, by 16-byte
// pieces of which a wavefront has U times 2 NB under way; its wavefronts take
// every kFewWaves-th 64 k, and their sums are joined in LDS. The tokens' rows, 16
// to a block, come from L2. Feed-forward of 4 tokens, 4,096 x 12,288: 36.8 us, 5.5
// TB/s (39.1 where the compiler may put loads behind products); of 32 50.8 (59.8).
constexpr int kFewWaves = 4;
constexpr int kFew = 32;  // tokens, at most: from 33 on tiles are as fast

template <class T, int NT, int NB, int U>
struct Few {
  f32x4 acc[NB][NT];

  // w[b]: the rows of block b, `off[b]` this lane's bytes from its first row on
  // (row lane % 16, k = 8 (lane / 16)); x and xoff the same of the tokens.
  __device__ __forceinline__ void run(const __amdgpu_buffer_rsrc_t (&w)[NB], const int (&off)[NB],
                                      __amdgpu_buffer_rsrc_t x, const int (&xoff)[NT], int K) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = (threadIdx.x & 63) >> 4 << 3;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0, 0, 0, 0};
    auto round = [&](int k0, auto whole) __attribute__((always_inline)) {
      s16x8 wf[U][2][NB], xf[U][2][NT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = k0 + u * kFewWaves * 64 + 32 * h, from = whole || k < K ? k * 2 : 0;
          const bool there = whole || k + at < K;
#pragma unroll
          for (int b = 0; b < NB; ++b)
            wf[u][h][b] = __builtin_bit_cast(s16x8, __builtin_amdgcn_raw_buffer_load_b128(w[b], there ? off[b] : kNowhere, from, 0));
#pragma unroll
          for (int t = 0; t < NT; ++t)
            xf[u][h][t] = __builtin_bit_cast(s16x8, __builtin_amdgcn_raw_buffer_load_b128(x, there ? xoff[t] : kNowhere, from, 0));
        }
      __builtin_amdgcn_sched_barrier(0);  // all loads first
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[b][t] = mfma(wf[u][h][b], xf[u][h][t], acc[b][t], T{});
    };
    constexpr int kRound = kFewWaves * 64 * U;
    int k0 = wave * 64;
    for (; k0 + kRound - (kFewWaves - 1) * 64 <= K; k0 += kRound) round(k0, std::true_type{});
    for (; k0 < K; k0 += kRound) round(k0, std::false_type{});
  }

  // Sums over the wavefronts, in their order: tokens t are then wavefront t %
  // kFewWaves's.
  __device__ __forceinline__ void join() {
    __shared__ f32x4 part[kFewWaves][NB * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t) part[wave][b * NT + t][lane] = acc[b][t];
    __syncthreads();
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (t % kFewWaves != wave) continue;
        f32x4 v = part[0][b * NT + t][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) v += part[w][b * NT + t][lane];
        acc[b][t] = v;
      }
  }
};

// A grid of mt by nt tiles in S parts of k, for the most rows there can be. Where
// the rows are counted on the device and are fewer, the same workgroups take
// more parts of k, at most `most`.
struct Grid {
  int32_t mt, nt, S, most;
};
__device__ __forceinline__ Grid counted(Grid g, int64_t count, int tile) {
  const int all = g.mt * g.nt * g.S;
  g.mt = (int)((count + tile - 1) / tile);
  if (g.mt < 1) g.mt = 1;
  const int s = all / (g.mt * g.nt);
  g.S = s < g.most ? s : g.most > g.S ? g.most : g.S;
  return g;
}

// The gradients' products: B is one operand, or two one after the other along
// k (the second begins at k1, a multiple of kStep). The rows of A may be
// counted on the device (*n), or k (COUNT_K): then B is b1 where fewer are
// counted than there are, else b. Written in T, times f scale where f is there,
// or, by S parts, as 32-bit sums [S][mt TM][cols], added to what is there where
// `add` is set.
struct Grad {
  Operand a, b, b1;
  int64_t k1;
  const uint32_t* n;
  Rows rows;
  float* sums;
  Grid grid;
  int32_t tile, add;  // rows of a tile
  const float* f;
  float scale;
  const int32_t* place;
};
__device__ __forceinline__ float factor_of(const Grad& g) { return g.f ? *g.f * g.scale : 1.0f; }

template <class TT, bool TWO, bool COUNT_K>
__device__ __forceinline__ void grad_body(Grad g, int block) {
  using T = typename TT::T;
  Grid grid = g.grid;
  if (g.n) {
    const int64_t count = __builtin_amdgcn_readfirstlane((int)*g.n);
    if (COUNT_K) {
      if (count < g.a.k) g.b = g.b1;
      g.a.k = g.b.k = count;
    } else {
      if (count == 0) return;
      grid = counted(grid, count, TT::TM);
      g.a.rows = count;
    }
  }
  if (block >= grid.S * grid.mt * grid.nt) return;
  int m, n, begin, end;
  const int part = tile_at(block, grid.mt, grid.nt, m, n, grid.S);
  const int64_t m0 = (int64_t)m * TT::TM, n0 = (int64_t)n * TT::TN;
  my_part(g.a.k, part, grid.S, begin, end);
  TT t;
  const typename TT::LoadA la(g.a, m0);
  const typename TT::LoadB lb(g.b, n0);
  if constexpr (TWO) {
    // one loop after the other: a choice between them at each load breaks the
    // order of the loop's instructions (gradients of 16,384 tokens, 4,096 wide
    // with 12,288 inside: 8,492 us in place of 5,406)
    const int k1 = (int)g.k1;
    t.run(la, lb, begin, end < k1 ? end : k1);
    g.b1.p = (const char*)g.b1.p - g.k1 * g.b1.stride * 2;  // its k count from k1 on
    g.b1.k += g.k1;
    t.template run<true>(la, typename TT::LoadB(g.b1, n0), begin > k1 ? begin : k1, end);
  } else {
    t.run(la, lb, begin, end);
  }
  const int lane = threadIdx.x & 63;
  const int64_t cols = g.b.rows;
  if (!g.sums) {
    const float f = factor_of(g);
#pragma unroll
    for (int i = 0; i < TT::FM; ++i) {
      const int64_t mine = m0 + TT::row_of(i) + (lane & 15);
      const bool none = g.place && mine < g.a.rows && g.place[mine] < 0;
      t.template write<0, 2>(i, cols - n0, [&](int j, int e) { return none ? 0.0f : t.acc[i][j][e] * f; },
                             [&](int r) {
                               T* row = m0 + r < g.a.rows ? row_at<T>(g.rows, m0 + r, cols) : nullptr;
                               return row ? row + n0 : nullptr;
                             });
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < TT::FM; ++i) {
    const int64_t row = m0 + TT::row_of(i) + (lane & 15);
    if (row >= g.a.rows) continue;
    float* sum = g.sums + ((int64_t)part * grid.mt * TT::TM + row) * cols;
#pragma unroll
    for (int j = 0; j < TT::FN; ++j) {
      const int64_t c = n0 + TT::col_of(j) + 4 * (lane >> 4);
      if (c >= cols) continue;  // cols is a multiple of 8
      float4 v = make_float4(t.acc[i][j][0], t.acc[i][j][1], t.acc[i][j][2], t.acc[i][j][3]);
      if (g.add) {
        const float4 o = *(const float4*)(sum + c);
        v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
      }
      *(float4*)(sum + c) = v;
    }
  }
}

// Both gradients of an operator: the input's (tiles X, A with k innermost) and
// the weights' (tiles W). The longer workgroups, `first` of them, go first.
template <class X, class W, bool TWO, bool COUNT_K>
__global__ __launch_bounds__(X::THREADS) void grad_pair(Grad x, Grad w, int first, int w_first) {
  const bool of_w = ((int)blockIdx.x < first) == (w_first != 0);
  const int block = (int)blockIdx.x < first ? blockIdx.x : blockIdx.x - first;
  if (of_w) grad_body<W, false, COUNT_K>(w, block);
  else grad_body<X, TWO, false>(x, block);
}

// Sum of the S parts, in their order, of eight columns.
__device__ __forceinline__ Vec<float, 8> sum_parts(const float* sums, const Grid& g, int tile, int64_t row, int64_t cols, int64_t c) {
  Vec<float, 8> v{};
  for (int s = 0; s < g.S; ++s) {
    const Vec<float, 8> a = load_vec<8>(sums + (((int64_t)s * g.mt * tile + row) * cols + c));
#pragma unroll
    for (int j = 0; j < 8; ++j) v.e[j] += a.e[j];
  }
  return v;
}

template <class T>
__global__ __launch_bounds__(256) void grad_join(Grad g, int64_t rows) {
  const int64_t cols = g.b.rows, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= rows * cols) return;
  const int64_t row = i / cols;
  T* out = row_at<T>(g.rows, row, cols);
  if (!out) return;
  const float f = factor_of(g);
  const Vec<float, 8> v = sum_parts(g.sums, g.grid, g.tile, row, cols, i - row * cols);
  Vec<T, 8> o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o.e[j] = (T)(v.e[j] * f);
  store_vec<8>(out + i - row * cols, o);
}

template <class T, bool ROWS_A, bool ROWS_B>
using Big = Tile<T, 256, 256, 2, 4, ROWS_A, ROWS_B>;
template <class T, bool ROWS_A, bool ROWS_B, int STAGES = 2>
using Small = Tile<T, 128, 128, 2, 2, ROWS_A, ROWS_B, STAGES>;
// Both operands with k innermost:
template <class T>
using Wide = Tile<T, 128, 256, 2, 4, true, true>;
template <class T>
using Middle = Tile<T, 192, 128, 2, 2, true, true>;
template <class T, int STAGES = 2>
using Short = Tile<T, 64, 128, 2, 2, true, true, STAGES>;

// Tiles of a forward product, by the time that their workgroups take. A CU holds
// `each` of them; where it has fewer, a step is shorter. Feed-forward (tokens,
// width, inner width), big, wide, middle, small and short tiles, us: 100 x 2,048 x
// 8,192 43, 34, 29, 26, 22; 300 x 2,048 x 8,192 46, 33, 32, 38, 42; 500 x 4,096 x 5,120
// 80, 60, 53, 70, 76; 1,000 x 1,000 x 2,720 29, 20, 25, 23, 25; 4,000 x 4,096 x 5,120 271,
// 281, 291, 310, 407.
constexpr int kCus = 256;
enum Kind { kBig, kWide, kMiddle, kSmall, kShort };
struct KindCost {
  int tm, tn, threads, each;
  float step[3], ends[3], once;  // us a step with 1, 2, 3 on a CU, a workgroup's ends, and once
};
// What a tile ends with: feed-forward's one output or three, or the cross entropy's
// exponentials, for which there are big, small and short tiles only.
enum Ends { kOne, kThree, kLoss };
inline Kind kind_of(int64_t rows, int64_t cols, int64_t k, Ends ends) {
  constexpr KindCost costs[] = {{256, 256, 512, 1, {1.18f, 0, 0}, {9.0f, 14.5f, 11.0f}, 0},
                                {128, 256, 512, 1, {0.87f, 0, 0}, {5.0f, 7.0f, 0}, 0},
                                {192, 128, 256, 2, {0.69f, 1.25f, 0}, {4.0f, 9.0f, 0}, 4.0f},
                                {128, 128, 256, 2, {0.72f, 1.05f, 0}, {2.0f, 5.5f, 3.5f}, 3.0f},
                                {64, 128, 256, 3, {0.55f, 0.85f, 1.13f}, {1.0f, 2.8f, 2.0f}, 3.0f}};
  const float steps = (float)ceil_div(k, kStep);
  Kind best = kBig;
  float least = 0;
  for (int i = 0; i < 5; ++i) {
    if (ends == kLoss && (i == kWide || i == kMiddle)) continue;
    const KindCost& c = costs[i];
    const int64_t n = ceil_div(rows, c.tm) * ceil_div(cols, c.tn), rounds = n / (c.each * kCus), rest = n - rounds * c.each * kCus;
    // an axis of a launch takes below 2^32 threads; the biggest tile's are always fewer
    if (i > 0 && n * c.threads >= (int64_t)1 << 32) continue;
    float t = c.once + (float)rounds * (steps * c.step[c.each - 1] + c.ends[ends]);
    if (rest) t += steps * c.step[ceil_div(rest, kCus) - 1] + c.ends[ends];
    if (i > 0 && t >= least) continue;
    least = t;
    best = (Kind)i;
  }
  return best;
}
// Calls go with the tile of a kind.
template <class T, bool LOSS, class F>
auto with_tile(int64_t rows, int64_t cols, int64_t k, bool three, F go) {
  const Kind kind = kind_of(rows, cols, k, LOSS ? kLoss : three ? kThree : kOne);
  if (kind == kBig) return go(Big<T, true, true>{});
  if constexpr (!LOSS) {
    if (kind == kWide) return go(Wide<T>{});
    if (kind == kMiddle) return go(Middle<T>{});
  }
  if (kind == kSmall) return go(Small<T, true, true>{});
  // one to a CU waits for its loads: four stages in place of two
  return ceil_div(rows, 64) * ceil_div(cols, 128) <= kCus ? go(Short<T, 4>{}) : go(Short<T>{});
}

// How the two gradients of an operator are taken: tiles and parts of k. Their
// workgroups share the chip, so that the parts of one fill what the tiles of the
// other leave: feed-forward gradient of 2,000 tokens, 2,048 wide with 5,120 inside 186
// us, 219 in two launches; of 4,000, 1,024 with 2,048 90 and 116. Of 75 plans tried by
// hand in each of nine cases none was more than 7% better than the one chosen.
struct Plan {
  bool big, deep, w_first;
  Grid x, w;  // no sums where S is 1
  int tile() const { return big ? 256 : 128; }
};
constexpr int64_t kPart = 512;  // k of a part, at least
constexpr int kMostParts = 64;

// The time that n1 workgroups of a1 and then n2 of a2 take on `slots` places.
inline float time_of(float n1, float a1, float n2, float a2, float slots) {
  const float rounds = floorf(n1 / slots), late = n1 - rounds * slots, t0 = rounds * a1, t1 = t0 + a1;
  if (n2 <= 0) return late > 0 ? t1 : t0;
  float j = floorf(((n1 * a1 + n2 * a2) / slots - t0) / a2), m;
  do {
    m = t0 + j * a2;
    j += 1;
  } while ((slots - late) * (j - 1) + late * fmaxf(0.0f, floorf((m - t1) / a2 + 1e-3f)) < n2);
  return late > 0 ? fmaxf(m, t1) : m;
}

inline Plan plan_grads(int64_t rows_x, int64_t k_x, int64_t rows_w, int64_t k_w, int64_t cols) {
  // Microseconds of a step of 64 k, and of a workgroup's start and end, which
  // writes 16 bits a value, or 32 for parts: measured as they are in rounds of
  // workgroups that fill the chip.
  struct How {
    int tile, slots;
    float step, ends, ends_sums;
  };
  constexpr How hows[3] = {{256, kCus, 1.4f, 8.0f, 14.0f}, {128, 2 * kCus, 1.05f, 4.0f, 6.0f}, {128, kCus, 0.62f, 3.0f, 4.0f}};
  constexpr int cuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  const float steps_x = (float)ceil_div(k_x, kStep), steps_w = (float)ceil_div(k_w, kStep);
  const int most_x = (int)(k_x / kPart < 1 ? 1 : k_x / kPart < kMostParts ? k_x / kPart : kMostParts);
  const int most_w = (int)(k_w / kPart < 1 ? 1 : k_w / kPart < kMostParts ? k_w / kPart : kMostParts);
  const float longest = steps_x > steps_w ? steps_x : steps_w;
  Plan best{};
  float least = 0;
  for (const How& kind : hows) {
    const int64_t mx = ceil_div(rows_x, kind.tile), mw = ceil_div(rows_w, kind.tile), n = ceil_div(cols, kind.tile);
    int was_x = 0, was_w = 0;
    for (int cut : cuts) {
      const float length = longest / (float)cut;
      const int sx = (int)fminf((float)most_x, fmaxf(1.0f, roundf(steps_x / length)));
      const int sw = (int)fminf((float)most_w, fmaxf(1.0f, roundf(steps_w / length)));
      if (sx == was_x && sw == was_w) continue;
      was_x = sx;
      was_w = sw;
      const float nx = (float)(mx * n * sx), nw = (float)(mw * n * sw);
      if (kind.tile == 128 && kind.slots == kCus && nx + nw > kCus) break;
      const float ax = ceilf(steps_x / sx) * kind.step + (sx > 1 ? kind.ends_sums : kind.ends);
      const float aw = ceilf(steps_w / sw) * kind.step + (sw > 1 ? kind.ends_sums : kind.ends);
      float t = aw > ax ? time_of(nw, aw, nx, ax, kind.slots) : time_of(nx, ax, nw, aw, kind.slots);
      // sums are read again, at 5 TB/s
      if (sx > 1) t += 4.0f + (float)sx * (float)(rows_x * cols) * 4e-6f / 5.0f;
      if (sw > 1) t += 4.0f + (float)sw * (float)(rows_w * cols) * 4e-6f / 5.0f;
      if (least > 0 && t >= least) continue;
      least = t;
      best = {kind.tile == 256, kind.tile == 128 && kind.slots == kCus, aw > ax,
              {(int32_t)mx, (int32_t)n, sx, most_x}, {(int32_t)mw, (int32_t)n, sw, most_w}};
    }
  }
  return best;
}
// 32-bit sums of a product.
inline size_t sums_bytes(const Plan& p, const Grid& g, int64_t cols) {
  return align256((size_t)g.S * (size_t)g.mt * (size_t)p.tile() * (size_t)cols * 4);
}

// The gradients of an operator's input and of its weights, of a plan's grids.
template <class T, bool TWO, bool COUNT_K>
hipError_t launch_grads(const Plan& p, Grad& x, Grad& w, hipStream_t st) {
  x.tile = w.tile = p.tile();
  const int nx = x.grid.mt * x.grid.nt * x.grid.S, nw = w.grid.mt * w.grid.nt * w.grid.S;
  auto go = [&](auto tx, auto tw) {
    using X = decltype(tx);
    hipLaunchKernelGGL((grad_pair<X, decltype(tw), TWO, COUNT_K>), dim3((unsigned)(nx + nw)), dim3(X::THREADS), 0, st, x, w,
                       p.w_first ? nw : nx, (int)p.w_first);
    return hipGetLastError();
  };
  if (p.big) return go(Big<T, true, false>{}, Big<T, false, false>{});
  return p.deep ? go(Small<T, true, false, 4>{}, Small<T, false, false, 4>{}) : go(Small<T, true, false>{}, Small<T, false, false>{});
}
template <class T>
hipError_t launch_join(const Grad& g, int64_t rows, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(grad_join<T>, dim3((unsigned)ceil_div(rows * g.b.rows, 8 * 256)), dim3(256), 0, st, g, rows);
  return hipGetLastError();
}

}  // namespace product
}  // namespace argus
