// Matrix products on bfloat16 or float16 tiles, with 32-bit sums: the part
// that the feed-forward block and the cross entropy share.
//
//   C[m][n] = sum over k of A(m, k) B(n, k)
//
// Either operand is stored with k innermost ("rows": x, weights in a forward
// product) or with k as the outer dimension ("columns": weights and inputs in
// gradients). A workgroup owns TM x TN of C and takes k in steps of 32 through
// kBuffers pairs of LDS tiles, loaded straight from memory.
//
// All products are v_mfma_f32_32x32x16 with B's rows as the instruction's
// first operand, so that a lane holds one m (its column) and groups of four
// consecutive n: with c = lane % 32 and h = lane / 32, register i of a block
// is n = 8 (i / 4) + 4 h + i % 4, m = c, and of both operands a lane holds
// k = 8 h + j, j = 0 .. 7.
#pragma once

#include <type_traits>

#include "ops_internal.h"

namespace argus {
namespace product {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 32;  // k of a tile

__device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c, bf16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c, f16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Past every buffer's end: reads as zeros.
constexpr int kNowhere = 0x7ffffff0;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int64_t bytes) {
  if (bytes < 0) bytes = 0;
  if (bytes > kNowhere) bytes = kNowhere;
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

// Loads of tiles of ROWS rows by 32 k with k innermost: 64 bytes a row, four
// pieces of 16 bytes. Piece c of row r lies at place c ^ (r >> 2 & 3), so that
// the 16 rows of one cycle's read take all 64 banks; a wavefront's lanes write
// consecutive places, so the exchange is made on the global side.
template <int ROWS, int THREADS>
struct LoadRows {
  static constexpr int N = ROWS * 4 / THREADS;
  static_assert(N >= 1 && ROWS * 4 % THREADS == 0);
  __amdgpu_buffer_rsrc_t r;
  int off[N], at, k;
  __device__ __forceinline__ LoadRows(const Operand& o, int64_t row0) {
    const int row = threadIdx.x >> 2, c = (threadIdx.x & 3) ^ ((threadIdx.x >> 4) & 3);
    r = buffer((const char*)o.p + row0 * o.stride * 2, ((o.rows - row0 - 1) * o.stride + o.k) * 2);
    at = c * 8;
    k = (int)o.k;
#pragma unroll
    for (int i = 0; i < N; ++i) off[i] = (int)(((row + i * (THREADS / 4)) * o.stride + c * 8) * 2);
  }
  // Tile of k = k0 .. k0 + 31. With whole set, all of them exist.
  template <class T>
  __device__ __forceinline__ void load(int k0, T* tile, bool whole) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < N; ++i)
      load_lds(r, tile + (i * THREADS + wave * 64) * 8, whole || k0 + at < k ? off[i] : kNowhere, k0 * 2);
  }
};

// Loads of tiles of 32 k by COLS columns with k as the outer dimension. Piece
// c of row k lies at place c ^ 4 (k & 3): a transposed read takes, of 32 lanes
// at a time, four neighbouring pieces of four rows, which are all 64 banks.
template <int COLS, int THREADS>
struct LoadCols {
  static constexpr int PIECES = COLS / 8, N = kStep * PIECES / THREADS;
  static_assert(N >= 1 && kStep * PIECES % THREADS == 0);
  const char* p;
  int64_t k, stride;
  int off[N], cols;
  __device__ __forceinline__ LoadCols(const Operand& o, int64_t col0) {
    p = (const char*)o.p + col0 * 2;
    k = o.k;
    stride = o.stride;
    cols = (int)(o.rows - col0 < COLS ? o.rows - col0 : COLS);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * THREADS + threadIdx.x, row = at / PIECES, c = (at % PIECES) ^ ((row & 3) << 2);
      off[i] = c * 8 < cols ? (int)((row * stride + c * 8) * 2) : kNowhere;
    }
  }
  template <class T>
  __device__ __forceinline__ void load(int k0, T* tile, bool) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const auto r = buffer(p + k0 * stride * 2, ((k - k0 - 1) * stride + cols) * 2);
#pragma unroll
    for (int i = 0; i < N; ++i) load_lds(r, tile + (i * THREADS + wave * 64) * 8, off[i], 0);
  }
};

// Reads of blocks of 32 rows (or columns) by 16 k as operands. BLOCKS of them,
// at rows first(0), first(1), .. of the tile.
template <bool ROWS, int WIDTH, int BLOCKS>
struct Read;
template <int WIDTH, int BLOCKS>
struct Read<true, WIDTH, BLOCKS> {
  uint32_t at[2];
  uint32_t row[BLOCKS];
  template <class F>
  __device__ __forceinline__ explicit Read(F first) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      at[ks] = (first(0) + (lane & 31)) * 64 + ((2 * ks + (lane >> 5)) ^ ((lane >> 2) & 3)) * 16;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) row[b] = (first(b) - first(0)) * 64;  // constants
  }
  template <class T>
  __device__ __forceinline__ s16x8 get(const T* tile, int b, int ks) const {
    typedef __attribute__((address_space(3))) const char* lds_ptr;
    const lds_ptr p = (lds_ptr)(__attribute__((address_space(3))) const void*)tile;
    return *(__attribute__((address_space(3))) const s16x8*)(p + at[ks] + row[b]);
  }
};
template <int WIDTH, int BLOCKS>
struct Read<false, WIDTH, BLOCKS> {
  uint32_t at[BLOCKS];
  template <class F>
  __device__ __forceinline__ explicit Read(F first) {
    const int lane = threadIdx.x & 63, i = lane & 15;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
      at[b] = ((lane >> 5) * 8 + (i >> 2)) * WIDTH * 2 + (((first(b) / 32) ^ (i >> 2)) * 4 + (lane & 16) / 8) * 16 + (i & 3) * 8;
  }
  // Sixteen lanes read four rows of sixteen columns and each gets one column.
  template <class T>
  __device__ __forceinline__ s16x8 get(const T* tile, int b, int ks) const {
    typedef __attribute__((address_space(3))) const char* lds_ptr;
    typedef __attribute__((address_space(3))) s16x4* tr_ptr;
    const lds_ptr p = (lds_ptr)(__attribute__((address_space(3))) const void*)tile;
    const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + at[b] + (16 * ks) * WIDTH * 2));
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + at[b] + (16 * ks + 4) * WIDTH * 2));
    return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Loads issued by this wavefront that may still be under way: at most n.
template <int n>
__device__ __forceinline__ void wait_loads() {
  static_assert(n < 64);
  __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | ((n >> 4) << 14));
}
// All wavefronts are here; nothing is waited for.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The tile of a workgroup. Wavefronts lie WM by WN over it; in n each takes a
// share of both halves of the tile, the same columns of each: a feed-forward
// tile holds gate columns in the one and up columns in the other.
template <class T_, int TM_, int TN_, int WM_, int WN_, bool ROWS_A, bool ROWS_B>
struct Tile {
  using T = T_;
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, THREADS = 64 * WM * WN;
  static constexpr int FM = TM / WM / 32, FN = TN / WN / 32;
  static_assert(FM >= 1 && FN >= 2 && FN % 2 == 0);
  using LoadA = std::conditional_t<ROWS_A, LoadRows<TM, THREADS>, LoadCols<TM, THREADS>>;
  using LoadB = std::conditional_t<ROWS_B, LoadRows<TN, THREADS>, LoadCols<TN, THREADS>>;
  static constexpr int kLoads = LoadA::N + LoadB::N;

  f32x16 acc[FM][FN];

  static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
  static __device__ __forceinline__ int row_of(int b) { return wave() / WN * (FM * 32) + 32 * b; }
  static __device__ __forceinline__ int col_of(int b) {
    return b / (FN / 2) * (TN / 2) + wave() % WN * (FN / 2 * 32) + b % (FN / 2) * 32;
  }

  // Order of a half step's instructions: its reads from LDS (of the next half
  // step's operands) and its loads one by one between the products.
  template <int LOADS>
  static __device__ __forceinline__ void interleave() {
    constexpr int kReads = FM * (ROWS_A ? 1 : 2) + FN * (ROWS_B ? 1 : 2), kProducts = FM * FN;
    constexpr int kEach = (kReads + LOADS + kProducts - 1) / kProducts;  // to a product
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int n = i * kEach + j;
        if (n < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        else if (n < kReads + LOADS) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // Adds the products of k = k_begin .. k_end - 1 (k_begin a multiple of 32).
  // load_b(k0, tile, whole) loads a tile of B. Four tiles deep: at the barrier
  // of a step the tiles of this one and the next have arrived, those of the
  // one after are under way, and the step before has left its buffers, which
  // the loads of the third go to.
  template <class LB>
  __device__ __forceinline__ void run(const LoadA& la, const LB& lb, int k_begin, int k_end) {
    __shared__ __align__(16) T a0[TM * kStep], a1[TM * kStep], a2[TM * kStep], a3[TM * kStep];
    __shared__ __align__(16) T b0[TN * kStep], b1[TN * kStep], b2[TN * kStep], b3[TN * kStep];
    const Read<ROWS_A, TM, FM> ra([](int b) { return row_of(b); });
    const Read<ROWS_B, TN, FN> rb([](int b) { return col_of(b); });
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    if (k_begin >= k_end) return;
    const int last = k_begin + ((k_end - k_begin - 1) / kStep) * kStep;  // k of the last tile
    auto load = [&](int k0, T* A, T* B) __attribute__((always_inline)) {
      // past the last tile the same one again, into a buffer that is read no
      // more: the count of loads under way stays the same
      const int k = k0 < last ? k0 : last;
      la.load(k, A, k + kStep <= k_end);
      lb.load(k, B, k + kStep <= k_end);
    };
    s16x8 fa[2][FM], fb[2][FN];
    auto read = [&](int to, const T* A, const T* B, int ks) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[to][i] = ra.get(A, i, ks);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[to][j] = rb.get(B, j, ks);
    };
    auto multiply = [&](int of) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma(fb[of][j], fa[of][i], acc[i][j], T{});
    };
    int k = k_begin;
    load(k, a0, b0);
    load(k + kStep, a1, b1);
    load(k + 2 * kStep, a2, b2);
    wait_loads<2 * kLoads>();
    meet();
    read(0, a0, b0, 0);
    auto step = [&](T* A, T* B, T* nextA, T* nextB, T* freeA, T* freeB) __attribute__((always_inline)) {
      wait_loads<kLoads>();
      meet();
      load(k + 3 * kStep, freeA, freeB);
      read(1, A, B, 1);
      multiply(0);
      interleave<kLoads>();
      read(0, nextA, nextB, 0);
      multiply(1);
      interleave<0>();
      k += kStep;
      return k <= last;
    };
    while (true) {
      if (!step(a0, b0, a1, b1, a3, b3)) break;
      if (!step(a1, b1, a2, b2, a0, b0)) break;
      if (!step(a2, b2, a3, b3, a1, b1)) break;
      if (!step(a3, b3, a0, b0, a2, b2)) break;
    }
    wait_loads<0>();  // none may write into LDS that another use has taken
    meet();
  }
};

// Tile (m, n) of this workgroup, of mt by nt. Workgroups go to the eight XCDs
// in turn; each XCD takes a consecutive part of the order, which runs through
// bands of kBand rows of tiles, so that tiles which share operands are in the
// same L2 at the same time.
constexpr int kBand = 8;
__device__ __forceinline__ void my_tile(int mt, int nt, int& m, int& n) {
  const int id = (int)xcd_item(blockIdx.x, (int64_t)mt * nt);
  const int band = id / (kBand * nt), in = id - band * (kBand * nt);
  const int high = mt - band * kBand < kBand ? mt - band * kBand : kBand;
  n = in / high;
  m = band * kBand + in - n * high;
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

// The gradients' products: B is one operand, or two one after the other along
// k (the second begins at k1, a multiple of kStep). The rows of A may be
// counted on the device (*n), or k (COUNT_K): then B is b1 where fewer are
// counted than there are, else b. Written in T, times f scale where f is there,
// or, by S parts, as 32-bit sums [S][rows][cols], added to what is there where
// `add` is set.
struct Grad {
  Operand a, b, b1;
  int64_t k1;
  const uint32_t* n;
  Rows rows;
  float* sums;
  int32_t mt, nt, S, add;
  const float* f;
  float scale;
};
__device__ __forceinline__ float factor_of(const Grad& g) { return g.f ? *g.f * g.scale : 1.0f; }

template <class TT, bool ROWS_A, bool TWO, bool COUNT_K>
__global__ __launch_bounds__(TT::THREADS) void grad_kernel(Grad g) {
  using T = typename TT::T;
  int m, n, begin, end;
  my_tile(g.mt, g.nt, m, n);
  const int64_t m0 = (int64_t)m * TT::TM, n0 = (int64_t)n * TT::TN;
  int64_t kept = g.rows.at1 + g.rows.n1;  // rows of the product
  if (g.n) {
    const int64_t count = __builtin_amdgcn_readfirstlane((int)*g.n);
    if (COUNT_K) {
      if (count < g.a.k) g.b = g.b1;
      g.a.k = g.b.k = count;
    } else {
      if (m0 >= count) return;
      g.a.rows = count;
    }
  }
  my_part(g.a.k, blockIdx.y, g.S, begin, end);
  TT t;
  const typename TT::LoadA la(g.a, m0);
  const typename TT::LoadB lb(g.b, n0), lb1(TWO ? g.b1 : g.b, n0);
  auto load_b = [&](int k0, T* tile, bool whole) __attribute__((always_inline)) {
    if (TWO && k0 >= g.k1) lb1.load(k0 - (int)g.k1, tile, whole);
    else lb.load(k0, tile, whole);
  };
  struct B {
    decltype(load_b)& f;
    __device__ __forceinline__ void load(int k0, T* tile, bool whole) const { f(k0, tile, whole); }
  };
  t.run(la, B{load_b}, begin, end);
  const int lane = threadIdx.x & 63;
  const int64_t cols = g.b.rows;
  const float f = factor_of(g);
#pragma unroll
  for (int i = 0; i < TT::FM; ++i) {
    const int64_t row = m0 + TT::row_of(i) + (lane & 31);
    T* out = row < g.a.rows ? row_at<T>(g.rows, row, cols) : nullptr;
    float* sum = row < g.a.rows && row < kept ? g.sums + ((int64_t)blockIdx.y * kept + row) * cols : nullptr;
#pragma unroll
    for (int j = 0; j < TT::FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int64_t c = n0 + TT::col_of(j) + 2 * e + 4 * (lane >> 5);
        if (c >= cols) continue;  // cols is a multiple of 8
        float4 v = make_float4(t.acc[i][j][e], t.acc[i][j][e + 1], t.acc[i][j][e + 2], t.acc[i][j][e + 3]);
        if (g.sums) {
          if (!sum) continue;
          if (g.add) {
            const float4 o = *(const float4*)(sum + c);
            v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
          }
          *(float4*)(sum + c) = v;
        } else if (out) {
          Vec<T, 4> o{{(T)(v.x * f), (T)(v.y * f), (T)(v.z * f), (T)(v.w * f)}};
          *(Vec<T, 4>*)(out + c) = o;
        }
      }
  }
}

// Adds the S parts' sums in their order, eight columns to a thread.
template <class T>
__global__ __launch_bounds__(256) void grad_join(Grad g, int64_t rows) {
  const int64_t cols = g.b.rows, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= rows * cols) return;
  const int64_t row = i / cols;
  T* out = row_at<T>(g.rows, row, cols);
  if (!out) return;
  const float f = factor_of(g);
  float v[8] = {};
  for (int s = 0; s < g.S; ++s) {
    const Vec<float, 8> a = load_vec<8>(g.sums + s * rows * cols + i);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += a.e[j];
  }
  Vec<T, 8> o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o.e[j] = (T)(v[j] * f);
  store_vec<8>(out + i - row * cols, o);
}

template <class T, bool ROWS_A, bool ROWS_B>
using Big = Tile<T, 256, 256, 2, 4, ROWS_A, ROWS_B>;
template <class T, bool ROWS_A, bool ROWS_B>
using Small = Tile<T, 128, 128, 2, 2, ROWS_A, ROWS_B>;

// Tiles of 256 x 256 need a CU's LDS each; of 128 x 128 two fit.
constexpr int kCus = 256;
inline bool is_big(int64_t rows, int64_t cols) { return ceil_div(rows, 256) * ceil_div(cols, 256) >= kCus * 3 / 4; }
inline int64_t tiles_of(int64_t rows, int64_t cols, bool big) {
  const int t = big ? 256 : 128;
  return ceil_div(rows, t) * ceil_div(cols, t);
}
// Parts of k where the tiles alone do not fill the chip: at least kPart of k in each.
constexpr int64_t kPart = 512;
inline int32_t parts_of(int64_t rows, int64_t cols, int64_t k) {
  if (rows <= 0 || is_big(rows, cols)) return 1;
  const int64_t want = 2 * kCus / tiles_of(rows, cols, false), most = k / kPart;
  const int64_t s = want < most ? want : most;
  return s < 1 ? 1 : s > 64 ? 64 : (int32_t)s;
}
inline size_t sums_bytes(int64_t rows, int64_t cols, int64_t k) {
  const int32_t s = parts_of(rows, cols, k);
  return s > 1 ? align256((size_t)s * (size_t)rows * (size_t)cols * 4) : 0;
}

// One gradient product of `rows` rows; S parts (1 and no sums: written in T at once).
template <class T, bool ROWS_A, bool TWO, bool COUNT_K>
hipError_t launch_grad(Grad g, int64_t rows, hipStream_t st) {
  auto go = [&](auto tile) {
    using TT = decltype(tile);
    g.mt = (int32_t)ceil_div(rows, TT::TM);
    g.nt = (int32_t)ceil_div(g.b.rows, TT::TN);
    hipLaunchKernelGGL((grad_kernel<TT, ROWS_A, TWO, COUNT_K>), dim3((unsigned)(g.mt * g.nt), (unsigned)g.S),
                       dim3(TT::THREADS), 0, st, g);
    return hipGetLastError();
  };
  if (rows <= 0 || g.b.rows <= 0) return hipSuccess;
  return is_big(rows, g.b.rows) ? go(Big<T, ROWS_A, false>{}) : go(Small<T, ROWS_A, false>{});
}
template <class T>
hipError_t launch_join(const Grad& g, int64_t rows, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(grad_join<T>, dim3((unsigned)ceil_div(rows * g.b.rows, 8 * 256)), dim3(256), 0, st, g, rows);
  return hipGetLastError();
}

}  // namespace product
}  // namespace argus
