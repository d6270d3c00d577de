// Tiles of the attention kernels: documents, rows in LDS, matrix operands.
//
// All products are v_mfma_f32_32x32x16_bf16. Its lanes are 32 columns in two
// halves h = lane / 32; with column c = lane % 32 and j = 0 .. 7,
//   A holds A[row c][k = 8 h + j], B holds B[k = 8 h + j][column c], and of
//   the result a lane holds rows 8 (i / 4) + 4 h + i % 4, i = 0 .. 15, of
//   column c.
// A result whose rows are the next product's k needs no exchange between
// lanes: registers 8 t .. 8 t + 7 are taken as the B operand of k-step t, and
// the A operand is read with the same order of k, which is rows
// 16 t + 4 h + (0 .. 3) and 16 t + 8 + 4 h + (0 .. 3). A row-major tile gives
// such an operand, transposed, by two ds_read_b64_tr_b16.
#pragma once

#include "ops_internal.h"

namespace argus {
namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Documents and the workspace's flag (1: the offsets are malformed).
struct Docs {
  const int64_t *q_off, *k_off;
  int32_t n_docs;
  int64_t n_q, n_k;
  const uint32_t* bad;
};
struct Doc {
  int64_t q0, k0;
  int32_t nq, nk;
};

__device__ __forceinline__ Doc doc_at(const Docs& d, int i) {
  if (!d.q_off) return {0, 0, (int32_t)d.n_q, (int32_t)d.n_k};
  const int64_t q0 = d.q_off[i], k0 = d.k_off[i];
  return {q0, k0, (int32_t)(d.q_off[i + 1] - q0), (int32_t)(d.k_off[i + 1] - k0)};
}

// Workgroups own tiles of kTile rows of a document, queries or keys. The
// plan lists them, those of long documents first (they would otherwise begin
// when the others end); entries past the last tile have the document -1.
// ceil((b - a) / kTile) <= b / kTile - a / kTile + 1, so tokens / kTile + 1 for
// each document is enough.
constexpr int kTile = 128;
struct Plan {
  const int2* tile;  // document, first row in it
  int32_t n;         // entries, at least as many as tiles
};
inline int64_t plan_entries(int64_t tokens, int32_t n_docs) { return tokens / kTile + n_docs; }

// Tile and head of this workgroup. Heads that divide evenly over the eight
// XCDs (workgroups go to them in turn) stay on one each, neighbours together,
// so that an XCD's L2 holds the keys and values of few heads.
__device__ __forceinline__ bool my_tile(const Plan& plan, int heads, int& head, int& doc, int& row0) {
  const int b = blockIdx.x;
  int nth;
  if (heads % 8 == 0) {
    const int per = heads / 8;
    nth = (b >> 3) / per;
    head = (b & 7) * per + (b >> 3) % per;
  } else {
    nth = b / heads;
    head = b % heads;
  }
  const int2 t = plan.tile[nth];
  doc = __builtin_amdgcn_readfirstlane(t.x);
  row0 = __builtin_amdgcn_readfirstlane(t.y);
  return doc >= 0;
}

// Rows [0, n) of a document's tile as a buffer: what lies past the last row
// reads as zeros. `stride` in elements.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const __bf16* first, int64_t n, int64_t stride, int dim) {
  int64_t bytes = n > 0 ? ((n - 1) * stride + dim) * 2 : 0;
  if (bytes > 0x7ffffff0) bytes = 0x7ffffff0;  // tiles past that have a base of their own
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<__bf16*>(first), (short)0, (int)bytes, 0x00020000);
}

// Place of 16-byte piece c of row r of a tile of DP elements a row: pieces are
// exchanged within a row so that in neither kind of read two lanes of one
// cycle (16 lanes of 16 bytes, 32 of 8: 64 banks) meet in a bank. Rows' reads
// take one piece of 16 rows; the transposed ones four neighbouring pieces of
// four rows. 64-element rows lie two to the banks' width.
template <int DP>
__device__ __forceinline__ int swz(int r, int c) {
  if constexpr (DP == 128) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
  else return c ^ (((r & 2) << 1) | ((r >> 2) & 3));
}

// Loads of a tile of ROWS rows straight into LDS, 16 bytes a lane. A
// wavefront's lanes write consecutive places, so the exchange of pieces is
// made on the global side: the lane of place c reads piece swz(row, c).
template <int DP, int ROWS, int THREADS>
struct TileLoad {
  static constexpr int PIECES = DP / 8;
  static constexpr int N = ROWS * PIECES / THREADS;
  static_assert(ROWS * PIECES % THREADS == 0);
  int off[N];  // bytes from the tile's first row
  __device__ __forceinline__ TileLoad(int64_t stride, int dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * THREADS + threadIdx.x, row = at / PIECES, c = swz<DP>(row, at % PIECES);
      // pieces past the head dimension read as zeros like rows past the end
      off[i] = c * 8 < dim ? (int)((row * stride + c * 8) * 2) : 0x7ffffff0;
    }
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, __bf16* tile) const {
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass has no 16-byte form and drops kernels that name it
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < N; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          r, (__attribute__((address_space(3))) void*)(tile + (i * THREADS + wave * 64) * 8), 16, off[i], 0, 0, 0);
#endif
  }
};

// 4 bytes a lane into consecutive words.
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, float* words, int off) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)words, 4, off, 0, 0, 0);
#endif
}

// All of this wavefront's loads have arrived.
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Reads of tiles of DP elements a row. A few byte offsets of the lane serve
// every tile: what else moves an operand is a constant, which the
// instructions hold.
template <int DP>
struct Reader {
  static constexpr int KS = DP / 16, DT = DP / 32;
  typedef __attribute__((address_space(3))) const char* lds_ptr;
  typedef __attribute__((address_space(3))) s16x4* tr_ptr;
  uint32_t row[KS], col[DT][2];
  __device__ __forceinline__ Reader() {
    const int lane = threadIdx.x & 63, r = lane & 31, i = lane & 15, c = (lane & 16) + 4 * (i & 3);
    const int rc = 4 * (lane >> 5) + (i >> 2);
#pragma unroll
    for (int j = 0; j < KS; ++j) row[j] = (r * DP + swz<DP>(r, 2 * j + (lane >> 5)) * 8) * 2;
#pragma unroll
    for (int j = 0; j < DT; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        col[j][u] = ((rc + 8 * u) * DP + swz<DP>(rc + 8 * u, (c >> 3) + 4 * j) * 8 + (c & 7)) * 2;
  }
  // Keeps the sums of offsets and constants out of registers: called once a
  // step, it hides that they are the same ones.
  __device__ __forceinline__ void fresh() {
#pragma unroll
    for (int j = 0; j < KS; ++j) asm volatile("" : "+v"(row[j]));
#pragma unroll
    for (int j = 0; j < DT; ++j) asm volatile("" : "+v"(col[j][0]), "+v"(col[j][1]));
  }
  // A (or B) operand: rows r0 + lane % 32, k = 16 ks + 8 h + j; r0 a multiple of 32.
  __device__ __forceinline__ bf16x8 rows(const __bf16* tile, int r0, int ks, uint32_t more = 0) const {
    const lds_ptr p = (lds_ptr)(__attribute__((address_space(3))) const void*)tile;
    return *(__attribute__((address_space(3))) const bf16x8*)(p + (row[ks] + more) + r0 * DP * 2);
  }
  // A operand, transposed: row index of A = column c0 + lane % 32 of the tile,
  // k = rows r0 + 4 h + (0 .. 3) and r0 + 8 + 4 h + (0 .. 3); r0 a multiple of
  // 16, c0 of 32. Sixteen lanes read four rows of sixteen columns and each
  // gets one column.
  __device__ __forceinline__ bf16x8 cols(const __bf16* tile, int r0, int c0) const {
    const lds_ptr p = (lds_ptr)(__attribute__((address_space(3))) const void*)tile;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + col[c0 / 32][0] + r0 * DP * 2));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + col[c0 / 32][1] + r0 * DP * 2));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Registers 8 t .. 8 t + 7 of a result, rounded to bfloat16, as a B operand.
__device__ __forceinline__ bf16x8 as_operand(const f32x16& x, int t) {
  bf16x8 r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = (__bf16)x[8 * t + j];
  return r;
}

// A row's operand in registers: row of the buffer, k as in an operand.
template <int DP>
__device__ __forceinline__ void load_operand(bf16x8 (&f)[DP / 16], __amdgpu_buffer_rsrc_t r, int row, int64_t stride,
                                             int dim) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const int c = 16 * ks + 8 * half;
    const int off = c < dim ? (int)(((int64_t)row * stride + c) * 2) : 0x7ffffff0;
    f[ks] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
  }
}

template <int DP>
__device__ __forceinline__ void clear(f32x16 (&x)[DP / 32]) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[d][i] = 0;
}

// Writes a transposed accumulator, times f: lane = row, registers = columns.
template <int DP>
__device__ __forceinline__ void write_rows(__bf16* row, const f32x16 (&x)[DP / 32], float f, int dim) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int at = 32 * d + 2 * i + 4 * half;
      bf16x4 o4;
#pragma unroll
      for (int j = 0; j < 4; ++j) o4[j] = (__bf16)(x[d][i + j] * f);
      if (at < dim) *(bf16x4*)(row + at) = o4;
    }
}

__device__ __forceinline__ float other_half(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __builtin_bit_cast(float, (uint32_t)((threadIdx.x & 32) ? s[0] : s[1]));
}

// Scale of the scores in units of log2. Not 0, so that a masked score, which
// is -infinity, stays that.
__device__ __forceinline__ float score_scale(float scale) { return fmaxf(scale * kLog2e, 0x1p-100f); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace attn
}  // namespace argus
