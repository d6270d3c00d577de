// Shared by the step operators' kernels (embedding, layer norm, balance,
// attention): element types, unaligned vectors, lane reductions, and the
// launch-side entry points. See include/argus_ops.h for the contract.
#pragma once

#include "../../include/argus_ops.h"
#include "argus_internal.h"

namespace argus {

using bf16_t = __bf16;
using f16_t = _Float16;

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_f32(float v) { return (T)v; }  // round to nearest even

// N elements that are aligned like one: rows of any stride and width are read
// and written with the widest instructions, which need no more than that
// alignment for global memory.
template <typename T, int N>
struct Vec {
  T e[N];
};
template <int N, typename T>
__device__ __forceinline__ Vec<T, N> load_vec(const T* p) {
  Vec<T, N> v;
  __builtin_memcpy(&v, p, sizeof(v));
  return v;
}
template <int N, typename T>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, N>& v) {
  __builtin_memcpy(p, &v, sizeof(v));
}

// Past the caches: for large outputs that are written once and not read here.
template <int N, typename T>
__device__ __forceinline__ void stream_vec(T* p, const Vec<T, N>& v) {
  if constexpr (sizeof(v) == 16) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p);
  } else {
    store_vec<N>(p, v);
  }
}

// Elements [i, i + N) of a row of n: whole vectors, and the elements that
// exist of the one across the row's end (the others are 0).
template <int N, typename T>
__device__ __forceinline__ Vec<T, N> load_row(const T* row, int i, int n) {
  if (i + N <= n) return load_vec<N>(row + i);
  Vec<T, N> v;
#pragma unroll
  for (int j = 0; j < N; ++j) v.e[j] = i + j < n ? row[i + j] : (T)0.0f;
  return v;
}
template <int N, typename T>
__device__ __forceinline__ void store_row(T* row, int i, int n, const Vec<T, N>& v) {
  if (i + N <= n) {
    store_vec<N>(row + i, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (i + j < n) row[i + j] = v.e[j];
}

template <int N, typename T>
__device__ __forceinline__ void stream_row(T* row, int i, int n, const Vec<T, N>& v) {
  if (i + N <= n) stream_vec<N>(row + i, v);
  else store_row<N>(row, i, n, v);
}

template <int CTRL>
__device__ __forceinline__ int dpp_i32(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
  return __builtin_bit_cast(float, dpp_i32<CTRL>(__builtin_bit_cast(int, v)));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

// Sum over the 16 lanes of a row, in every lane. Each step adds the value of
// the mirrored lane; the lanes of one half already agree, so a mirror serves
// as an exchange.
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f32<kXor1>(v);
  v += dpp_f32<kXor2>(v);
  v += dpp_f32<kHalfMirror>(v);
  v += dpp_f32<kMirror>(v);
  return v;
}
// Sum over the four rows of a wavefront, lane by lane, in every row.
__device__ __forceinline__ float rows_sum(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}
__device__ __forceinline__ float wave_sum_f32(float v) { return rows_sum(row_sum(v)); }

// Host side: calls fn with a value of the element type.
template <typename F>
hipError_t with_dtype(int32_t dtype, F fn) {
  switch (dtype) {
    case ARGUS_BF16: return fn(bf16_t{});
    case ARGUS_F16: return fn(f16_t{});
    default: return fn(float{});
  }
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

hipError_t launch_embedding(const argus_embedding_t& p, const void* table, void* out, hipStream_t st);
size_t embedding_bwd_workspace_bytes(const argus_embedding_t& p);
hipError_t launch_embedding_bwd(const argus_embedding_t& p, const void* dout, void* dtable, void* ws, hipStream_t st);

hipError_t launch_layer_norm(const argus_layer_norm_t& p, const void* x, const void* w, const void* b, void* y,
                             float* mean, float* rstd, hipStream_t st);
size_t layer_norm_bwd_workspace_bytes(const argus_layer_norm_t& p);
hipError_t launch_layer_norm_bwd(const argus_layer_norm_t& p, const void* dy, const void* x, const float* mean,
                                 const float* rstd, const void* w, void* dx, void* dw, void* db, void* ws,
                                 hipStream_t st);

size_t balance_workspace_bytes(const argus_balance_t& p);
hipError_t launch_balance(const argus_balance_t& p, const void* logits, const uint8_t* mask,
                          const argus_balance_out_t& o, void* ws, hipStream_t st);
hipError_t launch_balance_bwd(const argus_balance_t& p, const void* logits, const float* lse, const int32_t* expert,
                              const uint32_t* count, const uint32_t* n_valid, const float* dloss, const float* dgate,
                              void* dlogits, hipStream_t st);

size_t attention_workspace_bytes(const argus_attention_t& p);
hipError_t launch_attention(const argus_attention_t& p, const void* q, const void* k, const void* v, void* o,
                            float* lse, void* ws, hipStream_t st);
size_t attention_bwd_workspace_bytes(const argus_attention_t& p);
hipError_t launch_attention_bwd(const argus_attention_t& p, const void* d_o, const void* q, const void* k,
                                const void* v, const void* o, const float* lse, void* dq, void* dk, void* dv,
                                void* ws, hipStream_t st);

}  // namespace argus
