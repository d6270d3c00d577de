// Top-k router with its balance loss, and the gradient of both.
//
// Sixteen lanes hold a token's logits, 16 bytes of each 256 to a lane (the
// row is read once, in whole lines), so a wavefront takes four tokens and
// every reduction over a token is four steps inside a row of lanes.
//   forward   top_k times the largest key; a key orders the logit's bits and
//             then the lower index, so ties need no further step. The first
//             is the softmax's maximum. Sums of the probabilities per expert
//             stay in registers over all tokens of a workgroup, counts in its
//             LDS; the workgroups' sums are written once and added in their
//             order by one workgroup, which makes the loss (in doubles).
//   backward  p = exp(x - lse); the gates' gradients are put into a zeroed
//             LDS row of the token, read back by the lanes that own the
//             experts, and cleared.
// Bound by memory backward (logits read, dlogits written) and by the selection's
// instructions forward.
#include <type_traits>

#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace argus {
namespace {

constexpr int kBlock = 1024;              // threads of a forward workgroup
constexpr int kTokens = kBlock / 16;      // tokens it takes at a time
constexpr int kMaxGrid = 256;             // one workgroup to a CU: few partial sums to add

template <typename T>
constexpr int kVec = 16 / sizeof(T);

// Key of a logit: ascending with its value, and among equal values with
// falling index. -0 and +0 are one value. 0 is below every key.
template <typename T>
struct Key {
  using U = uint32_t;  // 16-bit types: the value's bits above the index's
  static __device__ __forceinline__ U make(T v, int e) {
    const uint32_t b = __builtin_bit_cast(uint16_t, (float)v == 0.0f ? (T)0.0f : v);
    return ((b & 0x8000u ? b ^ 0xffffu : b | 0x8000u) << 16) | (uint32_t)(0xffff - e);
  }
  static __device__ __forceinline__ int index(U k) { return 0xffff - (int)(k & 0xffffu); }
};
template <>
struct Key<float> {
  using U = uint64_t;
  static __device__ __forceinline__ U make(float v, int e) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v == 0.0f ? 0.0f : v);
    return ((uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | (uint32_t)(0xffff - e);
  }
  static __device__ __forceinline__ int index(U k) { return 0xffff - (int)(k & 0xffffu); }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_key(uint32_t v) { return (uint32_t)dpp_i32<CTRL>((int)v); }
template <int CTRL>
__device__ __forceinline__ uint64_t dpp_key(uint64_t v) {
  return ((uint64_t)(uint32_t)dpp_i32<CTRL>((int)(v >> 32)) << 32) | (uint32_t)dpp_i32<CTRL>((int)v);
}
template <typename U>
__device__ __forceinline__ U max_of(U a, U b) { return a > b ? a : b; }
template <typename U>
__device__ __forceinline__ U row_max(U v) {
  v = max_of(v, dpp_key<kXor1>(v));
  v = max_of(v, dpp_key<kXor2>(v));
  v = max_of(v, dpp_key<kHalfMirror>(v));
  return max_of(v, dpp_key<kMirror>(v));
}

struct BalArgs {
  int64_t n, stride;
  int32_t E, K;
  float alpha;
  const void* logits;
  const uint8_t* mask;
  int32_t* expert;
  float* gate;
  float* lse;
  float* psum;     // [workgroups][E]
  uint32_t* cnt;   // [workgroups][E]
  uint32_t* valid; // [workgroups][2]: tokens taking part; 1 if a token was left out for its logits
};

template <typename T, int NI>
__global__ __launch_bounds__(kBlock) void bal_fwd(BalArgs a) {
  constexpr int V = kVec<T>, N = NI * V;
  using KT = Key<T>;
  using U = typename KT::U;
  __shared__ float ps[ARGUS_MAX_EXPERTS];
  __shared__ uint32_t cnt[ARGUS_MAX_EXPERTS];
  __shared__ uint32_t nv[2];
  const int tid = threadIdx.x, lane = tid & 15, E = a.E;
  for (int e = tid; e < E; e += kBlock) {
    ps[e] = 0;
    cnt[e] = 0;
  }
  if (tid < 2) nv[tid] = 0;
  __syncthreads();
  const T* logits = (const T*)a.logits;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * kTokens; t0 < a.n; t0 += (int64_t)gridDim.x * kTokens) {
    const int64_t t = t0 + (tid >> 4);
    const bool in = t < a.n && (!a.mask || a.mask[t]);
    float x[N];
    U key[N];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int at = (i * 16 + lane) * V;
      Vec<T, V> v = {};
      if (in) v = load_row<V>(logits + t * a.stride, at, E);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const bool here = in && at + j < E;
        x[i * V + j] = here ? to_f32(v.e[j]) : -__builtin_inff();
        nan |= here && v.e[j] != v.e[j];
        // a logit of -infinity is never chosen
        key[i * V + j] = x[i * V + j] > -__builtin_inff() ? KT::make(v.e[j], at + j) : 0;
      }
    }
    const float any_nan = row_sum(nan ? 1.0f : 0.0f);
    U best = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) best = max_of(best, key[i]);
    best = row_max(best);
    // the largest logit, from the lane that holds it
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    m = fmaxf(m, dpp_f32<kXor1>(m));
    m = fmaxf(m, dpp_f32<kXor2>(m));
    m = fmaxf(m, dpp_f32<kHalfMirror>(m));
    m = fmaxf(m, dpp_f32<kMirror>(m));
    const bool ok = in && any_nan == 0.0f && m > -__builtin_inff() && m < __builtin_inff();
    float p[N], z = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      p[i] = ok ? __expf(x[i] - m) : 0.0f;
      z += p[i];
    }
    z = row_sum(z);
    const float rz = ok ? 1.0f / z : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      p[i] *= rz;
      acc[i] += p[i];
    }
    int mine = -1;      // lane j keeps the j-th choice
    float mine_p = 0;
    for (int k = 0; k < a.K; ++k) {
      int e = ok && best ? KT::index(best) : -1;
      float g = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const bool hit = key[i] == best;
        g = hit ? p[i] : g;
        key[i] = hit ? 0 : key[i];
      }
      g = row_sum(best ? g : 0.0f);
      if (lane == k) {
        mine = e;
        mine_p = e >= 0 ? g : 0.0f;
      }
      U nb = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) nb = max_of(nb, key[i]);
      best = row_max(nb);
    }
    if (t < a.n) {
      if (lane < a.K) {
        a.expert[t * a.K + lane] = mine;
        a.gate[t * a.K + lane] = mine_p;
        if (mine >= 0) atomicAdd(&cnt[mine], 1u);
      }
      if (lane == 0) {
        a.lse[t] = ok ? m + __logf(z) : -__builtin_inff();
        if (ok) atomicAdd(&nv[0], 1u);
        if (in && !ok) nv[1] = 1;
      }
    }
  }
  // the four tokens of a wavefront, then the wavefronts in their order
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v = acc[i];
    auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
    auto u = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    acc[i] = __builtin_bit_cast(float, (uint32_t)u[0]) + __builtin_bit_cast(float, (uint32_t)u[1]);
  }
  for (int w = 0; w < kBlock / 64; ++w) {
    if (tid >> 6 == w && (tid & 63) < 16) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = (i / V * 16 + lane) * V + i % V;
        if (e < E) ps[e] += acc[i];
      }
    }
    __syncthreads();
  }
  for (int e = tid; e < E; e += kBlock) {
    a.psum[(int64_t)blockIdx.x * E + e] = ps[e];
    a.cnt[(int64_t)blockIdx.x * E + e] = cnt[e];
  }
  if (tid < 2) a.valid[blockIdx.x * 2 + tid] = nv[tid];
}

__global__ __launch_bounds__(1024) void bal_join(BalArgs a, int32_t blocks, argus_balance_out_t o) {
  __shared__ float ps[1024];
  __shared__ uint32_t cs[1024];
  __shared__ double part[1024];
  __shared__ uint32_t tot[2];
  const int tid = threadIdx.x, E = a.E;
  int ep = 1;
  while (ep < E) ep *= 2;
  const int groups = 1024 / ep, e = tid % ep, g = tid / ep;
  float s = 0;
  uint32_t c = 0;
  if (e < E) {
#pragma unroll 8
    for (int b = g; b < blocks; b += groups) {
      s += a.psum[(int64_t)b * E + e];
      c += a.cnt[(int64_t)b * E + e];
    }
  }
  ps[tid] = s;
  cs[tid] = c;
  if (tid < 2) tot[tid] = 0;
  __syncthreads();
  if (tid < blocks) {
    if (a.valid[tid * 2]) atomicAdd(&tot[0], a.valid[tid * 2]);
    if (a.valid[tid * 2 + 1]) tot[1] = 1;
  }
  __syncthreads();
  const uint32_t n = tot[0];
  double term = 0;
  if (g == 0 && e < E) {
    for (int i = 1; i < groups; ++i) {
      s += ps[i * ep + e];
      c += cs[i * ep + e];
    }
    o.count[e] = c;
    o.prob[e] = n ? (float)((double)s / n) : 0.0f;
    term = n ? (double)c * (double)s / n : 0.0;
  }
  part[tid] = term;
  __syncthreads();
  for (int h = 512; h > 0; h >>= 1) {
    if (tid < h) part[tid] += part[tid + h];
    __syncthreads();
  }
  if (tid == 0) {
    o.n_valid[0] = n;
    o.loss[0] = n ? (float)((double)a.alpha * E * part[0] / ((double)a.K * n)) : 0.0f;
    if (o.dev_status) *o.dev_status = tot[1] ? (int32_t)ARGUS_DEV_LOGITS : 0;
  }
}

struct BalBwdArgs {
  int64_t n, stride;
  int32_t E, K;
  float alpha;
  const void* logits;
  const float* lse;
  const int32_t* expert;
  const uint32_t* count;
  const uint32_t* n_valid;
  const float* dloss;
  const float* dgate;
  void* dlogits;
};

template <typename T, int NI>
__global__ __launch_bounds__(256) void bal_bwd(BalBwdArgs a) {
  constexpr int V = kVec<T>, N = NI * V;
  __shared__ __align__(16) float rows[16][NI * 16 * V];
  const int tid = threadIdx.x, lane = tid & 15, E = a.E;
  float* row = rows[tid >> 4];
  float c[N];
  const float n = (float)a.n_valid[0];
  const float coef = n > 0 ? a.dloss[0] * a.alpha * (float)E / ((float)a.K * n) / n : 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = (i / V * 16 + lane) * V + i % V;
    c[i] = e < E ? coef * (float)a.count[e] : 0.0f;
    row[e] = 0;
  }
  const T* logits = (const T*)a.logits;
  T* out = (T*)a.dlogits;
  for (int64_t t = (int64_t)blockIdx.x * 16 + (tid >> 4); t < a.n; t += (int64_t)gridDim.x * 16) {
    const float l = a.lse[t];
    const bool ok = l > -__builtin_inff();
    Vec<T, V> v[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = load_row<V>(logits + t * a.stride, (i * 16 + lane) * V, E);
    int e = -1;
    if (a.dgate && lane < a.K) {
      e = a.expert[t * a.K + lane];
      if (e >= 0 && e < E) atomicAdd(&row[e], a.dgate[t * a.K + lane]);
      else e = -1;
    }
    // the token's row is this wavefront's own: LDS keeps its order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    float p[N], g[N], s = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int k = i * V + j, at = (i * 16 + lane) * V + j;
        p[k] = ok && at < E ? __expf(to_f32(v[i].e[j]) - l) : 0.0f;
        g[k] = c[k] + row[at];
        s += g[k] * p[k];
      }
    s = row_sum(s);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    if (e >= 0) row[e] = 0;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      Vec<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.e[j] = from_f32<T>(p[i * V + j] * (g[i * V + j] - s));
      store_row<V>(out + t * E, (i * 16 + lane) * V, E, o);
    }
  }
}

// Calls fn with the number of 256-byte pieces of a row, as a constant: the
// next of 1, 2, 3, 4, 6, 8, 12, 16.
template <typename T, typename F>
hipError_t with_pieces(int32_t E, F fn) {
  const int64_t n = ceil_div(E, 16 * kVec<T>);
  if (n <= 1) return fn(std::integral_constant<int, 1>{});
  if (n <= 2) return fn(std::integral_constant<int, 2>{});
  if (n <= 3) return fn(std::integral_constant<int, 3>{});
  if (n <= 4) return fn(std::integral_constant<int, 4>{});
  if (n <= 6) return fn(std::integral_constant<int, 6>{});
  if constexpr (sizeof(T) == 2) {
    return fn(std::integral_constant<int, 8>{});
  } else {
    if (n <= 8) return fn(std::integral_constant<int, 8>{});
    if (n <= 12) return fn(std::integral_constant<int, 12>{});
    return fn(std::integral_constant<int, 16>{});
  }
}

int64_t bal_grid(const argus_balance_t& p) {
  const int64_t need = ceil_div(p.n_tokens, kTokens);
  return need < 1 ? 1 : need < kMaxGrid ? need : kMaxGrid;
}

}  // namespace

size_t balance_workspace_bytes(const argus_balance_t& p) {
  const size_t g = (size_t)bal_grid(p);
  return 2 * align256(g * (size_t)p.n_experts * 4) + align256(g * 8);
}

hipError_t launch_balance(const argus_balance_t& p, const void* logits, const uint8_t* mask,
                          const argus_balance_out_t& o, void* ws, hipStream_t st) {
  const int64_t grid = bal_grid(p);
  const size_t part = align256((size_t)grid * (size_t)p.n_experts * 4);
  uint8_t* base = (uint8_t*)ws;
  BalArgs a{p.n_tokens, p.row_stride, p.n_experts, p.top_k, p.alpha, logits, mask, o.expert, o.gate, o.lse,
            (float*)base, (uint32_t*)(base + part), (uint32_t*)(base + 2 * part)};
  const hipError_t e = with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    return with_pieces<T>(p.n_experts, [&](auto ni) {
      hipLaunchKernelGGL((bal_fwd<T, decltype(ni)::value>), dim3((unsigned)grid), dim3(kBlock), 0, st, a);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(bal_join, dim3(1), dim3(1024), 0, st, a, (int32_t)grid, o);
  return hipGetLastError();
}

hipError_t launch_balance_bwd(const argus_balance_t& p, const void* logits, const float* lse, const int32_t* expert,
                              const uint32_t* count, const uint32_t* n_valid, const float* dloss, const float* dgate,
                              void* dlogits, hipStream_t st) {
  if (p.n_tokens == 0) return hipSuccess;
  BalBwdArgs a{p.n_tokens, p.row_stride, p.n_experts, p.top_k, p.alpha, logits, lse, expert, count, n_valid, dloss,
               dgate, dlogits};
  const int64_t need = ceil_div(p.n_tokens, 16), grid = need < 2048 ? need : 2048;
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    return with_pieces<T>(p.n_experts, [&](auto ni) {
      hipLaunchKernelGGL((bal_bwd<T, decltype(ni)::value>), dim3((unsigned)grid), dim3(256), 0, st, a);
      return hipGetLastError();
    });
  });
}

}  // namespace argus
