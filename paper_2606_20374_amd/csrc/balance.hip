// Top-k router with its balance loss, and the gradient of both.
//
// Sixteen lanes hold a token's logits, 16 bytes of each 256 to a lane (the
// row is read once, in whole lines), so a wavefront takes four tokens and
// every reduction over a token is four steps inside a row of lanes.
//   forward   a key orders a logit's value and then the lower index, so ties
//             need no further step. Each lane sorts its own keys, as many as
//             can be chosen, in registers (comparators of one maximum and one
//             minimum); then top_k times the largest of the sixteen heads is
//             taken and its lane moves up. The first is the softmax's
//             maximum. Sums of the probabilities per expert stay in registers
//             over all tokens of a workgroup, counts in its LDS; the
//             workgroups' sums are written once and added in their order by
//             a second launch, whose last workgroup makes the loss (in
//             doubles).
//   backward  p = exp(x - lse); the gates' gradients are put into a zeroed
//             LDS row of the token, read back by the lanes that own the
//             experts, and cleared.
// Backward is bound by memory (logits read, dlogits written): 262,144 tokens
// of 128 bf16 logits, top 8: 31 to 34 us, 30 at a large copy's 5.0 TB/s. Forward is
// bound by the selection's instructions: 131,072 tokens of 256 32-bit logits,
// top 8: 86 us, 29 at the copy's rate; the vector units are busy 77% of the
// cycles, 1,011 instructions to four tokens (counters).
#include <type_traits>

#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace argus {
namespace {

constexpr int kMaxGrid = 256;  // forward workgroups, one to a CU: few sums to add

template <typename T>
constexpr int kVec = 16 / sizeof(T);

// Key of a logit: ascending with its value, and among equal values with
// falling index; -0 and +0 are one value, and the keys of -infinity and of
// what is no logit are `none`, below all others. Keys of 16-bit types are
// 32-bit integers: the 32-bit float's bits, made ascending, of which the low
// ten are free for the index (1,024 experts at most). Those of 32-bit floats
// are doubles: the value leaves 29 bits of the mantissa free, and the minimum
// and maximum of doubles are single instructions.
constexpr uint32_t kIdx = ARGUS_MAX_EXPERTS - 1;
static_assert((ARGUS_MAX_EXPERTS & kIdx) == 0 && kIdx < (1u << 13), "an index fits below a half's 19 bits");

template <typename T>
struct Key {
  using U = uint32_t;
  static constexpr U kNone = 0;
  static __device__ __forceinline__ U make(float f, int e) {
    const uint32_t b = __builtin_bit_cast(uint32_t, f + 0.0f);  // -0 becomes +0
    const uint32_t up = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (up & ~kIdx) | (kIdx - (uint32_t)e);
  }
  static __device__ __forceinline__ bool none(U k) { return k < 0x00800000u; }  // -infinity's 0x007fffff and below
  static __device__ __forceinline__ int index(U k) { return (int)(kIdx - (k & kIdx)); }
  static __device__ __forceinline__ float value(U k) {
    return __builtin_bit_cast(float, (k & 0x80000000u ? k ^ 0x80000000u : ~k) & ~kIdx);
  }
  static __device__ __forceinline__ U largest(U a, U b) { return a > b ? a : b; }
  static __device__ __forceinline__ U smallest(U a, U b) { return a < b ? a : b; }
  template <int CTRL>
  static __device__ __forceinline__ U dpp(U v) { return (U)dpp_i32<CTRL>((int)v); }
};
template <>
struct Key<float> {
  using U = double;
  static constexpr U kNone = -1e300;
  static __device__ __forceinline__ U make(float f, int e) {
    // also a NaN becomes kNone
    const uint64_t b = __builtin_bit_cast(uint64_t, __builtin_fmax((double)(f + 0.0f), kNone));
    // a larger mantissa is a larger value above zero and a smaller one below
    const uint32_t low = (uint32_t)e ^ (~(uint32_t)((int64_t)b >> 63) & kIdx);
    return __builtin_bit_cast(double, b ^ low);  // kNone keeps its place below every value
  }
  static __device__ __forceinline__ bool none(U k) { return k < -1e200; }
  static __device__ __forceinline__ int index(U k) {
    const uint32_t b = (uint32_t)__builtin_bit_cast(uint64_t, k) & kIdx;
    return (int)(k < 0 ? b : kIdx - b);
  }
  static __device__ __forceinline__ float value(U k) {
    return (float)__builtin_bit_cast(double, __builtin_bit_cast(uint64_t, k) & ~(uint64_t)kIdx);
  }
  // fmax and fmin would first make each operand canonical, for NaNs; the only
  // keys that are one are +infinity's, whose token is left out by its sum
  static __device__ __forceinline__ U largest(U a, U b) {
    U r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
  }
  static __device__ __forceinline__ U smallest(U a, U b) {
    U r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
  }
  template <int CTRL>
  static __device__ __forceinline__ U dpp(U v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, ((uint64_t)(uint32_t)dpp_i32<CTRL>((int)(b >> 32)) << 32) | (uint32_t)dpp_i32<CTRL>((int)b));
  }
};

// exp(x - m); the difference is taken first, which gives no NaN for finite logits
// (the lowest values of a type among them). Its product with log2(e) is
// rounded, which puts the value off by |x - m| 2^-24 of itself: 2^-20 at a
// distance of 16, where a probability is below 2e-7. An exact product would be
// two more instructions for each logit of a kernel that instructions bound.
__device__ __forceinline__ float exp_from(float x, float m) {
  return __builtin_amdgcn_exp2f((x - m) * 1.4426950408889634f);
}

// NI vectors of a row of E elements, of each 16 V one to a lane; what lies
// past the row is `pad`.
template <int NI, typename T, int V = kVec<T>>
__device__ __forceinline__ void load_logits(Vec<T, V> (&v)[NI], const T* row, bool in, int E, T pad) {
  const int lane = threadIdx.x & 15;
  const bool whole = E % V == 0;  // no vector lies across the row's end
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int at = (i * 16 + lane) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) v[i].e[j] = pad;
    if (whole) {
      if (in && at < E) v[i] = load_vec<V>(row + at);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (in && at + j < E) v[i].e[j] = row[at + j];
    }
  }
}

template <typename K, typename U>
__device__ __forceinline__ U row_max(U v) {
  v = K::largest(v, K::template dpp<kXor1>(v));
  v = K::largest(v, K::template dpp<kXor2>(v));
  v = K::largest(v, K::template dpp<kHalfMirror>(v));
  return K::largest(v, K::template dpp<kMirror>(v));
}

// Sorts M keys, a power of two, descending (odd-even merges).
template <typename K, int M, typename U>
__device__ __forceinline__ void sort_keys(U (&k)[M]) {
#pragma unroll
  for (int p = 1; p < M; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < M; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < M && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const U a = k[i + j], b = k[i + j + q];
            k[i + j] = K::largest(a, b);
            k[i + j + q] = K::smallest(a, b);
          }
}

// The M largest of two descending lists of M, descending, into `a`.
template <typename K, int M, typename U>
__device__ __forceinline__ void merge_keys(U (&a)[M], const U (&b)[M]) {
#pragma unroll
  for (int i = 0; i < M; ++i) a[i] = K::largest(a[i], b[M - 1 - i]);
#pragma unroll
  for (int q = M / 2; q >= 1; q /= 2)
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (!(i & q)) {
        const U x = a[i], y = a[i + q];
        a[i] = K::largest(x, y);
        a[i + q] = K::smallest(x, y);
      }
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
  double* terms;   // [joining workgroups] the loss's
  uint32_t* ticket;
};

// Most threads of a forward workgroup: fewer where a lane holds more logits.
constexpr int fwd_block(int n) { return n <= 16 ? 1024 : n <= 32 ? 512 : 256; }

// KC: 8 or 16, not below top_k.
template <typename T, int NI, int KC>
__global__ __launch_bounds__(fwd_block(NI * kVec<T>)) void bal_fwd(BalArgs a) {
  constexpr int V = kVec<T>, N = NI * V;
  using KT = Key<T>;
  using U = typename KT::U;
  __shared__ float ps[ARGUS_MAX_EXPERTS];
  __shared__ uint32_t cnt[ARGUS_MAX_EXPERTS];
  __shared__ uint32_t nv[2];
  const int tid = threadIdx.x, lane = tid & 15, E = a.E, block = blockDim.x, tokens = block / 16;
  for (int e = tid; e < E; e += block) {
    ps[e] = 0;
    cnt[e] = 0;
  }
  if (tid < 2) nv[tid] = 0;
  if (blockIdx.x == 0 && tid == 0) *a.ticket = 0;
  __syncthreads();
  const T* logits = (const T*)a.logits;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0;
  const int64_t step = (int64_t)gridDim.x * tokens;
  int64_t t = (int64_t)blockIdx.x * tokens + (tid >> 4);
  Vec<T, V> v[NI];
  bool in = false;
  auto fetch = [&](int64_t at) {
    in = at < a.n && (!a.mask || a.mask[at]);
    load_logits(v, logits + at * a.stride, in, E, (T)-__builtin_inff());
  };
  fetch(t);
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < a.n; t0 += step, t += step) {
    const bool here = in;
    float x[N];
    U best[KC];  // the lane's largest keys, descending
#pragma unroll
    for (int c = 0; c < N; c += KC) {
      U k[KC];
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        k[j] = KT::kNone;
        if (c + j < N) {
          x[c + j] = to_f32(v[(c + j) / V].e[(c + j) % V]);
          k[j] = KT::make(x[c + j], ((c + j) / V * 16 + lane) * V + (c + j) % V);
        }
      }
      sort_keys<KT>(k);
      if (c == 0) {
#pragma unroll
        for (int j = 0; j < KC; ++j) best[j] = k[j];
      } else {
        merge_keys<KT>(best, k);
      }
    }
    fetch(t + step);
    U top = row_max<KT>(best[0]);
    // the largest logit; with a NaN or an infinity among them z is NaN below
    const float m = KT::value(top);
    float z = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = exp_from(x[i], m);
      z += x[i];
    }
    z = row_sum(z);
    const bool ok = here && !KT::none(top) && z < __builtin_inff();  // and no NaN
    const float rz = 1.0f / z;
    if (__ballot(!ok)) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = ok ? x[i] : 0.0f;
    }
    const float w = ok ? rz : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] += x[i] * w;
    U mine = KT::kNone;  // lane j keeps the j-th choice
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      if (k < a.K) {
        if (lane == k) mine = top;
        if (k + 1 < KC) {
          const bool won = best[0] == top;
#pragma unroll
          for (int j = 0; j + 1 < KC - k; ++j) best[j] = won ? best[j + 1] : best[j];
          top = row_max<KT>(best[0]);
        }
      }
    }
    if (t < a.n) {
      if (lane < a.K) {
        const bool chosen = ok && !KT::none(mine);
        const int e = chosen ? KT::index(mine) : -1;
        a.expert[t * a.K + lane] = e;
        a.gate[t * a.K + lane] = chosen ? exp_from(KT::value(mine), m) * rz : 0.0f;
        if (chosen) atomicAdd(&cnt[e], 1u);
      }
      if (lane == 0) {
        a.lse[t] = ok ? m + __logf(z) : -__builtin_inff();
        if (ok) atomicAdd(&nv[0], 1u);
        if (here && !ok) nv[1] = 1;
      }
    }
  }
  // the four tokens of a wavefront, then the wavefronts in their order
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = rows_sum(acc[i]);
  for (int w = 0; w < block / 64; ++w) {
    if (tid >> 6 == w && (tid & 63) < 16) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = (i / V * 16 + lane) * V + i % V;
        if (e < E) ps[e] += acc[i];
      }
    }
    __syncthreads();
  }
  for (int e = tid; e < E; e += block) {
    a.psum[(int64_t)blockIdx.x * E + e] = ps[e];
    a.cnt[(int64_t)blockIdx.x * E + e] = cnt[e];
  }
  if (tid < 2) a.valid[blockIdx.x * 2 + tid] = nv[tid];
}

constexpr int kJoin = 32;  // experts of a joining workgroup

// Adds the workgroups' sums in their order, 32 runs of them side by side and
// then the runs; the last workgroup to end adds the loss's terms.
__global__ __launch_bounds__(1024) void bal_join(BalArgs a, int32_t blocks, argus_balance_out_t o) {
  __shared__ float ps[32][kJoin];
  __shared__ uint32_t cs[32][kJoin];
  __shared__ uint32_t tot[2];
  __shared__ bool last;
  const int tid = threadIdx.x, E = a.E, c = tid % kJoin, g = tid / kJoin, e = blockIdx.x * kJoin + c;
  if (tid < 2) tot[tid] = 0;
  float s = 0;
  uint32_t n_of = 0;
  if (e < E) {
#pragma unroll 8
    for (int b = g; b < blocks; b += 32) {
      s += a.psum[(int64_t)b * E + e];
      n_of += a.cnt[(int64_t)b * E + e];
    }
  }
  ps[g][c] = s;
  cs[g][c] = n_of;
  __syncthreads();
  if (tid < blocks) {
    if (a.valid[tid * 2]) atomicAdd(&tot[0], a.valid[tid * 2]);
    if (a.valid[tid * 2 + 1]) tot[1] = 1;
  }
  __syncthreads();
  const uint32_t n = tot[0];
  if (tid < 64) {
    double term = 0;
    if (tid < kJoin && e < E) {
      float sum = 0;
      uint32_t cnt = 0;
      for (int i = 0; i < 32; ++i) {
        sum += ps[i][tid];
        cnt += cs[i][tid];
      }
      o.count[e] = cnt;
      o.prob[e] = n ? (float)((double)sum / n) : 0.0f;
      term = n ? (double)cnt * (double)sum / n : 0.0;
    }
    for (int h = 32; h > 0; h >>= 1) term += __shfl_xor(term, h, 64);
    if (tid == 0) {
      __hip_atomic_store(&a.terms[blockIdx.x], term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
  }
  __syncthreads();
  if (last && tid == 0) {
    double sum = 0;
    for (unsigned i = 0; i < gridDim.x; ++i)
      sum += __hip_atomic_load(&a.terms[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    o.n_valid[0] = n;
    o.loss[0] = n ? (float)((double)a.alpha * E * sum / ((double)a.K * n)) : 0.0f;
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

// Whether another of a row's 16 lanes holds the same value: rotations by one
// to eight places meet every pair. All lanes take part in each.
__device__ __forceinline__ bool repeated(int e) {
  constexpr int kRotate = 0x120;
  return (dpp_i32<kRotate + 1>(e) == e) | (dpp_i32<kRotate + 2>(e) == e) | (dpp_i32<kRotate + 3>(e) == e) |
         (dpp_i32<kRotate + 4>(e) == e) | (dpp_i32<kRotate + 5>(e) == e) | (dpp_i32<kRotate + 6>(e) == e) |
         (dpp_i32<kRotate + 7>(e) == e) | (dpp_i32<kRotate + 8>(e) == e);
}

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
    int e = -1 - lane;  // no choice: unlike every other lane's
    // the token's row is this wavefront's own: LDS keeps its order
    auto settle = [] {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    };
    if (a.dgate) {
      float dg = 0;
      if (lane < a.K) {
        const int at = a.expert[t * a.K + lane];
        if (at >= 0 && at < E) {
          e = at;
          dg = a.dgate[t * a.K + lane];
        }
      }
      // the router's choices are distinct; repeated ones of a caller's own list
      // are added one after the other, so that their order is fixed
      if (!__ballot(repeated(e))) {
        if (e >= 0) row[e] = dg;
      } else {
        for (int k = 0; k < a.K; ++k) {
          if (lane == k && e >= 0) row[e] += dg;
          settle();
        }
      }
    }
    settle();
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
      for (int j = 0; j < V; ++j)  // the choice matters where dloss is no number
        o.e[j] = from_f32<T>(ok ? p[i * V + j] * (g[i * V + j] - s) : 0.0f);
      stream_row<V>(out + t * E, (i * 16 + lane) * V, E, o);
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

// Forward workgroups, at most one to a CU, and their threads: no more than
// the tokens need, so that few tokens still spread over the CUs.
struct BalShape {
  int64_t grid;
  int block;
};
BalShape bal_shape(const argus_balance_t& p) {
  const int v = p.dtype == ARGUS_F32 ? 4 : 8, most = fwd_block((int)ceil_div(p.n_experts, 16 * v) * v);
  const int64_t even = ceil_div(ceil_div(p.n_tokens, kMaxGrid), 4) * 64;  // threads, a wavefront to four tokens
  const int block = (int)(even < 64 ? 64 : even < most ? even : most);
  const int64_t need = ceil_div(p.n_tokens, block / 16);
  return {need < 1 ? 1 : need < kMaxGrid ? need : kMaxGrid, block};
}

struct BalLayout {
  size_t cnt, valid, terms, ticket, total;
};
BalLayout bal_layout(const argus_balance_t& p) {
  const size_t g = (size_t)bal_shape(p).grid, part = align256(g * (size_t)p.n_experts * 4);
  BalLayout l;
  l.cnt = part;
  l.valid = 2 * part;
  l.terms = l.valid + align256(g * 8);
  l.ticket = l.terms + align256((size_t)ceil_div(p.n_experts, kJoin) * 8);
  l.total = l.ticket + 256;
  return l;
}

}  // namespace

size_t balance_workspace_bytes(const argus_balance_t& p) { return bal_layout(p).total; }

hipError_t launch_balance(const argus_balance_t& p, const void* logits, const uint8_t* mask,
                          const argus_balance_out_t& o, void* ws, hipStream_t st) {
  const BalShape shape = bal_shape(p);
  const int64_t grid = shape.grid;
  const BalLayout l = bal_layout(p);
  uint8_t* base = (uint8_t*)ws;
  BalArgs a{p.n_tokens, p.row_stride, p.n_experts, p.top_k, p.alpha, logits, mask, o.expert, o.gate, o.lse,
            (float*)base, (uint32_t*)(base + l.cnt), (uint32_t*)(base + l.valid), (double*)(base + l.terms),
            (uint32_t*)(base + l.ticket)};
  const hipError_t e = with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    return with_pieces<T>(p.n_experts, [&](auto ni) {
      constexpr int NI = decltype(ni)::value;
      const dim3 block(shape.block);
      if (p.top_k <= 8) hipLaunchKernelGGL((bal_fwd<T, NI, 8>), dim3((unsigned)grid), block, 0, st, a);
      else hipLaunchKernelGGL((bal_fwd<T, NI, 16>), dim3((unsigned)grid), block, 0, st, a);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(bal_join, dim3((unsigned)ceil_div(p.n_experts, kJoin)), dim3(1024), 0, st, a, (int32_t)grid, o);
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
