// Softmax cross entropy over a large vocabulary, straight from the last hidden
// states: the logits z = scale x w^T live in registers only.
//
// Tokens that are learned are numbered first, in order, and their rows of x
// copied together where some are left out, so that ignored tokens cost no
// product and whatever their rows hold reaches nothing.
// Forward: each tile of logits leaves its rows' maximum and sum of
// exponentials; a further launch joins a row's tiles.
// Backward: a piece of the vocabulary at a time, the logits again, and
//   dz = c / C (exp(z - lse) (1 + 2 z_loss lse) - [v = label]),
// rounded to bfloat16 as the operand of dw = C scale dz^T x, which is final for
// these ids, and dx += C scale dz w, which is summed over the pieces in 32
// bits. C is the largest |c|: with a factor that all tokens share in the
// operand, dz of most labels, -c, would round by the same part of itself, and
// the sums by as much (0.0029 of their norm for 0.0023).
#include "cross_entropy_plan.h"

namespace argus {
using namespace product;

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// The learned tokens, in order.
struct Tokens {
  uint32_t* n;     // [2] how many, and a counter of workgroups that are done
  float* most;     // [1] largest |c| that is finite, 1 where that is next to 0; backward
  int32_t* index;  // [n] token
  int32_t* label;  // [n] forward
  int32_t* place;  // [T] number of a token, -1: not learned; backward
  float4* row;     // [n] backward: -lse in units of log2, c, c (1 + 2 z_loss lse), label
  bf16_t* x;       // [n][W], where n < T
};

struct CeArgs {
  Tokens t;
  Operand x, w;
  const void* labels;
  int32_t ids_64;
  int64_t T, V;
  float scale, z_loss;
  int32_t* status;
};

// Where an operator is small, every token is taken and those that are not learned
// are dropped at the end: index is null, rows are tokens, and n is T.
__device__ __forceinline__ int64_t count_of(const CeArgs& a) {
  return a.t.index ? (int64_t)__builtin_amdgcn_readfirstlane((int)*a.t.n) : a.T;
}
__device__ __forceinline__ int64_t token_of(const CeArgs& a, int64_t row) { return a.t.index ? a.t.index[row] : row; }
// The label of a token, at or above V where it is out of range.
__device__ __forceinline__ int64_t raw_label(const CeArgs& a, int64_t t) {
  return a.ids_64 ? ((const int64_t*)a.labels)[t] : (int64_t)((const int32_t*)a.labels)[t];
}
__device__ __forceinline__ int64_t label_of(const CeArgs& a, int64_t row) {
  if (a.t.index) return a.t.label[row];
  const int64_t l = raw_label(a, row);
  return l >= 0 && l < a.V ? l : -1;
}

constexpr int kIndexThreads = 1024;

struct IndexArgs {
  float *loss, *lse_out;  // forward: of tokens that are not learned
  uint32_t* n_valid;
  const float *lse, *dloss, *dmean;  // backward
  const uint32_t* divisor;
  int32_t* status;
};

// Numbers the tokens, one to a thread. Each workgroup counts those before its own
// by itself, and the first looks at all of them for the totals: of 16,384 tokens
// that takes 6.5 us, one workgroup that goes through them 23.
__global__ __launch_bounds__(kIndexThreads) void ce_index(CeArgs a, IndexArgs o) {
  constexpr int kWaves = kIndexThreads / 64, kDeep = 8;  // loads of a thread under way
  __shared__ uint32_t sums[kWaves], before[kWaves];
  __shared__ float tops[kWaves];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const bool first = blockIdx.x == 0;
  float mean = 0;
  if (o.dmean) {
    const uint32_t d = *o.divisor;
    mean = *o.dmean / (float)(d ? d : 1);
  }
  const int64_t base = (int64_t)blockIdx.x * kIndexThreads, t = base + threadIdx.x;
  int64_t id = t < a.T ? raw_label(a, t) : -1;
  if (id >= a.V) id = -1;
  // the tokens before, or all
  const int64_t end = first ? a.T : base;
  uint32_t n = 0;
  float top = 0;
  bool range = false;
  for (int64_t i0 = threadIdx.x; i0 < end; i0 += kIndexThreads * kDeep) {
    int64_t ids[kDeep];
    float c[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const int64_t i = i0 + j * kIndexThreads;
      ids[j] = i < end ? raw_label(a, i) : -1;
      c[j] = first && o.dloss && i < end ? o.dloss[i] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      range |= ids[j] >= a.V;
      if (ids[j] < 0 || ids[j] >= a.V) continue;
      ++n;
      const float size = fabsf(mean + c[j]);
      if (size < __builtin_inff()) top = fmaxf(top, size);
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    n += __shfl_xor(n, d);
    top = fmaxf(top, __shfl_xor(top, d));
  }
  const uint64_t there = __ballot(id >= 0);
  if (lane == 0) {
    before[w] = n;
    sums[w] = (uint32_t)__popcll(there);
    tops[w] = top;
  }
  if (first && threadIdx.x == 0) {
    a.t.n[1] = 0;
    if (o.status) *o.status = 0;
  }
  __syncthreads();
  uint32_t at = (uint32_t)__popcll(there & (((uint64_t)1 << lane) - 1)), all = 0;
#pragma unroll
  for (int j = 0; j < kWaves; ++j) {
    all += before[j];
    if (j < w) at += sums[j];
  }
  if (!first) at += all;
  if (id >= 0) {
    a.t.index[at] = (int32_t)t;
    if (!a.t.row) {
      a.t.label[at] = (int32_t)id;
    } else {
      const float lse = o.lse[t], c = mean + (o.dloss ? o.dloss[t] : 0.0f);
      a.t.row[at] = make_float4(-lse * kLog2e, c, c * (1.0f + 2.0f * a.z_loss * lse), __int_as_float((int32_t)id));
    }
  } else if (o.loss && t < a.T) {
    o.loss[t] = 0.0f;
    o.lse_out[t] = -__builtin_inff();
  }
  if (a.t.place && t < a.T) a.t.place[t] = id >= 0 ? (int32_t)at : -1;
  if (!first) return;
  if (range && o.status) atomicOr(o.status, ARGUS_DEV_TOKEN_RANGE);
  if (threadIdx.x) return;
  *a.t.n = all;
  if (o.n_valid) *o.n_valid = all;
  if (a.t.most) {
    for (int j = 0; j < kWaves; ++j) top = fmaxf(top, tops[j]);
    *a.t.most = top > 0x1p-100f ? top : 1.0f;  // one that can be divided by
  }
}

// Backward, small: rows of zeros in the place of those of tokens that are not
// learned, and what ce_index notes of each token. A row to a wavefront.
__global__ __launch_bounds__(256) void ce_rows(CeArgs a, IndexArgs o) {
  __shared__ float tops[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 4 + w;
  float mean = 0;
  if (o.dmean) {
    const uint32_t d = *o.divisor;
    mean = *o.dmean / (float)(d ? d : 1);
  }
  if (row < a.T) {
    const int64_t id = label_of(a, row);
    const bf16_t* from = (const bf16_t*)a.x.p + row * a.x.stride;
    bf16_t* to = a.t.x + row * a.x.k;
    Vec<bf16_t, 8> none;
#pragma unroll
    for (int j = 0; j < 8; ++j) none.e[j] = (bf16_t)0.0f;
    for (int64_t c = lane * 8; c < a.x.k; c += 512) store_vec<8>(to + c, id >= 0 ? load_vec<8>(from + c) : none);
    if (lane == 0) {
      const float lse = id >= 0 ? o.lse[row] : 0.0f, c = mean + (o.dloss ? o.dloss[row] : 0.0f);
      // a token that is not learned: no label, and a dz of zeros
      a.t.row[row] = id >= 0 ? make_float4(-lse * kLog2e, c, c * (1.0f + 2.0f * a.z_loss * lse), __int_as_float((int32_t)id))
                             : make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));
      a.t.place[row] = id >= 0 ? (int32_t)row : -1;
    }
  }
  if (blockIdx.x) return;
  float top = 0;
  bool range = false;
  for (int64_t t = threadIdx.x; t < a.T; t += 256) {
    const int64_t id = raw_label(a, t);
    const float c = fabsf(mean + (o.dloss ? o.dloss[t] : 0.0f));
    if (id >= 0 && id < a.V && c < __builtin_inff()) top = fmaxf(top, c);
    range |= id >= a.V;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[w] = top;
  if (threadIdx.x == 0 && o.status) *o.status = 0;
  __syncthreads();
  if (range && o.status) atomicOr(o.status, ARGUS_DEV_TOKEN_RANGE);
  if (threadIdx.x) return;
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  *a.t.most = top > 0x1p-100f ? top : 1.0f;  // one that can be divided by
}

// A row to a wavefront.
__global__ __launch_bounds__(256) void ce_gather(CeArgs a) {
  const int64_t n = *a.t.n, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n == a.T || row >= n) return;
  const bf16_t* from = (const bf16_t*)a.x.p + a.t.index[row] * a.x.stride;
  bf16_t* to = a.t.x + row * a.x.k;
  for (int64_t c = (threadIdx.x & 63) * 8; c < a.x.k; c += 512) store_vec<8>(to + c, load_vec<8>(from + c));
}

__device__ __forceinline__ Operand learned(const CeArgs& a, int64_t n) {
  if (!a.t.index || n == a.T) return a.x;
  return {a.t.x, n, a.x.k, a.x.k};
}

// Maximum over the four rows of a wavefront, lane by lane, in every row.
__device__ __forceinline__ float rows_max(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// Before the join, where no launch has numbered the tokens.
__device__ __forceinline__ void clear_for_join(const CeArgs& a) {
  a.t.n[1] = 0;
  if (a.status) *a.status = 0;
}

template <class TT>
__global__ __launch_bounds__(TT::THREADS) void ce_fwd(CeArgs a, float2* part, float* own, int nt) {
  __shared__ float2 join[TT::WN][TT::TM];
  const int64_t count = count_of(a);
  if (!a.t.index && blockIdx.x == 0 && threadIdx.x == 0) clear_for_join(a);
  const int mt = (int)((count + TT::TM - 1) / TT::TM);
  if (blockIdx.x >= (unsigned)mt * nt) return;
  int m, n;
  tile_at(blockIdx.x, mt, nt, m, n);
  const int64_t m0 = (int64_t)m * TT::TM, n0 = (int64_t)n * TT::TN;
  TT t;
  const typename TT::LoadA la(learned(a, count), m0);
  const typename TT::LoadB lb(a.w, n0);
  t.run(la, lb, 0, (int)a.x.k);
  const int lane = threadIdx.x & 63, q = lane >> 4;
#pragma unroll
  for (int i = 0; i < TT::FM; ++i) {
    const int at = TT::row_of(i) + (lane & 15);
    const int64_t label = m0 + at < count ? label_of(a, m0 + at) - n0 : -1;
    float top = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < TT::FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float z = t.acc[i][j][e] * a.scale;
        if (n0 + TT::TN > a.V && n0 + TT::col_of(j) + 4 * q + e >= a.V) z = -__builtin_inff();
        t.acc[i][j][e] = z;
        top = fmaxf(top, z);
      }
    if (__any(label >= 0 && label < TT::TN)) {
#pragma unroll
      for (int j = 0; j < TT::FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (label == TT::col_of(j) + 4 * q + e) own[m0 + at] = t.acc[i][j][e];
    }
    top = rows_max(top);
    const float from = top == -__builtin_inff() ? 0.0f : top;  // no difference of infinities
    float sum = 0;
#pragma unroll
    for (int j = 0; j < TT::FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((t.acc[i][j][e] - from) * kLog2e);
    sum = rows_sum(sum);
    if (q == 0) join[TT::wave() % TT::WN][at] = make_float2(top, sum);
  }
  __syncthreads();
  for (int r = threadIdx.x; r < TT::TM; r += TT::THREADS) {
    if (m0 + r >= count) break;
    float top = -__builtin_inff(), sum = 0;
#pragma unroll
    for (int j = 0; j < TT::WN; ++j) top = fmaxf(top, join[j][r].x);
    const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int j = 0; j < TT::WN; ++j) sum += join[j][r].y * __builtin_amdgcn_exp2f((join[j][r].x - from) * kLog2e);
    part[(m0 + r) * nt + n] = make_float2(top, sum);
  }
}

// Operands of few tokens: NB blocks of 16 ids from v0 on, and the learned tokens,
// which need not lie together.
template <int NB>
__device__ __forceinline__ void few_weights(const CeArgs& a, int64_t v0, __amdgpu_buffer_rsrc_t (&w)[NB], int (&off)[NB]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t first = v0 + 16 * b < a.V ? v0 + 16 * b : a.V - 1;  // of a block past the end: dropped
    w[b] = buffer((const char*)a.w.p + first * a.w.stride * 2, ((a.V - first - 1) * a.w.stride + a.w.k) * 2);
    off[b] = (int)(((lane & 15) * a.w.stride + 8 * (lane >> 4)) * 2);
  }
}
template <int NT>
__device__ __forceinline__ void few_tokens(const CeArgs& a, int count, int (&xoff)[NT]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = t * 16 + (lane & 15);
    xoff[t] = row < count ? (int)((token_of(a, row) * a.x.stride + 8 * (lane >> 4)) * 2) : kNowhere;
  }
}

// As ce_fwd for at most kFew tokens: 16 NB ids to a workgroup.
template <int NT, int NB, int U>
__global__ __launch_bounds__(64 * kFewWaves) void ce_few(CeArgs a, float2* part, float* own, int nt) {
  const int lane = threadIdx.x & 63, q = lane >> 4, wave = threadIdx.x >> 6;
  const int count = (int)count_of(a), n = (int)xcd_item(blockIdx.x, nt);
  if (!a.t.index && blockIdx.x == 0 && threadIdx.x == 0) clear_for_join(a);
  const int64_t v0 = (int64_t)n * (16 * NB);
  __amdgpu_buffer_rsrc_t w[NB];
  int off[NB], xoff[NT];
  few_weights<NB>(a, v0, w, off);
  few_tokens<NT>(a, count, xoff);
  Few<bf16_t, NT, NB, U> s;
  s.run(w, off, buffer(a.x.p, ((a.T - 1) * a.x.stride + a.x.k) * 2), xoff, (int)a.x.k);
  s.join();
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = t * 16 + (lane & 15);
    if (t % kFewWaves != wave || t * 16 >= count) continue;
    const int64_t label = row < count ? label_of(a, row) - v0 : -1;
    float top = -__builtin_inff(), sum = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 16 * b + 4 * q + e;
        float z = s.acc[b][t][e] * a.scale;
        if (c == label) own[row] = z;
        if (v0 + c >= a.V) z = -__builtin_inff();
        s.acc[b][t][e] = z;
        top = fmaxf(top, z);
      }
    top = rows_max(top);
    const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((s.acc[b][t][e] - from) * kLog2e);
    sum = rows_sum(sum);
    if (q == 0 && row < count) part[(int64_t)row * nt + n] = make_float2(top, sum);
  }
}

// Adds the pair (top, sum) b to a.
__device__ __forceinline__ float2 both(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x), from = top == -__builtin_inff() ? 0.0f : top;
  return make_float2(top, a.y * __builtin_amdgcn_exp2f((a.x - from) * kLog2e) + b.y * __builtin_amdgcn_exp2f((b.x - from) * kLog2e));
}

// A token to WAVES wavefronts of four. With MEAN the workgroup that is done last
// takes the mean: losses are written past the caches of its XCD and read past
// them. Each workgroup then writes its XCD's cache back: of 16,384 tokens that
// took 133 us, a launch of its own after 22 us takes 5.
template <int WAVES, bool MEAN>
__global__ __launch_bounds__(256) void ce_join(CeArgs a, const float2* part, const float* own, int nt, float* loss,
                                               float* lse, float* mean, uint32_t* n_valid) {
  __shared__ float2 pairs[4];
  __shared__ double sums[4];
  __shared__ uint32_t counts[4];
  __shared__ bool last;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = threadIdx.x % (64 * WAVES);
  const int64_t n = count_of(a), row = (int64_t)blockIdx.x * (4 / WAVES) + wave / WAVES;
  float2 p = make_float2(-__builtin_inff(), 0.0f);
  if (row < n)
    for (int j = in; j < nt; j += 64 * WAVES) p = both(p, part[row * nt + j]);
#pragma unroll
  for (int d = 32; d; d >>= 1) p = both(p, make_float2(__shfl_xor(p.x, d), __shfl_xor(p.y, d)));
  if (WAVES > 1) {
    if (lane == 0) pairs[wave] = p;
    __syncthreads();
    p = pairs[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) p = both(p, pairs[w]);
  }
  if (row < n && in == 0) {
    const int64_t t = token_of(a, row);
    const float from = p.x == -__builtin_inff() ? 0.0f : p.x, rest = logf(p.y);
    float all = from + rest, l;
    if (a.t.index || (raw_label(a, t) >= 0 && raw_label(a, t) < a.V)) {
      // the largest logit's distance first: a sure token's loss is what is left of the sum
      l = (from - own[row]) + rest + a.z_loss * all * all;
    } else {
      l = 0.0f;
      all = -__builtin_inff();
      if (a.status && raw_label(a, t) >= a.V) atomicOr(a.status, ARGUS_DEV_TOKEN_RANGE);
    }
    __hip_atomic_store(loss + t, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    lse[t] = all;
  }
  if (!MEAN) return;
  __syncthreads();
  if (threadIdx.x == 0) last = __hip_atomic_fetch_add(a.t.n + 1, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  double s = 0;
  uint32_t c = 0;
  for (int64_t i = threadIdx.x; i < a.T; i += 256 * 4) {
    float v[4];  // all under way before the first is added
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t t = i + 256 * j;
      v[j] = t < a.T ? __hip_atomic_load(loss + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0f;
      c += t < a.T && raw_label(a, t) >= 0 && raw_label(a, t) < a.V;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s += v[j];
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    s += __shfl_xor(s, d);
    c += __shfl_xor(c, d);
  }
  if (lane == 0) {
    sums[wave] = s;
    counts[wave] = c;
  }
  __syncthreads();
  if (threadIdx.x) return;
  c = counts[0] + counts[1] + counts[2] + counts[3];
  *n_valid = c;
  *mean = (float)((sums[0] + sums[1] + sums[2] + sums[3]) / (double)(c ? c : 1));
}

__global__ __launch_bounds__(1024) void ce_mean(CeArgs a, const float* loss, float* mean) {
  __shared__ double sums[16];
  double s = 0;
  for (int64_t t = threadIdx.x; t < a.T; t += 1024) s += loss[t];
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = 0;
  for (int j = 0; j < 16; ++j) s += sums[j];
  *mean = (float)(s / (*a.t.n ? *a.t.n : 1));
}

// dz of the ids [v0, v0 + cols) of the vocabulary, `cols` a multiple of 64.
template <class TT>
__global__ __launch_bounds__(TT::THREADS) void ce_dz(CeArgs a, bf16_t* dz, int64_t v0, int64_t cols, int64_t stride,
                                                     int nt) {
  const int64_t count = count_of(a);
  const int mt = (int)((count + TT::TM - 1) / TT::TM);
  if (blockIdx.x >= (unsigned)mt * nt) return;
  int m, n;
  tile_at(blockIdx.x, mt, nt, m, n);
  const int64_t m0 = (int64_t)m * TT::TM, n0 = (int64_t)n * TT::TN;
  TT t;
  const typename TT::LoadA la(learned(a, count), m0);
  const typename TT::LoadB lb(a.w, v0 + n0);
  t.run(la, lb, 0, (int)a.x.k);
  const int lane = threadIdx.x & 63, q = lane >> 4;
  const float sc = a.scale * kLog2e, inv = 1.0f / *a.t.most;
  float4 rows[TT::FM];
#pragma unroll
  for (int i = 0; i < TT::FM; ++i) {
    const int64_t row = m0 + TT::row_of(i) + (lane & 15);
    rows[i] = a.t.row[row < count ? row : count - 1];  // computed and not written
  }
#pragma unroll
  for (int i = 0; i < TT::FM; ++i) {
    const float less = rows[i].x, f = rows[i].y * inv, more = rows[i].z * inv;
    const int64_t label = __float_as_int(rows[i].w) - v0 - n0;
#pragma unroll
    for (int j = 0; j < TT::FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) t.acc[i][j][e] = more * __builtin_amdgcn_exp2f(fmaf(t.acc[i][j][e], sc, less));
    // few tiles hold a label of their rows, or the vocabulary's end
    if (__any(label >= 0 && label < TT::TN)) {
#pragma unroll
      for (int j = 0; j < TT::FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (label == TT::col_of(j) + 4 * q + e) t.acc[i][j][e] -= f;
    }
    // not 0 times what its row of zeros gives: an infinite weight makes that NaN
    if (__any(__float_as_int(rows[i].w) < 0)) {
#pragma unroll
      for (int j = 0; j < TT::FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (__float_as_int(rows[i].w) < 0) t.acc[i][j][e] = 0.0f;
    }
    if (v0 + n0 + TT::TN > a.V) {
#pragma unroll
      for (int j = 0; j < TT::FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v0 + n0 + TT::col_of(j) + 4 * q + e >= a.V) t.acc[i][j][e] = 0.0f;
    }
    t.template write<0, 2>(i, cols - n0, [&](int j, int e) { return t.acc[i][j][e]; },
                           [&](int r) { return m0 + r < count ? dz + (m0 + r) * stride + n0 : nullptr; });
  }
}

// As ce_dz for at most kFew tokens and the whole vocabulary.
template <int NT, int NB, int U>
__global__ __launch_bounds__(64 * kFewWaves) void ce_dz_few(CeArgs a, bf16_t* dz, int64_t cols, int64_t stride) {
  const int lane = threadIdx.x & 63, q = lane >> 4, wave = threadIdx.x >> 6, count = (int)count_of(a);
  const int64_t v0 = xcd_item(blockIdx.x, gridDim.x) * (16 * NB);
  __amdgpu_buffer_rsrc_t w[NB];
  int off[NB], xoff[NT];
  few_weights<NB>(a, v0, w, off);
  few_tokens<NT>(a, count, xoff);
  Few<bf16_t, NT, NB, U> s;
  s.run(w, off, buffer(a.x.p, ((a.T - 1) * a.x.stride + a.x.k) * 2), xoff, (int)a.x.k);
  s.join();
  const float sc = a.scale * kLog2e, inv = 1.0f / *a.t.most;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = t * 16 + (lane & 15);
    if (t % kFewWaves != wave || row >= count) continue;
    const float4 r = a.t.row[row];
    const bool learned = __float_as_int(r.w) >= 0;
    const int64_t label = __float_as_int(r.w) - v0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int64_t c = v0 + 16 * b + 4 * q;
      Vec<bf16_t, 4> o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float p = r.z * inv * __builtin_amdgcn_exp2f(fmaf(s.acc[b][t][e], sc, r.x));
        if (16 * b + 4 * q + e == label) p -= r.y * inv;
        o.e[e] = (bf16_t)(learned && c + e < a.V ? p : 0.0f);
      }
      if (c < cols) store_vec<4>(dz + row * stride + c, o);
    }
  }
}

// dx of every token from the parts' sums: zeros where it is not learned.
__global__ __launch_bounds__(256) void ce_dx(Tokens t, Grad g, int64_t T, int64_t W, bf16_t* dx) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= T * W) return;
  const int64_t row = i / W, at = t.place[row];
  Vec<bf16_t, 8> o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o.e[j] = (bf16_t)0.0f;
  if (at >= 0) {
    const float f = factor_of(g);
    const Vec<float, 8> v = sum_parts(g.sums, g.n ? counted(g.grid, *g.n, g.tile) : g.grid, g.tile, at, W, i - row * W);
#pragma unroll
    for (int j = 0; j < 8; ++j) o.e[j] = (bf16_t)(v.e[j] * f);
  }
  store_vec<8>(dx + i, o);
}

__global__ __launch_bounds__(256) void ce_clear(bf16_t* p, int64_t n) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += (int64_t)gridDim.x * 2048)
    *(uint4*)(p + i) = make_uint4(0, 0, 0, 0);
}

struct Space {
  char* p;
  size_t at = 0;
  template <class T>
  T* take(size_t n) {
    T* r = (T*)(p + at);
    at += align256(n * sizeof(T));
    return r;
  }
};

struct Forward {
  Tokens t;
  float2* part;
  float* own;
  size_t bytes;
};
Forward forward_space(const argus_cross_entropy_t& p, void* ws) {
  Space s{(char*)ws};
  const size_t T = (size_t)p.n_tokens;
  Forward f{};
  f.t.n = s.take<uint32_t>(2);
  f.t.index = s.take<int32_t>(T);
  f.t.label = s.take<int32_t>(T);
  f.t.x = s.take<bf16_t>(T * (size_t)p.width);
  f.part = s.take<float2>(T * (size_t)tiles_n(p));
  f.own = s.take<float>(T);
  f.bytes = s.at;
  return f;
}

struct Backward {
  Tokens t;
  bf16_t* dz;
  float *dx, *dw;
  int64_t piece;
  Plan plan;  // of a piece
  size_t bytes;
};
Backward backward_space(const argus_cross_entropy_t& p, void* ws) {
  Space s{(char*)ws};
  const size_t T = (size_t)p.n_tokens;
  Backward b{};
  b.piece = piece_of(p);
  b.plan = plan_of(p);
  b.t.n = s.take<uint32_t>(2);
  b.t.most = s.take<float>(1);
  b.t.index = s.take<int32_t>(T);
  b.t.place = s.take<int32_t>(T);
  b.t.row = s.take<float4>(T);
  b.t.x = s.take<bf16_t>(T * (size_t)p.width);
  b.dz = s.take<bf16_t>(T * (size_t)b.piece);
  b.dx = s.take<float>(sums_bytes(b.plan, b.plan.x, p.width) / 4);
  b.dw = s.take<float>(b.plan.w.S > 1 ? sums_bytes(b.plan, b.plan.w, p.width) / 4 : 0);
  b.bytes = s.at;
  return b;
}

CeArgs args_of(const argus_cross_entropy_t& p, const Tokens& t, const void* x, const void* w) {
  return {t, {x, p.n_tokens, p.width, p.x_stride}, {w, p.n_vocab, p.width, p.w_stride},
          p.labels, p.ids_64, p.n_tokens, p.n_vocab, p.scale, p.z_loss, nullptr};
}

hipError_t launch_tokens(const CeArgs& a, const IndexArgs& o, bool rows, hipStream_t st) {
  hipLaunchKernelGGL(ce_index, dim3((unsigned)(a.T > 0 ? ceil_div(a.T, kIndexThreads) : 1)), dim3(kIndexThreads), 0, st, a, o);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !rows) return e;
  hipLaunchKernelGGL(ce_gather, dim3((unsigned)ceil_div(a.T, 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t cross_entropy_workspace_bytes(const argus_cross_entropy_t& p) { return forward_space(p, nullptr).bytes; }
size_t cross_entropy_bwd_workspace_bytes(const argus_cross_entropy_t& p) { return backward_space(p, nullptr).bytes; }

hipError_t launch_cross_entropy(const argus_cross_entropy_t& p, const void* x, const void* w,
                                const argus_cross_entropy_out_t& o, void* ws, hipStream_t st) {
  const Forward f = forward_space(p, ws);
  CeArgs a = args_of(p, f.t, x, w);
  const int64_t T = p.n_tokens, V = p.n_vocab, W = p.width;
  const bool small = T > 0 && is_small(p);
  a.status = o.dev_status;
  hipError_t e;
  if (small) a.t.index = nullptr;
  else if ((e = launch_tokens(a, {o.loss, o.lse, o.n_valid, nullptr, nullptr, nullptr, nullptr, o.dev_status}, T > 0, st)) != hipSuccess)
    return e;
  const int nt = (int)tiles_n(p);
  auto go = [&](auto tile) {
    using TT = decltype(tile);
    const int mt = (int)ceil_div(T, TT::TM);
    hipLaunchKernelGGL(ce_fwd<TT>, dim3((unsigned)(mt * nt)), dim3(TT::THREADS), 0, st, a, f.part, f.own, nt);
  };
  auto few = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((unsigned)nt), dim3(64 * kFewWaves), 0, st, a, f.part, f.own, nt);
  };
  if (T == 0) {
  } else if (is_few(p)) {
    if (few_ids(p) == 32) T <= 16 ? few(ce_few<1, 2, 4>) : few(ce_few<2, 2, 3>);
    else T <= 16 ? few(ce_few<1, 8, 1>) : few(ce_few<2, 8, 1>);
  } else {
    with_tile<bf16_t, true>(T, V, W, false, go);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  auto join = [&](auto kern, int64_t rows) {
    const int64_t need = ceil_div(T, rows);
    hipLaunchKernelGGL(kern, dim3((unsigned)(need > 0 ? need : 1)), dim3(256), 0, st, a, f.part, f.own, nt, o.loss, o.lse, o.mean, o.n_valid);
  };
  // few tokens: a workgroup to each
  if (T <= 1024) {
    join(ce_join<4, true>, 1);
    return hipGetLastError();
  }
  join(ce_join<1, false>, 4);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(ce_mean, dim3(1), dim3(1024), 0, st, a, o.loss, o.mean);
  return hipGetLastError();
}

hipError_t launch_cross_entropy_bwd(const argus_cross_entropy_t& p, const void* x, const void* w, const float* lse,
                                    const uint32_t* n_valid, const float* dmean, const float* dloss, void* dx, void* dw,
                                    int32_t* dev_status, void* ws, hipStream_t st) {
  const Backward b = backward_space(p, ws);
  const int64_t T = p.n_tokens, V = p.n_vocab, W = p.width;
  hipError_t e;
  if (T == 0) {
    if (dev_status) {
      const CeArgs a = args_of(p, b.t, x, w);
      if ((e = launch_tokens(a, {nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, dev_status}, false, st)) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(ce_clear, dim3(2048), dim3(256), 0, st, (bf16_t*)dw, V * W);
    return hipGetLastError();
  }
  CeArgs a = args_of(p, b.t, x, w);
  const IndexArgs io{nullptr, nullptr, nullptr, lse, dloss, dmean, n_valid, dev_status};
  const bool small = is_small(p);
  if (small) {
    a.t.index = nullptr;
    hipLaunchKernelGGL(ce_rows, dim3((unsigned)ceil_div(T, 4)), dim3(256), 0, st, a, io);
    e = hipGetLastError();
    a.x = {b.t.x, T, W, W};
  } else {
    e = launch_tokens(a, io, true, st);
  }
  if (e != hipSuccess) return e;
  const bool whole = small && b.piece >= V && b.plan.x.S == 1;  // dx leaves the product as it is
  Grad g{};
  for (int64_t v0 = 0; v0 < V; v0 += b.piece) {
    const int64_t ids = V - v0 < b.piece ? V - v0 : b.piece, cols = ceil_div(ids, 64) * 64;
    auto go = [&](auto tile) {
      using TT = decltype(tile);
      const int mt = (int)ceil_div(T, TT::TM), nt = (int)ceil_div(cols, TT::TN);
      hipLaunchKernelGGL(ce_dz<TT>, dim3((unsigned)(mt * nt)), dim3(TT::THREADS), 0, st, a, b.dz, v0, cols, b.piece, nt);
      return hipGetLastError();
    };
    auto few = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)ceil_div(cols, few_ids(p))), dim3(64 * kFewWaves), 0, st, a, b.dz, cols, b.piece);
      return hipGetLastError();
    };
    if (is_few(p)) {
      if (few_ids(p) == 32) e = T <= 16 ? few(ce_dz_few<1, 2, 4>) : few(ce_dz_few<2, 2, 3>);
      else e = T <= 16 ? few(ce_dz_few<1, 8, 1>) : few(ce_dz_few<2, 8, 1>);
    } else {
      e = with_tile<bf16_t, true>(T, cols, W, false, go);
    }
    if (e != hipSuccess) return e;
    g = Grad{};
    g.a = {b.dz, T, cols, b.piece};
    g.b = {(const char*)w + v0 * p.w_stride * 2, W, ids, p.w_stride};
    g.n = small ? nullptr : b.t.n;
    g.f = b.t.most;
    g.scale = p.scale;
    g.grid = b.plan.x;
    g.add = v0 > 0;
    if (whole) {
      g.rows = {dx, nullptr, T, T, 0};
      g.place = b.t.place;
    } else {
      g.sums = b.dx;
    }
    Grad d{};
    d.a = {b.dz, cols, T, b.piece};
    d.b = {a.x.p, W, T, a.x.stride};
    d.b1 = {b.t.x, W, T, W};
    d.n = g.n;
    d.f = b.t.most;
    d.scale = p.scale;
    d.rows = {(bf16_t*)dw + v0 * W, nullptr, ids, ids, 0};
    d.grid = b.plan.w;
    d.grid.mt = (int32_t)ceil_div(ids, b.plan.tile());
    d.sums = d.grid.S > 1 ? b.dw : nullptr;
    if ((e = launch_grads<bf16_t, false, true>(b.plan, g, d, st)) != hipSuccess) return e;
    if (d.sums && (e = launch_join<bf16_t>(d, ids, st)) != hipSuccess) return e;
  }
  if (whole) return hipSuccess;
  hipLaunchKernelGGL(ce_dx, dim3((unsigned)ceil_div(T * W, 2048)), dim3(256), 0, st, b.t, g, T, W, (bf16_t*)dx);
  return hipGetLastError();
}

}  // namespace argus
