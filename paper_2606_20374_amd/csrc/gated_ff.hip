// Gated feed-forward block, forward and backward.
//
// Forward: g = x Wg^T and u = x Wu^T of the same columns are summed in one
// workgroup's registers, h = act(g) u leaves it.
// Backward, from the forward's rounded g and u: dg = dh u act'(g) and
// du = dh act(g), rounded to x's type as the operands that the matrix
// instructions take (half a step each), lie side by side in the workspace;
// dx = [dg | du] [Wg; Wu], [dWg; dWu] = [dg | du]^T x.
// In float16 a power of two that brings the largest of them below 2^15 is taken
// out before and put back by the products' ends: the gradient of a mean over
// some thousand tokens lies where float16 has no digits left, and products of
// two of its values leave its range. What is within 2^28 of the largest rounds by half
// a step of its own.
#include "product.h"

namespace argus {
using namespace product;

namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

// act(g) and its derivative.
__device__ __forceinline__ float2 activation(float g, int act) {
  if (act == ARGUS_SILU) {
    const float s = logistic(g);
    return make_float2(g * s, s * (1.0f + g * (1.0f - s)));
  }
  if (act == ARGUS_GELU) {
    // Phi(-z) = exp(-z^2 / 2) t S(t), t = 1 / (1 + 0.28 z), for z >= 0: the form of
    // Abramowitz and Stegun 7.1.26, S fitted here to 5e-7 of the value itself, so
    // that the tail keeps its digits (1 + erf is a difference of ones there).
    const float e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * g * g), t = __builtin_amdgcn_rcpf(1.0f + 0.28f * fabsf(g));
    float s = 0.024720103f;
    for (float c : {-0.09359359f, 0.09242878f, -0.006449664f, 0.0727752f, 0.08363075f, 0.10308467f, 0.111699805f, 0.11170386f})
      s = fmaf(s, t, c);
    const float tail = e * t * s, cdf = g < 0.0f ? tail : 1.0f - tail;
    return make_float2(g * cdf, cdf + g * e * 0.39894228f);
  }
  // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y)), y = sqrt(2 / pi) (g + 0.044715 g^3)
  // In the slope s (1 - s) is 0 long before the square leaves 32 bits: 0, not 0 times
  // infinity.
  const float s = logistic(1.5957691f * (g + 0.044715f * g * g * g));
  return make_float2(g * s, s + g * s * (1.0f - s) * 1.5957691f * (1.0f + 0.134145f * fminf(g * g, 0x1p100f)));
}

struct FfArgs {
  Operand x, wg, wu;
  void *h, *g, *u;
  int32_t act, mt, nt;
};

template <class TT>
__global__ __launch_bounds__(TT::THREADS) void ff_fwd(FfArgs a) {
  using T = typename TT::T;
  int m, n;
  tile_at(blockIdx.x, a.mt, a.nt, m, n);
  const int64_t m0 = (int64_t)m * TT::TM, n0 = (int64_t)n * (TT::TN / 2), F = a.wg.rows;
  TT t;
  const typename TT::LoadA la(a.x, m0);
  const typename TT::LoadB lb(a.wg, n0, a.wu, n0);
  t.run(la, lb, 0, (int)a.x.k);
#pragma unroll
  for (int i = 0; i < TT::FM; ++i) {
    auto to = [&](void* p) {
      return [=](int r) { return m0 + r < a.x.rows ? (T*)p + (m0 + r) * F + n0 : nullptr; };
    };
    t.template write<0, 1>(i, F - n0, [&](int j, int e) { return activation(t.acc[i][j][e], a.act).x * t.acc[i][j + TT::HN][e]; }, to(a.h));
    if (a.g) {
      t.template write<0, 1>(i, F - n0, [&](int j, int e) { return t.acc[i][j][e]; }, to(a.g));
      t.template write<0, 1>(i, F - n0, [&](int j, int e) { return t.acc[i][j + TT::HN][e]; }, to(a.u));
    }
  }
}

// FB blocks of 16 gate rows and the same up rows, NT blocks of 16 tokens.
template <class T, int NT, int FB, int U>
__global__ __launch_bounds__(64 * kFewWaves) void ff_few(FfArgs a) {
  const int lane = threadIdx.x & 63, q = lane >> 4, wave = threadIdx.x >> 6;
  const int64_t F = a.wg.rows, N = a.x.rows, f0 = xcd_item(blockIdx.x, gridDim.x) * (16 * FB);
  __amdgpu_buffer_rsrc_t w[2 * FB];
  int off[2 * FB], xoff[NT];
#pragma unroll
  for (int b = 0; b < 2 * FB; ++b) {
    const Operand& o = b < FB ? a.wg : a.wu;
    const int64_t first = f0 + b % FB * 16;
    w[b] = buffer((const char*)o.p + first * o.stride * 2, ((F - first - 1) * o.stride + o.k) * 2);
    off[b] = (int)(((lane & 15) * o.stride + 8 * q) * 2);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t row = t * 16 + (lane & 15);
    xoff[t] = row < N ? (int)((row * a.x.stride + 8 * q) * 2) : kNowhere;
  }
  Few<T, NT, 2 * FB, U> s;
  s.run(w, off, buffer(a.x.p, ((N - 1) * a.x.stride + a.x.k) * 2), xoff, (int)a.x.k);
  s.join();
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t % kFewWaves != wave) continue;
    const int64_t row = t * 16 + (lane & 15);
#pragma unroll
    for (int b = 0; b < FB; ++b) {
      const int64_t c = f0 + b * 16 + 4 * q;
      if (row >= N || c >= F) continue;  // F is a multiple of 8
      Vec<T, 4> h, g, u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float gv = s.acc[b][t][e], uv = s.acc[FB + b][t][e];
        h.e[e] = (T)(activation(gv, a.act).x * uv);
        g.e[e] = (T)gv;
        u.e[e] = (T)uv;
      }
      store_vec<4>((T*)a.h + row * F + c, h);
      if (a.g) {
        store_vec<4>((T*)a.g + row * F + c, g);
        store_vec<4>((T*)a.u + row * F + c, u);
      }
    }
  }
}

// dg and du of eight columns of a row.
template <class T>
__device__ __forceinline__ void point_of(const T* dh, const T* g, const T* u, int act, float (&dg)[8], float (&du)[8]) {
  const Vec<T, 8> d = load_vec<8>(dh), gv = load_vec<8>(g), uv = load_vec<8>(u);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 f = activation((float)gv.e[j], act);
    dg[j] = (float)d.e[j] * (float)uv.e[j] * f.y;
    du[j] = (float)d.e[j] * f.x;
  }
}

// Maximum over a workgroup of four wavefronts, in every thread.
__device__ __forceinline__ float group_max(float v) {
  __shared__ float tops[4];
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
}

constexpr int kMostGroups = 1024;
struct Range {
  float* most;    // [groups] largest finite |dg| and |du| of each workgroup of ff_most
  float* factor;  // [1] what the operands are to be multiplied with
  int32_t groups;
};

// The largest finite |dg| and |du|, before they are rounded to float16. They are
// computed again by ff_point: kept in 32 bits they would be more to write and
// read than what they are made from. Bound by memory: 16,384 tokens of 12,288 231 us,
// 5.2 TB/s; 999 of 2,720 5.4 us.
template <class T>
__global__ __launch_bounds__(256) void ff_most(const T* dh, int64_t stride, const T* g, const T* u, Range r, int64_t rows,
                                               int32_t F, int32_t act) {
  const int per = F / 8;
  const int64_t all = rows * per;
  float top = 0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int c = (int)(i - row * per) * 8;
    float dg[8], du[8];
    point_of(dh + row * stride + c, g + row * F + c, u + row * F + c, act, dg, du);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (fabsf(dg[j]) < __builtin_inff()) top = fmaxf(top, fabsf(dg[j]));
      if (fabsf(du[j]) < __builtin_inff()) top = fmaxf(top, fabsf(du[j]));
    }
  }
  top = group_max(top);
  if (threadIdx.x == 0) r.most[blockIdx.x] = top;
}

// 2^n, n = -126 .. 127.
__device__ __forceinline__ float power_of_two(int n) { return __int_as_float((n + 127) << 23); }

// dg and du of a row, eight columns to a thread: [rows][2][wide], zeros from F on.
template <class T>
__global__ __launch_bounds__(256) void ff_point(const T* dh, int64_t stride, const T* g, const T* u, T* to, Range r,
                                                int64_t rows, int32_t F, int32_t wide, int32_t act) {
  float out = 1.0f;
  if constexpr (std::is_same_v<T, f16_t>) {
    float top = 0;
    for (int i = threadIdx.x; i < r.groups; i += 256) top = fmaxf(top, r.most[i]);
    top = group_max(top);
    // 2^at <= top < 2^(at + 1), where top is not next to 0: 2^114 is finite as well
    int at = (__float_as_int(top) >> 23) - 127;
    at = at < -100 ? -100 : at;
    out = power_of_two(14 - at);
    if (blockIdx.x == 0 && threadIdx.x == 0) *r.factor = power_of_two(at - 14);
  }
  const int per = wide / 8;
  const int64_t all = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int c = (int)(i - row * per) * 8;
    Vec<T, 8> dg, du;
#pragma unroll
    for (int j = 0; j < 8; ++j) dg.e[j] = du.e[j] = (T)0.0f;
    if (c < F) {
      float a[8], b[8];
      point_of(dh + row * stride + c, g + row * F + c, u + row * F + c, act, a, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dg.e[j] = (T)(a[j] * out);
        du.e[j] = (T)(b[j] * out);
      }
    }
    store_vec<8>(to + row * 2 * wide + c, dg);
    store_vec<8>(to + row * 2 * wide + wide + c, du);
  }
}

int64_t wide_of(const argus_gated_ff_t& p) { return ceil_div(p.ff, 64) * 64; }
size_t point_bytes(const argus_gated_ff_t& p) { return align256((size_t)p.n_tokens * 2 * (size_t)wide_of(p) * 2); }
size_t range_bytes(const argus_gated_ff_t& p) { return p.dtype == ARGUS_F16 ? align256((kMostGroups + 1) * sizeof(float)) : 0; }

Plan plan_of(const argus_gated_ff_t& p) { return plan_grads(p.n_tokens, 2 * wide_of(p), 2 * wide_of(p), p.n_tokens, p.width); }
size_t sums_of(const argus_gated_ff_t& p, const Plan& plan, const Grid& g) { return g.S > 1 ? sums_bytes(plan, g, p.width) : 0; }

template <class T>
hipError_t forward(const argus_gated_ff_t& p, const void* x, const void* wg, const void* wu, void* h, void* g, void* u,
                   hipStream_t st) {
  FfArgs a{{x, p.n_tokens, p.width, p.x_stride}, {wg, p.ff, p.width, p.wg_stride}, {wu, p.ff, p.width, p.wu_stride},
           h, g, u, p.act, 0, 0};
  auto go = [&](auto tile) {
    using TT = decltype(tile);
    a.mt = (int32_t)ceil_div(p.n_tokens, TT::TM);
    a.nt = (int32_t)ceil_div(p.ff, TT::TN / 2);
    hipLaunchKernelGGL(ff_fwd<TT>, dim3((unsigned)(a.mt * a.nt)), dim3(TT::THREADS), 0, st, a);
    return hipGetLastError();
  };
  auto few = [&](auto kern, int rows) {
    hipLaunchKernelGGL(kern, dim3((unsigned)ceil_div(p.ff, rows)), dim3(64 * kFewWaves), 0, st, a);
    return hipGetLastError();
  };
  if (p.n_tokens <= 16) return few(ff_few<T, 1, 1, 4>, 16);
  if (p.n_tokens <= kFew) return few(ff_few<T, 2, 1, 3>, 16);
  return with_tile<T, false>(p.n_tokens, 2 * (int64_t)p.ff, p.width, g != nullptr, go);
}

template <class T>
hipError_t backward(const argus_gated_ff_t& p, const void* dh, const void* x, const void* wg, const void* wu, const void* g,
                    const void* u, void* dx, void* dwg, void* dwu, void* ws, hipStream_t st) {
  const int64_t wide = wide_of(p), W = p.width, F = p.ff, N = p.n_tokens;
  const Plan plan = plan_of(p);
  T* point = (T*)ws;
  float* most = (float*)((char*)ws + point_bytes(p));
  float* sums = (float*)((char*)most + range_bytes(p));
  Range range{};
  hipError_t e;
  if (N > 0) {
    const int64_t need = ceil_div(N * (wide / 8), 256);
    if constexpr (std::is_same_v<T, f16_t>) {
      range = {most, most + kMostGroups, (int32_t)(need < kMostGroups ? need : kMostGroups)};
      hipLaunchKernelGGL(ff_most<T>, dim3((unsigned)range.groups), dim3(256), 0, st, (const T*)dh, p.dh_stride, (const T*)g,
                         (const T*)u, range, N, p.ff, p.act);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(ff_point<T>, dim3((unsigned)(need < 16384 ? need : 16384)), dim3(256), 0, st, (const T*)dh,
                       p.dh_stride, (const T*)g, (const T*)u, point, range, N, p.ff, (int32_t)wide, p.act);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  Grad dinput{}, dweights{};
  dinput.f = dweights.f = range.factor;
  dinput.scale = dweights.scale = 1.0f;
  dinput.a = {point, N, 2 * wide, 2 * wide};
  dinput.b = {wg, W, F, p.wg_stride};
  dinput.b1 = {wu, W, F, p.wu_stride};
  dinput.k1 = wide;
  dinput.rows = {dx, nullptr, N, N, 0};
  dinput.grid = plan.x;
  dinput.sums = dinput.grid.S > 1 ? sums : nullptr;
  dweights.a = {point, 2 * wide, N, 2 * wide};
  dweights.b = {x, W, N, p.x_stride};
  dweights.rows = {dwg, dwu, F, wide, F};
  dweights.grid = plan.w;
  dweights.sums = dweights.grid.S > 1 ? sums + sums_of(p, plan, plan.x) / 4 : nullptr;
  if ((e = launch_grads<T, true, false>(plan, dinput, dweights, st)) != hipSuccess) return e;
  if (dinput.sums && (e = launch_join<T>(dinput, N, st)) != hipSuccess) return e;
  return dweights.sums ? launch_join<T>(dweights, wide + F, st) : hipSuccess;
}

}  // namespace

size_t gated_ff_workspace_bytes(const argus_gated_ff_t&) { return 0; }

size_t gated_ff_bwd_workspace_bytes(const argus_gated_ff_t& p) {
  const Plan plan = plan_of(p);
  return point_bytes(p) + range_bytes(p) + sums_of(p, plan, plan.x) + sums_of(p, plan, plan.w);
}

hipError_t launch_gated_ff(const argus_gated_ff_t& p, const void* x, const void* wg, const void* wu, void* h, void* g,
                           void* u, void*, hipStream_t st) {
  if (p.n_tokens == 0) return hipSuccess;
  return p.dtype == ARGUS_F16 ? forward<f16_t>(p, x, wg, wu, h, g, u, st) : forward<bf16_t>(p, x, wg, wu, h, g, u, st);
}

hipError_t launch_gated_ff_bwd(const argus_gated_ff_t& p, const void* dh, const void* x, const void* wg, const void* wu,
                               const void* g, const void* u, void* dx, void* dwg, void* dwu, void* ws, hipStream_t st) {
  return p.dtype == ARGUS_F16 ? backward<f16_t>(p, dh, x, wg, wu, g, u, dx, dwg, dwu, ws, st)
                              : backward<bf16_t>(p, dh, x, wg, wu, g, u, dx, dwg, dwu, ws, st);
}

}  // namespace argus
