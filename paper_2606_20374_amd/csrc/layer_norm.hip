// Layer norm and its gradients.
//
// Forward, per row of cols elements: mean, then the sum of (x - mean)^2 over
// the row that is still in registers, y = (x - mean) rstd w + b. Backward,
// with xhat = (x - mean) rstd and g = dy w:
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  dw = sum dy xhat,
//   db = sum dy.
// Both are bound by memory: a row is read once (x; x and dy) and written once.
// A row belongs to one wavefront where it is at most two 16-byte vectors per
// lane wide (no barrier at all), to as many wavefronts as have a vector per
// lane up to 1,024 vectors, and to up to sixteen wavefronts of more vectors
// past that. Workgroups stay and take every n-th row, so that the weights and,
// backward, the sums of the weight's gradient live in registers. Forward the
// next row is loaded before the current one is reduced; backward its registers
// would cost a workgroup of the CU, which hides more (20,011 x 5,000 bf16, all
// launches: 232 us with, 135 us without). The gradient sums of the workgroups
// are written once each ([workgroups][2][cols]) and added in the order of the
// workgroups. All sums are 32-bit floats. 32,768 x 4,096 bf16 forward: 99 us,
// 5.4 TB/s, more than a large copy reaches (5.0).
#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace argus {
namespace {

template <typename T>
constexpr int kVec = 16 / sizeof(T);

struct LnArgs {
  int64_t rows, x_stride, dy_stride;
  int32_t cols;
  float eps;
  const void *x, *dy, *w, *b;
  void *y, *dx;
  float *mean, *rstd;
  float* part;  // [workgroups][2][cols]
  int32_t has_db;
};

constexpr int kMaxWaves = 16;

// Sums of M values over the threads of a row (a wavefront, or the workgroup),
// in every thread of it. `slot` alternates between calls, so one barrier per
// call is enough.
template <bool WAVE, int M>
__device__ __forceinline__ void row_sums(float (&v)[M], float* lds, int slot) {
#pragma unroll
  for (int m = 0; m < M; ++m) v[m] = wave_sum_f32(v[m]);
  if constexpr (!WAVE) {
    // sixteen places to a value: those of wavefronts that do not exist stay 0
    float* s = lds + slot * (kMaxWaves * M);
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int m = 0; m < M; ++m) s[m * kMaxWaves + w] = v[m];
    }
    lds_barrier();
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = row_sum(s[m * kMaxWaves + (threadIdx.x & 15)]);
  }
}

template <typename T, typename W, int N, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void ln_fwd(LnArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float lds[2 * kMaxWaves];
  const int tpr = WAVE ? 64 : blockDim.x, lane = WAVE ? threadIdx.x & 63 : threadIdx.x, cols = a.cols;
  constexpr int RPB = WAVE ? 4 : 1;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + (WAVE ? threadIdx.x >> 6 : 0);
  if (!WAVE) {
    if (threadIdx.x < 2 * kMaxWaves) lds[threadIdx.x] = 0;
    __syncthreads();
  }
  const T* x = (const T*)a.x;
  T* y = (T*)a.y;
  const float inv = 1.0f / (float)cols;
  Vec<W, V> w[N], b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = (i * tpr + lane) * V;
    w[i] = load_row<V>((const W*)a.w, at, cols);
    if (a.b) {
      b[i] = load_row<V>((const W*)a.b, at, cols);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) b[i].e[j] = (W)0.0f;
    }
  }
  Vec<T, V> nx[N];
  if (row < a.rows) {
#pragma unroll
    for (int i = 0; i < N; ++i) nx[i] = load_row<V>(x + row * a.x_stride, (i * tpr + lane) * V, cols);
  }
  for (; row < a.rows; row += step) {
    float f[N * V], s[1] = {0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        f[i * V + j] = to_f32(nx[i].e[j]);
        s[0] += f[i * V + j];
      }
    if (row + step < a.rows) {
#pragma unroll
      for (int i = 0; i < N; ++i) nx[i] = load_row<V>(x + (row + step) * a.x_stride, (i * tpr + lane) * V, cols);
    }
    row_sums<WAVE, 1>(s, lds, 0);
    const float mean = s[0] * inv;
    s[0] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float& d = f[i * V + j];
        d = (i * tpr + lane) * V + j < cols ? d - mean : 0.0f;
        s[0] += d * d;
      }
    row_sums<WAVE, 1>(s, lds, 1);
    const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
    if (lane == 0) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      Vec<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j)
        o.e[j] = from_f32<T>(f[i * V + j] * rstd * to_f32(w[i].e[j]) + to_f32(b[i].e[j]));
      store_row<V>(y + row * cols, (i * tpr + lane) * V, cols, o);
    }
  }
}

template <typename T, typename W, int N, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void ln_bwd(LnArgs a) {
  constexpr int V = kVec<T>;
  constexpr int RPB = WAVE ? 4 : 1;
  __shared__ float lds[2 * 2 * kMaxWaves];
  __shared__ float join[RPB > 1 ? (RPB - 1) * 64 * 2 : 1];
  const int tpr = WAVE ? 64 : blockDim.x, lane = WAVE ? threadIdx.x & 63 : threadIdx.x;
  const int sub = WAVE ? threadIdx.x >> 6 : 0, cols = a.cols;
  if (!WAVE) {
    if (threadIdx.x < 4 * kMaxWaves) lds[threadIdx.x] = 0;
    __syncthreads();
  }
  const int64_t step = (int64_t)gridDim.x * RPB;
  const T* x = (const T*)a.x;
  const T* dy = (const T*)a.dy;
  T* dx = (T*)a.dx;
  const float inv = 1.0f / (float)cols;
  Vec<W, V> w[N];
  float dw[N * V], db[N * V];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = load_row<V>((const W*)a.w, (i * tpr + lane) * V, cols);
#pragma unroll
  for (int i = 0; i < N * V; ++i) dw[i] = db[i] = 0;
  auto take = [&](int64_t row, int slot) {
    Vec<T, V> xv[N], dv[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      xv[i] = load_row<V>(x + row * a.x_stride, (i * tpr + lane) * V, cols);
      dv[i] = load_row<V>(dy + row * a.dy_stride, (i * tpr + lane) * V, cols);
    }
    const float mean = a.mean[row], rstd = a.rstd[row];
    float xh[N * V], g[N * V], s[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int k = i * V + j;
        // past the row's end dy is 0, so every sum is unaffected
        xh[k] = (to_f32(xv[i].e[j]) - mean) * rstd;
        const float d = to_f32(dv[i].e[j]);
        g[k] = d * to_f32(w[i].e[j]);
        dw[k] += d * xh[k];
        db[k] += d;
        s[0] += g[k];
        s[1] += g[k] * xh[k];
      }
    row_sums<WAVE, 2>(s, lds, slot);
    const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      Vec<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.e[j] = from_f32<T>(rstd * (g[i * V + j] - m0 - xh[i * V + j] * m1));
      store_row<V>(dx + row * cols, (i * tpr + lane) * V, cols, o);
    }
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  for (int slot = 0; row < a.rows; row += step, slot ^= 1) take(row, slot);
  float* pw = a.part + (int64_t)blockIdx.x * 2 * cols;
  if constexpr (RPB == 1) {
#pragma unroll
    for (int i = 0; i < N * V; ++i) {
      const int at = (i / V * tpr + lane) * V + i % V;
      if (at < cols) {
        pw[at] = dw[i];
        if (a.has_db) pw[cols + at] = db[i];
      }
    }
  } else {
    // the wavefronts' sums are added in their order
#pragma unroll
    for (int i = 0; i < N * V; ++i) {
      __syncthreads();
      if (sub) {
        join[(sub - 1) * 128 + lane] = dw[i];
        join[(sub - 1) * 128 + 64 + lane] = db[i];
      }
      __syncthreads();
      const int at = (i / V * tpr + lane) * V + i % V;
      if (sub == 0 && at < cols) {
        float u = dw[i], v = db[i];
#pragma unroll
        for (int k = 0; k < RPB - 1; ++k) {
          u += join[k * 128 + lane];
          v += join[k * 128 + 64 + lane];
        }
        pw[at] = u;
        if (a.has_db) pw[cols + at] = v;
      }
    }
  }
}

// dweight and dbias: the workgroups' sums, sixteen runs of them in turn and
// the runs' sums in their order.
template <typename W>
__global__ __launch_bounds__(1024) void ln_bwd_join(const float* part, int32_t n, int32_t cols, W* dw, W* db) {
  __shared__ float lds[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float s = 0;
  if (c < cols) {
    const float* p = part + (int64_t)blockIdx.y * cols + c;
    const int64_t pitch = 2 * (int64_t)cols;
#pragma unroll 8
    for (int i = w; i < n; i += 16) s += p[i * pitch];
  }
  lds[w][threadIdx.x & 63] = s;
  __syncthreads();
  if (w == 0 && c < cols) {
    float t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += lds[i][threadIdx.x];
    (blockIdx.y ? db : dw)[c] = from_f32<W>(t);
  }
}

// Threads and vectors per thread of a row of `vecs` 16-byte vectors.
struct LnShape {
  bool wave;
  int threads, n;  // of a workgroup, which has four rows at a time where a wavefront has one
};
LnShape ln_shape(const argus_layer_norm_t& p) {
  const int64_t vecs = ceil_div(p.cols, p.dtype == ARGUS_F32 ? 4 : 8);
  if (vecs <= 128) return {true, 256, (int)ceil_div(vecs, 64)};
  const int n = (int)ceil_div(vecs, 1024);
  return {false, (int)ceil_div(ceil_div(vecs, n), 64) * 64, n};
}

// Workgroups that take the rows in turn: `threads` of each CU (forward 32,768 x
// 4,096 bf16 with 2,048: 98.7 us, 1,536: 108, 8,192: 101). Those of one vector
// to a thread fit at once, but for the gradient's of f16 with 32-bit weights (82
// registers). Of more vectors registers admit fewer, and the rest begin as the
// first end: of the gradient's of 16-bit rows of 513 to 1,024 columns (129 to
// 132 registers) three workgroups fit a CU in place of six.
int64_t ln_grid(const argus_layer_norm_t& p, int64_t threads) {
  const LnShape s = ln_shape(p);
  const int64_t fit = threads / s.threads, most = 256 * (fit < 1 ? 1 : fit), need = ceil_div(p.rows, s.wave ? 4 : 1);
  return need < most ? need : most;
}

template <bool BWD>
hipError_t ln_launch(const argus_layer_norm_t& p, const LnArgs& a, int64_t grid, hipStream_t st) {
  const LnShape s = ln_shape(p);
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    auto by_weight = [&](auto wt) {
      using W = decltype(wt);
      auto go = [&](auto fwd, auto bwd) {
        hipLaunchKernelGGL(BWD ? bwd : fwd, dim3((unsigned)grid), dim3(s.threads), 0, st, a);
        return hipGetLastError();
      };
#define ARGUS_LN(N, WAVE) go(ln_fwd<T, W, N, WAVE>, ln_bwd<T, W, N, WAVE>)
      if (s.wave) return s.n == 1 ? ARGUS_LN(1, true) : ARGUS_LN(2, true);
      if (s.n == 1) return ARGUS_LN(1, false);
      if (s.n == 2) return ARGUS_LN(2, false);
      if constexpr (kVec<T> == 4) return s.n == 3 ? ARGUS_LN(3, false) : ARGUS_LN(4, false);  // up to 16,384 columns
#undef ARGUS_LN
      return hipErrorInvalidValue;
    };
    return p.weight_dtype == ARGUS_F32 ? by_weight(float{}) : by_weight(T{});
  });
}

}  // namespace

hipError_t launch_layer_norm(const argus_layer_norm_t& p, const void* x, const void* w, const void* b, void* y,
                             float* mean, float* rstd, hipStream_t st) {
  if (p.rows == 0) return hipSuccess;
  LnArgs a{p.rows, p.x_stride, 0, p.cols, p.eps, x, nullptr, w, b, y, nullptr, mean, rstd, nullptr, 0};
  return ln_launch<false>(p, a, ln_grid(p, 2048), st);
}

size_t layer_norm_bwd_workspace_bytes(const argus_layer_norm_t& p) {
  return align256((size_t)ln_grid(p, 1536) * 2 * (size_t)p.cols * sizeof(float));
}

hipError_t launch_layer_norm_bwd(const argus_layer_norm_t& p, const void* dy, const void* x, const float* mean,
                                 const float* rstd, const void* w, void* dx, void* dw, void* db, void* ws,
                                 hipStream_t st) {
  const int64_t grid = ln_grid(p, 1536);
  if (grid) {
    LnArgs a{p.rows, p.x_stride, p.dy_stride, p.cols, p.eps, x, dy, w, nullptr, nullptr, dx,
             const_cast<float*>(mean), const_cast<float*>(rstd), (float*)ws, db != nullptr};
    const hipError_t e = ln_launch<true>(p, a, grid, st);
    if (e != hipSuccess) return e;
  }
  return with_dtype(p.weight_dtype, [&](auto t) {
    using W = decltype(t);
    hipLaunchKernelGGL(ln_bwd_join<W>, dim3((unsigned)ceil_div(p.cols, 64), db ? 2 : 1), dim3(1024), 0, st,
                       (const float*)ws, (int32_t)grid, p.cols, (W*)dw, (W*)db);
    return hipGetLastError();
  });
}

}  // namespace argus
