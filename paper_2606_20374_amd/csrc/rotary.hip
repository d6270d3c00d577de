// Rotary positions: pairs of a head's elements turned by position times
// frequency, in either direction.
//
// The angle is taken in turns, position * frequency / 2 pi, in 64 bits, and
// only its fraction goes on in 32: at position 10^6 an angle in 32 bits would
// be off by 0.06. A workgroup makes the sines and cosines of its tokens' pairs
// once, in LDS, and uses them for all of the tokens' heads. Bound by memory.
#include "ops_internal.h"

namespace argus {
namespace {

constexpr int kThreads = 256;
constexpr int kPairs = 1024;  // sines and cosines that fit a workgroup's LDS

struct RotaryArgs {
  const void *x, *pos;
  void* out;
  const double* freq;
  int64_t n_tokens, x_tok, x_head, out_tok, out_head;
  int32_t heads, dim, pairs, pos_64, tokens;  // tokens of a workgroup
  float scale, sign;
};

template <typename T, bool NEIGHBOURS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 turn[kPairs];
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
  const int n = (int)(a.n_tokens - t0 < a.tokens ? a.n_tokens - t0 : a.tokens);
  for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
    const int t = i / a.pairs, p = i - t * a.pairs;
    const int64_t at = t0 + t;
    const double pos = !a.pos ? (double)at : a.pos_64 ? (double)((const int64_t*)a.pos)[at] : (double)((const int32_t*)a.pos)[at];
    double turns = pos * (a.freq[p] * 0.15915494309189535);
    turns -= rint(turns);
    float s, c;
    sincospif((float)(2.0 * turns), &s, &c);
    turn[i] = make_float2(c * a.scale, s * a.scale * a.sign);
  }
  __syncthreads();
  // elements of a head: pairs first, then what is only copied
  const int rest = a.dim - 2 * a.pairs, per = a.pairs + rest;
  for (int64_t i = threadIdx.x; i < (int64_t)n * a.heads * per; i += kThreads) {
    const int64_t row = i / per;
    const int e = (int)(i - row * per), t = (int)(row / a.heads), h = (int)(row - (int64_t)t * a.heads);
    const T* x = (const T*)a.x + (t0 + t) * a.x_tok + h * a.x_head;
    T* out = (T*)a.out + (t0 + t) * a.out_tok + h * a.out_head;
    if (e >= a.pairs) {
      out[e + a.pairs] = x[e + a.pairs];
      continue;
    }
    const float2 cs = turn[t * a.pairs + e];
    const int i0 = NEIGHBOURS ? 2 * e : e, i1 = NEIGHBOURS ? 2 * e + 1 : e + a.pairs;
    const float u = to_f32(x[i0]), v = to_f32(x[i1]);
    out[i0] = from_f32<T>(u * cs.x - v * cs.y);
    out[i1] = from_f32<T>(u * cs.y + v * cs.x);
  }
}

}  // namespace

hipError_t launch_rotary(const argus_rotary_t& p, const void* x, void* out, hipStream_t st) {
  if (p.n_tokens == 0 || p.n_heads == 0) return hipSuccess;
  RotaryArgs a{x, p.pos, out, p.freq, p.n_tokens, p.x_tok, p.x_head, p.out_tok, p.out_head,
               p.n_heads, p.head_dim, p.rot_dim / 2, p.pos_64, 1, p.scale, p.inverse ? -1.0f : 1.0f};
  a.tokens = kPairs / a.pairs < 16 ? kPairs / a.pairs : 16;
  const unsigned grid = (unsigned)ceil_div(p.n_tokens, a.tokens);
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    if (p.interleaved) hipLaunchKernelGGL((rotary_kernel<T, true>), dim3(grid), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((rotary_kernel<T, false>), dim3(grid), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  });
}

}  // namespace argus
