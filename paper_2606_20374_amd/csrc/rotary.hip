// Rotary positions: pairs of a head's elements turned by position times
// frequency, in either direction.
//
// The angle is taken in turns, position * frequency / 2 pi, in 64 bits, and
// only its fraction goes on in 32: at position 10^6 an angle in 32 bits would
// be off by 0.06. A workgroup makes the sines and cosines of its tokens' pairs
// once, in LDS, and uses them for all of the tokens' heads.
// Bound by memory: a thread takes 16 bytes (with the halves' layout 16 of each
// half), whatever the alignment, and writes past the caches. 65,536 tokens, 40
// heads of 128, bf16: 231 us, 5.8 TB/s (an element to a thread: 597); 20,011
// tokens, 24 heads of 96 of which 32 turn, f16: 45 us, 4.1 TB/s.
#include <type_traits>

#include "ops_internal.h"

namespace argus {
namespace {

constexpr int kThreads = 256;
constexpr int kTurns = 2048;   // sines and cosines that fit a workgroup's LDS
// Pieces that a workgroup takes where there are enough tokens (1,024: 252 us in the
// place of 232, 61 of 54; 256: 247 and 52).
constexpr int kItems = 512;
constexpr int kGroups = 1024;  // workgroups below which it takes fewer
constexpr int64_t kMaxGrid = 1 << 20;

struct RotaryArgs {
  const void *x, *pos;
  void* out;
  const double* freq;
  int64_t n_tokens, x_tok, x_head, out_tok, out_head;
  int32_t heads, dim, pairs, pos_64, tokens;  // tokens of a workgroup
  float scale, sign;
};

// Pieces of N elements of a head: of what is turned, then of what is copied.
template <int N, bool NEIGHBOURS>
__host__ __device__ __forceinline__ int turned_pieces(int pairs) { return ((NEIGHBOURS ? 2 * pairs : pairs) + N - 1) / N; }
template <int N>
__host__ __device__ __forceinline__ int copied_pieces(int rest) { return (rest + N - 1) / N; }

template <typename T, int N, bool NEIGHBOURS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ __align__(16) float2 turn[kTurns];
  const int turned = turned_pieces<N, NEIGHBOURS>(a.pairs), per = turned + copied_pieces<N>(a.dim - 2 * a.pairs);
  for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.n_tokens; t0 += (int64_t)gridDim.x * a.tokens) {
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
    const uint32_t all = (uint32_t)n * a.heads * per;  // below 2^25: kItems and one token's at most
    for (uint32_t i = threadIdx.x; i < all; i += kThreads) {
      const uint32_t row = i / (uint32_t)per, t = row / (uint32_t)a.heads;
      const int piece = (int)(i - row * per);
      const int64_t h = row - t * a.heads;
      const T* x = (const T*)a.x + (t0 + t) * a.x_tok + h * a.x_head;
      T* out = (T*)a.out + (t0 + t) * a.out_tok + h * a.out_head;
      const float2* cs = turn + t * a.pairs;
      if (piece >= turned) {
        const int e = (piece - turned) * N;
        x += 2 * a.pairs;
        stream_row<N>(out + 2 * a.pairs, e, a.dim - 2 * a.pairs, load_row<N>(x, e, a.dim - 2 * a.pairs));
      } else if constexpr (NEIGHBOURS) {
        const int e = piece * N;
        Vec<T, N> v = load_row<N>(x, e, 2 * a.pairs);
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          const float2 f = cs[e / 2 + j / 2 < a.pairs ? e / 2 + j / 2 : 0];
          const float p = to_f32(v.e[j]), q = to_f32(v.e[j + 1]);
          v.e[j] = from_f32<T>(p * f.x - q * f.y);
          v.e[j + 1] = from_f32<T>(p * f.y + q * f.x);
        }
        stream_row<N>(out, e, 2 * a.pairs, v);
      } else {
        const int e = piece * N;
        Vec<T, N> u = load_row<N>(x, e, a.pairs), v = load_row<N>(x + a.pairs, e, a.pairs);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float2 f = cs[e + j < a.pairs ? e + j : 0];
          const float p = to_f32(u.e[j]), q = to_f32(v.e[j]);
          u.e[j] = from_f32<T>(p * f.x - q * f.y);
          v.e[j] = from_f32<T>(p * f.y + q * f.x);
        }
        stream_row<N>(out, e, a.pairs, u);
        stream_row<N>(out + a.pairs, e, a.pairs, v);
      }
    }
    __syncthreads();  // the next tokens' turns take the place of these
  }
}

}  // namespace

hipError_t launch_rotary(const argus_rotary_t& p, const void* x, void* out, hipStream_t st) {
  if (p.n_tokens == 0) return hipSuccess;
  RotaryArgs a{x, p.pos, out, p.freq, p.n_tokens, p.x_tok, p.x_head, p.out_tok, p.out_head,
               p.n_heads, p.head_dim, p.rot_dim / 2, p.pos_64, 1, p.scale, p.inverse ? -1.0f : 1.0f};
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int kWide = 16 / sizeof(T);
    auto go = [&](auto n, auto neighbours) {
      constexpr int N = n;
      constexpr bool NEIGHBOURS = neighbours;
      const int64_t pieces = (int64_t)p.n_heads * (turned_pieces<N, NEIGHBOURS>(a.pairs) + copied_pieces<N>(p.head_dim - p.rot_dim));
      int64_t tokens = ceil_div(kItems, pieces);
      if (tokens > kTurns / a.pairs) tokens = kTurns / a.pairs;
      if (tokens > ceil_div(p.n_tokens, kGroups)) tokens = ceil_div(p.n_tokens, kGroups);
      a.tokens = (int32_t)tokens;
      const int64_t need = ceil_div(p.n_tokens, tokens);
      hipLaunchKernelGGL((rotary_kernel<T, N, NEIGHBOURS>), dim3((unsigned)(need < kMaxGrid ? need : kMaxGrid)),
                         dim3(kThreads), 0, st, a);
      return hipGetLastError();
    };
    using std::integral_constant;
    auto with = [&](auto neighbours) {
      // half a vector where that leaves no piece across a row's end, which is
      // taken element by element (30,000 tokens, 20 heads of 40: 27 us for 51)
      const int run = neighbours ? p.rot_dim : a.pairs, rest = p.head_dim - p.rot_dim;
      const bool half = (run % kWide || rest % kWide) && run % (kWide / 2) == 0 && rest % (kWide / 2) == 0;
      return half ? go(integral_constant<int, kWide / 2>{}, neighbours) : go(integral_constant<int, kWide>{}, neighbours);
    };
    return p.interleaved ? with(std::true_type{}) : with(std::false_type{});
  });
}

}  // namespace argus
