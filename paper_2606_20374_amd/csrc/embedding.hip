// Token embedding and the gradient of its table.
//
// Forward: out[t] = scale * table[ids[t]], a gather of rows; 16-byte vectors,
// as many lanes to a token as its row has vectors (at most a workgroup). The
// product is a 32-bit float in every type, then rounded.
//
// Backward: dtable[v] = scale * sum of dout[t] over ids[t] = v. The token
// numbers are sorted by id, equal ids in token order, so the sums need no
// floating-point atomics and have a fixed order; every row of dtable is then
// written once by the lanes that own it, zeros for ids that do not occur.
//   sort    up to kRankMax tokens: each token's place is counted against all
//           others (one launch). More: radix sort, 8 bits a pass, at most
//           kSortBlocks workgroups, two launches a pass (counts per workgroup
//           and digit; places from the counts of the workgroups before).
//   pieces  ids that occur more than 2 * kPiece times are summed by pieces of
//           kPiece sorted positions in 32 bits, so that a frequent token's
//           rows are read by many workgroups.
//   rows    kRowsPer table rows to a workgroup: their ranges in the sorted
//           order by binary search, then the sums (of rows, or of pieces).
// Bound by memory: dout is read once (and the pieces' sums, 1/kPiece of it in
// 32 bits, written and read), dtable written once.
#include "ops_internal.h"

namespace argus {
namespace {

constexpr int kRankMax = 1024;    // tokens that are ranked by counting
constexpr int kSortBlocks = 128;  // workgroups of a radix pass
constexpr int kPiece = 64;        // sorted positions of a piece
constexpr int kRowsPer = 16;      // table rows of a workgroup
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups of a lookup

template <typename T>
constexpr int kVec = 16 / sizeof(T);

__device__ __forceinline__ uint32_t key_of(const void* ids, int64_t t, int ids_64, int32_t V) {
  const int64_t id = ids_64 ? ((const int64_t*)ids)[t] : (int64_t)((const int32_t*)ids)[t];
  return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
}

// The 32-bit product, then rounded: in half precision one instruction would do
// both and skip the product's own rounding, and types would differ in that.
template <typename T>
__device__ __forceinline__ T scaled(float v, float scale) {
  float p = v * scale;
  asm("" : "+v"(p));
  return from_f32<T>(p);
}

template <typename T>
__global__ __launch_bounds__(256) void emb_fwd(const void* ids, int64_t n, int32_t ids_64, int32_t V, int32_t dim,
                                               int64_t stride, float scale, const T* table, T* out, int32_t tpr,
                                               int32_t* dev_status) {
  constexpr int E = kVec<T>;
  const int lane = threadIdx.x % tpr;
  const int64_t step = (int64_t)gridDim.x * (256 / tpr);
  for (int64_t t = (int64_t)blockIdx.x * (256 / tpr) + threadIdx.x / tpr; t < n; t += step) {
    const int64_t id = ids_64 ? ((const int64_t*)ids)[t] : (int64_t)((const int32_t*)ids)[t];
    if (id >= V && lane == 0 && dev_status) atomicOr(dev_status, (int32_t)ARGUS_DEV_TOKEN_RANGE);
    const bool ok = id >= 0 && id < V;
    const T* row = table + (ok ? id : 0) * stride;
    T* o = out + t * dim;
    for (int64_t i = lane * E; i < dim; i += tpr * E) {
      Vec<T, E> v = {};
      if (ok) {
        v = load_row<E>(row, (int)i, dim);
#pragma unroll
        for (int j = 0; j < E; ++j) v.e[j] = scaled<T>(to_f32(v.e[j]), scale);
      }
      store_row<E>(o, (int)i, dim, v);
    }
  }
}

// ------------------------------------------------------------------- sorting
// Sorted position of each of n <= kRankMax tokens: how many (id, token) pairs
// are below its own. 64 tokens to a workgroup, a quarter of the others to
// each of its wavefronts.
__global__ __launch_bounds__(256) void emb_rank(const void* ids, int32_t n, int32_t ids_64, int32_t V, uint32_t* skey,
                                                uint32_t* stok, int32_t* dev_status) {
  __shared__ uint32_t key[kRankMax];
  __shared__ int part[4][64];
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < kRankMax; i += 256) {
    uint32_t k = ~0u;
    if (i < n) {
      k = key_of(ids, i, ids_64, V);
      const int64_t id = ids_64 ? ((const int64_t*)ids)[i] : (int64_t)((const int32_t*)ids)[i];
      if (id >= V) bad = 1;
    }
    key[i] = k;
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, me = blockIdx.x * 64 + lane;
  const uint32_t mine = me < n ? key[me] : ~0u;
  const int per = (n + 3) / 4, lo = w * per, hi = min(n, lo + per);
  int c = 0;
  for (int j = lo; j < hi; ++j) {
    const uint32_t k = key[j];
    c += k < mine || (k == mine && j < me);
  }
  part[w][lane] = c;
  __syncthreads();
  if (w == 0 && me < n) {
    const int at = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
    skey[at] = mine;
    stok[at] = me;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0 && dev_status) *dev_status = bad ? (int32_t)ARGUS_DEV_TOKEN_RANGE : 0;
}

struct SortArgs {
  const void* ids;       // first pass: the ids themselves
  const uint32_t* key;   // later passes
  const uint32_t* tok;
  uint32_t *okey, *otok;
  uint32_t* hist;        // [workgroups][256]
  int32_t n, per, ids_64, V, shift;  // per: tokens of a workgroup, a multiple of 256
  int32_t* dev_status;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int i) {
  return a.ids ? key_of(a.ids, i, a.ids_64, a.V) : a.key[i];
}

__global__ __launch_bounds__(256) void emb_count(SortArgs a) {
  __shared__ uint32_t h[256];
  h[threadIdx.x] = 0;
  __syncthreads();
  const int lo = blockIdx.x * a.per, hi = min(a.n, lo + a.per);
  for (int i = lo + threadIdx.x; i < hi; i += 256) {
    atomicAdd(&h[(sort_key(a, i) >> a.shift) & 255], 1u);
    if (a.ids && a.dev_status) {
      const int64_t id = a.ids_64 ? ((const int64_t*)a.ids)[i] : (int64_t)((const int32_t*)a.ids)[i];
      if (id >= a.V) atomicOr(a.dev_status, (int32_t)ARGUS_DEV_TOKEN_RANGE);
    }
  }
  __syncthreads();
  a.hist[blockIdx.x * 256 + threadIdx.x] = h[threadIdx.x];
}

// Exclusive sum over the 256 threads.
__device__ __forceinline__ uint32_t scan256(uint32_t v, uint32_t* lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) lds[w] = s;
  __syncthreads();
  uint32_t before = 0;
  for (int i = 0; i < w; ++i) before += lds[i];
  return before + s - v;
}

__global__ __launch_bounds__(256) void emb_scatter(SortArgs a) {
  __shared__ uint32_t next[256];     // where the next token of each digit goes
  __shared__ uint32_t cnt[4][256];   // this round's tokens of each wavefront and digit
  __shared__ uint32_t lds[4];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, b = blockIdx.x;
  uint32_t before = 0, total = 0;
  for (int i = 0; i < (int)gridDim.x; ++i) {
    const uint32_t h = a.hist[i * 256 + tid];
    if (i < b) before += h;
    total += h;
  }
  next[tid] = before + scan256(total, lds);
  const int lo = b * a.per, hi = min(a.n, lo + a.per);
  for (int base = lo; base < hi; base += 256) {
#pragma unroll
    for (int i = 0; i < 4; ++i) cnt[i][tid] = 0;
    __syncthreads();
    const int i = base + tid;
    const bool on = i < hi;
    const uint32_t k = on ? sort_key(a, i) : 0, d = (k >> a.shift) & 255;
    const uint32_t tok = on ? (a.ids ? (uint32_t)i : a.tok[i]) : 0;
    // lanes of this wavefront with the same digit
    uint64_t same = __ballot(on);
#pragma unroll
    for (int bit = 0; bit < 8; ++bit) {
      const uint64_t m = __ballot((d >> bit) & 1);
      same &= (d >> bit) & 1 ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (on && rank == 0) cnt[w][d] = __popcll(same);
    __syncthreads();
    uint32_t at = rank;
    if (on) {
      at += next[d];
      for (int i2 = 0; i2 < w; ++i2) at += cnt[i2][d];
    }
    __syncthreads();
    next[tid] += cnt[0][tid] + cnt[1][tid] + cnt[2][tid] + cnt[3][tid];
    if (on) {
      a.okey[at] = k;
      a.otok[at] = tok;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------- sums
struct SumArgs {
  const uint32_t *skey, *stok;
  int32_t n, V, dim, tpr;
  int64_t stride;
  float scale;
  float* piece;  // [pieces][2][dim]: the run at a piece's left edge (or all of it), at its right edge
};

// Adds dout rows [lo, hi) of the sorted order to the E columns at c.
template <typename T>
__device__ __forceinline__ void add_rows(const SumArgs& a, const T* dout, int lo, int hi, int step, int c,
                                         float (&acc)[kVec<T>]) {
  constexpr int E = kVec<T>;
  int i = lo;
  for (; i + 3 * step < hi; i += 4 * step) {
    Vec<T, E> v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = load_row<E>(dout + (int64_t)a.stok[i + u * step] * a.stride, c, a.dim);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] += to_f32(v[u].e[j]);
  }
  for (; i < hi; i += step) {
    const Vec<T, E> v = load_row<E>(dout + (int64_t)a.stok[i] * a.stride, c, a.dim);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] += to_f32(v.e[j]);
  }
}

// First sorted position whose key is at least k.
__device__ __forceinline__ int lower_bound(const uint32_t* skey, int n, uint32_t k) {
  int lo = 0, len = n;
  while (len > 0) {
    const int half = len >> 1;
    if (skey[lo + half] < k) {
      lo += half + 1;
      len -= half + 1;
    } else {
      len = half;
    }
  }
  return lo;
}

// The sums of a piece's runs that belong to an id of more than 2 * kPiece
// tokens. Such an id's run touches an edge of every piece it is in.
template <typename T>
__global__ __launch_bounds__(256) void emb_pieces(SumArgs a, const T* dout) {
  constexpr int E = kVec<T>;
  __shared__ float lds[256][E + 1];
  const int first = blockIdx.x * kPiece, last = min(a.n, first + kPiece) - 1;
  const uint32_t ka = a.skey[first], kb = a.skey[last];
  const int tpr = a.tpr, lane = threadIdx.x % tpr, sub = threadIdx.x / tpr, groups = 256 / tpr;
  const int c = (blockIdx.y * tpr + lane) * E;
  for (int side = 0; side < 2; ++side) {
    int lo = first, hi = last + 1;
    bool heavy;
    if (ka == kb) {
      if (side) break;
      // the whole piece: a longer run goes on to one side or the other
      heavy = ka < (uint32_t)a.V && ((first > 0 && a.skey[first - 1] == ka) || (hi < a.n && a.skey[hi] == ka));
    } else if (side == 0) {
      hi = first + lower_bound(a.skey + first, last + 1 - first, ka + 1);
      heavy = hi - 1 - 2 * kPiece >= 0 && a.skey[hi - 1 - 2 * kPiece] == ka;  // ka < kb <= V
    } else {
      lo = first + lower_bound(a.skey + first, last + 1 - first, kb);
      heavy = kb < (uint32_t)a.V && lo + 2 * kPiece < a.n && a.skey[lo + 2 * kPiece] == kb;
    }
    if (!heavy) continue;  // uniform over the workgroup
    float acc[E] = {};
    if (c < a.dim) add_rows(a, dout, lo + sub, hi, groups, c, acc);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < E; ++j) lds[threadIdx.x][j] = acc[j];
    __syncthreads();
    if (sub == 0 && c < a.dim) {
      for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += lds[g * tpr + lane][j];
      float* o = a.piece + ((int64_t)blockIdx.x * 2 + side) * a.dim;
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c + j < a.dim) o[c + j] = acc[j];
    }
  }
}

template <typename T, typename G>
__global__ __launch_bounds__(256) void emb_rows(SumArgs a, const T* dout, G* dtable) {
  constexpr int E = kVec<T>;
  __shared__ int start[kRowsPer + 1];
  const int64_t r0 = (int64_t)blockIdx.x * kRowsPer;
  const int rows = (int)(a.V - r0 < kRowsPer ? a.V - r0 : kRowsPer);
  if ((int)threadIdx.x <= rows) start[threadIdx.x] = lower_bound(a.skey, a.n, (uint32_t)(r0 + threadIdx.x));
  __syncthreads();
  const int tpr = a.tpr, lane = threadIdx.x % tpr, sub = threadIdx.x / tpr, groups = 256 / tpr;
  const int c = (blockIdx.y * tpr + lane) * E;
  if (c >= a.dim) return;
  for (int r = sub; r < rows; r += groups) {
    const int s = start[r], e = start[r + 1];
    float acc[E] = {};
    if (e - s <= 2 * kPiece) {
      add_rows(a, dout, s, e, 1, c, acc);
    } else {
      for (int p = s / kPiece; p <= (e - 1) / kPiece; ++p) {
        // the id's run lies at the right edge of the first piece unless it fills it
        const int side = p == s / kPiece && s % kPiece != 0 ? 1 : 0;
        const Vec<float, E> v = load_row<E>(a.piece + ((int64_t)p * 2 + side) * a.dim, c, a.dim);
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += v.e[j];
      }
    }
    Vec<G, E> o;
#pragma unroll
    for (int j = 0; j < E; ++j) o.e[j] = scaled<G>(acc[j], a.scale);
    store_row<E>(dtable + (r0 + r) * a.dim, c, a.dim, o);
  }
}

// Lanes of a row: a power of two that covers its vectors, 8 to 256.
int lanes_of(int64_t vecs) {
  int t = 8;
  while (t < vecs && t < 256) t *= 2;
  return t;
}

struct BwdLayout {
  size_t key[2], tok[2], hist, piece, total;
};
BwdLayout bwd_layout(const argus_embedding_t& p) {
  BwdLayout l;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += align256(n); return o; };
  const size_t n = (size_t)p.n_tokens;
  l.key[0] = take(4 * n);
  l.tok[0] = take(4 * n);
  const bool sorted = p.n_tokens > kRankMax;
  l.key[1] = take(sorted ? 4 * n : 0);
  l.tok[1] = take(sorted ? 4 * n : 0);
  l.hist = take(sorted ? kSortBlocks * 256 * 4 : 0);
  l.piece = take(p.n_tokens > 2 * kPiece ? (size_t)ceil_div(p.n_tokens, kPiece) * 2 * (size_t)p.dim * 4 : 0);
  l.total = at;
  return l;
}

}  // namespace

hipError_t launch_embedding(const argus_embedding_t& p, const void* table, void* out, hipStream_t st) {
  if (p.dev_status) {
    const hipError_t e = launch_clear(p.dev_status, nullptr, st);
    if (e != hipSuccess) return e;
  }
  if (p.n_tokens == 0) return hipSuccess;
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    const int tpr = lanes_of(ceil_div(p.dim, kVec<T>));
    const int64_t need = ceil_div(p.n_tokens, 256 / tpr), grid = need < kMaxGrid ? need : kMaxGrid;
    hipLaunchKernelGGL(emb_fwd<T>, dim3((unsigned)grid), dim3(256), 0, st, p.ids,
                       p.n_tokens, p.ids_64, p.n_vocab, p.dim, p.row_stride, p.scale, (const T*)table, (T*)out, tpr,
                       p.dev_status);
    return hipGetLastError();
  });
}

size_t embedding_bwd_workspace_bytes(const argus_embedding_t& p) { return bwd_layout(p).total; }

hipError_t launch_embedding_bwd(const argus_embedding_t& p, const void* dout, void* dtable, void* ws, hipStream_t st) {
  const BwdLayout l = bwd_layout(p);
  uint8_t* base = (uint8_t*)ws;
  uint32_t *key[2], *tok[2];
  for (int i = 0; i < 2; ++i) {
    key[i] = (uint32_t*)(base + l.key[i]);
    tok[i] = (uint32_t*)(base + l.tok[i]);
  }
  const int32_t n = (int32_t)p.n_tokens;
  int cur = 0;
  hipError_t e;
  if (n <= kRankMax) {
    // at least one workgroup, which also sets the status word
    hipLaunchKernelGGL(emb_rank, dim3(n ? (unsigned)ceil_div(n, 64) : 1), dim3(256), 0, st, p.ids, n, p.ids_64,
                       p.n_vocab, key[0], tok[0], p.dev_status);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    if (p.dev_status && (e = launch_clear(p.dev_status, nullptr, st)) != hipSuccess) return e;
    const int32_t per = (int32_t)(ceil_div(ceil_div(n, kSortBlocks), 1024) * 1024);
    const unsigned blocks = (unsigned)ceil_div(n, per);
    for (int shift = 0; shift == 0 || ((uint32_t)p.n_vocab >> shift) != 0; shift += 8) {  // keys are 0 .. n_vocab
      SortArgs a{shift ? nullptr : p.ids, key[cur], tok[cur], key[cur ^ 1], tok[cur ^ 1],
                 (uint32_t*)(base + l.hist), n, per, p.ids_64, p.n_vocab, shift, shift ? nullptr : p.dev_status};
      hipLaunchKernelGGL(emb_count, dim3(blocks), dim3(256), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(emb_scatter, dim3(blocks), dim3(256), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      cur ^= 1;
    }
  }
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t vecs = ceil_div(p.dim, kVec<T>);
    const int tpr = lanes_of(vecs);
    const unsigned cb = (unsigned)ceil_div(vecs, tpr);
    SumArgs a{key[cur], tok[cur], n, p.n_vocab, p.dim, tpr, p.row_stride, p.scale, (float*)(base + l.piece)};
    if (n > 2 * kPiece) {
      hipLaunchKernelGGL(emb_pieces<T>, dim3((unsigned)ceil_div(n, kPiece), cb), dim3(256), 0, st, a, (const T*)dout);
      const hipError_t e2 = hipGetLastError();
      if (e2 != hipSuccess) return e2;
    }
    auto rows = [&](auto g) {
      using G = decltype(g);
      hipLaunchKernelGGL((emb_rows<T, G>), dim3((unsigned)ceil_div(p.n_vocab, kRowsPer), cb), dim3(256), 0, st, a,
                         (const T*)dout, (G*)dtable);
      return hipGetLastError();
    };
    return p.grad_dtype == ARGUS_F32 ? rows(float{}) : rows(T{});
  });
}

}  // namespace argus
