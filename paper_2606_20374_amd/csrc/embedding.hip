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
//           others (one launch). More: radix sort, 9 bits a pass, at most
//           kSortBlocks workgroups, two launches a pass (counts per workgroup
//           and digit; places from the counts of the workgroups before).
//   pieces  ids that occur more than 2 * kPiece times are summed by pieces of
//           kPiece sorted positions in 32 bits, so that a frequent token's
//           rows are read by many workgroups.
//   sums    workgroups take kWindow sorted positions each: the runs of equal
//           ids that begin there are summed (rows, or pieces) and written.
//           Further workgroups, of this launch and of the pieces', take
//           kFillRows table rows each and write zeros where no token was
//           counted: they begin while the last sums end (alternating with
//           the sums' from the start was slower, 311 us for 292).
// Bound by memory: dout is read once (and the pieces' sums, 1/kPiece of it in
// 32 bits, written and read), dtable written once. At 32,768 Zipf-distributed
// tokens, 128,000 x 4,096 bf16: 292 us, 4.5 TB/s; of it the sort 20, the sums
// without the zeros 111, the zeros (1.0 GB) the rest. The lookup of 65,536
// tokens: 131 us; plain stores in place of streaming ones 175 us.
#include "ops_internal.h"

namespace argus {
namespace {

constexpr int kRankMax = 1024;    // tokens that are ranked by counting
constexpr int kSortBlocks = 128;  // workgroups of a radix pass
constexpr int kPiece = 64;        // sorted positions of a piece, at most a wavefront's lanes
constexpr int kWindow = 32;       // sorted positions whose runs a workgroup sums
constexpr int kFillRows = 32;     // table rows of a workgroup that writes zeros
constexpr int kPieceMin = 4 * kPiece;  // tokens from which on frequent ids are summed by pieces
constexpr int kBits = 9, kDigits = 1 << kBits;  // of a radix pass
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups of a lookup

template <typename T>
constexpr int kVec = 16 / sizeof(T);

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

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
  constexpr int E = kVec<T>, U = 2;  // vectors of a row in flight
  const int lane = threadIdx.x % tpr;
  const int64_t step = (int64_t)gridDim.x * (256 / tpr);
  for (int64_t t = (int64_t)blockIdx.x * (256 / tpr) + threadIdx.x / tpr; t < n; t += step) {
    const int64_t id = ids_64 ? ((const int64_t*)ids)[t] : (int64_t)((const int32_t*)ids)[t];
    if (id >= V && lane == 0 && dev_status) atomicOr(dev_status, (int32_t)ARGUS_DEV_TOKEN_RANGE);
    const bool ok = id >= 0 && id < V;
    const T* row = table + (ok ? id : 0) * stride;
    T* o = out + t * dim;
    for (int64_t i = lane * E; i < dim; i += U * tpr * E) {
      Vec<T, E> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u] = Vec<T, E>{};
        if (ok && i + u * tpr * E < dim) v[u] = load_row<E>(row, (int)(i + u * tpr * E), dim);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[u].e[j] = ok ? scaled<T>(to_f32(v[u].e[j]), scale) : (T)0.0f;
        if (i + u * tpr * E < dim) stream_row<E>(o, (int)(i + u * tpr * E), dim, v[u]);
      }
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
  uint32_t* hist;        // [workgroups][kDigits]
  int32_t n, per, ids_64, V, shift;  // per: tokens of a workgroup, a multiple of 512
  uint8_t* seen;         // [V] first pass: set where a token is counted
  int32_t* dev_status;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int i) {
  return a.ids ? key_of(a.ids, i, a.ids_64, a.V) : a.key[i];
}

// Clears the table's marks (whole words: the buffer is padded) and the status.
__global__ __launch_bounds__(256) void emb_clear(u32x4_t* seen, int32_t words, int32_t* dev_status) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < words) seen[i] = u32x4_t{0, 0, 0, 0};
  if (i == 0 && dev_status) *dev_status = 0;
}

__global__ __launch_bounds__(kDigits) void emb_count(SortArgs a) {
  __shared__ uint32_t h[kDigits];
  h[threadIdx.x] = 0;
  __syncthreads();
  const int lo = blockIdx.x * a.per, hi = min(a.n, lo + a.per);
  for (int i = lo + threadIdx.x; i < hi; i += kDigits) {
    const uint32_t k = sort_key(a, i);
    atomicAdd(&h[(k >> a.shift) & (kDigits - 1)], 1u);
    if (a.ids) {
      if (k < (uint32_t)a.V) a.seen[k] = 1;
      const int64_t id = a.ids_64 ? ((const int64_t*)a.ids)[i] : (int64_t)((const int32_t*)a.ids)[i];
      if (id >= a.V && a.dev_status) atomicOr(a.dev_status, (int32_t)ARGUS_DEV_TOKEN_RANGE);
    }
  }
  __syncthreads();
  a.hist[blockIdx.x * kDigits + threadIdx.x] = h[threadIdx.x];
}

__global__ __launch_bounds__(kDigits) void emb_scatter(SortArgs a) {
  constexpr int W = kDigits / 64;
  __shared__ uint32_t next[kDigits];   // where the next token of each digit goes
  __shared__ uint32_t cnt[W][kDigits]; // this round's tokens of each wavefront and digit
  __shared__ uint32_t lds[W];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, b = blockIdx.x;
  const int lo = b * a.per, hi = min(a.n, lo + a.per);
  // the first round's tokens are on their way while the counts are added
  uint32_t nk = 0, nt = 0;
  auto fetch = [&](int base) {
    const int i = base + tid;
    if (i < hi) {
      nk = sort_key(a, i);
      nt = a.ids ? (uint32_t)i : a.tok[i];
    }
  };
  fetch(lo);
  uint32_t before = 0, total = 0;
#pragma unroll 16
  for (int i = 0; i < (int)gridDim.x; ++i) {
    const uint32_t h = a.hist[i * kDigits + tid];
    if (i < b) before += h;
    total += h;
  }
  uint32_t s = total;  // exclusive sum over the digits
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) lds[w] = s;
  __syncthreads();
  for (int i = 0; i < w; ++i) s += lds[i];
  next[tid] = before + s - total;
  for (int base = lo; base < hi; base += kDigits) {
#pragma unroll
    for (int i = 0; i < W; ++i) cnt[i][tid] = 0;
    __syncthreads();
    const bool on = base + tid < hi;
    const uint32_t k = nk, tok = nt, d = on ? (k >> a.shift) & (kDigits - 1) : 0;
    fetch(base + kDigits);
    // lanes of this wavefront with the same digit
    uint64_t same = __ballot(on);
#pragma unroll
    for (int bit = 0; bit < kBits; ++bit) {
      const uint64_t m = __ballot((d >> bit) & 1);
      same &= (d >> bit) & 1 ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (on && rank == 0) cnt[w][d] = __popcll(same);
    __syncthreads();
    uint32_t at = rank;
    if (on) {
      at += next[d];
      for (int i = 0; i < w; ++i) at += cnt[i][d];
    }
    __syncthreads();
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) sum += cnt[i][tid];
    next[tid] += sum;
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
  const uint8_t* seen;  // [V], or null: the few sorted keys are looked through
  int32_t work, cols;   // workgroups that sum, before those that write zeros; pieces of a row's columns
  int64_t fill0;        // first table row of the launch's zeros
};

// The vector at column c of a row, c a multiple of E below dim. `whole`: dim
// is a multiple of E, so no vector lies across a row's end and the load needs
// no branch.
template <int E, typename T>
__device__ __forceinline__ Vec<T, E> load_col(const T* row, int c, int dim, bool whole) {
  return whole ? load_vec<E>(row + c) : load_row<E>(row, c, dim);
}

// Adds the dout rows of tokens tok[lo], tok[lo + step], .. below hi to the E
// columns at c, eight of them in flight.
template <typename T>
__device__ __forceinline__ void add_rows(const SumArgs& a, const T* dout, const uint32_t* tok, int lo, int hi, int step,
                                         int c, float (&acc)[kVec<T>]) {
  constexpr int E = kVec<T>, U = 8;
  auto all = [&](bool whole) {
    for (int i = lo; i < hi; i += U * step) {
      Vec<T, E> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)  // past the end the first row again, which is not added
        v[u] = load_col<E>(dout + (int64_t)tok[i + u * step < hi ? i + u * step : lo] * a.stride, c, a.dim, whole);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u * step >= hi) break;
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += to_f32(v[u].e[j]);
      }
    }
  };
  if (a.dim % E == 0) all(true);
  else all(false);
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

// The same by a whole wavefront: 64 places are looked at together, so 32,768
// keys take three loads one after the other in place of fifteen.
__device__ __forceinline__ int wave_lower_bound(const uint32_t* skey, int n, uint32_t k) {
  int lo = 0, end = n;
  while (lo < end) {
    const int step = (end - lo + 63) / 64;
    const int64_t at = lo + ((int64_t)(threadIdx.x & 63) + 1) * step - 1;
    const int below = __popcll(__ballot(at < end && skey[at] < k));
    lo += below * step;
    end = min(end, lo + step - 1);
  }
  return lo;
}

// Zeros for the rows that occur nowhere; `there` holds kFillRows words.
template <typename G>
__device__ __forceinline__ void fill_rows(const SumArgs& a, int nth, G* dtable, uint32_t* there) {
  constexpr int E = kVec<G>;
  const int64_t r0 = a.fill0 + (int64_t)nth * kFillRows;
  const int rows = (int)(a.V - r0 < kFillRows ? a.V - r0 : kFillRows);
  if (threadIdx.x < kFillRows) there[threadIdx.x] = a.seen && (int)threadIdx.x < rows ? a.seen[r0 + threadIdx.x] : 0;
  __syncthreads();
  if (!a.seen) {
    for (int i = threadIdx.x; i < a.n; i += 256) {
      const int64_t at = (int64_t)a.skey[i] - r0;
      if (at >= 0 && at < rows) there[at] = 1;
    }
    __syncthreads();
  }
  const Vec<G, E> zero = {};
  for (int r = 0; r < rows; ++r) {
    if (there[r]) continue;  // uniform over the workgroup
    G* row = dtable + (r0 + r) * a.dim;
    for (int64_t c = threadIdx.x * E; c < a.dim; c += 256 * E) stream_row<E>(row, (int)c, a.dim, zero);
  }
}

// The sums of a piece's runs that belong to an id of more than 2 * kPiece
// tokens. Such an id's run touches an edge of every piece it is in.
template <typename T, typename G>
__global__ __launch_bounds__(256) void emb_pieces(SumArgs a, const T* dout, G* dtable) {
  constexpr int E = kVec<T>;
  __shared__ float lds[256][E + 1];
  // the piece's keys, and as many before and after it as tell a frequent id
  constexpr int kSide = 2 * kPiece;
  __shared__ uint32_t tok[kPiece], keys[kPiece + 2 * kSide];
  const int role = blockIdx.x;
  if (role >= a.work) return fill_rows(a, role - a.work, dtable, tok);
  const int piece = role / a.cols, first = piece * kPiece, len = min(a.n - first, kPiece);
  for (int i = threadIdx.x; i < kPiece + 2 * kSide; i += 256) {
    const int64_t at = (int64_t)first - kSide + i;
    keys[i] = at >= 0 && at < a.n ? a.skey[at] : ~0u;
  }
  __shared__ int edge[2];  // keys equal to the first, and to the last
  if ((int)threadIdx.x < len) tok[threadIdx.x] = a.stok[first + threadIdx.x];
  __syncthreads();
  if (threadIdx.x < 64) {
    const bool in = (int)threadIdx.x < len;
    const uint32_t mine = in ? keys[kSide + threadIdx.x] : ~0u;
    const int na = __popcll(__ballot(in && mine == keys[kSide])), nb = __popcll(__ballot(in && mine == keys[kSide + len - 1]));
    if (threadIdx.x == 0) {
      edge[0] = na;
      edge[1] = nb;
    }
  }
  __syncthreads();
  const uint32_t *key = keys + kSide, ka = key[0], kb = key[len - 1], V = (uint32_t)a.V;
  const int tpr = a.tpr, lane = threadIdx.x % tpr, sub = threadIdx.x / tpr, groups = 256 / tpr;
  const int c = (role % a.cols * tpr + lane) * E;
  for (int side = 0; side < 2; ++side) {
    int lo = 0, hi = len;
    bool heavy;
    if (ka == kb) {
      if (side) break;
      // the whole piece: a longer run goes on to one side or the other
      heavy = ka < V && (key[-1] == ka || key[len] == ka);
    } else if (side == 0) {
      hi = edge[0];
      heavy = key[hi - 1 - kSide] == ka;  // ka < kb <= V
    } else {
      lo = len - edge[1];
      heavy = kb < V && key[lo + kSide] == kb;
    }
    if (!heavy) continue;  // uniform over the workgroup
    float acc[E] = {};
    if (c < a.dim) add_rows(a, dout, tok, lo + sub, hi, groups, c, acc);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < E; ++j) lds[threadIdx.x][j] = acc[j];
    __syncthreads();
    if (sub == 0 && c < a.dim) {
      for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += lds[g * tpr + lane][j];
      float* o = a.piece + ((int64_t)piece * 2 + side) * a.dim;
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c + j < a.dim) o[c + j] = acc[j];
    }
  }
}

// A window of kWindow sorted positions to the lanes of a row: the runs that
// begin in it, one after the other in one stream of rows, eight of which are
// in flight whatever the runs' lengths.
constexpr int kSpan = kWindow + 2 * kPiece + 1;      // positions that decide the window's runs
constexpr int kWords = (kSpan + 31) / 32 + 1;        // of a mask of them, one to spare
constexpr int kStaged = 2 * (kSpan + 1) + 2 * ((kWords + 1) / 2);  // words of LDS of a window, the mask's an even number
static_assert(kWindow <= 64 && kPiece <= 64 && kStaged % 2 == 0);

template <typename T, typename G>
__global__ __launch_bounds__(256) void emb_sums(SumArgs a, const T* dout, G* dtable) {
  constexpr int E = kVec<T>, U = 8;
  extern __shared__ uint64_t lds64[];  // per window: a mask, then the keys and token numbers
  uint32_t* lds = (uint32_t*)lds64;
  const int role = blockIdx.x;
  if (role >= a.work) return fill_rows(a, role - a.work, dtable, lds);
  const int tpr = a.tpr, lane = threadIdx.x % tpr, sub = threadIdx.x / tpr, groups = 256 / tpr;
  const int64_t begin = ((int64_t)(role / a.cols) * groups + sub) * kWindow;
  uint32_t *mask = lds + sub * kStaged, *key = mask + 2 * ((kWords + 1) / 2), *tok = key + kSpan + 1;
  // key[i] is that of sorted position first - 1 + i. Ids that name no row sort
  // behind all others and have the key of the places past the last position:
  // the two are one run without an end, which is never summed or written.
  const int64_t first = begin < a.n ? begin : a.n;
  const uint32_t V = (uint32_t)a.V;
  for (int i = lane; i <= kSpan; i += tpr) {
    const int64_t at = first - 1 + i;
    const bool there = at >= 0 && at < a.n;
    const uint32_t k = there ? a.skey[at] : ~0u;
    key[i] = k < V ? k : ~0u;
    tok[i] = there ? a.stok[at] : 0;
  }
  for (int i = lane; i < 2 * ((kWords + 1) / 2); i += tpr) mask[i] = 0;
  __syncthreads();
  // bit i: a run ends at place i, and one begins at i + 1
  for (int i = lane; i < kSpan; i += tpr)
    if (key[i] != key[i + 1]) atomicOr(&mask[i >> 5], 1u << (i & 31));
  __syncthreads();
  const int c = (role % a.cols * tpr + lane) * E;
  // the stream: from the window's first run to the end of its last
  const uint64_t* mask64 = (const uint64_t*)mask;
  const uint64_t begins = mask64[0] & (~0ull >> (64 - kWindow));
  if (!begins) return;  // no run begins here
  int i = __builtin_ctzll(begins) + 1;
  const int last = 64 - __builtin_clzll(begins);
  int stop = 0;
  for (int w = last >> 5; w < kWords && !stop; ++w) {
    const uint32_t m = w == last >> 5 ? mask[w] & (~0u << (last & 31)) : mask[w];
    if (m) stop = w * 32 + __builtin_ctz(m) + 1;
  }
  const bool heavy = stop == 0 || stop - last > 2 * kPiece;  // a frequent id: below
  if (heavy) stop = last;
  const uint32_t id = key[last];
  const int s = (int)(first - 1) + last;
  // where its run ends (whole wavefronts search together)
  int e = 0;
  if (heavy && id < V) e = tpr >= 64 ? wave_lower_bound(a.skey, a.n, id + 1) : lower_bound(a.skey, a.n, id + 1);
  if (c >= a.dim) return;
  float acc[E] = {};
  auto write = [&](uint32_t to) {
    Vec<G, E> o;
#pragma unroll
    for (int j = 0; j < E; ++j) o.e[j] = scaled<G>(acc[j], a.scale);
    stream_row<E>(dtable + (int64_t)to * a.dim, c, a.dim, o);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = 0;
  };
  auto stream = [&](bool whole) {
    for (; i < stop; i += U) {
      Vec<T, E> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)  // past the end the last row again, which is not added
        v[u] = load_col<E>(dout + (int64_t)tok[min(i + u, stop - 1)] * a.stride, c, a.dim, whole);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= stop) break;
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += to_f32(v[u].e[j]);
        if (mask[(i + u) >> 5] >> ((i + u) & 31) & 1) write(key[i + u]);
      }
    }
  };
  if (a.dim % E == 0) stream(true);
  else stream(false);
  if (!e) return;
  if (!a.piece) {
    add_rows(a, dout, a.stok, s, e, 1, c, acc);
  } else {
    constexpr int UP = 8;
    const int p0 = s / kPiece, p1 = (e - 1) / kPiece;
    for (int p = p0; p <= p1; p += UP) {
      Vec<float, E> v[UP];
#pragma unroll
      for (int u = 0; u < UP; ++u) {
        // the id's run lies at the right edge of the first piece unless it fills it
        const int q = min(p + u, p1), side = q == p0 && s % kPiece != 0 ? 1 : 0;
        v[u] = load_row<E>(a.piece + ((int64_t)q * 2 + side) * a.dim, c, a.dim);
      }
#pragma unroll
      for (int u = 0; u < UP; ++u) {
        if (p + u > p1) break;
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += v[u].e[j];
      }
    }
  }
  write(id);
}

// Lanes of a row: a power of two that covers its vectors, 8 to 256.
int lanes_of(int64_t vecs) {
  int t = 8;
  while (t < vecs && t < 256) t *= 2;
  return t;
}

struct BwdLayout {
  size_t key[2], tok[2], hist, seen, piece, total;
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
  l.hist = take(sorted ? kSortBlocks * kDigits * 4 : 0);
  l.seen = take(sorted ? (size_t)p.n_vocab : 0);
  l.piece = take(p.n_tokens > kPieceMin ? (size_t)ceil_div(p.n_tokens, kPiece) * 2 * (size_t)p.dim * 4 : 0);
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
    hipLaunchKernelGGL(emb_fwd<T>, dim3((unsigned)grid), dim3(256), 0, st, p.ids, p.n_tokens, p.ids_64, p.n_vocab, p.dim,
                       p.row_stride, p.scale, (const T*)table, (T*)out, tpr, p.dev_status);
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
  uint8_t* seen = nullptr;
  if (n <= kRankMax) {
    // at least one workgroup, which also sets the status word
    hipLaunchKernelGGL(emb_rank, dim3(n ? (unsigned)ceil_div(n, 64) : 1), dim3(256), 0, st, p.ids, n, p.ids_64,
                       p.n_vocab, key[0], tok[0], p.dev_status);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    seen = base + l.seen;
    const int32_t words = (int32_t)ceil_div(p.n_vocab, 16);
    hipLaunchKernelGGL(emb_clear, dim3((unsigned)ceil_div(words, 256)), dim3(256), 0, st, (u32x4_t*)seen, words,
                       p.dev_status);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int32_t per = (int32_t)(ceil_div(ceil_div(n, kSortBlocks), kDigits) * kDigits);
    const unsigned blocks = (unsigned)ceil_div(n, per);
    for (int shift = 0; shift == 0 || ((uint32_t)p.n_vocab >> shift) != 0; shift += kBits) {  // keys are 0 .. n_vocab
      SortArgs a{shift ? nullptr : p.ids, key[cur], tok[cur], key[cur ^ 1], tok[cur ^ 1],
                 (uint32_t*)(base + l.hist), n, per, p.ids_64, p.n_vocab, shift, seen, p.dev_status};
      hipLaunchKernelGGL(emb_count, dim3(blocks), dim3(kDigits), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(emb_scatter, dim3(blocks), dim3(kDigits), 0, st, a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      cur ^= 1;
    }
  }
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t vecs = ceil_div(p.dim, kVec<T>);
    const int tpr = lanes_of(vecs);
    const int32_t cols = (int32_t)ceil_div(vecs, tpr);
    const bool pieces = n > kPieceMin;
    SumArgs a{key[cur], tok[cur], n, p.n_vocab, p.dim, tpr, p.row_stride, p.scale,
              pieces ? (float*)(base + l.piece) : nullptr, seen, 0, cols, 0};
    auto sums = [&](auto g) {
      using G = decltype(g);
      const int64_t fills = ceil_div(p.n_vocab, kFillRows), first = pieces ? fills / 2 : 0;
      if (pieces) {
        a.work = (int32_t)ceil_div(n, kPiece) * cols;
        hipLaunchKernelGGL((emb_pieces<T, G>), dim3((unsigned)(a.work + first)), dim3(256), 0, st, a, (const T*)dout,
                           (G*)dtable);
        const hipError_t e2 = hipGetLastError();
        if (e2 != hipSuccess) return e2;
      }
      const int groups = 256 / tpr;
      a.work = (int32_t)ceil_div(n, kWindow * groups) * cols;
      a.fill0 = first * kFillRows;
      hipLaunchKernelGGL((emb_sums<T, G>), dim3((unsigned)(a.work + fills - first)), dim3(256),
                         groups * kStaged * sizeof(uint32_t), st, a, (const T*)dout, (G*)dtable);
      return hipGetLastError();
    };
    return p.grad_dtype == ARGUS_F32 ? sums(float{}) : sums(T{});
  });
}

}  // namespace argus
