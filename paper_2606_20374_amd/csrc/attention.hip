// Softmax attention over packed documents, forward, and the plan of tiles that
// both directions use.
//
// S^T = K Q^T per tile of keys, with the running maximum and sum of each
// query, and O^T += V^T P^T. The transposed products keep a query in one lane
// (two lanes, one to each half of a tile's keys), so its maximum, sum and
// rescaling are plain registers, and P^T is the second product's operand as it
// comes out of the first, rounded to bfloat16: at most 2^-8 of each
// probability, as the values and the output have it, since the matrix
// instructions take no wider operand at this rate (o is off by 0.0021 of its
// norm, with 32-bit probabilities by 0.0016, the output's own rounding). The
// sum l is that of the unrounded ones, in 32 bits.
//
// A workgroup of four wavefronts owns 128 queries, 32 to a wavefront, and two
// such workgroups share a CU (at most 256 registers a lane: with one, 1,150 us
// in place of 682). Keys and values come straight into LDS, 64 at a time, the
// next tile while one is used (through registers 682 us, straight 583).
// Four sequences of 4,096, causal, 32 query and 8 key heads of 128: 556 to
// 592 us, 930 to 990 TFLOP/s, after some fifty runs one after the other; the
// first thirty take 600 to 760 us and the same cycles, at a lower clock. The
// matrix units are busy half of the cycles (counters). Tiles of 32 keys four deep (617 us), eight
// wavefronts with three tiles (594) and three workgroups to a CU (718) were
// not faster.
#include "attention_tile.h"

#pragma clang fp contract(fast)

namespace argus {
using namespace attn;
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;  // keys of a tile

struct FwdArgs {
  Docs d;
  const __bf16 *q, *k, *v;
  __bf16* o;
  float* lse;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;
  int32_t H, N, D, causal;
  Plan plan;
  float scale;
};

struct PlanArgs {
  Docs d;
  int32_t causal;
  uint32_t* bad;
  int32_t* dev_status;
  int2 *q_tile, *k_tile;  // k_tile may be null
  int32_t q_n, k_n;
};

// One workgroup checks the offsets, sets the status word and lists the tiles:
// documents by their length, longest first, in 64 classes, and of each the
// tiles with the most to do first. A document's tiles stay together, since
// they read the same keys (all tiles by their work alone: 602 us in place of
// 570 for four documents of 4,096).
__global__ __launch_bounds__(1024) void attn_plan(PlanArgs a) {
  __shared__ int any, most, count[64], place[64], tiles;
  const Docs& d = a.d;
  const int tid = threadIdx.x;
  if (tid == 0) any = d.q_off && (d.q_off[0] != 0 || d.k_off[0] != 0 || d.q_off[d.n_docs] != d.n_q ||
                                  d.k_off[d.n_docs] != d.n_k);
  __syncthreads();
  if (d.q_off) {
    bool b = false;
    for (int i = tid; i < d.n_docs; i += 1024) b |= d.q_off[i] > d.q_off[i + 1] || d.k_off[i] > d.k_off[i + 1];
    if (b) any = 1;
  }
  __syncthreads();
  if (tid == 0) {
    *a.bad = any;
    if (a.dev_status) *a.dev_status = any ? (int32_t)ARGUS_DEV_BAD_SEGMENT : 0;
  }
  if (any) return;
  const int wave = tid >> 6, lane = tid & 63;
  for (int side = 0; side < 2; ++side) {
    int2* out = side ? a.k_tile : a.q_tile;
    if (!out) continue;
    __syncthreads();
    if (tid < 64) count[tid] = 0;
    if (tid == 0) most = 1;
    __syncthreads();
    for (int i = tid; i < d.n_docs; i += 1024) {
      const Doc t = doc_at(d, i);
      atomicMax(&most, side ? t.nq : t.nk);
    }
    __syncthreads();
    const float per = 63.0f / (float)most;
    auto class_of = [&](const Doc& t) { return 63 - (int)((float)(side ? t.nq : t.nk) * per); };
    auto tiles_of = [&](const Doc& t) { return ((side ? t.nk : t.nq) + kTile - 1) / kTile; };
    for (int i = tid; i < d.n_docs; i += 1024) {
      const Doc t = doc_at(d, i);
      atomicAdd(&count[class_of(t)], tiles_of(t));
    }
    __syncthreads();
    if (tid == 0) {
      int at = 0;
      for (int c = 0; c < 64; ++c) {
        place[c] = at;
        at += count[c];
      }
      tiles = at;
    }
    __syncthreads();
    for (int i = wave; i < d.n_docs; i += 16) {
      const Doc t = doc_at(d, i);
      const int n = tiles_of(t);
      int at = 0;
      if (lane == 0) at = atomicAdd(&place[class_of(t)], n);
      at = __builtin_amdgcn_readfirstlane(at);
      // causal: the last queries see the most keys, the first keys the most queries
      for (int j = lane; j < n; j += 64) out[at + j] = make_int2(i, (a.causal && !side ? n - 1 - j : j) * kTile);
    }
    for (int i = tiles + tid; i < (side ? a.k_n : a.q_n); i += 1024) out[i] = make_int2(-1, 0);
  }
}

// Malformed offsets: every query sees no key.
__device__ void fill_empty(const FwdArgs& a) {
  const int64_t n = a.d.n_q * a.H;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    a.lse[i] = -__builtin_inff();
    for (int j = 0; j < a.D; ++j) a.o[i * a.D + j] = (__bf16)0.0f;
  }
}

template <int DP>
__global__ __launch_bounds__(kThreads, 2) void attn_fwd(FwdArgs a) {
  constexpr int KS = DP / 16, DT = DP / 32;
  // four arrays, not two of two: reads of one tile then do not wait for the
  // loads of the next
  __shared__ __align__(16) __bf16 kt0[kKeys * DP], kt1[kKeys * DP], vt0[kKeys * DP], vt1[kKeys * DP];
  if (*a.d.bad) return fill_empty(a);
  int h, di, row0;
  if (!my_tile(a.plan, a.H, h, di, row0)) return;
  const Doc doc = doc_at(a.d, di);
  const int n = h / (a.H / a.N);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, half = lane >> 5;
  const int q0 = row0 + w * 32, q = q0 + (lane & 31);  // the wavefront's first query, the lane's
  const int shift = doc.nk - doc.nq;                   // query i sees keys up to i + shift
  const float sc = score_scale(a.scale);

  bf16x8 qf[KS];
  load_operand<DP>(qf, rows_rsrc(a.q + (doc.q0 + row0) * a.q_tok + (int64_t)h * a.q_head, doc.nq - row0, a.q_tok, a.D),
                   w * 32 + (lane & 31), a.q_tok, a.D);
  f32x16 acc[DT];
  clear<DP>(acc);
  float m = -__builtin_inff(), l = 0;
  // keys that some query of the workgroup sees, and of the wavefront
  const int last_row = row0 + kTile - 1 < doc.nq - 1 ? row0 + kTile - 1 : doc.nq - 1;
  const int seen = a.causal ? last_row + shift + 1 : doc.nk;
  const int nk = seen < 0 ? 0 : seen < doc.nk ? seen : doc.nk;
  const int tiles = (nk + kKeys - 1) / kKeys;
  int wave_nk = q0 >= doc.nq ? 0 : nk;
  if (a.causal && q0 + 32 + shift < wave_nk) wave_nk = q0 + 32 + shift;
  int lim = a.causal ? q + shift : doc.nk - 1;  // the last key that the lane's query sees
  if (lim > doc.nk - 1) lim = doc.nk - 1;
  const __bf16* kb = a.k + doc.k0 * a.k_tok + (int64_t)n * a.k_head;
  const __bf16* vb = a.v + doc.k0 * a.v_tok + (int64_t)n * a.v_head;
  Reader<DP> rd;
  const TileLoad<DP, kKeys, kThreads> lk(a.k_tok, a.D), lv(a.v_tok, a.D);
  auto load = [&](int t, __bf16* K, __bf16* V) __attribute__((always_inline)) {
    const int64_t first = (int64_t)t * kKeys;
    lk.load(rows_rsrc(kb + first * a.k_tok, doc.nk - first, a.k_tok, a.D), K);
    lv.load(rows_rsrc(vb + first * a.v_tok, doc.nk - first, a.v_tok, a.D), V);
  };
  auto compute = [&](int key0, const __bf16* K, const __bf16* V) __attribute__((always_inline)) {
    rd.fresh();
    f32x16 s[kKeys / 32];
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[b] = mfma(rd.rows(K, 32 * b, ks), qf[ks], s[b]);
    }
    // the tiles at the causal edge and at the document's end
    if (key0 + kKeys > doc.nk || (a.causal && key0 + kKeys - 1 > q0 + shift)) {
#pragma unroll
      for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 32 * b + 8 * (i / 4) + 4 * half + i % 4;
          s[b][i] = key <= lim ? s[b][i] : -__builtin_inff();
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx = fmaxf(mx, other_half(mx)) * sc;
    // The sums are kept against an earlier maximum until it is passed by
    // 2^8: the probabilities then stay below 2^8, which 32 bits and a
    // bfloat16 operand hold as exactly as those below 1.
    const float mn = fmaxf(m, mx);
    if (__ballot(mn > m + 8.0f)) {
      const float al = exp2_fast(m - (mn > -__builtin_inff() ? mn : 0.0f));
      m = mn;
      l *= al;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= al;
    }
    const float mm = m > -__builtin_inff() ? m : 0.0f;
    float sum = 0;
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = exp2_fast(s[b][i] * sc - mm);
        s[b][i] = p;
        sum += p;
      }
    l += sum;
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        const bf16x8 p = as_operand(s[b], k2);
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = mfma(rd.cols(V, 32 * b + 16 * k2, 32 * d), p, acc[d]);
      }
  };
  auto step = [&](int t, const __bf16* K, const __bf16* V, __bf16* next_k, __bf16* next_v)
                  __attribute__((always_inline)) {
    if (t + 1 < tiles) load(t + 1, next_k, next_v);
    const int key0 = t * kKeys;
    if (key0 < wave_nk) compute(key0, K, V);
    wait_loads();
    __syncthreads();
  };
  if (tiles > 0) load(0, kt0, vt0);
  wait_loads();
  __syncthreads();
  for (int t = 0; t < tiles; t += 2) {
    step(t, kt0, vt0, kt1, vt1);
    if (t + 1 < tiles) step(t + 1, kt1, vt1, kt0, vt0);
  }
  const float z = l + other_half(l);
  if (q >= doc.nq) return;
  if (lim < 0) clear<DP>(acc);  // no key seen: 0 times what the hidden values hold may be NaN
  const int64_t row = (doc.q0 + q) * a.H + h;
  if (half == 0) a.lse[row] = z == 0 ? -__builtin_inff() : m * kLn2 + __logf(z);
  write_rows<DP>(a.o + row * a.D, acc, z > 0 ? 1.0f / z : z == 0 ? 0.0f : z, a.D);  // a NaN stays
}

}  // namespace

size_t attn_plan_bytes(const argus_attention_t& p, bool both) {
  return 256 + align256((size_t)plan_entries(p.n_q, p.n_docs) * 8) +
         (both ? align256((size_t)plan_entries(p.n_k, p.n_docs) * 8) : 0);
}

hipError_t launch_attn_plan(const argus_attention_t& p, void* ws, Plan* queries, Plan* keys, hipStream_t st) {
  uint8_t* base = (uint8_t*)ws;
  int2* qt = (int2*)(base + 256);
  const int32_t qn = (int32_t)plan_entries(p.n_q, p.n_docs), kn = (int32_t)plan_entries(p.n_k, p.n_docs);
  int2* kt = keys ? (int2*)(base + 256 + align256((size_t)qn * 8)) : nullptr;
  *queries = {qt, qn};
  if (keys) *keys = {kt, kn};
  PlanArgs a{{p.q_off, p.k_off, p.n_docs, p.n_q, p.n_k, nullptr}, p.causal, (uint32_t*)ws, p.dev_status, qt, kt, qn, kn};
  hipLaunchKernelGGL(attn_plan, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

size_t attention_workspace_bytes(const argus_attention_t& p) { return attn_plan_bytes(p, false); }

hipError_t launch_attention(const argus_attention_t& p, const void* q, const void* k, const void* v, void* o,
                            float* lse, void* ws, hipStream_t st) {
  Plan plan;
  const hipError_t e = launch_attn_plan(p, ws, &plan, nullptr, st);
  if (e != hipSuccess || p.n_q == 0) return e;
  FwdArgs a{{p.q_off, p.k_off, p.n_docs, p.n_q, p.n_k, (const uint32_t*)ws},
            (const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (__bf16*)o, lse,
            p.q_tok, p.q_head, p.k_tok, p.k_head, p.v_tok, p.v_head,
            p.n_heads, p.n_kv_heads, p.head_dim, p.causal, plan, p.scale};
  const unsigned grid = (unsigned)plan.n * p.n_heads;  // below 2^23: the caller has checked
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(grid), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  };
  return p.head_dim <= 64 ? go(attn_fwd<64>) : go(attn_fwd<128>);
}

}  // namespace argus
