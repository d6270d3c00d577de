// Softmax attention over packed documents, backward.
//
//   P = exp(S - lse),  dP = dO V^T,  dS = P (dP - delta),  delta = dO . O
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
// The probabilities are recomputed from q, k and lse. Launches, after that of
// the plan of tiles, which checks the offsets:
//   prep   delta and lse (in units of log2) per head and query
//   dkv    a workgroup owns 128 keys of a key head, 32 to a wavefront, with V
//          as operands in registers (K too where heads are at most 64 wide, in
//          LDS otherwise), and takes the queries of all its query heads
//          through LDS. S = Q K^T keeps a key in one lane, so P and dS are the
//          operands of dV^T += dO^T P and dK^T += Q^T dS as they are.
//   dq     a workgroup owns 128 queries and takes the keys through LDS:
//          S^T = K Q^T keeps a query in one lane, dQ^T += K^T dS^T.
// S and dP are computed in both: 7 products in place of 5, and no atomics:
// sums have a fixed order. Where tiles and heads are few, several workgroups
// share one (the queries of dkv's, the keys of dq's in equal parts) and write
// 32-bit sums that a further launch for each of dk, dv and dq adds in their
// order.
//
// Each rounding to bfloat16 is of an operand, P and dS, at most 2^-8 of each:
// the matrix instructions take no wider one at this rate (the gradients are
// off by 0.0024 of their norm, with both in 32 bits by 0.0017, the outputs' own
// rounding). Two workgroups share a CU, with at most 256 registers a lane. Two sequences of
// 8,192, causal, 32 query and 8 key heads of 128: 3,540 to 3,740 us in all from run
// to run, 735 to 776 TFLOP/s of the gradient's five products. Under the
// profiler dkv takes 2,047 us, dq 1,391 and prep 50 after forty runs; the matrix
// units are busy 59% of dkv's cycles and 64% of dq's (counters). 13 packed
// documents, the longest of 3,812 tokens, 16 heads of 64: 226 to 233 us (dkv
// 124, dq 92, prep 13 under the profiler).
#include "attention_tile.h"

#pragma clang fp contract(fast)

namespace argus {
using namespace attn;

size_t attn_plan_bytes(const argus_attention_t& p, bool both);
hipError_t launch_attn_plan(const argus_attention_t& p, void* ws, Plan* queries, Plan* keys, hipStream_t st);

namespace {

constexpr int kThreads = 256;
constexpr int kOwn = kTile;  // rows a workgroup owns
constexpr int kStep = 64;    // rows of the other side taken at a time

struct BwdArgs {
  Docs d;
  const __bf16 *q, *k, *v, *o, *go;
  const float* lse;
  __bf16 *dq, *dk, *dv;
  float* stat;   // [H][n_q][2]: lse in units of log2, delta
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;
  int32_t H, N, D, causal;
  Plan plan;
  int32_t parts;  // workgroups that share a tile and head
  float* sums;    // parts > 1: [parts][rows][D] (dkv: of dk, then of dv)
  float scale;
};

// A query and head to sixteen lanes.
__global__ __launch_bounds__(256) void attn_prep(BwdArgs a) {
  const int lane = threadIdx.x & 15;
  const int64_t n = a.d.n_q * a.H;
  for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < n; i += (int64_t)gridDim.x * 16) {
    float s = 0;
    const int c = lane * 8;
    if (c < a.D) {
      const bf16x8 x = *(const bf16x8*)(a.go + i * a.D + c), y = *(const bf16x8*)(a.o + i * a.D + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += (float)x[j] * (float)y[j];
    }
    s = row_sum(s);
    if (lane == 0) {
      const int64_t t = i / a.H, at = (i - t * a.H) * a.d.n_q + t;
      const float l = a.lse[i];
      // a query that sees nothing: exp2(s - infinity) = 0 for every key (a NaN
      // stays one: every key it sees shares its sum)
      *(float2*)(a.stat + 2 * at) = make_float2(l == -__builtin_inff() ? __builtin_inff() : l * kLog2e, s);
    }
  }
}

// Zeros for n rows of dim elements, spread over the grid.
__device__ void fill_zero(__bf16* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
    p[i] = (__bf16)0.0f;
}

// As write_rows, in 32 bits.
template <int DP>
__device__ __forceinline__ void write_sums(float* row, const f32x16 (&x)[DP / 32], int dim) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int at = 32 * d + 2 * i + 4 * half;
      if (at < dim) *(float4*)(row + at) = make_float4(x[d][i], x[d][i + 1], x[d][i + 2], x[d][i + 3]);
    }
}

// Adds the parts' sums in their order: n elements, eight to a thread.
__global__ __launch_bounds__(256) void attn_join(const float* sums, int32_t parts, int64_t n, float scale, __bf16* out,
                                                 const uint32_t* bad) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n || *bad) return;  // n is a multiple of 8
  float4 u = *(const float4*)(sums + i), v = *(const float4*)(sums + i + 4);
  for (int p = 1; p < parts; ++p) {
    const float4 a = *(const float4*)(sums + p * n + i), b = *(const float4*)(sums + p * n + i + 4);
    u = make_float4(u.x + a.x, u.y + a.y, u.z + a.z, u.w + a.w);
    v = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
  }
  const float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
  bf16x8 o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = (__bf16)(f[j] * scale);
  *(bf16x8*)(out + i) = o;
}

// Heads wider than 64 keep K in LDS, read anew for every step: with dK, dV, V
// and K in registers only one wavefront fits a SIMD, which then waits for each
// of its reads. Their steps are half as long, so that two workgroups fit a
// CU's LDS.
template <int DP>
__global__ __launch_bounds__(kThreads, 2) void attn_dkv(BwdArgs a) {
  constexpr int KS = DP / 16, DT = DP / 32;
  constexpr bool kInLds = DP > 64;
  constexpr int kQ = kInLds ? 32 : 64;  // queries of a step
  // arrays of their own, so that reads of one tile do not wait for the loads
  // of the next
  __shared__ __align__(16) __bf16 qt0[kQ * DP], qt1[kQ * DP], gt0[kQ * DP], gt1[kQ * DP];
  __shared__ __align__(16) __bf16 kt[kInLds ? kOwn * DP : 8];
  __shared__ __align__(16) float st0[2 * kQ], st1[2 * kQ];  // lse and delta of each query
  if (*a.d.bad) {
    fill_zero(a.dk, a.d.n_k * a.N * a.D);
    fill_zero(a.dv, a.d.n_k * a.N * a.D);
    return;
  }
  int vn, di, row0;
  if (!my_tile(a.plan, a.N * a.parts, vn, di, row0)) return;
  const Doc doc = doc_at(a.d, di);
  const int G = a.H / a.N, n = vn / a.parts, part = vn % a.parts;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, half = lane >> 5;
  const int shift = doc.nk - doc.nq, key0 = row0 + w * 32, key = key0 + (lane & 31);
  const float sc = score_scale(a.scale);
  const auto src_k = rows_rsrc(a.k + (doc.k0 + row0) * a.k_tok + (int64_t)n * a.k_head, doc.nk - row0, a.k_tok, a.D);
  bf16x8 kf[kInLds ? 1 : KS], vf[KS];
  if constexpr (kInLds) TileLoad<DP, kOwn, kThreads>(a.k_tok, a.D).load(src_k, kt);
  else load_operand<DP>(kf, src_k, w * 32 + (lane & 31), a.k_tok, a.D);
  load_operand<DP>(vf, rows_rsrc(a.v + (doc.k0 + row0) * a.v_tok + (int64_t)n * a.v_head, doc.nk - row0, a.v_tok, a.D),
                   w * 32 + (lane & 31), a.v_tok, a.D);
  f32x16 dk[DT], dv[DT];
  clear<DP>(dk);
  clear<DP>(dv);
  // queries from the first that sees a key of the workgroup on, so none that
  // sees no key at all, whatever its rows hold
  int first = 0;
  if (a.causal && row0 > shift) first = row0 - shift;
  const int per = first < doc.nq ? (doc.nq - first + kQ - 1) / kQ : 0;
  // this part's steps, of all heads' one after the other
  const int begin = (int)((int64_t)per * G * part / a.parts), end = (int)((int64_t)per * G * (part + 1) / a.parts);
  const int tiles = end - begin;
  const int64_t o_tok = (int64_t)a.H * a.D;
  Reader<DP> rd;
  const uint32_t own = w * 32 * DP * 2;  // the wavefront's keys in their tile
  const TileLoad<DP, kQ, kThreads> lq(a.q_tok, a.D), lg(o_tok, a.D);
  int lh = n * G + (per ? begin / per : 0), lt = per ? begin % per : 0;  // head and step of the next load
  auto load = [&](__bf16* Q, __bf16* GO, float* st) __attribute__((always_inline)) {
    const int q0 = first + lt * kQ;
    lq.load(rows_rsrc(a.q + (doc.q0 + q0) * a.q_tok + (int64_t)lh * a.q_head, doc.nq - q0, a.q_tok, a.D), Q);
    lg.load(rows_rsrc(a.go + (doc.q0 + q0) * o_tok + (int64_t)lh * a.D, doc.nq - q0, o_tok, a.D), GO);
    // past the last query zeros: with do = 0 there, neither P nor dS counts
    if (w < 2 * kQ / 64) {
      const int64_t left = (int64_t)(doc.nq - q0) * 8;
      const auto r = __builtin_amdgcn_make_buffer_rsrc(a.stat + 2 * ((int64_t)lh * a.d.n_q + doc.q0 + q0), (short)0,
                                                       (int)(left < 8 * kQ ? left : 8 * kQ), 0x00020000);
      load_words(r, st + 64 * __builtin_amdgcn_readfirstlane(w), threadIdx.x * 4);
    }
    if (++lt == per) {
      lt = 0;
      ++lh;
    }
  };
  auto arrive = [&]() __attribute__((always_inline)) {
    wait_loads();
    __syncthreads();
  };
  int q0 = first + lt * kQ;  // first query of the step
  auto step = [&](int t, const __bf16* Q, const __bf16* GO, const float* st, __bf16* next_q, __bf16* next_g,
                  float* next_st) __attribute__((always_inline)) {
    if (t + 1 < tiles) load(next_q, next_g, next_st);
    rd.fresh();
#pragma unroll
    for (int b = 0; b < kQ / 32; ++b) {
      // the wavefront owns no key, or none that a query of these sees
      if (key0 >= doc.nk || (a.causal && q0 + 32 * b + 31 + shift < key0)) continue;
      f32x16 s, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 k;
        if constexpr (kInLds) k = rd.rows(kt, 0, ks, own);
        else k = kf[ks];
        s = mfma(rd.rows(Q, 32 * b, ks), k, s);
        dp = mfma(rd.rows(GO, 32 * b, ks), vf[ks], dp);
      }
      if (key0 + 32 > doc.nk || (a.causal && key0 + 31 > q0 + 32 * b + shift)) {
        // the first of the step's rows that sees the key, counted from row 4 half on
        int from = a.causal ? key - shift - q0 - 32 * b - 4 * half : -64;
        if (key >= doc.nk) from = 64;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 >= from ? s[i] : -__builtin_inff();
      }
#pragma unroll
      for (int i4 = 0; i4 < 16; i4 += 4) {
        const int r = 32 * b + 2 * i4 + 4 * half;
        const float4 a4 = *(const float4*)&st[2 * r], b4 = *(const float4*)&st[2 * r + 4];
        const float lv[4] = {a4.x, a4.z, b4.x, b4.z}, dl[4] = {a4.y, a4.w, b4.y, b4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = exp2_fast(s[i4 + j] * sc - lv[j]);
          s[i4 + j] = p;
          dp[i4 + j] = p * (dp[i4 + j] - dl[j]);
        }
      }
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        const bf16x8 p = as_operand(s, k2), d = as_operand(dp, k2);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          dv[c] = mfma(rd.cols(GO, 32 * b + 16 * k2, 32 * c), p, dv[c]);
          dk[c] = mfma(rd.cols(Q, 32 * b + 16 * k2, 32 * c), d, dk[c]);
        }
      }
    }
    q0 = q0 + kQ < first + per * kQ ? q0 + kQ : first;
    arrive();
  };
  if (tiles > 0) load(qt0, gt0, st0);
  arrive();
  for (int t = 0; t < tiles; t += 2) {
    step(t, qt0, gt0, st0, qt1, gt1, st1);
    if (t + 1 < tiles) step(t + 1, qt1, gt1, st1, qt0, gt0, st0);
  }
  if (key < doc.nk) {
    const int64_t row = ((doc.k0 + key) * a.N + n) * a.D, all = a.d.n_k * a.N * a.D;
    if (a.parts == 1) {
      write_rows<DP>(a.dk + row, dk, a.scale, a.D);
      write_rows<DP>(a.dv + row, dv, 1.0f, a.D);
    } else {
      write_sums<DP>(a.sums + part * all + row, dk, a.D);
      write_sums<DP>(a.sums + (a.parts + part) * all + row, dv, a.D);
    }
  }
}

template <int DP>
__global__ __launch_bounds__(kThreads, 2) void attn_dq(BwdArgs a) {
  constexpr int KS = DP / 16, DT = DP / 32;
  __shared__ __align__(16) __bf16 kt0[kStep * DP], kt1[kStep * DP], vt0[kStep * DP], vt1[kStep * DP];
  if (*a.d.bad) return fill_zero(a.dq, a.d.n_q * a.H * a.D);
  int vh, di, row0;
  if (!my_tile(a.plan, a.H * a.parts, vh, di, row0)) return;
  const Doc doc = doc_at(a.d, di);
  const int h = vh / a.parts, part = vh % a.parts, n = h / (a.H / a.N);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, half = lane >> 5;
  const int q0 = row0 + w * 32, q = q0 + (lane & 31), shift = doc.nk - doc.nq;
  const float sc = score_scale(a.scale);
  const int64_t o_tok = (int64_t)a.H * a.D;
  bf16x8 qf[KS], gf[KS];
  load_operand<DP>(qf, rows_rsrc(a.q + (doc.q0 + row0) * a.q_tok + (int64_t)h * a.q_head, doc.nq - row0, a.q_tok, a.D),
                   w * 32 + (lane & 31), a.q_tok, a.D);
  load_operand<DP>(gf, rows_rsrc(a.go + (doc.q0 + row0) * o_tok + (int64_t)h * a.D, doc.nq - row0, o_tok, a.D),
                   w * 32 + (lane & 31), o_tok, a.D);
  float lse2 = __builtin_inff(), delta = 0;
  if (q < doc.nq) {
    const float2 st = *(const float2*)(a.stat + 2 * ((int64_t)h * a.d.n_q + doc.q0 + q));
    lse2 = st.x;
    delta = st.y;
  }
  f32x16 acc[DT];
  clear<DP>(acc);
  const int last_row = row0 + kOwn - 1 < doc.nq - 1 ? row0 + kOwn - 1 : doc.nq - 1;
  const int seen = a.causal ? last_row + shift + 1 : doc.nk;
  const int nk = seen < 0 ? 0 : seen < doc.nk ? seen : doc.nk, all_tiles = (nk + kStep - 1) / kStep;
  const int begin = (int)((int64_t)all_tiles * part / a.parts), tiles = (int)((int64_t)all_tiles * (part + 1) / a.parts);
  const __bf16* kb = a.k + doc.k0 * a.k_tok + (int64_t)n * a.k_head;
  const __bf16* vb = a.v + doc.k0 * a.v_tok + (int64_t)n * a.v_head;
  Reader<DP> rd;
  const TileLoad<DP, kStep, kThreads> lk(a.k_tok, a.D), lv(a.v_tok, a.D);
  auto load = [&](int t, __bf16* K, __bf16* V) __attribute__((always_inline)) {
    const int64_t f = (int64_t)t * kStep;
    lk.load(rows_rsrc(kb + f * a.k_tok, doc.nk - f, a.k_tok, a.D), K);
    lv.load(rows_rsrc(vb + f * a.v_tok, doc.nk - f, a.v_tok, a.D), V);
  };
  int lim = a.causal ? q + shift : doc.nk - 1;
  if (lim > doc.nk - 1) lim = doc.nk - 1;
  auto step = [&](int t, const __bf16* K, const __bf16* V, __bf16* next_k, __bf16* next_v)
                  __attribute__((always_inline)) {
    const int key0 = t * kStep;
    if (t + 1 < tiles) load(t + 1, next_k, next_v);
    rd.fresh();
#pragma unroll
    for (int b = 0; b < kStep / 32; ++b) {
      // the wavefront owns no query, or none that sees a key of these
      if (q0 >= doc.nq || (a.causal && key0 + 32 * b > q0 + 31 + shift)) continue;
      f32x16 s, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = mfma(rd.rows(K, 32 * b, ks), qf[ks], s);
        dp = mfma(rd.rows(V, 32 * b, ks), gf[ks], dp);
      }
      if (key0 + 32 * b + 32 > doc.nk || (a.causal && key0 + 32 * b + 31 > q0 + shift)) {
        const int to = lim - key0 - 32 * b - 4 * half;  // the last key of the step that is seen
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 <= to ? s[i] : -__builtin_inff();
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] = exp2_fast(s[i] * sc - lse2) * (dp[i] - delta);
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        const bf16x8 d = as_operand(dp, k2);
#pragma unroll
        for (int c = 0; c < DT; ++c) acc[c] = mfma(rd.cols(K, 32 * b + 16 * k2, 32 * c), d, acc[c]);
      }
    }
    wait_loads();
    __syncthreads();
  };
  if (begin < tiles) load(begin, kt0, vt0);
  wait_loads();
  __syncthreads();
  for (int t = begin; t < tiles; t += 2) {
    step(t, kt0, vt0, kt1, vt1);
    if (t + 1 < tiles) step(t + 1, kt1, vt1, kt0, vt0);
  }
  if (q < doc.nq) {
    if (lim < 0) clear<DP>(acc);  // no key seen: no gradient, whatever its row and the hidden ones hold
    const int64_t row = ((doc.q0 + q) * a.H + h) * a.D;
    if (a.parts == 1) write_rows<DP>(a.dq + row, acc, a.scale, a.D);
    else write_sums<DP>(a.sums + part * a.d.n_q * a.H * a.D + row, acc, a.D);
  }
}

}  // namespace

namespace {

// Workgroups that share a tile: as many as make kEnough in all (two to a CU,
// twice), while each still has kPart rows of a document of average length to
// take. One document of 8,192, 8 heads of 128 that share one key head: 2,595
// us unshared, 614 us shared; 32 heads over 8, two of 2,048: 451 and 310 us.
// Sharing where there are 1,456 workgroups, or documents of 512, loses the
// sums' traffic (13 packed documents: 232 us unshared, 298 with twice kEnough).
constexpr int64_t kEnough = 1024, kPart = 512, kMostParts = 8;
int32_t parts_of(int64_t own, int64_t other, int32_t n_docs, int64_t heads, int64_t heads_taken) {
  const int64_t blocks = plan_entries(own, n_docs) * heads;
  int64_t parts = ceil_div(kEnough, blocks), most = other / n_docs * heads_taken / kPart;
  if (parts > most) parts = most;
  if (parts > kMostParts) parts = kMostParts;
  return parts < 1 ? 1 : (int32_t)parts;
}
struct Parts {
  int32_t dkv, dq;
  size_t bytes;
};
Parts parts_of(const argus_attention_t& p) {
  Parts r;
  r.dkv = parts_of(p.n_k, p.n_q, p.n_docs, p.n_kv_heads, p.n_heads / p.n_kv_heads);
  r.dq = parts_of(p.n_q, p.n_k, p.n_docs, p.n_heads, 1);
  const size_t kv = r.dkv > 1 ? (size_t)2 * r.dkv * (size_t)p.n_k * p.n_kv_heads * p.head_dim * 4 : 0;
  const size_t q = r.dq > 1 ? (size_t)r.dq * (size_t)p.n_q * p.n_heads * p.head_dim * 4 : 0;
  r.bytes = align256(kv > q ? kv : q);
  return r;
}

}  // namespace

size_t attention_bwd_workspace_bytes(const argus_attention_t& p) {
  return attn_plan_bytes(p, true) + align256((size_t)p.n_q * (size_t)p.n_heads * 2 * sizeof(float)) + parts_of(p).bytes;
}

hipError_t launch_attention_bwd(const argus_attention_t& p, const void* d_o, const void* q, const void* k,
                                const void* v, const void* o, const float* lse, void* dq, void* dk, void* dv,
                                void* ws, hipStream_t st) {
  Plan queries, keys;
  hipError_t e = launch_attn_plan(p, ws, &queries, &keys, st);
  if (e != hipSuccess) return e;
  const Parts parts = parts_of(p);
  uint8_t* stat = (uint8_t*)ws + attn_plan_bytes(p, true);
  BwdArgs a{{p.q_off, p.k_off, p.n_docs, p.n_q, p.n_k, (const uint32_t*)ws},
            (const __bf16*)q, (const __bf16*)k, (const __bf16*)v, (const __bf16*)o, (const __bf16*)d_o, lse,
            (__bf16*)dq, (__bf16*)dk, (__bf16*)dv, (float*)stat,
            p.q_tok, p.q_head, p.k_tok, p.k_head, p.v_tok, p.v_head,
            p.n_heads, p.n_kv_heads, p.head_dim, p.causal, keys, parts.dkv,
            (float*)(stat + align256((size_t)p.n_q * (size_t)p.n_heads * 2 * sizeof(float))), p.scale};
  const bool wide = p.head_dim > 64;
  if (p.n_q > 0) {
    const int64_t need = ceil_div(p.n_q * p.n_heads, 16), grid = need < 8192 ? need : 8192;
    hipLaunchKernelGGL(attn_prep, dim3((unsigned)grid), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  auto go = [&](auto kern, int64_t heads) {
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.plan.n * heads * a.parts)), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  };
  auto join = [&](int64_t n, int first, float scale, void* out) {
    hipLaunchKernelGGL(attn_join, dim3((unsigned)ceil_div(n, 8 * 256)), dim3(256), 0, st, a.sums + first * n, a.parts, n,
                       scale, (__bf16*)out, (const uint32_t*)ws);
    return hipGetLastError();
  };
  if (p.n_k > 0) {
    if ((e = wide ? go(attn_dkv<128>, p.n_kv_heads) : go(attn_dkv<64>, p.n_kv_heads)) != hipSuccess) return e;
    const int64_t n = p.n_k * p.n_kv_heads * p.head_dim;
    if (a.parts > 1 && ((e = join(n, 0, p.scale, dk)) != hipSuccess || (e = join(n, a.parts, 1.0f, dv)) != hipSuccess))
      return e;
  }
  if (p.n_q == 0) return hipSuccess;
  a.plan = queries;
  a.parts = parts.dq;
  if ((e = wide ? go(attn_dq<128>, p.n_heads) : go(attn_dq<64>, p.n_heads)) != hipSuccess || a.parts == 1) return e;
  return join(p.n_q * p.n_heads * p.head_dim, 0, p.scale, dq);
}

}  // namespace argus
