/*
 * libargus: the operators of a training step, for rank checks.
 *
 * argus_cross_rank and argus_l2 name ranks and (rank, kernel) pairs that are
 * slow. Whether the machine is slow or its work was larger is answered by
 * running the same seeded step on it and on its peers, and comparing their
 * times through the same summaries and the bits of their outputs, and by the
 * per-expert token counts that argus_balance gives for the job's own router.
 * The operators each bound another part of the GPU:
 *
 *   argus_embedding    token lookup with scaling (gather), and the table's
 *                      gradient by sorted tokens (sort, segmented sums)
 *   argus_layer_norm   layer norm and its gradients (memory streaming,
 *                      reductions over rows and over columns)
 *   argus_attention    softmax attention over packed documents, and its
 *                      gradients, which recompute the probabilities (matrix
 *                      instructions)
 *   argus_balance      top-k router: softmax, chosen experts, per-expert
 *                      counts and the balance loss, and its gradient
 *   argus_rotary       rotary positions of queries and keys, and their
 *                      gradient (memory streaming, 64-bit angles)
 *   argus_gated_ff     gated feed-forward block: two products, activation
 *                      and gate, and its gradients (matrix instructions;
 *                      few tokens: memory streaming)
 *   argus_cross_entropy  the loss over a large vocabulary from the last
 *                      hidden states, without the logits in memory, and its
 *                      gradients (matrix instructions)
 *
 * The conventions are those of argus.h: device pointers owned by the caller,
 * a caller workspace where the *_workspace query is not 0 (256-byte aligned,
 * not shared by calls that may overlap), asynchronous on the caller's stream,
 * a host status before any launch, ARGUS_DEV_* bits in the optional
 * *dev_status, every element of every output written, nothing kept between
 * calls. Sums, softmax statistics and means are held in 32-bit floats (the
 * balance loss in doubles) and each output is rounded once to its own type;
 * the order of every sum is fixed by the sizes and the values of ids and
 * offsets, so equal inputs give equal bits.
 *
 * Strides are counted in elements and are those of the outer dimensions; the
 * innermost dimension is always contiguous. Rows need no alignment beyond
 * their element's (attention, gated_ff and cross_entropy: 16 bytes, see
 * there), and rows that are only read may coincide (stride 0, a broadcast
 * input; not those three's). Outputs may not overlap
 * inputs or each other, except where noted.
 */
#ifndef ARGUS_OPS_H
#define ARGUS_OPS_H

#include "argus.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ARGUS_F32 = 0, ARGUS_BF16 = 1, ARGUS_F16 = 2 }; /* element types */

#define ARGUS_MAX_LN_COLS 16384    /* argus_layer_norm: columns limit */
#define ARGUS_MAX_EXPERTS 1024     /* argus_balance: experts limit */
#define ARGUS_MAX_TOP_K 16         /* argus_balance: experts per token limit */
#define ARGUS_MAX_HEAD_DIM 128     /* argus_attention: head dimension limit */
#define ARGUS_MAX_ROTARY_DIM 1024  /* argus_rotary: head dimension limit */
#define ARGUS_MAX_FF_WIDTH 65536   /* argus_gated_ff: width limit */
#define ARGUS_MAX_FF 131072        /* argus_gated_ff: inner width limit */
#define ARGUS_MAX_CE_WIDTH 16384   /* argus_cross_entropy: width limit */
#define ARGUS_MAX_CE_VOCAB 1048576 /* argus_cross_entropy: vocabulary limit */

/* ---------------------------------------------------------------- embedding
 *
 * out[t][:] = scale * table[ids[t]][:], in 32 bits, rounded once. An id below
 * 0 is padding and one at or above n_vocab is an error (ARGUS_DEV_TOKEN_RANGE
 * is raised); both give a row of zeros and no gradient.
 */
typedef struct argus_embedding {
  const void* ids;      /* [n_tokens] int32 or int64 */
  int64_t n_tokens;     /* 0 .. 2^27 */
  int32_t ids_64;       /* 1: ids are int64 */
  int32_t n_vocab;      /* 1 .. 2^27 */
  int32_t dim;          /* 1 .. 65536 */
  int32_t dtype;        /* of table, out, dout */
  int32_t grad_dtype;   /* of dtable (argus_embedding_bwd) */
  float scale;
  int64_t row_stride;   /* of table (argus_embedding) or dout (argus_embedding_bwd); >= 0 */
  int32_t* dev_status;  /* optional (may be NULL) */
} argus_embedding_t;

/* out: [n_tokens][dim], contiguous. */
int argus_embedding(const argus_embedding_t* p, const void* table, void* out, void* stream);

/* The gradient of the table: dtable[v][:] = scale * sum of dout[t][:] over
 * the tokens t with ids[t] = v, in ascending t inside fixed pieces, zeros for
 * an id that does not occur. dtable: [n_vocab][dim], contiguous; every
 * element is written. */
size_t argus_embedding_bwd_workspace(const argus_embedding_t* p);
int argus_embedding_bwd(const argus_embedding_t* p, const void* dout, void* dtable, void* workspace,
                        size_t workspace_bytes, void* stream);

/* --------------------------------------------------------------- layer norm
 *
 * Per row: mean = sum x / cols, rstd = 1 / sqrt(sum (x - mean)^2 / cols +
 * eps), y = (x - mean) * rstd * weight + bias. The squares are summed in a
 * second pass over the row in registers, not from sum x^2.
 * Backward, from the forward's mean and rstd, with xhat = (x - mean) * rstd
 * and g = dy * weight: dx = rstd * (g - mean(g) - xhat * mean(g * xhat)),
 * dweight = sum over rows of dy * xhat, dbias = sum over rows of dy.
 */
typedef struct argus_layer_norm {
  int64_t rows;         /* 0 .. 2^31 - 1 */
  int32_t cols;         /* 1 .. ARGUS_MAX_LN_COLS */
  int32_t dtype;        /* of x, y, dy, dx */
  int32_t weight_dtype; /* of weight, bias, dweight, dbias: ARGUS_F32 or dtype */
  float eps;            /* >= 0 */
  int64_t x_stride;     /* row stride of x, >= 0 */
  int64_t dy_stride;    /* row stride of dy (argus_layer_norm_bwd), >= 0 */
} argus_layer_norm_t;

/* y: [rows][cols], contiguous; mean, rstd: [rows]; bias may be NULL. */
int argus_layer_norm(const argus_layer_norm_t* p, const void* x, const void* weight, const void* bias, void* y,
                     float* mean, float* rstd, void* stream);

/* dx: [rows][cols], contiguous; dweight, dbias: [cols]; dbias may be NULL. */
size_t argus_layer_norm_bwd_workspace(const argus_layer_norm_t* p);
int argus_layer_norm_bwd(const argus_layer_norm_t* p, const void* dy, const void* x, const float* mean,
                         const float* rstd, const void* weight, void* dx, void* dweight, void* dbias,
                         void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ balance
 *
 * The router of a layer of n_experts experts. A token takes part iff its mask
 * byte is not 0 (no mask: every token) and its largest logit is finite and
 * none is NaN; one that the mask lets in and that has no finite largest logit
 * raises ARGUS_DEV_LOGITS. n = number of tokens that take part. For one that
 * does: p = softmax(logits), lse = log sum exp(logits), expert = the top_k
 * largest logits in descending order, the lowest index of equal ones first
 * (a logit of -infinity is never chosen: expert -1, gate 0), gate = p of
 * those. For one that does not: expert -1, gate 0, lse -infinity.
 *   count[e] = how often e was chosen,  prob[e] = sum over tokens of p_e / n
 *   loss = alpha * n_experts * sum over e of count[e] / (top_k n) * prob[e]
 * (prob and loss 0 when n = 0).
 * Backward, with count taken as a constant: g_e = dloss * alpha * n_experts *
 * count[e] / (top_k n^2), plus dgate[j] at e = expert[j]; dlogits = p * (g -
 * sum over e of g_e p_e), zeros for a token that does not take part (its
 * logits are not used).
 */
typedef struct argus_balance {
  int64_t n_tokens;   /* 0 .. 2^31 - 1 */
  int32_t n_experts;  /* 1 .. ARGUS_MAX_EXPERTS */
  int32_t top_k;      /* 1 .. min(n_experts, ARGUS_MAX_TOP_K) */
  int32_t dtype;      /* of logits, dlogits */
  float alpha;
  int64_t row_stride; /* of logits, >= 0 */
} argus_balance_t;

typedef struct argus_balance_out {
  int32_t* expert;     /* [n_tokens][top_k] */
  float* gate;         /* [n_tokens][top_k] */
  float* lse;          /* [n_tokens] */
  uint32_t* count;     /* [n_experts] */
  float* prob;         /* [n_experts] */
  uint32_t* n_valid;   /* [1] n */
  float* loss;         /* [1] */
  int32_t* dev_status; /* optional (may be NULL) */
} argus_balance_out_t;

/* mask: [n_tokens] or NULL. */
size_t argus_balance_workspace(const argus_balance_t* p);
int argus_balance(const argus_balance_t* p, const void* logits, const uint8_t* mask, const argus_balance_out_t* out,
                  void* workspace, size_t workspace_bytes, void* stream);

/* lse, expert, count, n_valid: outputs of argus_balance over these logits.
 * dloss: [1]; dgate: [n_tokens][top_k] or NULL; dlogits: [n_tokens]
 * [n_experts], contiguous. */
int argus_balance_bwd(const argus_balance_t* p, const void* logits, const float* lse, const int32_t* expert,
                      const uint32_t* count, const uint32_t* n_valid, const float* dloss, const float* dgate,
                      void* dlogits, void* stream);

/* ---------------------------------------------------------------- attention
 *
 * Softmax attention over packed documents: document d has the queries
 * q_off[d] .. q_off[d+1] and the keys k_off[d] .. k_off[d+1] and sees nothing
 * else. NULL offsets: one document of all tokens. Query head h uses the key
 * and value head h / (n_heads / n_kv_heads). With causal set, query i of a
 * document of a queries and b keys sees keys j <= i + b - a (the last query
 * sees the last key), so the first a - b queries of a longer query side see
 * none. Per query and head, over the keys it sees:
 *   s_j = scale q . k_j,  lse = log sum exp(s_j),  o = sum exp(s_j - lse) v_j
 * A query that sees no key has o = 0, lse = -infinity and no gradient.
 * Backward, from q, k, v, o, lse and do: P_ij = exp(s_ij - lse_i),
 * dS_ij = P_ij (do_i . v_j - do_i . o_i), dq_i = scale sum_j dS_ij k_j,
 * dk_j = scale sum_i dS_ij q_i, dv_j = sum_i P_ij do_i, the last two summed
 * over the query heads of a key head as well. The products run on bfloat16
 * matrix instructions with 32-bit sums; P and dS are rounded to bfloat16 as
 * their operands.
 *
 * Offsets are read on the device: unless off[0] = 0, the offsets ascend and
 * off[n_docs] is the number of tokens, for both sides, ARGUS_DEV_BAD_SEGMENT
 * is raised and every query is taken to see no key.
 *
 * A query or key row that holds a NaN makes lse, o and dq of the queries that
 * see it NaN, and by them dk and dv of all keys these see.
 * A value row of a document that holds a NaN or an infinity may reach those
 * of its queries that do not see it under the causal mask. Backward, such a
 * key or value row may reach their dq, and such a row of q, o, d_o or lse the
 * dk and dv of keys that the query does not see. Nothing reaches the outputs of
 * a query that sees no key, nor passes from its row to a key, nor from one
 * document to another.
 */
typedef struct argus_attention {
  int32_t n_docs;      /* >= 1 */
  int32_t n_heads;     /* >= 1, a multiple of n_kv_heads; <= 65535 */
  int32_t n_kv_heads;  /* >= 1 */
  int32_t head_dim;    /* a multiple of 8, 8 .. ARGUS_MAX_HEAD_DIM */
  int32_t causal;      /* 0 or 1 */
  int32_t dtype;       /* ARGUS_BF16 */
  float scale;         /* finite, >= 0 */
  int64_t n_q, n_k;    /* tokens of all documents, 0 .. 2^30; (tokens / 128 + n_docs) times the heads below 2^23 */
  const int64_t* q_off; /* [n_docs + 1] or NULL (then k_off is NULL and n_docs 1) */
  const int64_t* k_off; /* [n_docs + 1] or NULL */
  /* strides of the token and head dimensions: multiples of 8, at least
   * head_dim, at most 2^21 (tokens) and 2^40 (heads); all pointers to vectors
   * are 16-byte aligned */
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;
  int32_t* dev_status; /* optional (may be NULL) */
} argus_attention_t;

/* o: [n_q][n_heads][head_dim], contiguous; lse: [n_q][n_heads]. */
size_t argus_attention_workspace(const argus_attention_t* p);
int argus_attention(const argus_attention_t* p, const void* q, const void* k, const void* v, void* o, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream);

/* d_o and o: [n_q][n_heads][head_dim], contiguous; lse: [n_q][n_heads];
 * dq like o; dk, dv: [n_k][n_kv_heads][head_dim], contiguous. */
size_t argus_attention_bwd_workspace(const argus_attention_t* p);
int argus_attention_bwd(const argus_attention_t* p, const void* d_o, const void* q, const void* k, const void* v,
                        const void* o, const float* lse, void* dq, void* dk, void* dv, void* workspace,
                        size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------- rotary
 *
 * Pair i of a token's head, i = 0 .. rot_dim / 2 - 1, is (x[i], x[i + rot_dim
 * / 2]), or with interleaved set (x[2 i], x[2 i + 1]). With the angle a = pos
 * freq[i], (u, v) becomes scale (u cos a - v sin a, u sin a + v cos a), in 32
 * bits, rounded once; with inverse set a is taken as -a, which is the
 * gradient's direction (the map's transpose). Elements from rot_dim on are
 * copied. pos freq[i] / 2 pi is taken in 64 bits and its fraction alone goes
 * on: positions up to 2^31 in size turn right to 1e-6 of a radian.
 */
typedef struct argus_rotary {
  int64_t n_tokens;    /* 0 .. 2^28 */
  int32_t n_heads;     /* 1 .. 65535 */
  int32_t head_dim;    /* 2 .. ARGUS_MAX_ROTARY_DIM */
  int32_t rot_dim;     /* even, 2 .. head_dim */
  int32_t interleaved; /* 0 or 1 */
  int32_t inverse;     /* 0 or 1 */
  int32_t dtype;       /* of x, out */
  float scale;         /* finite */
  int32_t pos_64;      /* 1: pos is int64 */
  const void* pos;     /* [n_tokens] int32 or int64, or NULL: 0, 1, 2, .. */
  const double* freq;  /* [rot_dim / 2] radians a position */
  int64_t x_tok, x_head;     /* strides of x, >= 0 */
  int64_t out_tok, out_head; /* strides of out; heads and tokens may not overlap */
} argus_rotary_t;

/* out may be x with the same strides. */
int argus_rotary(const argus_rotary_t* p, const void* x, void* out, void* stream);

/* ----------------------------------------------------------------- gated_ff
 *
 * g = x wg^T, u = x wu^T, h = act(g) u, with act(g) = g / (1 + exp(-g))
 * (ARGUS_SILU), g Phi(g) with the normal distribution's Phi (ARGUS_GELU), or
 * g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2 (ARGUS_GELU_TANH). The
 * products have 32-bit sums, h is made of those and rounded once.
 * Backward, from the rounded g and u: dg = d_h u act'(g), du = d_h act(g),
 * both rounded to dtype as operands (in float16 times a power of two that puts
 * the largest of them below 2^15); dx = dg wg + du wu, dwg = dg^T x,
 * dwu = du^T x. A row of x or d_h that holds a NaN or an infinity reaches its own
 * token's rows and the weights' gradients alone.
 */
enum { ARGUS_SILU = 0, ARGUS_GELU = 1, ARGUS_GELU_TANH = 2 };

typedef struct argus_gated_ff {
  int64_t n_tokens; /* 0 .. 2^20 */
  int32_t width;    /* a multiple of 8, 8 .. ARGUS_MAX_FF_WIDTH */
  int32_t ff;       /* a multiple of 8, 8 .. ARGUS_MAX_FF */
  int32_t dtype;    /* ARGUS_BF16 or ARGUS_F16, of every tensor */
  int32_t act;
  /* row strides: multiples of 8, at least the row's length, at most 2^21; all
   * pointers to tensors are 16-byte aligned */
  int64_t x_stride, wg_stride, wu_stride;
  int64_t dh_stride; /* of d_h (argus_gated_ff_bwd) */
} argus_gated_ff_t;

/* x: [n_tokens][width]; wg, wu: [ff][width]; h: [n_tokens][ff], contiguous;
 * g, u: like h, or both NULL where no backward pass follows. */
size_t argus_gated_ff_workspace(const argus_gated_ff_t* p);
int argus_gated_ff(const argus_gated_ff_t* p, const void* x, const void* wg, const void* wu, void* h, void* g, void* u,
                   void* workspace, size_t workspace_bytes, void* stream);

/* d_h: [n_tokens][ff]; g, u: the forward's, contiguous; dx: [n_tokens]
 * [width], dwg, dwu: [ff][width], contiguous. */
size_t argus_gated_ff_bwd_workspace(const argus_gated_ff_t* p);
int argus_gated_ff_bwd(const argus_gated_ff_t* p, const void* d_h, const void* x, const void* wg, const void* wu,
                       const void* g, const void* u, void* dx, void* dwg, void* dwu, void* workspace,
                       size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------ cross_entropy
 *
 * Per token: z = scale x w^T over the vocabulary, lse = log sum exp(z), loss =
 * lse - z[label] + z_loss lse^2; mean = sum of loss / n_valid, n_valid the
 * number of tokens that are learned (mean 0 if none). A token whose label is
 * below 0 is not learned; one whose label is at or above n_vocab neither, and
 * raises ARGUS_DEV_TOKEN_RANGE: loss 0, lse -infinity, and no gradient,
 * whatever their rows of x hold. The logits are not kept. A NaN among a learned
 * token's logits, or one of +infinity, makes its lse and loss, and by them the
 * mean, NaN; one of -infinity counts as an exponential of 0.
 * Backward, with c = dmean / max(n_valid, 1) + dloss[token] for a token that
 * is learned: dz[v] = c scale (exp(z[v] - lse) (1 + 2 z_loss lse) - [v =
 * label]), rounded to bfloat16 as an operand; dx = dz w, dw = dz^T x. n_valid
 * divides dmean alone: with tokens on several ranks it may be their total.
 */
typedef struct argus_cross_entropy {
  const void* labels; /* [n_tokens] int32 or int64 */
  int64_t n_tokens;   /* 0 .. 2^20; n_tokens n_vocab below 2^38 */
  int32_t ids_64;     /* 1: labels are int64 */
  int32_t n_vocab;    /* 1 .. ARGUS_MAX_CE_VOCAB */
  int32_t width;      /* a multiple of 8, 8 .. ARGUS_MAX_CE_WIDTH */
  int32_t dtype;      /* ARGUS_BF16, of x, w, dx, dw */
  float scale;        /* finite */
  float z_loss;       /* finite, >= 0 */
  /* row strides: multiples of 8, at least width, at most 2^21; all pointers to
   * tensors are 16-byte aligned */
  int64_t x_stride, w_stride;
} argus_cross_entropy_t;

typedef struct argus_cross_entropy_out {
  float* loss;         /* [n_tokens] */
  float* lse;          /* [n_tokens] */
  float* mean;         /* [1] */
  uint32_t* n_valid;   /* [1] */
  int32_t* dev_status; /* optional (may be NULL) */
} argus_cross_entropy_out_t;

/* x: [n_tokens][width]; w: [n_vocab][width]. */
size_t argus_cross_entropy_workspace(const argus_cross_entropy_t* p);
int argus_cross_entropy(const argus_cross_entropy_t* p, const void* x, const void* w,
                        const argus_cross_entropy_out_t* out, void* workspace, size_t workspace_bytes, void* stream);

/* lse: the forward's; dmean: [1], with n_valid [1], or NULL; dloss: [n_tokens]
 * or NULL; one of the two has to be there. dx: [n_tokens][width], dw: [n_vocab]
 * [width], contiguous; dev_status: optional. */
size_t argus_cross_entropy_bwd_workspace(const argus_cross_entropy_t* p);
int argus_cross_entropy_bwd(const argus_cross_entropy_t* p, const void* x, const void* w, const float* lse,
                            const uint32_t* n_valid, const float* dmean, const float* dloss, void* dx, void* dw,
                            int32_t* dev_status, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ARGUS_OPS_H */
