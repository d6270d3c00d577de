// C-ABI host wrapper of the step operators: argument checks and launches on
// the caller's stream. See include/argus_ops.h for the contract.
#include <cmath>

#include "ops_internal.h"

namespace argus {
namespace {

bool bad_dtype(int32_t d) { return d != ARGUS_F32 && d != ARGUS_BF16 && d != ARGUS_F16; }
uintptr_t size_of(int32_t d) { return d == ARGUS_F32 ? 4 : 2; }
bool misaligned(const void* q, uintptr_t m) { return (reinterpret_cast<uintptr_t>(q) & (m - 1)) != 0; }
bool bad_workspace(const void* ws, size_t have, size_t need) {
  return need > 0 && (!ws || misaligned(ws, 256) || have < need);
}

bool bad_embedding(const argus_embedding_t* p) {
  if (!p || p->n_tokens < 0 || p->n_tokens > (1 << 27) || p->n_vocab < 1 || p->n_vocab > (1 << 27) || p->dim < 1 ||
      p->dim > (1 << 16))
    return true;
  if (bad_dtype(p->dtype) || p->row_stride < 0 || !std::isfinite(p->scale)) return true;
  if (p->ids_64 != 0 && p->ids_64 != 1) return true;
  if (misaligned(p->dev_status, 4)) return true;
  return p->n_tokens > 0 && (!p->ids || misaligned(p->ids, p->ids_64 ? 8 : 4));
}

bool bad_grad_dtype(const argus_embedding_t* p) {
  return p->grad_dtype != ARGUS_F32 && p->grad_dtype != p->dtype;
}

bool bad_layer_norm(const argus_layer_norm_t* p) {
  if (!p || p->rows < 0 || p->rows > INT32_MAX || p->cols < 1 || p->cols > ARGUS_MAX_LN_COLS) return true;
  if (bad_dtype(p->dtype) || (p->weight_dtype != ARGUS_F32 && p->weight_dtype != p->dtype)) return true;
  return !(p->eps >= 0.0f) || !std::isfinite(p->eps) || p->x_stride < 0;
}

bool bad_balance(const argus_balance_t* p) {
  if (!p || p->n_tokens < 0 || p->n_tokens > INT32_MAX || p->n_experts < 1 || p->n_experts > ARGUS_MAX_EXPERTS)
    return true;
  if (p->top_k < 1 || p->top_k > ARGUS_MAX_TOP_K || p->top_k > p->n_experts) return true;
  return bad_dtype(p->dtype) || p->row_stride < 0 || !std::isfinite(p->alpha);
}

bool bad_attention(const argus_attention_t* p) {
  if (!p || p->n_docs < 1 || p->n_heads < 1 || p->n_heads > 65535 || p->n_kv_heads < 1 ||
      p->n_heads % p->n_kv_heads != 0)
    return true;
  if (p->head_dim < 8 || p->head_dim > ARGUS_MAX_HEAD_DIM || p->head_dim % 8 != 0) return true;
  if ((p->causal != 0 && p->causal != 1) || p->dtype != ARGUS_BF16) return true;
  if (!(p->scale >= 0.0f) || !std::isfinite(p->scale)) return true;
  if (p->n_q < 0 || p->n_q > (1 << 30) || p->n_k < 0 || p->n_k > (1 << 30)) return true;
  if ((p->q_off == nullptr) != (p->k_off == nullptr) || (!p->q_off && p->n_docs != 1)) return true;
  if (misaligned(p->q_off, 8) || misaligned(p->k_off, 8) || misaligned(p->dev_status, 4)) return true;
  // one launch takes all tiles of all heads
  if ((p->n_q / 128 + p->n_docs) * p->n_heads >= (1 << 23) || (p->n_k / 128 + p->n_docs) * p->n_kv_heads >= (1 << 23))
    return true;
  // a tile's rows are addressed with 32-bit offsets from its first one
  for (int64_t x : {p->q_tok, p->k_tok, p->v_tok})
    if (x < p->head_dim || x % 8 != 0 || x > (1 << 21)) return true;
  for (int64_t x : {p->q_head, p->k_head, p->v_head})
    if (x < p->head_dim || x % 8 != 0 || x > ((int64_t)1 << 40)) return true;
  return false;
}

bool bad_rotary(const argus_rotary_t* p) {
  if (!p || p->n_tokens < 0 || p->n_tokens > (1 << 28) || p->n_heads < 1 || p->n_heads > 65535) return true;
  if (p->head_dim < 2 || p->head_dim > ARGUS_MAX_ROTARY_DIM || p->rot_dim < 2 || p->rot_dim > p->head_dim ||
      p->rot_dim % 2 != 0)
    return true;
  for (int32_t flag : {p->interleaved, p->inverse, p->pos_64})
    if (flag != 0 && flag != 1) return true;
  if (bad_dtype(p->dtype) || !std::isfinite(p->scale)) return true;
  if (misaligned(p->pos, p->pos_64 ? 8 : 4) || !p->freq || misaligned(p->freq, 8)) return true;
  // a written head may not reach into another: heads inside a token, or tokens inside a head
  if (p->x_tok < 0 || p->x_head < 0 || p->out_tok < 0 || p->out_head < 0) return true;
  const int64_t T = p->n_tokens, H = p->n_heads, D = p->head_dim;
  if ((H > 1 && p->out_head < D) || (T > 1 && p->out_tok < D)) return true;
  const unsigned __int128 heads = (unsigned __int128)(H - 1) * p->out_head + D,
                          tokens = T > 0 ? (unsigned __int128)(T - 1) * p->out_tok + D : D;
  return H > 1 && T > 1 && (unsigned __int128)p->out_tok < heads && (unsigned __int128)p->out_head < tokens;
}

// Rows for the matrix products: strides in elements that 16-byte pieces divide.
bool bad_rows(int64_t stride, int64_t cols) { return stride < cols || stride % 8 != 0 || stride > (1 << 21); }

bool bad_gated_ff(const argus_gated_ff_t* p) {
  if (!p || p->n_tokens < 0 || p->n_tokens > (1 << 20)) return true;
  if (p->width < 8 || p->width > ARGUS_MAX_FF_WIDTH || p->width % 8 != 0) return true;
  if (p->ff < 8 || p->ff > ARGUS_MAX_FF || p->ff % 8 != 0) return true;
  if (p->dtype != ARGUS_BF16 && p->dtype != ARGUS_F16) return true;
  if (p->act < ARGUS_SILU || p->act > ARGUS_GELU_TANH) return true;
  return bad_rows(p->x_stride, p->width) || bad_rows(p->wg_stride, p->width) || bad_rows(p->wu_stride, p->width);
}

bool bad_cross_entropy(const argus_cross_entropy_t* p) {
  if (!p || p->n_tokens < 0 || p->n_tokens > (1 << 20) || p->n_vocab < 1 || p->n_vocab > ARGUS_MAX_CE_VOCAB) return true;
  if (p->n_tokens * p->n_vocab >= ((int64_t)1 << 38)) return true;
  if (p->width < 8 || p->width > ARGUS_MAX_CE_WIDTH || p->width % 8 != 0) return true;
  if (p->dtype != ARGUS_BF16 || (p->ids_64 != 0 && p->ids_64 != 1)) return true;
  if (!std::isfinite(p->scale) || !std::isfinite(p->z_loss) || p->z_loss < 0.0f) return true;
  if (p->n_tokens > 0 && (!p->labels || misaligned(p->labels, p->ids_64 ? 8 : 4))) return true;
  return bad_rows(p->x_stride, p->width) || bad_rows(p->w_stride, p->width);
}

}  // namespace
}  // namespace argus

using namespace argus;

extern "C" {

int argus_embedding(const argus_embedding_t* p, const void* table, void* out, void* stream) {
  if (bad_embedding(p)) return ARGUS_EINVAL;
  const uintptr_t s = size_of(p->dtype);
  if (!table || misaligned(table, s) || (p->n_tokens > 0 && (!out || misaligned(out, s)))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_embedding(*p, table, out, (hipStream_t)stream));
}

size_t argus_embedding_bwd_workspace(const argus_embedding_t* p) {
  if (!p || p->n_tokens < 0 || p->n_tokens > (1 << 27) || p->n_vocab < 1 || p->dim < 1 || p->dim > (1 << 16))
    return 0;
  return embedding_bwd_workspace_bytes(*p);
}

int argus_embedding_bwd(const argus_embedding_t* p, const void* dout, void* dtable, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (bad_embedding(p) || bad_grad_dtype(p)) return ARGUS_EINVAL;
  if (!dtable || misaligned(dtable, size_of(p->grad_dtype))) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!dout || misaligned(dout, size_of(p->dtype)))) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_embedding_bwd_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_embedding_bwd(*p, dout, dtable, workspace, (hipStream_t)stream));
}

int argus_layer_norm(const argus_layer_norm_t* p, const void* x, const void* weight, const void* bias, void* y,
                     float* mean, float* rstd, void* stream) {
  if (bad_layer_norm(p)) return ARGUS_EINVAL;
  const uintptr_t s = size_of(p->dtype), w = size_of(p->weight_dtype);
  if (!weight || misaligned(weight, w) || misaligned(bias, w)) return ARGUS_EINVAL;
  if (p->rows > 0 && (!x || !y || !mean || !rstd)) return ARGUS_EINVAL;
  if (misaligned(x, s) || misaligned(y, s) || misaligned(mean, 4) || misaligned(rstd, 4)) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_layer_norm(*p, x, weight, bias, y, mean, rstd, (hipStream_t)stream));
}

size_t argus_layer_norm_bwd_workspace(const argus_layer_norm_t* p) {
  if (!p || p->rows < 0 || p->cols < 1 || p->cols > ARGUS_MAX_LN_COLS || bad_dtype(p->dtype)) return 0;
  return layer_norm_bwd_workspace_bytes(*p);
}

int argus_layer_norm_bwd(const argus_layer_norm_t* p, const void* dy, const void* x, const float* mean,
                         const float* rstd, const void* weight, void* dx, void* dweight, void* dbias,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_layer_norm(p) || p->dy_stride < 0) return ARGUS_EINVAL;
  const uintptr_t s = size_of(p->dtype), w = size_of(p->weight_dtype);
  if (!weight || !dweight || misaligned(weight, w) || misaligned(dweight, w) || misaligned(dbias, w))
    return ARGUS_EINVAL;
  if (p->rows > 0 && (!dy || !x || !mean || !rstd || !dx)) return ARGUS_EINVAL;
  if (misaligned(dy, s) || misaligned(x, s) || misaligned(dx, s) || misaligned(mean, 4) || misaligned(rstd, 4))
    return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_layer_norm_bwd_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_layer_norm_bwd(*p, dy, x, mean, rstd, weight, dx, dweight, dbias, workspace,
                                         (hipStream_t)stream));
}

size_t argus_balance_workspace(const argus_balance_t* p) {
  return bad_balance(p) ? 0 : balance_workspace_bytes(*p);
}

int argus_balance(const argus_balance_t* p, const void* logits, const uint8_t* mask, const argus_balance_out_t* out,
                  void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_balance(p) || !out) return ARGUS_EINVAL;
  const argus_balance_out_t& o = *out;
  if (!o.count || !o.prob || !o.n_valid || !o.loss) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!logits || !o.expert || !o.gate || !o.lse)) return ARGUS_EINVAL;
  if (misaligned(logits, size_of(p->dtype))) return ARGUS_EINVAL;
  const void* ptrs[8] = {o.expert, o.gate, o.lse, o.count, o.prob, o.n_valid, o.loss, o.dev_status};
  for (const void* x : ptrs)
    if (misaligned(x, 4)) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_balance_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_balance(*p, logits, mask, o, workspace, (hipStream_t)stream));
}

int argus_balance_bwd(const argus_balance_t* p, const void* logits, const float* lse, const int32_t* expert,
                      const uint32_t* count, const uint32_t* n_valid, const float* dloss, const float* dgate,
                      void* dlogits, void* stream) {
  if (bad_balance(p) || !count || !n_valid || !dloss) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!logits || !lse || !dlogits || (dgate && !expert))) return ARGUS_EINVAL;
  if (misaligned(logits, size_of(p->dtype)) || misaligned(dlogits, size_of(p->dtype))) return ARGUS_EINVAL;
  const void* ptrs[6] = {lse, expert, count, n_valid, dloss, dgate};
  for (const void* x : ptrs)
    if (misaligned(x, 4)) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_balance_bwd(*p, logits, lse, expert, count, n_valid, dloss, dgate, dlogits,
                                      (hipStream_t)stream));
}

size_t argus_attention_workspace(const argus_attention_t* p) {
  return bad_attention(p) ? 0 : attention_workspace_bytes(*p);
}

int argus_attention(const argus_attention_t* p, const void* q, const void* k, const void* v, void* o, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_attention(p)) return ARGUS_EINVAL;
  if ((p->n_q > 0 && (!q || !o || !lse)) || (p->n_k > 0 && (!k || !v))) return ARGUS_EINVAL;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(o, 16) || misaligned(lse, 4))
    return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_attention_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_attention(*p, q, k, v, o, lse, workspace, (hipStream_t)stream));
}

size_t argus_attention_bwd_workspace(const argus_attention_t* p) {
  return bad_attention(p) ? 0 : attention_bwd_workspace_bytes(*p);
}

int argus_attention_bwd(const argus_attention_t* p, const void* d_o, const void* q, const void* k, const void* v,
                        const void* o, const float* lse, void* dq, void* dk, void* dv, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (bad_attention(p)) return ARGUS_EINVAL;
  if (p->n_q > 0 && (!d_o || !q || !o || !lse || !dq)) return ARGUS_EINVAL;
  if (p->n_k > 0 && (!k || !v || !dk || !dv)) return ARGUS_EINVAL;
  const void* ptrs[8] = {d_o, q, k, v, o, dq, dk, dv};
  for (const void* x : ptrs)
    if (misaligned(x, 16)) return ARGUS_EINVAL;
  if (misaligned(lse, 4)) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_attention_bwd_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_attention_bwd(*p, d_o, q, k, v, o, lse, dq, dk, dv, workspace, (hipStream_t)stream));
}

int argus_rotary(const argus_rotary_t* p, const void* x, void* out, void* stream) {
  if (bad_rotary(p)) return ARGUS_EINVAL;
  const uintptr_t s = size_of(p->dtype);
  if (p->n_tokens > 0 && (!x || !out)) return ARGUS_EINVAL;
  if (misaligned(x, s) || misaligned(out, s)) return ARGUS_EINVAL;
  if (x == out && (p->x_tok != p->out_tok || p->x_head != p->out_head)) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_rotary(*p, x, out, (hipStream_t)stream));
}

size_t argus_gated_ff_workspace(const argus_gated_ff_t* p) { return bad_gated_ff(p) ? 0 : gated_ff_workspace_bytes(*p); }

int argus_gated_ff(const argus_gated_ff_t* p, const void* x, const void* wg, const void* wu, void* h, void* g, void* u,
                   void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_gated_ff(p) || !wg || !wu || (g == nullptr) != (u == nullptr)) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!x || !h)) return ARGUS_EINVAL;
  const void* ptrs[6] = {x, wg, wu, h, g, u};
  for (const void* q : ptrs)
    if (misaligned(q, 16)) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_gated_ff_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_gated_ff(*p, x, wg, wu, h, g, u, workspace, (hipStream_t)stream));
}

size_t argus_gated_ff_bwd_workspace(const argus_gated_ff_t* p) {
  return bad_gated_ff(p) ? 0 : gated_ff_bwd_workspace_bytes(*p);
}

int argus_gated_ff_bwd(const argus_gated_ff_t* p, const void* d_h, const void* x, const void* wg, const void* wu,
                       const void* g, const void* u, void* dx, void* dwg, void* dwu, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (bad_gated_ff(p) || bad_rows(p->dh_stride, p->ff) || !wg || !wu || !dwg || !dwu) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!d_h || !x || !g || !u || !dx)) return ARGUS_EINVAL;
  const void* ptrs[9] = {d_h, x, wg, wu, g, u, dx, dwg, dwu};
  for (const void* q : ptrs)
    if (misaligned(q, 16)) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_gated_ff_bwd_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_gated_ff_bwd(*p, d_h, x, wg, wu, g, u, dx, dwg, dwu, workspace, (hipStream_t)stream));
}

size_t argus_cross_entropy_workspace(const argus_cross_entropy_t* p) {
  return bad_cross_entropy(p) ? 0 : cross_entropy_workspace_bytes(*p);
}

int argus_cross_entropy(const argus_cross_entropy_t* p, const void* x, const void* w,
                        const argus_cross_entropy_out_t* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_cross_entropy(p) || !w || !out || !out->mean || !out->n_valid) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!x || !out->loss || !out->lse)) return ARGUS_EINVAL;
  if (misaligned(x, 16) || misaligned(w, 16)) return ARGUS_EINVAL;
  const void* ptrs[5] = {out->loss, out->lse, out->mean, out->n_valid, out->dev_status};
  for (const void* q : ptrs)
    if (misaligned(q, 4)) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_cross_entropy_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_cross_entropy(*p, x, w, *out, workspace, (hipStream_t)stream));
}

size_t argus_cross_entropy_bwd_workspace(const argus_cross_entropy_t* p) {
  return bad_cross_entropy(p) ? 0 : cross_entropy_bwd_workspace_bytes(*p);
}

int argus_cross_entropy_bwd(const argus_cross_entropy_t* p, const void* x, const void* w, const float* lse,
                            const uint32_t* n_valid, const float* dmean, const float* dloss, void* dx, void* dw,
                            int32_t* dev_status, void* workspace, size_t workspace_bytes, void* stream) {
  if (bad_cross_entropy(p) || !w || !dw || (!dmean && !dloss) || (dmean && !n_valid)) return ARGUS_EINVAL;
  if (p->n_tokens > 0 && (!x || !lse || !dx)) return ARGUS_EINVAL;
  for (const void* q : {x, w, (const void*)dx, (const void*)dw})
    if (misaligned(q, 16)) return ARGUS_EINVAL;
  for (const void* q : {(const void*)lse, (const void*)n_valid, (const void*)dmean, (const void*)dloss, (const void*)dev_status})
    if (misaligned(q, 4)) return ARGUS_EINVAL;
  if (bad_workspace(workspace, workspace_bytes, argus_cross_entropy_bwd_workspace(p))) return ARGUS_EINVAL;
  const int rc = check_device();
  if (rc != ARGUS_OK) return rc;
  return status_of(launch_cross_entropy_bwd(*p, x, w, lse, n_valid, dmean, dloss, dx, dw, dev_status, workspace,
                                            (hipStream_t)stream));
}

}  // extern "C"
