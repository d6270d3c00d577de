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

}  // extern "C"
