// How the cross entropy takes a call: by size alone, on the host.
#pragma once

#include "product.h"

namespace argus {
namespace product {

// Ids that one workgroup of the forward product takes. Few tokens: enough to
// join a token's sums in a few steps, yet enough workgroups.
inline int few_ids(const argus_cross_entropy_t& p) { return p.n_vocab >= 65536 ? 128 : 32; }
inline bool is_few(const argus_cross_entropy_t& p) { return p.n_tokens <= kFew; }
// Numbering the tokens costs two launches, about 10 us; taking them all costs at
// most 4 G multiplications, about that.
inline bool is_small(const argus_cross_entropy_t& p) {
  return is_few(p) || (p.n_tokens <= 1024 && p.n_tokens * p.n_vocab * p.width <= (int64_t)1 << 32);
}
inline int64_t tiles_n(const argus_cross_entropy_t& p) {
  return ceil_div(p.n_vocab, is_few(p) ? few_ids(p) : kind_of(p.n_tokens, p.n_vocab, p.width, kLoss) == kBig ? 256 : 128);
}
// Ids of a piece: at most 2^27 values of dz where the tokens allow it, and as
// many in all pieces as tiles allow.
inline int64_t piece_of(const argus_cross_entropy_t& p) {
  int64_t ids = ((int64_t)1 << 27) / (p.n_tokens > 0 ? p.n_tokens : 1) / 256 * 256;
  if (ids < 4096) ids = 4096;
  const int64_t all = ceil_div(p.n_vocab, 64) * 64;
  return ids < all ? ceil_div(ceil_div(p.n_vocab, ceil_div(p.n_vocab, ids)), 256) * 256 : all;
}
// The gradients' products of a piece.
inline Plan plan_of(const argus_cross_entropy_t& p) {
  const int64_t ids = piece_of(p);
  return plan_grads(p.n_tokens > 0 ? p.n_tokens : 1, ids, ids, p.n_tokens, p.width);
}

}  // namespace product
}  // namespace argus
