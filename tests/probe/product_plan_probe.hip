// Host code only: how the matrix products of paper_2606_20374_amd/csrc/product.h
// and cross_entropy_plan.h are taken for a size.
#include "../../paper_2606_20374_amd/csrc/cross_entropy_plan.h"

using namespace argus::product;

namespace {
struct Chosen {
  int32_t tm, tn, threads, stages;
};
template <class T, int TM, int TN, int WM, int WN, bool A, bool B, int STAGES>
Chosen chosen(Tile<T, TM, TN, WM, WN, A, B, STAGES>*) { return {TM, TN, 64 * WM * WN, STAGES}; }
}  // namespace

extern "C" {

// out: rows, columns, threads and stages of the tile of a forward product; loss:
// of the cross entropy's logits; three: with feed-forward's three outputs.
void probe_forward_tile(int64_t rows, int64_t cols, int64_t k, int32_t loss, int32_t three, int32_t* out) {
  auto go = [](auto tile) { return chosen((decltype(tile)*)nullptr); };
  const Chosen c = loss ? with_tile<argus::bf16_t, true>(rows, cols, k, false, go)
                        : with_tile<argus::bf16_t, false>(rows, cols, k, three != 0, go);
  out[0] = c.tm;
  out[1] = c.tn;
  out[2] = c.threads;
  out[3] = c.stages;
}

// out: rows of a tile, whether it has four stages, parts of k of the input's and
// of the weights' gradient, threads, and workgroups of the launch.
void probe_gradient_plan(int64_t rows_x, int64_t k_x, int64_t rows_w, int64_t k_w, int64_t cols, int64_t* out) {
  const Plan p = plan_grads(rows_x, k_x, rows_w, k_w, cols);
  out[0] = p.tile();
  out[1] = p.deep;
  out[2] = p.x.S;
  out[3] = p.w.S;
  out[4] = p.big ? Big<argus::bf16_t, true, false>::THREADS : Small<argus::bf16_t, true, false>::THREADS;
  out[5] = (int64_t)p.x.mt * p.x.nt * p.x.S + (int64_t)p.w.mt * p.w.nt * p.w.S;
}

// out: whether tokens are few, whether they are not numbered, and the ids of a
// piece of the vocabulary.
void probe_loss_call(int64_t tokens, int32_t vocab, int32_t width, int64_t* out) {
  argus_cross_entropy_t p{};
  p.n_tokens = tokens;
  p.n_vocab = vocab;
  p.width = width;
  out[0] = is_few(p);
  out[1] = is_small(p);
  out[2] = piece_of(p);
}

}  // extern "C"
