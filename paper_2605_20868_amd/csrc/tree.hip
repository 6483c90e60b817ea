// Attention of drafted tokens (a tree, or a chunk of a prompt) over the quantized cache: the calls.  Kernels in tree_inl.h.
#include "tree_inl.h"

namespace cqa {

int64_t tree_ws_bytes(const Cache* c, int n_draft) {
  const int64_t heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  const int n_rows = n_draft * (c->desc.n_q_heads / c->desc.n_kv_heads);
  const auto most = [&](int rows) { return tree_splits(c->n_cu, heads, n_rows, rows, c->desc.max_tokens, n_draft + BLK - 1); };
  const int64_t sets = std::max(most(32), most(n_rows <= 64 ? 64 : (n_rows <= 128 ? 128 : 256)));
  return heads * ((n_rows + 31) / 32) * sets * T_FLOATS * 4;
}

int32_t launch_tree(const Cache* c, int layer, const __half* q, const __half* kd, const __half* vd, int n_draft, const uint64_t* mask,
                    const cqa_tolerances& tol, __half* O, cqa_node_cert* cert, uint32_t* flags, float* ws, hipStream_t st) {
  const int64_t head0 = head_index(c, layer, 0, 0);
  const int64_t heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  TreeArgs a;
  a.t1 = c->t1 + head0 * c->nq_cap * QUAD_BYTES;
  a.trail_k = c->trail_k + head0 * BLK * D;
  a.trail_v = c->trail_v + head0 * BLK * D;
  a.q = q;
  a.kd = kd;
  a.vd = vd;
  a.mask = mask;
  a.part = ws;
  a.nq_cap = c->nq_cap;
  a.nb = c->length[layer] / BLK;
  a.n = n_draft;
  a.words = (n_draft + 63) / 64;
  a.trail = (int)(c->length[layer] % BLK);
  a.n_kv = c->desc.n_kv_heads;
  a.group = c->desc.n_q_heads / c->desc.n_kv_heads;
  const int n_rows = n_draft * a.group;
  a.row_tiles = (n_rows + 31) / 32;
  const int rows = tree_rows(c->n_cu, heads, n_rows, a.nb * BLK, a.trail + a.n);
  a.nsplit = tree_splits(c->n_cu, heads, n_rows, rows, a.nb * BLK, a.trail + a.n);
  if (rows > 32) put_shares(a, rows, a.trail + a.n);
  a.O = O;
  a.cert = cert;
  a.flags = flags;
  a.tol = tol;
  if (const int32_t rc = launch_pass(a, heads, rows, a.trail + a.n, st)) return rc;
  return a.nsplit == 1 ? CQA_OK : launch_join(a, heads, a.nsplit, c->n_cu, st);
}

}  // namespace cqa
