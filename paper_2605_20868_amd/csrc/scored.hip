// Attention of nodes with scores of the caller's (a scale, a cap, a bias by distance, spans of cached tokens), and of nodes whose sequences share a
// beginning that is cached once: the calls.  Kernels in tree_inl.h.
//
// A beginning's cached tokens are one sequence for all who share it: their nodes are its rows, so that it is read and reconstructed once for up to 256 of
// them instead of once a sequence.  A pass over it and one over the sequences' own tokens leave partial sets, which one launch joins.
#include "light_inl.h"

namespace cqa {

// A row's sets of two passes: those of the beginning's, by whose rows the launch goes, then those of the sequence's own.
struct SetsOfTwo {
  SetsOf one, two;
  __device__ __forceinline__ int count() const { return one.n + two.n; }
  __device__ __forceinline__ const float* set(int i, int& r32) const {
    const bool first = i < one.n;
    r32 = first ? one.r32 : two.r32;
    return (first ? one.sets : two.sets) + (int64_t)(first ? i : i - one.n) * T_FLOATS;
  }
  __device__ __forceinline__ float quantity(int i, int t) const {
    int r;
    const float* const p = set(i, r);
    return p[T_OFLOATS + t * T_ROWS + r];
  }
  __device__ __forceinline__ float4 channels(int i, int c) const {
    int r;
    const float* const p = set(i, r);
    return reinterpret_cast<const float4*>(p)[c * T_ROWS + r];
  }
};
template <Scores SCORES>
struct JoinArgs : SetArgs<SCORES> {
  const float* own;              // the sequences' own sets [Bt * Hkv][own_tiles][own_sets][T_FLOATS]
  int own_tiles, own_sets;
  __device__ SetsOfTwo sets_of(const float* sets, int head, int r32, int r) const {
    r = min(r, this->n * this->group - 1);
    const int b = head / this->n_kv, kvh = head - b * this->n_kv;
    const int node = r / this->group, seq = node / this->each, row = (node - seq * this->each) * this->group + (r - node * this->group);
    const int64_t own_head = ((int64_t)b * (this->n / this->each) + seq) * this->n_kv + kvh;
    return {SetsOf{sets, T_FLOATS, this->nsplit, r32}, SetsOf{own + (own_head * own_tiles + row / T_ROWS) * own_sets * T_FLOATS, T_FLOATS, own_sets, row % T_ROWS}};
  }
};

static int row_count(const Cache* c, int64_t nodes) { return (int)(nodes * (c->desc.n_q_heads / c->desc.n_kv_heads)); }
// Rows of a KV group a workgroup takes, and the partial sets of a row.
struct Shape {
  int rows, nsplit;
};
static int light_splits(int n_cu, int64_t heads, int waves, int64_t sealed, int64_t others) {
  const int64_t most = std::max<int64_t>(1, 12 / waves * (int64_t)n_cu / heads), tiles = (sealed + 32 * waves - 1) / (32 * waves);
  return (int)std::min(most, tiles <= 1 && others <= L_EXACT ? 1 : tiles + (others + L_EXACT - 1) / L_EXACT);
}
static Shape shape_of(int n_cu, int64_t heads, int n_rows, int64_t sealed, int64_t others) {
  if (n_rows <= L_ROWS) {
    const int most = light_splits(n_cu, heads, 12, 1 << 30, 0);
    const int waves = heads <= n_cu && (sealed + 383) / 384 >= 3 * most ? 12 : 4;
    return {waves == 4 ? L_ROWS : L_ROWS + 1, light_splits(n_cu, heads, waves, sealed, others)};
  }
  const int rows = tree_rows(n_cu, heads, n_rows, sealed, others);
  return {rows, tree_splits(n_cu, heads, n_rows, rows, sealed, others)};
}
template <typename A>
static int32_t launch_rows(const A& a, int64_t heads, int rows, int others, hipStream_t st) {
  if (rows > L_ROWS + 1) return launch_pass(a, heads, rows, others, st);
  if (rows == L_ROWS)
    tree_light_kernel<4><<<dim3((uint32_t)heads, (uint32_t)a.nsplit), 256, 0, st>>>(a);
  else
    tree_light_kernel<12><<<dim3((uint32_t)heads, (uint32_t)a.nsplit), 768, 0, st>>>(a);
  CQA_HIP(hipGetLastError());
  return CQA_OK;
}
static int64_t set_floats(const Cache* c, int64_t nodes, int64_t others) {
  const int64_t heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  const int n_rows = row_count(c, nodes);
  const auto most = [&](int rows) { return (int64_t)tree_splits(c->n_cu, heads, n_rows, rows, c->desc.max_tokens, others); };
  if (n_rows <= L_ROWS) return heads * light_splits(c->n_cu, heads, 4, c->desc.max_tokens, others) * T_FLOATS;
  return heads * ((n_rows + 31) / 32) * std::max(most(32), most(n_rows <= 64 ? 64 : (n_rows <= 128 ? 128 : 256))) * T_FLOATS;
}
int64_t scored_ws_bytes(const Cache* shared, const Cache* c, int n) {
  int64_t floats = set_floats(c, n, n + BLK - 1);
  if (shared != nullptr) floats += set_floats(shared, (int64_t)n * (c->desc.batch / shared->desc.batch), BLK - 1);
  return floats * 4;
}

// What the pass over c's tokens takes, of `nodes` nodes of each of its sequences.  others: drafted tokens.
template <Scores SCORES>
static int put_pass(SetArgs<SCORES>& a, const Cache* c, int layer, int nodes, int drafts, int first, float* part) {
  const int64_t head0 = head_index(c, layer, 0, 0), heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  a.t1 = c->t1 + head0 * c->nq_cap * QUAD_BYTES;
  a.trail_k = c->trail_k + head0 * BLK * D;
  a.trail_v = c->trail_v + head0 * BLK * D;
  a.nq_cap = c->nq_cap;
  a.nb = c->length[layer] / BLK;
  a.trail = (int)(c->length[layer] % BLK);
  a.n = nodes;
  a.nd = drafts;
  a.first = first;
  a.part = part;
  const int n_rows = nodes * a.group, others = a.trail + drafts;
  a.row_tiles = (n_rows + 31) / 32;
  const Shape x = shape_of(c->n_cu, heads, n_rows, a.nb * BLK, others);
  a.nsplit = x.nsplit;
  if (x.rows > 32) {
    put_shares(a, x.rows, others);
  } else if (x.rows <= L_ROWS + 1) {
    const TileShares s = light_shares((int)((a.nb + 1) / 2), others, a.nsplit, x.rows == L_ROWS ? 4 : 12);
    a.share = s.share, a.over = s.over, a.least = s.least, a.last = s.last;
  }
  return x.rows;
}

template <Scores SCORES>
static int32_t run(const Cache* shared, const Cache* c, int layer, const NodeCall& x, float* ws, hipStream_t st) {
  SetArgs<SCORES> a = {};
  a.q = x.q;
  a.kd = x.kd;
  a.vd = x.vd;
  a.mask = x.mask;
  a.words = (x.n + 63) / 64;
  a.n_kv = c->desc.n_kv_heads;
  a.group = c->desc.n_q_heads / c->desc.n_kv_heads;
  a.O = x.O;
  a.cert = x.cert;
  a.flags = x.flags;
  a.tol = *x.tol;
  const int64_t beginning = shared != nullptr ? shared->length[layer] : 0, heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  a.each = x.n;
  a.cached = (int)(beginning + c->length[layer]);
  a.drafted = x.kd != nullptr;
  if (SCORES != PLAIN) {
    const cqa_scoring& s = *x.scoring;
    constexpr float LOG2E = 1.4426950408889634f;
    a.scale = s.scale != 0.0f ? s.scale : 0.08838834764831845f;
    a.cap = s.cap;
    a.cap_kind = s.cap == 0.0f ? CAP_NONE : (s.cap <= LOW_CAPS ? CAP_LOW : CAP_HIGH);
    a.gain = a.cap_kind == CAP_NONE ? 0.0f : (a.cap_kind == CAP_LOW ? 2.0f * LOG2E : 1.0f) * (a.scale / s.cap);
    a.per_unit = LOG2E * (a.cap_kind == CAP_NONE ? a.scale : (a.cap_kind == CAP_LOW ? 2.0f * s.cap : s.cap));
    a.level = a.cap_kind == CAP_NONE ? a.per_unit : 1.0f;
    a.offset = a.cap_kind == CAP_LOW ? s.cap : 0.0f;
    a.slopes = s.slopes_dev;
    a.places = s.places_dev;
    a.spans = s.spans_dev;
  }
  const int drafts = a.drafted ? x.n : 0;
  const bool own = beginning == 0 || c->length[layer] + drafts > 0;
  if (beginning == 0) {
    const int rows = put_pass(a, c, layer, x.n, drafts, 0, ws);
    if (const int32_t rc = launch_rows(a, heads, rows, a.trail + drafts, st)) return rc;
    return a.nsplit == 1 ? CQA_OK : launch_join(a, heads, a.nsplit, c->n_cu, st);
  }
  const int64_t shared_heads = (int64_t)shared->desc.batch * shared->desc.n_kv_heads;
  JoinArgs<SCORES> j = {};
  static_cast<SetArgs<SCORES>&>(j) = a;
  const int shared_rows = put_pass(static_cast<SetArgs<SCORES>&>(j), shared, layer, x.n * (c->desc.batch / shared->desc.batch), 0, 0, ws);
  j.row_sets = own;
  const SetArgs<SCORES>& s = j;
  if (!own) {
    if (const int32_t rc = launch_rows(s, shared_heads, shared_rows, s.trail, st)) return rc;
    return s.nsplit == 1 ? CQA_OK : launch_join(s, shared_heads, s.nsplit, c->n_cu, st);
  }
  a.row_sets = 1;
  const int rows = put_pass(a, c, layer, x.n, drafts, (int)beginning, ws + shared_heads * s.row_tiles * s.nsplit * T_FLOATS);
  if (shared_rows == L_ROWS && rows == L_ROWS && shared_heads * s.nsplit + heads * a.nsplit <= 3 * (int64_t)c->n_cu) {
    const TwoPasses<SetArgs<SCORES>> two = {s, a, (int)shared_heads, (int)shared_heads * s.nsplit, (int)heads};
    tree_light_two_kernel<4><<<dim3((uint32_t)(two.a_groups + heads * a.nsplit)), 256, 0, st>>>(two);
    CQA_HIP(hipGetLastError());
  } else {
    if (const int32_t rc = launch_rows(s, shared_heads, shared_rows, s.trail, st)) return rc;
    if (const int32_t rc = launch_rows(a, heads, rows, a.trail + drafts, st)) return rc;
  }
  j.own = a.part;
  j.own_tiles = a.row_tiles;
  j.own_sets = a.nsplit;
  return launch_join(j, shared_heads, j.nsplit + a.nsplit, c->n_cu, st);
}

int32_t launch_scored(const Cache* shared, const Cache* c, int layer, const NodeCall& x, float* ws, hipStream_t st) {
  const cqa_scoring* const s = x.scoring;
  if (s != nullptr && (s->slopes_dev != nullptr || s->spans_dev != nullptr)) return run<PLACED>(shared, c, layer, x, ws, st);
  if (s != nullptr && ((s->scale != 0.0f && s->scale != 0.08838834764831845f) || s->cap != 0.0f)) return run<SCALED>(shared, c, layer, x, ws, st);
  return run<PLAIN>(shared, c, layer, x, ws, st);
}

}  // namespace cqa
