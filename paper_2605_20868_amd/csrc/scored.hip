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
    const int node = this->node_of(r), seq = node / this->each, row = (node - seq * this->each) * this->group + (r - node * this->group);
    const int64_t own_head = ((int64_t)b * (this->n / this->each) + seq) * this->n_kv + kvh;
    return {SetsOf{sets, T_FLOATS, this->nsplit, r32}, SetsOf{own + (own_head * own_tiles + row / T_ROWS) * own_sets * T_FLOATS, T_FLOATS, own_sets, row % T_ROWS}};
  }
};

// ---- what a call launches --------------------------------------------------------------------------------------------------------------

// Rows of a KV group a workgroup takes, its waves, and the partial sets of a row.
struct Shape {
  int rows, waves, nsplit;
};
static int light_splits(int n_cu, int64_t heads, int waves, int64_t sealed, int64_t others) {
  const int64_t most = std::max<int64_t>(1, 12 / waves * (int64_t)n_cu / heads), tiles = (sealed + 32 * waves - 1) / (32 * waves);
  return (int)std::min(most, tiles <= 1 && others <= exact_of(waves) ? 1 : tiles + (others + exact_of(waves) - 1) / exact_of(waves));
}
// Up to 16 rows go by the light kernel: twelve waves a workgroup, one of which a compute unit holds, where these have three turns and more, for there are
// fewer sets to join; two where more heads are there than workgroups of four can be at a time, and short ones or no more than of two; else four
// (us a call in a graph with twelve and with four: 8 heads, 131072 tokens 64.1, 67.8; 4 x 8 heads, windows of 4096 in 32768 23.6, 24.4; 8 heads, 8000 tokens
// 14.4, 12.6; 64 x 8 heads, 1029 tokens 44.3, 33.6.  With four and with two: 512 heads, 263 tokens 15.1, 17.9; 640 19.7, 20.7; 800 25.4, 20.0; 3200 68.7, 59.8;
// 800 heads, 40 tokens 17.7, 10.9; 1029 tokens 57.3, 50.1; 4101 tokens 232, 234; 1024 heads, 517 tokens 37.8, 32.3; 1600 heads, 1029 tokens 110.7, 122.4).
// More rows: tree_rows.
static int light_waves(int n_cu, int64_t heads, int64_t sealed) {
  if (heads <= n_cu && (sealed + 383) / 384 >= 3 * (n_cu / heads)) return 12;
  return heads > 3 * n_cu && sealed <= (heads <= 6 * n_cu ? 2048 : 512) ? 2 : 4;
}
static Shape shape_of(int n_cu, int64_t heads, int n_rows, int64_t sealed, int64_t others) {
  if (n_rows <= L_ROWS) {
    const int waves = light_waves(n_cu, heads, sealed);
    return {L_ROWS, waves, light_splits(n_cu, heads, waves, sealed, others)};
  }
  const int rows = tree_rows(n_cu, heads, n_rows, sealed, others);
  return {rows, 8, tree_splits(n_cu, heads, n_rows, rows, sealed, others)};
}

static int row_count(const Cache* c, int64_t nodes) { return (int)(nodes * (c->desc.n_q_heads / c->desc.n_kv_heads)); }
static int64_t kv_groups(const Cache* c) { return (int64_t)c->desc.batch * c->desc.n_kv_heads; }
static int64_t set_floats(const Cache* c, int64_t nodes, int64_t others) {
  const int64_t heads = kv_groups(c);
  const int n_rows = row_count(c, nodes);
  // (of two waves there is one set a head)
  if (n_rows <= L_ROWS) return heads * light_splits(c->n_cu, heads, 4, c->desc.max_tokens, others) * T_FLOATS;
  const auto most = [&](int rows) { return (int64_t)tree_splits(c->n_cu, heads, n_rows, rows, c->desc.max_tokens, others); };
  return heads * ((n_rows + 31) / 32) * std::max(most(32), most(n_rows <= 64 ? 64 : (n_rows <= 128 ? 128 : 256))) * T_FLOATS;
}
int64_t scored_ws_bytes(const Cache* shared, const Cache* c, int n) {
  int64_t floats = set_floats(c, n, n + BLK - 1);
  if (shared != nullptr) floats += set_floats(shared, (int64_t)n * (c->desc.batch / shared->desc.batch), BLK - 1);
  return floats * 4;
}

// The pass over c's tokens of `nodes` nodes of each of its sequences.
struct Pass {
  int64_t heads;
  Shape shape;
  int others;      // trailing and drafted tokens
  int64_t floats;  // of its sets
};
template <Scores SCORES>
static Pass put_pass(SetArgs<SCORES>& a, const Cache* c, int layer, int nodes, int drafts, int first) {
  const int64_t head0 = head_index(c, layer, 0, 0);
  a.t1 = c->t1 + head0 * c->nq_cap * QUAD_BYTES;
  a.trail_k = c->trail_k + head0 * BLK * D;
  a.trail_v = c->trail_v + head0 * BLK * D;
  a.nq_cap = c->nq_cap;
  a.nb = c->length[layer] / BLK;
  a.trail = (int)(c->length[layer] % BLK);
  a.n = nodes;
  a.nd = drafts;
  a.first = first;
  const int n_rows = nodes * a.group;
  a.row_tiles = (n_rows + 31) / 32;
  Pass x;
  x.heads = kv_groups(c);
  x.others = a.trail + drafts;
  x.shape = shape_of(c->n_cu, x.heads, n_rows, a.nb * BLK, x.others);
  a.nsplit = x.shape.nsplit;
  if (x.shape.rows > 32) put_shares(a, x.shape.rows, x.others);
  if (x.shape.rows == L_ROWS) {
    const TileShares s = light_shares((int)((a.nb + 1) / 2), x.others, a.nsplit, x.shape.waves);
    a.share = s.share, a.over = s.over, a.least = s.least, a.last = s.last;
  }
  x.floats = x.heads * a.row_tiles * a.nsplit * T_FLOATS;
  return x;
}
// low: the pass takes its caps as CAP_LOW; any_low: this or the call's other pass
template <Scores SCORES>
static void put_scores(SetArgs<SCORES>& a, const cqa_scoring& s, bool low, bool any_low) {
  constexpr float LOG2E = 1.4426950408889634f;
  a.scale = s.scale != 0.0f ? s.scale : PLAIN_SCALE;
  a.cap = s.cap;
  a.cap_kind = s.cap == 0.0f ? CAP_NONE : (low ? CAP_LOW : CAP_HIGH);
  a.rounded = any_low && s.slopes_dev == nullptr;
  a.gain = a.cap_kind == CAP_NONE ? 0.0f : (low ? 2.0f * LOG2E : 1.0f) * (a.scale / s.cap);
  if (a.cap_kind == CAP_HIGH) {
    const bool powers = a.gain >= 1e-4f && a.gain <= 1e4f;   // the seventh, by the smallest coefficient, is a normal number
    a.series_end = SERIES_END / a.gain;
    a.pre = powers ? 1.0f : a.gain;
    double power = powers ? a.gain : 1.0;
    for (int i = 0; i < 4; ++i, power *= powers ? (double)a.gain * a.gain : 1.0) a.series[i] = (float)(SERIES[i] * power);
  }
  a.per_unit = LOG2E * (a.cap_kind == CAP_NONE ? a.scale : s.cap);
  a.slopes = s.slopes_dev;
  a.places = s.places_dev;
  a.spans = s.spans_dev;
}
template <typename A>
static int32_t launch_rows(const A& a, const Pass& x, hipStream_t st) {
  if (x.shape.rows != L_ROWS) return launch_pass(a, x.heads, x.shape.rows, x.others, st);
  const dim3 grid((uint32_t)x.heads, (uint32_t)a.nsplit);
  if (x.shape.waves == 2)
    tree_light_kernel<2><<<grid, 128, 0, st>>>(a);
  else if (x.shape.waves == 4)
    tree_light_kernel<4><<<grid, 256, 0, st>>>(a);
  else
    tree_light_kernel<12><<<grid, 768, 0, st>>>(a);
  CQA_HIP(hipGetLastError());
  return CQA_OK;
}
// A pass that is all of its rows'.
template <typename A>
static int32_t launch_alone(const A& a, const Pass& x, int n_cu, hipStream_t st) {
  if (const int32_t rc = launch_rows(a, x, st)) return rc;
  return a.nsplit == 1 ? CQA_OK : launch_join(a, x.heads, a.nsplit, n_cu, st);
}

template <Scores SCORES>
static int32_t run(const Cache* shared, const Cache* c, int layer, const NodeCall& call, float* ws, hipStream_t st) {
  SetArgs<SCORES> a = {};
  a.q = call.q;
  a.kd = call.kd;
  a.vd = call.vd;
  a.mask = call.mask;
  a.words = (call.n + 63) / 64;
  a.n_kv = c->desc.n_kv_heads;
  a.group = c->desc.n_q_heads / c->desc.n_kv_heads;
  a.O = call.O;
  a.cert = call.cert;
  a.flags = call.flags;
  a.tol = *call.tol;
  a.part = ws;
  const int64_t beginning = shared != nullptr ? shared->length[layer] : 0;
  const int drafts = call.kd != nullptr ? call.n : 0;
  a.each = call.n;
  a.cached = (int)(beginning + c->length[layer]);
  a.drafted = drafts != 0;
  // The sequences' own tokens and the beginning's, a pass each where there are any; the first also where there are none at all.
  JoinArgs<SCORES> both = {};
  SetArgs<SCORES>& b = both;
  b = a;
  const bool has_own = beginning == 0 || c->length[layer] + drafts > 0, has_shared = beginning != 0;
  const Pass own = put_pass(a, c, layer, call.n, drafts, (int)beginning);
  const Pass theirs = has_shared ? put_pass(b, shared, layer, call.n * (c->desc.batch / shared->desc.batch), 0, 0) : Pass{};
  if constexpr (SCORES != PLAIN) {
    const bool may = call.scoring->cap != 0.0f && call.scoring->cap <= LOW_CAPS;
    const bool low = may && has_own && own.shape.rows >= 128, their_low = may && has_shared && theirs.shape.rows >= 128;
    put_scores(a, *call.scoring, low, low || their_low);
    put_scores(b, *call.scoring, their_low, low || their_low);
  }
  if (!has_shared) return launch_alone(a, own, c->n_cu, st);
  if (!has_own) return launch_alone(b, theirs, c->n_cu, st);
  a.row_sets = b.row_sets = 1;
  a.part = ws + theirs.floats;
  const int64_t groups = theirs.heads * b.nsplit + own.heads * a.nsplit;
  if (theirs.shape.rows == L_ROWS && own.shape.rows == L_ROWS && theirs.shape.waves == 4 && own.shape.waves == 4 && groups <= 3 * (int64_t)c->n_cu) {
    // (as many as the device holds at a time: 2 sequences behind 1029 tokens, 1 KV head 13.0 us, by two launches 18.7)
    const TwoPasses<SetArgs<SCORES>> two = {b, a, (int)theirs.heads, (int)(theirs.heads * b.nsplit), (int)own.heads};
    tree_light_two_kernel<4><<<dim3((uint32_t)groups), 256, 0, st>>>(two);
    CQA_HIP(hipGetLastError());
  } else {
    if (const int32_t rc = launch_rows(b, theirs, st)) return rc;
    if (const int32_t rc = launch_rows(a, own, st)) return rc;
  }
  both.own = a.part;
  both.own_tiles = a.row_tiles;
  both.own_sets = a.nsplit;
  return launch_join(both, theirs.heads, both.nsplit + a.nsplit, c->n_cu, st);
}

int32_t launch_scored(const Cache* shared, const Cache* c, int layer, const NodeCall& call, float* ws, hipStream_t st) {
  const cqa_scoring* const s = call.scoring;
  if (s != nullptr && (s->slopes_dev != nullptr || s->spans_dev != nullptr)) return run<PLACED>(shared, c, layer, call, ws, st);
  if (s != nullptr && ((s->scale != 0.0f && s->scale != PLAIN_SCALE) || s->cap != 0.0f)) return run<SCALED>(shared, c, layer, call, ws, st);
  return run<PLAIN>(shared, c, layer, call, ws, st);
}

}  // namespace cqa
