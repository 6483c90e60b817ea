// Attention of up to 16 rows a KV group over the quantized cache: the split pass of single tokens and of few drafted ones.
//
// The mathematics and the partial sets are tree_inl.h's; the products are 16x16x32 MFMA, whose accumulators and queries take half the registers of 32
// rows, so that three waves share a SIMD instead of two.  What bounds it is the reconstruction on the vector ALU, which does not depend on the number of
// rows, and the latency of its loads, which the third wave hides; the softmax of 32 rows, of which a single token's are four, is a quarter of the vector
// operations, that of 16 an eighth.
// 8 KV heads of 131072 tokens, one token of 4 query heads, capped: 63 us in a trace (a call 68) for 302 MB, 4.8 TB/s; vector ALU 55 % busy, waves wait 35 % of
// their cycles; 60 us is the time of a copy of as many bytes.
//
//   S^T [32 tokens][16 rows] = K^ Q^T as two tiles of 16 tokens.  A lane (n, g), n = l & 15, g = l >> 4, gets four tokens of each tile for row n.  The tiles
//     are tokens 0 - 3 and 4 - 7 of the pair's four octets, so that these eight are octet g: of one block, one dword of value codes, and packed
//     pairwise they are the B operand of
//   O^T [128 channels][16 rows] += V^T P^T, 32 tokens a product.
// Both tiles' A operands are of the same block in a lane, n >> 3, so that a channel's sigma and z are read once for two keys.
#pragma once
#include "tree_inl.h"

namespace cqa {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr int L_ROWS = 16;
constexpr int L_SET_O = D * L_ROWS, L_SET = L_SET_O + 8 * L_ROWS;      // floats of a wave's set in LDS: [four channels][row], then the quantities
constexpr int L_KM_BLK = KM_BYTES + 32, L_VM_BLK = VM_BYTES + 32;      // bytes; padded: the addresses of a read lie in different banks
constexpr int L_W_RUN = 16 * 16 + 16;                                  // widths [run of 8 channels][16 blocks]
constexpr int L_KM = 0, L_VM = L_KM + 2 * L_KM_BLK, L_W = L_VM + 2 * L_VM_BLK, L_META_END = L_W + D / 8 * L_W_RUN;
constexpr int exact_of(int waves) { return waves < 4 ? 32 : 64; }      // trailing and drafted tokens of a turn
constexpr int L_Q = L_ROWS * Q_ROW;
static_assert(L_META_END <= L_SET * 4 && 2 * exact_of(4) * D * 2 <= 4 * L_SET * 4 && 2 * exact_of(2) * D * 2 <= 2 * L_SET * 4 && L_VM % 16 == 0 && L_W % 16 == 0, "a wave's part of LDS, of four waves'");

// Pairs by workgroup: a turn of the trailing and drafted tokens takes as long as two of the sealed ones.
__host__ __device__ inline TileShares light_shares(int pairs, int others, int nsplit, int waves) {
  return tile_shares(pairs, (others + exact_of(waves) - 1) / exact_of(waves), nsplit, 2 * waves);
}

struct LightRows {
  f16x8 q[4];      // channels (i >> 1) 64 + g 16 + (i & 1) 8 + 0 .. 7
  f32x4 o[8];      // channels ct 16 + g 4 + 0 .. 3
  float m, sum, sealed, ev, evmax, dmax, vmax;
  int node;
  template <typename F>
  __device__ __forceinline__ void each_sum(F f) {
#pragma unroll
    for (int ct = 0; ct < 8; ++ct)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[ct][r] = f(o[ct][r]);
  }
};
// Places of trailing and drafted tokens in the operands: of 32 tokens, the two tiles; octets of channels in their order.
struct PlacesLight {
  static __device__ __forceinline__ int key(int t) { return (t >> 5) * 32 + ((t >> 2) & 1) * 16 + ((t >> 3) & 3) * 4 + (t & 3); }
  static __device__ __forceinline__ int value(int oct, int c) { return oct * D + c; }
};

__device__ __forceinline__ float max_over_groups(float x) { return max_x32(max_x16(x)); }
__device__ __forceinline__ float sum_over_groups(float x) { return sum_x32(sum_x16(x)); }

// Scores of a lane's eight tokens, of its octet, to weights; p: the B operand.  bits, where masked: those its row attends.
template <typename A, typename Rows>
__device__ __forceinline__ void softmax8(const A& a, Rows& w, f32x8 (&s)[1], uint32_t (&p)[1][4], bool masked, uint32_t bits, float eta, bool silent = false) {
  // (the block's other octet is 16 lanes away)
  softmax_sets<1, 8>(a, w, s, p, masked, [&](int) { return bits; }, [&](int) { return eta; }, [](float x) { return max_over_groups(x); }, [](float x) { return sum_x16(x); }, silent);
}
__device__ __forceinline__ f32x8 both(f32x4 x, f32x4 y) { return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ f32x4 product16(uint4 x, f16x8 y, f32x4 z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), y, z, 0, 0, 0); }

struct LightLds {
  float (*set)[L_SET];   // [waves]
  uint8_t* q;            // [L_Q]
  float* norm;           // [L_EXACT]
  uint8_t* bad;          // [L_EXACT]
  int* place;            // [L_EXACT], PLACED
  Spans* span;           // [L_ROWS], PLACED
};

// A wave's rows to its set.
template <typename Rows>
__device__ __forceinline__ void put_light(const Rows& w, float* to) {
  const int l = threadIdx.x & 63, row = l & 15, g = l >> 4;
  float none = 0.0f;   // stays, unless a channel is no finite number
#pragma unroll
  for (int ct = 0; ct < 8; ++ct) {
    reinterpret_cast<float4*>(to)[(ct * 4 + g) * L_ROWS + row] = make_float4(w.o[ct][0], w.o[ct][1], w.o[ct][2], w.o[ct][3]);
#pragma unroll
    for (int r = 0; r < 4; ++r) none = fmaf(0.0f, w.o[ct][r], none);
  }
  const float bad = max_over_groups(none == 0.0f ? 0.0f : 1.0f);
  if (g == 0) {
    float* const st = to + L_SET_O + row;
    st[T_M * L_ROWS] = w.m;
    st[T_L * L_ROWS] = w.sum;
    st[T_SEALED * L_ROWS] = w.sealed;
    st[T_EV * L_ROWS] = w.ev;
    st[T_EVMAX * L_ROWS] = w.evmax;
    st[T_DMAX * L_ROWS] = w.dmax;
    st[T_VMAX * L_ROWS] = w.vmax;
    st[T_BAD * L_ROWS] = bad;
  }
}
// The waves' sets, joined: to a set of the pass, or to the outputs.
template <int WAVES, typename A>
__device__ __forceinline__ void end_light(const A& a, const float (*sets)[L_SET], int head, int split, int tid) {
  const int row = tid & 15, rows = a.n * a.group;
  if (row >= rows) return;
  float f[WAVES], M = -INFINITY, L = 0.0f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    f[i] = sets[i][L_SET_O + T_M * L_ROWS + row];
    M = fmaxf(M, f[i]);
  }
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    f[i] = set_weight(a, f[i], M);
    L = fmaf(f[i], sets[i][L_SET_O + T_L * L_ROWS + row], L);
  }
  const bool leaves = leaves_sets(a);
  float* const to = leaves ? set_of(a, head, 0, split) : nullptr;
  const int64_t out = row_out(a, head, row);
  const float inv = mean_factor(L);
#pragma unroll
  for (int c = tid >> 4; c < 32; c += 4 * WAVES) {
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float4 y = reinterpret_cast<const float4*>(sets[i])[c * L_ROWS + row];
      x.x = fmaf(f[i], y.x, x.x), x.y = fmaf(f[i], y.y, x.y), x.z = fmaf(f[i], y.z, x.z), x.w = fmaf(f[i], y.w, x.w);
    }
    if (leaves)
      reinterpret_cast<float4*>(to)[c * T_ROWS + row] = x;
    else
      put_channels(a, out, c, x, inv);
  }
  if (tid >= L_ROWS) return;
  float SL = 0.0f, E = 0.0f, EM = 0.0f, DM = 0.0f, VM = 0.0f, bad = 0.0f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    const float* const st = sets[i] + L_SET_O + row;
    SL = fmaf(f[i], st[T_SEALED * L_ROWS], SL);
    E = fmaf(f[i], st[T_EV * L_ROWS], E);
    EM = fmaxf(EM, f[i] * st[T_EVMAX * L_ROWS]);
    DM = fmaxf(DM, st[T_DMAX * L_ROWS]);
    VM = fmaxf(VM, st[T_VMAX * L_ROWS]);
    bad = fmaxf(bad, st[T_BAD * L_ROWS]);
  }
  if (!leaves) {
    put_certificate(a, out, certificate(a, M, L, SL, E, EM, DM, VM, out_offset(a, head, row)), bad != 0.0f);
    return;
  }
  float* const st = to + T_OFLOATS + row;
  st[T_M * T_ROWS] = M;
  st[T_L * T_ROWS] = L;
  st[T_SEALED * T_ROWS] = SL;
  st[T_EV * T_ROWS] = E;
  st[T_EVMAX * T_ROWS] = EM;
  st[T_DMAX * T_ROWS] = DM;
  st[T_VMAX * T_ROWS] = VM;
  st[T_BAD * T_ROWS] = bad;
}

template <int WAVES, typename A>
__device__ __forceinline__ void attend_light(const A& a, int64_t head, int split, const LightLds& lds) {
  const int tid = threadIdx.x, l = tid & 63, n16 = l & 15, g = l >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int L_EXACT = exact_of(WAVES);
  const int b = (int)(head / a.n_kv), kvh = (int)(head - (int64_t)b * a.n_kv);
  uint8_t* const wave = reinterpret_cast<uint8_t*>(lds.set[w]);
  std::conditional_t<A::SCORED, Scored<LightRows>, LightRows> rows;
  const int last_row = a.n * a.group - 1;
  rows.node = a.node_of(min(n16, last_row));
  // four rows of the queries at a time by each of four waves, or of two: 16 lanes a row
  constexpr int Q_TURNS = WAVES < 4 ? 4 / WAVES : 1;
  const auto q_row = [&](int i) { return 4 * ((w + i * WAVES) & 3) + g; };
  uint4 q_in[Q_TURNS];
#pragma unroll
  for (int i = 0; i < Q_TURNS; ++i) {
    const int row = min(q_row(i), last_row), node = a.node_of(row);
    q_in[i] = ld16_any(a.q + (((int64_t)b * a.n + node) * a.n_kv * a.group + kvh * a.group + (row - node * a.group)) * D + n16 * 8);
  }

  const uint8_t* const base = a.t1 + head * a.nq_cap * QUAD_BYTES;
  int units = (int)((a.nb + 1) >> 1);                       // pairs of sealed blocks
  Active active;
  bool spans = false;
  if constexpr (A::PLACED) {
    const int64_t node = (int64_t)b * a.n + rows.node;
    const SpansGiven given = spans_given(a, node);
    const RowBias x = row_bias(a, node, kvh * a.group + (min(n16, last_row) - rows.node * a.group), given);
    rows.slope = x.slope * (1.0f / (a.per_unit * LN2));
    rows.place = x.place - a.first;
    rows.near = x.near;
    spans = a.spans != nullptr;
    rows.idle = false;
    if (spans) {
      const Spans mine = spans_among(given, a.first, (int)a.nb * BLK + a.trail);
      rows.idle = mine.hi0 == 0 && mine.hi1 == 0;
      if (l < L_ROWS) lds.span[l] = mine;                   // (every wave the same)
      active = active_units(hull_of<L_ROWS>(mine), (int)a.nb * BLK, 2 * BLK);
      units = active.units;
    }
  }
  const auto pair_at = [&](int u) {
    if constexpr (A::PLACED) return spans ? active.at(u) : u;
    return u;
  };
  // the workgroup's pairs: from .. units - 1
  const TileShares sh = spans ? light_shares(units, a.trail + a.drafts(), a.nsplit, WAVES) : TileShares{a.share, a.over, a.least, a.last};
  const int even = a.nsplit - sh.last, mid = min(split, even);
  const int from = mid * sh.share + min(mid, sh.over) + (split - mid) * sh.least;
  units = from + (split < even ? sh.share + (split < sh.over) : sh.least);
  const int kb = n16 >> 3, tok = ((n16 >> 2) & 1) * 8 + (n16 & 3);   // the keys' block of the pair, and the first tile's token of it
  const int vb = g >> 1;                                             // the octet's block
  uint4 k00, k01, k10, k11, km0, km1, vc0, vc1, vm;                  // keys (tile, half of the channels)
  float2 an;
  const auto record = [&](int u) { return base + (int64_t)(u < units ? pair_at(u) >> 1 : 0) * QUAD_BYTES; };
  const auto load_keys = [&](int u) {
    const uint8_t* const p = record(u) + Q_KC + ((pair_at(u) & 1) * 2 + kb) * KC_BYTES + g * 256 + tok * 16;
    k00 = *reinterpret_cast<const uint4*>(p), k10 = *reinterpret_cast<const uint4*>(p + 64);
    k01 = *reinterpret_cast<const uint4*>(p + 1024), k11 = *reinterpret_cast<const uint4*>(p + 1088);
  };
  const auto load_meta = [&](int u) {
    const uint8_t* const r = record(u);
    const int b0 = (pair_at(u) & 1) * 2;
    km0 = reinterpret_cast<const uint4*>(r + Q_KM + b0 * KM_BYTES)[l];
    km1 = reinterpret_cast<const uint4*>(r + Q_KM + (b0 + 1) * KM_BYTES)[l];
    vm = reinterpret_cast<const uint4*>(r + Q_VM + b0 * VM_BYTES)[l];
    an = reinterpret_cast<const float2*>(r + Q_AN)[b0 + vb];
  };
  const auto load_values = [&](int u) {
    const uint8_t* const p = record(u) + Q_VC + ((pair_at(u) & 1) * 2 + vb) * VC_BYTES + (g & 1) * 512 + n16 * 16;
    vc0 = *reinterpret_cast<const uint4*>(p);
    vc1 = *reinterpret_cast<const uint4*>(p + 256);
  };
  int u = from + w;
  load_meta(u);
  load_keys(u);
  load_values(u);
#pragma unroll
  for (int i = 0; i < Q_TURNS; ++i) *reinterpret_cast<uint4*>(lds.q + q_row(i) * Q_ROW + n16 * 16) = q_in[i];   // (of each four waves the same)
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) rows.q[i] = *reinterpret_cast<const f16x8*>(lds.q + n16 * Q_ROW + (i >> 1) * 128 + g * 32 + (i & 1) * 16);
  rows.m = -INFINITY;
  rows.sum = rows.sealed = rows.ev = rows.evmax = rows.dmax = rows.vmax = 0.0f;
#pragma unroll
  for (int ct = 0; ct < 8; ++ct)
#pragma unroll
    for (int r = 0; r < 4; ++r) rows.o[ct][r] = 0.0f;
  if constexpr (A::SCORED) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 x = __builtin_bit_cast(uint4, rows.q[i]);
      bad |= !(finite2(x.x) & finite2(x.y) & finite2(x.z) & finite2(x.w));
    }
    rows.undefined = max_over_groups(bad ? 1.0f : 0.0f) != 0.0f;
    zero_undefined(rows, rows.q);
  }

  uint32_t open = 0u;     // what the lane's row has attended
  bool partial = false;   // PLACED: some row does not attend all of the blocks whose widths have come
  for (int turn = 0; u < units; u += WAVES, ++turn) {
    const int pair = pair_at(u);
    uint32_t there = (int64_t)pair * 2 + vb < a.nb ? 0xffu : 0u;
    bool silent = false;
    bool masked = (int64_t)pair * 2 + 2 > a.nb;
    if constexpr (A::PLACED)
      if (spans && !active.open(pair * 2 * BLK, (pair + 1) * 2 * BLK)) {
        masked = partial = true;
        there &= span_bits(lds.span[n16], (pair * 4 + g) * 8);
      }
    if constexpr (A::PLACED) {
      silent = rows.idle;
      there = silent ? 0u : there;
    }
    open |= there;
    float eta = value_error(an);
    if constexpr (A::PLACED)
      if (spans) {
        uint32_t flawed[2];
        mend_pair(km0, km1, vm, flawed);
        if (there & (vb ? flawed[1] : flawed[0]) >> (g & 1) * 8) rows.sum = NAN;   // stays
        eta = there == 0u ? 0.0f : eta;
      }
    // metadata
    reinterpret_cast<uint4*>(wave + L_KM)[l] = km0;
    reinterpret_cast<uint4*>(wave + L_KM + L_KM_BLK)[l] = km1;
    *reinterpret_cast<uint4*>(wave + L_VM + (l >> 5) * L_VM_BLK + (l & 31) * 16) = paired(vm);
    rows.vmax = fmaxf(rows.vmax, A::PLACED && there == 0u ? 0.0f : an.y);
    load_meta(u + WAVES);
    wave_sync();
    // widths: four channels a lane
    {
      const int c = (l & 31) * 4;
      const float* const p = reinterpret_cast<const float*>(wave + L_KM + (l >> 5) * L_KM_BLK) + c;
      const float4 s4 = *reinterpret_cast<const float4*>(p), z4 = *reinterpret_cast<const float4*>(p + D);
      *reinterpret_cast<uint2*>(wave + L_W + (c >> 3) * L_W_RUN + ((turn & 7) * 2 + (l >> 5)) * 16 + (c & 4) * 2) =
          make_uint2(key_width(s4.x, z4.x) | key_width(s4.y, z4.y) << 16, key_width(s4.z, z4.z) | key_width(s4.w, z4.w) << 16);
    }
    f32x4 x0 = {0.0f, 0.0f, 0.0f, 0.0f}, x1 = x0;
    const float* const sg = reinterpret_cast<const float*>(wave + L_KM + kb * L_KM_BLK) + g * 16;
    each<4>([&](auto i_) {
      constexpr int i = i_.value;
      const float* const p = sg + (i >> 1) * 64 + (i & 1) * 8;
      const float4 s0 = *reinterpret_cast<const float4*>(p), s1 = *reinterpret_cast<const float4*>(p + 4);
      const float4 z0 = *reinterpret_cast<const float4*>(p + D), z1 = *reinterpret_cast<const float4*>(p + D + 4);
      const uint4 c0 = i >> 1 ? k01 : k00, c1 = i >> 1 ? k11 : k10;
      x0 = product16(i & 1 ? keys8(c0.z, c0.w, s0, s1, z0, z1) : keys8(c0.x, c0.y, s0, s1, z0, z1), rows.q[i], x0);
      x1 = product16(i & 1 ? keys8(c1.z, c1.w, s0, s1, z0, z1) : keys8(c1.x, c1.y, s0, s1, z0, z1), rows.q[i], x1);
    });
    load_keys(u + WAVES);
    if ((turn & 7) == 7 || u + WAVES >= units) {
      wave_sync();
      const int last = (turn & 7) * 2 + 1, slot = min(n16, last), first = u - (turn & 7) * WAVES;
      f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
      uint32_t no_signs = 0x7fff7fffu;
      asm volatile("" : "+s"(no_signs));   // |q| is formed here, not kept
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 y = __builtin_bit_cast(uint4, rows.q[i]);
        y.x &= no_signs, y.y &= no_signs, y.z &= no_signs, y.w &= no_signs;
        d = product16(*reinterpret_cast<const uint4*>(wave + L_W + ((i >> 1) * 8 + g * 2 + (i & 1)) * L_W_RUN + slot * 16), __builtin_bit_cast(f16x8, y), d);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int s = min(g * 4 + r, last);
        float x = d[r];
        if constexpr (A::PLACED)
          if (partial) x = some_of(lds.span[n16], pair_at(first + (s >> 1) * WAVES) * 2 + (s & 1)) ? x : 0.0f;
        rows.dmax = fmaxf(rows.dmax, x);
      }
      partial = false;
      wave_sync();
    }
    f32x8 s[1] = {both(x0, x1)};
    uint32_t p[1][4];
    if constexpr (A::SCORED) score<8>(a, rows, s[0], RunFar<8>(rows, (pair * 4 + g) * 8));
    softmax8(a, rows, s, p, masked, there, eta, silent);
    const f16x8 weights = __builtin_bit_cast(f16x8, make_uint4(p[0][0], p[0][1], p[0][2], p[0][3]));
    const uint8_t* const sc = wave + L_VM + vb * L_VM_BLK + (g & 1) * 128;
    each<8>([&](auto i_) {
      constexpr int ct = i_.value;
      const uint4 v = ct >> 2 ? vc1 : vc0;
      const uint32_t c = (ct & 3) == 0 ? v.x : ((ct & 3) == 1 ? v.y : ((ct & 3) == 2 ? v.z : v.w));
      rows.o[ct] = product16(values8(c, *reinterpret_cast<const uint4*>(sc + ct * 16), *reinterpret_cast<const uint4*>(sc + 256 + ct * 16)), weights, rows.o[ct]);
    });
    load_values(u + WAVES);
    wave_sync();
  }
  if constexpr (A::PLACED) rows.dmax = rows.idle ? 0.0f : rows.dmax;
  rows.sealed = rows.sum;
  // The other tokens, 32 to a wave: dealt to the workgroups from the last one down.
  for (int t0 = (a.nsplit - 1 - split) * L_EXACT; t0 < a.trail + a.drafts(); t0 += a.nsplit * L_EXACT) {
    uint4* const s_k = reinterpret_cast<uint4*>(lds.set);
    uint4* const s_v = s_k + 16 * L_EXACT;
    const int at = t0 + w * 32 + g * 8;   // the lane's octet
    uint32_t bits = open_tokens(a, b, rows.node, at & ~15) >> (at & 8) & 0xffu;
    if constexpr (A::PLACED) {
      if (spans) bits &= span_bits(lds.span[n16], (int)a.nb * BLK + at) | ~trailing_bits(a, at);
      if (a.slopes != nullptr && tid < L_EXACT) lds.place[tid] = exact_place(a, b, t0 + tid);
    }
    if (tid < L_EXACT / 4) reinterpret_cast<uint32_t*>(lds.bad)[tid] = 0u;
    __syncthreads();
    constexpr int LOADERS = WAVES < 8 ? 64 * WAVES : 512;
    if (WAVES <= 8 || tid < LOADERS) load_exact<LOADERS, L_EXACT, PlacesLight>(a, head, t0, tid, s_k, s_v, lds.norm, lds.bad);
    __syncthreads();
    if (w * 32 < min(L_EXACT, a.trail + a.drafts() - t0)) {
      const int in = w * 32 + g * 8;
      open |= bits;
      uint32_t hit = 0u;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        hit |= (reinterpret_cast<const uint32_t*>(lds.bad + in)[i] * 0x10204080u >> 28) << (4 * i);   // a bit per byte
        const float4 x = reinterpret_cast<const float4*>(lds.norm + in)[i];
        rows.vmax = fmaxf(rows.vmax, fmaxf(fmaxf(bits >> (4 * i) & 1u ? x.x : 0.0f, bits >> (4 * i + 1) & 1u ? x.y : 0.0f),
                                           fmaxf(bits >> (4 * i + 2) & 1u ? x.z : 0.0f, bits >> (4 * i + 3) & 1u ? x.w : 0.0f)));
      }
      if (bits & hit) rows.sum = NAN;   // stays
      f32x4 x0 = {0.0f, 0.0f, 0.0f, 0.0f}, x1 = x0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4* const k = s_k + ((i >> 1) * 8 + g * 2 + (i & 1)) * L_EXACT + w * 32 + n16;
        x0 = product16(k[0], rows.q[i], x0);
        x1 = product16(k[16], rows.q[i], x1);
      }
      f32x8 s[1] = {both(x0, x1)};
      uint32_t p[1][4];
      if constexpr (A::SCORED) score<8>(a, rows, s[0], [&](int r) { return (float)(abs(rows.place - lds.place[in + r]) - rows.near); });
      softmax8(a, rows, s, p, true, bits, 0.0f);
      const f16x8 weights = __builtin_bit_cast(f16x8, make_uint4(p[0][0], p[0][1], p[0][2], p[0][3]));
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) rows.o[ct] = product16(s_v[(w * 4 + g) * D + ct * 16 + n16], weights, rows.o[ct]);
    }
    __syncthreads();   // (the next ones, or the waves' sets, come where these are)
  }
  // the groups of lanes joined (end_rows)
  const float any = max_over_groups(open != 0u ? 1.0f : 0.0f);
  rows.sum = sum_over_groups(rows.sum);
  if (rows.sum == 0.0f && any != 0.0f) rows.sum = NAN;
  if constexpr (A::SCORED)
    if (rows.undefined && any != 0.0f) rows.sum = NAN;
  rows.sealed = sum_over_groups(rows.sealed);
  rows.ev = sum_over_groups(rows.ev);
  rows.evmax = max_over_groups(rows.evmax);
  rows.dmax = max_over_groups(rows.dmax) * a.half_scale();
  rows.vmax = max_over_groups(rows.vmax);
  put_light(rows, lds.set[w]);
  __syncthreads();
  end_light<WAVES>(a, lds.set, (int)head, split, tid);
}

template <int WAVES, typename F>
__device__ __forceinline__ void with_light_lds(F f) {
  constexpr int L_EXACT = exact_of(WAVES);
  __shared__ __align__(16) float s_set[WAVES][L_SET];
  __shared__ __align__(16) uint8_t s_q[L_Q];
  __shared__ __align__(16) float s_norm[L_EXACT];
  __shared__ __align__(16) uint8_t s_bad[L_EXACT];
  __shared__ __align__(16) int s_place[L_EXACT];
  __shared__ __align__(16) Spans s_span[L_ROWS];
  f(LightLds{s_set, s_q, s_norm, s_bad, s_place, s_span});
}
template <int WAVES, typename A>
__global__ __launch_bounds__(64 * WAVES, 3) void tree_light_kernel(A a) {
  fetch_args<sizeof(A)>();
  with_light_lds<WAVES>([&](const LightLds& lds) { attend_light<WAVES>(a, blockIdx.x, blockIdx.y, lds); });
}
// Two passes in one launch, a's workgroups first. 
template <typename A>
struct TwoPasses {
  A a, b;
  int a_heads, a_groups, b_heads;   // KV groups, a's workgroups
};
template <int WAVES, typename A>
__global__ __launch_bounds__(64 * WAVES, 3) void tree_light_two_kernel(TwoPasses<A> x) {
  fetch_args<sizeof(TwoPasses<A>)>();
  const int i = (int)blockIdx.x;
  with_light_lds<WAVES>([&](const LightLds& lds) {
    if (i < x.a_groups)
      attend_light<WAVES>(x.a, i % x.a_heads, i / x.a_heads, lds);
    else
      attend_light<WAVES>(x.b, (i - x.a_groups) % x.b_heads, (i - x.a_groups) / x.b_heads, lds);
  });
}

}  // namespace cqa
