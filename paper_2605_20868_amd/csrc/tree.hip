// Attention of drafted tokens (a tree, or a chunk of a prompt) over the quantized cache, with the certificate of every
// (node, query head): split pass on the matrix cores and the joining of its partial sets.
//
// The rows of a KV group are its n_draft nodes times its G query heads, and all of them attend the same sealed blocks.  Two kernels: 32 rows a workgroup, whose
// waves reconstruct pairs of blocks in registers, each for itself; or up to 256 rows, for which a workgroup reconstructs a tile of keys and values
// once, into LDS (tree_rows says when).
//   k^ = FP16(code sigma + z),  v^ = FP16(code scale + offset)
// FP16 operands, FP32 accumulation: with the two-term scaled queries of the single-token pass the operand forming would cost
// 128 multiplications per (row, block), more than the products.  What the rounding of the reconstruction adds is in the certificate:
// the originals are FP16 numbers, so rounding k^ to FP16 moves it by at most |k - k^| <= sigma / 2, and by at most half a step of FP16;
// the key's width in Delta_b is therefore
//   w_c = sigma_c + 2 min(sigma_c / 2, 2^-11 max |k^_c| + 2^-25),   Delta_b = (1 / (2 sqrt d)) sum_c |q_c| w_c
// and the block's value error  eta_b + min(eta_b, 2^-11 (nu_b + eta_b) + 2^-21).  w is rounded up to FP16, where |q| w is exact on the
// matrix cores (a bound stays one, at most 2^-10 wider).
//
// Products, 32x32x16 MFMA:
//   S^T [32 tokens][32 rows] = K^ Q^T.  The tile's 32 token rows are dealt to two blocks so that a lane's 16 results are the 16 tokens of
//     one block for one row: the block's sum S_b is an in-lane sum, and what the lane holds is, packed, the B operand of
//   O^T [128 channels][32 rows] += V^T P^T, whose 8 consecutive tokens per lane are what one dword of value codes holds.
// Softmax in FP32 (running maximum per row, FP32 sums); the weights enter the second product as FP16, off by 2^-11 of a weight at most: two terms
// of each would double the products with the values, and O is rounded to FP16 itself.
//
// Trailing FP16 tokens and drafted ones, which are exact, are attended behind the sealed ones, under the mask, by the workgroups that have
// the fewest of those.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "cqa_internal.h"
#include "reduce_inl.h"

namespace cqa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float SCORE = 0.08838834764831845f * 1.4426950408889634f;   // 1 / sqrt(d), in the exponent's base 2
constexpr float HALF_SCORE = 0.5f * 0.08838834764831845f;
constexpr float F16_MAX = 65504.0f;
constexpr float MOST = 14.0f;   // the largest weight is 2^MOST: see softmax32
constexpr float LN2 = 0.6931471805599453f;

// f(0), f(1), ... f(N - 1), each with its index as a constant
template <typename F, int... I>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}

// ---- partial set of a split and 32 rows: the accumulators by (four channels, row), then one float per row for each quantity
enum { T_M = 0, T_L, T_SEALED, T_EV, T_EVMAX, T_DMAX, T_VMAX, T_BAD };   // T_BAD: 1 where an accumulator is no finite number, else 0
constexpr int T_ROWS = 32;
constexpr int T_OFLOATS = D * T_ROWS;
constexpr int T_FLOATS = T_OFLOATS + 8 * T_ROWS;

struct TreeArgs {
  const uint8_t* t1;       // layer base of the quad records
  const __half* trail_k;   // layer base [Bt * Hkv][16][128]
  const __half* trail_v;
  const __half* q;         // [Bt][n][Hq][128]
  const __half* kd;        // [Bt][Hkv][n][128]
  const __half* vd;
  const uint64_t* mask;    // [Bt][n][words], or null: node i attends nodes 0 .. i
  float* part;             // [Bt * Hkv][row tiles][nsplit][T_FLOATS]
  int64_t nq_cap;
  int64_t nb;              // sealed blocks
  int n, words, trail;     // drafted nodes, mask words of one, trailing tokens
  int n_kv, group;
  int row_tiles;           // of 32 rows
  int nsplit;              // partial sets per row; 1: the split pass finishes the rows itself
  int share, over, least, last;   // many rows: sealed tiles of a workgroup, how many have one more, those of the `last` workgroups
  __half* O;               // [Bt][n][Hq][128]
  cqa_node_cert* cert;     // [Bt][n][Hq]
  uint32_t* flags;
  cqa_tolerances tol;
};

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}
// Two keys, code sigma + z in FP32 and then rounded to FP16: the codes as FP16 integers by the mantissa of 1024 (the stored bytes are
// code + 128), which the multiply-add takes as they are.
template <int I>
__device__ __forceinline__ uint32_t key2(uint32_t codes, float s0, float s1, float z0, float z1) {
  const uint32_t biased = __builtin_amdgcn_perm(0x64646464u, codes, I ? 0x04030402u : 0x04010400u);
  const f16x2 code = __builtin_bit_cast(f16x2, biased) - f16x2{(_Float16)1152.0f, (_Float16)1152.0f};
  float x = fmaf((float)code[0], s0, z0), y = fmaf((float)code[1], s1, z1);
  asm("" : "+v"(x), "+v"(y));   // both are binary32 numbers first (as_rounded)
  return pack_f16(x, y);
}
__device__ __forceinline__ uint4 keys8(uint32_t c0, uint32_t c1, float4 s0, float4 s1, float4 z0, float4 z1) {
  return make_uint4(key2<0>(c0, s0.x, s0.y, z0.x, z0.y), key2<1>(c0, s0.z, s0.w, z0.z, z0.w), key2<0>(c1, s1.x, s1.y, z1.x, z1.y),
                    key2<1>(c1, s1.z, s1.w, z1.z, z1.w));
}
// Eight tokens are paired 0 4, 1 5, 2 6, 3 7, for then one mask takes two codes out of a dword; weights, scales and offsets go along.
__device__ __forceinline__ uint4 paired(uint4 x) {
  return make_uint4(__builtin_amdgcn_perm(x.z, x.x, 0x05040100u), __builtin_amdgcn_perm(x.z, x.x, 0x07060302u),
                    __builtin_amdgcn_perm(x.w, x.y, 0x05040100u), __builtin_amdgcn_perm(x.w, x.y, 0x07060302u));
}
// Two values: code scale + offset, rounded once; the codes as FP16 integers by the mantissa of 1024, which leaves exactly.  The scale's
// rounding to FP16 can take the largest code beyond the group's maximum, and beyond FP16's range where that is at its end (keys cannot:
// z and sigma are FP32, the largest code is the maximum within 2^-23).
template <int I>
__device__ __forceinline__ uint32_t value2(uint32_t codes, uint32_t scale, uint32_t off) {
  // (odd ones where they are, on the mantissa of 64: shifts are common to two of them)
  uint32_t bias = I & 1 ? 0x54005400u : 0x64006400u;
  asm("" : "+v"(bias));   // (in a register, so that mask and bias are one operation)
  const uint32_t biased = (codes >> (8 * (I >> 1)) & (I & 1 ? 0x00f000f0u : 0x000f000fu)) | bias;
  const f16x2 code = __builtin_bit_cast(f16x2, biased) - __builtin_bit_cast(f16x2, bias);
  const f16x2 x = __builtin_elementwise_fma(code, __builtin_bit_cast(f16x2, scale), __builtin_bit_cast(f16x2, off));
  const f16x2 most = {(_Float16)F16_MAX, (_Float16)F16_MAX};
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_minimum(x, most));
}
__device__ __forceinline__ uint4 values8(uint32_t d, uint4 scale, uint4 off) {
  return make_uint4(value2<0>(d, scale.x, off.x), value2<1>(d, scale.y, off.y), value2<2>(d, scale.z, off.z), value2<3>(d, scale.w, off.w));
}
// the width of a key channel in the bound, rounded up to FP16
__device__ __forceinline__ uint32_t key_width(float sigma, float z) {
  const float most = fmaxf(fabsf(fmaf(-128.0f, sigma, z)), fabsf(fmaf(127.0f, sigma, z)));
  const float w = as_rounded(fmaf(2.0f, fminf(0.5f * sigma, fmaf(most, 0x1p-11f, 0x1p-25f)), sigma));
  const _Float16 h = (_Float16)w;
  const uint32_t u = __builtin_bit_cast(uint16_t, h);
  return (float)h < w ? u + 1u : u;
}
__device__ __forceinline__ float value_error(float2 an) { return an.x + fminf(an.x, fmaf(an.y + an.x, 0x1p-11f, 0x1p-21f)); }

// What a wave holds of its 32 rows: lane l has row l & 31; its two halves have the tokens of different blocks.
struct TreeRows {
  f16x8 q[8];     // run of 8 channels (half * 8 + ks)
  f32x16 o[4];
  float m, sum, sealed, ev, evmax, dmax, vmax;
  int node;
};

// Rows of the queries on their way to the operands: 16 lanes fetch a row, four rows a request (a lane that fetched its own operand's
// pieces would ask for a line each), and the operands' pieces are read back, 16 bytes more between rows.
constexpr int Q_ROW = D * 2 + 16, Q_TILE = T_ROWS * Q_ROW;
__device__ __forceinline__ uint4 fetch_rows(const TreeArgs& a, int b, int kvh, int first) {
  const int l = threadIdx.x & 63, r = min(first + (l >> 4), a.n * a.group - 1), node = r / a.group;
  return ld16_any(a.q + (((int64_t)b * a.n + node) * a.n_kv * a.group + kvh * a.group + (r - node * a.group)) * D + (l & 15) * 8);
}
__device__ __forceinline__ void keep_rows(uint8_t* at, int row, uint4 x) {
  const int l = threadIdx.x & 63;
  *reinterpret_cast<uint4*>(at + (row + (l >> 4)) * Q_ROW + (l & 15) * 16) = x;
}
__device__ __forceinline__ void start_rows(TreeRows& s, const TreeArgs& a, int tile, const uint8_t* at) {
  const int l = threadIdx.x & 63;
  s.node = min(tile * T_ROWS + (l & 31), a.n * a.group - 1) / a.group;
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) s.q[ks] = *reinterpret_cast<const f16x8*>(at + (l & 31) * Q_ROW + ((l >> 5) * 8 + ks) * 16);
  s.m = -INFINITY;
  s.sum = s.sealed = s.ev = s.evmax = s.dmax = s.vmax = 0.0f;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) s.o[ct][r] = 0.0f;
}

// Products of 32 tokens with the wave's rows.  key(ks), value(oct, ct): the A operands.
template <typename Key>
__device__ __forceinline__ void scores32(const TreeRows& w, f32x16& s, Key key) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(key(ks), w.q[ks], s, 0, 0, 0);
}
template <typename Value>
__device__ __forceinline__ void values32(TreeRows& w, const uint32_t (&p)[8], Value value) {
#pragma unroll
  for (int oct = 0; oct < 2; ++oct)
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
      w.o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
          value(oct, ct), __builtin_bit_cast(f16x8, make_uint4(p[4 * oct], p[4 * oct + 1], p[4 * oct + 2], p[4 * oct + 3])), w.o[ct], 0, 0, 0);
}
// What weights relative to a largest score m are worth beside a largest one M >= m (-inf: there are none).
__device__ __forceinline__ float set_weight(float m, float M) { return m == M ? 1.0f : __builtin_amdgcn_exp2f((m - M) * SCORE); }
// Scores of MT times 32 tokens to weights, 2^MOST for a row's largest score so far, the row's m.  The weights enter
// the product with the values as FP16: those down to 2^-28 of the largest keep 11 bits, and a million lighter ones are together off by 2^-19
// of it.  (With 1 for the largest, tokens of 2^-25 of it vanished, and all of the result with them where the heavy ones' values are zero.)
// m is taken off ahead of the scaling, which costs an operation a score (8 heads, 131072 tokens, 64 nodes 184.0, 186.3 us; 20000 tokens, 256 nodes
// 65.4, 66.2): a scaled maximum has FP32's spacing, 8 and more from 2^26 on, and the largest weight then is more than FP16 holds, or nothing.
// bits(mt), where masked: the tokens of the lane's block that its row attends; eta(mt): the block's value error.
template <int MT, typename Bits, typename Eta>
__device__ __forceinline__ void softmax32(TreeRows& w, f32x16 (&s)[MT], uint32_t (&p)[MT][8], bool masked, Bits bits, Eta eta) {
  if (masked) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const uint32_t x = bits(mt);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = x >> r & 1u ? s[mt][r] : -INFINITY;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[mt][r]);
  top = max_x32(top);
  if (__any(top > w.m)) {
    const float mn = fmaxf(w.m, top);
    const float f = set_weight(w.m, mn);
    w.m = mn;
    w.sum *= f;
    w.sealed *= f;
    w.ev *= f;
    w.evmax *= f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[ct][r] *= f;
  }
  const float most = w.m == -INFINITY ? 0.0f : w.m;   // nothing attended yet: every weight is exp2(-inf) = 0
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float bs = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int i = (r & 4) * 2 + (r & 3);   // tokens i and i + 4
      const float x = __builtin_amdgcn_exp2f(fmaf(s[mt][i] - most, SCORE, MOST));
      const float y = __builtin_amdgcn_exp2f(fmaf(s[mt][i + 4] - most, SCORE, MOST));
      bs += x + y;
      p[mt][r] = pack_f16(x, y);
    }
    const float e = bs * eta(mt);
    w.sum += bs;
    w.ev += e;
    w.evmax = fmaxf(w.evmax, e);
  }
}
// All of it, of exact tokens.
template <typename Key, typename Value>
__device__ __forceinline__ void attend32(TreeRows& w, uint32_t bits, Key key, Value value) {
  f32x16 s[1];
  uint32_t p[1][8];
  scores32(w, s[0], key);
  softmax32<1>(w, s, p, true, [&](int) { return bits; }, [&](int) { return 0.0f; });
  values32(w, p[0], value);
}

// Delta of 32 blocks (or of fewer, repeated); width(ks): the A operand
template <typename Width>
__device__ __forceinline__ void bound_scores(TreeRows& w, Width width) {
  f32x16 d;
#pragma unroll
  for (int r = 0; r < 16; ++r) d[r] = 0.0f;
  uint32_t no_signs = 0x7fff7fffu;
  asm volatile("" : "+s"(no_signs));   // |q| is formed here: kept over the callers' loops it would take 32 registers
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    uint4 y = __builtin_bit_cast(uint4, w.q[ks]);
    y.x &= no_signs, y.y &= no_signs, y.z &= no_signs, y.w &= no_signs;
    d = __builtin_amdgcn_mfma_f32_32x32x16_f16(width(ks), __builtin_bit_cast(f16x8, y), d, 0, 0, 0);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) w.dmax = fmaxf(w.dmax, d[r]);
}

// place of token t of block `blk` among the keys of a tile: the A operand's rows are dealt to two blocks
__device__ __forceinline__ int key_place(int blk, int t) { return (blk >> 1) * 32 + (t >> 2) * 8 + (blk & 1) * 4 + (t & 3); }
// run of 8 tokens of channel c among the values of a tile: the A operand's rows are (c >> 6, c & 15), its tiles (c >> 4) & 3
__device__ __forceinline__ int value_place(int oct, int c) { return oct * D + ((c >> 4) & 3) * 32 + (c >> 6) * 16 + (c & 15); }

// Trailing and drafted tokens t0 .. t0 + TOK - 1 (of trail + n; zeros behind the last) by THREADS threads, thread `tid`.
//   keys [16 runs of 8 channels][TOK], values [TOK / 8][128] by value_place, norms [TOK], bad [TOK]: 1 for a token with a number that
//   is not finite (zeros before)
// Such a number must not meet the zero weight of a row that does not attend its token: it is taken out, and the rows that do attend
// the token get a sum that is no number.
template <int THREADS, int TOK>
__device__ __forceinline__ void load_exact(const TreeArgs& a, int64_t head, int t0, int tid, uint4* keys, uint4* values, float* norms, uint8_t* bad) {
  const int total = a.trail + a.n;
  const auto finite = [](uint32_t x) { return (uint32_t)((x & 0x7c00u) != 0x7c00u) & (uint32_t)((x & 0x7c000000u) != 0x7c000000u); };
  // (every address is a token's: the requests stand in no branch, and all come first)
  const __half* const tk = a.trail_k + head * BLK * D;
  const __half* const tv = a.trail_v + head * BLK * D;
  const __half* const dk = a.kd + (head * a.n - a.trail) * D;
  const __half* const dv = a.vd + (head * a.n - a.trail) * D;
  const auto token = [&](const __half* trail, const __half* drafts, int pos) {
    pos = min(pos, total - 1);
    return (pos < a.trail ? trail : drafts) + pos * D;
  };
  constexpr int NK = TOK * 16 / THREADS, NV = (TOK * 4 + THREADS - 1) / THREADS;
  uint4 kx[NK];
  uint2 vx[NV][8];
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const int i = tid + k * THREADS;
    kx[k] = ld16_any(token(tk, dk, t0 + (i >> 4)) + (i & 15) * 8);
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = tid + k * THREADS;
    if (THREADS > TOK * 4 && i >= TOK * 4) break;   // (whole waves)
#pragma unroll
    for (int j = 0; j < 8; ++j) vx[k][j] = ld8_any(token(tv, dv, t0 + (i >> 5) * 8 + j) + (i & 31) * 4);
  }
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const int i = tid + k * THREADS, t = i >> 4;
    uint4 x = kx[k];
    const uint32_t ok = finite(x.x) & finite(x.y) & finite(x.z) & finite(x.w), there = t0 + t < total;
    if (there & (ok ^ 1u)) bad[t] = 1;
    const uint32_t keep = 0u - (there & ok);
    x.x &= keep, x.y &= keep, x.z &= keep, x.w &= keep;
    keys[(i & 15) * TOK + key_place(t / BLK, t % BLK)] = x;
  }
  // four channels of eight tokens
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = tid + k * THREADS, oct = i >> 5, c = (i & 31) * 4;
    if (THREADS > TOK * 4 && i >= TOK * 4) break;
    uint32_t x[8][2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j][0] = vx[k][j].x;
      x[j][1] = vx[k][j].y;
    }
    float norm2 = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = oct * 8 + j;
      const f16x2 u = __builtin_bit_cast(f16x2, x[j][0]), v = __builtin_bit_cast(f16x2, x[j][1]);
      float sq = fmaf((float)u[0], (float)u[0], fmaf((float)u[1], (float)u[1], fmaf((float)v[0], (float)v[0], (float)v[1] * (float)v[1])));
      sq = sum_x16(row_sum(sq));   // the 32 lanes that have the token
      norm2 = (i & 31) == j ? sq : norm2;
      const uint32_t ok = finite(x[j][0]) & finite(x[j][1]), there = t0 + t < total;
      if (there & (ok ^ 1u)) bad[t] = 1;
      x[j][0] &= 0u - (there & ok);
      x[j][1] &= 0u - (there & ok);
    }
    if ((i & 31) < 8) norms[oct * 8 + (i & 31)] = sqrtf(norm2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = __builtin_amdgcn_perm(x[j + 4][e >> 1], x[j][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
      values[value_place(oct, c + e)] = make_uint4(h[0], h[1], h[2], h[3]);
    }
  }
}

// The open ones among the 16 trailing and drafted tokens from `first` on, for a node of sequence b.
__device__ __forceinline__ uint32_t open_tokens(const TreeArgs& a, int b, int node, int first) {
  const int j = first - a.trail;   // drafted node of the first token; below 0: trailing ones ahead of it
  if (a.mask == nullptr) {
    const int seen = node - j + 1;   // tokens up to the node itself
    return seen >= BLK ? 0xffffu : (seen > 0 ? (1u << seen) - 1u : 0u);
  }
  uint32_t x = 0u;
  const int lo = max(j, 0);
  if (j + BLK > 0 && lo < a.n) {
    const uint64_t* const mw = a.mask + ((int64_t)b * a.n + node) * a.words;
    uint64_t y = mw[lo >> 6] >> (lo & 63);
    if ((lo & 63) + BLK > 64 && (lo >> 6) + 1 < a.words) y |= mw[(lo >> 6) + 1] << (64 - (lo & 63));
    x = ((uint32_t)y & ((1u << min(a.n - lo, BLK)) - 1u)) << (lo - j);
  }
  if (j < 0) x |= (1u << min(-j, BLK)) - 1u;
  return x & 0xffffu;
}
// What the lane's row takes from its open tokens besides: the largest value norm, and no sum where one is not a number
__device__ __forceinline__ void open_exact(TreeRows& w, uint32_t bits, const float* norms, const uint8_t* bad) {
  uint32_t hit = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hit |= (reinterpret_cast<const uint32_t*>(bad)[i] * 0x10204080u >> 28) << (4 * i);   // a bit per byte
    const float4 x = reinterpret_cast<const float4*>(norms)[i];
    w.vmax = fmaxf(w.vmax, fmaxf(fmaxf(bits >> (4 * i) & 1u ? x.x : 0.0f, bits >> (4 * i + 1) & 1u ? x.y : 0.0f),
                                 fmaxf(bits >> (4 * i + 2) & 1u ? x.z : 0.0f, bits >> (4 * i + 3) & 1u ? x.w : 0.0f)));
  }
  if (bits & hit) w.sum = NAN;   // stays
}

// Joins the halves of the rows.  open: not 0 where the lane's row attends tokens that the wave has had.  Where these have left it no weight, all its scores are
// -inf, as a query that is not finite has them: the sum is no number, and 0 is that of a row that attends nothing.
__device__ __forceinline__ void end_rows(TreeRows& w, uint32_t open) {
  w.sum = sum_x32(w.sum);
  const float any = max_x32(open != 0u ? 1.0f : 0.0f);
  if (w.sum == 0.0f && any != 0.0f) w.sum = NAN;
  w.sealed = sum_x32(w.sealed);
  w.ev = sum_x32(w.ev);
  w.evmax = max_x32(w.evmax);
  w.dmax = max_x32(w.dmax) * HALF_SCORE;
  w.vmax = max_x32(w.vmax);
}
__device__ __forceinline__ void put_rows(const TreeRows& w, float* to) {
  const int l = threadIdx.x & 63, row = l & 31, half = l >> 5;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      // rows 8 r4 + 4 half + 0 .. 3 of the A operand: channels (r4 >> 1) 64 + ct 16 + (r4 & 1) 8 + half 4 + 0 .. 3
      const int c = (r4 >> 1) * 16 + ct * 4 + (r4 & 1) * 2 + half;
      reinterpret_cast<float4*>(to)[c * T_ROWS + row] = make_float4(w.o[ct][4 * r4], w.o[ct][4 * r4 + 1], w.o[ct][4 * r4 + 2], w.o[ct][4 * r4 + 3]);
    }
  float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // stay, unless a channel is no finite number
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) none[ct] = fmaf(0.0f, w.o[ct][r], none[ct]);
  const float bad = max_x32(none[0] + none[1] + none[2] + none[3] == 0.0f ? 0.0f : 1.0f);
  if (half == 0) {
    float* const st = to + T_OFLOATS + row;
    st[T_BAD * T_ROWS] = bad;
    st[T_M * T_ROWS] = w.m;
    st[T_L * T_ROWS] = w.sum;
    st[T_SEALED * T_ROWS] = w.sealed;
    st[T_EV * T_ROWS] = w.ev;
    st[T_EVMAX * T_ROWS] = w.evmax;
    st[T_DMAX * T_ROWS] = w.dmax;
    st[T_VMAX * T_ROWS] = w.vmax;
  }
}
// Joins N sets, `stride` floats apart, into one by THREADS threads (whole groups of 32).
template <int N, int THREADS>
__device__ __forceinline__ void join_sets(const float* sets, int stride, float* to, int tid) {
  const int row = tid & 31;
  float f[N], M = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    f[i] = sets[i * stride + T_OFLOATS + T_M * T_ROWS + row];
    M = fmaxf(M, f[i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = set_weight(f[i], M);
  for (int c = tid >> 5; c < 32; c += THREADS / 32) {
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float4 y = reinterpret_cast<const float4*>(sets + i * stride)[c * T_ROWS + row];
      x.x = fmaf(f[i], y.x, x.x), x.y = fmaf(f[i], y.y, x.y), x.z = fmaf(f[i], y.z, x.z), x.w = fmaf(f[i], y.w, x.w);
    }
    reinterpret_cast<float4*>(to)[c * T_ROWS + row] = x;
  }
  if (tid < 32) {
    float L = 0.0f, SL = 0.0f, E = 0.0f, EM = 0.0f, DM = 0.0f, VM = 0.0f, bad = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float* const st = sets + i * stride + T_OFLOATS + row;
      L = fmaf(f[i], st[T_L * T_ROWS], L);
      SL = fmaf(f[i], st[T_SEALED * T_ROWS], SL);
      E = fmaf(f[i], st[T_EV * T_ROWS], E);
      EM = fmaxf(EM, f[i] * st[T_EVMAX * T_ROWS]);
      DM = fmaxf(DM, st[T_DMAX * T_ROWS]);
      VM = fmaxf(VM, st[T_VMAX * T_ROWS]);
      bad = fmaxf(bad, st[T_BAD * T_ROWS]);
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
}
// ---- rows whose sets are all there: outputs --------------------------------------------------------------------------------------------

// Row r of a KV group among the outputs.
__device__ __forceinline__ int64_t row_out(const TreeArgs& a, int head, int r) {
  const int b = head / a.n_kv, kvh = head - b * a.n_kv, node = r / a.group;
  return ((int64_t)b * a.n + node) * a.n_kv * a.group + kvh * a.group + (r - node * a.group);
}
// Four channels; whether one is no finite number.
__device__ __forceinline__ bool put_channels(const TreeArgs& a, int64_t out, int c, float4 x, float inv) {
  // (a mean of values: where the rounding of the weights takes it beyond FP16's range, the values' largest, it stays there)
  const auto mean = [&](float v) { return v *= inv, isfinite(v) ? __builtin_amdgcn_fmed3f(v, -F16_MAX, F16_MAX) : v; };
  const float y[4] = {mean(x.x), mean(x.y), mean(x.z), mean(x.w)};
  reinterpret_cast<uint2*>(a.O + out * D)[c] = make_uint2(pack_f16(y[0], y[1]), pack_f16(y[2], y[3]));
  return !(isfinite(y[0]) && isfinite(y[1]) && isfinite(y[2]) && isfinite(y[3]));
}
__device__ __forceinline__ float mean_factor(float L) { return L == 0.0f ? 0.0f : 1.0f / L; }   // 0: the row attends nothing
struct Certificate {
  cqa_node_cert ct;
  uint32_t flags;
};
__device__ __forceinline__ Certificate certificate(const TreeArgs& a, float M, float L, float sealed, float E, float EM, float DM, float VM) {
  const float inv = mean_factor(L);
  const bool empty = L == 0.0f;
  Certificate x;
  cqa_node_cert& ct = x.ct;
  ct.E_val = E * inv;
  ct.delta_h = DM;
  ct.v_max = VM;
  ct.alpha_tail_hat = sealed * inv;
  ct.lse = empty ? -INFINITY : fmaf(M, SCORE * LN2, logf(L) - MOST * LN2);
  ct.max_block_contrib = EM * inv;
  ct.reserved = 0.0f;
  float tail = 0.0f;
  // (Sealed weights below 2^-126 are lost, 2^30 of them at most beside a sum of 2^14: a mass of 2^-110, which e^(4 Delta) can make a certain one.)
  if (a.nb > 0 && DM != 0.0f)
    tail = fminf(1.0f, expf((float)a.tol.mass_exp * DM) * (ct.alpha_tail_hat < 0x1p-110f ? 0x1p-110f : ct.alpha_tail_hat)) * expm1f(2.0f * DM);
  const float full = tanhf(DM);
  ct.E_key = 2.0f * VM * (a.tol.key_bound_mode == 0 ? fminf(full, tail) : (a.tol.key_bound_mode == 1 ? tail : full));
  uint32_t fl = a.tol.force_flags;
  if (ct.E_key > a.tol.eps_key) fl |= CQA_FLAG_KEY;
  if (ct.E_val > a.tol.eps_val || ct.max_block_contrib > a.tol.v_tol) fl |= CQA_FLAG_VAL;
  if (ct.E_key + ct.E_val > a.tol.eps_total) fl |= CQA_FLAG_TOTAL;
  if (!isfinite(ct.E_key) || !isfinite(ct.E_val) || !isfinite(DM) || !isfinite(VM) || (!empty && !isfinite(ct.lse))) fl |= CQA_FLAG_PRECOND;
  x.flags = fl;
  return x;
}
__device__ __forceinline__ void put_certificate(const TreeArgs& a, int64_t out, const Certificate& x, bool bad) {
  a.cert[out] = x.ct;
  a.flags[out] = x.flags | (bad ? CQA_FLAG_PRECOND : 0u);
}
// A wave's rows, from its registers.
__device__ __forceinline__ void finish_rows(const TreeRows& w, const TreeArgs& a, int head, int tile) {
  const int l = threadIdx.x & 63, half = l >> 5, r = tile * T_ROWS + (l & 31);
  if (r >= a.n * a.group) return;   // (both halves)
  const int64_t out = row_out(a, head, r);
  const float inv = mean_factor(w.sum);
  bool bad = false;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      bad |= put_channels(a, out, (r4 >> 1) * 16 + ct * 4 + (r4 & 1) * 2 + half, make_float4(w.o[ct][4 * r4], w.o[ct][4 * r4 + 1], w.o[ct][4 * r4 + 2], w.o[ct][4 * r4 + 3]), inv);
  bad = __shfl_xor((int)bad, 32) != 0 || bad;
  if (half == 0) put_certificate(a, out, certificate(a, w.m, w.sum, w.sealed, w.ev, w.evmax, w.dmax, w.vmax), bad);
}
// ROWS rows from r32 = `first` of a tile on, of which all sets, up to N of them (n, `stride` floats apart), are at `sets`, by THREADS threads:
// the last 64 have the certificates, the others the channels.
template <int N, int ROWS, int THREADS>
__device__ __forceinline__ void finish_sets(const float* sets, int64_t stride, int n, const TreeArgs& a, int head, int tile, int first, int tid) {
  constexpr int WIDE = THREADS - 64;
  static_assert(WIDE > 0 && WIDE % ROWS == 0 && ROWS <= 64, "whole rows");
  const int row = tid % ROWS, r32 = first + row, r = tile * T_ROWS + r32;
  const bool there = r < a.n * a.group, certifies = there && tid >= WIDE && tid < WIDE + ROWS;
  const int64_t out = row_out(a, head, r);
  // (places behind the last set read it again, with weight 0: no request stands in a branch, and none waits for another)
  const auto set = [&](int i) { return sets + (int64_t)min(i, n - 1) * stride; };
  const auto quantity = [&](int i, int t) { return set(i)[T_OFLOATS + t * T_ROWS + r32]; };
  float f[N], l[N], M = -INFINITY, L = 0.0f;
  const auto weigh = [&] {   // the sets' maxima in f become their weights
#pragma unroll
    for (int i = 0; i < N; ++i) M = fmaxf(M, f[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f[i] = set_weight(f[i], M) * (i < n ? 1.0f : 0.0f);
      L = fmaf(f[i], l[i], L);
    }
  };
  if (certifies) {
    float z[N][6];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f[i] = quantity(i, T_M);
      l[i] = quantity(i, T_L);
#pragma unroll
      for (int t = 0; t < 6; ++t) z[i][t] = quantity(i, T_SEALED + t);
    }
    weigh();
    float SL = 0.0f, E = 0.0f, EM = 0.0f, DM = 0.0f, VM = 0.0f, bad = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      SL = fmaf(f[i], z[i][0], SL);
      E = fmaf(f[i], z[i][1], E);
      EM = fmaxf(EM, f[i] * z[i][2]);
      DM = fmaxf(DM, z[i][3]);
      VM = fmaxf(VM, z[i][4]);
      bad = fmaxf(bad, z[i][5]);
    }
    put_certificate(a, out, certificate(a, M, L, SL, E, EM, DM, VM), bad != 0.0f);
  } else if (there && tid < WIDE) {
    int c = tid / ROWS;
    float4 y[N];
    const auto request = [&] {
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = reinterpret_cast<const float4*>(set(i))[c * T_ROWS + r32];
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f[i] = quantity(i, T_M);
      l[i] = quantity(i, T_L);
    }
    request();
    weigh();
    const float inv = mean_factor(L);
    while (true) {
      float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < N; ++i) x.x = fmaf(f[i], y[i].x, x.x), x.y = fmaf(f[i], y[i].y, x.y), x.z = fmaf(f[i], y[i].z, x.z), x.w = fmaf(f[i], y[i].w, x.w);
      put_channels(a, out, c, x, inv);
      c += WIDE / ROWS;
      if (c >= 32) break;
      request();
    }
  }
}

__device__ __forceinline__ float* set_of(const TreeArgs& a, int64_t head, int tile, int split) {
  return a.part + ((head * a.row_tiles + tile) * a.nsplit + split) * T_FLOATS;
}

// ---- 32 rows a workgroup: bound by the cache's bytes and their reconstruction ------------------------------------------------------------
//
// A wave takes pairs of blocks by itself and reconstructs them in registers, in the operands' layout: a 16-byte piece of key codes (16
// channels of a token) is two operands' part of its lane, a dword of value codes (8 tokens of a channel) one.  Only the metadata, which 16
// lanes share, goes through LDS, the wave's own part of it, so that no wave waits for another until the waves' sets are joined.
// Two waves a SIMD: what one is to read from LDS is requested a product ahead, and a pair's metadata and codes as soon as those of the pair before
// are used.  4 x 8 KV heads of 32768 tokens, 5 nodes of 4 query heads: 60 - 64 us for 303 MB, 4.7 - 5.0 TB/s, about what a large copy reaches (each read
// where it is used took a tenth more, the widths' products for each pair by itself among it); vector ALU 65 - 70 % busy, matrix cores 15 %.
constexpr int FEW_WAVES = 8;
constexpr int FEW_KM_HALF = 64 + 4, FEW_KM_KIND = 2 * FEW_KM_HALF, FEW_KM_BLK = 2 * FEW_KM_KIND + 8;   // floats; padded: the four
constexpr int FEW_VM_BLK = VM_BYTES + 32, FEW_W_RUN = 32 * 16 + 16;                                   // addresses of a read in four sets of banks
constexpr int FEW_KM = 0, FEW_VM = FEW_KM + 2 * FEW_KM_BLK * 4, FEW_W = FEW_VM + 2 * FEW_VM_BLK, FEW_META_END = FEW_W + D / 8 * FEW_W_RUN;   // widths [run of 8 channels][32 blocks]
constexpr int FEW_EXACT = 96;   // trailing and drafted tokens of a turn, at most
static_assert(FEW_META_END <= T_FLOATS * 4 && 2 * FEW_EXACT * D * 2 <= FEW_WAVES * T_FLOATS * 4 && FEW_VM % 16 == 0 && FEW_W % 16 == 0,
              "a wave's part of LDS");

// EXACT: tokens of a turn of the trailing and drafted ones.  64 where they are no more, for each thread fetches its share of EXACT (1 KV head, 1029 tokens, 8 nodes
// of 4 query heads 10.7 us a call in a graph, with 96 11.3; 8 heads, 60 tokens, 12 nodes 9.9, 10.4), else 96 (64 nodes 10.6, by turns of 64 12.8; 256 nodes, 500
// tokens 22.6, 26.1).
template <int EXACT>
__global__ __launch_bounds__(512, 2) void tree_few_kernel(TreeArgs a) {
  static_assert(EXACT <= FEW_EXACT, "LDS");
  fetch_args<sizeof(TreeArgs)>();
  __shared__ __align__(16) float s_set[FEW_WAVES][T_FLOATS];
  __shared__ __align__(16) uint8_t s_q[Q_TILE];
  __shared__ __align__(16) float s_norm[EXACT];
  __shared__ __align__(16) uint8_t s_bad[EXACT];
  const int tid = threadIdx.x, l = tid & 63, n32 = l & 31, half = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t head = blockIdx.x;
  const int split = blockIdx.y, tile = blockIdx.z;
  const int b = (int)(head / a.n_kv), kvh = (int)(head - (int64_t)b * a.n_kv);
  uint8_t* const mine = reinterpret_cast<uint8_t*>(s_set[w]);
  TreeRows rows;

  const uint8_t* const base = a.t1 + head * a.nq_cap * QUAD_BYTES;
  const int units = (int)((a.nb + 1) >> 1);                 // pairs of sealed blocks
  const int step = FEW_WAVES * a.nsplit;
  const int bsel = (n32 >> 2) & 1, tok = (n32 >> 3) * 4 + (n32 & 3);   // the lane's token as a row of the keys' operand
  uint4 kc[4], km0, km1, vc0, vc1, vm;   // (arrays of two went to LDS)
  float2 an;
  // (behind the last pair: the head's first, which is not used)
  const auto record = [&](int u) { return base + (int64_t)(u < units ? u >> 1 : 0) * QUAD_BYTES; };
  const auto load_keys = [&](int u) {
    const uint8_t* const r = record(u);
    const int b0 = (u & 1) * 2;
    const uint8_t* const p = r + Q_KC + (b0 + bsel) * KC_BYTES + half * 1024 + tok * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) kc[i] = *reinterpret_cast<const uint4*>(p + i * 256);
  };
  const auto load_meta = [&](int u) {
    const uint8_t* const r = record(u);
    const int b0 = (u & 1) * 2;
    km0 = reinterpret_cast<const uint4*>(r + Q_KM + b0 * KM_BYTES)[l];
    km1 = reinterpret_cast<const uint4*>(r + Q_KM + (b0 + 1) * KM_BYTES)[l];
    vm = reinterpret_cast<const uint4*>(r + Q_VM + b0 * VM_BYTES)[l];
    an = reinterpret_cast<const float2*>(r + Q_AN)[b0 + half];
  };
  const auto load_values = [&](int u) {
    const uint8_t* const r = record(u);
    const int b0 = (u & 1) * 2;
    vc0 = reinterpret_cast<const uint4*>(r + Q_VC + (b0 + half) * VC_BYTES)[n32];
    vc1 = reinterpret_cast<const uint4*>(r + Q_VC + (b0 + half) * VC_BYTES + 512)[n32];
  };
  int u = split * FEW_WAVES + w;
  const uint4 q_in = fetch_rows(a, b, kvh, tile * T_ROWS + 4 * w);
  load_meta(u);
  load_keys(u);
  load_values(u);
  keep_rows(s_q, 4 * w, q_in);
  __syncthreads();
  start_rows(rows, a, tile, s_q);

  const float* const sg = reinterpret_cast<const float*>(mine + FEW_KM) + bsel * FEW_KM_BLK + half * FEW_KM_HALF;
  const uint8_t* const sc = mine + FEW_VM + half * FEW_VM_BLK + (n32 >> 4) * 64;
  for (int turn = 0; u < units; u += step, ++turn) {
    // metadata: sigma and z by (block, kind, half of the channels), scales and offsets by block
    float* const skm = reinterpret_cast<float*>(mine + FEW_KM);
    float* const at = skm + half * FEW_KM_KIND + ((l >> 4) & 1) * FEW_KM_HALF + (l & 15) * 4;
    *reinterpret_cast<uint4*>(at) = km0;
    *reinterpret_cast<uint4*>(at + FEW_KM_BLK) = km1;
    *reinterpret_cast<uint4*>(mine + FEW_VM + half * FEW_VM_BLK + n32 * 16) = paired(vm);
    const float eta = value_error(an);
    rows.vmax = fmaxf(rows.vmax, an.y);
    load_meta(u + step);
    wave_sync();
    // Operands' metadata are read a product ahead of their use.
    float4 m4[2][4];
    const auto key_meta = [&](auto ks_) {
      constexpr int ks = ks_.value;
#pragma unroll
      for (int i = 0; i < 4; ++i) m4[ks & 1][i] = *reinterpret_cast<const float4*>(sg + (i >> 1) * FEW_KM_KIND + ks * 8 + (i & 1) * 4);
    };
    key_meta(std::integral_constant<int, 0>{});
    // widths: four channels a lane
    {
      const int c = n32 * 4;
      const float* const p = skm + half * FEW_KM_BLK + (c >> 6) * FEW_KM_HALF + (c & 63);
      const float4 s4 = *reinterpret_cast<const float4*>(p), z4 = *reinterpret_cast<const float4*>(p + FEW_KM_KIND);
      *reinterpret_cast<uint2*>(mine + FEW_W + (c >> 3) * FEW_W_RUN + ((turn & 15) * 2 + half) * 16 + (c & 4) * 2) =
          make_uint2(key_width(s4.x, z4.x) | key_width(s4.y, z4.y) << 16, key_width(s4.z, z4.z) | key_width(s4.w, z4.w) << 16);
    }
    f32x16 x[1];
    uint32_t p[1][8];
#pragma unroll
    for (int r = 0; r < 16; ++r) x[0][r] = 0.0f;
    each<8>([&](auto ks_) {
      constexpr int ks = ks_.value;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (ks < 7) key_meta(std::integral_constant<int, ks + 1>{});
      const uint32_t c0 = ks & 1 ? kc[ks >> 1].z : kc[ks >> 1].x, c1 = ks & 1 ? kc[ks >> 1].w : kc[ks >> 1].y;
      const float4* const m = m4[ks & 1];
      x[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, keys8(c0, c1, m[0], m[1], m[2], m[3])), rows.q[ks], x[0], 0, 0, 0);
    });
    __builtin_amdgcn_sched_barrier(0);
    load_keys(u + step);
    uint4 v4[2][2];
    const auto value_meta = [&](auto i_) {
      constexpr int I = i_.value;   // (octet, channel tile)
      const uint8_t* const p = sc + (I >> 2) * 128 + (I & 3) * 16;
      v4[I & 1][0] = *reinterpret_cast<const uint4*>(p);
      v4[I & 1][1] = *reinterpret_cast<const uint4*>(p + 256);
    };
    value_meta(std::integral_constant<int, 0>{});
    if ((turn & 15) == 15 || u + step >= units) {
      wave_sync();
      const int blk = min(n32, (turn & 15) * 2 + 1);
      bound_scores(rows, [&](int ks) { return *reinterpret_cast<const f16x8*>(mine + FEW_W + (half * 8 + ks) * FEW_W_RUN + blk * 16); });
      wave_sync();
    }
    softmax32<1>(
        rows, x, p, (int64_t)u * 2 + 2 > a.nb, [&](int) { return (int64_t)u * 2 + half < a.nb ? 0xffffu : 0u; }, [&](int) { return eta; });
    each<8>([&](auto i_) {
      constexpr int I = i_.value, ct = I & 3, oct = I >> 2;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (I < 7) value_meta(std::integral_constant<int, I + 1>{});
      const uint4 v = oct ? vc1 : vc0;
      const uint32_t c = ct == 0 ? v.x : (ct == 1 ? v.y : (ct == 2 ? v.z : v.w));
      rows.o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, values8(c, v4[I & 1][0], v4[I & 1][1])),
                                                          __builtin_bit_cast(f16x8, make_uint4(p[0][4 * oct], p[0][4 * oct + 1], p[0][4 * oct + 2], p[0][4 * oct + 3])),
                                                          rows.o[ct], 0, 0, 0);
    });
    __builtin_amdgcn_sched_barrier(0);
    load_values(u + step);
    wave_sync();
  }
  rows.sealed = rows.sum;
  uint32_t open = split * FEW_WAVES + w < units;
  // The other tokens, dealt from the workgroup on whose turn is the next, which fetches them together; as many of its waves as they have pairs of blocks attend them.
  for (int t0 = (split + a.nsplit - (units + FEW_WAVES - 1) / FEW_WAVES % a.nsplit) % a.nsplit * EXACT; t0 < a.trail + a.n; t0 += a.nsplit * EXACT) {
    uint4* const s_k = reinterpret_cast<uint4*>(s_set);
    uint4* const s_v = s_k + 16 * EXACT;
    const int blk = 2 * w + half;
    const uint32_t bits = open_tokens(a, b, rows.node, t0 + blk * BLK);
    if (tid < EXACT / 4) reinterpret_cast<uint32_t*>(s_bad)[tid] = 0u;
    __syncthreads();
    load_exact<64 * FEW_WAVES, EXACT>(a, head, t0, tid, s_k, s_v, s_norm, s_bad);
    __syncthreads();
    if (w * 32 < min(EXACT, a.trail + a.n - t0)) {
      open |= bits;
      open_exact(rows, bits, s_norm + blk * BLK, s_bad + blk * BLK);
      attend32(
          rows, bits, [&](int ks) { return __builtin_bit_cast(f16x8, s_k[(half * 8 + ks) * EXACT + w * 32 + n32]); },
          [&](int oct, int ct) { return __builtin_bit_cast(f16x8, s_v[(blk * 2 + oct) * D + ct * 32 + n32]); });
    }
    __syncthreads();   // (the next ones, or the waves' sets, come where these are)
  }
  end_rows(rows, open);
  put_rows(rows, s_set[w]);
  __syncthreads();
  if (a.nsplit > 1) {
    join_sets<FEW_WAVES, 512>(s_set[0], T_FLOATS, set_of(a, head, tile, split), tid);
    return;
  }
  finish_sets<FEW_WAVES, T_ROWS, 512>(s_set[0], T_FLOATS, FEW_WAVES, a, (int)head, tile, 0, tid);
}

// ---- many rows: bound by the products -------------------------------------------------------------------------------------------------
//
// Eight waves, WR side by side over rows (32 each) and WT over tokens; four of them reconstruct the tile's keys and four its values
// into LDS, a block each, for all.  A SIMD has a wave of either kind, and they take turns with a barrier between the phases: while one
// multiplies (the last tile's weights with its values, the next one's keys with the queries) and reconstructs between its products,
// the other one turns scores into weights, so that the matrix cores and the vector ALU of a SIMD both have work.  Phases numbered from 0:
//   keys' waves    phase 2 t      values of t - 1, scores of t, reconstruct the keys of t + 1      phase 2 t + 1  weights of t
//   values' waves  phase 2 t + 1  values of t - 1, scores of t, reconstruct the values of t        phase 2 t + 2  weights of t
// Keys of t are read in 2 t and 2 t + 1 and replaced (t + 2) in 2 t + 2; values of t are read in 2 t + 2 and 2 t + 3 and replaced
// in 2 t + 5: two tiles in LDS.  eta of t comes with the keys in 2 t - 2 and is read until 2 t + 2: four of them.  Codes are requested a tile
// ahead.  (Reconstruction in the weights' phase: products 1310 cycles, weights and reconstruction 2600, of which the products' wave waited half.)
// 8 KV heads of 131072 tokens, 64 nodes of 4 query heads: 173 - 208 us in a trace (178 of a call of 187) for 142 GFLOP, 680 - 820 TFLOP/s; vector ALU 71 % and matrix
// cores 46 % busy, at a clock that falls from 2.4 to 1.6 - 1.8 GHz meanwhile.
template <int WR>
struct ManyShape {
  static constexpr int WT = 8 / WR;
  static constexpr int MT = WR == 8 ? 2 : 1;      // times 32 tokens a wave takes of a tile
  static constexpr int TOK = 32 * MT * WT;
  static constexpr int QUADS = TOK / 64, BLKS = TOK / BLK;
  static constexpr int TILE = 2 * TOK * D * 2;    // keys [16 runs][TOK], values [TOK / 8][128], 16 bytes each
  // LDS: two tiles, the waves' metadata of a block (16 bytes more behind each 64 floats), the widths of 32 blocks while the next 32 come;
  // at the end the waves' sets, where there are some to be joined
  static constexpr int META = KM_BYTES + 4 * 16, META_AT = 2 * TILE, WIDTH_AT = META_AT + 8 * META, END = WIDTH_AT + 2 * 32 * D * 2;
  static constexpr int BYTES = WT > 1 && 8 * T_FLOATS * 4 > END ? 8 * T_FLOATS * 4 : END;
};

template <int WR>
__global__ __launch_bounds__(512, 2) void tree_many_kernel(TreeArgs a) {
  fetch_args<sizeof(TreeArgs)>();
  using S = ManyShape<WR>;
  constexpr int MT = S::MT, TOK = S::TOK, QUADS = S::QUADS, BLKS = S::BLKS;
  __shared__ __align__(16) uint8_t s_main[S::BYTES];
  __shared__ float s_eta[4][BLKS];
  __shared__ __align__(16) float s_norm[TOK];
  __shared__ __align__(16) uint8_t s_bad[TOK];

  const int tid = threadIdx.x, l = tid & 63, n32 = l & 31, half = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = w % WR, wt = w / WR, wb = w & 3;
  const int64_t head = blockIdx.x;
  const int split = blockIdx.y;
  const int b = (int)(head / a.n_kv), kvh = (int)(head - (int64_t)b * a.n_kv);
  const int tile0 = blockIdx.z * WR;
  uint8_t* const s_meta = s_main + S::META_AT + w * S::META;
  // [ring][run of 8 channels][block], 16 bytes
  const auto width_at = [&](int ring, int run, int blk) { return s_main + S::WIDTH_AT + ((ring * (D / 8) + run) * 32 + blk) * 16; };
  TreeRows rows;

  const uint8_t* const base = a.t1 + head * a.nq_cap * QUAD_BYTES;
  const int nquads = (int)((a.nb + 3) >> 2);
  const int even = a.nsplit - a.last, mid = min(split, even);
  const int from = mid * a.share + min(mid, a.over) + (split - mid) * a.least;
  const int units = from + (split < even ? a.share + (split < a.over) : a.least);   // the workgroup's tiles: from .. units - 1
  // the wave's block of each quad of the tile: keys, lane (run pair c8, token t8) has 16 channels of tokens t8 and t8 + 8; values, lane (octet
  // oc, n = gh 16 + n16) has four channels of eight tokens
  const int t8 = l & 7, c8 = l >> 3;
  uint4 raw[QUADS][3];
  float2 an[QUADS];
  float nu = 0.0f;
  // The same requests for either kind of waves, at their own offsets: in a branch, what joins behind it is waited for there.
  const uint32_t at0 = w < 4 ? Q_KC + wb * KC_BYTES + c8 * 256 + t8 * 16 : Q_VC + wb * VC_BYTES + l * 16;
  const uint32_t at1 = w < 4 ? at0 + 128 : at0;
  const uint32_t at2 = w < 4 ? Q_KM + wb * KM_BYTES + l * 16 : Q_VM + wb * VM_BYTES + n32 * 16;
  const auto load = [&](int u) {
#pragma unroll
    for (int qd = 0; qd < QUADS; ++qd) {
      int quad = u * QUADS + qd;
      if (u >= units || quad >= nquads) quad = 0;   // behind the last: any record of the head
      const uint8_t* const r = base + (int64_t)quad * QUAD_BYTES;
      raw[qd][0] = *reinterpret_cast<const uint4*>(r + at0);
      raw[qd][1] = *reinterpret_cast<const uint4*>(r + at1);
      raw[qd][2] = *reinterpret_cast<const uint4*>(r + at2);
      an[qd] = reinterpret_cast<const float2*>(r + Q_AN)[wb];
    }
  };
  int u = from;
  load(u);
  {
    static_assert(8 * Q_TILE <= S::BYTES, "the queries on their way");
    uint8_t* const s_q = s_main + w * Q_TILE;
    uint4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fetch_rows(a, b, kvh, (tile0 + wr) * T_ROWS + 4 * i);
#pragma unroll
    for (int i = 0; i < 8; ++i) keep_rows(s_q, 4 * i, x[i]);
    wave_sync();
    start_rows(rows, a, tile0 + wr, s_q);
  }
  int fresh = 0, ring = 0;   // blocks whose widths have come into the half `ring`
  int buf = 0;
  __syncthreads();

  const auto key_of = [&](const uint4* s_k, int unit, int ks) { return __builtin_bit_cast(f16x8, s_k[(half * 8 + ks) * TOK + unit * 32 + n32]); };
  // From one phase to the next: nothing of either is moved across.
  const auto turn_over = [] {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto value_of = [&](const uint4* s_v, int blk, int oct, int ct) { return __builtin_bit_cast(f16x8, s_v[(blk * 2 + oct) * D + ct * 32 + n32]); };
  // The wave's part of a tile, keys and widths and eta, or values.  Metadata go through LDS (stage): 512 bytes of either kind, the
  // second one (zero points, offsets) 544 bytes behind the first.
  const auto stage = [&](auto keys, int qd) {
    if constexpr (keys.value)
      *reinterpret_cast<uint4*>(s_meta + (l * 4 + (l >> 4) * 4) * 4) = raw[qd][2];
    else if (half == 0)
      *reinterpret_cast<uint4*>(s_meta + (n32 >> 4) * 544 + (n32 & 15) * 16) = paired(raw[qd][2]);
    wave_sync();
  };
  // The reconstruction of the wave's block of quad qd in PIECES pieces of some five operations, J = 0, 1, ...; metadata are read a group of
  // five pieces ahead of their use, the first ones by begin.
  constexpr int PIECES = 24;
  uint4 m4[2][4], out4;
  float2 w2[2];
  const auto begin = [&](auto keys) {
    const uint8_t* const m = s_meta + (keys.value ? (c8 * 16 + (c8 >> 2) * 4) * 4 : (l >> 5) * 128 + ((l >> 4) & 1) * 64);
    if constexpr (keys.value) {
#pragma unroll
      for (int i = 0; i < 4; ++i) m4[0][i] = *reinterpret_cast<const uint4*>(m + (i >> 1) * 544 + (i & 1) * 16);
    } else {
      m4[0][0] = *reinterpret_cast<const uint4*>(m);
      m4[0][1] = *reinterpret_cast<const uint4*>(m + 544);
    }
  };
  const auto reconstruct = [&](auto keys, auto qd_, auto j_, int buf, int ring, int slot, int turn) {
    constexpr int qd = qd_.value, J = j_.value, G = J / 5, R = J % 5;
    uint4* const s_k = reinterpret_cast<uint4*>(s_main + buf * S::TILE);
    uint4* const s_v = s_k + 16 * TOK;
    const int blk = qd * 4 + wb;
    if constexpr (keys.value) {
      const uint8_t* const m = s_meta + (c8 * 16 + (c8 >> 2) * 4) * 4;
      const int ch = c8 * 16 + 2 * t8;
      if constexpr (G < 4 && R == 0) {
        if constexpr (G == 1)
#pragma unroll
          for (int i = 0; i < 4; ++i) m4[1][i] = *reinterpret_cast<const uint4*>(m + 32 + (i >> 1) * 544 + (i & 1) * 16);
        if constexpr (G == 2) {   // of the widths: two channels a lane
          w2[0] = reinterpret_cast<const float2*>(m)[t8];
          w2[1] = reinterpret_cast<const float2*>(m + 544)[t8];
        }
      } else if constexpr (G < 4) {
        // eight channels E of token t8 + 8 T, two a piece
        constexpr int E = G >> 1, T = G & 1, I = R - 1;
        const uint4& x = raw[qd][T];
        const uint32_t c = E ? (I < 2 ? x.z : x.w) : (I < 2 ? x.x : x.y);
        const uint4 sg = m4[E][I >> 1], zz = m4[E][2 + (I >> 1)];
        const uint32_t y = key2<(I & 1)>(c, __uint_as_float(I & 1 ? sg.z : sg.x), __uint_as_float(I & 1 ? sg.w : sg.y),
                                         __uint_as_float(I & 1 ? zz.z : zz.x), __uint_as_float(I & 1 ? zz.w : zz.y));
        (I == 0 ? out4.x : I == 1 ? out4.y : I == 2 ? out4.z : out4.w) = y;
        if constexpr (I == 3) s_k[(2 * c8 + E) * TOK + key_place(blk, t8 + 8 * T)] = out4;
      } else if constexpr (R == 0) {
        out4.x = key_width(w2[0].x, w2[1].x);
      } else if constexpr (R == 1) {
        *reinterpret_cast<uint32_t*>(width_at(ring, ch >> 3, slot + blk) + (ch & 7) * 2) = out4.x | key_width(w2[0].y, w2[1].y) << 16;
      } else if constexpr (R == 2) {
        s_eta[turn & 3][blk] = value_error(an[qd]);   // (every lane the same)
        nu = fmaxf(nu, an[qd].y);
      }
    } else if constexpr (G < 4) {
      // eight tokens of octet oc of channel (gh 4 + G) 16 + n16, two a piece
      const int oc = l >> 5, gh = (l >> 4) & 1, n16 = l & 15;
      if constexpr (R == 0) {
        if constexpr (G < 3) {
          const uint8_t* const m = s_meta + oc * 128 + gh * 64 + (G + 1) * 16;
          m4[(G + 1) & 1][0] = *reinterpret_cast<const uint4*>(m);
          m4[(G + 1) & 1][1] = *reinterpret_cast<const uint4*>(m + 544);
        }
      } else {
        constexpr int I = R - 1;
        const uint4 &x = raw[qd][0], &sc = m4[G & 1][0], &of = m4[G & 1][1];
        const uint32_t y = value2<I>(G == 0 ? x.x : G == 1 ? x.y : G == 2 ? x.z : x.w, I == 0 ? sc.x : I == 1 ? sc.y : I == 2 ? sc.z : sc.w,
                                     I == 0 ? of.x : I == 1 ? of.y : I == 2 ? of.z : of.w);
        (I == 0 ? out4.x : I == 1 ? out4.y : I == 2 ? out4.z : out4.w) = y;
        if constexpr (I == 3) s_v[value_place(blk * 2 + oc, (gh * 4 + G) * 16 + n16)] = out4;
      }
    }
  };
  f32x16 sc[MT];
  uint32_t p[MT][8];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int r = 0; r < 8; ++r) p[mt][r] = 0u;
  const auto add_values = [&](int buf) {
    const uint4* const s_v = reinterpret_cast<const uint4*>(s_main + buf * S::TILE) + 16 * TOK;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) values32(rows, p[mt], [&](int oct, int ct) { return value_of(s_v, (wt * MT + mt) * 2 + half, oct, ct); });
  };
  // The products of a phase in their order, operands read AHEAD products ahead, and behind each some pieces of the reconstruction.  (Left to
  // the compiler, which cannot tell the tiles apart, each operand was read when it was needed: 3310 cycles a phase.)
  constexpr int PRODUCTS = 16 * MT, AHEAD = 6, FROM = 2, EACH = QUADS == 2 ? 4 : 2, BEHIND = FROM + PIECES * QUADS / EACH;
  static_assert(PIECES * QUADS % EACH == 0 && BEHIND < PRODUCTS, "the pieces end ahead of the products");
  const auto sealed_tiles = [&](auto keys) {
    for (int turn = 0; u < units; ++u, buf ^= 1, ++turn) {
      const bool last = u + 1 >= units, full = fresh == 32;
      const int ring1 = full ? ring ^ 1 : ring, slot = full ? 0 : fresh;   // where the next tile's widths go
      const uint4* const s_k = reinterpret_cast<const uint4*>(s_main + buf * S::TILE);
      const uint4* const s_v = reinterpret_cast<const uint4*>(s_main + (buf ^ 1) * S::TILE) + 16 * TOK;
      f16x8 f[AHEAD];
      // product I: values (mt, octet, channel tile), then keys (channels, mt): the accumulators take turns
      const auto operand = [&](auto i_) {
        constexpr int I = i_.value, K = I - 8 * MT;
        if constexpr (K < 0)
          f[I % AHEAD] = value_of(s_v, (wt * MT + I / 8) * 2 + half, (I & 7) >> 2, I & 3);
        else
          f[I % AHEAD] = key_of(s_k, wt * MT + K % MT, K / MT);
      };
      const auto product = [&](auto i_) {
        constexpr int I = i_.value, K = I - 8 * MT;
        if constexpr (K < 0) {
          const uint32_t* const x = &p[I / 8][(I & 4)];
          rows.o[I & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[I % AHEAD], __builtin_bit_cast(f16x8, make_uint4(x[0], x[1], x[2], x[3])), rows.o[I & 3], 0, 0, 0);
        } else {
          if constexpr (K < MT)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[K][r] = 0.0f;
          sc[K % MT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[I % AHEAD], rows.q[K / MT], sc[K % MT], 0, 0, 0);
        }
      };
      __builtin_amdgcn_s_setprio(1);
      stage(keys, 0);
      each<AHEAD>(operand);
      begin(keys);
      __builtin_amdgcn_sched_barrier(0);
      each<PRODUCTS>([&](auto i_) {
        constexpr int I = i_.value;
        product(i_);
        if constexpr (I + AHEAD < PRODUCTS) operand(std::integral_constant<int, I + AHEAD>{});
        // (keys, behind the last tile: of the head's first record, which nothing reads)
        if constexpr (I >= FROM)
          each<EACH>([&](auto k_) {
            constexpr int P = (I - FROM) * EACH + k_.value, QD = P / PIECES, J = P % PIECES;
            if constexpr (P < PIECES * QUADS) {
              if constexpr (QD > 0 && J == 0) {
                stage(keys, QD);
                begin(keys);
              }
              reconstruct(keys, std::integral_constant<int, QD>{}, std::integral_constant<int, J>{}, keys.value ? buf ^ 1 : buf, ring1, slot, turn + 1);
            }
          });
        if constexpr (I == BEHIND) load(keys.value ? u + 2 : u + 1);
        __builtin_amdgcn_sched_barrier(0);
      });
      if (full || last) {
        // (up to the last block that has come: on the last tile, other waves write the first record's widths behind it meanwhile)
        const int blk = min(n32, fresh - 1);
        if (wt == 0) bound_scores(rows, [&](int ks) { return *reinterpret_cast<const f16x8*>(width_at(ring, half * 8 + ks, blk)); });
      }
      ring = ring1;
      fresh = slot + BLKS;
      __builtin_amdgcn_s_setprio(0);
      turn_over();
      softmax32<MT>(
          rows, sc, p, (int64_t)(u + 1) * BLKS > a.nb, [&](int mt) { return (int64_t)u * BLKS + (wt * MT + mt) * 2 + half < a.nb ? 0xffffu : 0u; },
          [&](int mt) { return s_eta[turn & 3][(wt * MT + mt) * 2 + half]; });
      turn_over();
    }
  };
  if (u < units) {
    // the values that the first turn's weights, zeros, meet
    for (int i = tid; i < 16 * TOK; i += 512) (reinterpret_cast<uint4*>(s_main + S::TILE) + 16 * TOK)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (w < 4) {
      each<QUADS>([&](auto qd) {
        stage(std::true_type{}, qd.value);
        begin(std::true_type{});
        each<PIECES>([&](auto j) { reconstruct(std::true_type{}, qd, j, 0, 0, 0, 0); });
      });
      load(u + 1);
    }
    fresh = BLKS;
    __syncthreads();
    if (w < 4) {
      sealed_tiles(std::true_type{});
      turn_over();
    } else {
      turn_over();
      sealed_tiles(std::false_type{});
    }
    add_values(buf ^ 1);
  }
  rows.sealed = rows.sum;
  uint32_t open = fresh != 0 && (S::WT == 1 || (int64_t)from * BLKS + wt * MT * 2 < a.nb);   // it has had tiles, and the wave a block of the first
  // the other tokens' tiles: dealt to the workgroups from the last one down
  for (int t0 = (a.nsplit - 1 - split) * TOK; t0 < a.trail + a.n; t0 += a.nsplit * TOK, buf ^= 1) {
    uint4* const s_k = reinterpret_cast<uint4*>(s_main + buf * S::TILE);
    uint4* const s_v = s_k + 16 * TOK;
    uint32_t bits[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) bits[mt] = open_tokens(a, b, rows.node, t0 + ((wt * MT + mt) * 2 + half) * BLK);
    __syncthreads();   // norms and bad tokens of the last tile are done with
    if (tid < TOK) s_bad[tid] = 0;
    __syncthreads();
    load_exact<512, TOK>(a, head, t0, tid, s_k, s_v, s_norm, s_bad);
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int unit = wt * MT + mt, blk = unit * 2 + half;
      open |= bits[mt];
      open_exact(rows, bits[mt], s_norm + blk * BLK, s_bad + blk * BLK);
      attend32(
          rows, bits[mt], [&](int ks) { return key_of(s_k, unit, ks); }, [&](int oct, int ct) { return value_of(s_v, blk, oct, ct); });
    }
  }
  __syncthreads();
  if (w < 4 && l == 0) s_norm[w] = nu;
  __syncthreads();
  rows.vmax = fmaxf(rows.vmax, fmaxf(fmaxf(s_norm[0], s_norm[1]), fmaxf(s_norm[2], s_norm[3])));
  end_rows(rows, open);
  if constexpr (S::WT == 1) {
    if (tile0 + wr >= a.row_tiles) return;
    if (a.nsplit > 1)
      put_rows(rows, set_of(a, head, tile0 + wr, split));
    else
      finish_rows(rows, a, (int)head, tile0 + wr);
  } else {
    // the token waves' sets are joined through LDS
    float* const sets = reinterpret_cast<float*>(s_main);
    put_rows(rows, sets + w * T_FLOATS);
    __syncthreads();
    constexpr int PER = 512 / WR;   // threads a joined set: set i of row wave r is that of wave i * WR + r
    const int r = tid / PER;
    if (a.nsplit > 1) {
      if (tile0 + r < a.row_tiles) join_sets<S::WT, PER>(sets + r * T_FLOATS, WR * T_FLOATS, set_of(a, head, tile0 + r, split), tid % PER);
      return;
    }
    finish_sets<S::WT, T_ROWS, PER>(sets + r * T_FLOATS, WR * T_FLOATS, S::WT, a, (int)head, tile0 + r, 0, tid % PER);
  }
}

// ---- joining the partial sets ---------------------------------------------------------------------------------------------------------

// Up to N sets: eight rows a workgroup, four channels of one a thread, and a wave for the certificates.  Every thread requests N sets, so there
// are two of these and the one for any number (us a call in a graph: 8 heads, 8229 tokens, 26 nodes of 4 query heads, 8 sets: 24.1 with N = 8, 25.0 with 16; 2000
// tokens, 256 nodes of 2, 16 sets: 23.7 with 16, 27.7 by the one below; 8000 tokens, 4 nodes of 4, 31 sets: 16.7 with 32, 16.1 below).
constexpr int JOIN_ROWS = 8, JOIN_FEW_THREADS = JOIN_ROWS * 32 + 64;
template <int N>
__global__ __launch_bounds__(JOIN_FEW_THREADS) void tree_join_few_kernel(TreeArgs a) {
  const int head = blockIdx.x, tile = blockIdx.y >> 2, first = (blockIdx.y & 3) * JOIN_ROWS;
  finish_sets<N, JOIN_ROWS, JOIN_FEW_THREADS>(set_of(a, head, tile, 0), T_FLOATS, a.nsplit, a, head, tile, first, threadIdx.x);
}

// Many sets: eight rows a workgroup, and a PARTS-th of their channels.  First every set's quantities of the rows, a set a thread, which gives the sets'
// weights; then the accumulators, four channels of a row and every G-th set a thread, JOIN_AHEAD sets at a time, the first ones requested
// ahead of the weights.  Four parts where more sets than one has requests for at a time meet few workgroups (us a call in a graph, 4 query heads: 1 head, 131000
// tokens, 8 nodes, 256 sets 25.6, undivided 35.1; 2 heads, 64000 tokens, 32 nodes, 128 sets 30.3, 35.3; 4 heads, 64 sets 41.1, 42.7; 64 nodes, 128 workgroups
// undivided, 59.5, 58.0).
constexpr int JOIN_AHEAD = 8;
template <int PARTS>
__global__ __launch_bounds__(1024) void tree_join_kernel(TreeArgs a) {
  constexpr int R = JOIN_ROWS, C = 32 / PARTS, G = 4 * PARTS;
  extern __shared__ float s_f[];                     // [nsplit][R] weights
  __shared__ __align__(16) float4 s_o[G][C][R];
  __shared__ float s_m[16][R];
  __shared__ float s_q[16][7][R];
  const int tid = threadIdx.x, row = tid % R, w = tid >> 6;
  const int cc = tid / R % C, c = blockIdx.z * C + cc, g = tid / (C * R);   // channels 4 c .. 4 c + 3, sets g, g + G, ...
  const int head = blockIdx.x, tile = blockIdx.y / (T_ROWS / R), r32 = blockIdx.y % (T_ROWS / R) * R + row;
  const int r = tile * 32 + r32;
  const float* const sets = a.part + ((int64_t)head * a.row_tiles + tile) * a.nsplit * T_FLOATS;
  const auto channels = [&](int i) { return reinterpret_cast<const float4*>(sets + (int64_t)i * T_FLOATS)[c * T_ROWS + r32]; };
  float4 y[JOIN_AHEAD];
#pragma unroll
  for (int k = 0; k < JOIN_AHEAD; ++k) y[k] = channels(min(g + G * k, a.nsplit - 1));

  const auto lanes_max = [](float x) { return max_x32(max_x16(fmaxf(x, dpp_mov<0x128>(x)))); };   // over the lanes of a row: 8, 16, 32 apart
  const auto lanes_sum = [](float x) { return sum_x32(sum_x16(x + dpp_mov<0x128>(x))); };
  constexpr int TRIP = 1024 / R;   // sets of a trip of the workgroup
  const auto quantity = [&](int i, int t) { return sets[(int64_t)min(i, a.nsplit - 1) * T_FLOATS + T_OFLOATS + t * T_ROWS + r32]; };
  const int i0 = tid / R;
  float z[8], m = -INFINITY;
  if (w * (64 / R) < a.nsplit) {   // the first trip's quantities at once
#pragma unroll
    for (int t = 0; t < 8; ++t) z[t] = quantity(i0, t);
    m = z[T_M];
  }
  for (int i = i0 + TRIP; i < a.nsplit; i += TRIP) m = fmaxf(m, quantity(i, T_M));
  m = lanes_max(m);
  if ((tid & 63) < R) s_m[w][row] = m;
  __syncthreads();
  float M = s_m[0][row];
#pragma unroll
  for (int i = 1; i < 16; ++i) M = fmaxf(M, s_m[i][row]);
  float q[7] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};   // sums: L, sealed, EV; maxima: EVMAX, DMAX, VMAX, BAD
  const auto take = [&](int i, const float* y) {
    if (i >= a.nsplit) return;
    const float f = set_weight(y[T_M], M);
    s_f[i * R + row] = f;
    q[0] = fmaf(f, y[T_L], q[0]);
    q[1] = fmaf(f, y[T_SEALED], q[1]);
    q[2] = fmaf(f, y[T_EV], q[2]);
    q[3] = fmaxf(q[3], f * y[T_EVMAX]);
    q[4] = fmaxf(q[4], y[T_DMAX]);
    q[5] = fmaxf(q[5], y[T_VMAX]);
    q[6] = fmaxf(q[6], y[T_BAD]);
  };
  if (w * (64 / R) < a.nsplit) take(i0, z);
  for (int i = i0 + TRIP; i < a.nsplit; i += TRIP) {
#pragma unroll
    for (int t = 0; t < 8; ++t) z[t] = quantity(i, t);
    take(i, z);
  }
#pragma unroll
  for (int k = 0; k < 7; ++k) {
    q[k] = k < 3 ? lanes_sum(q[k]) : lanes_max(q[k]);
    if ((tid & 63) < R) s_q[w][k][row] = q[k];
  }
  __syncthreads();
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const auto add = [&](float f, const float4& v) { x.x = fmaf(f, v.x, x.x), x.y = fmaf(f, v.y, x.y), x.z = fmaf(f, v.z, x.z), x.w = fmaf(f, v.w, x.w); };
  for (int i = g;; i += G * JOIN_AHEAD) {
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k)
      if (i + G * k < a.nsplit) add(s_f[(i + G * k) * R + row], y[k]);
    if (i + G * JOIN_AHEAD >= a.nsplit) break;
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k) y[k] = channels(min(i + G * (JOIN_AHEAD + k), a.nsplit - 1));
  }
  s_o[g][cc][row] = x;
  __syncthreads();
  const bool certifies = tid >= 512 && tid < 512 + R && blockIdx.z == 0;
  if (r >= a.n * a.group || (tid >= C * R && !certifies)) return;
#pragma unroll
  for (int k = 0; k < 7; ++k) {
    q[k] = s_q[0][k][row];
#pragma unroll
    for (int i = 1; i < 16; ++i) q[k] = k < 3 ? q[k] + s_q[i][k][row] : fmaxf(q[k], s_q[i][k][row]);
  }
  if (certifies) {
    put_certificate(a, row_out(a, head, r), certificate(a, M, q[0], q[1], q[2], q[3], q[4], q[5]), q[6] != 0.0f);
  } else {
#pragma unroll
    for (int k = 1; k < G; ++k) add(1.0f, s_o[k][cc][row]);
    put_channels(a, row_out(a, head, r), c, x, mean_factor(q[0]));
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------------------

// Rows of a KV group a workgroup takes: 32, by the first kernel, where its waves have few turns each (it has them over sooner, and fewer sets to join),
// else up to 256 by the second, which reconstructs a tile once for all of them.  One of the trailing and drafted tokens takes as long as two sealed
// ones.  us a call in a graph by the first and the second kernel, turns a wave:
//   64 rows   8 heads, 2000 tokens 12.2, 15.8 (0.5)   8 heads, 32000 35.8, 36.6 (8)   8 heads, 64000 54.6, 51.4 (16)
//   128 rows  8 heads, 2000 14.1, 17.0 (1)   2 heads, 32000 22.8, 25.6 (4)   8 heads, 8000 22.1, 22.2 (4)   4 heads, 32000 31.8, 28.7 (8)
//   256 rows  8 heads, 4000 22.2, 24.7 (4)   1 head, 32000 23.0, 31.7 (4)   8 heads, 8000 32.6, 29.6 (8)
//   512 rows  4 heads, 4000 23.3, 27.0 (4.2)   8 heads, 2000 23.3, 22.9 (4.4)
static int tree_rows(int n_cu, int64_t heads, int n_rows, int64_t sealed, int64_t others) {
  const int64_t work = (sealed + 2 * others) * heads * ((n_rows + 31) / 32), turn = (int64_t)32 * FEW_WAVES * n_cu;
  if (n_rows <= 32 || 2 * work <= (n_rows <= 64 ? 16 : 9) * turn) return 32;
  return n_rows <= 64 ? 64 : (n_rows <= 128 ? 128 : 256);
}

// Tokens of a tile, or of a turn of the first kernel's waves.
static int tile_tokens(int rows) { return rows == 32 ? 32 * FEW_WAVES : (rows == 64 ? 128 : 64); }

// Partial sets: as many workgroups as the device holds at a time, each with a tile of sealed blocks or of the other tokens.  Of 32 rows a workgroup
// the first tile and the other tokens are one workgroup's, which needs no second launch (us a call in a graph, 8 heads of 4 query heads: 12 nodes, 60 tokens 9.9, by
// two workgroups 10.9; 4 nodes, 200 tokens 10.7, 10.6; two tiles, 4 nodes, 400 tokens, by one 13.4, by three 10.8).
static int tree_splits(int n_cu, int64_t heads, int n_rows, int rows, int64_t sealed, int64_t others) {
  const int tok = tile_tokens(rows), exact = rows == 32 ? FEW_EXACT : tok;   // (64 others at most are a turn as well)
  const int64_t z = (n_rows + rows - 1) / rows, most = std::max<int64_t>(1, (int64_t)n_cu / (heads * z));
  const int64_t tiles = (sealed + tok - 1) / tok, turns = tiles + (others + exact - 1) / exact;
  return (int)std::min(most, rows == 32 && tiles <= 1 && others <= exact ? 1 : turns);
}

// Sealed tiles of the second kernel by workgroup: the trailing and drafted tokens' tiles are the last workgroups', EXACT tiles' work each, and
// the sealed ones are dealt so that all end together.
constexpr int EXACT = 3;
static void tree_shares(TreeArgs& a, int rows) {
  const int tok = tile_tokens(rows);
  const int tiles = (int)(((a.nb + 3) / 4 * 64 + tok - 1) / tok), exact = (a.trail + a.n + tok - 1) / tok;
  a.last = exact < a.nsplit ? exact : 0;
  a.least = std::max(0, (tiles + EXACT * exact) / a.nsplit - EXACT);
  const int rest = tiles - a.last * a.least, even = a.nsplit - a.last;
  a.share = rest / even;
  a.over = rest % even;
}

int64_t tree_ws_bytes(const Cache* c, int n_draft) {
  const int64_t heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  const int n_rows = n_draft * (c->desc.n_q_heads / c->desc.n_kv_heads);
  const auto most = [&](int rows) { return tree_splits(c->n_cu, heads, n_rows, rows, c->desc.max_tokens, n_draft + BLK - 1); };
  const int64_t sets = std::max(most(32), most(n_rows <= 64 ? 64 : (n_rows <= 128 ? 128 : 256)));
  return heads * ((n_rows + 31) / 32) * sets * T_FLOATS * 4;
}

template <int WR>
static void launch_many(const TreeArgs& a, int64_t heads, hipStream_t st) {
  tree_many_kernel<WR><<<dim3((uint32_t)heads, (uint32_t)a.nsplit, (uint32_t)((a.row_tiles + WR - 1) / WR)), 512, 0, st>>>(a);
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
  if (rows > 32) tree_shares(a, rows);
  a.O = O;
  a.cert = cert;
  a.flags = flags;
  a.tol = tol;
  switch (rows) {
    case 32: {
      const dim3 grid((uint32_t)heads, (uint32_t)a.nsplit, (uint32_t)a.row_tiles);
      if (a.trail + a.n <= 64)
        tree_few_kernel<64><<<grid, 64 * FEW_WAVES, 0, st>>>(a);
      else
        tree_few_kernel<FEW_EXACT><<<grid, 64 * FEW_WAVES, 0, st>>>(a);
      break;
    }
    case 64: launch_many<2>(a, heads, st); break;
    case 128: launch_many<4>(a, heads, st); break;
    default: launch_many<8>(a, heads, st); break;
  }
  CQA_HIP(hipGetLastError());
  if (a.nsplit == 1) return CQA_OK;
  const dim3 grid((uint32_t)heads, (uint32_t)a.row_tiles * (T_ROWS / JOIN_ROWS));
  if (a.nsplit <= 8)
    tree_join_few_kernel<8><<<grid, JOIN_FEW_THREADS, 0, st>>>(a);
  else if (a.nsplit <= 16)
    tree_join_few_kernel<16><<<grid, JOIN_FEW_THREADS, 0, st>>>(a);
  else if (a.nsplit > 4 * JOIN_AHEAD && heads * a.row_tiles * (T_ROWS / JOIN_ROWS) * 4 <= c->n_cu)
    tree_join_kernel<4><<<dim3(grid.x, grid.y, 4), 1024, (size_t)a.nsplit * JOIN_ROWS * 4, st>>>(a);
  else
    tree_join_kernel<1><<<grid, 1024, (size_t)a.nsplit * JOIN_ROWS * 4, st>>>(a);
  CQA_HIP(hipGetLastError());
  return CQA_OK;
}

}  // namespace cqa
