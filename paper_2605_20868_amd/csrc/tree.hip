// Attention of drafted tokens (a tree, or a chunk of a prompt) over the quantized cache, with the certificate of every
// (node, query head): split pass on the matrix cores and the joining of its partial sets.
//
// The rows of a KV group are its n_draft nodes times its G query heads, and all of them attend the same sealed blocks, so one
// workgroup reconstructs a tile of keys and values once, in FP16, into LDS, and its waves multiply it with up to 256 rows.
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
// Softmax in FP32 (running maximum per row, FP32 sums); the weights enter the second product as FP16, 2^-12 of a weight at most.
//
// A further workgroup per group of rows attends the trailing FP16 tokens and the drafted ones, which are exact, under the mask.
#include <algorithm>

#include "cqa_internal.h"

namespace cqa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float SCORE = 0.08838834764831845f * 1.4426950408889634f;   // 1 / sqrt(d), in the exponent's base 2
constexpr float F16_MAX = 65504.0f;
constexpr float LN2 = 0.6931471805599453f;

// ---- partial set of a split and 32 rows: the accumulators by (four channels, row), then one float per row for each quantity
enum { T_M = 0, T_L, T_EV, T_EVMAX, T_DMAX, T_VMAX, T_STATS };
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
  float* part;             // [Bt * Hkv][row tiles][nsplit + 1][T_FLOATS]
  int64_t nq_cap;
  int64_t nb;              // sealed blocks
  int n, words, trail;     // drafted nodes, mask words of one, trailing tokens
  int n_kv, group;
  int row_tiles;           // of 32 rows
  int nsplit;              // partial sets of the sealed blocks; one more of the other tokens
};

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}
// code scale + offset of two tokens, rounded once.  The scale's rounding to FP16 can take the largest code beyond the group's maximum, and
// beyond FP16's range where that is at its end (keys cannot: z and sigma are FP32, the largest code is the maximum within 2^-23).
__device__ __forceinline__ uint32_t value2(uint32_t code, uint32_t scale, uint32_t off) {
  const f16x2 x = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, code), __builtin_bit_cast(f16x2, scale), __builtin_bit_cast(f16x2, off));
  const f16x2 most = {(_Float16)F16_MAX, (_Float16)F16_MAX};
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_minimum(x, most));
}
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// the width of a key channel in the bound, rounded up to FP16
__device__ __forceinline__ uint16_t key_width(float sigma, float z) {
  const float most = fmaxf(fabsf(fmaf(-128.0f, sigma, z)), fabsf(fmaf(127.0f, sigma, z)));
  const float w = fmaf(2.0f, fminf(0.5f * sigma, fmaf(most, 0x1p-11f, 0x1p-25f)), sigma);
  const _Float16 h = (_Float16)w;
  uint16_t u = __builtin_bit_cast(uint16_t, h);
  if ((float)h < w) ++u;
  return u;
}

// NT tiles of 32 rows per wave, WR waves side by side over rows, WT over tokens; four waves.
template <int NT, int WR, int WT>
struct TreeShape {
  static constexpr int MT = WT == 1 ? 2 : 1;                 // tiles of 32 tokens a wave takes of a tile
  static constexpr int TOK = 32 * MT * WT;                   // tokens of a tile
  static constexpr int QUADS = TOK / 64;
  static constexpr int BLKS = TOK / BLK;
  static constexpr int ROWS = 32 * NT * WR;
  static constexpr int KV_BYTES = 2 * TOK * D * 2;
  static constexpr int OUT_BYTES = WT > 1 ? 4 * T_FLOATS * 4 : 0;   // the waves' sets, joined through LDS
  static constexpr int MAIN_BYTES = KV_BYTES > OUT_BYTES ? KV_BYTES : OUT_BYTES;
};

template <int NT, int WR, int WT>
__global__ __launch_bounds__(256, NT * WR > 2 ? 1 : 2) void tree_split_kernel(TreeArgs a) {
  using S = TreeShape<NT, WR, WT>;
  constexpr int MT = S::MT, TOK = S::TOK, BLKS = S::BLKS;
  __shared__ __align__(16) uint8_t s_main[S::MAIN_BYTES];   // keys [16 runs of 8 channels][TOK] x 16 B, values [TOK / 8][128] x 16 B
  __shared__ __align__(16) uint16_t s_width[D / 8][32][8];  // key widths of the last 32 blocks
  __shared__ float s_eta[BLKS];
  __shared__ float s_norm[TOK];
  __shared__ uint32_t s_bad[BLKS];
  uint4* const s_k = reinterpret_cast<uint4*>(s_main);
  uint4* const s_v = s_k + 16 * TOK;

  const int tid = threadIdx.x, l = tid & 63, n32 = l & 31, half = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = w % WR, wt = w / WR;
  const int head = blockIdx.x;   // (batch, KV head)
  const int split = blockIdx.y;
  const int b = head / a.n_kv, kvh = head - b * a.n_kv;
  const int n_rows = a.n * a.group;
  const int tile0 = blockIdx.z * (NT * WR) + wr * NT;   // first row tile of the wave

  f16x8 qf[NT][8];
  int node[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = min((tile0 + nt) * 32 + n32, n_rows - 1);
    node[nt] = r / a.group;
    const __half* row = a.q + (((int64_t)b * a.n + node[nt]) * a.n_kv * a.group + kvh * a.group + (r - node[nt] * a.group)) * D;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qf[nt][ks] = __builtin_bit_cast(f16x8, ld16_any(row + ks * 16 + half * 8));
  }
  f32x16 o[NT][4];
  float m[NT], sum[NT], ev[NT], evmax[NT], dmax[NT], vmax[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    sum[nt] = ev[nt] = evmax[nt] = dmax[nt] = vmax[nt] = 0.0f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[nt][ct][r] = 0.0f;
  }
  float nu = 0.0f;

  // Scores, softmax and values of the tile in LDS.  bits, where masked: the tokens of the lane's block that its row attends.
  const auto attend = [&](bool masked, const uint32_t (&bits)[NT][MT]) {
    f32x16 s[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[mt][nt][r] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const f16x8 k = __builtin_bit_cast(f16x8, s_k[(2 * ks + half) * TOK + (wt * MT + mt) * 32 + n32]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[mt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, qf[nt][ks], s[mt][nt], 0, 0, 0);
      }
    }
    uint32_t p[MT][NT][8];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float top = -INFINITY;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (masked) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[mt][nt][r] = bits[nt][mt] >> r & 1u ? s[mt][nt][r] : -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[mt][nt][r]);
      }
      top = fmaxf(top, other_half(top)) * SCORE;
      if (__any(top > m[nt])) {
        const float mn = fmaxf(m[nt], top);
        const float f = mn == m[nt] ? 1.0f : __builtin_amdgcn_exp2f(m[nt] - mn);
        m[nt] = mn;
        sum[nt] *= f;
        ev[nt] *= f;
        evmax[nt] *= f;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[nt][ct][r] *= f;
      }
      const float base = m[nt] == -INFINITY ? 0.0f : m[nt];   // nothing attended yet: every weight is exp2(-inf) = 0
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float bs = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[mt][nt][r], SCORE, -base));
          const float y = __builtin_amdgcn_exp2f(fmaf(s[mt][nt][r + 1], SCORE, -base));
          bs += x + y;
          p[mt][nt][r / 2] = pack_f16(x, y);
        }
        const float e = bs * s_eta[(wt * MT + mt) * 2 + half];
        sum[nt] += bs;
        ev[nt] += e;
        evmax[nt] = fmaxf(evmax[nt], e);
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int oct = 0; oct < 2; ++oct)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
          const f16x8 v = __builtin_bit_cast(f16x8, s_v[(((wt * MT + mt) * 2 + half) * 2 + oct) * D + ct * 32 + n32]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const uint32_t* x = &p[mt][nt][4 * oct];
            o[nt][ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, __builtin_bit_cast(f16x8, make_uint4(x[0], x[1], x[2], x[3])), o[nt][ct], 0, 0, 0);
          }
        }
  };
  // Delta of the 32 blocks whose widths are in LDS
  const auto bound_scores = [&] {
    if (wt != 0) return;
    f32x16 d[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 16; ++r) d[nt][r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const f16x8 x = *reinterpret_cast<const f16x8*>(s_width[2 * ks + half][n32]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint4 y = __builtin_bit_cast(uint4, qf[nt][ks]);
        y.x &= 0x7fff7fffu, y.y &= 0x7fff7fffu, y.z &= 0x7fff7fffu, y.w &= 0x7fff7fffu;
        d[nt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(f16x8, y), d[nt], 0, 0, 0);
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 16; ++r) dmax[nt] = fmaxf(dmax[nt], d[nt][r]);
  };
  // token t of block `blk` of the tile has this place among the keys: the A operand's rows, see attend
  const auto place = [](int blk, int t) { return (blk >> 1) * 32 + (t >> 2) * 8 + (blk & 1) * 4 + (t & 3); };

  const bool sealed = split < a.nsplit;
  const int64_t nquads = (a.nb + 3) >> 2;
  const int total = a.trail + a.n;   // of the other tokens: trailing ones, then drafted ones
  // sealed tokens: tiles split, split + nsplit, ..., so that the workgroups of a head move through it side by side
  const int64_t tiles = sealed ? (nquads + S::QUADS - 1) / S::QUADS : (total + TOK - 1) / TOK;
  const int64_t step = sealed ? a.nsplit : 1;
  int fresh = 0;   // blocks whose widths have come since bound_scores
  if (sealed)
    for (int i = tid; i < (int)sizeof(s_width) / 4; i += 256) reinterpret_cast<uint32_t*>(s_width)[i] = 0u;

  for (int64_t tile = sealed ? split : 0; tile < tiles; tile += step) {
    uint32_t bits[NT][MT];
    bool masked;
    __syncthreads();   // the last tile is done with
    if (sealed) {
      const uint8_t* const base = a.t1 + (int64_t)head * a.nq_cap * QUAD_BYTES;
#pragma unroll
      for (int qd = 0; qd < S::QUADS; ++qd) {
        int64_t quad = tile * S::QUADS + qd;
        if (quad >= nquads) quad = 0;   // behind the last: any record of the head, its scores are masked
        const uint8_t* const rec = base + quad * QUAD_BYTES;
        const int blk = qd * 4 + (tid >> 6);   // a wave: one block
        {
          // keys: lane (run pair c8, token t8) has 16 channels of tokens t8 and t8 + 8
          const int t8 = tid & 7, c8 = (tid >> 3) & 7;
          const uint8_t* const kc = rec + Q_KC + (tid >> 6) * KC_BYTES + (c8 >> 2) * 1024 + (c8 & 3) * 256;
          const float* const km = reinterpret_cast<const float*>(rec + Q_KM + (tid >> 6) * KM_BYTES) + c8 * 16;
          float sg[16], z[16];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            *reinterpret_cast<float4*>(&sg[4 * e]) = reinterpret_cast<const float4*>(km)[e];
            *reinterpret_cast<float4*>(&z[4 * e]) = reinterpret_cast<const float4*>(km + D)[e];
          }
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            const uint4 c4 = *reinterpret_cast<const uint4*>(kc + (t8 + 8 * tt) * 16);
            const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t x = c[e >> 1] >> (16 * (e & 1));
              h[e] = pack_f16(fmaf((float)(x & 255u) - 128.0f, sg[2 * e], z[2 * e]),
                              fmaf((float)(x >> 8 & 255u) - 128.0f, sg[2 * e + 1], z[2 * e + 1]));
            }
            const int at = place(blk, t8 + 8 * tt);
            s_k[(2 * c8) * TOK + at] = make_uint4(h[0], h[1], h[2], h[3]);
            s_k[(2 * c8 + 1) * TOK + at] = make_uint4(h[4], h[5], h[6], h[7]);
          }
          // widths: two channels a lane
          const int ch = c8 * 16 + 2 * t8;
          const float2 s2 = *reinterpret_cast<const float2*>(km + 2 * t8), z2 = *reinterpret_cast<const float2*>(km + D + 2 * t8);
          const uint32_t w2 = key_width(s2.x, z2.x) | (uint32_t)key_width(s2.y, z2.y) << 16;
          *reinterpret_cast<uint32_t*>(&s_width[ch >> 3][fresh + blk][ch & 7]) = w2;
        }
        {
          // values: lane (octet oc, group set gh, channel n) has four channels of eight tokens, one dword each
          const int n16 = tid & 15, gh = (tid >> 4) & 1, oc = (tid >> 5) & 1;
          const uint4 c4 = reinterpret_cast<const uint4*>(rec + Q_VC)[tid];
          const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
          const uint8_t* const vm = rec + Q_VM + (tid >> 6) * VM_BYTES + oc * 128 + gh * 64;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint4 sc = reinterpret_cast<const uint4*>(vm)[g], of = reinterpret_cast<const uint4*>(vm + 256)[g];
            const uint32_t d = c[g];
            // codes of tokens (2 i, 2 i + 1) as FP16 integers: dropped into the mantissa of 1024, which leaves exactly
            const auto codes = [&](int i) {
              const uint32_t x = d >> (8 * i);
              const uint32_t pair = (x & 0xfu) | (x << 12 & 0xf0000u) | 0x64006400u;
              return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, pair) - __builtin_bit_cast(f16x2, 0x64006400u));
            };
            s_v[((tid >> 6) + qd * 4) * 2 * D + oc * D + (gh * 4 + g) * 16 + n16] =
                make_uint4(value2(codes(0), sc.x, of.x), value2(codes(1), sc.y, of.y), value2(codes(2), sc.z, of.z), value2(codes(3), sc.w, of.w));
          }
        }
        if (tid < 4) {
          const float2 an = reinterpret_cast<const float2*>(rec + Q_AN)[tid];   // eta, nu; zeros where not sealed
          s_eta[qd * 4 + tid] = an.x + fminf(an.x, fmaf(an.y + an.x, 0x1p-11f, 0x1p-21f));
          nu = fmaxf(nu, an.y);
        }
      }
      fresh += BLKS;
      const int64_t left = a.nb - tile * BLKS;   // sealed blocks from the tile's first on
      masked = left < BLKS;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) bits[nt][mt] = (wt * MT + mt) * 2 + half < left ? 0xffffu : 0u;
      __syncthreads();
    } else {
      const int t0 = (int)tile * TOK;
      masked = true;
      if (tid < BLKS) {
        s_eta[tid] = 0.0f;   // exact tokens
        s_bad[tid] = 0u;
      }
      __syncthreads();
      // a wave takes a token at a time: 2 channels a lane; rows behind the last token are zeros
      for (int t = w; t < TOK; t += 4) {
        const int i = t0 + t;
        uint32_t k2 = 0u, v2 = 0u;
        if (i < total) {
          const bool old = i < a.trail;
          k2 = ld4_any((old ? a.trail_k + ((int64_t)head * BLK + i) * D : a.kd + ((int64_t)head * a.n + i - a.trail) * D) + 2 * l);
          v2 = ld4_any((old ? a.trail_v + ((int64_t)head * BLK + i) * D : a.vd + ((int64_t)head * a.n + i - a.trail) * D) + 2 * l);
        }
        const f16x2 k = __builtin_bit_cast(f16x2, k2), v = __builtin_bit_cast(f16x2, v2);
        const float x = (float)v[0], y = (float)v[1];
        // A number that is not finite must not meet the zero weight of a row that does not attend its token: the token is
        // taken out, and the rows that do attend it get a sum that is no number.
        const bool bad = __any(!(fabsf(x) <= F16_MAX && fabsf(y) <= F16_MAX && fabsf((float)k[0]) <= F16_MAX && fabsf((float)k[1]) <= F16_MAX));
        float sq = fmaf(x, x, y * y);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sq += __shfl_xor(sq, d);
        if (l == 0) {
          s_norm[t] = sqrtf(sq);
          if (bad) atomicOr(&s_bad[t / BLK], 1u << (t % BLK));
        }
        if (bad) k2 = v2 = 0u;
        reinterpret_cast<uint32_t*>(s_k)[((l >> 2) * TOK + place(t / BLK, t % BLK)) * 4 + (l & 3)] = k2;
        uint16_t* const vh = reinterpret_cast<uint16_t*>(s_v);
        vh[((t >> 3) * D + 2 * l) * 8 + (t & 7)] = (uint16_t)v2;
        vh[((t >> 3) * D + 2 * l + 1) * 8 + (t & 7)] = (uint16_t)(v2 >> 16);
      }
      __syncthreads();
      // a row's open tokens among the 16 of the lane's block
      const auto open = [&](int nt, int mt) -> uint32_t {
        const int j = t0 + ((wt * MT + mt) * 2 + half) * BLK - a.trail;   // drafted node of the block's first token; below 0: trailing ones
        uint32_t x = 0u;
        if (a.mask == nullptr) {
          const int seen = node[nt] - j + 1;   // tokens up to the node itself
          return seen >= BLK ? 0xffffu : (seen > 0 ? (1u << seen) - 1u : 0u);
        }
        const int lo = max(j, 0);
        if (j + BLK > 0 && lo < a.n) {
          const uint64_t* const mw = a.mask + ((int64_t)b * a.n + node[nt]) * a.words;
          uint64_t y = mw[lo >> 6] >> (lo & 63);
          if ((lo & 63) + BLK > 64 && (lo >> 6) + 1 < a.words) y |= mw[(lo >> 6) + 1] << (64 - (lo & 63));
          x = ((uint32_t)y & ((1u << min(a.n - lo, BLK)) - 1u)) << (lo - j);
        }
        if (j < 0) x |= (1u << min(-j, BLK)) - 1u;
        return x & 0xffffu;
      };
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int blk = (wt * MT + mt) * 2 + half;
          bits[nt][mt] = open(nt, mt);
          for (int r = 0; r < BLK; ++r)
            if (bits[nt][mt] >> r & 1u) vmax[nt] = fmaxf(vmax[nt], s_norm[blk * BLK + r]);
          if (bits[nt][mt] & s_bad[blk]) sum[nt] = NAN;   // stays
        }
    }
    attend(masked, bits);
    if (sealed && (fresh == 32 || tile + step >= tiles)) {
      bound_scores();
      fresh = 0;
    }
  }
  if (sealed) {
    if (tid < 4) s_norm[tid] = nu;
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) vmax[nt] = fmaxf(fmaxf(s_norm[0], s_norm[1]), fmaxf(s_norm[2], s_norm[3]));
  }

  // the halves of a row have the tokens of different blocks
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    sum[nt] += other_half(sum[nt]);
    ev[nt] += other_half(ev[nt]);
    evmax[nt] = fmaxf(evmax[nt], other_half(evmax[nt]));
    dmax[nt] = fmaxf(dmax[nt], other_half(dmax[nt])) * (0.5f * 0.08838834764831845f);
    vmax[nt] = fmaxf(vmax[nt], other_half(vmax[nt]));
  }
  const auto put = [&](float* to, int nt) {
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)   // channels ct * 32 + r4 * 8 + half * 4 + 0 .. 3
        reinterpret_cast<float4*>(to)[(ct * 8 + r4 * 2 + half) * T_ROWS + n32] =
            make_float4(o[nt][ct][4 * r4], o[nt][ct][4 * r4 + 1], o[nt][ct][4 * r4 + 2], o[nt][ct][4 * r4 + 3]);
    if (half == 0) {
      float* const st = to + T_OFLOATS + n32;
      st[T_M * T_ROWS] = m[nt];
      st[T_L * T_ROWS] = sum[nt];
      st[T_EV * T_ROWS] = ev[nt];
      st[T_EVMAX * T_ROWS] = evmax[nt];
      st[T_DMAX * T_ROWS] = dmax[nt];
      st[T_VMAX * T_ROWS] = vmax[nt];
    }
  };
  const auto set_of = [&](int tile) { return a.part + (((int64_t)head * a.row_tiles + tile) * (a.nsplit + 1) + split) * T_FLOATS; };
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if constexpr (WT == 1) {
      if (tile0 + nt < a.row_tiles) put(set_of(tile0 + nt), nt);
    } else {
      // the token waves' sets are joined through LDS
      float* const sets = reinterpret_cast<float*>(s_main);
      __syncthreads();
      put(sets + w * T_FLOATS, nt);
      __syncthreads();
      constexpr int PER = 256 / WR;   // threads a joined set
      const int mine = tid / PER, lane = tid % PER;
      const int tile = blockIdx.z * (NT * WR) + mine * NT + nt;
      if (tile < a.row_tiles) {
        float* const to = set_of(tile);
        const int row = lane & 31;
        float f[WT], M = -INFINITY;
#pragma unroll
        for (int i = 0; i < WT; ++i) {
          f[i] = sets[(i * WR + mine) * T_FLOATS + T_OFLOATS + T_M * T_ROWS + row];
          M = fmaxf(M, f[i]);
        }
#pragma unroll
        for (int i = 0; i < WT; ++i) f[i] = f[i] == M ? 1.0f : __builtin_amdgcn_exp2f(f[i] - M);
        for (int c = lane >> 5; c < 32; c += PER / 32) {
          float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int i = 0; i < WT; ++i) {
            const float4 y = reinterpret_cast<const float4*>(sets + (i * WR + mine) * T_FLOATS)[c * T_ROWS + row];
            x.x = fmaf(f[i], y.x, x.x), x.y = fmaf(f[i], y.y, x.y), x.z = fmaf(f[i], y.z, x.z), x.w = fmaf(f[i], y.w, x.w);
          }
          reinterpret_cast<float4*>(to)[c * T_ROWS + row] = x;
        }
        if (lane < 32) {
          float L = 0.0f, E = 0.0f, EM = 0.0f, DM = 0.0f, VM = 0.0f;
#pragma unroll
          for (int i = 0; i < WT; ++i) {
            const float* const st = sets + (i * WR + mine) * T_FLOATS + T_OFLOATS + row;
            L = fmaf(f[i], st[T_L * T_ROWS], L);
            E = fmaf(f[i], st[T_EV * T_ROWS], E);
            EM = fmaxf(EM, f[i] * st[T_EVMAX * T_ROWS]);
            DM = fmaxf(DM, st[T_DMAX * T_ROWS]);
            VM = fmaxf(VM, st[T_VMAX * T_ROWS]);
          }
          float* const st = to + T_OFLOATS + row;
          st[T_M * T_ROWS] = M;
          st[T_L * T_ROWS] = L;
          st[T_EV * T_ROWS] = E;
          st[T_EVMAX * T_ROWS] = EM;
          st[T_DMAX * T_ROWS] = DM;
          st[T_VMAX * T_ROWS] = VM;
        }
      }
    }
  }
}

// ---- joining: a workgroup has 8 rows, a thread four channels of one ----------------------------------------------------------------

struct TreeJoinArgs {
  const float* part;
  __half* O;               // [Bt][n][Hq][128]
  cqa_node_cert* cert;     // [Bt][n][Hq]
  uint32_t* flags;
  cqa_tolerances tol;
  int n, n_kv, group, row_tiles, nsplit;
};

__global__ __launch_bounds__(256) void tree_join_kernel(TreeJoinArgs a) {
  const int row = threadIdx.x & 7, c = threadIdx.x >> 3;
  const int head = blockIdx.x, tile = blockIdx.y >> 2, r32 = (blockIdx.y & 3) * 8 + row;
  const int r = tile * 32 + r32;
  const float* const sets = a.part + ((int64_t)head * a.row_tiles + tile) * (a.nsplit + 1) * T_FLOATS;
  __shared__ uint32_t s_bad[8];
  if (threadIdx.x < 8) s_bad[threadIdx.x] = 0u;
  __syncthreads();
  float M = -INFINITY;
  for (int i = 0; i <= a.nsplit; ++i) M = fmaxf(M, sets[i * T_FLOATS + T_OFLOATS + T_M * T_ROWS + r32]);
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float L = 0.0f, sealed = 0.0f, E = 0.0f, EM = 0.0f, DM = 0.0f, VM = 0.0f;
  for (int i = 0; i <= a.nsplit; ++i) {
    const float* const st = sets + i * T_FLOATS + T_OFLOATS + r32;
    const float mi = st[T_M * T_ROWS];
    const float f = mi == M ? 1.0f : __builtin_amdgcn_exp2f(mi - M);
    const float4 y = reinterpret_cast<const float4*>(sets + i * T_FLOATS)[c * T_ROWS + r32];
    x.x = fmaf(f, y.x, x.x), x.y = fmaf(f, y.y, x.y), x.z = fmaf(f, y.z, x.z), x.w = fmaf(f, y.w, x.w);
    L = fmaf(f, st[T_L * T_ROWS], L);
    if (i < a.nsplit) sealed = L;
    E = fmaf(f, st[T_EV * T_ROWS], E);
    EM = fmaxf(EM, f * st[T_EVMAX * T_ROWS]);
    DM = fmaxf(DM, st[T_DMAX * T_ROWS]);
    VM = fmaxf(VM, st[T_VMAX * T_ROWS]);
  }
  const bool empty = L == 0.0f;   // the row attends nothing
  const float inv = empty ? 0.0f : 1.0f / L;
  // (a mean of values: where the rounding of the weights takes it beyond FP16's range, the values' largest, it stays there)
  const auto mean = [&](float y) { return y *= inv, isfinite(y) ? __builtin_amdgcn_fmed3f(y, -F16_MAX, F16_MAX) : y; };
  const f32x2 lo = {mean(x.x), mean(x.y)}, hi = {mean(x.z), mean(x.w)};
  const bool mine = r < a.n * a.group;
  const int b = head / a.n_kv, kvh = head - b * a.n_kv, node = r / a.group;
  const int64_t out = ((int64_t)b * a.n + node) * a.n_kv * a.group + kvh * a.group + (r - node * a.group);
  if (mine) {
    reinterpret_cast<uint2*>(a.O + out * D)[c] =
        make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, f16x2)), __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, f16x2)));
    if (!(isfinite(lo[0]) && isfinite(lo[1]) && isfinite(hi[0]) && isfinite(hi[1]))) atomicOr(&s_bad[row], 1u);
  }
  __syncthreads();
  if (!mine || c != 0) return;
  cqa_node_cert ct;
  ct.E_val = E * inv;
  ct.delta_h = DM;
  ct.v_max = VM;
  ct.alpha_tail_hat = sealed * inv;
  ct.lse = empty ? -INFINITY : M * LN2 + logf(L);
  ct.max_block_contrib = EM * inv;
  ct.reserved = 0.0f;
  float tail = 0.0f;
  if (ct.alpha_tail_hat > 0.0f && DM != 0.0f)
    tail = fminf(1.0f, expf((float)a.tol.mass_exp * DM) * ct.alpha_tail_hat) * expm1f(2.0f * DM);
  const float full = tanhf(DM);
  ct.E_key = 2.0f * VM * (a.tol.key_bound_mode == 0 ? fminf(full, tail) : (a.tol.key_bound_mode == 1 ? tail : full));
  uint32_t fl = a.tol.force_flags;
  if (ct.E_key > a.tol.eps_key) fl |= CQA_FLAG_KEY;
  if (ct.E_val > a.tol.eps_val || ct.max_block_contrib > a.tol.v_tol) fl |= CQA_FLAG_VAL;
  if (ct.E_key + ct.E_val > a.tol.eps_total) fl |= CQA_FLAG_TOTAL;
  if (s_bad[row] != 0u || !isfinite(ct.E_key) || !isfinite(ct.E_val) || !isfinite(DM) || !isfinite(VM) || (!empty && !isfinite(ct.lse)))
    fl |= CQA_FLAG_PRECOND;
  a.cert[out] = ct;
  a.flags[out] = fl;
}

// ---- host --------------------------------------------------------------------------------------------------------------------------

// Rows of a KV group a workgroup takes: few rows spare the accumulators, and the waves share the tokens instead.
static int tree_rows(int n_rows) { return n_rows <= 32 ? 32 : (n_rows <= 64 ? 64 : (n_rows <= 128 ? 128 : 256)); }

// Partial sets of the sealed blocks: as many workgroups as the device holds at a time.
static int tree_splits(int n_cu, int64_t heads, int n_rows, int64_t nb) {
  const int rows = tree_rows(n_rows);
  const int64_t z = (n_rows + rows - 1) / rows;
  const int64_t most = std::max<int64_t>(1, (rows <= 64 ? 2 : 1) * (int64_t)n_cu / (heads * z));
  const int64_t quads = (nb + 3) / 4;
  const int64_t tiles = rows == 32 ? (quads + 1) / 2 : quads;
  return (int)std::min(most, tiles);
}

int64_t tree_ws_bytes(const Cache* c, int n_draft) {
  const int64_t heads = (int64_t)c->desc.batch * c->desc.n_kv_heads;
  const int n_rows = n_draft * (c->desc.n_q_heads / c->desc.n_kv_heads);
  return heads * ((n_rows + 31) / 32) * (tree_splits(c->n_cu, heads, n_rows, c->nb_cap) + 1) * T_FLOATS * 4;
}

template <int NT, int WR, int WT>
static void launch_tree_shape(const TreeArgs& a, int64_t heads, hipStream_t st) {
  const uint32_t z = (uint32_t)((a.row_tiles + NT * WR - 1) / (NT * WR));
  tree_split_kernel<NT, WR, WT><<<dim3((uint32_t)heads, (uint32_t)a.nsplit + 1, z), 256, 0, st>>>(a);
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
  a.nsplit = tree_splits(c->n_cu, heads, n_rows, a.nb);
  switch (tree_rows(n_rows)) {
    case 32: launch_tree_shape<1, 1, 4>(a, heads, st); break;
    case 64: launch_tree_shape<1, 2, 2>(a, heads, st); break;
    case 128: launch_tree_shape<2, 2, 2>(a, heads, st); break;
    default: launch_tree_shape<2, 4, 1>(a, heads, st); break;
  }
  CQA_HIP(hipGetLastError());
  TreeJoinArgs j;
  j.part = ws;
  j.O = O;
  j.cert = cert;
  j.flags = flags;
  j.tol = tol;
  j.n = n_draft;
  j.n_kv = a.n_kv;
  j.group = a.group;
  j.row_tiles = a.row_tiles;
  j.nsplit = a.nsplit;
  tree_join_kernel<<<dim3((uint32_t)heads, (uint32_t)a.row_tiles * 4), 256, 0, st>>>(j);
  CQA_HIP(hipGetLastError());
  return CQA_OK;
}

}  // namespace cqa
