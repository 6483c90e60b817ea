// Reading the cache back: the reconstruction of tokens of every sequence, k = code sigma + z (one fused multiply-add in FP32) and
// v = code scale + offset, rounded once to the asked type; trailing tokens are their FP16 originals.
//
// What bounds it: bytes, 288 read and 512 (FP16) written per token and KV head.  One wave a block of 16 tokens: lane (cp, tq) has
// channels 8 cp .. 8 cp + 7 of tokens tq, tq + 4, tq + 8, tq + 12, so that sigma and z are fetched once for four tokens, a dword of value
// codes (one channel of eight tokens) serves two of the lane's, and a wave's store is four whole rows.
#include "cqa_internal.h"

namespace cqa {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8r __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x8r __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x8r __attribute__((ext_vector_type(8), aligned(4)));

struct ReadArgs {
  const uint8_t* t1;        // layer base of the quad records
  const __half* trail_k;    // layer base [Bt * Hkv][16][128]
  const __half* trail_v;
  int64_t nq_cap;
  int64_t nb;               // sealed blocks
  int64_t first, end;       // tokens
  int64_t blk0;             // first / 16
  void* k;
  void* v;                  // either may be null
  cqa_strides st;
  int n_kv;
};

template <int T>
__device__ __forceinline__ void put8(void* base, int64_t i, f32x8 x) {
  if constexpr (T == CQA_TYPE_FP16) *(f16x8r*)((_Float16*)base + i) = __builtin_convertvector(x, f16x8r);
  else if constexpr (T == CQA_TYPE_BF16) *(bf16x8r*)((__bf16*)base + i) = __builtin_convertvector(x, bf16x8r);
  else *(f32x8r*)((float*)base + i) = x;
}

template <int T>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
  const int l = threadIdx.x & 63, cp = l & 15, tq = l >> 4;
  const int64_t blk = a.blk0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (blk * BLK >= a.end) return;
  const int64_t head = (int64_t)blockIdx.z * a.n_kv + blockIdx.y;
  const int64_t out0 = (int64_t)blockIdx.z * a.st.batch + (int64_t)blockIdx.y * a.st.head + 8 * cp;
  const auto row = [&](int t, int64_t& i) {   // of the block's token t; false: not asked for
    const int64_t tok = blk * BLK + t;
    i = out0 + (tok - a.first) * a.st.token;
    return tok >= a.first && tok < a.end;
  };
  if (blk >= a.nb) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = tq + 4 * r;
      int64_t i;
      if (!row(t, i)) continue;
      const int64_t src = (head * BLK + t) * D + 8 * cp;
      if (a.k != nullptr) put8<T>(a.k, i, __builtin_convertvector(*(const f16x8r*)((const _Float16*)a.trail_k + src), f32x8));
      if (a.v != nullptr) put8<T>(a.v, i, __builtin_convertvector(*(const f16x8r*)((const _Float16*)a.trail_v + src), f32x8));
    }
    return;
  }
  const int64_t rec = head * a.nq_cap;
  const int g = cp >> 1;
  if (a.k != nullptr) {
    const uint8_t* const kc = a.t1 + t1_offset(rec, blk, Q_KC, KC_BYTES);
    const float* const km = reinterpret_cast<const float*>(a.t1 + t1_offset(rec, blk, Q_KM, KM_BYTES));
    const f32x8 sigma = *(const f32x8r*)(km + 8 * cp), z = *(const f32x8r*)(km + D + 8 * cp);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = tq + 4 * r;
      const uint2 code = *reinterpret_cast<const uint2*>(kc + kc_offset(t, 8 * cp));
      int64_t i;
      if (!row(t, i)) continue;
      f32x8 x;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = e < 4 ? code.x : code.y;
        x[e] = fmaf((float)((w >> (8 * (e & 3))) & 255u) - 128.0f, sigma[e], z[e]);
      }
      put8<T>(a.k, i, x);
    }
  }
  if (a.v != nullptr) {
    const uint8_t* const vc = a.t1 + t1_offset(rec, blk, Q_VC, VC_BYTES);
    const _Float16* const vm = reinterpret_cast<const _Float16*>(a.t1 + t1_offset(rec, blk, Q_VM, VM_BYTES));
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint32_t*>(vc + vc_dword_offset(o, 8 * cp + e));
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int t = 8 * o + tq + 4 * r;
        int64_t i;
        if (!row(t, i)) continue;
        const _Float16 scale = vm[vm_index(t, g)], off = vm[BLK * NG + vm_index(t, g)];
        f32x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t code = (w[e] >> (4 * (t & 7))) & 15u;
          // To FP16 by one FP16 operation: rounded once.  The scale's rounding can take the largest code beyond the group's
          // maximum, and out of range where that is FP16's largest number.
          x[e] = T == CQA_TYPE_FP16 ? (float)__builtin_elementwise_minimum(__builtin_elementwise_fma((_Float16)code, scale, off), (_Float16)65504.0f)
                                    : fmaf((float)code, (float)scale, (float)off);
        }
        put8<T>(a.v, i, x);
      }
    }
  }
}

int32_t launch_read(const Cache* c, int layer, int64_t first, int64_t n, int type, void* k, void* v, const cqa_strides& strides,
                    hipStream_t st) {
  const int64_t head0 = head_index(c, layer, 0, 0);
  ReadArgs a;
  a.t1 = c->t1 + head0 * c->nq_cap * QUAD_BYTES;
  a.trail_k = c->trail_k + head0 * BLK * D;
  a.trail_v = c->trail_v + head0 * BLK * D;
  a.nq_cap = c->nq_cap;
  a.nb = c->length[layer] / BLK;
  a.first = first;
  a.end = first + n;
  a.blk0 = first / BLK;
  a.k = k;
  a.v = v;
  a.st = strides;
  a.n_kv = c->desc.n_kv_heads;
  const int64_t blocks = (a.end - 1) / BLK - a.blk0 + 1;
  const dim3 grid((uint32_t)((blocks + 3) / 4), (uint32_t)c->desc.n_kv_heads, (uint32_t)c->desc.batch);
  if (type == CQA_TYPE_FP16) read_kernel<CQA_TYPE_FP16><<<grid, 256, 0, st>>>(a);
  else if (type == CQA_TYPE_BF16) read_kernel<CQA_TYPE_BF16><<<grid, 256, 0, st>>>(a);
  else read_kernel<CQA_TYPE_FP32><<<grid, 256, 0, st>>>(a);
  CQA_HIP(hipGetLastError());
  return CQA_OK;
}

}  // namespace cqa
