// Reading the cache back: the reconstruction of tokens of every sequence, k = code sigma + z (one fused multiply-add in FP32) and
// v = code scale + offset, rounded once to the asked type; trailing tokens are their FP16 originals.
//
// What bounds it: bytes, 288 read and 512 (FP16) written per token and KV head.  One wave a block of 16 tokens, a lane 16 bytes of a row: C = 8
// channels of tokens tq, tq + 4, tq + 8, tq + 12, or, of FP32 rows, C = 4 of tokens tq, tq + 2, ..., so that sigma and z are fetched
// once for all of the lane's tokens, a dword of value codes (one channel of eight tokens) serves half of them, and each
// store of a wave is whole rows, past the caches (128K tokens of 8 heads to FP16 180 -> 172 us; 4 x 8 heads x 9400 to FP32, token-major, 94 ->
// 82, and 117 with 8 channels a lane).
#include "cqa_internal.h"

namespace cqa {

typedef _Float16 f16x8r __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x8r __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4r __attribute__((ext_vector_type(4), aligned(4)));

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

template <int T, int C>
__device__ __forceinline__ void put(void* base, int64_t i, const float (&x)[C]) {
  if constexpr (T == CQA_TYPE_FP32) {
    f32x4r y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[e];
    __builtin_nontemporal_store(y, (f32x4r*)((float*)base + i));
  } else if constexpr (T == CQA_TYPE_FP16) {
    f16x8r y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (_Float16)x[e];
    __builtin_nontemporal_store(y, (f16x8r*)((_Float16*)base + i));
  } else {
    bf16x8r y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];
    __builtin_nontemporal_store(y, (bf16x8r*)((__bf16*)base + i));
  }
}

template <int T>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
  constexpr int C = T == CQA_TYPE_FP32 ? 4 : 8, LANES = D / C, SIDE = 64 / LANES;   // channels a lane, lanes a row, rows side by side
  const int l = threadIdx.x & 63, cp = l % LANES, tq = l / LANES;
  const int64_t blk = a.blk0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (blk * BLK >= a.end) return;
  const int64_t head = (int64_t)blockIdx.z * a.n_kv + blockIdx.y;
  const int64_t out0 = (int64_t)blockIdx.z * a.st.batch + (int64_t)blockIdx.y * a.st.head + C * cp;
  const auto row = [&](int t, int64_t& i) {   // of the block's token t; false: not asked for
    const int64_t tok = blk * BLK + t;
    i = out0 + (tok - a.first) * a.st.token;
    return tok >= a.first && tok < a.end;
  };
  if (blk >= a.nb) {
#pragma unroll
    for (int r = 0; r < BLK / SIDE; ++r) {
      const int t = tq + SIDE * r;
      int64_t i;
      if (!row(t, i)) continue;
      const int64_t src = (head * BLK + t) * D + C * cp;
      float x[C];
      if (a.k != nullptr) {
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = __half2float(a.trail_k[src + e]);
        put<T>(a.k, i, x);
      }
      if (a.v != nullptr) {
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = __half2float(a.trail_v[src + e]);
        put<T>(a.v, i, x);
      }
    }
    return;
  }
  const int64_t rec = head * a.nq_cap;
  const int g = C * cp / VG;
  if (a.k != nullptr) {
    const uint8_t* const kc = a.t1 + t1_offset(rec, blk, Q_KC, KC_BYTES);
    const float* const km = reinterpret_cast<const float*>(a.t1 + t1_offset(rec, blk, Q_KM, KM_BYTES)) + C * cp;
    float sigma[C], z[C];
#pragma unroll
    for (int e = 0; e < C; e += 4) {
      *reinterpret_cast<float4*>(sigma + e) = *reinterpret_cast<const float4*>(km + e);
      *reinterpret_cast<float4*>(z + e) = *reinterpret_cast<const float4*>(km + D + e);
    }
#pragma unroll
    for (int r = 0; r < BLK / SIDE; ++r) {
      const int t = tq + SIDE * r;
      uint32_t code[C / 4];
#pragma unroll
      for (int e = 0; e < C / 4; ++e) code[e] = reinterpret_cast<const uint32_t*>(kc + kc_offset(t, C * cp))[e];
      int64_t i;
      if (!row(t, i)) continue;
      float x[C];
#pragma unroll
      for (int e = 0; e < C; ++e) x[e] = as_rounded(fmaf((float)((code[e >> 2] >> (8 * (e & 3))) & 255u) - 128.0f, sigma[e], z[e]));
      put<T>(a.k, i, x);
    }
  }
  if (a.v != nullptr) {
    const uint8_t* const vc = a.t1 + t1_offset(rec, blk, Q_VC, VC_BYTES);
    const _Float16* const vm = reinterpret_cast<const _Float16*>(a.t1 + t1_offset(rec, blk, Q_VM, VM_BYTES));
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      uint32_t w[C];
#pragma unroll
      for (int e = 0; e < C; ++e) w[e] = *reinterpret_cast<const uint32_t*>(vc + vc_dword_offset(o, C * cp + e));
#pragma unroll
      for (int r = 0; r < 8 / SIDE; ++r) {
        const int t = 8 * o + tq + SIDE * r;
        int64_t i;
        if (!row(t, i)) continue;
        const _Float16 scale = vm[vm_index(t, g)], off = vm[BLK * NG + vm_index(t, g)];
        float x[C];
#pragma unroll
        for (int e = 0; e < C; ++e) {
          const uint32_t code = (w[e] >> (4 * (t & 7))) & 15u;
          // To FP16 by one FP16 operation: rounded once.  The scale's rounding can take the largest code beyond the group's
          // maximum, and out of range where that is FP16's largest number.
          x[e] = T == CQA_TYPE_FP16 ? (float)__builtin_elementwise_minimum(__builtin_elementwise_fma((_Float16)code, scale, off), (_Float16)65504.0f)
                                    : as_rounded(fmaf((float)code, (float)scale, (float)off));
        }
        put<T>(a.v, i, x);
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
