// Rotary positions of the queries' and keys' rows ahead of cqa_cache_append and the decode calls.
//
// A pair of channels (a, b) of a row at position p turns by the angle p f_i:
//   a' = m (a cos - b sin),   b' = m (a sin + b cos).
// The angle is kept in turns as a 64-bit binary fraction: the host rounds f_i / 2 pi to 64 bits behind the point, p times that
// modulo 2^64 is the fraction of a turn exactly (for negative p as well).  What is left of an angle has an error of
// |p| 2^-64 turns (f_i's own rounding on the host and this one), below that of FP32 up to |p| = 2^40, and the sine and cosine of
// its upper 32 bits are within 2^-24 of a turn's.
//
// What bounds it: bytes, each row is read and written once.  A thread owns 8 pairs (16 channels) of one token and walks over the
// token's heads, so that the 8 sines and cosines are computed once for all of them.  Rows are written past the caches: a prompt of 8192
// tokens x 40 heads, BF16 to FP16, 43 -> 36 us (168 MB, 4.7 TB/s), 2 x 4099 x 24 in FP32 45 -> 43.
#include "cqa_internal.h"

namespace cqa {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8r __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x8r __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x8r __attribute__((ext_vector_type(8), aligned(4)));

// eight consecutive channels as FP32 numbers, from and to any address that one number may have
template <int T>
__device__ __forceinline__ f32x8 load8(const void* base, int64_t i) {
  if constexpr (T == CQA_TYPE_FP16) return __builtin_convertvector(*(const f16x8r*)((const _Float16*)base + i), f32x8);
  if constexpr (T == CQA_TYPE_BF16) return __builtin_convertvector(*(const bf16x8r*)((const __bf16*)base + i), f32x8);
  return *(const f32x8r*)((const float*)base + i);
}
template <int T>
__device__ __forceinline__ void store8(void* base, int64_t i, f32x8 x) {
  if constexpr (T == CQA_TYPE_FP16) __builtin_nontemporal_store(__builtin_convertvector(x, f16x8r), (f16x8r*)((_Float16*)base + i));
  else if constexpr (T == CQA_TYPE_BF16) __builtin_nontemporal_store(__builtin_convertvector(x, bf16x8r), (bf16x8r*)((__bf16*)base + i));
  else __builtin_nontemporal_store((f32x8r)x, (f32x8r*)((float*)base + i));
}
template <int T>
__device__ __forceinline__ float load1(const void* base, int64_t i) {
  if constexpr (T == CQA_TYPE_FP16) return (float)((const _Float16*)base)[i];
  if constexpr (T == CQA_TYPE_BF16) return (float)((const __bf16*)base)[i];
  return ((const float*)base)[i];
}
template <int T>
__device__ __forceinline__ void store1(void* base, int64_t i, float x) {
  if constexpr (T == CQA_TYPE_FP16) ((_Float16*)base)[i] = (_Float16)x;
  else if constexpr (T == CQA_TYPE_BF16) ((__bf16*)base)[i] = (__bf16)x;
  else ((float*)base)[i] = x;
}

struct RotaryArgs {
  uint64_t turn[D / 2];        // f_i / 2 pi, 64 bits behind the point
  const int64_t* positions;
  int64_t pos_batch;
  int64_t n_tokens;
  cqa_rotary_rows rows[2];     // the second with n_heads = 0: there is none
  float magnitude;
  int half;                    // pairs that turn
  int interleaved;
  int tok_shift;               // a workgroup takes 2^tok_shift tokens side by side ...
  int heads_per;               // ... and so many heads of each
};

__device__ __forceinline__ void sin_cos_of(uint64_t turn, int64_t p, float m, float& s, float& c) {
  const int32_t x = (int32_t)((turn * (uint64_t)p) >> 32);
  sincospif((float)x * 0x1p-31f, &s, &c);
  s *= m;
  c *= m;
}

// P = 8: a thread has 8 pairs, where their channels come in whole runs of 8 (rot_dim a multiple of 16); P = 1: one pair, any rot_dim (the two prompts
// of the figures above by P = 1: 86 us for 35, 73 for 42).
template <int TI, int TO, int P>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  constexpr int UNITS = D / 2 / P;   // threads a row takes
  const int unit = threadIdx.x % UNITS, slot = threadIdx.x / UNITS;
  const int64_t t = ((int64_t)blockIdx.x << a.tok_shift) + (slot & ((1 << a.tok_shift) - 1));
  if (t >= a.n_tokens) return;
  const int64_t b = blockIdx.z;
  const int side = (256 / UNITS) >> a.tok_shift;   // heads side by side
  const int n_all = a.rows[0].n_heads + a.rows[1].n_heads;
  const int h_end = min(n_all, ((int)blockIdx.y + 1) * a.heads_per);
  const int i0 = unit * P;
  const bool turns = i0 < a.half;
  // first channels of the thread's two runs
  const int ca = turns ? (a.interleaved ? 2 * i0 : i0) : 2 * i0;
  const int cb = turns ? (a.interleaved ? 2 * i0 + P : i0 + a.half) : 2 * i0 + P;
  float s[P], c[P];
  if (turns) {
    const int64_t p = a.positions[b * a.pos_batch + t];
#pragma unroll
    for (int e = 0; e < P; ++e) sin_cos_of(a.turn[i0 + e], p, a.magnitude, s[e], c[e]);
  }
  for (int h = (int)blockIdx.y * a.heads_per + (slot >> a.tok_shift); h < h_end; h += side) {
    const bool second = h >= a.rows[0].n_heads;
    const cqa_rotary_rows& r = second ? a.rows[1] : a.rows[0];
    const int64_t hh = second ? h - a.rows[0].n_heads : h;
    const int64_t in = b * r.in_strides.batch + hh * r.in_strides.head + t * r.in_strides.token;
    const int64_t out = b * r.out_strides.batch + hh * r.out_strides.head + t * r.out_strides.token;
    if constexpr (P == 8) {
      f32x8 x = load8<TI>(r.in_dev, in + ca), y = load8<TI>(r.in_dev, in + cb);
      if (turns) {
        if (a.interleaved) {
          // runs hold (a, b) (a, b) ..: the pairs of x are the thread's first four
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float xa = x[2 * e], xb = x[2 * e + 1], ya = y[2 * e], yb = y[2 * e + 1];
            x[2 * e] = fmaf(xa, c[e], -xb * s[e]);
            x[2 * e + 1] = fmaf(xa, s[e], xb * c[e]);
            y[2 * e] = fmaf(ya, c[4 + e], -yb * s[4 + e]);
            y[2 * e + 1] = fmaf(ya, s[4 + e], yb * c[4 + e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float xa = x[e], xb = y[e];
            x[e] = fmaf(xa, c[e], -xb * s[e]);
            y[e] = fmaf(xa, s[e], xb * c[e]);
          }
        }
      }
      store8<TO>(r.out_dev, out + ca, x);
      store8<TO>(r.out_dev, out + cb, y);
    } else {
      float x = load1<TI>(r.in_dev, in + ca), y = load1<TI>(r.in_dev, in + cb);
      if (turns) {
        const float xa = x, xb = y;
        x = fmaf(xa, c[0], -xb * s[0]);
        y = fmaf(xa, s[0], xb * c[0]);
      }
      store1<TO>(r.out_dev, out + ca, x);
      store1<TO>(r.out_dev, out + cb, y);
    }
  }
}

template <int TI, int TO>
static void launch_types(const RotaryArgs& a, bool wide, dim3 grid, hipStream_t st) {
  if (wide)
    rotary_kernel<TI, TO, 8><<<grid, 256, 0, st>>>(a);
  else
    rotary_kernel<TI, TO, 1><<<grid, 256, 0, st>>>(a);
}
template <int TI>
static void launch_from(const RotaryArgs& a, int out_type, bool wide, dim3 grid, hipStream_t st) {
  if (out_type == CQA_TYPE_FP16) launch_types<TI, CQA_TYPE_FP16>(a, wide, grid, st);
  else if (out_type == CQA_TYPE_BF16) launch_types<TI, CQA_TYPE_BF16>(a, wide, grid, st);
  else launch_types<TI, CQA_TYPE_FP32>(a, wide, grid, st);
}

int32_t launch_rotary(const Rotary& r, const int64_t* positions, int64_t pos_batch, int batch, int64_t n_tokens,
                      const cqa_rotary_rows* rows, int n_rows, int in_type, int out_type, hipStream_t st) {
  RotaryArgs a;
  for (int i = 0; i < D / 2; ++i) a.turn[i] = r.turn[i];
  a.positions = positions;
  a.pos_batch = pos_batch;
  a.n_tokens = n_tokens;
  a.rows[0] = rows[0];
  a.rows[1] = rows[n_rows - 1];
  if (n_rows < 2) a.rows[1].n_heads = 0;
  a.magnitude = r.magnitude;
  a.half = r.rot_dim / 2;
  a.interleaved = r.layout == CQA_ROTARY_INTERLEAVED;
  const bool wide = r.rot_dim % 16 == 0;
  const int slots = wide ? 32 : 4;   // rows side by side in a workgroup
  a.tok_shift = 0;
  while ((1 << a.tok_shift) < slots && (1 << a.tok_shift) < n_tokens) ++a.tok_shift;
  // As many heads a thread as leave the device's 256 compute units 8 workgroups each: the sines are shared by them.  (4, 8, 16, 32 each: 8192 tokens x 40 heads,
  // BF16 to FP16, 33.9, 35.3, 36.0, 39.8 us; 2 x 4099 x 24 in FP32 45.7, 42.4, 41.3, 41.3; a row requested ahead of the one before 36.3, 34.6 and 49.9, 45.1.)
  const int n_all = a.rows[0].n_heads + a.rows[1].n_heads;
  const int64_t tiles = ((n_tokens - 1) >> a.tok_shift) + 1;
  a.heads_per = slots >> a.tok_shift;
  while (a.heads_per < n_all && tiles * batch * ((n_all + 2 * a.heads_per - 1) / (2 * a.heads_per)) >= 2048) a.heads_per *= 2;
  const int64_t gy = (n_all + a.heads_per - 1) / a.heads_per;
  if (tiles > 0xffffff || gy > 65535) return CQA_ERR_UNSUPPORTED;
  const dim3 grid((uint32_t)tiles, (uint32_t)gy, (uint32_t)batch);
  if (in_type == CQA_TYPE_FP16) launch_from<CQA_TYPE_FP16>(a, out_type, wide, grid, st);
  else if (in_type == CQA_TYPE_BF16) launch_from<CQA_TYPE_BF16>(a, out_type, wide, grid, st);
  else launch_from<CQA_TYPE_FP32>(a, out_type, wide, grid, st);
  CQA_HIP(hipGetLastError());
  return CQA_OK;
}

}  // namespace cqa
