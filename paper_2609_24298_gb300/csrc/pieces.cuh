// A head's basis (and vectors) as sums of bf16 pieces, the operands of tensor-core projections: each piece is the
// rounding of what the ones before leave, so N of them leave 2^-(9N - 1) of a value behind (bf16 rounds by 2^-8 at
// most, just above a power of two; what is left then lies below one).
#pragma once

#include "common.cuh"

namespace cobra {

// Two fp32 values to N pieces each; what is left of them.
template <int N>
__device__ __forceinline__ float2 split_pieces(float a, float b, uint32_t (&p)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    p[k] = pack_bf16(a, b);
    a -= __uint_as_float(p[k] << 16);
    b -= __uint_as_float(p[k] & 0xFFFF0000u);
  }
  return make_float2(a, b);
}

// The r rows of W to [piece][dimensions 0 .. 63, 64 .. 127][channel], 128-byte rows, swizzled (K-major): a warp of
// kWarps per channel, a lane per four dimensions, kRows channels i0, i0 + kWarps, ... at a time: their loads, and
// what is made of them.  norm(channel, f.x |w|^2 + f.y |w2|^2 + f.z |w - w1 - w2|^2) in every lane, where kNorms
// (of three pieces: f.x |w|^2).  A head without channels has no rows, and
// its offset need not be one that 16 bytes can be read at.
template <int kWarps, int kRows>
__device__ __forceinline__ void load_basis(float4 (&w)[kRows], const float* W, int r, int i0) {
#pragma unroll
  for (int k = 0; k < kRows; ++k)
    w[k] = r > 0 ? reinterpret_cast<const float4*>(W + min(i0 + k * kWarps, r - 1) * kD)[threadIdx.x & 31]
                 : make_float4(0.f, 0.f, 0.f, 0.f);
}
template <int N, int kWarps, bool kNorms, int kRows, typename F>
__device__ __forceinline__ void lay_basis(unsigned char (*to)[2][kD * 128], const float4 (&w)[kRows], int r, int i0, float3 f, F norm) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int i = i0 + k * kWarps;
    if (i >= r) break;
    uint32_t p[N], q[N];
    const float2 u = split_pieces(w[k].x, w[k].y, p), v = split_pieces(w[k].z, w[k].w, q);
    if (kNorms) {
      float n2 = f.x * (w[k].x * w[k].x + w[k].y * w[k].y + w[k].z * w[k].z + w[k].w * w[k].w);
      if (N == 2) {
        const float x = __uint_as_float(p[1] << 16), y = __uint_as_float(p[1] & 0xFFFF0000u), z = __uint_as_float(q[1] << 16),
                    t = __uint_as_float(q[1] & 0xFFFF0000u);
        n2 = fmaf(f.y, x * x + y * y + z * z + t * t, fmaf(f.z, u.x * u.x + u.y * u.y + v.x * v.x + v.y * v.y, n2));
      }
#pragma unroll
      for (int m = 16; m; m >>= 1) n2 += __shfl_xor_sync(0xffffffffu, n2, m);
      norm(i, n2);
    }
    const int at = i * 128 + ((((lane & 15) >> 1) ^ (i & 7)) << 4) + 8 * (lane & 1);
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<uint2*>(to[n][lane >> 4] + at) = make_uint2(p[n], q[n]);
  }
}

// A lane's dimensions 2 l, 2 l + 1 and the ones 64 behind, as two words; `wide`: 4-byte aligned (else 2-byte).
__device__ __forceinline__ void load_pairs(const __nv_bfloat16* x, bool wide, uint32_t& a, uint32_t& b) {
  const int lane = threadIdx.x & 31;
  if (wide) {
    a = reinterpret_cast<const uint32_t*>(x)[lane];
    b = reinterpret_cast<const uint32_t*>(x)[lane + 32];
  } else {
    const unsigned short* h = reinterpret_cast<const unsigned short*>(x);
    a = h[2 * lane] | (uint32_t)h[2 * lane + 1] << 16;
    b = h[2 * lane + 64] | (uint32_t)h[2 * lane + 65] << 16;
  }
}
// where those words lie in vector v's row
__device__ __forceinline__ int pair_at(int v) {
  const int lane = threadIdx.x & 31;
  return v * 128 + (((lane >> 2) ^ (v & 7)) << 4) + 4 * (lane & 3);
}

}  // namespace cobra
