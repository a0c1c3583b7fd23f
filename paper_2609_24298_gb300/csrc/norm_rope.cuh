// Per-head norms of queries and keys with the rotary rotation in the same pass:
//   y = R(pos) (x / sqrt(mean(x^2) + eps) * w)   per head vector x of 128,
// R(x) as in rope.cuh: pair (j, j + 64) turned by pos theta^(-2j/128).  The mean, the norm and the
// rotation are in fp32; the result is rounded to bf16 once.
//
// Bound: HBM (256 bytes in and out per head vector, some 60 instructions per 16 of its elements).
// Eight lanes hold a head vector, lane l elements 8 l .. 8 l + 7 of both halves: a lane has whole
// pairs, loads and stores 16 bytes at a time, and the sum of squares takes three shuffles.  A warp
// takes a token and four heads at a time; the token's angles are composed once per lane (from the
// coarse and fine rows of the angle table) and kept in registers over `per_warp` groups of four heads.
// 16383 tokens x 72 heads: 100 us, 6.0 TB/s.
#pragma once

#include "common.cuh"
#include "rope_angles.cuh"

namespace cobra {

constexpr int kNormThreads = 128;
constexpr int kNormAhead = 2;  // groups in flight (16383 tokens x 72 heads: 116 us with one, 101 with two, 113 with three)

struct NormSide {
  const __nv_bfloat16* x;
  __nv_bfloat16* out;
  const float* w;  // 128 weights or null
  long long st, sh, ot, oh;
  int heads;
};
struct NormArgs {
  NormSide q, k;
  const int* pos;
  const float* table;  // null: no rotation
  int n_coarse, n_tok, norm;
  float eps;
  int q_groups, groups;  // groups of four heads: of q, of q and k
  int per_warp;          // groups a warp takes
};

__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f[2 * k] = __uint_as_float(w[k] << 16);
    f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
  }
}

// Vectors whose squares leave fp32's range (`far`): scaled by the power of two that takes the larger of the largest element
// and sqrt(eps) to [1, 2), which leaves x / sqrt(mean(x^2) + eps) as it is.  The reciprocal roots, of the others too.
__device__ __forceinline__ float norm_scaled(float (&lo)[8], float (&hi)[8], float eps, bool far) {
  float m = sqrtf(eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fmaxf(fabsf(lo[i]), fabsf(hi[i])));
#pragma unroll
  for (int x = 4; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  // 2^-k in two factors (k may be -126); an infinite element is left as it is
  const int k = far && m < INFINITY ? max((int)(__float_as_uint(m) >> 23), 1) - 127 : 0, k1 = k / 2;
  const float f = __uint_as_float((uint32_t)(127 - k1) << 23), g = __uint_as_float((uint32_t)(127 - (k - k1)) << 23);
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = lo[i] * f * g, hi[i] = hi[i] * f * g;
    ss = fmaf(lo[i], lo[i], fmaf(hi[i], hi[i], ss));
  }
#pragma unroll
  for (int x = 4; x; x >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, x);
  return rsqrtf(fmaf(ss, 1.f / kD, eps * f * f * g * g));
}

__global__ void __launch_bounds__(kNormThreads, 8) norm_rope_kernel(NormArgs a) {
  grid_dep_launch();
  // the vectors may come from the kernel ahead, or still be read by it where the output goes
  grid_dep_wait();
  const int lane = threadIdx.x & 31, l8 = lane & 7;
  const int runs = (a.groups + a.per_warp - 1) / a.per_warp;
  const long long wid = (long long)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
  const int tok = (int)(wid / runs), g0 = (int)(wid % runs) * a.per_warp, g1 = min(a.groups, g0 + a.per_warp);
  if (tok >= a.n_tok) return;
  // cos and sin of the lane's pairs j = 8 l8 + i; entry (n, jj) of a table row holds pair 4 n + jj
  float c[8], s[8];
  if (a.table) {
    int p = a.pos[tok];
    const int max_pos = kRopeFine * a.n_coarse;
    if (p < 0 || p >= max_pos) {  // outside the table: reported, computed with the nearest angles
      if (lane == 0 && g0 == 0) atomicOr(&g_status, 2u);
      p = min(max(p, 0), max_pos - 1);
    }
    const float4* fine = reinterpret_cast<const float4*>(a.table + (size_t)(p & 15) * kRopeRowFloats);
    const float4* crs = reinterpret_cast<const float4*>(a.table + (size_t)(kRopeFine + (p >> 4)) * kRopeRowFloats);
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const float4 f = fine[jj * 8 + l8], m = crs[jj * 8 + l8];
      rope_compose(m.x, m.y, f.x, f.y, c[jj], s[jj]);
      rope_compose(m.z, m.w, f.z, f.w, c[4 + jj], s[4 + jj]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = 1.f, s[i] = 0.f;
  }
  // the lane's halves of group g's vector (x and out may be the same memory, so the compiler would not load the
  // next groups' ahead of a store)
  auto load = [&](int g, uint4& ulo, uint4& uhi) {
    const bool key = g >= a.q_groups;
    const NormSide& sd = key ? a.k : a.q;
    const int head = 4 * (key ? g - a.q_groups : g) + (lane >> 3);
    ulo = uhi = make_uint4(0u, 0u, 0u, 0u);
    if (g < g1 && head < sd.heads) {
      const uint4* x = reinterpret_cast<const uint4*>(sd.x + tok * sd.st + head * sd.sh);
      ulo = x[l8];
      uhi = x[8 + l8];
    }
  };
  auto turn = [&](int g, const uint4& ulo, const uint4& uhi) {
    const bool key = g >= a.q_groups;
    const NormSide& sd = key ? a.k : a.q;
    const int head = 4 * (key ? g - a.q_groups : g) + (lane >> 3);
    const bool live = g < g1 && head < sd.heads;
    float lo[8], hi[8];
    unpack8(ulo, lo);
    unpack8(uhi, hi);
    if (a.norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(lo[i], lo[i], fmaf(hi[i], hi[i], ss));
#pragma unroll
      for (int m = 4; m; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
      const float mean = fmaf(ss, 1.f / kD, a.eps);
      float inv = rsqrtf(mean);  // (2 units in the last place)
      const bool far = live && !(mean >= 1e-30f && mean < INFINITY);
      if (__any_sync(0xffffffffu, far)) inv = norm_scaled(lo, hi, a.eps, far);
      if (sd.w) {
        const float4* w4 = reinterpret_cast<const float4*>(sd.w);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 wl = __ldg(w4 + 2 * l8 + h), wh = __ldg(w4 + 16 + 2 * l8 + h);
          lo[4 * h] *= inv * wl.x, lo[4 * h + 1] *= inv * wl.y, lo[4 * h + 2] *= inv * wl.z, lo[4 * h + 3] *= inv * wl.w;
          hi[4 * h] *= inv * wh.x, hi[4 * h + 1] *= inv * wh.y, hi[4 * h + 2] *= inv * wh.z, hi[4 * h + 3] *= inv * wh.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) lo[i] *= inv, hi[i] *= inv;
      }
    }
    uint32_t ol[4], oh[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float a0 = lo[2 * k], a1 = lo[2 * k + 1], b0 = hi[2 * k], b1 = hi[2 * k + 1];
      if (a.table) {
        const float c0 = c[2 * k], s0 = s[2 * k], c1 = c[2 * k + 1], s1 = s[2 * k + 1];
        const float ra0 = fmaf(a0, c0, -b0 * s0), rb0 = fmaf(a0, s0, b0 * c0);
        const float ra1 = fmaf(a1, c1, -b1 * s1), rb1 = fmaf(a1, s1, b1 * c1);
        a0 = ra0, b0 = rb0, a1 = ra1, b1 = rb1;
      }
      ol[k] = pack_bf16(a0, a1);
      oh[k] = pack_bf16(b0, b1);
    }
    if (live) {
      uint4* o = reinterpret_cast<uint4*>(sd.out + tok * sd.ot + head * sd.oh);
      o[l8] = make_uint4(ol[0], ol[1], ol[2], ol[3]);
      o[8 + l8] = make_uint4(oh[0], oh[1], oh[2], oh[3]);
    }
  };
  uint4 lo0[kNormAhead], hi0[kNormAhead];
#pragma unroll
  for (int k = 0; k < kNormAhead; ++k) load(g0 + k, lo0[k], hi0[k]);
  for (int g = g0; g < g1; g += kNormAhead) {
#pragma unroll
    for (int k = 0; k < kNormAhead; ++k) {
      turn(g + k, lo0[k], hi0[k]);
      load(g + k + kNormAhead, lo0[k], hi0[k]);
    }
  }
}

}  // namespace cobra
