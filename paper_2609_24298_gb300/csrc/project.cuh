// The fp32 projection of a few vectors of a head on its basis, O[v][i] = sum_d W[i][d] X[v][d], by one
// CTA: the appends and the query projections run it.
#pragma once

#include "common.cuh"

namespace cobra {

// One CTA of 256 threads stages the head's basis in shared memory once (row stride kProjLd floats, so
// that a warp's 16-byte row reads are conflict-free) and its warps share out (4 vectors) x (32, 64 or
// 128 channels) units, so that one sequence's vectors keep every warp busy as well as 32 vectors do.
// Each output is summed over d in the same order whatever the split: the codes do not depend on it.
constexpr int kAppendThreads = 256;
constexpr int kProjWarps = kAppendThreads / 32;
constexpr int kProjLd = 132;
constexpr int kProjVecs = 40;  // vectors per pass (32 queries and the new tokens of their sequences)
__host__ __device__ constexpr size_t proj_smem_bytes() {
  return sizeof(float) * ((size_t)kD * kProjLd + (size_t)kProjVecs * kD + (size_t)kProjVecs * kProjLd + kD + kProjVecs);
}
// the shared memory of a projecting CTA
struct ProjSmem {
  float* Ws;   // [kD][kProjLd] basis row i = channel i (rows past r are not written)
  float* Xs;   // [kProjVecs][kD] vectors of this pass
  float* Os;   // [kProjVecs][kProjLd] their projections
  float* wmu;  // [kD] W^T mu
  int* pos;    // [kProjVecs] positions of the pass's new tokens
  __device__ explicit ProjSmem(float* base)
      : Ws(base), Xs(Ws + kD * kProjLd), Os(Xs + kProjVecs * kD), wmu(Os + kProjVecs * kProjLd),
        pos(reinterpret_cast<int*>(wmu + kD)) {}
};

// nv vectors of 128 bf16 into Xs; row(v) is vector v's address.  `wide`: every row is 16-byte
// aligned (in general they are only 2-byte aligned).
template <typename Row>
__device__ __forceinline__ void proj_load(int nv, bool wide, Row row, float* Xs) {
  if (wide) {
#pragma unroll 3
    for (int idx = threadIdx.x; idx < nv * (kD / 8); idx += kAppendThreads) {
      const int v = idx / (kD / 8), c = idx % (kD / 8);
      const uint4 u = reinterpret_cast<const uint4*>(row(v))[c];
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      float f[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[2 * k] = __uint_as_float(w[k] << 16);
        f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
      float4* o = reinterpret_cast<float4*>(Xs + v * kD + 8 * c);
      o[0] = make_float4(f[0], f[1], f[2], f[3]);
      o[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
  } else {
#pragma unroll 16
    for (int idx = threadIdx.x; idx < nv * kD; idx += kAppendThreads) Xs[idx] = __bfloat162float(row(idx / kD)[idx % kD]);
  }
}

// A warp's unit: vectors 4 vg .. 4 vg + 3 times CB blocks of 32 channels from block cb.  Rows of
// Ws past r hold anything; their results are not stored.
template <int CB>
__device__ __forceinline__ void proj_unit(const ProjSmem& sm, int vg, int cb, int nv, int r) {
  const int lane = threadIdx.x & 31;
  float acc[CB][4];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[c][v] = 0.f;
  const float* Wp = sm.Ws + (lane + 32 * cb) * kProjLd;
  const float* Xp = sm.Xs + 4 * vg * kD;
#pragma unroll 4
  for (int d = 0; d < kD; d += 4) {
    float4 w[CB], x[4];
#pragma unroll
    for (int c = 0; c < CB; ++c) w[c] = *reinterpret_cast<const float4*>(Wp + 32 * c * kProjLd + d);
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = *reinterpret_cast<const float4*>(Xp + v * kD + d);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        acc[c][v] += w[c].x * x[v].x + w[c].y * x[v].y + w[c].z * x[v].z + w[c].w * x[v].w;
  }
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const int ch = lane + 32 * (cb + c);
    if (ch >= r) continue;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (4 * vg + v < nv) sm.Os[(4 * vg + v) * kProjLd + ch] = acc[c][v];
  }
}
// Os <- projections of the nv vectors in Xs on the r channels.  Wider units read each basis value
// for more vectors' worth of work per shared-memory access; they are used once there are enough
// of them for the 8 warps, and no wider than the head's channels.
template <int CB>
__device__ __forceinline__ void proj_units(const ProjSmem& sm, int nv, int r) {
  const int ng = (nv + 3) >> 2, nc = ((r + 31) / 32 + CB - 1) / CB;
  for (int u = threadIdx.x >> 5; u < ng * nc; u += kProjWarps) proj_unit<CB>(sm, u / nc, CB * (u % nc), nv, r);
}
__device__ __forceinline__ void project(const ProjSmem& sm, int nv, int r) {
  const int units = ((nv + 3) >> 2) * ((r + 31) / 32);
  if (units <= kProjWarps)
    proj_units<1>(sm, nv, r);
  else if (units <= 2 * kProjWarps || r <= 64)
    proj_units<2>(sm, nv, r);
  else
    proj_units<4>(sm, nv, r);
}

// Issues the copies of a head's W^T mu and basis rows [0, r) (parameters: this may run before the
// wait for the kernel ahead).  The caller waits with cp_async_wait_all and synchronises the block.
// W^T mu is r floats; the pool is padded to 32 floats, so whole 16-byte chunks stay in it.
__device__ __forceinline__ void proj_stage_issue(const ProjSmem& sm, const float* pool, const HeadEntry& he) {
  const int tid = threadIdx.x;
  if (tid < (he.r + 3) / 4) cp_async16(smem_addr(sm.wmu + 4 * tid), pool + he.wmu_off + 4 * tid);
  const float* W = pool + he.w_off;
  for (int idx = tid; idx < he.r * (kD / 4); idx += kAppendThreads)
    cp_async16(smem_addr(sm.Ws + (idx >> 5) * kProjLd + 4 * (idx & 31)), W + (size_t)idx * 4);
}

}  // namespace cobra
