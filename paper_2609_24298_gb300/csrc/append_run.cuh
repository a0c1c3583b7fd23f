// Runs of new tokens into the packed cache, K and V in one launch (Table alg:kvrobin step 7 for several
// tokens per sequence, at any position): y = W^T (R(pos) x - mu), code = clamp(floor(y / Delta +
// 2^{b-1}), 0, 2^b - 1), format v1; R turns keys to their positions where a table is given, else R = 1.
//
// Codes are those of the exact y: the projection runs on the tensor cores with a bound on its error, and a value
// that lies within the bound of a cell's border is done again by its warp, four dimensions a lane: in pairs of
// fp32, and in fp64 (two lanes' worth of it per cycle and SM) if those still cannot tell.  So the codes depend
// neither on the order of summation nor on how tokens are grouped.
//
// The projection: W = w1 + w2 + w3, a turned x = x1 + x2 + x3 in bf16 pieces (each the rounding of what the ones
// before leave: 2^-26 of a value is left behind), a plain x is bf16 already; the products w_i x_j with i + j <= 4
// (w_i x_1) accumulate in fp32, the small ones first.  M = 128 channels, N = up to 128 vectors, K = 128.
// A sum of 16 products and the accumulator keeps bits down to 2^-25 of its largest addend and is cut to 24 bits
// (measured; addends 1 and s, s = 2^-16 .. 2^-31), so an instruction is off by at most (16 2^-25 + 2^-23) |w| |x|
// (Cauchy-Schwarz), the last eight make 1.25 2^-18 |w| |x| of it and the ones before, of sums below 2^-7 of
// that, little.  With the pieces' rest and the turned x (6 2^-24 (|xa| + |xb|) per element) that is below
// 2^-17 |w| |x|, and W^T mu adds its rounding, 2^-24 of it; at worst 2^-20.8 |w| |x| was seen (40 x 8192 sums, heavy tails).
//
// A CTA works through its share of all (side, layer, kv head, code row): it lays a head's
// basis out in pieces, takes rows of up to kTokens tokens together (all new tokens of a sequence in one code row go
// together), keeps their codes in shared memory and then merges every touched word of the rows once: a plain
// read and write, because nobody else has the row.
//
// What bounds it: chains of memory round trips per batch (positions, vectors and angles, products, codes, words),
// and the instructions that turn and split keys.  32 layers x 8 kv heads x 64 sequences x 4 tokens, K turned: 128 us,
// of whose touched sectors 200 MB have to move (30 us); 2001 tokens of a layer 29 us; 304 and 61 with the projection
// in fp32 on the CUDA cores.
#pragma once

#include "common.cuh"
#include "pieces.cuh"
#include "rope_angles.cuh"
#include "tc.cuh"

namespace cobra {

// Long runs: 128 tokens per batch (a whole code row), one CTA per SM.
struct RunMany {
  static constexpr int kThreads = 512, kTokens = 128, kPieces = 3, kPerSm = 1;
};
// Shorter ones: 64 or 32 tokens per batch, and W and x in two pieces, so that two CTAs fit: one's products run beside
// the other's loads, and the next call's basis is laid out while this one still runs.
struct RunMid {
  static constexpr int kThreads = 256, kTokens = 64, kPieces = 2, kPerSm = 2;
};
struct RunFew {
  static constexpr int kThreads = 256, kTokens = 32, kPieces = 2, kPerSm = 2;
};
// The error of a projection is below 2^-18 |x| times the root of a sum over the channel's basis,
//   f.x |w|^2 + f.y |w2|^2 + f.z |w - w1 - w2|^2   (the first term alone with three pieces: 2^-17 |w| |x|).
// With two pieces, in units of 2^-18 |x|: the sums' 1.27 |w|; 2^18 |w - w1 - w2|; and for a turned x what its second piece
// leaves, 2 |w|, the turn's 0.2 |w| and the dropped w2 x2, 2^10 |w2| (x2 is 2^-8 of x at most, and so may w2 be of w;
// as a rule it is a third of that, and a bound for the worst case would send 1.7 times as many codes to be done again:
// 131 us for 129, 32 layers x 64 sequences x 4 tokens).  By Cauchy-Schwarz
// (a + b + c)^2 <= a^2 / A + b^2 / B + c^2 / C where A + B + C = 1, best with A, B, C as the terms are.
template <class C>
__device__ __forceinline__ float3 run_error(bool turn) {
  if (C::kPieces == 3) return make_float3(4.f, 0.f, 0.f);
  return turn ? make_float3(3.48f * 3.48f / 0.64f, 1.01f * 1048576.f / 0.24f, 68719476736.f / 0.12f)
              : make_float3(1.27f * 1.27f / 0.66f, 0.f, 68719476736.f / 0.34f);
}
constexpr int kRunSegs = 32;             // code rows per batch
constexpr int kRunSeqs = 256;            // sequences per block of the row count
constexpr int kRunCodeLd = 132;
constexpr uint64_t kRunWaitNs = 2000000000ull;

struct RunArgs {
  const unsigned char* block;
  const __nv_bfloat16* x[2];  // K, V
  unsigned char* cache;
  const int *page_table, *pos, *n_new, *index;
  const double* table;  // cobra_rope_table64, or null
  long long sl, ss, st, sh;
  int head0[2], layer_stride, n_layers, n_kv, n_seqs, max_new, n_src, rows_per_seq, pages_per_seq;
  int n_coarse;
};

struct RunSeg {
  int seq, row, t0, n, j0, v0;  // sequence, code row, first token in the row, tokens, first new token, first vector
};
template <class C>
struct RunSmem {
  static constexpr int kWarps = C::kThreads / 32, kGroups = C::kTokens / 32;
  // operands: [piece][dimensions 0 .. 63, 64 .. 127][channel or vector] 128-byte rows, swizzled
  unsigned char w[C::kPieces][2][kD * 128], x[C::kPieces][2][C::kTokens * 128];
  uint8_t codes[C::kTokens * kRunCodeLd];
  float wmu[kD], werr[kD];  // W^T mu; the projection's error over |x|
  float xnorm[C::kTokens];
  int pre[kRunSeqs + 1];  // rows of the block's sequences before each
  int pos[kRunSeqs], n[kRunSeqs];  // their runs
  int warp_sum[kWarps];
  RunSeg seg[kRunSegs];
  int n_seg, n_vec;
  long long vec_at[C::kTokens];                  // first element of each vector in x
  int vec_src[C::kTokens], vec_pos[C::kTokens];  // source token (-1: skipped) and position
  // per channel and 32 vectors, where the vectors lay: codes to be done again, and whose border was not above the
  // first result
  __device__ uint32_t* near() { return reinterpret_cast<uint32_t*>(x); }
  __device__ uint32_t* above() { return near() + kD * kGroups; }
  unsigned long long done;
  uint32_t tmem;
};

// Exclusive prefix sum over the CTA's threads; *total is the sum.
template <class C>
__device__ __forceinline__ int run_scan(RunSmem<C>& sm, int v, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, m);
    if (lane >= m) x += y;
  }
  if (lane == 31) sm.warp_sum[warp] = x;
  __syncthreads();
  int base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < RunSmem<C>::kWarps; ++w) {
    if (w < warp) base += sm.warp_sum[w];
    sum += sm.warp_sum[w];
  }
  __syncthreads();
  *total = sum;
  return base + x - v;
}

// A sequence's run: position and number of the tokens that fit the cache (what does not is reported).
__device__ __forceinline__ void run_of(const RunArgs& a, int s, bool report, int& pos, int& n) {
  const long long cap = min(0x7fffffffLL, 128LL * (a.page_table ? 2LL * a.pages_per_seq : (long long)a.rows_per_seq));
  pos = a.pos[s];
  n = a.n_new ? a.n_new[s] : a.max_new;
  bool bad = n < 0 || n > a.max_new;
  n = min(max(n, 0), a.max_new);
  if (n > 0 && (pos < 0 || pos + (long long)n > cap)) {
    bad = true;
    n = pos < 0 || pos >= cap ? 0 : (int)(cap - pos);
  }
  if (bad && report) atomicOr(&g_status, 2u);
}

// Cosine and sine of pos omega_j in fp64: table rows of 64 (cos, sin) pairs, fine then coarse.
__device__ __forceinline__ void run_angle(const RunArgs& a, int pos, int j, double& c, double& s) {
  const double2 f = reinterpret_cast<const double2*>(a.table)[(pos & 15) * (kD / 2) + j];
  const double2 m = reinterpret_cast<const double2*>(a.table)[(size_t)(kRopeFine + (pos >> 4)) * (kD / 2) + j];
  c = m.x * f.x - m.y * f.y;
  s = m.y * f.x + m.x * f.y;
}

// The nearest float of a cosine or sine (|x| <= 1; 0 below 2^-126), on its bits: conversions from fp64 run at its
// rate (128 vectors loaded, turned and split: 20000 cycles with them, 11000 without).
__device__ __forceinline__ float run_single(double x) {
  const unsigned long long bits = (unsigned long long)__double_as_longlong(x) + 0x10000000ull;  // half a unit in the last place
  const uint32_t hi = (uint32_t)(bits >> 32), h = __funnelshift_l((uint32_t)bits, hi, 3);
  // exponents 897 .. 1023 become 1 .. 127, as 896 is a multiple of 128
  return (hi & 0x7FF00000u) < (897u << 20) ? 0.f : __uint_as_float((h & 0x3FFFFFFFu) | (hi & 0x80000000u));
}

// y - W^T mu of one channel in fp64, by the warp: lane l has the dimension pairs l and l + 32.
__device__ __forceinline__ double run_exact(const RunArgs& a, const __nv_bfloat16* x, const float* w, const float* mu,
                                            bool turn, int pos) {
  const int lane = threadIdx.x & 31;
  double y = 0.0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int j = lane + 32 * u;
    double xa = (double)__bfloat162float(x[j]), xb = (double)__bfloat162float(x[j + 64]);
    if (turn) {
      double c, s;
      run_angle(a, pos, j, c, s);
      const double ya = xa * c - xb * s;
      xb = xa * s + xb * c;
      xa = ya;
    }
    y += (double)w[j] * (xa - (double)mu[j]) + (double)w[j + 64] * (xb - (double)mu[j + 64]);
  }
#pragma unroll
  for (int m = 16; m; m >>= 1) y += __shfl_xor_sync(0xffffffffu, y, m);
  return y;
}

// y - W^T mu - `border` of one channel in pairs of fp32 (each value a sum of two, products and sums with their
// rounding errors), by the warp, and a bound on its error: the pairs lose less than 2^-40 of the sum of
// magnitudes (roundings of the low parts, 2^-48 of a term each, some twenty deep), and angles composed in fp32
// turn x within 6 2^-24 of |xa| + |xb|.
__device__ __forceinline__ float run_close(const RunArgs& a, const __nv_bfloat16* x, const float* w, const float* mu,
                                           bool turn, int pos, float half_steps, float delta, float& bound) {
  const int lane = threadIdx.x & 31;
  float hi = 0.f, lo = 0.f, size = 0.f;
  auto add = [&](float p, float e) {  // (hi, lo) += p + e
    const float t = hi + p, q = t - hi;
    lo += (hi - (t - q)) + (p - q) + e;
    hi = t;
  };
  auto term = [&](float wd, float xh, float xl, float m) {  // wd (xh + xl - m)
    const float h = xh - m, q = h - xh, l = (xh - (h - q)) + (-m - q) + xl, p = wd * h;
    add(p, fmaf(wd, h, -p) + wd * l);
    size += fabsf(wd) * (fabsf(xh) + fabsf(m));
  };
  bound = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int j = lane + 32 * u;
    float xa = __bfloat162float(x[j]), xb = __bfloat162float(x[j + 64]), la = 0.f, lb = 0.f;
    if (turn) {
      const double2 f = reinterpret_cast<const double2*>(a.table)[(pos & 15) * (kD / 2) + j];
      const double2 m = reinterpret_cast<const double2*>(a.table)[(size_t)(kRopeFine + (pos >> 4)) * (kD / 2) + j];
      float c, s;
      rope_compose(run_single(m.x), run_single(m.y), run_single(f.x), run_single(f.y), c, s);
      bound += 3.6e-7f * (fabsf(w[j]) + fabsf(w[j + 64])) * (fabsf(xa) + fabsf(xb));
      const float p0 = xa * c, p1 = -xb * s, p2 = xa * s, p3 = xb * c;
      const float ya = p0 + p1, qa = ya - p0, yb = p2 + p3, qb = yb - p2;
      la = (p0 - (ya - qa)) + (p1 - qa) + fmaf(xa, c, -p0) + fmaf(-xb, s, -p1);
      lb = (p2 - (yb - qb)) + (p3 - qb) + fmaf(xa, s, -p2) + fmaf(xb, c, -p3);
      xa = ya, xb = yb;
    }
    term(w[j], xa, la, mu[j]);
    term(w[j + 64], xb, lb, mu[j + 64]);
  }
#pragma unroll
  for (int m = 16; m; m >>= 1) {
    const float h = __shfl_xor_sync(0xffffffffu, hi, m), l = __shfl_xor_sync(0xffffffffu, lo, m);
    add(h, l);
    size += __shfl_xor_sync(0xffffffffu, size, m);
    bound += __shfl_xor_sync(0xffffffffu, bound, m);
  }
  const float p = half_steps * delta;
  add(-p, -fmaf(half_steps, delta, -p));
  bound = 1.01f * bound + 9.1e-13f * (size + fabsf(p));  // 2^-40
  return hi + lo;
}

// The head's basis in pieces, W^T mu and the columns' errors, by all warps but the first.
template <class C>
__device__ __forceinline__ void run_basis(RunSmem<C>& sm, const float* pool, const HeadEntry& he, bool turn) {
  const int lane = threadIdx.x & 31, i = threadIdx.x - 32;
  if (i < he.r) sm.wmu[i] = pool[he.wmu_off + i];
  constexpr int kWarps = C::kThreads / 32 - 1, kRows = 9;  // rows in flight
  float4 w[kRows];
  for (int i0 = i >> 5; i0 < he.r; i0 += kRows * kWarps) {
    load_basis<kWarps>(w, pool + he.w_off, he.r, i0);
    lay_basis<C::kPieces, kWarps, true>(sm.w, w, he.r, i0, run_error<C>(turn), [&](int ch, float n2) {
      if (lane == 0) sm.werr[ch] = 3.8147e-6f * sqrtf(n2);
    });
  }
}

// The batch's vectors in pieces, turned to their positions, and their norms: a warp per vector, lane l has the
// dimensions 2 l, 2 l + 1 and the ones 64 behind; kVecs vectors are in flight per warp.
template <bool TURN, int kVecs, class C>
__device__ __forceinline__ void run_vectors(const RunArgs& a, RunSmem<C>& sm, const __nv_bfloat16* x, bool wide, int nv) {
  constexpr int kWarps = C::kThreads / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int v0 = warp; v0 < nv; v0 += kVecs * RunSmem<C>::kWarps) {
    uint32_t xa[kVecs], xb[kVecs];
    double2 fine[kVecs][2], coarse[kVecs][2];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int v = min(v0 + k * RunSmem<C>::kWarps, nv - 1);  // (the last one again where there are no more)
      load_pairs(x + sm.vec_at[v], wide, xa[k], xb[k]);
      if (TURN) {
        const int pos = sm.vec_pos[v];
        const double2* f = reinterpret_cast<const double2*>(a.table) + (pos & 15) * (kD / 2) + 2 * lane;
        const double2* m = reinterpret_cast<const double2*>(a.table) + (size_t)(kRopeFine + (pos >> 4)) * (kD / 2) + 2 * lane;
        fine[k][0] = f[0], fine[k][1] = f[1], coarse[k][0] = m[0], coarse[k][1] = m[1];
      }
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int v = min(v0 + k * RunSmem<C>::kWarps, nv - 1);
      float xs[4] = {__uint_as_float(xa[k] << 16), __uint_as_float(xa[k] & 0xFFFF0000u), __uint_as_float(xb[k] << 16),
                     __uint_as_float(xb[k] & 0xFFFF0000u)};
      const int at = pair_at(v);
      if (TURN) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float c, s;
          rope_compose(run_single(coarse[k][h].x), run_single(coarse[k][h].y), run_single(fine[k][h].x),
                       run_single(fine[k][h].y), c, s);
          const float p = xs[h], q = xs[h + 2];
          xs[h] = fmaf(p, c, -q * s);
          xs[h + 2] = fmaf(p, s, q * c);
        }
        uint32_t p[C::kPieces], q[C::kPieces];
        split_pieces(xs[0], xs[1], p);
        split_pieces(xs[2], xs[3], q);
#pragma unroll
        for (int n = 0; n < C::kPieces; ++n) {
          *reinterpret_cast<uint32_t*>(sm.x[n][0] + at) = p[n];
          *reinterpret_cast<uint32_t*>(sm.x[n][1] + at) = q[n];
        }
      } else {
        *reinterpret_cast<uint32_t*>(sm.x[0][0] + at) = xa[k];
        *reinterpret_cast<uint32_t*>(sm.x[0][1] + at) = xb[k];
      }
      float n2 = xs[0] * xs[0] + xs[1] * xs[1] + xs[2] * xs[2] + xs[3] * xs[3];
#pragma unroll
      for (int m = 16; m; m >>= 1) n2 += __shfl_xor_sync(0xffffffffu, n2, m);
      if (lane == 0) sm.xnorm[v] = sqrtf(n2);
    }
  }
}

// The batch's nv vectors to codes; false: a wait has expired.
template <class C>
__device__ __forceinline__ bool run_codes(const RunArgs& a, RunSmem<C>& sm, uint32_t tmem, uint32_t phase, const HeadEntry& he,
                                          const __nv_bfloat16* x, const float* W, const float* mu, bool turn, bool wide,
                                          int nv) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = he.r, b = he.b;
  constexpr int kWarps = C::kThreads / 32, kGroups = C::kTokens / 32, kPieces = C::kPieces;
  if (nv <= kWarps)
    turn ? run_vectors<true, 1>(a, sm, x, wide, nv) : run_vectors<false, 1>(a, sm, x, wide, nv);
  else
    turn ? run_vectors<true, 2>(a, sm, x, wide, nv) : run_vectors<false, 4>(a, sm, x, wide, nv);
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    // kind::f16, bf16 A and B, fp32 D, M = 128, N = vectors (those behind the last hold anything)
    const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(2 * ((nv + 15) >> 4)) << 17) | (8u << 24);
    const uint64_t wd = umma_desc_sw128(smem_addr(sm.w)), xd = umma_desc_sw128(smem_addr(sm.x));
    if (elect_one()) {
      bool more = false;
#pragma unroll
      for (int t = 0; t < 6; ++t) {
        constexpr int kW[6] = {2, 1, 0, 1, 0, 0}, kX[6] = {0, 1, 2, 0, 1, 0};
        if (kW[t] + kX[t] >= kPieces || (kX[t] > 0 && !turn)) continue;
#pragma unroll
        for (int kt = 0; kt < 8; ++kt) {
          const uint64_t at = (kt & 3) * 2;
          tc_mma_bf16_ss(tmem, wd + (uint64_t)((2 * kW[t] + (kt >> 2)) * (kD * 128) >> 4) + at,
                         xd + (uint64_t)((2 * kX[t] + (kt >> 2)) * (C::kTokens * 128) >> 4) + at, idesc, more);
          more = true;
        }
      }
      tc_commit(smem_addr(&sm.done));
    }
    __syncwarp();
  }
  const bool ok = mbar_wait_bounded(smem_addr(&sm.done), phase, kRunWaitNs);
  if (__syncthreads_or(!ok)) return false;
  tc_fence_after();
  // u = y / Delta + 2^{b-1} adds two roundings of a value below 2^{b+1} to the error
  const float half = (float)(1 << (b - 1)), inv_delta = he.inv_delta, top = (float)((1 << b) - 1);
  auto slack = [&](int ch) { return inv_delta * sm.werr[ch]; };
  auto least = [&](int ch) { return 2.4e-7f * inv_delta * fabsf(sm.wmu[ch]) + 4.8e-7f * (top + 1.f); };
  const int blocks = (r + 31) / 32, block = warp & 3, v0 = 32 * (warp >> 2), i = 32 * block + lane;
  if (block < blocks && v0 < nv) {  // the lane's channel, 32 vectors
    const int ch = min(i, r - 1);
    const float wmu = sm.wmu[ch], sl = slack(ch), le = least(ch);
    uint32_t y[32], near = 0u, above = 0u;
    tc_ld32(tmem + ((uint32_t)(32 * block) << 16) + v0, y);
    float xn[32];
#pragma unroll
    for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(xn + j) = *reinterpret_cast<const float4*>(sm.xnorm + v0 + j);
    tc_wait_ld(y);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float u = fmaf(__uint_as_float(y[j]) - wmu, inv_delta, half), tol = fmaf(sl, xn[j], le);
      const float e = rintf(u);  // borders that tell codes apart: 1 .. 2^b - 1
      // (as negations: a NaN, which pieces of an infinity give, is left to the exact sum)
      if (!(fabsf(u - e) > tol) && !(u <= 0.5f - tol) && !(u >= top + 0.5f + tol)) near |= 1u << j;
      if (u >= e) above |= 1u << j;
      y[j] = (uint32_t)fminf(fmaxf(u, 0.f), top);
    }
    if (i < r) {
#pragma unroll
      for (int j = 0; j < 32; ++j) sm.codes[(v0 + j) * kRunCodeLd + i] = (uint8_t)y[j];
      sm.near()[kGroups * i + (v0 >> 5)] = nv - v0 < 32 ? near & ((1u << (nv - v0)) - 1u) : near;
      sm.above()[kGroups * i + (v0 >> 5)] = above;
    }
  }
  tc_fence_before();
  __syncthreads();
  // lane l of warp w looks for codes to be done again in word w + kWarps l
  const int groups = (nv + 31) >> 5, word = warp + kWarps * lane;
  const uint32_t mine = word / kGroups < r && word % kGroups < groups ? sm.near()[word] : 0u;
  for (unsigned some = __ballot_sync(0xffffffffu, mine != 0u); some; some &= some - 1) {
    const int from = __ffs(some) - 1, k = warp + kWarps * from, ch = k / kGroups;
    for (unsigned todo = __shfl_sync(0xffffffffu, mine, from); todo; todo &= todo - 1) {
      const int bit = __ffs(todo) - 1, v = 32 * (k % kGroups) + bit;
      uint8_t& slot = sm.codes[v * kRunCodeLd + ch];
      const __nv_bfloat16* xv = x + sm.vec_at[v];
      const float e = (float)slot + ((sm.above()[k] >> bit) & 1u ? 0.f : 1.f);  // the border in question
      float bound;
      const float past = run_close(a, xv, W + ch * kD, mu, turn, sm.vec_pos[v], e - half, he.delta, bound);
      float code = fminf(fmaxf(past > 0.f ? e : e - 1.f, 0.f), top);
      // (a first error of half a cell or more may have missed the border)
      const bool told = fmaf(slack(ch), sm.xnorm[v], least(ch)) < 0.4f && fabsf(past) > bound;
      if (!__shfl_sync(0xffffffffu, told, 0)) {
        const double y = run_exact(a, xv, W + ch * kD, mu, turn, sm.vec_pos[v]);
        code = (float)fmin(fmax(floor(y / (double)he.delta + (double)half), 0.0), (double)top);
      }
      __syncwarp();  // (all lanes have read the slot)
      if (lane == 0) slot = (uint8_t)code;
    }
  }
  __syncthreads();
  return true;
}

// The touched words of the batch's rows: codes in, the other tokens' bits as they are.  A warp (or 2 to 16 of
// them, where rows are few) takes a row, a thread a piece of every few strips: which words, bits and tokens it
// touches there is the same for all of them.  It asks for the first and last touched word of kStrips strips, the only
// ones that other tokens share, and then builds the words in one walk over the tokens.
template <int SIDE, int kStrips, class C>
__device__ __forceinline__ void run_write(const RunArgs& a, RunSmem<C>& sm, const HeadEntry& he) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int strips = he.r >> 1, b = he.b, n_seg = sm.n_seg;
  const uint32_t rb = 16u * he.r * b, ones = (1u << b) - 1u;
  constexpr int kWarps = C::kThreads / 32;
  int ways = kWarps;
  while (ways > 1 && ways * n_seg > kWarps) ways >>= 1;
  for (int k = warp / ways; k < n_seg; k += kWarps / ways) {
    const RunSeg g = sm.seg[k];
    const int t1 = g.t0 + g.n - 1;
    // pieces of a strip that hold any of the tokens: K piece t % 8; V pieces (t / 2) % 4 (+ 4: odd channel)
    const int p0 = SIDE == 0 ? g.t0 & 7 : (g.t0 >> 1) & 3;
    const int np = SIDE == 0 ? min(g.n, 8) : min((t1 >> 1) - (g.t0 >> 1) + 1, 4);
    const int lp = np > 4 ? 3 : np > 2 ? 2 : np - 1;  // 2^lp >= np
    const int item = lane + 32 * (warp % ways), step = (32 * ways) >> (lp + SIDE);
    const int q = item & ((1 << lp) - 1), odd = SIDE & (item >> lp);
    if (q >= np) continue;
    const int p = SIDE == 0 ? (p0 + q) & 7 : (p0 + q) & 3;
    // the piece's tokens in the run: ta + 8 rho (V: and the one after), rho in [ra, rz], words [wa, wz]
    const int ta = SIDE == 0 ? p : 2 * p, ra = (g.t0 - ta - SIDE + 7) >> 3, rz = (t1 - ta) >> 3;
    const int wa = (ra * b) >> 4, wz = (rz * b + b - 1) >> 4;
    uint32_t* const piece = reinterpret_cast<uint32_t*>(a.cache + row_offset(he.cache_off, rb, g.seq, g.row, a.page_table,
                                                                             a.pages_per_seq, a.rows_per_seq)) +
                            (p + 4 * odd) * b;
    for (int s0 = item >> (lp + SIDE); s0 < strips; s0 += kStrips * step) {
      uint32_t old_a[kStrips], old_z[kStrips], bits[kStrips], mask = 0u;
      const uint8_t* codes[kStrips];
#pragma unroll
      for (int u = 0; u < kStrips; ++u) {
        const int s = min(s0 + u * step, strips - 1);  // (one behind the last is not written)
        old_a[u] = piece[s * 8 * b + wa];
        old_z[u] = piece[s * 8 * b + wz];
        bits[u] = 0u;
        codes[u] = sm.codes + 2 * s + odd;
      }
      int w = wa;
      auto flush = [&] {
        if (!mask) return;
#pragma unroll
        for (int u = 0; u < kStrips; ++u)
          if (s0 + u * step < strips) {
            uint32_t* const at = piece + (s0 + u * step) * 8 * b + w;
            *at = mask == 0xFFFFFFFFu ? bits[u] : ((w == wa ? old_a[u] : w == wz ? old_z[u] : *at) & ~mask) | bits[u];
          }
      };
      for (int rho = ra; rho <= rz; ++rho) {
        const int v = g.v0 + 8 * rho + ta - g.t0, v1 = min(v + 1, C::kTokens - 1), vc = max(v, 0);
        uint32_t live;  // of the two codes of a rho: channels 2 s and 2 s + 1 of a token; two tokens of a channel
        if (SIDE == 0)
          live = sm.vec_src[v] >= 0 ? 0x00010001u : 0u;
        else
          live = (8 * rho + ta >= g.t0 && sm.vec_src[vc] >= 0 ? 1u : 0u) |
                 (8 * rho + ta < t1 && sm.vec_src[v1] >= 0 ? 0x00010000u : 0u);
        // a code may end in the word behind: its upper off + b - 16 bits
        const int off = rho * b - 16 * w, more = max(off + b - 16, 0);
        const uint32_t in = live * ((ones << off) & 0xFFFFu), out = live * ((1u << more) - 1u);
        mask |= in;
        uint32_t two[kStrips];
#pragma unroll
        for (int u = 0; u < kStrips; ++u) {
          if (SIDE == 0) {
            const uint32_t c = *reinterpret_cast<const uint16_t*>(codes[u] + v * kRunCodeLd);
            two[u] = __byte_perm(c, 0u, 0x4140);
          } else {
            two[u] = codes[u][vc * kRunCodeLd] | (uint32_t)codes[u][v1 * kRunCodeLd] << 16;
          }
          // (off > 8 where a code goes on, so what it loses falls outside of the other one's bits)
          bits[u] |= (two[u] << off) & in;
        }
        if (off + b >= 16) {
          flush();
          ++w;
          mask = out;
#pragma unroll
          for (int u = 0; u < kStrips; ++u) bits[u] = (two[u] >> (16 - off)) & out;
        }
      }
      flush();
    }
  }
}

// grid: at most C::kPerSm CTAs per SM; CTA c has the c-th share of all (side, layer, kv head) x code rows
template <class C>
__global__ void __launch_bounds__(C::kThreads, C::kPerSm) append_run_kernel(RunArgs a) {
  constexpr int kWarps = C::kThreads / 32;
  extern __shared__ unsigned char run_raw[];
  const uint32_t raw = smem_addr(run_raw);
  RunSmem<C>& sm = *reinterpret_cast<RunSmem<C>*>(run_raw + (((raw + 1023u) & ~1023u) - raw));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dep_launch();
  const int n_heads = reinterpret_cast<const BlockHeader*>(a.block)->n_heads;
  const float* pool = param_pool(a.block);
  if (tid == 0) {
    mbar_init(smem_addr(&sm.done), 1);
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc(smem_addr(&sm.tmem), C::kTokens);
  const int heads = a.n_layers * a.n_kv;
  auto entry = [&](int hs, HeadEntry& he) {  // false: the block does not hold the head
    const int side = hs >= heads, head = hs - side * heads;
    const int h = a.head0[side] + head / a.n_kv * a.layer_stride + head % a.n_kv;
    if (h >= n_heads) return false;
    he = head_table(a.block)[h];
    return true;
  };
  // the share's first head does not depend on the number of rows: floor(floor(H rows c / C) / rows) = floor(H c / C)
  const int hs0 = (int)(2LL * heads * blockIdx.x / gridDim.x);
  HeadEntry he = {};
  bool known = entry(hs0, he);
  if (warp > 0 && he.r > 0) run_basis(sm, pool, he, hs0 < heads && a.table);
  // the tokens, positions and the cache may be produced or read by the kernels ahead
  grid_dep_wait();
  int held = 0, sum = 0;  // the block of sequences that lies in shared memory, its code rows
  auto count = [&](int s0, bool report) {
    int pos = 0, n = 0;
    if (tid < kRunSeqs && s0 + tid < a.n_seqs) run_of(a, s0 + tid, report, pos, n);
    const int before = run_scan(sm, n > 0 ? ((pos + n - 1) >> 7) - (pos >> 7) + 1 : 0, &sum);
    if (tid < kRunSeqs) {
      sm.pre[tid] = before;
      sm.pos[tid] = pos;
      sm.n[tid] = n;
    }
    if (tid == 0) sm.pre[kRunSeqs] = sum;
    held = s0;
  };
  int total = 0;  // the call's code rows
  for (int s0 = 0; s0 < a.n_seqs; s0 += kRunSeqs) {
    count(s0, blockIdx.x == 0);
    total += sum;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  uint32_t phase = 0;
  bool ok = true;
  const long long units = 2LL * heads * total;
  const long long lo = units * blockIdx.x / gridDim.x, hi = units * (blockIdx.x + 1) / gridDim.x;
  for (int hs = lo < hi ? hs0 : 2 * heads; ok && hs < 2 * heads && (long long)hs * total < hi; ++hs) {
    bool fresh = hs > hs0;  // the basis is not laid out yet
    if (fresh) known = entry(hs, he);
    if (!known) {
      if (tid == 0) atomicOr(&g_status, 2u);
      continue;
    }
    if (he.r == 0) continue;
    const int side = hs >= heads, head = hs - side * heads, layer = head / a.n_kv, kv = head % a.n_kv;
    const float *mu = pool + he.mu_off, *W = pool + he.w_off;
    const __nv_bfloat16* x = a.x[side] + layer * a.sl + kv * a.sh;
    const bool turn = side == 0 && a.table != nullptr;
    const bool wide = ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(2 * a.ss) | (uintptr_t)(2 * a.st)) & 3) == 0;
    const int first = (int)max(lo - (long long)hs * total, 0LL), last = (int)min(hi - (long long)hs * total, (long long)total);
    HeadEntry next;  // the next head's basis is wanted soon
    if ((long long)(hs + 1) * total < hi && entry(hs + 1, next) && tid < 4 * next.r) prefetch_l2(pool + next.w_off + 32 * tid);
    int base = 0;  // rows before the block of sequences
    for (int s0 = 0; ok && s0 < a.n_seqs && base < last; s0 += kRunSeqs) {
      if (held != s0) {
        count(s0, false);
        __syncthreads();
      }
      const int g1 = min(last - base, sum);
      for (int g = max(first - base, 0); g < g1;) {
        // warp 0: the rows g, g + 1, ... that make up to C::kTokens tokens
        if (tid < 32) {
          RunSeg sg = {};
          if (g + lane < g1) {
            int lo = 0, hi = kRunSeqs;  // the last sequence whose rows begin at or before this one
            while (hi - lo > 1) {
              const int mid = (lo + hi) >> 1;
              if (sm.pre[mid] <= g + lane) lo = mid; else hi = mid;
            }
            const int pos = sm.pos[lo], n = sm.n[lo];
            const int k = g + lane - sm.pre[lo], row = (pos >> 7) + k;
            const int begin = max(pos, row << 7), end = min(pos + n, (row + 1) << 7);
            sg = RunSeg{s0 + lo, row, begin & 127, end - begin, begin - pos, 0};
          }
          int sum_n = sg.n;
#pragma unroll
          for (int m = 1; m < 32; m <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum_n, m);
            if (lane >= m) sum_n += y;
          }
          sg.v0 = sum_n - sg.n;
          const bool in = sg.n > 0 && sum_n <= C::kTokens;
          const unsigned taken = __ballot_sync(0xffffffffu, in);
          if (in) sm.seg[lane] = sg;
          if (lane == __popc(taken) - 1) sm.n_vec = sum_n;
          if (lane == 0) sm.n_seg = __popc(taken);
        } else if (fresh) {
          run_basis(sm, pool, he, turn);
        }
        fresh = false;
        __syncthreads();
        const int n_seg = sm.n_seg, nv = sm.n_vec;
        // the rows' bytes are wanted at the batch's end
        for (int k = warp; k < n_seg; k += kWarps) {
          const uint32_t rb = 16u * he.r * he.b;
          const unsigned char* row = a.cache + row_offset(he.cache_off, rb, sm.seg[k].seq, sm.seg[k].row, a.page_table,
                                                          a.pages_per_seq, a.rows_per_seq);
          for (uint32_t o = 128u * lane; o < rb; o += 4096u) prefetch_l2(row + o);
        }
        if (tid < nv) {
          int k = 0;  // the last row whose vectors begin at or before this one
#pragma unroll
          for (int step = kRunSegs / 2; step; step >>= 1)
            if (k + step < n_seg && sm.seg[k + step].v0 <= tid) k += step;
          const RunSeg& sg = sm.seg[k];
          const int j = sg.j0 + tid - sg.v0;
          int src = a.index ? a.index[(long long)sg.seq * a.max_new + j] : j;
          if (src < 0 || src >= a.n_src) {
            src = -1;
            atomicOr(&g_status, 2u);
          }
          int p = 128 * sg.row + sg.t0 + tid - sg.v0;
          if (turn && p >= kRopeFine * a.n_coarse) {  // past the table: reported, the last angles are used
            atomicOr(&g_status, 2u);
            p = kRopeFine * a.n_coarse - 1;
          }
          sm.vec_at[tid] = sg.seq * a.ss + (long long)max(src, 0) * a.st;
          sm.vec_src[tid] = src;
          sm.vec_pos[tid] = p;
        }
        __syncthreads();
        ok = run_codes(a, sm, tmem, phase, he, x, W, mu, turn, wide, nv);
        if (!ok) break;
        phase ^= 1u;
        // with up to two rows there are as many threads as pieces
        if (side == 0)
          n_seg > 2 ? run_write<0, 4>(a, sm, he) : run_write<0, 1>(a, sm, he);
        else
          n_seg > 2 ? run_write<1, 4>(a, sm, he) : run_write<1, 1>(a, sm, he);
        __syncthreads();
        g += n_seg;
      }
      base += sum;
      __syncthreads();  // the prefix sums are rewritten by the next block of sequences
    }
  }
  if (!ok && tid == 0) {  // products in flight are given time to end
    atomicOr(&g_status, 1u);
    mbar_wait_bounded(smem_addr(&sm.done), phase, 1000000ull);
  }
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, C::kTokens);
}

// fp64 angle table: row x < 16 holds position x, row 16 + m position 16 m, 64 (cos, sin) pairs each.
__global__ void rope_table64_kernel(double* table, int n_rows, double theta) {
  grid_dep_wait();  // an earlier append may still read the table being overwritten
  grid_dep_launch();
  const int idx = blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= n_rows * (kD / 2)) return;
  const int x = idx / (kD / 2), j = idx % (kD / 2);
  const double pos = x < kRopeFine ? (double)x : 16.0 * (double)(x - kRopeFine);
  double s, c;
  sincos(pos * pow(theta, -2.0 * (double)j / (double)kD), &s, &c);
  reinterpret_cast<double2*>(table)[idx] = make_double2(c, s);
}

}  // namespace cobra
