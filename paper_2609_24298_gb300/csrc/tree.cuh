// Attention of a tree of drafted tokens over the packed cache (Table alg:kvrobin step 8 for several query
// tokens per sequence), with optional score caps, distance biases and sliding windows.
//
// Sequence s has n <= max_draft drafted tokens; token i and query head g of a kv head make column
// c = i G + g of that head.  In log2 units,
//   cached token t   z = q~_c . (c^K_t - 2^{b-1} + 1/2) + c0_c,  q~ = (Delta_K log2e / sqrt d) W_K^T q,
//                    c0 = (log2e / sqrt d) q . mu_K
//   drafted token j  z = (log2e / sqrt d) q . k_j, for the bits j of the token's mask row
//   cap              z <- cap2 tanh(z / cap2)
//   bias             z <- z + slope2_g (t - p_i)
//   seen             p_i - window < t <= p_i, and t below the sequence's length
// and o_c = sum_t 2^z_t V_t / sum_t 2^z_t, the cached values accumulated in rank space (deviations from
// the code centre) and mapped back once.  A column that sees nothing gives zeros; one whose scores are not finite
// (a query, drafted key or slope with a NaN or an infinity, or beyond fp32) gives NaN, as the definition does.
//
//   tree_prepare_kernel  per (head, sequence, 32 columns) q~ as f16 with a power-of-two scale, c0, and
//                        the drafted tokens' own softmax partial; one CTA lays out the scan's work
//   tree_scan_kernel     the packed rows, split evenly over the CTAs
//   tree_combine_kernel  the parts of each column together, back-projection, bf16 out
//
// Work split.  The rows of all (head, sequence, column tile) units lie on a line in this order, each row
// as long as its head's cost; CTA c of C takes the rows that begin in [c, c + 1) / C of it.  A unit's
// rows are then shared by consecutive CTAs, and the part of CTA c in unit u goes to slot c + u (both
// grow along the line, so no two parts meet): nothing is counted or reset between launches.
#pragma once

#include <type_traits>

#include "pieces.cuh"
#include "tc.cuh"
#include "unpack_tc.cuh"

namespace cobra {

constexpr int kTreeMaxDraft = 64;
constexpr uint64_t kTreeWaitNs = 2000000000ull;  // 2 s
constexpr int kTreeChunk = 32;    // columns of a prepare unit
constexpr int kTreePart = kD + 4;  // floats of a column's partial: m, l, -, -, O[128]
constexpr float kTreeCapPlain = 512.f;  // caps up to here (log2 units, 355 of a score) take the formula alone: see tree_cap
constexpr float kTreeLargest = 1e38f;   // magnitude of a score that fp32 holds with its parts
constexpr float kTreeLowest = -3e38f;   // stands for a drafted score of -inf: below every other, but seen
constexpr float kTreeBound = 80.f;  // scores this near their reference need no running maximum: 2^80 times codes of 2^7, summed over 2^31 tokens, is finite
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInvSqrtD = 0.088388347648318440f;

struct TreeCol {     // what the scan knows of a column
  float c0, slope2;
  int pos;
  float scale;       // 2^-e, if 2^e scales the column's q~
  int lo, hi;        // cached tokens [lo, hi) that it sees
  int bounded;       // 1: scores of the chunk's columns, less their biases, are within kTreeBound of c0 (0 with a cap);
                     // -1: not so, and some of its columns are scaled
  int bad;           // scores that are not finite: the scan has zeros for the column, the combine makes it NaN
};
static_assert(sizeof(TreeCol) == 32, "copied as 16-byte units");

struct TreeArgs {
  const unsigned char* block;
  const unsigned char* cache;
  const int *page_table, *seq_lens, *n_draft, *q_pos;
  const unsigned long long* mask;
  const float* slopes;
  const __nv_bfloat16 *q, *kd, *vd;
  __nv_bfloat16* out;
  long long q_sl, q_ss, q_st, d_sl, d_ss, d_st, d_sh, o_sl, o_ss, o_st;
  int k_head0, v_head0, layer_stride, n_layers, n_kv, group, n_seqs, max_draft;
  int rows_per_seq, pages_per_seq, window;
  float cap2;          // cap in log2 units, 0: none
  int nc, tiles, chunks;  // columns per tile, tiles and 32-column chunks per (head, sequence)
  int ctas;            // scan CTAs
  uint32_t top_f16, top_bf16;  // kTopF16, kTopBf16 (see Bases)
  // workspace
  int *row0, *rows, *live;        // [n_seqs] first row seen, rows seen, column tiles in use
  int* row_bytes;                 // [2] the largest K and V code row of the call's heads
  int* start;                     // [ctas][2] head and sequence at the beginning of each CTA's stretch
  long long *rpre, *wpre;         // prefix sums: rows x tiles of the sequences, costs of the heads
  unsigned char* img;             // [unit][2 nc 128 bytes] f16 q~ (tree_img_at)
  TreeCol* col;                   // [unit][nc]
  float *draft, *part;            // [head][seq][columns][kTreePart], [slot][nc][kTreePart]
};

// ---------------------------------------------------------------------------------------
// The work line
// ---------------------------------------------------------------------------------------
// x / d for x >= 0, d > 0: most quotients here are of 32-bit numbers, and a 64-bit division is a hundred instructions
__device__ __forceinline__ long long tree_div(long long x, long long d) {
  return ((x | d) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)d) : x / d;
}
struct TreeLine {
  long long rows, total;  // row-tiles of all sequences, length of the line
  long long share;        // total / ctas
  int ctas, rest;         // total % ctas
  __device__ TreeLine(const TreeArgs& a) : rows(a.rpre[a.n_seqs]), ctas(a.ctas) {
    total = a.wpre[a.n_layers * a.n_kv] * rows;
    share = tree_div(total, ctas);
    rest = (int)(total - share * ctas);
  }
  __device__ long long begin(int c) const {  // floor(total c / ctas)
    return share * c + (uint32_t)(rest * c) / (uint32_t)ctas;
  }
  // rows of a unit at `base` with n rows of cost w that begin before x
  __device__ static int before(long long x, long long base, int n, int w) {
    const long long d = x - base;
    return d <= 0 ? 0 : d > (n - 1LL) * w ? n : (int)tree_div(d + w - 1, w);
  }
};
// The index i in [0, n) with pre[i] <= x < pre[i + 1], and both, by a converged warp: 32 entries at a time.
struct TreeFound {
  int i;
  long long lo, hi;
};
__device__ __forceinline__ TreeFound tree_find(const long long* pre, int n, long long x) {
  const int lane = threadIdx.x & 31;
  int base = 0;
  while (n > 32) {
    const int step = (n + 31) / 32, at = min((lane + 1) * step, n);
    const int k = __popc(__ballot_sync(0xffffffffu, pre[base + at] <= x && (lane + 1) * step < n));
    base += k * step;
    n = min(step, n - k * step);
  }
  const long long lo = pre[base + min(lane, n - 1)], hi = pre[base + min(lane, n - 1) + 1];
  const int k = __popc(__ballot_sync(0xffffffffu, lane < n - 1 && hi <= x));
  return TreeFound{base + k, __shfl_sync(0xffffffffu, lo, k), __shfl_sync(0xffffffffu, hi, k)};
}
// a head's parameters; a head that the block does not hold is reported and stands for one without codes
__device__ __forceinline__ HeadEntry tree_head(const TreeArgs& a, int head0, int head, bool& known) {
  const int h = head0 + head / a.n_kv * a.layer_stride + head % a.n_kv;
  known = h < reinterpret_cast<const BlockHeader*>(a.block)->n_heads;
  HeadEntry e = head_table(a.block)[known ? h : 0];
  if (!known) e.r = 0;
  return e;
}
// cached tokens of a sequence: its length within the cache
__device__ __forceinline__ int tree_len(const TreeArgs& a, int s, bool report) {
  const long long cap = 128LL * (a.page_table ? 2LL * a.pages_per_seq : (long long)a.rows_per_seq);
  const int T = a.seq_lens[s];
  if (report && (T < 0 || T > cap)) atomicOr(&g_status, 2u);
  return T < 0 ? 0 : T > cap ? (int)cap : T;
}
__device__ __forceinline__ int tree_drafts(const TreeArgs& a, int s, bool report) {
  const int n = a.n_draft ? a.n_draft[s] : a.max_draft;
  if (report && (n < 0 || n > a.max_draft)) atomicOr(&g_status, 2u);
  return min(max(n, 0), a.max_draft);
}
__device__ __forceinline__ int tree_pos(const TreeArgs& a, int s, int i, int T) {
  return a.q_pos ? a.q_pos[(long long)s * a.max_draft + i] : T + i;
}
// cached tokens [x, y) that a query at position p of a sequence of T tokens sees
__device__ __forceinline__ int2 tree_seen(const TreeArgs& a, long long p, int T) {
  const long long x = a.window > 0 ? max(0LL, p - a.window + 1) : 0LL, y = min((long long)T, p + 1);
  return x < y ? make_int2((int)x, (int)y) : make_int2(0, 0);
}
// byte of place p of a column in a unit's image of q~: rows of 64 places, 128-byte swizzle; a tile's 16
// channels are in the order of the unpacked codes (tc_k_channel)
__device__ __forceinline__ int tree_img_at(int nc, int col, int p) {
  return (p >> 6) * nc * 128 + col * 128 + ((((p & 63) >> 3) ^ (col & 7)) << 4) + (p & 7) * 2;
}
// z with the cap: cap2 tanh(z / cap2) = cap2 (1 - 2 / (1 + e^{2 z / cap2})).  The difference loses relative, not
// absolute accuracy near 0: the score is within 2^-20 cap2, for caps up to kTreeCapPlain 2^-11 of a log2 unit.
__device__ __forceinline__ float tree_cap(float z, float cap2, float k) {  // cap2 <= kTreeCapPlain, k = tree_cap_k
  return cap2 - __fdividef(2.f * cap2, 1.f + ex2_approx(z * k));
}
__device__ __forceinline__ float tree_cap_k(float cap2) {  // 2 log2e / cap2, finite (0 times it has to be 0)
  return cap2 > 0.f ? fminf(__fdiv_rn(2.f * kLog2e, cap2), 3e38f) : 0.f;
}
// The same for larger caps (with one of 1e5 the above would be off by 0.1): below 0.3 cap2 the series of tanh to x^9, whose
// rest is below 2^-24 of it, so that the result is within 2^-19 of itself.
__device__ __forceinline__ float tree_cap_large(float z, float cap2, float k) {
  const float x = z * k * (0.5f / kLog2e), x2 = x * x;
  const float series = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  return fabsf(x) < 0.3f ? z * series : tree_cap(z, cap2, k);
}

// ---------------------------------------------------------------------------------------
// Prepare
// ---------------------------------------------------------------------------------------
struct TreeDraftSmem {
  float q[kTreeChunk][kD + 4];
  float kv[kTreeMaxDraft][kD + 4];
  float z[kTreeChunk][kTreeMaxDraft + 1];
  float p[kTreeMaxDraft][kTreeChunk + 4];  // probabilities, [drafted token][column]
  int pos[kTreeMaxDraft];                  // of the drafted tokens,
  unsigned long long mask[kTreeMaxDraft];  // and what each sees of them
};

// prefix sum over the CTA's 256 threads
__device__ __forceinline__ long long tree_scan(long long* sums, long long v, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, m);
    if (lane >= m) x += y;
  }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  long long base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    if (w < warp) base += sums[w];
    sum += sums[w];
  }
  __syncthreads();
  *total = sum;
  return base + x - v;
}

// The scan's work: rows and tiles per sequence, costs per head.
__device__ __forceinline__ void tree_layout(const TreeArgs& a, long long* sums) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  for (int s = warp; s < a.n_seqs; s += 8) {
    const int T = tree_len(a, s, lane == 0), n = tree_drafts(a, s, lane == 0);
    int lo = 0x7fffffff, hi = 0;
    for (int i = lane; i < n; i += 32) {
      const int2 seen = tree_seen(a, tree_pos(a, s, i, T), T);
      if (seen.y > 0) {
        lo = min(lo, seen.x);
        hi = max(hi, seen.y);
      }
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) {
      lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, m));
      hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    if (lane == 0) {
      const int row0 = hi > 0 ? lo >> 7 : 0;
      a.row0[s] = row0;
      a.rows[s] = ((hi + 127) >> 7) - row0;
      a.live[s] = (n * a.group + a.nc - 1) / a.nc;
    }
  }
  __syncthreads();
  long long base = 0, sum;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 256) {
    const int s = s0 + tid;
    const long long v = s < a.n_seqs ? (long long)a.rows[s] * a.live[s] : 0;
    const long long x = tree_scan(sums, v, &sum);
    if (s < a.n_seqs) a.rpre[s] = base + x;
    base += sum;
  }
  if (tid == 0) a.rpre[a.n_seqs] = base;
  base = 0;
  const int heads = a.n_layers * a.n_kv;
  __shared__ int row_bytes[2];
  if (tid < 2) row_bytes[tid] = 0;
  __syncthreads();
  for (int h0 = 0; h0 < heads; h0 += 256) {
    const int h = h0 + tid;
    long long v = 0;
    if (h < heads) {
      bool kk, kv;
      const HeadEntry ek = tree_head(a, a.k_head0, h, kk), ev = tree_head(a, a.v_head0, h, kv);
      if (!kk || !kv) atomicOr(&g_status, 2u);
      v = 512 + ek.r + ev.r;
      atomicMax(row_bytes, 16 * ek.r * ek.b);
      atomicMax(row_bytes + 1, 16 * ev.r * ev.b);
    }
    const long long x = tree_scan(sums, v, &sum);
    if (h < heads) a.wpre[h] = base + x;
    base += sum;
  }
  if (tid == 0) a.wpre[heads] = base;
  if (tid < 2) a.row_bytes[tid] = row_bytes[tid];
  __syncthreads();
  // where the CTAs' stretches begin: the scan need not search for it while nothing else runs (four round trips)
  const TreeLine line(a);
  if (line.total == 0) return;
  auto find = [](const long long* pre, int n, long long x) {  // the last i with pre[i] <= x
    int lo = 0;
    for (int hi = n; hi - lo > 1;) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
  };
  for (int c = tid; c < a.ctas; c += 256) {
    const long long x = line.begin(c);
    const int h = find(a.wpre, heads, tree_div(x, line.rows));
    const long long w0 = a.wpre[h];
    a.start[2 * c] = h;
    a.start[2 * c + 1] = find(a.rpre, a.n_seqs, tree_div(x - w0 * line.rows, a.wpre[h + 1] - w0));
  }
}

constexpr int kTreeProjLd = kD + 4;
struct TreeProjSmem {
  unsigned char w[2][2][kD * 128], x[2][kTreeChunk * 128];  // operands on 1024-byte boundaries
  float os[kTreeChunk][kTreeProjLd];
  float dot[kTreeChunk], red[2][8];
  int bad[kTreeChunk], exp[kTreeChunk];  // not finite; exponent of the scale
  unsigned long long done;
  uint32_t tmem;
};

// q~ and c0 of 32 columns.  The projection is a product of bf16 queries with the basis in two bf16 pieces, summed
// in fp32: 2^-17 |w| |q| off by the pieces and half as much by the sums (append_run.cuh), below the 2^-11 of an element
// that f16 takes.  (In fp32 on the CUDA cores, bound by shared-memory reads, the product alone took 4.3 us.)
__device__ __forceinline__ void tree_project(const TreeArgs& a, TreeProjSmem& sm, int head, int s, int chunk) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  bool known;
  // ahead of the parameters too: the kernel ahead may write them, and asking for them earlier gained nothing (the
  // smallest call takes 22.4 us either way)
  grid_dep_wait();
  const HeadEntry he = tree_head(a, a.k_head0, head, known);
  const float* pool = param_pool(a.block);
  const float* mu = pool + he.mu_off;
  const int r = he.r, layer = head / a.n_kv, kv = head % a.n_kv, G = a.group;
  float m4[4];  // the lane's dimensions: 2 l, 2 l + 1 and the ones 64 behind
#pragma unroll
  for (int k = 0; k < 4; ++k) m4[k] = known ? mu[2 * lane + (k & 1) + 64 * (k >> 1)] : 0.f;
  float4 basis[kD / 8];  // on its way while the queries come
  load_basis<8>(basis, pool + he.w_off, r, warp);
  const int T = tree_len(a, s, false), n = tree_drafts(a, s, false);
  const int c0 = chunk * kTreeChunk, nv = max(0, min(kTreeChunk, n * G - c0));
  if (c0 / a.nc * a.nc >= n * G) return;  // nobody reads this tile (idle columns of a tile in use get zeros)
  const __nv_bfloat16* q = a.q + layer * a.q_sl + (long long)s * a.q_ss + (long long)(kv * G) * kD;
  const bool wide = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)(2 * a.q_sl) | (uintptr_t)(2 * a.q_ss) |
                      (uintptr_t)(2 * a.q_st)) & 3) == 0;
  if (tid == 0) {
    mbar_init(smem_addr(&sm.done), 1);
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc(smem_addr(&sm.tmem), kTreeChunk);
  const int ti = tid < nv ? (c0 + tid) / G : 0;  // the thread's column: its token
  const int p = tree_pos(a, s, ti, T);
  const int2 seen = tid < nv ? tree_seen(a, p, T) : make_int2(0, 0);
  const float slope = a.slopes && tid < nv ? a.slopes[kv * G + (c0 + tid) % G] * kLog2e : 0.f;
  constexpr int kEach = kTreeChunk / 8;
  uint32_t xa[kEach], xb[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int c = c0 + warp + 8 * k;
    xa[k] = xb[k] = 0u;
    if (warp + 8 * k < nv) load_pairs(q + (long long)(c / G) * a.q_st + c % G * kD, wide, xa[k], xb[k]);
  }
  lay_basis<2, 8, false>(sm.w, basis, r, warp, float3{}, [](int, float) {});
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int c = warp + 8 * k;
    *reinterpret_cast<uint32_t*>(sm.x[0] + pair_at(c)) = xa[k];
    *reinterpret_cast<uint32_t*>(sm.x[1] + pair_at(c)) = xb[k];
    float d = fmaf(__uint_as_float(xa[k] << 16), m4[0], __uint_as_float(xa[k] & 0xFFFF0000u) * m4[1]);
    d = fmaf(__uint_as_float(xb[k] << 16), m4[2], fmaf(__uint_as_float(xb[k] & 0xFFFF0000u), m4[3], d));
#pragma unroll
    for (int m = 16; m; m >>= 1) d += __shfl_xor_sync(0xffffffffu, d, m);
    if (lane == 0) sm.dot[c] = d;
  }
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  if (warp == 0) {
    // kind::f16, bf16 A and B, fp32 D, M = 128 channels, N = 32 columns; the basis' small pieces first
    constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTreeChunk >> 3) << 17) | (8u << 24);
    const uint64_t wd = umma_desc_sw128(smem_addr(sm.w)), xd = umma_desc_sw128(smem_addr(sm.x));
    if (elect_one()) {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int half = (t >> 2) & 1, piece = 1 - (t >> 3);
        tc_mma_bf16_ss(tmem, wd + (uint64_t)((2 * piece + half) * (kD * 128) >> 4) + (t & 3) * 2,
                       xd + (uint64_t)(half * (kTreeChunk * 128) >> 4) + (t & 3) * 2, kIdesc, t > 0);
      }
      tc_commit(smem_addr(&sm.done));
    }
    __syncwarp();
  }
  if (!mbar_wait_bounded(smem_addr(&sm.done), 0, kTreeWaitNs)) atomicOr(&g_status, 1u);
  __syncwarp();
  tc_fence_after();
  if (warp < 4) {
    uint32_t y[32];
    tc_ld32(tmem + ((uint32_t)(32 * warp) << 16), y);
    tc_wait_ld(y);
#pragma unroll
    for (int c = 0; c < kTreeChunk; ++c) sm.os[c][tid] = __uint_as_float(y[c]);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, kTreeChunk);
  const float f = he.delta * kInvSqrtD * kLog2e;
  // per column: the largest |q~|, how far a score can be from c0 (sum |q~| (2^{b-1} - 1/2), a little more for the
  // roundings; with a cap from 0: the cap).  An element that is not finite makes q . mu such; columns with one are left out.
  float top = 0.f, far = 0.f;
  for (int c = warp; c < nv; c += 8) {
    float s1 = 0.f, most = 0.f;
#pragma unroll
    for (int k = 0; k < kD / 32; ++k) {
      const int i = lane + 32 * k;
      const float x = i < r ? fabsf(sm.os[c][i] * f) : 0.f;
      most = fmaxf(most, x);
      s1 += x;
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) s1 += __shfl_xor_sync(0xffffffffu, s1, m);
    s1 *= ((float)(1 << (he.b > 0 ? he.b - 1 : 0)) - 0.5f) * 1.01f;
    const bool bad = !(s1 + fabsf(sm.dot[c]) * (kInvSqrtD * kLog2e) < kTreeLargest);
#pragma unroll
    for (int m = 16; m; m >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, m));
    // f16 rounds an element by 2^-11 of it (finer than the bf16 query's own 2^-8) down to 2^-14, and smaller ones
    // by 2^-25, which the codes of a head make 2^-11 of a score's log2 unit at most: a column's q~ is scaled only
    // where it would overflow
    if (lane == 0) {
      int ex = 15;
      if (!bad && most >= 32768.f) frexpf(most, &ex);
      sm.bad[c] = bad;
      sm.exp[c] = 15 - ex;
    }
    if (bad) continue;
    top = fmaxf(top, most);
    far = fmaxf(far, s1);
  }
  if (__any_sync(0xffffffffu, !(fabsf(slope) < 1e20f))) far = INFINITY;  // (times 2^31 it would not be finite)
  if (lane == 0) sm.red[0][warp] = top, sm.red[1][warp] = far;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = fmaxf(top, sm.red[0][w]), far = fmaxf(far, sm.red[1][w]);
  const long long unit = ((long long)head * a.n_seqs + s) * a.tiles + c0 / a.nc;
  const int cb = c0 % a.nc;  // the chunk's first column in its tile
  unsigned char* img = a.img + unit * (2 * a.nc * 128);
  const int ncol = min(kTreeChunk, a.nc);
  for (int idx = tid; idx < ncol * (kD / 8); idx += 256) {  // 8 places of a column
    const int c = idx / (kD / 8), p = 8 * (idx % (kD / 8));
    const bool fed = c < nv && !sm.bad[c];
    const float up = fed ? ldexpf(f, sm.exp[c]) : 0.f;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = tc_k_channel(p + 2 * k + h);
        x[h] = fed && i < r ? sm.os[c][i] * up : 0.f;
      }
      w[k] = pack_f16(x[0], x[1]);
    }
    *reinterpret_cast<uint4*>(img + tree_img_at(a.nc, cb + c, p)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  const int bounded = top >= 32768.f ? -1 : a.cap2 > 0.f ? a.cap2 <= kTreeBound && far < INFINITY : far <= kTreeBound;
  if (tid < ncol) {
    const int bad = tid < nv ? sm.bad[tid] : 0;
    const float c0f = tid < nv && !bad ? sm.dot[tid] * (kInvSqrtD * kLog2e) : 0.f;
    a.col[unit * a.nc + cb + tid] = TreeCol{c0f, slope, p, ldexpf(1.f, tid < nv ? -sm.exp[tid] : 0), seen.x, seen.y, bounded, bad};
  }
}

// The drafted tokens' own part of 32 columns: m, l and O in the model's dimensions.
__device__ __forceinline__ void tree_draft_part(const TreeArgs& a, TreeDraftSmem& sm, int head, int s, int chunk) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.group;
  const int layer = head / a.n_kv, kv = head % a.n_kv;
  const int T = tree_len(a, s, false), n = tree_drafts(a, s, false);
  const int c0 = chunk * kTreeChunk, nv = min(kTreeChunk, n * G - c0);
  if (nv <= 0) return;
  const __nv_bfloat16* q = a.q + layer * a.q_sl + (long long)s * a.q_ss + (long long)(kv * G) * kD;
  const long long d0 = layer * a.d_sl + (long long)s * a.d_ss + kv * a.d_sh;
  // 8 elements at a time where every row is 16-byte aligned
  auto stage = [&](auto row, int rows, bool wide, float f, float(*to)[kD + 4]) {
    if (wide) {
      for (int idx = tid; idx < rows * (kD / 8); idx += 256) {
        const int r = idx / (kD / 8), c = idx % (kD / 8);
        const uint4 u = reinterpret_cast<const uint4*>(row(r))[c];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          to[r][8 * c + 2 * k] = f * __uint_as_float(w[k] << 16);
          to[r][8 * c + 2 * k + 1] = f * __uint_as_float(w[k] & 0xFFFF0000u);
        }
      }
    } else {
      for (int idx = tid; idx < rows * kD; idx += 256) to[idx / kD][idx % kD] = f * __bfloat162float(row(idx / kD)[idx % kD]);
    }
  };
  auto aligned16 = [](const void* p, long long x, long long y, long long z) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(2 * x) | (uintptr_t)(2 * y) | (uintptr_t)(2 * z)) & 15) == 0;
  };
  const bool q_wide = aligned16(a.q, a.q_sl, a.q_ss, a.q_st);
  const bool d_wide = aligned16(a.kd, a.d_sl, a.d_ss, a.d_st | a.d_sh) && aligned16(a.vd, 0, 0, 0);
  stage([&](int c) { return q + (long long)((c0 + c) / G) * a.q_st + ((c0 + c) % G) * kD; }, nv, q_wide, kInvSqrtD * kLog2e, sm.q);
  stage([&](int j) { return a.kd + d0 + (long long)j * a.d_st; }, n, d_wide, 1.f, sm.kv);
  if (tid < n) {
    sm.pos[tid] = tree_pos(a, s, tid, T);
    sm.mask[tid] = a.mask ? a.mask[(long long)s * a.max_draft + tid] : ~0ull >> (63 - tid);
  }
  __syncthreads();
  // scores: a warp has four columns, its lanes the drafted tokens lane and lane + 32
  const float k2 = tree_cap_k(a.cap2);
  {
    float z[4][2] = {};
    const int j0 = min(lane, n - 1), j1 = min(lane + 32, n - 1), cw = 4 * warp;
    if (cw < nv) {
#pragma unroll 4
      for (int d = 0; d < kD; d += 4) {
        const float4 k0 = *reinterpret_cast<const float4*>(&sm.kv[j0][d]), k1 = *reinterpret_cast<const float4*>(&sm.kv[j1][d]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float4 x = *reinterpret_cast<const float4*>(&sm.q[min(cw + c, nv - 1)][d]);
          z[c][0] = fmaf(x.x, k0.x, fmaf(x.y, k0.y, fmaf(x.z, k0.z, fmaf(x.w, k0.w, z[c][0]))));
          z[c][1] = fmaf(x.x, k1.x, fmaf(x.y, k1.y, fmaf(x.z, k1.z, fmaf(x.w, k1.w, z[c][1]))));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int c = cw + (u >> 1), j = lane + 32 * (u & 1), i = (c0 + c) / G, g = (c0 + c) % G;
      if (c >= nv || j >= n) continue;
      const long long dist = (long long)sm.pos[j] - sm.pos[i];
      const bool seen = (sm.mask[i] >> j & 1ull) != 0ull && (a.window <= 0 || dist > -(long long)a.window);
      float y = z[u >> 1][u & 1];
      if (a.cap2 > 0.f) y = a.cap2 <= kTreeCapPlain ? tree_cap(y, a.cap2, k2) : tree_cap_large(y, a.cap2, k2);
      if (a.slopes) y = fmaf(a.slopes[kv * G + g] * kLog2e, (float)dist, y);
      sm.z[c][j] = !seen ? -INFINITY : y < kTreeLowest ? kTreeLowest : y;
    }
  }
  __syncthreads();
  stage([&](int j) { return a.vd + d0 + (long long)j * a.d_st; }, n, d_wide, 1.f, sm.kv);
  float* part = a.draft + (((long long)head * a.n_seqs + s) * a.max_draft * G + c0) * kTreePart;
  for (int c = warp; c < kTreeChunk; c += 8) {
    const float z0 = c < nv && lane < n ? sm.z[c][lane] : -INFINITY, z1 = c < nv && lane + 32 < n ? sm.z[c][lane + 32] : -INFINITY;
    float m = fmaxf(z0, z1);
#pragma unroll
    for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
    const float p0 = z0 == -INFINITY ? 0.f : exp2f(z0 - m), p1 = z1 == -INFINITY ? 0.f : exp2f(z1 - m);
    float l = p0 + p1;
#pragma unroll
    for (int k = 16; k; k >>= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
    sm.p[lane][c] = p0;
    sm.p[lane + 32][c] = p1;
    if (lane == 0 && c < nv) {
      part[c * kTreePart] = m;
      part[c * kTreePart + 1] = l;
    }
  }
  __syncthreads();
  // values: a thread has one dimension of 16 columns.  A token that a column does not see has p = 0,
  // whatever its value is.
  const int d = tid & 127, cb = 16 * (tid >> 7);
  float o[16] = {};
  for (int j = 0; j < n; ++j) {
    const float v = sm.kv[j][d];
    float p[16];
#pragma unroll
    for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(p + k) = *reinterpret_cast<const float4*>(&sm.p[j][cb + k]);
    if (fabsf(v) < INFINITY) {
#pragma unroll
      for (int k = 0; k < 16; ++k) o[k] = fmaf(p[k], v, o[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) o[k] = cb + k >= nv || sm.z[cb + k][j] == -INFINITY ? o[k] : fmaf(p[k], v, o[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 16; ++k)
    if (cb + k < nv) part[(cb + k) * kTreePart + 4 + d] = o[k];
}

// grid: (head, sequence, chunk) projections, as many drafted parts where there are drafted keys, one more
__global__ void __launch_bounds__(256, 2) tree_prepare_kernel(TreeArgs a) {
  extern __shared__ unsigned char tree_raw[];
  unsigned char* const tree_smem = tree_raw + ((1024u - (smem_addr(tree_raw) & 1023u)) & 1023u);
  const long long n = (long long)a.n_layers * a.n_kv * a.n_seqs * a.chunks;
  long long b = blockIdx.x;
  if (b == 0) {
    grid_dep_wait();
    tree_layout(a, reinterpret_cast<long long*>(tree_smem));
    return;
  }
  --b;
  const bool draft = b >= n;
  if (draft) b -= n;
  const int chunk = (int)(b % a.chunks), s = (int)(b / a.chunks % a.n_seqs), head = (int)(b / a.chunks / a.n_seqs);
  if (!draft) {
    tree_project(a, *reinterpret_cast<TreeProjSmem*>(tree_smem), head, s, chunk);
    grid_dep_launch();  // not ahead of the work: the scan's CTAs need whole SMs
  } else {
    grid_dep_wait();
    tree_draft_part(a, *reinterpret_cast<TreeDraftSmem*>(tree_smem), head, s, chunk);
  }
}

// ---------------------------------------------------------------------------------------
// Scan
// ---------------------------------------------------------------------------------------
struct TreeSeg {
  int head, s, tile, k0, k1;  // rows [k0, k1) of the unit, from the sequence's first one, row0
  int row0, drafts;
  long long unit;
};
// Walks the parts of CTA c along the line (a converged warp).
struct TreeWalk {
  TreeLine line;
  long long x0, x1, at;  // the CTA's stretch and where the walk has come to
  int head, s;           // where it begins
  __device__ TreeWalk(const TreeArgs& a, int c)
      : line(a), x0(line.begin(c)), x1(line.begin(c + 1)), at(x0), head(a.start[2 * c]), s(a.start[2 * c + 1]) {}
  __device__ bool next(const TreeArgs& a, TreeSeg& g) {
    while (at < x1) {
      TreeFound h, f;
      if (head >= 0) {
        h = TreeFound{head, a.wpre[head], a.wpre[head + 1]};
        f = TreeFound{s, a.rpre[s], 0};
        head = -1;
      } else {
        h = tree_find(a.wpre, a.n_layers * a.n_kv, tree_div(at, line.rows));
        f = tree_find(a.rpre, a.n_seqs, tree_div(at - h.lo * line.rows, h.hi - h.lo));
      }
      const int w = (int)(h.hi - h.lo);
      const long long hbase = h.lo * line.rows;
      const int n = a.rows[f.i], row0 = a.row0[f.i], drafts = tree_drafts(a, f.i, false);
      const long long sbase = hbase + f.lo * w;
      const int tile = (int)tree_div(at - sbase, (long long)n * w);
      const long long base = sbase + (long long)tile * n * w;
      g = TreeSeg{h.i, f.i, tile, TreeLine::before(x0, base, n, w), TreeLine::before(x1, base, n, w), row0, drafts,
                  ((long long)h.i * a.n_seqs + f.i) * a.tiles + tile};
      at = base + (long long)n * w;
      if (g.k0 < g.k1) return true;
    }
    return false;
  }
};

// ---------------------------------------------------------------------------------------
// The scan kernel.  A CTA per SM walks its stretch of the line row by row, as a pipeline of warps:
//   producer     walks the stretch, copies q~ images, columns and code rows (bulk copies) into rings
//   K unpackers  (4 warps, thread = token) codes of a K row into TMEM, exact f16 deviations
//   products     (a warp each) S[token][column] = A_K q~  (M = 128 tokens, N = columns, K = channels), and
//                O[channel][column] += A_V P  (M = 128 channels, K = 128 tokens), A from TMEM; the columns'
//                sums l are O's row behind the last channel, whose A is a constant (a product of their own,
//                M = 64 equal rows, for heads of rank 128)
//   V unpackers  (4 warps, thread = channel) codes of a V row into TMEM
//   softmax      (4 warps per 32 columns, thread = token) scores from TMEM, probabilities as bf16 into shared
//                memory: rows of 64 columns per token, the MN-major operand of the second product
// KA, VA and S have two buffers and P three, so that a row's five steps run beside those of its neighbours.
//
// The fed probabilities 2^(z - reference) are bf16 (a rounding of 2^-8, as the result's own; the sums l are of
// the fed values, so the weights are normalised exactly; it makes the result 1.1e-3 less exact than f16 would): its exponents hold all that fp32 does, so the
// reference need not follow the maximum.  Where the codes bound the scores to within kTreeBound of c0 (or a cap
// bounds them), c0 (0) and the largest bias are the reference, a score goes from TMEM into the exponential as it is
// (or capped and with its bias), and the warps of a row need not agree on anything.  Else (large queries) a
// reference is raised when a score
// exceeds it by kTreeTau (one vote per row and 32 columns), and the columns' sums and O are rescaled.  Queries of standard
// deviation 1.5, bounded, and 4, with votes: 64 columns, 131072 tokens at 0.5 bpd 284 and 397 us a call; 8 x 32768 at
// 1 bpd 107 and 136; single tokens with biases over 32 ragged sequences of up to 16384 at 4 bpd 74 and 111.
//
// What bounds it: a row takes 1300 to 1600 cycles, of which the products' own are 80 (16 columns) to 512.  The issue
// slots of an SM's four quarters are used to 0.61 on average and to 0.74 in the fullest: the K, V and softmax warps of
// the same 32 TMEM lanes share one, and ranks up to 64 leave two quarters without V codes.  The rest are the two
// chains of hand-overs (product, softmax, next product into the same buffer; codes, product, next codes): when the first
// case above took 306 us, it took 260 with the unpacking left out and 244 with the exponentials left out too.
// ---------------------------------------------------------------------------------------
constexpr float kTreeTau = 60.f;
constexpr int kTreeRingBytes = 57344;    // K rows in flight, and V rows: as many as fit, 3 of the largest at least
constexpr int kTreeRing = 16;            // and this many at most

struct TreeDesc {  // a part of a unit, as the warps see it
  int n, row0, rk, bk, rv, bv, n_col;  // rows (0: no more parts), first row, ranks and widths, live columns
  long long slot;
};
template <int NCW>
struct alignas(16) TreeWg {  // per softmax warpgroup
  float c0[NCW], sub[NCW];     // c0, and what is subtracted from a score: the reference (sub: c0 - reference, plain)
  float ref[NCW], alpha[NCW];
  float slope[NCW], sc[NCW];
  int pos[NCW], lo[NCW], hi[NCW];
  float red[4][NCW];
};
template <int NC, int NCW>
struct TreeScanSmem {
  static constexpr int kWg = NC == 64 ? 2 : 1;  // (at most 8 columns are part of a product of 16)
  static constexpr int kThreads = 32 * (8 + 4 * kWg + 3);
  unsigned char p[3][128 * 128];          // [token][64 columns] bf16, swizzled
  unsigned char ones[64 * 128];           // bf16 1.0: A of the product that sums the probabilities
  unsigned char img[2][2 * NC * 128];     // (operands of the products lie on 1024-byte boundaries)
  unsigned char k[kTreeRingBytes], v[kTreeRingBytes];
  alignas(16) uint32_t half[36 * 4];      // 16 b bytes for every width b: codes 2^{b-1}, deviation 1/2
  alignas(16) TreeCol col[2][NC];
  TreeWg<NCW> wg[kWg];
  TreeDesc desc[2];
  unsigned long long seg_full[2], seg_empty[2], kf[kTreeRing], ke[kTreeRing], vf[kTreeRing], ve[kTreeRing];
  // operands of a row's first product ready (codes in KA, S read), its result; of the second (VA, P), done
  unsigned long long s_ready[2], s_full[2], pv_ready[3], pv_done[3], o_empty, drain;
  uint32_t tmem;
  int fail;
};

// f with the width as a constant (0: nothing to unpack)
template <typename F>
__device__ __forceinline__ void tree_by_width(int b, F f) {
  switch (b) {
    case 0: f(std::integral_constant<int, 0>{}); break;
    case 1: f(std::integral_constant<int, 1>{}); break;
    case 2: f(std::integral_constant<int, 2>{}); break;
    case 3: f(std::integral_constant<int, 3>{}); break;
    case 4: f(std::integral_constant<int, 4>{}); break;
    case 5: f(std::integral_constant<int, 5>{}); break;
    case 6: f(std::integral_constant<int, 6>{}); break;
    case 7: f(std::integral_constant<int, 7>{}); break;
    default: f(std::integral_constant<int, 8>{}); break;
  }
}
// the rest of a wait whose first look failed; out of line: every copy of it would take room in the caches
__device__ __noinline__ bool tree_wait_on(uint32_t bar, uint32_t parity) {
  return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, kTreeWaitNs));
}
template <int N>
__device__ __forceinline__ void tree_ld(uint32_t taddr, uint32_t (&v)[N]) {
  if constexpr (N == 32) {
    tc_ld32(taddr, v);
  } else if constexpr (N == 16) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
  } else {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr)
                 : "memory");
  }
}
// Wait for this thread's TMEM loads; v passes through, so that no use of it is scheduled ahead.
template <int N>
__device__ __forceinline__ void tree_wait_ld(uint32_t (&v)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(v[i]));
}
template <int N>
__device__ __forceinline__ void tree_st(uint32_t taddr, const uint32_t (&v)[N]) {
#pragma unroll
  for (int c = 0; c < N / 8; ++c) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = v[8 * c + i];
    tc_st32x8(taddr + 8 * c, w);
  }
}
// v[j] over the warp's 32 lanes for every j by halving exchanges: the lane's result is that of column
// tree_owned<N>(lane)
template <int N>
__device__ __forceinline__ int tree_owned(int lane) {
  return N == 32 ? lane : N == 16 ? lane >> 1 : lane >> 2;
}
template <int N, typename Op>
__device__ __forceinline__ float tree_reduce(float (&v)[N], Op op) {
  const int lane = threadIdx.x & 31;
  int n = N;
#pragma unroll
  for (int m = 16; m; m >>= 1) {
    const bool up = lane & m;
    if (n > 1) {
      n >>= 1;
#pragma unroll
      for (int j = 0; j < N / 2; ++j)
        if (j < n) {
          const float send = up ? v[j] : v[j + n], keep = up ? v[j + n] : v[j];
          v[j] = op(keep, __shfl_xor_sync(0xffffffffu, send, m));
        }
    } else {
      v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], m));
    }
  }
  return v[0];
}
// Scores of the thread's token against the columns: absolute (log2 units) or less the reference.  A column without a
// reference has sub = +3e38 (plain) or -3e38 (ref), so that any score it sees asks for one.
template <int NCW, bool ABS, bool LARGE>
__device__ __forceinline__ void tree_scores(const TreeArgs& a, const TreeWg<NCW>& w, const uint32_t (&x)[NCW], float k2,
                                            bool plain, bool masked, int tok, float (&z)[NCW]) {
  if (plain) {
    const float* add = ABS ? w.c0 : w.sub;
    const f32x2 one = pack2(1.f, 1.f);
#pragma unroll
    for (int j = 0; j < NCW; j += 4) {
      const float4 c = *reinterpret_cast<const float4*>(add + j);
      const float2 y0 = unpack2(fma2(pack2(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), one, pack2(c.x, c.y)));
      const float2 y1 = unpack2(fma2(pack2(__uint_as_float(x[j + 2]), __uint_as_float(x[j + 3])), one, pack2(c.z, c.w)));
      z[j] = y0.x, z[j + 1] = y0.y, z[j + 2] = y1.x, z[j + 3] = y1.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NCW; ++j) {
      float y = __uint_as_float(x[j]) + w.c0[j];
      if (a.cap2 > 0.f) y = LARGE ? tree_cap_large(y, a.cap2, k2) : tree_cap(y, a.cap2, k2);
      if (a.slopes) y = fmaf(w.slope[j], (float)(tok - w.pos[j]), y);
      z[j] = ABS ? y : y - w.sub[j];
    }
  }
  if (masked) {
#pragma unroll
    for (int j = 0; j < NCW; ++j)
      if (tok < w.lo[j] || tok >= w.hi[j]) z[j] = -INFINITY;
  }
}

// LARGE: caps above kTreeCapPlain (a kernel of their own: with both formulas in one, calls with biases and loud queries
// took 142 us for 111, 32 ragged sequences of up to 16384 tokens)
template <int NC, int NCW, bool LARGE>
__global__ void __launch_bounds__(TreeScanSmem<NC, NCW>::kThreads, 1) tree_scan_kernel(TreeArgs a) {
  using Smem = TreeScanSmem<NC, NCW>;
  constexpr int kWg = Smem::kWg, kMmaWarp = 8 + 4 * kWg;
  constexpr int kKa = 0, kVa = 128, kS = 256, kO = 384, kL = 448;  // TMEM columns (64 per buffer)
  // instruction descriptors, kind::f16: f16 A and B (bf16 in the second), fp32 D, M = 128, N = NC; the second's
  // B is MN-major
  constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(NC >> 3) << 17) | (8u << 24), kIdescO = kIdescS | (1u << 16) | (1u << 7) | (1u << 10);
  constexpr uint32_t kIdescL = (kIdescO & ~(31u << 24)) | (4u << 24);  // M = 64
  extern __shared__ unsigned char tree_raw[];
  const uint32_t raw = smem_addr(tree_raw);
  Smem& sm = *reinterpret_cast<Smem*>(tree_raw + (((raw + 1023u) & ~1023u) - raw));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto bar = [](unsigned long long& b) { return smem_addr(&b); };
  if (warp == kMmaWarp && lane == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(sm.seg_full[i]), 1);
      mbar_init(bar(sm.seg_empty[i]), 8 + 4 * kWg + 2);
      mbar_init(bar(sm.s_ready[i]), 4 + 4 * kWg);
      mbar_init(bar(sm.s_full[i]), 1);
    }
    // (as many as P has buffers: the softmax warps may be two rows ahead of the V unpackers)
    for (int i = 0; i < 3; ++i) {
      mbar_init(bar(sm.pv_ready[i]), 4 + 4 * kWg);
      mbar_init(bar(sm.pv_done[i]), 1);
    }
    for (int i = 0; i < kTreeRing; ++i) {
      mbar_init(bar(sm.kf[i]), 1);
      mbar_init(bar(sm.ke[i]), 4);
      mbar_init(bar(sm.vf[i]), 1);
      mbar_init(bar(sm.ve[i]), 4);
    }
    mbar_init(bar(sm.o_empty), 4 * kWg);
    mbar_init(bar(sm.drain), 2);
    fence_mbar_init();
  }
  if (tid == 0) sm.fail = 0;
  for (int i = tid; i < (int)sizeof(sm.ones) / 4; i += Smem::kThreads) reinterpret_cast<uint32_t*>(sm.ones)[i] = 0x3F803F80u;
  for (int i = tid; i < 36 * 4; i += Smem::kThreads) {  // words of b: from 4 (1 + .. + b - 1), word q b + n of piece q
    int b = 1, at = i;
    while (at >= 4 * b) at -= 4 * b++;
    uint32_t x = 0;
    for (int rho = 0; rho < 16; ++rho) {  // the top bit of every code, in both sub-streams
      const int bit = rho * b + b - 1;
      if (bit >> 4 == at % b) x |= 0x00010001u << (bit & 15);
    }
    sm.half[i] = x;
  }
  fence_proxy_async_smem();
  if (warp == 0) tmem_alloc(smem_addr(&sm.tmem), 512);
  grid_dep_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  // slots of the largest row's size (the last channel tile of a K row is read whole, up to 1.8 KB behind
  // the row: any bits there are finite codes, against zeros of q~)
  const int k_slot = max(128, (a.row_bytes[0] + 127) & ~127), v_slot = max(128, (a.row_bytes[1] + 127) & ~127);
  const int ring = min(kTreeRing, kTreeRingBytes / max(k_slot, v_slot));
  // a wait of the whole warp; after one that has expired the warp's later ones pass at once, it leaves its loop,
  // and the others' waits for it expire in turn
  bool ok = true;
  auto wait = [&](unsigned long long& b, uint32_t parity) {
    if (!__all_sync(0xffffffffu, mbar_try_wait(bar(b), parity)) && ok) ok = tree_wait_on(bar(b), parity);
    return ok;
  };
  auto arrive = [&](unsigned long long& b) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(b));
  };
  // the next part of the stretch: false when there is none
  TreeDesc d;
  auto next_part = [&](int seg) {
    if (!wait(sm.seg_full[seg & 1], (seg >> 1) & 1)) return false;
    d = sm.desc[seg & 1];
    return d.n > 0;
  };

  if (warp == kMmaWarp + 2) {
    // ---- producer ----
    TreeWalk walk(a, blockIdx.x);
    TreeSeg g;
    int n = 0, st = 0;  // rows so far, the next one's slot and its phase
    uint32_t ph = 0;
    for (int seg = 0;; ++seg) {
      const bool more = walk.next(a, g);
      if (seg >= 2 && !wait(sm.seg_empty[seg & 1], ((seg >> 1) - 1) & 1)) break;
      bool kk, kv;
      HeadEntry hk, hv;
      if (more) hk = tree_head(a, a.k_head0, g.head, kk), hv = tree_head(a, a.v_head0, g.head, kv);
      const uint32_t rbk = more ? 16u * hk.r * hk.b : 0u, rbv = more ? 16u * hv.r * hv.b : 0u;
      const int row0 = more ? g.row0 + g.k0 : 0, rows = more ? g.k1 - g.k0 : 0;
      if (lane == 0) {
        TreeDesc& o = sm.desc[seg & 1];
        o.n = rows;
        if (more) {
          o = TreeDesc{rows, row0, hk.r, hk.b, hv.r, hv.b, min(NC, g.drafts * a.group - g.tile * NC),
                       (long long)blockIdx.x + g.unit};
          // channels past the rank's last tile of 64 are not read
          const uint32_t img = (hk.r > 64 ? 2u : 1u) * NC * 128u;
          fence_proxy_async_smem();
          mbar_arrive_expect_tx(bar(sm.seg_full[seg & 1]), img + NC * (uint32_t)sizeof(TreeCol));
          bulk_g2s(smem_addr(sm.img[seg & 1]), a.img + g.unit * (2 * NC * 128), img, bar(sm.seg_full[seg & 1]));
          bulk_g2s(smem_addr(sm.col[seg & 1]), a.col + g.unit * NC, NC * (uint32_t)sizeof(TreeCol), bar(sm.seg_full[seg & 1]));
        } else {
          mbar_arrive(bar(sm.seg_full[seg & 1]));
        }
      }
      __syncwarp();
      if (!more) break;
      int page = 0;
      for (int k = 0; k < rows && ok; ++k, ++n) {
        const int row = row0 + k;
        if (a.page_table) {  // lane l looks up the page of row k + l
          if (k % 32 == 0 && k + lane < rows) page = a.page_table[(long long)g.s * a.pages_per_seq + ((row + lane) >> 1)];
        }
        const long long slot = a.page_table ? 2LL * __shfl_sync(0xffffffffu, page, k % 32) + (row & 1)
                                            : (long long)g.s * a.rows_per_seq + row;
        if (n >= ring && (!wait(sm.ke[st], ph ^ 1u) || !wait(sm.ve[st], ph ^ 1u))) break;
        if (lane == 0) {
          fence_proxy_async_smem();
          mbar_arrive_expect_tx(bar(sm.kf[st]), rbk);
          if (rbk) bulk_g2s(smem_addr(sm.k + st * k_slot), a.cache + hk.cache_off + slot * rbk, rbk, bar(sm.kf[st]));
          mbar_arrive_expect_tx(bar(sm.vf[st]), rbv);
          if (rbv) bulk_g2s(smem_addr(sm.v + st * v_slot), a.cache + hv.cache_off + slot * rbv, rbv, bar(sm.vf[st]));
        }
        __syncwarp();
        if (++st == ring) st = 0, ph ^= 1u;
      }
      if (!ok) break;
    }
  } else if (warp == kMmaWarp) {
    // ---- first products, issued by one thread ----
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    int n = 0;
    for (int seg = 0; next_part(seg); ++seg) {
      const int nk = (d.rk + 15) >> 4;
      const uint64_t qd = umma_desc_sw128(smem_addr(sm.img[seg & 1]));
      for (int k = 0; k < d.n && ok; ++k, ++n) {
        const int u = n & 1;
        if (!wait(sm.s_ready[u], (n >> 1) & 1)) break;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kt = 0; kt < 8; ++kt)
            if (kt < nk)
              tc_mma_bf16_ts(tm + kS + 64 * u, tm + kKa + 64 * u + 8 * kt,
                             qd + (uint64_t)((kt >> 2) * (NC * 128) >> 4) + (kt & 3) * 2, kIdescS, kt > 0);
          tc_commit(bar(sm.s_full[u]));
          if (k == d.n - 1) tc_commit(bar(sm.seg_empty[seg & 1]));  // the image has been read
        }
        __syncwarp();
      }
      if (!ok) break;
    }
  } else if (warp == kMmaWarp + 1) {
    // ---- second products ----
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t od = umma_desc_sw128(smem_addr(sm.ones)), pd = umma_desc_sw128(smem_addr(sm.p[0]));
    int n = 0, pb = 0, ph = 0;
    for (int seg = 0; next_part(seg); ++seg) {
      arrive(sm.seg_empty[seg & 1]);
      // the part's first product overwrites O: the softmax warps have read the part's before
      if (seg > 0 && !wait(sm.o_empty, (seg - 1) & 1)) break;
      for (int k = 0; k < d.n && ok; ++k, ++n) {
        if (!wait(sm.pv_ready[pb], ph)) break;
        tc_fence_after();
        // P: 8 tokens x 64 columns are a 1024-byte block, a k-tile of 16 tokens is two of them
        const uint64_t p = pd + (uint64_t)(pb * 128 * 128 >> 4);
        const uint32_t va = tm + kVa + 64 * (n & 1);
        if (elect_one()) {
#pragma unroll
          for (int kt = 0; kt < 8; ++kt)
            tc_mma_bf16_ts(tm + kO, va + 8 * kt, p + (uint64_t)(kt * 2048 >> 4), kIdescO, k > 0 || kt > 0);
          if (d.rv == kD) {
#pragma unroll
            for (int kt = 0; kt < 8; ++kt)
              tc_mma_bf16_ss(tm + kL, od, p + (uint64_t)(kt * 2048 >> 4), kIdescL, k > 0 || kt > 0);
          }
          tc_commit(bar(sm.pv_done[pb]));
        }
        __syncwarp();
        if (++pb == 3) pb = 0, ph ^= 1;
      }
      if (!ok) break;
    }
  } else if (warp < 4) {
    // ---- K unpackers ----
    const uint32_t ka = tmem + ((uint32_t)(32 * warp) << 16) + kKa;
    int n = 0, st = 0;
    uint32_t ph = 0;
    for (int seg = 0; next_part(seg); ++seg) {
      arrive(sm.seg_empty[seg & 1]);
      const int nk = (d.rk + 15) >> 4;
      tree_by_width(nk ? d.bk : 0, [&](auto width) {  // (a loop over rows for each width: short code)
        constexpr int B = decltype(width)::value;
        const KUnpack<B ? B : 1> unpack(warp, a.top_f16);
        for (int k = 0; k < d.n && ok; ++k, ++n) {
          const int u = n & 1;
          if (!wait(sm.kf[st], ph)) break;
          if (n >= 2 && !wait(sm.s_full[u], ((n >> 1) - 1) & 1)) break;  // the product before has read the buffer
          tc_fence_after();
          if constexpr (B > 0) {
            unpack(sm.k + st * k_slot, nk, ka + 64 * u);
            tc_wait_st();
          }
          arrive(sm.ke[st]);
          if (++st == ring) st = 0, ph ^= 1u;
          tc_fence_before();
          arrive(sm.s_ready[u]);
        }
      });
      if (!ok) break;
    }
  } else if (warp < 8) {
    // ---- V unpackers: channels 64 .. 127 in the first two warps' lanes (the SM quarters of the other two have
    //      neither the products' nor the copies' warp, and most ranks are below 64) ----
    const int ch = (tid - 64) & 127;
    const uint32_t va = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kVa;
    int n = 0, st = 0, pb = 0, pd = 1;  // (pd: phase of row n - 2 on its barrier, (pb + 1) % 3)
    uint32_t ph = 0;
    for (int seg = 0; next_part(seg); ++seg) {
      arrive(sm.seg_empty[seg & 1]);
      // channels 0 .. r - 1, then the constant row of the sums (lanes behind it hold anything)
      tree_by_width((ch & ~31) > d.rv ? 0 : d.rv > 0 ? d.bv : 1, [&](auto width) {
        constexpr int B = decltype(width)::value;
        const uint8_t* half = reinterpret_cast<const uint8_t*>(sm.half + 2 * B * (B - 1));
        for (int k = 0; k < d.n && ok; ++k, ++n) {
          const int u = n & 1;
          if (!wait(sm.vf[st], ph)) break;
          const int next = pb == 2 ? 0 : pb + 1;
          if (next == 0) pd ^= 1;
          if (n >= 2 && !wait(sm.pv_done[next], pd)) break;  // the product of row n - 2 has read the buffer
          tc_fence_after();
          if constexpr (B > 0) {
            tc_unpack_v<B>(ch < d.rv ? sm.v + st * v_slot + 16 * B * ch : half, va + 64 * u, a.top_bf16);
            tc_wait_st();
          }
          arrive(sm.ve[st]);
          if (++st == ring) st = 0, ph ^= 1u;
          tc_fence_before();
          arrive(sm.pv_ready[pb]);
          pb = next;
        }
      });
      if (!ok) break;
    }
  } else {
    // ---- softmax ----
    const int wg = (warp - 8) >> 2, wq = warp & 3, t = 32 * wq + lane;
    const uint32_t lanes = (uint32_t)(32 * wq) << 16;
    TreeWg<NCW>& w = sm.wg[wg];
    const bool plain = !(a.cap2 > 0.f) && !a.slopes;
    const float k2 = tree_cap_k(a.cap2);
    int n = 0, pb = 0, ph = 1;  // row, its buffer of P and the phase of the buffer's last product
    arrive(sm.s_ready[0]);  // both buffers of S are free
    arrive(sm.s_ready[1]);
    for (int seg = 0;; ++seg) {
      const bool more = next_part(seg);
      // the warps leave together, whichever has an expired wait: they meet at barriers all through a part
      // (where an expired wait makes the later ones pass at once)
      if (wg_any(wg, !ok)) ok = false;
      if (!ok || !more) break;
      const TreeCol* col = sm.col[seg & 1] + wg * NCW;
      const int live = min(NCW, d.n_col - wg * NCW);  // may be <= 0
      const int kind = col[0].bounded;
      const bool bounded = kind > 0;
      if (t < NCW) {
        const TreeCol c = col[t];
        w.c0[t] = c.c0;
        // bounded: the reference is c0, or 0 of capped scores, and the largest bias, that of the last token seen
        // (the first one where the slope is negative)
        const float mid = a.cap2 > 0.f ? 0.f : c.c0;
        const int at = c.slope2 < 0.f ? c.lo : c.hi - 1;
        w.sub[t] = plain ? -kTreeLowest : bounded ? mid : kTreeLowest;
        w.ref[t] = !bounded ? -INFINITY : a.slopes ? fmaf(c.slope2, (float)((long long)at - c.pos), mid) : mid;
        w.slope[t] = c.slope2;
        w.sc[t] = c.scale;
        w.pos[t] = bounded ? at : c.pos;
        w.lo[t] = c.lo;
        w.hi[t] = c.hi;
      }
      // rows [lo, hi) are seen whole by every live column
      int lo = 0, hi = 0x7fffffff;
      for (int j = 0; j < live; ++j) lo = max(lo, col[j].lo), hi = min(hi, col[j].hi);
      wg_sync(wg);
      for (int k = 0; k < d.n; ++k, ++n) {
        const int u = n & 1, base = 128 * (d.row0 + k), tok = base + t;
        const bool masked = base < lo || base + 128 > hi;
        wait(sm.s_full[u], (n >> 1) & 1);
        tc_fence_after();
        if (n >= 3) wait(sm.pv_done[pb], ph);  // P's buffer has been read
        unsigned char* const prow = sm.p[pb] + t * 128;
        unsigned long long& p_ready = sm.pv_ready[pb];
        if (++pb == 3) pb = 0, ph ^= 1;
        auto put = [&](int c, const float(&y)[8]) {  // the probabilities of columns 8 c .. 8 c + 7
          uint32_t h[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = pack_bf16(ex2_approx(y[2 * i]), ex2_approx(y[2 * i + 1]));
          *reinterpret_cast<uint4*>(prow + (((wg * (NCW / 8) + c) ^ (t & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        };
        if (bounded && !masked && d.rk > 0) {
          const uint32_t at = tmem + lanes + kS + 64 * u + wg * NCW;
          if (plain) {  // scores as they are, eight columns at a time; the next ones are on their way meanwhile
            uint32_t x[8];
            tree_ld<8>(at, x);
#pragma unroll
            for (int c = 0; c < NCW / 8; ++c) {
              float y[8];
              tree_wait_ld<8>(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(x[i]);
              if (c + 1 < NCW / 8) tree_ld<8>(at + 8 * (c + 1), x);
              put(c, y);
            }
          } else if (!a.slopes) {  // capped
            uint32_t x[8];
            tree_ld<8>(at, x);
#pragma unroll 1
            for (int c = 0; c < NCW / 8; ++c) {
              const float4 p = *reinterpret_cast<const float4*>(w.c0 + 8 * c), q = *reinterpret_cast<const float4*>(w.c0 + 8 * c + 4);
              const float c8[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
              float y[8];
              tree_wait_ld<8>(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(x[i]) + c8[i];
              if (c + 1 < NCW / 8) tree_ld<8>(at + 8 * (c + 1), x);
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = tree_cap(y[i], a.cap2, k2);
              put(c, y);
            }
          } else {  // with a bias, capped or not
            uint32_t x[8];
            tree_ld<8>(at, x);
#pragma unroll 1
            for (int c = 0; c < NCW / 8; ++c) {
              float y[8];
              tree_wait_ld<8>(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(x[i]);
              if (c + 1 < NCW / 8) tree_ld<8>(at + 8 * (c + 1), x);
              if (a.cap2 > 0.f) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = tree_cap(y[i] + w.c0[8 * c + i], a.cap2, k2);
              }
              if (a.slopes) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = fmaf(w.slope[8 * c + i], (float)(tok - w.pos[8 * c + i]), y[i]);
              }
              put(c, y);
            }
          }
          tc_fence_before();
          arrive(sm.s_ready[u]);  // for the row after the next
          fence_proxy_async_smem();
          arrive(p_ready);
          continue;
        }
        // a chunk with scaled columns: the scales taken off S in place, in little code (as part of tree_scores, loud queries
        // on 64 columns take 149 us for 136, 8 x 32768 tokens, where no column is scaled either)
        if (kind < 0 && d.rk > 0) {
          const uint32_t at = tmem + lanes + kS + 64 * u + wg * NCW;
#pragma unroll 1
          for (int c = 0; c < NCW; c += 8) {
            uint32_t x[8];
            tree_ld<8>(at + c, x);
            tree_wait_ld<8>(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * w.sc[c + i]);
            tree_st<8>(at + c, x);
          }
          tc_wait_st();
        }
        float z[NCW];
        auto load = [&](auto use) {
          uint32_t x[NCW];
          if (d.rk > 0) {
            tree_ld<NCW>(tmem + lanes + kS + 64 * u + wg * NCW, x);
            tree_wait_ld<NCW>(x);
          } else {
#pragma unroll
            for (int j = 0; j < NCW; ++j) x[j] = 0u;
          }
          use(x);
        };
        auto scores = [&](auto abs) {
          load([&](const uint32_t(&x)[NCW]) { tree_scores<NCW, decltype(abs)::value, LARGE>(a, w, x, k2, plain, masked, tok, z); });
        };
        float top = -INFINITY;
        if (bounded && plain) {
          load([&](const uint32_t(&x)[NCW]) {
#pragma unroll
            for (int j = 0; j < NCW; ++j) z[j] = __uint_as_float(x[j]);
          });
          if (masked) {
#pragma unroll
            for (int j = 0; j < NCW; ++j)
              if (tok < w.lo[j] || tok >= w.hi[j]) z[j] = -INFINITY;
          }
        } else {
          scores(std::false_type{});
          if (!bounded) {
#pragma unroll
            for (int j = 0; j < NCW; ++j) top = fmaxf(top, z[j]);
          }
        }
        if (!bounded && wg_any(wg, top > kTreeTau)) {
          // the columns' maxima over the row, new references where they are exceeded
          scores(std::true_type{});
          const float mine = tree_reduce<NCW>(z, [](float p, float q) { return fmaxf(p, q); });
          w.red[wq][tree_owned<NCW>(lane)] = mine;
          wg_sync(wg);
          if (t < NCW) {
            const float best = fmaxf(fmaxf(w.red[0][t], w.red[1][t]), fmaxf(w.red[2][t], w.red[3][t]));
            const float ref = w.ref[t];
            float al = 1.f;
            if (best > ref + kTreeTau && best < INFINITY) {
              const float r = best;
              al = ex2_approx(ref - r);
              w.ref[t] = r;
              w.sub[t] = plain ? w.c0[t] - r : r;
            }
            w.alpha[t] = al;
          }
          wg_sync(wg);
          if (k > 0) {
            wait(sm.pv_done[(n - 1) % 3], ((n - 1) / 3) & 1);
            tc_fence_after();
#pragma unroll 1
            for (int at = kO; at <= (d.rv == kD ? kL : kO); at += kL - kO) {
              uint32_t o[NCW];
              tree_ld<NCW>(tmem + lanes + at + wg * NCW, o);
              tree_wait_ld<NCW>(o);
#pragma unroll
              for (int j = 0; j < NCW; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * w.alpha[j]);
              tree_st<NCW>(tmem + lanes + at + wg * NCW, o);
            }
            tc_wait_st();
          }
          scores(std::false_type{});
        }
        tc_fence_before();
        arrive(sm.s_ready[u]);  // for the row after the next
#pragma unroll
        for (int c = 0; c < NCW / 8; ++c) {
          float y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = z[8 * c + i];
          put(c, y);
        }
        fence_proxy_async_smem();
        arrive(p_ready);
      }
      // ---- the part's sums ----
      const int last = n - 1;
      float* part = a.part + (d.slot * NC + wg * NCW) * kTreePart;
      wait(sm.pv_done[last % 3], (last / 3) & 1);
      tc_fence_after();
      uint32_t o[NCW];
      tree_ld<NCW>(tmem + lanes + kO + wg * NCW, o);
      tree_wait_ld<NCW>(o);
      const int ch = (t + 64) & 127;
#pragma unroll
      for (int j = 0; j < NCW; ++j)
        if (j < live) {
          if (ch < d.rv) part[j * kTreePart + 4 + ch] = __uint_as_float(o[j]);
          if (ch == d.rv)  // the row of halves
            *reinterpret_cast<float2*>(part + j * kTreePart) = make_float2(w.ref[j], 2.f * __uint_as_float(o[j]));
        }
      if (d.rv == kD && wq == 0) {  // l's rows are equal: lane 0 has one
        tree_ld<NCW>(tmem + kL + wg * NCW, o);
        tree_wait_ld<NCW>(o);
#pragma unroll
        for (int j = 0; j < NCW; ++j)
          if (j < live && lane == 0)
            *reinterpret_cast<float2*>(part + j * kTreePart) = make_float2(w.ref[j], __uint_as_float(o[j]));
      }
      tc_fence_before();
      arrive(sm.o_empty);
      arrive(sm.seg_empty[seg & 1]);
    }
  }
  // only now: CTAs of the kernels behind that came early would keep a later call's CTAs from their SMs (8 x 32768
  // tokens, 16 drafted: 150 us a call, 173 with the launch at the start of this kernel and the one before it)
  grid_dep_launch();
  if (!ok && lane == 0) {
    sm.fail = 1;
    atomicOr(&g_status, 1u);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (sm.fail && (warp == kMmaWarp || warp == kMmaWarp + 1) && lane == 0) {
    // after an expired wait: products and copies in flight are given time to land before the shared memory
    // and TMEM go away
    tc_commit(bar(sm.drain));
    mbar_wait_bounded(bar(sm.drain), 0, 1000000ull);
    for (int par = 0; par < 2; ++par) {
      for (int i = 0; i < 2; ++i) mbar_wait_bounded(bar(sm.seg_full[i]), par, 1000000ull);
      for (int i = 0; i < kTreeRing; ++i) {
        mbar_wait_bounded(bar(sm.kf[i]), par, 1000000ull);
        mbar_wait_bounded(bar(sm.vf[i]), par, 1000000ull);
      }
    }
  }
  __syncthreads();
  if (warp == 0) {
    __syncwarp();
    tmem_dealloc(tmem, 512);
  }
}

// ---------------------------------------------------------------------------------------
// Combine: grid (head, sequence, 8 columns), one warp per column for the weights; then thread = channel quad x
// column for the weighted sums of the parts, and warp = every eighth channel, lane = four dimensions for the
// back-projection, whose sums meet in shared memory.  A chain of memory round trips (layout, parts), so each
// step's loads go out together; the basis is in registers and the mean asked for ahead of the wait for the scan (its
// CTAs, past their own wait when they let this kernel start, came behind whatever wrote the parameters).
// ---------------------------------------------------------------------------------------
constexpr int kTreeCombine = 8;      // columns of a CTA
constexpr int kTreeParts = 192;      // parts of a unit at most: the scan's CTAs
__global__ void __launch_bounds__(256) tree_combine_kernel(TreeArgs a) {
  __shared__ float wt[kTreeCombine][kTreeParts];
  __shared__ int list[kTreeParts];
  __shared__ float wd_s[kTreeCombine], pc_s[kTreeCombine];
  __shared__ __align__(16) float zbar[kTreeCombine][kD];
  __shared__ __align__(16) float sums[8][kTreeCombine][kD];  // per warp
  __shared__ int n_list;
  grid_dep_launch();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.group;
  const int cols = a.max_draft * G, per = (cols + kTreeCombine - 1) / kTreeCombine;
  const int c0 = (int)(blockIdx.x % per) * kTreeCombine;
  const int s = (int)(blockIdx.x / per % a.n_seqs), head = (int)(blockIdx.x / per / a.n_seqs);
  bool known;
  const HeadEntry hv = tree_head(a, a.v_head0, head, known);
  const float* pool = param_pool(a.block);
  const float4* W = reinterpret_cast<const float4*>(pool + hv.w_off) + lane;
  constexpr int kRows = kD / 8;
  float4 wv[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) wv[k] = 8 * k + warp < hv.r ? __ldg(W + (8 * k + warp) * (kD / 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
  const int dim = tid & 127;
  const float mu = known ? pool[hv.mu_off + dim] : 0.f;
  grid_dep_wait();
  const int layer = head / a.n_kv, kv = head % a.n_kv;
  // the parts of the columns' unit: CTAs first .. last, less those that have no row of it
  const int tile = c0 / a.nc, n = a.rows[s];
  const long long unit = ((long long)head * a.n_seqs + s) * a.tiles + tile;
  const TreeLine line(a);
  const long long w0 = a.wpre[head], w1 = a.wpre[head + 1], r0 = a.rpre[s];
  const int live = min(kTreeCombine, tree_drafts(a, s, false) * G - c0);
  if (live <= 0) return;
  if (warp == 0) {
    int count = 0;
    if (n > 0) {
      const int w = (int)(w1 - w0);
      const long long base = w0 * line.rows + (r0 + (long long)tile * n) * w, end = base + (long long)(n - 1) * w;
      int first = (int)((float)base / (float)line.total * a.ctas);  // near enough: at most one off
      first = max(0, min(first, a.ctas - 1));
      while (first > 0 && line.begin(first) > base) --first;
      for (int c = first + lane; ; c += 32) {
        const bool in = c < a.ctas && line.begin(c) <= end;
        const bool has = in && TreeLine::before(line.begin(c), base, n, w) < TreeLine::before(line.begin(c + 1), base, n, w);
        const unsigned m = __ballot_sync(0xffffffffu, has);
        const int at = count + __popc(m & ((1u << lane) - 1u));
        if (has && at < kTreeParts) list[at] = c;
        count += __popc(m);
        if (!__all_sync(0xffffffffu, in)) break;
      }
    }
    if (lane == 0) n_list = min(count, kTreeParts);
  }
  __syncthreads();
  const int np = n_list;
  auto part = [&](int k, int col) { return a.part + ((list[k] + unit) * a.nc + (c0 + col) % a.nc) * kTreePart; };
  const float* draft = a.kd ? a.draft + (((long long)head * a.n_seqs + s) * cols + c0) * kTreePart : nullptr;
  // the drafted part's values of the thread's outputs
  float dv[4] = {};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c8 = 4 * (tid >> 7) + k;
    if (draft && c8 < live) dv[k] = draft[c8 * kTreePart + 4 + dim];
  }
  if (warp < live) {
    const float2 dr = draft ? *reinterpret_cast<const float2*>(draft + warp * kTreePart) : make_float2(-INFINITY, 0.f);
    const TreeCol* col = a.col + unit * a.nc + (c0 + warp) % a.nc;
    const int cached = col->hi > col->lo, bad = col->bad;
    float M = dr.x, l = 0.f;
    constexpr int kAt = kTreeParts / 32;
    float2 ml[kAt];
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      ml[k] = lane + 32 * k < np ? *reinterpret_cast<const float2*>(part(lane + 32 * k, warp)) : make_float2(-INFINITY, 0.f);
      if (ml[k].y == 0.f) ml[k].x = -INFINITY;  // (a bounded column has its reference whether it sees a token or not)
      M = fmaxf(M, ml[k].x);
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      const float e = ml[k].y == 0.f ? 0.f : exp2f(ml[k].x - M);
      l = fmaf(e, ml[k].y, l);  // (a sum that is not finite stays so)
      ml[k].x = e;
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    const float wd = dr.y == 0.f ? 0.f : exp2f(dr.x - M);
    const float sum = fmaf(wd, dr.y, l);
    // NaN: the combined scores are not finite, all of them are -inf, or their sum is not a number
    const float inv = !cached && dr.y == 0.f ? 0.f
                      : bad || M <= kTreeLowest || !(sum > 0.f && sum < INFINITY) ? __int_as_float(0x7fffffff) : 1.f / sum;
#pragma unroll
    for (int k = 0; k < kAt; ++k)
      if (lane + 32 * k < np) wt[warp][lane + 32 * k] = ml[k].x * inv;
    if (lane == 0) {
      wd_s[warp] = dr.y == 0.f ? -1.f : wd * inv;  // (a value that is not finite shows whatever its weight)
      pc_s[warp] = l * inv;
    }
  }
  __syncthreads();
  {  // rank-space averages (deviations from the code centre)
    const int cq = lane, c8 = warp;  // channels 4 cq .. 4 cq + 3
    float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c8 < live && 4 * cq < hv.r) {
#pragma unroll 8
      for (int k = 0; k < np; ++k) {
        // (an empty part's values may never have been written: asked for all the same, so that the loads of
        // several parts go out together, and passed over)
        const float w = wt[c8][k];
        const float4 x = *reinterpret_cast<const float4*>(part(k, c8) + 4 + 4 * cq);
        if (w > 0.f) z.x = fmaf(w, x.x, z.x), z.y = fmaf(w, x.y, z.y), z.z = fmaf(w, x.z, z.z), z.w = fmaf(w, x.w, z.w);
      }
    }
    const float f = hv.delta;
    const float e[4] = {f * z.x, f * z.y, f * z.z, f * z.w};
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = 4 * cq + k < hv.r ? e[k] : 0.f;
    *reinterpret_cast<float4*>(&zbar[c8][4 * cq]) = make_float4(y[0], y[1], y[2], y[3]);
  }
  __syncthreads();
  float o[kTreeCombine][4] = {};
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (8 * k + warp >= hv.r) break;
#pragma unroll
    for (int c = 0; c < kTreeCombine; ++c) {
      const float z = zbar[c][8 * k + warp];
      o[c][0] = fmaf(wv[k].x, z, o[c][0]), o[c][1] = fmaf(wv[k].y, z, o[c][1]);
      o[c][2] = fmaf(wv[k].z, z, o[c][2]), o[c][3] = fmaf(wv[k].w, z, o[c][3]);
    }
  }
#pragma unroll
  for (int c = 0; c < kTreeCombine; ++c)
    *reinterpret_cast<float4*>(&sums[warp][c][4 * lane]) = make_float4(o[c][0], o[c][1], o[c][2], o[c][3]);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c8 = 4 * (tid >> 7) + k, col = c0 + c8;
    if (c8 >= live) continue;
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) y += sums[w][c8][dim];
    y = fmaf(mu, pc_s[c8], y);
    if (wd_s[c8] >= 0.f) y = fmaf(dv[k], wd_s[c8], y);
    a.out[layer * a.o_sl + (long long)s * a.o_ss + (long long)(col / G) * a.o_st + (kv * G + col % G) * kD + dim] = __float2bfloat16_rn(y);
  }
}

}  // namespace cobra
