// Packed code rows into the tensor cores' A operand in TMEM, as exact 16-bit deviations from the code centre.
#pragma once

#include "tc.cuh"

namespace cobra {

// 8 consecutive TMEM columns of the warp's 32 lanes: column (taddr + j) of this lane = v[j]
__device__ __forceinline__ void tc_st32x8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(v[0]),
               "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// named barrier of a warpgroup, and the same returning whether `p` holds in any of its threads
__device__ __forceinline__ void wg_sync(int wg) { asm volatile("bar.sync %0, 128;" ::"r"(1 + wg) : "memory"); }
__device__ __forceinline__ bool wg_any(int wg, bool p) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n bar.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((int)p), "r"(1 + wg)
      : "memory");
  return r != 0;
}

// The codes of token t of a K row into the A operand: TMEM lane t, column s = channels (2 s, 2 s + 1),
// nk tiles of 8 columns.  Codes of strips past the row are whatever the buffer holds (finite, against
// zero columns of W').  The rotation brings the code to mantissa bit 1; what wraps around is masked.
template <int B>
__device__ __forceinline__ void tc_unpack_k_row(const uint8_t* krow, int nk, int t, uint32_t a_tmem) {
  const int p = t & 7, rho = 2 * (t >> 4) + ((t >> 3) & 1);
  const int wi = (rho * B) >> 4, off = (rho * B) & 15, nlo = min(B, 16 - off), rot = (off + 31) & 31;
  const uint32_t m0 = (((1u << nlo) - 1u) << 1) * 0x00010001u;
  const uint32_t m1 = ((((1u << B) - 1u) & ~((1u << nlo) - 1u)) << 1) * 0x00010001u;
  const __half2 cen = __float2half2_rn(512.f + (float)(1 << (B - 1)) - 0.5f);
  const uint8_t* src = krow + p * 4 * B + 4 * wi;
  const int next = wi + 1 < B ? 4 : 0;
#pragma unroll 2
  for (int kt = 0; kt < nk; ++kt) {
    uint32_t v[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const uint8_t* w = src + (8 * kt + s) * 32 * B;
      const uint32_t x = *reinterpret_cast<const uint32_t*>(w);
      uint32_t c = (__funnelshift_r(x, x, rot) & m0) | 0x60006000u;
      if constexpr (16 % B != 0)  // a code may straddle two words
        c |= (*reinterpret_cast<const uint32_t*>(w + next) << (nlo + 1)) & m1;
      const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&c), cen);
      v[s] = *reinterpret_cast<const uint32_t*>(&h);
    }
    tc_st32x8(a_tmem + 8 * kt, v);
  }
}
__device__ __forceinline__ void tc_unpack_k(int b, const uint8_t* krow, int nk, int t, uint32_t a_tmem) {
  switch (b) {
    case 1: tc_unpack_k_row<1>(krow, nk, t, a_tmem); break;
    case 2: tc_unpack_k_row<2>(krow, nk, t, a_tmem); break;
    case 3: tc_unpack_k_row<3>(krow, nk, t, a_tmem); break;
    case 4: tc_unpack_k_row<4>(krow, nk, t, a_tmem); break;
    case 5: tc_unpack_k_row<5>(krow, nk, t, a_tmem); break;
    case 6: tc_unpack_k_row<6>(krow, nk, t, a_tmem); break;
    case 7: tc_unpack_k_row<7>(krow, nk, t, a_tmem); break;
    default: tc_unpack_k_row<8>(krow, nk, t, a_tmem); break;
  }
}

// ---------------------------------------------------------------------------------------
// Codes to 16-bit floats.  A code is masked into mantissa bits [k, k + b) of a float with base 2^(m - k) (m
// mantissa bits: 10 of f16, 7 of bf16), which reads 2^(m - k) + code, and the base and the code centre are
// subtracted: exact, because the centred code has b bits and k >= 1 leaves one for its half.
// ---------------------------------------------------------------------------------------
// The pairs 2^(m - k), one register each: mask and base as two immediates would take two instructions.  top: the
// pair of k = 0, from a kernel argument (a constant that the compiler knows becomes an immediate again).
template <int M>
struct Bases {
  uint32_t r[M];
  __device__ __forceinline__ explicit Bases(uint32_t top) {
#pragma unroll
    for (int k = 0; k < M; ++k) r[k] = top - (uint32_t)(k << M) * 0x00010001u;
  }
};
constexpr uint32_t kTopF16 = 0x64006400u, kTopBf16 = 0x43004300u;  // 2^10 in f16, 2^7 in bf16

// Codes of a window of a 16-bit sub-stream pair that begins at bit `Base` of each half: registers u = 0 .. N - 1
// hold codes u (both sub-streams), centred.  Base 1 (b <= 2) needs no shifts.
template <int B, int Base, int N>
__device__ __forceinline__ void tc_window(uint32_t x, uint32_t (&v)[N], const Bases<10>& bases) {
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int o = Base + u * B, sh = o == 0 ? -1 : o + B <= 10 ? 0 : o >= 7 && o - 6 + B <= 10 ? 6 : 3, k = o - sh;
    static_assert(Base == 1 ? B <= 2 : Base == 0, "places checked for these");
    const uint32_t y = sh < 0 ? x << -sh : x >> sh;
    const uint32_t c = (y & pair_mask(B, k)) | bases.r[k];
    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&c),
                              __float2half2_rn((float)(1 << (10 - k)) + (float)(1 << (B - 1)) - 0.5f));
    v[u] = *reinterpret_cast<const uint32_t*>(&h);
  }
}

// ---------------------------------------------------------------------------------------
// V rows: thread = channel (TMEM lane), column c = tokens (2 c, 2 c + 1), as bf16 (see tree.cuh: the
// probabilities they meet are bf16 for its range).  A channel's codes are the bytes [16 b i, 16 b (i + 1)) of
// the row: pieces q = 0..3 of its parity; register rho of piece q is column 4 rho + q.
// ---------------------------------------------------------------------------------------
template <int B>
struct VPlace {
  static constexpr int kTop = 7 - (B < 7 ? B : 6);  // the highest k
  __host__ __device__ static constexpr int off(int rho) { return (rho * B) & 15; }
  __host__ __device__ static constexpr bool straddles(int rho) { return off(rho) + B > 16; }
  // right shift of the word (negative: left), shared by neighbouring codes where they fit
  __host__ __device__ static constexpr int shift(int rho) {
    const int o = off(rho);
    return straddles(rho) ? o - kTop : o == 0 ? -1 : (o - 1) / kTop * kTop;
  }
  __host__ __device__ static constexpr int k(int rho) { return off(rho) - shift(rho); }
};
template <int B>
__device__ __forceinline__ uint32_t tc_centred(const uint32_t (&w)[B], int rho, const Bases<7>& bases) {
  const int wi = (rho * B) >> 4, o = (rho * B) & 15;
  if constexpr (B <= 6) {
    const int k = VPlace<B>::k(rho), sh = VPlace<B>::shift(rho);
    const uint32_t x = sh < 0 ? w[wi] << -sh : w[wi] >> sh;
    uint32_t v;
    if (VPlace<B>::straddles(rho)) {
      const int lo = 16 - o;  // bits of the code in this word
      const uint32_t y = w[wi + 1 < B ? wi + 1 : wi] << (k + lo);
      v = (x & pair_mask(lo, k)) | (y & pair_mask(B - lo, k + lo)) | bases.r[k];
    } else {
      v = (x & pair_mask(B, k)) | bases.r[k];
    }
    const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v),
                                     __float2bfloat162_rn((float)(1 << (7 - k)) + (float)(1 << (B - 1)) - 0.5f));
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {  // 7 and 8 bits leave no bit for the half: by way of fp32
    uint32_t c = (w[wi] >> o) & pair_mask(B < 16 - o ? B : 16 - o, 0);
    if (o + B > 16) c |= (w[wi + 1 < B ? wi + 1 : wi] << (16 - o)) & pair_mask(o + B - 16, 16 - o);
    const float cen = (float)(1 << (B - 1)) - 0.5f;
    return pack_bf16((float)(c & 0xFFFFu) - cen, (float)(c >> 16) - cen);
  }
}
// One or two bits: four codes of each piece at a time in a rolled loop.  (Each kind of warp of the scan runs code
// of its own; straight-line code of a few hundred instructions each does not stay in the instruction caches.)
template <int B>
__device__ __forceinline__ void tc_unpack_v_small(const uint8_t* src, uint32_t a_tmem, uint32_t top) {
  static_assert(B == 1 || B == 2, "whole windows of four codes in a word");
  const Bases<7> bases(top);
  const uint4 u = reinterpret_cast<const uint4*>(src)[0];
  uint4 n = u;
  if constexpr (B == 2) n = reinterpret_cast<const uint4*>(src)[1];
  // words of the four pieces, turned a bit up: code u of a window begins at bit 1 + u b of each half
  auto up = [](uint32_t x) { return __funnelshift_l(x, x, 1); };
  uint32_t w[4] = {up(u.x), up(B == 1 ? u.y : u.z), up(B == 1 ? u.z : n.x), up(B == 1 ? u.w : n.z)};
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t v[16];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int o = 1 + i * B, sh = o + B <= 7 ? 0 : 5, k = o - sh;
        const uint32_t x = ((w[q] >> sh) & pair_mask(B, k)) | bases.r[k];
        const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x),
                                         __float2bfloat162_rn((float)(1 << (7 - k)) + (float)(1 << (B - 1)) - 0.5f));
        v[4 * i + q] = *reinterpret_cast<const uint32_t*>(&h);
      }
      w[q] = __funnelshift_r(w[q], w[q], 4 * B);
    }
    if (B == 2 && c == 1) w[0] = up(u.y), w[1] = up(u.w), w[2] = up(n.y), w[3] = up(n.w);
    tc_st32x16(a_tmem + 16 * c, v);
  }
}
template <int B>
__device__ __forceinline__ void tc_unpack_v_row(const uint8_t* src, uint32_t a_tmem, uint32_t top) {
  const Bases<7> bases(top);
  uint32_t w[4][B];
#pragma unroll
  for (int n = 0; n < B; ++n) {
    const uint4 u = reinterpret_cast<const uint4*>(src)[n];
    const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[(4 * n + i) / B][(4 * n + i) % B] = x[i];
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {  // rho 4 c .. 4 c + 3
    uint32_t v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = tc_centred<B>(w[u & 3], 4 * c + (u >> 2), bases);
    tc_st32x16(a_tmem + 16 * c, v);
  }
}
// src: the channel's 16 b bytes
template <int B>
__device__ __forceinline__ void tc_unpack_v(const uint8_t* src, uint32_t a_tmem, uint32_t top) {
  if constexpr (B <= 2)
    tc_unpack_v_small<B>(src, a_tmem, top);
  else
    tc_unpack_v_row<B>(src, a_tmem, top);
}

// ---------------------------------------------------------------------------------------
// K rows, by pieces: warp w of four takes the tokens 32 w .. 32 w + 31 (its TMEM lanes), which are codes
// rho = 4 w .. 4 w + 3 of the 8 pieces of every strip.  Lane (g, j) = (lane / 4, lane % 4) reads piece g of
// strips j and j + 4 of a tile of 8 strips, one or two words each, so that a word gives four registers (a
// token per thread would use one code pair of each word).  The registers are stored by 16x256b: lanes g, g + 8
// of each half of the warp's lanes, columns 2 j and 2 j + 1: column 2 s holds strip s < 4 of a tile, column
// 2 s + 1 strip s + 4 (tc_k_channel).
// ---------------------------------------------------------------------------------------
// channel at place p of the 16 elements of a tile
__host__ __device__ constexpr int tc_k_channel(int p) {
  const int c = (p & 15) >> 1;
  return (p & ~15) | (2 * ((c >> 1) + 4 * (c & 1)) + (p & 1));
}
__device__ __forceinline__ void tc_st16x256(uint32_t taddr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x1.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r0), "r"(r1), "r"(r2),
               "r"(r3)
               : "memory");
}
// where a warp finds its N codes of b bits in a piece, from bit x of the sub-streams
template <int B, int N>
struct KFetch {
  static constexpr int Base = B <= 2 ? 1 : 0;
  static constexpr bool two = 16 % (N * B) != 0;  // the codes may straddle two words
  struct Raw {
    uint32_t x, y;
  };
  int wi, wj;         // words
  int rot;            // right rotation of the first
  int up;             // left shift of the second
  uint32_t m0, m1;
  __device__ explicit KFetch(int x) {
    const int off = x & 15, lo = min(N * B, 16 - off);
    wi = x >> 4;
    wj = lo < N * B ? wi + 1 : wi;
    rot = (off - Base) & 31;
    up = lo;
    m0 = ((1u << lo) - 1u) * 0x00010001u;
    m1 = (((1u << (N * B)) - 1u) & ~((1u << lo) - 1u)) * 0x00010001u;
  }
  __device__ __forceinline__ Raw load(const uint8_t* piece) const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(piece);
    return Raw{w[wi], two ? w[wj] : 0u};
  }
  __device__ __forceinline__ uint32_t operator()(const Raw& r) const {
    if constexpr (!two) return __funnelshift_r(r.x, r.x, rot);
    return ((r.x >> rot) & m0) | ((r.y << up) & m1);
  }
};
// The unpacking of K rows of width B by warp `warp` of four.
template <int B>
struct KUnpack {
  static constexpr int N = B <= 4 ? 4 : 2, F = 4 / N;  // codes per fetch, fetches per strip
  using Fetch = KFetch<B, N>;
  Fetch f[2];
  Bases<10> bases;
  int at;  // the lane's first piece in a row
  __device__ __forceinline__ KUnpack(int warp, uint32_t top)
      : f{Fetch(4 * warp * B), Fetch(4 * warp * B + (F - 1) * 2 * B)}, bases(top),
        at((threadIdx.x & 3) * 32 * B + ((threadIdx.x & 31) >> 2) * 4 * B) {}
  __device__ __forceinline__ void operator()(const uint8_t* krow, int nk, uint32_t a_tmem) const {
    const uint8_t* src = krow + at;
    typename Fetch::Raw raw[2][F];  // the next tile's words are loaded ahead of this one's stores
    auto load = [&] {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < F; ++i) raw[s][i] = f[i].load(src + s * 4 * 32 * B);
      src += 8 * 32 * B;
    };
    load();
#pragma unroll 1
    for (int kt = 0; kt < nk; ++kt) {
      uint32_t x[2][F];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < F; ++i) x[s][i] = f[i](raw[s][i]);
      if (kt + 1 < nk) load();
      uint32_t v[2][4];  // [strip j, j + 4][rho]
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if constexpr (N == 4) {
          tc_window<B, Fetch::Base, 4>(x[s][0], v[s], bases);
        } else {
          uint32_t a[2], b[2];
          tc_window<B, 0, 2>(x[s][0], a, bases);
          tc_window<B, 0, 2>(x[s][F - 1], b, bases);
          v[s][0] = a[0], v[s][1] = a[1], v[s][2] = b[0], v[s][3] = b[1];
        }
      }
      tc_st16x256(a_tmem, v[0][0], v[1][0], v[0][1], v[1][1]);
      tc_st16x256(a_tmem + (16u << 16), v[0][2], v[1][2], v[0][3], v[1][3]);
      a_tmem += 8;
    }
  }
};

}  // namespace cobra
