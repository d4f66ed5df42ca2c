// Attention over the paged cache (the kernel template; one translation unit per
// cache format instantiates it).
//
//   o_i = sum_j softmax_j(q_i . K_j / sqrt(dh)) V_j
//
// over a sequence's cached tokens j, or over those of the pages listed for row
// i, of a window up to the row's own token, or of a context and the drafted tokens that
// the row's mask names (PagedLook).  The rows of one sequence that share a key head (its query heads times
// the sequence's rows, "packed rows") form tiles of 16; a workgroup takes up
// to RT tiles and a range of the keys, its wavefronts alternating 32-key
// tiles.  Per 32 keys a wavefront forms S^T = K Q^T (16 keys x 16 rows per
// instruction), so that lane (c, g) holds row c's logits of keys 4g .. 4g + 3
// of both 16-key halves; these eight are just the reduction slots that the
// second product O^T += V^T P^T wants from the lane, if V^T's slots name the
// same keys: P never leaves the lane, the row maximum takes two lane swaps,
// and the rescale is a per-lane scalar.  V^T's operand wants eight keys of one
// channel per lane where a row of memory has the channels side by side: a lane
// loads four (head width 128: eight) channels of its eight keys and
// transposes them among its own registers, one byte permutation per two
// elements.  The main loop has no barrier: a wavefront keeps the next tile's loads
// in flight while it computes, and meets the others only when their parts are
// joined at the end.
//
// K's operand wants 16 keys side by side in the lanes, whose rows lie apart: read
// straight from memory, 16 neighbouring lanes touch 16 lines.  Where a wavefront
// has 32 rows or float32 ones, rows of more than 64 bytes are therefore loaded
// in order, whole lines at a time, and change places in LDS of the wavefront's own
// (paged_stage; 4 x 16 heads of 64 bf16, 512 rows over 4096 tokens: 90.9 us
// straight, 65.6 staged; int8 rows of 80, 36 .. 100 rows over 1088 tokens:
// 62.4, 44.5).  Rows of 64 bytes lose by it (38.7, 39.9), and for 16 rows memory is
// the bound either way (one row over 64 caches of 4096 tokens: 176.8, 178.6).
//
// Softmax statistics and O are float32; the maximum that P is taken against
// trails the true one by at most 2^8, which saves most rescales.  P is rounded
// to bf16 (half a step, 2^-8 of each weight; the products' other operand V is
// exact in bf16 for every format, int8 with its exponent in P).  float32 rows are
// split into three bf16 parts (24 bits, nothing lost) and so is P; infinite keys
// and values meet the first parts only (a second pass, where there are any).
//
// Bound: single rows by the cache's bytes (16 int8 caches of 4000 .. 32768
// tokens, 607 MB: 119 us, 118 at a copy's rate); many rows by the latency of
// loads and of dependent instructions at two or three wavefronts a SIMD (100
// rows over 32 caches of 1088 bf16 tokens: 49 us; all from the same few pages
// 36, without loads 27, and without exponentials no less).  Handing page ids
// on from tile to tile, or loading two tiles ahead, took no less time.
#pragma once

#include <algorithm>
#include <type_traits>

#include "paged_device.h"
#include "paged_walk.h"

namespace marche {

// Two bf16 (or the high halves of two floats) from dwords a and b.
__device__ __forceinline__ uint32_t lo16(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t hi16(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

__device__ __forceinline__ uint32_t as_u32(bf16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// Largest over the four lanes that share c (lanes c, c + 16, c + 32, c + 48).
__device__ __forceinline__ float quad_max(float v) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// Global memory at a uniform address that the compiler takes as it is.
typedef __attribute__((address_space(1))) char gbyte;
__device__ __forceinline__ const gbyte *scalar(const void *p) {
  const gbyte *q = (const gbyte *)p;
  asm("" : "+s"(q));
  return q;
}
// (the lane offset is kept from being widened outside the loop, where the
// addressing mode would no longer be seen)
template <typename V>
__device__ __forceinline__ V at(const gbyte *p, uint32_t lane_offset, int offset) {
  asm("" : "+v"(lane_offset));
  return *(const __attribute__((address_space(1))) V *)(p + lane_offset + offset);
}

// Raw registers of 32 keys of a lane: K for its key c of each half (STAGE: every
// 64th piece of the half, in the order of memory), V for its eight keys,
// exponent bytes.
template <int FMT, int DH, bool STAGE>
struct KvRaw {
  static constexpr bool W = FMT == BF;               // 2-byte elements
  static constexpr int ES = W ? 2 : 1;
  static constexpr int KQ = W ? DH / 32 : DH / 64;   // 16-byte pieces per key and lane
  static constexpr int RB = DH * ES;                 // bytes of a row
  static constexpr int RP = RB / 16;                 // 16-byte pieces of a row
  static constexpr int KL = RB / 64;                 // whole-line loads of 16 keys: of 16 bytes,
  static constexpr int KT = RB % 64 / 16;            // and one more of KT dwords
  static constexpr bool T = DH % 32 != 0;            // a 16-channel tail (dh 80)
  static constexpr int NC = DH / 32 + T;             // 32-deep products of S; the tail fills half of one
  static constexpr int VC = DH == 128 ? 8 : 4;       // channels per lane
  static constexpr int VW = VC * ES / 4;             // dwords of them
  static constexpr int M = DH / 16;                  // 16-channel tiles of O
  static_assert(DH == 64 || DH == 80 || DH == 128, "head width");

  u32x4 k[2][KL];
  uint32_t kt[2][2];
  uint32_t v[8][VW];
  uint32_t vt[8];
  uint32_t ke[2], ve[2];  // ke: the byte of key c (e4m3), the four of keys 4g.. (int8)

  // half u of the tile: 16 tokens from `slot` (uniform) on
  __device__ __forceinline__ void load(int u, const void *kb, const void *vb, const uint8_t *kx,
                                       const uint8_t *vx, size_t slot, int c, int g) {
    // Uniform bases in scalar registers, lane offsets of 32 bits: left to itself
    // the compiler adds the lane offsets to the pool's base once and keeps a
    // 64-bit address per load (30 registers and eight additions per tile).
    const gbyte *kp = scalar(static_cast<const char *>(kb) + slot * (DH * ES));
    const gbyte *vp = scalar(static_cast<const char *>(vb) + slot * (DH * ES));
    if constexpr (!STAGE) {
      const uint32_t ko = (uint32_t)(c * RB + 16 * g), to = (uint32_t)(c * RB + 64 * ES + 4 * ES * g);
#pragma unroll
      for (int m = 0; m < KQ; ++m) k[u][m] = at<u32x4>(kp, ko, 64 * m);
      if constexpr (T && W) {
        const u32x2 y = at<u32x2>(kp, to, 0);
        kt[u][0] = y.x, kt[u][1] = y.y;
      } else if constexpr (T) {
        kt[u][0] = at<uint32_t>(kp, to, 0);
      }
    } else {
      const uint32_t lane = 16 * g + c;
#pragma unroll
      for (int m = 0; m < KL; ++m) {
        const uint32_t key = 64 / RP * m + lane / RP;  // (rows of 8 or 16 pieces)
        const uint32_t ko = RP % 8 ? 16 * lane : 16 * (lane ^ swizzle(key));
        k[u][m] = at<u32x4>(kp, ko, 1024 * m);
      }
      if constexpr (KT == 2) {
        const u32x2 y = at<u32x2>(kp, 8 * lane, 1024 * KL);
        kt[u][0] = y.x, kt[u][1] = y.y;
      } else if constexpr (KT == 1) {
        kt[u][0] = at<uint32_t>(kp, 4 * lane, 1024 * KL);
      }
    }
    const uint32_t vo = (uint32_t)(4 * g * DH * ES + c * VC * ES);
    const uint32_t vto = (uint32_t)(4 * g * DH * ES + 64 * ES + c * ES);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      uint32_t(&x)[VW] = v[4 * u + r];
      if constexpr (VW == 1) {
        x[0] = at<uint32_t>(vp, vo, r * DH * ES);
      } else if constexpr (VW == 2) {
        const u32x2 y = at<u32x2>(vp, vo, r * DH * ES);
        x[0] = y.x, x[1] = y.y;
      } else {
        const u32x4 y = at<u32x4>(vp, vo, r * DH * ES);
        x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
      }
      if constexpr (T) {
        if constexpr (W) vt[4 * u + r] = at<uint16_t>(vp, vto, r * DH * ES);
        else vt[4 * u + r] = at<uint8_t>(vp, vto, r * DH * ES);
      }
    }
    if constexpr (!W) {
      const gbyte *ep = scalar(kx + slot), *xp = scalar(vx + slot);
      if constexpr (FMT == E4) ke[u] = at<uint8_t>(ep, (uint32_t)c, 0);
      else ke[u] = at<uint32_t>(ep, (uint32_t)(4 * g), 0);
      ve[u] = at<uint32_t>(xp, (uint32_t)(4 * g), 0);
    }
  }
  // Piece i of key c's row lies at piece i ^ swizzle(c) in LDS, so that 8 keys' pieces i
  // are in different banks (rows of 80 channels are so by themselves, or nearly).
  static __device__ __forceinline__ uint32_t swizzle(uint32_t key) { return RP % 8 == 0 ? key % 8 : 0; }
  // K to the wavefront's LDS, rows side by side
  __device__ __forceinline__ void stage(char *s_k, int lane) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int m = 0; m < KL; ++m) *reinterpret_cast<u32x4 *>(s_k + 16 * RB * u + 1024 * m + 16 * lane) = k[u][m];
      char *rest = s_k + 16 * RB * u + 1024 * KL;
      if constexpr (KT == 2) *reinterpret_cast<u32x2 *>(rest + 8 * lane) = u32x2{kt[u][0], kt[u][1]};
      else if constexpr (KT == 1) *reinterpret_cast<uint32_t *>(rest + 4 * lane) = kt[u][0];
    }
  }
  // V of keys n .. 15 of half u becomes zero (they hold nothing, or another
  // sequence's leavings, which may not even be finite).
  __device__ __forceinline__ void clear(int u, int n, int g) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (4 * g + r >= n) {
#pragma unroll
        for (int w = 0; w < VW; ++w) v[4 * u + r][w] = 0u;
        if constexpr (T) vt[4 * u + r] = 0u;
        if constexpr (!W) ve[u] = (ve[u] & ~(0xFFu << (8 * r))) | (0x7Fu << (8 * r));
      }
  }
  // K of half u as operands: product n covers the eight channels from chan(n, g)
  // on (the tail's: four, and zeros; a 16-deep instruction of its own is no faster).
  __device__ __forceinline__ void keys(int u, const char *s_k, int c, int g, bf16x8 (&f)[NC]) const {
    u32x4 k[KQ];
    u32x2 kt = {this->kt[u][0], this->kt[u][1]};
    const char *row = s_k + 16 * RB * u + c * RB;
#pragma unroll
    for (int m = 0; m < KQ; ++m)
      k[m] = STAGE ? *reinterpret_cast<const u32x4 *>(row + 16 * ((4 * m + g) ^ swizzle(c))) : this->k[u][m];
    if constexpr (STAGE && T && W) kt = *reinterpret_cast<const u32x2 *>(row + 128 + 8 * g);
    if constexpr (STAGE && T && !W) kt.x = *reinterpret_cast<const uint32_t *>(row + 64 + 4 * g);
    if constexpr (W) {
#pragma unroll
      for (int n = 0; n < DH / 32; ++n) f[n] = __builtin_bit_cast(bf16x8, k[n]);
      if constexpr (T) f[NC - 1] = __builtin_bit_cast(bf16x8, u32x4{kt.x, kt.y, 0u, 0u});
    } else {
      const float sc = FMT == E4 ? exp_scale(ke[u]) : 1.f;
#pragma unroll
      for (int n = 0; n < DH / 32; ++n) {
        const uint32_t a = k[n / 2][2 * (n % 2)], b = k[n / 2][2 * (n % 2) + 1];
        f[n] = __builtin_bit_cast(bf16x8, u32x4{pair(a, sc, 0), pair(a, sc, 1), pair(b, sc, 0), pair(b, sc, 1)});
      }
      if constexpr (T)
        f[NC - 1] = __builtin_bit_cast(bf16x8, u32x4{pair(kt.x, sc, 0), pair(kt.x, sc, 1), 0u, 0u});
    }
  }
  // bytes 2 h, 2 h + 1 of a dword as two bf16 (e4m3: times the scale)
  static __device__ __forceinline__ uint32_t pair(uint32_t w, float sc, int h) {
    if constexpr (FMT == E4) {
      return h ? as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, true))
               : as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, false));
    } else {
      const float a = (float)(int8_t)(w >> (16 * h)), b = (float)(int8_t)(w >> (16 * h + 8));
      return hi16(__float_as_uint(a), __float_as_uint(b));  // at most 8 significant bits: exact
    }
  }
  // V^T of the eight keys as operands, tiles m and m + 1 (the last one of an
  // odd count alone): channels vchan(m, c), vchan(m + 1, c).
  __device__ __forceinline__ void values(int m, bf16x8 &f0, bf16x8 &f1) const {
    uint32_t o[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // keys 2 i and 2 i + 1
      const int a = 2 * i, b = a + 1, u = a / 4;
      const float sa = FMT == E4 ? exp_scale((ve[u] >> (8 * (a % 4))) & 0xFFu) : 1.f;
      const float sb = FMT == E4 ? exp_scale((ve[u] >> (8 * (b % 4))) & 0xFFu) : 1.f;
      if (T && m == M - 1) {
        if constexpr (FMT == I8)
          o[0][i] = hi16(__float_as_uint((float)(int8_t)vt[a]), __float_as_uint((float)(int8_t)vt[b]));
        else if constexpr (FMT == E4)
          o[0][i] = lo16(pair(vt[a], sa, 0), pair(vt[b], sb, 0));
        else
          o[0][i] = lo16(vt[a], vt[b]);
      } else if constexpr (FMT == I8) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          o[e][i] = hi16(__float_as_uint((float)(int8_t)(v[a][m / 4] >> (8 * (m % 4 + e)))),
                         __float_as_uint((float)(int8_t)(v[b][m / 4] >> (8 * (m % 4 + e)))));
      } else {
        uint32_t x, y;
        if constexpr (FMT == E4) x = pair(v[a][m / 4], sa, m / 2 % 2), y = pair(v[b][m / 4], sb, m / 2 % 2);
        else x = v[a][m / 2], y = v[b][m / 2];
        o[0][i] = lo16(x, y);
        o[1][i] = hi16(x, y);
      }
    }
    f0 = __builtin_bit_cast(bf16x8, u32x4{o[0][0], o[0][1], o[0][2], o[0][3]});
    if (!(T && m == M - 1)) f1 = __builtin_bit_cast(bf16x8, u32x4{o[1][0], o[1][1], o[1][2], o[1][3]});
  }
  // first channel of product n's eight in lane group g
  static __device__ __forceinline__ int chan(int n, int g) {
    return T && n == NC - 1 ? 64 + 4 * g : W ? 32 * n + 8 * g : 64 * (n / 2) + 16 * g + 8 * (n % 2);
  }
  // channel of row x of O's tile m
  static __device__ __forceinline__ int vchan(int m, int x) { return m < VC ? VC * x + m : 64 + x; }
};

// One bf16, or three whose sum is the float32 value: its first 8 bits cut off (rounded,
// the largest finite values would become infinite) and the 16 behind them in two
// parts (an infinity's are zero; a NaN's are NaN, should the first part not be).
template <int T>
__device__ __forceinline__ void split(float x, bf16 (&o)[T]) {
  static_assert(T == 1 || T == 3, "parts");
  if constexpr (T == 1) {
    o[0] = (bf16)x;
  } else {
    const float top = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
    o[0] = __builtin_bit_cast(bf16, (uint16_t)(__float_as_uint(x) >> 16));
    x = fabsf(x) == INFINITY ? 0.f : x - top;
    o[1] = (bf16)x;
    o[2] = (bf16)(x - (float)o[1]);
  }
}

// Eight bf16 with zeros for infinities and NaN.
__device__ __forceinline__ bf16x8 finite(bf16x8 x) {
  u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
    if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0xFFFFu;
  }
  return __builtin_bit_cast(bf16x8, w);
}

// Tokens that a row at token t sees of `len`: those of [lo, hi), and of [0, hi) those
// below the number of sinks (hi = 0: none).
__device__ __forceinline__ void window_of(const PagedAttnArgs &a, int len, int t, int &lo, int &hi) {
  hi = t < 0 ? 0 : min(t, len - 1) + 1;
  lo = t < 0 ? 0 : max(t - (a.window - 1), 0);
}
// Which of the 16 keys from `key` on these are, as bits.
__device__ __forceinline__ uint32_t below16(int n) { return n <= 0 ? 0u : n >= 16 ? 0xFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t window_bits(int lo, int hi, int sinks, int key) {
  return below16(hi - key) & (~below16(lo - key) | below16(sinks - key));
}
// Of a block's rows: the smallest and largest lo and hi (rows that see nothing
// count in hi_min and lo_max, so that no tile is taken to be whole for them).
struct Span {
  int lo_min, lo_max, hi_min, hi_max;
};
__device__ __forceinline__ Span span_of(const PagedAttnArgs &a, int len, int row, int rows, int lane) {
  int lo = 0, hi = 0;
  window_of(a, len, a.q_idx[row + min(lane, rows - 1)], lo, hi);
  // (none of them is negative)
  auto least = [](int v) { return (int)~wave_max_u32(~(uint32_t)v); };
  return Span{least(hi > 0 ? lo : INT32_MAX), (int)wave_max_u32((uint32_t)lo), least(hi), (int)wave_max_u32((uint32_t)hi)};
}
// Bits `at` .. at + 15 of a row's mask; those before bit 0 (the context) are set, those
// behind the last word are not.
__device__ __forceinline__ uint32_t tree_bits(const uint32_t *mask, int words, int at) {
  const int w = at >> 5;  // (-1 for the context's last tokens)
  if (w < -1) return 0xFFFFu;
  const uint32_t lo = w < 0 ? 0xFFFFFFFFu : w < words ? mask[w] : 0u;
  const uint32_t hi = w + 1 < words ? mask[w + 1] : 0u;
  return (uint32_t)((((uint64_t)hi << 32) | lo) >> (at & 31)) & 0xFFFFu;
}

// Whether K goes through LDS (the text above).
template <int FMT, int DH, int RT, typename RowT>
constexpr bool paged_stage = DH * (FMT == BF ? 2 : 1) > 64 && (RT == 2 || sizeof(RowT) == 4);

// Attention of a block's packed rows [p0, p1) over the tokens that each of them
// looks at, a wavefront per row, 16 keys at a time (lanes 0 .. 15 a key each):
// the plain loop, for blocks in which a row's masked keys have values that are not
// finite.  first(pos): the key at the block's position pos (a multiple of 16); look(i, key):
// whether row i sees it.  Slow: one such value among 36 .. 100 rows over 8 of 34 bf16
// pages makes the call take 1.9 ms for 72 us, in a prompt of 8192 rows over windows of 1024 9.1
// ms for 0.18 (4.5 and 27.9 with a channel and a key at a time).
template <int FMT, int DH, typename RowT, typename First, typename Look>
__device__ __forceinline__ void one_by_one(const PagedAttnArgs &a, const int32_t *tab, First first, Look look, int p0,
                                           int p1, int row0, int h, int split_i, int len, int pos0, int end, int wave,
                                           int waves, int lane) {
  const int page = 1 << a.page_log2;
  // eight channels of a key
  auto eight = [&](size_t slot, int d, float (&o)[8]) {
    if constexpr (FMT == BF) {
      load8(static_cast<const bf16 *>(a.k) + slot * DH + d, o);
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2 *>(static_cast<const char *>(a.k) + slot * DH + d);
      const float s = exp_scale(a.k_exp[slot]);
      unpack4<FMT>(w.x, s, o);
      unpack4<FMT>(w.y, s, o + 4);
    }
  };
  auto at = [&](const void *x, const uint8_t *ex, size_t slot, int d) {
    if constexpr (FMT == BF) return (float)static_cast<const bf16 *>(x)[slot * DH + d];
    const uint32_t q = static_cast<const uint8_t *>(x)[slot * DH + d];
    const float s = exp_scale(ex[slot]);
    return FMT == E4 ? __builtin_amdgcn_cvt_f32_fp8((int)q, 0) * s : (float)(int8_t)q * s;
  };
  for (int pr = p0 + wave; pr < p1; pr += waves) {
    const int i = (int)a.d_group.div(pr), hg = pr - i * a.group;
    const RowT *q = static_cast<const RowT *>(a.q) + (size_t)(row0 + i) * a.q_stride + (size_t)(h * a.group + hg) * DH;
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    bool seen = false;
#pragma unroll 1
    for (int pos = pos0; pos < end; pos += 16) {
      const int key = first(pos);
      const int n = min(len - key, 16);
      if (n <= 0) continue;
      const unsigned long long sees = __ballot(lane < n && look(i, key + lane));
      if (!sees) continue;
      const int phys = tab[key >> a.page_log2];
      if ((unsigned)phys >= (unsigned)a.n_pages) continue;
      const size_t slot = (((size_t)phys * a.n_heads + h) << a.page_log2) + (key & (page - 1));
      const bool mine = (sees >> lane) & 1u;
      seen = true;
      float s = 0.f;
      if (mine) {
#pragma unroll 1
        for (int d = 0; d < DH; d += 8) {
          float x[8], y[8];
          load8(q + d, x);
          eight(slot + lane, d, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
        }
        s *= a.sl2;
      }
      const float m_new = fmaxf(m, wave_max(mine ? s : -INFINITY));
      const float al = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      const float p = mine ? __builtin_amdgcn_exp2f(s - (m_new == -INFINITY ? 0.f : m_new)) : 0.f;
      m = m_new;
      l = l * al + wave_sum(p);
      acc[0] *= al;
      acc[1] *= al;
#pragma unroll 1
      for (int r0 = 0; r0 < n; r0 += 4) {
        float v[4][2];  // (loads of keys behind the last repeat it)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = min(r0 + u, n - 1);
          v[u][0] = at(a.v, a.v_exp, slot + r, lane);
          v[u][1] = at(a.v, a.v_exp, slot + r, DH > 64 ? min(lane + 64, DH - 1) : lane);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (r0 + u >= n || !((sees >> (r0 + u)) & 1u)) continue;
          const float w = __shfl(p, r0 + u, 64);
          acc[0] = fmaf(w, v[u][0], acc[0]);
          if (lane + 64 < DH) acc[1] = fmaf(w, v[u][1], acc[1]);
        }
      }
    }
    const size_t row = (size_t)(row0 + i) * (a.n_heads * a.group) + h * a.group + hg;
    const size_t part = (size_t)split_i * a.q_total * (a.n_heads * a.group) + row;
    const float inv = a.splits > 1 ? 1.f : seen ? 1.f / l : 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int d = lane + 64 * j;
      if (d >= DH) break;
      if (a.splits > 1) a.part_o[part * DH + d] = acc[j];
      else static_cast<RowT *>(a.o)[row * DH + d] = (RowT)(acc[j] * inv);
    }
    if (a.splits > 1 && lane == 0) {
      a.part_ml[2 * part] = m;
      a.part_ml[2 * part + 1] = seen ? l : -1.f;
    }
  }
}

// MODE: which keys a row sees (PagedLook).  (Trees of two row tiles of 128 bf16 stay within
// 256 registers, two wavefronts a SIMD, if they have to: 32 rows over 40 caches of 2000 tokens, 8 heads, 82.0 us
// otherwise, 71.5 so.  Windows spill then: 15.8 us become 21.6 with 30 .. 60 rows over 6 caches.)
template <int FMT, int DH, int RT, typename RowT, int MODE>
__global__ __launch_bounds__(RT == 1 ? 512 : 256, MODE == PAGED_TREE ? 2 : 1) void paged_attn_kernel(PagedAttnArgs a,
                                                                         const int32_t *__restrict__ table) {
  constexpr bool SEL = MODE == PAGED_LISTED, WIN = MODE == PAGED_WINDOW, TREE = MODE == PAGED_TREE;
  constexpr bool STAGE = paged_stage<FMT, DH, RT, RowT>;
  using Raw = KvRaw<FMT, DH, STAGE>;
  constexpr int TERMS = sizeof(RowT) == 4 ? 3 : 1;
  constexpr int NC = Raw::NC, M = Raw::M;
  constexpr int OS = DH + 4;              // row stride of the joined parts
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;

  // (sequence, key head, row block, key range): consecutive workgroup ids go
  // round the 8 XCDs, so (sequence, head) pairs are dealt to them one by one
  // and the blocks and ranges of a pair follow each other on its XCD, whose L2
  // they share.  (Contiguous sequences per XCD leave most XCDs idle at the end
  // where sequences differ.)
  int split_i, chunk = a.chunk, rb, b, h;
  if constexpr (WIN) {
    const PagedUnit u(a, blockIdx.x, a.n_seqs * a.n_heads);
    rb = u.block;
    split_i = u.split;
    b = (int)a.d_heads.div(u.pair);
    h = u.pair - b * a.n_heads;
  } else {
    const int at0 = blockIdx.x >> 3;
    const int at1 = a.d_splits.div(at0);
    const int at2 = a.d_blocks.div(at1);
    rb = at1 - at2 * a.row_blocks;
    const int pair = 8 * at2 + (blockIdx.x & 7);
    split_i = at0 - at1 * a.splits;
    b = a.d_heads.div(pair);
    h = pair - b * a.n_heads;
  }
  if (!SEL && !WIN && a.budget > 0) {
    if (b >= a.budget) return;
    const Shares sh(a, lane);
    chunk = sh.chunk;
    b = __builtin_amdgcn_readfirstlane(TREE ? sh.find_long_first(b, lane, split_i) : sh.find(b, lane, split_i));
    if (b < 0) return;
  } else if (b >= a.n_seqs) {
    return;
  }

  // The lists' entries that a workgroup starts from are loaded together: the
  // length, the rows and the page of its first tile (where that lies if the
  // sequence is long enough).
  const int page = 1 << a.page_log2;
  const int32_t *tab = table + (size_t)b * a.max_pages;
  int first = split_i * chunk + wave;
  const int ahead = SEL || WIN ? 0 : tab[min((32 * first) >> a.page_log2, a.max_pages - 1)];
  const int len = min(paged_len(a.lens[b], a.max_pages, a.page_log2), a.len_max);
  int row0 = b * a.rows_each, row1 = row0 + a.rows_each;  // the sequence's rows
  if (a.q_off) {
    row0 = min(max(a.q_off[b], 0), a.q_total);
    row1 = min(max(a.q_off[b + 1], row0), a.q_total);
  }
  const int packed = min(row1 - row0, a.q_max) * a.group;
  const int p0 = rb * 16 * RT;
  if (p0 >= packed) return;

  // LDS: joined O parts (before: the wavefront's staged keys, which need no
  // more), maxima and sums of every wavefront and the rows' places in the output
  // (several wavefronts only), then the page bits of the block's rows and the
  // list of pages that any of them looks at
  static_assert(32 * Raw::RB <= 16 * OS * 4, "staged keys in the place of O");
  float *s_o = reinterpret_cast<float *>(smem);             // [waves][RT*16][OS]
  char *s_k = reinterpret_cast<char *>(s_o + wave * RT * 16 * OS);
  float *s_m = s_o + (waves > 1 ? waves * RT * 16 * OS : STAGE ? 8 * Raw::RB : 0);  // [waves][RT*16]
  float *s_l = s_m + (waves > 1 ? waves * RT * 16 : 0);       // [waves][RT*16]
  int *s_row = reinterpret_cast<int *>(s_l + (waves > 1 ? waves * RT * 16 : 0));  // [RT*16]
  uint32_t *s_bits = reinterpret_cast<uint32_t *>(s_row + (waves > 1 ? RT * 16 : 0));
  const int words = TREE ? a.mask_words : (a.max_pages + 31) >> 5;
  auto row_of = [&](int p) { return (int)a.d_group.div(p); };  // a packed row's row
  const int i0 = row_of(p0), i1 = row_of(min(p0 + 16 * RT, packed) - 1);  // the block's rows
  uint32_t *s_any = s_bits + (SEL ? a.bit_rows * words : 0);
  uint16_t *s_list = reinterpret_cast<uint16_t *>(s_any + words);
  int n_list = 0;
  if constexpr (SEL) {
    const int rows = i1 - i0 + 1;
    for (int x = tid; x < rows * words; x += blockDim.x) s_bits[x] = 0u;
    __syncthreads();
    const int n_p = (len + page - 1) >> a.page_log2;
    for (int x = tid; x < rows * a.n_select; x += blockDim.x) {
      const int i = x / a.n_select, j = x - i * a.n_select;
      const int p = a.pages[((size_t)(row0 + i0 + i) * a.n_heads + h) * a.n_select + j];
      if (p >= 0 && p < n_p) atomicOr(&s_bits[i * words + (p >> 5)], 1u << (p & 31));
    }
    __syncthreads();
    for (int x = tid; x < words; x += blockDim.x) {
      uint32_t any = 0;
      for (int i = 0; i < rows; ++i) any |= s_bits[i * words + x];
      s_any[x] = any;
    }
    __syncthreads();
    // the union's pages in ascending order (every wavefront counts; the first writes)
    for (int x0 = 0; x0 < words; x0 += 64) {
      const uint32_t w = x0 + lane < words ? s_any[x0 + lane] : 0u;
      int before = __popc(w);
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(before, o, 64);
        if (lane >= o) before += y;
      }
      const int sum = __shfl(before, 63, 64);
      if (wave == 0) {
        int to = n_list + before - __popc(w);
        for (uint32_t v = w; v; v &= v - 1) s_list[to++] = (uint16_t)(32 * (x0 + lane) + __ffs(v) - 1);
      }
      n_list += sum;
    }
    __syncthreads();
  }
  n_list = __builtin_amdgcn_readfirstlane(n_list);
  int n_keys = SEL ? n_list << a.page_log2 : len;  // positions the block walks through
  // drafted tokens: the rows' bits for those behind the context
  const int ctx = TREE ? max(a.ctx[b], 0) : 0;
  if constexpr (TREE) {
    const int n = (i1 - i0 + 1) * words;
    for (int x = tid; x < n; x += blockDim.x) s_bits[x] = a.mask[(size_t)(row0 + i0) * words + x];
    __syncthreads();
  }
  // windows: what any row of the block sees (paged_walk.h)
  Span sp;
  WindowWalk<32> walk{};
  if constexpr (WIN) {
    sp = span_of(a, len, row0 + i0, i1 - i0 + 1, lane);
    walk = WindowWalk<32>::of(sp.lo_min, sp.hi_max, a.sinks);
    n_keys = 32 * walk.tiles;
    chunk = ((int)a.d_splits.div(walk.tiles + a.splits - 1) + waves - 1) / waves * waves;
    first = split_i * chunk + wave;
  }
  const int t1 = min((split_i + 1) * chunk, (n_keys + 31) >> 5);  // the range's last tile

  // queries: lane (c, g) holds row c of each tile (columns behind the last row
  // repeat the block's first: computed and never stored)
  bf16x8 qf[RT][TERMS][NC];
  int w_lo[RT], w_hi[RT];  // windows: the row's first token and the one behind its last
  int loc[RT];  // the row within the block
  int out[RT];  // and its (row, query head) in the output, or -1
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int pr = p0 + rt * 16 + c;
    const bool on = pr < packed;
    const int i = on ? row_of(pr) : i0, hg = on ? pr - i * a.group : 0;
    loc[rt] = i - i0;
    if constexpr (WIN) window_of(a, len, a.q_idx[row0 + i], w_lo[rt], w_hi[rt]);
    out[rt] = on ? (row0 + i) * (a.n_heads * a.group) + h * a.group + hg : -1;
    const RowT *q = static_cast<const RowT *>(a.q) + (size_t)(row0 + i) * a.q_stride +
                    (size_t)(h * a.group + hg) * DH;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      float x[8];
      if (Raw::T && n == NC - 1) {
        load4(q + Raw::chan(n, g), x);
#pragma unroll
        for (int e = 4; e < 8; ++e) x[e] = 0.f;
      } else {
        load8(q + Raw::chan(n, g), x);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        bf16 p[TERMS];
        split<TERMS>(x[e], p);
#pragma unroll
        for (int s = 0; s < TERMS; ++s) qf[rt][s][n][e] = p[s];
      }
    }
  }

  // Where the halves of a 32-key tile lie: first slots in the pool, how many of
  // the 16 tokens exist, and (selected pages) the logical pages.  All uniform.
  struct Tile {
    size_t slot[2];
    int n[2], lp[2], key[2];
  };
  auto place = [&](int t, bool start) {
    Tile x;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int pos = (WIN ? walk.key(t) : 32 * t) + 16 * u;
      x.key[u] = pos;
      if (u == 1 && a.page_log2 > 4) {  // the same page
        x.lp[1] = x.lp[0];
        x.slot[1] = x.slot[0] + 16;
        x.n[1] = x.n[0] < 16 ? 0 : min(max(len - (SEL ? (x.lp[0] << a.page_log2) + (pos & (page - 1)) : pos), 0), 16);
        break;
      }
      bool ok = pos < (WIN ? len : n_keys);
      int lp = ok ? pos >> a.page_log2 : 0, key = pos;
      if constexpr (SEL) {
        lp = __builtin_amdgcn_readfirstlane((int)s_list[lp]);
        key = (lp << a.page_log2) + (pos & (page - 1));
      }
      const int phys = !ok ? 0 : !SEL && !WIN && start && u == 0 ? ahead : tab[lp];
      ok = ok && (unsigned)phys < (unsigned)a.n_pages;
      x.n[u] = ok ? min(max(len - key, 0), 16) : 0;
      x.slot[u] = (((size_t)(ok ? phys : 0) * a.n_heads + h) << a.page_log2) + (pos & (page - 1));
      x.lp[u] = lp;
    }
    return x;
  };

  // The words that say which rows look at a tile's pages (bit lp & 31), read from
  // LDS a tile ahead by two row tiles: read where they are used, 36 .. 100 rows
  // over 8 pages each of 32 x 16 heads of 64, the selection included, take 78 us
  // for 72 (34 bf16 pages), 217 for 187 (63 e4m3 pages).  One row tile has the same
  // latency once and more wavefronts to hide it, and the words' registers cost
  // more (20 .. 60 fp32 rows over 8 of 34 int8 pages, 16 x 16 heads of 80: 60.1 us
  // ahead, 53.2 in place; one row of 32 heads over 32 of 512 pages 27.4 and 26.6).
  // Two row tiles of 128 bf16 have no registers for them.
  constexpr bool AHEAD = SEL && RT == 2 && !(FMT == BF && DH == 128);
  struct Bits {
    uint32_t w[RT][2];
  };
  auto row_bits = [&](const Tile &x) {
    Bits b;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      b.w[rt][0] = s_bits[loc[rt] * words + (x.lp[0] >> 5)];
      b.w[rt][1] = a.page_log2 > 4 ? b.w[rt][0] : s_bits[loc[rt] * words + (x.lp[1] >> 5)];
    }
    return b;
  };

  f32x4 acc[RT][M];
  float m_run[RT], l_run[RT];
  bool seen[RT];

  // (again: the products with the lower parts of fp32 queries and weights leave
  // out keys and values that are not finite, see below)
  auto pass = [&](auto again) {
    constexpr bool AGAIN = again.value;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m_run[rt] = -INFINITY;
      l_run[rt] = 0.f;
      seen[rt] = false;
#pragma unroll
      for (int m = 0; m < M; ++m) acc[rt][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int t = first;
    if (t >= t1) return;
    Raw raw;
    Tile x = place(t, true);
    raw.load(0, a.k, a.v, a.k_exp, a.v_exp, x.slot[0], c, g);
    raw.load(1, a.k, a.v, a.k_exp, a.v_exp, x.slot[1], c, g);
    Tile y = t + waves < t1 ? place(t + waves, false) : x;
    Bits bits, bits_next;
    if constexpr (AHEAD) bits = row_bits(x);
    while (true) {
      // the next tile's loads, and the page ids of the one after it
      const bool more = t + waves < t1;
      Raw next;
      Tile z = y;
      if (more) {
        next.load(0, a.k, a.v, a.k_exp, a.v_exp, y.slot[0], c, g);
        next.load(1, a.k, a.v, a.k_exp, a.v_exp, y.slot[1], c, g);
        if constexpr (AHEAD) bits_next = row_bits(y);
        if (t + 2 * waves < t1) z = place(t + 2 * waves, false);
      }
      const bool part = x.n[0] + x.n[1] < 32;
      if (part) {
        raw.clear(0, x.n[0], g);
        raw.clear(1, x.n[1], g);
      }
      // Every step runs over all row tiles before the next begins: their chains
      // of dependent instructions overlap (a lone chain leaves most issue
      // slots empty).
      if constexpr (STAGE) {
        raw.stage(s_k, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      f32x4 s[RT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8 kf[NC];
        raw.keys(u, s_k, c, g, kf);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = TERMS - 1; e >= 0; --e)
#pragma unroll
          for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              s[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(AGAIN && e > 0 ? finite(kf[n]) : kf[n], qf[rt][e][n], s[rt][u], 0, 0, 0);
      }
      if constexpr (FMT == I8) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float sc = exp_scale((raw.ke[u] >> (8 * r)) & 0xFFu);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][u][r] *= sc;
          }
      }
      if (part) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * g + r >= x.n[u]) {
#pragma unroll
              for (int rt = 0; rt < RT; ++rt) s[rt][u][r] = -INFINITY;
            }
      }
      float mx[RT];
      bool raise = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        mx[rt] = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bool look = true;
          uint32_t bits16 = 0xFFFFu;  // which of the half's keys the row sees
          if constexpr (WIN) {
            if (!(x.key[u] + 16 <= sp.hi_min && (x.key[u] >= sp.lo_max || x.key[u] + 16 <= a.sinks))) {
              bits16 = window_bits(w_lo[rt], w_hi[rt], a.sinks, x.key[u]);
              look = (bits16 & ((1u << x.n[u]) - 1u)) != 0;
            }
          }
          if constexpr (TREE) {
            if (x.key[u] + 16 > ctx) {
              bits16 = tree_bits(s_bits + loc[rt] * words, words, x.key[u] - ctx);
              look = (bits16 & ((1u << x.n[u]) - 1u)) != 0;
            }
          }
          if constexpr (SEL) {
            const uint32_t w = AHEAD ? bits.w[rt][u] : s_bits[loc[rt] * words + (x.lp[u] >> 5)];
            look = (w >> (x.lp[u] & 31)) & 1u;
          }
          seen[rt] |= look && x.n[u] > 0;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (SEL && !look) s[rt][u][r] = -INFINITY;
            if ((WIN || TREE) && !((bits16 >> (4 * g + r)) & 1u)) s[rt][u][r] = -INFINITY;
            mx[rt] = fmaxf(mx[rt], s[rt][u][r]);
          }
        }
        raise |= mx[rt] * a.sl2 > m_run[rt] + 8.f;
      }
      if (__any(raise)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const float m_new = fmaxf(m_run[rt], quad_max(mx[rt]) * a.sl2);
          const float al = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
          m_run[rt] = m_new;
          l_run[rt] *= al;
#pragma unroll
          for (int m = 0; m < M; ++m) acc[rt][m] *= al;
        }
      }
      bf16x8 pb[RT][TERMS];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float mm = m_run[rt] == -INFINITY ? 0.f : -m_run[rt];
        float sum[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float p[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[rt][u][r], a.sl2, mm));
          sum[u] = (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if constexpr (FMT == I8) p[r] *= exp_scale((raw.ve[u] >> (8 * r)) & 0xFFu);
            bf16 q[TERMS];
            split<TERMS>(p[r], q);
#pragma unroll
            for (int e = 0; e < TERMS; ++e) pb[rt][e][4 * u + r] = q[e];
          }
        }
        l_run[rt] += sum[0] + sum[1];
      }
#pragma unroll
      for (int m = 0; m < M; m += 2) {
        bf16x8 vf[2];
        raw.values(m, vf[0], vf[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (m + j == M) break;
#pragma unroll
          for (int e = TERMS - 1; e >= 0; --e)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              acc[rt][m + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(AGAIN && e > 0 ? finite(vf[j]) : vf[j], pb[rt][e], acc[rt][m + j], 0, 0, 0);
        }
      }
      if (!more) break;
      t += waves;
      raw = next;
      if constexpr (AHEAD) bits = bits_next;
      x = y;
      y = z;
    }
  };

  // Four channels from d on of tile rt's row c, for every such group of the lane.
  auto groups = [&](int rt, auto f) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int m = 0; m < Raw::VC; m += 4)
        f(Raw::VC * (4 * g + r) + m, f32x4{acc[rt][m][r], acc[rt][m + 1][r], acc[rt][m + 2][r], acc[rt][m + 3][r]});
    if constexpr (Raw::T) f(64 + 4 * g, acc[rt][M - 1]);
  };
  auto store = [&](int row, int d, f32x4 v) {
    if (a.splits > 1) {
      const size_t part = (size_t)split_i * a.q_total * (a.n_heads * a.group) + row;
      *reinterpret_cast<f32x4 *>(a.part_o + part * DH + d) = v;
    } else if constexpr (sizeof(RowT) == 4) {
      *reinterpret_cast<f32x4 *>(static_cast<float *>(a.o) + (size_t)row * DH + d) = v;
    } else {
      *reinterpret_cast<bf16x4 *>(static_cast<bf16 *>(a.o) + (size_t)row * DH + d) =
          bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    }
  };

  // Joins the wavefronts' parts and writes them.  l = -1 stands for "no key at
  // all" (the row gets zeros; a sum of 0 over keys that all have logit -inf
  // gives 0 / 0).
  auto join = [&]() {
    float scale[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      l_run[rt] += __shfl_xor(l_run[rt], 16, 64);
      l_run[rt] += __shfl_xor(l_run[rt], 32, 64);
      if (waves > 1 && g == 0) {
        s_m[wave * RT * 16 + rt * 16 + c] = m_run[rt];
        s_l[wave * RT * 16 + rt * 16 + c] = seen[rt] ? l_run[rt] : -1.f;
        if (wave == 0) s_row[rt * 16 + c] = out[rt];
      }
    }
    if (waves > 1) __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float m = m_run[rt], l = l_run[rt];
      bool any = seen[rt];
      scale[rt] = 1.f;
      if (waves > 1) {
        m = -INFINITY;
        for (int w = 0; w < waves; ++w) m = fmaxf(m, s_m[w * RT * 16 + rt * 16 + c]);
        l = 0.f;
        any = false;
        for (int w = 0; w < waves; ++w) {
          const float lw = s_l[w * RT * 16 + rt * 16 + c], mw = s_m[w * RT * 16 + rt * 16 + c];
          if (lw == -1.f) continue;
          any = true;
          l += lw * (mw == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(mw - m));
        }
        scale[rt] = m_run[rt] == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(m_run[rt] - m);
      }
      if (a.splits == 1) {
        scale[rt] *= any ? 1.f / l : 0.f;
      } else if (wave == 0 && g == 0 && out[rt] >= 0) {
        const size_t part = (size_t)split_i * a.q_total * (a.n_heads * a.group) + out[rt];
        a.part_ml[2 * part] = m;
        a.part_ml[2 * part + 1] = any ? l : -1.f;
      }
    }
    if (waves == 1) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
        if (out[rt] >= 0) groups(rt, [&](int d, f32x4 v) { store(out[rt], d, v * scale[rt]); });
      return;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float *o = s_o + ((wave * RT + rt) * 16 + c) * OS;
      groups(rt, [&](int d, f32x4 v) { *reinterpret_cast<f32x4 *>(o + d) = v * scale[rt]; });
    }
    __syncthreads();
    for (int x = tid; x < RT * 16 * (DH / 4); x += blockDim.x) {
      const int col = x / (DH / 4), d = (x - col * (DH / 4)) * 4;
      const int row = s_row[col];
      if (row < 0) continue;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < waves; ++w) sum += *reinterpret_cast<const f32x4 *>(s_o + (w * RT * 16 + col) * OS + d);
      store(row, d, sum);
    }
  };

  // Whether anything is not finite; with `own`, apart from rows whose weights' sum is
  // NaN: their own logits make all of them NaN.
  auto spoiled = [&](bool own) {
    bool bad = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float l = l_run[rt] + __shfl_xor(l_run[rt], 16, 64);
      l += __shfl_xor(l, 32, 64);
      bool x = false;
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) x |= !(fabsf(acc[rt][m][r]) < INFINITY);
      bad |= x && !(own && l != l);
    }
    return __syncthreads_or(bad);
  };

  pass(std::false_type());
  // An infinite bf16 key or value times a part of an fp32 query or weight that is
  // zero, or of the other sign than the whole, is NaN where none is due.
  if constexpr (FMT == BF && TERMS > 1)
    if (spoiled(false)) pass(std::true_type());
  // A weight of zero times an infinite or NaN value that only another row looks at (or
  // none, in a tile that some row sees a part of) is NaN: such a block is computed
  // again, row by row over each row's own keys.
  if constexpr (MODE != PAGED_ALL) {
    if ((!SEL || i1 > i0) && spoiled(true)) {
      one_by_one<FMT, DH, RowT>(
          a, tab,
          [&](int pos) {
            if constexpr (SEL) return ((int)s_list[pos >> a.page_log2] << a.page_log2) + (pos & (page - 1));
            else return WIN && pos >= 32 * walk.sink_tiles ? pos + 32 * walk.jump : pos;
          },
          [&](int i, int key) {
            if constexpr (SEL) {
              const int lp = key >> a.page_log2;
              return ((s_bits[(i - i0) * words + (lp >> 5)] >> (lp & 31)) & 1u) != 0;
            } else if constexpr (WIN) {
              int lo, hi;
              window_of(a, len, a.q_idx[row0 + i], lo, hi);
              return key < hi && (key >= lo || key < a.sinks);
            } else {
              return (tree_bits(s_bits + (i - i0) * words, words, key - ctx) & 1u) != 0;
            }
          },
          p0, min(p0 + 16 * RT, packed), row0, h, split_i, len, 32 * split_i * chunk, min(32 * t1, n_keys), wave,
          waves, lane);
      return;
    }
  }
  join();
}

template <int FMT, int DH, int RT, typename RowT, int MODE>
hipError_t launch_paged_attn(const PagedAttnArgs &a, hipStream_t s) {
  constexpr int OS = DH + 4;
  const int words = (a.max_pages + 31) / 32;
  size_t lds = paged_stage<FMT, DH, RT, RowT> ? 32 * DH * (FMT == BF ? 2 : 1) : 0;
  if (a.waves > 1) lds = ((size_t)a.waves * (RT * 16 * OS + 2 * RT * 16) + RT * 16) * 4;
  if (MODE == PAGED_LISTED) lds += ((size_t)(a.bit_rows + 1) * words) * 4 + (size_t)words * 64;
  if (MODE == PAGED_TREE) lds += (size_t)a.bit_rows * a.mask_words * 4;
  auto kernel = paged_attn_kernel<FMT, DH, RT, RowT, MODE>;
  if (lds > 65536) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int64_t grid = paged_grid(a);
  launch_kernel(kernel, dim3((unsigned)grid), dim3(64 * a.waves), (uint32_t)lds, s, a, a.table);
  return hipGetLastError();
}

template <int FMT, int DH, typename RowT, int MODE>
hipError_t launch_paged_rt(const PagedAttnArgs &a, hipStream_t s) {
  if (a.row_tiles == 1) return launch_paged_attn<FMT, DH, 1, RowT, MODE>(a, s);
  if constexpr (sizeof(RowT) == 2)
    if (a.row_tiles == 2) return launch_paged_attn<FMT, DH, 2, RowT, MODE>(a, s);
  return hipErrorInvalidValue;
}

// MASKED: windows and trees; otherwise every token, or listed pages.
template <int FMT, int DH, bool MASKED, typename RowT>
hipError_t launch_paged_mode(const PagedAttnArgs &a, hipStream_t s) {
  if constexpr (MASKED)
    return a.look == PAGED_TREE ? launch_paged_rt<FMT, DH, RowT, PAGED_TREE>(a, s)
                                : launch_paged_rt<FMT, DH, RowT, PAGED_WINDOW>(a, s);
  else
    return a.pages ? launch_paged_rt<FMT, DH, RowT, PAGED_LISTED>(a, s) : launch_paged_rt<FMT, DH, RowT, PAGED_ALL>(a, s);
}

template <int FMT, bool MASKED>
hipError_t launch_paged_fmt(DType dt, int head_dim, const PagedAttnArgs &a, hipStream_t s) {
  auto go = [&](auto dh) {
    return dt == DType::BF16 ? launch_paged_mode<FMT, dh.value, MASKED, bf16>(a, s)
                             : launch_paged_mode<FMT, dh.value, MASKED, float>(a, s);
  };
  switch (head_dim) {
    case 64: return go(std::integral_constant<int, 64>());
    case 80: return go(std::integral_constant<int, 80>());
    case 128: return go(std::integral_constant<int, 128>());
  }
  return hipErrorInvalidValue;
}

}  // namespace marche
