// Attention over the paged cache (the kernel template; one translation unit per
// cache format instantiates it).
//
//   o_i = sum_j softmax_j(q_i . K_j / sqrt(dh)) V_j
//
// over a sequence's cached tokens j, or over those of the pages listed for row
// i.  The rows of one sequence that share a key head (its query heads times
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
// elements.  Nothing goes through LDS until the wavefronts' parts are joined
// at the end, so the main loop has no barrier and each wavefront keeps the next
// tile's loads in flight while it computes.
//
// Softmax statistics and O are float32; the maximum that P is taken against
// trails the true one by at most 2^8, which saves most rescales.  P is rounded
// to bf16 (half a step, 2^-9 of each weight, as the products' other operand V
// is exact in bf16 for every format).  float32 rows are split into three bf16
// parts (24 bits, nothing lost) and so is P.
//
// Bound: single rows by the cache's bytes, many rows by the softmax's vector
// work.
#pragma once

#include <algorithm>

#include "paged_device.h"

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

// Raw registers of 32 keys of a lane: K for its key c of each half, V for its
// eight keys, exponent bytes.
template <int FMT, int DH>
struct KvRaw {
  static constexpr bool W = FMT == BF;               // 2-byte elements
  static constexpr int ES = W ? 2 : 1;
  static constexpr int KQ = W ? DH / 32 : DH / 64;   // 16-byte loads per key
  static constexpr bool T = DH % 32 != 0;            // a 16-channel tail (dh 80)
  static constexpr int NC = DH / 32 + T;             // 32-deep products of S; the tail fills half of one
  static constexpr int VC = DH == 128 ? 8 : 4;       // channels per lane
  static constexpr int VW = VC * ES / 4;             // dwords of them
  static constexpr int M = DH / 16;                  // 16-channel tiles of O
  static_assert(DH == 64 || DH == 80 || DH == 128, "head width");

  u32x4 k[2][KQ];
  u32x2 kt[2];
  uint32_t v[8][VW];
  uint32_t vt[8];
  uint32_t ke[2], ve[2];  // ke: the byte of key c (e4m3), the four of keys 4g.. (int8)

  // half u of the tile: 16 tokens from `slot` (uniform) on
  __device__ __forceinline__ void load(int u, const void *kb, const void *vb, const uint8_t *kx,
                                       const uint8_t *vx, size_t slot, int c, int g) {
    const char *kp = static_cast<const char *>(kb) + slot * (DH * ES);
    const char *vp = static_cast<const char *>(vb) + slot * (DH * ES);
    const uint32_t ko = c * DH * ES;
#pragma unroll
    for (int m = 0; m < KQ; ++m) k[u][m] = *reinterpret_cast<const u32x4 *>(kp + ko + 64 * m + 16 * g);
    if constexpr (T) {
      if constexpr (W) kt[u] = *reinterpret_cast<const u32x2 *>(kp + ko + 64 * ES + 8 * g);
      else kt[u].x = *reinterpret_cast<const uint32_t *>(kp + ko + 64 * ES + 4 * g);
    }
    const uint32_t vo = 4 * g * DH * ES + c * VC * ES;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const char *p = vp + vo + r * DH * ES;
      uint32_t(&x)[VW] = v[4 * u + r];
      if constexpr (VW == 1) {
        x[0] = *reinterpret_cast<const uint32_t *>(p);
      } else if constexpr (VW == 2) {
        const u32x2 y = *reinterpret_cast<const u32x2 *>(p);
        x[0] = y.x, x[1] = y.y;
      } else {
        const u32x4 y = *reinterpret_cast<const u32x4 *>(p);
        x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
      }
      if constexpr (T) {
        const char *t = vp + 4 * g * DH * ES + r * DH * ES + 64 * ES + c * ES;
        if constexpr (W) vt[4 * u + r] = *reinterpret_cast<const uint16_t *>(t);
        else vt[4 * u + r] = *reinterpret_cast<const uint8_t *>(t);
      }
    }
    if constexpr (!W) {
      if constexpr (FMT == E4) ke[u] = kx[slot + c];
      else ke[u] = *reinterpret_cast<const uint32_t *>(kx + slot + 4 * g);
      ve[u] = *reinterpret_cast<const uint32_t *>(vx + slot + 4 * g);
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
  // on (the tail's: four, and zeros.  Its own 16-deep instruction is no faster,
  // and following a 32-deep one on the same accumulators gave wrong sums).
  __device__ __forceinline__ void keys(int u, bf16x8 (&f)[NC]) const {
    if constexpr (W) {
#pragma unroll
      for (int n = 0; n < DH / 32; ++n) f[n] = __builtin_bit_cast(bf16x8, k[u][n]);
      if constexpr (T) f[NC - 1] = __builtin_bit_cast(bf16x8, u32x4{kt[u].x, kt[u].y, 0u, 0u});
    } else {
      const float sc = FMT == E4 ? exp_scale(ke[u]) : 1.f;
#pragma unroll
      for (int n = 0; n < DH / 32; ++n) {
        const uint32_t a = k[u][n / 2][2 * (n % 2)], b = k[u][n / 2][2 * (n % 2) + 1];
        f[n] = __builtin_bit_cast(bf16x8, u32x4{pair(a, sc, 0), pair(a, sc, 1), pair(b, sc, 0), pair(b, sc, 1)});
      }
      if constexpr (T)
        f[NC - 1] = __builtin_bit_cast(bf16x8, u32x4{pair(kt[u].x, sc, 0), pair(kt[u].x, sc, 1), 0u, 0u});
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
  // V^T of the eight keys as operands, tile m: channel vchan(m, c).
  __device__ __forceinline__ void values(bf16x8 (&f)[M]) const {
    uint32_t o[M][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // keys 2 i and 2 i + 1
      const int a = 2 * i, b = a + 1, u = a / 4;
      if constexpr (FMT == I8) {
#pragma unroll
        for (int m = 0; m < VC; ++m)
          o[m][i] = hi16(__float_as_uint((float)(int8_t)(v[a][m / 4] >> (8 * (m % 4)))),
                         __float_as_uint((float)(int8_t)(v[b][m / 4] >> (8 * (m % 4)))));
        if constexpr (T)
          o[4][i] = hi16(__float_as_uint((float)(int8_t)vt[a]), __float_as_uint((float)(int8_t)vt[b]));
      } else {
        const float sa = FMT == E4 ? exp_scale((ve[u] >> (8 * (a % 4))) & 0xFFu) : 1.f;
        const float sb = FMT == E4 ? exp_scale((ve[u] >> (8 * (b % 4))) & 0xFFu) : 1.f;
#pragma unroll
        for (int p = 0; p < VC / 2; ++p) {
          uint32_t x, y;
          if constexpr (FMT == E4) x = pair(v[a][p / 2], sa, p % 2), y = pair(v[b][p / 2], sb, p % 2);
          else x = v[a][p], y = v[b][p];
          o[2 * p][i] = lo16(x, y);
          o[2 * p + 1][i] = hi16(x, y);
        }
        if constexpr (T) {
          if constexpr (FMT == E4) o[4][i] = lo16(pair(vt[a], sa, 0), pair(vt[b], sb, 0));
          else o[4][i] = lo16(vt[a], vt[b]);
        }
      }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) f[m] = __builtin_bit_cast(bf16x8, u32x4{o[m][0], o[m][1], o[m][2], o[m][3]});
  }
  // first channel of product n's eight in lane group g
  static __device__ __forceinline__ int chan(int n, int g) {
    return T && n == NC - 1 ? 64 + 4 * g : W ? 32 * n + 8 * g : 64 * (n / 2) + 16 * g + 8 * (n % 2);
  }
  // channel of row x of O's tile m
  static __device__ __forceinline__ int vchan(int m, int x) { return m < VC ? VC * x + m : 64 + x; }
};

// T parts of a float32 whose sum is the value to 8 T bits (an infinity's other
// parts are zero).
template <int T>
__device__ __forceinline__ void split(float x, bf16 (&o)[T]) {
  o[0] = (bf16)x;
  if constexpr (T > 1) x = fabsf(x) == INFINITY ? 0.f : x - (float)o[0];
#pragma unroll
  for (int i = 1; i < T; ++i) {
    o[i] = (bf16)x;
    x -= (float)o[i];
  }
}

template <int FMT, int DH, int RT, typename RowT, bool SEL>
__global__ __launch_bounds__(RT == 1 ? 512 : 256) void paged_attn_kernel(PagedAttnArgs a,
                                                                         const int32_t *__restrict__ table) {
  using Raw = KvRaw<FMT, DH>;
  constexpr int TERMS = sizeof(RowT) == 4 ? 3 : 1;
  constexpr int NC = Raw::NC, M = Raw::M;
  constexpr int OS = DH + 4;  // row stride of the joined parts
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;

  // (sequence, key head, row block, key range), ranges and blocks of one
  // sequence and head side by side on one XCD
  int at = xcd_remap(blockIdx.x, gridDim.x);
  const int split_i = at % a.splits;
  at /= a.splits;
  const int rb = at % a.row_blocks;
  at /= a.row_blocks;
  const int h = at % a.n_heads, b = at / a.n_heads;

  int row0, n_rows;  // the sequence's rows
  if (a.q_off) {
    row0 = min(max(a.q_off[b], 0), a.q_total);
    n_rows = min(max(a.q_off[b + 1], row0), a.q_total) - row0;
  } else {
    row0 = b * a.rows_each;
    n_rows = a.rows_each;
  }
  const int packed = min(n_rows, a.q_max) * a.group;
  const int p0 = rb * 16 * RT;
  if (p0 >= packed) return;
  const int n_rt = min(RT, (packed - p0 + 15) >> 4);
  const int len = min(paged_len(a.lens[b], a.max_pages, a.page_log2), a.len_max);
  const int page = 1 << a.page_log2;
  const int32_t *tab = table + (size_t)b * a.max_pages;

  // LDS: joined O parts, maxima and sums of every wavefront, then the page
  // bits of the block's rows and the list of pages that any of them looks at
  float *s_o = reinterpret_cast<float *>(smem);             // [waves][16][OS]
  float *s_m = s_o + waves * 16 * OS;                       // [waves][RT*16]
  float *s_l = s_m + waves * RT * 16;                       // [waves][RT*16]
  uint32_t *s_bits = reinterpret_cast<uint32_t *>(s_l + waves * RT * 16);
  const int words = (a.max_pages + 31) >> 5;
  const int i0 = p0 / a.group, i1 = (min(p0 + 16 * RT, packed) - 1) / a.group;  // the block's rows
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
  const int n_keys = SEL ? n_list << a.page_log2 : len;  // positions the block walks through
  const int t0 = min(split_i * a.chunk, (n_keys + 31) >> 5), t1 = min(t0 + a.chunk, (n_keys + 31) >> 5);

  // queries: lane (c, g) holds row c of each tile
  bf16x8 qf[RT][TERMS][NC];
  int bit_at[RT];  // the row's page bits
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int pr = p0 + rt * 16 + c;
    const bool on = pr < packed;
    const int i = on ? pr / a.group : i0, hg = on ? pr - i * a.group : 0;
    const RowT *q = static_cast<const RowT *>(a.q) + (size_t)(row0 + i) * a.q_stride +
                    (size_t)(h * a.group + hg) * DH;
    bit_at[rt] = (i - i0) * words;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
      if (on) {
        if (Raw::T && n == NC - 1) load4(q + Raw::chan(n, g), x);
        else load8(q + Raw::chan(n, g), x);
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

  // Where a tile's halves lie: first slot in the pool, how many of the 16
  // tokens exist, and (selected pages) the logical page.
  struct Half {
    size_t slot;
    int n, lp;
  };
  auto half = [&](int pos, int only) {
    Half x;
    int lp = pos >> a.page_log2, key = pos;
    bool ok = pos < n_keys;
    if constexpr (SEL) {
      lp = __builtin_amdgcn_readfirstlane((int)s_list[ok ? lp : 0]);
      if (!ok) lp = 0;
      key = (lp << a.page_log2) + (pos & (page - 1));
      if (only >= 0) ok = ok && ((s_bits[only * words + (lp >> 5)] >> (lp & 31)) & 1u);
    }
    const int phys = ok ? tab[lp] : 0;
    ok = ok && (unsigned)phys < (unsigned)a.n_pages;
    x.n = __builtin_amdgcn_readfirstlane(ok ? min(max(len - key, 0), 16) : 0);
    const int ph = __builtin_amdgcn_readfirstlane(ok ? phys : 0);
    x.slot = (((size_t)ph * a.n_heads + h) << a.page_log2) + (pos & (page - 1));
    x.lp = lp;
    return x;
  };

  f32x4 acc[RT][M];
  float m_run[RT], l_run[RT];
  bool seen[RT];

  // every row at once (only < 0), or, where that met values that are not
  // finite, row `only` over its own pages
  auto pass = [&](int only) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m_run[rt] = -INFINITY;
      l_run[rt] = 0.f;
      seen[rt] = false;
#pragma unroll
      for (int m = 0; m < M; ++m) acc[rt][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int t = t0 + wave;
    if (t >= t1) return;
    Raw raw;
    Half x0 = half(32 * t, only), x1 = half(32 * t + 16, only);
    raw.load(0, a.k, a.v, a.k_exp, a.v_exp, x0.slot, c, g);
    raw.load(1, a.k, a.v, a.k_exp, a.v_exp, x1.slot, c, g);
    Half y0 = x0, y1 = x1;
    if (t + waves < t1) y0 = half(32 * (t + waves), only), y1 = half(32 * (t + waves) + 16, only);
    while (true) {
      // the next tile's loads, and the page ids of the one after it
      const bool more = t + waves < t1;
      Raw next;
      Half z0 = y0, z1 = y1;
      if (more) {
        next.load(0, a.k, a.v, a.k_exp, a.v_exp, y0.slot, c, g);
        next.load(1, a.k, a.v, a.k_exp, a.v_exp, y1.slot, c, g);
        if (t + 2 * waves < t1)
          z0 = half(32 * (t + 2 * waves), only), z1 = half(32 * (t + 2 * waves) + 16, only);
      }
      const int nv[2] = {x0.n, x1.n}, lp[2] = {x0.lp, x1.lp};
      const bool part = nv[0] + nv[1] < 32;
      if (part) {
        raw.clear(0, nv[0], g);
        raw.clear(1, nv[1], g);
      }
      if (nv[0] + nv[1] > 0) {
        bf16x8 kf[2][NC], vf[M];
        raw.keys(0, kf[0]);
        raw.keys(1, kf[1]);
        raw.values(vf);
        float ks[2][4], vs[2][4];
        if constexpr (FMT == I8) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              ks[u][r] = exp_scale((raw.ke[u] >> (8 * r)) & 0xFFu) * a.sl2;
              vs[u][r] = exp_scale((raw.ve[u] >> (8 * r)) & 0xFFu);
            }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          if (rt >= n_rt) break;
          float s[2][4];
          float mx = -INFINITY;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = TERMS - 1; e >= 0; --e)
#pragma unroll
              for (int n = 0; n < NC; ++n)
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u][n], qf[rt][e][n], d, 0, 0, 0);
            bool look = true;
            if constexpr (SEL) {
              look = (s_bits[bit_at[rt] + (lp[u] >> 5)] >> (lp[u] & 31)) & 1u;
              seen[rt] |= look && nv[u] > 0;
            } else {
              seen[rt] = true;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              s[u][r] = d[r] * (FMT == I8 ? ks[u][r] : a.sl2);
              if (SEL ? !look : false) s[u][r] = -INFINITY;
              if (part && 4 * g + r >= nv[u]) s[u][r] = -INFINITY;
              mx = fmaxf(mx, s[u][r]);
            }
          }
          if (__any(mx > m_run[rt] + 8.f)) {
            const float m_new = fmaxf(m_run[rt], quad_max(mx));
            const float al = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
            m_run[rt] = m_new;
            l_run[rt] *= al;
#pragma unroll
            for (int m = 0; m < M; ++m) acc[rt][m] *= al;
          }
          const float mm = m_run[rt] == -INFINITY ? 0.f : m_run[rt];
          bf16x8 pb[TERMS];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float p = __builtin_amdgcn_exp2f(s[u][r] - mm);
              l_run[rt] += p;
              if constexpr (FMT == I8) p *= vs[u][r];
              bf16 y[TERMS];
              split<TERMS>(p, y);
#pragma unroll
              for (int e = 0; e < TERMS; ++e) pb[e][4 * u + r] = y[e];
            }
#pragma unroll
          for (int e = TERMS - 1; e >= 0; --e)
#pragma unroll
            for (int m = 0; m < M; ++m)
              acc[rt][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[m], pb[e], acc[rt][m], 0, 0, 0);
        }
      }
      if (!more) break;
      t += waves;
      raw = next;
      x0 = y0, x1 = y1;
      y0 = z0, y1 = z1;
    }
  };

  // Joins the wavefronts' parts and writes them; `only`: that row alone.
  // l = -1 stands for "no key at all" (the row gets zeros; a sum of 0 over
  // keys that all have logit -inf gives 0 / 0).
  auto join = [&](int only) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float l = l_run[rt];
      l += __shfl_xor(l, 16, 64);
      l += __shfl_xor(l, 32, 64);
      if (g == 0) {
        s_m[wave * RT * 16 + rt * 16 + c] = m_run[rt];
        s_l[wave * RT * 16 + rt * 16 + c] = seen[rt] ? l : -1.f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (rt >= n_rt) break;
      const int col = rt * 16 + c;
      float m = -INFINITY;
      for (int w = 0; w < waves; ++w) m = fmaxf(m, s_m[w * RT * 16 + col]);
      const float al = m_run[rt] == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(m_run[rt] - m);
      float *o = s_o + (wave * 16 + c) * OS;
#pragma unroll
      for (int m4 = 0; m4 < M; ++m4)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[Raw::vchan(m4, 4 * g + r)] = acc[rt][m4][r] * al;
      __syncthreads();
      for (int x = tid; x < 16 * (DH / 4); x += blockDim.x) {
        const int cc = x / (DH / 4), d = (x - cc * (DH / 4)) * 4, cl = rt * 16 + cc;
        const int pr = p0 + cl;
        if (pr >= packed) continue;
        const int i = pr / a.group, hg = pr - i * a.group;
        if (only >= 0 && i != only) continue;
        float mt = -INFINITY;
        for (int w = 0; w < waves; ++w) mt = fmaxf(mt, s_m[w * RT * 16 + cl]);
        float l = 0.f;
        bool any = false;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < waves; ++w) {
          const float lw = s_l[w * RT * 16 + cl], mw = s_m[w * RT * 16 + cl];
          if (lw == -1.f) continue;
          any = true;
          l += lw * (mw == -INFINITY ? (mt == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(mw - mt));
          sum += *reinterpret_cast<const f32x4 *>(s_o + (w * 16 + cc) * OS + d);
        }
        const size_t row = (size_t)(row0 + i) * (a.n_heads * a.group) + h * a.group + hg;
        if (a.splits > 1) {
          const size_t part = (size_t)split_i * a.q_total * (a.n_heads * a.group) + row;
          *reinterpret_cast<f32x4 *>(a.part_o + part * DH + d) = sum;
          if (d == 0) {
            a.part_ml[2 * part] = mt;
            a.part_ml[2 * part + 1] = any ? l : -1.f;
          }
        } else {
          const float inv = any ? 1.f / l : 0.f;
          RowT *out = static_cast<RowT *>(a.o) + row * DH + d;
          if constexpr (sizeof(RowT) == 4) {
            f32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = any ? sum[e] * inv : 0.f;
            *reinterpret_cast<f32x4 *>(out) = y;
          } else {
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (bf16)(any ? sum[e] * inv : 0.f);
            *reinterpret_cast<bf16x4 *>(out) = y;
          }
        }
      }
      __syncthreads();
    }
  };

  pass(-1);
  if constexpr (SEL) {
    // A weight of zero times an infinite or NaN value of a page that only
    // another row looks at would be NaN: rows of a block in which anything is
    // not finite are computed again, each over its own pages alone.
    bool bad = false;
    if (i1 > i0) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r) bad |= !(fabsf(acc[rt][m][r]) < INFINITY);
    }
    if (__syncthreads_or(bad)) {
      for (int i = i0; i <= i1; ++i) {
        pass(i - i0);
        join(i);
      }
      return;
    }
  }
  join(-1);
}

template <int FMT, int DH, int RT, typename RowT, bool SEL>
hipError_t launch_paged_attn(const PagedAttnArgs &a, hipStream_t s) {
  constexpr int OS = DH + 4;
  const int words = (a.max_pages + 31) / 32;
  size_t lds = (size_t)a.waves * (16 * OS + 2 * RT * 16) * 4;
  if (SEL) lds += ((size_t)(a.bit_rows + 1) * words) * 4 + (size_t)words * 64;
  auto kernel = paged_attn_kernel<FMT, DH, RT, RowT, SEL>;
  if (lds > 65536) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int64_t grid = (int64_t)a.n_seqs * a.n_heads * a.row_blocks * a.splits;
  launch_kernel(kernel, dim3((unsigned)grid), dim3(64 * a.waves), (uint32_t)lds, s, a, a.table);
  return hipGetLastError();
}

template <int FMT, int DH, typename RowT, bool SEL>
hipError_t launch_paged_rt(const PagedAttnArgs &a, hipStream_t s) {
  switch (a.row_tiles) {
    case 1: return launch_paged_attn<FMT, DH, 1, RowT, SEL>(a, s);
    case 2: return launch_paged_attn<FMT, DH, 2, RowT, SEL>(a, s);
    case 4:
      if constexpr (sizeof(RowT) == 2) return launch_paged_attn<FMT, DH, 4, RowT, SEL>(a, s);
  }
  return hipErrorInvalidValue;
}

template <int FMT, int DH>
hipError_t launch_paged_dh(DType dt, const PagedAttnArgs &a, hipStream_t s) {
  if (dt == DType::BF16)
    return a.pages ? launch_paged_rt<FMT, DH, bf16, true>(a, s) : launch_paged_rt<FMT, DH, bf16, false>(a, s);
  return a.pages ? launch_paged_rt<FMT, DH, float, true>(a, s) : launch_paged_rt<FMT, DH, float, false>(a, s);
}

template <int FMT>
hipError_t launch_paged_fmt(DType dt, int head_dim, const PagedAttnArgs &a, hipStream_t s) {
  switch (head_dim) {
    case 64: return launch_paged_dh<FMT, 64>(dt, a, s);
    case 80: return launch_paged_dh<FMT, 80>(dt, a, s);
    case 128: return launch_paged_dh<FMT, 128>(dt, a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace marche
