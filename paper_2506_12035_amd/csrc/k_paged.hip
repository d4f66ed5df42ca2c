// Paged key/value cache: quantising rows as they are written, reading tokens
// back, key bounds of pages, page selection and attention over the cache.
//
// A pool holds pages [n_pages][H][page][dh] for K and for V; a page belongs to
// one head's `page` consecutive tokens of one sequence.  8-bit formats carry
// one exponent byte per (page, head, token) and value = q * 2^(code - 127).
// With powers of two, quantising (a product by 2^-e and one rounding to the
// format) and reading back (q * 2^e, exact in bf16: both formats have at most
// 8 significant bits) give the same bits whatever the order of operations, and
// the page scores below are whole numbers times powers of two.
//
// Page ids and lengths come from device memory.  Every kernel checks a page id
// against the pool before it forms an address from it and clamps lengths to
// the page table, so that no list reaches outside the pool; a page id outside
// the pool reads as "no tokens there" and a write to it is dropped.
#include <algorithm>
#include <type_traits>

#include "paged_device.h"

namespace marche {

// ------------------------------------------------------------------ write

// One (row, head) of new keys and values per GROUP lanes, 8 elements of each
// per lane: the row's largest magnitude by lane exchanges, its exponent, one
// rounding, one 8-byte (16 for bf16) store.  Bound by bytes: each new row is
// read once and its slot written once.  (Two or four pairs a thread, to find
// the rows' sequences less often: 59.0 and 64.6 us for 56.4 on 40960 rows of 16
// heads of 64, bf16 to int8, without STREAM; now, with it, 52.5, 4.8 TB/s.)
// STREAM: the rows are loaded past the caches, for calls whose rows do not fit
// them anyway.  The loads wait for the range of the rows that have a sequence
// (a clamped row instead of a branch, behind which they were waited for at once:
// 53.2 us for 55.3).
template <int FMT, int DH, typename InT, bool STREAM>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedWriteArgs a) {
  constexpr int PER = paged_write_pairs(DH), GROUP = 256 / PER;
  constexpr int NV = sizeof(InT) == 4 ? 2 : 1;  // 16-byte loads of 8 elements
  __shared__ int s_b0;
  const int tid = threadIdx.x, lane = tid & 63, c = tid % GROUP;
  const uint32_t u0 = blockIdx.x * PER, unit = u0 + tid / GROUP;  // pairs are below 2^31
  const int r = (int)a.d_heads.div(unit), h = (int)(unit - (uint32_t)r * a.n_heads);
  const RowRange own(a.a_off, a.n_seqs, a.a_total);
  if (own.none()) return;
  const int rr = own.nearest(r);  // (what is loaded for others is not used)
  const bool on = r == rr && c < DH / 8;

  // the values and the token, in flight while the row's sequence is found
  u32x4 kx[NV], vx[NV];
  {
    const size_t at = (size_t)rr * a.row_stride + (size_t)h * DH + (c < DH / 8 ? 8 * c : 0);
    const u32x4 *kp = reinterpret_cast<const u32x4 *>(static_cast<const InT *>(a.k_new) + at);
    const u32x4 *vp = reinterpret_cast<const u32x4 *>(static_cast<const InT *>(a.v_new) + at);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      kx[i] = STREAM ? __builtin_nontemporal_load(kp + i) : kp[i];
      vx[i] = STREAM ? __builtin_nontemporal_load(vp + i) : vp[i];
    }
  }
  const int tok = a.a_idx[rr];
  int b;
  if (a.a_off) {
    if (tid < 64) {
      const int f = wave_find_seq(a.a_off, a.n_seqs, min((int)a.d_heads.div(u0), a.a_total - 1), lane);
      if (tid == 0) s_b0 = f;
    }
    __syncthreads();
    b = s_b0;  // of the workgroup's first row; on from there
    while (b < a.n_seqs && a.a_off[b + 1] <= rr) ++b;
  } else {
    b = (int)a.d_rows.div((uint32_t)rr);
  }
  const bool ok = on && b < a.n_seqs && tok >= 0 && (tok >> a.page_log2) < a.max_pages;
  const int page = ok ? a.table[(size_t)b * a.max_pages + (tok >> a.page_log2)] : -1;
  int kc = 0, vc = 0;
  if constexpr (FMT != BF) {
    kc = exp_code<FMT>(__uint_as_float(group_max<GROUP>(on ? largest<InT>(kx) : 0u)));
    vc = exp_code<FMT>(__uint_as_float(group_max<GROUP>(on ? largest<InT>(vx) : 0u)));
  }
  if ((unsigned)page >= (unsigned)a.n_pages) return;
  const size_t slot = (((size_t)page * a.n_heads + h) << a.page_log2) + (tok & ((1 << a.page_log2) - 1));
  const size_t at = slot * DH + 8 * c;
  if constexpr (FMT == BF) {
    u32x4 ko = kx[0], vo = vx[0];
    if constexpr (sizeof(InT) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int w = i / 2, e = i % 2 * 2;
        ko[i] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)__uint_as_float(kx[w][e]), (bf16)__uint_as_float(kx[w][e + 1])});
        vo[i] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)__uint_as_float(vx[w][e]), (bf16)__uint_as_float(vx[w][e + 1])});
      }
    }
    *reinterpret_cast<u32x4 *>(static_cast<bf16 *>(a.k) + at) = ko;
    *reinterpret_cast<u32x4 *>(static_cast<bf16 *>(a.v) + at) = vo;
  } else {
    *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.k) + at) = pack8<FMT, InT>(kx, kc);
    *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.v) + at) = pack8<FMT, InT>(vx, vc);
    if (c == 0) {
      a.k_exp[slot] = (uint8_t)kc;
      a.v_exp[slot] = (uint8_t)vc;
    }
  }
}

// ------------------------------------------------------------------ read

// PAGED_READ_TOKENS tokens of one (sequence, head) of K and of V per workgroup.  Within a
// page the tokens of a head lie one after another on both sides, so a thread
// takes EP consecutive elements whatever the head width, EP such that its
// stores are 16 bytes and a wavefront's are contiguous.  Bound by bytes.  STREAM:
// past the caches, for outputs that do not fit them (64 sequences of 1088
// tokens, e4m3 to bf16: 83.3 us without, 77.0 with, 5.6 TB/s).
template <int FMT, int DH, typename OutT, bool STREAM>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedReadArgs a) {
  constexpr int EP = 16 / sizeof(OutT), CH = DH / EP, N = 4;  // N pieces in flight
  const int blk = blockIdx.x % a.blocks, bh = blockIdx.x / a.blocks;
  const int b = bh / a.n_heads, h = bh - b * a.n_heads;
  const int len = min(paged_len(a.lens[b], a.max_pages, a.page_log2), a.n_tokens);
  const int t0 = blk * PAGED_READ_TOKENS;
  if (t0 >= len) return;
  const int n = min(len - t0, PAGED_READ_TOKENS) * CH;
  const int32_t *tab = a.table + (size_t)b * a.max_pages;
  using In = std::conditional_t<FMT == BF, std::conditional_t<EP == 8, u32x4, u32x2>,
                                std::conditional_t<EP == 8, u32x2, uint32_t>>;
  for (int x0 = threadIdx.x; x0 < n; x0 += 256 * N) {
    size_t slot[N];
    bool on[N];
    In in[2][N];
    uint32_t code[2][N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = t0 + min(x0 + 256 * j, n - 1) / CH;
      const int page = tab[t >> a.page_log2];
      on[j] = x0 + 256 * j < n && (unsigned)page < (unsigned)a.n_pages;
      slot[j] = (((size_t)(on[j] ? page : 0) * a.n_heads + h) << a.page_log2) + (t & ((1 << a.page_log2) - 1));
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int d = min(x0 + 256 * j, n - 1) % CH * EP;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const char *src = static_cast<const char *>(w ? a.v : a.k) + (slot[j] * DH + d) * (FMT == BF ? 2 : 1);
        const In *from = reinterpret_cast<const In *>(src);
        in[w][j] = STREAM ? __builtin_nontemporal_load(from) : *from;
        if constexpr (FMT != BF) code[w][j] = (w ? a.v_exp : a.k_exp)[slot[j]];
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (!on[j]) continue;
      const int x = x0 + 256 * j;
      const size_t to = ((size_t)bh * a.n_tokens + t0) * DH + (size_t)x * EP;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t *q = reinterpret_cast<const uint32_t *>(&in[w][j]);
        u32x4 o;
        if constexpr (FMT == BF && EP == 8) {
          o = in[w][j];
        } else {
          float f[EP];
          if constexpr (FMT == BF) {
#pragma unroll
            for (int i = 0; i < EP; ++i) f[i] = __uint_as_float(i % 2 ? q[i / 2] & 0xFFFF0000u : q[i / 2] << 16);
          } else {
            const float s = exp_scale(code[w][j]);
#pragma unroll
            for (int i = 0; i < EP / 4; ++i) unpack4<FMT>(q[i], s, f + 4 * i);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (EP == 4) o[i] = __float_as_uint(f[i]);
            else o[i] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)f[2 * i], (bf16)f[2 * i + 1]});
          }
        }
        u32x4 *out = reinterpret_cast<u32x4 *>(static_cast<OutT *>(w ? a.v_out : a.k_out) + to);
        if constexpr (STREAM) __builtin_nontemporal_store(o, out);
        else *out = o;
      }
    }
  }
}

// ------------------------------------------------------------------ bounds

// One wavefront per (sequence, page, head): lanes hold four channels, LPT lanes
// a token and TPW tokens a load, each lane the largest and smallest of its
// channels over its tokens; the TPW parts are joined by lane swaps at the
// end.  Bound by bytes and, close behind, by the comparisons: two per key
// element (two tokens at a time share a three-operand one); 64 sequences of 1024
// .. 1088 tokens, 16 heads of 64 in e4m3: 18.1 us, 4.1 TB/s.  STREAM: keys
// past the caches, where they do not fit them: 29.9 us without, 24.8 with on
// 142 MB of bf16 keys, but 18.4 without, 19.7 with on 71 MB.
template <int FMT, int DH, bool STREAM>
__global__ __launch_bounds__(256) void paged_bounds_kernel(PagedBoundsArgs a) {
  constexpr int LPT = DH / 4, TPW = 64 / LPT, ES = FMT == BF ? 2 : 1;
  using In = std::conditional_t<FMT == BF, u32x2, uint32_t>;
  const int lane = threadIdx.x & 63;
  const uint32_t unit = blockIdx.x * PAGED_BOUNDS_PAIRS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // below 2^31
  const uint32_t bp = a.d_heads.div(unit);
  const int h = unit - bp * a.n_heads, b = a.d_span.div(bp);
  if (b >= a.n_seqs) return;
  const int len = paged_len(a.lens[b], a.max_pages, a.page_log2);
  const int first = a.first ? max(a.first[b], 0) : 0;
  const int p = (first >> a.page_log2) + (int)(bp - (uint32_t)b * a.span);
  if (p >= a.max_pages || ((int64_t)p << a.page_log2) >= len) return;
  const int page = a.table[(size_t)b * a.max_pages + p];
  if ((unsigned)page >= (unsigned)a.n_pages) return;
  const int n = min(len - (p << a.page_log2), 1 << a.page_log2);
  const size_t slot0 = ((size_t)page * a.n_heads + h) << a.page_log2;
  const int t_in = min(lane / LPT, TPW - 1), l = lane % LPT;  // (left-over lanes repeat a token's)
  const char *src = static_cast<const char *>(a.k) + slot0 * (DH * ES);
  const uint8_t *ex = FMT == BF ? nullptr : a.k_exp + slot0;
  float hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) hi[i] = -INFINITY, lo[i] = INFINITY;
  uint32_t most = 0;  // exponent codes; bf16: the values' bits without sign, in halves
  // eight loads in flight; tokens behind the last repeat it
  for (int t0 = t_in; t0 < n; t0 += 8 * TPW) {
    In in[8];
    uint32_t code[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t t = min(t0 + j * TPW, n - 1);
      const In *from = reinterpret_cast<const In *>(src + (t * (DH * ES) + 4 * ES * l));
      in[j] = STREAM ? __builtin_nontemporal_load(from) : *from;
      if constexpr (FMT != BF) code[j] = ex[t];
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      float f[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if constexpr (FMT == BF) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t w = in[j + u][i];
            f[u][2 * i] = __uint_as_float(w << 16);
            f[u][2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
            most |= (w & 0x7F807F80u) + 0x00800080u;  // bit 15 or 31: an exponent of all ones
          }
        } else if constexpr (FMT == E4) {
          const float s = exp_scale(code[j + u]);
          const auto x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(in[j + u], s, false);
          const auto y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(in[j + u], s, true);
          f[u][0] = x[0], f[u][1] = x[1], f[u][2] = y[0], f[u][3] = y[1];
          most = max(most, code[j + u]);
        } else {
          unpack4<FMT>(in[j + u], exp_scale(code[j + u]), f[u]);
          most = max(most, code[j + u]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = fmaxf(hi[i], fmaxf(f[0][i], f[1][i]));
        lo[i] = fminf(lo[i], fminf(f[0][i], f[1][i]));
      }
    }
  }
  bool bad = FMT == BF ? (most & 0x80008000u) != 0 : most == 255;
  // join the tokens' parts, then the largest magnitude
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (LPT == 20) {
      const float h0 = hi[i], l0 = lo[i];
#pragma unroll
      for (int k = 1; k < TPW; ++k) {
        hi[i] = fmaxf(hi[i], __shfl(h0, min(lane + k * LPT, 63), 64));
        lo[i] = fminf(lo[i], __shfl(l0, min(lane + k * LPT, 63), 64));
      }
    } else {
      if constexpr (LPT == 16) {
        auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(hi[i]), __float_as_uint(hi[i]), false, false);
        auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(lo[i]), __float_as_uint(lo[i]), false, false);
        hi[i] = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
        lo[i] = fminf(__uint_as_float(q[0]), __uint_as_float(q[1]));
      }
      auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(hi[i]), __float_as_uint(hi[i]), false, false);
      auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(lo[i]), __float_as_uint(lo[i]), false, false);
      hi[i] = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
      lo[i] = fminf(__uint_as_float(q[0]), __uint_as_float(q[1]));
    }
    amax = fmaxf(amax, fmaxf(fabsf(hi[i]), fabsf(lo[i])));
  }
  bad = __ballot(bad) != 0;
  amax = __uint_as_float(wave_max_u32(lane < LPT ? __float_as_uint(amax) & 0x7FFFFFFFu : 0u));
  const int code = bad ? 255 : exp_code<I8>(amax);
  const size_t out = (size_t)page * a.n_heads + h;
  if (code == TOP_CODE<I8>) {
    const float top = int8_top(code);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = __builtin_amdgcn_fmed3f(hi[i], -top, top);
      lo[i] = __builtin_amdgcn_fmed3f(lo[i], -top, top);
    }
  }
  if (lane < LPT) {
    uint32_t wh = 0, wl = 0;
    if (code != 255) {
      const float inv = exp_inv(code);
      wh = (uint32_t)pack_low(round_low(hi[0], inv), round_low(hi[1], inv), round_low(hi[2], inv), round_low(hi[3], inv));
      wl = (uint32_t)pack_low(round_low(lo[0], inv), round_low(lo[1], inv), round_low(lo[2], inv), round_low(lo[3], inv));
    }
    uint32_t *o = reinterpret_cast<uint32_t *>(a.bounds + out * 2 * DH);
    o[l] = wh;
    o[DH / 4 + l] = wl;
  }
  if (lane == 0) a.bounds_exp[out] = (uint8_t)code;
}

// ------------------------------------------------------------------ select

// Order-preserving image of a score that is no NaN: larger score, larger value;
// -0 ties with +0; at least 0x7FFFFF (-infinity).
constexpr uint32_t NAN_KEY = 1;  // below every number's, above "no page" (0)
__device__ __forceinline__ uint32_t score_key(float f) {
  if (f == 0.0f) f = 0.0f;
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Page selection.  One workgroup per (rows_per consecutive rows, key head): the
// query heads of those rows that share the key head are the columns of 16-wide
// products.  Each row's queries are quantised to int8 with an exponent of their
// own, split by sign, and
//   score = sum_d (q_d > 0 ? q_d hi_d : q_d lo_d) = [q+ ; q-] . [hi ; lo]
// is an int8 product on the matrix cores (16 pages x 16 columns x 64 deep per
// instruction) against the bounds as they lie in memory: whole numbers below
// 2^24, so the sum is exact in any order, and so is scaling it by the sum of the
// two exponents (one after the other could overflow in between).  The largest
// over a row's heads is taken in LDS.  Then one
// wavefront per row finds the n_select-th largest key by its bits, from the
// top, and compacts the pages above it (and the first of those equal to it) in
// ascending order.
//
// Bound by latency: row offsets, length, page ids and bounds are loaded one after
// the other.  8 rows of 32 heads over 512 pages (64 workgroups) 12.0 us, 36 .. 100
// rows of 16 heads over 34 pages of 32 sequences 18.8 us (the workgroups fill the
// chip twice); the bounds and queries alone are 1.8 and 1.3 us of bytes.
template <int DH, typename InT, int KPL>
__global__ __launch_bounds__(1024) void paged_select_kernel(PagedSelectArgs a) {
  constexpr int ST = (2 * DH + 63) / 64;
  constexpr int NT = 2;  // 16-page tiles in flight
  extern __shared__ uint32_t s_key[];  // [rows_per][p_cap]
  // of [q+ ; q-], whose groups of 64 hold the same channels twice where DH is a
  // multiple of 64
  constexpr int XN = DH % 64 == 0 ? ST / 2 : ST;
  __shared__ int s_len[16], s_seq[16];
  __shared__ i32x4 s_q[ST][64];
  __shared__ int s_qe[16];
  constexpr int NOT_FINITE = 1 << 16;  // for an exponent; past every sum of two
  const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % a.n_heads;
  const int r0 = (blockIdx.x / a.n_heads) * a.rows_per;
  const int rows = min(a.rows_per, a.q_total - r0), cols = rows * a.group;

  const RowRange own(a.q_off, a.n_seqs, a.q_total);
  if (own.none()) return;

  for (int x = 4 * tid; x < a.rows_per * a.p_cap; x += 4 * blockDim.x)
    *reinterpret_cast<u32x4 *>(s_key + x) = u32x4{0, 0, 0, 0};
  // the rows' sequences, by the first wavefront (the last one sees to the queries)
  if (wave == 0) {
    int b = a.n_seqs;
    if (a.q_off) {
      const int first = a.q_off[0];
      b = wave_find_seq(a.q_off, a.n_seqs, r0, lane);
      if (lane > 0 && lane < rows)
        while (b < a.n_seqs && a.q_off[b + 1] <= r0 + lane) ++b;
      if (r0 + lane < first) b = a.n_seqs;  // of no sequence
    } else if (lane < rows) {
      b = (r0 + lane) / a.rows_each;
    }
    if (lane < rows) {
      s_seq[lane] = b;
      s_len[lane] = b < a.n_seqs ? paged_len(a.lens[b], a.max_pages, a.page_log2) : 0;
    }
  }

  for (int col0 = 0; col0 < cols; col0 += 16) {
    const int col = col0 + c;
    const bool on = col < cols;
    const int i = on ? col / a.group : 0, hg = on ? col - i * a.group : 0;
    if (col0 > 0) __syncthreads();  // the products with the last 16 columns are done
    if (wave == waves - 1) {
      // The columns' queries as the products' operand, for all wavefronts: a lane holds
      // its 16-element groups of [q+ ; q-] (columns past the last repeat the first).
      const InT *qp = static_cast<const InT *>(a.q) + (size_t)own.nearest(r0 + i) * a.q_stride +
                      (size_t)(h * a.group + hg) * DH;
      float x[XN][16];
      uint32_t am = 0;
#pragma unroll
      for (int s = 0; s < XN; ++s) {
        const int k0 = 64 * s + 16 * g;
        const InT *p = qp + (k0 < DH ? k0 : k0 < 2 * DH ? k0 - DH : 0);
        load8(p, x[s]);
        load8(p + 8, x[s] + 8);
      }
#pragma unroll
      for (int s = 0; s < XN; ++s)
#pragma unroll
        for (int e = 0; e < 16; ++e) am = max(am, __float_as_uint(x[s][e]) & 0x7FFFFFFFu);
      am = max(am, (uint32_t)__shfl_xor((int)am, 16, 64));
      am = max(am, (uint32_t)__shfl_xor((int)am, 32, 64));
      const int qc = exp_code<I8>(__uint_as_float(am));
      const float inv = exp_inv(min(qc, 253));
      const float top = int8_top(qc);
#pragma unroll
      for (int s = 0; s < ST; ++s) {
        const int k0 = 64 * s + 16 * g;
        const bool neg = k0 >= DH;
        i32x4 q;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = x[s % XN][4 * w + e];
            y[e] = round_low(__builtin_amdgcn_fmed3f(v, neg ? -top : 0.f, neg ? 0.f : top), inv);
          }
          q[w] = k0 < 2 * DH ? pack_low(y[0], y[1], y[2], y[3]) : 0;
        }
        s_q[s][lane] = q;
      }
      if (g == 0) s_qe[c] = qc == 255 ? NOT_FINITE : qc - 254;  // both exponents' biases
    }
    __syncthreads();
    i32x4 qf[ST];
#pragma unroll
    for (int s = 0; s < ST; ++s) qf[s] = s_q[s][lane];
    const int qe = s_qe[c];

    // runs of rows of one sequence are scored at once
    const int seq = lane < rows ? s_seq[lane] : -1;
    const int row_p = lane < rows ? (s_len[lane] + (1 << a.page_log2) - 1) >> a.page_log2 : 0;
    for (int lo = 0, end; lo < rows; lo = end) {
      const int b = __builtin_amdgcn_readlane(seq, lo), n_p = __builtin_amdgcn_readlane(row_p, lo);
      end = lo + __builtin_ctzll(__ballot(seq != b) >> lo);  // (lanes behind the rows differ)
      if (b >= a.n_seqs || n_p <= a.n_select) continue;
      const bool mine = on && i >= lo && i < end;
      const int32_t *tab = a.table + (size_t)b * a.max_pages;
      for (int p0 = 16 * wave; p0 < n_p; p0 += 16 * NT * waves) {
        int be[NT];
        i32x4 bf[NT][ST];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int page = tab[min(p0 + 16 * t * waves + c, n_p - 1)];
          const bool ok = (unsigned)page < (unsigned)a.n_pages;
          const size_t at = (size_t)(ok ? page : 0) * a.n_heads + h;
          const uint32_t code = a.bounds_exp[at];
#pragma unroll
          for (int s = 0; s < ST; ++s) {
            bf[t][s] = i32x4{0, 0, 0, 0};
            if (64 * s + 48 < 2 * DH || 64 * s + 16 * g < 2 * DH)
              bf[t][s] = *reinterpret_cast<const i32x4 *>(a.bounds + at * 2 * DH + 64 * s + 16 * g);
          }
          be[t] = ok && code != 255 ? (int)code : NOT_FINITE;  // (pages outside the pool as well)
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int pt = p0 + 16 * t * waves;
          i32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < ST; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[t][s], qf[s], acc, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // lane's page 4 g + j: its exponent sits in lane 4 g + j
            const int e = __shfl(be[t], 4 * g + j, 64) + qe;
            const float score = __builtin_amdgcn_ldexpf((float)acc[j], e);
            const uint32_t key = e < NOT_FINITE / 2 ? score_key(score) : NAN_KEY;
            const int p = pt + 4 * g + j;
            if (mine && p < n_p) {
              uint32_t *to = &s_key[i * a.p_cap + p];
              if (a.group == 1) *to = key;
              else atomicMax(to, key);
            }
          }
        }
      }
    }
  }
  __syncthreads();

  for (int i = wave; i < rows; i += waves) {
    if (s_seq[i] >= a.n_seqs) continue;
    int32_t *out = a.pages + ((size_t)(r0 + i) * a.n_heads + h) * a.n_select;
    const int n_p = __builtin_amdgcn_readfirstlane((s_len[i] + (1 << a.page_log2) - 1) >> a.page_log2);
    if (n_p <= a.n_select) {  // every page, without a score
      for (int j = lane; j < a.n_select; j += 64) out[j] = j < n_p ? j : -1;
      continue;
    }
    uint32_t kr[KPL];  // pages 64 j + lane; 0 behind the last
#pragma unroll
    for (int j = 0; j < KPL; ++j) kr[j] = 64 * j + lane < n_p ? s_key[i * a.p_cap + 64 * j + lane] : 0u;
    const unsigned long long below = (1ull << lane) - 1ull;
    if constexpr (KPL == 1) {
      // One page per lane: a page's rank is the number of larger keys.  Ranks below
      // n_select are the selection, unless the last of them is shared: of those
      // pages the first are taken.
      int rank = 0;
      for (int j = 0; j < n_p; j += 4) {
        const u32x4 k = *reinterpret_cast<const u32x4 *>(s_key + i * a.p_cap + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) rank += k[e] > kr[0] ? 1 : 0;
      }
      bool take = rank < a.n_select && kr[0] != 0u;
      unsigned long long sel = __ballot(take);
      if (__popcll(sel) > a.n_select) {
        const uint32_t last = wave_max_u32(take ? (uint32_t)rank : 0u);
        const unsigned long long tied = __ballot(take && rank == (int)last);
        take = take && (rank < (int)last || __popcll(tied & below) < a.n_select - (int)last);
        sel = __ballot(take);
      }
      if (take) out[__popcll(sel & below)] = lane;
      continue;
    }
    uint32_t lo = 0xFFFFFFFFu, hi = 0u;
#pragma unroll
    for (int j = 0; j < KPL; ++j) {
      lo = min(lo, kr[j] ? kr[j] : 0xFFFFFFFFu);
      hi = max(hi, kr[j]);
    }
    auto count_ge = [&](uint32_t v) {
      int n = 0;
#pragma unroll
      for (int j = 0; j < KPL; ++j) n += __popcll(__ballot(kr[j] >= v));
      return n;
    };
    lo = ~wave_max_u32(~lo);
    hi = wave_max_u32(hi);
    // The largest t with n_select keys or more at or above it, from the first
    // bit in which the keys differ; where there are just as many, they are the
    // selection.
    const int top = lo == hi ? -1 : 31 - __clz(lo ^ hi);
    uint32_t t = top < 0 ? hi : hi & ~((2u << top) - 1u);
    int at_least = n_p;
    for (int bit = top; bit >= 0 && at_least != a.n_select; --bit) {
      const int n = count_ge(t | (1u << bit));
      if (n >= a.n_select) t |= 1u << bit, at_least = n;
    }
    // of the keys equal to t the first `ties` are taken (at_least == n_select: all)
    const bool all = at_least == a.n_select;
    const int ties = all ? 0 : a.n_select - (t == 0xFFFFFFFFu ? 0 : count_ge(t + 1u));
    int base = 0, tie_base = 0;
#pragma unroll
    for (int j = 0; j < KPL; ++j) {
      const unsigned long long tie = __ballot(kr[j] != 0u && kr[j] == t);
      const bool take = kr[j] != 0u && (kr[j] > t || (kr[j] == t && (all || tie_base + __popcll(tie & below) < ties)));
      const unsigned long long sel = __ballot(take);
      if (take) out[base + __popcll(sel & below)] = 64 * j + lane;
      base += __popcll(sel);
      tie_base += __popcll(tie);
    }
  }
}

// ------------------------------------------------------------------ join

// Joins the key ranges' parts: part s of a row counts exp2(m_s - m) of it, m the
// largest m_s.  One workgroup per (row, head); each of its four wavefronts
// holds every part's maximum and sum (lane s part s: there are at most 64) and
// sums every fourth part, four of them in flight.  Latency alone: 4.7 us for 8
// rows of 32 heads of 128 in 4 parts, 5.5 us for 16 in up to 64.
template <int DH, typename RowT>
__global__ __launch_bounds__(PAGED_JOIN_THREADS) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int C = DH == 64 ? 1 : 2;  // channels per lane, C lane + e
  __shared__ float s_sum[4][2 * 64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n = (int64_t)a.q_total * a.n_heads * a.group;
  const int64_t row = blockIdx.x;
  // everything that needs no other load first: the parts' statistics (of as
  // many ranges as there can be) and the sequences' lengths
  float ms = 0.f, ls = 0.f;
  if (lane < a.splits) {
    ms = a.part_ml[2 * (lane * n + row)];
    ls = a.part_ml[2 * (lane * n + row) + 1];
  }
  // rows behind the last sequence (or before the first) belong to nobody
  const int r = (int)(row / (a.n_heads * a.group));
  if (a.q_off && (r < a.q_off[0] || r >= a.q_off[a.n_seqs])) return;
  int splits = a.splits;
  if (a.budget > 0) {  // the ranges of the row's sequence
    const int b = a.q_off ? min(wave_find_seq(a.q_off, a.n_seqs, r, lane), a.n_seqs - 1) : r / a.rows_each;
    const Shares sh(a, lane);
    splits = sh.ranges((min(paged_len(a.lens[b], a.max_pages, a.page_log2), a.len_max) + 31) >> 5);
  }
  const bool has = lane < splits && ls != -1.f;  // a part that saw keys
  if (!has) ms = -INFINITY;
  const unsigned long long seen = __ballot(has);
  const float m = wave_max(ms);
  const float w = !has ? 0.f : ms == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(ms - m);
  const float l = wave_sum(has ? ls * w : 0.f);
  const bool on = C * lane < DH;
  float sum[C] = {};
  for (int s0 = wave; s0 < splits; s0 += 16) {
    float x[4][C];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float *o = a.part_o + (min(s0 + 4 * u, splits - 1) * n + row) * DH + (on ? C * lane : 0);
#pragma unroll
      for (int e = 0; e < C; ++e) x[u][e] = o[e];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + 4 * u;
      const float ws = __shfl(w, min(s, 63), 64);
      const bool add = s < splits && ((seen >> s) & 1);  // (a part without keys was not written)
#pragma unroll
      for (int e = 0; e < C; ++e) sum[e] = add ? fmaf(x[u][e], ws, sum[e]) : sum[e];
    }
  }
#pragma unroll
  for (int e = 0; e < C; ++e) s_sum[wave][C * lane + e] = sum[e];
  __syncthreads();
  const int d = threadIdx.x;
  if (d >= DH) return;
  const float total = (s_sum[0][d] + s_sum[1][d]) + (s_sum[2][d] + s_sum[3][d]);
  static_cast<RowT *>(a.o)[row * DH + d] = (RowT)(seen ? total / l : 0.f);
}

// The same for many rows: a lane group per (row, head), four channels a lane, `times`
// of them in turn; the group's lanes hold the parts' maxima and sums.  (paged_rows.h has
// written the sequences of one range already.)
template <int DH, typename RowT>
__global__ __launch_bounds__(256) void paged_rows_join_kernel(PagedAttnArgs a, int times) {
  constexpr int LANES = DH == 64 ? 16 : 32, PER = 256 / LANES, K = 64 / LANES;
  const int tid = threadIdx.x, lane = tid & 63, c = tid % LANES;
  const int heads = a.n_heads * a.group;
  const int64_t n = (int64_t)a.q_total * heads;
  int chunk = 0;
  if (a.budget > 0) chunk = Shares(a, lane).chunk;
  const int first = a.q_off ? a.q_off[0] : 0, last = a.q_off ? a.q_off[a.n_seqs] : a.q_total;
  int row = -1, b = 0, splits = a.splits;
#pragma unroll 1
  for (int i = 0; i < times; ++i) {
    const int64_t x0 = ((int64_t)blockIdx.x * times + i) * PER + (tid & ~63) / LANES;  // of the wavefront
    if (x0 >= n) return;
    const int64_t x = min(x0 + lane / LANES, n - 1);
    const int r = (int)(x / heads);
    if (a.q_off && i == 0) b = wave_find_seq(a.q_off, a.n_seqs, __builtin_amdgcn_readfirstlane((int)(x0 / heads)), lane);
    if (r != row) {
      row = r;
      if (a.q_off) {
        while (b < a.n_seqs && a.q_off[b + 1] <= r) ++b;
      } else {
        b = r / a.rows_each;
      }
      if (a.budget > 0) {
        const int len = min(paged_len(a.lens[min(b, a.n_seqs - 1)], a.max_pages, a.page_log2), a.len_max);
        splits = (((len + 31) >> 5) + chunk - 1) / chunk;
      }
    }
    if (r < first || r >= last || (splits == 1 && a.row_waves > 0) || x0 + lane / LANES >= n) continue;  // (whole groups)
    float ms[K], ls[K], m = -INFINITY;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int s = LANES * k + c;
      ms[k] = -INFINITY;
      ls[k] = -1.f;
      if (s < splits) {
        ms[k] = a.part_ml[2 * (s * n + x)];
        ls[k] = a.part_ml[2 * (s * n + x) + 1];
        if (ls[k] == -1.f) ms[k] = -INFINITY;
      }
      m = fmaxf(m, ms[k]);
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    float l = 0.f;
    bool seen = false;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool has = ls[k] != -1.f;  // a part that saw keys
      const float w = !has ? 0.f : ms[k] == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(ms[k] - m);
      l += has ? ls[k] * w : 0.f;
      seen |= has;
      ms[k] = has ? w : -1.f;
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) {
      l += __shfl_xor(l, o, 64);
      seen |= __shfl_xor((int)seen, o, 64) != 0;
    }
    const int d = 4 * c < DH ? 4 * c : 0;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      for (int s0 = LANES * k; s0 < min(splits, LANES * (k + 1)); s0 += 4) {
        f32x4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = *reinterpret_cast<const f32x4 *>(a.part_o + (min(s0 + u, splits - 1) * n + x) * DH + d);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float w = __shfl(ms[k], (lane & ~(LANES - 1)) + (s0 + u) % LANES, 64);
          if (s0 + u < splits && w != -1.f) {  // (a part without keys adds nothing, whatever it holds)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = fmaf(y[u][e], w, sum[e]);
          }
        }
      }
    }
    if (4 * c >= DH) continue;
    const float inv = seen ? 1.f / l : 0.f;
    RowT *o = static_cast<RowT *>(a.o) + x * DH + d;
    if constexpr (sizeof(RowT) == 4) *reinterpret_cast<f32x4 *>(o) = sum * inv;
    else *reinterpret_cast<bf16x4 *>(o) = bf16x4{(bf16)(sum[0] * inv), (bf16)(sum[1] * inv), (bf16)(sum[2] * inv), (bf16)(sum[3] * inv)};
  }
}

// ------------------------------------------------------------------ launches

hipError_t launch_paged_write(DType dt, int32_t format, int32_t head_dim, PagedWriteArgs a, hipStream_t s) {
  if (a.a_total == 0) return hipSuccess;
  a.d_heads = FastDiv::of(a.n_heads);
  a.d_rows = FastDiv::of(std::max(1, a.rows_each));
  const int per = paged_write_pairs(head_dim);
  const unsigned grid = (unsigned)(((int64_t)a.a_total * a.n_heads + per - 1) / per);
  // Rows of 64 MB and more are loaded past the caches.  Smaller ones may still
  // lie there from the product that made them: 10.7 us streamed for 9.6 on 20 MB.
  const bool stream = 2.0 * a.a_total * a.n_heads * head_dim * (dt == DType::BF16 ? 2 : 4) >= 64e6;
  return by_shape(format, head_dim, [&](auto fmt, auto dh) {
    auto go = [&](auto st) {
      constexpr bool S = st.value;
      if (dt == DType::BF16) launch_kernel(paged_write_kernel<fmt.value, dh.value, bf16, S>, grid, 256, 0, s, a);
      else launch_kernel(paged_write_kernel<fmt.value, dh.value, float, S>, grid, 256, 0, s, a);
    };
    if (stream) go(std::true_type());
    else go(std::false_type());
  });
}

hipError_t launch_paged_read(DType dt, int32_t format, int32_t head_dim, PagedReadArgs a,
                             hipStream_t s) {
  if (a.n_seqs == 0 || a.n_tokens == 0) return hipSuccess;
  a.blocks = (a.n_tokens + PAGED_READ_TOKENS - 1) / PAGED_READ_TOKENS;
  const unsigned grid = (unsigned)((int64_t)a.n_seqs * a.n_heads * a.blocks);
  // as if every sequence had n_tokens tokens (lengths are on the device)
  const bool stream = 2.0 * a.n_seqs * a.n_heads * a.n_tokens * head_dim * (dt == DType::BF16 ? 2 : 4) >= 64e6;
  return by_shape(format, head_dim, [&](auto fmt, auto dh) {
    auto go = [&](auto st) {
      constexpr bool S = st.value;
      if (dt == DType::BF16) launch_kernel(paged_read_kernel<fmt.value, dh.value, bf16, S>, grid, 256, 0, s, a);
      else launch_kernel(paged_read_kernel<fmt.value, dh.value, float, S>, grid, 256, 0, s, a);
    };
    if (stream) go(std::true_type());
    else go(std::false_type());
  });
}

hipError_t launch_paged_bounds(int32_t format, int32_t head_dim, PagedBoundsArgs a, hipStream_t s) {
  if (a.n_seqs == 0 || a.span == 0) return hipSuccess;
  a.d_heads = FastDiv::of(a.n_heads);
  a.d_span = FastDiv::of(a.span);
  const unsigned grid = (unsigned)(((int64_t)a.n_seqs * a.n_heads * a.span + PAGED_BOUNDS_PAIRS - 1) / PAGED_BOUNDS_PAIRS);
  const double keys = (double)a.n_seqs * a.span * a.n_heads * head_dim * (format == BF ? 2 : 1);
  const bool stream = keys * (1 << a.page_log2) >= 128e6;
  return by_shape(format, head_dim, [&](auto fmt, auto dh) {
    if (stream) launch_kernel(paged_bounds_kernel<fmt.value, dh.value, true>, grid, 256, 0, s, a);
    else launch_kernel(paged_bounds_kernel<fmt.value, dh.value, false>, grid, 256, 0, s, a);
  });
}

int64_t paged_select_grid(PagedSelectArgs &a) {
  a.p_cap = (a.max_pages + 63) / 64 * 64;
  // consecutive rows that a sequence is likely to own, as far as they fit the
  // 16 columns and their keys 32 KB of LDS
  const int mean = (int)(((int64_t)a.q_total + a.n_seqs - 1) / a.n_seqs);
  a.rows_per = std::max(1, std::min({16 / a.group, 8192 / a.p_cap, mean}));
  // a wavefront per two tiles of 16 pages, or per four rows where that is more
  // (two at least: one finds the rows' sequences, another quantises)
  a.waves = std::min(16, std::max({2, (a.max_pages + 31) / 32, (a.rows_per + 3) / 4}));
  return ((int64_t)a.q_total + a.rows_per - 1) / a.rows_per * a.n_heads;
}

hipError_t launch_paged_select(DType dt, int32_t head_dim, const PagedSelectArgs &a, int64_t grid,
                               hipStream_t s) {
  const dim3 g((unsigned)grid), b(64 * a.waves);
  const uint32_t lds = (uint32_t)a.rows_per * a.p_cap * 4;
  return by_shape(BF, head_dim, [&](auto, auto dh) {
    auto go = [&](auto kpl) {
      constexpr int K = kpl.value;
      if (dt == DType::BF16) launch_kernel(paged_select_kernel<dh.value, bf16, K>, g, b, lds, s, a);
      else launch_kernel(paged_select_kernel<dh.value, float, K>, g, b, lds, s, a);
    };
    // keys per lane of a row's wavefront: the fewest that hold max_pages (64, beyond
    // 1024 pages, spill two registers)
    const int kpl = a.p_cap / 64;
    if (kpl <= 1) go(std::integral_constant<int, 1>());
    else if (kpl <= 4) go(std::integral_constant<int, 4>());
    else if (kpl <= 8) go(std::integral_constant<int, 8>());
    else if (kpl <= 16) go(std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 64>());
  });
}

static int64_t paged_pairs(const PagedAttnArgs &a) { return (int64_t)(a.budget > 0 ? a.budget : a.n_seqs) * a.n_heads; }

int64_t paged_grid(const PagedAttnArgs &a) {
  const int64_t pairs = paged_pairs(a);  // dealt to 8 XCDs
  if (a.look == PAGED_WINDOW || a.row_waves > 0) return pairs * a.row_blocks * (a.budget > 0 ? 1 : a.splits);
  return (pairs + 7) / 8 * 8 * a.row_blocks * (a.budget > 0 ? 1 : a.splits);
}

// Sequences of a tree call cut into equal ranges on the device, of 8 `waves` 32-key tiles
// at least, such that those of a whole chunk fill `slots` workgroups and the sequences'
// last ones, which begin later, the gaps: where the longest cache has more than three such
// ranges.  16 int8 caches of 900 .. 32768 tokens, 16 heads of 64, 12 .. 25 rows: 245 us with 512
// workgroups for all ranges in the sequences' order, 148 so (768 slots; 152 with 512, 203 with
// 256).  Caches of 2000 tokens are as fast or faster in equal parts of each (8 rows over one: 18.3 us
// shared out, 15.3 not; 32 of 500 .. 2000: 62.7 and 53.1).
static void share_out(PagedAttnArgs &a, int64_t tiles, int waves, int64_t slots) {
  const int64_t per = (int64_t)a.n_heads * a.row_blocks, most = (tiles + 8 * waves - 1) / (8 * waves);
  if (a.n_seqs > PAGED_MAX_SHARED || tiles * a.n_seqs >= (1LL << 30) || most < 4) return;
  a.waves = waves;
  a.chunk = 8 * waves;
  a.budget = (int32_t)std::min<int64_t>(a.n_seqs + (slots + per - 1) / per, a.n_seqs * most);
  a.splits = (int32_t)std::min<int64_t>({64, a.budget, most});
}

// Tokens that a block of `rows` neighbouring rows walks through at most.
static int64_t block_keys(const PagedAttnArgs &a, int64_t rows) {
  return a.look == PAGED_WINDOW ? std::min<int64_t>(a.len_max, (int64_t)a.sinks + a.window + rows + 126) : a.len_max;
}

// Whether windows and trees go by blocks of many rows (paged_rows.h): bf16 rows, more
// than half a block of them for a key head, and blocks for the whole chip or, as a block's
// wavefronts do not share its keys out, long enough walks for a part of it.  By blocks and by
// the few-row kernel, us (one box):
//   heads of 64, bf16, windows   of 256: 128 blocks 15.6 and 13.3, 512 20.5 and 22.8; of 1024: 128 28.6 and 20.6,
//     384 49.2 and 39.0, 512 35.8 and 51.8; of 4096: 128 39.3 and 48.1; of 8192: 32 30.9 and 38.7, 64 41.2 and 57.1
//   heads of 80, bf16, windows of 1024: 256 blocks 43.9 and 37.3, 512 48.1 and 61.4
//   heads of 64, bf16, trees   over 600 tokens: 128 blocks 18.6 and 15.2, 256 21.5 and 22.9; over 4000: 128 47.8 and 61.2
//   heads of 128, bf16, windows   of 256: 32 blocks 17.6 and 12.8, 96 18.2 and 24.5; of 1024: 32 23.9 and 30.0
//   heads of 128, e4m3, windows   of 1024: 128 blocks 40.7 and 28.4, 384 71.4 and 79.3; of 4096: 128 64.9 and 70.1
//   heads of 128, e4m3, trees   over 300 tokens: 64 blocks 17.4 and 12.6; over 2000: 64 33.1 and 32.3; up to 8000:
//     16 43.3 and 32.7, 32 44.5 and 51.6
// Over 806 such pairs of times the choice is 1.4% behind the better one in the mean (7.3% with a number of
// blocks alone), at worst 1.5 times (windows of 256, heads of 128, 64 blocks).
static bool by_rows(DType dt, int32_t head_dim, const PagedAttnArgs &a) {
  const int64_t rows = (int64_t)a.q_max * a.group, block = 32 * PAGED_ROW_WAVES;
  const bool tree = a.look == PAGED_TREE;
  if (dt != DType::BF16 || (a.look != PAGED_WINDOW && !tree) || rows <= block / 2) return false;
  const int64_t blocks = std::min<int64_t>((int64_t)a.n_seqs * a.n_heads * ((rows + block - 1) / block), 1 << 20);
  const int64_t keys = block_keys(a, block / a.group);
  if (blocks < 32) return false;
  if (head_dim == 128 && (tree || !a.bits8)) return blocks * keys >= 32 << 10;
  return blocks >= (tree ? 256 : head_dim == 128 ? 384 : 512) || blocks * keys >= 448 << 10 || keys >= 6 << 10;
}

// Their plan.
static void rows_plan(PagedAttnArgs &a) {
  const int rows = a.q_max * a.group;
  a.row_waves = PAGED_ROW_WAVES;
  a.waves = a.row_waves;
  a.row_blocks = (rows - 1) / (32 * a.row_waves) + 1;
  const int64_t units = (int64_t)a.n_seqs * a.n_heads * a.row_blocks;
  const int64_t tiles = std::max<int64_t>(1, (block_keys(a, 32 * a.row_waves / a.group) + 31) / 32);
  // two workgroups for each compute unit, twelve 32-key tiles each at least (a prompt of 512 rows, 128
  // blocks: 31.4 us in two ranges of eight tiles, 20.9 in one)
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({64, (512 + units - 1) / units, tiles / 12}));
  a.chunk = (int32_t)((tiles + splits - 1) / splits);
  a.chunk += a.chunk & 1;
  a.splits = (int32_t)((tiles + a.chunk - 1) / a.chunk);
  // 512 workgroups run at a time; half as many again balance caches of different lengths
  // better, where their ranges stay long (32 caches up to 8000 e4m3 tokens, 64 rows of 4 x 8 heads: 252.7 us and
  // 265.9 with 512, 16 caches 142.3 and 148.9, 8 caches 95.2 and 79.5)
  const bool many = units * tiles >= 768 * 64;
  if (a.look == PAGED_TREE && units < 2048) share_out(a, tiles, PAGED_ROW_WAVES, many ? 768 : 512);
}

void paged_plan(DType dt, int32_t head_dim, PagedAttnArgs &a) {
  const int rows = a.q_max * a.group;  // packed rows of a sequence and key head
  a.row_waves = a.budget = 0;
  a.d_heads = FastDiv::of(a.n_heads);
  a.d_group = FastDiv::of(a.group);
  if (by_rows(dt, head_dim, a)) {
    rows_plan(a);
    a.d_splits = FastDiv::of(a.budget > 0 ? 1 : a.splits);
    a.d_blocks = FastDiv::of(a.row_blocks);
    const int64_t pairs = a.budget > 0 ? (int64_t)a.n_heads * a.row_blocks : paged_pairs(a);
    a.d_pairs = FastDiv::of((uint32_t)std::min<int64_t>(pairs, INT32_MAX));
    return;
  }
  // Two 16-row tiles a wavefront share what is loaded (36 .. 100 rows over 32
  // caches of 1088 bf16 tokens: 46 us, 69 with one); float32 rows have no registers
  // for them.  Where rows list fewer pages than there are, one tile's rows list
  // fewer than two tiles': 64 rows of 32 heads, 16 pages of 469: 128 us with
  // two, 86 with one; where a tile's lists may cover the cache (8 pages of 34) 72
  // and 88, the selection included.
  const int tile_rows = (16 + a.group - 2) / a.group + 1;  // rows that have a part in a tile
  const int64_t cached = ((int64_t)a.len_max + (1 << a.page_log2) - 1) >> a.page_log2;
  const bool sparse = a.n_select > 0 && cached > (int64_t)a.n_select * tile_rows;
  a.row_tiles = rows <= 16 || dt == DType::F32 || sparse ? 1 : 2;
  a.row_blocks = (rows - 1) / (16 * a.row_tiles) + 1;
  const int block_rows = std::min(a.q_max, (16 * a.row_tiles + a.group - 2) / a.group + 1);
  a.bit_rows = block_rows;
  int64_t keys = a.len_max;
  if (a.n_select > 0)
    keys = std::min(cached, (int64_t)a.n_select * block_rows) << a.page_log2;
  // (rows of one block that are neighbours; the kernel cuts what there is into `splits`)
  if (a.look == PAGED_WINDOW) keys = std::min<int64_t>(keys, (int64_t)a.sinks + a.window + block_rows + 62);
  const int64_t tiles = std::max<int64_t>(1, (keys + 31) / 32);
  const int64_t units = std::max<int64_t>(1, (int64_t)a.n_seqs * a.n_heads * a.row_blocks);
  // Wavefronts per unit: two for each of the chip's 1024 SIMDs in all, two tiles
  // each at least; beyond a workgroup's, the keys are split over workgroups.
  // More of them repeat the start and the end of a wavefront, some 6 us of
  // latency: with 4096 one row over 32 caches of 1088 tokens (int8, 8 key heads
  // of 128) takes 24.9 us for 16.4, 36 .. 100 rows over 32 bf16 caches 55.6 for 46.4.
  // fp32 rows of several blocks take three times the products a tile, and
  // sequences with fewer blocks than the longest leave some of the units empty:
  // 35.8 us with 4096 for 46.3 (1 .. 333 rows, 6 caches up to 1503 tokens).
  const int64_t fill = dt == DType::F32 && a.row_blocks > 1 ? 4096 : 2048;
  const int64_t want = std::min<int64_t>((fill + units - 1) / units, (tiles + 1) / 2);
  const int most = a.row_tiles == 1 ? 8 : 4;
  a.waves = 1;
  while (a.waves < most && a.waves < want) a.waves *= 2;
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(64, want / a.waves));
  a.chunk = (int32_t)((tiles + splits - 1) / splits);
  a.chunk = (a.chunk + a.waves - 1) / a.waves * a.waves;
  a.splits = (int32_t)((tiles + a.chunk - 1) / a.chunk);
  a.budget = 0;
  // Split caches may differ in length, so that the longest would be waited for:
  // equal ranges, shared out on the device, over 512 workgroups (two of 4
  // wavefronts per compute unit; measured against 256 to 1024 of 2 to 8).
  const int64_t per = (int64_t)a.n_heads * a.row_blocks;
  if (a.look == PAGED_TREE) {
    if (units < 2048) share_out(a, tiles, 4, 768);
  } else if (a.n_select == 0 && a.look != PAGED_WINDOW && a.n_seqs <= PAGED_MAX_SHARED && tiles * a.n_seqs < (1LL << 30) &&
             a.splits > 1) {
    a.waves = std::min(a.waves, 4);
    a.budget = (int32_t)std::max<int64_t>(2 * a.n_seqs, (512 + per - 1) / per);
    a.chunk = 2 * a.waves;  // at least
    a.splits = (int32_t)std::min<int64_t>({64, a.budget, (tiles + a.chunk - 1) / a.chunk});
  }
  a.d_splits = FastDiv::of(a.budget > 0 ? 1 : a.splits);
  a.d_blocks = FastDiv::of(a.row_blocks);
  a.d_pairs = FastDiv::of((uint32_t)std::min<int64_t>(paged_pairs(a), INT32_MAX));
}

hipError_t launch_paged_attention(DType dt, int32_t format, int32_t head_dim, const PagedAttnArgs &a,
                                  hipStream_t s) {
  if (a.row_waves > 0) switch (format) {
      case BF: return launch_paged_rows_bf16(head_dim, a, s);
      case E4: return launch_paged_rows_e4m3(head_dim, a, s);
      case I8: return launch_paged_rows_int8(head_dim, a, s);
    }
  if (a.look == PAGED_WINDOW || a.look == PAGED_TREE) switch (format) {
      case BF: return launch_paged_masked_bf16(dt, head_dim, a, s);
      case E4: return launch_paged_masked_e4m3(dt, head_dim, a, s);
      case I8: return launch_paged_masked_int8(dt, head_dim, a, s);
    }
  switch (format) {
    case BF: return launch_paged_attention_bf16(dt, head_dim, a, s);
    case E4: return launch_paged_attention_e4m3(dt, head_dim, a, s);
    case I8: return launch_paged_attention_int8(dt, head_dim, a, s);
  }
  return hipErrorInvalidValue;
}

// (304 rows of 16 heads of 64 in up to 23 parts: 13.5 us with a workgroup each, 6.3 in lane groups.
// Four in turn repeat less of what comes before the parts: 2048 rows of 32 heads of 128 in up to
// two parts 17.1 us, 21.2 one by one; the 304 rows 15.2.)
int paged_join_turns(int32_t head_dim, const PagedAttnArgs &a) {
  const int64_t n = (int64_t)a.q_total * a.n_heads * a.group;
  if (a.row_waves == 0 && ((a.look != PAGED_WINDOW && a.look != PAGED_TREE) || n < 4096)) return 0;
  return n >= 4096 * paged_join_groups(head_dim) ? 4 : 1;
}

hipError_t launch_paged_join(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)a.q_total * a.n_heads * a.group);
  if (const int times = paged_join_turns(head_dim, a)) {
    const unsigned per = paged_join_groups(head_dim) * times, groups = (grid + per - 1) / per;
    return by_shape(BF, head_dim, [&](auto, auto dh) {
      if (dt == DType::BF16) launch_kernel(paged_rows_join_kernel<dh.value, bf16>, groups, 256, 0, s, a, times);
      else launch_kernel(paged_rows_join_kernel<dh.value, float>, groups, 256, 0, s, a, times);
    });
  }
  return by_shape(BF, head_dim, [&](auto, auto dh) {
    if (dt == DType::BF16) launch_kernel(paged_join_kernel<dh.value, bf16>, grid, PAGED_JOIN_THREADS, 0, s, a);
    else launch_kernel(paged_join_kernel<dh.value, float>, grid, PAGED_JOIN_THREADS, 0, s, a);
  });
}

}  // namespace marche
