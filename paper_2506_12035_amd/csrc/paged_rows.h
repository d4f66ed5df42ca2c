// Attention of many rows over windows and drafted trees in the paged cache (the kernel
// template; one translation unit per cache format instantiates it).
//
// The packed rows of a sequence and key head (its query heads times the sequence's rows)
// go 32 to a wavefront and QB wavefronts to a workgroup, which share tiles of 64 keys in
// LDS, in bf16 whatever the cache's format: a key is loaded and converted once for 32 QB
// rows.  Tiles go memory -> registers -> one of two LDS slots, the next one's loads in
// flight during a tile's products.  S^T = K Q^T (32 keys x 32 rows an instruction): lane l owns row l & 31, so
// that the row maximum takes one exchange between the halves and the rescale is a
// per-lane factor; O^T += V^T P^T with P in registers and V^T from the transposing LDS
// read.  Softmax statistics and O are float32, the maximum trails by at most 2^8, P is
// rounded to bf16 (half a step, 2^-8 of each weight; not in the weights' sum).
//
// Bound: LDS, which every wavefront reads 32 KB a tile from (heads of 128) for 32 products'
// 1024 cycles, beside 1100 cycles of vector instructions: 8192 rows of 32 heads over
// windows of 8192 take 537 .. 599 us by the box (0.92 .. 1.02 PFLOP/s); where they took 599, 479 without its
// reads, 503 without loads to it, 368 without either.  Over windows of 1024 (172 .. 190 us by the box, 0.68 .. 0.75
// PFLOP/s) the start and the end of each workgroup count too: windows of one token take 57 us.  8-bit formats
// convert a tile once for the workgroup: 213 .. 218 us in e4m3, 231 in int8.
#pragma once

#include "paged_attn.h"

namespace marche {

constexpr int ROWS_TK = 64;  // keys of a tile

// Bytes of LDS of a workgroup: two for each compute unit fit.
template <int FMT, int DH>
constexpr int rows_lds = ROWS_TK * DH * (FMT == BF ? 8 : 10) + (DH == 80 && FMT == BF ? 64 : 0);

// A tile's K or V in LDS: rows of DH bf16 one after another, as wide loads to LDS place
// them.  Chunks of 16 bytes of a row are permuted by an XOR with the row's reversed low
// bits, so that the 16 rows of a K fragment read, and the four rows by four chunks of a
// V^T read, lie in different banks (rows of 80, at 160 bytes, do so nearly by themselves).
template <int DH>
struct RowsLay {
  static constexpr int CPR = DH / 8;             // chunks of a row
  static constexpr int RB = 2 * DH;              // bytes of a row
  static constexpr int TILE = ROWS_TK * RB;
  static constexpr int DB = (DH + 31) / 32;      // 32-channel blocks of O
  // (V's last channels of a 32-channel block past 80 are read from the next row, the last
  // row's from behind the tile: they only reach outputs that do not exist)
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (DH == 128) return (int)(__builtin_bitreverse32((uint32_t)row) >> 28);
    else if constexpr (DH == 64) return (int)(__builtin_bitreverse32((uint32_t)row >> 1) >> 29);
    else return 0;
  }
  static __device__ __forceinline__ int at(int row, int c) { return row * RB + ((c ^ swz(row)) << 4); }
};

typedef short rows_s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ rows_s16x4 rows_read_tr(const char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((rows_s16x4 __attribute__((address_space(3))) *)(
      (__attribute__((address_space(3))) char *)(uintptr_t)p));
}

// 16 bytes a lane from memory to LDS, lane l's to lds + 16 l.  Written out, as the compiler
// waits for the builtin's loads before every LDS read that it cannot tell from their
// target; no register waits for the data, and rows_arrive() does.
__device__ __forceinline__ void load_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds(uint32_t lds, const void *at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds), "v"(at) : "memory", "m0");
}
__device__ __forceinline__ void rows_arrive() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0); the compiler counts by it too
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ uint64_t below64(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

// Largest of the two lanes that share a row.
__device__ __forceinline__ float half_max(float v) {
  auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// (Three workgroups a compute unit for 8-bit heads of 64, which spill 6 or 7 registers for it: 8192 rows
// of 12 heads over windows of 1024 in e4m3 59.8 us, 75.4 with two and no spill; 32 trees of 64 x 4 x 8 over 1100 ..
// 8000 tokens 154 and 168; windows of 8192 206 and 196.)
template <int FMT, int DH, int QB, int MODE>
__global__ __launch_bounds__(QB * 64, DH == 64 && FMT != BF ? 3 : 2) void paged_rows_kernel(PagedAttnArgs a, const int32_t *__restrict__ table) {
  using L = RowsLay<DH>;
  constexpr bool WIN = MODE == PAGED_WINDOW;
  constexpr int T = QB * 64;
  constexpr int ES = FMT == BF ? 2 : 1;
  constexpr int PPR = DH * ES / 16;                  // 16-byte pieces of a cached row
  constexpr int PIECES = ROWS_TK * PPR;              // of a tile's K, and of its V
  constexpr int N = (PIECES + T - 1) / T;            // of those per thread
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // tiles of K, K, V, V; 8-bit rows of K, V
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hf = lane >> 5;

  // (sequence, head, row block, key range): see PagedUnit; where sequences are cut into equal
  // ranges on the device, the longest ranges come first, a range's heads and blocks together.
  const bool shared = !WIN && a.budget > 0;
  int split_i, chunk = a.chunk, ranges = a.splits, b, h, rb;
  if (shared) {
    const int x = (int)a.d_pairs.div(blockIdx.x), y = blockIdx.x - x * (a.n_heads * a.row_blocks);
    rb = (int)a.d_heads.div(y);
    h = y - rb * a.n_heads;
    const Shares sh(a, lane);
    chunk = sh.chunk;
    b = __builtin_amdgcn_readfirstlane(sh.find_long_first(x, lane, split_i));
    if (b < 0) return;
  } else {
    const PagedUnit u(a, blockIdx.x, a.n_seqs * a.n_heads);
    split_i = u.split;
    rb = u.block;
    b = (int)a.d_heads.div(u.pair);
    h = u.pair - b * a.n_heads;
  }
  const int32_t *tab = table + (size_t)b * a.max_pages;
  const int len = min(paged_len(a.lens[b], a.max_pages, a.page_log2), a.len_max);
  if (shared) ranges = max(1, (((len + 31) >> 5) + chunk - 1) / chunk);
  int row0 = b * a.rows_each, row1 = row0 + a.rows_each;
  if (a.q_off) {
    row0 = min(max(a.q_off[b], 0), a.q_total);
    row1 = min(max(a.q_off[b + 1], row0), a.q_total);
  }
  const int packed = min(row1 - row0, a.q_max) * a.group;
  const int p0 = rb * 32 * QB;
  if (p0 >= packed) return;
  auto row_of = [&](int p) { return (int)a.d_group.div(p); };
  const int i0 = row_of(p0), i1 = row_of(min(p0 + 32 * QB, packed) - 1);

  // This lane's row; columns behind the last row repeat the block's first.
  const int pr = p0 + 32 * wave + col;
  const bool live = p0 + 32 * wave < packed;
  const bool on = pr < packed;
  const int i = on ? row_of(pr) : i0, hg = on ? pr - i * a.group : 0;
  const int out = on ? (row0 + i) * (a.n_heads * a.group) + h * a.group + hg : -1;
  const bf16 *q = static_cast<const bf16 *>(a.q) + (size_t)(row0 + i) * a.q_stride + (size_t)(h * a.group + hg) * DH;
  bf16x8 qf[DH / 16];
#pragma unroll
  for (int s = 0; s < DH / 16; ++s) qf[s] = *reinterpret_cast<const bf16x8 *>(q + 16 * s + 8 * hf);

  // The range's keys, in tiles; all uniform.
  const int ctx = WIN ? 0 : max(a.ctx[b], 0);
  const uint32_t *mask = WIN ? nullptr : a.mask + (size_t)(row0 + i) * a.mask_words;
  int w_lo = 0, w_hi = 0, base = 0, end = len, t0, t1;
  Span sp{};
  WindowWalk<ROWS_TK> walk{};
  if constexpr (WIN) {
    window_of(a, len, a.q_idx[row0 + i], w_lo, w_hi);
    // of the block's rows, 64 at a time
    sp = span_of(a, len, row0 + i0, min(i1 - i0 + 1, 64), lane);
    if (i1 - i0 >= 64) {
      const Span s2 = span_of(a, len, row0 + i0 + 64, i1 - i0 - 63, lane);
      sp = Span{min(sp.lo_min, s2.lo_min), max(sp.lo_max, s2.lo_max), min(sp.hi_min, s2.hi_min), max(sp.hi_max, s2.hi_max)};
    }
    end = sp.hi_max;
    walk = WindowWalk<ROWS_TK>::of(sp.lo_min, end, a.sinks);
    chunk = (int)((uint32_t)(walk.tiles + a.splits - 1) / (uint32_t)a.splits);
    t0 = split_i * chunk;
    t1 = min(t0 + chunk, walk.tiles);
  } else {
    base = 32 * chunk * split_i;
    end = min(len, base + 32 * chunk);
    t0 = 0;
    t1 = (max(end - base, 0) + ROWS_TK - 1) / ROWS_TK;
  }
  auto key_of = [&](int t) { return WIN ? walk.key(t) : base + ROWS_TK * t; };

  // Page ids of a tile's four 16-key parts, -1 where there are no tokens.  Uniform, from a
  // register that holds those of 16 tiles, the last of which may lie behind the range, asked
  // for in order (scalar loads in the loop would make the waits for LDS reads waits for them).
  struct Pages {
    int id[4];
  };
  int ids = -1, ids_at = t0 - 16;
  auto pages_of = [&](int t) {
    if (t - ids_at >= 16) {
      ids_at = t;
      const int key = token_of(key_of, t + (lane >> 2), t1, lane & 3, end);
      const int x = key >= 0 ? tab[key >> a.page_log2] : -1;
      ids = (unsigned)x < (unsigned)a.n_pages ? x : -1;
    }
    Pages p;
#pragma unroll
    for (int j = 0; j < 4; ++j) p.id[j] = __builtin_amdgcn_readlane(ids, 4 * (t - ids_at) + j);
    return p;
  };
  auto slot_of = [&](int id, int key) {
    return (((size_t)max(id, 0) * a.n_heads + h) << a.page_log2) + (key & ((1 << a.page_log2) - 1));
  };
  // whether all of a tile's tokens exist
  auto full = [&](int key, const Pages &p) { return key + ROWS_TK <= end && (p.id[0] | p.id[1] | p.id[2] | p.id[3]) >= 0; };

  // A tile's K or V straight to LDS, 1 KB an instruction, lane l to the l-th 16 bytes: bf16 to
  // its place (a lane fetches the chunk that belongs there), 8 bits as they are, row by row,
  // for convert().  Rows without a token get what lies there.
  constexpr int OPS = PIECES / 64;
  auto fetch = [&](const void *from, int t, const Pages &p, char *to) {
    const int key = key_of(t);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int op = n * QB + wave;
      if (OPS % QB != 0 && op >= OPS) break;
      const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(to + 1024 * op));
      if constexpr (DH == 80) {
        const int x = 64 * op + lane, row = x / PPR, j = row >> 4;
        const int id = j == 0 ? p.id[0] : j == 1 ? p.id[1] : j == 2 ? p.id[2] : p.id[3];
        load_lds(lds, static_cast<const char *>(from) + slot_of(id, key + row) * (DH * ES) + 16 * (x - row * PPR));
      } else {  // (the instruction's rows lie in one 16-key part)
        const int row = 64 * op / PPR, j = row >> 4, in = lane / PPR;
        const int id = j == 0 ? p.id[0] : j == 1 ? p.id[1] : j == 2 ? p.id[2] : p.id[3];
        const int c = FMT == BF ? (lane % PPR) ^ L::swz(row + in) : lane % PPR;
        load_lds(lds, static_cast<const char *>(from) + slot_of(id, key + row) * (DH * ES), (uint32_t)(in * (DH * ES) + 16 * c));
      }
    }
  };
  // The exponent codes of the rows whose pieces this lane fetches.
  struct Codes {
    uint8_t c[N];
  };
  auto fetch_codes = [&](const uint8_t *exps, int t, const Pages &p) {
    Codes o;
    const int key = key_of(t);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int op = min(n * QB + wave, OPS - 1), row = (64 * op + (DH == 80 ? lane : 0)) / PPR, j = row >> 4;
      const int id = j == 0 ? p.id[0] : j == 1 ? p.id[1] : j == 2 ? p.id[2] : p.id[3];
      if constexpr (DH == 80) o.c[n] = exps[slot_of(id, key + row)];
      else o.c[n] = at<uint8_t>(scalar(exps + slot_of(id, key + row)), (uint32_t)(lane / PPR), 0);
    }
    return o;
  };
  // The pieces that this lane fetched, in bf16 to their places (rows without a token: zeros).
  struct Raw {
    u32x4 w[N];
  };
  auto read_raw = [&](const char *raw) {
    Raw o;
#pragma unroll
    for (int n = 0; n < N; ++n) o.w[n] = *reinterpret_cast<const u32x4 *>(raw + 16 * min(64 * (n * QB + wave) + lane, PIECES - 1));
    return o;
  };
  auto convert = [&](const Raw &raw, const Codes &codes, int t, const Pages &p, char *to) {
    const bool whole = full(key_of(t), p);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      __builtin_amdgcn_sched_barrier(0);  // (a piece at a time: there are no registers for more)
      const int op = n * QB + wave;
      if (OPS % QB != 0 && op >= OPS) break;
      const int x = 64 * op + lane, row = x / PPR, part = x - row * PPR;
      u32x4 w = raw.w[n];
      float s = exp_scale(codes.c[n]);
      if (!whole) {
        const int j = row >> 4, id = j == 0 ? p.id[0] : j == 1 ? p.id[1] : j == 2 ? p.id[2] : p.id[3];
        if (id < 0 || key_of(t) + row >= end) w = u32x4{0u, 0u, 0u, 0u}, s = 1.f;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (FMT == E4) {
            o[2 * j] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + j], s, false));
            o[2 * j + 1] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + j], s, true));
          } else {  // (a whole number of seven bits times a power of two: exact)
            float f[4];
            unpack4<I8>(w[2 * i + j], s, f);
            o[2 * j] = hi16(__float_as_uint(f[0]), __float_as_uint(f[1]));
            o[2 * j + 1] = hi16(__float_as_uint(f[2]), __float_as_uint(f[3]));
          }
        }
        *reinterpret_cast<u32x4 *>(to + L::at(row, 2 * part + i)) = o;
      }
    }
  };
  // zeros for V's rows without a token: they may hold anything
  auto clear = [&](int t, const Pages &p, char *to) {
    const int key = key_of(t);
    for (int x = tid; x < ROWS_TK * L::CPR; x += T) {
      const int row = x / L::CPR, j = row >> 4;
      const int id = j == 0 ? p.id[0] : j == 1 ? p.id[1] : j == 2 ? p.id[2] : p.id[3];
      if (id < 0 || key + row >= end) *reinterpret_cast<u32x4 *>(to + 16 * x) = u32x4{0u, 0u, 0u, 0u};
    }
  };

  float m_run = -INFINITY, l_run = 0.f;
  bool seen = false;
  f32x16 acc[L::DB];
#pragma unroll
  for (int d = 0; d < L::DB; ++d) acc[d] = f32x16{};

  // Fragment addresses within a tile: one base each, the chunk by an XOR.
  const int g = lane >> 4, e = (lane & 15) >> 2, qd = lane & 3;
  const uint32_t k_base = L::at(col, hf);
  const uint32_t v_base = L::at(4 * hf + e, 2 * (g & 1) + (qd >> 1)) + 8 * (qd & 1);
  // K's rows 32 kb + col, chunk 2 st + hf
  auto k_frag = [&](const char *kt, uint32_t kbase, int kb, int st) {
    const uint32_t at = DH == 80 ? kbase + 32 * st : kbase ^ (32 * st);
    return *reinterpret_cast<const bf16x8 *>(kt + at + 32 * kb * L::RB);
  };
  // V^T's channels 32 db .. of keys 16 y + 4 hf .. + 3 and 8 further on
  auto v_frag = [&](const char *vt, uint32_t vbase, int y, int db) {
    const uint32_t at = DH == 80 ? vbase + 64 * db : vbase ^ (64 * db);
    const uint32_t at8 = DH == 80 ? vbase + 64 * db : vbase ^ (64 * db ^ 16);
    const rows_s16x4 v8[2] = {rows_read_tr(vt + at + 16 * y * L::RB), rows_read_tr(vt + at8 + (16 * y + 8) * L::RB)};
    return *reinterpret_cast<const bf16x8 *>(v8);
  };
  // masks and the running maximum
  auto settle = [&](int key, const Pages &p, f32x16 (&s)[2]) {
    bool whole = full(key, p);
    if constexpr (WIN) whole &= key + ROWS_TK <= sp.hi_min && (key >= sp.lo_max || key + ROWS_TK <= a.sinks);
    else whole &= key + ROWS_TK <= ctx;
    if (whole) {
      seen = true;
    } else {
      uint64_t ok = below64(end - key);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (p.id[j] < 0) ok &= ~(0xFFFFull << (16 * j));
      if constexpr (WIN) {
        ok &= below64(w_hi - key) & (~below64(w_lo - key) | below64(a.sinks - key));
      } else {
        uint64_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m |= (uint64_t)tree_bits(mask, a.mask_words, key + 16 * j - ctx) << (16 * j);
        ok &= m;
      }
      seen |= ok != 0;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t w = (uint32_t)(ok >> (32 * kb)) >> (4 * hf);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!((w >> ((r >> 2) * 8 + (r & 3))) & 1u)) s[kb][r] = -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    if (__any(mx * a.sl2 > m_run + 8.f)) {
      const float m_new = fmaxf(m_run, half_max(mx) * a.sl2);
      const float al = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= al;
#pragma unroll
      for (int d = 0; d < L::DB; ++d) acc[d] *= al;
    }
  };
  // The tile's softmax and product with V, and between them the next tile's logits, a quarter
  // at a time: quarter y is the keys 16 y + 4 hf .. + 3 and 8 further on, whose weights are
  // formed during the products of the quarter before, whose fragments are read from LDS
  // half a quarter ahead.  The order is written out (the barriers only bind the compiler):
  // left to itself it reads every fragment right before its product.
  constexpr int ST = DH / 16;  // products of 32 keys' logits
  auto work = [&](const char *vt, const char *kt, f32x16 (&s)[2], f32x16 (&s_next)[2]) {
    uint32_t kbase = k_base, vbase = v_base;
    asm("" : "+v"(kbase), "+v"(vbase));  // (their XORs are not kept outside the loop)
    bf16x8 kf[(ST + 1) / 2], vf[L::DB];
    auto read_k = [&](int y) {
#pragma unroll
      for (int n = ST * y / 2; n < ST * (y + 1) / 2; ++n) kf[n - ST * y / 2] = k_frag(kt, kbase, n / ST, n % ST);
    };
    auto read_v = [&](int y) {
#pragma unroll
      for (int db = 0; db < L::DB; ++db) vf[db] = v_frag(vt, vbase, y, db);
    };
    read_k(0);
    read_v(0);
    __builtin_amdgcn_sched_barrier(0);
    // (products first: the other workgroup's wavefront fills what they leave; 580 us without
    // for 8192 rows over windows of 8192, 561 with)
    __builtin_amdgcn_s_setprio(1);
    const float mm = m_run == -INFINITY ? 0.f : -m_run;
    float x[8];
    auto weight = [&](int y, int i) {
      x[i] = __builtin_amdgcn_exp2f(fmaf(s[y / 2][8 * (y % 2) + i], a.sl2, mm));
    };
    bf16x8 pb;
    auto round_weights = [&]() {
      l_run += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
      for (int i = 0; i < 8; ++i) pb[i] = (bf16)x[i];
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) weight(0, i);
    round_weights();
    s_next[0] = s_next[1] = f32x16{};
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int n0 = ST * y / 2, ns = ST * (y + 1) / 2 - n0, nm = ns + L::DB;
#pragma unroll
      for (int j = 0; j < ns + L::DB; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        if (j < ns) {
          const int n = n0 + j;
          s_next[n / ST] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], qf[n % ST], s_next[n / ST], 0, 0, 0);
        } else {
          acc[j - ns] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j - ns], pb, acc[j - ns], 0, 0, 0);
        }
        if (y < 3) {
#pragma unroll
          for (int i = 8 * j / nm; i < 8 * (j + 1) / nm; ++i) weight(y + 1, i);
          if (j == ns - 1) read_k(y + 1);
        }
      }
      if (y < 3) {
        read_v(y + 1);
        round_weights();
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
  };
  // Tile t's logits are formed during tile t - 1's softmax and product: K runs a tile ahead of
  // V.  Slot x of K and of V holds tiles of parity x; behind them lie the 8-bit rows.
  auto k_slot = [&](int x) { return smem + x * L::TILE; };
  auto v_slot = [&](int x) { return smem + (2 + x) * L::TILE; };
  char *k_raw = smem + 4 * L::TILE, *v_raw = k_raw + 16 * PIECES;
  if (t0 < t1) {
    Pages p0 = pages_of(t0), p1 = pages_of(min(t0 + 1, t1 - 1)), p2 = pages_of(min(t0 + 2, t1 - 1));
    const int second = min(t0 + 1, t1 - 1);
    if constexpr (FMT == BF) {
      fetch(a.k, t0, p0, k_slot(0));
      fetch(a.v, t0, p0, v_slot(0));
      fetch(a.k, second, p1, k_slot(1));
      rows_arrive();
      __syncthreads();
      if (!full(key_of(t0), p0)) {
        clear(t0, p0, v_slot(0));
        __syncthreads();
      }
    } else {
      // (the third one's rows where V's tile 1 will be)
      fetch(a.k, t0, p0, k_raw);
      fetch(a.v, t0, p0, v_raw);
      fetch(a.k, second, p1, v_slot(1));
      const Codes c0 = fetch_codes(a.k_exp, t0, p0), c1 = fetch_codes(a.v_exp, t0, p0), c2 = fetch_codes(a.k_exp, second, p1);
      rows_arrive();
      const Raw r0 = read_raw(k_raw), r1 = read_raw(v_raw), r2 = read_raw(v_slot(1));
      convert(r0, c0, t0, p0, k_slot(0));
      convert(r1, c1, t0, p0, v_slot(0));
      convert(r2, c2, second, p1, k_slot(1));
      __syncthreads();
    }
    f32x16 sa[2], sb[2];
    if (live) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        sa[kb] = f32x16{};
#pragma unroll
        for (int st = 0; st < DH / 16; ++st)
          sa[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(k_slot(0), k_base, kb, st), qf[st], sa[kb], 0, 0, 0);
      }
    }
    __syncthreads();  // (the first tile's K is read: the third one's takes its place)
    // one tile of parity `par` (behind the last tile the logits are of what lies in LDS, and
    // not used)
    auto step = [&](int t, auto par, f32x16 (&s)[2], f32x16 (&s_next)[2]) {
      constexpr int X = par.value;
      const bool second = t + 1 < t1, third = t + 2 < t1;
      Codes kc, vc;
      if (third) fetch(a.k, t + 2, p2, FMT == BF ? k_slot(X) : k_raw);
      if (second) fetch(a.v, t + 1, p1, FMT == BF ? v_slot(1 - X) : v_raw);
      if constexpr (FMT != BF) {
        kc = fetch_codes(a.k_exp, min(t + 2, t1 - 1), p2);
        vc = fetch_codes(a.v_exp, min(t + 1, t1 - 1), p1);
      }
      const Pages p3 = pages_of(min(t + 3, t1 - 1));
      if (live) {
        settle(key_of(t), p0, s);
        work(v_slot(X), k_slot(1 - X), s, s_next);
      }
      rows_arrive();
      if constexpr (FMT != BF) {
        const Raw kr = read_raw(k_raw), vr = read_raw(v_raw);
        if (third) convert(kr, kc, t + 2, p2, k_slot(X));
        if (second) convert(vr, vc, t + 1, p1, v_slot(1 - X));
      }
      __syncthreads();
      if constexpr (FMT == BF) {
        if (second && !full(key_of(t + 1), p1)) {
          clear(t + 1, p1, v_slot(1 - X));
          __syncthreads();
        }
      }
      p0 = p1;
      p1 = p2;
      p2 = p3;
    };
#pragma unroll 1
    for (int t = t0; t < t1; t += 2) {
      step(t, std::integral_constant<int, 0>(), sa, sb);
      if (t + 1 < t1) step(t + 1, std::integral_constant<int, 1>(), sb, sa);
    }
  }

  // channel of register r of block d
  auto chan = [&](int d, int r) { return 32 * d + (r >> 2) * 8 + 4 * hf + (r & 3); };
  const float l = half_sum(l_run);
  bool bad = false;
#pragma unroll
  for (int d = 0; d < L::DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (32 * d + (r >> 2) * 8 < DH) bad |= !(fabsf(acc[d][r]) < INFINITY);
  // A weight of zero times an infinite or NaN value that this row does not see is NaN:
  // such a block is computed again, row by row over each row's own keys (rows whose own
  // logits are NaN aside: all of theirs is NaN).
  const bool direct = ranges == 1;
  // (the tiles have been read; a last one's barrier lies behind)
  volatile int *again = reinterpret_cast<int *>(smem);
  if (tid == 0) *again = 0;
  __syncthreads();
  if (bad && l == l) *again = 1;
  __syncthreads();
  if (*again) {
    PagedAttnArgs one = a;
    if (direct) one.splits = 1;
    one_by_one<FMT, DH, bf16>(
        one, tab, [&](int pos) { return WIN && pos >= ROWS_TK * walk.sink_tiles ? pos + ROWS_TK * walk.jump : pos; },
        [&](int x, int key) {
          if constexpr (WIN) {
            int lo, hi;
            window_of(a, len, a.q_idx[row0 + x], lo, hi);
            return key < hi && (key >= lo || key < a.sinks);
          } else {
            return key < end && (tree_bits(a.mask + (size_t)(row0 + x) * a.mask_words, a.mask_words, key - ctx) & 1u) != 0;
          }
        },
        p0, min(p0 + 32 * QB, packed), row0, h, split_i, len, base + ROWS_TK * t0, base + ROWS_TK * t1, wave, QB, lane);
    return;
  }
  if (out < 0) return;
  if (direct) {
    const float inv = seen ? 1.f / l : 0.f;
    bf16 *o = static_cast<bf16 *>(a.o) + (size_t)out * DH;
#pragma unroll
    for (int d = 0; d < L::DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        if (32 * d + 2 * r < DH)
          *reinterpret_cast<bf16x4 *>(o + chan(d, r)) = bf16x4{(bf16)(acc[d][r] * inv), (bf16)(acc[d][r + 1] * inv),
                                                               (bf16)(acc[d][r + 2] * inv), (bf16)(acc[d][r + 3] * inv)};
    return;
  }
  const size_t part = (size_t)split_i * a.q_total * (a.n_heads * a.group) + out;
#pragma unroll
  for (int d = 0; d < L::DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      if (32 * d + 2 * r < DH)
        *reinterpret_cast<f32x4 *>(a.part_o + part * DH + chan(d, r)) = f32x4{acc[d][r], acc[d][r + 1], acc[d][r + 2], acc[d][r + 3]};
  if (hf == 0) {
    a.part_ml[2 * part] = m_run;
    a.part_ml[2 * part + 1] = seen ? l : -1.f;
  }
}

template <int FMT, int DH, int QB, int MODE>
hipError_t launch_paged_rows_mode(const PagedAttnArgs &a, hipStream_t s) {
  constexpr int lds = rows_lds<FMT, DH>;
  auto kernel = paged_rows_kernel<FMT, DH, QB, MODE>;
  if (lds > 65536) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  launch_kernel(kernel, dim3((unsigned)paged_grid(a)), dim3(64 * QB), (uint32_t)lds, s, a, a.table);
  return hipGetLastError();
}

template <int FMT>
hipError_t launch_paged_rows(int32_t head_dim, const PagedAttnArgs &a, hipStream_t s) {
  auto go = [&](auto dh) {
    return a.look == PAGED_TREE ? launch_paged_rows_mode<FMT, dh.value, PAGED_ROW_WAVES, PAGED_TREE>(a, s)
                                : launch_paged_rows_mode<FMT, dh.value, PAGED_ROW_WAVES, PAGED_WINDOW>(a, s);
  };
  switch (head_dim) {
    case 64: return go(std::integral_constant<int, 64>());
    case 80: return go(std::integral_constant<int, 80>());
    case 128: return go(std::integral_constant<int, 128>());
  }
  return hipErrorInvalidValue;
}

}  // namespace marche
