// Device-side helpers of the paged cache's kernels.
#pragma once

#include "device_common.h"

namespace marche {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int BF = 0, E4 = 1, I8 = 2;  // marche_cache_format_t

// ------------------------------------------------------------------ exponents

// Exponent code (e + 127) of a row with largest magnitude amax: the least
// e >= -111 with amax <= M 2^e, M = 448 (e4m3) or 127 (int8).  amax =
// f 2^x with f in [1, 2): e = x - 8 if f <= 1.75 and x - 7 beyond (448 = 1.75
// 2^8); e = x - 6 if f <= 1.984375 and x - 5 beyond (127 = 1.984375 2^6).  The floor
// keeps the smallest e4m3 value (2^-9) times 2^e a normal bf16.  255: not finite.
template <int FMT>
__device__ __forceinline__ int exp_code(float amax) {
  constexpr uint32_t top = FMT == E4 ? 0x600000u : 0x7E0000u;
  const uint32_t u = __float_as_uint(amax);
  const int x = (int)(u >> 23);  // biased
  if (x == 255) return 255;
  const int e = x - (FMT == E4 ? 8 : 6) + ((u & 0x7FFFFFu) > top ? 1 : 0);
  return max(e, 16);
}
// 2^(code - 127); the code 255 gives infinity.
__device__ __forceinline__ float exp_scale(uint32_t code) { return __uint_as_float(code << 23); }
// The code of the largest finite rows, and, as float bits, the largest magnitude
// in them: what would be rounded to 2^128 becomes the number before it, 240 2^120
// or 63 2^122 (off by up to a step, not half a one), so that finite rows read back
// finite.
template <int FMT>
constexpr int TOP_CODE = FMT == E4 ? 247 : 249;
template <int FMT>
constexpr uint32_t TOP_BITS = FMT == E4 ? 0x7F700000u : 0x7F7C0000u;
// Of an int8 row with this code: the magnitude that its values are held to.
__device__ __forceinline__ float int8_top(int code) {
  return code == TOP_CODE<I8> ? __uint_as_float(TOP_BITS<I8>) : INFINITY;
}
// 2^(127 - code), exact for every code a finite row has (16 .. 249).
__device__ __forceinline__ float exp_inv(int code) { return __uint_as_float((uint32_t)(254 - code) << 23); }

// Four values of a dword of the format.
template <int FMT>
__device__ __forceinline__ void unpack4(uint32_t w, float scale, float *o) {
  if constexpr (FMT == E4) {
    // (times a power of two after the conversion is exact, and keeps the code 255
    // a NaN)
    o[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale;
    o[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale;
    o[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * scale;
    o[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * scale;
  } else {
    o[0] = (float)(int8_t)(w) * scale;
    o[1] = (float)(int8_t)(w >> 8) * scale;
    o[2] = (float)(int8_t)(w >> 16) * scale;
    o[3] = (float)(int8_t)(w >> 24) * scale;
  }
}

// ------------------------------------------------------------------ sequences

// Tokens of a sequence that its page table can hold.
__device__ __forceinline__ int paged_len(int len, int max_pages, int page_log2) {
  const int64_t cap = (int64_t)max_pages << page_log2;
  return max(0, (int)(len < cap ? len : cap));
}

// The rows that belong to any sequence: [lo, hi) of [0, total).  What lies
// outside may not even be there.
struct RowRange {
  int lo, hi;
  __device__ __forceinline__ RowRange(const int32_t *off, int n_seqs, int total) : lo(0), hi(total) {
    if (off) lo = max(off[0], 0), hi = min(off[n_seqs], total);
  }
  __device__ __forceinline__ bool none() const { return hi <= lo; }
  __device__ __forceinline__ int nearest(int r) const { return min(max(r, lo), hi - 1); }
};

// Eight consecutive values of a row.
__device__ __forceinline__ void load8(const float *p, float *o) {
  const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = a[i], o[4 + i] = b[i];
}
__device__ __forceinline__ void load8(const bf16 *p, float *o) {
  const bf16x8 a = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = (float)a[i];
}

__device__ __forceinline__ void load4(const float *p, float *o) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = a[i];
}
__device__ __forceinline__ void load4(const bf16 *p, float *o) {
  const bf16x4 a = *reinterpret_cast<const bf16x4 *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = (float)a[i];
}

// Sequence of row r: the b with off[b] <= r < off[b+1] (the last b with
// off[b] <= r), or n_seqs for a row behind the last one.  One wavefront per
// call, r uniform: each round 64 probes cut the range 64-fold.
__device__ __forceinline__ int wave_find_seq(const int32_t *off, int n_seqs, int r, int lane) {
  int lo = 0, n = n_seqs;  // among the ends off[lo + 1 .. lo + n], how many are <= r
  while (n > 0) {
    const int step = (n + 63) / 64;
    const int at = min((lane + 1) * step, n);
    const bool le = off[lo + at] <= r;
    const int full = __popcll(__ballot(le));
    if (full == 64) return lo + n;
    lo += min(full * step, n);
    n = min(step - 1, n_seqs - lo);
  }
  return lo;
}

// ------------------------------------------------------------------ shares of long caches

// Sequences of different lengths are cut into ranges of one length, `chunk`
// 32-key tiles, so that `budget` ranges or fewer cover all of them: with total
// the sum of the sequences' tiles, ceil(total / (budget - n_seqs)) is enough, as each
// sequence adds less than one range to total / chunk.  At most 64 ranges a
// sequence.  One wavefront per call; n_seqs <= PAGED_MAX_SHARED.
struct Shares {
  int chunk;
  int tiles[PAGED_MAX_SHARED / 64];  // of sequence 64 k + lane
  __device__ __forceinline__ Shares(const PagedAttnArgs &a, int lane) {
    int sum = 0, most = 0;
#pragma unroll
    for (int k = 0; k < PAGED_MAX_SHARED / 64; ++k) {
      const int b = 64 * k + lane;
      const int len = b < a.n_seqs ? min(paged_len(a.lens[b], a.max_pages, a.page_log2), a.len_max) : 0;
      tiles[k] = (len + 31) >> 5;
      sum += tiles[k];
      most = max(most, tiles[k]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      sum += __shfl_xor(sum, o, 64);
      most = max(most, __shfl_xor(most, o, 64));
    }
    const int room = a.budget - a.n_seqs;
    chunk = max(max((sum + room - 1) / room, (most + 63) >> 6), a.chunk);
    chunk = __builtin_amdgcn_readfirstlane(chunk);
  }
  __device__ __forceinline__ int ranges(int n) const { return (int)((uint32_t)(n + chunk - 1) / (uint32_t)chunk); }
  // Range x of all: its sequence (-1: there are fewer) and place in it.
  __device__ __forceinline__ int find(int x, int lane, int &part) const {
    int before = 0;
#pragma unroll
    for (int k = 0; k < PAGED_MAX_SHARED / 64; ++k) {
      const int n = ranges(tiles[k]);
      int end = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(end, o, 64);
        if (lane >= o) end += y;
      }
      end += before;
      const unsigned long long past = __ballot(end > x);
      if (past) {
        const int l = __ffsll((long long)past) - 1;
        part = __builtin_amdgcn_readfirstlane(x - __shfl(end - n, l, 64));
        return 64 * k + l;
      }
      before = __shfl(end, 63, 64);
    }
    return -1;
  }
};

}  // namespace marche
