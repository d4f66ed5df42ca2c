// Appending rows to the paged cache: queries and keys turned by their positions,
// the turned queries written out, keys and values quantised into their slots.
//
// Pair i of a head's channels (x, y) at position p (on the pair's axis) becomes
//   (x cos t - y sin t, y cos t + x sin t),   t = p * freq_i.
// The angle is formed in turns and in 64 bits and reduced there to an eighth of a turn
// to either side, as float32 has no bits left for far positions (2^20 times any
// frequency is off by 0.06 radians); sine and cosine of what is left are float32
// polynomials.  Keys go from float32 to the cache's format by one rounding.
#include <algorithm>

#include "paged_device.h"

namespace marche {

// Sine and cosine of 2 pi pos turn: Taylor's sums on [-pi/4, pi/4], whose next terms are
// below 2e-9 (sine, x^11 / 11!) and 2e-10 (cosine, x^12 / 12!).
__device__ __forceinline__ void turn(int pos, double per, float &sn, float &cs) {
  double t = (double)pos * per;
  t -= rint(t);
  const double quarter = rint(4.0 * t);  // -2 .. 2
  const float x = (float)fma(-0.25, quarter, t) * 6.28318530717958648f;
  const float z = x * x;
  float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(z, s, 8.33333333e-3f);
  s = fmaf(z, s, -1.66666667e-1f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  c = fmaf(z, c, -1.38888889e-3f);
  c = fmaf(z, c, 4.16666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const int q = (int)quarter & 3;
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  sn = q & 2 ? -a : a;
  cs = (q + 1) & 2 ? -b : b;
}

// A lane holds four pairs of a head: eight channels, in two pieces of four (HALVES: the
// pairs' first and second channels, or, behind the turned ones, any eight; otherwise
// eight neighbours).  A group of lanes takes N heads of one row, queries' before
// keys' before values', so that the angles are formed once for them.
template <int FMT, int DH, typename InT, bool HALVES, int N>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedTurns turns, PagedAppendArgs a) {
  constexpr int PER = paged_write_pairs(DH), GROUP = 256 / PER;
  using Piece = std::conditional_t<sizeof(InT) == 4, u32x4, u32x2>;
  __shared__ int s_b0;
  const int tid = threadIdx.x, lane = tid & 63, c = tid % GROUP;
  const uint32_t u0 = blockIdx.x * PER, unit = u0 + tid / GROUP;  // below 2^31
  const int r = (int)a.d_slots.div(unit), slot = (int)(unit - (uint32_t)r * a.slots);
  const RowRange own(a.a_off, a.n_seqs, a.a_total);
  if (own.none()) return;
  const int rr = own.nearest(r);  // (what is loaded for others is not used)
  const bool on = r == rr && c < DH / 8;

  // the pieces' channels
  const int P = a.n_pairs, cc = c < DH / 8 ? c : 0;
  const bool split = HALVES && 4 * cc < P;
  const int first = split ? 4 * cc : 8 * cc, second = split ? P + 4 * cc : 8 * cc + 4;

  const int heads = a.q_heads + 2 * a.n_heads;
  Piece in[N][2];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = min(slot + i * a.slots, heads - 1);
    const int h = x < a.q_heads ? x : x < a.q_heads + a.n_heads ? x - a.q_heads : x - a.q_heads - a.n_heads;
    const void *base = x < a.q_heads ? a.q : x < a.q_heads + a.n_heads ? a.k_new : a.v_new;
    const InT *p = static_cast<const InT *>(base) + (size_t)rr * a.row_stride + (size_t)h * DH;
    in[i][0] = *reinterpret_cast<const Piece *>(p + first);
    in[i][1] = *reinterpret_cast<const Piece *>(p + second);
  }

  const int tok = a.a_idx[rr];
  float sn[4], cs[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int pair = min(4 * cc + e, 63);
    const int pos = a.pos ? a.pos[(size_t)turns.axis[pair] * a.a_total + rr] : tok;
    turn(pos, turns.turn[pair], sn[e], cs[e]);
  }

  int b;
  if (a.a_off) {
    if (tid < 64) {
      const int f = wave_find_seq(a.a_off, a.n_seqs, own.nearest((int)a.d_slots.div(u0)), lane);
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

#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = slot + i * a.slots;
    if (x >= heads) break;
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(InT) == 4) f[e] = __uint_as_float(in[i][e / 4][e % 4]);
      else f[e] = __uint_as_float(e % 2 ? in[i][e / 4][e % 4 / 2] & 0xFFFF0000u : in[i][e / 4][e % 4 / 2] << 16);
    }
    if (x < a.q_heads + a.n_heads) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (4 * cc + e >= P) break;
        const int u = HALVES ? e : 2 * e, v = HALVES ? 4 + e : 2 * e + 1;
        const float p = f[u], q = f[v];
        f[u] = fmaf(-q, sn[e], p * cs[e]);
        f[v] = fmaf(p, sn[e], q * cs[e]);
      }
    }
    auto bf = [&](int e) { return __builtin_bit_cast(uint32_t, bf16x2{(bf16)f[e], (bf16)f[e + 1]}); };
    auto raw = [&](int e) { return __float_as_uint(f[e]); };
    if (x < a.q_heads) {
      InT *o = static_cast<InT *>(a.q_out) + (size_t)rr * a.q_out_stride + (size_t)x * DH;
      if (!on) continue;
      if constexpr (sizeof(InT) == 4) {
        *reinterpret_cast<u32x4 *>(o + first) = u32x4{raw(0), raw(1), raw(2), raw(3)};
        *reinterpret_cast<u32x4 *>(o + second) = u32x4{raw(4), raw(5), raw(6), raw(7)};
      } else {
        *reinterpret_cast<u32x2 *>(o + first) = u32x2{bf(0), bf(2)};
        *reinterpret_cast<u32x2 *>(o + second) = u32x2{bf(4), bf(6)};
      }
      continue;
    }
    const bool is_v = x >= a.q_heads + a.n_heads;
    const int h = x - a.q_heads - (is_v ? a.n_heads : 0);
    const size_t at = (((size_t)max(page, 0) * a.n_heads + h) << a.page_log2) + (tok & ((1 << a.page_log2) - 1));
    const bool fits = (unsigned)page < (unsigned)a.n_pages;
    if constexpr (FMT == BF) {
      if (!fits) continue;
      bf16 *o = static_cast<bf16 *>(is_v ? a.v : a.k) + at * DH;
      *reinterpret_cast<u32x2 *>(o + first) = u32x2{bf(0), bf(2)};
      *reinterpret_cast<u32x2 *>(o + second) = u32x2{bf(4), bf(6)};
    } else {
      u32x4 y[2] = {{raw(0), raw(1), raw(2), raw(3)}, {raw(4), raw(5), raw(6), raw(7)}};
      const int code = exp_code<FMT>(__uint_as_float(group_max<GROUP>(on ? largest<float>(y) : 0u)));
      const u32x2 o = pack8<FMT, float>(y, code);
      if (!fits) continue;
      char *to = static_cast<char *>(is_v ? a.v : a.k) + at * DH;
      *reinterpret_cast<uint32_t *>(to + first) = o.x;
      *reinterpret_cast<uint32_t *>(to + second) = o.y;
      if (c == 0) (is_v ? a.v_exp : a.k_exp)[at] = (uint8_t)code;
    }
  }
}

int paged_append_heads(int32_t head_dim, int64_t rows, int32_t heads) {
  return rows * heads >= 4096 ? 4 : 1;
}

hipError_t launch_paged_append(DType dt, int32_t format, int32_t head_dim, bool halves, const PagedTurns &turns,
                               PagedAppendArgs a, hipStream_t s) {
  const int heads = a.q_heads + 2 * a.n_heads, n = paged_append_heads(head_dim, a.a_total, heads);
  a.slots = (heads + n - 1) / n;
  a.d_slots = FastDiv::of(a.slots);
  a.d_rows = FastDiv::of(std::max(1, a.rows_each));
  const int per = paged_write_pairs(head_dim);
  const unsigned grid = (unsigned)(((int64_t)a.a_total * a.slots + per - 1) / per);
  return by_shape(format, head_dim, [&](auto fmt, auto dh) {
    auto go = [&](auto half, auto several) {
      constexpr bool H = half.value;
      constexpr int N = several.value ? 4 : 1;
      if (dt == DType::BF16) launch_kernel(paged_append_kernel<fmt.value, dh.value, bf16, H, N>, grid, 256, 0, s, turns, a);
      else launch_kernel(paged_append_kernel<fmt.value, dh.value, float, H, N>, grid, 256, 0, s, turns, a);
    };
    auto by_n = [&](auto half) {
      if (n > 1) go(half, std::true_type());
      else go(half, std::false_type());
    };
    if (halves) by_n(std::true_type());
    else by_n(std::false_type());
  });
}

}  // namespace marche
