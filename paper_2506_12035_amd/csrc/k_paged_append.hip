// Appending rows to the paged cache: queries and keys turned by their positions,
// the turned queries written out, keys and values quantised into their slots.
//
// Pair i of a head's channels (x, y) at position p (on the pair's axis) becomes
//   (x cos t - y sin t, y cos t + x sin t),   t = p * freq_i.
// The angle is formed in turns and in 64 bits and reduced there to an eighth of a turn
// to either side, as float32 has no bits left for far positions (at 2^20 a frequency
// near 1 gives angles off by up to 0.06 radians); sine and cosine of what is left are
// polynomials in 64 bits, rounded once (12.0 us for 1826 fp32 rows of 48 heads of 80, 11.7 with sums in
// float32, which were off by up to 1.8 times what the products may be).  Keys go from float32 to
// the cache's format by one rounding.
//
// Bound by bytes: 40960 rows of 12 heads of 64, three axes, bf16 to int8, 316 MB: 76.9 us,
// 4.1 TB/s (93.6 with queries, keys and values of a row side by side in a wavefront, which
// then ran each other's instructions).  One row of 48 heads: 3.0 us, latency.
#include <algorithm>

#include "paged_device.h"

namespace marche {

// Sine and cosine of 2 pi pos turn, the nearest float32 numbers: Taylor's sums on [-pi/4, pi/4] in
// 64 bits, whose next terms are below 1e-11 (sine, x^13 / 13!) and 2e-10 (cosine, x^12 / 12!).
__device__ __forceinline__ void turn(int pos, double per, float &sn, float &cs) {
  double t = (double)pos * per;
  t -= rint(t);
  const double quarter = rint(4.0 * t);  // -2 .. 2
  const double x = fma(-0.25, quarter, t) * 6.283185307179586477;
  const double z = x * x;
  double s = fma(z, -1.0 / 39916800, 1.0 / 362880);
  s = fma(z, s, -1.0 / 5040);
  s = fma(z, s, 1.0 / 120);
  s = fma(z, s, -1.0 / 6);
  s = fma(x * z, s, x);
  double c = fma(z, -1.0 / 3628800, 1.0 / 40320);
  c = fma(z, c, -1.0 / 720);
  c = fma(z, c, 1.0 / 24);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const int q = (int)quarter & 3;
  const float a = (float)(q & 1 ? c : s), b = (float)(q & 1 ? s : c);
  sn = q & 2 ? -a : a;
  cs = (q + 1) & 2 ? -b : b;
}

// Workgroups of the queries come first, then the keys', then the values', so that a
// wavefront does one thing.  A lane holds eight channels of a head in two pieces of four: of
// queries and keys four pairs (HALVES: their first and their second channels, or, behind the
// turned ones, any eight; otherwise eight neighbours), of values neighbours.  A group of
// lanes takes N heads of one row, so that angles, row and page are found once for them.
// STREAM: rows past the caches, for calls whose rows do not fit them anyway.
template <int FMT, int DH, typename InT, bool HALVES, int N, bool STREAM>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedTurns turns, PagedAppendArgs a) {
  constexpr int PER = paged_write_pairs(DH), GROUP = 256 / PER;
  using Piece = std::conditional_t<sizeof(InT) == 4, u32x4, u32x2>;
  __shared__ int s_b0;
  const int tid = threadIdx.x, lane = tid & 63, c = tid % GROUP;
  const RowRange own(a.a_off, a.n_seqs, a.a_total);
  if (own.none()) return;

  auto run = [&](auto kind, uint32_t block) {
    constexpr int KIND = kind.value;  // 0 queries, 1 keys, 2 values
    const int heads = KIND == 0 ? a.q_heads : a.n_heads, slots = KIND == 0 ? a.q_slots : a.kv_slots;
    const FastDiv d_slots = KIND == 0 ? a.d_q_slots : a.d_kv_slots;
    const uint32_t u0 = block * PER, unit = u0 + tid / GROUP;  // below 2^31
    const int r = (int)d_slots.div(unit), h0 = (int)(unit - (uint32_t)r * slots) * N;
    const int rr = own.nearest(r);  // (what is loaded for others is not used)
    const int cc = c < DH / 8 ? c : 0;
    const bool on = r == rr && c < DH / 8;

    const int P = a.n_pairs;
    const bool split = KIND < 2 && HALVES && 4 * cc < P;
    const int first = split ? 4 * cc : 8 * cc, second = split ? P + 4 * cc : 8 * cc + 4;
    const InT *from = static_cast<const InT *>(KIND == 0 ? a.q : KIND == 1 ? a.k_new : a.v_new) + (size_t)rr * a.row_stride;
    Piece in[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const InT *p = from + (size_t)min(h0 + i, heads - 1) * DH;
      const Piece *x = reinterpret_cast<const Piece *>(p + first), *y = reinterpret_cast<const Piece *>(p + second);
      in[i][0] = STREAM ? __builtin_nontemporal_load(x) : *x;
      in[i][1] = STREAM ? __builtin_nontemporal_load(y) : *y;
    }

    const int tok = a.a_idx[rr];
    float sn[4], cs[4];
    if constexpr (KIND < 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pair = min(4 * cc + e, 63);
        const int pos = a.pos ? a.pos[(size_t)turns.axis[pair] * a.a_total + rr] : tok;
        turn(pos, turns.turn[pair], sn[e], cs[e]);
      }
    }
    size_t at = 0;
    bool fits = on;
    if constexpr (KIND > 0) {
      int b;
      if (a.a_off) {
        if (tid < 64) {
          const int f = wave_find_seq(a.a_off, a.n_seqs, own.nearest((int)d_slots.div(u0)), lane);
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
      fits = (unsigned)page < (unsigned)a.n_pages;
      at = (((size_t)max(page, 0) * a.n_heads + h0) << a.page_log2) + (tok & ((1 << a.page_log2) - 1));
    }

#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (h0 + i >= heads) break;
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (sizeof(InT) == 4) f[e] = __uint_as_float(in[i][e / 4][e % 4]);
        else f[e] = __uint_as_float(e % 2 ? in[i][e / 4][e % 4 / 2] & 0xFFFF0000u : in[i][e / 4][e % 4 / 2] << 16);
      }
      if constexpr (KIND < 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int u = HALVES ? e : 2 * e, v = HALVES ? 4 + e : 2 * e + 1;
          const float x = fmaf(-f[v], sn[e], f[u] * cs[e]), y = fmaf(f[u], sn[e], f[v] * cs[e]);
          const bool turned = HALVES ? 4 * cc < P : 4 * cc + e < P;
          f[u] = turned ? x : f[u];
          f[v] = turned ? y : f[v];
        }
      }
      auto bf = [&](int e) { return __builtin_bit_cast(uint32_t, bf16x2{(bf16)f[e], (bf16)f[e + 1]}); };
      auto raw = [&](int e) { return __float_as_uint(f[e]); };
      auto put = [&](auto *to, auto x, auto y) {
        using V = decltype(x);
        if (STREAM && KIND == 0) {
          __builtin_nontemporal_store(x, reinterpret_cast<V *>(to + first));
          __builtin_nontemporal_store(y, reinterpret_cast<V *>(to + second));
        } else {
          *reinterpret_cast<V *>(to + first) = x;
          *reinterpret_cast<V *>(to + second) = y;
        }
      };
      if constexpr (KIND == 0) {
        InT *o = static_cast<InT *>(a.q_out) + (size_t)rr * a.q_out_stride + (size_t)(h0 + i) * DH;
        if (!fits) continue;
        if constexpr (sizeof(InT) == 4) put(o, u32x4{raw(0), raw(1), raw(2), raw(3)}, u32x4{raw(4), raw(5), raw(6), raw(7)});
        else put(o, u32x2{bf(0), bf(2)}, u32x2{bf(4), bf(6)});
      } else if constexpr (FMT == BF) {
        if (!fits) continue;
        put(static_cast<bf16 *>(KIND == 2 ? a.v : a.k) + (at + ((size_t)i << a.page_log2)) * DH, u32x2{bf(0), bf(2)}, u32x2{bf(4), bf(6)});
      } else {
        u32x4 y[2] = {{raw(0), raw(1), raw(2), raw(3)}, {raw(4), raw(5), raw(6), raw(7)}};
        const int code = exp_code<FMT>(__uint_as_float(group_max<GROUP>(on ? largest<float>(y) : 0u)));
        const u32x2 o = pack8<FMT, float>(y, code);
        if (!fits) continue;
        const size_t x = at + ((size_t)i << a.page_log2);
        put(static_cast<uint8_t *>(KIND == 2 ? a.v : a.k) + x * DH, o.x, o.y);
        if (c == 0) (KIND == 2 ? a.v_exp : a.k_exp)[x] = (uint8_t)code;
      }
    }
  };
  const uint32_t id = blockIdx.x;
  if (id < a.q_blocks) run(std::integral_constant<int, 0>(), id);
  else if (id < a.q_blocks + a.kv_blocks) run(std::integral_constant<int, 1>(), id - a.q_blocks);
  else run(std::integral_constant<int, 2>(), id - a.q_blocks - a.kv_blocks);
}

// Four heads a lane group share the angles where that leaves 1024 wavefronts or more of 64
// channels (2048 of 80 and 128); below, a head each is the shorter way.
PagedAppendPlan paged_append_plan(DType dt, int32_t head_dim, int32_t a_total, int32_t q_heads, int32_t n_heads) {
  const int64_t pairs = (int64_t)a_total * (q_heads + 2 * n_heads);
  return PagedAppendPlan{pairs >= 32768 && n_heads >= 4 ? 4 : 1, (double)pairs * head_dim * (dt == DType::BF16 ? 2 : 4) >= 64e6};
}

hipError_t launch_paged_append(DType dt, int32_t format, int32_t head_dim, bool halves, const PagedTurns &turns,
                               PagedAppendArgs a, hipStream_t s) {
  const PagedAppendPlan plan = paged_append_plan(dt, head_dim, a.a_total, a.q_heads, a.n_heads);
  const int n = plan.heads;
  const bool stream = plan.stream;
  const int per = paged_write_pairs(head_dim);
  a.q_slots = std::max(1, (a.q_heads + n - 1) / n);
  a.kv_slots = (a.n_heads + n - 1) / n;
  a.d_q_slots = FastDiv::of(a.q_slots);
  a.d_kv_slots = FastDiv::of(a.kv_slots);
  a.d_rows = FastDiv::of(std::max(1, a.rows_each));
  a.q_blocks = a.q_heads ? (uint32_t)(((int64_t)a.a_total * a.q_slots + per - 1) / per) : 0;
  a.kv_blocks = (uint32_t)(((int64_t)a.a_total * a.kv_slots + per - 1) / per);
  const unsigned grid = a.q_blocks + 2 * a.kv_blocks;
  return by_shape(format, head_dim, [&](auto fmt, auto dh) {
    auto go = [&](auto half, auto several, auto st) {
      constexpr bool H = half.value, S = st.value;
      constexpr int N = several.value ? 4 : 1;
      if (dt == DType::BF16) launch_kernel(paged_append_kernel<fmt.value, dh.value, bf16, H, N, S>, grid, 256, 0, s, turns, a);
      else launch_kernel(paged_append_kernel<fmt.value, dh.value, float, H, N, S>, grid, 256, 0, s, turns, a);
    };
    auto by_n = [&](auto half) {
      if (n > 1 && stream) go(half, std::true_type(), std::true_type());
      else if (n > 1) go(half, std::true_type(), std::false_type());
      else go(half, std::false_type(), std::false_type());
    };
    if (halves) by_n(std::true_type());
    else by_n(std::false_type());
  });
}

}  // namespace marche
