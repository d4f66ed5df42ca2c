// Internal declarations shared by the host API and the HIP kernels of
// libmarche.so.  Not part of the public ABI (include/marche.h is).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace marche {

typedef __bf16 bf16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Where active row r of the packed activations lives: image b, token tok,
// and its row in the [batch][n_tokens][d_model] residual stream.
struct RowMap {
  int32_t x_row;  // b * n_tokens + tok
  int32_t b;
  int32_t tok;
  int32_t pad;
};

// Kernel timing of the library's profiling mode (marche_profile_*): while a
// timed call runs on a thread, the first kernel it launches through
// launch_kernel() (device_common.h) carries the call's two events on its
// dispatch (hipExtLaunchKernel), so they hold the kernel's own start and end,
// not the stream's dispatch gap before it.
struct KernelEvents {
  hipEvent_t start = nullptr, stop = nullptr;
  bool used = false;
};
// This thread's slot: the timed call in progress, or nullptr.
KernelEvents *&kernel_events();

// Element type of the packed activations, weights and KV cache.
enum class DType { F32 = 0, BF16 = 1 };

// ---- elementwise / indexing (k_elementwise.hip) ----
hipError_t launch_row_map(RowMap *map, const int32_t *a_idx, const int32_t *a_off, int32_t batch,
                          int32_t n_tokens, hipStream_t s);
hipError_t launch_gather_ln(DType dt, void *out, const float *x, const RowMap *map, const float *g,
                            const float *b, int32_t rows, int32_t d_model, float eps, hipStream_t s);
hipError_t launch_decoder_input(float *x, const float *cls, const float *value, const float *mask,
                                const float *pos, const int32_t *rank, int32_t batch,
                                int32_t n_tokens, int32_t n_buf, int32_t d_model, int32_t n_known,
                                hipStream_t s);
hipError_t launch_fill_zero(void *dst, size_t bytes, hipStream_t s);
// Debug-mode check of a step's active lists; report[0] = 0 or 1 + code*batch + image
// (codes: 0 offsets, 1 token range, 2 duplicate token, 3 n_gen).
hipError_t launch_check_active(const int32_t *a_idx, const int32_t *a_off, const int32_t *n_gen,
                               int32_t batch, int32_t n_tokens, int32_t a_total, int32_t a_max,
                               int32_t gen_max, int32_t *report, hipStream_t s);

// ---- the rest of a MAR step (k_mar.hip) ----
// Encoder input rows [batch][n_buf + n_known][d_model] (Eq. 1).
hipError_t launch_encoder_input(float *x, const float *cls, const float *tok, const float *w_z,
                                const float *b_z, const float *pe, const int32_t *known,
                                int32_t batch, int32_t n_buf, int32_t n_img, int32_t n_known,
                                int32_t d_model, int32_t c_tok, hipStream_t s);
// Masked rows of the decoder input (Eq. 2).
hipError_t launch_mask_fill(float *x, const float *mask, const float *pe, const int32_t *rank,
                           int32_t batch, int32_t n_tokens, int32_t n_buf, int32_t n_known,
                           int32_t d_model, hipStream_t s);
// out[r] = LN(x[rows ? rows[r] : r]) * g + b (+ add[src % n_tokens - n_buf]).
hipError_t launch_ln_rows(DType dt, void *out, const float *x, const int32_t *rows_idx,
                          const float *g, const float *b, const float *add, int32_t rows,
                          int32_t n_tokens, int32_t n_buf, int32_t d_model, float eps,
                          hipStream_t s);
// Sinusoidal time embedding table [n_steps][freq].
hipError_t launch_time_sinus(DType dt, void *out, int32_t n_steps, int32_t freq, hipStream_t s);
// sc = SiLU(cond + temb_row), [rows][width].
hipError_t launch_silu_cond(DType dt, void *sc, const float *cond, const float *temb, int32_t rows,
                            int32_t width, hipStream_t s);
// w_t = w^T for a [rows][cols] float32 matrix.
hipError_t launch_transpose_f32(float *w_t, const float *w, int32_t rows, int32_t cols,
                                hipStream_t s);
// a = LN(h) (1 + scale) + shift (slices of mod at the offsets).
hipError_t launch_head_mod(DType dt, void *a, const float *h, const void *mod, int32_t mod_ld,
                           int32_t shift_off, int32_t scale_off, int32_t rows, int32_t width,
                           float eps, hipStream_t s);
// Coefficients of one DDPM step (see head_step_kernel).
struct HeadStep {
  float sra, srm1, c1, c2, sigma;
};
// Everything between two sampling steps' blocks, row by row (see
// head_step_kernel).  `out`: this step's output projection and DDPM update
// (final modulation at shift_off, scale_off); `in`: the next step's input
// projection and first modulated norm (slices 0 and width of mod; a == NULL:
// without the norm, which the next launch forms itself); sc != NULL:
// SiLU(cond + temb) into it.
struct HeadRows {
  bool out, in;
  float *h;
  void *a;
  const void *mod;
  int32_t mod_ld, shift_off, scale_off;
  const float *w_out, *b_out;    // [C][W], [C]
  const float *w_in, *w_in_t;    // [W][C] and its transpose
  const float *b_in;             // [W]
  const float *x_cur, *noise;    // [rows][C]
  float *x_next, *tok_out;       // tok_out: last step only
  const int32_t *out_rows;
  HeadStep st;
  void *sc;
  const float *cond, *temb;      // [rows][W], [W]
  int32_t rows, c_tok;
  float eps;
};
hipError_t launch_head_step(DType dt, const HeadRows &p, int32_t width, hipStream_t s);

// ---- GEMMs with fused epilogues (k_gemm.hip) ----
// C[M][N] = A[M][K] . W[N][K]^T (+ bias) followed by one epilogue:
//   qkv:   columns [0,D) -> q [M][D]; [D,2D) -> K cache, [2D,3D) -> V cache
//          (scattered to [b][h][tok][d] of one layer's cache)
//   resid: x[map[r].x_row][c] += C + bias        (float32 residual stream)
//   gelu:  h[r][c] = GELU(C + bias)
struct QkvOut {
  void *q;
  void *k_cache;  // layer base
  void *v_cache;  // layer base
  int32_t d_model, head_dim, n_heads, n_tokens;
};
// `shared`: the call computes a part of its cache's images, so that others may
// run beside it (see gemm_tile_kind).
hipError_t launch_gemm_qkv(DType dt, const void *a, const void *w, const float *bias, int32_t m,
                           int32_t n, int32_t k, const RowMap *map, QkvOut out, bool shared,
                           hipStream_t s);
// tag: 0 = output projection, 1 = fc2 (separate kernel symbols)
hipError_t launch_gemm_resid(DType dt, const void *a, const void *w, const float *bias, int32_t m,
                             int32_t n, int32_t k, const RowMap *map, float *x, int32_t tag,
                             bool shared, hipStream_t s);
hipError_t launch_gemm_gelu(DType dt, const void *a, const void *w, const float *bias, int32_t m,
                            int32_t n, int32_t k, void *h, bool shared, hipStream_t s);
// Sampler GEMMs: out[r][c] = act(C + bias) as out_dt (row-major, row stride
// ld), act SiLU or the identity; a float32 GEMM writes float32 only.
hipError_t launch_gemm_plain(DType dt, const void *a, const void *w, const float *bias, int32_t m,
                             int32_t n, int32_t k, void *out, DType out_dt, bool silu_act,
                             int32_t ld, hipStream_t s);
// The two products of a sampler block (width x width): y = SiLU(a w^T + bias),
// and h += gate (a w^T + bias) with the gate a slice of the modulations.  Side
// products out = a w^T + bias (bf16, same rows and reduction length as the
// main one, n columns a multiple of 128, ld = HeadSides::ld) share the launch:
// a block product of a few hundred rows leaves most compute units idle.
struct HeadSide {
  const void *a, *w;
  const float *bias;
  void *out;
  int32_t n;
};
struct HeadSides {
  HeadSide s[2];
  int32_t ld;
};
// 128-column side tiles per launch that fit beside the main product in one
// wave of workgroups (0: none, or no side products for this type).
int head_side_tiles(DType dt, int32_t m, int32_t width);
hipError_t launch_head_gemm_silu(DType dt, const void *a, const void *w, const float *bias,
                                 int32_t m, int32_t width, void *y, const HeadSides &sides,
                                 hipStream_t s);
// The first with its activations a = LN(h) (1 + scale) + shift formed in the
// same launch (bf16, where head_norm_fits: up to 16 rows, by width).
bool head_norm_fits(DType dt, int32_t m, int32_t width);
hipError_t launch_head_gemm_norm_silu(const float *h, const void *mod, int32_t mod_ld,
                                      int32_t shift_off, int32_t scale_off, float eps,
                                      const void *w, const float *bias, int32_t m, int32_t width,
                                      void *y, const HeadSides &sides, hipStream_t s);
hipError_t launch_head_gemm_gate(DType dt, const void *a, const void *w, const float *bias,
                                 int32_t m, int32_t width, float *h, const void *gate,
                                 int32_t mod_ld, const HeadSides &sides, hipStream_t s);
// Decoder embedding of the encoder rows scattered to their sequence positions
// (n = d_model): x[b][j][c] = C + bias + pe[j][c], j the position encoder row
// r = b * n_enc + i holds (i < n_buf: i; else n_buf + known[b][i - n_buf]).
hipError_t launch_gemm_embed(DType dt, const void *a, const void *w, const float *bias, int32_t m,
                             int32_t n, int32_t k, float *x, const float *pe, const int32_t *known,
                             int32_t n_enc, int32_t n_buf, int32_t n_known, int32_t n_tokens,
                             hipStream_t s);
// bf16 GEMM workgroup tile of an M x N x K product (rows x columns).
enum GemmTile {
  GEMM_TILE_256 = 0, GEMM_TILE_320, GEMM_TILE_64x128, GEMM_TILE_128, GEMM_TILE_192x128,
  GEMM_TILE_256x128, GEMM_TILE_64x64, GEMM_TILE_32x64, GEMM_TILE_32x32, GEMM_TILE_COUNT
};
int gemm_tile_kind(DType dt, int32_t m, int32_t n, int32_t k, bool shared = false);
// The tile of a sampler block's bf16 product (width x width) with side products
// of n_side columns.
int head_tile_kind(int32_t m, int32_t width, int32_t n_side);
// Whether a sampler launch of m rows and n columns (side products among them)
// over K = k runs the few-row kernel instead.
bool gemm_few_rows(DType dt, int32_t m, int32_t n, int32_t k);
// Compute units of the current device (queried once per device, then cached).
int device_cu_count();

// ---- attention (k_attn.hip) ----
struct AttnArgs {
  const void *q;        // [a_total][D] packed queries
  const void *k_cache;  // layer base [B][H][N][dh] (keys 0..N-1; the first segment)
  const void *v_cache;
  void *o;              // [a_total][D]
  const int32_t *a_off; // CSR rows per image; NULL: image b owns rows [b*a_max, (b+1)*a_max)
  const RowMap *map;
  int32_t batch, n_heads, n_tokens, head_dim, d_model, a_total, a_max;
  // Optional second key/value segment [B][H][n2][dh], attended after the
  // first in the same online-softmax pass (bf16 attention only).
  const void *k2 = nullptr;
  const void *v2 = nullptr;
  int32_t n2 = 0;
  // Optional attention mass of the generating rows (the first n_gen[b] rows
  // of image b), scores[b][h][j], written by the same kernel where
  // attn_fuses_scores() holds (one key segment).
  const int32_t *n_gen = nullptr;
  float *scores = nullptr;
  int32_t gen_max = 0;  // largest n_gen[b]
  // Optional row statistics [a_total][n_heads][2] (maximum logit, 1 / sum) for
  // launch_attn_scores, written by the kernels that run where
  // attn_fuses_scores() does not hold (and by every fp32 one).
  float *stats = nullptr;
};
hipError_t launch_attention(DType dt, const AttnArgs &a, hipStream_t s);
// Whether these bf16 arguments run the resident-K/V kernel (one workgroup per
// (image, head)).
bool attn_resident(const AttnArgs &a);
// Whether bf16 attention with these sizes runs the register-staged streaming
// kernel (head width 64, one key segment of whole tiles).
bool attn_streams(int32_t head_dim, int32_t n_tokens, bool two_segments);
// Wavefronts of 32 queries per workgroup of the streaming kernel that these
// bf16 arguments run (where the resident one does not).
int attn_query_blocks(const AttnArgs &a);
// Whether bf16 attention with these sizes can write the score pass itself:
// the resident kernel (every key of a head in LDS), or the streaming kernel
// when the generating rows fit its first query chunk.
bool attn_fuses_scores(int32_t a_max, int32_t n_tokens, int32_t head_dim, int32_t gen_max);
// dst[b][h] = [a[b][h] (na rows) ; c[b][h] (nc rows)], rows of dh elements, for
// K and V: the concatenation of the active and cached segments.
hipError_t launch_concat_kv(DType dt, void *k_dst, void *v_dst, const void *k_a, const void *v_a,
                            const void *k_c, const void *v_c, int32_t bh, int32_t na, int32_t nc,
                            int32_t head_dim, hipStream_t s);
// scores[b][h][j] = sum over the first n_gen[b] active rows i of P_h[i][j]
hipError_t launch_attn_scores(DType dt, const AttnArgs &a, const int32_t *n_gen, float *scores,
                              hipStream_t s);

// ---- selection (k_select.hip) ----
// lowest = false: highest scores first; true: lowest scores first.
hipError_t launch_select_topk(const float *scores, int32_t n_parts, const int32_t *excl_idx,
                              const int32_t *excl_off, int32_t batch, int32_t n_tokens, int32_t k,
                              int32_t *out_idx, const int32_t *out_off, bool lowest,
                              hipStream_t s);

// ---- paged cache (k_paged.hip, k_paged_attn_*.hip) ----
// Pointers are one layer's; formats are marche_cache_format_t; a page holds
// 1 << page_log2 tokens.  *_off NULL: every sequence has rows_each rows.
// Division of numbers below 2^31 by a constant known at launch: with s the
// bits of d - 1 and m = ceil(2^(32 + s) / d) - 2^32 < 2^32,
// n / d = (n m / 2^32 + n) / 2^s.
struct FastDiv {
  uint32_t m, s;
  static FastDiv of(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {(uint32_t)(((1ull << (32 + s)) + d - 1) / d - (1ull << 32)), s};
  }
  __host__ __device__ uint32_t div(uint32_t n) const {
    return (uint32_t)(((((uint64_t)n * m) >> 32) + n) >> s);
  }
};
struct PagedWriteArgs {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  const int32_t *table, *a_idx, *a_off;
  const void *k_new, *v_new;
  int64_t row_stride;
  int32_t n_pages, n_heads, page_log2, max_pages, n_seqs, a_total, rows_each;
  FastDiv d_heads, d_rows;  // set by the launch
};
// (row, head) pairs of a workgroup of 256 threads
constexpr int paged_write_pairs(int32_t head_dim) { return head_dim == 64 ? 32 : 16; }
hipError_t launch_paged_write(DType dt, int32_t format, int32_t head_dim, PagedWriteArgs a,
                              hipStream_t s);
// The rotation of an append: of pair i the turns (2 pi) per position, and its axis.
struct PagedTurns {
  double turn[64];
  uint8_t axis[64];
};
struct PagedAppendArgs {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  const int32_t *table, *a_idx, *a_off, *pos;  // pos NULL: a_idx on every axis
  const void *q, *k_new, *v_new;
  void *q_out;
  int64_t row_stride, q_out_stride;
  int32_t n_pages, n_heads, q_heads, page_log2, max_pages, n_seqs, a_total, rows_each, n_pairs;
  // set by the launch: lane groups per row and workgroups of the queries, and of the keys
  int32_t q_slots, kv_slots;
  uint32_t q_blocks, kv_blocks;
  FastDiv d_q_slots, d_kv_slots, d_rows;
};
// Heads of a row that a lane group takes, and whether rows go past the caches.
struct PagedAppendPlan {
  int heads;
  bool stream;
};
PagedAppendPlan paged_append_plan(DType dt, int32_t head_dim, int32_t a_total, int32_t q_heads, int32_t n_heads);
hipError_t launch_paged_append(DType dt, int32_t format, int32_t head_dim, bool halves, const PagedTurns &turns,
                               PagedAppendArgs a, hipStream_t s);
constexpr int PAGED_READ_TOKENS = 128;  // tokens per workgroup of the read kernel
struct PagedReadArgs {
  const void *k, *v;
  const uint8_t *k_exp, *v_exp;
  const int32_t *table, *lens;
  void *k_out, *v_out;
  int32_t n_pages, n_heads, page_log2, max_pages, n_seqs, n_tokens, blocks;
};
hipError_t launch_paged_read(DType dt, int32_t format, int32_t head_dim, PagedReadArgs a,
                             hipStream_t s);
struct PagedBoundsArgs {
  const void *k;
  const uint8_t *k_exp;
  int8_t *bounds;
  uint8_t *bounds_exp;
  const int32_t *table, *lens, *first;
  int32_t n_pages, n_heads, page_log2, max_pages, n_seqs, span;
  FastDiv d_heads, d_span;  // set by the launch
};
constexpr int PAGED_BOUNDS_PAIRS = 4;  // (page, head) pairs of a workgroup of 256 threads
hipError_t launch_paged_bounds(int32_t format, int32_t head_dim, PagedBoundsArgs a, hipStream_t s);
constexpr int64_t PAGED_MAX_THREADS = 1LL << 32;  // of a launch
constexpr int64_t PAGED_MAX_ROWS = 1 << 30;  // rows of queries times their heads
constexpr int PAGED_MAX_PAGES = 4096;  // pages of a sequence, where pages are selected
struct PagedSelectArgs {
  const int8_t *bounds;
  const uint8_t *bounds_exp;
  const int32_t *table, *lens, *q_off;
  const void *q;
  int32_t *pages;
  int64_t q_stride;
  int32_t n_pages, n_heads, page_log2, max_pages, n_seqs, q_total, rows_each, group, n_select;
  int32_t rows_per, p_cap, waves;  // paged_select_grid: rows per workgroup, keys per row in LDS, wavefronts
};
// Fills these and returns the workgroups of the launch.
int64_t paged_select_grid(PagedSelectArgs &a);
hipError_t launch_paged_select(DType dt, int32_t head_dim, const PagedSelectArgs &a, int64_t grid,
                               hipStream_t s);
// Which keys a row of the attention sees: every token; those of listed pages; those
// of a window up to its own token, and the sequence's first ones; a context and the
// drafted tokens that its mask names.
enum PagedLook : int32_t { PAGED_ALL = 0, PAGED_LISTED = 1, PAGED_WINDOW = 2, PAGED_TREE = 3 };
constexpr int PAGED_ROW_WAVES = 4;  // wavefronts of 32 rows of a workgroup of paged_rows.h
constexpr int PAGED_MAX_MASK_WORDS = 64;  // of 32 drafted tokens each
constexpr int PAGED_JOIN_THREADS = 256;  // of the join's workgroup, one per (row, query head)
constexpr int paged_join_groups(int32_t head_dim) { return head_dim == 64 ? 16 : 8; }  // lane groups of the rows' join
constexpr int PAGED_MAX_SHARED = 256;  // sequences of a call whose ranges are shared out on the device
struct PagedAttnArgs {
  const void *k, *v;
  const uint8_t *k_exp, *v_exp;
  const int32_t *table, *lens, *q_off;
  const void *q;
  void *o;
  const int32_t *pages;  // [q_total][n_heads][n_select], or NULL: every token
  const int32_t *q_idx;  // [q_total]: the rows' tokens (windows)
  const int32_t *ctx;    // [n_seqs]: tokens before the drafted ones (trees)
  const uint32_t *mask;  // [q_total][mask_words]: drafted tokens that a row sees
  float *part_o, *part_ml;
  int64_t q_stride;
  int32_t n_pages, n_heads, page_log2, max_pages, n_seqs, q_total, q_max, rows_each, group, len_max,
      n_select;
  int32_t look, window, sinks, mask_words;  // PagedLook
  int32_t bits8;  // whether the cache holds 8 bits
  float sl2;  // log2(e) / sqrt(head_dim)
  // the plan (paged_plan): 16-row tiles and wavefronts per workgroup, row
  // blocks per sequence, key ranges, 32-key tiles per range, rows of a block
  // (with selected pages).  budget > 0: sequences are cut into equal ranges on
  // the device (Shares), at most `splits` each and `budget` in all, of `chunk`
  // tiles at least.
  int32_t row_tiles, waves, row_blocks, splits, chunk, bit_rows, budget;
  // row_waves > 0: blocks of 32 row_waves rows (paged_rows.h), otherwise of 16 row_tiles
  int32_t row_waves;
  FastDiv d_pairs;  // (sequence, head) pairs (PagedUnit)
  FastDiv d_splits, d_blocks, d_heads, d_group;
};
// Workgroups of the attention launch.
int64_t paged_grid(const PagedAttnArgs &a);
// Fills the plan from the sizes.
void paged_plan(DType dt, int32_t head_dim, PagedAttnArgs &a);
hipError_t launch_paged_attention(DType dt, int32_t format, int32_t head_dim, const PagedAttnArgs &a,
                                  hipStream_t s);
// How many (row, query head) pairs a lane group of the join takes in turn, or 0: a workgroup each.
int paged_join_turns(int32_t head_dim, const PagedAttnArgs &a);
hipError_t launch_paged_join(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_attention_bf16(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_attention_e4m3(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_attention_int8(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
// windows and trees
hipError_t launch_paged_masked_bf16(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_masked_e4m3(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_masked_int8(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_rows_bf16(int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_rows_e4m3(int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);
hipError_t launch_paged_rows_int8(int32_t head_dim, const PagedAttnArgs &a, hipStream_t s);

}  // namespace marche
