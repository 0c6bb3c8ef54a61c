// C-ABI front end of the serving operators: the cache append and the attention of new tokens over the
// whole cache. Argument checks (host only, before any HIP call) and launches. See include/lsa.h.
#include "api_common.hpp"
#include "launch.hpp"

using lsa::aligned;
using lsa::cdiv;
using lsa::fail;
using lsa::g_err;
using lsa::hip_fail;

namespace {

lsa_status check_append_params(const lsa_append_params* p) {
  LSA_REQUIRE(p != nullptr, LSA_ERR_INVALID_ARG, "params is NULL");
  LSA_REQUIRE(p->n_heads >= 0 && p->n_heads <= 4096, LSA_ERR_INVALID_ARG, "n_heads=%d not in [0, 4096]", p->n_heads);
  LSA_REQUIRE(p->n_kv_heads >= 1 && p->n_kv_heads <= 4096, LSA_ERR_INVALID_ARG, "n_kv_heads=%d not in [1, 4096]",
              p->n_kv_heads);
  LSA_REQUIRE(p->d_k >= 16 && p->d_k <= 1024 && p->d_k % 16 == 0, LSA_ERR_UNSUPPORTED,
              "d_k=%d must be a multiple of 16 in [16, 1024]", p->d_k);
  LSA_REQUIRE(p->d_v >= 0 && p->d_v <= 1024 && p->d_v % 16 == 0, LSA_ERR_UNSUPPORTED,
              "d_v=%d must be a multiple of 16 in [0, 1024]", p->d_v);
  LSA_REQUIRE(p->rot_start >= 0 && p->rot_dim >= 0 && p->rot_start <= p->d_k && p->rot_dim <= p->d_k - p->rot_start,
              LSA_ERR_INVALID_ARG, "rotated dims [%d, +%d) exceed d_k=%d", p->rot_start, p->rot_dim, p->d_k);
  LSA_REQUIRE(p->rot_start % 16 == 0 && p->rot_dim % 16 == 0, LSA_ERR_UNSUPPORTED,
              "rot_start=%d and rot_dim=%d must be multiples of 16", p->rot_start, p->rot_dim);
  LSA_REQUIRE(p->interleaved == 0 || p->interleaved == 1, LSA_ERR_INVALID_ARG, "interleaved=%d must be 0 or 1",
              p->interleaved);
  LSA_REQUIRE(p->key_dtype == LSA_KEY_BF16 || p->key_dtype == LSA_KEY_FP8_E4M3FN, LSA_ERR_INVALID_ARG,
              "key_dtype=%d unknown", p->key_dtype);
  return LSA_OK;
}

// An input [n_tok, heads, width] whose tokens lie `stride` elements apart.
lsa_status check_tokens(const char* name, const void* x, int64_t stride, int64_t heads, int64_t width) {
  LSA_REQUIRE(x != nullptr, LSA_ERR_INVALID_ARG, "%s is NULL", name);
  LSA_REQUIRE(aligned(x, 16) && stride % 8 == 0, LSA_ERR_INVALID_ARG,
              "%s must be 16-byte aligned and its stride (%lld) a multiple of 8", name, (long long)stride);
  LSA_REQUIRE(stride >= heads * width, LSA_ERR_INVALID_ARG, "%s: a stride of %lld is less than a token's %lld elements",
              name, (long long)stride, (long long)(heads * width));
  return LSA_OK;
}

lsa_status check_decode_params(const lsa_decode_attn_params* p) {
  LSA_REQUIRE(p != nullptr, LSA_ERR_INVALID_ARG, "params is NULL");
  LSA_REQUIRE(p->latent == 0 || p->latent == 1, LSA_ERR_INVALID_ARG, "latent=%d must be 0 or 1", p->latent);
  LSA_REQUIRE(p->n_heads >= 1 && p->n_heads <= 1024 && p->n_kv_heads >= 1 && p->n_heads % p->n_kv_heads == 0,
              LSA_ERR_INVALID_ARG, "n_heads=%d must be a multiple of n_kv_heads=%d and at most 1024", p->n_heads,
              p->n_kv_heads);
  LSA_REQUIRE(p->key_dtype == LSA_KEY_BF16 || p->key_dtype == LSA_KEY_FP8_E4M3FN, LSA_ERR_INVALID_ARG,
              "key_dtype=%d unknown", p->key_dtype);
  const bool mla = p->latent == 1 && p->n_kv_heads == 1 && p->d_qk == 576 && p->d_v == 512 && p->key_dtype == LSA_KEY_BF16;
  const bool gqa = p->latent == 0 && (p->d_qk == 64 || p->d_qk == 128) && p->d_v == p->d_qk;
  LSA_REQUIRE(mla || gqa, LSA_ERR_UNSUPPORTED,
              "attention shape (n_kv_heads=%d, d_qk=%d, d_v=%d, latent=%d, key_dtype=%d) not supported; use widths "
              "(64,64) or (128,128), or a bf16 latent cache of (576,512) with one head",
              p->n_kv_heads, p->d_qk, p->d_v, p->latent, p->key_dtype);
  LSA_REQUIRE(p->k_sink >= 0 && p->k_swa >= 0, LSA_ERR_INVALID_ARG, "k_sink=%d / k_swa=%d must be >= 0", p->k_sink,
              p->k_swa);
  LSA_REQUIRE(p->sm_scale > 0.f && p->sm_scale < 1e30f, LSA_ERR_INVALID_ARG, "sm_scale must be positive and finite");
  return LSA_OK;
}

lsa_status check_decode_sizes(const lsa_decode_attn_params* p, int32_t n_seq, int32_t rows_per_seq, int32_t max_pages,
                              int32_t kv_page_size) {
  LSA_REQUIRE(n_seq >= 0, LSA_ERR_INVALID_ARG, "n_seq=%d < 0", n_seq);
  LSA_REQUIRE(rows_per_seq >= 1 && max_pages >= 1 && kv_page_size >= 1, LSA_ERR_INVALID_ARG,
              "rows_per_seq, max_pages and kv_page_size must be >= 1");
  LSA_REQUIRE((int64_t)max_pages * kv_page_size < (1LL << 31), LSA_ERR_UNSUPPORTED, "positions must fit in int32");
  LSA_REQUIRE(rows_per_seq <= 1024 && (int64_t)n_seq * rows_per_seq * p->n_heads < (1LL << 30), LSA_ERR_UNSUPPORTED,
              "rows_per_seq must be <= 1024 and the call have < 2^30 rows of all heads");
  return LSA_OK;
}

// How a call is dealt out (decode_attn.hip): `grid` workgroups take equal stretches of all tiles.
struct DecodePlan {
  int grid, stretches, waves, min_tiles, block_cols, blocks, M, pass_tiles;  // (see DecodeGeom)
  bool cut;  // may a stretch end inside a (sequence, head)?
  int64_t all_tiles;  // at most
  bool together;
  size_t off_ml, off_parts, total;
};
constexpr int64_t kCus = 256;
constexpr int kTile = 32;          // positions of a tile
constexpr int kPageSlots = 2048;   // page-table entries a workgroup stages at a time
constexpr int kLatentPages = 1024; // the same, latent cache

// A (sequence, head, query row block) of at most that many tiles is left whole: a workgroup each, no scan of the lengths, no
// partials and no join. What the host knows is the tables' capacity, so the bound, at most 64 tiles, also limits what one long
// sequence among short ones can cost. It follows the kernels' time (a cut call costs the host 3 us more, for its second launch; a
// graph of the step has neither): with few workgroups a whole one is faster for as many tiles as scan, partials and join are
// worth, `base`, more where stretches of several sequences end inside them, and the more workgroups there are, the fewer can a
// cut call add. us on the GPU, cut / whole, at capacities around so many tiles, the lengths 0.6 to 1 of them:
//   lone: 16 rows of 128, 1 head 20 9.2 / 8.9, 24 9.3 / 9.4, 32 9.4 / 11.7; 8 heads 20 9.0 / 8.7, 24 9.0 / 9.2, 32 10.5 / 11.7; fp8 20 8.8 / 8.5, 24 8.6 /
//     9.2; 32 rows 16 11.1 / 11.0, 24 11.1 / 12.2; 64 wide, 12 heads 28 8.7 / 8.3, 36 8.4 / 8.9; 32 rows 24 8.9 / 8.7, 28 8.8 / 9.8; 33 to 64 rows 8 13.8 /
//     13.1, 12 13.7 / 15.4, 64 wide 12 10.6 / 10.7; latent 4 10.4 / 9.2, 8 10.5 / 11.2
//   16 rows of 128, sequences x heads: 2 x 8 28 12.8 / 11.4, 32 11.8 / 11.9, 46 13.1 / 14.1; 4 x 8 40 14.8 / 13.3, 52 15.4 / 15.4; 8 x 8 46 19.2 / 18.5, 52 20.0 /
//     21.4; 8 x 1 46 14.0 / 14.0; 32 x 1 64 17.9 / 17.9; 12 x 8 52 25.5 / 24.6, 58 26.9 / 26.2; 96 x 1 64 32.5 / 29.8; fp8 8 x 8 64 17.2 / 17.3
//   32 rows: 8 x 1 40 17.6 / 16.4, 52 17.7 / 18.7; 64 x 1 58 28.1 / 25.9; 64 wide: 2 x 4 36 8.8 / 8.9; 4 x 4 46 10.9 / 11.1; 8 x 4 58 12.8 / 12.7; 32 x 1 64 15.7 / 15.3
//   33 to 64 rows: 4 x 1 28 21.9 / 23.6; 32 x 1 32 24.7 / 25.2; 64 x 1 46 34.8 / 33.4, 52 36.0 / 37.0; 96 x 1 52 42.1 / 38.6; 64 wide 4 x 1 24 15.2 / 14.4; 32 x 1 32 18.5 /
//     18.6; 64 x 1 46 24.1 / 23.5; two new tokens 4 x 2 24 25.7 / 25.5; 16 x 2 24 26.8 / 26.3; 32 x 2 32 33.4 / 33.4; 48 x 2 46 44.6 / 44.5; 64 x 2 52 51.1 / 50.1
//   latent, one block: 4 8 12.1 / 11.3, 12 13.0 / 15.0; 16 12 15.7 / 15.6; 28 16 17.6 / 18.8; 64 20 24.1 / 22.1, 24 25.6 / 24.7, 28 27.8 / 29.3; 80 28 31.4 / 30.8, 32
//     33.1 / 33.8; 96 32 36.4 / 35.4, 40 41.5 / 42.7; 112 46 49.9 / 45.3, 64 61.4 / 60.2; 128 64 66.6 / 61.5; two blocks: 4 8 13.7 / 11.6, 12 14.4 / 15.3; 32 20 22.9 /
//     22.4; 64 28 32.9 / 31.1, 36 35.3 / 36.8; blocks of 64: 8 12 19.2 / 19.2; 28 20 25.5 / 26.4; 64 28 36.4 / 37.1; 97 46 57.0 / 54.3, 64 68.9 / 71.9; 128 64 81.5 / 74.8
int64_t whole_tiles(const lsa_decode_attn_params* p, int block_cols, int64_t n_seq, int64_t pairs) {
  const bool lone = n_seq == 1;
  int64_t t;
  if (p->latent) {  // (the two blocks of 32 rows of a sequence share its rows of the cache and count as one workgroup)
    const int64_t n = pairs / 2 > n_seq ? pairs / 2 : n_seq;
    t = (lone ? 6 : 9) + n / 4 + (n > 80 ? (n - 80) * 2 / 3 : 0);
  } else {
    const int64_t base = block_cols == 64 ? (lone ? 10 : 22) : !lone ? 36 : p->d_qk == 128 ? 22 : 28;
    t = base + pairs / 3;
  }
  return t < 64 ? t : 64;
}

DecodePlan plan_decode(const lsa_decode_attn_params* p, int32_t n_seq, int32_t rows_per_seq, int32_t max_pages,
                       int32_t kv_page_size) {
  DecodePlan pl{};
  const bool latent = p->latent != 0;
  const int64_t cap = (int64_t)max_pages * kv_page_size;
  int64_t tiles = cdiv(cap, kTile);  // of one (sequence, head), at most
  if (p->k_swa > 0) {
    const int64_t window = cdiv(p->k_sink, kTile) + cdiv((int64_t)p->k_swa + rows_per_seq, kTile) + 1;
    tiles = window < tiles ? window : tiles;
  }
  // The query rows of a key/value head, in blocks. More rows a block read the cache fewer times; latent blocks of 32 go to
  // twice the workgroups, at 0.6 us a tile instead of 0.95, with half the partials. us of 64 heads in blocks of 32 / 64: 1 x 200
  // 10.5 / 12.6, 1 x 16K 21.4 / 24.3, 1 x 64K 30.1 / 32.5, 8 x 16K 53.5 / 50.9, 64 x 300 15.6 / 18.2, 64 x 1000 30.8 / 36.2, 128 x 300 20.2 /
  // 19.3, 128 x 700 33.6 / 31.4.
  const int64_t cols = (int64_t)rows_per_seq * (p->n_heads / p->n_kv_heads), blocks64 = n_seq * cdiv(cols, 64);
  if (latent) pl.block_cols = cols <= 32 || (blocks64 <= 96 && blocks64 * tiles <= 2048) ? 32 : 64;
  else pl.block_cols = cols <= 16 ? 16 : cols <= 32 ? 32 : 64;
  pl.blocks = (int)cdiv(cols, pl.block_cols);
  pl.M = p->n_kv_heads * pl.blocks;
  const int64_t pairs = (int64_t)n_seq * pl.M;
  pl.min_tiles = latent ? 2 : 4;  // (grouped heads: one per wave)
  pl.all_tiles = pairs * tiles;
  const int64_t some = cdiv(pl.all_tiles, lsa::least_tiles(pl.all_tiles, pl.min_tiles)), most = some > pairs ? some : pairs;
  const int64_t wgs = kCus * (latent ? 1 : lsa::gqa_per_cu(p->d_qk, pl.block_cols / 16, rows_per_seq > 1, 4));
  const int64_t n = (most < wgs ? most : wgs) / pl.M;
  pl.stretches = (int)(n > 1 ? n : 1);
  pl.together = pl.blocks > 1 && pl.stretches >= 8;
  if (pl.together) pl.stretches &= -8;
  pl.cut = tiles > whole_tiles(p, pl.block_cols, n_seq, pairs);
  // Left whole, a (sequence, head) has one workgroup: of 8 waves where the workgroups are fewer than the CUs and their tiles
  // enough for 8. us with 4 / 8 waves, 32 heads on 8: 8 x 2000 22.8 / 17.4, 16 x 1001 15.1 / 15.2, 24 x 1000 19.4 / 20.0, 32 x 1000
  // 26.5 / 27.0, 1 x 250 6.5 / 6.7, 1 x 500 8.5 / 8.0; 16 heads on one, 69 x 2000 23.3 / 18.1; fp8 24 x 1000 15.5 / 14.2.
  pl.waves = !latent && !pl.cut && pairs <= kCus * 3 / 4 && tiles > 8 && pl.block_cols <= 32 ? 8 : 4;
  pl.grid = (int)(pl.cut ? (int64_t)pl.stretches * pl.M : pairs);
  // pages of a pass: tiles * 32 / P, and two more at the ends of each of two parts
  const int64_t pass = (int64_t)((latent ? kLatentPages : kPageSlots) - 4) * kv_page_size / kTile;
  pl.pass_tiles = (int)(pass < (1 << 26) ? pass : (1 << 26));
  const size_t parts = pl.cut ? (size_t)2 * pl.grid * pl.block_cols : 0;
  pl.off_ml = lsa::round_up(parts * p->d_v * 4, 256);
  pl.off_parts = pl.off_ml + lsa::round_up(parts * 2 * 4, 256);
  pl.total = pl.off_parts + (pl.cut ? lsa::round_up((size_t)pairs * 16, 256) : 0);
  return pl;
}

// lsa_cache_append (norm NULL) and lsa_norm_append
lsa_status append(const lsa_append_params* p, const lsa_append_norm* norm, const lsa_append_tensors* t, int64_t n_tok, int32_t n_seq,
                  int32_t rows_per_seq, int32_t max_pages, int32_t kv_page_size, int64_t n_phys, void* stream) {
  g_err[0] = 0;
  lsa_status s = check_append_params(p);
  if (s != LSA_OK) return s;
  LSA_REQUIRE(t != nullptr, LSA_ERR_INVALID_ARG, "tensors is NULL");
  LSA_REQUIRE(n_tok >= 0 && n_seq >= 0, LSA_ERR_INVALID_ARG, "n_tok=%lld / n_seq=%d < 0", (long long)n_tok, n_seq);
  if (n_tok == 0) return LSA_OK;  // nothing to read or write
  LSA_REQUIRE(n_tok < (1LL << 28), LSA_ERR_UNSUPPORTED, "n_tok must be < 2^28 per call");
  LSA_REQUIRE(n_seq >= 1 && rows_per_seq >= 1 && max_pages >= 1 && kv_page_size >= 1 && n_phys >= 1,
              LSA_ERR_INVALID_ARG, "n_seq, rows_per_seq, max_pages, kv_page_size and n_phys must be >= 1");
  LSA_REQUIRE((int64_t)max_pages * kv_page_size < (1LL << 31), LSA_ERR_UNSUPPORTED, "positions must fit in int32");
  LSA_REQUIRE(n_phys < (1LL << 31) && n_phys * kv_page_size < (1LL << 31) / p->n_kv_heads, LSA_ERR_UNSUPPORTED,
              "n_phys * kv_page_size * n_kv_heads must be < 2^31");
  LSA_REQUIRE(t->page_table != nullptr || (max_pages == 1 && n_phys >= n_seq), LSA_ERR_INVALID_ARG,
              "without a page table each sequence has one page: max_pages must be 1 and n_phys >= n_seq");
  LSA_REQUIRE((t->pos != nullptr) != (t->ctx_len != nullptr), LSA_ERR_INVALID_ARG,
              "exactly one of pos and ctx_len must be given");
  LSA_REQUIRE(t->pos != nullptr || (t->seq == nullptr && n_tok == (int64_t)n_seq * rows_per_seq), LSA_ERR_INVALID_ARG,
              "with ctx_len the tokens are rows_per_seq of every sequence: n_tok must be n_seq * rows_per_seq, seq NULL");
  const bool fp8 = p->key_dtype == LSA_KEY_FP8_E4M3FN, rot = p->rot_dim > 0;
  LSA_REQUIRE(rot == (t->rope != nullptr) && t->rope_rows >= 0, LSA_ERR_INVALID_ARG,
              "rope must be given exactly when rot_dim > 0, rope_rows must be >= 0");
  LSA_REQUIRE((t->k_rot == nullptr && t->q_rot == nullptr) || (rot && p->rot_start > 0 && p->rot_start + p->rot_dim == p->d_k),
              LSA_ERR_INVALID_ARG, "k_rot / q_rot need a rotation of the last rot_dim dims, fewer than d_k");
  LSA_REQUIRE((t->q != nullptr) == (p->n_heads > 0) && (t->q_out != nullptr) == (p->n_heads > 0) &&
                  (t->q_rot == nullptr || p->n_heads > 0),
              LSA_ERR_INVALID_ARG, "q and q_out must be given exactly when n_heads > 0, q_rot only then");
  LSA_REQUIRE((t->v != nullptr) == (p->d_v > 0) && (t->v_cache != nullptr) == (p->d_v > 0), LSA_ERR_INVALID_ARG,
              "v and v_cache must be given exactly when d_v > 0");
  LSA_REQUIRE(t->k_cache != nullptr, LSA_ERR_INVALID_ARG, "k_cache is NULL");
  LSA_REQUIRE((t->k_scale != nullptr) == fp8 && (t->v_scale != nullptr) == (fp8 && p->d_v > 0), LSA_ERR_INVALID_ARG,
              "k_scale / v_scale must be given exactly for fp8 caches");
  const int64_t k_width = t->k_rot ? p->d_k - p->rot_dim : p->d_k, q_width = t->q_rot ? p->d_k - p->rot_dim : p->d_k;
  s = check_tokens("k", t->k, t->k_stride, p->n_kv_heads, k_width);
  if (s == LSA_OK && t->k_rot) s = check_tokens("k_rot", t->k_rot, t->k_rot_stride, p->n_kv_heads, p->rot_dim);
  if (s == LSA_OK && t->v) s = check_tokens("v", t->v, t->v_stride, p->n_kv_heads, p->d_v);
  if (s == LSA_OK && t->q) s = check_tokens("q", t->q, t->q_stride, p->n_heads, q_width);
  if (s == LSA_OK && t->q_rot) s = check_tokens("q_rot", t->q_rot, t->q_rot_stride, p->n_heads, p->rot_dim);
  if (s != LSA_OK) return s;
  LSA_REQUIRE(t->q == nullptr || t->q_out != t->q || (t->q_rot == nullptr && t->q_stride == (int64_t)p->n_heads * p->d_k),
              LSA_ERR_INVALID_ARG, "q_out may be q only when q is contiguous and whole");
  LSA_REQUIRE(aligned(t->q_out, 16) && aligned(t->k_cache, 16) && aligned(t->v_cache, 16) && aligned(t->rope, 16),
              LSA_ERR_INVALID_ARG, "q_out, k_cache, v_cache and rope must be 16-byte aligned");
  LSA_REQUIRE(aligned(t->seq, 4) && aligned(t->pos, 4) && aligned(t->ctx_len, 4) && aligned(t->page_table, 4) &&
                  aligned(t->k_scale, 4) && aligned(t->v_scale, 4) && aligned(t->rows, 8),
              LSA_ERR_INVALID_ARG, "seq, pos, ctx_len, page_table and scales must be 4-byte aligned, rows 8-byte");
  if (norm != nullptr) {
    LSA_REQUIRE(norm->eps > 0.f && norm->eps < 1e30f, LSA_ERR_INVALID_ARG, "eps must be positive and finite");
    LSA_REQUIRE(norm->q_weight == nullptr || p->n_heads > 0, LSA_ERR_INVALID_ARG, "q_weight must be NULL with n_heads = 0");
    LSA_REQUIRE(aligned(norm->q_weight, 16) && aligned(norm->k_weight, 16) && aligned(norm->k_out, 16), LSA_ERR_INVALID_ARG,
                "q_weight, k_weight and k_out must be 16-byte aligned");
    LSA_REQUIRE(norm->k_out == nullptr || norm->k_out != t->k || (t->k_rot == nullptr && t->k_stride == (int64_t)p->n_kv_heads * p->d_k),
                LSA_ERR_INVALID_ARG, "k_out may be k only when k is contiguous and whole");
  }

  lsa::AppendGeom g{};
  if (norm != nullptr) {
    g.q_weight = static_cast<const uint16_t*>(norm->q_weight);
    g.k_weight = static_cast<const uint16_t*>(norm->k_weight);
    g.k_out = static_cast<uint16_t*>(norm->k_out);
    g.eps = norm->eps;
  }
  g.q = static_cast<const uint16_t*>(t->q);
  g.q_rot = static_cast<const uint16_t*>(t->q_rot);
  g.k = static_cast<const uint16_t*>(t->k);
  g.k_rot = static_cast<const uint16_t*>(t->k_rot);
  g.v = static_cast<const uint16_t*>(t->v);
  g.q_stride = t->q_stride;
  g.q_rot_stride = t->q_rot_stride;
  g.k_stride = t->k_stride;
  g.k_rot_stride = t->k_rot_stride;
  g.v_stride = t->v_stride;
  g.rope = t->rope;
  g.rope_rows = t->rope_rows;
  g.seq = t->seq;
  g.pos = t->pos;
  g.ctx_len = t->ctx_len;
  g.page_table = t->page_table;
  g.q_out = static_cast<uint16_t*>(t->q_out);
  g.k_cache = t->k_cache;
  g.v_cache = t->v_cache;
  g.k_scale = t->k_scale;
  g.v_scale = t->v_scale;
  g.rows = t->rows;
  g.n_tok = (int)n_tok;
  g.n_phys = n_phys;
  g.H = p->n_heads;
  g.Hkv = p->n_kv_heads;
  g.d_k = p->d_k;
  g.d_v = p->d_v;
  g.rot_start = p->rot_start;
  g.rot_dim = p->rot_dim;
  g.interleaved = p->interleaved;
  g.fp8 = fp8;
  g.n_seq = n_seq;
  g.by_rows = lsa::fast_div((uint32_t)rows_per_seq);
  g.max_pages = max_pages;
  g.P = kv_page_size;
  const hipError_t e = lsa::launch_append(g, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "cache append");
  return LSA_OK;
}

}  // namespace

extern "C" {

lsa_status lsa_cache_append(const lsa_append_params* p, const lsa_append_tensors* t, int64_t n_tok, int32_t n_seq,
                            int32_t rows_per_seq, int32_t max_pages, int32_t kv_page_size, int64_t n_phys,
                            void* stream) {
  return append(p, nullptr, t, n_tok, n_seq, rows_per_seq, max_pages, kv_page_size, n_phys, stream);
}

lsa_status lsa_norm_append(const lsa_append_params* p, const lsa_append_norm* norm, const lsa_append_tensors* t, int64_t n_tok,
                           int32_t n_seq, int32_t rows_per_seq, int32_t max_pages, int32_t kv_page_size, int64_t n_phys,
                           void* stream) {
  g_err[0] = 0;
  LSA_REQUIRE(norm != nullptr, LSA_ERR_INVALID_ARG, "norm is NULL");
  return append(p, norm, t, n_tok, n_seq, rows_per_seq, max_pages, kv_page_size, n_phys, stream);
}

size_t lsa_decode_attn_workspace_size(const lsa_decode_attn_params* p, int32_t n_seq, int32_t rows_per_seq,
                                      int32_t max_pages, int32_t kv_page_size) {
  if (check_decode_params(p) != LSA_OK || check_decode_sizes(p, n_seq, rows_per_seq, max_pages, kv_page_size) != LSA_OK) return 0;
  return n_seq == 0 ? 0 : plan_decode(p, n_seq, rows_per_seq, max_pages, kv_page_size).total;
}

lsa_status lsa_decode_attn(const lsa_decode_attn_params* p, int32_t n_seq, int32_t rows_per_seq, const void* q,
                           const void* k_cache, const float* k_scale, const void* v_cache, const float* v_scale,
                           const int32_t* ctx_len, const int32_t* page_table, int32_t max_pages, int32_t kv_page_size,
                           int64_t n_phys, void* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  lsa_status s = check_decode_params(p);
  if (s != LSA_OK) return s;
  s = check_decode_sizes(p, n_seq, rows_per_seq, max_pages, kv_page_size);
  if (s != LSA_OK) return s;
  if (n_seq == 0) return LSA_OK;  // nothing to read or write
  LSA_REQUIRE(n_phys >= 1 && n_phys < (1LL << 31) && n_phys * kv_page_size < (1LL << 31) / p->n_kv_heads,
              LSA_ERR_UNSUPPORTED, "n_phys must be >= 1 and n_phys * kv_page_size * n_kv_heads < 2^31");
  LSA_REQUIRE(page_table != nullptr || (max_pages == 1 && n_phys >= n_seq), LSA_ERR_INVALID_ARG,
              "without a page table each sequence has one page: max_pages must be 1 and n_phys >= n_seq");
  const bool fp8 = p->key_dtype == LSA_KEY_FP8_E4M3FN, latent = p->latent != 0;
  LSA_REQUIRE(q && k_cache && ctx_len && out, LSA_ERR_INVALID_ARG, "q, k_cache, ctx_len and out must be non-NULL");
  LSA_REQUIRE(latent == (v_cache == nullptr), LSA_ERR_INVALID_ARG,
              latent ? "v_cache must be NULL for a latent cache" : "v_cache is NULL");
  LSA_REQUIRE(fp8 == (k_scale != nullptr) && fp8 == (v_scale != nullptr), LSA_ERR_INVALID_ARG,
              "k_scale and v_scale must be given exactly for fp8 caches");
  LSA_REQUIRE(aligned(q, 16) && aligned(k_cache, 16) && aligned(v_cache, 16) && aligned(out, 16), LSA_ERR_INVALID_ARG,
              "q, k_cache, v_cache and out must be 16-byte aligned");
  LSA_REQUIRE(aligned(k_scale, 4) && aligned(v_scale, 4) && aligned(ctx_len, 4) && aligned(page_table, 4) && aligned(lse, 4),
              LSA_ERR_INVALID_ARG, "scales, ctx_len, page_table and lse must be 4-byte aligned");
  const DecodePlan pl = plan_decode(p, n_seq, rows_per_seq, max_pages, kv_page_size);
  LSA_REQUIRE(pl.all_tiles <= (1LL << 30), LSA_ERR_UNSUPPORTED,
              "n_seq * max_pages * kv_page_size / 32 * n_kv_heads must be <= 2^30");
  const size_t need = pl.total;
  LSA_REQUIRE(need == 0 || (workspace != nullptr && aligned(workspace, 256)), LSA_ERR_WORKSPACE,
              "workspace must be non-NULL and 256-byte aligned");
  LSA_REQUIRE(ws_bytes >= need, LSA_ERR_WORKSPACE, "workspace of %zu bytes < %zu needed", ws_bytes, need);
  lsa::DecodeGeom g{};
  g.q = static_cast<const uint16_t*>(q);
  g.k = k_cache;
  g.v = v_cache;
  g.k_scale = k_scale;
  g.v_scale = v_scale;
  g.ctx_len = ctx_len;
  g.page_table = page_table;
  g.out = static_cast<uint16_t*>(out);
  g.lse = lse;
  g.n_phys = n_phys;
  g.n_seq = n_seq;
  g.R = rows_per_seq;
  g.H = p->n_heads;
  g.Hkv = p->n_kv_heads;
  g.d_qk = p->d_qk;
  g.d_v = p->d_v;
  g.latent = latent;
  g.fp8 = fp8;
  g.max_pages = max_pages;
  g.P = kv_page_size;
  g.cap = max_pages * kv_page_size;
  // (a window of all positions is none, and without a window there is no separate sink)
  g.k_swa = p->k_swa < g.cap ? p->k_swa : 0;
  g.k_sink = g.k_swa == 0 ? 0 : p->k_sink < g.cap ? p->k_sink : g.cap;
  g.scale_log2 = p->sm_scale * 1.4426950408889634f;
  g.by_page = lsa::fast_div((uint32_t)kv_page_size);
  g.pass_tiles = pl.pass_tiles;
  g.whole_tiles = kv_page_size % kTile == 0;
  g.block_cols = pl.block_cols;
  g.by_group = lsa::fast_div((uint32_t)(p->n_heads / p->n_kv_heads));
  g.by_blocks = lsa::fast_div((uint32_t)pl.blocks);
  g.M = pl.M;
  g.by_m = lsa::fast_div((uint32_t)pl.M);
  g.grid = pl.grid;
  g.by_stretches = lsa::fast_div((uint32_t)pl.stretches);
  g.together = pl.cut && pl.together;
  g.by_seqs = lsa::fast_div((uint32_t)n_seq);
  g.waves = pl.waves;
  g.min_tiles = pl.min_tiles;
  if (pl.cut) {
    g.part_o = static_cast<float*>(workspace);
    g.part_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + pl.off_ml);
    g.parts = reinterpret_cast<int4*>(static_cast<uint8_t*>(workspace) + pl.off_parts);
  }
  const hipError_t e = lsa::launch_decode_attn(g, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "decode attention");
  return LSA_OK;
}

}  // extern "C"
