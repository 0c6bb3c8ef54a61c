// C-ABI front end of the prompt side of serving: reading a paged cache back, attention of packed prompts and of chunks of new
// tokens over a paged cache. Argument checks (host only, before any HIP
// call) and launches. See include/lsa.h.
#include "api_common.hpp"
#include "launch.hpp"

using lsa::aligned;
using lsa::fail;
using lsa::g_err;
using lsa::hip_fail;

namespace {

// Calls of at most so many blocks of rows are cut along their keys into about so many pieces, one per CU. us of 32 heads on 8 of 128, with the limit
// of blocks at 0 / 256 / 512 / 1024: 16 tokens behind 32K (8 blocks) in fp8 872 / 47 / 47 / 47; 1024 behind 7K (136) 226 / 162 / 159 / 159; 24 sequences,
// 2048 tokens (456) 238 / 231 / 207 / 203, in fp8 309 / 304 / 237 / 237; 2048 behind 6K (264) 256 / 260 / 264 / 264; 3900 behind 4K (496) 393 / 401 / 407
// / 406. From 256 blocks on it is blocks of unequal lengths that gain; equal ones lose 1 to 4%, but the host has the sizes alone and cannot tell them apart. For
// the same reason calls are planned as cut whose blocks then stay whole (short prompts, of which only the sum of keys is known, and windows), and
// pay for the join's launch: 16 prompts of 100 28.5, 25.2 without the plan; window of 1024, 12 heads of 64, 8192 tokens 66.7, 62.5, 2048 of 32 on 8 51.4, 48.2, 24
// sequences 96, 92. With 128 / 256 / 512 pieces: 16 behind 32K in fp8 69 / 47 / 56, 512 behind 8K 144 / 102 / 121, 24 sequences 239 / 207 / 222.
constexpr int64_t kMostCutBlocks = 512;
constexpr int kPieces = 256;
// They have to have more than so many keys: the more blocks, the more CUs are busy with them whole, and the more partial results there are. us whole
// and cut: 16 tokens of 500 keys (8 blocks) 17.4, 15.6, of 900 23.3, 16.6, of 2K 43, 16.4; 200 of 900 (32) 34.0, 27.8; 16 heads on one,
// prompts of 700 (45) 27.3, 28.0; 12 heads of 64, 900 (48) 23.4, 22.3; 32 on 8, 300 (40) 17.1, 24.2, 700 (88) 28.4, 37, 1024 (136) 37, 41,
// 1500 (192) 67, 55.
constexpr int64_t least_cut_keys(int64_t blocks) { return lsa::kPromptKeys * (blocks < 32 ? 8 : blocks > 64 ? 16 : blocks / 4); }

// Every workgroup looks through the sequences, 64 at a time, so that a call's time grows with their square (figures beside lsa_chunk_attn in lsa.h;
// 2^21 sequences would hold the GPU for minutes). And with at most so many the device's sums over sequences (pieces of calls that are cut: per sequence
// kMostCutBlocks blocks and Hkv more) stay below 2^31 whatever the offsets hold, also where they do not ascend.
constexpr int32_t kMostSequences = 1 << 16;

// The pages of a call's caches
lsa_status check_pages(const int32_t* page_table, int32_t n_seq, int32_t max_pages, int32_t kv_page_size, int64_t n_phys, int32_t n_kv_heads) {
  LSA_REQUIRE(max_pages >= 1 && kv_page_size >= 1 && n_phys >= 1, LSA_ERR_INVALID_ARG,
              "max_pages, kv_page_size and n_phys must be >= 1");
  LSA_REQUIRE((int64_t)max_pages * kv_page_size < (1LL << 31), LSA_ERR_UNSUPPORTED, "positions must fit in int32");
  LSA_REQUIRE(n_phys < (1LL << 31) && n_phys * kv_page_size < (1LL << 31) / n_kv_heads, LSA_ERR_UNSUPPORTED,
              "n_phys * kv_page_size * n_kv_heads must be < 2^31");
  LSA_REQUIRE(page_table != nullptr || (max_pages == 1 && n_phys >= n_seq), LSA_ERR_INVALID_ARG,
              "without a page table each sequence has one page: max_pages must be 1 and n_phys >= n_seq");
  return LSA_OK;
}

lsa_status check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t k_sink, int32_t k_swa, float sm_scale) {
  LSA_REQUIRE(n_heads >= 1 && n_heads <= 1024 && n_kv_heads >= 1 && n_heads % n_kv_heads == 0, LSA_ERR_INVALID_ARG,
              "n_heads=%d must be a multiple of n_kv_heads=%d and at most 1024", n_heads, n_kv_heads);
  LSA_REQUIRE(k_sink >= 0 && k_swa >= 0, LSA_ERR_INVALID_ARG, "k_sink=%d / k_swa=%d must be >= 0", k_sink, k_swa);
  LSA_REQUIRE(sm_scale > 0.f && sm_scale < 1e30f, LSA_ERR_INVALID_ARG, "sm_scale must be positive and finite");
  return LSA_OK;
}

lsa_status check_prefill_params(const lsa_prefill_attn_params* p) {
  LSA_REQUIRE(p != nullptr, LSA_ERR_INVALID_ARG, "params is NULL");
  LSA_REQUIRE((p->d_qk == 64 && p->d_v == 64) || (p->d_qk == 128 && p->d_v == 128) || (p->d_qk == 192 && p->d_v == 128),
              LSA_ERR_UNSUPPORTED, "attention shape (d_qk=%d, d_v=%d) not supported; use (64,64), (128,128) or (192,128)", p->d_qk,
              p->d_v);
  LSA_REQUIRE(p->causal == 0 || p->causal == 1, LSA_ERR_INVALID_ARG, "causal=%d must be 0 or 1", p->causal);
  LSA_REQUIRE(p->causal || (p->k_swa == 0 && p->k_sink == 0), LSA_ERR_UNSUPPORTED, "a window and a sink need causal = 1");
  return check_heads(p->n_heads, p->n_kv_heads, p->k_sink, p->k_swa, p->sm_scale);
}

lsa_status check_chunk_params(const lsa_decode_attn_params* p) {
  LSA_REQUIRE(p != nullptr, LSA_ERR_INVALID_ARG, "params is NULL");
  LSA_REQUIRE(p->latent == 0 || p->latent == 1, LSA_ERR_INVALID_ARG, "latent=%d must be 0 or 1", p->latent);
  LSA_REQUIRE(p->latent == 0 && (p->d_qk == 64 || p->d_qk == 128) && p->d_v == p->d_qk, LSA_ERR_UNSUPPORTED,
              "attention shape (d_qk=%d, d_v=%d, latent=%d) not supported; use (64,64) or (128,128), not latent", p->d_qk, p->d_v,
              p->latent);
  LSA_REQUIRE(p->key_dtype == LSA_KEY_BF16 || p->key_dtype == LSA_KEY_FP8_E4M3FN, LSA_ERR_INVALID_ARG, "key_dtype=%d unknown",
              p->key_dtype);
  return check_heads(p->n_heads, p->n_kv_heads, p->k_sink, p->k_swa, p->sm_scale);
}

lsa_status check_tokens(int32_t n_seq, int64_t n_tok, int32_t n_heads, int32_t n_kv_heads) {
  LSA_REQUIRE(n_seq >= 0 && n_tok >= 0, LSA_ERR_INVALID_ARG, "n_seq=%d / n_tok=%lld < 0", n_seq, (long long)n_tok);
  LSA_REQUIRE(n_seq <= kMostSequences, LSA_ERR_UNSUPPORTED, "n_seq=%d must be at most %d per call", n_seq, kMostSequences);
  LSA_REQUIRE(n_tok < (1LL << 30) && n_tok * n_heads < (1LL << 30) && (int64_t)n_seq * n_kv_heads < (1LL << 24), LSA_ERR_UNSUPPORTED,
              "n_tok * n_heads must be < 2^30 and n_seq * n_kv_heads < 2^24");
  return LSA_OK;
}

lsa_status check_rows(const char* name, const void* x, int64_t stride, int64_t heads, int64_t width) {
  LSA_REQUIRE(x != nullptr, LSA_ERR_INVALID_ARG, "%s is NULL", name);
  LSA_REQUIRE(aligned(x, 16) && stride % 8 == 0, LSA_ERR_INVALID_ARG,
              "%s must be 16-byte aligned and its stride (%lld) a multiple of 8", name, (long long)stride);
  LSA_REQUIRE(stride >= heads * width, LSA_ERR_INVALID_ARG, "%s: a stride of %lld is less than a row's %lld elements", name,
              (long long)stride, (long long)(heads * width));
  LSA_REQUIRE(stride < (1LL << 24), LSA_ERR_UNSUPPORTED, "%s: a stride of %lld is not below 2^24", name, (long long)stride);
  return LSA_OK;
}

// What both attentions have of their sizes.
void set_heads(lsa::PromptGeom& g, int32_t n_seq, int64_t n_tok, int32_t n_heads, int32_t n_kv_heads, int32_t d_qk, int32_t d_v,
               int32_t k_sink, int32_t k_swa, int64_t most_keys, float sm_scale) {
  g.n_seq = n_seq;
  g.n_tok = (int)n_tok;
  g.H = n_heads;
  g.Hkv = n_kv_heads;
  g.d_qk = d_qk;
  g.d_v = d_v;
  // (a window of all positions is none, and without a window there is no separate sink)
  g.k_swa = k_swa < most_keys ? k_swa : 0;
  g.k_sink = g.k_swa == 0 ? 0 : (int)(k_sink < most_keys ? k_sink : most_keys);
  g.scale_log2 = sm_scale * 1.4426950408889634f;
  g.by_group = lsa::fast_div((uint32_t)(n_heads / n_kv_heads));
  // Of each sequence every XCD takes turns at a class of heads (prompt_attn.hip), as many turns of each head as blocks of rows over
  // the XCDs that share it, rounded up: the sum of roundings is below the sequences that have tokens.
  g.head_classes = n_kv_heads % 8 == 0 ? 8 : n_kv_heads % 4 == 0 ? 4 : n_kv_heads % 2 == 0 ? 2 : 1;
  const int64_t per_turn = (int64_t)lsa::kPromptRows * (8 / g.head_classes), rows = n_tok * (n_heads / n_kv_heads);
  g.items = 8 * (n_kv_heads / g.head_classes) * (rows / per_turn + (n_seq < n_tok ? n_seq : n_tok));
}

// Whether a call's blocks of rows are cut along their keys, and its workspace.
struct PromptPlan {
  int pieces, blocks, slot_rows;
  size_t off_ml, off_joins, off_n, total;
};
PromptPlan plan_prompt(int32_t n_seq, int64_t n_tok, int32_t n_heads, int32_t n_kv_heads, int32_t d_v, int32_t k_sink, int32_t k_swa,
                       int64_t most_keys) {
  PromptPlan pl{};
  const int64_t rows = n_tok * (n_heads / n_kv_heads), blocks = n_kv_heads * (rows / lsa::kPromptRows + (n_seq < n_tok ? n_seq : n_tok));
  int64_t keys = most_keys;
  if (k_swa > 0 && (int64_t)k_sink + k_swa + lsa::kPromptRows < keys) keys = (int64_t)k_sink + k_swa + lsa::kPromptRows;
  if (n_tok == 0 || n_seq == 0 || blocks > kMostCutBlocks || keys <= least_cut_keys(blocks)) return pl;
  pl.pieces = kPieces;
  pl.blocks = (int)blocks;
  pl.slot_rows = (int)(rows < lsa::kPromptRows ? rows : lsa::kPromptRows);
  const size_t slots = (size_t)pl.pieces + pl.blocks;
  pl.off_ml = lsa::round_up(slots * pl.slot_rows * d_v * 4, 256);
  pl.off_joins = pl.off_ml + lsa::round_up(slots * pl.slot_rows * 8, 256);
  pl.off_n = pl.off_joins + lsa::round_up((size_t)blocks * 32, 256);
  pl.total = pl.off_n + 256;
  return pl;
}

lsa_status set_plan(lsa::PromptGeom& g, const PromptPlan& pl, void* workspace, size_t ws_bytes) {
  if (pl.total == 0) return LSA_OK;
  LSA_REQUIRE(workspace != nullptr && aligned(workspace, 256), LSA_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  LSA_REQUIRE(ws_bytes >= pl.total, LSA_ERR_WORKSPACE, "workspace of %zu bytes < %zu needed", ws_bytes, pl.total);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  g.pieces = pl.pieces;
  g.blocks = pl.blocks;
  g.slot_rows = pl.slot_rows;
  g.part_o = reinterpret_cast<float*>(ws);
  g.part_ml = reinterpret_cast<float*>(ws + pl.off_ml);
  g.joins = reinterpret_cast<int4*>(ws + pl.off_joins);
  g.n_joins = reinterpret_cast<int32_t*>(ws + pl.off_n);
  return LSA_OK;
}

}  // namespace

extern "C" {

lsa_status lsa_cache_read(const lsa_cache_read_params* p, int64_t n_tok, int32_t n_seq, const void* k_cache, const float* k_scale,
                          const void* v_cache, const float* v_scale, const int32_t* cu, const int32_t* start,
                          const int32_t* page_table, int32_t max_pages, int32_t kv_page_size, int64_t n_phys, void* k_out,
                          void* v_out, void* stream) {
  g_err[0] = 0;
  LSA_REQUIRE(p != nullptr, LSA_ERR_INVALID_ARG, "params is NULL");
  LSA_REQUIRE(p->n_kv_heads >= 1 && p->n_kv_heads <= 4096, LSA_ERR_INVALID_ARG, "n_kv_heads=%d not in [1, 4096]", p->n_kv_heads);
  LSA_REQUIRE(p->d_k >= 16 && p->d_k <= 1024 && p->d_k % 16 == 0, LSA_ERR_UNSUPPORTED,
              "d_k=%d must be a multiple of 16 in [16, 1024]", p->d_k);
  LSA_REQUIRE(p->d_v >= 0 && p->d_v <= 1024 && p->d_v % 16 == 0, LSA_ERR_UNSUPPORTED,
              "d_v=%d must be a multiple of 16 in [0, 1024]", p->d_v);
  LSA_REQUIRE(p->key_dtype == LSA_KEY_BF16 || p->key_dtype == LSA_KEY_FP8_E4M3FN, LSA_ERR_INVALID_ARG, "key_dtype=%d unknown",
              p->key_dtype);
  LSA_REQUIRE(n_tok >= 0 && n_seq >= 0, LSA_ERR_INVALID_ARG, "n_tok=%lld / n_seq=%d < 0", (long long)n_tok, n_seq);
  if (n_tok == 0 || n_seq == 0) return LSA_OK;  // nothing to read or write
  LSA_REQUIRE(n_tok < (1LL << 28), LSA_ERR_UNSUPPORTED, "n_tok must be < 2^28 per call");
  const lsa_status s = check_pages(page_table, n_seq, max_pages, kv_page_size, n_phys, p->n_kv_heads);
  if (s != LSA_OK) return s;
  const bool fp8 = p->key_dtype == LSA_KEY_FP8_E4M3FN, values = p->d_v > 0;
  LSA_REQUIRE(k_cache && cu && k_out, LSA_ERR_INVALID_ARG, "k_cache, cu and k_out must be non-NULL");
  LSA_REQUIRE((v_cache != nullptr) == values && (v_out != nullptr) == values, LSA_ERR_INVALID_ARG,
              "v_cache and v_out must be given exactly when d_v > 0");
  LSA_REQUIRE((k_scale != nullptr) == fp8 && (v_scale != nullptr) == (fp8 && values), LSA_ERR_INVALID_ARG,
              "k_scale / v_scale must be given exactly for fp8 caches");
  LSA_REQUIRE(aligned(k_cache, 16) && aligned(v_cache, 16) && aligned(k_out, 16) && aligned(v_out, 16), LSA_ERR_INVALID_ARG,
              "k_cache, v_cache, k_out and v_out must be 16-byte aligned");
  LSA_REQUIRE(aligned(k_scale, 4) && aligned(v_scale, 4) && aligned(cu, 4) && aligned(start, 4) && aligned(page_table, 4),
              LSA_ERR_INVALID_ARG, "scales, cu, start and page_table must be 4-byte aligned");
  lsa::CacheReadGeom g{};
  g.k = k_cache;
  g.v = v_cache;
  g.k_scale = k_scale;
  g.v_scale = v_scale;
  g.cu = cu;
  g.start = start;
  g.page_table = page_table;
  g.k_out = static_cast<uint16_t*>(k_out);
  g.v_out = static_cast<uint16_t*>(v_out);
  g.n_tok = n_tok;
  g.n_phys = n_phys;
  g.n_seq = n_seq;
  g.Hkv = p->n_kv_heads;
  g.d_k = p->d_k;
  g.d_v = p->d_v;
  g.fp8 = fp8;
  g.max_pages = max_pages;
  g.P = kv_page_size;
  const hipError_t e = lsa::launch_cache_read(g, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "cache read");
  return LSA_OK;
}

size_t lsa_prefill_attn_workspace_size(const lsa_prefill_attn_params* p, int32_t n_seq, int64_t n_tok, int64_t n_kv) {
  if (check_prefill_params(p) != LSA_OK || check_tokens(n_seq, n_tok, p->n_heads, p->n_kv_heads) != LSA_OK || n_kv < 0 || n_kv >= (1LL << 31))
    return 0;
  return plan_prompt(n_seq, n_tok, p->n_heads, p->n_kv_heads, p->d_v, p->k_sink, p->k_swa, n_kv).total;
}

lsa_status lsa_prefill_attn(const lsa_prefill_attn_params* p, int32_t n_seq, int64_t n_tok, int64_t n_kv, const void* q,
                            int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int32_t* cu_q, const int32_t* cu_kv, void* out, float* lse, void* workspace, size_t ws_bytes,
                            void* stream) {
  g_err[0] = 0;
  lsa_status s = check_prefill_params(p);
  if (s != LSA_OK) return s;
  s = check_tokens(n_seq, n_tok, p->n_heads, p->n_kv_heads);
  if (s != LSA_OK) return s;
  LSA_REQUIRE(n_kv >= 0, LSA_ERR_INVALID_ARG, "n_kv=%lld < 0", (long long)n_kv);
  LSA_REQUIRE(n_kv < (1LL << 31), LSA_ERR_UNSUPPORTED, "n_kv must be < 2^31");
  if (n_tok == 0 || n_seq == 0) return LSA_OK;  // nothing to read or write
  LSA_REQUIRE(cu_q && out, LSA_ERR_INVALID_ARG, "cu_q and out must be non-NULL");
  LSA_REQUIRE(cu_kv != nullptr || n_kv == n_tok, LSA_ERR_INVALID_ARG, "without cu_kv the keys are the tokens': n_kv must be n_tok");
  s = check_rows("q", q, q_stride, p->n_heads, p->d_qk);
  if (s == LSA_OK && n_kv > 0) s = check_rows("k", k, k_stride, p->n_kv_heads, p->d_qk);
  if (s == LSA_OK && n_kv > 0) s = check_rows("v", v, v_stride, p->n_kv_heads, p->d_v);
  if (s != LSA_OK) return s;
  LSA_REQUIRE(aligned(out, 16) && aligned(cu_q, 4) && aligned(cu_kv, 4) && aligned(lse, 4), LSA_ERR_INVALID_ARG,
              "out must be 16-byte aligned, cu_q, cu_kv and lse 4-byte");
  lsa::PromptGeom g{};
  g.q = static_cast<const uint16_t*>(q);
  g.k = k;
  g.v = v;
  g.q_stride = q_stride;
  g.k_stride = k_stride;
  g.v_stride = v_stride;
  g.cu_q = cu_q;
  g.cu_kv = cu_kv ? cu_kv : cu_q;
  g.out = static_cast<uint16_t*>(out);
  g.lse = lse;
  g.n_kv = (int)n_kv;
  g.causal = p->causal;
  set_heads(g, n_seq, n_tok, p->n_heads, p->n_kv_heads, p->d_qk, p->d_v, p->k_sink, p->k_swa, n_kv, p->sm_scale);
  s = set_plan(g, plan_prompt(n_seq, n_tok, p->n_heads, p->n_kv_heads, p->d_v, p->k_sink, p->k_swa, n_kv), workspace, ws_bytes);
  if (s != LSA_OK) return s;
  const hipError_t e = lsa::launch_prompt_attn(g, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "prefill attention");
  return LSA_OK;
}

size_t lsa_chunk_attn_workspace_size(const lsa_decode_attn_params* p, int32_t n_seq, int64_t n_tok, int32_t max_pages,
                                     int32_t kv_page_size) {
  if (check_chunk_params(p) != LSA_OK || check_tokens(n_seq, n_tok, p->n_heads, p->n_kv_heads) != LSA_OK || max_pages < 1 || kv_page_size < 1)
    return 0;
  return plan_prompt(n_seq, n_tok, p->n_heads, p->n_kv_heads, p->d_v, p->k_sink, p->k_swa, (int64_t)max_pages * kv_page_size).total;
}

lsa_status lsa_chunk_attn(const lsa_decode_attn_params* p, int32_t n_seq, int64_t n_tok, const void* q, const void* k_cache,
                          const float* k_scale, const void* v_cache, const float* v_scale, const int32_t* cu_q,
                          const int32_t* ctx_len, const int32_t* page_table, int32_t max_pages, int32_t kv_page_size,
                          int64_t n_phys, void* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  lsa_status s = check_chunk_params(p);
  if (s != LSA_OK) return s;
  s = check_tokens(n_seq, n_tok, p->n_heads, p->n_kv_heads);
  if (s != LSA_OK) return s;
  if (n_tok == 0 || n_seq == 0) return LSA_OK;  // nothing to read or write
  s = check_pages(page_table, n_seq, max_pages, kv_page_size, n_phys, p->n_kv_heads);
  if (s != LSA_OK) return s;
  const bool fp8 = p->key_dtype == LSA_KEY_FP8_E4M3FN;
  LSA_REQUIRE(q && k_cache && v_cache && cu_q && ctx_len && out, LSA_ERR_INVALID_ARG,
              "q, k_cache, v_cache, cu_q, ctx_len and out must be non-NULL");
  LSA_REQUIRE(fp8 == (k_scale != nullptr) && fp8 == (v_scale != nullptr), LSA_ERR_INVALID_ARG,
              "k_scale and v_scale must be given exactly for fp8 caches");
  LSA_REQUIRE(aligned(q, 16) && aligned(k_cache, 16) && aligned(v_cache, 16) && aligned(out, 16), LSA_ERR_INVALID_ARG,
              "q, k_cache, v_cache and out must be 16-byte aligned");
  LSA_REQUIRE(aligned(k_scale, 4) && aligned(v_scale, 4) && aligned(cu_q, 4) && aligned(ctx_len, 4) && aligned(page_table, 4) && aligned(lse, 4),
              LSA_ERR_INVALID_ARG, "scales, cu_q, ctx_len, page_table and lse must be 4-byte aligned");
  lsa::PromptGeom g{};
  g.q = static_cast<const uint16_t*>(q);
  g.q_stride = (int64_t)p->n_heads * p->d_qk;
  g.k = k_cache;
  g.v = v_cache;
  g.k_scale = k_scale;
  g.v_scale = v_scale;
  g.cu_q = cu_q;
  g.ctx_len = ctx_len;
  g.page_table = page_table;
  g.out = static_cast<uint16_t*>(out);
  g.lse = lse;
  g.n_phys = n_phys;
  g.fp8 = fp8;
  g.causal = 1;
  g.max_pages = max_pages;
  g.P = kv_page_size;
  g.cap = max_pages * kv_page_size;
  g.by_page = lsa::fast_div((uint32_t)kv_page_size);
  const int64_t pass = (int64_t)(lsa::kPromptPages - 2) * kv_page_size / lsa::kPromptKeys;  // (two pages more at the ends)
  g.pass_tiles = (int)(pass < (1 << 26) ? pass : (1 << 26));
  set_heads(g, n_seq, n_tok, p->n_heads, p->n_kv_heads, p->d_qk, p->d_v, p->k_sink, p->k_swa, g.cap, p->sm_scale);
  s = set_plan(g, plan_prompt(n_seq, n_tok, p->n_heads, p->n_kv_heads, p->d_v, p->k_sink, p->k_swa, g.cap), workspace, ws_bytes);
  if (s != LSA_OK) return s;
  const hipError_t e = lsa::launch_prompt_attn(g, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "chunk attention");
  return LSA_OK;
}

}  // extern "C"
