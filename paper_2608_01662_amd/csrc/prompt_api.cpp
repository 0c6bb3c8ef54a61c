// C-ABI front end of the prompt side of serving: reading a paged cache back. Argument checks (host only, before any HIP
// call) and launches. See include/lsa.h.
#include "api_common.hpp"
#include "launch.hpp"

using lsa::aligned;
using lsa::fail;
using lsa::g_err;
using lsa::hip_fail;

namespace {

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

}  // extern "C"
