// Internal interface between the C-ABI front end (lsa_api.cpp) and the HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

namespace lsa {

// Everything the indexer kernels need to know about one call, passed by value.
struct IndexGeom {
  int H, D, fp8;                 // indexer heads, head dim, fp8 keys
  int P, B, M;                   // page, sub-block, kept pages (M <= 0: flat)
  int minmax;                    // coarse stage: min-max pooling (block keys [k_max | k_min])
  int k_sparse, k_sink, k_swa, C;
  int page_subs, tile_pages;     // coarse stage: sub-blocks per page, whole pages in a tile of 32 block keys
  int sub_recip;                 // ceil(2^16 / page_subs): (j * sub_recip) >> 16 = j / page_subs for j < 32
  int64_t q_start;               // prefill: position of row 0
  int64_t n_kv;                  // prefill: cached tokens
  int64_t n_sub;                 // mean keys available
  const int32_t* ctx_len;        // decode: [rows] (nullptr for prefill)
  const int32_t* page_table;     // decode: [rows, max_pages]
  int max_pages, kv_page;
  int64_t n_phys;
};

// Block cache of the coarse stage: mean keys [n_sub, D] or min-max extrema [n_sub, 2D]. rows == nullptr:
// every sub-block 0..n_items-1; otherwise the sub-blocks holding token rows[0..n_items).
hipError_t launch_block_keys(int64_t n_items, const int64_t* rows, int64_t n_tok, int D, int B, bool fp8, bool minmax,
                             const void* k, const float* ks, uint16_t* out, hipStream_t st);
hipError_t launch_coarse(const IndexGeom& g, int64_t n_rows, const uint16_t* q, const float* w, const uint16_t* kmean,
                         uint32_t* page_keys, int64_t ld, int64_t max_tiles, hipStream_t st);
// Page selection; with phys != nullptr (paged decode) it also writes each recalled page's physical
// page to phys[row * ld + k], which may alias page_keys (the row's keys are read first).
hipError_t launch_page_select(const IndexGeom& g, int64_t n_rows, const uint32_t* page_keys, int64_t ld,
                              int32_t* pages, int32_t* phys, int64_t max_elig, hipStream_t st);
// Dynamic LDS bytes of the page selection over rows of up to max_elig eligible pages.
inline size_t page_select_lds_bytes(int64_t max_elig, bool with_phys) {
  return (size_t)(max_elig > 0 ? max_elig : 1) * (with_phys ? 8 : 4);
}
// Fine scoring; paged decode reads the recalled pages' physical pages from phys (row stride ldp)
// as the page selection wrote them (nullptr in flat mode: looked up in the page table).
hipError_t launch_fine(const IndexGeom& g, int64_t n_rows, const uint16_t* q, const float* w, const void* k,
                       const float* ks, const int32_t* pages, const int32_t* phys, int64_t ldp, uint32_t* fine_keys,
                       int64_t ldf, int64_t max_sel, hipStream_t st);
// Dynamic LDS bytes of the token selection; rows of up to kSelectRegMax candidates keep their keys
// in registers (20 KB of static LDS), larger ones stage them in LDS (4 KB of static LDS).
constexpr int64_t kSelectRegMax = 512 * 64;
// Calls with at most this many rows (decode batches) select tokens (rows of 1025 to 8192 candidates) and
// pages with more threads per row: with few rows the GPU is mostly idle and per-row latency counts.
constexpr int64_t kSelectFewRows = 1024;
size_t token_select_lds_bytes(int64_t slots_cap, int k_cap, int M);
inline size_t token_select_static_lds(int64_t slots_cap) { return slots_cap <= kSelectRegMax ? 20 * 1024 : 4 * 1024; }
hipError_t launch_token_select(const IndexGeom& g, int64_t n_rows, const uint32_t* fine_keys, int64_t ldf,
                               const int32_t* pages, int32_t* idx, int32_t* count, int32_t* runs, int32_t* run_count,
                               int64_t slots_cap, hipStream_t st);
hipError_t prepare_index_kernels();
// p[0..n) = v (a kernel, so that the call also records correctly inside a captured graph).
hipError_t launch_fill_i32(int32_t* p, int64_t n, int32_t v, hipStream_t st);
// Run encoding -> position list: idx[r, 0..count[r]) from runs[r, 0..run_count[r]) (int32 pairs).
hipError_t launch_expand_runs(const int32_t* runs, const int32_t* run_count, int64_t n_rows, int k_cap, int32_t* idx,
                              int32_t* count, hipStream_t st);

// Sparse attention over gathered rows.
struct AttnGeom {
  const uint16_t* q;       // [n_rows, H, d_qk]
  const uint16_t* kv;      // latent [n_kv_rows, d_qk] or K
  const uint16_t* v;       // V [n_kv_rows, d_v] or nullptr
  int64_t n_kv_rows;
  const int32_t* rows;     // [n_rows, k_cap] cache rows to attend (positions, or translated rows)
  const int32_t* count;    // [n_rows]
  int k_cap;
  uint16_t* out;           // [n_rows, H, d_v]
  float* lse;              // [n_rows, H] or nullptr
  uint16_t* part_o;        // split partials, each normalised by its own sum, bf16 [n_rows - n_whole, n_split, H, d_v]
  float* part_f32;         // the same in fp32 (then part_o is unused), or nullptr
  float* part_ml;          // [n_rows - n_whole, n_split, H, 2]
  int64_t n_rows;
  int64_t n_whole;         // with n_split > 1: the last rows, taken whole; the earlier ones are cut into pieces
  int n_split;             // pieces per row, of whole tiles (some without any where the list is short)
  int short_tiles;         // lists of at most that many 32-entry tiles are not cut
  float scale_log2;        // sm_scale * log2(e)
  // Windowed lists (MLA list form; k_swa < 0: plain lists): row r's list is its entries before the
  // window and then the contiguous positions [t - w + 1, t], t = q_pos0 + r, w = min(k_swa, t + 1).
  int k_swa;
  int64_t q_pos0;
  // Run form of the lists (MLA only; nullptr = use rows/count): row r's list is the concatenation
  // of the runs (start, length) runs[r, 0..run_count[r]), int32 pairs with row stride k_cap.
  const int32_t* runs;
  const int32_t* run_count;
  // Paged cache (list form; nullptr = rows are cache rows): rows holds positions, and position
  // s of query row r is cache row page_table[(r / rows_per_seq) * max_pages + s / kv_page] *
  // kv_page + s % kv_page, translated while the list is staged.
  const int32_t* page_table;
  int max_pages, kv_page, rows_per_seq;
};

hipError_t launch_mla_attn(const AttnGeom& a, hipStream_t st);
hipError_t launch_mqa_attn(const AttnGeom& a, hipStream_t st);
hipError_t launch_attn_combine(const AttnGeom& a, hipStream_t st);  // MLA: 64 heads x 512

// Exact division of 0 <= n < 2^31 by d >= 1: n / d = (n * mul) >> shift with mul = floor(2^shift / d) + 1,
// shift = 31 + ceil(log2 d), so that the error n (mul d - 2^shift) / (d 2^shift) stays below 1 / d.
struct FastDiv {
  uint32_t d, shift;
  uint64_t mul;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while (l < 32 && (uint64_t(1) << l) < d) ++l;
  const uint32_t shift = 31 + l;
  return FastDiv{d, shift, (uint64_t(1) << shift) / d + 1};
}
__host__ __device__ inline int fdiv(const FastDiv& f, int n) { return (int)(((uint64_t)(uint32_t)n * f.mul) >> f.shift); }

// Launches a kernel and returns the status of this launch. (hipGetLastError would also return, and clear, an error that an
// earlier call of the thread left, when the kernel has been enqueued all the same.)
template <class... A>
inline hipError_t launch_kernel(void (*kernel)(A...), dim3 grid, dim3 block, hipStream_t st, A... args) {
  void* at[] = {&args...};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, 0, st);
  if (e != hipSuccess) (void)hipGetLastError();  // reported by the call, not by the thread's next check
  return e;
}

// One cache append (lsa_append_tensors and lsa_append_norm, checked).
struct AppendGeom {
  const uint16_t *q, *q_rot, *k, *k_rot, *v;
  const uint16_t *q_weight, *k_weight;  // of normed heads, or nullptr
  uint16_t* k_out;                      // the keys beside the cache, or nullptr
  float eps;
  int64_t q_stride, q_rot_stride, k_stride, k_rot_stride, v_stride;
  const float* rope;
  int64_t rope_rows;
  const int32_t *seq, *pos, *ctx_len, *page_table;
  uint16_t* q_out;
  void *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int64_t* rows;
  int64_t n_phys;
  int n_tok;
  int H, Hkv, d_k, d_v, rot_start, rot_dim, interleaved, fp8;
  int n_seq, max_pages, P;
  FastDiv by_rows;  // division by rows_per_seq
  // set by the launcher: first token of the launch (seq, pos, ctx_len and rows are indexed from the call's first), and
  // divisions by the threads of a head, the heads of a token and P
  int tok0;
  FastDiv by_q_units, by_q_heads, by_kv_heads, by_k_lanes, by_v_lanes, by_page;
};
hipError_t launch_append(const AppendGeom& g, hipStream_t st);

// One read of a paged cache (lsa_cache_read, checked).
struct CacheReadGeom {
  const void *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *cu, *start, *page_table;
  uint16_t *k_out, *v_out;
  int64_t n_tok, n_phys;
  int n_seq, Hkv, d_k, d_v, fp8, max_pages, P;
  // set by the launcher: rows of a workgroup, and divisions by the 16-value units of a token and of a head, and by P
  int tokens;
  FastDiv by_units, by_k_units, by_v_units, by_page;
};
hipError_t launch_cache_read(const CacheReadGeom& g, hipStream_t st);

// One call of the attention of prompts or chunks (lsa_prefill_attn, lsa_chunk_attn, checked).
struct PromptGeom {
  const uint16_t* q;  // [n_tok, H, d_qk], tokens q_stride apart
  const void *k, *v;  // packed rows [n_kv, Hkv, d], k_stride / v_stride apart, or (with ctx_len) caches [n_phys, Hkv, P, d]
  int64_t q_stride, k_stride, v_stride;
  const float *k_scale, *v_scale;
  const int32_t *cu_q, *cu_kv, *ctx_len, *page_table;
  uint16_t* out;
  float* lse;  // or nullptr
  int64_t n_phys;
  int n_tok, n_kv, n_seq, H, Hkv, d_qk, d_v, fp8, causal;
  int max_pages, P, cap;
  int k_sink, k_swa;  // both below the most keys of a sequence, or 0
  float scale_log2;   // sm_scale * log2(e)
  FastDiv by_group, by_page;
  int pass_tiles;     // tiles whose page-table entries fit the LDS area
  int head_classes;   // greatest common divisor of Hkv and 8 (the XCDs)
  int64_t items;      // workgroups of all blocks of kPromptRows query rows, at most
  int first;          // set by the launcher: first item of the launch
  // Calls whose blocks' keys are cut into pieces (pieces > 0; about so many, and at most blocks more):
  int pieces, blocks;          // blocks of kPromptRows query rows of all heads, at most
  int slot_rows;               // rows of a piece's partial results
  float *part_o, *part_ml;     // [pieces + blocks, slot_rows, d_v] unnormalised, [.., 2] maximum and sum
  int4* joins;                 // [blocks, 2]: pieces, slot of the first (of the others Hkv apart), head, row0; rows, first token
  int32_t* n_joins;
};
constexpr int kPromptRows = 256, kPromptKeys = 64, kPromptPages = 2048;
hipError_t launch_prompt_attn(const PromptGeom& g, hipStream_t st);

// One call of the attention over the whole cache (lsa_decode_attn, checked).
struct DecodeGeom {
  const uint16_t* q;  // [n_seq * R, H, d_qk]
  const void *k, *v;  // [n_phys, Hkv, P, d]; v unused with a latent cache
  const float *k_scale, *v_scale;
  const int32_t *ctx_len, *page_table;
  uint16_t* out;
  float* lse;  // or nullptr
  int64_t n_phys;
  int n_seq, R, H, Hkv, d_qk, d_v, latent, fp8;
  int max_pages, P;
  int k_sink, k_swa;  // both below cap, or 0
  float scale_log2;   // sm_scale * log2(e)
  // the plan
  int cap;            // positions a sequence can have: max_pages * P
  FastDiv by_page;    // division by P
  int whole_tiles;    // no tile lies in two pages (P is a multiple of the tile)
  int pass_tiles;     // tiles whose page-table entries fit the LDS area
  int block_cols;     // query rows of one key/value head that a workgroup takes together
  FastDiv by_group;   // division by H / Hkv
  FastDiv by_blocks;  // by the blocks of block_cols of a head's query rows
  int M;              // such blocks of a sequence (of all heads)
  int first;          // set by the launcher: first workgroup of the launch, a large call takes several (read first, with M)
  FastDiv by_m;       // by M
  int grid;           // workgroups
  FastDiv by_stretches;  // division by the stretches the tiles are dealt in (grid = stretches * M)
  FastDiv by_seqs;    // by n_seq
  int together;       // the M workgroups of a stretch on one XCD (stretches are a multiple of 8)
  int waves;          // of a workgroup (grouped heads)
  int min_tiles;      // fewest tiles of a workgroup (see least_tiles)
  float *part_o, *part_ml;  // two partials per workgroup: [block_cols, d_v], [block_cols, 2]; nullptr: none is cut
  int4* parts;        // [n_seq, M]: first and last stretch of each, slot of the first one's partial, r
};
// Tiles that pay for a workgroup in a call of `total` tiles: n workgroups take total / n tiles each and leave n partials
// to be written and joined, and the sum of both is least at n ~ sqrt(total). In steps of `step` (grouped heads: four
// waves). us at fixed tiles per workgroup: latent 1000 positions (32 tiles) 2 14.0, 4 15.1; 16K (512) 4 25.4, 6 23.9, 12 26.7; 64K
// (2048) 8 34.0, 12 32.5, 16 33.7; MQA 16K (512) 4 11.8, 8 11.9; 128K (4096) 8 21.7, 16 20.5.
__host__ __device__ inline int least_tiles(int64_t total, int step) {
  const int t = (int)(__builtin_sqrtf((float)total) * 0.25f + 0.5f);
  return t < step ? step : step == 4 ? t & -4 : t;
}
// Waves of the grouped-head kernel per SIMD: two where the registers of nb blocks of 16 query rows allow it; and
// workgroups of w waves per CU.
constexpr int gqa_waves_per_simd(int d, int nb, bool multi) { return nb <= 2 || (d == 64 && !multi) ? 2 : 1; }
constexpr int gqa_per_cu(int d, int nb, bool multi, int w) { return 4 * gqa_waves_per_simd(d, nb, multi) / w; }
hipError_t launch_decode_attn(const DecodeGeom& g, hipStream_t st);

}  // namespace lsa
