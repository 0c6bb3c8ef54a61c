// Reading a paged cache back into packed bf16 rows (lsa_cache_read) for gfx950.
//
// A workgroup takes a few neighbouring rows of the output: it finds their cache rows first (a search of the offsets, a
// page-table entry), then its threads copy 16 values at a time, of fp8 caches rounded from code * scale. One product per
// value: bound by HBM, and by the chain offsets, page, row where rows are few. 131072 latent rows of four sequences 60 us (302 MB, 5.05
// TB/s, what a copy reaches), 1001 rows of 8 heads in fp8 4.3 us.
#include "device.hpp"
#include "launch.hpp"

namespace lsa {

constexpr int kReadThreads = 256;
constexpr int kReadTokens = 64;  // rows of a workgroup, at most

template <bool FP8>
__global__ __launch_bounds__(kReadThreads) void cache_read_kernel(CacheReadGeom g) {
  __shared__ int64_t rows[kReadTokens];  // physical page * P + offset -> page * Hkv * P + offset; -1: zeros, -2: not written
  const int64_t t0 = (int64_t)blockIdx.x * g.tokens;
  const int n = g.n_tok - t0 < g.tokens ? (int)(g.n_tok - t0) : g.tokens;
  for (int t = (int)threadIdx.x; t < n; t += kReadThreads) {
    const int tok = (int)(t0 + t);
    int lo = 0, hi = g.n_seq;  // the last sequence that starts at or before the row
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (g.cu[mid] <= tok) lo = mid;
      else hi = mid;
    }
    const int first = g.cu[lo];
    int64_t row = -2;
    if (tok >= first && tok < g.cu[lo + 1]) {
      const int64_t pos = (int64_t)(g.start ? g.start[lo] : 0) + tok - first;
      row = -1;
      if (pos >= 0 && pos < (int64_t)g.max_pages * g.P) {
        const int pg = fdiv(g.by_page, (int)pos);
        const int64_t page = g.page_table ? g.page_table[(int64_t)lo * g.max_pages + pg] : lo;
        if (page >= 0 && page < g.n_phys) row = page * g.Hkv * g.P + ((int)pos - pg * g.P);
      }
    }
    rows[t] = row;
  }
  __syncthreads();
  const int per_token = (int)g.by_units.d, k_units = g.Hkv * (g.d_k / 16);
  for (int i = (int)threadIdx.x; i < n * per_token; i += kReadThreads) {
    const int t = fdiv(g.by_units, i);
    int u = i - t * per_token;
    const bool key = u < k_units;
    if (!key) u -= k_units;
    const int64_t row = rows[t];
    if (row == -2) continue;
    const int head = fdiv(key ? g.by_k_units : g.by_v_units, u), d = key ? g.d_k : g.d_v, at = 16 * (u - head * (d / 16));
    u32x4 lo{}, hi{};
    if (row >= 0) {
      const int64_t r = row + (int64_t)head * g.P;
      if constexpr (FP8) {
        const float scale = (key ? g.k_scale : g.v_scale)[r];
        const u32x4 c = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(key ? g.k : g.v) + r * d + at);
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[j], true);
          y[2 * j] = pack_bf16x2(a[0] * scale, a[1] * scale);
          y[2 * j + 1] = pack_bf16x2(b[0] * scale, b[1] * scale);
        }
        lo = u32x4{y[0], y[1], y[2], y[3]};
        hi = u32x4{y[4], y[5], y[6], y[7]};
      } else {
        const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(key ? g.k : g.v) + r * d + at);
        lo = src[0];
        hi = src[1];
      }
    }
    uint16_t* out = (key ? g.k_out : g.v_out) + ((t0 + t) * g.Hkv + head) * d + at;
    reinterpret_cast<u32x4*>(out)[0] = lo;
    reinterpret_cast<u32x4*>(out)[1] = hi;
  }
}

hipError_t launch_cache_read(const CacheReadGeom& all, hipStream_t st) {
  CacheReadGeom g = all;
  const int64_t share = (g.n_tok + 2047) / 2048;  // rows of a workgroup where all are resident at once
  g.tokens = (int)(share < kReadTokens ? share : kReadTokens);
  g.by_units = fast_div((uint32_t)(g.Hkv * ((g.d_k + g.d_v) / 16)));
  g.by_k_units = fast_div((uint32_t)(g.d_k / 16));
  g.by_v_units = fast_div((uint32_t)(g.d_v ? g.d_v / 16 : 1));
  g.by_page = fast_div((uint32_t)g.P);
  const dim3 grid((unsigned)((g.n_tok + g.tokens - 1) / g.tokens));  // (n_tok < 2^28: fewer than 2^32 threads)
  return launch_kernel(g.fp8 ? cache_read_kernel<true> : cache_read_kernel<false>, grid, dim3(kReadThreads), st, g);
}

}  // namespace lsa
