// Attention of new tokens over the whole of a paged cache (lsa_decode_attn) for gfx950.
//
// A call is bound by reading the cache once: 4 flops per byte with 32 query heads on 8 bf16 key heads, 121
// with 64 heads on an MLA latent row, where the card has about 250. So the work is dealt out by cache tiles, not by sequences: the
// tiles (32 positions of one key/value head) of all sequences stand in one line, sequence after sequence, and
// every workgroup takes an equal stretch of it, whatever the lengths are. A stretch that covers a (sequence,
// head) whole writes its output; the others leave a partial (running maximum, sum and unnormalised fp32
// accumulators of the online softmax) and a second kernel joins the partials. The lengths are on the device, so
// every workgroup finds its stretch by itself from the lengths.
#include "attn_tile.hpp"
#include "device.hpp"
#include "launch.hpp"

namespace lsa {

constexpr int kTile = 32;  // positions of a tile

// What loads of positions that nobody attends to read instead (behind the context, in unmapped pages): zeros,
// since a weight of zero does not silence a NaN or an infinity in V.
__device__ __attribute__((aligned(256))) const uint8_t zero_row[1152] = {};

// The tiles of a sequence that any of its new tokens attends to: 0 .. ns - 1 (the sink) and then ns + skip ..
struct Span {
  int c;         // cached positions, 0 where the length is out of range
  int lo;        // first position of the window of the first new token
  int ns, skip;  // tile i of the span is tile i of the sequence, from ns on tile i + skip
  int nt;        // tiles in all
};
__device__ __forceinline__ Span span_of(const DecodeGeom& g, int ctx) {
  Span s;
  s.c = ctx < 0 || ctx > g.cap ? 0 : ctx;
  const int t1 = s.c - g.R + 1;  // (first new token) + 1
  s.lo = g.k_swa > 0 && t1 > g.k_swa ? t1 - g.k_swa : 0;
  const int sink = g.k_sink < s.c ? g.k_sink : s.c, total = (int)(((uint32_t)s.c + kTile - 1) / kTile);
  const int st = (int)(((uint32_t)sink + kTile - 1) / kTile), first = s.lo / kTile;
  s.ns = first <= st ? total : st;
  s.skip = first <= st ? 0 : first - st;
  s.nt = total - s.skip;
  return s;
}

// (a wave-uniform value that the compiler cannot know to be: kept in a scalar register)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// 2^(s scale - m), the product rounded as where the maximum m was taken: one rounding for both (an fma) leaves the largest
// score's exponent at m's rounding error, which overflows from scores of 2^31 on.
__device__ __forceinline__ float exp2_below(float s, float scale, float m) {
#pragma clang fp contract(off)
  const float z = s * scale;
  return fast_exp2(z - m);
}

// Values over the sum of their weights, 0 where there are none or all are 0 (every score -inf). Selected, since 0 times what a
// value of a weight of 0 left (a NaN or an infinity times 0) is NaN.
__device__ __forceinline__ f32x4 average(f32x4 acc, float sum) {
  const float inv = 1.f / sum;
  f32x4 y;
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = sum == 0.f ? 0.f : acc[k] * inv;
  return y;
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8: within rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15: rows 0 and 2 into 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31: row 1 into 2 and 3
  return x;
}

// The rows of a sequence that attend to nothing (d: width of an output row).
__device__ __forceinline__ void empty_rows(const DecodeGeom& g, int b, int d) {
  const int64_t n = (int64_t)g.R * g.H * d;
  for (int64_t i = 8 * (int64_t)threadIdx.x; i < n; i += 8 * (int64_t)blockDim.x) *reinterpret_cast<u32x4*>(g.out + b * n + i) = u32x4{};
  if (g.lse)
    for (int i = (int)threadIdx.x; i < g.R * g.H; i += (int)blockDim.x) g.lse[(int64_t)b * g.R * g.H + i] = -INFINITY;
}

// Deals this workgroup its work. The tiles of all sequences (of one head) stand in one line, and workgroup (y, r) takes
// stretch y of it, an equal share of all, but no fewer tiles than pay for a workgroup, for r, one of the g.M (head, query row
// block)s of every sequence; the g.M of a stretch are neighbours in the launch, so that what they share is read at one time. Calls
// segment(sequence, r, span, first tile, last tile + 1, whole, slot of the partial), and tells the join about every
// (sequence, r) whose first tile is here. Then the rows of sequences without a tile, dealt to the workgroups. d: width of an output
// row. (Tiles of all in all fit 30 bits: the host refuses more.)
//
// What precedes the first load of a row is a chain of round trips, so the first 64 lengths are loaded once and
// scanned in registers, and divisions by what the host knows are products.
template <class F>
__device__ __forceinline__ void deal(const DecodeGeom& g, int d, F&& segment) {
  const int M = g.M, lane = threadIdx.x & 63;
  const bool cut = g.parts != nullptr;
  // (together: workgroups i, i + 8, .. run on one XCD, whose L2 then reads the rows that the g.M share once. A call that is cut
  // has few workgroups, all of one launch.)
  const int q = g.together ? (int)blockIdx.x >> 3 : g.first + (int)blockIdx.x, yq = fdiv(g.by_m, q), r = q - yq * M;
  const int y = g.together ? 8 * yq + ((int)blockIdx.x & 7) : yq;
  auto length = [&](int b) { return b < g.n_seq ? g.ctx_len[b] : 0; };
  int ctx0 = 0, share = 0;
  int at = 0, end = 0, b = 0, before = 0;  // tiles [at, end), the sequence of `at`, the tiles before that sequence
  if (!cut) {  // a workgroup per (sequence, r); `before` counts from its own sequence
    b = y;
    ctx0 = uniform(g.ctx_len[b]);
    end = span_of(g, ctx0).nt;
  } else {
    ctx0 = length(lane);
    const int inc0 = wave_scan(span_of(g, ctx0).nt);
    int total = __builtin_amdgcn_readlane(inc0, 63);
    for (int b0 = 64; b0 < g.n_seq; b0 += 64) total += __builtin_amdgcn_readlane(wave_scan(span_of(g, length(b0 + lane)).nt), 63);
    share = fdiv(g.by_stretches, total + (int)g.by_stretches.d - 1);
    int least = least_tiles(total * M, g.min_tiles);
    // (where workgroups are idle, one of fewer tiles rather than one for several short sequences)
    const int mean = fdiv(g.by_seqs, total + g.n_seq - 1);
    least = mean < least ? mean : least;
    share = share < least ? least : share;
    const int64_t first = (int64_t)y * share;
    if (first < total) {
      at = (int)first;
      end = total - at < share ? total : at + share;
      for (int inc = inc0, ctx = ctx0;;) {
        const uint64_t past = __ballot(before + inc > at);
        if (past) {
          const int i = __ffsll((unsigned long long)past) - 1;
          before += __builtin_amdgcn_readlane(inc, i) - span_of(g, __builtin_amdgcn_readlane(ctx, i)).nt;
          b += i;
          break;
        }
        before += __builtin_amdgcn_readlane(inc, 63);
        b += 64;
        ctx = length(b + lane);
        inc = wave_scan(span_of(g, ctx).nt);
      }
    }
  }
  const int start = at;
  while (at < end) {
    const Span sp = span_of(g, !cut ? ctx0 : b < 64 ? __builtin_amdgcn_readlane(ctx0, b) : uniform(g.ctx_len[b]));
    if (sp.nt == 0) {
      ++b;
      continue;
    }
    const int t0 = uniform(at - before), n = uniform(end - at < sp.nt - t0 ? end - at : sp.nt - t0);
    const int slot = 2 * (y * M + r) + (at != start);
    segment(b, r, sp, t0, t0 + n, n == sp.nt, slot);
    if (t0 == 0 && cut && threadIdx.x == 0)  // first stretch and last one, and the first one's partial
      g.parts[(int64_t)b * M + r] = int4{y, (int)((uint32_t)(at + sp.nt - 1) / (uint32_t)share), slot, r};
    at += n;
    if (t0 + n == sp.nt) {
      before += sp.nt;
      ++b;
    }
  }
  // sequences without a tile
  if (!cut) {
    if (end == 0 && r == 0) empty_rows(g, b, d);
    return;
  }
  for (int e = blockIdx.x; e < g.n_seq; e += g.grid) {
    if (span_of(g, g.ctx_len[e]).nt != 0) continue;
    empty_rows(g, e, d);
    for (int i = (int)threadIdx.x; i < M; i += (int)blockDim.x) g.parts[(int64_t)e * M + i] = int4{0, 0, 0, 0};
  }
}

// ---------------------------------------------------------------- direct global -> LDS loads
// 16 (4) bytes per lane from `src` to LDS bytes lds + 16 (4) lane. The compiler does not see these loads, so
// that it does not drain them before every LDS read; callers wait with explicit vmcnt counts. M0 holds the LDS
// address and is restored; the s_nop is the wait state before a load may read it.
__device__ __forceinline__ void lds_dma16(const uint8_t* src, uint32_t lds) {
  uint32_t save;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
               : "=&s"(save) : "v"(src), "s"(lds) : "memory");
}
// N <= 4 KB of neighbouring cache rows from `base`: load j takes base + 1024 j + off[j] per lane to LDS bytes lds + 1024 j +
// 16 lane. (The immediate offset counts for both addresses.)
template <int N>
__device__ __forceinline__ void lds_dma16_rows(const uint8_t* base, uint32_t off, uint32_t x1, uint32_t x2, uint32_t x3, uint32_t lds) {
  uint32_t save;
  if constexpr (N == 4)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:2048\n\tglobal_load_lds_dwordx4 %5, %1 offset:3072\n\ts_mov_b32 m0, %0"
                 : "=&s"(save) : "s"(base), "v"(off), "v"(off ^ x1), "v"(off ^ x2), "v"(off ^ x3), "s"(lds) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\ts_mov_b32 m0, %0"
                 : "=&s"(save) : "s"(base), "v"(off), "v"(off ^ x1), "s"(lds) : "memory");
}
__device__ __forceinline__ void lds_dma4(const uint8_t* src, uint32_t lds) {
  uint32_t save;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
               : "=&s"(save) : "v"(src), "s"(lds) : "memory");
}

// eight e4m3 codes -> eight bf16 (exact)
__device__ __forceinline__ u32x4 fp8x8_bf16(uint32_t lo, uint32_t hi) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
}
typedef __attribute__((ext_vector_type(2))) int i32x2;
// Transposed read of 8-bit values: in a 16-lane group, source lane s supplies 8 bytes of row s / 2 (columns
// 8 (s % 2) ..), and lane i receives column i of the 8 rows.
__device__ __forceinline__ u32x2 tr8(const uint8_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(p)));
}

// ============================================================================ grouped heads, 64 or 128 wide
// One workgroup = W waves that share no tiles: wave w streams tiles w, w + W, .. of the stretch through a
// ring in LDS of its own, K and V apart, by direct loads of whole rows, and refills a tile's K as soon as it is
// scored and its V as soon as it is multiplied, so that most of its 16 KB (32 where registers leave one wave per
// SIMD) are on their way at any time, 128 KB per CU. (A step of the ring needs no barrier, only a count of the wave's own
// loads.) At the stretch's end the waves' results are merged through LDS.
//
// Bound by HBM: 64 sequences of up to 16K, 32 heads on 8 in bf16 (mean 2.1 GB) 372 us, 5.8 TB/s; 48 of 4K to 32K in fp8, two
// new tokens each (1.9 GB) 337 us, 5.5 TB/s; 33 windows of 1024, 12 heads of 64, pages of 20 (104 MB) 22 us; one
// sequence of 128K, 16 heads on one (67 MB) 21 us, of which the join 5; one of 1001, 32 on 8, 9.0 us, all latency. Two waves per
// SIMD hide one's softmax behind the other's products: one wave took 402 and 400 us in place of the first two's 356 and 306 at
// that time. 33 to 64 query rows per key head need the registers of one wave per SIMD: 64 heads on one, 64 x 16K (537 MB) 115 us, 4.7
// TB/s, but in fp8 97 us, 2.9 TB/s, bound by that wave's issue, as are chunks of new tokens (512 on 16 x 8K, 32 heads on 8, 2.9 ms, 374
// TFLOP/s), which walk the cache once per 64 query rows.
//
// The rows of the products are query rows: the heads of the group of all new tokens, in blocks of 16 (NB
// blocks per wave); S^T = K Q^T on 16x16x32 products with tokens on the rows, in an order that gives lane
// (g = lane / 16) the scores of tokens 8 g .. + 7 of its column, which is the layout of the B operand of
// O^T += V^T P^T: P never leaves the registers.
constexpr int kPageSlots = 2048;      // page-table entries staged in LDS at a time

template <int D, bool FP8, int NB, bool MULTI, int W>
struct GqaTile {
  static constexpr int kPerCu = gqa_per_cu(D, NB, MULTI, W);
  static constexpr int kRing = 128 * 1024 / (kPerCu * W);  // LDS ring bytes per wave
  static constexpr int kRow = D * (FP8 ? 1 : 2);          // bytes of a cache row
  static constexpr int kBytes = kTile * kRow;             // of a K or V tile
  static constexpr int kChunks = kRow / 16;               // 16-byte chunks of a row
  static constexpr int kLoads = kBytes / 1024;            // direct loads of a K or V tile
  static constexpr int kStages = kRing / (2 * kBytes); // tiles in the ring
  static constexpr int kK = kLoads + (FP8 ? 1 : 0);       // loads issued with K: its rows, and both scales
  static constexpr int kPair = kK + kLoads;
  // Chunk c of token t lies in 16-byte slot c ^ swz(t) of its row. The K reads (16 tokens of one chunk per 16
  // lanes) and the transposed V reads (per 32 lanes 8 or 16 tokens x 32 or 16 bytes) then fall on all
  // banks alike: with t = 16 a1 + 8 a0 + 4 b + 2 k1 + k0, a K read varies a1, a0, k1, k0, a V read of 32 lanes a0, k1, k0
  // (fp8: and b), and rows of less than 256 bytes spread by their own low token bits.
  static constexpr __host__ __device__ __forceinline__ int swz(int t) {
    const int a1 = (t >> 4) & 1, a0 = (t >> 3) & 1, b = (t >> 2) & 1;
    if constexpr (kChunks == 16) return a1 | (t & 3) << 1 | a0 << 3;
    if constexpr (kChunks == 8) return (a1 ^ b) | (t & 2) | a0 << 2;
    return a0 | (a1 ^ b) << 1;
  }
};

template <int D, bool FP8, int NB, bool MULTI, int W>  // MULTI: several new tokens per sequence; W waves
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(gqa_waves_per_simd(D, NB, MULTI), gqa_waves_per_simd(D, NB, MULTI))))
void gqa_decode_kernel(DecodeGeom g) {
  using T = GqaTile<D, FP8, NB, MULTI, W>;
  constexpr int NS = T::kStages, KS = D / 32, CD = D / 16, COLS = 16 * NB;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[W][T::kRing];
  __shared__ __attribute__((aligned(16))) float scales[FP8 ? W : 1][FP8 ? NS : 1][64];
  __shared__ int pages[kPageSlots];
  __shared__ uint32_t seen_bits[W][NS];  // of the tiles in the ring: tokens somebody attends to
  __shared__ float pm[W][COLS], pl[W][COLS];
  static_assert(COLS * D * 4 <= T::kRing, "the accumulators are merged in the ring");
  const int lane = threadIdx.x & 63, q4 = lane >> 4, i16 = lane & 15;
  const int wv = uniform((int)(threadIdx.x >> 6));
  uint8_t* const lk = ring[wv];                    // K tiles, then V tiles
  uint8_t* const lv = ring[wv] + NS * T::kBytes;
  const int group = (int)g.by_group.d, cols = g.R * group, cb_n = (int)g.by_blocks.d;  // query rows of a head, and their blocks

  // LDS offsets of this lane's operands: K of token block mt at chunk 4 s + q4, V of value block c
  int k_off[2], k_swz[2];
#pragma unroll
  for (int mt = 0; mt < 2; ++mt) {
    const int t = 8 * (i16 >> 2) + 4 * mt + (i16 & 3);
    k_off[mt] = t * T::kRow;
    k_swz[mt] = T::swz(t);
  }
  const int v_t0 = FP8 ? 8 * q4 + (i16 >> 1) : 8 * q4 + (i16 >> 2), v_t1 = v_t0 + 4;  // (bf16: rows of both reads)
  // direct load j: tokens j * 64 / chunks .., lane -> token lane / chunks of them, slot lane % chunks
  constexpr int LT = 64 / T::kChunks;  // tokens per load
  const int ld_t = lane / T::kChunks, ld_slot = lane % T::kChunks;

  // bits of the tokens t8 .. + 7 that a query at position t attends to
  auto sees8 = [&](int t8, int t) -> uint32_t {
    auto first = [](int n) { return (1u << (n < 0 ? 0 : n > 8 ? 8 : n)) - 1u; };  // the first n of them
    const uint32_t window = g.k_swa == 0 ? 0xFFu : ~first(t - g.k_swa + 1 - t8) | first(g.k_sink - t8);
    return first(t + 1 - t8) & window;
  };

  auto segment = [&](int b, int r, const Span& sp, int t0, int t1, bool whole, int slot) {
    const int kvh = fdiv(g.by_blocks, r), col0 = (r - kvh * cb_n) * COLS;
    const int ncols = cols - col0 < COLS ? cols - col0 : COLS;
    // ---- Q as the B operand: column 16 nb + i16 = (new token j, head of the group), dims of k-step s. (Columns past the
    // last query row repeat the first one's and are not stored.)
    u32x4 qb[NB][KS];
    int tcol[NB];  // position of the column's token
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int col = col0 + 16 * nb + i16;
      const bool ok = 16 * nb + i16 < ncols;
      const int j = fdiv(g.by_group, ok ? col : col0), hh = (ok ? col : col0) - j * group;
      tcol[nb] = sp.c - g.R + j;
      const uint8_t* qp = reinterpret_cast<const uint8_t*>(g.q + (((int64_t)b * g.R + j) * g.H + kvh * group + hh) * D);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        // bf16: chunk 4 s + q4 of the row; fp8: a 16-byte K chunk 4 (s / 2) + q4 holds the dims of two k-steps
        const int dim = FP8 ? 64 * (s >> 1) + 16 * q4 + 8 * (s & 1) : 32 * s + 8 * q4;
        qb[nb][s] = *reinterpret_cast<const u32x4*>(qp + 2 * dim);
      }
    }
    f32x4 o[NB][CD];
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb] = kNoRef;
      l[nb] = 0.f;
#pragma unroll
      for (int c = 0; c < CD; ++c) o[nb][c] = f32x4{};
    }
    for (int p0 = t0; p0 < t1; p0 += g.pass_tiles) {
      const int p1 = t1 - p0 < g.pass_tiles ? t1 : p0 + g.pass_tiles;
      // ---- page-table entries of tiles [p0, p1): those before the skipped ones, then the others
      const int e1 = p1 < sp.ns ? p1 : sp.ns, b2 = p0 > sp.ns ? p0 : sp.ns;
      int f1 = 0, n1 = 0, f2 = 0, n2 = 0;  // first page and pages of both parts
      if (p0 < e1) {
        f1 = fdiv(g.by_page, p0 * kTile);
        const int last = e1 <= (sp.c - 1) / kTile ? e1 * kTile - 1 : sp.c - 1;  // (e1 * kTile may be 2^31)
        n1 = fdiv(g.by_page, last) - f1 + 1;
      }
      if (b2 < p1) {
        f2 = fdiv(g.by_page, (b2 + sp.skip) * kTile);
        const int64_t end = (int64_t)(p1 + sp.skip) * kTile - 1;
        n2 = fdiv(g.by_page, end < sp.c ? (int)end : sp.c - 1) - f2 + 1;
      }
      for (int i = (int)threadIdx.x; i < n1 + n2; i += 64 * W) {
        const int pg = i < n1 ? f1 + i : f2 + i - n1;
        const int ph = g.page_table ? g.page_table[(int64_t)b * g.max_pages + pg] : b;
        pages[i] = ph >= 0 && ph < g.n_phys ? ph : -1;
      }
      // Q (and everything else on its way) has arrived before the first direct load: the compiler, which does
      // not know of those, would wait for all of them together with Q
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      const int nw = p1 - p0 > wv ? (p1 - p0 - wv + W - 1) / W : 0;  // this wave's tiles
      auto tile_pos = [&](int i) {
        const int t = p0 + wv + W * i;
        return (t < sp.ns ? t : t + sp.skip) * kTile;
      };
      // Where this wave's tile i lies: the cache row of token lane % 32, -1 where nobody attends to it (bits: the tokens
      // somebody attends to). A tile that lies whole in one page and is attended to whole needs its first row only.
      struct Where {
        int rows;
        uint32_t row0, bits;
      };
      auto locate = [&](int i) {
        Where w{-1, 0u, 0u};
        const int t = p0 + wv + W * i, s0 = tile_pos(i), s = s0 + (lane & 31);
        const bool seen = s < sp.c && (s >= sp.lo || s < g.k_sink);
        const int shift = t < sp.ns ? f1 : f2 - n1;
        if (g.whole_tiles) {
          const int pg = fdiv(g.by_page, s0), ph = uniform(pages[pg - shift]);
          w.row0 = ((uint32_t)ph * (uint32_t)g.Hkv + (uint32_t)kvh) * (uint32_t)g.P + (uint32_t)(s0 - pg * g.P);
          if (ph >= 0) {
            w.bits = (uint32_t)__ballot(seen);
            if (w.bits != ~0u) w.rows = seen ? (int)w.row0 + (lane & 31) : -1;
          }
          return w;
        }
        if (seen) {
          const int pg = fdiv(g.by_page, s), ph = pages[pg - shift];
          if (ph >= 0) w.rows = (int)(((uint32_t)ph * (uint32_t)g.Hkv + (uint32_t)kvh) * (uint32_t)g.P + (uint32_t)(s - pg * g.P));
        }
        w.bits = (uint32_t)__ballot(w.rows >= 0);
        return w;
      };
      auto issue = [&](const void* base, uint8_t* dst, const Where& w) {
        if (g.whole_tiles && w.bits == ~0u) {
          constexpr int N = T::kLoads < 4 ? T::kLoads : 4;
          // (swz(t + u) = swz(t) ^ swz(u) where the bits of t and u are apart)
          constexpr uint32_t x1 = T::swz(LT) * 16, x2 = T::swz(2 * LT) * 16, x3 = T::swz(3 * LT) * 16;
          const uint32_t off = (uint32_t)(ld_t * T::kRow + (ld_slot ^ T::swz(ld_t)) * 16);
          const uint8_t* src = static_cast<const uint8_t*>(base) + (int64_t)(uint32_t)uniform((int)w.row0) * T::kRow;
#pragma unroll
          for (int j = 0; j < T::kLoads; j += N) lds_dma16_rows<N>(src + j * 1024, off ^ (T::swz(j * LT) * 16), x1, x2, x3, lds_addr(dst + j * 1024));
          return;
        }
#pragma unroll
        for (int j = 0; j < T::kLoads; ++j) {
          const int t = j * LT + ld_t, row = __shfl(w.rows, t);
          const uint8_t* src = row >= 0 ? static_cast<const uint8_t*>(base) + (int64_t)row * T::kRow : zero_row;
          lds_dma16(src + (ld_slot ^ T::swz(t)) * 16, lds_addr(dst + j * 1024));
        }
      };
      auto issue_k = [&](int st, const Where& w) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage's last reads are done
        if constexpr (FP8) {
          const float* sc = lane < 32 ? g.k_scale : g.v_scale;
          const int row = g.whole_tiles && w.bits == ~0u ? (int)w.row0 + (lane & 31) : w.rows;
          lds_dma4(row >= 0 ? reinterpret_cast<const uint8_t*>(sc + row) : zero_row, lds_addr(scales[wv][st]));
        }
        issue(g.k, lk + st * T::kBytes, w);
      };
      auto issue_v = [&](int st, const Where& w) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        issue(g.v, lv + st * T::kBytes, w);
      };
      // (the stages are not unrolled: eight copies of the body passed the instruction cache)
#pragma nounroll
      for (int i = 0; i < NS && i < nw; ++i) {
        const Where w = locate(i);
        seen_bits[wv][i] = w.bits;
        issue_k(i, w);
        issue_v(i, w);
      }
      {
        int st = 0;
#pragma nounroll
        for (int i = 0; i < nw; ++i, st = st + 1 == NS ? 0 : st + 1) {
          const bool more = uniform(i + NS < nw);  // tile i + NS takes this one's place
          const uint32_t bits = (uint32_t)uniform((int)seen_bits[wv][st]);
          Where w{};
          if (more) w = locate(i + NS);
          // K of tile i has landed: behind it are its V and the other stages' tiles (fewer at the stretch's end)
          if (i + NS <= nw) vm_wait<T::kLoads + (NS - 1) * T::kPair>();
          else vm_wait<0>();
          // ---- S^T = K Q^T
          const uint8_t* kt = lk + st * T::kBytes;
          f32x4 s4[2][NB];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s4[mt][nb] = f32x4{};
            if constexpr (FP8) {
#pragma unroll
              for (int s = 0; s < KS; s += 2) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(kt + k_off[mt] + ((2 * s + q4) ^ k_swz[mt]) * 16);
                const u32x4 a = fp8x8_bf16(x.x, x.y), b = fp8x8_bf16(x.z, x.w);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                  s4[mt][nb] = mfma16(a, qb[nb][s], s4[mt][nb]);
                  s4[mt][nb] = mfma16(b, qb[nb][s + 1], s4[mt][nb]);
                }
              }
            } else {
#pragma unroll
              for (int s = 0; s < KS; ++s) {
                const u32x4 a = *reinterpret_cast<const u32x4*>(kt + k_off[mt] + ((4 * s + q4) ^ k_swz[mt]) * 16);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s4[mt][nb] = mfma16(a, qb[nb][s], s4[mt][nb]);
              }
            }
          }
          // scores of tokens 8 q4 .. + 7 of the columns, in units of log2
          float z[NB][8], vs[8];
          if constexpr (FP8) {
            const f32x4* sk = reinterpret_cast<const f32x4*>(&scales[wv][st][8 * q4]);
            const f32x4* sv = reinterpret_cast<const f32x4*>(&scales[wv][st][32 + 8 * q4]);
            const f32x4 a = sk[0], b = sk[1], c = sv[0], d = sv[1];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float ks = (k < 4 ? a[k & 3] : b[k & 3]) * g.scale_log2;
              vs[k] = k < 4 ? c[k & 3] : d[k & 3];
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) z[nb][k] = s4[k >> 2][nb][k & 3] * ks;
            }
          } else {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int k = 0; k < 8; ++k) z[nb][k] = s4[k >> 2][nb][k & 3] * g.scale_log2;
          }
          if (more) issue_k(st, w);
          const int s0 = tile_pos(i);
          // several new tokens: does the tile reach to where they see different positions?
          const bool uneven = MULTI && uniform((s0 > sp.c - g.R + 1 - kTile || (g.k_swa > 0 && s0 < sp.c - g.k_swa)));
          if (bits != ~0u || uneven) {
            const int t8 = s0 + 8 * q4;  // this lane's first token
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint32_t own = (bits >> (8 * q4)) & (uneven ? sees8(t8, tcol[nb]) : 0xFFu);
#pragma unroll
              for (int k = 0; k < 8; ++k) z[nb][k] = (own >> k) & 1u ? z[nb][k] : -INFINITY;
            }
          }
          // ---- online softmax; the reference maximum moves when it grows by more than 2^8
          u32x4 pb[NB];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float mx = z[nb][0];
#pragma unroll
            for (int k = 1; k < 8; ++k) mx = fmaxf(mx, z[nb][k]);
            mx = max4_xor16_32(mx);
            const bool need = mx > m[nb] + kLazy;
            if (__ballot(need)) {
              const float alpha = need ? fast_exp2(m[nb] - mx) : 1.f;
#pragma unroll
              for (int c = 0; c < CD; ++c) o[nb][c] *= alpha;
              l[nb] *= alpha;
              m[nb] = need ? mx : m[nb];
            }
            float p[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              p[k] = fast_exp2(z[nb][k] - m[nb]);  // -inf -> 0
              l[nb] += p[k];
              if constexpr (FP8) p[k] = z[nb][k] == -INFINITY ? 0.f : p[k] * vs[k];  // (masked: also from a NaN scale)
            }
            // The weights' one rounding, to the 8 significant bits that a matrix product with bf16 takes (V's codes and values are
            // exact there; an fp8 row's scale goes into the weight before it). The sum above takes them unrounded. Against 64 bits
            // the output is off by 2.2e-3 to 2.4e-3 of its norm, 1.7e-3 of which are its own rounding to bf16; weights in two bf16
            // terms would bring it to that, for twice the value products.
            pb[nb] = u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
          }
          // V of tile i has landed: behind it are the other stages' tiles and the K just requested
          if (more) vm_wait<(NS - 1) * T::kPair + T::kK>();
          else if (i + NS == nw) vm_wait<(NS - 1) * T::kPair>();
          else vm_wait<0>();
          // ---- O^T += V^T P^T
          const uint8_t* vt = lv + st * T::kBytes;
          auto value = [&](int c) {
            if constexpr (FP8) {
              const u32x2 x = tr8(vt + v_t0 * T::kRow + (c ^ T::swz(v_t0)) * 16 + (i16 & 1) * 8);
              return fp8x8_bf16(x.x, x.y);
            } else {
              const int ch = 2 * c + ((i16 >> 1) & 1), half = (i16 & 1) * 8;
              return tr16_pair(vt + v_t0 * T::kRow + (ch ^ T::swz(v_t0)) * 16 + half,
                               vt + v_t1 * T::kRow + (ch ^ T::swz(v_t1)) * 16 + half);
            }
          };
          bool apart = false;
          if (uneven) {  // (adding 1 to an exponent of ones carries into the sign bit)
            uint32_t odd = 0;
#pragma nounroll
            for (int c = 0; c < CD; ++c) {  // (unrolled, its operands would be held together and spill)
              const u32x4 a = value(c);
#pragma unroll
              for (int k = 0; k < 4; ++k) odd |= (a[k] & 0x7F807F80u) + 0x00800080u;
            }
            apart = uniform(__ballot((odd & 0x80008000u) != 0) != 0);
          }
          if (!apart) {
#pragma unroll
            for (int c = 0; c < CD; ++c) {
              const u32x4 a = value(c);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) o[nb][c] = mfma16(a, pb[nb], o[nb][c]);
            }
          } else {
            // A weight of zero does not silence a NaN or an infinity in a row of V that some of the columns see: one product
            // per new token, its unseen rows of V zeroed, taken by its own columns.
            for (int j = fdiv(g.by_group, col0); j <= fdiv(g.by_group, col0 + ncols - 1); ++j) {
              const int t = sp.c - g.R + j;
              const uint32_t own = sees8(s0 + 8 * q4, t);
              u32x4 keep;
#pragma unroll
              for (int k = 0; k < 4; ++k) keep[k] = ((own >> (2 * k)) & 1u ? 0xFFFFu : 0u) | ((own >> (2 * k + 1)) & 1u ? 0xFFFF0000u : 0u);
#pragma unroll
              for (int c = 0; c < CD; ++c) {
                const u32x4 a = value(c) & keep;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                  const f32x4 x = mfma16(a, pb[nb], f32x4{});
#pragma unroll
                  for (int k = 0; k < 4; ++k) o[nb][c][k] = tcol[nb] == t ? o[nb][c][k] + x[k] : o[nb][c][k];
                }
              }
            }
          }
          if (more) {
            seen_bits[wv][st] = w.bits;
            issue_v(st, w);
          }
        }
      }
      __syncthreads();  // every wave is done with `pages` and its ring
    }
    // ---- the waves' results, weighted by 2^(m_w - M) and summed. Column and dims 4 u .. lie in 16-byte slot u ^ column of the
    // column's row, so that 16 lanes of one u fall on all banks. (The lane is made opaque, or these offsets are computed
    // before the loop over stretches and spill.)
    int el = lane;
    asm volatile("" : "+v"(el));
    const int e16 = el & 15, e4 = el >> 4;
    constexpr int U = D / 4;
    f32x4* const po = reinterpret_cast<f32x4*>(ring[wv]);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int c = 0; c < CD; ++c) po[(16 * nb + e16) * U + ((4 * c + e4) ^ e16)] = o[nb][c];
      const float lt = sum4_xor16_32(l[nb]);
      if (e4 == 0) {
        pm[wv][16 * nb + e16] = m[nb];
        pl[wv][16 * nb + e16] = lt;
      }
    }
    __syncthreads();
    for (int x = 64 * wv + el; x < ncols * U; x += 64 * W) {
      const int col = x / U, u = x % U, d = 4 * u;
      float mx = pm[0][col];
#pragma unroll
      for (int w = 1; w < W; ++w) mx = fmaxf(mx, pm[w][col]);
      float sum = 0.f;
      f32x4 acc = {};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = fast_exp2(pm[w][col] - mx);
        sum += pl[w][col] * f;
        acc += f * reinterpret_cast<const f32x4*>(ring[w])[col * U + (u ^ (col & 15))];
      }
      if (whole) {
        const int at = col0 + col, j = fdiv(g.by_group, at);
        const int64_t row = ((int64_t)b * g.R + j) * g.H + kvh * group + at - j * group;
        const f32x4 y = average(acc, sum);
        *reinterpret_cast<u32x2*>(g.out + row * D + d) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        if (g.lse && d == 0) g.lse[row] = sum == 0.f ? -INFINITY : (mx + __log2f(sum)) * kLn2;
      } else {
        const int64_t pc = (int64_t)slot * COLS + col;
        *reinterpret_cast<f32x4*>(g.part_o + pc * D + d) = acc;
        if (d == 0) *reinterpret_cast<f32x2*>(g.part_ml + 2 * pc) = f32x2{mx, sum};
      }
    }
    __syncthreads();
  };

  deal(g, D, segment);
}

// ============================================================================ latent cache
// One workgroup = eight waves = 32 HB columns, query rows of a sequence (its new tokens' heads, token by token, so that
// few heads of several tokens share one pass over the cache). Two waves per SIMD, split by role as in the
// sparse attention (attention.hip, whose tile and operand layouts these are): four scorers compute S^T = K Q^T of 16 tokens x
// 16 HB columns each, do the online softmax and leave P (bf16) and the reference maximum of their token half in an LDS slot;
// four value waves, one tile behind, accumulate O^T += V^T P^T for all columns and 128 value dims each, from V operands read a
// tile ahead. One barrier per tile.
//
// Here the tiles are whole stretches of cache rows, so nothing is gathered through a list: a value wave's lane finds
// the row of its token from the staged page-table entries. A call is bound by the cache's bytes, not by the
// products, so kLatBufs tile buffers keep kLatBufs - 1 tiles on their way while one is scored (at barrier `it`
// the buffer of tile it - 1 is free: its V operands are in registers).
//
// Measured, 64 heads: 64 sequences of 16K to 128K (5.4 GB) 885 us, 6.2 TB/s, bound by HBM; two new tokens on 64 x 16K 345 us,
// 0.85 PFLOP/s, each row of the cache read by two workgroups of one XCD; 1 x 16K 21.4 us, of which about 5 are the lengths,
// pages and Q before the first tile, 0.6 a tile, and the partials' way through the join 5 and more. 16 heads: 64 x 16K 220 us, with
// three new tokens 241 in one pass over the cache (498 with a workgroup per token).
constexpr int kLatBufs = 4;
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
constexpr int kLatPages = 1024;  // page-table entries staged in LDS at a time

template <int HB, bool MULTI>  // blocks of 32 query rows; MULTI: of several new tokens
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void latent_decode_kernel(DecodeGeom g) {
  constexpr int COLS = 32 * HB;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLatBufs * kMlaTile + 2 * kMlaPSlot];
  __shared__ int pages[kLatPages];
  __shared__ float fin[2 * 2 * COLS];  // per (token half, column): reference maximum and sum
  const int lane = threadIdx.x & 63, wv = uniform((int)(threadIdx.x >> 6));
  const int i16 = lane & 15, q4 = lane >> 4, w4 = wv & 3;
  const bool scorer = wv < 4;
  uint8_t* const pslots = lds + kLatBufs * kMlaTile;
  const uint8_t* kvb = static_cast<const uint8_t*>(g.k);

  auto segment = [&](int b, int r, const Span& sp, int t0, int t1, bool whole, int slot) {
    // columns: rows col0 .. of the sequence's R * H; positions of the first and the last one's new token
    const int col0 = r * COLS, ncols = g.R * g.H - col0 < COLS ? g.R * g.H - col0 : COLS;
    const int tq0 = sp.c - g.R + fdiv(g.by_group, col0);
    const int tq1 = MULTI ? sp.c - g.R + fdiv(g.by_group, col0 + ncols - 1) : tq0;
    const int64_t row0 = (int64_t)b * g.R * g.H + col0;  // output row of column 0
    auto token_of = [&](int col) { return MULTI ? sp.c - g.R + fdiv(g.by_group, col0 + (col < ncols ? col : 0)) : tq0; };
    auto sees = [&](int s, int t) { return s <= t && (g.k_swa == 0 || t - s < g.k_swa || s < g.k_sink); };
    // several new tokens: does a tile from position s0 on reach to where they see different positions? (s0 + kTile may be 2^31)
    auto uneven = [&](int s0) { return MULTI && uniform(tq0 != tq1 && (s0 > tq0 + 1 - kTile || (g.k_swa > 0 && s0 <= tq1 - g.k_swa))); };
    auto first_pos = [&](int t) { return (t < sp.ns ? t : t + sp.skip) * kTile; };
    // page-table entries of tiles [p0, p1): those before the skipped ones, then the others
    int f1 = 0, n1 = 0, f2 = 0;
    auto stage = [&](int p0, int p1) {
      const int e1 = p1 < sp.ns ? p1 : sp.ns, b2 = p0 > sp.ns ? p0 : sp.ns;
      int n2 = 0;
      f1 = n1 = f2 = 0;
      if (p0 < e1) {
        f1 = fdiv(g.by_page, p0 * kTile);
        const int last = e1 <= (sp.c - 1) / kTile ? e1 * kTile - 1 : sp.c - 1;  // (e1 * kTile may be 2^31)
        n1 = fdiv(g.by_page, last) - f1 + 1;
      }
      if (b2 < p1) {
        f2 = fdiv(g.by_page, (b2 + sp.skip) * kTile);
        const int64_t end = (int64_t)(p1 + sp.skip) * kTile - 1;
        n2 = fdiv(g.by_page, end < sp.c ? (int)end : sp.c - 1) - f2 + 1;
      }
      // (barriers that wait for LDS alone, and no entries loaded by value waves: their direct loads of Q may still be on
      // their way)
      lds_barrier();  // the previous entries' readers are done
      if (scorer)
        for (int i = (int)threadIdx.x; i < n1 + n2; i += 256) {
          const int pg = i < n1 ? f1 + i : f2 + i - n1;
          const int ph = g.page_table ? g.page_table[(int64_t)b * g.max_pages + pg] : b;
          pages[i] = ph >= 0 && ph < g.n_phys ? ph : -1;
        }
      lds_barrier();
    };
    // cache row of token `tok` of tile t, -1 where no column attends to it
    auto row_of = [&](int t, int tok) {
      const int s = first_pos(t) + tok;
      if (s > tq1 || !(g.k_swa == 0 || tq0 - s < g.k_swa || s < g.k_sink)) return -1;
      const int pg = fdiv(g.by_page, s);
      const int ph = pages[t < sp.ns ? pg - f1 : n1 + pg - f2];
      return ph >= 0 ? ph * g.P + (s - pg * g.P) : -1;
    };
    if (scorer) {
      const int th = w4 & 1, pair = w4 >> 1;  // tokens 16 th .. + 15, columns 16 HB pair ..
      const int ksw = mla_swz(i16 >> 3, i16 & 7);
      const int k_row = th * kMlaHalf + 9 * (i16 >> 3) * 1024 + 8 * (i16 & 7) * 16;
      const int k_even = k_row + ((0 + q4) ^ ksw) * 16, k_odd = k_row + ((4 + q4) ^ ksw) * 16;
      u32x4 qb[HB][18];  // Q^T as the B operand: column 16 (HB pair + nb) + i16, k-step s covers dims 32 s + 8 q4 ..
      float m[HB], l[HB];
      int tcol[HB];  // positions of the columns' new tokens
#pragma unroll
      for (int nb = 0; nb < HB; ++nb) {
        m[nb] = kNoRef;
        l[nb] = 0.f;
        tcol[nb] = token_of(16 * (HB * pair + nb) + i16);
      }
      for (int p0 = t0; p0 < t1; p0 += g.pass_tiles) {
        const int nt = t1 - p0 < g.pass_tiles ? t1 - p0 : g.pass_tiles;
        stage(p0, p0 + nt);
        if (p0 == t0) {  // Q has landed as tiles of 32 columns, whose rows lie as a K tile's
          lds_barrier();
          const uint8_t* qt = lds + (kLatBufs - 2) * kMlaTile + pair * (HB == 2 ? kMlaTile : kMlaHalf) - th * kMlaHalf;
#pragma unroll
          for (int nb = 0; nb < HB; ++nb)
#pragma unroll
            for (int s = 0; s < 18; ++s) qb[nb][s] = *reinterpret_cast<const u32x4*>(qt + nb * kMlaHalf + ((s & 1) ? k_odd : k_even) + (s >> 1) * 1024);
          lds_barrier();
        }
        uint32_t cur = 0;
        for (int it = 0; it <= nt; ++it) {
          // tile it has landed; this scorer's P of tile it - 1 is written
          asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
          const uint8_t* tb = lds + __builtin_amdgcn_readfirstlane(cur);
          cur = cur + kMlaTile == kLatBufs * kMlaTile ? 0 : cur + kMlaTile;
          if (it == nt) continue;  // (the value waves' last tile)
          const uint32_t vmask = (uint32_t)__ballot(row_of(p0 + it, lane & 31) >= 0);
          float mp[2] = {-INFINITY, -INFINITY};  // the other token half's reference of tile it - 1
          if (it > 0) {
            const uint8_t* pr = pslots + ((it - 1) & 1) * kMlaPSlot + 64 * kMlaPHead + (1 - th) * 256;
#pragma unroll
            for (int nb = 0; nb < HB; ++nb) mp[nb] = *reinterpret_cast<const float*>(pr + 4 * (16 * (HB * pair + nb) + i16));
          }
          constexpr int KB = 3;  // K operands requested ahead of the products
          f32x4 sacc[HB];
#pragma unroll
          for (int nb = 0; nb < HB; ++nb) sacc[nb] = f32x4{};
          u32x4 ka[2][KB];
#pragma unroll
          for (int s6 = 0; s6 < KB; ++s6) ka[0][s6] = *reinterpret_cast<const u32x4*>(tb + ((s6 & 1) ? k_odd : k_even) + (s6 >> 1) * 1024);
#pragma unroll
          for (int bt = 0; bt < 18 / KB; ++bt) {
            if (bt + 1 < 18 / KB) {
#pragma unroll
              for (int s6 = 0; s6 < KB; ++s6) {
                const int s = KB * (bt + 1) + s6;
                ka[(bt + 1) & 1][s6] = *reinterpret_cast<const u32x4*>(tb + ((s & 1) ? k_odd : k_even) + (s >> 1) * 1024);
              }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s6 = 0; s6 < KB; ++s6)
#pragma unroll
              for (int nb = 0; nb < HB; ++nb) sacc[nb] = mfma16(ka[bt & 1][s6], qb[nb][KB * bt + s6], sacc[nb]);
            __builtin_amdgcn_sched_barrier(0);
          }
          const uint32_t hmask = (vmask >> (16 * th)) & 0xFFFFu;
          if (hmask != 0xFFFFu) {
#pragma unroll
            for (int nb = 0; nb < HB; ++nb)
#pragma unroll
              for (int k = 0; k < 4; ++k) sacc[nb][k] = ((hmask >> (4 * q4 + k)) & 1u) ? sacc[nb][k] : -INFINITY;
          }
          if (const int s0 = first_pos(p0 + it); uneven(s0)) {
#pragma unroll
            for (int nb = 0; nb < HB; ++nb)
#pragma unroll
              for (int k = 0; k < 4; ++k) sacc[nb][k] = sees(s0 + 16 * th + 4 * q4 + k, tcol[nb]) ? sacc[nb][k] : -INFINITY;
          }
          uint8_t* ps = pslots + (it & 1) * kMlaPSlot;
          float smx[HB];
#pragma unroll
          for (int nb = 0; nb < HB; ++nb) smx[nb] = fmaxf(fmaxf(sacc[nb][0], sacc[nb][1]), fmaxf(sacc[nb][2], sacc[nb][3]));
          if constexpr (HB == 2) max4_xor16_32_pair(smx[0], smx[1]);
          else smx[0] = max4_xor16_32(smx[0]);
#pragma unroll
          for (int nb = 0; nb < HB; ++nb) {
            const float mx = smx[nb] * g.scale_log2;
            // the reference moves when the maximum grows by more than 2^8, or to the other half's when that is larger
            float tgt = mx > m[nb] + kLazy ? mx : m[nb];
            tgt = fmaxf(tgt, mp[nb]);
            const bool up = tgt > m[nb];
            if (__ballot(up)) {
              l[nb] = up ? l[nb] * fast_exp2(m[nb] - tgt) : l[nb];
              m[nb] = up ? tgt : m[nb];
            }
            float p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              p[k] = exp2_below(sacc[nb][k], g.scale_log2, m[nb]);  // -inf -> 0
              l[nb] += p[k];
            }
            const int lh = 16 * (HB * pair + nb) + i16;
            // (rounded to bf16, what the value products take, which also halves the slot; the sums take them unrounded)
            *reinterpret_cast<u32x2*>(ps + lh * kMlaPHead + 32 * th + 8 * q4) = u32x2{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])};
            if (q4 == 0) *reinterpret_cast<float*>(ps + 64 * kMlaPHead + th * 256 + 4 * lh) = m[nb];
          }
        }
      }
#pragma unroll
      for (int nb = 0; nb < HB; ++nb) {
        const float lt = sum4_xor16_32(l[nb]);
        if (q4 == 0) {
          const int lh = 16 * (HB * pair + nb) + i16;
          fin[2 * (COLS * th + lh)] = m[nb];
          fin[2 * (COLS * th + lh) + 1] = lt;
        }
      }
      __syncthreads();
      return;
    }
    // ---- value wave w4: dims 128 w4 .. + 127 of all columns
    const int G = lane >> 4, sl = lane & 15;
    int v_off[2][2];
#pragma unroll
    for (int rd = 0; rd < 2; ++rd)
#pragma unroll
      for (int par = 0; par < 2; ++par) {
        const int tk = 8 * (G >> 1) + 4 * rd + (sl >> 2), o8 = tk >> 3, j8 = tk & 7;
        const int ch = 4 * par + 2 * (G & 1) + ((sl >> 1) & 1);
        v_off[rd][par] = (9 * o8 + 2 * w4) * 1024 + (8 * j8 + (ch ^ mla_swz(o8, j8))) * 16 + (sl & 1) * 8;
      }
    const int oj = lane & 31;
    f32x16 o[4 * HB];  // block 4 hb + c: columns 32 hb .., dims 128 w4 + 32 c ..
#pragma unroll
    for (int c = 0; c < 4 * HB; ++c) o[c] = f32x16{};
    bool marred = false;  // was a value taken as 0?
    float m_o[HB];  // reference maxima of the accumulators
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) m_o[hb] = -INFINITY;
    // this wave loads tokens 8 w4 .. of a tile: lane 8 jj + u takes chunk u ^ swz of token jj of them, nine times
    const int dj = lane >> 3, dma_tok = 8 * w4 + dj;
    const int64_t dma_col = ((lane & 7) ^ mla_swz(w4, dj)) * 16;
    // Q goes through the last tile buffers. (Columns past the last repeat the first and are not stored.)
#pragma unroll
    for (int t = 0; t < HB; ++t) {
      const int h = 32 * t + dma_tok;
      lds_dma_row9(reinterpret_cast<const uint8_t*>(g.q) + (row0 + (h < ncols ? h : 0)) * 1152 + dma_col,
                   lds_addr(lds + (kLatBufs - 2 + t) * kMlaTile + w4 * (kMlaLoads * 1024)));
    }
    for (int p0 = t0; p0 < t1; p0 += g.pass_tiles) {
      const int nt = t1 - p0 < g.pass_tiles ? t1 - p0 : g.pass_tiles;
      stage(p0, p0 + nt);
      auto issue = [&](int it, uint32_t buf) {
        const int row = row_of(p0 + it, dma_tok);
        lds_dma_row9((row >= 0 ? kvb + (int64_t)row * 1152 : zero_row) + dma_col, lds_addr(lds + buf + w4 * (kMlaLoads * 1024)));
      };
      uint32_t cur = 0, next = 0;  // buffers of tile it, and of the next tile to load
      auto fill = [&](int i) {
        if (i < nt) {
          issue(i, next);
          next += kMlaTile;
        }
      };
      if (p0 == t0) {
        fill(0);
        fill(1);
        // Q has landed (behind it are one or two tiles), and the scorers have read it
        if (nt > 1) vm_wait<2 * kMlaLoads>();
        else vm_wait<kMlaLoads>();
        lds_barrier();
        lds_barrier();
      } else {
        fill(0);
        fill(1);
      }
      fill(2);
      static_assert(kLatBufs == 4, "two buffers for Q, two to fill meanwhile");
      u32x4 va[4][2];  // V operands of tile it - 1
      for (int it = 0; it <= nt; ++it) {
        // tile it has landed (behind it are the kLatBufs - 2 next ones, fewer at the end); the scorers' P of tile
        // it - 1 is in its slot; the buffer of tile it - 1 is free
        if (it + kLatBufs - 2 < nt) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kMlaLoads * (kLatBufs - 2)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + kLatBufs - 1 < nt) {
          issue(it + kLatBufs - 1, next = next == kLatBufs * kMlaTile ? 0 : next);
          next += kMlaTile;
        }
        const uint32_t at = cur;
        cur = cur + kMlaTile == kLatBufs * kMlaTile ? 0 : cur + kMlaTile;
        auto read_v = [&]() {
          const uint8_t* tp = lds + __builtin_amdgcn_readfirstlane(at);
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
              va[c][ks] = tr16_pair(tp + v_off[0][c & 1] + ks * kMlaHalf + (c >> 1) * 1024, tp + v_off[1][c & 1] + ks * kMlaHalf + (c >> 1) * 1024);
        };
        if (it == 0) {  // (nothing scored yet)
          read_v();
          continue;
        }
        if (const int s0 = first_pos(p0 + it - 1); uneven(s0)) {
          uint32_t odd = 0;  // (adding 1 to an exponent of ones carries into the sign bit)
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
              for (int k = 0; k < 4; ++k) odd |= (va[c][ks][k] & 0x7F807F80u) + 0x00800080u;
          // A weight of zero does not silence a NaN or an infinity in a row of V that only some of the columns see. It is taken
          // as 0 here, and those that see it get their NaN after the stores.
          if (uniform(__ballot((odd & 0x80008000u) != 0) != 0)) {
            marred = true;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int k = 0; k < 4; ++k) va[c][ks][k] &= ~(((((va[c][ks][k] & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xFFFFu);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        const uint8_t* ps = pslots + ((it - 1) & 1) * kMlaPSlot;
        float mA[HB], mB[HB];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
          mA[hb] = *reinterpret_cast<const float*>(ps + 64 * kMlaPHead + 4 * (32 * hb + oj));
          mB[hb] = *reinterpret_cast<const float*>(ps + 64 * kMlaPHead + 256 + 4 * (32 * hb + oj));
        }
        u32x4 pb[HB][2];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
            pb[hb][ks] = *reinterpret_cast<const u32x4*>(ps + (32 * hb + oj) * kMlaPHead + 32 * ks + 16 * (lane >> 5));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
          const float mn = fmaxf(mA[hb], mB[hb]);  // >= m_o: the references never decrease
          if (__ballot(mA[hb] != mB[hb] || mn > m_o[hb])) {  // rare once the halves agree
            const float alpha = mn > m_o[hb] ? fast_exp2(m_o[hb] - mn) : 1.f;  // m_o = -inf -> 0
            m_o[hb] = mn;
            if (__ballot(alpha != 1.f)) {
#pragma unroll
              for (int c = 0; c < 4; ++c) o[4 * hb + c] *= alpha;
            }
            // (a half whose reference is lower: its weights are scaled and rounded to bf16 once more, which leaves them within 2^-8;
            // from the next tile on both halves have one reference)
            const float fa = mA[hb] == mn ? 1.f : fast_exp2(mA[hb] - mn), fb = mB[hb] == mn ? 1.f : fast_exp2(mB[hb] - mn);
            if (__ballot(fa != 1.f)) pb[hb][0] = scale_bf16x8(pb[hb][0], fa);
            if (__ballot(fb != 1.f)) pb[hb][1] = scale_bf16x8(pb[hb][1], fb);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int hb = 0; hb < HB; ++hb) o[4 * hb + c] = mfma32(va[c][ks], pb[hb][ks], o[4 * hb + c]);
        if (it < nt) {
          __builtin_amdgcn_sched_barrier(0);
          read_v();
        }
      }
    }
    __syncthreads();  // the scorers' reference maxima and sums
    float mfin[HB], lt[HB];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      const int lh = 32 * hb + oj;
      const float ma = fin[2 * lh], la = fin[2 * lh + 1], mb = fin[2 * (COLS + lh)], lb = fin[2 * (COLS + lh) + 1];
      mfin[hb] = fmaxf(ma, mb);
      lt[hb] = la * fast_exp2(ma - mfin[hb]) + lb * fast_exp2(mb - mfin[hb]);
      if (w4 == 0 && lane < 32 && lh < ncols) {
        if (whole) {
          if (g.lse) g.lse[row0 + lh] = lt[hb] == 0.f ? -INFINITY : (mfin[hb] + __log2f(lt[hb])) * kLn2;
        } else {
          *reinterpret_cast<f32x2*>(g.part_ml + 2 * ((int64_t)slot * COLS + lh)) = f32x2{mfin[hb], lt[hb]};
        }
      }
    }
    // An output goes row by row through the tile buffers, idle since the barrier, so that a store instruction
    // writes whole lines.
    // Lane l, register r of block 4 hb + c holds column 32 c + 8 (r / 4) + 4 (l / 32) + r % 4 of head 32 hb + l % 32.
    // (the lane made opaque here, or these offsets are computed before the loop over stretches and spill)
    int el = lane;
    asm volatile("" : "+v"(el));
    const int ej = el & 31;
    if (whole) {
      uint8_t* ost = lds + w4 * (64 * 272);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x16& ob = o[4 * hb + c];
            const f32x4 y = average(f32x4{ob[4 * q], ob[4 * q + 1], ob[4 * q + 2], ob[4 * q + 3]}, lt[hb]);
            *reinterpret_cast<u32x2*>(ost + (32 * hb + ej) * 272 + (32 * c + 8 * q + 4 * (el >> 5)) * 2) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
          }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (this wave's own writes)
#pragma unroll
      for (int k = 0; k < 8 * HB; ++k) {
        const int hh = 4 * k + (el >> 4);
        const u32x4 v = *reinterpret_cast<const u32x4*>(ost + hh * 272 + 16 * (el & 15));
        if (hh < ncols) *reinterpret_cast<u32x4*>(g.out + (row0 + hh) * 512 + 128 * w4 + 8 * (el & 15)) = v;
      }
    } else {  // a partial in the accumulators' order, whole lines per store: [4 waves][4 HB blocks][4][64 lanes][4]
      f32x4* dst = reinterpret_cast<f32x4*>(g.part_o) + (int64_t)slot * (4096 * HB) + w4 * (1024 * HB) + el;
#pragma unroll
      for (int c = 0; c < 4 * HB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) dst[(4 * c + q) * 64] = f32x4{o[c][4 * q], o[c][4 * q + 1], o[c][4 * q + 2], o[c][4 * q + 3]};
    }
    // (A value that is no number or infinite is part of K too: a column that sees it has a score that is none or infinite, so
    // that all its output is NaN already unless the score is -inf, whose weight of 0 times the value is NaN. Columns of no other
    // score stay 0; a partial's may have other scores elsewhere.)
    if (MULTI && marred) {
      for (int t = t0; t < t1; ++t) {
        const int s0 = first_pos(t);
        if (!uneven(s0)) continue;
        for (int s = s0; s - s0 < kTile && s <= tq1; ++s) {
          const int pg = fdiv(g.by_page, s), ph = g.page_table ? g.page_table[(int64_t)b * g.max_pages + pg] : b;
          if (ph < 0 || ph >= g.n_phys) continue;
          const uint16_t* v = reinterpret_cast<const uint16_t*>(kvb + ((int64_t)ph * g.P + (s - pg * g.P)) * 1152) + 128 * w4;
          for (int d = lane; d < 128; d += 64) {
            if ((v[d] & 0x7F80u) != 0x7F80u) continue;
            for (int col = 0; col < ncols; ++col) {
              if (!sees(s, token_of(col))) continue;
              if (whole && fin[2 * col + 1] == 0.f && fin[2 * (COLS + col) + 1] == 0.f) continue;
              if (whole) g.out[(row0 + col) * 512 + 128 * w4 + d] = 0x7FC0;
              else g.part_o[(((int64_t)slot * 16 * HB + w4 * 4 * HB + 4 * (col / 32) + d / 32) * 4 + (d / 8) % 4) * 256 + (col % 32 + 32 * ((d / 4) % 2)) * 4 + d % 4] = __builtin_nanf("");
            }
          }
        }
      }
    }
  };
  deal(g, 512, segment);
}

// ============================================================================ joining the partials
// A thread takes four dims of one output row and every S-th of the row's partials, with a running maximum; the
// S threads of a row and dims meet in LDS. Bound by two round trips to what other XCDs have just written: which
// workgroups have partials (left there by the first of them), and the partials. Nothing to do where one
// stretch covered a (sequence, head) whole. 4 to 6 us for up to 16 MB of partials, 12 for the 42 MB of 64 latent sequences.
struct Joined {
  float m, l;
  f32x4 acc;
};
// partial v of the parts p: slot of the first workgroup's, then the first slot of each following stretch's
__device__ __forceinline__ int part_slot(const int4& p, int v, int M) { return v == 0 ? p.z : 2 * ((p.x + v) * M + p.w); }

template <int S, int U, class ML, class O>  // U partials requested together
__device__ __forceinline__ Joined join_parts(const int4& p, int M, int sub, ML&& load_ml, O&& load_o) {
  const int n = p.y - p.x + 1;
  Joined r{kNoRef, 0.f, f32x4{}};
  for (int v = sub; v < n; v += S * U) {
    f32x2 ml[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int slot = part_slot(p, v + u * S < n ? v + u * S : v, M);
      ml[u] = load_ml(slot);
      x[u] = load_o(slot);
    }
    float mx = r.m;
#pragma unroll
    for (int u = 0; u < U; ++u) mx = fmaxf(mx, ml[u][0]);
    const float a = fast_exp2(r.m - mx);
    r.l *= a;
    r.acc *= a;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v + u * S >= n) break;
      const float f = fast_exp2(ml[u][0] - mx);
      r.l += ml[u][1] * f;
      r.acc += f * x[u];
    }
    r.m = mx;
  }
  return r;
}
__device__ __forceinline__ void join_two(Joined& r, const Joined& q) {
  const float mx = fmaxf(r.m, q.m), a = fast_exp2(r.m - mx), f = fast_exp2(q.m - mx);
  r.l = r.l * a + q.l * f;
  r.acc = r.acc * a + q.acc * f;
  r.m = mx;
}
// The sum over the S threads x, x + T, .. of a workgroup of S T threads (in its first T), first within waves.
template <int S, int T>
__device__ __forceinline__ Joined join_threads(Joined r, Joined* lds) {
  constexpr int TW = T < 64 ? T : 64, W = S * T / 64, G = W * TW / T;  // threads of a wave apart, waves, entries per thread
#pragma unroll
  for (int o = TW; o < 64; o <<= 1) {
    Joined q;
    q.m = __shfl_xor(r.m, o);
    q.l = __shfl_xor(r.l, o);
#pragma unroll
    for (int k = 0; k < 4; ++k) q.acc[k] = __shfl_xor(r.acc[k], o);
    join_two(r, q);
  }
  if constexpr (G > 1) {
    const int wv = threadIdx.x >> 6, at = wv * TW + (threadIdx.x & 63);  // = group * T + x, T threads of neighbouring waves
    if ((threadIdx.x & 63) < TW) lds[at] = r;
    __syncthreads();
    if ((int)threadIdx.x < T)
#pragma unroll
      for (int k = 1; k < G; ++k) join_two(r, lds[k * T + (int)threadIdx.x]);
  }
  return r;
}
__device__ __forceinline__ void join_store(const DecodeGeom& g, const Joined& r, int64_t row, int width, int d) {
  const f32x4 y = average(r.acc, r.l);
  *reinterpret_cast<u32x2*>(g.out + row * width + d) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  if (g.lse && d == 0) g.lse[row] = r.l == 0.f ? -INFINITY : (r.m + __log2f(r.l)) * kLn2;
}

// Grouped heads: a workgroup per output row and 4 T of its dims.
template <int D, int COLS, int S, int T>
__global__ __launch_bounds__(S * T) void gqa_join_kernel(DecodeGeom g) {
  __shared__ Joined lds[S * T < 64 ? 1 : S * T / 64 * (T < 64 ? T : 64)];
  const int group = (int)g.by_group.d, cols = g.R * group, cb_n = (int)g.by_blocks.d;
  const int nth = g.first + (int)blockIdx.x, unit = (int)((uint32_t)nth / (uint32_t)cols), col = nth - unit * cols;  // (sequence, key/value head)
  const int4 p = g.parts[(int64_t)unit * cb_n + col / COLS];
  if (p.x == p.y) return;
  const int d = 4 * (T * (int)blockIdx.y + (int)threadIdx.x % T), cc = col % COLS;
  Joined r = join_parts<S, 4>(p, g.M, threadIdx.x / T, [&](int slot) { return *reinterpret_cast<const f32x2*>(g.part_ml + 2 * ((int64_t)slot * COLS + cc)); },
                              [&](int slot) { return *reinterpret_cast<const f32x4*>(g.part_o + ((int64_t)slot * COLS + cc) * D + d); });
  r = join_threads<S, T>(r, lds);
  if ((int)threadIdx.x >= T) return;
  const int b = unit / g.Hkv, kvh = unit - b * g.Hkv, j = fdiv(g.by_group, col);
  join_store(g, r, ((int64_t)b * g.R + j) * g.H + kvh * group + col - j * group, D, d);
}

// Latent: a workgroup per (sequence, block of columns) and T of the partial's 4096 HB vectors of four, 64 of which are 32
// columns x 8 dims in the accumulators' order.
template <int HB, int S, int T>
__global__ __launch_bounds__(S * T) void latent_join_kernel(DecodeGeom g) {
  static_assert(HB <= 2 && T % 64 == 0, "a wave's threads share their partials");
  __shared__ Joined lds[S * T / 64 * 64];
  const int nth = g.first + (int)blockIdx.x;
  const int4 p = g.parts[nth];
  if (p.x == p.y) return;
  const int vec = T * (int)blockIdx.y + (int)threadIdx.x % T;
  const int lane = vec & 63, q = (vec >> 6) & 3, c = (vec >> 8) & 3, hb = (vec >> 10) & (HB - 1), w4 = vec >> (9 + HB);
  const int lh = 32 * hb + (lane & 31), d = 128 * w4 + 32 * c + 8 * q + 4 * (lane >> 5);
  Joined r = join_parts<S, (S > 1 ? 8 : 4)>(p, g.M, threadIdx.x / T, [&](int slot) { return *reinterpret_cast<const f32x2*>(g.part_ml + 2 * ((int64_t)slot * (32 * HB) + lh)); },
                           [&](int slot) { return reinterpret_cast<const f32x4*>(g.part_o)[(int64_t)slot * (4096 * HB) + vec]; });
  r = join_threads<S, T>(r, lds);
  if (threadIdx.x >= T) return;
  const int b = fdiv(g.by_m, nth), col = 32 * HB * (nth - b * g.M) + lh;
  if (col < g.R * g.H) join_store(g, r, (int64_t)b * g.R * g.H + col, 512, d);
}

// ============================================================================ host launchers
// Launches n (times y) workgroups, in as many launches as it takes: the runtime counts the threads of a launch's dimension in 32
// bits, and a launch of more runs the rest modulo 2^32 without an error.
static hipError_t launch_all(void (*kernel)(DecodeGeom), DecodeGeom g, int64_t n, unsigned y, unsigned threads, hipStream_t st) {
  const int64_t most = (int64_t(1) << 31) / threads;
  for (int64_t at = 0; at < n; at += most) {
    g.first = (int)at;
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)(n - at < most ? n - at : most), y), dim3(threads), st, g);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Calls of few rows, whose rows have many partials, take few dims per workgroup and share the partials among
// more threads.
constexpr int64_t kJoinFew = 2048;  // workgroups
template <int D, bool FP8, int NB>
static hipError_t launch_gqa(const DecodeGeom& g, hipStream_t st) {
  auto kernel = g.R > 1 ? gqa_decode_kernel<D, FP8, NB, true, 4> : gqa_decode_kernel<D, FP8, NB, false, 4>;
  if constexpr (NB <= 2)
    if (g.waves == 8) kernel = g.R > 1 ? gqa_decode_kernel<D, FP8, NB, true, 8> : gqa_decode_kernel<D, FP8, NB, false, 8>;
  const hipError_t e = launch_all(kernel, g, g.grid, 1, 64 * (unsigned)g.waves, st);
  if (e != hipSuccess || g.part_o == nullptr) return e;
  const int64_t rows = (int64_t)g.n_seq * g.R * g.H;
  if (rows * (D / 32) <= kJoinFew) {
    // (at most that many partials of a row, if the sequences are alike)
    if ((int)g.by_stretches.d / g.n_seq > 32) return launch_all(gqa_join_kernel<D, 16 * NB, 128, 8>, g, rows, D / 32, 1024, st);
    return launch_all(gqa_join_kernel<D, 16 * NB, 32, 8>, g, rows, D / 32, 256, st);
  }
  return launch_all(gqa_join_kernel<D, 16 * NB, 1024 / D, D / 4>, g, rows, 1, 256, st);
}
template <int D, bool FP8>
static hipError_t launch_gqa(const DecodeGeom& g, hipStream_t st) {
  const int nb = g.block_cols / 16;
  return nb == 1 ? launch_gqa<D, FP8, 1>(g, st) : nb == 2 ? launch_gqa<D, FP8, 2>(g, st) : launch_gqa<D, FP8, 4>(g, st);
}

template <int HB>
static hipError_t launch_latent(const DecodeGeom& g, hipStream_t st) {
  const auto kernel = g.R > 1 && g.H % (32 * HB) != 0 ? latent_decode_kernel<HB, true> : latent_decode_kernel<HB, false>;
  const hipError_t e = launch_all(kernel, g, g.grid, 1, 512, st);
  if (e != hipSuccess || g.part_o == nullptr) return e;
  const int64_t units = (int64_t)g.n_seq * g.M;
  // us with 16 / 4 / 1 threads a vector: 64 heads, 1 x 16K 21.1 / 23.0 / 37.3, 4 x 8000 26.0 / 25.3 / 29.5, 8 x 16K 50.6 / 47.4 /
  // 50.9, 64 x 1500 70.4 / 49.6 / 45.2; 16 heads, 1 x 64K 27.2 / 35.3 / 76.5, 20 x 4000 33.1 / 29.3 / 30.7
  const int64_t few = units * 64 * HB;
  if (few <= 128) return launch_all(latent_join_kernel<HB, 16, 64>, g, units, 64 * HB, 1024, st);
  if (few <= 2048) return launch_all(latent_join_kernel<HB, 4, 64>, g, units, 64 * HB, 256, st);
  return launch_all(latent_join_kernel<HB, 1, 256>, g, units, 16 * HB, 256, st);
}

hipError_t launch_decode_attn(const DecodeGeom& g, hipStream_t st) {
  if (g.latent) return g.block_cols == 32 ? launch_latent<1>(g, st) : launch_latent<2>(g, st);
  if (g.d_qk == 64) return g.fp8 ? launch_gqa<64, true>(g, st) : launch_gqa<64, false>(g, st);
  return g.fp8 ? launch_gqa<128, true>(g, st) : launch_gqa<128, false>(g, st);
}

}  // namespace lsa
