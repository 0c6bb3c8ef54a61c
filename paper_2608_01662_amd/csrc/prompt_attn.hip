// Attention of packed prompts over their own keys and values (lsa_prefill_attn) and of ragged chunks of new tokens over a
// paged cache (lsa_chunk_attn) for gfx950.
//
// The query rows of a key/value head are the heads of its group of all new tokens of a sequence, token after token: a row of
// them attends to o = sum_j 2^(z_j - m) v_j / l with z_j = scale log2(e) q.k_j, m the largest z_j, l = sum_j 2^(z_j - m). A workgroup takes
// 256 rows, eight waves of 32, and walks the tiles of 64 keys that any of them attends to, each tile once through LDS for all, in
// halves of 32 keys, with a running m (moved when a row's grew by more than 2^8, by the row's own scores) and l in fp32.
// S^T = K Q^T on 32x32x16 products: a lane holds 16 scores of one row and half, which are, rounded to bf16, the B operand of
// O^T += V^T P^T as they lie, so that P never leaves the registers; V^T comes from LDS by transposed reads. Queries and accumulators
// stay in registers (two waves per SIMD, 256 each; see waves_per_simd). The scores of the next half and the values of the last run on the matrix
// cores while this half's weights are computed.
//
// What bounds it: long calls neither the matrix cores (busy 0.39 to 0.43 of the cycles) nor the vector unit (0.29 to 0.48 beside the products), but that they
// take turns, and the clock, which falls under them. 32 heads on 8, 8192 x 8192 keys without a mask: 1125 us, 977 TFLOP/s, where a large matrix product reaches
// 1224 to 1407 (192/128 wide 1006, 64 wide, whose softmax is twice as much per product, 811). A wave's products of a tile take 1024 cycles (64 wide 512) and two
// waves of a SIMD need about 3900 for a tile each. Calls of few rows: the bytes of K and V, and the way to the first tile. Measured and not kept: 64 rows of a wave, one
// wave per SIMD (1333 us against 1190 at the time); scores weighed before the maximum is known, in one block with the products (1309
// against 1151); the instructions' order by hand or by groups (1318 against 1151); wave priorities (no change).
#include "attn_tile.hpp"
#include "device.hpp"
#include "launch.hpp"
#include "serve_tile.hpp"

namespace lsa {

constexpr int kRows = kPromptRows;  // query rows of a workgroup
constexpr int kKeys = kPromptKeys;  // keys of a tile
constexpr int kPageSlots = kPromptPages;  // page-table entries staged in LDS at a time

// Where 16-byte chunk c of row r of a tile lies: slot c ^ swz(r) of the row. The reads of a product's K operand (16 rows of one
// chunk at a time) and the transposed reads of V (4 rows of 4 chunks) then fall on all banks alike: rows of 256
// bytes cover all of them, of 128 or 384 bytes two rows do.
template <int CHUNKS>
__device__ __forceinline__ int swz(int r) {
  if constexpr (CHUNKS == 16) return (r & 3) << 2 | ((r >> 2) & 3);
  return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}

// A workgroup's share: rows row0 .. of the rows of one key/value head of sequence b, and the tiles of its keys: 0 .. ns - 1
// (the sink) and then from ns + skip on, nt in all.
struct Share {
  int b, head, row0, rows;
  int n, c;         // new tokens and keys of the sequence
  int64_t q0, kv0;  // its first token, its first key of contiguous ones
  int ns, skip, nt;
  int p0, p1;       // tiles [p0, p1) of the span are this workgroup's
  int slot;         // of its partial results, -1: it has all tiles and writes the output
};

__device__ __forceinline__ int new_tokens(const PromptGeom& g, int b, int& first) {
  const int a = g.cu_q[b], e = g.cu_q[b + 1];
  first = a;
  return a >= 0 && e >= a && e <= g.n_tok ? e - a : 0;
}

// The keys of sequence b, and the first one's row.
__device__ __forceinline__ int keys_of(const PromptGeom& g, int b, int& first) {
  if (g.ctx_len) {
    const int c = g.ctx_len[b];
    first = 0;
    return c < 0 || c > g.cap ? 0 : c;
  }
  const int a = g.cu_kv[b], e = g.cu_kv[b + 1];
  first = a;
  return a >= 0 && e >= a && e <= g.n_kv ? e - a : 0;
}
// The tiles of a block of rows: completes w from its sequence, row0 and rows.
__device__ __forceinline__ void span_of(const PromptGeom& g, Share& w) {
  const int last = (w.rows - w.row0 < kRows ? w.rows : w.row0 + kRows) - 1;
  const int t_lo = g.causal ? w.c - w.n + fdiv(g.by_group, w.row0) : w.c - 1, t_hi = g.causal ? w.c - w.n + fdiv(g.by_group, last) : w.c - 1;
  const int end = t_hi + 1 > 0 ? t_hi + 1 : 0, total = (int)(((uint32_t)end + kKeys - 1) / kKeys);  // (t_hi < c)
  const int lo = g.k_swa > 0 && t_lo >= g.k_swa ? t_lo - g.k_swa + 1 : 0, first = lo / kKeys;
  const int sink = g.k_sink < end ? g.k_sink : end, st = (int)(((uint32_t)sink + kKeys - 1) / kKeys);
  w.ns = first <= st ? total : st;
  w.skip = first <= st ? 0 : first - st;
  w.nt = total - w.skip;
}

// The work of workgroup `item` of a call that leaves the keys of a block whole, false when there is none. Workgroups i, i + 8, .. run
// on one XCD, whose L2 should read the keys that they share once: so with u = gcd(heads, 8) XCD x takes the heads = x mod u, one
// after the other, and every 8 / u th block of rows of each (which ones, turns with the sequence), from the last, which has the most
// keys, to the first. Some workgroups at the ends of sequences have nothing to do.
__device__ __forceinline__ bool find_whole(const PromptGeom& g, int item, Share& w) {
  const int lane = threadIdx.x & 63, group = (int)g.by_group.d, u = g.head_classes, step = 8 / u, per_class = g.Hkv / u;
  const int xcd = item & 7, at = item >> 3;
  int before = 0;
  for (int b0 = 0; b0 < g.n_seq; b0 += 64) {
    const int b = b0 + lane;
    int first = 0;
    const int n = b < g.n_seq ? new_tokens(g, b, first) : 0;
    int kv0 = 0;
    const int c = b < g.n_seq ? keys_of(g, b, kv0) : 0;
    const int turns = ((n * group + kRows - 1) / kRows + step - 1) / step, inc = wave_scan(turns * per_class);
    const uint64_t past = __ballot(before + inc > at);
    if (past) {
      const int i = __ffsll((unsigned long long)past) - 1;
      w.b = b0 + i;
      w.n = __builtin_amdgcn_readlane(n, i);
      w.q0 = __builtin_amdgcn_readlane(first, i);
      w.rows = w.n * group;
      const int nt = __builtin_amdgcn_readlane(turns, i), k = at - (before + __builtin_amdgcn_readlane(inc, i) - nt * per_class);
      const int nth = k / nt, block = (w.rows + kRows - 1) / kRows - 1 - ((xcd / u + w.b) % step + step * (k - nth * nt));
      if (block < 0) return false;
      w.head = xcd % u + u * nth;
      w.row0 = block * kRows;
      w.c = __builtin_amdgcn_readlane(c, i);
      w.kv0 = __builtin_amdgcn_readlane(kv0, i);
      span_of(g, w);
      w.p0 = 0;
      w.p1 = w.nt;
      w.slot = -1;
      return true;
    }
    before += __builtin_amdgcn_readlane(inc, 63);
  }
  return false;
}

// The same of a call that has few blocks of rows: the keys of a sequence's blocks are cut into equal pieces, as many as make the
// call's pieces cost about 1 / g.pieces of all, but of kLeastTiles at least: a piece's way to its first tile and its partial results, which
// the join reads again, take as long as some tiles. (us with 4 tiles, and with 4 to 16 that go with the rows: 64 tokens behind 8K 33.5, 42.4; 128
// behind 2K 29.9, 42.4; 16 behind 2K 16.4, 20.7, with 2 to 6 15.9.) A tile costs 2 with up to 128 rows, a wave per SIMD, and 3 with more (1 and 2: 24
// sequences 212 for 202). The largest pieces come first, of up to 64 sequences (24 of 1 to 342 tokens behind 1389 to 8423: 202 us, in the
// sequences' order and by equal tiles 231). Of a sequence the heads come one after the other, so that an XCD keeps to a class of them, and a block's pieces lie Hkv
// apart; the last block, which has the most keys, first (3900 tokens behind 4292, 32 heads on 8: 407 us, blocks of a head from the first on 470,
// not cut at all 393). The first piece of a block tells the join about it.
constexpr int kLeastTiles = 4;
__device__ __forceinline__ bool find_piece(const PromptGeom& g, int id, Share& w) {
  const int lane = threadIdx.x & 63, group = (int)g.by_group.d;
  struct Seq {
    int n, q0, c, kv0, blocks, tiles;  // tiles: of its last block, the most
  };
  auto load = [&](int b) {
    Seq s{};
    if (b >= g.n_seq) return s;
    s.n = new_tokens(g, b, s.q0);
    s.c = keys_of(g, b, s.kv0);
    const int rows = s.n * group;
    s.blocks = (rows + kRows - 1) / kRows;
    if (s.blocks > 0) {
      Share x;
      x.rows = rows;
      x.row0 = (s.blocks - 1) * kRows;
      x.n = s.n;
      x.c = s.c;
      span_of(g, x);
      s.tiles = x.nt;
    }
    return s;
  };
  auto cost = [&](const Seq& s) { return s.n * group <= kRows / 2 ? 2 : 3; };
  Seq s = load(lane);
  // (in float: the sum may pass 31 bits)
  auto all = [&](const Seq& y) { return (float)(cost(y) * y.blocks) * (float)(y.tiles) * (float)g.Hkv; };
  float total = all(s);
  for (int b = lane + 64; b < g.n_seq; b += 64) total += all(load(b));
  for (int k = 32; k >= 1; k >>= 1) total += __shfl_xor(total, k);
  const float share = total / (float)g.pieces;
  const int slots = g.pieces + g.blocks;
  int before = 0, items = 0;
  for (int b0 = 0; b0 < g.n_seq; b0 += 64) {
    if (b0 > 0) s = load(b0 + lane);
    const float even = share / (float)cost(s);
    const int each = even > (float)kLeastTiles ? (even < 1e9f ? (int)even + 1 : 1000000000) : kLeastTiles;
    const int pieces = s.tiles > each ? (s.tiles + each - 1) / each : 1;
    int count = s.blocks * g.Hkv * pieces, count_items = s.blocks * g.Hkv, from = lane;
    if (g.n_seq <= 64) {
      const int size = cost(s) * (s.tiles / pieces);
      int rank = 0;
      for (int k = 0; k < g.n_seq; ++k) {
        const int other = __builtin_amdgcn_readlane(size, k);
        rank += other > size || (other == size && k < lane);
      }
      if (lane >= g.n_seq) rank = lane;
      count = __builtin_amdgcn_ds_permute(4 * rank, count);
      count_items = __builtin_amdgcn_ds_permute(4 * rank, count_items);
      from = __builtin_amdgcn_ds_permute(4 * rank, lane);
    }
    const int inc = wave_scan(count), inc_items = wave_scan(count_items);
    const uint64_t past = id < slots ? __ballot(before + inc > id) : 0;
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1, i = __builtin_amdgcn_readlane(from, at);
      w.b = b0 + i;
      w.n = __builtin_amdgcn_readlane(s.n, i);
      w.q0 = __builtin_amdgcn_readlane(s.q0, i);
      w.c = __builtin_amdgcn_readlane(s.c, i);
      w.kv0 = __builtin_amdgcn_readlane(s.kv0, i);
      w.rows = w.n * group;
      const int np = __builtin_amdgcn_readlane(pieces, i), nb = __builtin_amdgcn_readlane(s.blocks, i);
      const int k = id - (before + __builtin_amdgcn_readlane(inc, at) - nb * g.Hkv * np), rest = k / g.Hkv, nth = rest / np, piece = rest - nth * np;
      w.head = k - rest * g.Hkv;
      const int item = items + __builtin_amdgcn_readlane(inc_items, at) - (nb - nth) * g.Hkv + w.head;
      if (item >= g.blocks) return false;  // (offsets that are not ascending)
      w.row0 = (nb - 1 - nth) * kRows;
      span_of(g, w);
      w.p0 = (int)((int64_t)w.nt * piece / np);
      w.p1 = (int)((int64_t)w.nt * (piece + 1) / np);
      w.slot = np > 1 ? id : -1;
      if (piece == 0 && threadIdx.x == 0) {
        g.joins[2 * item] = int4{np, id, w.head, w.row0};
        g.joins[2 * item + 1] = int4{w.rows, (int)w.q0, 0, 0};
      }
      return true;
    }
    before += __builtin_amdgcn_readlane(inc, 63);
    items += __builtin_amdgcn_readlane(inc_items, 63);
  }
  // the launch has one workgroup more than there can be pieces, which tells the join how many blocks there are
  if (id == slots && threadIdx.x == 0) *g.n_joins = before <= slots && items <= g.blocks ? items : 0;
  return false;
}

// The maximum and the sum of lanes l and l ^ 32 (see max4_xor16_32).
__device__ __forceinline__ float max2_xor32(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum2_xor32(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// ---------------------------------------------------------------- sizes, LDS layout, operand offsets
constexpr int kWaves = kRows / 32, kThreads = 64 * kWaves;  // a wave has 32 rows, the columns of its products
template <int DQK, int DV, int KIND>  // KIND 0: contiguous bf16, 1: paged bf16, 2: paged fp8
struct Prompt {
  static constexpr bool FP8 = KIND == 2;
  static constexpr int CK = DQK / 8, CV = DV / 8, KS = DQK / 16, DB = DV / 32;
  static constexpr int kK = kKeys * DQK * 2, kV = kKeys * DV * 2;  // bytes of a tile
  static constexpr int kLoadsK = kK / 512 / kWaves, kLoadsV = kV / 512 / kWaves;   // direct loads of a wave, keys or values
  // Tile buffers. Step i reads keys i and i + 1 and values i, while tiles up to i + kLead are on their way: as many as fit. Of fp8
  // caches tile i + 2 is written in bf16 meanwhile, from the kRaw buffers that the tiles up to i + 2 + kRaw come into.
  static constexpr int kLead = FP8 || DQK == 192 ? 2 : 3, kBufs = kLead + 1, kRaw = 3;
  struct Lds {
    uint8_t k[kBufs][kK], v[kBufs][kV];
    uint8_t raw[FP8 ? kRaw : 1][FP8 ? kK : 16];  // of fp8 tiles the keys, then the values
    float raw_scales[FP8 ? kRaw : 1][2][FP8 ? kKeys : 4];
    float scales[FP8 ? kBufs : 1][2][FP8 ? kKeys : 4];  // of keys (times the softmax scale) and of values
    int pages[KIND ? kPageSlots : 1];
  };
  // LDS offsets of this lane's operands in a tile: of K at k-step 0 (at s: ^ 32 s, or by 4 k-steps), of the first four and of the second four values
  // of a k-step in block 0 (in d: ^ 64 d).
  int k_off, v_off[2];
  __device__ __forceinline__ explicit Prompt(int lane) {
    const int h = lane >> 5, l32 = lane & 31, i = lane & 15, cc = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    k_off = l32 * DQK * 2 + ((h ^ swz<CK>(l32)) << 4);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = 8 * half + 4 * h + (i >> 2);
      v_off[half] = row * DV * 2 + ((cc ^ swz<CV>(row)) << 4) + 8 * (i & 1);
    }
  }
  // (in a loop over tiles: the operands' addresses are made from these where they are used, one instruction each; kept over the loop,
  // as the compiler would have them, they take the registers of the accumulators)
  __device__ __forceinline__ void refresh() { asm volatile("" : "+v"(k_off), "+v"(v_off[0]), "+v"(v_off[1])); }
  // The K operand of a k-step, and the V operand of a block of 32 dims: `at` is the LDS address of the tile's half (a multiple of
  // 256, and a row starts at a multiple of what the exclusive or reaches) and for V of the k-step's first key.
  __device__ __forceinline__ u32x4 k_operand(uint32_t at, int s) const {
    constexpr int X = CK == 16 ? 8 : 4;  // k-steps that the exclusive or of the chunks reaches
    const uint32_t p = ((at + (uint32_t)k_off) ^ (uint32_t)(32 * (s % X))) + 32 * X * (s / X);
    return *(const __attribute__((address_space(3))) u32x4*)(p);
  }
  __device__ __forceinline__ u32x4 v_operand(uint32_t at, int ks, int d) const {
    u32x2 y[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t p = ((at + (uint32_t)v_off[half]) ^ (uint32_t)(64 * d)) + 16 * ks * DV * 2;
      y[half] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
    }
    return u32x4{y[0].x, y[0].y, y[1].x, y[1].y};
  }
};

// x, made anew here: what is computed from it is not kept in registers over the loop around it.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

__device__ __forceinline__ const uint8_t* uniform_ptr(const uint8_t* p) {
  const uint64_t x = (uint64_t)(uintptr_t)p;
  return (const uint8_t*)(uintptr_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// A bf16 cache's weight exponent: s scale - m in one rounding. That leaves the largest score's at m's rounding error, the same for all
// keys of a row, which cancels; but from scores of 2^28 on it may overflow, and the careful form takes both roundings.
constexpr float kFarScore = 268435456.f;

// The first n of 32 bits.
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

__device__ __forceinline__ float scaled_below(float s, float scale, float m) {
#pragma clang fp contract(off)
  const float z = s * scale;
  return z - m;
}

// This lane's query row.
template <int KS>
struct Query {
  u32x4 q[KS];  // B operands: columns are rows, dims of k-step s
  int t;        // position of the row's token, -1 and less: none
};
template <int DQK>
__device__ __forceinline__ Query<DQK / 16> load_query(const PromptGeom& g, const Share& w, int wrow, int lane) {
  Query<DQK / 16> x;
  const int group = (int)g.by_group.d;
  const int row = wrow + (lane & 31), r = row < w.rows ? row : w.rows - 1, j = fdiv(g.by_group, r);
  x.t = g.causal ? w.c - w.n + j : w.c - 1;
  const uint16_t* p = g.q + (w.q0 + j) * g.q_stride + (int64_t)(w.head * group + r - j * group) * DQK + 8 * (lane >> 5);
#pragma unroll
  for (int s = 0; s < DQK / 16; ++s) x.q[s] = *reinterpret_cast<const u32x4*>(p + 16 * s);
  return x;
}
// They have arrived here: the compiler would wait for them where it first uses them, in a loop at every turn, and for the direct
// loads, of which it does not know, with them.
template <int KS>
__device__ __forceinline__ void arrived(Query<KS>& x) {
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(x.q[s]));
}

// Which of the 32 keys from s0 on the query at t attends to, of those in `there`.
__device__ __forceinline__ uint32_t sees32(const PromptGeom& g, int t, int s0, uint32_t there) {
  const int rel = t - s0;  // (-2^30 and less only where t is: s0 is a position)
  uint32_t m = first_bits(rel + 1) & there;
  if (g.k_swa > 0) m &= ~first_bits(rel - g.k_swa + 1) | first_bits(g.k_sink - s0);
  return m;
}

// ---------------------------------------------------------------- output
template <int DV>
__device__ __forceinline__ void store_row(const PromptGeom& g, const Share& w, int wrow, int lane, const f32x16 (&o)[DV / 32], float m, float l) {
  const int group = (int)g.by_group.d, h = lane >> 5;
  const int row = wrow + (lane & 31);
  const float sum = sum2_xor32(l), inv = 1.f / sum;
  const bool in = row < w.rows;
  if (w.slot >= 0) {
    if (!in) return;
    const int64_t at = (int64_t)w.slot * g.slot_rows + row - w.row0;
    if (h == 0) *reinterpret_cast<f32x2*>(g.part_ml + 2 * at) = f32x2{m, sum};
#pragma unroll
    for (int d = 0; d < DV / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<f32x4*>(g.part_o + at * DV + 32 * d + 2 * r + 4 * h) = f32x4{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
    return;
  }
  const int j = fdiv(g.by_group, row);
  const int64_t at = (w.q0 + j) * g.H + w.head * group + row - j * group;
  if (g.lse && in && h == 0) g.lse[at] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2;
#pragma unroll
  for (int d = 0; d < DV / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 8) {
      // dims 2 r + 4 h and 2 r + 8 + 4 h, four each: swapped with lane l ^ 32 into eight from 2 r + 8 h on
      uint32_t y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        y[k] = pack_bf16x2(sum == 0.f ? 0.f : o[d][r + 2 * k] * inv, sum == 0.f ? 0.f : o[d][r + 2 * k + 1] * inv);
      const auto lo = __builtin_amdgcn_permlane32_swap(y[0], y[2], false, false), hi = __builtin_amdgcn_permlane32_swap(y[1], y[3], false, false);
      if (in) *reinterpret_cast<u32x4*>(g.out + at * DV + 32 * d + 2 * r + 8 * h) = u32x4{lo[0], hi[0], lo[1], hi[1]};
    }
}

// The pieces of a block joined: o = sum_k 2^(m_k - m) o_k / sum_k 2^(m_k - m) l_k. Workgroup (i, y) takes rows of block y, DV / 4 threads
// a row of few pieces, and four times as many a row of more, each of which joins every fourth piece, kJoinAhead of them at a time: what few
// rows of many pieces wait for is the chain of loads (16 tokens behind 32K, 31 pieces: 3.4 us from its start to its end, one group of threads and one piece after the
// other 5 and more). With 8 pieces at a time 4 tokens behind 100K, 256 pieces, 30.7 against 33.4 us in all, but 512 behind 8K, few pieces
// of many rows, 106 against 97.
constexpr int kJoinGroups = 4, kJoinAhead = 4;  // (pieces that a thread loads at a time)
template <int DV>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptGeom g) {
  constexpr int T = DV / 4, kR = 256 / (T * kJoinGroups);
  __shared__ float part[kJoinGroups][kR][2];
  __shared__ f32x4 part_o[kJoinGroups][kR][T];
  const int item = blockIdx.y, n = *g.n_joins;
  const int4 a = g.joins[2 * item], b = g.joins[2 * item + 1];  // (of an item that is none: whatever was there)
  if (item >= n) return;
  const int np = a.x, groups = np <= kJoinAhead ? 1 : kJoinGroups, R = kR * kJoinGroups / groups;  // (rows at a time)
  const int x = (int)threadIdx.x % T, grp = (int)threadIdx.x / T & (groups - 1), lr = (int)threadIdx.x / (T * groups);
  const int row0 = a.w, rows = b.x - row0 < kRows ? b.x - row0 : kRows, d = 4 * x;
  if (np <= 1) return;
  const int64_t step = (int64_t)g.slot_rows * g.Hkv;  // from a piece to the next
  const int group = (int)g.by_group.d;
  for (int r0 = (int)blockIdx.x * R; r0 < rows; r0 += (int)gridDim.x * R) {
    const int r = r0 + lr, row = row0 + r;
    const bool in = r < rows;
    const int64_t at = (int64_t)a.y * g.slot_rows + (in ? r : r0);
    const f32x2* ml = reinterpret_cast<const f32x2*>(g.part_ml) + at;
    float top = kNoRef, sum = 0.f;
    f32x4 y{};
    for (int k0 = grp; k0 < np; k0 += groups * kJoinAhead) {
      f32x2 z[kJoinAhead];
      f32x4 o[kJoinAhead];
#pragma unroll
      for (int e = 0; e < kJoinAhead; ++e) {
        const int k = k0 + groups * e;
        z[e] = f32x2{kNoRef, 0.f};
        o[e] = f32x4{};
        if (k < np) {
          z[e] = ml[k * step];
          o[e] = *reinterpret_cast<const f32x4*>(g.part_o + (at + k * step) * DV + d);
        }
      }
      float tn = top;
#pragma unroll
      for (int e = 0; e < kJoinAhead; ++e) tn = fmaxf(tn, z[e].x);
      const float f0 = fast_exp2(top - tn);
      top = tn;
      sum *= f0;
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] *= f0;
#pragma unroll
      for (int e = 0; e < kJoinAhead; ++e) {
        const float f = fast_exp2(z[e].x - top);
        sum += f * z[e].y;
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] += f * o[e][q];
      }
    }
    if (groups > 1) {
      __syncthreads();  // everyone is done with the rows before
      if (x == 0) {
        part[grp][lr][0] = top;
        part[grp][lr][1] = sum;
      }
      part_o[grp][lr][x] = y;
      __syncthreads();
      if (grp != 0) continue;
#pragma unroll
      for (int k = 1; k < kJoinGroups; ++k) top = fmaxf(top, part[k][lr][0]);
      sum = 0.f;
      y = f32x4{};
#pragma unroll
      for (int k = 0; k < kJoinGroups; ++k) {
        const float f = fast_exp2(part[k][lr][0] - top);
        sum += f * part[k][lr][1];
        const f32x4 o = part_o[k][lr][x];
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] += f * o[q];
      }
    }
    if (!in) continue;
    const int j = fdiv(g.by_group, row);
    const int64_t to = ((int64_t)b.y + j) * g.H + a.z * group + row - j * group;
    if (g.lse && x == 0) g.lse[to] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    const float inv = 1.f / sum;
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = sum == 0.f ? 0.f : y[q] * inv;
    *reinterpret_cast<u32x2*>(g.out + to * DV + d) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  }
}

// ---------------------------------------------------------------- items with values that are no finite numbers
// A weight of 0 does not silence a NaN or an infinity in V, and a tile is multiplied whole. So an item whose outputs are not all
// finite is done again here, a tile at a time, with such values taken out of the product and added to the rows that attend to them
// (and to no others). Nothing else takes this way: it is written to be right, not fast.
template <int DQK, int DV, int KIND>
__device__ __forceinline__ void careful_item(const PromptGeom& g, const Share& w, typename Prompt<DQK, DV, KIND>::Lds& lds) {
  using T = Prompt<DQK, DV, KIND>;
  constexpr int KS = T::KS, DB = T::DB;
  constexpr bool FP8 = T::FP8;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
  const int wrow = w.row0 + 32 * wave;
  const bool active = wrow < w.rows;
  T f(lane);
  const Query<KS> x = load_query<DQK>(g, w, wrow, lane);
  f32x16 o[DB];
  float m = kNoRef, l = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16{};
  uint8_t *lk = lds.k[0], *lv = lds.v[0];
  for (int i = w.p0; i < w.p1; ++i) {
    const int s0 = (i < w.ns ? i : i + w.skip) * kKeys;
    __syncthreads();
    // row of the cache (or of the sequence's packed keys) of a key, -1: none
    auto row_of = [&](int key) -> int64_t {
      const uint32_t s = (uint32_t)s0 + key;
      if (s >= (uint32_t)w.c) return -1;
      if constexpr (KIND == 0) return w.kv0 + s;
      const int pg = fdiv(g.by_page, (int)s);
      const int64_t ph = g.page_table ? g.page_table[(int64_t)w.b * g.max_pages + pg] : w.b;
      return ph >= 0 && ph < g.n_phys ? (ph * g.Hkv + w.head) * g.P + ((int)s - pg * g.P) : -1;
    };
    auto load = [&](const void* base, int64_t stride, uint8_t* dst, auto width) {
      constexpr int D = decltype(width)::value, C = D / 8;
      for (int e = (int)threadIdx.x; e < kKeys * C; e += kThreads) {
        const int r = e / C, c = e % C;
        const int64_t row = row_of(r);
        u32x4 y{};
        if (row >= 0 && !FP8) y = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + row * stride + 8 * c);
        if (row >= 0 && FP8) {
          const u32x2 z = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(base) + row * D + 8 * c);
          y = fp8x8_bf16(z.x, z.y);
        }
        *reinterpret_cast<u32x4*>(dst + r * D * 2 + ((c ^ swz<C>(r)) << 4)) = y;
      }
    };
    load(KIND ? g.k : static_cast<const void*>(static_cast<const uint16_t*>(g.k) + w.head * DQK), KIND ? DQK : g.k_stride, lk,
         std::integral_constant<int, DQK>{});
    load(KIND ? g.v : static_cast<const void*>(static_cast<const uint16_t*>(g.v) + w.head * DV), KIND ? DV : g.v_stride, lv,
         std::integral_constant<int, DV>{});
    const int64_t own = row_of(lane);
    if constexpr (FP8) {
      if (wave == 0) {
        lds.scales[0][0][lane] = own >= 0 ? g.k_scale[own] * g.scale_log2 : 0.f;
        lds.scales[0][1][lane] = own >= 0 ? g.v_scale[own] : 0.f;
      }
    }
    __syncthreads();
    if (!active) continue;
    const uint64_t there = __ballot(own >= 0);
#pragma nounroll
    for (int kb = 0; kb < 2; ++kb) {  // (halves of a tile and sums in the order of the steps below: other rows keep their bits)
      f.refresh();
      f32x16 s{};
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const u32x4 a = f.k_operand((uint32_t)(uintptr_t)lk + kb * 32 * DQK * 2, st);
        s = mfma32(a, x.q[st], s);
      }
      u32x4 p[2];     // [k-step of 16]
      float top = -INFINITY;
      const uint32_t seen = sees32(g, x.t, s0 + 32 * kb, (uint32_t)(there >> (32 * kb))) >> (4 * h);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r >> 2) + (r & 3);
        if constexpr (FP8) s[r] *= lds.scales[0][0][32 * kb + 4 * h + key];
        s[r] = (seen >> key) & 1 ? s[r] : -INFINITY;
        top = fmaxf(top, s[r]);
      }
      top = max2_xor32(FP8 ? top : top * g.scale_log2);
      if (top > m + kLazy) {
        const float al = fast_exp2(m - top);
        m = top;
        l *= al;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= al;
      }
      uint32_t live = 0;  // scores that are not -inf
      const bool far = !(fabsf(m) < kFarScore) && m != kNoRef;
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float e[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float z = s[r + k];
          const bool in = z != -INFINITY;
          if (in) live |= 1u << (r + k);
          e[k] = fast_exp2(FP8 ? z - m : far ? scaled_below(z, g.scale_log2, m) : fmaf(z, g.scale_log2, -m));
          l += e[k];
          if constexpr (FP8) e[k] = in ? e[k] * lds.scales[0][1][32 * kb + 8 * (r >> 2) + 4 * h + ((r + k) & 3)] : 0.f;
        }
        p[r >> 3][(r & 7) >> 1] = pack_bf16x2(e[0], e[1]);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const u32x4 a = f.v_operand((uint32_t)(uintptr_t)lv + 32 * kb * DV * 2, ks, d);
          u32x4 up{}, down{}, fin = a;  // 1 where a value is +inf or NaN, -inf or NaN; the others
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t v = (a[k] >> (16 * half)) & 0xFFFFu, one = 0x3F80u << (16 * half);
              const bool odd = (v & 0x7F80u) == 0x7F80u, nan = odd && (v & 0x7Fu) != 0;
              fin[k] &= odd ? (half ? 0xFFFFu : 0xFFFF0000u) : ~0u;
              up[k] |= nan || (odd && !(v & 0x8000u)) ? one : 0u;
              down[k] |= nan || (odd && (v & 0x8000u)) ? one : 0u;
            }
          u32x4 one;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t bits = live >> (8 * ks + 2 * k);
            one[k] = (bits & 1 ? 0x3F80u : 0u) | (bits & 2 ? 0x3F800000u : 0u);
          }
          o[d] = mfma32(fin, p[ks], o[d]);
          const f32x16 plus = mfma32(up, one, f32x16{}), minus = mfma32(down, one, f32x16{});
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            o[d][r] += plus[r] > 0.f ? INFINITY : 0.f;
            o[d][r] -= minus[r] > 0.f ? INFINITY : 0.f;
          }
        }
    }
  }
  if (active) store_row<DV>(g, w, wrow, lane, o, m, l);
}

// ---------------------------------------------------------------- direct loads of tiles
// N direct loads of a tile's rows: load j takes base + off[j] + 1024 (j % 4) per lane to LDS bytes lds + 1024 j + 16 lane (the
// immediate offset, less than 4096, counts for both addresses).
template <int N>
__device__ __forceinline__ void lds_dma16_tile(const uint8_t* base, const uint32_t* off, uint32_t lds) {
  if constexpr (N > 4) {
    lds_dma16_tile<4>(base, off, lds);
    lds_dma16_tile<N - 4>(base, off + 4, lds + 4096);
    return;
  }
  uint32_t save;
  if constexpr (N == 4)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:2048\n\tglobal_load_lds_dwordx4 %5, %1 offset:3*1024\n\ts_mov_b32 m0, %0"
                 : "=&s"(save) : "s"(base), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(lds) : "memory");
  else if constexpr (N == 3)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:2048\n\ts_mov_b32 m0, %0"
                 : "=&s"(save) : "s"(base), "v"(off[0]), "v"(off[1]), "v"(off[2]), "s"(lds) : "memory");
  else if constexpr (N == 2)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\ts_mov_b32 m0, %0"
                 : "=&s"(save) : "s"(base), "v"(off[0]), "v"(off[1]), "s"(lds) : "memory");
  else if constexpr (N == 1)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\ts_mov_b32 m0, %0"
                 : "=&s"(save) : "s"(base), "v"(off[0]), "s"(lds) : "memory");
}
// Wait until at most N direct loads of this wave are on their way and its LDS reads are done, then join the barrier.
template <int N>
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Heads of 64 in bf16 run two workgroups per CU, four waves per SIMD. What does not fit their 128 registers is spilled: of the careful form, and over a paged
// cache also a few addresses of the load path and one register of the masked tiles; not those of fp8 caches, whose products' operands would be. us with two waves
// per SIMD and with four. Packed: 12 heads, 8192 x 8192 keys 771, 678, window of 1024 81, 68. Paged, 32 heads on 8: 24 sequences mixed 137, 129; 8192 behind 8K
// 984, 870; 4096 behind 60K 2500, 2260; 4096 of four behind 16K 215, 205; 8 of one token behind 16K 106, 65; 2048 behind 6K 178, 178; 512 behind 4K 42, 44; 16
// behind 32K 28.7, 29.8; 300 alone 13.3, 14.6; 12 on 12, 8192 alone 169, 177. In fp8, 24 mixed: 181, 472.
constexpr int waves_per_simd(int d_qk, int kind) { return d_qk == 64 && kind != 2 ? 4 : 2; }
template <int DQK, int DV, int KIND>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(waves_per_simd(DQK, KIND), waves_per_simd(DQK, KIND)))) void prompt_attn_kernel(PromptGeom g) {
  using T = Prompt<DQK, DV, KIND>;
  constexpr int KS = T::KS, DB = T::DB, NB = T::kBufs, NR = T::kRaw;
  constexpr bool FP8 = T::FP8;
  __shared__ __attribute__((aligned(1024))) typename T::Lds lds;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
  Share w;
  if (!(g.pieces ? find_piece(g, (int)blockIdx.x, w) : find_whole(g, g.first + (int)blockIdx.x, w))) return;
  const int wrow = w.row0 + 32 * wave;
  const bool active = wrow < w.rows;
  T f(lane);
  Query<KS> x;
  bool fresh = true;
  // positions of the wave's first and last token
  const int wlast = (w.rows - wrow < 32 ? w.rows : wrow + 32) - 1;
  const int t_first = !active ? -1 : g.causal ? w.c - w.n + fdiv(g.by_group, wrow) : w.c - 1;
  const int t_last = !active ? -1 : g.causal ? w.c - w.n + fdiv(g.by_group, wlast) : w.c - 1;
  f32x16 o[DB];
  float m = kNoRef, l = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16{};

  const bool whole_tiles = KIND == 0 || g.P % kKeys == 0;  // (no tile lies in two pages)
  const int64_t row_k = KIND ? DQK * (FP8 ? 1 : 2) : g.k_stride * 2, row_v = KIND ? DV * (FP8 ? 1 : 2) : g.v_stride * 2;  // bytes
  const uint8_t* const base_k = static_cast<const uint8_t*>(g.k) + (KIND ? 0 : w.head * DQK * 2 + w.kv0 * row_k);
  const uint8_t* const base_v = static_cast<const uint8_t*>(g.v) + (KIND ? 0 : w.head * DV * 2 + w.kv0 * row_v);
  // Direct loads: half the waves load the keys of a tile, half the values; load j of a wave fills slots 64 (loads part + j) + lane.
  constexpr int LK = T::kLoadsK, LV = T::kLoadsV, LM = LK > LV ? LK : LV;
  const bool loads_k = wave < kWaves / 2;
  const int part = wave % (kWaves / 2);
  const uint8_t* const base = loads_k ? base_k : base_v;
  const int64_t row_bytes = loads_k ? row_k : row_v;
  auto slot_of = [&](int j, int ln, int& r) {  // byte of its row that the slot of load j and lane ln holds
    const int e = 64 * ((loads_k ? LK : LV) * part + j) + ln;
    r = loads_k ? e / T::CK : e / T::CV;
    return loads_k ? ((e % T::CK) ^ swz<T::CK>(r)) << 4 : ((e % T::CV) ^ swz<T::CV>(r)) << 4;
  };
  uint32_t dma[LM];
  if constexpr (!FP8) {
#pragma unroll
    for (int j = 0; j < LM; ++j) {
      int r;
      const int c = slot_of(j, lane, r);
      dma[j] = (uint32_t)(r * (int)row_bytes + c) - 1024 * (j & 3);
    }
  }
  const uint32_t lds_k = (uint32_t)(uintptr_t)&lds.k[0][0], lds_v = (uint32_t)(uintptr_t)&lds.v[0][0];
  auto next_k = [&](uint32_t at) { return at + T::kK == lds_k + NB * T::kK ? lds_k : at + T::kK; };
  auto next_v = [&](uint32_t at) { return at + T::kV == lds_v + NB * T::kV ? lds_v : at + T::kV; };

  // Tiles [a, b) of the sequence, the pages of which (from page f1 on) are in LDS; mapped: none of them is missing.
  auto run = [&](int a, int b, int f1, bool mapped) {
    auto row_of = [&](int tile) {  // row of key `lane` of a tile, -1: none
      const uint32_t s = (uint32_t)tile * kKeys + lane;
      if (s >= (uint32_t)w.c) return -1;
      if constexpr (KIND == 0) return (int)s;
      const int pg = fdiv(g.by_page, (int)s), ph = lds.pages[pg - f1];
      return ph >= 0 ? (ph * g.Hkv + w.head) * g.P + ((int)s - pg * g.P) : -1;
    };
    // The tile to be loaded next, where tiles do not lie in two pages and every page is mapped: it starts at row `off` of page `ph`
    // (read a step before it is used).
    const int start = a * kKeys, pg0 = KIND ? fdiv(g.by_page, start) : 0;
    int off = KIND ? start - pg0 * g.P : start, entry = pg0 - f1, ph = KIND ? lds.pages[entry] : 0;
    // the first row of tile a + i, which is next; -1: its rows are to be looked up one by one
    auto next_rows = [&](int i) {
      int row = -1;
      if (whole_tiles) {
        if (mapped && (uint32_t)(a + i + 1) * kKeys <= (uint32_t)w.c) row = KIND ? (uniform(ph) * g.Hkv + w.head) * g.P + off : off;
        off += kKeys;
        if (KIND != 0 && off == g.P) {
          off = 0;
          ++entry;
        }
        if constexpr (KIND != 0) ph = lds.pages[entry];  // (behind the last tile: an entry that is not used)
      }
      return row;
    };

    // -- bf16: tile a + i by direct loads into its buffers
    uint32_t ring = loads_k ? lds_k : lds_v;  // of the next tile to be loaded
    auto issue = [&](int i) {
      const int row0 = next_rows(i);
      const uint32_t to = (uint32_t)uniform((int)(ring + part * (loads_k ? LK : LV) * 1024));
      ring = loads_k ? next_k(ring) : next_v(ring);
      if (row0 >= 0) {
        const uint8_t* from = uniform_ptr(base + (int64_t)row0 * row_bytes);
        if (LK == LV || loads_k) lds_dma16_tile<LK>(from, dma, to);
        else lds_dma16_tile<LV>(from, dma, to);
        return;
      }
      const int ln = here(lane), own = row_of(a + i);
#pragma unroll
      for (int j = 0; j < LM; ++j) {
        if (j >= (loads_k ? LK : LV)) break;
        int r;
        const int c = slot_of(j, ln, r), row = __shfl(own, r & 63);
        lds_dma16(row >= 0 ? base + (int64_t)(uint32_t)row * row_bytes + c : zero_row, to + j * 1024);
      }
    };
    // -- fp8: tile a + i by direct loads as it is, and from there in bf16 into its buffers; a thread converts what it has loaded itself
    constexpr int kUnits = kKeys * DQK / 16, RL = FP8 ? 2 * kUnits / kThreads : 1;  // 16-byte units of a tile's keys or values; loads of a wave
    static_assert(!FP8 || RL * kThreads == 2 * kUnits, "whole loads");
    auto unit_of = [&](int j, bool& keys) {
      const int e = kThreads * j + (int)threadIdx.x;
      keys = RL == 2 ? j == 0 : wave < kWaves / 2;
      return e % kUnits;
    };
    auto fetch = [&](int i) {
      const int row0 = next_rows(i), own = row0 >= 0 ? row0 + lane : row_of(a + i);
      const int slot = i % NR;
      const uint32_t to = (uint32_t)uniform((int)((uint32_t)(uintptr_t)&lds.raw[slot][0] + 1024 * wave));
#pragma unroll
      for (int j = 0; j < RL; ++j) {
        bool keys;
        const int u = unit_of(j, keys);
        const uint8_t* const from = keys ? base_k : base_v;
        if (row0 >= 0) {
          const uint32_t byte = 16 * u;
          lds_dma16_tile<1>(uniform_ptr(from + (int64_t)row0 * DQK), &byte, to + 1024 * kWaves * j);
        } else {
          const int row = __shfl(own, u / (DQK / 16));
          lds_dma16(row >= 0 ? from + (int64_t)row * DQK + 16 * (u % (DQK / 16)) : zero_row, to + 1024 * kWaves * j);
        }
      }
      if (wave < 2)
        lds_dma4(own >= 0 ? reinterpret_cast<const uint8_t*>((wave == 0 ? g.k_scale : g.v_scale) + own) : zero_row,
                 (uint32_t)uniform((int)(uint32_t)(uintptr_t)&lds.raw_scales[slot][wave & 1][0]));
    };
    auto commit = [&](int i) {
      const int slot = i % NR;
#pragma unroll
      for (int j = 0; j < RL; ++j) {
        bool keys;
        const int u = unit_of(j, keys), r = u / (DQK / 16), c = 2 * (u % (DQK / 16));
        const u32x4 y = *reinterpret_cast<const u32x4*>(&lds.raw[slot][16 * (kThreads * j + (int)threadIdx.x)]);
        uint8_t* const to = (keys ? lds.k[i % NB] : lds.v[i % NB]) + r * DQK * 2;
        *reinterpret_cast<u32x4*>(to + ((c ^ swz<T::CK>(r)) << 4)) = fp8x8_bf16(y.x, y.y);
        *reinterpret_cast<u32x4*>(to + (((c + 1) ^ swz<T::CK>(r)) << 4)) = fp8x8_bf16(y.z, y.w);
      }
      if (wave < 2) {
        const float y = lds.raw_scales[slot][wave][lane];
        lds.scales[i % NB][wave][lane] = wave == 0 ? y * g.scale_log2 : y;
      }
    };

    const int nt = b - a;
    // the tiles that some row of this wave attends to are the first nw
    const int seen_end = t_last < 0 ? 0 : t_last / kKeys + 1;
    const int nw = seen_end <= a ? 0 : seen_end < b ? seen_end - a : nt;

    // -- the pieces of a step, which takes half a tile: keys 32 kb .. + 31
    // The operands of a product are read from LDS while the one before runs: those of KA k-steps of the scores (all, where the
    // registers allow it), and all of the values.
    constexpr int KA = DQK == 192 ? 6 : KS;
    u32x4 kf[KA], vf[2][DB];
    auto load_k = [&](uint32_t lk) {
#pragma unroll
      for (int st = 0; st < KA; ++st) kf[st] = f.k_operand(lk, st);
    };
    auto load_v = [&](uint32_t lv) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < DB; ++d) vf[ks][d] = f.v_operand(lv, ks, d);
    };
    auto scores = [&](uint32_t lk, f32x16& s) {
      s = f32x16{};
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const u32x4 y = st < KA ? kf[st < KA ? st : 0] : f.k_operand(lk, st);
        s = mfma32(y, x.q[st], s);
      }
    };
    u32x4 p[2];  // weights: B operands of k-steps of 16
    auto values = [&] {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < DB; ++d)
          o[d] = mfma32(vf[ks][d], p[ks], o[d]);
    };
    // the scores' maximum per row, in base-2 units (those of an fp8 cache with the keys' scales first)
    auto scale_max = [&](int i, int kb, f32x16& s, float& top) {
      f32x4 sc[4];
      if constexpr (FP8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[k] = *reinterpret_cast<const f32x4*>(&lds.scales[i % NB][0][32 * kb + 8 * k + 4 * h]);
      }
      top = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (FP8) s[r] *= sc[r >> 2][r & 3];
        top = fmaxf(top, s[r]);
      }
    };
    // the same of those that the rows attend to (a path of its own beside the products, so that these exist once)
    auto mask = [&](int i, int kb, f32x16& s, float& top) {
      const uint32_t keys = (uint32_t)(__ballot(row_of(a + i) >= 0) >> (32 * kb));
      top = -INFINITY;
      const uint32_t seen = sees32(g, x.t, (a + i) * kKeys + 32 * kb, keys) >> (4 * h);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = (seen >> (8 * (r >> 2) + (r & 3))) & 1 ? s[r] : -INFINITY;
        top = fmaxf(top, s[r]);
      }
    };
    auto rescale = [&](float& top) {
      top = max2_xor32(FP8 ? top : top * g.scale_log2);
      const bool grown = top > m + kLazy;
      if (__any(grown)) {
        // (each row by its own scores, whatever the wave's others do)
        const float mn = grown ? top : m, al = fast_exp2(m - mn);
        m = mn;
        l *= al;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= al;
      }
    };
    // The weights, rounded to bf16 for the product with V (half a step, 2^-8, of each; their sum l takes them as they are in fp32): one product in place of the
    // two that their high and low halves would need. It moves an output's relative error from 1.7e-3, which its own rounding makes, to 2.2e-3. Those of an fp8
    // cache are multiplied by the values' scales first, so that there is one rounding too.
    auto weights = [&](int i, int kb, const f32x16& s) {
      f32x4 sc[4];
      if constexpr (FP8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[k] = *reinterpret_cast<const f32x4*>(&lds.scales[i % NB][1][32 * kb + 8 * k + 4 * h]);
      }
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float e0 = fast_exp2(FP8 ? s[r] - m : fmaf(s[r], g.scale_log2, -m));
        float e1 = fast_exp2(FP8 ? s[r + 1] - m : fmaf(s[r + 1], g.scale_log2, -m));
        l += e0;
        l += e1;
        if constexpr (FP8) {
          e0 *= sc[r >> 2][r & 3];
          e1 *= sc[r >> 2][(r & 3) + 1];
        }
        p[r >> 3][(r & 7) >> 1] = pack_bf16x2(e0, e1);
      }
    };
    auto is_clear = [&](int i) {  // every row of the wave attends to every key of tile a + i
      const int s0 = (a + i) * kKeys;
      return mapped && s0 <= t_first - (kKeys - 1) && (g.k_swa == 0 || s0 > t_last - g.k_swa || s0 <= g.k_sink - kKeys);
    };
    // start of step i: tile i + 1 has arrived, everyone is done with tile i - 1 (and the first half of keys i); tile i + kLead sets out
    constexpr int LEAD = T::kLead;
    auto wait = [&](auto tiles) {  // until at most so many tiles are on their way
      constexpr int N = decltype(tiles)::value;
      if constexpr (FP8) {  // (and tile i + 2 as it is)
        if (wave < 2) tile_barrier<N * (RL + 1)>();
        else tile_barrier<N * RL>();
      } else if (LK == LV || loads_k) tile_barrier<N * LK>();
      else tile_barrier<N * LV>();
    };
    auto advance = [&](int i) {
      if constexpr (FP8) {
        if (i + 1 + NR < nt) wait(std::integral_constant<int, NR - 1>{});
        else wait(std::integral_constant<int, 0>{});
        if (i + 2 < nt) commit(i + 2);
        if (i + 2 + NR < nt) fetch(i + 2 + NR);
      } else {
        if (i + LEAD - 1 < nt) wait(std::integral_constant<int, LEAD - 2>{});
        else wait(std::integral_constant<int, 0>{});
        if (i + LEAD < nt) issue(i + LEAD);
      }
    };

    // -- first tiles (the queries of a paged cache's call have set out with the first page table entries)
    if (KIND != 0 && fresh) arrived(x);
    if constexpr (FP8) {
      for (int i = 0; i < NR && i < nt; ++i) fetch(i);
      if (nt >= NR) wait(std::integral_constant<int, NR - 2>{});
      else wait(std::integral_constant<int, 0>{});
      for (int i = 0; i < 2 && i < nt; ++i) {
        commit(i);
        if (i + NR < nt) fetch(i + NR);
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    } else {
      issue(0);
      if (KIND == 0 && fresh) {
        x = load_query<DQK>(g, w, wrow, lane);
        arrived(x);
      }
      for (int i = 1; i < LEAD && i < nt; ++i) issue(i);
      if (nt >= LEAD) wait(std::integral_constant<int, LEAD - 1>{});
      else wait(std::integral_constant<int, 0>{});
    }
    fresh = false;
    f32x16 sa, sb;
    if (nw > 0) {
      load_k(lds_k);
      scores(lds_k, sa);
      load_v(lds_v + 32 * DV * 2);
    }
    // (before the first half there are no weights: zeros, on values that are there; and after the last one scores of what is left
    // in the buffers, which nobody reads)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      p[ks] = u32x4{};
    constexpr uint32_t HK = 32 * DQK * 2, HV = 32 * DV * 2;  // bytes of half a tile
    uint32_t kc = lds_k, vc = lds_v;                         // buffers of tile i
    for (int i = 0; i < nt; ++i) {
      advance(i);
      const uint32_t k = kc, v = vc;
      kc = next_k(kc);
      vc = next_v(vc);
      if (i >= nw) continue;
      f.refresh();
      const bool clear = is_clear(i);
      float top;
      load_k(k + HK);
      values();
      scale_max(i, 0, sa, top);
      if (!clear) mask(i, 0, sa, top);
      rescale(top);
      load_v(v);
      scores(k + HK, sb);
      weights(i, 0, sa);
      load_k(kc);
      values();
      scale_max(i, 1, sb, top);
      if (!clear) mask(i, 1, sb, top);
      rescale(top);
      load_v(v + HV);
      scores(kc, sa);
      weights(i, 1, sb);
    }
    if (nw > 0) values();
  };

  if constexpr (KIND != 0) x = load_query<DQK>(g, w, wrow, lane);
  // The span's two stretches of tiles, and of a paged cache as many at a time as their pages fit in LDS.
  for (int part = 0; part < 2; ++part) {
    const int first = part ? (w.p0 > w.ns ? w.p0 : w.ns) + w.skip : w.p0, last = part ? w.p1 + w.skip : (w.ns < w.p1 ? w.ns : w.p1);
    for (int a = first; a < last;) {
      int b = last, f1 = 0;
      bool mapped = true;
      __syncthreads();  // everyone is done with the buffers
      if constexpr (KIND != 0) {
        if (b - a > g.pass_tiles) b = a + g.pass_tiles;
        f1 = fdiv(g.by_page, a * kKeys);
        const int64_t end = (int64_t)b * kKeys - 1;
        const int n = fdiv(g.by_page, end < w.c ? (int)end : w.c - 1) - f1 + 1;
        bool missing = false;
        for (int i = (int)threadIdx.x; i < n; i += kThreads) {
          const int64_t ph = g.page_table ? g.page_table[(int64_t)w.b * g.max_pages + f1 + i] : w.b;
          const bool there = ph >= 0 && ph < g.n_phys;
          missing |= !there;
          lds.pages[i] = there ? (int)ph : -1;
        }
        mapped = !__syncthreads_or(missing);
      }
      run(a, b, f1, mapped);
      a = b;
    }
  }
  // (a value that is no finite number leaves every accumulator it was multiplied into so)
  float odd[4] = {};
  odd[0] = fmaf(l, 0.f, odd[0]);
  if (!FP8 && !(fabsf(m) < kFarScore) && m != kNoRef) odd[0] = 1.f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd[r & 3] = fmaf(o[d][r], 0.f, odd[r & 3]);
  if (__syncthreads_or((odd[0] + odd[1]) + (odd[2] + odd[3]) != 0.f)) {  // (NaN != 0)
    careful_item<DQK, DV, KIND>(g, w, lds);
    return;
  }
  if (active) store_row<DV>(g, w, wrow, lane, o, m, l);
}

hipError_t launch_prompt_attn(const PromptGeom& all, hipStream_t st) {
  PromptGeom g = all;
  auto* kernel = g.ctx_len == nullptr ? (g.d_qk == 64    ? prompt_attn_kernel<64, 64, 0>
                                         : g.d_qk == 128 ? prompt_attn_kernel<128, 128, 0>
                                                         : prompt_attn_kernel<192, 128, 0>)
                 : g.fp8 ? (g.d_qk == 64 ? prompt_attn_kernel<64, 64, 2> : prompt_attn_kernel<128, 128, 2>)
                         : (g.d_qk == 64 ? prompt_attn_kernel<64, 64, 1> : prompt_attn_kernel<128, 128, 1>);
  if (g.pieces) {
    hipError_t e = launch_kernel(kernel, dim3((unsigned)(g.pieces + g.blocks + 1)), dim3(kThreads), st, g);
    if (e != hipSuccess) return e;
    // (workgroups of a block: one for as many rows as it takes at a time, but few where there are many blocks, most of them whole. With 4096 / 8192 /
    // 32768 in all, us: prompts of 2048, none cut, 68.3 / 70.0 / 75.3, 24 sequences mixed 207 / 205 / 209)
    const int rows = 256 / (g.d_v / 4 * kJoinGroups), groups = (g.slot_rows + rows - 1) / rows, most = 4096 / g.blocks > 8 ? 4096 / g.blocks : 8;
    return launch_kernel(g.d_v == 64 ? prompt_join_kernel<64> : prompt_join_kernel<128>, dim3((unsigned)(groups < most ? groups : most), (unsigned)g.blocks),
                         dim3(256), st, g);
  }
  constexpr int64_t kMost = 1 << 22;  // workgroups of a launch (2^32 threads and more are taken modulo 2^32)
  for (int64_t i = 0; i < all.items; i += kMost) {
    g.first = (int)i;
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)(all.items - i < kMost ? all.items - i : kMost)), dim3(kThreads), st, g);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace lsa
