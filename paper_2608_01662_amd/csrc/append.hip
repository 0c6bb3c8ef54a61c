// Cache append with position rotation (lsa_cache_append) for gfx950: queries and keys rotated, keys and
// values written to their rows of a paged cache in bf16 or e4m3 with a scale per row.
//
// A thread takes 16 values of one head of one token: eight pairs of the rotated part (both halves of each
// pair, so that every input is loaded once), or 16 neighbours elsewhere. Nothing is shared between threads
// but the maximum of an fp8 row, an exchange within the lanes that hold the row.
//
// Six flops per rotated pair against 8 bytes: bound by HBM, from a few thousand tokens on; below that by the chain
// of round trips (position, page-table entry and angles, then rows) and the launch. Measured, GPU time alone: one token of 32
// fp8 indexer heads 3.3 us; 64 tokens of 64 latent heads 4.7; 4001 tokens of 32 heads on 8 in bf16 (100 MB) 18.4, 5.5 TB/s; 8192
// in fp8 (187 MB) 39.5, 4.7 TB/s; 32768 of 32 indexer heads (559 MB) 105, 5.3 TB/s, where a copy of 2 GiB reaches 5.0.
// (Non-temporal stores were 20% slower.)
#include "device.hpp"
#include "launch.hpp"

namespace lsa {

constexpr int kAppendThreads = 256;

// What token t of this launch is: its sequence and position (pos < 0: none).
struct AppendToken {
  int seq, pos;
};
__device__ __forceinline__ AppendToken append_token(const AppendGeom& g, int t) {
  AppendToken r;
  const int nth = g.tok0 + t, by_rows = fdiv(g.by_rows, nth);
  r.seq = g.seq ? g.seq[nth] : by_rows;
  if (r.seq < 0 || r.seq >= g.n_seq) return AppendToken{0, -1};
  const int rows = (int)g.by_rows.d;
  const int64_t p = g.pos ? g.pos[nth] : (int64_t)g.ctx_len[r.seq] - rows + (nth - by_rows * rows);
  const bool ok = p >= 0 && p < (int64_t)g.max_pages * g.P && (g.rot_dim == 0 || p < g.rope_rows);
  r.pos = ok ? (int)p : -1;
  return r;
}

__device__ __forceinline__ void unpack8(u32x4 v, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float* x) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// The 16 values of unit u of a head: dims `lo` .. + 7 and `hi` .. + 7.
struct Unit {
  int lo, hi, pair;  // pair: first pair of the rotated part, -1 outside it
};
__device__ __forceinline__ Unit unit_of(const AppendGeom& g, int u) {
  const int c = u - g.rot_start / 16;
  if (c < 0 || c >= g.rot_dim / 16) return Unit{16 * u, 16 * u + 8, -1};
  if (g.interleaved) return Unit{16 * u, 16 * u + 8, 8 * c};
  return Unit{g.rot_start + 8 * c, g.rot_start + g.rot_dim / 2 + 8 * c, 8 * c};
}

// The angles of a unit's pairs at a position.
struct Angles {
  f32x4 c0, c1, s0, s1;
};
__device__ __forceinline__ Angles load_angles(const AppendGeom& g, const Unit& u, int pos) {
  const f32x4* cs = reinterpret_cast<const f32x4*>(g.rope + (int64_t)pos * g.rot_dim + u.pair);
  const f32x4* sn = reinterpret_cast<const f32x4*>(g.rope + (int64_t)pos * g.rot_dim + g.rot_dim / 2 + u.pair);
  return Angles{cs[0], cs[1], sn[0], sn[1]};
}
// y[0..8) and y[8..16) are the values at dims lo and hi.
__device__ __forceinline__ void rotate(const AppendGeom& g, const Angles& an, float* y) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = i < 4 ? an.c0[i & 3] : an.c1[i & 3], s = i < 4 ? an.s0[i & 3] : an.s1[i & 3];
    const float a = g.interleaved ? y[2 * i] : y[i], b = g.interleaved ? y[2 * i + 1] : y[i + 8];
    const float ra = a * c - b * s, rb = b * c + a * s;
    if (g.interleaved) {
      y[2 * i] = ra;
      y[2 * i + 1] = rb;
    } else {
      y[i] = ra;
      y[i + 8] = rb;
    }
  }
}
// Where a unit of head `head` of token t lies: in x, or with the rotated dims apart in x or `part`.
__device__ __forceinline__ const uint16_t* unit_base(const AppendGeom& g, const uint16_t* x, int64_t stride, const uint16_t* part,
                                                     int64_t part_stride, int t, int head, const Unit& u) {
  if (part == nullptr) return x + (int64_t)t * stride + (int64_t)head * g.d_k;
  if (u.pair < 0) return x + (int64_t)t * stride + (int64_t)head * (g.d_k - g.rot_dim);
  return part + (int64_t)t * part_stride + (int64_t)head * g.rot_dim - g.rot_start;
}

// Eight values as e4m3 codes (round to nearest even; NaN stays NaN; |x| < 464).
__device__ __forceinline__ u32x2 pack_fp8x8(const float* x) {
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
  return u32x2{(uint32_t)lo, (uint32_t)hi};
}

// Blocks [0, bq) rotate queries, [bq, bq + bk) append keys, the rest values. A head's units are dealt to
// `lanes` neighbouring threads: as many as it has, or for fp8 rows the next power of two, so that the lanes
// of a row exchange their maximum within one wave.
template <int HEADS>  // query heads per thread
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendGeom g, int bq, int bk) {
  const int blk = (int)blockIdx.x;
  if (blk < bq) {
    const int item = blk * kAppendThreads + (int)threadIdx.x, vec = fdiv(g.by_q_units, item), t = fdiv(g.by_q_heads, vec);
    if (t >= g.n_tok) return;
    const AppendToken tok = append_token(g, t);
    const Unit u = unit_of(g, item - vec * (int)g.by_q_units.d);
    const int head = (vec - t * (int)g.by_q_heads.d) * HEADS;
    u32x4 x[HEADS][2];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      const uint16_t* p = unit_base(g, g.q, g.q_stride, g.q_rot, g.q_rot_stride, t, head + h, u);
      x[h][0] = *reinterpret_cast<const u32x4*>(p + u.lo);
      x[h][1] = *reinterpret_cast<const u32x4*>(p + u.hi);
    }
    const bool turn = u.pair >= 0 && tok.pos >= 0;
    Angles an{};
    if (turn) an = load_angles(g, u, tok.pos);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      float y[16];
      unpack8(x[h][0], y);
      unpack8(x[h][1], y + 8);
      if (turn) rotate(g, an, y);
      if (tok.pos < 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.f;
      }
      uint16_t* o = g.q_out + ((int64_t)t * g.H + head + h) * g.d_k;
      *reinterpret_cast<u32x4*>(o + u.lo) = pack8(y);
      *reinterpret_cast<u32x4*>(o + u.hi) = pack8(y + 8);
    }
    return;
  }
  const bool key = blk < bq + bk;
  const FastDiv& by_lanes = key ? g.by_k_lanes : g.by_v_lanes;
  const int d = key ? g.d_k : g.d_v, units = d / 16, lanes = (int)by_lanes.d;
  const int item = (key ? blk - bq : blk - bq - bk) * kAppendThreads + (int)threadIdx.x;
  const int vec = fdiv(by_lanes, item), t = fdiv(g.by_kv_heads, vec);
  if (t >= g.n_tok) return;  // (whole groups of lanes leave)
  const int head = vec - t * g.Hkv, ui = item - vec * lanes;
  const AppendToken tok = append_token(g, t);
  const int pg = tok.pos < 0 ? 0 : fdiv(g.by_page, tok.pos), off = tok.pos < 0 ? 0 : tok.pos - pg * g.P;
  int64_t page = -1;
  if (tok.pos >= 0) page = g.page_table ? g.page_table[(int64_t)tok.seq * g.max_pages + pg] : tok.seq;
  if (page >= g.n_phys) page = -1;
  if (key && head == 0 && ui == 0 && g.rows) g.rows[g.tok0 + t] = page < 0 ? -1 : page * g.P + off;
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = 0.f;
  Unit u{16 * ui, 16 * ui + 8, -1};
  if (ui < units) {
    if (key) u = unit_of(g, ui);
    const uint16_t* p = key ? unit_base(g, g.k, g.k_stride, g.k_rot, g.k_rot_stride, t, head, u) : g.v + (int64_t)t * g.v_stride + head * d;
    unpack8(*reinterpret_cast<const u32x4*>(p + u.lo), y);
    unpack8(*reinterpret_cast<const u32x4*>(p + u.hi), y + 8);
    if (u.pair >= 0 && tok.pos >= 0) rotate(g, load_angles(g, u, tok.pos), y);
  }
  const int64_t row = (page * g.Hkv + head) * g.P + off;
  if (!g.fp8) {
    if (page < 0 || ui >= units) return;
    uint16_t* o = static_cast<uint16_t*>(key ? g.k_cache : g.v_cache) + row * d;
    *reinterpret_cast<u32x4*>(o + u.lo) = pack8(y);
    *reinterpret_cast<u32x4*>(o + u.hi) = pack8(y + 8);
    return;
  }
  // the row's largest magnitude, on the bits, so that a NaN or infinity counts
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
  for (int o = 1; o < lanes; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  float scale = __uint_as_float(top) / 448.f;
  scale = top == 0 ? 1.f : scale < 1.17549435e-38f ? 1.17549435e-38f : scale;
  if (page < 0) return;
  float* sc = key ? g.k_scale : g.v_scale;
  if (ui == 0) sc[row] = scale;
  if (ui >= units) return;
  const float inv = 1.f / scale;
#pragma unroll
  for (int i = 0; i < 16; ++i) {  // y / scale: the product with the reciprocal, corrected by its remainder
    const float q = y[i] * inv;
    y[i] = fmaf(fmaf(-q, scale, y[i]), inv, q);
  }
  uint8_t* o = static_cast<uint8_t*>(key ? g.k_cache : g.v_cache) + row * d;
  *reinterpret_cast<u32x2*>(o + u.lo) = pack_fp8x8(y);
  *reinterpret_cast<u32x2*>(o + u.hi) = pack_fp8x8(y + 8);
}

static int append_lanes(int units, bool fp8) {
  if (!fp8) return units;
  int l = 1;
  while (l < units) l *= 2;
  return l;
}

// Units of queries from which a thread takes four heads: their position, row and angles are found once, for a quarter of the
// threads. us of one / four heads a thread: 32 heads of 128, bf16, 64 tokens (2^14 units) 3.4 / 3.8, 512 4.9 / 4.9, 1024 7.5 / 7.2, 4096 19.4 / 18.5, 8192 39.3 /
// 39.6; with one fp8 indexer key 256 4.1 / 4.0, 1024 6.9 / 6.0, 4096 14.6 / 13.7; 8 heads of 64 2048 (2^16) 4.7 / 5.2, 4096 7.2 / 7.6, 8192 (2^18) 11.7 / 11.4;
// latent, 64 heads, 64 (2^17) 4.7 / 4.5, 256 10.4 / 10.7, 512 15.9 / 15.1.
constexpr int64_t kManyUnits = 1 << 18;
hipError_t launch_append(const AppendGeom& all, hipStream_t st) {
  AppendGeom g = all;
  const int q_units = g.H ? g.d_k / 16 : 1, k_lanes = append_lanes(g.d_k / 16, g.fp8), v_lanes = g.d_v ? append_lanes(g.d_v / 16, g.fp8) : 1;
  const int heads = g.H % 4 == 0 && (int64_t)all.n_tok * g.H * q_units >= kManyUnits ? 4 : 1;
  g.by_q_units = fast_div((uint32_t)q_units);
  g.by_q_heads = fast_div((uint32_t)(g.H ? g.H / heads : 1));
  g.by_kv_heads = fast_div((uint32_t)g.Hkv);
  g.by_k_lanes = fast_div((uint32_t)k_lanes);
  g.by_v_lanes = fast_div((uint32_t)v_lanes);
  g.by_page = fast_div((uint32_t)g.P);
  // A launch of as many tokens as 31 bits count threads for, those of queries, keys and values together (each part's last
  // workgroup is not full): the runtime takes a launch of 2^32 threads or more modulo 2^32, without an error.
  const int64_t each = (int64_t)g.H * q_units + (int64_t)g.Hkv * (k_lanes + (g.d_v ? v_lanes : 0));
  const int64_t tokens = ((int64_t(1) << 31) - 3 * kAppendThreads) / each;
  auto blocks = [](int64_t items) { return (int)((items + kAppendThreads - 1) / kAppendThreads); };
  for (int64_t t0 = 0; t0 < all.n_tok; t0 += tokens) {
    g.tok0 = (int)t0;
    g.n_tok = (int)(all.n_tok - t0 < tokens ? all.n_tok - t0 : tokens);
    if (all.q) g.q = all.q + t0 * g.q_stride;
    if (all.q_rot) g.q_rot = all.q_rot + t0 * g.q_rot_stride;
    if (all.q_out) g.q_out = all.q_out + t0 * g.H * g.d_k;
    g.k = all.k + t0 * g.k_stride;
    if (all.k_rot) g.k_rot = all.k_rot + t0 * g.k_rot_stride;
    if (all.v) g.v = all.v + t0 * g.v_stride;
    const int bq = g.H ? blocks((int64_t)g.n_tok * (g.H / heads) * q_units) : 0, bk = blocks((int64_t)g.n_tok * g.Hkv * k_lanes);
    const int bv = g.d_v ? blocks((int64_t)g.n_tok * g.Hkv * v_lanes) : 0;
    const hipError_t e = launch_kernel(heads == 4 ? append_kernel<4> : append_kernel<1>, dim3((unsigned)bq + (unsigned)bk + (unsigned)bv),
                                       dim3(kAppendThreads), st, g, bq, bk);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace lsa
