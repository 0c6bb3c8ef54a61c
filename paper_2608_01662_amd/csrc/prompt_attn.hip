// Attention of packed prompts over their own keys and values (lsa_prefill_attn) and of ragged chunks of new tokens over a
// paged cache (lsa_chunk_attn) for gfx950.
//
// The query rows of a key/value head are the heads of its group of all new tokens of a sequence, token after token. A
// workgroup takes 256 of them, four waves of 64, and walks the tiles of 64 keys that any of them attends to, with the running
// maximum and sum of an online softmax. S^T = K Q^T on 32x32x16 products: a lane holds the scores of one query row,
// which are, rounded to bf16, the B operand of O^T += V^T P^T as they lie, so that P never leaves the registers.
#include "attn_tile.hpp"
#include "device.hpp"
#include "launch.hpp"
#include "serve_tile.hpp"

namespace lsa {

constexpr int kRows = kPromptRows;  // query rows of a workgroup
constexpr int kKeys = 64;           // keys of a tile
constexpr int kThreads = 256;

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
  int clear0, clear1;  // tiles [clear0, clear1) of the span are attended to whole by every row
};

__device__ __forceinline__ int new_tokens(const PromptGeom& g, int b, int& first) {
  const int a = g.cu_q[b], e = g.cu_q[b + 1];
  first = a;
  return a >= 0 && e >= a && e <= g.n_tok ? e - a : 0;
}

// The work item of this workgroup, false when there is none. Items of a sequence: heads outermost, blocks of rows from the last
// (which has the most keys) to the first.
__device__ __forceinline__ bool find_share(const PromptGeom& g, int item, Share& w) {
  const int lane = threadIdx.x & 63, group = (int)g.by_group.d;
  int before = 0;
  for (int b0 = 0; b0 < g.n_seq; b0 += 64) {
    const int b = b0 + lane;
    int first = 0;
    const int n = b < g.n_seq ? new_tokens(g, b, first) : 0;
    const int blocks = (n * group + kRows - 1) / kRows, inc = wave_scan(blocks * g.Hkv);
    const uint64_t past = __ballot(before + inc > item);
    if (past) {
      const int i = __ffsll((unsigned long long)past) - 1;
      w.b = b0 + i;
      w.n = __builtin_amdgcn_readlane(n, i);
      w.q0 = __builtin_amdgcn_readlane(first, i);
      const int nb = __builtin_amdgcn_readlane(blocks, i);
      const int at = item - (before + __builtin_amdgcn_readlane(inc, i) - nb * g.Hkv);
      w.head = at / nb;
      w.row0 = (nb - 1 - (at - w.head * nb)) * kRows;
      w.rows = w.n * group;
      break;
    }
    before += __builtin_amdgcn_readlane(inc, 63);
    if (b0 + 64 >= g.n_seq) return false;
  }
  if (g.ctx_len) {
    const int c = uniform(g.ctx_len[w.b]);
    w.c = c < 0 || c > g.cap ? 0 : c;
    w.kv0 = 0;
  } else {
    const int a = uniform(g.cu_kv[w.b]), e = uniform(g.cu_kv[w.b + 1]);
    w.c = a >= 0 && e >= a && e <= g.n_kv ? e - a : 0;
    w.kv0 = a;
  }
  const int last = (w.rows - w.row0 < kRows ? w.rows : w.row0 + kRows) - 1;
  const int t_lo = g.causal ? w.c - w.n + fdiv(g.by_group, w.row0) : w.c - 1, t_hi = g.causal ? w.c - w.n + fdiv(g.by_group, last) : w.c - 1;
  const int end = t_hi + 1 > 0 ? t_hi + 1 : 0, total = (int)(((uint32_t)end + kKeys - 1) / kKeys);  // (t_hi < c)
  const int lo = g.k_swa > 0 && t_lo >= g.k_swa ? t_lo - g.k_swa + 1 : 0, first = lo / kKeys;
  const int sink = g.k_sink < end ? g.k_sink : end, st = (int)(((uint32_t)sink + kKeys - 1) / kKeys);
  w.ns = first <= st ? total : st;
  w.skip = first <= st ? 0 : first - st;
  w.nt = total - w.skip;
  return true;
}

__device__ __forceinline__ float swap32(float x) {  // the value of lane l ^ 32
  return __shfl_xor(x, 32);
}

template <int DQK, int DV, int KIND>  // KIND 0: contiguous bf16, 1: paged bf16, 2: paged fp8
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void prompt_attn_kernel(PromptGeom g) {
  constexpr int CK = DQK / 8, CV = DV / 8, KS = DQK / 16, DB = DV / 32, NQ = 2;
  constexpr bool FP8 = KIND == 2;
  __shared__ __attribute__((aligned(1024))) uint8_t lk[kKeys * DQK * 2], lv[kKeys * DV * 2];
  __shared__ __attribute__((aligned(16))) float scales[FP8 ? 2 : 1][FP8 ? kKeys : 1];
  __shared__ int mapped[kKeys];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5, l32 = lane & 31;
  Share w;
  if (!find_share(g, g.first + (int)blockIdx.x, w)) return;
  const int group = (int)g.by_group.d, wrow = w.row0 + 64 * wave;
  const bool active = wrow < w.rows;

  u32x4 qf[NQ][KS];
  int t[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int row = wrow + 32 * nq + l32, r = row < w.rows ? row : w.rows - 1, j = fdiv(g.by_group, r);
    t[nq] = g.causal ? w.c - w.n + j : w.c - 1;
    const uint16_t* p = g.q + (w.q0 + j) * g.q_stride + (int64_t)(w.head * group + r - j * group) * DQK + 8 * h;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[nq][s] = *reinterpret_cast<const u32x4*>(p + 16 * s);
  }
  f32x16 o[DB][NQ];
  float m[NQ], l[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    m[nq] = kNoRef;
    l[nq] = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d][nq] = f32x16{};
  }
  // LDS offsets of this lane's operands
  int k_off[KS], v_off[2][DB];
#pragma unroll
  for (int s = 0; s < KS; ++s) k_off[s] = l32 * DQK * 2 + (((2 * s + h) ^ swz<CK>(l32)) << 4);
  {
    const int i = lane & 15, cc = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = 8 * half + 4 * h + (i >> 2);
#pragma unroll
      for (int d = 0; d < DB; ++d) v_off[half][d] = row * DV * 2 + (((4 * d + cc) ^ swz<CV>(row)) << 4) + 8 * (i & 1);
    }
  }

  for (int i = 0; i < w.nt; ++i) {
    const int s0 = (i < w.ns ? i : i + w.skip) * kKeys;
    __syncthreads();
    // row of the cache (or of the packed keys) of a key, -1: none
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
      if constexpr (FP8) {
        for (int e = (int)threadIdx.x; e < kKeys * (D / 16); e += kThreads) {
          const int r = e / (D / 16), u = e % (D / 16);
          const int64_t row = row_of(r);
          u32x4 x{};
          if (row >= 0) x = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(base) + row * D + 16 * u);
          *reinterpret_cast<u32x4*>(dst + r * D * 2 + (((2 * u) ^ swz<C>(r)) << 4)) = fp8x8_bf16(x.x, x.y);
          *reinterpret_cast<u32x4*>(dst + r * D * 2 + (((2 * u + 1) ^ swz<C>(r)) << 4)) = fp8x8_bf16(x.z, x.w);
        }
      } else {
        for (int e = (int)threadIdx.x; e < kKeys * C; e += kThreads) {
          const int r = e / C, c = e % C;
          const int64_t row = row_of(r);
          u32x4 x{};
          if (row >= 0) x = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + row * stride + 8 * c);
          *reinterpret_cast<u32x4*>(dst + r * D * 2 + ((c ^ swz<C>(r)) << 4)) = x;
        }
      }
    };
    load(KIND ? g.k : static_cast<const void*>(static_cast<const uint16_t*>(g.k) + w.head * DQK), KIND ? DQK : g.k_stride, lk,
         std::integral_constant<int, DQK>{});
    load(KIND ? g.v : static_cast<const void*>(static_cast<const uint16_t*>(g.v) + w.head * DV), KIND ? DV : g.v_stride, lv,
         std::integral_constant<int, DV>{});
    if (threadIdx.x < kKeys) {
      const int64_t row = row_of((int)threadIdx.x);
      mapped[threadIdx.x] = row >= 0;
      if constexpr (FP8) {
        scales[0][threadIdx.x] = row >= 0 ? g.k_scale[row] : 0.f;
        scales[1][threadIdx.x] = row >= 0 ? g.v_scale[row] : 0.f;
      }
    }
    __syncthreads();
    if (!active) continue;
    const uint64_t there = __ballot(mapped[lane] != 0);
    f32x16 s[2][NQ];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) s[kb][nq] = f32x16{};
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(lk + k_off[st] + kb * 32 * DQK * 2);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) s[kb][nq] = mfma32(a, qf[nq][st], s[kb][nq]);
      }
    u32x4 p[2][2][NQ];      // [key block][k-step of 16]
    uint32_t live[2][NQ];   // scores that are not -inf
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      float top = -INFINITY;
      const int rel = t[nq] - s0, win = g.k_swa > 0 ? rel - g.k_swa : -1, sink = g.k_swa > 0 ? g.k_sink - s0 : 0;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * kb + 8 * (r >> 2) + 4 * h + (r & 3);
          const bool seen = key <= rel && (key > win || key < sink) && ((there >> key) & 1);
          float z = s[kb][nq][r] * g.scale_log2;
          if constexpr (FP8) z *= scales[0][key];
          s[kb][nq][r] = seen ? z : -INFINITY;
          top = fmaxf(top, s[kb][nq][r]);
        }
      top = fmaxf(top, swap32(top));
      const bool grown = top > m[nq] + kLazy;
      if (__any(grown)) {  // (each row by its own scores, whatever the wave's others do)
        const float mn = grown ? top : m[nq], al = fast_exp2(m[nq] - mn);
        m[nq] = mn;
        l[nq] *= al;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][nq][r] *= al;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        live[kb][nq] = 0;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          float e[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float z = s[kb][nq][r + k];
            const bool in = z != -INFINITY;
            if (in) live[kb][nq] |= 1u << (r + k);
            e[k] = fast_exp2(z - m[nq]);
            l[nq] += e[k];
            if constexpr (FP8) e[k] = in ? e[k] * scales[1][32 * kb + 8 * (r >> 2) + 4 * h + ((r + k) & 3)] : 0.f;
          }
          p[kb][r >> 3][nq][(r & 7) >> 1] = pack_bf16x2(e[0], e[1]);
        }
      }
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const uint8_t* base = lv + (32 * kb + 16 * ks) * DV * 2;
          u32x4 a = tr16_pair(base + v_off[0][d], base + v_off[1][d]);
          // Values that are no finite numbers, of keys that some row attends to and others do not: a weight of 0 does not
          // silence them, so they are taken out of the product and added where they belong.
          uint32_t odd = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) odd |= ((a[k] & 0x7F80u) == 0x7F80u) | ((a[k] & 0x7F800000u) == 0x7F800000u);
          if (__any(odd)) {
            u32x4 up{}, down{}, fin = a;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                const uint32_t v = (a[k] >> (16 * half)) & 0xFFFFu;
                if ((v & 0x7F80u) == 0x7F80u) {
                  const bool nan = (v & 0x7Fu) != 0;
                  fin[k] &= half ? 0xFFFFu : 0xFFFF0000u;
                  if (nan || !(v & 0x8000u)) up[k] |= 0x3F80u << (16 * half);
                  if (nan || (v & 0x8000u)) down[k] |= 0x3F80u << (16 * half);
                }
              }
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
              u32x4 one;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t bits = live[kb][nq] >> (8 * ks + 2 * k);
                one[k] = (bits & 1 ? 0x3F80u : 0u) | (bits & 2 ? 0x3F800000u : 0u);
              }
              o[d][nq] = mfma32(fin, p[kb][ks][nq], o[d][nq]);
              const f32x16 plus = mfma32(up, one, f32x16{}), minus = mfma32(down, one, f32x16{});
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                if (plus[r] > 0.f) o[d][nq][r] += INFINITY;
                if (minus[r] > 0.f) o[d][nq][r] -= INFINITY;
              }
            }
          } else {
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) o[d][nq] = mfma32(a, p[kb][ks][nq], o[d][nq]);
          }
        }
  }
  if (!active) return;
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int row = wrow + 32 * nq + l32;
    const float sum = l[nq] + swap32(l[nq]), inv = 1.f / sum;
    if (row >= w.rows) continue;
    const int j = fdiv(g.by_group, row);
    const int64_t at = (w.q0 + j) * g.H + w.head * group + row - j * group;
    if (g.lse && h == 0) g.lse[at] = sum == 0.f ? -INFINITY : (m[nq] + __builtin_amdgcn_logf(sum)) * kLn2;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = sum == 0.f ? 0.f : o[d][nq][r + k] * inv;
        *reinterpret_cast<u32x2*>(g.out + at * DV + 32 * d + 2 * r + 4 * h) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
      }
  }
}

hipError_t launch_prompt_attn(const PromptGeom& all, hipStream_t st) {
  PromptGeom g = all;
  auto* kernel = g.ctx_len == nullptr ? (g.d_qk == 64 ? prompt_attn_kernel<64, 64, 0> : g.d_qk == 128 ? prompt_attn_kernel<128, 128, 0> : prompt_attn_kernel<192, 128, 0>)
                 : g.fp8              ? (g.d_qk == 64 ? prompt_attn_kernel<64, 64, 2> : prompt_attn_kernel<128, 128, 2>)
                                      : (g.d_qk == 64 ? prompt_attn_kernel<64, 64, 1> : prompt_attn_kernel<128, 128, 1>);
  constexpr int64_t kMost = 1 << 22;  // workgroups of a launch (2^32 threads and more are taken modulo 2^32)
  for (int64_t i = 0; i < all.items; i += kMost) {
    g.first = (int)i;
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)(all.items - i < kMost ? all.items - i : kMost)), dim3(kThreads), st, g);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace lsa
