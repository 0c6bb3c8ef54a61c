// Attention of new tokens over the whole of a paged cache (lsa_decode_attn) for gfx950.
#include "device.hpp"
#include "launch.hpp"

namespace lsa {

constexpr float kLn2 = 0.69314718055994530942f;

// One wave per (row, head), 64 positions at a time: a lane scores one position, then holds d_v / 64 columns
// of the output. The plain form of the operator: every head reads its rows by itself.
__global__ __launch_bounds__(64) void decode_attn_kernel(DecodeGeom g) {
  __shared__ float qs[576];
  __shared__ float ps[64];
  __shared__ int rows[64];
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x / g.H;
  const int h = (int)(blockIdx.x - r * g.H), kvh = h / (g.H / g.Hkv);
  const int b = (int)(r / g.R), j = (int)(r - (int64_t)b * g.R);
  for (int i = lane; i < g.d_qk; i += 64) qs[i] = __uint_as_float((uint32_t)g.q[(r * g.H + h) * g.d_qk + i] << 16);
  const int ctx = g.ctx_len[b];
  const int t = ctx < 0 || ctx > g.max_pages * g.P ? -1 : ctx - g.R + j;
  const int cols = g.d_v / 64;
  float o[8] = {}, m = -INFINITY, l = 0.f;
  auto value = [&](const void* base, const float* scale, int64_t row, int d, int i) {
    if (!g.fp8) return __uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[row * d + i] << 16);
    return __builtin_amdgcn_cvt_f32_fp8((int) static_cast<const uint8_t*>(base)[row * d + i], 0) * scale[row];
  };
  __syncthreads();
  for (int s0 = 0; s0 <= t; s0 += 64) {
    const int s = s0 + lane;
    bool seen = s <= t && (g.k_swa == 0 || s > t - g.k_swa || s < g.k_sink);
    int64_t ph = -1;
    if (seen) ph = g.page_table ? g.page_table[(int64_t)b * g.max_pages + s / g.P] : b;
    seen = seen && ph >= 0 && ph < g.n_phys;
    const int64_t row = (ph * g.Hkv + kvh) * g.P + s % g.P;
    float z = -INFINITY;
    if (seen) {
      float acc = 0.f;
      for (int i = 0; i < g.d_qk; ++i) acc += qs[i] * value(g.k, g.k_scale, row, g.d_qk, i);
      z = acc * g.scale_log2;
    }
    const float mx = fmaxf(wave_max(z), m);
    const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
    const float p = seen && z != -INFINITY ? __builtin_amdgcn_exp2f(z - mx) : 0.f;
    float sum = p;
    for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
    l = l * alpha + sum;
    m = mx;
    ps[lane] = p;
    rows[lane] = seen ? (int)row : -1;
    __syncthreads();
    for (int c = 0; c < cols; ++c) o[c] *= alpha;
    for (int k = 0; k < 64; ++k) {
      if (rows[k] < 0) continue;
      for (int c = 0; c < cols; ++c)
        o[c] += ps[k] * (g.latent ? value(g.k, nullptr, rows[k], g.d_qk, 64 * c + lane)
                                  : value(g.v, g.v_scale, rows[k], g.d_v, 64 * c + lane));
    }
    __syncthreads();
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int c = 0; c < cols; ++c)
    g.out[(r * g.H + h) * g.d_v + 64 * c + lane] = (uint16_t)pack_bf16x2(l == 0.f ? 0.f : o[c] * inv, 0.f);
  if (g.lse && lane == 0) g.lse[r * g.H + h] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

hipError_t launch_decode_attn(const DecodeGeom& g, hipStream_t st) {
  hipLaunchKernelGGL(decode_attn_kernel, dim3((unsigned)(g.n_seq * g.R * g.H)), dim3(64), 0, st, g);
  return hipGetLastError();
}

}  // namespace lsa
