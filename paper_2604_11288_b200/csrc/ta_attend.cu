// Attention of new tokens over a cache.
#include <math.h>

#include "ta_cache.cuh"

namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ float cache_value(const ta_cache_dev& c, const uint8_t* row, int j) {
  if (c.format == TA_CACHE_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[j]);
  if (c.format == TA_CACHE_E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw(row[j], __NV_E4M3)));
  return (float)reinterpret_cast<const int8_t*>(row)[j];
}

// A block per query row: its warps take every kWarps-th cache row each, with a running maximum and sum, and join at the end.
// grid.x = units, grid.y = rows of a unit. scores: [unit][row][max_len] for the attention mass, or null.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) ta_attend_kernel(ta_attend_args a, float* scores, float* row_lse,
                                                                 ta_dev_status* status) {
  ta_wait_for_prior_grid();
  constexpr int N = D / 32;
  __shared__ float s_q[D], s_m[kWarps], s_l[kWarps], s_o[kWarps][D];
  const ta_cache_dev& c = a.cache;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int unit = blockIdx.x, g = unit % c.Hkv, b = unit / c.Hkv % c.batch, l = unit / c.Hkv / c.batch;
  const int G = a.Hq / c.Hkv, t = blockIdx.y / G, h = g * G + blockIdx.y % G;
  long long n = (long long)ta_cache_len(c, l, b, g) + a.new_rows;
  const long long most = min((long long)a.max_len, (long long)c.wide * c.page);
  if (n > most) {
    if (threadIdx.x == 0) ta_report_bounds(status, 32, b, (int)min(n, 0x7fffffffLL));
    n = most;
  }
  const int seen = (int)max(0LL, n - (a.causal ? a.T - 1 - t : 0));
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q.ptr) + l * a.q.stride_l + b * a.q.stride_b + h * a.q.stride_h +
                           t * a.q.stride_n;
  for (int j = threadIdx.x; j < D; j += kWarps * 32) {
    float v = __bfloat162float(q[j]);
    if (a.rot.phase && j < a.rot.d_rot) {
      const int half = a.rot.d_rot / 2;
      const int position = a.rot.positions ? a.rot.positions[b * a.T + t] : (int)n - a.T + t;
      const bool second = a.rot.interleaved ? (j & 1) : j >= half;
      const int p = a.rot.interleaved ? j >> 1 : (second ? j - half : j);
      const int other = a.rot.interleaved ? j ^ 1 : (second ? j - half : j + half);
      const float2 cs = ta_cos_sin(a.rot, a.rot.phase[p], position);
      const float o = __bfloat162float(q[other]);
      v = second ? o * cs.y + v * cs.x : v * cs.x - o * cs.y;
    }
    s_q[j] = v;
  }
  __syncthreads();
  float qf[N], o[N] = {}, m = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) qf[e] = s_q[lane + 32 * e];
  float* sc = scores ? scores + ((long long)unit * gridDim.y + blockIdx.y) * a.max_len : nullptr;
  for (int r = warp; r < seen; r += kWarps) {
    const ta_row_at at = ta_cache_row(c, b, r);
    if (at.row < 0) {
      if (lane == 0) ta_report_bounds(status, 33, b, r);
      if (sc && lane == 0) sc[r] = -INFINITY;
      continue;
    }
    const long long base = l * c.sl + g * c.sh + at.row, sbase = l * c.ssl + g * c.ssh + at.scale;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) s += qf[e] * cache_value(c, c.k + base, lane + 32 * e);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
    s *= a.scale * (c.format == TA_CACHE_BF16 ? 1.0f : c.ks[sbase]);
    if (sc && lane == 0) sc[r] = s;
    const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.0f : top;
    const float keep = __expf(m - ref), p = __expf(s - ref);
    const float pv = p * (c.format == TA_CACHE_BF16 ? 1.0f : c.vs[sbase]);
    sum = sum * keep + p;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = o[e] * keep + pv * cache_value(c, c.v + base, lane + 32 * e);
    m = top;
  }
  if (lane == 0) s_m[warp] = m, s_l[warp] = sum;
#pragma unroll
  for (int e = 0; e < N; ++e) s_o[warp][lane + 32 * e] = o[e];
  __syncthreads();
  float top = -INFINITY, z = 0.0f;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w]);
  const float ref = top == -INFINITY ? 0.0f : top;
  for (int w = 0; w < kWarps; ++w) z += s_l[w] == 0.0f ? 0.0f : s_l[w] * __expf(s_m[w] - ref);
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(a.out.ptr)) + l * a.out.stride_l + b * a.out.stride_b +
                       h * a.out.stride_h + t * a.out.stride_n;
  for (int j = threadIdx.x; j < D; j += kWarps * 32) {
    float x = 0.0f;
    for (int w = 0; w < kWarps; ++w) x += s_l[w] == 0.0f ? 0.0f : s_o[w][j] * __expf(s_m[w] - ref);
    out[j] = __float2bfloat16(z == 0.0f ? 0.0f : x / z);
  }
  if (threadIdx.x == 0) {
    const float lse = z == 0.0f ? -INFINITY : ref + logf(z);
    if (a.lse) a.lse[(((long long)l * c.batch + b) * a.Hq + h) * a.T + t] = lse;
    if (row_lse) row_lse[(long long)unit * gridDim.y + blockIdx.y] = lse;
  }
}

// Attention mass per cache row. grid.x = units, grid.y = blocks of rows.
__global__ void __launch_bounds__(256) ta_attend_mass_kernel(ta_attend_args a, const float* scores, const float* row_lse) {
  ta_wait_for_prior_grid();
  const ta_cache_dev& c = a.cache;
  const int unit = blockIdx.x, g = unit % c.Hkv, b = unit / c.Hkv % c.batch, l = unit / c.Hkv / c.batch;
  const int G = a.Hq / c.Hkv, R = G * a.T;
  long long n = (long long)ta_cache_len(c, l, b, g) + a.new_rows;
  n = min(n, min((long long)a.max_len, (long long)c.wide * c.page));
  for (long long j = blockIdx.y * 256 + threadIdx.x; j < a.mass_stride; j += gridDim.y * 256) {
    float m = 0.0f;
    for (int r = 0; r < R; ++r) {
      const long long seen = n - (a.causal ? a.T - 1 - r / G : 0);
      if (j < seen) m += __expf(scores[((long long)unit * R + r) * a.max_len + j] - row_lse[(long long)unit * R + r]);
    }
    a.mass[unit * a.mass_stride + j] = m;
  }
}

}  // namespace

size_t ta_attend_scratch(int units, int rows, int d, int max_len, bool with_mass) {
  return with_mass ? (size_t)units * rows * ((size_t)max_len + 1) * 4 : 0;
}

cudaError_t ta_launch_attend(const ta_attend_args& a, ta_dev_status* status, cudaStream_t stream) {
  const int units = a.n_layers * a.cache.batch * a.cache.Hkv, rows = a.Hq / a.cache.Hkv * a.T;
  float* row_lse = a.mass ? reinterpret_cast<float*>(a.scratch) : nullptr;
  float* scores = a.mass ? row_lse + (size_t)units * rows : nullptr;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)units, (unsigned)rows, 1);
  cfg.blockDim = dim3(kWarps * 32, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  ta_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = a.d == 64 ? cudaLaunchKernelEx(&cfg, ta_attend_kernel<64>, a, scores, row_lse, status)
                            : cudaLaunchKernelEx(&cfg, ta_attend_kernel<128>, a, scores, row_lse, status);
  if (e != cudaSuccess || !a.mass) return e;
  cfg.gridDim = dim3((unsigned)units, (unsigned)((a.mass_stride + 255) / 256), 1);
  cfg.blockDim = dim3(256, 1, 1);
  return cudaLaunchKernelEx(&cfg, ta_attend_mass_kernel, a, (const float*)scores, (const float*)row_lse);
}
