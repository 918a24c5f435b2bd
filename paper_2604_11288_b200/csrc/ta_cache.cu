// Writing new keys and values into a cache, in its format, and reading rows back.
#include "ta_cache.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Token {
  int b, i;  // sequence and index in it
};
__device__ __forceinline__ Token token_of(const ta_seq_desc& seq, long long tok) {
  if (!seq.cu) {
    const int b = (int)(tok / seq.n_uniform);
    return {b, (int)(tok - (long long)b * seq.n_uniform)};
  }
  int lo = 0, hi = seq.batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (seq.cu[mid] <= tok) lo = mid;
    else hi = mid;
  }
  return {lo, (int)(tok - seq.cu[lo])};
}
__device__ __forceinline__ long long view_at(const ta_bf16_view& v, const ta_seq_desc& seq, int l, int g, Token t, long long tok) {
  return l * v.stride_l + g * v.stride_h + (seq.cu ? tok * v.stride_n : t.b * v.stride_b + t.i * v.stride_n);
}
// entry of `rows` for a token: [L][B][Hkv][n], or [L][Hkv][total] where the batch is ragged
__device__ __forceinline__ long long rows_at(const ta_seq_desc& seq, int Hkv, int l, int g, Token t, long long tok) {
  return seq.cu ? ((long long)l * Hkv + g) * seq.total + tok : (((long long)l * seq.batch + t.b) * Hkv + g) * seq.n_uniform + t.i;
}

// A warp per row of k and of v: lane j holds coordinates j, j + 32, ...
template <int D>
__global__ void __launch_bounds__(kThreads) ta_cache_append_kernel(ta_cache_move_args a, ta_dev_status* status) {
  ta_wait_for_prior_grid();
  constexpr int N = D / 32;
  __shared__ float s_row[kWarps][D];
  const ta_cache_dev& c = a.cache;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long w = (long long)blockIdx.x * kWarps + warp;
  const int l = blockIdx.y;
  if (w >= a.seq.total * c.Hkv) return;
  const long long tok = w / c.Hkv;
  const int g = (int)(w - tok * c.Hkv);
  const Token t = token_of(a.seq, tok);
  const long long row = a.rows ? a.rows[rows_at(a.seq, c.Hkv, l, g, t, tok)] : (long long)ta_cache_len(c, l, t.b, g) + t.i;
  if (row < 0) {
    if (!a.rows && lane == 0) ta_report_bounds(status, 30, t.b, (int)row);
    return;
  }
  const ta_row_at at = row < 0x7fffffff ? ta_cache_row(c, t.b, (int)row) : ta_row_at{-1, 0};
  if (at.row < 0) {
    if (lane == 0) ta_report_bounds(status, 30, t.b, (int)row);
    return;
  }
  for (int kv = 0; kv < 2; ++kv) {
    const ta_bf16_view& src = kv ? a.v : a.k;
    const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(src.ptr) + view_at(src, a.seq, l, g, t, tok);
    uint8_t* dst = (kv ? c.v : c.k) + l * c.sl + g * c.sh + at.row;
    const bool turned = !kv && a.rot.phase;
    if (c.format == TA_CACHE_BF16 && !turned) {
#pragma unroll
      for (int e = 0; e < N; ++e) reinterpret_cast<__nv_bfloat16*>(dst)[lane + 32 * e] = x[lane + 32 * e];
      continue;
    }
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = __bfloat162float(x[lane + 32 * e]);
    if (turned) {
      const int position = a.rot.positions ? a.rot.positions[tok] : (int)row, half = a.rot.d_rot / 2;
#pragma unroll
      for (int e = 0; e < N; ++e) s_row[warp][lane + 32 * e] = f[e];
      __syncwarp();
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int j = lane + 32 * e;
        if (j >= a.rot.d_rot) continue;
        const bool second = a.rot.interleaved ? (j & 1) : j >= half;
        const int p = a.rot.interleaved ? j >> 1 : (second ? j - half : j);
        const int other = a.rot.interleaved ? j ^ 1 : (second ? j - half : j + half);
        const float2 cs = ta_cos_sin(a.rot, a.rot.phase[p], position);
        const float o = s_row[warp][other];
        f[e] = second ? o * cs.y + f[e] * cs.x : f[e] * cs.x - o * cs.y;
      }
      __syncwarp();
    }
    if (c.format == TA_CACHE_BF16) {
#pragma unroll
      for (int e = 0; e < N; ++e) reinterpret_cast<__nv_bfloat16*>(dst)[lane + 32 * e] = __float2bfloat16(f[e]);
      continue;
    }
    float m = 0x1p-100f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      m = fmaxf(m, fabsf(f[e]));
      bad = bad || !(fabsf(f[e]) <= 3.402823466e38f);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    bad = __any_sync(0xffffffffu, bad);
    const float full = c.format == TA_CACHE_E4M3 ? 448.0f : 127.0f;
    const float inv = bad ? 0.0f : __fdiv_rn(full, m);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float y = bad ? 0.0f : f[e] * inv;
      if (c.format == TA_CACHE_E4M3) dst[lane + 32 * e] = __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3);
      else reinterpret_cast<int8_t*>(dst)[lane + 32 * e] = (int8_t)__float2int_rn(y);
    }
    if (lane == 0) (kv ? c.vs : c.ks)[l * c.ssl + g * c.ssh + at.scale] = bad ? __int_as_float(0x7fc00000) : __fdiv_rn(m, full);
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads) ta_cache_read_kernel(ta_cache_move_args a, ta_dev_status* status) {
  ta_wait_for_prior_grid();
  constexpr int N = D / 32;
  const ta_cache_dev& c = a.cache;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long w = (long long)blockIdx.x * kWarps + warp;
  const int l = blockIdx.y;
  if (w >= a.seq.total * c.Hkv) return;
  const long long tok = w / c.Hkv;
  const int g = (int)(w - tok * c.Hkv);
  const Token t = token_of(a.seq, tok);
  const int row = a.rows ? a.rows[rows_at(a.seq, c.Hkv, l, g, t, tok)] : t.i;
  const ta_row_at at = row >= 0 ? ta_cache_row(c, t.b, row) : ta_row_at{-1, 0};
  if (row >= 0 && at.row < 0 && lane == 0) ta_report_bounds(status, 31, t.b, row);
  for (int kv = 0; kv < 2; ++kv) {
    const ta_bf16_view& out = kv ? a.v : a.k;
    __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(out.ptr)) + view_at(out, a.seq, l, g, t, tok);
    const uint8_t* src = (kv ? c.v : c.k) + l * c.sl + g * c.sh + at.row;
    const float scale = at.row >= 0 && c.format != TA_CACHE_BF16 ? (kv ? c.vs : c.ks)[l * c.ssl + g * c.ssh + at.scale] : 1.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int j = lane + 32 * e;
      __nv_bfloat16 o = __float2bfloat16(0.0f);
      if (at.row >= 0) {
        if (c.format == TA_CACHE_BF16) o = reinterpret_cast<const __nv_bfloat16*>(src)[j];
        else if (c.format == TA_CACHE_E4M3)
          o = __float2bfloat16(__half2float(__half(__nv_cvt_fp8_to_halfraw(src[j], __NV_E4M3))) * scale);
        else o = __float2bfloat16((float)reinterpret_cast<const int8_t*>(src)[j] * scale);
      }
      y[j] = o;
    }
  }
}

template <class K>
cudaError_t launch(K kernel, const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  const long long rows = a.seq.total * a.cache.Hkv;
  if (rows == 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((rows + kWarps - 1) / kWarps), (unsigned)a.n_layers, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  ta_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, status);
}

}  // namespace

cudaError_t ta_launch_cache_append(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  return a.d == 64 ? launch(ta_cache_append_kernel<64>, a, status, stream) : launch(ta_cache_append_kernel<128>, a, status, stream);
}
cudaError_t ta_launch_cache_read(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  return a.d == 64 ? launch(ta_cache_read_kernel<64>, a, status, stream) : launch(ta_cache_read_kernel<128>, a, status, stream);
}
