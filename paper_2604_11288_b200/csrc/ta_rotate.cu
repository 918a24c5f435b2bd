// Rotary positions of a batch's queries and keys.
#include "ta_cache.cuh"

namespace {

constexpr int kThreads = 256;

// One pair per thread and round: grid.x = tokens, grid.y = layers.
__global__ void __launch_bounds__(kThreads) ta_rotate_kernel(ta_rotate_args a) {
  ta_wait_for_prior_grid();
  const long long tok = blockIdx.x;
  const int l = blockIdx.y, half = a.rot.d_rot / 2;
  int b, i;
  if (a.seq.cu) {
    int lo = 0, hi = a.seq.batch;  // the last sequence that begins at or before the token
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.seq.cu[mid] <= tok) lo = mid;
      else hi = mid;
    }
    b = lo;
    i = (int)(tok - a.seq.cu[b]);
  } else {
    b = (int)(tok / a.seq.n_uniform);
    i = (int)(tok - (long long)b * a.seq.n_uniform);
  }
  const int position = a.rot.positions ? a.rot.positions[tok] : i;
  extern __shared__ float2 s_cs[];
  for (int p = threadIdx.x; p < half; p += kThreads) s_cs[p] = ta_cos_sin(a.rot, a.rot.phase[p], position);
  __syncthreads();
  const int per_head = half + (a.d - a.rot.d_rot);
  for (int w = threadIdx.x; w < (a.Hq + a.Hkv) * per_head; w += kThreads) {
    const int head = w / per_head, p = w - head * per_head;
    const bool is_q = head < a.Hq;
    const int h = is_q ? head : head - a.Hq;
    const ta_bf16_view& vi = is_q ? a.q : a.k;
    const ta_bf16_view& vo = is_q ? a.q_out : a.k_out;
    const long long at = a.seq.cu ? tok : i;
    const long long bi = a.seq.cu ? 0 : b;
    const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(vi.ptr) + l * vi.stride_l + bi * vi.stride_b + h * vi.stride_h +
                             at * vi.stride_n;
    __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(vo.ptr)) + l * vo.stride_l + bi * vo.stride_b +
                       h * vo.stride_h + at * vo.stride_n;
    if (p >= half) {
      const int c = a.rot.d_rot + p - half;
      y[c] = x[c];
      continue;
    }
    const int c0 = a.rot.interleaved ? 2 * p : p, c1 = a.rot.interleaved ? 2 * p + 1 : p + half;
    const float u = __bfloat162float(x[c0]), v = __bfloat162float(x[c1]);
    const float2 cs = s_cs[p];
    y[c0] = __float2bfloat16(u * cs.x - v * cs.y);
    y[c1] = __float2bfloat16(u * cs.y + v * cs.x);
  }
}

}  // namespace

cudaError_t ta_launch_rotate(const ta_rotate_args& a, cudaStream_t stream) {
  if (a.seq.total == 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.seq.total, (unsigned)a.n_layers, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = a.rot.d_rot / 2 * sizeof(float2);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  ta_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, ta_rotate_kernel, a);
}
