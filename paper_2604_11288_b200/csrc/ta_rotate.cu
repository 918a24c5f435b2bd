// Rotary positions of a batch's queries and keys.
//
// Every value is read and written once: 4 bytes of traffic for an element against one product and one multiply-add, so memory is
// the bound, as long as sine and cosine are not formed per head, and addresses not per 16 bytes: a block takes the heads of
// a few tokens, forms their angles once in shared memory, and a thread keeps one part of a head (V coordinates of both sides
// of its pairs), takes its angles to registers once a token, and steps through the heads with a constant stride, kAhead
// 16-byte loads ahead of their use. Blocks are small (64 threads, many an SM): one block's angles are formed while others
// stream. 131072 tokens of 32 + 8 heads of 128: 432 us, 6.2 TB/s read and written (neighbouring pairs 419 us, 6.4 TB/s); with
// 128 threads a block 490, with 256 and addresses per vector 507. 8 + 2 heads, 524288 tokens: 462 us.
#include "ta_cache.cuh"

namespace {

constexpr int kThreads = 64;
constexpr int kAhead = 4;  // 16-byte loads of a thread before the first is used
constexpr int kTokens = 4;  // tokens of a thread

struct Cut {  // a block's work: `tokens` tokens; a thread has one part of a head, every lanes-th head and every tok_lanes-th token
  int tokens, pairs, per_head, lanes, tok_lanes;  // pairs: parts that are rotated, the others are copied
};

template <int V>
struct Vec {
  uint32_t w[V / 2];
};
template <int V>
__device__ __forceinline__ Vec<V> load(const __nv_bfloat16* p) {
  Vec<V> v;
  if constexpr (V == 8)
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "l"(p));
  else
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "l"(p));
  return v;
}
template <int V>
__device__ __forceinline__ void store(__nv_bfloat16* p, const Vec<V>& v) {
  if constexpr (V == 8) ta_st_stream(reinterpret_cast<uint4*>(p), make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]));
  else *reinterpret_cast<uint2*>(p) = make_uint2(v.w[0], v.w[1]);
}
__device__ __forceinline__ float2 both(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// grid.x = groups of cut.tokens tokens, grid.y = layers. INTER: neighbouring coordinates are a pair.
template <int V, bool INTER>
__global__ void __launch_bounds__(kThreads) ta_rotate_kernel(ta_rotate_args a, Cut cut) {
  ta_wait_for_prior_grid();
  ta_launch_dependents();
  extern __shared__ __align__(16) float2 s_cs[];  // [token][pair]
  const int l = blockIdx.y, half = a.rot.d_rot / 2;
  const long long tok0 = (long long)blockIdx.x * cut.tokens;
  const int tokens = (int)min((long long)cut.tokens, a.seq.total - tok0);
  for (int w = threadIdx.x; w < tokens * half; w += kThreads) {
    const int t = w / half, p = w - t * half;
    const long long tok = tok0 + t;
    int position;
    if (a.rot.positions) {
      position = a.rot.positions[tok];
    } else if (a.seq.cu) {
      int lo = 0, hi = a.seq.batch;  // the last sequence that begins at or before the token
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.seq.cu[mid] <= tok) lo = mid;
        else hi = mid;
      }
      position = (int)(tok - a.seq.cu[lo]);
    } else {
      position = (int)((unsigned)tok % (unsigned)a.seq.n_uniform);
    }
    s_cs[w] = ta_cos_sin(a.rot, a.rot.phase[p], position);
  }
  __syncthreads();
  const int part = threadIdx.x % cut.per_head, unit = threadIdx.x / cut.per_head, lane = unit % cut.lanes;
  if (unit >= cut.lanes * cut.tok_lanes) return;
  const bool turned = part < cut.pairs;
  const int c = turned ? part * V : a.rot.d_rot + (part - cut.pairs) * V;
  constexpr int NP = INTER ? V / 2 : V;  // pairs of a part
  constexpr int U = INTER ? kAhead : kAhead / 2;
  for (int t = unit / cut.lanes; t < tokens; t += cut.tok_lanes) {
    float2 cs[NP];
    if (turned) {
      const float4* f = reinterpret_cast<const float4*>(s_cs + t * half + part * NP);
#pragma unroll
      for (int e = 0; e < NP / 2; ++e) {
        const float4 v = f[e];
        cs[2 * e] = make_float2(v.x, v.y);
        cs[2 * e + 1] = make_float2(v.z, v.w);
      }
    }
    long long b = 0, i = tok0 + t;
    if (!a.seq.cu) {
      b = (unsigned)i / (unsigned)a.seq.n_uniform;
      i -= b * a.seq.n_uniform;
    }
    auto heads = [&](const ta_bf16_view& vi, const ta_bf16_view& vo, int H) {
      const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(vi.ptr) + l * vi.stride_l + b * vi.stride_b + i * vi.stride_n +
                                 lane * vi.stride_h + c;
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(vo.ptr)) + l * vo.stride_l + b * vo.stride_b +
                           i * vo.stride_n + lane * vo.stride_h + c;
      const long long in_step = cut.lanes * vi.stride_h, out_step = cut.lanes * vo.stride_h;
      for (int h = lane; h < H; h += U * cut.lanes) {
        Vec<V> x[U], y[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
          if (h + k * cut.lanes < H) {
            x[k] = load<V>(src);
            if (!INTER && turned) y[k] = load<V>(src + half);
          }
          src += in_step;
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
          if (h + k * cut.lanes < H) {
            Vec<V> u, v;
            if (!turned) {
              store<V>(dst, x[k]);
            } else if constexpr (INTER) {
#pragma unroll
              for (int e = 0; e < V / 2; ++e) {
                const float2 f = both(x[k].w[e]), r = cs[e];
                u.w[e] = pack(f.x * r.x - f.y * r.y, f.x * r.y + f.y * r.x);
              }
              store<V>(dst, u);
            } else {
#pragma unroll
              for (int e = 0; e < V / 2; ++e) {
                const float2 f = both(x[k].w[e]), g = both(y[k].w[e]), r = cs[2 * e], q = cs[2 * e + 1];
                u.w[e] = pack(f.x * r.x - g.x * r.y, f.y * q.x - g.y * q.y);
                v.w[e] = pack(f.x * r.y + g.x * r.x, f.y * q.y + g.y * q.x);
              }
              store<V>(dst, u);
              store<V>(dst + half, v);
            }
          }
          dst += out_step;
        }
      }
    };
    heads(a.q, a.q_out, a.Hq);
    if (a.Hkv) heads(a.k, a.k_out, a.Hkv);
  }
}

}  // namespace

cudaError_t ta_launch_rotate(const ta_rotate_args& a, cudaStream_t stream) {
  if (a.seq.total == 0) return cudaSuccess;
  const int half = a.rot.d_rot / 2;
  const bool inter = a.rot.interleaved;
  const int V = inter || half % 8 == 0 ? 8 : 4;
  const int pairs = inter ? a.rot.d_rot / V : half / V;
  // nothing to copy where every output view is its input
  auto same = [](const ta_bf16_view& x, const ta_bf16_view& y) {
    return x.ptr == y.ptr && x.stride_l == y.stride_l && x.stride_b == y.stride_b && x.stride_h == y.stride_h && x.stride_n == y.stride_n;
  };
  const bool in_place = same(a.q, a.q_out) && (a.Hkv == 0 || same(a.k, a.k_out));
  const int per_head = pairs + (in_place ? 0 : (a.d - a.rot.d_rot) / V);
  // four heads a thread, so that their angles are fetched once for as many, then other tokens
  const int units = kThreads / per_head > 0 ? kThreads / per_head : 1, by_heads = a.Hq / 4 > 1 ? a.Hq / 4 : 1;
  const int lanes = units < by_heads ? units : by_heads, tok_lanes = units / lanes;
  // a block's tokens: kTokens a thread, but fewer while that does not fill the 148 SMs with eight blocks each
  const long long spread = a.seq.total * a.n_layers / (8 * 148);
  int tokens = kTokens * tok_lanes;
  if (tokens > spread) tokens = (int)spread;
  if (tokens < 1) tokens = 1;
  const Cut cut = {tokens, pairs, per_head, lanes, tok_lanes};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((a.seq.total + tokens - 1) / tokens), (unsigned)a.n_layers, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)tokens * half * sizeof(float2);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  ta_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (inter) return cudaLaunchKernelEx(&cfg, ta_rotate_kernel<8, true>, a, cut);
  return V == 8 ? cudaLaunchKernelEx(&cfg, ta_rotate_kernel<8, false>, a, cut)
                : cudaLaunchKernelEx(&cfg, ta_rotate_kernel<4, false>, a, cut);
}
