// Writing new keys and values into a cache, in its format, and reading rows back.
//
// Both move every row once: 2 d bytes of bf16 on one side and 2 d or d + 4 on the other, for some operations an element; memory
// is the bound where the instructions stay under about 130 a row and warp. A row is held by d / 8 lanes, 16 bytes of bf16 each
// (8 of codes), so a warp holds two rows (d = 128) or four. What does not depend on a lane is found once, by a thread per row,
// and handed on in shared memory: where the row lies (kept per lane: 4382 us where this takes 2266, both without the next
// two), angles of the tokens (for all heads), and of a row's keys and values only one lane's division each. The largest magnitude of a
// row meets in three or four shuffles; a lane's partner coordinates (half layout) come by four of packed pairs.
// 2 x 16 x 32768 tokens of 8 heads, written and read: bf16 2632 us, 6.5 TB/s; e4m3 2044, 6.4 TB/s; rotated on the way bf16 2691,
// 6.4 TB/s, e4m3 2662, 4.9 TB/s (bound by instructions: issue slots 74 % taken).
#include <math.h>

#include "ta_cache.cuh"

namespace {

constexpr int kThreads = 128;
// Rows of k, and of v, of a block: 32 keep memory busy (16: 2989 us where 32 take 2722, rotated into e4m3 and read), 8 spread a call
// with few rows over more SMs (64 tokens of 8 heads 6.9 us, 11.6 with 32).
constexpr int kItems = 32, kFewItems = 8;
constexpr long long kFewRows = 148 * 32;

struct Token {
  int b, i;  // sequence and index in it
};
// What the tokens of a block are looked up in: the offsets of the sequences and, where every sequence has one, their lengths.
// Few of them are brought to shared memory, all at once: one wait where a search and a length would be one after another.
constexpr int kKept = 256;
struct Kept {
  int cu[kKept + 1], len[kKept];
};
__device__ __forceinline__ bool keeps(const ta_seq_desc& seq) { return seq.batch <= kKept; }
__device__ __forceinline__ void keep(Kept& s, const ta_seq_desc& seq, const ta_cache_dev& c, bool with_lens) {
  if (!keeps(seq)) return;
  for (int i = threadIdx.x; i <= seq.batch; i += kThreads) {
    if (seq.cu) s.cu[i] = seq.cu[i];
    if (with_lens && i < seq.batch) s.len[i] = c.lens && !c.lens_per_unit ? c.lens[i] : c.len_uniform;
  }
}
__device__ __forceinline__ Token token_of(const Kept& s, const ta_seq_desc& seq, long long tok) {
  if (!seq.cu) {
    const int b = (int)((unsigned)tok / (unsigned)seq.n_uniform);
    return {b, (int)(tok - (long long)b * seq.n_uniform)};
  }
  const int* cu = keeps(seq) ? s.cu : seq.cu;
  int lo = 0, hi = seq.batch;  // the last sequence that begins at or before the token
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (cu[mid] <= tok) lo = mid;
    else hi = mid;
  }
  return {lo, (int)(tok - cu[lo])};
}
__device__ __forceinline__ int len_of(const Kept& s, const ta_seq_desc& seq, const ta_cache_dev& c, int l, int b, int g) {
  return keeps(seq) && !(c.lens && c.lens_per_unit) ? s.len[b] : ta_cache_len(c, l, b, g);
}
__device__ __forceinline__ long long view_at(const ta_bf16_view& v, const ta_seq_desc& seq, int l, int g, Token t, long long tok) {
  return l * v.stride_l + g * v.stride_h + (seq.cu ? tok * v.stride_n : t.b * v.stride_b + t.i * v.stride_n);
}
// entry of `rows` for a token: [L][B][Hkv][n], or [L][Hkv][total] where the batch is ragged
__device__ __forceinline__ long long rows_at(const ta_seq_desc& seq, int Hkv, int l, int g, Token t, long long tok) {
  return seq.cu ? ((long long)l * Hkv + g) * seq.total + tok : (((long long)l * seq.batch + t.b) * Hkv + g) * seq.n_uniform + t.i;
}
__device__ __forceinline__ float2 both(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load8(const void* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 y, %4, %3;\n\tmov.b32 %0, {x, y};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// whole numbers -127..127 to nearest even: added to 1.5 * 2^23 they stand in the mantissa's lowest byte
__device__ __forceinline__ uint32_t int8x4(float a, float b, float c, float d) {
  constexpr float M = 12582912.0f;
  const uint32_t x = __float_as_uint(__fadd_rn(a, M)), y = __float_as_uint(__fadd_rn(b, M));
  const uint32_t z = __float_as_uint(__fadd_rn(c, M)), w = __float_as_uint(__fadd_rn(d, M));
  return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
}

struct Place {  // of an item, a token's row of one head, in the cache
  long long row, scale;  // offsets of the row (bytes; -1: there is none) and of its scale
};
struct Sides {  // of an item in the views
  long long k, v;
};

// What a lane has of a row: coordinates 8 lane .. 8 lane + 7. A group of D / 8 lanes takes a row at a time.
template <int D>
struct Lanes {
  static constexpr int N = D / 8, GROUPS = kThreads / N;
};

// Items are counted token * Hkv + head. grid.x = ITEMS of them, grid.y = layers.
template <int D, int FMT, bool TURN, int ITEMS>
__global__ void __launch_bounds__(kThreads, 8) ta_cache_append_kernel(ta_cache_move_args a, ta_dev_status* status) {
  ta_wait_for_prior_grid();
  ta_launch_dependents();
  constexpr int N = Lanes<D>::N, GROUPS = Lanes<D>::GROUPS, PER = ITEMS / GROUPS;
  constexpr bool CODES = FMT != TA_CACHE_BF16;
  // positions looked up once a token, behind the places (2662 us, beside them 2870), or, in a call with few rows, once an angle,
  // beside them (64 tokens 7.1 us, 7.4 behind)
  constexpr bool ONCE = ITEMS == kItems;
  extern __shared__ __align__(16) float2 s_cs[];  // [token][pair]
  __shared__ Place s_place[ITEMS];
  __shared__ int s_position[ITEMS];
  __shared__ Kept s_kept;
  const ta_cache_dev& c = a.cache;
  const int lane = threadIdx.x % N, group = threadIdx.x / N, l = blockIdx.y, half = a.rot.d_rot / 2;
  const unsigned first = blockIdx.x * ITEMS, todo = min((unsigned)ITEMS, (unsigned)a.seq.total * c.Hkv - first);
  const unsigned tok0 = first / c.Hkv, tokens = (first + todo - 1) / c.Hkv - tok0 + 1;
  // a group of lanes has PER items that follow one another: heads of one token, as a rule
  uint4 k[PER], v[PER];
  {
    const unsigned w = first + group * PER;
    unsigned tok = w / c.Hkv;
    int g = (int)(w - tok * c.Hkv);
    const __nv_bfloat16 *kp = nullptr, *vp = nullptr;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i == 0 || g == 0) {  // a token's first item here
        Token t = {0, 0};
        if (!a.seq.cu) t = token_of(s_kept, a.seq, tok);
        kp = reinterpret_cast<const __nv_bfloat16*>(a.k.ptr) + view_at(a.k, a.seq, l, g, t, tok) + lane * 8;
        vp = reinterpret_cast<const __nv_bfloat16*>(a.v.ptr) + view_at(a.v, a.seq, l, g, t, tok) + lane * 8;
      }
      if (group * PER + i < todo) {
        k[i] = load16(kp);
        v[i] = load16(vp);
      }
      kp += a.k.stride_h;
      vp += a.v.stride_h;
      if (++g == c.Hkv) g = 0, ++tok;
    }
  }
  keep(s_kept, a.seq, c, true);
  __syncthreads();
  // one thread finds an item's place
  if (threadIdx.x < todo) {
    const unsigned w = first + threadIdx.x, tok = w / c.Hkv;
    const int g = (int)(w - tok * c.Hkv);
    const Token t = token_of(s_kept, a.seq, tok);
    Place p;
    const long long row = a.rows ? (long long)a.rows[rows_at(a.seq, c.Hkv, l, g, t, tok)] : (long long)len_of(s_kept, a.seq, c, l, t.b, g) + t.i;
    ta_row_at at = {-1, 0};
    if (row >= 0 && row < 0x7fffffff) at = ta_cache_row(c, t.b, (int)row);
    if (at.row < 0 && (row >= 0 || !a.rows)) ta_report_bounds(status, 30, t.b, (int)row);
    p.row = at.row < 0 ? -1 : l * c.sl + g * c.sh + at.row;
    p.scale = l * c.ssl + g * c.ssh + at.scale;
    s_place[threadIdx.x] = p;
    // without positions a token's is its row, the same for all layers and heads
    if constexpr (TURN && ONCE) s_position[tok - tok0] = a.rot.positions ? a.rot.positions[tok] : (int)row;
  }
  if constexpr (TURN && ONCE) __syncthreads();
  if constexpr (TURN) {
    for (unsigned w = kThreads - 1 - threadIdx.x; w < tokens * half; w += kThreads) {
      const unsigned i = w / half, p = w - i * half;
      int position;
      if constexpr (ONCE) {
        position = s_position[i];
      } else if (a.rot.positions) {
        position = a.rot.positions[tok0 + i];
      } else {
        const Token t = token_of(s_kept, a.seq, tok0 + i);
        position = len_of(s_kept, a.seq, c, l, t.b, 0) + t.i;
      }
      s_cs[w] = ta_cos_sin(a.rot, a.rot.phase[p], position);
    }
  }
  __syncthreads();
  // the row's coordinates of this lane, rotated
  float2 cs[8];
  unsigned of_cs = ~0u;  // the token that they are of
  auto turn = [&](float (&f)[8], const uint4& x, int w) {
    const unsigned tok = (first + w) / c.Hkv - tok0;
    const int at = lane * 8;
    if (a.rot.interleaved) {
      if (at < a.rot.d_rot && tok != of_cs) {
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e] = s_cs[tok * half + lane * 4 + e];
      }
      if (at < a.rot.d_rot) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = f[2 * e], q = f[2 * e + 1];
          f[2 * e] = p * cs[e].x - q * cs[e].y;
          f[2 * e + 1] = p * cs[e].y + q * cs[e].x;
        }
      }
    } else {  // partners are `half` coordinates away: a multiple of 4
      const uint32_t word[4] = {x.x, x.y, x.z, x.w};
      uint32_t o[4];
      const int leader = (threadIdx.x & 31) - lane;
      if ((half & 7) == 0) {
        const int from = leader + (((at < half ? at + half : at - half) >> 3) & (N - 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __shfl_sync(0xffffffffu, word[e], from);
      } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {  // four coordinates of one side
          const int mine = at + 4 * q, other = mine < half ? mine + half : mine - half;
          const int from = leader + ((other >> 3) & (N - 1));
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t lo = __shfl_sync(0xffffffffu, word[e], from), hi = __shfl_sync(0xffffffffu, word[2 + e], from);
            o[2 * q + e] = (other & 4) ? hi : lo;  // the partners are a lane's lower or upper four
          }
        }
      }
      if (at < a.rot.d_rot) {  // (a multiple of 8)
        if (tok != of_cs) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int mine = at + 4 * q;
            const float4* r = reinterpret_cast<const float4*>(s_cs + tok * half + (mine < half ? mine : mine - half));
            const float sign = mine < half ? -1.0f : 1.0f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float4 two = r[e];
              cs[4 * q + 2 * e] = make_float2(two.x, two.y * sign);
              cs[4 * q + 2 * e + 1] = make_float2(two.z, two.w * sign);
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = both(o[e]);
          f[2 * e] = f[2 * e] * cs[2 * e].x + p.x * cs[2 * e].y;
          f[2 * e + 1] = f[2 * e + 1] * cs[2 * e + 1].x + p.y * cs[2 * e + 1].y;
        }
      }
    }
    of_cs = tok;
  };
  auto open = [&](const uint4& x, float (&f)[8]) {
    const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 p = both(word[e]);
      f[2 * e] = p.x;
      f[2 * e + 1] = p.y;
    }
  };
  auto largest = [&](const float (&f)[8]) {  // magnitude in a row; a NaN is larger than all
    float m = fabsf(f[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) m = max_nan(m, fabsf(f[e]));
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
  };
  auto code = [&](const float (&f)[8], float inv, bool fine) {
    uint2 r;
    if constexpr (FMT == TA_CACHE_E4M3)
      r = make_uint2(e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), e4m3x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
    else r = make_uint2(int8x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), int8x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
    return fine ? r : make_uint2(0u, 0u);
  };
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int w = group * PER + i;
    const bool is = w < todo;  // a group without an item goes along (shuffles) and writes nothing
    if (!is) k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
    const Place place = s_place[is ? w : 0];
    const bool put = is && place.row >= 0;
    float f[8];
    if constexpr (!CODES) {
      if constexpr (TURN) {
        open(k[i], f);
        turn(f, k[i], is ? w : 0);
        k[i] = make_uint4(pack(f[0], f[1]), pack(f[2], f[3]), pack(f[4], f[5]), pack(f[6], f[7]));
      }
      if (put) {
        *reinterpret_cast<uint4*>(c.k + place.row + lane * 16) = k[i];
        *reinterpret_cast<uint4*>(c.v + place.row + lane * 16) = v[i];
      }
    } else {
      float h[8];
      open(k[i], f);
      if constexpr (TURN) turn(f, k[i], is ? w : 0);
      open(v[i], h);
      const float mk = largest(f), mv = largest(h);
      // one lane divides for the keys, the next for the values
      constexpr float FULL = FMT == TA_CACHE_E4M3 ? 448.0f : 127.0f;
      const float mine = (lane & 1) ? mv : mk, m = fmaxf(mine, 0x1p-100f), quotient = __fdiv_rn(FULL, m);
      const int leader = (threadIdx.x & 31) - lane;
      const float ik = __shfl_sync(0xffffffffu, quotient, leader), iv = __shfl_sync(0xffffffffu, quotient, leader + 1);
      const uint2 ck = code(f, ik, mk < INFINITY), cv = code(h, iv, mv < INFINITY);
      if (put) {
        *reinterpret_cast<uint2*>(c.k + place.row + lane * 8) = ck;
        *reinterpret_cast<uint2*>(c.v + place.row + lane * 8) = cv;
        if (lane < 2) (lane ? c.vs : c.ks)[place.scale] = mine < INFINITY ? ta_div_by(m, FULL, __frcp_rn(FULL)) : __int_as_float(0x7fc00000);
      }
    }
  }
}

// Items in the order [B][Hkv][n], or [Hkv][total] where the batch is ragged. grid.x = ITEMS of them, grid.y = layers.
template <int D, int FMT, int ITEMS>
__global__ void __launch_bounds__(kThreads) ta_cache_read_kernel(ta_cache_move_args a, ta_dev_status* status) {
  ta_wait_for_prior_grid();
  ta_launch_dependents();
  constexpr int N = Lanes<D>::N, GROUPS = Lanes<D>::GROUPS, PER = ITEMS / GROUPS;
  constexpr bool CODES = FMT != TA_CACHE_BF16;
  __shared__ Place s_place[ITEMS];
  __shared__ Kept s_kept;
  __shared__ Sides s_side[ITEMS];
  __shared__ float2 s_scale[ITEMS];
  const ta_cache_dev& c = a.cache;
  const int lane = threadIdx.x % N, group = threadIdx.x / N, l = blockIdx.y;
  const unsigned first = blockIdx.x * ITEMS, todo = min((unsigned)ITEMS, (unsigned)a.seq.total * c.Hkv - first);
  if (a.seq.cu) {
    keep(s_kept, a.seq, c, false);
    __syncthreads();
  }
  if (threadIdx.x < todo) {  // one thread finds an item's places
    const unsigned w = first + threadIdx.x;
    Token t;
    int g;
    unsigned tok = 0;
    if (a.seq.cu) {
      g = (int)(w / (unsigned)a.seq.total);
      tok = w - (unsigned)g * (unsigned)a.seq.total;
      t = token_of(s_kept, a.seq, tok);
    } else {
      const unsigned u = w / (unsigned)a.seq.n_uniform;
      t.i = (int)(w - u * a.seq.n_uniform);
      t.b = (int)(u / (unsigned)c.Hkv);
      g = (int)(u - (unsigned)t.b * c.Hkv);
    }
    s_side[threadIdx.x] = {view_at(a.k, a.seq, l, g, t, tok), view_at(a.v, a.seq, l, g, t, tok)};
    const int row = a.rows ? a.rows[rows_at(a.seq, c.Hkv, l, g, t, tok)] : t.i;
    const ta_row_at at = row >= 0 ? ta_cache_row(c, t.b, row) : ta_row_at{-1, 0};
    if (row >= 0 && at.row < 0) ta_report_bounds(status, 31, t.b, row);
    const long long at_scale = l * c.ssl + g * c.ssh + at.scale;
    s_place[threadIdx.x] = {at.row < 0 ? -1 : l * c.sl + g * c.sh + at.row, at_scale};
    if constexpr (CODES) {
      s_scale[threadIdx.x] = at.row < 0 ? make_float2(0.0f, 0.0f) : make_float2(c.ks[at_scale], c.vs[at_scale]);
    }
  }
  __syncthreads();
  uint4 x[PER][CODES ? 1 : 2];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int w = group + k * GROUPS;
    const long long row = s_place[w].row + lane * (CODES ? 8 : 16);
    const bool is = w < todo && s_place[w].row >= 0;
    if constexpr (CODES) {
      uint2 p = make_uint2(0u, 0u), q = p;
      if (is) {
        p = load8(c.k + row);
        q = load8(c.v + row);
      }
      x[k][0] = make_uint4(p.x, p.y, q.x, q.y);
    } else {
      x[k][0] = x[k][1] = make_uint4(0u, 0u, 0u, 0u);
      if (is) {
        x[k][0] = load16(c.k + row);
        x[k][1] = load16(c.v + row);
      }
    }
  }
  auto value = [&](uint32_t w, int e) {  // code e of a word
    if constexpr (FMT == TA_CACHE_E4M3) {
      const __half h = __half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)(w >> (8 * e)), __NV_E4M3));
      return __half2float(h);
    } else {
      return (float)(int)(int8_t)(w >> (8 * e));
    }
  };
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int w = group + k * GROUPS;
    if (w >= todo) break;
    const float2 scales = CODES ? s_scale[w] : make_float2(0.0f, 0.0f);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint4 o;
      if constexpr (CODES) {
        const uint32_t p = kv ? x[k][0].z : x[k][0].x, q = kv ? x[k][0].w : x[k][0].y;
        const float s = kv ? scales.y : scales.x;
        o.x = pack(value(p, 0) * s, value(p, 1) * s);
        o.y = pack(value(p, 2) * s, value(p, 3) * s);
        o.z = pack(value(q, 0) * s, value(q, 1) * s);
        o.w = pack(value(q, 2) * s, value(q, 3) * s);
      } else {
        o = x[k][kv];
      }
      uint16_t* dst = reinterpret_cast<uint16_t*>(const_cast<void*>(kv ? a.v.ptr : a.k.ptr)) + (kv ? s_side[w].v : s_side[w].k) + lane * 8;
      ta_st_stream(reinterpret_cast<uint4*>(dst), o);
    }
  }
}

cudaLaunchConfig_t config(const ta_cache_move_args& a, int items, cudaStream_t stream, cudaLaunchAttribute* attr) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((a.seq.total * a.cache.Hkv + items - 1) / items), (unsigned)a.n_layers, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = stream;
  ta_pdl_attribute(attr);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}
template <int D, int FMT, int ITEMS>
cudaError_t append(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(a, ITEMS, stream, attr);
  if (!a.rot.phase) return cudaLaunchKernelEx(&cfg, ta_cache_append_kernel<D, FMT, false, ITEMS>, a, status);
  const int tokens = (ITEMS + a.cache.Hkv - 2) / a.cache.Hkv + 1;  // that a block's items may belong to
  cfg.dynamicSmemBytes = (size_t)tokens * (a.rot.d_rot / 2) * sizeof(float2);
  return cudaLaunchKernelEx(&cfg, ta_cache_append_kernel<D, FMT, true, ITEMS>, a, status);
}
template <int D, int FMT, int ITEMS>
cudaError_t read(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(a, ITEMS, stream, attr);
  return cudaLaunchKernelEx(&cfg, ta_cache_read_kernel<D, FMT, ITEMS>, a, status);
}
template <int D, int FMT>
cudaError_t move(bool write, const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  // (a block has 128 / (D / 8) groups of lanes and at least one row for each)
  constexpr int FEW = kFewItems > Lanes<D>::GROUPS ? kFewItems : Lanes<D>::GROUPS;
  if (a.seq.total * a.cache.Hkv * a.n_layers <= kFewRows)
    return write ? append<D, FMT, FEW>(a, status, stream) : read<D, FMT, FEW>(a, status, stream);
  return write ? append<D, FMT, kItems>(a, status, stream) : read<D, FMT, kItems>(a, status, stream);
}
template <int D>
cudaError_t move(bool write, const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  if (a.cache.format == TA_CACHE_BF16) return move<D, TA_CACHE_BF16>(write, a, status, stream);
  if (a.cache.format == TA_CACHE_E4M3) return move<D, TA_CACHE_E4M3>(write, a, status, stream);
  return move<D, TA_CACHE_INT8>(write, a, status, stream);
}

}  // namespace

cudaError_t ta_launch_cache_append(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  if (a.seq.total == 0) return cudaSuccess;
  return a.d == 64 ? move<64>(true, a, status, stream) : move<128>(true, a, status, stream);
}
cudaError_t ta_launch_cache_read(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream) {
  if (a.seq.total == 0) return cudaSuccess;
  return a.d == 64 ? move<64>(false, a, status, stream) : move<128>(false, a, status, stream);
}
