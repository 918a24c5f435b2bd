// Attention of new tokens over a cache.
//
// A unit (layer, sequence, KV head) has R = (Hq / Hkv) * T query rows that read the same n cache rows, each once: 4 d R
// operations for 4 d bytes (bf16), so up to some tens of query rows the cache's bytes are the bound, and everything below
// serves to keep them coming. The cache rows of a unit are cut into pieces, a block each; a block's warps take its tiles (16
// or 32 rows) in turn, each with two slots of its own in shared memory that asynchronous 16-byte copies fill a tile ahead, so
// no warp waits for another before the end. Any page size and any strides: a lane looks up one row of a tile a tile before
// that. Rows that are not there are filled with zeros and masked.
//
// Per tile and warp: scores S = Q K^T on the tensor cores (m16n8k16, fp32 sums), a running maximum and sum per query row,
// O = O + P V on the tensor cores with P straight from the score registers. Products have 8 to 32 rows: far too few for a
// tcgen05 tile of 128 to pay, and what moves the data is the same. The order of the d coordinates inside a product is free as
// long as both operands use the same one: a lane's 16 bytes of a key row serve as its fragments of two (bf16) or four (8-bit)
// products without a shuffle.
//
// Precision. bf16 caches: products of bf16 values. 8-bit caches: codes are exact in fp16; queries are scaled per row by a power
// of two into fp16's range (and back in the score's factor), the scale of a key row multiplies its scores, that of a value row
// its probabilities, relative to a power of two that is a query row's own. Probabilities and rotated queries
// enter their products as a sum of two 16-bit parts, hi + lo: with up to 8 query rows the lower half of the 16-row product,
// which would be empty, holds the lo parts at no cost (MB = 0); with more rows the lo parts are a second product.
//
// What bounds it. bf16: memory, 16 x 32768 rows of 8 heads in 306 us, 7.0 TB/s. 8-bit: instructions, 914 for a tile of 32 rows, of
// which 384 turn codes into fp16 and 64 are products: 36 x 16384 e4m3 rows of 8 heads 225 us, 5.5 TB/s. With 16 query rows 1170 for a
// tile, and latency: issue slots 52 % taken, tensor cores 46 %, memory 41 %, three warps a scheduler that wait for their own
// results (4 x 100001 to 131072 int8 rows of 4 heads 130 us, 3.6 TB/s). Cache rows as the long side of the products (S^T = K Q^T, half of them and of the
// accumulators, four blocks an SM instead of three) were slower, 275 us where this took 238: no fewer instructions, and less
// distance between those that depend on one another. Tiles of 16 rows for codes: 297 for 251. Bulk copies for codes: 511 for 296 row by
// row, 247 for 250 in runs of 16 rows.
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "ta_cache.cuh"
#include "ta_sm100.cuh"

namespace {

using ta_sm100::ex2;
using ta_sm100::smem_u32;

template <int D, int FMT, int W>  // W: warps of a block
struct Shape {
  static constexpr bool CODES = FMT != TA_CACHE_BF16;
  static constexpr int ROW = D * (CODES ? 1 : 2);                 // bytes of a row
  static constexpr int CHUNKS = ROW / 16;
  static constexpr int TK = (CODES || D == 64) ? 32 : 16;         // cache rows of a tile
  static constexpr int TILE = TK * ROW;                           // bytes of K, and of V, in a stage
  static constexpr int STAGE = 2 * TILE + (CODES ? 2 * TK * 4 : 0);
  static constexpr int STAGES = 2;
  static constexpr int KS = D / 16;                               // products along d
  static constexpr int RING = W * STAGES * STAGE;
};
template <int D, int FMT, int MB, int W>
constexpr int smem_bytes() {
  constexpr int R = ta_attend_rows(MB);
  constexpr int q32 = R * D * 4;  // queries in fp32, then (MB > 0) their fragments, hi and lo, in the same place
  constexpr int join = W * R * (D + 4) * 4;
  constexpr int ring = Shape<D, FMT, W>::RING > join ? Shape<D, FMT, W>::RING : join;
  return ring + q32 + R * 4 /* row factors */ + W * R * 8 /* maxima and sums */ + W * Shape<D, FMT, W>::STAGES * 4 + 16;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ const void* at16(const void* base, uint32_t units) {  // base + 16 * units, in one product
  uint64_t r;
  asm("mad.wide.u32 %0, %1, 16, %2;" : "=l"(r) : "r"(units), "l"(base));
  return reinterpret_cast<const void*>(r);
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ float2 lds_f2(uint32_t a) {
  const uint2 v = lds64(a);
  return make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a));
}
template <bool CODES>  // fp16 operands for 8-bit caches, bf16 otherwise
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (CODES)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x and y as a pair of 16-bit values (x in the lower half), and what the rounding left
template <bool CODES>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  uint32_t r;
  if constexpr (CODES) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
template <bool CODES>
__device__ __forceinline__ float2 unpack2(uint32_t p) {
  if constexpr (CODES) return __half22float2(*reinterpret_cast<__half2*>(&p));
  else return make_float2(__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u));
}
template <bool CODES>
__device__ __forceinline__ uint32_t rest2(float x, float y, uint32_t hi) {
  const float2 h = unpack2<CODES>(hi);
  return pack2<CODES>(x - h.x, y - h.y);
}
// Codes as fp16, exactly, without the conversion unit (16 lanes a clock: cvt.f16x2.e4m3x2 kept the whole kernel at a fifth of the
// memory's rate). Bytes i of x and y become a pair:
//   E4M3: both bytes with their signs spread over the byte above (one permute), shifted so that the four exponent and three
//     mantissa bits stand where fp16 has the last four and first three of its own, the sign that lands on the fifth exponent
//     bit masked out: the value times 2^-8 (kCodeUnit), subnormals included. The shift is a product with a number that the
//     compiler does not know: the other two instructions load the integer pipe, this one the multipliers.
//   INT8: the byte with its upper bit turned over is c + 128; under the exponent of 1024 that is 1152 + c, less 1152. (A number put under
//     the exponent that makes its unit the mantissa's last place: a published way to convert integers, the constants follow from fp16.)
template <int FMT, int I>
__device__ __forceinline__ uint32_t pair_of(uint32_t x, uint32_t y, uint32_t times128) {
  if constexpr (FMT == TA_CACHE_E4M3) {
    constexpr uint32_t SEL = (uint32_t)I | (uint32_t)(I + 8) << 4 | (uint32_t)(I + 4) << 8 | (uint32_t)(I + 12) << 12;
    uint32_t p;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(p) : "r"(x), "r"(y), "n"(SEL));
    return (p * times128) & 0xbf80bf80u;
  } else {
    constexpr uint32_t SEL = (uint32_t)I | (uint32_t)I << 4 | (uint32_t)(I + 4) << 8 | (uint32_t)(I + 4) << 12;
    const uint32_t p = (__byte_perm(x, y, SEL) & 0x00ff00ffu) ^ 0x64806480u;
    const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&p), __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}
template <int FMT>
constexpr int kCodeUnit = FMT == TA_CACHE_E4M3 ? 8 : 0;  // fp16 operands are the codes times 2^-kCodeUnit
// the four codes of a word of a key row, as pairs (0, 1) and (2, 3)
template <int FMT>
__device__ __forceinline__ void expand(uint32_t w, uint32_t& lo, uint32_t& hi, uint32_t times128) {
  if constexpr (FMT == TA_CACHE_E4M3) {  // (the permute takes the bytes where they are)
    uint32_t p, q;
    asm("prmt.b32 %0, %1, %1, 0x9180;" : "=r"(p) : "r"(w));
    asm("prmt.b32 %0, %1, %1, 0xb3a2;" : "=r"(q) : "r"(w));
    lo = (p * times128) & 0xbf80bf80u;
    hi = (q * times128) & 0xbf80bf80u;
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t p = __byte_perm(u, 0x64646464u, 0x4140), q = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&p), off), y = __hsub2(*reinterpret_cast<const __half2*>(&q), off);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }  // -126 <= e <= 127

struct Unit {
  int l, b, g, n;  // n: rows that are there
};
__device__ __forceinline__ Unit unit_of(const ta_attend_args& a, int unit) {  // n still to come
  const ta_cache_dev& c = a.cache;
  const int lb = unit / c.Hkv, l = lb / c.batch;
  return {l, lb - l * c.batch, unit - lb * c.Hkv, 0};
}
__device__ __forceinline__ int rows_of_unit(const ta_attend_args& a, const Unit& u, int len, bool report, ta_dev_status* status) {
  const long long asked = (long long)len + a.new_rows;
  const long long most = min((long long)a.max_len, (long long)a.cache.wide * a.cache.page);
  if (asked > most && report) ta_report_bounds(status, 32, u.b, (int)min(asked, 0x7fffffffLL));
  return (int)max(0LL, min(asked, most));
}

struct Cut {                     // how the kernel's blocks share the cache rows of a unit's row block
  int pieces, piece, row_blocks;
  int target;               // 0, or: pieces are as long as gives this many in the whole call; `piece` is not used then
  int groups_per_sequence;  // units and row blocks of a sequence, for that
};
struct Scratch {    // of one call (null: not used)
  float* part;      // [unit][row block][piece][row][D], unnormalised
  float2* part_ml;  // [unit][row block][piece][row]: maximum (in bits) and sum
  int* ticket;      // [unit][row block], zero between calls
  float* score;     // [unit][row][score_stride], in bits
  float2* row_ml;   // [unit][row]: maximum and 1 / sum for the attention mass
  long long score_stride;
};

// blockIdx.x = (unit * row blocks + block) * pieces + piece
template <int D, int FMT, int MB, int W>
__global__ void __launch_bounds__(W * 32, (MB < 2 ? 12 : 8) / W) ta_attend_kernel(ta_attend_args a, Scratch sc, Cut cut,
                                                              uint32_t times128, ta_dev_status* status) {
  using S = Shape<D, FMT, W>;
  constexpr int kWarps = W, kThreads = W * 32;
  constexpr bool CODES = S::CODES, NARROW = MB == 0;
  constexpr int TK = S::TK, NT = TK / 8, KS = S::KS, R = ta_attend_rows(MB), MBN = NARROW ? 1 : MB, NR = NARROW ? 1 : 2 * MB;
  constexpr int NJ = D / 8;  // 8-wide tiles of the output
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int join_bytes = kWarps * R * (D + 4) * 4;
  uint8_t* s_at = smem + (S::RING > join_bytes ? S::RING : join_bytes);
  float* s_q = reinterpret_cast<float*>(s_at);
  uint4* s_frag = reinterpret_cast<uint4*>(s_at);  // [hi, lo][mb][ks][lane]
  s_at += R * D * 4;
  float* s_factor = reinterpret_cast<float*>(s_at);
  float2* s_ml = reinterpret_cast<float2*>(s_factor + R);
  uint32_t* s_there = reinterpret_cast<uint32_t*>(s_ml + kWarps * R);
  int* s_last = reinterpret_cast<int*>(s_there + kWarps * S::STAGES);

  ta_wait_for_prior_grid();
  ta_launch_dependents();
  const ta_cache_dev& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
  const int group = blockIdx.x / cut.pieces, part = blockIdx.x - group * cut.pieces;
  const int unit = group / cut.row_blocks, r0 = (group - unit * cut.row_blocks) * R;
  Unit u = unit_of(a, unit);
  const int G = a.Hq / c.Hkv, rows = G * a.T;
  const int len = ta_cache_len(c, u.l, u.b, u.g);
  // A lane's row of a coming tile: its page's number is read a tile early, the first one's beside the length, and not looked at
  // before the row is fetched.
  int page_id = 0, page_row = 0;
  auto look_up = [&](int r) {
    const int j = c.page_shift >= 0 ? r >> c.page_shift : (int)((unsigned)r / (unsigned)c.page);
    page_row = r - j * c.page;
    page_id = -1;
    if (j < c.wide) {
      if (c.table) page_id = c.table[u.b * (long long)c.wide + j];
      else page_id = u.b * c.wide + j;
    }
  };
  if (!cut.target) look_up(part * cut.piece + warp * TK + lane);
  u.n = rows_of_unit(a, u, len, part == 0 && r0 == 0 && tid == 0, status);
  int piece = cut.piece;
  if (cut.target) {  // pieces of all sequences' rows shared out evenly, not of max_len
    const int most = (int)min((long long)a.max_len, (long long)c.wide * c.page);
    int sum = 0;
    for (int b = tid; b < c.batch; b += kThreads) sum += (int)max(0LL, min((long long)c.lens[b] + a.new_rows, (long long)most));
    sum = __reduce_add_sync(0xffffffffu, sum);
    if (lane == 0) s_there[warp] = (uint32_t)sum;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all += s_there[w];
    __syncthreads();  // (the words are used again)
    all *= cut.groups_per_sequence;
    const int even = (int)((all + cut.target - 1) / cut.target), least = (most + cut.pieces - 1) / cut.pieces;
    piece = (max(max(even, least), 1) + kAttendPieceUnit - 1) / kAttendPieceUnit * kAttendPieceUnit;
  }
  const int n_pieces = max(1, (u.n + piece - 1) / piece);  // at least one, which writes the empty result
  if (part >= n_pieces) return;
  const int begin = part * piece, end = min(u.n, begin + piece);
  const int tiles = (end - begin + TK - 1) / TK, mine = tiles > warp ? (tiles - warp + kWarps - 1) / kWarps : 0;

  // ---- the ring
  constexpr uint32_t kAllRows = TK == 32 ? 0xffffffffu : (1u << TK) - 1;
  const uint8_t *k_base = c.k + u.l * c.sl + u.g * c.sh, *v_base = c.v + u.l * c.sl + u.g * c.sh;
  const uint32_t sp16 = (uint32_t)(c.sp >> 4), sr16 = (uint32_t)(c.sr >> 4);
  const uint32_t ring = smem_u32(smem) + warp * S::STAGES * S::STAGE;
  uint32_t* there_w = s_there + warp * S::STAGES;
  auto row_at = [&](int i) { return begin + (warp + i * kWarps) * TK + lane; };  // the lane's row of the warp's i-th tile
  uint32_t at_row = 0, at_scale = 0;  // in units of 16 bytes, and of the scale
  bool at_there = false;
  auto place = [&](int i) {
    const bool asked = lane < TK && row_at(i) < end;
    at_there = asked && page_id >= 0 && page_id < c.n_pages;
    if (asked && !at_there) ta_report_bounds(status, 33, u.b, row_at(i));
    at_row = at_there ? (uint32_t)page_id * sp16 + (uint32_t)page_row * sr16 : 0u;
    at_scale = at_there ? (uint32_t)page_id * (uint32_t)c.ssp + (uint32_t)page_row * (uint32_t)c.ssr : 0u;
  };
  // A lane's 16 bytes of a row are the same for all the tile's rows that it copies, CHUNKS / 32 rows apart. Swizzles: eight lanes
  // that read 16 bytes each at a time meet all banks (keys: two rows and four chunks; values: eight rows of one chunk through
  // ldmatrix, or, of codes, four even rows and two chunks).
  constexpr int ROWS_AT_ONCE = 32 / S::CHUNKS;
  const int my_row = lane / S::CHUNKS, my_chunk = lane % S::CHUNKS;
  const uint8_t *k_lane = k_base + my_chunk * 16, *v_lane = v_base + my_chunk * 16;
  const float *ks_base = c.ks + u.l * c.ssl + u.g * c.ssh, *vs_base = c.vs + u.l * c.ssl + u.g * c.ssh;
  auto copy = [&](uint32_t dst, auto all) {  // all: every row is there
    uint32_t there = 0;
    if constexpr (!decltype(all)::value) there = __ballot_sync(0xffffffffu, at_there);
#pragma unroll
    for (int k = 0; k < TK / ROWS_AT_ONCE; ++k) {
      const int row = k * ROWS_AT_ONCE + my_row;
      const uint32_t at = __shfl_sync(0xffffffffu, at_row, row);
      const int kx = S::CHUNKS >= 8 ? (row & 1) << 2 : 0;
      const int vx = !CODES ? row & 7 : S::CHUNKS >= 8 ? ((row >> 1) & 3) << 1 : (row >> 1) & 3;
      const uint32_t to_k = dst + row * S::ROW + ((my_chunk ^ kx) << 4), to_v = dst + S::TILE + row * S::ROW + ((my_chunk ^ vx) << 4);
      if constexpr (decltype(all)::value) {
        cp16(to_k, at16(k_lane, at));
        cp16(to_v, at16(v_lane, at));
      } else {  // (a row that is not there stands at the pool's start and is not read)
        cp16(to_k, at16(k_lane, at), (there >> row) & 1);
        cp16(to_v, at16(v_lane, at), (there >> row) & 1);
      }
    }
    if constexpr (CODES) {
      cp4(dst + 2 * S::TILE + lane * 4, ks_base + at_scale, at_there);
      cp4(dst + 2 * S::TILE + TK * 4 + lane * 4, vs_base + at_scale, at_there);
    }
  };
  auto issue = [&](int i) {
    if (i < mine) {
      const int stage = i % S::STAGES;
      const uint32_t dst = ring + stage * S::STAGE;
      place(i);
      const uint32_t there = __ballot_sync(0xffffffffu, at_there);
      if (lane == 0) there_w[stage] = there;
      if (there == kAllRows) copy(dst, std::true_type{});
      else copy(dst, std::false_type{});
      look_up(row_at(i + 1));
    }
    cp_commit();
  };
  if (cut.target) look_up(row_at(0));
#pragma unroll
  for (int i = 0; i < S::STAGES - 1; ++i) issue(i);

  // ---- the queries
  auto limit_of = [&](int r) {  // cache rows that the block's row r sees
    const int row = r0 + r;
    return row < rows ? max(0, u.n - (a.causal ? a.T - 1 - row / G : 0)) : 0;
  };
  auto query = [&](int row) {
    const int t = row / G, h = u.g * G + row - t * G;
    return reinterpret_cast<const __nv_bfloat16*>(a.q.ptr) + u.l * a.q.stride_l + u.b * a.q.stride_b + h * a.q.stride_h +
           t * a.q.stride_n;
  };
  // up to 8 rows that are not rotated go straight to the fragments, others to shared memory in fp32 first
  const bool straight = NARROW && !a.rot.phase;
  const int n_rows = min(R, rows - r0);
  if (!straight) {
    const int half = a.rot.phase ? a.rot.d_rot / 2 : 0, rest = (D - 2 * half) / 4;  // pairs, and fours that are not rotated
    for (int w = tid; w < n_rows * half; w += kThreads) {
      const int r = w / half, p = w - r * half, row = r0 + r;
      const int c0 = a.rot.interleaved ? 2 * p : p, c1 = a.rot.interleaved ? 2 * p + 1 : p + half;
      const __nv_bfloat16* q = query(row);
      const float x = __bfloat162float(q[c0]), y = __bfloat162float(q[c1]);
      const int position = a.rot.positions ? a.rot.positions[u.b * a.T + row / G] : u.n - a.T + row / G;
      const float2 cs = ta_cos_sin(a.rot, a.rot.phase[p], position);
      s_q[r * D + c0] = x * cs.x - y * cs.y;
      s_q[r * D + c1] = x * cs.y + y * cs.x;
    }
    for (int w = tid; w < n_rows * rest; w += kThreads) {
      const int r = w / rest, c0 = 2 * half + (w - r * rest) * 4;
      const uint2 x = *reinterpret_cast<const uint2*>(query(r0 + r) + c0);
      const float2 lo = unpack2<false>(x.x), hi = unpack2<false>(x.y);
      *reinterpret_cast<float4*>(s_q + r * D + c0) = make_float4(lo.x, lo.y, hi.x, hi.y);
    }
    for (int w = tid + n_rows * (D / 4); w < R * (D / 4); w += kThreads)
      reinterpret_cast<float4*>(s_q)[w] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncthreads();
  }
  // a row's part of four coordinates for product ks: the order in which a lane's bytes of a key row come
  auto coordinate = [&](int ks) { return CODES ? (t4 + 4 * (ks / 4)) * 16 + (ks % 4) * 4 : (t4 + 4 * (ks / 2)) * 8 + (ks % 2) * 4; };
  const float bits = a.scale * 1.4426950408889634f * pow2(kCodeUnit<FMT>);
  // 8-bit caches: a power of two that brings a row's largest value into [1, 2); m: the largest of this lane's
  auto row_scale = [&](float m, float& down) {
    if constexpr (CODES) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    }
    const int e = CODES ? min(max((int)(__float_as_uint(m) >> 23) - 127, -100), 126) : 0;
    down = pow2(-e);
    return bits * pow2(e);
  };
  auto largest = [](float m, const float4& v) { return fmaxf(m, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w)))); };
  auto staged = [&](int r, int at) { return *reinterpret_cast<const float4*>(s_q + r * D + at); };
  auto staged_scale = [&](int r, float& down) {
    float m = 0.0f;
    if constexpr (CODES) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) m = largest(m, staged(r, coordinate(ks)));
    }
    return row_scale(m, down);
  };
  uint32_t qf[NARROW ? KS : 1][4];
  float factor[NR];
  int limit[NR];
  if constexpr (NARROW) {
    float down;
    limit[0] = limit_of(g8);
    if (straight) {
      const bool is = r0 + g8 < rows;
      const __nv_bfloat16* q = is ? query(r0 + g8) : nullptr;
      uint2 w[KS];
      float m = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) w[ks] = is ? *reinterpret_cast<const uint2*>(q + coordinate(ks)) : make_uint2(0u, 0u);
      if constexpr (CODES) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const float2 x = unpack2<false>(w[ks].x), y = unpack2<false>(w[ks].y);
          m = largest(m, make_float4(x.x, x.y, y.x, y.y));
        }
      }
      factor[0] = row_scale(m, down);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if constexpr (CODES) {
          const float2 x = unpack2<false>(w[ks].x), y = unpack2<false>(w[ks].y);
          qf[ks][0] = pack2<CODES>(x.x * down, x.y * down);
          qf[ks][2] = pack2<CODES>(y.x * down, y.y * down);
          qf[ks][1] = rest2<CODES>(x.x * down, x.y * down, qf[ks][0]);
          qf[ks][3] = rest2<CODES>(y.x * down, y.y * down, qf[ks][2]);
        } else {
          qf[ks][0] = w[ks].x;
          qf[ks][2] = w[ks].y;
          qf[ks][1] = qf[ks][3] = 0u;
        }
      }
    } else {
      factor[0] = staged_scale(g8, down);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const float4 v = staged(g8, coordinate(ks));
        qf[ks][0] = pack2<CODES>(v.x * down, v.y * down);
        qf[ks][2] = pack2<CODES>(v.z * down, v.w * down);
        qf[ks][1] = rest2<CODES>(v.x * down, v.y * down, qf[ks][0]);
        qf[ks][3] = rest2<CODES>(v.z * down, v.w * down, qf[ks][2]);
      }
    }
  } else {
    constexpr int PER_WARP = KS / kWarps;  // products of a warp, of every 16 rows
    uint4 hi[MB][PER_WARP], lo[MB][PER_WARP];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      float d0, d1;
      const float f0 = staged_scale(mb * 16 + g8, d0), f1 = staged_scale(mb * 16 + g8 + 8, d1);
      if (warp == 0 && t4 == 0) s_factor[mb * 16 + g8] = f0, s_factor[mb * 16 + g8 + 8] = f1;
#pragma unroll
      for (int i = 0; i < PER_WARP; ++i) {
        const int at = coordinate(warp * PER_WARP + i);
        const float4 v = staged(mb * 16 + g8, at), w = staged(mb * 16 + g8 + 8, at);
        uint4 &h = hi[mb][i], &r = lo[mb][i];
        h.x = pack2<CODES>(v.x * d0, v.y * d0);
        h.y = pack2<CODES>(w.x * d1, w.y * d1);
        h.z = pack2<CODES>(v.z * d0, v.w * d0);
        h.w = pack2<CODES>(w.z * d1, w.w * d1);
        r.x = rest2<CODES>(v.x * d0, v.y * d0, h.x);
        r.y = rest2<CODES>(w.x * d1, w.y * d1, h.y);
        r.z = rest2<CODES>(v.z * d0, v.w * d0, h.z);
        r.w = rest2<CODES>(w.z * d1, w.w * d1, h.w);
      }
    }
    __syncthreads();  // the fragments take the queries' place
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int i = 0; i < PER_WARP; ++i) {
        s_frag[(mb * KS + warp * PER_WARP + i) * 32 + lane] = hi[mb][i];
        s_frag[((MB + mb) * KS + warp * PER_WARP + i) * 32 + lane] = lo[mb][i];
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      factor[i] = s_factor[(i / 2) * 16 + (i & 1) * 8 + g8];
      limit[i] = limit_of((i / 2) * 16 + (i & 1) * 8 + g8);
    }
  }
  const bool q_parts = a.rot.phase != nullptr;  // queries that are not rotated have no second part
  const uint32_t frag = smem_u32(s_frag) + lane * 16;
  const int seen_by_all = limit_of(0);  // the block's first row has the lowest limit

  float o[MBN][NJ][4], m[NR], l[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
  for (int i = 0; i < MBN; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][j][e] = 0.0f;
  // 8-bit caches: exponents that probabilities times value rows' scales are taken relative to, at least kLeastRef (the smallest scale
  // that ta_cache_append writes is above 2^-109)
  constexpr int kLeastRef = -112;
  int ref[CODES ? NR : 1];
  if constexpr (CODES) {
#pragma unroll
    for (int r = 0; r < NR; ++r) ref[r] = kLeastRef;
  }

  for (int i = 0; i < mine; ++i) {
    cp_wait<S::STAGES - 2>();
    __syncwarp();
    issue(i + S::STAGES - 1);
    const int stage = i % S::STAGES, first = begin + (warp + i * kWarps) * TK;
    const uint32_t kt = ring + stage * S::STAGE, vt = kt + S::TILE, st = kt + 2 * S::TILE;
    const uint32_t there = there_w[stage];
    const bool whole = there == kAllRows && first + TK <= seen_by_all;

    // ---- scores
    float s[MBN][NT][4];
#pragma unroll
    for (int x = 0; x < MBN; ++x)
#pragma unroll
      for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[x][y][e] = 0.0f;
    constexpr int PER = CODES ? 4 : 2;  // products that 16 bytes of a key row serve
#pragma unroll
    for (int k = 0; k < KS / PER; ++k) {
      uint4 w[NT];
#pragma unroll
      for (int y = 0; y < NT; ++y) {
        const int kx = S::CHUNKS >= 8 ? (g8 & 1) << 2 : 0;
        w[y] = lds128(kt + (y * 8 + g8) * S::ROW + (((t4 + 4 * k) ^ kx) << 4));
      }
#pragma unroll
      for (int h = 0; h < PER; ++h) {
        uint32_t b0[NT], b1[NT];
#pragma unroll
        for (int y = 0; y < NT; ++y) {
          const uint32_t* wy = reinterpret_cast<const uint32_t*>(&w[y]);
          if constexpr (CODES) expand<FMT>(wy[h], b0[y], b1[y], times128);
          else b0[y] = wy[2 * h], b1[y] = wy[2 * h + 1];
        }
        if constexpr (NARROW) {
#pragma unroll
          for (int y = 0; y < NT; ++y) mma<CODES>(s[0][y], qf[k * PER + h], b0[y], b1[y]);
        } else {
#pragma unroll
          for (int x = 0; x < MB; ++x) {
            uint4 q = lds128(frag + (x * KS + k * PER + h) * 512);
            const uint32_t qa[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int y = 0; y < NT; ++y) mma<CODES>(s[x][y], qa, b0[y], b1[y]);
            if (q_parts) {
              q = lds128(frag + ((MB + x) * KS + k * PER + h) * 512);
              const uint32_t ql[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
              for (int y = 0; y < NT; ++y) mma<CODES>(s[x][y], ql, b0[y], b1[y]);
            }
          }
        }
      }
    }
    // this thread's scores, in bits: x[row][8-row tile][2]
    float x[NR][NT][2];
    float2 vs[NT];
#pragma unroll
    for (int y = 0; y < NT; ++y) {
      float2 ks = make_float2(1.0f, 1.0f);
      vs[y] = ks;
      if constexpr (CODES) {
        ks = lds_f2(st + (y * 8 + 2 * t4) * 4);
        vs[y] = lds_f2(st + (TK + y * 8 + 2 * t4) * 4);
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        if constexpr (NARROW) {
          x[0][y][0] = (s[0][y][0] + s[0][y][2]) * (factor[0] * ks.x);
          x[0][y][1] = (s[0][y][1] + s[0][y][3]) * (factor[0] * ks.y);
        } else {
          x[r][y][0] = s[r / 2][y][(r & 1) * 2] * (factor[r] * ks.x);
          x[r][y][1] = s[r / 2][y][(r & 1) * 2 + 1] * (factor[r] * ks.y);
        }
      }
    }
    if (!whole) {
#pragma unroll
      for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int k = y * 8 + 2 * t4 + e;
          const bool is = (there >> k) & 1;
#pragma unroll
          for (int r = 0; r < NR; ++r)
            if (!is || first + k >= limit[r]) {
              x[r][y][e] = -INFINITY;
              if constexpr (CODES && NARROW) (e ? vs[y].y : vs[y].x) = 0.0f;  // (may be NaN)
            }
        }
    }
    if (sc.score) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int row = r0 + (NARROW ? g8 : (r / 2) * 16 + (r & 1) * 8 + g8);
        if (row < rows) {
          float* to = sc.score + ((long long)unit * rows + row) * sc.score_stride + first;
#pragma unroll
          for (int y = 0; y < NT; ++y)
            if (first + y * 8 + 2 * t4 < end) *reinterpret_cast<float2*>(to + y * 8 + 2 * t4) = make_float2(x[r][y][0], x[r][y][1]);
        }
      }
    }

    // ---- running maximum and sum
    float keep[NR];
    bool grew = false;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float top = m[r];
#pragma unroll
      for (int y = 0; y < NT; ++y) top = fmaxf(top, fmaxf(x[r][y][0], x[r][y][1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float from = top == -INFINITY ? 0.0f : top;
      keep[r] = ex2(m[r] - from);
      const int fell = CODES ? (int)fminf(from - m[r], 512.0f) : 0;  // whole bits by which what came before is taken down
      grew |= top > m[r];
      m[r] = top;
      float sum = 0.0f;
#pragma unroll
      for (int y = 0; y < NT; ++y) {
        x[r][y][0] = ex2(x[r][y][0] - from);
        x[r][y][1] = ex2(x[r][y][1] - from);
        sum += x[r][y][0] + x[r][y][1];
      }
      l[r] = l[r] * keep[r] + sum;
      if constexpr (CODES) {
        ref[r] -= fell;
        keep[r] *= pow2(min(fell, 126));
      }
    }
    if constexpr (CODES) {
      // Probabilities times their value rows' scales, for each query row relative to 2^ref, the largest that it has met (in the frame
      // of its running maximum), and times 2^14: at most 2^15, and 2^-38 of the largest is still told from zero. A scale that a
      // row does not see, or sees with next to no probability, takes nothing from the others, however large it is. (One reference for
      // all rows of a warp, from the scales alone, let such a scale wipe out what the other rows hold. A query row's own costs 2 to 4 %
      // with more than 8 rows and nothing with fewer.)
      if (NARROW || whole) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int y = 0; y < NT; ++y) {
            x[r][y][0] *= vs[y].x;
            x[r][y][1] *= vs[y].y;
          }
      } else {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int k = y * 8 + 2 * t4 + e;
              x[r][y][e] *= e ? vs[y].y : vs[y].x;
              if (!((there >> k) & 1) || first + k >= limit[r]) x[r][y][e] = 0.0f;  // (its scale may be NaN)
            }
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float top = 0.0f;
#pragma unroll
        for (int y = 0; y < NT; ++y) top = fmaxf(top, fmaxf(fabsf(x[r][y][0]), fabsf(x[r][y][1])));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int now = max(max(ref[r], (int)(__float_as_uint(top) >> 23) - 127), kLeastRef);
        const int by = now - ref[r];
        keep[r] *= by > 126 ? 0.0f : pow2(-by);
        grew |= by != 0;
        ref[r] = now;
        const float up = pow2(14 - now);
#pragma unroll
        for (int y = 0; y < NT; ++y) {
          x[r][y][0] *= up;
          x[r][y][1] *= up;
        }
      }
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int y = 0; y < MBN; ++y)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const float k0 = keep[NARROW ? 0 : 2 * y], k1 = keep[NARROW ? 0 : 2 * y + 1];
          o[y][j][0] *= k0;
          o[y][j][1] *= k0;
          o[y][j][2] *= k1;
          o[y][j][3] *= k1;
        }
    }

    // ---- values. Rows that a later token sees and an earlier one does not meet probabilities of zero; where such a row is
    // not finite, every token's rows are taken by themselves.
    bool apart = false;
    if (!CODES && first + TK > seen_by_all && seen_by_all < end) {  // (codes are finite, and scales were dealt with)
      bool bad = false;
      for (int w = lane; w < TK * S::CHUNKS; w += 32) {
        const int row = w / S::CHUNKS;
        if (first + row < seen_by_all) continue;
        const uint4 v = lds128(vt + row * S::ROW + (w % S::CHUNKS) * 16);
        const uint32_t* p = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          bad |= (p[k] & 0x7f80u) == 0x7f80u || (p[k] & 0x7f800000u) == 0x7f800000u;
        }
      }
      apart = __any_sync(0xffffffffu, bad);
    }
#pragma unroll
    for (int kk = 0; kk < TK / 16; ++kk) {
      uint32_t ph[MBN][4], pl[MBN][4];
#pragma unroll
      for (int y = 0; y < MBN; ++y) {
        if constexpr (NARROW) {
          ph[0][0] = pack2<CODES>(x[0][2 * kk][0], x[0][2 * kk][1]);
          ph[0][2] = pack2<CODES>(x[0][2 * kk + 1][0], x[0][2 * kk + 1][1]);
          ph[0][1] = rest2<CODES>(x[0][2 * kk][0], x[0][2 * kk][1], ph[0][0]);
          ph[0][3] = rest2<CODES>(x[0][2 * kk + 1][0], x[0][2 * kk + 1][1], ph[0][2]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 2 * y + (e & 1), tile = 2 * kk + (e >> 1);
            ph[y][e] = pack2<CODES>(x[r][tile][0], x[r][tile][1]);
            pl[y][e] = rest2<CODES>(x[r][tile][0], x[r][tile][1], ph[y][e]);
          }
        }
      }
      auto product = [&](int j, uint32_t b0, uint32_t b1) {
        if (!apart) {
#pragma unroll
          for (int y = 0; y < MBN; ++y) {
            mma<CODES>(o[y][j], ph[y], b0, b1);
            if constexpr (!NARROW) mma<CODES>(o[y][j], pl[y], b0, b1);
          }
          return;
        }
        int before = -1;
        for (int r = 0; r < R; ++r) {  // one product per limit; a row takes the result of its own
          const int lim = limit_of(r);
          if (lim == before) continue;
          before = lim;
          auto cut = [&](uint32_t v, int k) {
            if (first + kk * 16 + k >= lim) v &= 0xffff0000u;
            if (first + kk * 16 + k + 1 >= lim) v &= 0x0000ffffu;
            return v;
          };
          const uint32_t c0 = cut(b0, 2 * t4), c1 = cut(b1, 2 * t4 + 8);
#pragma unroll
          for (int y = 0; y < MBN; ++y) {
            float own[4] = {o[y][j][0], o[y][j][1], o[y][j][2], o[y][j][3]};
            mma<CODES>(own, ph[y], c0, c1);
            if constexpr (!NARROW) mma<CODES>(own, pl[y], c0, c1);
            const bool u0 = limit[NARROW ? 0 : 2 * y] == lim, u1 = limit[NARROW ? 0 : 2 * y + 1] == lim;
            if (u0) o[y][j][0] = own[0], o[y][j][1] = own[1];
            if (u1) o[y][j][2] = own[2], o[y][j][3] = own[3];
          }
        }
      };
      if constexpr (!CODES) {
#pragma unroll
        for (int j = 0; j < NJ / 2; ++j) {
          const int key = kk * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), ch = 2 * j + (lane >> 4);
          uint32_t b[4];
          ldmatrix4_trans(b, vt + key * S::ROW + ((ch ^ (key & 7)) << 4));
          product(2 * j, b[0], b[1]);
          product(2 * j + 1, b[2], b[3]);
        }
      } else {
        constexpr int WORDS = D / 32;  // words of a lane's part of a row: D / 8 coordinates
        uint32_t v[4][WORDS];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = kk * 16 + 2 * t4 + (e & 1) + (e >> 1) * 8;
          if constexpr (WORDS == 4) {
            const uint4 q = lds128(vt + key * S::ROW + ((g8 ^ (((key >> 1) & 3) << 1)) << 4));
            v[e][0] = q.x, v[e][1] = q.y, v[e][2] = q.z, v[e][3] = q.w;
          } else {
            const uint2 q = lds64(vt + key * S::ROW + (((g8 >> 1) ^ ((key >> 1) & 3)) << 4) + (g8 & 1) * 8);
            v[e][0] = q.x, v[e][1] = q.y;
          }
        }
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          uint32_t b0[4], b1[4];  // pairs of two rows, one coordinate each
          b0[0] = pair_of<FMT, 0>(v[0][w], v[1][w], times128), b0[1] = pair_of<FMT, 1>(v[0][w], v[1][w], times128);
          b0[2] = pair_of<FMT, 2>(v[0][w], v[1][w], times128), b0[3] = pair_of<FMT, 3>(v[0][w], v[1][w], times128);
          b1[0] = pair_of<FMT, 0>(v[2][w], v[3][w], times128), b1[1] = pair_of<FMT, 1>(v[2][w], v[3][w], times128);
          b1[2] = pair_of<FMT, 2>(v[2][w], v[3][w], times128), b1[3] = pair_of<FMT, 3>(v[2][w], v[3][w], times128);
#pragma unroll
          for (int e = 0; e < 4; ++e) product(4 * w + e, b0[e], b1[e]);
        }
      }
    }
  }

  // ---- the warps join
  cp_wait<0>();
  __syncthreads();  // the rings are free
  constexpr int LD = D + 4;
  float* s_o = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    const int row = NARROW ? g8 : (r / 2) * 16 + (r & 1) * 8 + g8;
    if (t4 == 0) s_ml[warp * R + row] = make_float2(m[r], l[r]);
    if (r0 + row >= rows) continue;
    float* to = s_o + (warp * R + row) * LD;
    float unit_of_o = 1.0f;
    if constexpr (CODES) unit_of_o = pow2(ref[r] - 14 + kCodeUnit<FMT>);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float v0 = NARROW ? o[0][j][0] + o[0][j][2] : o[r / 2][j][(r & 1) * 2];
      const float v1 = NARROW ? o[0][j][1] + o[0][j][3] : o[r / 2][j][(r & 1) * 2 + 1];
      if constexpr (CODES) {
        to[2 * t4 * NJ + j] = v0 * unit_of_o;
        to[(2 * t4 + 1) * NJ + j] = v1 * unit_of_o;
      } else {
        *reinterpret_cast<float2*>(to + j * 8 + 2 * t4) = make_float2(v0, v1);
      }
    }
  }
  __syncthreads();
  auto finish = [&](int row, int j, float mm, float ll, float4 x) {
    const int t = row / G, h = u.g * G + row - t * G;
    const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;  // (a sum of NaN stays one)
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(a.out.ptr)) + u.l * a.out.stride_l +
                         u.b * a.out.stride_b + h * a.out.stride_h + t * a.out.stride_n;
    *reinterpret_cast<uint2*>(out + j) = make_uint2(pack2<false>(x.x * inv, x.y * inv), pack2<false>(x.z * inv, x.w * inv));
    if (j == 0) {
      if (a.lse)
        a.lse[(((long long)u.l * c.batch + u.b) * a.Hq + h) * a.T + t] =
            ll == 0.0f ? -INFINITY : mm * 0.6931471805599453f + logf(ll);
      if (sc.row_ml) sc.row_ml[(long long)unit * rows + row] = make_float2(mm, inv);
    }
  };
  for (int w = tid; w < n_rows * (D / 4); w += kThreads) {
    const int r = w / (D / 4), j = (w - r * (D / 4)) * 4;
    float mm = -INFINITY, ll = 0.0f;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) mm = fmaxf(mm, s_ml[k * R + r].x);
    const float from = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float2 ml = s_ml[k * R + r];
      const float f = ex2(ml.x - from);
      const float4 y = *reinterpret_cast<const float4*>(s_o + (k * R + r) * LD + j);
      if (ml.y == 0.0f) continue;
      ll += ml.y * f;
      x.x += y.x * f;
      x.y += y.y * f;
      x.z += y.z * f;
      x.w += y.w * f;
    }
    if (n_pieces == 1) {
      finish(r0 + r, j, mm, ll, x);
    } else {
      const long long slot = ((long long)group * cut.pieces + part) * R + r;
      *reinterpret_cast<float4*>(sc.part + slot * D + j) = x;
      if (j == 0) sc.part_ml[slot] = make_float2(mm, ll);
    }
  }
  if (n_pieces == 1) return;

  // ---- the pieces join: the block that comes last reads them in their order
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    const int came = atomicAdd(&sc.ticket[group], 1);
    *s_last = came == n_pieces - 1;
    if (*s_last) sc.ticket[group] = 0;
  }
  __syncthreads();
  if (!*s_last) return;
  __threadfence();
  const long long at0 = (long long)group * cut.pieces * R;
  float2* s_w = reinterpret_cast<float2*>(smem);  // [piece][row], at most kAttendJoined of them: maximum and sum, then what a piece weighs
  // Lanes that share a row, all rows at once: a warp per row takes four or eight rows one after another (8 units' 32 query rows
  // over 129 to 4096 rows 23 to 38 us, so 19 to 33, and 18 to 27 with the loads below). With 8 rows a warp has two at most, and the plainer code leaves the loop faster
  // (64 ragged conversations in e4m3 264 us, 281 with the other).
  if constexpr (R > 8) {
#pragma unroll 4
    for (int w = tid; w < n_pieces * R; w += kThreads) s_w[w] = __ldcg(&sc.part_ml[at0 + w]);
    __syncthreads();
    constexpr int PER_ROW = kThreads / R;  // lanes that share a row
    const int r = tid / PER_ROW, sub = tid % PER_ROW;
    float mm = -INFINITY, ll = 0.0f;
    for (int k = sub; k < n_pieces; k += PER_ROW) mm = fmaxf(mm, s_w[k * R + r].x);
#pragma unroll
    for (int w = PER_ROW / 2; w > 0; w >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, w));
    const float from = mm == -INFINITY ? 0.0f : mm;
    for (int k = sub; k < n_pieces; k += PER_ROW) {
      const float2 p = s_w[k * R + r];
      const float f = p.y == 0.0f ? 0.0f : ex2(p.x - from);
      s_w[k * R + r].x = f;
      if (p.y != 0.0f) ll += p.y * f;
    }
#pragma unroll
    for (int w = PER_ROW / 2; w > 0; w >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, w);
    if (sub == 0) s_ml[r] = make_float2(mm, ll);
  } else {
    for (int r = warp; r < n_rows; r += kWarps) {   // a warp per row
      const float2* ml = sc.part_ml + at0 + r;
      float mm = -INFINITY, ll = 0.0f;
      for (int k = lane; k < n_pieces; k += 32) {
        const float2 p = __ldcg(&ml[(long long)k * R]);
        s_w[k * R + r] = p;
        mm = fmaxf(mm, p.x);
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, w));
      const float from = mm == -INFINITY ? 0.0f : mm;
      for (int k = lane; k < n_pieces; k += 32) {
        const float2 p = s_w[k * R + r];
        const float f = p.y == 0.0f ? 0.0f : ex2(p.x - from);
        s_w[k * R + r].x = f;
        if (p.y != 0.0f) ll += p.y * f;
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, w);
      if (lane == 0) s_ml[r] = make_float2(mm, ll);
    }
  }
  __syncthreads();
  if constexpr (R > 8) {
    // A thread has four coordinates of every LANES-th row, and all their loads on their way: none under a condition (rows and pieces
    // that are not there repeat the last one, with no weight), nothing stored before the last.
    constexpr int LANES = kThreads / (D / 4), ITEMS = R / LANES, AHEAD = 16 / ITEMS < 4 ? 4 : 16 / ITEMS;
    const int r_first = tid / (D / 4), j = tid % (D / 4) * 4;
    float4 x[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float* part_of = sc.part + at0 * D + j;
    for (int k0 = 0; k0 < n_pieces; k0 += AHEAD) {
      float4 y[AHEAD][ITEMS];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
          y[k][i] = __ldcg(reinterpret_cast<const float4*>(
              part_of + ((long long)min(k0 + k, n_pieces - 1) * R + min(r_first + i * LANES, n_rows - 1)) * D));
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          const float f = k0 + k < n_pieces ? s_w[(k0 + k) * R + r_first + i * LANES].x : 0.0f;
          x[i].x += y[k][i].x * f;
          x[i].y += y[k][i].y * f;
          x[i].z += y[k][i].z * f;
          x[i].w += y[k][i].w * f;
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int r = r_first + i * LANES;
      if (r < n_rows) finish(r0 + r, j, s_ml[r].x, s_ml[r].y, x[i]);
    }
  } else {
    for (int w = tid; w < n_rows * (D / 4); w += kThreads) {
      const int r = w / (D / 4), j = (w - r * (D / 4)) * 4;
      const float* part_of = sc.part + (at0 + r) * D + j;
      float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
      for (int k = 0; k < n_pieces; ++k) {
        const float4 y = __ldcg(reinterpret_cast<const float4*>(part_of + (long long)k * R * D));
        const float f = s_w[k * R + r].x;
        x.x += y.x * f;
        x.y += y.y * f;
        x.z += y.z * f;
        x.w += y.w * f;
      }
      finish(r0 + r, j, s_ml[r].x, s_ml[r].y, x);
    }
  }
}

// Attention mass per cache row, from the scores and the rows' maxima and sums; a thread has four cache rows. grid.x = units,
// grid.y = stretches of 1024 rows, or as many as a grid can have. (Formed at the end of the attention's own blocks, where a unit is one block, it took longer:
// 32 x 16 x 8 units of 257 rows 135 us a step where this takes 128, of 1025 rows 423 and 388.)
__global__ void __launch_bounds__(256) ta_attend_mass_kernel(ta_attend_args a, Scratch sc) {
  ta_wait_for_prior_grid();
  ta_launch_dependents();
  const int unit = blockIdx.x, G = a.Hq / a.cache.Hkv, rows = G * a.T;
  const Unit u = unit_of(a, unit);
  const int n = rows_of_unit(a, u, ta_cache_len(a.cache, u.l, u.b, u.g), false, nullptr);
  const float2* row_ml = sc.row_ml + (long long)unit * rows;
  const float* score = sc.score + (long long)unit * rows * sc.score_stride;
  for (long long j = 4LL * (blockIdx.y * 256 + threadIdx.x); j < a.mass_stride; j += 1024LL * gridDim.y) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (j < n) {
#pragma unroll 4
      for (int r = 0; r < rows; ++r) {
        const float2 ml = row_ml[r];
        const float4 x = *reinterpret_cast<const float4*>(score + r * sc.score_stride + j);
        const int seen = n - (a.causal ? a.T - 1 - r / G : 0);
        if (ml.y == 0.0f) continue;  // a token that sees nothing
        if (j < seen) sum[0] += ex2(x.x - ml.x) * ml.y;
        if (j + 1 < seen) sum[1] += ex2(x.y - ml.x) * ml.y;
        if (j + 2 < seen) sum[2] += ex2(x.z - ml.x) * ml.y;
        if (j + 3 < seen) sum[3] += ex2(x.w - ml.x) * ml.y;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < a.mass_stride) a.mass[unit * a.mass_stride + j + e] = sum[e];
  }
}

template <int D, int FMT, int MB, int W>
cudaError_t launch(const ta_attend_args& a, const Scratch& sc, const ta_attend_plan& p, cudaLaunchConfig_t& cfg, ta_dev_status* status) {
  constexpr int smem = smem_bytes<D, FMT, MB, W>();
  static_assert(W < 4 || Shape<D, FMT, W>::RING >= kAttendJoined * 8, "the join's weights take the ring's place");
  static bool set[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!set[dev & 63]) {
    e = cudaFuncSetAttribute(ta_attend_kernel<D, FMT, MB, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    set[dev & 63] = true;
  }
  cfg.blockDim = dim3(W * 32, 1, 1);
  cfg.dynamicSmemBytes = smem;
  return cudaLaunchKernelEx(&cfg, ta_attend_kernel<D, FMT, MB, W>, a, sc,
                            Cut{p.pieces, p.piece, p.row_blocks, p.target, a.n_layers * a.cache.Hkv * p.row_blocks}, 128u, status);
}
template <int D, int FMT>
cudaError_t launch(const ta_attend_args& a, const Scratch& sc, const ta_attend_plan& p, cudaLaunchConfig_t& cfg, ta_dev_status* status) {
  if (p.mb == 0) return p.warps == 2 ? launch<D, FMT, 0, 2>(a, sc, p, cfg, status) : launch<D, FMT, 0, 4>(a, sc, p, cfg, status);
  if (p.mb == 1) return launch<D, FMT, 1, 4>(a, sc, p, cfg, status);
  return launch<D, FMT, 2, 4>(a, sc, p, cfg, status);
}
template <int D>
cudaError_t launch(const ta_attend_args& a, const Scratch& sc, const ta_attend_plan& p, cudaLaunchConfig_t& cfg, ta_dev_status* status) {
  if (a.cache.format == TA_CACHE_BF16) return launch<D, TA_CACHE_BF16>(a, sc, p, cfg, status);
  if (a.cache.format == TA_CACHE_E4M3) return launch<D, TA_CACHE_E4M3>(a, sc, p, cfg, status);
  return launch<D, TA_CACHE_INT8>(a, sc, p, cfg, status);
}

// The call's scratch; null: its size alone
size_t carve(long long units, int rows, int d, int max_len, bool codes, int ragged_batch, bool with_mass, uint8_t* base,
             Scratch* sc) {
  const ta_attend_plan p = ta_attend_plan_of(units, rows, max_len, codes, ragged_batch);
  const ta_attend_sizes z = ta_attend_sizes_of(units, rows, d, max_len, ta_attend_slots(p, units), with_mass);
  if (sc) {
    sc->part = reinterpret_cast<float*>(base);
    sc->part_ml = reinterpret_cast<float2*>(base + z.part);
    if (with_mass) {
      sc->score_stride = ta_attend_score_stride(max_len);
      sc->score = reinterpret_cast<float*>(base + z.part + z.part_ml);
      sc->row_ml = reinterpret_cast<float2*>(base + z.part + z.part_ml + z.score);
    }
  }
  return z.all();
}

}  // namespace

size_t ta_attend_scratch(int units, int rows, int d, int max_len, bool codes, int ragged_batch, bool with_mass) {
  return carve(units, rows, d, max_len, codes, ragged_batch, with_mass, nullptr, nullptr);
}

cudaError_t ta_launch_attend(const ta_attend_args& a, int* tickets, ta_dev_status* status, cudaStream_t stream) {
  const int units = a.n_layers * a.cache.batch * a.cache.Hkv, rows = a.Hq / a.cache.Hkv * a.T;
  const bool codes = a.cache.format != TA_CACHE_BF16;
  const int ragged_batch = a.cache.lens && !a.cache.lens_per_unit ? a.cache.batch : 0;
  const ta_attend_plan p = ta_attend_plan_of(units, rows, a.max_len, codes, ragged_batch);
  Scratch sc = {};
  carve(units, rows, a.d, a.max_len, codes, ragged_batch, a.mass != nullptr, a.scratch, &sc);
  sc.ticket = tickets;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((long long)units * p.row_blocks * p.pieces), 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  ta_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = a.d == 64 ? launch<64>(a, sc, p, cfg, status) : launch<128>(a, sc, p, cfg, status);
  if (e != cudaSuccess || !a.mass || a.mass_stride == 0) return e;
  const long long stretches = (a.mass_stride + 1023) / 1024;
  cfg.gridDim = dim3((unsigned)units, (unsigned)(stretches < 65535 ? stretches : 65535), 1);
  cfg.blockDim = dim3(256, 1, 1);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, ta_attend_mass_kernel, a, sc);
}
