// What the kernels of the cache, the rotation and the attention share: where a row lies, how it is held, and the angle of a
// position.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "ta_attend_rule.h"
#include "ta_internal.cuh"

struct ta_cache_dev {  // a ta_cache for kernels: strides of rows in bytes, of scales in floats
  uint8_t *k, *v;
  float *ks, *vs;
  long long sl, sp, sh, sr;
  long long ssl, ssp, ssh, ssr;
  const int32_t* table;
  const int32_t* lens;
  int batch, Hkv, format;
  int page, page_shift;  // page_shift >= 0: page is that power of two
  int n_pages, wide;     // wide: pages of a sequence
  int lens_per_unit, len_uniform;
};

struct ta_rotary_dev {
  const uint64_t* phase;  // null: nothing is rotated
  const int32_t* positions;
  int d_rot, interleaved, inverse;
  float magnitude;
};

struct ta_rotate_args {
  ta_seq_desc seq;
  int n_layers, Hq, Hkv, d;
  ta_rotary_dev rot;
  ta_bf16_view q, q_out, k, k_out;
};
cudaError_t ta_launch_rotate(const ta_rotate_args& a, cudaStream_t stream);

struct ta_cache_move_args {  // append: k and v are read; read: they are written
  ta_cache_dev cache;
  ta_seq_desc seq;
  int n_layers, d;
  ta_rotary_dev rot;
  ta_bf16_view k, v;
  const int32_t* rows;
};
cudaError_t ta_launch_cache_append(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream);
cudaError_t ta_launch_cache_read(const ta_cache_move_args& a, ta_dev_status* status, cudaStream_t stream);

struct ta_attend_args {
  ta_cache_dev cache;
  int n_layers, Hq, d, T, new_rows, max_len, causal;
  float scale;
  ta_rotary_dev rot;
  ta_bf16_view q, out;
  float* lse;
  float* mass;
  long long mass_stride;
  uint8_t* scratch;
};
// What a call takes. ragged_batch: sequences, where every one has a length of its own, else 0
size_t ta_attend_scratch(int units, int rows, int d, int max_len, bool codes, int ragged_batch, bool with_mass);
// tickets: kAttendTickets words, zero before and after
cudaError_t ta_launch_attend(const ta_attend_args& a, int* tickets, ta_dev_status* status, cudaStream_t stream);

#ifdef __CUDACC__
// Cosine and sine of a position's angle, with the factor on both: the product modulo 2^64 is the angle in turns, exactly, and
// its upper half as a signed number times 2^-31 the angle in half turns.
__device__ __forceinline__ float2 ta_cos_sin(const ta_rotary_dev& r, uint64_t phase, int position) {
  const uint64_t turns = phase * (uint64_t)(long long)position;
  float s, c;
  sincospif((float)(int)(turns >> 32) * 0x1p-31f, &s, &c);
  return make_float2(c * r.magnitude, (r.inverse ? -s : s) * r.magnitude);
}

__device__ __forceinline__ void ta_report_bounds(ta_dev_status* status, int where, int detail0, int detail1) {
  if (atomicCAS(&status->code, 0, (int)TA_ERR_DEVICE_BOUNDS) == 0) {
    status->where = where;
    status->detail0 = detail0;
    status->detail1 = detail1;
  }
}

struct ta_row_at {
  long long row, scale;  // byte offset of the row in k and v, offset of its scale; row -1: there is none
};
// Where row r (>= 0) of sequence b lies, layer and head left out.
__device__ __forceinline__ ta_row_at ta_cache_row(const ta_cache_dev& c, int b, int r) {
  const int j = c.page_shift >= 0 ? r >> c.page_shift : (int)((unsigned)r / (unsigned)c.page);
  const int in_page = r - j * c.page;
  if (j >= c.wide) return {-1, 0};
  const int id = c.table ? c.table[(long long)b * c.wide + j] : b * c.wide + j;
  if (id < 0 || id >= c.n_pages) return {-1, 0};
  return {id * c.sp + in_page * c.sr, id * c.ssp + in_page * c.ssr};
}
__device__ __forceinline__ int ta_cache_len(const ta_cache_dev& c, int l, int b, int g) {
  if (!c.lens) return c.len_uniform;
  return c.lens[c.lens_per_unit ? ((long long)l * c.batch + b) * c.Hkv + g : b];
}
#endif
