// Packed rows of several sequences: what the kernels of rope_append.hip, attn_kvq.h and attn_rows.h share (layouts: include/oomb.h).
#pragma once
#include "common.h"

namespace oomb {

struct RowsParams {
  int32_t Hq, Hkv, G, D, P, n_seqs, n_rows, max_rows, max_len, log2_p;
  float sm_scale;
  int64_t table_stride, num_phys, pool_page_stride, pool_head_stride, pool_tok_stride;
  const int32_t* tables;
  const int32_t* lens;
  const int32_t* starts;
  // rotation
  const float* cos;
  const float* sin;
  int32_t rot_dim, interleaved;
  // rows (read or written as the entry point says)
  oomb_rows q, q_out, k, v;
  void* k_pool;
  void* v_pool;
  float* kbar;
  // attention
  const int32_t* sel;
  const int32_t* sel_count;
  int32_t sel_stride;
  float* lse;
};

// One sequence: its first row, its rows and the position of the first of them, all within the host's bounds.
struct Seq {
  int32_t row, n, pos, len;   // n: rows to process; pos < 0: that many rows do not exist
};
__device__ __forceinline__ Seq seq_of(const RowsParams& p, int b) {
  int32_t s0, s1, len = p.max_len;
  if (p.starts) {
    s0 = p.starts[b];
    s1 = p.starts[b + 1];
  } else {
    const int32_t each = p.n_rows / p.n_seqs;
    s0 = b * each;
    s1 = s0 + each;
  }
  if (p.lens) len = min(max(p.lens[b], 0), p.max_len);
  s0 = min(max(s0, 0), p.n_rows);
  s1 = min(max(s1, s0), p.n_rows);
  return {s0, min(s1 - s0, p.max_rows), len - (s1 - s0), len};
}
// physical page of logical page l (below ceil(max_len / P)) of sequence b, -1 if there is none
__device__ __forceinline__ int32_t page_of(const RowsParams& p, int b, int32_t l) {
  const int32_t x = p.tables[(int64_t)b * p.table_stride + l];
  return x >= 0 && x < p.num_phys ? x : -1;
}
// pages that n rows touch at most
__host__ __device__ __forceinline__ int32_t pages_touched(int32_t n, int32_t P) { return (int32_t)(((int64_t)n + P - 2) / P) + 1; }

// ---- tiles of a 4-bit pool -----------------------------------------------------------------
constexpr int kvq_row_bytes(int D) { return D / 2; }
__host__ __device__ constexpr int64_t kvq_tile_bytes(int P, int D) { return (int64_t)P * (D / 2 + D / 32); }
// the float that a scale byte stands for; in the conversions of gfx950 an exponent of 255 makes every code NaN
__device__ __forceinline__ float kvq_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// Scale byte of a block whose largest magnitude has these bits: mantissas up to 1.75 = 7 / 4 take the exponent less two.
__device__ __forceinline__ uint32_t kvq_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  return min(max((int)((top + 0x1fffffu) >> 23) - 2, 2), 252);
}

hipError_t launch_append_rope(const RowsParams& p, bool is_bf16, bool kvq, hipStream_t st);
hipError_t launch_append_rope_bwd(const RowsParams& p, bool is_bf16, bool grad_bf16, hipStream_t st);
hipError_t launch_kvq_read(const RowsParams& p, bool is_bf16, hipStream_t st);
size_t kvq_attn_workspace_bytes(const RowsParams& p, bool is_bf16, int32_t sel_stride);
hipError_t launch_attn_kvq(const RowsParams& p, bool is_bf16, void* ws, hipStream_t st);
hipError_t launch_attn_kvq_bf16_128(const RowsParams& p, void* ws, hipStream_t st);
hipError_t launch_attn_kvq_bf16_64(const RowsParams& p, void* ws, hipStream_t st);
hipError_t launch_attn_kvq_f32_128(const RowsParams& p, void* ws, hipStream_t st);
hipError_t launch_attn_kvq_f32_64(const RowsParams& p, void* ws, hipStream_t st);
size_t rows_attn_workspace_bytes(const RowsParams& p, bool is_bf16, int32_t sel_stride);
hipError_t launch_attn_rows(const RowsParams& p, bool is_bf16, void* ws, hipStream_t st);
hipError_t launch_attn_rows_bf16_128(const RowsParams& p, void* ws, hipStream_t st);
hipError_t launch_attn_rows_bf16_64(const RowsParams& p, void* ws, hipStream_t st);
hipError_t launch_attn_rows_f32_128(const RowsParams& p, void* ws, hipStream_t st);
hipError_t launch_attn_rows_f32_64(const RowsParams& p, void* ws, hipStream_t st);
// workgroups that a launch would take (the grid may hold 2^24 - 1 of 256 threads)
int64_t append_rope_blocks(const RowsParams& p, bool kvq);
int64_t kvq_read_blocks(const RowsParams& p);
int64_t kvq_attn_blocks(const RowsParams& p, bool is_bf16, int32_t sel_stride);
int64_t rows_attn_blocks(const RowsParams& p, bool is_bf16, int32_t sel_stride);

}  // namespace oomb
