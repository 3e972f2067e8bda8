// Steps of generation between two passes of attention: pages of a cache forked, copied and compacted on the device (page_fork.hip), the selection of beam
// search (beam_topk.hip).  What api_gen.hip checks and passes on; layouts in include/oomb.h.
#pragma once
#include "common.h"

namespace oomb {

struct ForkParams {
  int32_t n_seqs, n_out, log2_p, cols, out_cols;
  int64_t stride, out_stride;
  int32_t num_phys;
  const int32_t* tables;
  const int32_t* lens;
  const int32_t* parents;
  const int32_t* grow;      // may be NULL
  const int32_t* refs;
  int32_t* tables_out;
  int32_t* lens_out;
  int32_t* refs_out;
  int32_t* copies;          // [n_out][3]
  int32_t* status;          // [2]
};
constexpr int FORK_MOST_SEQS = 4096;   // before and after: counters of both lie in the LDS of one workgroup
size_t fork_workspace_bytes(int32_t n_seqs, int32_t n_out, int64_t num_phys);
int64_t fork_blocks(const ForkParams& p);
hipError_t launch_page_fork(const ForkParams& p, void* ws, hipStream_t st);

struct CompactParams {
  int32_t n_seqs, page, log2_p, cols;
  int64_t stride, out_stride;
  int32_t num_phys;
  const int32_t* tables;
  const int32_t* lens;
  const int32_t* refs;
  int32_t* tables_out;
  int32_t* refs_out;
  int32_t* moves;           // [>= num_phys / 2][3]
  int32_t* map;             // [num_phys]
  int32_t* status;          // [2]
};
size_t compact_workspace_bytes(int64_t num_phys);
int64_t compact_blocks(const CompactParams& p);
hipError_t launch_page_compact(const CompactParams& p, void* ws, hipStream_t st);

struct CopyParams {
  int32_t n_heads, page, row_bytes, n_copies;
  int32_t num_phys;
  int64_t page_stride, head_stride, tok_stride;   // bytes; tok_stride 0: a page of a head is one piece of row_bytes
  const int32_t* copies;    // [n_copies][3]
  const int32_t* count;     // may be NULL
};
constexpr int COPY_POOLS = 64;         // of a launch
struct CopyPools { unsigned char* at[COPY_POOLS]; };
hipError_t launch_page_copy(const CopyParams& p, void* const* pools, int32_t n_pools, hipStream_t st);

struct BeamParams {
  int32_t n_groups, n_beams, vocab, n_out, pad_token;
  int64_t row_stride;       // elements
  const void* logits;       // [n_groups * n_beams][vocab]
  const float* scores;      // [n_groups][n_beams]
  const int32_t* done;      // may be NULL
  int32_t* parents;         // [n_groups][n_out]
  int32_t* tokens;
  float* best;
};
constexpr int BEAM_MOST_OUT = 64, BEAM_MOST_BEAMS = 64;
size_t beam_workspace_bytes(const BeamParams& p, bool is_bf16);
int64_t beam_blocks(const BeamParams& p, bool is_bf16);
hipError_t launch_beam_topk(const BeamParams& p, bool is_bf16, void* ws, hipStream_t st);

}  // namespace oomb
