// Attention of packed rows, what its kernels over 4-bit codes (attn_kvq.h) and over bf16 / fp32 pools (attn_rows.h) share: the parts that a call is cut
// into over workgroups, counted on the device from the lengths as they are, and the sum of a row's parts in their order.
#pragma once
#include "common.h"
#include "mfma_common.h"
#include "rows.h"
#include "rowsum.h"

namespace oomb {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float MOST = 512.0f;           // of a lane's weights of a unit, before the reference moves
constexpr int NO_TOKEN = 0x7fffff00;     // position of the tokens of a tile that does not exist
constexpr int PAD = 4;                   // floats between the rows of a merge buffer: conflict-free for 16-byte accesses
constexpr int COMBINE_THREADS = 256;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// what is left of a and b after their bf16 roundings, packed as `w`
__device__ __forceinline__ void less(float& a, float& b, uint32_t w) {
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
}

// A page of one head: buffer loads take its base, a lane's offset and the tile's from three registers, so that addresses cost next to no
// instruction; what lies past the page reads as zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_buffer(const unsigned char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, bytes, 0x00027000);
}

struct AttnArgs {
  int row_blocks;              // per (sequence, KV head)
  int split;                   // parts over workgroups (else one part per (sequence, KV head))
  int target, min_units;       // parts to aim at; units of a part at least
  int2* parts;                 // [sequence * Hkv + KV head]: first part, number of parts
  float* part;                 // [part][row block][row of the block][D] sums
  float* part_ml;              // [part][row block][row][2]: reference, sum
};

// Queries that are needed in every step are waited for here, once.
template <int RT, int QT, int NC> __device__ __forceinline__ void landed(uint4 (&q)[RT][QT][NC]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(q[rt][t][c].x), "+v"(q[rt][t][c].y), "+v"(q[rt][t][c].z), "+v"(q[rt][t][c].w));
}

// ---- the parts of a call ------------------------------------------------------------------------------------------------
// A bound of the units that the rows of (sequence, KV head) e see, -1 if it has no rows.  (No branch on a lane's values: a lane asks for several.)
__device__ __forceinline__ int units_of(const RowsParams& p, int e) {
  const Seq s = seq_of(p, e / p.Hkv);
  const int64_t tokens = p.sel ? (int64_t)min(max(p.sel_count[e], 0), p.sel_stride) * p.P : s.len;
  const int units = (int)((min(tokens, (int64_t)p.max_len) + 31) >> 5);
  return s.n == 0 ? -1 : units;
}
struct Part { int e, first, index, count; };   // (sequence, KV head), its first part, this one of it, its number of parts
// Part x of the call, by every lane of a wave; e < 0: there are fewer.
__device__ __forceinline__ Part part_at(const RowsParams& p, const AttnArgs& a, int x, int lane) {
  const int n = p.n_seqs * p.Hkv;
  if (!a.split) return {x, x, 0, 1};
  constexpr int HELD = 4;   // of a lane, loaded together (256 in all; more are asked for again)
  int held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = 64 * i < n ? units_of(p, min(64 * i + lane, n - 1)) : -1;
  float total = 0.0f;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (64 * i + lane >= n) held[i] = -1;
    total += (float)max(held[i], 0);
  }
  for (int e = 64 * HELD + lane; e < n; e += 64) total += (float)max(units_of(p, e), 0);
#pragma unroll
  for (int w = 1; w < 64; w *= 2) total += __shfl_xor(total, w, 64);
  const int per = max(a.min_units, (int)(total / (float)a.target) + 1);   // (the same sum in every wave)
  int before = 0;
  for (int e0 = 0; e0 < n; e0 += 64) {
    int units = -1;
    if (e0 >= 64 * HELD) {
      units = e0 + lane < n ? units_of(p, e0 + lane) : -1;
    } else {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (e0 == 64 * i) units = held[i];
    }
    const int parts = units < 0 ? 0 : max(1, (int)((uint32_t)(units + per - 1) / (uint32_t)per));
    int upto = parts;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
      const int y = __shfl_up(upto, w, 64);
      if (lane >= w) upto += y;
    }
    const uint64_t past = __ballot(before + upto > x);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int count = __builtin_amdgcn_readlane(parts, l), first = before + __builtin_amdgcn_readlane(upto, l) - count;
      return {e0 + l, first, x - first, count};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, 0, 0};
}

// The parts of a row, in order: a workgroup per row of a row block and slice of DW dims, its threads in groups of DW / 4 that take every
// (256 / (DW / 4))-th part each.  A compute unit takes in about 10 B/ns of lines that others wrote, so a few rows of many parts go in slices of a
// line (7 x 4 rows of 127 parts: 10.3 us whole).
template <typename T, int D, int DW>
__global__ __launch_bounds__(COMBINE_THREADS) void rows_combine_kernel(RowsParams p, AttnArgs a, int block_rows, int rows) {   // rows: of a block that there can be at most
  constexpr int LANES = DW / 4, GROUPS = COMBINE_THREADS / LANES;
  __shared__ __align__(16) float lds[GROUPS][DW + PAD];
  __shared__ float lds_ml[GROUPS][2];
  int x = blockIdx.x;
  const int slice = x % (D / DW);
  x /= D / DW;
  const int r = x % rows;
  x /= rows;
  const int block = x % a.row_blocks, e = x / a.row_blocks;
  const int b = e / p.Hkv, g = e - b * p.Hkv;
  const Seq s = seq_of(p, b);
  const int row = block * block_rows + r;
  if (row >= s.n * p.G) return;
  const int2 parts = a.parts[e];
  if (parts.y <= 1) return;
  const int grp = threadIdx.x / LANES, d = (threadIdx.x - grp * LANES) * 4;
  float ref = -INFINITY, sum = 0.0f, y[4] = {0.f, 0.f, 0.f, 0.f};
  constexpr int AT_ONCE = 4;   // (loads in flight: a chain of single ones takes a microsecond a part)
  for (int k0 = grp; k0 < parts.y; k0 += AT_ONCE * GROUPS) {
    float2 ml[AT_ONCE];
    float4 v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int64_t at = ((int64_t)(parts.x + min(k0 + i * GROUPS, parts.y - 1)) * a.row_blocks + block) * block_rows + r;
      ml[i] = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
      v[i] = *reinterpret_cast<const float4*>(a.part + at * D + slice * DW + d);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (k0 + i * GROUPS >= parts.y) break;
      const float to = fmaxf(ref, ml[i].x);
      const float f0 = ref == to ? 1.0f : __builtin_amdgcn_exp2f(ref - to), f1 = ml[i].x == to ? 1.0f : __builtin_amdgcn_exp2f(ml[i].x - to);
      ref = to;
      sum = sum * f0 + ml[i].y * f1;
      y[0] = y[0] * f0 + v[i].x * f1; y[1] = y[1] * f0 + v[i].y * f1; y[2] = y[2] * f0 + v[i].z * f1; y[3] = y[3] * f0 + v[i].w * f1;
    }
  }
  *reinterpret_cast<float4*>(&lds[grp][d]) = make_float4(y[0], y[1], y[2], y[3]);
  if (d == 0) { lds_ml[grp][0] = ref; lds_ml[grp][1] = sum; }
  __syncthreads();
  if (grp) return;
  float top = -INFINITY, total = 0.0f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, lds_ml[k][0]);
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) {
    const float f = lds_ml[k][0] == top ? 1.0f : __builtin_amdgcn_exp2f(lds_ml[k][0] - top);
    const float4 v = *reinterpret_cast<const float4*>(&lds[k][d]);
    total += lds_ml[k][1] * f;
    o[0] += v.x * f; o[1] += v.y * f; o[2] += v.z * f; o[3] += v.w * f;
  }
  const int i = row / p.G, h = g * p.G + (row - i * p.G);
  const float f = total == 0.0f ? 0.0f : 1.0f / total;
  T* dst = (T*)p.q_out.data + (int64_t)(s.row + i) * p.q_out.tok_stride + (int64_t)h * p.q_out.head_stride + slice * DW + d;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2_bf16(o[0] * f, o[1] * f), pack2_bf16(o[2] * f, o[3] * f));
  else *reinterpret_cast<float4*>(dst) = make_float4(o[0] * f, o[1] * f, o[2] * f, o[3] * f);
  if (d == 0 && slice == 0) p.lse[(int64_t)h * p.n_rows + s.row + i] = total == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * LN2;
}

}  // namespace
}  // namespace oomb
