// Attention of packed rows over pools of bf16 / fp32 rows (layouts: include/oomb.h, rows.h).
//
// A wave holds RT tiles of 16 query rows and walks steps of 32 tokens (fp32: 16), tiles of 16 that lie inside a page; the G query heads of
// a KV head share its cache: query row r of a sequence and KV head is token r / G, head r % G.  Operands come straight from memory, no LDS and no
// exchange of lanes.  With lane = 16 kg + m:
//   S^T = K Q^T: lane (m, kg) reads 16 bytes of token m at 64 c + 16 kg for every c: with v_mfma_f32_16x16x32_bf16 (lane l holds
//       A[l % 16][8 (l / 16) + 0..7], C[4 (l / 16) + r][l % 16] in register r) the operand of step c; with v_mfma_f32_16x16x4_f32 (A[l % 16][l / 16]) its
//       four floats are those of four steps.  The queries lie alike.
//   O^T += V^T P^T: a lane's accumulators of S^T are tokens 4 kg + 0..3 of a tile for query m, in this order the B operand.  Lane (m, kg) reads
//       dims D/16 m .. of those four tokens; fp32: float j of token 4 kg + r is the A operand of step r that gives dims D/16 m + j; bf16: pairs of tokens are put
//       together with byte permutes, and an operand takes both tiles.
// bf16 rows: weights in two bf16 terms (16 bits), so that the output's own rounding is the larger one.  fp32 rows: fp32 products.
//
// Softmax in one pass: weights are taken against a reference of the row that moves only when the weights of a lane in a step exceed 2^9 together; so no
// maximum is formed on the way, and sums stay far inside a float.
//
// The waves of a workgroup share a row block and split its tokens; long caches are cut into parts of equal work over workgroups, counted on the
// device from the lengths as they are, and attn_combine adds a row's parts in their order.
//
// What bounds it.  Few rows: the reading of the cache (28 heads over 4 of 128 dims, bf16, 1M tokens: 2.1 GB in 323 us, 6.6 TB/s, of which the join takes 6; fp32 5.5),
// where it is short two launches and a chain of loads that wait for each other (lengths, page, rows; 1000 tokens 11 us).  So a wave keeps 32 KB in
// flight, and the loop carries no LDS, no barrier and no exchange but the test of the weights.  Many rows read the cache again per block of rows: then
// attn_tiles_kernel, below, shares a reading among 128 rows (three prompts of up to 1021 rows: 945 us here, 342 to 350 there); fp32 stays here, where the
// fp32 matrix instructions bound it (1024 rows over 16K tokens, 28 / 4 heads of 128: 2219 us, 105 TFLOP/s; the library's fp32 product 136).
#pragma once
#include <type_traits>

#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "rows.h"
#include "wave.h"

namespace oomb {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float MOST = 512.0f;           // of a lane's weights of a step, before the reference moves
constexpr int NO_TOKEN = 0x7fffff00;     // position of the tokens of a tile that does not exist
constexpr int PAD = 4;                   // floats between the rows of a merge buffer: conflict-free for 16-byte accesses
constexpr int COMBINE_THREADS = 256;
constexpr int WGS = 512;                 // workgroups that a call is cut into
constexpr int WAVES = 4;                 // that split the tokens of a block (100 sequences of 500 tokens: 23 us; eight, one workgroup a compute unit, 34; two the same, fp32 48 for 39)

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma4(uint32_t a, uint32_t b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// what is left of a and b after their bf16 roundings, packed as `w`
__device__ __forceinline__ void less(float& a, float& b, uint32_t w) {
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
}
// whether a half (of a word of two bf16) or a float is an infinity or a NaN
__device__ __forceinline__ bool wild16(uint32_t w, int half) { return ((half ? w >> 16 : w) & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool wild32(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }
// A page of one head: buffer loads take its base, a lane's offset and the tile's from three registers, so that addresses cost next to no
// instruction.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_buffer(const unsigned char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, bytes, 0x00027000);
}

// ---- how a call is cut --------------------------------------------------------------------------------------------------
// (sequence, KV head) e has blocks of its rows, and every block is cut into the same number of parts, so that parts are of about equal work in the
// whole call: counted on the device from the rows and lengths as they are.
struct AttnArgs {
  int block_rows, step;        // rows of a block; tokens that the work is counted in
  int split;                   // whether blocks may be cut
  int even;                    // into equal shares of the longest
  int target, min_steps;       // workgroups to aim at; steps of a part at least
  int full;                    // whether the blocks fill the chip as they are: about equal ones are not cut
  int planned;                 // whether attn_plan counts, for the whole call; else every workgroup does
  int2* parts;                 // [sequence * Hkv + KV head]: its first workgroup, parts of each of its blocks; planned: one more, the workgroups of all
  float* part;                 // [workgroup][row of the block][D] sums
  float* part_ml;              // [workgroup][row of the block][2]: reference, sum
  int blocks;                  // workgroups of the launch
};
struct Load { int blocks, steps; Seq s; };   // of (sequence, KV head) e; steps: a bound of what its rows see
__device__ __forceinline__ Load load_of(const RowsParams& p, const AttnArgs& a, int e) {   // (no branch on a lane's values: a lane asks for several)
  const Seq s = seq_of(p, e / p.Hkv);
  const int64_t tokens = p.sel ? (int64_t)min(max(p.sel_count[e], 0), p.sel_stride) * p.P : s.len;
  const int steps = (int)((min(tokens, (int64_t)p.max_len) + a.step - 1) / a.step);
  return {(int)(((int64_t)s.n * p.G + a.block_rows - 1) / a.block_rows), max(steps, 1), s};
}
struct Item { int e, block, first, index, count; Seq s; };   // e, block of its rows, the block's first workgroup, this one of it, its number of parts
// Steps of a part.  Tiles: an equal share of the longest, as many as fit one round of workgroups (224 blocks of 250 steps in
// 1, 2, 3, 4 parts: 427, 362, 378, 365 us; 112 of 512: 823, 437, 434, 365); else by the work alone, so that short parts even out.
__device__ __forceinline__ int steps_of_part(const AttnArgs& a, float total, int most) {
  if (!a.split) return 0x7fffffff;
  const int shares = max(1, (int)((float)a.target * (float)most / max(total, 1.0f) + 1e-3f));
  const int per = max(a.min_steps, a.even ? (most + shares - 1) / shares : (int)(total / (float)a.target) + 1);
  return a.full && most <= 2 * per ? max(most, per) : per;
}
__device__ __forceinline__ int parts_of(const AttnArgs& a, const Load& l, int per) { return a.split ? (int)(((uint32_t)l.steps + (uint32_t)per - 1) / (uint32_t)per) : 1; }
__device__ __forceinline__ int workgroups_of(const Load& l, int parts) { return (int)min((int64_t)l.blocks * parts, (int64_t)1 << 24); }   // (a launch holds fewer; row_starts may be anything)

// Workgroup x's item, by every lane of a wave; e < 0: there are fewer.
__device__ __forceinline__ Item item_at(const RowsParams& p, const AttnArgs& a, int x, int lane) {
  if (a.planned) {   // the last e that begins at x or before
    const int n = p.n_seqs * p.Hkv;
    if (x >= a.parts[n].x) return {-1, 0, 0, 0, 0, {}};
    int e = 0;
    for (int size = n; size > 1;) {
      const int stride = (size + 63) >> 6;
      const uint64_t upto = __ballot(lane * stride < size && a.parts[min(e + lane * stride, n - 1)].x <= x);
      const int last = max(__popcll(upto) - 1, 0);
      e += last * stride;
      size = min(stride, size - last * stride);
    }
    e = __builtin_amdgcn_readfirstlane(e);
    const int2 at = a.parts[e];
    const Load l = load_of(p, a, e);
    const int count = __builtin_amdgcn_readfirstlane(max(at.y, 1)), nth = __builtin_amdgcn_readfirstlane((x - at.x) / count), blocks = __builtin_amdgcn_readfirstlane(l.blocks);
    if (nth < 0 || nth >= blocks) return {-1, 0, 0, 0, 0, {}};
    const int index = __builtin_amdgcn_readfirstlane(x - at.x) - nth * count;
    return {e, blocks - 1 - nth, x - index, index, count,
            {__builtin_amdgcn_readfirstlane(l.s.row), __builtin_amdgcn_readfirstlane(l.s.n), __builtin_amdgcn_readfirstlane(l.s.pos), 0}};
  }
  const int n = p.n_seqs * p.Hkv;
  constexpr int HELD = 4;   // of a lane, loaded together (256 in all; more are asked for again)
  Load held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = 64 * i < n ? load_of(p, a, min(64 * i + lane, n - 1)) : Load{0, 1, {}};
  float total = 0.0f;
  int most = 1;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (64 * i + lane >= n) held[i].blocks = 0;
    total += (float)held[i].blocks * (float)held[i].steps;
    most = max(most, held[i].blocks ? held[i].steps : 1);
  }
  for (int e = 64 * HELD + lane; e < n; e += 64) {
    const Load l = load_of(p, a, e);
    total += (float)l.blocks * (float)l.steps;
    most = max(most, l.blocks ? l.steps : 1);
  }
  total = last_lane(wave_upto(total, 0.0f, [](float a, float b) { return a + b; }));
  most = last_lane(wave_upto(most, 1, [](int a, int b) { return max(a, b); }));
  const int per = steps_of_part(a, total, most);   // (the same in every wave)
  int before = 0;
  for (int e0 = 0; e0 < n; e0 += 64) {
    Load l{0, 1, {}};
    if (e0 >= 64 * HELD) {
      if (e0 + lane < n) l = load_of(p, a, e0 + lane);
    } else {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (e0 == 64 * i) l = held[i];
    }
    const int parts = parts_of(a, l, per), own = workgroups_of(l, parts);
    const int upto = wave_upto(own, 0, [](int a, int b) { return a + b; });
    const uint64_t past = __ballot(before + upto > x);
    if (past) {
      const int at = __builtin_ctzll(past), count = __builtin_amdgcn_readlane(parts, at), blocks = __builtin_amdgcn_readlane(l.blocks, at);
      const int start = before + __builtin_amdgcn_readlane(upto - own, at), nth = (x - start) / count, index = x - start - nth * count;
      return {e0 + at, blocks - 1 - nth, x - index, index, count,     // (the last rows, which see the most, first)
              {__builtin_amdgcn_readlane(l.s.row, at), __builtin_amdgcn_readlane(l.s.n, at), __builtin_amdgcn_readlane(l.s.pos, at), 0}};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, 0, 0, 0, {}};
}
// What the sum of parts needs to know of e; by the workgroup of its last block's first part.
__device__ __forceinline__ void note_parts(const RowsParams& p, const AttnArgs& a, const Item& it, int n_rows) {
  if (a.split && !a.planned && it.index == 0 && it.block == (n_rows - 1) / a.block_rows && threadIdx.x == 0) a.parts[it.e] = make_int2(it.first, it.count);
}

// The same for the whole call, by one workgroup, where there are many sequences (counted by each workgroup, 1024 sequences of 2048 tokens, four KV heads, took
// 1117 us instead of 654).
constexpr int PLAN_THREADS = 1024, PLAN_EACH = 4, PLANNED = 512;   // more (sequence, KV head) than this
__global__ __launch_bounds__(PLAN_THREADS) void attn_plan_kernel(RowsParams p, AttnArgs a) {
  __shared__ float sums[PLAN_THREADS / 64];
  __shared__ int most_of[PLAN_THREADS / 64], ends[PLAN_THREADS / 64];
  const int n = p.n_seqs * p.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float total = 0.0f;
  int most = 1;
  Load l[PLAN_EACH];
  auto load = [&](int e0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < PLAN_EACH; ++j) {
      const int e = e0 + PLAN_EACH * tid + j;
      l[j] = load_of(p, a, min(e, n - 1));
      if (e >= n) l[j].blocks = 0;
    }
  };
  if (a.split) {
    for (int e0 = 0; e0 < n; e0 += PLAN_EACH * PLAN_THREADS) {
      load(e0);
#pragma unroll
      for (int j = 0; j < PLAN_EACH; ++j) {
        total += (float)l[j].blocks * (float)l[j].steps;
        most = max(most, l[j].blocks ? l[j].steps : 1);
      }
    }
    total = wave_upto(total, 0.0f, [](float a, float b) { return a + b; });
    most = wave_upto(most, 1, [](int a, int b) { return max(a, b); });
    if (lane == 63) { sums[wave] = total; most_of[wave] = most; }
    __syncthreads();
    total = 0.0f;
    most = 1;
    for (int w = 0; w < PLAN_THREADS / 64; ++w) { total += sums[w]; most = max(most, most_of[w]); }
  }
  const int per = steps_of_part(a, total, most);
  int before = 0;
  for (int e0 = 0; e0 < n; e0 += PLAN_EACH * PLAN_THREADS) {
    load(e0);
    int parts[PLAN_EACH], own[PLAN_EACH], mine = 0;
#pragma unroll
    for (int j = 0; j < PLAN_EACH; ++j) {
      parts[j] = parts_of(a, l[j], per);
      own[j] = workgroups_of(l[j], parts[j]);
      mine += own[j];
    }
    const int upto = wave_upto(mine, 0, [](int a, int b) { return a + b; });
    __syncthreads();
    if (lane == 63) ends[wave] = upto;
    __syncthreads();
    int at = before + upto - mine;
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
      at += w < wave ? ends[w] : 0;
      before += ends[w];
    }
#pragma unroll
    for (int j = 0; j < PLAN_EACH; ++j) {
      const int e = e0 + PLAN_EACH * tid + j;
      if (e < n) a.parts[e] = make_int2(at, parts[j]);
      at += own[j];
    }
  }
  if (tid == 0) a.parts[n] = make_int2(before, 0);
}

// The tiles of 16 tokens that a row at max_pos sees: all up to it, or the listed ones of pages that begin at or before it.
struct Tiles { int entries, tiles; };
__device__ __forceinline__ Tiles tiles_to(const RowsParams& p, int e, const int32_t* list, int max_pos, int lane) {
  if (max_pos < 0) return {0, 0};
  if (!list) return {(max_pos >> p.log2_p) + 1, (max_pos >> 4) + 1};
  for (int end = min(max(p.sel_count[e], 0), p.sel_stride); end > 0;) {   // (ascending: the last such entry is near the end)
    const int base = max(end - 64, 0), at = base + lane;
    const int id = at < end ? list[at] : -1;
    const uint64_t seen = __ballot(id >= 0 && id <= (max_pos >> p.log2_p));
    if (seen) {
      const int entries = base + 64 - __builtin_clzll(seen);
      return {entries, entries << (p.log2_p - 4)};
    }
    end = base;
  }
  return {0, 0};
}

// Pages of 64 consecutive entries, one per lane: logical page (-1: there is nothing) and where it lies in the pools.
struct Window {
  int first, log;
  uint32_t lo, hi;
  __device__ __forceinline__ void fill(const RowsParams& p, int b, const int32_t* list, int n_entries, int e0, int lane, int es) {
    first = e0;
    const int e = e0 + lane, n_pages = (p.max_len + p.P - 1) >> p.log2_p;
    log = e < n_entries ? (list ? list[e] : e) : -1;
    const int phys = log >= 0 && log < n_pages ? page_of(p, b, log) : -1;
    if (phys < 0) log = -1;
    const uint64_t at = (uint64_t)max(phys, 0) * (uint64_t)p.pool_page_stride * es;
    lo = (uint32_t)at;
    hi = (uint32_t)(at >> 32);
  }
  __device__ __forceinline__ int page(int e) const { return __builtin_amdgcn_readlane(log, e - first); }
  __device__ __forceinline__ uint64_t where(int e) const {
    return (uint32_t)__builtin_amdgcn_readlane(lo, e - first) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, e - first) << 32;
  }
};

template <typename T, int D> struct Shape {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int ES = sizeof(T), TILES = BF ? 2 : 1, STEP = 16 * TILES;
  static constexpr int KC = D * ES / 64;        // pieces of 16 bytes of a token's key in a lane
  static constexpr int VW = D * ES / 64;        // words of a token's value in a lane
  static constexpr int NJ = D / 16, NZ = 4 * TILES;
};
// Keys and values of a step as a lane reads them.
template <typename T, int D> struct Raw {
  u32x4 k[Shape<T, D>::TILES][Shape<T, D>::KC];
  uint32_t v[Shape<T, D>::TILES][4][Shape<T, D>::VW];
};

// tile i of a step: `at` is the offset of its first token in the page, `tok` that from token to token
template <typename T, int D, bool STREAM>
__device__ __forceinline__ void load_tile(__amdgpu_buffer_rsrc_t kp, __amdgpu_buffer_rsrc_t vp, int at, int tok, uint32_t k_lane, uint32_t v_lane, Raw<T, D>& r, int i) {
  constexpr int AUX = STREAM ? 2 : 0;   // (non-temporal)
  using S = Shape<T, D>;
#pragma unroll
  for (int c = 0; c < S::KC; ++c) r.k[i][c] = __builtin_amdgcn_raw_buffer_load_b128(kp, k_lane + 64 * c, at, AUX);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (S::VW == 2) {
      const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(vp, v_lane, at + j * tok, AUX);
      r.v[i][j][0] = x.x; r.v[i][j][1] = x.y;
    } else {
#pragma unroll
      for (int w = 0; w < S::VW; w += 4) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(vp, v_lane + 4 * w, at + j * tok, AUX);
        r.v[i][j][w] = x.x; r.v[i][j][w + 1] = x.y; r.v[i][j][w + 2] = x.z; r.v[i][j][w + 3] = x.w;
      }
    }
  }
}

template <int RT, int NC> __device__ __forceinline__ void queries_landed(u32x4 (&q)[RT][NC]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(q[rt][c]));
}

// WIDE: pages of 32 tokens and more, a step lies in one (fp32: always).  STREAM: the cache is read past the caches (1 GB in pages of 16 tokens: 179, 160 us).
template <typename T, int D, int RT, bool WIDE, bool STREAM>
__global__ __launch_bounds__(64 * WAVES, 2) void attn_rows_kernel(RowsParams p, AttnArgs a) {
  extern __shared__ __align__(16) float merge[];
  using S = Shape<T, D>;
  constexpr int W = WAVES, TILES = S::TILES, KC = S::KC, VW = S::VW, NJ = S::NJ, NZ = S::NZ, ES = S::ES, ROWS = 16 * RT;
  const int lane = threadIdx.x & 63, m = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Item item = item_at(p, a, blockIdx.x, lane);
  if (item.e < 0) return;
  const int b = item.e / p.Hkv, g = item.e - b * p.Hkv;
  const Seq s = item.s;
  const int n_rows = s.n * p.G;
  note_parts(p, a, item, n_rows);
  const int r0 = item.block * ROWS;
  const int r_last = min(r0 + ROWS, n_rows) - 1;
  const int min_pos = s.pos + r0 / p.G, max_pos = s.pos + r_last / p.G;

  // queries: row 16 rt + m of the block
  u32x4 q[RT][KC];
  int pos[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(r0 + 16 * rt + m, r_last), i = r / p.G, h = g * p.G + (r - i * p.G);
    pos[rt] = s.pos + i;
    const T* row = (const T*)p.q.data + (int64_t)(s.row + i) * p.q.tok_stride + (int64_t)h * p.q.head_stride + kg * (16 / ES);
#pragma unroll
    for (int c = 0; c < KC; ++c) q[rt][c] = *reinterpret_cast<const u32x4*>(row + c * (64 / ES));
  }

  const int log_tpp = p.log2_p - 4;
  const int32_t* list = p.sel ? p.sel + (int64_t)item.e * p.sel_stride : nullptr;
  const Tiles seen = tiles_to(p, item.e, list, max_pos, lane);
  const int n_steps = (seen.tiles + TILES - 1) / TILES;
  const int parts = item.count * W, mine = item.index * W + wave;
  const int each = (int)((uint32_t)n_steps / (uint32_t)parts), more = n_steps - each * parts;   // (one more for the first `more`)
  const int u_first = each * mine + min(mine, more), u_end = u_first + each + (mine < more);
  int u = u_first;

  f32x4 acc[RT][NJ];
  float ref[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    ref[rt] = -INFINITY;
    sum[rt] = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[rt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale = p.sm_scale * LOG2E;

  Window win;
  const unsigned char* kbase = (const unsigned char*)p.k_pool + (int64_t)g * p.pool_head_stride * ES;
  const unsigned char* vbase = (const unsigned char*)p.v_pool + (int64_t)g * p.pool_head_stride * ES;
  const int tok = (int)p.pool_tok_stride * ES, page_bytes = (p.P - 1) * tok + D * ES;
  const uint32_t k_lane = (uint32_t)(m * tok + 16 * kg), v_lane = (uint32_t)(4 * kg * tok + m * (4 * VW));
  auto fetch = [&](int step, Raw<T, D>& r, int (&t0)[TILES]) __attribute__((always_inline)) {   // t0: positions of the tiles' first tokens
#pragma unroll
    for (int i = 0; i < (WIDE ? 1 : TILES); ++i) {
      const int t = TILES * step + i, e = t >> log_tpp, off = (t & ((1 << log_tpp) - 1)) << 4;
      if (e - win.first >= 64) win.fill(p, b, list, seen.entries, e, lane, ES);
      const int page = win.page(e);
      const uint64_t where = win.where(e);
      const __amdgpu_buffer_rsrc_t kp = page_buffer(kbase + where, page_bytes), vp = page_buffer(vbase + where, page_bytes);
      t0[i] = page < 0 ? NO_TOKEN : (page << p.log2_p) + off;
      load_tile<T, D, STREAM>(kp, vp, off * tok, tok, k_lane, v_lane, r, i);
      if constexpr (WIDE && TILES == 2) {
        t0[1] = t0[0] + 16;
        load_tile<T, D, STREAM>(kp, vp, (off + 16) * tok, tok, k_lane, v_lane, r, 1);
      }
    }
  };

  bool wild_seen = false;
  auto one_step = [&](Raw<T, D>& raw, const int (&t0)[TILES]) __attribute__((always_inline)) {
    const bool masked = (TILES == 1 ? t0[0] : WIDE ? t0[TILES - 1] : max(t0[0], t0[TILES - 1])) + 15 > min_pos;
    // Tokens that not every row sees.  Their V is zero where nothing of it is seen (it may be anything), and so are their values that are not
    // finite: a weight of zero does not stop those, so the rows that do see them get them at the end.
    bool wild = false;
    if (masked) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = t0[i] + 4 * kg + j;
          const bool partly = t > min_pos, unseen = t > max_pos;
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            uint32_t x = raw.v[i][j][w];
            if constexpr (S::BF) {
              const bool lo = wild16(x, 0), hi = wild16(x, 1);
              wild |= partly && !unseen && (lo || hi);
              x = partly && (unseen || lo) ? x & 0xffff0000u : x;
              x = partly && (unseen || hi) ? x & 0x0000ffffu : x;
            } else {
              const bool bad = wild32(x);
              wild |= partly && !unseen && bad;
              x = partly && (unseen || bad) ? 0 : x;
            }
            raw.v[i][j][w] = x;
          }
        }
      }
    }

    // S^T
    f32x4 st[RT][TILES];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int i = 0; i < TILES; ++i) st[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          if constexpr (S::BF) {
            st[rt][i] = mfma16(raw.k[i][c], q[rt][c], st[rt][i]);
          } else {
#pragma unroll
            for (int x = 0; x < 4; ++x) st[rt][i] = mfma4(raw.k[i][c][x], q[rt][c][x], st[rt][i]);
          }
        }

    float z[RT][NZ], all[RT];
    auto weights = [&](int rt, float from) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < NZ; ++e) z[rt][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[rt][e >> 2][e & 3], scale, -from));
      if (masked) {
#pragma unroll
        for (int e = 0; e < NZ; ++e) z[rt][e] = t0[e >> 2] + 4 * kg + (e & 3) <= pos[rt] ? z[rt][e] : 0.0f;
      }
      all[rt] = (z[rt][0] + z[rt][1]) + (z[rt][2] + z[rt][3]);
      if constexpr (NZ == 8) all[rt] += (z[rt][4] + z[rt][5]) + (z[rt][6] + z[rt][7]);
    };
    bool up = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      weights(rt, ref[rt]);
      up |= !(all[rt] <= MOST);
    }
    if (__any(up)) {   // (the first step of a row: its reference is -infinity, so weights are infinite, or NaN where the logit is -infinity too)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < NZ; ++e) {
          const bool visible = !masked || t0[e >> 2] + 4 * kg + (e & 3) <= pos[rt];
          top = fmaxf(top, visible ? st[rt][e >> 2][e & 3] * scale : -INFINITY);
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float to = fmaxf(ref[rt], top);
        const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref[rt] - to);
        ref[rt] = to;
        sum[rt] *= f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[rt][j] *= f;
        weights(rt, to == -INFINITY ? 0.0f : to);   // (all that was seen may be -infinity: no weight)
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sum[rt] += all[rt];

    if constexpr (S::BF) {
      u32x4 pf[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = pack2_bf16(z[rt][2 * e], z[rt][2 * e + 1]);
            if (t == 0) less(z[rt][2 * e], z[rt][2 * e + 1], w[e]);
          }
          pf[rt][t] = u32x4{w[0], w[1], w[2], w[3]};
        }
      // V: word x holds dims 2 x and 2 x + 1 of this lane's; tokens (i, 2 y), (i, 2 y + 1) make word 2 i + y of an operand
#pragma unroll
      for (int x = 0; x < VW; ++x) {
        u32x4 lo, hi;
        lo.x = low_halves(raw.v[0][0][x], raw.v[0][1][x]); lo.y = low_halves(raw.v[0][2][x], raw.v[0][3][x]);
        lo.z = low_halves(raw.v[TILES - 1][0][x], raw.v[TILES - 1][1][x]); lo.w = low_halves(raw.v[TILES - 1][2][x], raw.v[TILES - 1][3][x]);
        hi.x = high_halves(raw.v[0][0][x], raw.v[0][1][x]); hi.y = high_halves(raw.v[0][2][x], raw.v[0][3][x]);
        hi.z = high_halves(raw.v[TILES - 1][0][x], raw.v[TILES - 1][1][x]); hi.w = high_halves(raw.v[TILES - 1][2][x], raw.v[TILES - 1][3][x]);
#pragma unroll
        for (int t = 1; t >= 0; --t)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            acc[rt][2 * x] = mfma16(lo, pf[rt][t], acc[rt][2 * x]);
            acc[rt][2 * x + 1] = mfma16(hi, pf[rt][t], acc[rt][2 * x + 1]);
          }
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][j] = mfma4(raw.v[0][r][j], __float_as_uint(z[rt][r]), acc[rt][j]);
    }
    wild_seen |= wild;
  };

  // steps in flight: a wave that waits for its next one idles its share of the memory's latency (about a microsecond); two of 128 dims do not fit the registers
  // in fp32 (1 GB of cache, one row: two 195 us, one 180), nor beside two row tiles
  constexpr int AHEAD = D == 128 && (sizeof(T) == 4 || RT == 2) ? 1 : 2;
  Raw<T, D> raw[AHEAD];
  int t0[AHEAD][TILES];
  // The wait for a step lets every later fetch fly on, if the compiler can count them: the steady loop fetches without a condition,
  // and the queries have landed before it.
  if (u < u_end) win.fill(p, b, list, seen.entries, (TILES * u) >> log_tpp, lane, ES);
  if (u + 2 * AHEAD <= u_end) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(u + k, raw[k], t0[k]);
    queries_landed(q);
    for (; u + 2 * AHEAD <= u_end; u += AHEAD) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        one_step(raw[k], t0[k]);
        fetch(u + k + AHEAD, raw[k], t0[k]);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (u + k < u_end) fetch(u + k, raw[k], t0[k]);
  }
  for (; u < u_end; u += AHEAD) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (u + k >= u_end) break;
      one_step(raw[k], t0[k]);
      if (u + k + AHEAD < u_end) fetch(u + k + AHEAD, raw[k], t0[k]);
    }
  }

  // lane (m, kg): query m, dims D/4 kg + D/16 i + j of acc[.][j][i]
  if (__any(wild_seen)) {
    for (int tile = min(TILES * u_end, seen.tiles) - 1; tile >= TILES * u_first; --tile) {
      const int e = tile >> log_tpp, off = (tile & ((1 << log_tpp) - 1)) << 4, page = list ? list[e] : e;
      const int phys = page >= 0 && page < (p.max_len + p.P - 1) >> p.log2_p ? page_of(p, b, page) : -1, start = (page << p.log2_p) + off;
      if (phys < 0) continue;
      if (start + 15 <= min_pos) break;
      for (int t = max(0, min_pos + 1 - start); t < 16 && start + t <= max_pos; ++t) {
        const T* v = reinterpret_cast<const T*>(vbase + (int64_t)phys * p.pool_page_stride * ES + (int64_t)(off + t) * tok) + kg * (D / 4);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const float y = Elem<T>::load(v + NJ * x + j);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              if (wild32(__float_as_uint(y)) && start + t <= pos[rt]) acc[rt][j][x] += y;
          }
      }
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] += __shfl_xor(sum[rt], 16, 64);
    sum[rt] += __shfl_xor(sum[rt], 32, 64);
  }
  // the waves' sums, one row tile at a time: [wave][16][D + PAD] floats, [wave][16][2] references and sums of weights
  float* ml = merge + W * 16 * (D + PAD);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt) __syncthreads();
    if (kg == 0) *reinterpret_cast<float2*>(ml + (wave * 16 + m) * 2) = make_float2(ref[rt], sum[rt]);
    __syncthreads();
    float to = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) to = fmaxf(to, ml[(w * 16 + m) * 2]);
    const float f = ref[rt] == to ? 1.0f : __builtin_amdgcn_exp2f(ref[rt] - to);
    float* at = merge + (wave * 16 + m) * (D + PAD) + (D / 4) * kg;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; j += 4)
        *reinterpret_cast<float4*>(at + NJ * i + j) = make_float4(acc[rt][j][i] * f, acc[rt][j + 1][i] * f, acc[rt][j + 2][i] * f, acc[rt][j + 3][i] * f);
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * (D / 4); e += 64 * W) {
      const int r = e / (D / 4), d = (e - r * (D / 4)) * 4;
      if (r0 + 16 * rt + r >= n_rows) break;
      float y[4] = {0.f, 0.f, 0.f, 0.f}, ref_r = -INFINITY, sum_r = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) ref_r = fmaxf(ref_r, ml[(w * 16 + r) * 2]);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float4 v = *reinterpret_cast<const float4*>(merge + (w * 16 + r) * (D + PAD) + d);
        const float2 mw = *reinterpret_cast<const float2*>(ml + (w * 16 + r) * 2);
        const float fw = mw.x == ref_r ? 1.0f : __builtin_amdgcn_exp2f(mw.x - ref_r);
        sum_r += mw.y * fw;
        y[0] += v.x; y[1] += v.y; y[2] += v.z; y[3] += v.w;
      }
      const int row = r0 + 16 * rt + r;
      if (item.count > 1) {
        const int64_t to_part = (int64_t)blockIdx.x * ROWS + 16 * rt + r;
        *reinterpret_cast<float4*>(a.part + to_part * D + d) = make_float4(y[0], y[1], y[2], y[3]);
        if (d == 0) *reinterpret_cast<float2*>(a.part_ml + to_part * 2) = make_float2(ref_r, sum_r);
      } else {
        const int i = row / p.G, h = g * p.G + (row - i * p.G);
        const float fr = sum_r == 0.0f ? 0.0f : 1.0f / sum_r;
        T* dst = (T*)p.q_out.data + (int64_t)(s.row + i) * p.q_out.tok_stride + (int64_t)h * p.q_out.head_stride + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2_bf16(y[0] * fr, y[1] * fr), pack2_bf16(y[2] * fr, y[3] * fr));
        else *reinterpret_cast<float4*>(dst) = make_float4(y[0] * fr, y[1] * fr, y[2] * fr, y[3] * fr);
        if (d == 0) p.lse[(int64_t)h * p.n_rows + s.row + i] = sum_r == 0.0f ? -INFINITY : (ref_r + __builtin_amdgcn_logf(sum_r)) * LN2;
      }
    }
  }
}

// The parts of a row, in order: a workgroup per row and slice of DW dims, its threads in groups of DW / 4 that take every
// (256 / (DW / 4))-th part each.  A compute unit takes in about 10 B/ns of lines that others wrote, so a few rows of many parts go in slices of a line.
// MANY: rows of few parts, a group of threads a row.
template <typename T, int D, int DW, bool MANY>
__global__ __launch_bounds__(COMBINE_THREADS) void attn_combine_kernel(RowsParams p, AttnArgs a, int rows) {   // rows: of (sequence, KV head) that there can be at most
  constexpr int LANES = DW / 4, GROUPS = COMBINE_THREADS / LANES;
  __shared__ __align__(16) float lds[GROUPS][DW + PAD];
  __shared__ float lds_ml[GROUPS][2];
  const int grp = threadIdx.x / LANES, d = (threadIdx.x - grp * LANES) * 4;
  int x = blockIdx.x;
  const int slice = x % (D / DW);
  x /= D / DW;
  const int per_e = MANY ? (rows + GROUPS - 1) / GROUPS : rows;
  const int e = x / per_e, row = MANY ? (x - e * per_e) * GROUPS + grp : x - e * per_e;
  const int b = e / p.Hkv, g = e - b * p.Hkv;
  const int2 parts = a.parts[e];
  const Seq s = seq_of(p, b);
  if (row >= s.n * p.G || parts.y <= 1) return;   // (without rows, nobody wrote parts)
  const int block = row / a.block_rows, last = (s.n * p.G - 1) / a.block_rows;
  const int64_t first = parts.x + (int64_t)(last - block) * parts.y;
  if (first < 0 || first + parts.y > a.blocks) return;   // (rows beyond what the bounds allow have no workgroups)
  float ref = -INFINITY, sum = 0.0f, y[4] = {0.f, 0.f, 0.f, 0.f};
  constexpr int AT_ONCE = 4;   // (loads in flight: a chain of single ones takes a microsecond a part)
  const int step = MANY ? 1 : GROUPS;
  for (int k0 = MANY ? 0 : grp; k0 < parts.y; k0 += AT_ONCE * step) {
    float2 ml[AT_ONCE];
    float4 v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int64_t at = (first + min(k0 + i * step, parts.y - 1)) * a.block_rows + (row - block * a.block_rows);
      ml[i] = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
      v[i] = *reinterpret_cast<const float4*>(a.part + at * D + slice * DW + d);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (k0 + i * step >= parts.y) break;
      const float to = fmaxf(ref, ml[i].x);
      const float f0 = ref == to ? 1.0f : __builtin_amdgcn_exp2f(ref - to), f1 = ml[i].x == to ? 1.0f : __builtin_amdgcn_exp2f(ml[i].x - to);
      ref = to;
      sum = sum * f0 + ml[i].y * f1;
      y[0] = y[0] * f0 + v[i].x * f1; y[1] = y[1] * f0 + v[i].y * f1; y[2] = y[2] * f0 + v[i].z * f1; y[3] = y[3] * f0 + v[i].w * f1;
    }
  }
  if constexpr (!MANY) {
    *reinterpret_cast<float4*>(&lds[grp][d]) = make_float4(y[0], y[1], y[2], y[3]);
    if (d == 0) { lds_ml[grp][0] = ref; lds_ml[grp][1] = sum; }
    __syncthreads();
    if (grp) return;
    ref = -INFINITY; sum = 0.0f;
    y[0] = y[1] = y[2] = y[3] = 0.0f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) ref = fmaxf(ref, lds_ml[k][0]);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const float f = lds_ml[k][0] == ref ? 1.0f : __builtin_amdgcn_exp2f(lds_ml[k][0] - ref);
      const float4 v = *reinterpret_cast<const float4*>(&lds[k][d]);
      sum += lds_ml[k][1] * f;
      y[0] += v.x * f; y[1] += v.y * f; y[2] += v.z * f; y[3] += v.w * f;
    }
  }
  const int i = row / p.G, h = g * p.G + (row - i * p.G);
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* dst = (T*)p.q_out.data + (int64_t)(s.row + i) * p.q_out.tok_stride + (int64_t)h * p.q_out.head_stride + slice * DW + d;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2_bf16(y[0] * f, y[1] * f), pack2_bf16(y[2] * f, y[3] * f));
  else *reinterpret_cast<float4*>(dst) = make_float4(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
  if (d == 0 && slice == 0) p.lse[(int64_t)h * p.n_rows + s.row + i] = sum == 0.0f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * LN2;
}

// ---- many rows: tiles of keys and values in the LDS -------------------------------------------------------------------------
// Four waves of 32 query rows each share stages of 64 tokens (four tiles of 16, each inside a page), which come into the LDS by direct copies a stage ahead.
// With v_mfma_f32_32x32x16_bf16 and the row tiles of mfma_common.h: S^T = K Q^T from rows of K, O^T += V^T P^T from transposing reads of V, a lane
// holds one query row.  The softmax as above.
// What bounds it: the matrix unit and the power it draws (4096 rows over 16K tokens, 28 / 4 heads of 128: 1175 us, 0.72 PFLOP/s, 1.08 with the weights' second
// terms; a library product of 8192^3 1.21).  32 rows a wave and a stage of 64 tokens twice are what registers and LDS hold for two workgroups a compute unit.  First form,
// softmax and products one after the other, 396 us for three prompts; in one pipeline with the accumulators where they are 342 to 350.
// A row tile in the LDS: rows of 2 D bytes, granule c (16 bytes) of row r at c ^ f(r).  Head dim 128: that of mfma_common.h.  Head dim 64: two rows share a
// line of 256 bytes, f(r) = 4 ((r / 2) % 2) + (r / 4) % 4: 16 rows read at one granule, and the 4 rows x 64 bytes of a transposing read, use every bank once.
constexpr int TILE_ROWS = 128, TILE_STAGE = 64, TILE_THREADS = 256;
template <int D> constexpr int STAGE_BYTES = TILE_STAGE * 2 * D;            // of K, and of V
template <int D> constexpr int TILE_LDS = 4 * STAGE_BYTES<D> + 16;          // K and V, two stages, a flag
template <int D> __device__ __forceinline__ uint32_t swizzle(uint32_t r) { return D == 128 ? row_tile_f(r) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3); }

// the LDS at a byte
template <typename V> __device__ __forceinline__ V lds_at(uint32_t at) { return *(const __attribute__((address_space(3))) V*)at; }
// eight 16-bit words of one column of a row tile, from the addresses of rows 0 and 8 (mfma_common.h)
__device__ __forceinline__ u32x4 column_frag(uint32_t a0, uint32_t a1) {
  const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)a0));
  const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)a1));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
}
// LDS operations of a group of operands: groups of K, then of V
template <int D> constexpr int tile_ops(int group) { return group >= D / 16 ? 0 : group < D / 32 ? 2 : 4; }
// The lane, asked for anew: what a loop full of operands does not need is not kept over it.
__device__ __forceinline__ int lane_again() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

template <int D> __global__ __launch_bounds__(TILE_THREADS, 2) void attn_tiles_kernel(RowsParams p, AttnArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int STAGE = STAGE_BYTES<D>, TILE = 32 * D, HALF = 2 * TILE;    // bytes of a stage, of a tile of 16 tokens, of a unit of 32
  constexpr int NK = D / 16, NJ = D / 32;                                  // steps of a product over the dims; blocks of 32 of them
  const int lane = threadIdx.x & 63, lq = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Item item = item_at(p, a, blockIdx.x, lane);
  if (item.e < 0) return;
  const int b = item.e / p.Hkv, g = item.e - b * p.Hkv;
  const Seq s = item.s;
  const int n_rows = s.n * p.G;
  note_parts(p, a, item, n_rows);
  const int r0 = item.block * TILE_ROWS, w0 = r0 + 32 * wave;
  const int r_last = min(r0 + TILE_ROWS, n_rows) - 1, w_last = min(w0 + 32, n_rows) - 1;
  const int block_pos = s.pos + r_last / p.G;               // the last row's of the workgroup
  const int min_pos = s.pos + min(w0, r_last) / p.G;
  const int s0_pos = s.pos;

  u32x4 q[NK];
  {
    const int row = min(w0 + lq, r_last), token = row / p.G, head = g * p.G + (row - token * p.G);
    const bf16_t* x = (const bf16_t*)p.q.data + (int64_t)(s.row + token) * p.q.tok_stride + (int64_t)head * p.q.head_stride + 8 * hh;
#pragma unroll
    for (int k = 0; k < NK; ++k) q[k] = *reinterpret_cast<const u32x4*>(x + 16 * k);
  }

  const int log_tpp = p.log2_p - 4;
  const int32_t* list = p.sel ? p.sel + (int64_t)item.e * p.sel_stride : nullptr;
  const Tiles seen = tiles_to(p, item.e, list, block_pos, lane);
  const int n_stages = (seen.tiles + 3) >> 2;
  const int each = (int)((uint32_t)n_stages / (uint32_t)item.count), more = n_stages - each * item.count;   // (one more for the first `more`)
  const int first = each * item.index + min(item.index, more), end = first + each + (item.index < more);

  f32x16 acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[j][x] = 0.f;
  float ref = -INFINITY, sum = 0.0f;
  const float scale = p.sm_scale * LOG2E;

  // A stage lies in the LDS as K, then V; K comes a stage earlier.  Wave w brings tile w of both.
  const unsigned char* kbase = (const unsigned char*)p.k_pool + (int64_t)g * p.pool_head_stride * 2;
  const unsigned char* vbase = (const unsigned char*)p.v_pool + (int64_t)g * p.pool_head_stride * 2;
  const uint32_t row_bytes = (uint32_t)p.pool_tok_stride * 2;
  uint32_t src_off[NJ];          // of a lane's granules in a tile, a KiB of the LDS each
#pragma unroll
  for (int c = 0; c < NJ; ++c) {
    constexpr int PER_ROW = D / 8;
    const uint32_t r = (64 / PER_ROW) * c + lane / PER_ROW;
    src_off[c] = r * row_bytes + (((lane % PER_ROW) ^ swizzle<D>(r)) << 4) - 1024 * c;
  }
  Window win;
  win.first = -64;
  struct Stage { int t0[4]; uint64_t where; };   // positions of the tiles' first tokens; where this wave's tile lies in the pools
  auto locate = [&](int stage) __attribute__((always_inline)) -> Stage {
    Stage x;
    if (stage >= end) return {{NO_TOKEN, NO_TOKEN, NO_TOKEN, NO_TOKEN}, 0};   // (its copies read the pool's first page, so that every stage has its copies)
    const int t = 4 * stage, e0 = t >> log_tpp, e3 = (t + 3) >> log_tpp, tw = t + wave;
    if (e3 - win.first >= 64) win.fill(p, b, list, seen.entries, e0, lane, 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int page = win.page((t + i) >> log_tpp), off = ((t + i) & ((1 << log_tpp) - 1)) << 4;
      x.t0[i] = page < 0 ? NO_TOKEN : (page << p.log2_p) + off;
    }
    x.where = win.where(tw >> log_tpp) + (uint64_t)((tw & ((1 << log_tpp) - 1)) << 4) * row_bytes;
    return x;
  };
  auto copy_tile = [&](const unsigned char* src, uint32_t dst) __attribute__((always_inline)) {
    if constexpr (D == 128) copy_rows16_to_lds(src, src_off, dst);
    else copy_rows_to_lds(src, src_off[0], src_off[1], dst);
  };
  auto copy_k = [&](const Stage& x, uint32_t at) __attribute__((always_inline)) { copy_tile(kbase + x.where, at + wave * TILE); };
  auto copy_v = [&](const Stage& x, uint32_t at) __attribute__((always_inline)) { copy_tile(vbase + x.where, at + STAGE + wave * TILE); };

  // operands of a lane: granule 2 k + hh of its row of K (step k); of V, for dim block j, rows 4 hh + (lane % 16) / 4 (and + 8), four dims
  uint32_t n_at, t_at;
  {
    const uint32_t L = lane & 15, gq = lane >> 4, r = 4 * (gq >> 1) + (L >> 2);
    n_at = lq * (2 * D) + ((swizzle<D>(lq) ^ hh) << 4);
    t_at = STAGE + r * (2 * D) + (((2 * (gq & 1) + ((L & 3) >> 1)) ^ swizzle<D>(r)) << 4) + 8 * (L & 1);
  }
  // (the other steps', blocks' and rows' addresses differ in bits: one instruction each, out of the compiler's sight, as kept they would not fit the registers)
  auto with_bits = [](uint32_t x, const uint32_t bits) __attribute__((always_inline)) {
    if (bits) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(x) : "i"(bits), "v"(x));
    return x;
  };

  // One step of the pipeline, a unit being half a stage (32 tokens): the matrix instructions of S_{u+1} = K_{u+1} Q^T (D / 16) and of O += V_u P_u (D / 8) between
  // slices of the softmax of S_u, in slots that are kept in order; operands come from the LDS in groups of two, two groups ahead.
  constexpr int GK = NK / 2, GV = NJ, GROUPS = GK + GV;   // groups of K, then of V
  u32x4 fr[3][2];
  auto fetch = [&](uint32_t k_at, uint32_t v_at, int gr) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (gr < GK) {
        fr[gr % 3][i] = lds_at<u32x4>(with_bits(k_at, (2 * gr + i) << 5));
      } else {
        const int u = (gr - GK) / (NJ / 2), j = 2 * ((gr - GK) % (NJ / 2)) + i;
        fr[gr % 3][i] = column_frag(with_bits(v_at, j << 6) + TILE * u, with_bits(v_at, j << 6 | 32) + TILE * u + TILE / 2);
      }
    }
  };
  float from = 0.0f;            // the reference, 0 while it is -infinity
  // before a unit's weights: what a row does not see is -infinity, and the reference moves if a weight would pass 2^9
  auto refer = [&](f32x16& s, bool masked, int ta, int tb) __attribute__((always_inline)) {
    if (masked) {
      const int l = lane_again(), mine = s0_pos + min(w0 + (l & 31), r_last) / p.G - 4 * (l >> 5);   // this row's position, less the lane's first token
#pragma unroll
      for (int x = 0; x < 16; ++x) s[x] = (x < 8 ? ta : tb) + 8 * ((x >> 2) & 1) + (x & 3) <= mine ? s[x] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) top = fmaxf(top, s[x]);
    top *= scale;
    if (__any(top > ref + 9.0f)) {
      const float to = fmaxf(ref, half_max(top));
      const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      from = to == -INFINITY ? 0.0f : to;
      sum *= f;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[j][x] *= f;
    }
  };
  // k_buf, v_buf: LDS offsets of K of unit u + 1 and V of unit u; (ta, tb): positions of unit u's tiles
  auto step = [&](uint32_t k_buf, uint32_t v_buf, f32x16& s_in, f32x16& s_out, bool masked, int ta, int tb) __attribute__((always_inline)) {
    const uint32_t k_at = n_at + k_buf, v_at = t_at + v_buf;
    u32x4 pr[2][2];              // [16 tokens][term]
    auto weigh = [&](int e) __attribute__((always_inline)) {   // a pair of logits
      float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s_in[2 * e], scale, -from)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(s_in[2 * e + 1], scale, -from));
      sum += x + y;
      const uint32_t w = pack2_bf16(x, y);
      less(x, y, w);
      pr[e >> 2][0][e & 3] = w;
      pr[e >> 2][1][e & 3] = pack2_bf16(x, y);
    };
    fetch(k_at, v_at, 0);
    fetch(k_at, v_at, 1);
    refer(s_in, masked, ta, tb);
    auto group = [&](auto number) __attribute__((always_inline)) {
      constexpr int gr = decltype(number)::value;
      if constexpr (gr + 2 < GROUPS) fetch(k_at, v_at, gr + 2);
      __builtin_amdgcn_s_waitcnt(0xC07F | (tile_ops<D>(gr + 1) + tile_ops<D>(gr + 2)) << 8);   // lgkmcnt: what was fetched after this group
      __builtin_amdgcn_sched_barrier(0);   // keep the fetch ahead of this group's matrix instructions
      if constexpr (gr < GK) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (gr == 0 && i == 0) {
            f32x16 zero;
#pragma unroll
            for (int x = 0; x < 16; ++x) zero[x] = 0.f;
            s_out = mfma32(__builtin_bit_cast(bf16x8, fr[0][0]), __builtin_bit_cast(bf16x8, q[0]), zero);
          } else {
            s_out = mfma32(__builtin_bit_cast(bf16x8, fr[gr % 3][i]), __builtin_bit_cast(bf16x8, q[2 * gr + i]), s_out);
          }
          if (GK == 2) weigh(2 * gr + i);
          else if (i == 0) weigh(gr);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        constexpr int u = (gr - GK) / (NJ / 2), j = 2 * ((gr - GK) % (NJ / 2));
#pragma unroll
        for (int t = 1; t >= 0; --t) {
#pragma unroll
          for (int i = 0; i < 2; ++i) acc[j + i] = mfma32(__builtin_bit_cast(bf16x8, fr[gr % 3][i]), __builtin_bit_cast(bf16x8, pr[u][t]), acc[j + i]);
          if (u == 0) {
            if (NJ == 4) weigh(4 + j + (1 - t));
            else { weigh(4 + 2 * (1 - t)); weigh(5 + 2 * (1 - t)); }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    group(std::integral_constant<int, 0>{});
    group(std::integral_constant<int, 1>{});
    group(std::integral_constant<int, 2>{});
    group(std::integral_constant<int, 3>{});
    if constexpr (GROUPS == 8) {
      group(std::integral_constant<int, 4>{});
      group(std::integral_constant<int, 5>{});
      group(std::integral_constant<int, 6>{});
      group(std::integral_constant<int, 7>{});
    }
  };
  auto beyond = [&](const Stage& x, int from_pos) { return max(max(x.t0[0], x.t0[1]), max(x.t0[2], x.t0[3])) + 15 > from_pos; };   // whether it goes past a position
  // Tokens of a stage that not every row of the workgroup sees: their V becomes zero where no row sees it (it may be anything), and so do their
  // values that are not finite: a weight of zero does not stop those, so the rows that do see them get them at the end of the stage.
  const int block_min = s.pos + r0 / p.G;
  volatile int* const wild_seen = reinterpret_cast<volatile int*>(smem + 4 * STAGE);
  auto tame = [&](const Stage& x, uint32_t v_at) __attribute__((always_inline)) {
    const int tid = 64 * wave + lane_again(), r = tid >> 2, i = r >> 4, t = (i == 0 ? x.t0[0] : i == 1 ? x.t0[1] : i == 2 ? x.t0[2] : x.t0[3]) + (r & 15);
    bool wild = false;
    if (t > block_min) {
      uint4* at = reinterpret_cast<uint4*>(smem + v_at + STAGE + r * (2 * D) + (tid & 3) * (D / 2));
      for (int c = 0; c < D / 32; ++c) {
        uint4 v = at[c];
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool lo = wild16(w[e], 0), hi = wild16(w[e], 1);
          wild |= t <= block_pos && (lo || hi);
          w[e] = t > block_pos ? 0 : w[e] & (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
        }
        at[c] = v;
      }
    }
    if (wild) *wild_seen = 1;
    __syncthreads();
  };
  f32x16 sA, sB;
  Stage cur = locate(first), next = locate(first + 1);
  if (first < end) {
    if (threadIdx.x == 0) *wild_seen = 0;
    copy_k(cur, 0);
    copy_v(cur, 0);
    copy_k(next, 2 * STAGE);
    wait_copies<2 * NJ>();
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 16; ++x) sA[x] = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) sA = mfma32(__builtin_bit_cast(bf16x8, lds_at<u32x4>(with_bits(n_at, k << 5))), __builtin_bit_cast(bf16x8, q[k]), sA);
  }
  // Copies complete in order, as many of a wave for K as for V; each has a stage of time.  (A wave without rows works on the last row.)
  uint32_t at = 0;               // LDS offset of this stage; the other one's: at ^ 2 STAGE
  for (int stage = first; stage < end; ++stage) {
    wait_copies<NJ>();            // V of this stage has landed, and every wave is done with the one before
    __syncthreads();
    copy_v(next, at ^ 2 * STAGE);
    if (beyond(cur, block_min)) tame(cur, at);
    const bool masked = beyond(cur, min_pos);
    step(at + HALF, at, sA, sB, masked, cur.t0[0], cur.t0[1]);
    const Stage after = locate(stage + 2);
    wait_copies<NJ>();            // K of the next stage has landed, and every wave is done with this one's
    __syncthreads();
    copy_k(after, at);
    step(at ^ 2 * STAGE, at + HALF, sB, sA, masked, cur.t0[2], cur.t0[3]);
    cur = next;
    next = after;
    at ^= 2 * STAGE;
  }

  wait_copies<0>();              // (the last ones, which nobody reads, before the LDS is another's)
  const int l = lane_again(), lr = l & 31, half = l >> 5, row = min(w0 + lr, r_last), token = row / p.G, head = g * p.G + (row - token * p.G), pos = s.pos + token;
  if (first < end && *wild_seen) {   // a lane holds dims 32 j + 8 (x / 4) + 4 hh + x % 4 of its row in acc[j][x]
    for (int tile = min(4 * end, seen.tiles) - 1; tile >= 4 * first; --tile) {
      const int e = tile >> log_tpp, off = (tile & ((1 << log_tpp) - 1)) << 4, page = list ? list[e] : e;
      const int phys = page >= 0 && page < (p.max_len + p.P - 1) >> p.log2_p ? page_of(p, b, page) : -1;
      if (phys < 0) continue;
      const int t0 = (page << p.log2_p) + off;
      if (t0 + 15 <= block_min) break;
      for (int t = max(0, block_min + 1 - t0); t < 16 && t0 + t <= block_pos; ++t) {
        const bf16_t* v = reinterpret_cast<const bf16_t*>(vbase + (int64_t)phys * p.pool_page_stride * 2 + (int64_t)(off + t) * row_bytes) + 4 * half;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const float y = bf16_to_f32(v[32 * j + 8 * (x >> 2) + (x & 3)]);
            if (wild32(__float_as_uint(y)) && t0 + t <= pos) acc[j][x] += y;
          }
      }
    }
  }
  sum = half_sum(sum);
  if (w0 >= n_rows || w0 + lr > w_last) return;
  if (item.count > 1) {
    const int64_t to = (int64_t)blockIdx.x * TILE_ROWS + 32 * wave + lr;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int x = 0; x < 16; x += 4)
        *reinterpret_cast<float4*>(a.part + to * D + 32 * j + 2 * x + 4 * half) = make_float4(acc[j][x], acc[j][x + 1], acc[j][x + 2], acc[j][x + 3]);
    if (half == 0) *reinterpret_cast<float2*>(a.part_ml + to * 2) = make_float2(ref, sum);
    return;
  }
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  bf16_t* dst = (bf16_t*)p.q_out.data + (int64_t)(s.row + token) * p.q_out.tok_stride + (int64_t)head * p.q_out.head_stride + 4 * half;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int x = 0; x < 16; x += 4)
      *reinterpret_cast<uint2*>(dst + 32 * j + 2 * x) = make_uint2(pack2_bf16(acc[j][x] * f, acc[j][x + 1] * f), pack2_bf16(acc[j][x + 2] * f, acc[j][x + 3] * f));
  if (half == 0) p.lse[(int64_t)head * p.n_rows + s.row + token] = sum == 0.0f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * LN2;
}

// How a call is cut.
struct Plan {
  int tiles, rt, stream, split, planned, full, block_rows, step, target, min_steps;
  int64_t blocks;   // workgroups at most
};
Plan plan_of(const RowsParams& p, bool is_bf16, int32_t sel_stride) {
  Plan c{};
  const int64_t rows = (int64_t)p.max_rows * p.G, heads = (int64_t)p.n_seqs * p.Hkv;
  int64_t tokens = p.max_len;
  if (sel_stride >= 0 && (int64_t)sel_stride * p.P < tokens) tokens = (int64_t)sel_stride * p.P;
  const int64_t reach = heads * tokens, held = p.num_phys * p.Hkv * p.P, cache_bytes = (reach < held ? reach : held) * 2 * p.D * (is_bf16 ? 2 : 4);
  // Readings of the caches after the first, in bytes, at 16 and at 32 rows a block.
  const int64_t again_16 = ((rows + 15) / 16 - 1) * cache_bytes, again_32 = ((rows + 31) / 32 - 1) * cache_bytes;
  // Tiles once the caches are read by a second block of 32 rows and that costs more than their start (one sequence, D 128, us without and with: 4 heads of 4096
  // tokens, 35 rows 17, 16; of 65,536, 54, 40; 64 of 2048, one head, 64 rows 36, 31; 16 of 4096, D 64, one head, 96 rows 20, 21).
  // It goes by the most rows of a sequence, for the whole call: single tokens beside a prompt's piece go in tiles too, seven rows in place of 128 (31 of up to 32K tokens and a
  // piece of 1000 rows: 610 us; in two calls 107 and 340).
  c.tiles = is_bf16 && rows > 32 && again_32 > (48ll << 20) && p.pool_tok_stride <= (1 << 24);   // (offsets of a lane in a tile: 32 bits)
  // Two row tiles a wave where rows need them; at head dim 128 for bf16 and caches that are worth it, one step in flight instead of two (32 rows of one head, us
  // with one and two: 4096 tokens 12, 14; 65,536, 25, 23; 28 rows of four heads over 500,000, in tiles 224, in two 167: 6.1 TB/s).
  c.rt = rows > 16 && (p.D == 64 || (is_bf16 && again_16 > (16ll << 20))) ? 2 : 1;
  c.block_rows = c.tiles ? TILE_ROWS : 16 * c.rt;
  c.step = c.tiles ? TILE_STAGE : 32;
  const int64_t steps = (tokens + c.step - 1) / c.step;
  // blocks of rows of all sequences at most
  const int64_t each = (rows + c.block_rows - 1) / c.block_rows;
  int64_t blocks = ((int64_t)p.n_rows * p.G / c.block_rows + p.n_seqs) * p.Hkv;
  if (blocks > each * heads) blocks = each * heads;
  c.min_steps = c.tiles ? 8 : 4;
  c.planned = heads > PLANNED;
  c.split = steps > 16 && blocks <= (c.planned && !c.tiles ? 16 * WGS : 2 * WGS);   // (more fill the chip; parts of tiles take up to 66 KB a workgroup, others 8 or 16)
  // Parts come out rounded up, half a part more for each block: one round of workgroups for few blocks (32 ragged sequences, 128 blocks: to 448, 704 workgroups 48.7, 53
  // us), shorter parts that even out for many (512 of them: to 2048, 2304 in 599, 587 us), but equal ones stay whole (1024 of 2048 tokens: 666, in halves 737).
  c.full = !c.tiles && blocks > WGS;
  c.target = (int)(c.tiles ? WGS : c.full ? blocks + WGS / 2 : blocks < WGS ? WGS - blocks / 2 : blocks);
  const int64_t most = (steps + c.min_steps - 1) / c.min_steps;
  const int64_t parts = c.target + blocks + 2;   // (what item_at comes to at most; two for its roundings)
  c.blocks = !c.split ? blocks : blocks * most < parts ? blocks * most : parts;
  // Measured where a byte is read once (single tokens); rows that read the caches again, prompts in fp32, lose by it (1000 rows, 28 / 4 heads of 128 dims, 336 MB: 23.2 ms,
  // through the caches 11.5; 14 / 2 of 64 dims, 338 MB: 12.1, 10.6; 1000 rows of 2000 tokens in a pool of 600 MB: 0.226, 0.220).
  c.stream = cache_bytes > (256ll << 20);
  return c;
}
// The sum of parts runs where c.split: a workgroup per row (before slices, which only a few rows have), or per eight (head dim 64: sixteen).
bool combine_many(const RowsParams& p) { return (int64_t)p.n_seqs * p.Hkv * p.max_rows * p.G > 4096; }   // (then a row has few parts)
int64_t combine_blocks(const RowsParams& p, const Plan& c) {
  const int64_t rows = (int64_t)p.max_rows * p.G, heads = (int64_t)p.n_seqs * p.Hkv, at_once = 4 * COMBINE_THREADS / p.D;
  return combine_many(p) ? heads * ((rows + at_once - 1) / at_once) : heads * rows;
}
size_t part_bytes(const RowsParams& p, const Plan& c) {
  return (c.split ? (size_t)c.blocks * c.block_rows * (p.D + 2) * sizeof(float) : 0) + (c.split || c.planned ? ((size_t)p.n_seqs * p.Hkv + 1) * sizeof(int2) : 0);
}

template <typename T, int D, typename K> hipError_t run(const RowsParams& p, const Plan& c, K kernel, int threads, size_t lds, DeviceOnce& once, void* ws, hipStream_t st) {
  AttnArgs a{c.block_rows, c.step, c.split, c.tiles, c.target, c.min_steps, c.full, c.planned, (int2*)ws, nullptr, nullptr, (int)c.blocks};
  if (c.split) {
    a.part = (float*)ws;
    a.part_ml = a.part + c.blocks * c.block_rows * D;
    a.parts = (int2*)(a.part_ml + c.blocks * c.block_rows * 2);
  }
  if (c.planned) {
    ProfScope prof_("attn_plan", st);
    attn_plan_kernel<<<dim3(1), dim3(PLAN_THREADS), 0, st>>>(p, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  {
    ProfScope prof_(c.tiles ? "attn_tiles" : "attn_rows", st);
    if (lds > 65536) {
      const hipError_t e = ensure_max_dynamic_lds(once, (const void*)kernel, (int)lds);
      if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)c.blocks), dim3(threads), lds, st>>>(p, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !c.split) return e;
  }
  ProfScope prof_("attn_combine", st);
  const int rows = p.max_rows * p.G;
  const int64_t wgs = combine_blocks(p, c);
  if (combine_many(p)) attn_combine_kernel<T, D, D, true><<<dim3((unsigned)wgs), dim3(COMBINE_THREADS), 0, st>>>(p, a, rows);
  else if (wgs < 256 && c.blocks > 32 * (int64_t)p.n_seqs * p.Hkv) attn_combine_kernel<T, D, 32, false><<<dim3((unsigned)(wgs * (D / 32))), dim3(COMBINE_THREADS), 0, st>>>(p, a, rows);
  else attn_combine_kernel<T, D, D, false><<<dim3((unsigned)wgs), dim3(COMBINE_THREADS), 0, st>>>(p, a, rows);
  return hipGetLastError();
}
template <typename T, int D, int RT, bool WIDE, bool STREAM> hipError_t run_rows(const RowsParams& p, const Plan& c, void* ws, hipStream_t st) {
  static DeviceOnce once;
  return run<T, D>(p, c, attn_rows_kernel<T, D, RT, WIDE, STREAM>, 64 * WAVES, (size_t)(WAVES * 16 * (D + PAD) + WAVES * 16 * 2) * sizeof(float), once, ws, st);
}
template <typename T, int D, int RT> hipError_t run_rows(const RowsParams& p, const Plan& c, void* ws, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (p.P < 32) return c.stream ? run_rows<T, D, RT, false, true>(p, c, ws, st) : run_rows<T, D, RT, false, false>(p, c, ws, st);
  }
  return c.stream ? run_rows<T, D, RT, true, true>(p, c, ws, st) : run_rows<T, D, RT, true, false>(p, c, ws, st);
}
// (instantiated for one type and head dim per source file, which are compiled side by side)
template <typename T, int D> hipError_t attn(const RowsParams& p, void* ws, hipStream_t st) {
  const Plan c = plan_of(p, sizeof(T) == 2, p.sel ? p.sel_stride : -1);
  if constexpr (sizeof(T) == 2) {
    static DeviceOnce once;
    if (c.tiles) return run<T, D>(p, c, attn_tiles_kernel<D>, TILE_THREADS, TILE_LDS<D>, once, ws, st);
  }
  if constexpr (D == 64 || sizeof(T) == 2) {
    if (c.rt == 2) return run_rows<T, D, 2>(p, c, ws, st);
  }
  return run_rows<T, D, 1>(p, c, ws, st);
}

}  // namespace
}  // namespace oomb
