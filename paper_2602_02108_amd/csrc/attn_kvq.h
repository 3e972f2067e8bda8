// Attention of packed rows over a cache of 4-bit codes (layouts: include/oomb.h, rows.h).
//
// A wave holds RT tiles of 16 query rows and walks units of 32 tokens (two tiles of 16, each inside a page); the G query heads of
// a KV head share its cache: query row r of a sequence and KV head is token r / G, head r % G.  Operands come straight from
// memory, no LDS and no exchange of lanes.  With lane = 16 kg + m:
//   v_mfma_f32_16x16x32_bf16: lane l holds A[l % 16][8 (l / 16) + 0..7], B alike with columns, C[4 (l / 16) + r][l % 16] in register r
//   S^T = K Q^T: lane (m, kg) reads the codes of dims D/4 kg .. of token m in one load (at D = 128 one block of 32 dims, one scale)
//       and converts a word at a time into the operands of the steps c; the queries are laid out to match: k index 8 kg + j of step c is dim
//       D/4 kg + 8 c + j
//   O^T += V^T P^T: a lane's accumulators of S^T are tokens 4 kg + 0..3 of both tiles of query m: in this order they are the B operand.
//       For the A operand lane (m, kg) reads those eight tokens' codes of dims D/16 m .., converts each with its own scale and puts pairs of tokens
//       together with byte permutes; operand j holds dims D/16 m + j
// Conversions are v_cvt_scalef32_pk_bf16_fp4 (two values each, scale applied, exact); every value of the cache is exact in bf16.  fp32
// rows: Q and P in three bf16 terms (24 bits).  bf16 rows: P in two (16 bits), so that the output's own rounding is the larger one, whatever else is in the
// call (in one term a bf16 output is 2.3e-3 from 64 bits instead of 1.7e-3, which is its own rounding).  (The codes could be a matrix operand as they are, v_mfma_scale_f32_16x16x128_f8f6f4 against e4m3 terms of the queries: its sums
// were off by 2^-16 of the largest product, where these are fp32 sums of exact products.)
//
// Softmax in one pass: weights are taken against a reference of the row that moves only when the eight weights of a lane in a unit
// exceed 2^9 together; so no maximum is formed on the way, and sums stay far inside a float.
//
// The waves of a workgroup share a row block and split its tokens; long caches are cut into parts of equal work over workgroups, counted on the
// device from the lengths as they are, and kvq_combine adds a row's parts in their order.
//
// Measured (28 / 4 heads, D 128, P 128): one token against 1,048,001: 103 us, 5.5 TB/s of the cache, bound by memory; 2048 rows over 80
// listed pages: 381 us, 0.71 PFLOP/s, bound by the vector unit (240 vector instructions for 48 matrix ones in a unit of two row tiles, 64 of them
// conversions, 32 permutes, 16 exponentials, 40 for the second terms of the weights); 32 sequences of one to 32K tokens: 22 us.  Two row tiles a wave and not more: with four, one wave per SIMD
// is left and its instructions wait for each other (599 us), three spill.
#pragma once
#include <type_traits>

#include "common.h"
#include "launch.h"
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
constexpr int WGS = 512;                 // workgroups that a call is cut into

typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
template <int SEL> __device__ __forceinline__ uint32_t cvt2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// what is left of a and b after their bf16 roundings, packed as `w`
__device__ __forceinline__ void less(float& a, float& b, uint32_t w) {
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
}

struct AttnArgs {
  int row_blocks;              // per (sequence, KV head)
  int split;                   // parts over workgroups (else one part per (sequence, KV head))
  int target, min_units;       // parts to aim at; units of a part at least
  int2* parts;                 // [sequence * Hkv + KV head]: first part, number of parts
  float* part;                 // [part][row block][row of the block][D] sums
  float* part_ml;              // [part][row block][row][2]: reference, sum
};

// Codes and scales of a unit as a lane reads them.
template <int D> struct Raw {
  uint32_t k[2][D / 32];
  uint32_t ks[2];
  uint32_t v[2][4];
  uint32_t vs[2];
};

// Where a lane's share of a tile lies: offsets from the tile's codes (its row of the page) and from its scales.
struct Lane { uint32_t k, ks, v, vs; };
template <int D> __device__ __forceinline__ Lane lane_at(int P, int m, int kg) {
  const int kb = D == 128 ? kg : kg >> 1, vb = D == 128 ? m >> 2 : m >> 3;
  return {(uint32_t)(m * (D / 2) + kg * (D / 8)), (uint32_t)(kb * P + m), (uint32_t)(4 * kg * (D / 2) + m * (D / 32)), (uint32_t)(vb * P + 4 * kg)};
}
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// A page of one head: buffer loads take its base, a lane's offset and the tile's from three registers, so that addresses cost next to no
// instruction; what lies past the page reads as zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_buffer(const unsigned char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, bytes, 0x00027000);
}
// tile i of a unit: `codes` and `scales` are the offsets of the unit's first token in the page, `further` tokens lie before the tile
template <int D, bool STREAM> __device__ __forceinline__ void load_tile(__amdgpu_buffer_rsrc_t kp, __amdgpu_buffer_rsrc_t vp, int codes, int scales, int further, const Lane& l, Raw<D>& r, int i) {
  constexpr int AUX = STREAM ? 2 : 0;   // (non-temporal)
  const int c = further * (D / 2);
  if constexpr (D == 128) {
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(kp, l.k + c, codes, AUX);
    r.k[i][0] = x.x; r.k[i][1] = x.y; r.k[i][2] = x.z; r.k[i][3] = x.w;
  } else {
    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(kp, l.k + c, codes, AUX);
    r.k[i][0] = x.x; r.k[i][1] = x.y;
  }
  r.ks[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(kp, l.ks + further, scales, 0);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (D == 128) r.v[i][j] = __builtin_amdgcn_raw_buffer_load_b32(vp, l.v + c + j * (D / 2), codes, AUX);
    else r.v[i][j] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(vp, l.v + c + j * (D / 2), codes, AUX);
  }
  r.vs[i] = __builtin_amdgcn_raw_buffer_load_b32(vp, l.vs + further, scales, 0);
}

// This lane's D / 4 dims of a query row, as operands of the steps and terms.
template <typename T, int D, int QT> __device__ __forceinline__ void query_terms(const T* row, uint4 (&q)[QT][D / 32]) {
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    if constexpr (QT == 1) {
      q[0][c] = *reinterpret_cast<const uint4*>(row + 8 * c);
    } else {
      float f[8];
      Vec16<float>::unpack(reinterpret_cast<const uint4*>(row + 8 * c)[0], f);
      Vec16<float>::unpack(reinterpret_cast<const uint4*>(row + 8 * c)[1], f + 4);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = pack2_bf16(f[2 * e], f[2 * e + 1]);
          less(f[2 * e], f[2 * e + 1], w[e]);
        }
        q[t][c] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

// Queries that are needed in every step are waited for here, once.
template <int RT, int QT, int NC> __device__ __forceinline__ void landed(uint4 (&q)[RT][QT][NC]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(q[rt][t][c].x), "+v"(q[rt][t][c].y), "+v"(q[rt][t][c].z), "+v"(q[rt][t][c].w));
}

// Byte X of a tile's four tokens' codes converted: words of tokens (0, 1) and (2, 3) for its even and its odd dim.
template <int X, int D> __device__ __forceinline__ void pairs(const Raw<D>& raw, int i, uint32_t* lo, uint32_t* hi) {
#pragma unroll
  for (int y = 0; y < 2; ++y) {   // (of a scale the conversion takes the exponent's bits alone)
    const float sa = __uint_as_float(raw.vs[i] << (y ? 7 : 23)), sb = __uint_as_float(y ? raw.vs[i] >> 1 : raw.vs[i] << 15);
    const uint32_t va = cvt2<X>(raw.v[i][2 * y], sa), vb = cvt2<X>(raw.v[i][2 * y + 1], sb);
    lo[y] = low_halves(va, vb);
    hi[y] = high_halves(va, vb);
  }
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

// WIDE: pages of 32 tokens and more, a unit lies in one.  STREAM: codes past the caches.
template <typename T, int D, int RT, int W, bool WIDE, bool STREAM>
__global__ __launch_bounds__(64 * W, RT == 1 && W == 4 && sizeof(T) == 2 ? 3 : 2) void attn_kvq_kernel(RowsParams p, AttnArgs a) {
  extern __shared__ __align__(16) float merge[];
  constexpr int QT = sizeof(T) == 2 ? 1 : 3, PT = sizeof(T) == 2 ? 2 : 3, NC = D / 32, NJ = D / 16, ROWS = 16 * RT;
  const int lane = threadIdx.x & 63, m = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int px = blockIdx.x / a.row_blocks, block = blockIdx.x - px * a.row_blocks;
  const Part part = part_at(p, a, px, lane);
  if (part.e < 0) return;
  const int b = part.e / p.Hkv, g = part.e - b * p.Hkv;
  const Seq s = seq_of(p, b);
  if (a.split && part.index == 0 && block == 0 && threadIdx.x == 0) a.parts[part.e] = make_int2(part.first, part.count);
  const int n_rows = s.n * p.G;
  const int r0 = block * ROWS;
  if (r0 >= n_rows) return;
  const int r_last = min(r0 + ROWS, n_rows) - 1;
  const int min_pos = s.pos + r0 / p.G, max_pos = s.pos + r_last / p.G;

  // queries: row 16 rt + m of the block
  uint4 q[RT][QT][NC];
  int pos[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(r0 + 16 * rt + m, r_last), i = r / p.G, h = g * p.G + (r - i * p.G);
    pos[rt] = s.pos + i;
    query_terms<T, D, QT>((const T*)p.q.data + (int64_t)(s.row + i) * p.q.tok_stride + (int64_t)h * p.q.head_stride + kg * (D / 4), q[rt]);
  }

  // the tiles that some row sees: entries of the list up to the last row's page
  const int log_tpp = p.log2_p - 4, n_pages = (p.max_len + p.P - 1) >> p.log2_p;
  const int32_t* list = p.sel ? p.sel + (int64_t)part.e * p.sel_stride : nullptr;
  int n_entries = 0, n_tiles = 0;
  if (max_pos >= 0) {
    if (list) {
      int e = min(max(p.sel_count[part.e], 0), p.sel_stride);
      while (e > 0) {      // (ascending: the last entry that begins at or before max_pos is near the end)
        const int base = max(e - 64, 0), at = base + lane;
        const int id = at < e ? list[at] : -1;
        const uint64_t seen = __ballot(id >= 0 && id <= (max_pos >> p.log2_p));
        if (seen) {
          n_entries = base + 64 - __builtin_clzll(seen);
          break;
        }
        e = base;
      }
      n_tiles = n_entries << log_tpp;
    } else {
      n_tiles = (max_pos >> 4) + 1;
      n_entries = (max_pos >> p.log2_p) + 1;
    }
  }
  const int n_units = (n_tiles + 1) >> 1;
  const int parts = part.count * W, mine = part.index * W + wave;
  const int each = (int)((uint32_t)n_units / (uint32_t)parts), more = n_units - each * parts;   // (one more for the first `more`)
  int u = each * mine + min(mine, more);
  const int u_end = u + each + (mine < more);

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

  // pages of 64 consecutive entries, one per lane: logical page (-1: there is nothing) and where it lies in the pools
  int win = 0, w_log = -1;
  uint32_t w_lo = 0, w_hi = 0;
  auto window = [&](int e0) __attribute__((always_inline)) {
    win = e0;
    const int e = e0 + lane;
    w_log = e < n_entries ? (list ? list[e] : e) : -1;
    const int phys = w_log >= 0 && w_log < n_pages ? page_of(p, b, w_log) : -1;
    if (phys < 0) w_log = -1;
    const uint64_t at = (uint64_t)max(phys, 0) * (uint64_t)p.pool_page_stride;
    w_lo = (uint32_t)at;
    w_hi = (uint32_t)(at >> 32);
  };
  const unsigned char* kbase = (const unsigned char*)p.k_pool + (int64_t)g * p.pool_head_stride;
  const unsigned char* vbase = (const unsigned char*)p.v_pool + (int64_t)g * p.pool_head_stride;
  const Lane at_lane = lane_at<D>(p.P, m, kg);
  const int tile_bytes = p.P * (D / 2 + D / 32), first_scale = p.P * (D / 2);
  auto fetch = [&](int unit, Raw<D>& r, int (&t0)[2]) __attribute__((always_inline)) {   // t0: positions of the tiles' first tokens
#pragma unroll
    for (int i = 0; i < (WIDE ? 1 : 2); ++i) {
      const int t = 2 * unit + i, e = t >> log_tpp, off = (t & ((1 << log_tpp) - 1)) << 4;
      if (e - win >= 64) window(e);
      const int at = e - win, page = __builtin_amdgcn_readlane(w_log, at);
      const uint64_t where = (uint32_t)__builtin_amdgcn_readlane(w_lo, at) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(w_hi, at) << 32;
      const __amdgpu_buffer_rsrc_t kp = page_buffer(kbase + where, tile_bytes), vp = page_buffer(vbase + where, tile_bytes);
      const int codes = off * (D / 2), scales = first_scale + off;
      t0[i] = page < 0 ? NO_TOKEN : (page << p.log2_p) + off;
      load_tile<D, STREAM>(kp, vp, codes, scales, 0, at_lane, r, i);
      if constexpr (WIDE) {
        t0[1] = t0[0] + 16;
        load_tile<D, STREAM>(kp, vp, codes, scales, 16, at_lane, r, 1);
      }
    }
  };

  auto unit = [&](int number, Raw<D>& raw, const int (&t0)[2]) __attribute__((always_inline)) {
    const bool masked = (WIDE ? t0[1] : max(t0[0], t0[1])) + 15 > min_pos;
    // Tokens that not every row sees.  Their V is zero where nothing of it is seen (it may be anything) and where it is NaN: a
    // weight of zero does not stop a NaN, so the rows that do see it get theirs below.
    bool nan_seen = false;
    if (masked) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = t0[i] + 4 * kg + j;
          const bool partly = t > min_pos, unseen = t > max_pos, bad = ((raw.vs[i] >> (8 * j)) & 255) == 255;
          if (partly && (unseen || bad)) {
            raw.v[i][j] = 0;
            raw.vs[i] = (raw.vs[i] & ~(255u << (8 * j))) | (127u << (8 * j));
          }
          nan_seen |= partly && !unseen && bad;
        }
      }
    }

    // S^T
    f32x4 st[RT][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float ks = kvq_scale(raw.ks[i]);
      uint4 kf[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c)
        kf[c] = make_uint4(cvt2<0>(raw.k[i][c], ks), cvt2<1>(raw.k[i][c], ks), cvt2<2>(raw.k[i][c], ks), cvt2<3>(raw.k[i][c], ks));
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) st[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = QT - 1; t >= 0; --t)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) st[rt][i] = mfma16(kf[c], q[rt][t][c], st[rt][i]);
    }

    float z[RT][8], all[RT];
    auto weights = [&](int rt, float from) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[rt][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[rt][e >> 2][e & 3], scale, -from));
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[rt][e] = t0[e >> 2] + 4 * kg + (e & 3) <= pos[rt] ? z[rt][e] : 0.0f;
      }
      all[rt] = ((z[rt][0] + z[rt][1]) + (z[rt][2] + z[rt][3])) + ((z[rt][4] + z[rt][5]) + (z[rt][6] + z[rt][7]));
    };
    bool up = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      weights(rt, ref[rt]);
      up |= !(all[rt] <= MOST);
    }
    if (__any(up)) {   // (the first unit of a row: its reference is -infinity, so weights are infinite, or NaN where the logit is -infinity too)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool seen = !masked || t0[e >> 2] + 4 * kg + (e & 3) <= pos[rt];
          top = fmaxf(top, seen ? st[rt][e >> 2][e & 3] * scale : -INFINITY);
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
    uint4 pf[RT][PT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      sum[rt] += all[rt];
#pragma unroll
      for (int t = 0; t < PT; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = pack2_bf16(z[rt][2 * e], z[rt][2 * e + 1]);
          if (t + 1 < PT) less(z[rt][2 * e], z[rt][2 * e + 1], w[e]);
        }
        pf[rt][t] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }

    // V: dims 2 x and 2 x + 1 of this lane's; tokens (i, 2 y), (i, 2 y + 1) make word 2 i + y of an operand
    auto add = [&](int j, const uint4& va) __attribute__((always_inline)) {
#pragma unroll
      for (int t = PT - 1; t >= 0; --t)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][j] = mfma16(va, pf[rt][t], acc[rt][j]);
    };
    auto dims = [&](auto sel) __attribute__((always_inline)) {
      constexpr int X = decltype(sel)::value;
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) pairs<X>(raw, i, lo + 2 * i, hi + 2 * i);
      add(2 * X, make_uint4(lo[0], lo[1], lo[2], lo[3]));
      add(2 * X + 1, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    };
    dims(std::integral_constant<int, 0>{});
    dims(std::integral_constant<int, 1>{});
    if constexpr (D == 128) {
      dims(std::integral_constant<int, 2>{});
      dims(std::integral_constant<int, 3>{});
    }

    if (__any(nan_seen)) {
      const int vb = D == 128 ? kg : kg >> 1;      // this lane's output dims are D/4 kg .. + D/4 - 1
      for (int i = 0; i < 2; ++i) {
        const int tile = 2 * number + i, e = tile >> log_tpp, off = (tile & ((1 << log_tpp) - 1)) << 4;
        if (t0[i] >= NO_TOKEN) continue;
        const unsigned char* vs = vbase + (int64_t)page_of(p, b, list ? list[e] : e) * p.pool_page_stride + p.P * (D / 2) + vb * p.P + off;
        for (int t = 0; t < 16; ++t) {
          const int at = t0[i] + t;
          if (at <= min_pos || at > max_pos || vs[t] != 255) continue;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            if (at <= pos[rt]) {
#pragma unroll
              for (int j = 0; j < NJ; ++j) acc[rt][j] = f32x4{NAN, NAN, NAN, NAN};
            }
        }
      }
    }
  };

  // units in flight: a wave that waits for its next unit idles its share of the memory's latency (about a microsecond)
  constexpr int AHEAD = 2;
  Raw<D> raw[AHEAD];
  int t0[AHEAD][2];
  // The wait for a unit lets every later fetch fly on, if the compiler can count them: the steady loop fetches without a condition,
  // and the queries have landed before it.
  if (u < u_end) window((2 * u) >> log_tpp);
  if (u + 2 * AHEAD <= u_end) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(u + k, raw[k], t0[k]);
    landed(q);
    for (; u + 2 * AHEAD <= u_end; u += AHEAD) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        unit(u + k, raw[k], t0[k]);
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
      unit(u + k, raw[k], t0[k]);
      if (u + k + AHEAD < u_end) fetch(u + k + AHEAD, raw[k], t0[k]);
    }
  }

  // lane (m, kg): query m, dims D/4 kg + D/16 i + j of acc[.][j][i]
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] += __shfl_xor(sum[rt], 16, 64);
    sum[rt] += __shfl_xor(sum[rt], 32, 64);
  }
  auto put = [&](int r, int d, const float* y, float ref_r, float sum_r, bool first) __attribute__((always_inline)) {   // four dims of row r of the block
    const int row = r0 + r;
    if (row >= n_rows) return;
    if (part.count > 1) {
      const int64_t at = (int64_t)blockIdx.x * ROWS + r;
      *reinterpret_cast<float4*>(a.part + at * D + d) = make_float4(y[0], y[1], y[2], y[3]);
      if (first) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(ref_r, sum_r);
      return;
    }
    const int i = row / p.G, h = g * p.G + (row - i * p.G);
    const float f = sum_r == 0.0f ? 0.0f : 1.0f / sum_r;
    T* dst = (T*)p.q_out.data + (int64_t)(s.row + i) * p.q_out.tok_stride + (int64_t)h * p.q_out.head_stride + d;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2_bf16(y[0] * f, y[1] * f), pack2_bf16(y[2] * f, y[3] * f));
    else *reinterpret_cast<float4*>(dst) = make_float4(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
    if (first) p.lse[(int64_t)h * p.n_rows + s.row + i] = sum_r == 0.0f ? -INFINITY : (ref_r + __builtin_amdgcn_logf(sum_r)) * LN2;
  };

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
    float* mine = merge + (wave * 16 + m) * (D + PAD) + (D / 4) * kg;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; j += 4)
        *reinterpret_cast<float4*>(mine + NJ * i + j) = make_float4(acc[rt][j][i] * f, acc[rt][j + 1][i] * f, acc[rt][j + 2][i] * f, acc[rt][j + 3][i] * f);
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
      put(16 * rt + r, d, y, ref_r, sum_r, d == 0);
    }
  }
}

// The parts of a row, in order: a workgroup per row of a row block and slice of DW dims, its threads in groups of DW / 4 that take every
// (256 / (DW / 4))-th part each.  A compute unit takes in about 10 B/ns of lines that others wrote, so a few rows of many parts go in slices of a
// line (7 x 4 rows of 127 parts: 10.3 us whole).
template <typename T, int D, int DW>
__global__ __launch_bounds__(COMBINE_THREADS) void kvq_combine_kernel(RowsParams p, AttnArgs a, int block_rows, int rows) {   // rows: of a block that there can be at most
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

// How a call is cut.
struct Plan {
  int rt, waves, stream, row_blocks, split, target, min_units;
  int64_t parts;   // at most
};
Plan plan_of(const RowsParams& p, bool is_bf16, int32_t sel_stride) {
  Plan c{};
  const int64_t rows = (int64_t)p.max_rows * p.G, heads = (int64_t)p.n_seqs * p.Hkv;
  c.rt = rows <= 16 || (!is_bf16 && p.D == 128) ? 1 : 2;   // (fp32 terms of two row tiles at head dim 128 do not fit the registers)
  c.row_blocks = (int)((rows + 16 * c.rt - 1) / (16 * c.rt));
  int64_t tokens = p.max_len;
  if (sel_stride >= 0 && (int64_t)sel_stride * p.P < tokens) tokens = (int64_t)sel_stride * p.P;
  const int64_t units = (tokens + 31) / 32;
  // A part's sums are written and read again, which takes as long as a few units: eight of a row tile at head dim 128.
  const int least = c.rt * p.D / 16 < 8 ? 8 : c.rt * p.D / 16;
  c.min_units = least;
  const int64_t each = (units + c.min_units - 1) / c.min_units;
  // Up to 40 units eight waves without a second launch are faster (1000 tokens: 9.4 us, 10.5 in parts; 2000: 13.4, 10.7).  A lone row block
  // is cut in any case: the lengths of many sequences may differ (32 of 1 to 32K tokens: 25 us, 127 whole).  Several are cut
  // where they leave workgroups idle (1024 rows x 7 over 8K tokens, 896 workgroups: 148 us, 170 in parts).
  // (the parts may be `heads` more than the target: kept within what the chip holds at once, as far as that leaves half of it)
  const int64_t room = WGS / c.row_blocks, aim = room - heads > room / 2 ? room - heads : room / 2;
  const int64_t target = c.row_blocks == 1 && aim < 2 * heads ? 2 * heads : aim;
  c.split = units > 40 && each > 1 && target >= 2 * heads;
  c.target = (int)(target < 1 ? 1 : target);
  c.parts = !c.split ? heads : heads * each < target + heads ? heads * each : target + heads;
  c.waves = c.split || (is_bf16 && rows > 64) ? 4 : 8;   // (4096 rows over 16K tokens: eight waves 1270 us, four 1176; 64 rows of 7 heads: 39.8, 41.0)
  // Codes past the caches once they would not stay in the last one (256 MiB) to the next call: 570 MB 117 -> 105 us, 62 MB 22.0 -> 23.6
  // (bf16 rows of head dim 128, where both were timed; the other forms are without it).  What is read is bounded by the lengths' bound and by the
  // pools: a batch whose bound alone is large (32 sequences of up to 32K tokens, 570 MB, that hold 62) goes by its pools, and one of short sequences
  // in large pools under a large bound loses the 7 %.
  const int64_t reach = heads * tokens, held = p.num_phys * p.Hkv * p.P;
  c.stream = (reach < held ? reach : held) * 2 * (p.D / 2 + p.D / 32) > (256ll << 20);
  return c;
}
// Rows that the combine has a workgroup for, and its workgroups (before slices, which only a few rows have); it runs where c.split.
int combine_rows(const RowsParams& p, const Plan& c) { return c.row_blocks == 1 ? p.max_rows * p.G : 16 * c.rt; }
int64_t combine_blocks(const RowsParams& p, const Plan& c) { return (int64_t)p.n_seqs * p.Hkv * c.row_blocks * combine_rows(p, c); }

template <typename T, int D, int RT, int W, bool WIDE, bool STREAM> hipError_t run(const RowsParams& p, const Plan& c, void* ws, hipStream_t st) {
  AttnArgs a{c.row_blocks, c.split, c.target, c.min_units, nullptr, nullptr, nullptr};
  const int64_t heads = (int64_t)p.n_seqs * p.Hkv, blocks = c.parts * c.row_blocks;
  if (c.split) {
    a.part = (float*)ws;
    a.part_ml = a.part + blocks * 16 * RT * D;
    a.parts = (int2*)(a.part_ml + blocks * 16 * RT * 2);
  }
  {
    ProfScope prof_("attn_kvq", st);
    constexpr size_t lds = (size_t)(W * 16 * (D + PAD) + W * 16 * 2) * sizeof(float);
    const auto kernel = attn_kvq_kernel<T, D, RT, W, WIDE, STREAM>;
    if (lds > 65536) {
      static DeviceOnce once;
      const hipError_t e = ensure_max_dynamic_lds(once, (const void*)kernel, (int)lds);
      if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)blocks), dim3(64 * W), lds, st>>>(p, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !c.split) return e;
  }
  ProfScope prof_("kvq_combine", st);
  const int rows = combine_rows(p, c);
  const int64_t wgs = combine_blocks(p, c);
  if (wgs < 256 && c.parts > 32 * heads) kvq_combine_kernel<T, D, 32><<<dim3((unsigned)(wgs * (D / 32))), dim3(COMBINE_THREADS), 0, st>>>(p, a, 16 * RT, rows);
  else kvq_combine_kernel<T, D, D><<<dim3((unsigned)wgs), dim3(COMBINE_THREADS), 0, st>>>(p, a, 16 * RT, rows);
  return hipGetLastError();
}
template <typename T, int D, int RT, int W> hipError_t run(const RowsParams& p, const Plan& c, void* ws, hipStream_t st) {
  if (p.P < 32) return run<T, D, RT, W, false, false>(p, c, ws, st);
  if constexpr (RT == 1 && W == 4 && D == 128 && sizeof(T) == 2) {
    if (c.stream) return run<T, D, RT, W, true, true>(p, c, ws, st);
  }
  return run<T, D, RT, W, true, false>(p, c, ws, st);
}
template <typename T, int D, int RT> hipError_t run(const RowsParams& p, const Plan& c, void* ws, hipStream_t st) {
  return c.waves == 8 ? run<T, D, RT, 8>(p, c, ws, st) : run<T, D, RT, 4>(p, c, ws, st);
}
// (instantiated for one type and head dim per source file, which are compiled side by side)
template <typename T, int D> hipError_t attn(const RowsParams& p, void* ws, hipStream_t st) {
  const Plan c = plan_of(p, sizeof(T) == 2, p.sel ? p.sel_stride : -1);
  if constexpr (sizeof(T) == 2 || D == 64) {
    if (c.rt == 2) return run<T, D, 2>(p, c, ws, st);
  }
  return run<T, D, 1>(p, c, ws, st);
}

}  // namespace
}  // namespace oomb
