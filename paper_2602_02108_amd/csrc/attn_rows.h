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
// device from the lengths as they are, and rows_combine adds a row's parts in their order.
#pragma once
#include <type_traits>

#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "rows.h"
#include "rows_parts.h"

namespace oomb {

namespace {

constexpr int WGS = 512;                 // workgroups that a call is cut into

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

__device__ __forceinline__ f32x4 mfma4(uint32_t a, uint32_t b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16v(const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// whether a half (of a word of two bf16) or a float is an infinity or a NaN
__device__ __forceinline__ bool wild16(uint32_t w, int half) { return ((half ? w >> 16 : w) & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool wild32(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }

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

// WIDE: pages of 32 tokens and more, a step lies in one (fp32: always).  STREAM: the cache is read past the caches.
template <typename T, int D, int RT, int W, bool WIDE, bool STREAM>
__global__ __launch_bounds__(64 * W, 2) void attn_rows_kernel(RowsParams p, AttnArgs a) {
  extern __shared__ __align__(16) float merge[];
  using S = Shape<T, D>;
  constexpr int TILES = S::TILES, KC = S::KC, VW = S::VW, NJ = S::NJ, NZ = S::NZ, ES = S::ES, ROWS = 16 * RT;
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
  const int n_steps = (n_tiles + TILES - 1) / TILES;
  const int parts = part.count * W, mine = part.index * W + wave;
  const int each = (int)((uint32_t)n_steps / (uint32_t)parts), more = n_steps - each * parts;   // (one more for the first `more`)
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
    const uint64_t at = (uint64_t)max(phys, 0) * (uint64_t)p.pool_page_stride * ES;
    w_lo = (uint32_t)at;
    w_hi = (uint32_t)(at >> 32);
  };
  const unsigned char* kbase = (const unsigned char*)p.k_pool + (int64_t)g * p.pool_head_stride * ES;
  const unsigned char* vbase = (const unsigned char*)p.v_pool + (int64_t)g * p.pool_head_stride * ES;
  const int tok = (int)p.pool_tok_stride * ES, page_bytes = (p.P - 1) * tok + D * ES;
  const uint32_t k_lane = (uint32_t)(m * tok + 16 * kg), v_lane = (uint32_t)(4 * kg * tok + m * (4 * VW));
  auto fetch = [&](int step, Raw<T, D>& r, int (&t0)[TILES]) __attribute__((always_inline)) {   // t0: positions of the tiles' first tokens
#pragma unroll
    for (int i = 0; i < (WIDE ? 1 : TILES); ++i) {
      const int t = TILES * step + i, e = t >> log_tpp, off = (t & ((1 << log_tpp) - 1)) << 4;
      if (e - win >= 64) window(e);
      const int at = e - win, page = __builtin_amdgcn_readlane(w_log, at);
      const uint64_t where = (uint32_t)__builtin_amdgcn_readlane(w_lo, at) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(w_hi, at) << 32;
      const __amdgpu_buffer_rsrc_t kp = page_buffer(kbase + where, page_bytes), vp = page_buffer(vbase + where, page_bytes);
      t0[i] = page < 0 ? NO_TOKEN : (page << p.log2_p) + off;
      load_tile<T, D, STREAM>(kp, vp, off * tok, tok, k_lane, v_lane, r, i);
      if constexpr (WIDE && TILES == 2) {
        t0[1] = t0[0] + 16;
        load_tile<T, D, STREAM>(kp, vp, (off + 16) * tok, tok, k_lane, v_lane, r, 1);
      }
    }
  };

  auto one_step = [&](int number, Raw<T, D>& raw, const int (&t0)[TILES]) __attribute__((always_inline)) {
    const bool masked = (TILES == 1 ? t0[0] : WIDE ? t0[TILES - 1] : max(t0[0], t0[TILES - 1])) + 15 > min_pos;
    // Tokens that not every row sees.  Their V is zero where nothing of it is seen (it may be anything), and so are their values that are not
    // finite: a weight of zero does not stop those, so the rows that do see them get them below.
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
            st[rt][i] = mfma16v(raw.k[i][c], q[rt][c], st[rt][i]);
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
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sum[rt] += all[rt];

    if constexpr (S::BF) {
      uint4 pf[RT][2];
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
          pf[rt][t] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      // V: word x holds dims 2 x and 2 x + 1 of this lane's; tokens (i, 2 y), (i, 2 y + 1) make word 2 i + y of an operand
#pragma unroll
      for (int x = 0; x < VW; ++x) {
        uint4 lo, hi;
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

    if (__any(wild)) {   // values that are not finite, to the rows that see them: lane (m, kg) holds dims D/4 kg + D/16 i + j of query m in acc[.][j][i]
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int tile = TILES * number + i, e = tile >> log_tpp, off = (tile & ((1 << log_tpp) - 1)) << 4;
        if (t0[i] >= NO_TOKEN) continue;
        const unsigned char* page = vbase + (int64_t)page_of(p, b, list ? list[e] : e) * p.pool_page_stride * ES;
        for (int t = 0; t < 16; ++t) {
          const int at = t0[i] + t;
          if (at <= min_pos || at > max_pos) continue;
          const T* v = reinterpret_cast<const T*>(page + (int64_t)(off + t) * tok) + kg * (D / 4);
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
              const float y = Elem<T>::load(v + NJ * x + j);
              const bool bad = wild32(__float_as_uint(y));
#pragma unroll
              for (int rt = 0; rt < RT; ++rt)
                if (bad && at <= pos[rt]) acc[rt][j][x] += y;
            }
        }
      }
    }
  };

  // steps in flight: a wave that waits for its next one idles its share of the memory's latency (about a microsecond)
  constexpr int AHEAD = 2;
  Raw<T, D> raw[AHEAD];
  int t0[AHEAD][TILES];
  // The wait for a step lets every later fetch fly on, if the compiler can count them: the steady loop fetches without a condition,
  // and the queries have landed before it.
  if (u < u_end) window((TILES * u) >> log_tpp);
  if (u + 2 * AHEAD <= u_end) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(u + k, raw[k], t0[k]);
    queries_landed(q);
    for (; u + 2 * AHEAD <= u_end; u += AHEAD) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        one_step(u + k, raw[k], t0[k]);
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
      one_step(u + k, raw[k], t0[k]);
      if (u + k + AHEAD < u_end) fetch(u + k + AHEAD, raw[k], t0[k]);
    }
  }

  // lane (m, kg): query m, dims D/4 kg + D/16 i + j of acc[.][j][i]
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
      if (part.count > 1) {
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

// How a call is cut.
struct Plan {
  int rt, waves, stream, row_blocks, split, target, min_units;
  int64_t parts;   // at most
};
Plan plan_of(const RowsParams& p, bool is_bf16, int32_t sel_stride) {
  Plan c{};
  const int64_t rows = (int64_t)p.max_rows * p.G, heads = (int64_t)p.n_seqs * p.Hkv;
  c.rt = rows <= 16 || p.D == 128 ? 1 : 2;
  c.row_blocks = (int)((rows + 16 * c.rt - 1) / (16 * c.rt));
  int64_t tokens = p.max_len;
  if (sel_stride >= 0 && (int64_t)sel_stride * p.P < tokens) tokens = (int64_t)sel_stride * p.P;
  const int64_t units = (tokens + 31) / 32;
  c.min_units = 8;
  const int64_t each = (units + c.min_units - 1) / c.min_units;
  const int64_t room = WGS / c.row_blocks, aim = room - heads > room / 2 ? room - heads : room / 2;
  const int64_t target = c.row_blocks <= 4 && aim < 2 * heads ? 2 * heads : aim;
  c.split = units > 16 && each > 1 && target >= 2 * heads;
  c.target = (int)(target < 1 ? 1 : target);
  c.parts = !c.split ? heads : heads * each < target + heads ? heads * each : target + heads;
  c.waves = c.split || (is_bf16 && rows > 64) ? 4 : 8;
  const int64_t reach = heads * tokens, held = p.num_phys * p.Hkv * p.P;
  c.stream = (reach < held ? reach : held) * 2 * p.D * (is_bf16 ? 2 : 4) > (256ll << 20);
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
    ProfScope prof_("attn_rows", st);
    constexpr size_t lds = (size_t)(W * 16 * (D + PAD) + W * 16 * 2) * sizeof(float);
    const auto kernel = attn_rows_kernel<T, D, RT, W, WIDE, STREAM>;
    if (lds > 65536) {
      static DeviceOnce once;
      const hipError_t e = ensure_max_dynamic_lds(once, (const void*)kernel, (int)lds);
      if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)blocks), dim3(64 * W), lds, st>>>(p, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !c.split) return e;
  }
  ProfScope prof_("rows_combine", st);
  const int rows = combine_rows(p, c);
  const int64_t wgs = combine_blocks(p, c);
  if (wgs < 256 && c.parts > 32 * heads) rows_combine_kernel<T, D, 32><<<dim3((unsigned)(wgs * (D / 32))), dim3(COMBINE_THREADS), 0, st>>>(p, a, 16 * RT, rows);
  else rows_combine_kernel<T, D, D><<<dim3((unsigned)wgs), dim3(COMBINE_THREADS), 0, st>>>(p, a, 16 * RT, rows);
  return hipGetLastError();
}
template <typename T, int D, int RT, int W> hipError_t run(const RowsParams& p, const Plan& c, void* ws, hipStream_t st) {
  if (sizeof(T) == 2 && p.P < 32) return run<T, D, RT, W, sizeof(T) != 2, false>(p, c, ws, st);
  if constexpr (RT == 1 && W == 4) {
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
  if constexpr (D == 64) {
    if (c.rt == 2) return run<T, D, 2>(p, c, ws, st);
  }
  return run<T, D, 1>(p, c, ws, st);
}

}  // namespace
}  // namespace oomb
