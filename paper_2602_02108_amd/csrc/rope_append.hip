// Rows on their way into the paged cache with the position rotation applied, into pools of their type or of 4-bit codes; the
// backward of the former; and the values of rows that a 4-bit cache holds.
//
// A row of a head is cut into units of 16 dims that a thread turns by 8 angles: unit u of a rotated row holds dims 8 u .. 8 u + 7 and
// rot_dim / 2 + 8 u .. + 7 (pairs in halves) or 16 u .. 16 u + 15 (neighbours), angles 8 u .. 8 u + 7 either way; a unit past rot_dim
// holds dims 16 u .. 16 u + 15 as they are.  So every access is 16 bytes of one row and a rotation never leaves its thread.
//
// One launch: the first workgroups take the K or V rows that fall into one page of one KV head, the others the queries.
#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "rows.h"
#include "rowsum.h"

#pragma clang fp contract(off)

namespace oomb {

namespace {

constexpr int THREADS = 256;
constexpr int UNIT = 16;

struct UnitAt { int lo, hi, angle; bool turns; };   // first dims of the halves of a unit, its first angle
__device__ __forceinline__ UnitAt unit_at(const RowsParams& p, int u) {
  if (u * UNIT >= p.rot_dim) return {u * UNIT, u * UNIT + 8, 0, false};
  if (p.interleaved) return {u * UNIT, u * UNIT + 8, 8 * u, true};
  return {8 * u, p.rot_dim / 2 + 8 * u, 8 * u, true};
}

template <typename T> __device__ __forceinline__ void load8(const T* src, float* x) {
  if constexpr (sizeof(T) == 2) {
    Vec16<T>::unpack(*reinterpret_cast<const uint4*>(src), x);
  } else {
    Vec16<T>::unpack(reinterpret_cast<const uint4*>(src)[0], x);
    Vec16<T>::unpack(reinterpret_cast<const uint4*>(src)[1], x + 4);
  }
}
template <typename T> __device__ __forceinline__ void store8(T* dst, const float* x) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]), pack2_bf16(x[4], x[5]), pack2_bf16(x[6], x[7]));
  } else {
    reinterpret_cast<float4*>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}
__device__ __forceinline__ void load_angles(const RowsParams& p, int pos, const UnitAt& a, float* c, float* s) {
  const int64_t at = (int64_t)pos * (p.rot_dim / 2) + a.angle;
  load8(p.cos + at, c);
  load8(p.sin + at, s);
}

// y1 = x1 c - x2 s, y2 = x2 c + x1 s; back: by the opposite angle
template <bool BACK> __device__ __forceinline__ void turn1(float& x1, float& x2, float c, float s) {
  const float a = x1, b = x2;
  if (BACK) s = -s;
  x1 = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  x2 = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
}
template <bool BACK> __device__ __forceinline__ void turn(const RowsParams& p, float* x, const float* c, const float* s) {
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn1<BACK>(x[2 * i], x[2 * i + 1], c[i], s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn1<BACK>(x[i], x[8 + i], c[i], s[i]);
  }
}

// A double rounded to float, to nearest -- or to odd, which keeps every comparison with a value of fewer than 24 bits: that is
// how a rotated key is quantised as if from 64 bits.
template <bool ODD> __device__ __forceinline__ float narrow(double x) {
  float f = (float)x;
  if (ODD) {
    const double d = (double)f;
    if (d != x && x == x) {
      uint32_t b = __float_as_uint(f);
      if (fabs(d) > fabs(x)) --b;
      f = __uint_as_float(b | 1);
    }
  }
  return f;
}
// The products of a 24-bit value and a 24-bit cosine are exact in 64 bits.  A key's rounding decides what is kept of it, a code or
// a bit of its type, so it is made from the right number; the few operations are hidden behind the row's loads.
template <bool ODD> __device__ __forceinline__ void turn1_wide(float& x1, float& x2, float c, float s) {
  const double a = x1, b = x2;
  x1 = narrow<ODD>(a * c - b * s);
  x2 = narrow<ODD>(b * c + a * s);
}
template <bool ODD> __device__ __forceinline__ void turn_wide(const RowsParams& p, float* x, const float* c, const float* s) {
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn1_wide<ODD>(x[2 * i], x[2 * i + 1], c[i], s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn1_wide<ODD>(x[i], x[8 + i], c[i], s[i]);
  }
}

// The tokens of one page that are new rows of one KV head, and where they lie.
struct Span {
  int b, g, page;      // sequence, KV head, logical page
  int first, last;     // positions [first, last)
  int32_t row, phys;   // row of `first`
};
__device__ __forceinline__ bool span_of(const RowsParams& p, int x, Span& s) {
  const int slots = pages_touched(p.max_rows, p.P);
  s.g = x % p.Hkv;
  x /= p.Hkv;
  const int slot = x % slots;
  s.b = x / slots;
  const Seq q = seq_of(p, s.b);
  const int from = max(q.pos, 0), to = q.pos + q.n;
  s.page = (from >> p.log2_p) + slot;
  s.first = max(from, s.page << p.log2_p);
  s.last = min(to, (s.page + 1) << p.log2_p);
  if (s.first >= s.last) return false;
  s.row = q.row + (s.first - q.pos);
  s.phys = page_of(p, s.b, s.page);
  return true;
}

// ---- queries: a thread takes one unit of one row for `heads` heads, so that its angles are loaded once --------------------
template <typename T, int D, bool BACK>
__device__ __forceinline__ void turn_queries(const RowsParams& p, int x, int blocks_per_seq, int heads) {
  constexpr int U = D / UNIT;
  const int b = x / blocks_per_seq;
  const int groups = (p.Hq + heads - 1) / heads;
  const int64_t at = (int64_t)(x - b * blocks_per_seq) * THREADS + threadIdx.x;
  const int u = (int)(at % U);
  const int64_t y = at / U;
  const int i = (int)(y / groups), h0 = (int)(y - (int64_t)i * groups) * heads;
  const Seq s = seq_of(p, b);
  const int pos = s.pos + i;
  if (i >= s.n || pos < 0) return;
  const UnitAt a = unit_at(p, u);
  float c[8], sn[8];
  if (a.turns) load_angles(p, pos, a, c, sn);
  const T* src = (const T*)p.q.data + (int64_t)(s.row + i) * p.q.tok_stride;
  T* dst = (T*)p.q_out.data + (int64_t)(s.row + i) * p.q_out.tok_stride;
  const int h1 = min(h0 + heads, p.Hq);
  float v[4][16];   // (four rows' loads in flight)
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const T* r = src + (int64_t)min(h0 + k, h1 - 1) * p.q.head_stride;
    load8(r + a.lo, v[k]);
    load8(r + a.hi, v[k] + 8);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (h0 + k >= h1) break;
    if (a.turns) turn<BACK>(p, v[k], c, sn);
    T* r = dst + (int64_t)(h0 + k) * p.q_out.head_stride;
    store8(r + a.lo, v[k]);
    store8(r + a.hi, v[k] + 8);
  }
}

// ---- keys and values into pools of the rows' type: a workgroup takes four units (64 dims) of its span ------------------
// Means: the page's keys in LDS (those before the new rows from the pool), then a thread per dim or two walks them in order.
template <typename T, int D>
__device__ __forceinline__ void append_page(const RowsParams& p, int x) {
  extern __shared__ __align__(16) unsigned char lds[];
  constexpr int SL = D / 64, U = 4;
  const int slice = x % SL;
  x /= SL;
  const bool keys = (x & 1) == 0;
  Span s;
  if (!span_of(p, x >> 1, s)) return;
  const oomb_rows& rows = keys ? p.k : p.v;
  const T* src = (const T*)rows.data + (int64_t)s.row * rows.tok_stride + (int64_t)s.g * rows.head_stride;
  // (a page that is not there is found out at the first store: the rows' loads do not wait for its number)
  T* pool = (T*)(keys ? p.k_pool : p.v_pool) + (int64_t)s.phys * p.pool_page_stride + (int64_t)s.g * p.pool_head_stride;
  const int t0 = s.page << p.log2_p, tid = threadIdx.x;
  const int ul = tid & (U - 1);
  const UnitAt a = unit_at(p, slice * U + ul);
  const bool turns = keys && a.turns;
  const bool sums = keys && p.kbar && s.last == t0 + p.P;
  T* tile = reinterpret_cast<T*>(lds);
  auto put = [&](int t, const float* v) __attribute__((always_inline)) {
    T* r = tile + (t - t0) * 64 + ul * UNIT;
    store8(r, v);
    store8(r + 8, v + 8);
  };
  for (int t = s.first + (tid >> 2); t < s.last; t += 2 * (THREADS / U)) {
    float v[2][16], c[2][8], sn[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tk = min(t + k * (THREADS / U), s.last - 1);
      const T* r = src + (int64_t)(tk - s.first) * rows.tok_stride;
      load8(r + a.lo, v[k]);
      load8(r + a.hi, v[k] + 8);
      if (turns) load_angles(p, tk, a, c[k], sn[k]);
    }
    if (s.phys < 0) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tk = t + k * (THREADS / U);
      if (tk >= s.last) break;
      if (turns) turn_wide<false>(p, v[k], c[k], sn[k]);
      T* r = pool + (int64_t)(tk - t0) * p.pool_tok_stride;
      store8(r + a.lo, v[k]);
      store8(r + a.hi, v[k] + 8);
      if (sums) put(tk, v[k]);
    }
  }
  if (!sums || s.phys < 0) return;
  if (t0 + (tid >> 2) < s.first) {   // (a page has 128 tokens at most: two a thread)
    float v[2][16];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const T* r = pool + (int64_t)(min(t0 + (tid >> 2) + k * (THREADS / U), s.first - 1) - t0) * p.pool_tok_stride;
      load8(r + a.lo, v[k]);
      load8(r + a.hi, v[k] + 8);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) put(min(t0 + (tid >> 2) + k * (THREADS / U), s.first - 1), v[k]);
  }
  __syncthreads();
  float* out = p.kbar + (((int64_t)s.b * p.table_stride + s.page) * p.Hkv + s.g) * D;
  lds_row_sum<T, 64>(p.P, lds, [&](int d, float sum) __attribute__((always_inline)) {
    const UnitAt w = unit_at(p, slice * U + d / UNIT);
    const int e = d % UNIT;
    out[e < 8 ? w.lo + e : w.hi + e - 8] = __fmul_rn(sum, 1.0f / (float)p.P);
  });
}

// ---- keys and values into pools of 4-bit codes: a workgroup takes whole rows, the units of a row lie in neighbouring lanes ----
__device__ __forceinline__ uint32_t codes8(const float* x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}
// the eight values of a word of codes, in bf16 (exact)
__device__ __forceinline__ uint4 values8(uint32_t codes, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}

template <typename T, int D>
__device__ __forceinline__ void append_page_kvq(const RowsParams& p, int x) {
  extern __shared__ __align__(16) unsigned char lds[];
  constexpr int U = D / UNIT, NB = D / 32, TOK = THREADS / U;
  const bool keys = (x & 1) == 0;
  Span s;
  if (!span_of(p, x >> 1, s)) return;
  const oomb_rows& rows = keys ? p.k : p.v;
  const T* src = (const T*)rows.data + (int64_t)s.row * rows.tok_stride + (int64_t)s.g * rows.head_stride;
  unsigned char* tile = (unsigned char*)(keys ? p.k_pool : p.v_pool) + (int64_t)s.phys * p.pool_page_stride + (int64_t)s.g * p.pool_head_stride;
  unsigned char* scales = tile + p.P * (D / 2);
  const int t0 = s.page << p.log2_p, tid = threadIdx.x, u = tid & (U - 1);
  UnitAt a = unit_at(p, u);
  if (!keys) a = {u * UNIT, u * UNIT + 8, 0, false};
  const bool sums = keys && p.kbar && s.last == t0 + p.P;
  bf16_t* held = reinterpret_cast<bf16_t*>(lds);
  auto put = [&](int t, uint32_t lo, uint32_t hi, float slo, float shi) __attribute__((always_inline)) {
    bf16_t* r = held + (t - t0) * D;
    *reinterpret_cast<uint4*>(r + a.lo) = values8(lo, slo);
    *reinterpret_cast<uint4*>(r + a.hi) = values8(hi, shi);
  };
  // (lanes past the last token go along with the last one's values: every lane takes part in the exchange of maxima)
  for (int tb = s.first; tb < s.last; tb += 2 * TOK) {
    float v[2][16], c[2][8], sn[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tk = min(tb + tid / U + k * TOK, s.last - 1);
      const T* r = src + (int64_t)(tk - s.first) * rows.tok_stride;
      load8(r + a.lo, v[k]);
      load8(r + a.hi, v[k] + 8);
      if (a.turns) load_angles(p, tk, a, c[k], sn[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tk = tb + tid / U + k * TOK;
      if (a.turns) turn_wide<true>(p, v[k], c[k], sn[k]);
      uint32_t mlo = 0, mhi = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mlo = max(mlo, __float_as_uint(v[k][i]) & 0x7fffffffu);
        mhi = max(mhi, __float_as_uint(v[k][8 + i]) & 0x7fffffffu);
      }
      uint32_t top[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) top[j] = max(a.lo / 32 == j ? mlo : 0u, a.hi / 32 == j ? mhi : 0u);
#pragma unroll
      for (int w = 1; w < U; w *= 2) {
#pragma unroll
        for (int j = 0; j < NB; ++j) top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], w, 64));
      }
      uint32_t blo = 0, bhi = 0, mine = 0;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const uint32_t y = kvq_scale_byte(top[j]);
        if (a.lo / 32 == j) blo = y;
        if (a.hi / 32 == j) bhi = y;
        if (u == j) mine = y;
      }
      if (tk >= s.last || s.phys < 0) continue;
      const uint32_t lo = blo == 255 ? 0 : codes8(v[k], kvq_scale(blo)), hi = bhi == 255 ? 0 : codes8(v[k] + 8, kvq_scale(bhi));
      unsigned char* r = tile + (tk - t0) * (D / 2);
      *reinterpret_cast<uint32_t*>(r + a.lo / 2) = lo;
      *reinterpret_cast<uint32_t*>(r + a.hi / 2) = hi;
      if (u < NB) scales[u * p.P + (tk - t0)] = (unsigned char)mine;
      if (sums) put(tk, lo, hi, kvq_scale(blo), kvq_scale(bhi));
    }
  }
  if (!sums || s.phys < 0) return;
  if (t0 + tid / U < s.first) {   // (a page has 128 tokens at most)
    constexpr int K = 128 / TOK;
    uint32_t lo[K], hi[K];
    unsigned char slo[K], shi[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int at = min(t0 + tid / U + k * TOK, s.first - 1) - t0;
      const unsigned char* r = tile + at * (D / 2);
      lo[k] = *reinterpret_cast<const uint32_t*>(r + a.lo / 2);
      hi[k] = *reinterpret_cast<const uint32_t*>(r + a.hi / 2);
      slo[k] = scales[(a.lo / 32) * p.P + at];
      shi[k] = scales[(a.hi / 32) * p.P + at];
    }
#pragma unroll
    for (int k = 0; k < K; ++k) put(min(t0 + tid / U + k * TOK, s.first - 1), lo[k], hi[k], kvq_scale(slo[k]), kvq_scale(shi[k]));
  }
  __syncthreads();
  float* out = p.kbar + (((int64_t)s.b * p.table_stride + s.page) * p.Hkv + s.g) * D;
  lds_row_sum<bf16_t, D>(p.P, lds, [&](int d, float sum) __attribute__((always_inline)) { out[d] = __fmul_rn(sum, 1.0f / (float)p.P); });
}

template <typename T, int D, bool KVQ>
__global__ __launch_bounds__(THREADS) void append_rope_kernel(RowsParams p, int page_blocks, int blocks_per_seq, int heads) {
  const int x = blockIdx.x;
  if (x >= page_blocks) return turn_queries<T, D, false>(p, x - page_blocks, blocks_per_seq, heads);
  if constexpr (KVQ) append_page_kvq<T, D>(p, x);
  else append_page<T, D>(p, x);
}

// ---- backward: the rows' gradients out of the pools ---------------------------------------------------------------------
template <typename T, typename GT, int D>
__device__ __forceinline__ void gather_page(const RowsParams& p, int x) {
  constexpr int SL = D / 64, U = 4;
  const int slice = x % SL;
  x /= SL;
  const bool keys = (x & 1) == 0;
  Span s;
  if (!span_of(p, x >> 1, s)) return;
  const oomb_rows& rows = keys ? p.k : p.v;
  T* dst = (T*)rows.data + (int64_t)s.row * rows.tok_stride + (int64_t)s.g * rows.head_stride;
  const GT* pool = (const GT*)(keys ? p.k_pool : p.v_pool) + (int64_t)max(s.phys, 0) * p.pool_page_stride + (int64_t)s.g * p.pool_head_stride;
  const int t0 = s.page << p.log2_p, tid = threadIdx.x;
  const UnitAt a = unit_at(p, slice * U + (tid & (U - 1)));
  const bool turns = keys && a.turns;
  for (int t = s.first + (tid >> 2); t < s.last; t += 2 * (THREADS / U)) {
    float v[2][16], c[2][8], sn[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tk = min(t + k * (THREADS / U), s.last - 1);
      const GT* r = pool + (int64_t)(tk - t0) * p.pool_tok_stride;
      load8(r + a.lo, v[k]);
      load8(r + a.hi, v[k] + 8);
      if (turns) load_angles(p, tk, a, c[k], sn[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tk = t + k * (THREADS / U);
      if (tk >= s.last) break;
      if (turns) turn<true>(p, v[k], c[k], sn[k]);
      if (s.phys < 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[k][i] = 0.0f;
      }
      T* r = dst + (int64_t)(tk - s.first) * rows.tok_stride;
      store8(r + a.lo, v[k]);
      store8(r + a.hi, v[k] + 8);
    }
  }
}
template <typename T, typename GT, int D>
__global__ __launch_bounds__(THREADS) void append_rope_bwd_kernel(RowsParams p, int page_blocks, int blocks_per_seq, int heads) {
  const int x = blockIdx.x;
  if (x >= page_blocks) turn_queries<T, D, true>(p, x - page_blocks, blocks_per_seq, heads);
  else gather_page<T, GT, D>(p, x);
}

// ---- values of rows in a 4-bit cache: a thread per 8 dims of a row (a word of codes, neighbouring lanes store neighbouring
// words; 32 dims to a thread took 10.5 us for 8192 rows of 8 heads), key heads first -----------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void kvq_read_kernel(RowsParams p, int blocks_per_seq) {
  constexpr int NW = D / 8;
  const int b = blockIdx.x / blocks_per_seq;
  const int64_t at = (int64_t)(blockIdx.x - b * blocks_per_seq) * THREADS + threadIdx.x;
  const int j = (int)(at % NW);
  const int64_t y = at / NW;
  const int i = (int)(y / (2 * p.Hkv)), w = (int)(y - (int64_t)i * 2 * p.Hkv), g = w >= p.Hkv ? w - p.Hkv : w;
  const Seq s = seq_of(p, b);
  const int pos = s.pos + i;
  if (i >= s.n || pos < 0) return;
  const int32_t phys = page_of(p, b, pos >> p.log2_p);
  const int slot = pos & (p.P - 1);
  const oomb_rows& rows = w >= p.Hkv ? p.v : p.k;
  T* dst = (T*)rows.data + (int64_t)(s.row + i) * rows.tok_stride + (int64_t)g * rows.head_stride + 8 * j;
  uint32_t codes = 0, byte = 127;
  if (phys >= 0) {
    const unsigned char* tile = (const unsigned char*)(w >= p.Hkv ? p.v_pool : p.k_pool) + (int64_t)phys * p.pool_page_stride + (int64_t)g * p.pool_head_stride;
    codes = *reinterpret_cast<const uint32_t*>(tile + slot * (D / 2) + 4 * j);
    byte = tile[p.P * (D / 2) + (j / 4) * p.P + slot];
  }
  const uint4 v = values8(codes, kvq_scale(byte));
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(dst) = v;
  } else {
    float f[8];
    Vec16<bf16_t>::unpack(v, f);
    store8(dst, f);
  }
}

// Heads per thread of the queries: up to the four whose loads are in flight together, as many as leave 128 Ki threads (half of what
// the chip holds at this kernel's registers).  A chunk of 4096 rows x 28 heads: one head 19.5 us, three 17.8, seven in two goes 19.6.
int query_heads(const RowsParams& p) {
  const int64_t units = (int64_t)p.n_rows * p.Hq * (p.D / UNIT) >> 17;
  return (int)(units < 1 ? 1 : units > 4 ? 4 : units);
}
int64_t query_blocks_per_seq(const RowsParams& p, int heads) {
  const int64_t threads = (int64_t)p.max_rows * ((p.Hq + heads - 1) / heads) * (p.D / UNIT);
  return p.q.data ? (threads + THREADS - 1) / THREADS : 0;
}
int64_t page_blocks(const RowsParams& p, bool kvq) {
  return (int64_t)p.n_seqs * pages_touched(p.max_rows, p.P) * p.Hkv * 2 * (kvq ? 1 : p.D / 64);
}

template <typename T, int D, bool KVQ> hipError_t append(const RowsParams& p, hipStream_t st) {
  ProfScope prof_(KVQ ? "kvq_append_rope" : "kv_append_rope", st);
  const int heads = query_heads(p);
  const int64_t pages = page_blocks(p, KVQ), per_seq = query_blocks_per_seq(p, heads);
  const size_t lds = !p.kbar ? 0 : (size_t)p.P * (KVQ ? D * 2 : 64 * sizeof(T));   // (at most 32 KiB)
  append_rope_kernel<T, D, KVQ><<<dim3((unsigned)(pages + per_seq * p.n_seqs)), dim3(THREADS), lds, st>>>(p, (int)pages, (int)per_seq, heads);
  return hipGetLastError();
}
template <typename T, typename GT, int D> hipError_t append_bwd(const RowsParams& p, hipStream_t st) {
  ProfScope prof_("kv_append_rope_bwd", st);
  const int heads = query_heads(p);
  const int64_t pages = page_blocks(p, false), per_seq = query_blocks_per_seq(p, heads);
  append_rope_bwd_kernel<T, GT, D><<<dim3((unsigned)(pages + per_seq * p.n_seqs)), dim3(THREADS), 0, st>>>(p, (int)pages, (int)per_seq, heads);
  return hipGetLastError();
}
template <typename T, int D> hipError_t append(const RowsParams& p, bool kvq, hipStream_t st) {
  return kvq ? append<T, D, true>(p, st) : append<T, D, false>(p, st);
}
template <typename T, int D> hipError_t append_bwd(const RowsParams& p, bool grad_bf16, hipStream_t st) {
  return grad_bf16 ? append_bwd<T, bf16_t, D>(p, st) : append_bwd<T, float, D>(p, st);
}
int64_t read_blocks_per_seq(const RowsParams& p) { return ((int64_t)p.max_rows * 2 * p.Hkv * (p.D / 8) + THREADS - 1) / THREADS; }
template <typename T, int D> hipError_t read(const RowsParams& p, hipStream_t st) {
  ProfScope prof_("kvq_read", st);
  const int64_t per_seq = read_blocks_per_seq(p);
  kvq_read_kernel<T, D><<<dim3((unsigned)(per_seq * p.n_seqs)), dim3(THREADS), 0, st>>>(p, (int)per_seq);
  return hipGetLastError();
}

}  // namespace

int64_t append_rope_blocks(const RowsParams& p, bool kvq) { return page_blocks(p, kvq) + query_blocks_per_seq(p, query_heads(p)) * p.n_seqs; }
int64_t kvq_read_blocks(const RowsParams& p) { return read_blocks_per_seq(p) * p.n_seqs; }

hipError_t launch_append_rope(const RowsParams& p, bool is_bf16, bool kvq, hipStream_t st) {
  if (is_bf16) return p.D == 128 ? append<bf16_t, 128>(p, kvq, st) : append<bf16_t, 64>(p, kvq, st);
  return p.D == 128 ? append<float, 128>(p, kvq, st) : append<float, 64>(p, kvq, st);
}
hipError_t launch_append_rope_bwd(const RowsParams& p, bool is_bf16, bool grad_bf16, hipStream_t st) {
  if (is_bf16) return p.D == 128 ? append_bwd<bf16_t, 128>(p, grad_bf16, st) : append_bwd<bf16_t, 64>(p, grad_bf16, st);
  return p.D == 128 ? append_bwd<float, 128>(p, grad_bf16, st) : append_bwd<float, 64>(p, grad_bf16, st);
}
hipError_t launch_kvq_read(const RowsParams& p, bool is_bf16, hipStream_t st) {
  if (is_bf16) return p.D == 128 ? read<bf16_t, 128>(p, st) : read<bf16_t, 64>(p, st);
  return p.D == 128 ? read<float, 128>(p, st) : read<float, 64>(p, st);
}

}  // namespace oomb
