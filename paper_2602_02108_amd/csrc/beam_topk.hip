// Beam search's selection: the n_out best continuations of every group over its beams' vocabularies (layouts: include/oomb.h).
//
//   candidate(w, v) = score[w] + x[w][v] - log sum_u exp(x[w][u])
//
// The first kernel reads the logits once, a slice of a row per workgroup: for each thread the maximum of its elements (a "cell" of the slice) and their sum of
// exponentials against it.  The second one, a workgroup per group, adds the sums, which makes candidates of different beams comparable, and looks for the K best
// through the cells: the K-th best cell maximum is a bound that K candidates reach at least; only the few cells that reach it are read again, and the rank of
// each of their values above the bound is counted.  Candidates are compared in 64 bits, ties go to the lowest w * vocab + v.
// Where very many values are equal (logits masked with a finite value, fewer than K others) the bound does not sort them out; then the K-th best cell is found in 64
// bits, and those equal to it are taken in order of their places.  Rows that fill fewer than K lanes (vocab / 4 in fp32, / 8 in bf16) have no first bound: with more than
// CELLS of them their group goes that way too (64 beams of 240 in fp32, 64 best: 60 us; of 1200: 21).
//
// What bounds it: the first kernel, the reading of the logits (256 rows of 130,999 bf16: 67 MB in 15.4 us, 4.4 TB/s; a maximum costs one instruction an element, where the
// best of each slice kept on the way made both kernels 154 us instead of 25); the second, one workgroup a group and its chain of steps (cells, bound, values, ranks):
// 8.7 us for one group of 4 x 32,000, 10.3 for 8 x 130,999, 10.7 for 32 such.  A cell that is read again holds vocab / (256 slices) values, which counts where many beams leave
// one slice a row: 34 us for 64 x 200,001 (fp32; the first kernel as many), 243 for 33 x 4,000,004 (beside 810).
#include <algorithm>
#include <cfloat>

#include "gen.h"

namespace oomb {

namespace {

constexpr int THREADS = 256;                    // of the first kernel
constexpr int LOADS = 4;                        // of 16 bytes, of a thread at a time
constexpr int MOST_LISTS = 64;                  // slices of a group's rows (or one a row): the second kernel takes in 10 B/ns (one group of 8 x 130,999 in fp32, both kernels: 16 us, with 256 lists 41)
constexpr int GROUP_THREADS = 1024;             // of the second
constexpr int GROUP_WAVES = GROUP_THREADS / 64;
constexpr int HELD = MOST_LISTS * THREADS / GROUP_THREADS;   // cells of a thread of it
static_assert(BEAM_MOST_BEAMS <= MOST_LISTS, "a row has a list at least");
constexpr int CELLS = 1024;                     // that reach the first bound (about 300 of equally distributed values at most, where there is one)
constexpr int HOLDERS = 256;                    // of them, that reach the bound
constexpr int ROOM = GROUP_THREADS;             // candidates that do
constexpr int PARTS = 8;                        // threads that count a rank together
template <typename T> constexpr int VEC = 16 / (int)sizeof(T);
template <typename T> constexpr int EACH = LOADS * VEC<T>;       // elements of a thread at a time
template <typename T> constexpr int TILE = THREADS * EACH<T>;

// log2(e) in two floats: the product with a difference is then right to the last bit.  An exponential of a difference above -32 is off by 2.5 * 2^-20 at most (half
// a step of the difference, of the product, the hardware's step), sums of a tile's by 0.6 * 2^-20 more, and the factors between references, of which as many as still
// matter are few, by less than what is left of 2^-18: so much the log-sum is off, for every vocabulary.
constexpr float LOG2E_HI = 1.44269502162933349609375f, LOG2E_LO = 1.925963033500011e-8f;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(__builtin_fmaf(d, LOG2E_HI, d * LOG2E_LO)); }
// e^(a - b), a finite: the exponent in 64 bits, its fraction's power the hardware's (2^-23).  (The library's 64-bit exponential holds 22 registers more: 32 groups of 8 x
// 130,999 in 25.5 us instead of 25.2.)
__device__ __forceinline__ double exp_between(float a, float b) {
  const double y = ((double)a - (double)b) * 1.4426950408889634, n = rint(y);
  return ldexp((double)__builtin_amdgcn_exp2f((float)(y - n)), (int)fmax(n, -4096.0));
}

struct BeamWs { double* sums; float* tops; float* cells; };   // of a (row, slice): sum against the maximum, maximum, [THREADS] maxima
__host__ __device__ BeamWs beam_ws(void* ws, int64_t lists) {
  BeamWs w;
  w.sums = (double*)ws;
  w.tops = (float*)(w.sums + lists);
  w.cells = w.tops + lists;
  return w;
}

template <typename T> __device__ __forceinline__ void unpack(const uint4& v, float* f);
template <> __device__ __forceinline__ void unpack<float>(const uint4& v, float* f) {
  f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
}
template <> __device__ __forceinline__ void unpack<bf16_t>(const uint4& v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// A row.  Positions count from the 16-byte boundary at or before its first element, which lies `lead` elements behind it.
template <typename T> struct Row {
  const T* from;                                 // (only ever read inside the row)
  int lead;
  int64_t end;
  __device__ __forceinline__ Row(const BeamParams& p, int64_t row) {
    const T* x = (const T*)p.logits + row * p.row_stride;
    lead = (int)(((uintptr_t)x & 15) / sizeof(T));
    from = x - lead;
    end = (int64_t)lead + p.vocab;
  }
  // 16 bytes at a position; what lies outside the row: -infinity
  __device__ __forceinline__ uint4 load(int64_t at) const {
    if (at >= lead && at + VEC<T> <= end) return *reinterpret_cast<const uint4*>(from + at);
    uint32_t word[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) {
        word[j] = at + j >= lead && at + j < end ? __float_as_uint(from[at + j]) : 0xff800000u;
      } else {
        const int64_t lo = at + 2 * j, hi = lo + 1;
        word[j] = (lo >= lead && lo < end ? (uint32_t)from[lo] : 0xff80u) | (hi >= lead && hi < end ? (uint32_t)from[hi] : 0xff80u) << 16;
      }
    }
    return make_uint4(word[0], word[1], word[2], word[3]);
  }
};
// piece i of a slice, of a thread
template <typename T> __device__ __forceinline__ int64_t place_of(int slice, int slice_tiles, int i, int thread) {
  return (int64_t)slice * slice_tiles * TILE<T> + ((int64_t)i * THREADS + thread) * VEC<T>;
}

template <typename T>
__global__ __launch_bounds__(THREADS, 4) void beam_rows_kernel(BeamParams p, void* ws, int slices, int slice_tiles) {
  const int row = blockIdx.x / slices, slice = blockIdx.x - row * slices, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (p.done && p.done[row]) return;
  const float score = p.scores[row];
  if (!(fabsf(score) < INFINITY)) return;
  constexpr int WAVES = THREADS / 64;
  __shared__ double wave_sum[WAVES];
  __shared__ float wave_top[WAVES];
  const Row<T> x(p, row);
  // Of this thread's elements: the maximum; the sum of exponentials against a reference that moves by more than 4 at a time.  A tile is summed in fp32; beyond
  // it are as many sums as a row is long, and factors of a reference that creeps up would be too, so both are in 64 bits.
  float top = -INFINITY, ref = -INFINITY;
  double sum = 0.0;
  uint4 raw[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) raw[i] = x.load(place_of<T>(slice, slice_tiles, i, tid));
  for (int t = 0; t < slice_tiles; ++t) {
    const int64_t base = place_of<T>(slice, slice_tiles, t * LOADS, 0);
    if (base >= x.end) break;
    float f[EACH<T>];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) unpack<T>(raw[i], f + i * VEC<T>);
    if (t + 1 < slice_tiles && base + TILE<T> < x.end) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) raw[i] = x.load(place_of<T>(slice, slice_tiles, (t + 1) * LOADS + i, tid));
    }
    float here = f[0];
#pragma unroll
    for (int j = 1; j < EACH<T>; ++j) here = fmaxf(here, f[j]);   // (not a NaN, unless all are)
    top = fmaxf(top, here);
    if (here > ref + 4.0f) {
      if (ref > -INFINITY) sum *= exp_between(ref, here);   // (else there is none yet)
      ref = here;
    }
    const float from = ref == -INFINITY ? 0.0f : ref;
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < EACH<T>; ++j) s4[j & 3] += exp_of(f[j] - from);
    sum += (double)((s4[0] + s4[1]) + (s4[2] + s4[3]));
  }
  const int64_t list = (int64_t)row * slices + slice;
  const BeamWs w = beam_ws(ws, (int64_t)p.n_groups * p.n_beams * slices);
  w.cells[list * THREADS + tid] = top;
  float m = top;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k, 64));
  if (lane == 0) wave_top[wave] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) m = fmaxf(m, wave_top[i]);
  double s = top > -INFINITY ? sum * exp_between(ref, m) : sum;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) s += __shfl_xor(s, k, 64);
  if (lane == 0) wave_sum[wave] = s;
  __syncthreads();
  if (tid == 0) {
    w.tops[list] = m;
    w.sums[list] = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
  }
}

// a double as a number in the same order (-0 as 0); 0: nothing (below every value)
__device__ __forceinline__ uint64_t ordered64(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return u ^ ((uint64_t)((int64_t)u >> 63) | 1ull << 63);
}
__device__ __forceinline__ double unordered64(uint64_t k) { return __longlong_as_double((long long)(k ^ ((uint64_t)((int64_t)~k >> 63) | 1ull << 63))); }

// Candidates in the LDS: a value, and where it stands: beam << 32 | token.
struct Cands {
  uint64_t val[ROOM + BEAM_MOST_OUT + 8 * PARTS];
  uint64_t at[ROOM + BEAM_MOST_OUT + 8 * PARTS];
  uint64_t best_val[BEAM_MOST_OUT], best_at[BEAM_MOST_OUT];   // in order
};
// The K best of `fresh` candidates and of the n_best best so far, in order; the new n_best.  (By every thread of a workgroup; no candidate twice.)
__device__ int keep_best(Cands& c, int fresh, int n_best, int K) {
  const int tid = threadIdx.x, all = fresh + n_best;
  if (tid < n_best) { c.val[fresh + tid] = c.best_val[tid]; c.at[fresh + tid] = c.best_at[tid]; }
  if (tid >= 64 && tid < 64 + 8 * PARTS) c.val[all + tid - 64] = 0;   // (loops of eight)
  __syncthreads();
  for (int i0 = 0; i0 < all; i0 += GROUP_THREADS / PARTS) {
    const int i = i0 + tid / PARTS;
    const uint64_t v = c.val[min(i, all)], at = c.at[min(i, all)];
    int r = 0;
    for (int k = 8 * (tid % PARTS); k < all; k += 8 * PARTS) {
      uint64_t v8[8], at8[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) { v8[j] = c.val[k + j]; at8[j] = c.at[k + j]; }
#pragma unroll
      for (int j = 0; j < 8; ++j) r += (int)(v8[j] > v) | ((int)(v8[j] == v) & (int)(at8[j] < at));
    }
#pragma unroll
    for (int k = 1; k < PARTS; k *= 2) r += __shfl_xor(r, k, 64);
    if (i < all && tid % PARTS == 0 && r < K) { c.best_val[r] = v; c.best_at[r] = at; }
  }
  __syncthreads();
  return min(all, K);
}

template <typename T> __global__ __launch_bounds__(GROUP_THREADS) void beam_group_kernel(BeamParams p, void* ws, int slices, int slice_tiles) {
  const int group = blockIdx.x, K = p.n_out, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lists = p.n_beams * slices, n_cells = lists * THREADS;
  const BeamWs w = beam_ws(ws, (int64_t)p.n_groups * p.n_beams * slices);
  __shared__ double base[BEAM_MOST_BEAMS];       // score less log-sum; -infinity: the row offers nothing
  __shared__ uint8_t beam_of[MOST_LISTS];
  __shared__ uint32_t tops[GROUP_THREADS], first_bound, bound;
  __shared__ __align__(16) uint32_t cell_key[CELLS + 8 * PARTS];
  __shared__ uint32_t cell_id[CELLS];
  __shared__ uint32_t holder[HOLDERS];
  __shared__ uint64_t ended_val[BEAM_MOST_BEAMS], ended_at[BEAM_MOST_BEAMS];
  __shared__ int n_cell, n_hold, n_cand;
  __shared__ uint8_t ties[BEAM_MOST_BEAMS];        // whether a beam has cells that equal the K-th best
  __shared__ __align__(16) Cands c;
  const float* cells = w.cells + (int64_t)group * n_cells;
  float held[HELD];                              // (on their way while the log-sums are formed; of a row that offers nothing they are not used)
#pragma unroll
  for (int j = 0; j < HELD; ++j)
    if (j * GROUP_THREADS < n_cells) held[j] = cells[min(tid + j * GROUP_THREADS, n_cells - 1)];
  if (tid < lists) beam_of[tid] = (uint8_t)(tid / slices);
  if (tid == 0) { n_cell = n_hold = n_cand = 0; bound = 0; }
  __syncthreads();
  for (int beam = wave; beam < p.n_beams; beam += GROUP_WAVES) {
    const int64_t row = (int64_t)group * p.n_beams + beam;
    const bool mine = lane < slices;             // (at most 64)
    const float score = p.scores[row], t = mine ? w.tops[row * slices + lane] : -INFINITY;
    const int over = p.done ? p.done[row] : 0;
    const double part = mine ? w.sums[row * slices + lane] : 0.0;
    const bool alive = fabsf(score) < INFINITY;
    double z = INFINITY;
    if (alive && !over) {
      float m = t;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k, 64));
      double s = t > -INFINITY ? part * exp((double)t - (double)m) : part;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) s += __shfl_xor(s, k, 64);
      z = (double)m + log(s);
    }
    if (lane == 0) {
      base[beam] = fabs(z) < (double)INFINITY ? (double)score - z : -(double)INFINITY;
      if (alive && over) {                       // a beam that has ended offers one candidate
        const int i = atomicAdd(&n_cand, 1);
        c.val[i] = ended_val[i] = ordered64((double)score);
        c.at[i] = ended_at[i] = (uint64_t)beam << 32 | (uint32_t)p.pad_token;
      }
    }
  }
  __syncthreads();
  const int n_ended = n_cand;
  auto value = [&](int beam, float x) -> uint64_t {   // 0: nothing
    const double v = base[beam] + (double)x;
    return x > -INFINITY && v > -(double)INFINITY ? ordered64(v) : 0;
  };
  auto cell = [&](int i, float x) -> uint32_t { return i < n_cells ? (uint32_t)(value(beam_of[i / THREADS], x) >> 32) : 0; };
  uint32_t mine = 0, keys[HELD];
#pragma unroll
  for (int j = 0; j < HELD; ++j) {
    keys[j] = 0;
    if (j * GROUP_THREADS < n_cells) mine = max(mine, keys[j] = cell(tid + j * GROUP_THREADS, held[j]));
  }
  // A bound that K cells reach at least: of the maxima of 64 groups of threads (of each lane over the waves: short rows fill the first threads of a list) the K-th
  // best, by one wave
  tops[tid] = mine;
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < GROUP_WAVES; ++w) mine = max(mine, tops[64 * w + lane]);
    const uint32_t key = (mine & ~63u) | (63 - lane);   // (no two alike; what the last bits held is let in)
    int rank = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) rank += (uint32_t)__builtin_amdgcn_readlane(key, i) > key;
    if (rank == K - 1) first_bound = max(key & ~63u, 1u);
    mine = tops[lane];
  }
  __syncthreads();
  const uint32_t limit = first_bound;
  auto note = [&](int i, uint32_t key) __attribute__((always_inline)) {
    if (key < limit) return;
    const int to = atomicAdd(&n_cell, 1);
    if (to < CELLS) { cell_key[to] = key; cell_id[to] = i; }
  };
  if (mine >= limit) {
#pragma unroll
    for (int j = 0; j < HELD; ++j)
      if (j * GROUP_THREADS < n_cells) note(tid + j * GROUP_THREADS, keys[j]);
  }
  __syncthreads();
  const int noted = n_cell;
  int n_best = 0;
  bool found = noted <= CELLS;
  if (found) {
    // the K-th best of them (equal ones in any order: what equals it counts)
    if (tid < 8 * PARTS) cell_key[noted + tid] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < noted; i0 += GROUP_THREADS / PARTS) {
      const int i = i0 + tid / PARTS;
      const uint32_t key = cell_key[min(i, noted)];
      int more = 0, same = 0;
      for (int k = 8 * (tid % PARTS); k < noted; k += 8 * PARTS) {
        uint32_t k8[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) k8[j] = cell_key[k + j];
#pragma unroll
        for (int j = 0; j < 8; ++j) { more += k8[j] > key; same += k8[j] == key; }
      }
#pragma unroll
      for (int k = 1; k < PARTS; k *= 2) { more += __shfl_xor(more, k, 64); same += __shfl_xor(same, k, 64); }
      if (i < noted && more < K && more + same >= K) bound = key;   // (whoever writes writes the same)
    }
    __syncthreads();
    for (int i = tid; i < noted; i += GROUP_THREADS)
      if (cell_key[i] >= bound) {
        const int to = atomicAdd(&n_hold, 1);
        if (to < HOLDERS) holder[to] = cell_id[i];
      }
    __syncthreads();
    const int n_holders = n_hold;
    found = n_holders <= HOLDERS;
    if (found) {
      // their values once more, a piece of 16 bytes a thread
      const uint64_t least = max((uint64_t)bound << 32, 1ull);
      const int each = slice_tiles * LOADS;
      for (int e = tid; e < n_holders * each; e += GROUP_THREADS) {
        const int h = e / each, i = e - h * each, id = holder[h], list = id / THREADS, beam = beam_of[list];
        const Row<T> x(p, (int64_t)group * p.n_beams + beam);
        const int64_t at = place_of<T>(list - beam * slices, slice_tiles, i, id % THREADS);
        float f[VEC<T>];
        unpack<T>(x.load(at), f);
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j) {
          const uint64_t v = value(beam, f[j]);
          if (v < least) continue;
          const int to = atomicAdd(&n_cand, 1);
          if (to < ROOM) { c.val[to] = v; c.at[to] = (uint64_t)beam << 32 | (uint32_t)(at + j - x.lead); }
        }
      }
      __syncthreads();
      found = n_cand <= ROOM;
      if (found) n_best = keep_best(c, n_cand, 0, K);
    }
  }
  if (!found) {
    // Very many values are equal, or very many cells have no first bound.  The K-th best cell in 64 bits: what reaches it stands in the cells that do, and if they are many, in the fewer than K above
    // it and at the lowest places that equal it.
    if (tid < n_ended) { c.val[tid] = ended_val[tid]; c.at[tid] = ended_at[tid]; }
    if (tid < p.n_beams) ties[tid] = 0;
    n_best = keep_best(c, n_ended, 0, K);
    if (tid == 0) n_hold = 0;
    uint64_t top[HELD];
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int i = tid + j * GROUP_THREADS;
      top[j] = i < n_cells ? value(beam_of[i / THREADS], cells[i]) : 0;
    }
    uint64_t edge = 0;
    int reach = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t to = edge | 1ull << bit;
      int n = 0;
#pragma unroll
      for (int j = 0; j < HELD; ++j) n += __popcll(__ballot(top[j] >= to));
      if (lane == 0) tops[(bit & 1) * GROUP_WAVES + wave] = n;
      __syncthreads();
      int all = 0;
#pragma unroll
      for (int w = 0; w < GROUP_WAVES; ++w) all += tops[(bit & 1) * GROUP_WAVES + w];
      if (all >= K) { edge = to; reach = all; }
    }
    edge = max(edge, (uint64_t)1);               // (fewer than K cells hold anything: all of it)
    const bool few = reach <= HOLDERS;
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      if (top[j] > edge || (few && top[j] == edge)) holder[atomicAdd(&n_hold, 1)] = tid + j * GROUP_THREADS;
      else if (top[j] == edge) ties[beam_of[(tid + j * GROUP_THREADS) / THREADS]] = 1;
    }
    __syncthreads();
    auto offer = [&](uint64_t v, uint64_t at) __attribute__((always_inline)) {   // a candidate of each thread; 0: none
      const uint64_t worst = n_best == K ? c.best_val[K - 1] : 0, worst_at = n_best == K ? c.best_at[K - 1] : 0;
      const bool better = v > worst || (v && v == worst && at < worst_at);
      if (tid == 0) n_cand = 0;
      if (!__syncthreads_or(better)) return;
      if (better) {
        const int to = atomicAdd(&n_cand, 1);
        c.val[to] = v;
        c.at[to] = at;
      }
      __syncthreads();
      n_best = keep_best(c, n_cand, n_best, K);
    };
    const int each = slice_tiles * LOADS * VEC<T>;
    const int64_t n_held = (int64_t)n_hold * each;
    for (int64_t e0 = 0; e0 < n_held; e0 += GROUP_THREADS) {
      const int64_t e = min(e0 + tid, n_held - 1);
      const int h = (int)(e / each), i = (int)(e - (int64_t)h * each), id = holder[h], list = id / THREADS, beam = beam_of[list];
      const Row<T> x(p, (int64_t)group * p.n_beams + beam);
      const int64_t at = place_of<T>(list - beam * slices, slice_tiles, i / VEC<T>, id % THREADS) + i % VEC<T>;
      const uint64_t v = e0 + tid < n_held && at >= x.lead && at < x.end ? value(beam, Elem<T>::load(x.from + at)) : 0;
      offer(v >= edge ? v : 0, (uint64_t)beam << 32 | (uint32_t)(at - x.lead));
    }
    for (int beam = 0; beam < p.n_beams; ++beam) {
      if (!ties[beam]) continue;
      const Row<T> x(p, (int64_t)group * p.n_beams + beam);
      for (int64_t v0 = 0; v0 < p.vocab; v0 += GROUP_THREADS) {
        if (n_best == K && (c.best_val[K - 1] > edge || (c.best_val[K - 1] == edge && c.best_at[K - 1] < ((uint64_t)beam << 32 | (uint32_t)v0)))) break;
        const int64_t at = x.lead + min(v0 + tid, (int64_t)p.vocab - 1);
        uint64_t v = v0 + tid < p.vocab ? value(beam, Elem<T>::load(x.from + at)) : 0;
        if (v == edge) {                         // (in a cell above the edge it has been offered)
          const int slice = (int)(at / ((int64_t)slice_tiles * TILE<T>)), thread = (int)(at / VEC<T> % THREADS);
          if (value(beam, cells[(beam * slices + slice) * THREADS + thread]) != edge) v = 0;
        }
        offer(v == edge ? v : 0, (uint64_t)beam << 32 | (uint32_t)(at - x.lead));
      }
    }
  }
  if (tid < K) {
    const int64_t to = (int64_t)group * K + tid;
    const bool is = tid < n_best;
    p.parents[to] = is ? group * p.n_beams + (int)(c.best_at[tid] >> 32) : -1;
    p.tokens[to] = is ? (int)(uint32_t)c.best_at[tid] : -1;
    p.best[to] = is ? (float)unordered64(c.best_val[tid]) : -INFINITY;
  }
}

// How a row is cut: enough workgroups to fill the chip, few enough lists for the second kernel.
struct Cut { int slices, tiles; };
template <typename T> Cut cut_of(const BeamParams& p) {
  const int64_t rows = (int64_t)p.n_groups * p.n_beams;
  const int tiles = (int)(((int64_t)p.vocab + VEC<T> - 1 + TILE<T> - 1) / TILE<T>);   // (a row may begin anywhere in 16 bytes)
  int most = MOST_LISTS / p.n_beams;
  const int64_t wanted = (1024 + rows - 1) / rows;
  most = (int)std::min<int64_t>(most, std::max<int64_t>(1, wanted));
  const int each = (tiles + std::min(tiles, most) - 1) / std::min(tiles, most);
  return {(tiles + each - 1) / each, each};
}
Cut cut_of(const BeamParams& p, bool is_bf16) { return is_bf16 ? cut_of<bf16_t>(p) : cut_of<float>(p); }

template <typename T> hipError_t run(const BeamParams& p, void* ws, hipStream_t st) {
  const Cut c = cut_of<T>(p);
  {
    ProfScope prof_("beam_rows", st);
    beam_rows_kernel<T><<<dim3((unsigned)(p.n_groups * p.n_beams * c.slices)), dim3(THREADS), 0, st>>>(p, ws, c.slices, c.tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope prof_("beam_group", st);
  beam_group_kernel<T><<<dim3((unsigned)p.n_groups), dim3(GROUP_THREADS), 0, st>>>(p, ws, c.slices, c.tiles);
  return hipGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(const BeamParams& p, bool is_bf16) {
  const int64_t lists = (int64_t)p.n_groups * p.n_beams * cut_of(p, is_bf16).slices;
  return (size_t)(lists * (12 + 4 * THREADS));
}
int64_t beam_blocks(const BeamParams& p, bool is_bf16) {   // (in workgroups of 256 threads)
  return std::max((int64_t)p.n_groups * p.n_beams * cut_of(p, is_bf16).slices, (int64_t)p.n_groups * (GROUP_THREADS / 256));
}
hipError_t launch_beam_topk(const BeamParams& p, bool is_bf16, void* ws, hipStream_t st) { return is_bf16 ? run<bf16_t>(p, ws, st) : run<float>(p, ws, st); }

}  // namespace oomb
