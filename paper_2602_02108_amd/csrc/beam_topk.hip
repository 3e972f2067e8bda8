// Beam search's selection: the n_out best continuations of every group over its beams' vocabularies (layouts: include/oomb.h).
//
//   candidate(w, v) = score[w] + x[w][v] - log sum_u exp(x[w][u])
//
// Within a row the order is that of the logits, so the first kernel needs no log-sum: a workgroup reads a slice of a row once, for the maximum and the
// sum of exponentials against it, and for the slice's best.  The second kernel, one workgroup per group, adds the slices' sums, takes the candidates in 64 bits and keeps the best.
// Ties go to the lowest w * vocab + v throughout.
//
// The best K of many: the K-th best of the threads' maxima is a bound that K values reach at least, and few others: these are written to the LDS and
// each one's rank is counted.
#include <algorithm>

#include "gen.h"

namespace oomb {

namespace {

constexpr int THREADS = 256;
constexpr int LOADS = 4;                        // of 16 bytes, of a thread at a time
constexpr int MOST_LISTS = 256;                 // slices of a group's rows
constexpr int MOST_SLICES = 64;
template <typename T> constexpr int VEC = 16 / (int)sizeof(T);
template <typename T> constexpr int EACH = LOADS * VEC<T>;       // elements of a thread at a time
template <typename T> constexpr int TILE = THREADS * EACH<T>;

// log2(e) in two floats: the product with a difference is then right to the last bit, so that sums of many exponentials are off by those alone
constexpr float LOG2E_HI = 1.44269502162933349609375f, LOG2E_LO = 1.925963033500011e-8f;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(__builtin_fmaf(d, LOG2E_HI, d * LOG2E_LO)); }

struct BeamWs { double* sums; float* tops; float* vals; int32_t* ids; };   // of a (row, slice): sum against the maximum, maximum, its K best, descending
__host__ __device__ BeamWs beam_ws(void* ws, int64_t lists, int k) {
  BeamWs w;
  w.sums = (double*)ws;
  w.tops = (float*)(w.sums + lists);
  w.vals = w.tops + lists;
  w.ids = (int32_t*)(w.vals + lists * k);
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

__device__ __forceinline__ bool better(float a, int i, float b, int j) { return a > b || (a == b && i < j); }

// One slice of one row.  Positions count from the 16-byte boundary at or before the row's first element, which lies `lead` elements behind it.
template <typename T>
__global__ __launch_bounds__(THREADS) void beam_rows_kernel(BeamParams p, void* ws, int slices, int slice_tiles) {
  const int row = blockIdx.x / slices, slice = blockIdx.x - row * slices, K = p.n_out, tid = threadIdx.x;
  if (p.done && p.done[row]) return;
  const float score = p.scores[row];
  if (!(fabsf(score) < INFINITY)) return;
  const BeamWs w = beam_ws(ws, (int64_t)p.n_groups * p.n_beams * slices, K);
  __shared__ float top_of[THREADS];
  __shared__ int id_of[THREADS];
  __shared__ float bound;
  __shared__ int bound_id, n_cand;
  __shared__ double wave_sum[THREADS / 64];
  __shared__ float wave_top[THREADS / 64];
  extern __shared__ __align__(16) char room[];
  float* cand = (float*)room;                    // [K * EACH + K]
  int* cand_id = (int*)(cand + K * EACH<T> + K);
  float* best = (float*)(cand_id + K * EACH<T> + K);   // [K], descending; ids from 0 to n_best - 1
  int* best_id = (int*)(best + K);

  const T* x = (const T*)p.logits + (int64_t)row * p.row_stride;
  const int lead = (int)(((uintptr_t)x & 15) / sizeof(T));
  const T* from = x - lead;                      // (only ever read inside the row)
  const int64_t end = (int64_t)lead + p.vocab, first = (int64_t)slice * slice_tiles * TILE<T>;
  float top = -INFINITY, sum = 0.0f;             // of this thread's elements
  int n_best = 0;
  float worst = -INFINITY;                       // the K-th best so far; what equals it comes later and loses
  for (int t = 0; t < slice_tiles; ++t) {
    const int64_t base = first + (int64_t)t * TILE<T>;
    if (base >= end) break;
    float f[EACH<T>];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int64_t at = base + ((int64_t)i * THREADS + tid) * VEC<T>;
      if (at >= lead && at + VEC<T> <= end) {
        unpack<T>(*reinterpret_cast<const uint4*>(from + at), f + i * VEC<T>);
      } else {
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j) f[i * VEC<T> + j] = at + j >= lead && at + j < end ? Elem<T>::load(from + at + j) : -INFINITY;
      }
    }
    float here = f[0];
    int where = 0;
#pragma unroll
    for (int j = 1; j < EACH<T>; ++j) {
      where = f[j] > here || !(here == here) ? j : where;
      here = fmaxf(here, f[j]);
    }
    const float to = fmaxf(top, here);
    if (to > -INFINITY) {
      sum *= exp_of(top - to);                   // (top -infinity: 0)
      float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < EACH<T>; ++j) s4[j & 3] += exp_of(f[j] - to);
      sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
      top = to;
    } else {
#pragma unroll
      for (int j = 0; j < EACH<T>; ++j) sum += f[j] == f[j] ? 0.0f : f[j];   // NaN
    }
    if (!__syncthreads_or(here > worst)) continue;

    // the bound: the K-th best of the threads' maxima
    auto id_at = [&](int j) { return (int)(base + ((int64_t)(j / VEC<T>) * THREADS + tid) * VEC<T> + j % VEC<T> - lead); };
    const int here_id = id_at(where);
    top_of[tid] = here;
    id_of[tid] = here_id;
    if (tid == 0) { n_cand = 0; bound = -INFINITY; bound_id = 0x7fffffff; }
    __syncthreads();
    int rank = 0;
    for (int i = 0; i < THREADS; ++i) rank += better(top_of[i], id_of[i], here, here_id);
    if (rank == K - 1 && here > -INFINITY) { bound = here; bound_id = here_id; }
    __syncthreads();
    const float b = bound;
    const int b_id = bound_id;
    if (here > worst && !better(b, b_id, here, here_id)) {
#pragma unroll
      for (int j = 0; j < EACH<T>; ++j)
        if (f[j] > worst && !better(b, b_id, f[j], id_at(j))) {
          const int c = atomicAdd(&n_cand, 1);
          cand[c] = f[j];
          cand_id[c] = id_at(j);
        }
    }
    __syncthreads();
    const int fresh = n_cand, all = fresh + n_best;
    for (int i = tid; i < n_best; i += THREADS) { cand[fresh + i] = best[i]; cand_id[fresh + i] = best_id[i]; }
    __syncthreads();
    for (int c = tid; c < all; c += THREADS) {
      const float v = cand[c];
      const int id = cand_id[c];
      int r = 0;
      for (int i = 0; i < all; ++i) r += better(cand[i], cand_id[i], v, id);
      if (r < K) { best[r] = v; best_id[r] = id; }
    }
    __syncthreads();
    n_best = min(all, K);
    if (n_best == K) worst = best[K - 1];
  }

  const int64_t list = (int64_t)row * slices + slice;
  for (int i = tid; i < K; i += THREADS) {
    w.vals[list * K + i] = i < n_best ? best[i] : -INFINITY;
    w.ids[list * K + i] = i < n_best ? best_id[i] : -1;
  }
  // the slice's maximum and sum
  float m = top;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k, 64));
  if ((tid & 63) == 0) wave_top[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
  double s = top > -INFINITY ? (double)sum * (double)exp_of(top - m) : (double)sum;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) s += __shfl_xor(s, k, 64);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    w.tops[list] = m;
    w.sums[list] = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
  }
}

__device__ __forceinline__ bool better64(double a, int i, double b, int j) { return a > b || (a == b && i < j); }

// One group: lists in order of beam and slice, so that of equal candidates the one of the lower list, and in it the first, wins.
__global__ __launch_bounds__(THREADS) void beam_group_kernel(BeamParams p, void* ws, int slices) {
  const int group = blockIdx.x, K = p.n_out, tid = threadIdx.x, lists = p.n_beams * slices;
  const BeamWs w = beam_ws(ws, (int64_t)p.n_groups * p.n_beams * slices, K);
  __shared__ double base[BEAM_MOST_BEAMS];       // score less log-sum; -infinity: the row offers nothing
  __shared__ double key[MOST_LISTS];
  __shared__ int ended[BEAM_MOST_BEAMS], n_cand;
  __shared__ double bound;
  __shared__ int bound_list;
  extern __shared__ __align__(16) char room[];
  double* cand = (double*)room;                  // [K * K + K]
  int* cand_at = (int*)(cand + K * K + K);       // list * K + place
  for (int beam = tid >> 6; beam < p.n_beams; beam += THREADS / 64) {
    const int lane = tid & 63;
    const int64_t row = (int64_t)group * p.n_beams + beam;
    const float score = p.scores[row];
    const int over = p.done ? p.done[row] : 0;
    const bool alive = fabsf(score) < INFINITY;
    float m = -INFINITY;
    double s = 0.0, z = 0.0;
    if (alive && !over) {
      const bool mine = lane < slices;           // (at most 64)
      const float t = mine ? w.tops[row * slices + lane] : -INFINITY;
      m = t;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k, 64));
      const double part = mine ? w.sums[row * slices + lane] : 0.0;
      s = t > -INFINITY ? part * exp((double)t - (double)m) : part;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) s += __shfl_xor(s, k, 64);
      z = (double)m + log(s);
    }
    if (lane == 0) {
      ended[beam] = alive && over;
      base[beam] = alive && !over && fabs(z) < (double)INFINITY ? (double)score - z : -(double)INFINITY;
    }
  }
  if (tid == 0) { n_cand = 0; bound = -(double)INFINITY; bound_list = 0x7fffffff; }
  __syncthreads();
  // candidate `at` of a list; an ended beam has one, in its first list
  auto value = [&](int list, int at) -> double {
    const int beam = list / slices;
    if (ended[beam]) return list == beam * slices && at == 0 ? (double)p.scores[(int64_t)group * p.n_beams + beam] : -(double)INFINITY;
    if (!(base[beam] > -(double)INFINITY)) return -(double)INFINITY;
    return base[beam] + (double)w.vals[((int64_t)group * lists + list) * K + at];
  };
  // With K or more lists their firsts give the bound; fewer are compared at the depth where they hold K together.
  const int depth = (K + lists - 1) / lists - 1, want = (K + depth) / (depth + 1);
  const double mine = tid < lists ? value(tid, depth) : -(double)INFINITY;
  if (tid < lists) key[tid] = mine;
  __syncthreads();
  if (tid < lists && mine > -(double)INFINITY) {
    int rank = 0;
    for (int i = 0; i < lists; ++i) rank += better64(key[i], i, mine, tid);
    if (rank == want - 1) { bound = mine; bound_list = tid; }
  }
  __syncthreads();
  if (tid < lists) {
    const double b = bound;
    const int b_list = bound_list;
    for (int i = 0; i < K; ++i) {
      const double v = value(tid, i);
      // (in its own list the bound lies at `depth`: what is there and before it counts, and equals behind it do not)
      if (!(v > -(double)INFINITY) || better64(b, b_list, v, tid) || (tid == b_list && i > depth)) break;
      const int c = atomicAdd(&n_cand, 1);
      cand[c] = v;
      cand_at[c] = tid * K + i;
    }
  }
  __syncthreads();
  const int all = n_cand;
  for (int c = tid; c < all; c += THREADS) {
    const double v = cand[c];
    const int at = cand_at[c];
    int r = 0;
    for (int i = 0; i < all; ++i) r += better64(cand[i], cand_at[i], v, at);
    if (r < K) {
      const int list = at / K, beam = list / slices;
      const int64_t to = (int64_t)group * K + r;
      p.parents[to] = group * p.n_beams + beam;
      p.tokens[to] = ended[beam] ? p.pad_token : w.ids[((int64_t)group * lists) * K + at];
      p.best[to] = (float)v;
    }
  }
  for (int r = all + tid; r < K; r += THREADS) {
    const int64_t to = (int64_t)group * K + r;
    p.parents[to] = -1;
    p.tokens[to] = -1;
    p.best[to] = -INFINITY;
  }
}

// How a row is cut: enough workgroups to fill the chip, few enough lists for the second kernel.
struct Cut { int slices, tiles; };
template <typename T> Cut cut_of(const BeamParams& p) {
  const int64_t rows = (int64_t)p.n_groups * p.n_beams;
  const int tiles = (int)(((int64_t)p.vocab + VEC<T> - 1 + TILE<T> - 1) / TILE<T>);   // (a row may begin anywhere in 16 bytes)
  int most = std::min(MOST_SLICES, MOST_LISTS / p.n_beams);
  const int64_t wanted = (2048 + rows - 1) / rows;
  most = (int)std::min<int64_t>(most, std::max<int64_t>(1, wanted));
  const int each = (tiles + std::min(tiles, most) - 1) / std::min(tiles, most);
  return {(tiles + each - 1) / each, each};
}
Cut cut_of(const BeamParams& p, bool is_bf16) { return is_bf16 ? cut_of<bf16_t>(p) : cut_of<float>(p); }

template <typename T> hipError_t run(const BeamParams& p, void* ws, hipStream_t st) {
  const Cut c = cut_of<T>(p);
  const size_t K = p.n_out, rows_lds = (K * EACH<T> + 2 * K) * 8, group_lds = (K * K + K) * 12;
  {
    ProfScope prof_("beam_rows", st);
    beam_rows_kernel<T><<<dim3((unsigned)(p.n_groups * p.n_beams * c.slices)), dim3(THREADS), rows_lds, st>>>(p, ws, c.slices, c.tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope prof_("beam_group", st);
  beam_group_kernel<<<dim3((unsigned)p.n_groups), dim3(THREADS), group_lds, st>>>(p, ws, c.slices);
  return hipGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(const BeamParams& p, bool is_bf16) {
  const int64_t lists = (int64_t)p.n_groups * p.n_beams * cut_of(p, is_bf16).slices;
  return (size_t)(lists * (12 + 8 * (int64_t)p.n_out));
}
int64_t beam_blocks(const BeamParams& p, bool is_bf16) { return (int64_t)p.n_groups * p.n_beams * cut_of(p, is_bf16).slices; }
hipError_t launch_beam_topk(const BeamParams& p, bool is_bf16, void* ws, hipStream_t st) { return is_bf16 ? run<bf16_t>(p, ws, st) : run<float>(p, ws, st); }

}  // namespace oomb
