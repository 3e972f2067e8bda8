// Pages of a cache with reference counts on the device: the sequences of the next step from those of this one (fork), copies of pages, and the used pages
// moved to the front (compact).  Results do not depend on scheduling: free pages go out in ascending order, by ranks counted with prefix sums, and what is
// added to a reference count is added as integers.
//
// What bounds it: launches and loads that wait for each other (parent, length, page, count), so few pages take one workgroup that holds the counts in the
// LDS (tables of 64 rows of 34: 6 us in one launch, 9 in two).  More pages: the plan (one workgroup, since every child's new pages follow from the needs of those
// before it) reads the counts only as far as free pages are needed, of a large pool the whole chip lists them first; the tables are written by the whole chip.
// Copies: memory, 236 MB read and written in 45 to 49 us (of the same pools again, partly out of the caches, 35).
#include "gen.h"
#include "wave.h"

namespace oomb {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int SCAN = 8;             // reference counts of a thread at a time
constexpr int ROW_THREADS = 256, ROW_ENTRIES = 1024;   // of a workgroup that rewrites a part of a table's row
constexpr int COPY_THREADS = 256;
constexpr int COMPACT_THREADS = 1024, COMPACT_EACH = 4, COMPACT_BLOCK = COMPACT_THREADS * COMPACT_EACH;   // pages of a workgroup that counts
constexpr int LARGE_POOL = 32768;   // a fork counts the free pages of more with many workgroups (150,000 pages, the free ones last: 10 us, by the plan alone 79)

__host__ __device__ int page_blocks(int64_t num_phys) { return (int)((num_phys + COMPACT_BLOCK - 1) / COMPACT_BLOCK); }

// What the plan leaves for the second kernel.
struct Child { int32_t was, now, first, copied; };      // tokens before and after, its first new page among all, whether the partly filled page is copied
struct Parent { int32_t children, keeps, pages, held; };   // whether a child keeps the partly filled page; entries that its row counts; full pages that children share
struct ForkWs { int32_t* found; Child* child; Parent* parent; int32_t *free_pages, *counts; };   // counts: free pages of each block of pages, in a large pool
__host__ __device__ ForkWs fork_ws(void* ws, int32_t n_seqs, int32_t n_out, int32_t num_phys) {
  ForkWs w;
  w.found = (int32_t*)ws;
  w.child = (Child*)((char*)ws + 16);
  w.parent = (Parent*)(w.child + n_out);
  w.free_pages = (int32_t*)(w.parent + n_seqs);
  w.counts = w.free_pages + num_phys;
  return w;
}

// Sum of x over the lanes below and over the workgroup's waves before: exclusive prefix and total.  `sums`: one int per wave.
template <int THREADS> __device__ __forceinline__ int block_scan(int x, int* sums, int& total) {
  constexpr int WAVES = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = wave_upto(x, 0, [](int a, int b) { return a + b; });
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int y = sums[w];
    before += w < wave ? y : 0;
    total += y;
  }
  return before + upto - x;
}

__device__ __forceinline__ int valid(const ForkParams& p, int x) { return x >= 0 && x < p.num_phys ? x : -1; }

// The free pages of each block of a large pool; the counts in their other place, if they get one.
__global__ __launch_bounds__(COMPACT_THREADS) void fork_count_kernel(ForkParams p, void* ws) {
  __shared__ int sums[COMPACT_THREADS / 64];
  const int64_t at = (int64_t)blockIdx.x * COMPACT_BLOCK + threadIdx.x * COMPACT_EACH;
  int n = 0, total;
#pragma unroll
  for (int j = 0; j < COMPACT_EACH; ++j)
    if (at + j < p.num_phys) {
      const int r = p.refs[at + j];
      n += r == 0;
      if (p.refs_out != p.refs) p.refs_out[at + j] = r;
    }
  block_scan<COMPACT_THREADS>(n, sums, total);
  if (threadIdx.x == 0) fork_ws(ws, p.n_seqs, p.n_out, p.num_phys).counts[blockIdx.x] = total;
}

// Workgroup 0 plans.  The others: in a large pool the free pages of a block each, ascending; else the reference counts in their other place, if they get one.
__global__ __launch_bounds__(PLAN_THREADS) void fork_plan_kernel(ForkParams p, void* ws, int blocks) {   // blocks: of a large pool; else 0
  const ForkWs w = fork_ws(ws, p.n_seqs, p.n_out, p.num_phys);
  __shared__ int sums[PLAN_THREADS / 64];
  if (blockIdx.x > 0 && blocks) {
    const int block = blockIdx.x - 1;
    int lower = 0, before, total;
    for (int i = threadIdx.x; i < block; i += PLAN_THREADS) lower += w.counts[i];
    block_scan<PLAN_THREADS>(lower, sums, before);
    const int64_t at = (int64_t)block * COMPACT_BLOCK + threadIdx.x * COMPACT_EACH;
    bool is[COMPACT_EACH];
    int n = 0;
#pragma unroll
    for (int j = 0; j < COMPACT_EACH; ++j) n += is[j] = at + j < p.num_phys && p.refs[at + j] == 0;
    int k = before + block_scan<PLAN_THREADS>(n, sums, total);
#pragma unroll
    for (int j = 0; j < COMPACT_EACH; ++j)
      if (is[j]) w.free_pages[k++] = (int)(at + j);
    return;
  }
  if (blockIdx.x > 0) {
    const int64_t i = (int64_t)(blockIdx.x - 1) * PLAN_THREADS + threadIdx.x;
    if (i < p.num_phys) p.refs_out[i] = p.refs[i];
    return;
  }
  __shared__ int children[FORK_MOST_SEQS], first[FORK_MOST_SEQS];
  for (int s = threadIdx.x; s < p.n_seqs; s += PLAN_THREADS) { children[s] = 0; first[s] = 0x7fffffff; }
  __syncthreads();
  for (int b = threadIdx.x; b < p.n_out; b += PLAN_THREADS) {
    const int s = p.parents[b];
    if (s >= 0 && s < p.n_seqs) {
      atomicAdd(&children[s], 1);
      atomicMin(&first[s], b);
    }
  }
  __syncthreads();
  const int P = 1 << p.log2_p, cap = p.cols << p.log2_p, out_cap = p.out_cols << p.log2_p;
  // the partly filled page of a sequence, and whether its first child may keep it
  auto last_page = [&](int s, int was) { return was & (P - 1) ? valid(p, p.tables[(int64_t)s * p.stride + (was >> p.log2_p)]) : -1; };
  for (int s = threadIdx.x; s < p.n_seqs; s += PLAN_THREADS) {
    const int len = min(max(p.lens[s], 0), cap), was = min(len, out_cap), page = last_page(s, was);
    Parent r;
    r.children = children[s];
    r.keeps = children[s] > 0 && page >= 0 && p.refs[page] <= 1;
    r.pages = (len + P - 1) >> p.log2_p;
    r.held = was >> p.log2_p;
    w.parent[s] = r;
  }
  int need_before = 0;
  for (int b0 = 0; b0 < p.n_out; b0 += PLAN_THREADS) {
    const int b = b0 + threadIdx.x;
    Child c{0, 0, 0, 0};
    int need = 0;
    if (b < p.n_out) {
      const int s = p.parents[b];
      const bool of = s >= 0 && s < p.n_seqs;
      if (of) {
        c.was = min(min(max(p.lens[s], 0), cap), out_cap);
        const int page = last_page(s, c.was);
        c.copied = page >= 0 && (first[s] != b || p.refs[page] > 1);
      }
      if (of || s == OOMB_FORK_BEGINS) {
        const int64_t more = p.grow ? max(p.grow[b], 0) : 0;
        c.now = (int)min(c.was + more, (int64_t)out_cap);
      }
      need = c.copied + ((c.now + P - 1) >> p.log2_p) - ((c.was + P - 1) >> p.log2_p);
    }
    int total;
    c.first = need_before + block_scan<PLAN_THREADS>(need, sums, total);
    need_before += total;
    if (b < p.n_out) w.child[b] = c;
  }

  // the free pages, ascending, as many as are needed
  int found = 0;
  if (blocks) {
    int n = 0;
    for (int i = threadIdx.x; i < blocks; i += PLAN_THREADS) n += w.counts[i];
    block_scan<PLAN_THREADS>(n, sums, found);
  }
  for (int64_t i0 = 0; !blocks && i0 < p.num_phys && found < need_before; i0 += PLAN_THREADS * SCAN) {
    const int64_t at = i0 + (int64_t)threadIdx.x * SCAN;
    int r[SCAN];
#pragma unroll
    for (int j = 0; j < SCAN; ++j) r[j] = at + j < p.num_phys ? p.refs[at + j] : 1;
    int n = 0;
#pragma unroll
    for (int j = 0; j < SCAN; ++j) n += r[j] == 0;
    int total;
    int k = found + block_scan<PLAN_THREADS>(n, sums, total);
#pragma unroll
    for (int j = 0; j < SCAN; ++j)
      if (r[j] == 0) {
        if (k < need_before) w.free_pages[k] = (int)(at + j);
        ++k;
      }
    found += total;
  }
  if (threadIdx.x == 0) {
    const int got = min(found, need_before);
    *w.found = got;
    p.status[0] = got;
    p.status[1] = need_before - got;
  }
}

// Workgroups of children write their rows, workgroups of parents take their references back.
__global__ __launch_bounds__(ROW_THREADS) void fork_rows_kernel(ForkParams p, void* ws, int pieces) {
  const ForkWs w = fork_ws(ws, p.n_seqs, p.n_out, p.num_phys);
  const int row = blockIdx.x / pieces, l0 = (blockIdx.x - row * pieces) * ROW_ENTRIES + threadIdx.x;
  const int P = 1 << p.log2_p;
  if (row < p.n_out) {
    const Child c = w.child[row];
    const int found = *w.found, s = p.parents[row];
    const int kept = ((c.was + P - 1) >> p.log2_p) - c.copied, pages = (c.now + P - 1) >> p.log2_p;
    const int32_t* from = p.tables + (int64_t)(s >= 0 && s < p.n_seqs ? s : 0) * p.stride;
    int32_t* to = p.tables_out + (int64_t)row * p.out_stride;
#pragma unroll
    for (int j = 0; j < ROW_ENTRIES / ROW_THREADS; ++j) {
      const int l = l0 + j * ROW_THREADS;
      if (l >= p.out_cols) break;
      int x = -1;
      if (l < kept) {
        x = valid(p, from[l]);
      } else if (l < pages) {
        const int k = c.first + l - kept;
        x = k < found ? w.free_pages[k] : -1;
        if (x >= 0) atomicAdd(p.refs_out + x, 1);
      }
      to[l] = x;
    }
    if (l0 == 0) {
      p.lens_out[row] = c.now;
      const bool copy = c.copied && c.first < found;
      p.copies[3 * row] = copy ? from[c.was >> p.log2_p] : -1;
      p.copies[3 * row + 1] = copy ? w.free_pages[c.first] : -1;
      p.copies[3 * row + 2] = copy ? c.was & (P - 1) : 0;
    }
    return;
  }
  const Parent r = w.parent[row - p.n_out];
  const int32_t* from = p.tables + (int64_t)(row - p.n_out) * p.stride;
#pragma unroll
  for (int j = 0; j < ROW_ENTRIES / ROW_THREADS; ++j) {
    const int l = l0 + j * ROW_THREADS;
    if (l >= r.pages) break;
    const int more = (l < r.held ? r.children : l == r.held ? r.keeps : 0) - 1;
    const int x = more ? valid(p, from[l]) : -1;
    if (x >= 0) atomicAdd(p.refs_out + x, more);
  }
}

// ---- copies ---------------------------------------------------------------------------------------------------------------
// A workgroup takes one head of a page of one pool at a time, 16 bytes a thread, eight loads in flight.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(COPY_THREADS) void page_copy_kernel(CopyParams p, CopyPools pools) {
  const int pool = blockIdx.y / p.n_heads, head = blockIdx.y - pool * p.n_heads;
  const int n = p.count ? min(max(*p.count, 0), p.n_copies) : p.n_copies;
  unsigned char* const base = pools.at[pool] + head * p.head_stride;
  const bool whole = p.tok_stride == 0 || p.tok_stride == p.row_bytes;
  const int row_units = p.row_bytes / 16;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int src = p.copies[3 * (int64_t)i], dst = p.copies[3 * (int64_t)i + 1], tokens = min(p.copies[3 * (int64_t)i + 2], p.page);
    if (src < 0 || src >= p.num_phys || dst < 0 || dst >= p.num_phys || src == dst || tokens <= 0) continue;
    const unsigned char* from = base + src * p.page_stride;
    unsigned char* to = base + dst * p.page_stride;
    const int units = p.tok_stride == 0 ? row_units : tokens * row_units;
    constexpr int AT_ONCE = 8;
    for (int u0 = threadIdx.x; u0 < units; u0 += AT_ONCE * COPY_THREADS) {
      u32x4 v[AT_ONCE];
      int64_t at[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int u = min(u0 + j * COPY_THREADS, units - 1);
        at[j] = whole ? (int64_t)u * 16 : (u / row_units) * p.tok_stride + (u % row_units) * 16;
        if (u0 + j * COPY_THREADS < units) v[j] = *reinterpret_cast<const u32x4*>(from + at[j]);
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if (u0 + j * COPY_THREADS < units) __builtin_nontemporal_store(v[j], reinterpret_cast<u32x4*>(to + at[j]));   // (past the caches: a compact and its copies of 236 MB 60 -> 53 us)
    }
  }
}

// ---- compact --------------------------------------------------------------------------------------------------------------
// n used pages; the i-th used page from n on moves to the i-th free page below n.
struct CompactWs { int32_t* counts; int32_t* becomes; };   // used pages of each block; a page's new number: -1, itself, or num_phys + i if it is the i-th to move
__host__ __device__ CompactWs compact_ws(void* ws, int32_t num_phys) {
  const int32_t blocks = page_blocks(num_phys);
  return {(int32_t*)ws, (int32_t*)ws + ((blocks + 3) & ~3)};
}
__device__ __forceinline__ int used_of(const CompactParams& p, int64_t at, int64_t end, bool (&used)[COMPACT_EACH]) {
  int n = 0;
#pragma unroll
  for (int j = 0; j < COMPACT_EACH; ++j) {
    used[j] = at + j < end && p.refs[at + j] > 0;
    n += used[j];
  }
  return n;
}

__global__ __launch_bounds__(COMPACT_THREADS) void compact_count_kernel(CompactParams p, void* ws) {
  __shared__ int sums[COMPACT_THREADS / 64];
  bool used[COMPACT_EACH];
  int total;
  block_scan<COMPACT_THREADS>(used_of(p, (int64_t)blockIdx.x * COMPACT_BLOCK + threadIdx.x * COMPACT_EACH, p.num_phys, used), sums, total);
  if (threadIdx.x == 0) compact_ws(ws, p.num_phys).counts[blockIdx.x] = total;
}

__global__ __launch_bounds__(COMPACT_THREADS) void compact_rank_kernel(CompactParams p, void* ws, int blocks) {
  __shared__ int sums[COMPACT_THREADS / 64];
  const CompactWs w = compact_ws(ws, p.num_phys);
  int mine = 0, before_me = 0;
  for (int i = threadIdx.x; i < blocks; i += COMPACT_THREADS) {
    const int c = w.counts[i];
    mine += c;
    before_me += i < (int)blockIdx.x ? c : 0;
  }
  int n, before, low;
  block_scan<COMPACT_THREADS>(mine, sums, n);
  block_scan<COMPACT_THREADS>(before_me, sums, before);
  // used pages below n: whole blocks, and the part of the one that n lies in
  const int edge = n / COMPACT_BLOCK;
  int below = 0;
  for (int i = threadIdx.x; i < edge; i += COMPACT_THREADS) below += w.counts[i];
  bool used[COMPACT_EACH];
  below += used_of(p, (int64_t)edge * COMPACT_BLOCK + threadIdx.x * COMPACT_EACH, n, used);
  block_scan<COMPACT_THREADS>(below, sums, low);
  const int64_t at = (int64_t)blockIdx.x * COMPACT_BLOCK + threadIdx.x * COMPACT_EACH;
  int total, rank = used_of(p, at, p.num_phys, used);
  rank = before + block_scan<COMPACT_THREADS>(rank, sums, total);
#pragma unroll
  for (int j = 0; j < COMPACT_EACH; ++j) {
    const int64_t i = at + j;
    if (i >= p.num_phys) break;
    if (used[j]) {
      if (i < n) {
        w.becomes[i] = p.map[i] = (int)i;
        p.refs_out[i] = p.refs[i];
      } else {
        w.becomes[i] = p.num_phys + (rank - low);
        p.moves[3 * (int64_t)(rank - low)] = (int)i;
      }
    } else {
      w.becomes[i] = p.map[i] = -1;
      if (i < n) {
        const int64_t k = i - rank;
        p.moves[3 * k + 1] = (int)i;
        p.moves[3 * k + 2] = p.page;
      } else {
        p.refs_out[i] = 0;
      }
    }
    rank += used[j];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.status[0] = n;
    p.status[1] = n - low;
  }
}

// Workgroups of moves (the counts of the pages that move, and the map), then of the tables' rows.
__global__ __launch_bounds__(ROW_THREADS) void compact_rows_kernel(CompactParams p, void* ws, int move_blocks, int pieces) {
  const CompactWs w = compact_ws(ws, p.num_phys);
  if ((int)blockIdx.x < move_blocks) {
    const int moves = p.status[1];
    for (int k = blockIdx.x * ROW_THREADS + threadIdx.x; k < moves; k += move_blocks * ROW_THREADS) {
      const int src = p.moves[3 * (int64_t)k], dst = p.moves[3 * (int64_t)k + 1];
      const int r = p.refs[src];
      p.map[src] = dst;
      p.refs_out[dst] = r;
      p.refs_out[src] = 0;
    }
    return;
  }
  const int block = blockIdx.x - move_blocks, s = block / pieces, l0 = (block - s * pieces) * ROW_ENTRIES + threadIdx.x;
  const int len = min(max(p.lens[s], 0), p.cols << p.log2_p), pages = (len + p.page - 1) >> p.log2_p;
#pragma unroll
  for (int j = 0; j < ROW_ENTRIES / ROW_THREADS; ++j) {
    const int l = l0 + j * ROW_THREADS;
    if (l >= p.cols) break;
    int x = l < pages ? p.tables[(int64_t)s * p.stride + l] : -1;
    x = x >= 0 && x < p.num_phys ? w.becomes[x] : -1;
    if (x >= p.num_phys) x = p.moves[3 * (int64_t)(x - p.num_phys) + 1];
    p.tables_out[(int64_t)s * p.out_stride + l] = x;
  }
}

// ---- few pages and sequences: a fork, or a compact, in one workgroup -------------------------------------------------------
// The reference counts lie in the LDS, and what needs them there needs no second launch (a table of 64 rows of 34: 9 us in two, 6 in one).
constexpr int SMALL_PAGES = 8192, SMALL_SEQS = 1024, SMALL_ENTRIES = 65536;
constexpr int SMALL_EACH = SMALL_PAGES / PLAN_THREADS;
// row of entry e of a table of `cols` columns: magic = ceil(2^32 / cols), exact below 2^16 entries
__device__ __forceinline__ int row_of(int e, int cols, uint32_t magic) { return cols == 1 ? e : (int)__umulhi((uint32_t)e, magic); }

__global__ __launch_bounds__(PLAN_THREADS) void fork_small_kernel(ForkParams p, uint32_t in_magic, uint32_t out_magic) {
  extern __shared__ __align__(16) int room[];
  __shared__ int sums[PLAN_THREADS / 64];
  int* const count = room;                                  // [num_phys]
  Child* const child = (Child*)(count + ((p.num_phys + 3) & ~3));   // [n_out]
  Parent* const parent = (Parent*)(child + p.n_out);        // [n_seqs]
  int* const first = (int*)(parent + p.n_seqs);             // [n_seqs]
  int* const last = first + p.n_seqs;                       // [n_seqs] partly filled page
  uint16_t* const free_pages = (uint16_t*)(last + p.n_seqs);   // [num_phys]
  const int tid = threadIdx.x, P = 1 << p.log2_p, cap = p.cols << p.log2_p, out_cap = p.out_cols << p.log2_p;
  // loads that wait for nothing
  const int s_of = tid < p.n_out ? p.parents[tid] : -1, more = tid < p.n_out && p.grow ? max(p.grow[tid], 0) : 0;
  const int len = tid < p.n_seqs ? min(max(p.lens[tid], 0), cap) : 0, was = min(len, out_cap);
  const int each = (p.num_phys + PLAN_THREADS - 1) / PLAN_THREADS;
  int refs[SMALL_EACH];
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j)
    if (j < each) refs[j] = tid * each + j < p.num_phys ? p.refs[tid * each + j] : 1;
  const int page = was & (P - 1) ? valid(p, p.tables[(int64_t)tid * p.stride + (was >> p.log2_p)]) : -1;
  if (tid < p.n_seqs) {
    parent[tid] = {0, 0, (len + P - 1) >> p.log2_p, was >> p.log2_p};
    first[tid] = 0x7fffffff;
    last[tid] = page;
  }
  int n_free = 0;
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j)
    if (j < each) {
      if (tid * each + j < p.num_phys) count[tid * each + j] = refs[j];
      n_free += refs[j] == 0;
    }
  __syncthreads();
  const bool of = s_of >= 0 && s_of < p.n_seqs;
  if (of) {
    atomicAdd(&parent[s_of].children, 1);
    atomicMin(&first[s_of], tid);
  }
  int total_free;
  int k = block_scan<PLAN_THREADS>(n_free, sums, total_free);
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j)
    if (j < each && refs[j] == 0) free_pages[k++] = (uint16_t)(tid * each + j);
  if (tid < p.n_seqs) parent[tid].keeps = parent[tid].children > 0 && page >= 0 && count[page] <= 1;
  Child c{0, 0, 0, 0};
  int need = 0;
  if (tid < p.n_out) {
    if (of) {
      const int l = last[s_of];
      c.copied = l >= 0 && (first[s_of] != tid || count[l] > 1);
      c.was = min(min(max(p.lens[s_of], 0), cap), out_cap);
    }
    if (of || s_of == OOMB_FORK_BEGINS) c.now = (int)min((int64_t)c.was + more, (int64_t)out_cap);
    need = c.copied + ((c.now + P - 1) >> p.log2_p) - ((c.was + P - 1) >> p.log2_p);
  }
  int total;
  c.first = block_scan<PLAN_THREADS>(need, sums, total);
  if (tid < p.n_out) child[tid] = c;
  __syncthreads();
  if (tid < p.n_out) {
    p.lens_out[tid] = c.now;
    const bool copy = c.copied && c.first < total_free;
    p.copies[3 * tid] = copy ? last[s_of] : -1;
    p.copies[3 * tid + 1] = copy ? free_pages[c.first] : -1;
    p.copies[3 * tid + 2] = copy ? c.was & (P - 1) : 0;
  }
  if (tid == 0) {
    p.status[0] = min(total, total_free);
    p.status[1] = total - min(total, total_free);
  }
  // the children's rows, then what the parents' rows counted; four entries of a thread at a time
  constexpr int AT_ONCE = 4;
  for (int e0 = tid; e0 < p.n_out * p.out_cols; e0 += AT_ONCE * PLAN_THREADS) {
    int x[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int e = e0 + j * PLAN_THREADS, row = row_of(e, p.out_cols, out_magic), l = e - row * p.out_cols;
      x[j] = -1;
      if (e < p.n_out * p.out_cols) {
        const Child h = child[row];
        if (l < ((h.was + P - 1) >> p.log2_p) - h.copied) x[j] = valid(p, p.tables[(int64_t)p.parents[row] * p.stride + l]);
      }
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int e = e0 + j * PLAN_THREADS, row = row_of(e, p.out_cols, out_magic), l = e - row * p.out_cols;
      if (e >= p.n_out * p.out_cols) break;
      const Child h = child[row];
      const int kept = ((h.was + P - 1) >> p.log2_p) - h.copied;
      if (l >= kept && l < (h.now + P - 1) >> p.log2_p && h.first + l - kept < total_free) {
        x[j] = free_pages[h.first + l - kept];
        atomicAdd(&count[x[j]], 1);
      }
      p.tables_out[(int64_t)row * p.out_stride + l] = x[j];
    }
  }
  for (int e0 = tid; e0 < p.n_seqs * p.cols; e0 += AT_ONCE * PLAN_THREADS) {
    int x[AT_ONCE], more_of[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int e = e0 + j * PLAN_THREADS, row = row_of(e, p.cols, in_magic), l = e - row * p.cols;
      x[j] = -1;
      more_of[j] = 0;
      if (e < p.n_seqs * p.cols) {
        const Parent r = parent[row];
        more_of[j] = l >= r.pages ? 0 : (l < r.held ? r.children : l == r.held ? r.keeps : 0) - 1;
        if (more_of[j]) x[j] = valid(p, p.tables[(int64_t)row * p.stride + l]);
      }
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (x[j] >= 0) atomicAdd(&count[x[j]], more_of[j]);
  }
  __syncthreads();
  for (int i = tid; i < p.num_phys; i += PLAN_THREADS) p.refs_out[i] = count[i];
}

__global__ __launch_bounds__(PLAN_THREADS) void compact_small_kernel(CompactParams p, uint32_t magic) {
  extern __shared__ __align__(16) int room[];
  __shared__ int sums[PLAN_THREADS / 64];
  int* const count = room;                                  // [num_phys]
  int* const becomes = count + p.num_phys;                  // [num_phys]: -1, itself, or num_phys + i if it is the i-th to move
  uint16_t* const src = (uint16_t*)(becomes + p.num_phys);  // [num_phys / 2]
  uint16_t* const dst = src + p.num_phys / 2;
  const int tid = threadIdx.x, each = (p.num_phys + PLAN_THREADS - 1) / PLAN_THREADS;
  int refs[SMALL_EACH], used = 0, n, low;
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j)
    if (j < each) refs[j] = tid * each + j < p.num_phys ? p.refs[tid * each + j] : 0;
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j)
    if (j < each) {
      if (tid * each + j < p.num_phys) count[tid * each + j] = refs[j];
      used += refs[j] > 0;
    }
  int rank = block_scan<PLAN_THREADS>(used, sums, n);
  int below = 0;
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j)
    if (j < each) below += refs[j] > 0 && tid * each + j < n;
  block_scan<PLAN_THREADS>(below, sums, low);
#pragma unroll
  for (int j = 0; j < SMALL_EACH; ++j) {
    const int i = tid * each + j;
    if (j >= each || i >= p.num_phys) break;
    if (refs[j] > 0) {
      becomes[i] = i < n ? i : p.num_phys + rank - low;
      if (i >= n) src[rank - low] = (uint16_t)i;
    } else {
      becomes[i] = -1;
      if (i < n) dst[i - rank] = (uint16_t)i;
    }
    rank += refs[j] > 0;
  }
  __syncthreads();
  const int moves = n - low;
  for (int i = tid; i < p.num_phys; i += PLAN_THREADS) {
    const int b = becomes[i];
    p.map[i] = b < p.num_phys ? b : dst[b - p.num_phys];
    if (b >= 0 || i >= n) p.refs_out[i] = b == i ? count[i] : 0;   // (holes below n: with the moves)
  }
  for (int k = tid; k < moves; k += PLAN_THREADS) {
    p.moves[3 * k] = src[k];
    p.moves[3 * k + 1] = dst[k];
    p.moves[3 * k + 2] = p.page;
    p.refs_out[dst[k]] = count[src[k]];
  }
  if (tid == 0) {
    p.status[0] = n;
    p.status[1] = moves;
  }
  constexpr int AT_ONCE = 4;
  for (int e0 = tid; e0 < p.n_seqs * p.cols; e0 += AT_ONCE * PLAN_THREADS) {
    int x[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int e = e0 + j * PLAN_THREADS, row = row_of(e, p.cols, magic), l = e - row * p.cols;
      x[j] = -1;
      if (e < p.n_seqs * p.cols) {
        const int len = min(max(p.lens[row], 0), p.cols << p.log2_p);
        x[j] = p.tables[(int64_t)row * p.stride + l];
        if (l >= (len + p.page - 1) >> p.log2_p) x[j] = -1;
      }
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int e = e0 + j * PLAN_THREADS, row = row_of(e, p.cols, magic), l = e - row * p.cols;
      if (e >= p.n_seqs * p.cols) break;
      int y = x[j] >= 0 && x[j] < p.num_phys ? becomes[x[j]] : -1;
      if (y >= p.num_phys) y = dst[y - p.num_phys];
      p.tables_out[(int64_t)row * p.out_stride + l] = y;
    }
  }
}

int pieces_of(int32_t cols) { return (cols + ROW_ENTRIES - 1) / ROW_ENTRIES; }
int fork_pieces(const ForkParams& p) { return pieces_of(p.cols > p.out_cols ? p.cols : p.out_cols); }
int compact_move_blocks(const CompactParams& p) {
  const int most = (p.num_phys / 2 + ROW_THREADS - 1) / ROW_THREADS;
  return most < 1 ? 1 : most < 64 ? most : 64;
}

bool few(int64_t num_phys, int64_t n_seqs, int64_t n_out, int64_t entries) {
  return num_phys <= SMALL_PAGES && n_seqs <= SMALL_SEQS && n_out <= SMALL_SEQS && entries <= SMALL_ENTRIES;
}
uint32_t magic_of(int32_t cols) { return (uint32_t)(((1ull << 32) + cols - 1) / cols); }

}  // namespace

size_t fork_workspace_bytes(int32_t n_seqs, int32_t n_out, int64_t num_phys) {
  return 16 + sizeof(Child) * (size_t)n_out + sizeof(Parent) * (size_t)n_seqs + sizeof(int32_t) * (size_t)(num_phys + page_blocks(num_phys));
}
int64_t fork_blocks(const ForkParams& p) { return ((int64_t)p.n_out + p.n_seqs) * fork_pieces(p); }
hipError_t launch_page_fork(const ForkParams& p, void* ws, hipStream_t st) {
  const int64_t in = (int64_t)p.n_seqs * p.cols, out = (int64_t)p.n_out * p.out_cols;
  if (few(p.num_phys, p.n_seqs, p.n_out, in > out ? in : out)) {
    ProfScope prof_("fork_small", st);
    const size_t lds = (size_t)((p.num_phys + 3) & ~3) * 4 + sizeof(Child) * p.n_out + (sizeof(Parent) + 8) * p.n_seqs + (size_t)p.num_phys * 2;
    if (lds > 65536 - 1024) {
      static DeviceOnce once;
      const hipError_t e = ensure_max_dynamic_lds(once, (const void*)fork_small_kernel, SMALL_PAGES * 6 + SMALL_SEQS * 40);
      if (e != hipSuccess) return e;
    }
    fork_small_kernel<<<dim3(1), dim3(PLAN_THREADS), lds, st>>>(p, magic_of(p.cols), magic_of(p.out_cols));
    return hipGetLastError();
  }
  {
    ProfScope prof_("fork_plan", st);
    const int blocks = p.num_phys > LARGE_POOL ? page_blocks(p.num_phys) : 0;
    if (blocks) {
      fork_count_kernel<<<dim3((unsigned)blocks), dim3(COMPACT_THREADS), 0, st>>>(p, ws);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    const unsigned more = blocks ? (unsigned)blocks : p.refs_out == p.refs ? 0 : (unsigned)(((int64_t)p.num_phys + PLAN_THREADS - 1) / PLAN_THREADS);
    fork_plan_kernel<<<dim3(1 + more), dim3(PLAN_THREADS), 0, st>>>(p, ws, blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope prof_("fork_rows", st);
  fork_rows_kernel<<<dim3((unsigned)fork_blocks(p)), dim3(ROW_THREADS), 0, st>>>(p, ws, fork_pieces(p));
  return hipGetLastError();
}

size_t compact_workspace_bytes(int64_t num_phys) {
  const int64_t blocks = page_blocks(num_phys);
  return sizeof(int32_t) * (size_t)(((blocks + 3) & ~3) + num_phys);
}
int64_t compact_blocks(const CompactParams& p) { return compact_move_blocks(p) + (int64_t)p.n_seqs * pieces_of(p.cols); }
hipError_t launch_page_compact(const CompactParams& p, void* ws, hipStream_t st) {
  if (few(p.num_phys, p.n_seqs, p.n_seqs, (int64_t)p.n_seqs * p.cols)) {
    ProfScope prof_("compact_small", st);
    const size_t lds = (size_t)p.num_phys * 10 + 16;
    if (lds > 65536 - 1024) {
      static DeviceOnce once;
      const hipError_t e = ensure_max_dynamic_lds(once, (const void*)compact_small_kernel, SMALL_PAGES * 10 + 16);
      if (e != hipSuccess) return e;
    }
    compact_small_kernel<<<dim3(1), dim3(PLAN_THREADS), lds, st>>>(p, magic_of(p.cols));
    return hipGetLastError();
  }
  const unsigned blocks = (unsigned)page_blocks(p.num_phys);
  {
    ProfScope prof_("compact_rank", st);
    compact_count_kernel<<<dim3(blocks), dim3(COMPACT_THREADS), 0, st>>>(p, ws);
    compact_rank_kernel<<<dim3(blocks), dim3(COMPACT_THREADS), 0, st>>>(p, ws, (int)blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope prof_("compact_rows", st);
  compact_rows_kernel<<<dim3((unsigned)compact_blocks(p)), dim3(ROW_THREADS), 0, st>>>(p, ws, compact_move_blocks(p), pieces_of(p.cols));
  return hipGetLastError();
}

hipError_t launch_page_copy(const CopyParams& p, void* const* pools, int32_t n_pools, hipStream_t st) {
  for (int32_t first = 0; first < n_pools; first += COPY_POOLS) {
    const int32_t n = n_pools - first < COPY_POOLS ? n_pools - first : COPY_POOLS;
    CopyPools at{};
    for (int32_t i = 0; i < n; ++i) at.at[i] = (unsigned char*)pools[first + i];
    const int32_t rows = n * p.n_heads, most = rows < 8192 ? 8192 / rows : 1;   // (a list that may be long is walked: most of its room may be unused)
    ProfScope prof_("page_copy", st);
    page_copy_kernel<<<dim3((unsigned)(p.n_copies < most ? p.n_copies : most), (unsigned)rows), dim3(COPY_THREADS), 0, st>>>(p, at);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace oomb
