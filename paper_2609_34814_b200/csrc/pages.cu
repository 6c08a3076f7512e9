// Pages of a cache's pool: the rows of a page table go on from rows of the last one (forking, growing, cutting back, ending), the pages
// in use go to the lowest numbers of the pool, pages go from one cache to another.
//
// Which page goes where is decided by the pages' counts: how many rows hold each.  Sums over the pool and over the rows decide the
// places, so the result does not depend on the order in which threads run.  A call that decides has two launches: one thread block or
// one cluster of up to sixteen does the sums (its phases are separated by the cluster's own barrier; no thread waits on a flag in memory),
// then a grid over all SMs copies what the decision says.  The first is latency (a few round trips to memory), the second
// memory traffic: a warp has four 16-byte loads under way a lane before it stores any.
#include <algorithm>
#include <climits>
#include "host_common.h"

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kCluster = 16;                         // thread blocks that decide, at most (the largest cluster; eight where that does not fit)
constexpr int kCopyThreads = 256, kCopyBlocks = 8;   // blocks an SM
constexpr int kUnroll = 4;                           // vectors of a lane under way
constexpr int kSegment = 32 * kUnroll;               // vectors of a warp's turn
constexpr int kRun = 512;                            // table entries of a warp's turn

__device__ void report(int* status, int code, int site, int where, int value) {
  if (status && atomicCAS(status, 0, code) == 0) status[1] = site, status[2] = where, status[3] = value;
}

__device__ __forceinline__ void sync_plan() {
  if (gridDim.x == 1) {
    __syncthreads();
  } else {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
  }
}

// ------------------------------------------------------------------ copying pages

// One of a cache's two tensors, in vectors (of 16 bytes, or of one element where something is not aligned to that)
struct Side { long long page, head, token; };
struct PageShape {
  int heads, vecs;         // vectors of a token's head
  int shift;               // log2 of the page's tokens
  int token_major;         // which of head and token is the inner one in the destination's memory
  int packed;              // both sides hold a page in one piece, in the same order
  unsigned total;          // vectors of a page (below 2^31)
  int segments;            // warps' turns of a page
  Side from[2], to[2];
};

// A warp's turn: vectors [segment * kSegment, ...) of the first `tokens` tokens of a page.
template <class V>
__device__ __forceinline__ void copy_segment(const PageShape& s, const V* from, V* to, int which, int segment, int tokens, int lane) {
  V x[kUnroll];
  long long at[kUnroll];
  const unsigned first = (unsigned)segment * kSegment + lane;
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const unsigned i = first + 32 * u;
    at[u] = -1;
    if (i >= s.total) continue;
    if (s.packed && tokens >> s.shift) {             // (the whole page)
      at[u] = i;
      x[u] = __ldg(from + i);
      continue;
    }
    const unsigned row = i / (unsigned)s.vecs, col = i - row * s.vecs;
    unsigned head, token;
    if (s.token_major) {
      token = row / (unsigned)s.heads, head = row - token * s.heads;
    } else {
      head = row >> s.shift, token = row & ((1u << s.shift) - 1);
    }
    if ((int)token >= tokens) continue;
    at[u] = head * s.to[which].head + token * s.to[which].token + col;
    x[u] = __ldg(from + head * s.from[which].head + token * s.from[which].token + col);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (at[u] >= 0) to[at[u]] = x[u];
}

struct Tensors { const void* from[2]; void* to[2]; };

// turn `i` of a pair of pages: its tensor and its segment
template <class V>
__device__ __forceinline__ void copy_turn(const PageShape& s, const Tensors& t, int from, int to, int i, int tokens, int lane) {
  const int which = i >= s.segments, segment = i - which * s.segments;
  copy_segment<V>(s, static_cast<const V*>(t.from[which]) + from * s.from[which].page, static_cast<V*>(t.to[which]) + to * s.to[which].page, which, segment,
                  tokens, lane);
}

struct CopyParams {
  PageShape shape;
  Tensors t;
  const int *from_pages, *to_pages;
  int count, from_n, to_n;
  int* dev_status;
};

template <class V>
__global__ void __launch_bounds__(kCopyThreads) k_copy_pages(const __grid_constant__ CopyParams p) {
  const int lane = threadIdx.x & 31;
  const long long turns = 2ll * p.shape.segments * p.count, step = (long long)gridDim.x * (kCopyThreads / 32);
#pragma unroll 1
  for (long long w = (long long)blockIdx.x * (kCopyThreads / 32) + threadIdx.x / 32; w < turns; w += step) {
    const int pair = (int)(w / (2 * p.shape.segments)), i = (int)(w - (long long)pair * 2 * p.shape.segments);
    const int from = p.from_pages[pair], to = p.to_pages[pair];
    if (from == -1 || to == -1) continue;
    if (from < 0 || from >= p.from_n || to < 0 || to >= p.to_n) {
      if (i == 0 && lane == 0) report(p.dev_status, WAVEAL_ERR_BAD_MASK, from < 0 || from >= p.from_n ? 89 : 90, pair, from < 0 || from >= p.from_n ? from : to);
      continue;
    }
    copy_turn<V>(p.shape, p.t, from, to, i, 1 << p.shape.shift, lane);
  }
}

// ------------------------------------------------------------------ sums over a thread block

// of the threads in front of this one; total: of all.  (Two barriers; shared: 33 words.)
__device__ __forceinline__ int scan_block(int x, int* shared, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  int upto = x;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  __syncthreads();                                   // (the words may still be read from the last call)
  if (lane == 31) shared[warp] = upto;
  __syncthreads();
  int sums = shared[lane];                           // kPlanThreads / 32 == 32 warps
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, sums, d);
    if (lane >= d) sums += y;
  }
  total = __shfl_sync(0xffffffffu, sums, 31);
  const int before = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
  return upto - x + (warp ? before : 0);
}
static_assert(kPlanThreads == 32 * 32, "scan_block");

// The counts of a pool, sixteen bytes at a time where they are aligned to that: one, eight or sixteen thread blocks read them all, so what a thread has under
// way at once decides (1.3 MB of counts took 10 us a pass one by one).
__device__ __forceinline__ bool by_four(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}
__device__ __forceinline__ void copy_counts(int* to, const int* from, int n, int tid, int threads) {
  int done = 0;
  if (by_four(to, from)) {
    done = n / 4 * 4;
#pragma unroll 4
    for (int i = tid; i < n / 4; i += threads) reinterpret_cast<int4*>(to)[i] = __ldg(reinterpret_cast<const int4*>(from) + i);
  }
#pragma unroll 1
  for (int i = done + tid; i < n; i += threads) to[i] = __ldg(from + i);
}
// LOCAL: in shared memory
template <bool LOCAL, class T> __device__ __forceinline__ T load_state(const T* at) {
  if constexpr (LOCAL) return *at;
  else return __ldcg(at);
}
// eight counts from i on (those from `end` on: `none`)
template <bool LOCAL = false> __device__ __forceinline__ void load_counts(const int* counts, int i, int end, bool four, int none, int (&v)[8]) {
  if (four && i + 8 <= end) {
    const int4* at = reinterpret_cast<const int4*>(counts + i);
    const int4 a = load_state<LOCAL>(at), b = load_state<LOCAL>(at + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = i + k < end ? load_state<LOCAL>(counts + i + k) : none;
  }
}

// this block's part of n things, begin a multiple of kPerThread
constexpr int kPerThread = 8;                        // pages of a thread's turn: a 32-byte sector of their counts
struct Part { int begin, end; };
__device__ __forceinline__ Part part_of(int n) {
  const long long each = ((long long)n + gridDim.x - 1) / gridDim.x, up = (each + kPerThread - 1) / kPerThread * kPerThread;
  return {(int)min((long long)n, up * blockIdx.x), (int)min((long long)n, up * (blockIdx.x + 1))};
}

// ------------------------------------------------------------------ forking

struct ForkParams {
  PageShape shape;
  Tensors t;
  int old_rows, rows, old_pages, pages, n_pages;
  long long old_stride, stride;
  const int *old_table, *held, *refs, *parents, *keep, *room;
  int *table, *new_refs;
  // workspace
  int* kids;               // [2][old_rows]: rows that go on from this one; the fewest full pages that they keep
  int* ends;               // [n_pages], of pages that rows end in: the first of these rows
  int4* row;               // [rows]: parent or -1, full pages kept, pages in all, tokens in the page filled in part (bit 30: the row keeps that page)
  int2* last;              // [rows]: the page filled in part (-1: none), where the row's fresh pages begin
  int* fresh;              // [n_pages]: free pages in ascending order, as many as are needed
  int* sums;               // [2][kCluster]
  int* free_pages;         // [1]
  int* dev_status;
};
constexpr int kStays = 1 << 30;

__device__ __forceinline__ int held_tokens(const ForkParams& p, int r) {
  const int n = p.held[r];
  return n < 0 || n > (long long)p.old_pages << p.shape.shift ? 0 : n;
}

// What the phases hand on (counts, rows): LOCAL, where one thread block decides, in shared memory (eight phases read in turn what the one before has
// written: 10.5 us of 16 rows of 63 pages instead of 12.6 through L2, 19.5 of 64 rows in beams instead of 21.6), else in the results and the workspace.
struct ForkState {
  int *refs, *ends, *count, *fewest;
  int4* row;
  int2* last;
};
__host__ __device__ inline size_t fork_state_bytes(long long n_pages, long long old_rows, long long rows) {
  return (size_t)(rows * (sizeof(int4) + sizeof(int2)) + (2 * ((n_pages + 3) / 4 * 4) + 2 * old_rows) * sizeof(int));
}

template <bool LOCAL>
__global__ void __launch_bounds__(kPlanThreads, 1) k_fork_plan(const __grid_constant__ ForkParams p) {
  __shared__ int shared[33], list[kPlanThreads * kPerThread];
  extern __shared__ __align__(16) unsigned char local[];
  ForkState s = {p.new_refs, p.ends, p.kids, p.kids + p.old_rows, p.row, p.last};
  if constexpr (LOCAL) {
    const int n = (p.n_pages + 3) / 4 * 4;
    s.row = reinterpret_cast<int4*>(local);
    s.refs = reinterpret_cast<int*>(s.row + p.rows);
    s.ends = s.refs + n;
    s.last = reinterpret_cast<int2*>(s.ends + n);
    s.count = reinterpret_cast<int*>(s.last + p.rows), s.fewest = s.count + p.old_rows;
  }
  waveal::let_next_kernel_start();
  const int tid = blockIdx.x * kPlanThreads + threadIdx.x, threads = gridDim.x * kPlanThreads;
  const int warp = tid / 32, warps = threads / 32, lane = threadIdx.x & 31;
  const int shift = p.shape.shift, mask = (1 << shift) - 1;

  copy_counts(s.refs, p.refs, p.n_pages, tid, threads);
#pragma unroll 1
  for (int r = tid; r < p.old_rows; r += threads) {
    s.count[r] = 0, s.fewest[r] = INT_MAX;
    const int n = p.held[r];
    if (n < 0 || n > (long long)p.old_pages << shift) report(p.dev_status, WAVEAL_ERR_BAD_MASK, 81, r, n);
  }
  sync_plan();

  // ---- what every row keeps
#pragma unroll 1
  for (int b = tid; b < p.rows; b += threads) {
    int parent = p.parents ? p.parents[b] : b, keep = p.keep[b], room = p.room[b];
    if (parent >= p.old_rows) report(p.dev_status, WAVEAL_ERR_BAD_MASK, 80, b, parent), parent = -1;
    if (parent >= 0 && (keep < 0 || keep > held_tokens(p, parent))) report(p.dev_status, WAVEAL_ERR_BAD_MASK, 82, b, keep), parent = -1;
    room = max(room, keep);
    if (parent >= 0 && room > (long long)p.pages << shift) report(p.dev_status, WAVEAL_ERR_BAD_MASK, 83, b, room), parent = -1;
    int4 row = {-1, 0, 0, 0};
    int page = -1;
    if (parent >= 0) {
      row = {parent, keep >> shift, (int)(((long long)room + mask) >> shift), keep & mask};
      if (row.w) {
        page = p.old_table[parent * p.old_stride + row.y];
        if (page < 0 || page >= p.n_pages) {
          report(p.dev_status, WAVEAL_ERR_BAD_MASK, 84, b, page);
          page = -1;
        } else {
          s.ends[page] = INT_MAX;
        }
      }
      atomicAdd(s.count + parent, 1);
      atomicMin(s.fewest + parent, row.y);
    }
    s.row[b] = row;
    s.last[b] = {page, 0};
  }
  sync_plan();

  // ---- counts: a page of an old row that k rows share goes from one holder to k.  (Rows of one child: no change up to what it keeps.)
  const int old_runs = (p.old_pages + kRun - 1) / kRun, runs = (p.pages + kRun - 1) / kRun;
#pragma unroll 1
  for (long long u = warp; u < (long long)p.old_rows * old_runs; u += warps) {
    const int r = (int)(u / old_runs), run = (int)(u - (long long)r * old_runs);
    const int kids = load_state<LOCAL>(s.count + r), all = kids ? load_state<LOCAL>(s.fewest + r) : 0, pages = (int)(((long long)held_tokens(p, r) + mask) >> shift);
#pragma unroll 4
    for (int j = max(run * kRun, kids == 1 ? all : 0) + lane; j < min(pages, (run + 1) * kRun); j += 32) {
      const int change = (j < all ? kids : 0) - 1, page = p.old_table[r * p.old_stride + j];
      if (change && page >= 0 && page < p.n_pages) atomicAdd(s.refs + page, change);
    }
  }
#pragma unroll 1
  for (long long u = warp; u < (long long)p.rows * runs; u += warps) {
    const int b = (int)(u / runs), run = (int)(u - (long long)b * runs);
    const int4 row = load_state<LOCAL>(s.row + b);
    if (row.x < 0) continue;
#pragma unroll 4
    for (int j = max(run * kRun, load_state<LOCAL>(s.fewest + row.x)) + lane; j < min(row.y, (run + 1) * kRun); j += 32) {
      const int page = p.old_table[row.x * p.old_stride + j];
      if (page >= 0 && page < p.n_pages) atomicAdd(s.refs + page, 1);
    }
  }
#pragma unroll 1
  for (int b = tid; b < p.rows; b += threads) {
    const int page = load_state<LOCAL>(s.last + b).x;
    if (page >= 0) atomicMin(s.ends + page, b);
  }
  sync_plan();

  // ---- a page filled in part stays with the first row that ends in it, if nobody else holds it
#pragma unroll 1
  for (int b = tid; b < p.rows; b += threads) {
    int4 row = load_state<LOCAL>(s.row + b);
    const int page = load_state<LOCAL>(s.last + b).x;
    bool stays = row.w && page < 0;                  // (no page to copy from: the row gets -1 there)
    if (page >= 0 && load_state<LOCAL>(s.ends + page) == b && load_state<LOCAL>(s.refs + page) <= 0) {
      stays = true;
      s.refs[page] = 1;
    }
    if (stays) s.row[b].w = row.w | kStays;
    s.last[b].y = row.z - row.y - stays;             // fresh pages
  }
  sync_plan();

  // ---- sums of the blocks' parts: free pages, fresh pages
  const Part pages = part_of(p.n_pages), rows = part_of(p.rows);
  int free_here = 0, need_here = 0, total;
  const bool four = LOCAL || by_four(s.refs, s.refs);
#pragma unroll 2
  for (int i = pages.begin + threadIdx.x * kPerThread; i < pages.end; i += kPlanThreads * kPerThread) {
    int v[kPerThread];
    load_counts<LOCAL>(s.refs, i, pages.end, four, 1, v);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) free_here += v[k] <= 0;
  }
#pragma unroll 1
  for (int b = rows.begin + threadIdx.x; b < rows.end; b += kPlanThreads) need_here += load_state<LOCAL>(s.last + b).y;
  scan_block(free_here, shared, total);
  if (threadIdx.x == 0) p.sums[blockIdx.x] = total;
  scan_block(need_here, shared, total);
  if (threadIdx.x == 0) p.sums[kCluster + blockIdx.x] = total;
  sync_plan();
  int free_before = 0, need_before = 0, free_all = 0, need_all = 0;
#pragma unroll
  for (int i = 0; i < kCluster; ++i) {
    const int f = i < (int)gridDim.x ? __ldcg(p.sums + i) : 0, n = i < (int)gridDim.x ? __ldcg(p.sums + kCluster + i) : 0;
    if (i < (int)blockIdx.x) free_before += f, need_before += n;
    free_all += f, need_all += n;
  }
  if (tid == 0) *p.free_pages = free_all;

  // ---- where every row's fresh pages begin, and which pages these are
#pragma unroll 1
  for (int b0 = rows.begin; b0 < rows.end; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x, need = b < rows.end ? load_state<LOCAL>(s.last + b).y : 0;
    const int begin = need_before + scan_block(need, shared, total);
    need_before += total;
    if (b < rows.end) {
      s.last[b].y = begin;
      if (begin <= free_all && begin + need > free_all) report(p.dev_status, WAVEAL_ERR_NO_PAGES, 85, b, need_all - free_all);
    }
  }
#pragma unroll 1
  for (int i0 = pages.begin; i0 < pages.end && free_before < need_all; i0 += kPlanThreads * kPerThread) {
    const int i = i0 + threadIdx.x * kPerThread;
    int v[kPerThread];
    load_counts<LOCAL>(s.refs, min(i, pages.end), pages.end, four, 1, v);
    unsigned is_free = 0;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) is_free |= (unsigned)(v[k] <= 0) << k;
    // (the list goes through shared memory, the counts back eight at once: a store whose lanes lie apart costs as many as there are lanes)
    int at = scan_block(__popc(is_free), shared, total);
    const int take = min(total, need_all - free_before);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k)
      if (is_free >> k & 1) {
        if (at < take) list[at] = i + k, v[k] = 1;
        ++at;
      }
    if (is_free) {
      if (four && i + kPerThread <= pages.end) {
        int4* to = reinterpret_cast<int4*>(s.refs + i);
        to[0] = make_int4(v[0], v[1], v[2], v[3]), to[1] = make_int4(v[4], v[5], v[6], v[7]);
      } else {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k)
          if (i + k < pages.end) s.refs[i + k] = v[k];
      }
    }
    __syncthreads();
#pragma unroll 1
    for (int k = threadIdx.x; k < take; k += kPlanThreads) p.fresh[free_before + k] = list[k];
    free_before += total;
  }
  if constexpr (LOCAL) {
    __syncthreads();
    const bool wide = by_four(p.new_refs, p.new_refs);
#pragma unroll 1
    for (int i = tid; wide && i < p.n_pages / 4; i += threads) reinterpret_cast<int4*>(p.new_refs)[i] = reinterpret_cast<int4*>(s.refs)[i];
#pragma unroll 1
    for (int i = (wide ? p.n_pages / 4 * 4 : 0) + tid; i < p.n_pages; i += threads) p.new_refs[i] = s.refs[i];
#pragma unroll 1
    for (int b = tid; b < p.rows; b += threads) p.row[b] = s.row[b], p.last[b] = s.last[b];
  }
}

template <class V>
__global__ void __launch_bounds__(kCopyThreads) k_fork_apply(const __grid_constant__ ForkParams p) {
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * (kCopyThreads / 32) + threadIdx.x / 32, warps = (long long)gridDim.x * (kCopyThreads / 32);
  const int turns = 2 * p.shape.segments;
  waveal::wait_for_previous_kernel();
  const int free_all = *p.free_pages;
  // the pages that rows filled in part and do not keep
#pragma unroll 1
  for (long long w = warp; w < (long long)p.rows * turns; w += warps) {
    const int b = (int)(w / turns);
    const int4 row = p.row[b];
    const int2 last = p.last[b];
    if (row.w == 0 || row.w & kStays || last.y >= free_all) continue;
    copy_turn<V>(p.shape, p.t, last.x, p.fresh[last.y], (int)(w - (long long)b * turns), row.w, lane);
  }
  // the table
  const int runs = (p.pages + kRun - 1) / kRun;
#pragma unroll 1
  for (long long u = warp; u < (long long)p.rows * runs; u += warps) {
    const int b = (int)(u / runs), run = (int)(u - (long long)b * runs);
    const int4 row = p.row[b];
    const int2 last = p.last[b];
    const int stays = row.w & kStays ? 1 : 0, end = min(p.pages, (run + 1) * kRun);
    // (four entries of a lane at once: they come from the last table or from the list of fresh pages)
#pragma unroll 1
    for (int j0 = run * kRun + lane; j0 < end; j0 += 4 * 32) {
      int page[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + 32 * k, i = last.y + j - row.y - stays;
        const bool old = j < row.y, fresh = !old && j < row.z && !(j == row.y && stays) && i < free_all;
        page[k] = j == row.y && stays ? last.x : -1;
        if (j < end && (old || fresh)) page[k] = old ? p.old_table[row.x * p.old_stride + j] : p.fresh[i];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + 32 * k;
        if (j >= end) continue;
        if (j < row.y && (page[k] < 0 || page[k] >= p.n_pages)) {
          report(p.dev_status, WAVEAL_ERR_BAD_MASK, 84, b, page[k]);
          page[k] = -1;
        }
        p.table[b * p.stride + j] = page[k];
      }
    }
  }
}

// ------------------------------------------------------------------ compacting

struct CompactParams {
  PageShape shape;
  Tensors t;
  int rows, pages, n_pages, prefix;
  long long old_stride, stride;
  const int *refs, *old_table, *old_prefix;
  int *new_refs, *table, *new_prefix, *place, *used;
  // workspace
  int* from;               // [n_pages]: pages in use behind the first n, at the number of pages in use in front of them
  int* to;                 // [n_pages]: free pages among the first n
  int* sums;               // [kCluster]
  int* first;              // [1]: pages in use among the first n: where `from` begins
};

__global__ void __launch_bounds__(kPlanThreads, 1) k_compact_plan(const __grid_constant__ CompactParams p) {
  __shared__ int shared[33];
  waveal::let_next_kernel_start();
  const Part pages = part_of(p.n_pages);
  int here = 0, total;
  const bool four = by_four(p.refs, p.refs);
#pragma unroll 2
  for (int i = pages.begin + threadIdx.x * kPerThread; i < pages.end; i += kPlanThreads * kPerThread) {
    int v[kPerThread];
    load_counts(p.refs, i, pages.end, four, 0, v);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) here += v[k] > 0;
  }
  scan_block(here, shared, total);
  if (threadIdx.x == 0) p.sums[blockIdx.x] = total;
  sync_plan();
  int before = 0, n = 0;
#pragma unroll
  for (int i = 0; i < kCluster; ++i) {
    const int x = i < (int)gridDim.x ? __ldcg(p.sums + i) : 0;
    if (i < (int)blockIdx.x) before += x;
    n += x;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *p.used = n;
    if (n == p.n_pages) *p.first = n;
  }
  // the i-th page in use from n on goes to the i-th free page below n
#pragma unroll 1
  for (int i0 = pages.begin; i0 < pages.end; i0 += kPlanThreads * kPerThread) {
    const int i = i0 + threadIdx.x * kPerThread;
    int v[kPerThread];
    load_counts(p.refs, min(i, pages.end), pages.end, four, 0, v);
    unsigned in_use = 0;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) in_use |= (unsigned)(v[k] > 0) << k;
    int at = before + scan_block(__popc(in_use), shared, total);
    before += total;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int page = i + k;
      if (page >= pages.end) break;
      const bool u = in_use >> k & 1;
      if (page == n) *p.first = at;
      if (u && page >= n) p.from[at] = page;
      if (!u && page < n) p.to[page - at] = page;
      p.place[page] = at;                            // (for the next pass)
      at += u;
    }
  }
  sync_plan();
  const int first = __ldcg(p.first);
#pragma unroll 1
  for (int page = pages.begin + threadIdx.x; page < pages.end; page += kPlanThreads) {
    const int count = p.refs[page];
    int place = -1;
    if (count > 0) {
      place = page < n ? page : __ldcg(p.to + (__ldcg(p.place + page) - first));
      p.new_refs[place] = count;
    }
    if (page >= n) p.new_refs[page] = 0;
    p.place[page] = place;
  }
}

template <class V>
__global__ void __launch_bounds__(kCopyThreads) k_compact_apply(const __grid_constant__ CompactParams p) {
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * (kCopyThreads / 32) + threadIdx.x / 32, warps = (long long)gridDim.x * (kCopyThreads / 32);
  waveal::wait_for_previous_kernel();
  const int first = *p.first, moves = *p.used - first, turns = 2 * p.shape.segments;
#pragma unroll 1
  for (long long w = warp; w < (long long)moves * turns; w += warps) {
    const int i = (int)(w / turns);
    copy_turn<V>(p.shape, p.t, p.from[first + i], p.to[i], (int)(w - (long long)i * turns), 1 << p.shape.shift, lane);
  }
  auto moved = [&](int page) { return page >= 0 && page < p.n_pages ? p.place[page] : -1; };
  const int runs = (p.pages + kRun - 1) / kRun;
#pragma unroll 1
  for (long long u = warp; u < (long long)p.rows * runs; u += warps) {
    const int b = (int)(u / runs), run = (int)(u - (long long)b * runs);
#pragma unroll 4
    for (int j = run * kRun + lane; j < min(p.pages, (run + 1) * kRun); j += 32) p.table[b * p.stride + j] = moved(p.old_table[b * p.old_stride + j]);
  }
#pragma unroll 1
  for (long long i = warp * 32 + lane; i < p.prefix; i += warps * 32) p.new_prefix[i] = moved(p.old_prefix[i]);
}

// ------------------------------------------------------------------ host

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

waveal_status check_pool(const waveal_cache_desc* c) {
  if (!c) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "cache is NULL");
  if (waveal_status e = waveal::check_cache(c)) return e;
  if (c->head_dim < 2 || c->head_dim > 512) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "head_dim %d (supported: 2 .. 512)", c->head_dim);
  if ((long long)c->kv_heads * c->page_size * c->head_dim > INT_MAX) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^31 - 1 elements in a page");
  return WAVEAL_OK;
}

// Threads walk through rows, pages of a row and pages of the pool in steps of up to 2^14 with 32-bit numbers, which must not run over.
constexpr int kMost = 1 << 30;
waveal_status check_counts(const waveal_cache_desc* c, int rows_a, int rows_b, int pages_a, int pages_b) {
  if (c->n_pages > kMost || std::max(rows_a, rows_b) > kMost || std::max(pages_a, pages_b) > kMost)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^30 pages of the pool, rows of a table or entries of a row");
  return WAVEAL_OK;
}

// a cache's tensors, or two caches', as the copying kernels see them; wide: 16-byte vectors.  Where anything is not aligned to that, all of it goes element by
// element, at a third of the rate (1.3 GB in one order: 2.1 TB/s instead of 6.2) or a sixth (other order: 0.9 instead of 6.1); the few pages of a step take as long.
bool page_shape(PageShape& s, Tensors& t, const waveal_cache_desc* from, const void* from_k, const void* from_v, const waveal_cache_desc* to, void* to_k,
                void* to_v) {
  const int64_t *in[2] = {from->k_stride, from->v_stride}, *out[2] = {to->k_stride, to->v_stride};
  t = {{from_k, from_v}, {to_k, to_v}};
  bool wide = from->head_dim % 8 == 0;
  for (int i = 0; i < 2; ++i) {
    wide = wide && waveal::aligned(t.from[i], 16) && waveal::aligned(t.to[i], 16);
    for (int j = 0; j < 3; ++j) wide = wide && in[i][j] % 8 == 0 && out[i][j] % 8 == 0;
  }
  const int64_t vec = wide ? 8 : 1, dim = from->head_dim, heads = from->kv_heads, tokens = from->page_size;
  s.heads = from->kv_heads, s.vecs = (int)(dim / vec), s.shift = __builtin_ctz((unsigned)from->page_size);
  s.token_major = out[0][2] > out[0][1];
  s.packed = 1;
  for (int i = 0; i < 2; ++i) {
    s.from[i] = {in[i][0] / vec, in[i][1] / vec, in[i][2] / vec}, s.to[i] = {out[i][0] / vec, out[i][1] / vec, out[i][2] / vec};
    const bool by_head = in[i][2] == dim && out[i][2] == dim && in[i][1] == dim * tokens && out[i][1] == dim * tokens;
    const bool by_token = in[i][1] == dim && out[i][1] == dim && in[i][2] == dim * heads && out[i][2] == dim * heads;
    if (!by_head && !by_token) s.packed = 0;
  }
  s.total = (unsigned)(heads * tokens * s.vecs);
  s.segments = (int)((s.total + kSegment - 1) / kSegment);
  return wide;
}

// blocks of a copying grid: one for every eight warps' turns, at most what the SMs hold
unsigned copy_grid(long long turns) {
  const long long blocks = (turns + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  return (unsigned)std::max(1ll, std::min(blocks, (long long)waveal::sm_count() * kCopyBlocks));
}

constexpr size_t kLocalBytes = 192 << 10;           // (beside the 32 KB and more of the kernel's own)

// Thread blocks that decide about a fork: one with its state in shared memory, a cluster of eight or of sixteen, by the counts and table entries that they walk
// through.  us of growing / forking a table of 64 rows, half of the pool in it:
//   pages                    one           eight         sixteen
//   1,024                    10.9 / 11.8   16.2 / 16.7   20.7 / 21.3
//   16,384                   13.6 / 14.6   17.1 / 19.3   21.8 / 24.0
//   32,768                   does not fit  17.6 / 22.1   21.9 / 26.5   (one, its state in L2: 18.9 / 27.5)
//   131,072                                21.0 / 27.6   24.9 / 31.4   (35.6 / 69.5)
//   327,680                                24.9 / 40.6   26.1 / 34.9   (64 / 151)
// 10,000 pages, 64 rows of 1,024 entries: 17.1 / 21.7, 17.9 / 21.3, 22.4 / 26.1; 8,192 pages, 256 rows of 512: 24.8 / 44.6, 19.8 / 26.3, 23.6 / 29.4.  Two and
// four are never more than 1 us ahead of the better neighbour.
// A new row's entries are walked where it keeps more than another child of its parent, so rows beyond the old ones' number count, an entry a quarter.  us where
// every child keeps another length / all keep everything, pools of 4,096 to 20,000 pages:
//   rows           one           eight         sixteen
//   1 x 1,000: 64  15.4 / 13.1   22.1 / 19.3   27.9 / 25.0
//   4 x 1,000: 128 20.9 / 14.7   22.3 / 19.5   27.6 / 25.2
//   1 x 1,000: 256 28.5 / 17.0   27.2 / 19.9   29.5 / 24.9
//   1 x 8,000: 64  44.0 / 21.9   39.5 / 20.9   39.0 / 25.6
//   2 x 2,000: 500 96.1 / 31.3   61.6 / 23.8   49.4 / 27.6
//   the same: 2,000 (not in one) 184 / 41.0    118 / 38.9
long long fork_work(long long pool, const waveal_fork_desc* f) {
  const long long more = std::max(0ll, (long long)f->rows - f->old_rows);
  return pool + (long long)f->old_rows * f->old_pages + more * std::min(f->old_pages, f->pages) / 4;
}
int fork_blocks(long long work, size_t state) { return work <= 65536 && state <= kLocalBytes ? 1 : work <= 400000 ? 8 : 16; }
// The same for compacting, us with the copies of half of the pool's small pages: 1,024 pages 7.3 (one), 8.5 (eight), 9.8 (sixteen); 4,096 11.7, 9.4, 11.0;
// 16,384 29.0, 13.2, 13.3; 32,768 52, 17.8, 16.7; 131,072 188, 46, 36.
int compact_blocks(long long pages) { return pages <= 2048 ? 1 : pages <= 16384 ? 8 : 16; }

// What a kernel has been given leave to on a device: nothing yet, what it asked for, clusters of eight at most.
enum Leave : char { kUnasked = 0, kAsWanted, kEightAtMost };

template <class P>
waveal_status launch_plan(void (*kernel)(P), Leave (&leave)[64], const P& p, int blocks, size_t smem, cudaStream_t st) {
  int dev = 0;
  WAVEAL_CUDA_OK(cudaGetDevice(&dev));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)blocks, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr, cfg.numAttrs = 1;
  // More than 48 KB have to be asked for, and more than eight blocks a cluster, which need as many SMs in one part of the GPU: where there are fewer
  // (part of a GPU is all that the program has), eight do the same work.
  if (blocks > 8 || smem) {
    Leave l = dev < 64 ? leave[dev] : kUnasked;
    if (l == kUnasked) {
      l = kAsWanted;
      if (smem) {
        WAVEAL_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLocalBytes));
      } else {
        WAVEAL_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        int clusters = 0;
        WAVEAL_CUDA_OK(cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg));
        if (clusters < 1) l = kEightAtMost;
      }
      if (dev < 64) leave[dev] = l;
    }
    if (l == kEightAtMost) cfg.gridDim.x = attr[0].val.clusterDim.x = 8;
  }
  WAVEAL_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, p));
  return WAVEAL_OK;
}

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return x && y && x < y + b_bytes && y < x + a_bytes;
}
size_t table_bytes(int rows, int pages, int64_t stride) { return rows && pages ? ((size_t)(rows - 1) * stride + pages) * sizeof(int) : 0; }

waveal_status check_fork(const waveal_cache_desc* c, const waveal_fork_desc* f) {
  if (waveal_status e = check_pool(c)) return e;
  if (!f) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "fork is NULL");
  if (f->old_rows < 0 || f->rows < 0 || f->old_pages < 0 || f->pages < 0)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "rows and pages must not be negative");
  if (waveal_status e = check_counts(c, f->old_rows, f->rows, f->old_pages, f->pages)) return e;
  if (f->old_stride < f->old_pages || f->stride < f->pages) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "a table's stride is smaller than its pages");
  if ((long long)f->old_rows * f->old_pages > INT_MAX || (long long)f->rows * f->pages > INT_MAX)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^31 - 1 entries in a table");
  return WAVEAL_OK;
}

struct ForkLayout { size_t kids, ends, row, last, fresh, sums, bytes; };
ForkLayout fork_layout(const waveal_cache_desc* c, const waveal_fork_desc* f) {
  ForkLayout l;
  l.sums = 0;
  l.kids = up256((2 * kCluster + 1) * sizeof(int));
  l.ends = l.kids + up256((size_t)f->old_rows * 2 * sizeof(int));
  l.row = l.ends + up256((size_t)c->n_pages * sizeof(int));
  l.last = l.row + up256((size_t)f->rows * sizeof(int4));
  l.fresh = l.last + up256((size_t)f->rows * sizeof(int2));
  l.bytes = l.fresh + up256((size_t)c->n_pages * sizeof(int));
  return l;
}

struct CompactLayout { size_t from, to, sums, bytes; };
CompactLayout compact_layout(const waveal_cache_desc* c) {
  CompactLayout l;
  l.sums = 0;
  l.from = up256((kCluster + 1) * sizeof(int));
  l.to = l.from + up256((size_t)c->n_pages * sizeof(int));
  l.bytes = l.to + up256((size_t)c->n_pages * sizeof(int));
  return l;
}

waveal_status check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return waveal::fail(WAVEAL_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : 0, need);
  if (!waveal::aligned(ws, 256)) return waveal::fail(WAVEAL_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return WAVEAL_OK;
}

waveal_status check_tensors(const void* k, const void* v) {
  if (!k || !v) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "the caches' keys and values are required");
  if (!waveal::aligned(k, 2) || !waveal::aligned(v, 2)) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "a tensor is not aligned to its element");
  return WAVEAL_OK;
}

// (behind all other checks)
waveal_status check_device() {
  return waveal::sm_count() > 0 ? WAVEAL_OK : waveal::fail(WAVEAL_ERR_CUDA, "number of SMs not available");
}

}  // namespace

extern "C" waveal_status waveal_cache_copy(const waveal_cache_desc* to, const waveal_cache_desc* from, int32_t count, const void* from_k,
                                           const void* from_v, void* to_k, void* to_v, const int32_t* from_pages, const int32_t* to_pages,
                                           int32_t* dev_status, void* cuda_stream) {
  if (waveal_status e = check_pool(to)) return e;
  if (waveal_status e = check_pool(from)) return e;
  if (to->page_size != from->page_size || to->kv_heads != from->kv_heads || to->head_dim != from->head_dim || to->dtype != from->dtype)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "the caches differ in page_size, kv_heads, head_dim or dtype");
  if (count < 0) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "count must not be negative");
  if (count == 0) {
    waveal::launch_counter() = 0;
    return WAVEAL_OK;
  }
  if (!from_pages || !to_pages) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "from_pages and to_pages are required");
  if (waveal_status e = check_tensors(from_k, from_v)) return e;
  if (waveal_status e = check_tensors(to_k, to_v)) return e;
  if (waveal_status e = check_device()) return e;
  CopyParams p = {};
  const bool wide = page_shape(p.shape, p.t, from, from_k, from_v, to, to_k, to_v);
  p.from_pages = from_pages, p.to_pages = to_pages, p.count = count;
  p.from_n = from->n_pages, p.to_n = to->n_pages, p.dev_status = dev_status;
  const unsigned grid = copy_grid(2ll * p.shape.segments * count);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (wide) k_copy_pages<uint4><<<grid, kCopyThreads, 0, st>>>(p);
  else k_copy_pages<unsigned short><<<grid, kCopyThreads, 0, st>>>(p);
  WAVEAL_CUDA_OK(cudaGetLastError());
  waveal::launch_counter() = 1;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_cache_fork_workspace_bytes(const waveal_cache_desc* cache, const waveal_fork_desc* fork, size_t* bytes) {
  if (!bytes) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "bytes is NULL");
  if (waveal_status e = check_fork(cache, fork)) return e;
  *bytes = fork_layout(cache, fork).bytes;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_cache_fork(const waveal_cache_desc* c, const waveal_fork_desc* f, void* k_cache, void* v_cache,
                                           const int32_t* old_table, const int32_t* held_len, const int32_t* page_refs, const int32_t* parents,
                                           const int32_t* keep_len, const int32_t* room_len, int32_t* table, int32_t* new_refs, void* ws,
                                           size_t ws_bytes, int32_t* dev_status, void* cuda_stream) {
  if (waveal_status e = check_fork(c, f)) return e;
  if (!page_refs || !new_refs || (f->old_rows && !held_len) || (f->old_rows && f->old_pages && !old_table) || (f->rows && (!keep_len || !room_len)) ||
      (f->rows && f->pages && !table))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "page_refs and new_refs are required, held_len and old_table with old rows, keep_len, room_len and table "
                                                "with rows");
  if (!parents && f->rows && f->rows != f->old_rows) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "without parents there are as many rows as before");
  if (waveal_status e = check_tensors(k_cache, v_cache)) return e;
  const size_t refs = (size_t)c->n_pages * sizeof(int);
  if (overlap(page_refs, refs, new_refs, refs) ||
      overlap(old_table, table_bytes(f->old_rows, f->old_pages, f->old_stride), table, table_bytes(f->rows, f->pages, f->stride)))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "the new table and counts must not lie over the old ones");
  const ForkLayout l = fork_layout(c, f);
  if (waveal_status e = check_workspace(ws, ws_bytes, l.bytes)) return e;
  if (waveal_status e = check_device()) return e;
  ForkParams p = {};
  const bool wide = page_shape(p.shape, p.t, c, k_cache, v_cache, c, k_cache, v_cache);
  p.old_rows = f->old_rows, p.rows = f->rows, p.old_pages = f->old_pages, p.pages = f->pages, p.n_pages = c->n_pages;
  p.old_stride = f->old_stride, p.stride = f->stride;
  p.old_table = old_table, p.held = held_len, p.refs = page_refs, p.parents = parents, p.keep = keep_len, p.room = room_len;
  p.table = table, p.new_refs = new_refs;
  char* w = static_cast<char*>(ws);
  p.sums = reinterpret_cast<int*>(w + l.sums), p.free_pages = p.sums + 2 * kCluster;
  p.kids = reinterpret_cast<int*>(w + l.kids), p.ends = reinterpret_cast<int*>(w + l.ends);
  p.row = reinterpret_cast<int4*>(w + l.row), p.last = reinterpret_cast<int2*>(w + l.last), p.fresh = reinterpret_cast<int*>(w + l.fresh);
  p.dev_status = dev_status;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  static Leave leave[2][64] = {};
  const size_t state = fork_state_bytes(c->n_pages, f->old_rows, f->rows);
  const int blocks = fork_blocks(fork_work(c->n_pages, f), state);
  if (waveal_status e = blocks == 1 ? launch_plan(k_fork_plan<true>, leave[1], p, 1, state, st) : launch_plan(k_fork_plan<false>, leave[0], p, blocks, 0, st)) return e;
  const unsigned grid = copy_grid((long long)f->rows * (2 * p.shape.segments + (f->pages + kRun - 1) / kRun));
  if (wide) WAVEAL_CUDA_OK(waveal::launch_chained(k_fork_apply<uint4>, dim3(grid), kCopyThreads, 0, st, p));
  else WAVEAL_CUDA_OK(waveal::launch_chained(k_fork_apply<unsigned short>, dim3(grid), kCopyThreads, 0, st, p));
  waveal::launch_counter() = 2;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_cache_compact_workspace_bytes(const waveal_cache_desc* cache, size_t* bytes) {
  if (!bytes) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "bytes is NULL");
  if (waveal_status e = check_pool(cache)) return e;
  if (waveal_status e = check_counts(cache, 0, 0, 0, 0)) return e;
  *bytes = compact_layout(cache).bytes;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_cache_compact(const waveal_cache_desc* c, const waveal_compact_desc* d, void* k_cache, void* v_cache,
                                              const int32_t* page_refs, const int32_t* old_table, const int32_t* old_prefix, int32_t* new_refs,
                                              int32_t* table, int32_t* prefix, int32_t* place, int32_t* used, void* ws, size_t ws_bytes,
                                              void* cuda_stream) {
  if (waveal_status e = check_pool(c)) return e;
  if (!d) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "compact is NULL");
  if (d->rows < 0 || d->pages < 0 || d->prefix_pages < 0)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "rows, pages and prefix_pages must not be negative");
  if (waveal_status e = check_counts(c, d->rows, 0, d->pages, 0)) return e;
  if (d->old_stride < d->pages || d->stride < d->pages) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "a table's stride is smaller than its pages");
  if ((long long)d->rows * d->pages > INT_MAX) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^31 - 1 entries in a table");
  const bool has_table = d->rows && d->pages;
  if (!page_refs || !new_refs || !place || !used || (has_table && (!old_table || !table)) || (d->prefix_pages && (!old_prefix || !prefix)))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "page_refs, new_refs, place and used are required, both tables with rows, both lists with prefix_pages");
  if (waveal_status e = check_tensors(k_cache, v_cache)) return e;
  const size_t refs = (size_t)c->n_pages * sizeof(int), list = (size_t)d->prefix_pages * sizeof(int);
  if (overlap(page_refs, refs, new_refs, refs) || overlap(old_prefix, list, prefix, list) ||
      overlap(old_table, table_bytes(d->rows, d->pages, d->old_stride), table, table_bytes(d->rows, d->pages, d->stride)))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "the new tables and counts must not lie over the old ones");
  const CompactLayout l = compact_layout(c);
  if (waveal_status e = check_workspace(ws, ws_bytes, l.bytes)) return e;
  if (waveal_status e = check_device()) return e;
  CompactParams p = {};
  const bool wide = page_shape(p.shape, p.t, c, k_cache, v_cache, c, k_cache, v_cache);
  p.rows = d->rows, p.pages = d->pages, p.n_pages = c->n_pages, p.prefix = d->prefix_pages;
  p.old_stride = d->old_stride, p.stride = d->stride;
  p.refs = page_refs, p.old_table = old_table, p.old_prefix = old_prefix;
  p.new_refs = new_refs, p.table = table, p.new_prefix = prefix, p.place = place, p.used = used;
  char* w = static_cast<char*>(ws);
  p.sums = reinterpret_cast<int*>(w + l.sums), p.first = p.sums + kCluster;
  p.from = reinterpret_cast<int*>(w + l.from), p.to = reinterpret_cast<int*>(w + l.to);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  static Leave leave[64] = {};
  if (waveal_status e = launch_plan(k_compact_plan, leave, p, compact_blocks(c->n_pages), 0, st)) return e;
  // (how many pages move is known on the device only: half of the pool at most)
  const unsigned grid = copy_grid((long long)(c->n_pages / 2) * 2 * p.shape.segments + (long long)d->rows * ((d->pages + kRun - 1) / kRun));
  if (wide) WAVEAL_CUDA_OK(waveal::launch_chained(k_compact_apply<uint4>, dim3(grid), kCopyThreads, 0, st, p));
  else WAVEAL_CUDA_OK(waveal::launch_chained(k_compact_apply<unsigned short>, dim3(grid), kCopyThreads, 0, st, p));
  waveal::launch_counter() = 2;
  return WAVEAL_OK;
}
