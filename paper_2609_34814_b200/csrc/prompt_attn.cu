// Attention of whole prompts: every token over its own sequence, causal or not, grouped heads, any lengths in one call.
//
//   o[h, t] = sum_j p_j v_j / sum_j p_j,   p_j = 2^(sl2 (q[h, t] . k_j - m)),   sl2 = scale log2(e),   j over what token t sees.
// Any m gives the same o as long as nothing overflows or vanishes.  A row's m is the largest of its first 16 scores, so that no tile of keys
// waits for another one's maximum; what overflows shows in the results, and such a row tile is computed again with maxima of every tile (m
// follows when a maximum has outgrown it by more than 2^8, O and the sum are scaled).
//
// A row tile is 128 rows of S: tq = 128 / G tokens with the G query heads that share a key head, so that a key head's tiles are
// loaded once for all of them and the causal diagonal crosses few of a tile's columns.  A thread block takes row tiles one after another (a ticket
// each, the ones with most keys first), and their key tiles of 128 as one stream:
//   S = Q K^T (one of three buffers in tensor memory) -> exponentials, P over S's columns -> O += P V (tensor memory).
// Two teams of eight warps take the tiles of the stream in turn, also across row tiles: one row tile's end (its last products, its
// results on their way out) runs beside the next one's first tiles.
//
// Warps: 0-7 and 8-15 the teams (two threads a row, 64 keys of a tile each: a warp by itself issues an instruction in four clocks, so
// that four of them a scheduler are needed), 16 items, Q and K, 17 and 18 products, 19 V, 20-23 results.
//
// What bounds it: a tile of 128 x 128 at head_dim 128 is 1,024 clk of the tensor pipe and 1,024 clk of the exponentials' unit, and takes 1,370 to
// 1,450; the rest is the way round of a buffer (products, 1,950 clk of a team's softmax, products) through three buffers, which is all that tensor
// memory holds beside O.  In a row of calls, under the power cap, with the SM clock that was sampled meanwhile / in the first 4 ms after a pause:
//   32,760 causal tokens, 32 query and 8 key heads          7.4 ms at 1,387 MHz / 6.2 to 6.6     1,180 TFLOP/s: 86 % of a library product kept up, 71 % of its burst
//   16 prompts of 20 to 2,000 tokens, the same heads        195 us at 1,470 MHz / 169            11,400 clk a row tile of 5.8 key tiles: 3,000 beside the loop's pace
//   6 frames of 1,560 tokens, 40 heads, not causal          328 us at 1,432 MHz / 287            910 TFLOP/s; 13 key tiles whose last one has 24 keys, 22 turns of row tiles
//   150 prompts of up to 700 tokens, head_dim 64, fp16      228 us at 1,687 MHz / 196            4,700 clk a row tile of 2.4 key tiles
// Short row tiles: a team needs 2,100 to 2,700 clk for a row tile's first or last tile (reference, mask, exponentials) and 700 to get to the next one.
// The same 32,760 tokens on the way here: the row's scores in registers of one thread, 11.4 ms (its code did not fit the instruction caches: 4.2 warps
// an issue waited for instructions); rolled loops that read S twice, 8.5; products issued by two warps, 7.9; two threads a row, 7.2; three buffers and
// one stream, 6.8; results by warps of their own, 6.7; tiles without a mask or a first score apart, 6.55.  Without gain: polynomials for an eighth to three
// eighths of the exponentials, waits that sleep, results through shared memory, loads of S ahead of their use in pieces of 16 columns, masks applied in
// registers, items made by a warp of their own (a 25th: all have 72 registers then), products of a cut tile without a loop.
//
// Values that a token must not see: their probabilities are zero, but zero times NaN is not.  A row tile whose results are not finite is computed
// again: then warp 19 writes zeros over what lies behind a sequence's end and looks through the values of tiles that the causal mask cuts; where one is
// not finite, the softmax warps add that tile's products themselves, each row's visible keys alone.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>
#include "host_common.h"
#include "sm100.h"

namespace {

using namespace waveal::sm100;

constexpr int kThreads = 768;
constexpr int kLoadWarp = 16, kScoreWarp = 17, kProductWarp = 18, kValueWarp = 19;
constexpr int kTile = 128;                           // keys of a tile, rows of a row tile
constexpr int kItems = 4;                            // row tiles under way: their descriptions, references and sums
constexpr int kItemReaders = 23;                     // two issuers, the V loader, sixteen softmax warps, four for the results
constexpr int kChecks = 8;                           // masked tiles whose verdicts are under way (more than the ring has V tiles)
constexpr long long kTimeoutCycles = 4000000000ll;   // ~2 s at boost clock
constexpr long long kSelfTestCycles = 4000000ll;     // ~2 ms
constexpr float kGrowth = 8.0f;                      // log2 of how far a row's maximum may outgrow its reference
// Most row tiles need only one reference: that of their first tile of keys.  Nothing is lost while no number overflows: P of bf16, the sums and O
// have the range of fp32, P of fp16 has 2^16.  What overflows shows in the results: an element of O is not finite, or a sum beyond what divides well.
constexpr float kSumLimit = 0x1p100f;

template <int D> struct Geo {
  static constexpr int SLABS = D / 64;               // 128-byte-swizzled slabs of 64 channels
  static constexpr int SLAB_BYTES = kTile * 128;
  static constexpr int TILE_BYTES = SLABS * SLAB_BYTES;
  static constexpr int NKS = D == 128 ? 2 : 4, NVS = NKS;   // stages of the rings of K and V tiles
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + NKS * TILE_BYTES, OFF_END = OFF_V + NVS * TILE_BYTES;
  static constexpr int S_COL = 0, O_COL = 384;       // tensor memory: S (and P) 0-127, 128-255, 256-383, O 384..
  static constexpr int OS = D == 128 ? 1 : 2;        // accumulators: at head_dim 64 two row tiles have one each
};

// ------------------------------------------------------------------ what there is to do

// In the workspace, made by the planning kernel: the sequences by descending length (row tiles; longer ones than 1,022 row tiles in any
// order), each with the number of row tiles of the ones in front of it.
struct Plan {
  int4* seq;               // [batch] {first token, tokens, row tiles in front, 0}
  int* again;              // [tickets]: chains of row tiles that are computed again (each with the one before it)
  int* head;               // [4] {row tiles of all sequences, tickets given out, sequences with tokens, 0}
};

struct Params {
  Plan plan;
  const int *seq_start, *seq_len;
  int batch, tokens, kv_heads, group, tq, causal;
  void* o;
  float* lse;
  long long o_stride_h, o_stride_t;
  int* dev_status;
  long long wait_limit;
  int drop_tile, wide_o;   // wide_o: o in 32-byte pieces
  int direct;              // no planning kernel: a row tile a thread block at most, of 32 sequences at most
  float sl2;               // scale * log2(e)
};

__host__ __device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

__device__ __noinline__ void report(int* status, int code, int site, int where, int value) {
  if (status && atomicCAS(status, 0, code) == 0) status[1] = site, status[2] = where, status[3] = value;
}

// {first token, tokens}; none of a malformed sequence (-1: its starts are)
__device__ inline int2 read_sequence(const Params& p, int b, bool tell) {
  const int start = p.seq_start[b], end = p.seq_start[b + 1];
  if (start < 0 || end < start || end > p.tokens) {
    if (tell) report(p.dev_status, WAVEAL_ERR_BAD_MASK, 100, b, start < 0 ? start : end);
    return make_int2(0, -1);
  }
  int n = end - start;
  if (p.seq_len) {
    const int len = p.seq_len[b];
    if (len < 0 || len > n) {
      if (tell) report(p.dev_status, WAVEAL_ERR_BAD_MASK, 101, b, len);
      return make_int2(0, 0);
    }
    n = len;
  }
  return make_int2(start, n);
}

constexpr int kPlanThreads = 1024;

// of the threads in front of this one; total: of all (two barriers; shared: 32 words)
__device__ __forceinline__ int scan_block(int x, int* shared, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  int upto = x;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  __syncthreads();
  if (lane == 31) shared[warp] = upto;
  __syncthreads();
  int sums = shared[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, sums, d);
    if (lane >= d) sums += y;
  }
  total = __shfl_sync(0xffffffffu, sums, 31);
  const int before = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
  return upto - x + (warp ? before : 0);
}

// One thread block sorts the sequences and adds up their row tiles: latency, hidden in part behind the start of the attention kernel's blocks.
__global__ void __launch_bounds__(kPlanThreads, 1) k_prompt_plan(const __grid_constant__ Params p) {
  __shared__ int count[kPlanThreads], shared[32], malformed;
  waveal::let_next_kernel_start();
  count[threadIdx.x] = 0;
  if (threadIdx.x == 0) malformed = 0;
  __syncthreads();
  // bucket 0: the longest; the last one: no tokens
  auto bucket = [&](int n) { return kPlanThreads - 1 - min(ceil_div(n, p.tq), kPlanThreads - 1); };
#pragma unroll 1
  for (int b = threadIdx.x; b < p.batch; b += kPlanThreads) {
    const int n = read_sequence(p, b, true).y;
    if (n < 0) malformed = 1;
    atomicAdd(&count[bucket(max(n, 0))], 1);
  }
  __syncthreads();
  int total;
  const bool some_left_out = malformed;
  if (some_left_out) {
    // Starts that go back would let sequences claim the same tokens, and make more row tiles than the workspace has places for: a
    // sequence that begins in front of an earlier start has no tokens either (said in the places of the chains, of which there are more than sequences).
    int top = -1;
#pragma unroll 1
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
      const int b = b0 + threadIdx.x, start = b < p.batch ? p.seq_start[b] : -1;
      __syncthreads();
      count[threadIdx.x] = start > p.tokens ? -1 : start;
      __syncthreads();
#pragma unroll 1
      for (int d = 1; d < kPlanThreads; d *= 2) {
        const int y = threadIdx.x >= d ? count[threadIdx.x - d] : -1;
        __syncthreads();
        count[threadIdx.x] = max(count[threadIdx.x], y);
        __syncthreads();
      }
      if (b < p.batch) p.plan.again[b] = max(top, count[threadIdx.x]) > start;
      top = max(top, count[kPlanThreads - 1]);
    }
    __syncthreads();
    count[threadIdx.x] = 0;
    __syncthreads();
  }
  auto sequence = [&](int b) {
    const int2 q = read_sequence(p, b, false);
    return q.y <= 0 || (some_left_out && p.plan.again[b]) ? make_int2(0, 0) : q;
  };
  if (some_left_out) {
#pragma unroll 1
    for (int b = threadIdx.x; b < p.batch; b += kPlanThreads) atomicAdd(&count[bucket(sequence(b).y)], 1);
    __syncthreads();
  }
  const int first = scan_block(count[threadIdx.x], shared, total);
  __syncthreads();
  count[threadIdx.x] = first;
  if (threadIdx.x == kPlanThreads - 1) p.plan.head[2] = first;
  __syncthreads();
#pragma unroll 1
  for (int b = threadIdx.x; b < p.batch; b += kPlanThreads) {
    const int2 q = sequence(b);
    p.plan.seq[atomicAdd(&count[bucket(q.y)], 1)] = make_int4(q.x, q.y, 0, 0);
  }
  __syncthreads();
  int tiles = 0;
#pragma unroll 1
  for (int r0 = 0; r0 < p.batch; r0 += kPlanThreads) {
    const int r = r0 + threadIdx.x, mine = r < p.batch ? ceil_div(p.plan.seq[r].y, p.tq) : 0;
    const int at = tiles + scan_block(mine, shared, total);
    if (r < p.batch) p.plan.seq[r].z = at;
    tiles += total;
  }
  if (threadIdx.x == 0) p.plan.head[0] = tiles, p.plan.head[1] = 0;
}

// The plan of at most 32 sequences, one a lane, in their own order (row tiles that have a thread block each are in no need of another): what Plan::seq
// would hold, sequences without tokens included, which share their number with the next one.
__device__ inline int4 plan_few(const Params& p, int lane, int& row_tiles) {
  const bool tell = blockIdx.x == 0;
  int2 q = lane < p.batch ? read_sequence(p, lane, tell) : make_int2(0, 0);
  if (__any_sync(0xffffffffu, q.y < 0)) {              // (as the planning kernel does)
    const int start = lane < p.batch ? p.seq_start[lane] : -1;
    int top = start > p.tokens ? -1 : start;
#pragma unroll 1
    for (int d = 1; d < 32; d *= 2) {
      const int y = __shfl_up_sync(0xffffffffu, top, d);
      if (lane >= d) top = max(top, y);
    }
    if (top > start) q.y = 0;
  }
  q.y = max(q.y, 0);
  const int mine = ceil_div(q.y, p.tq);
  int upto = mine;
#pragma unroll 1
  for (int d = 1; d < 32; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  row_tiles = __shfl_sync(0xffffffffu, upto, 31);
  return make_int4(q.x, q.y, upto - mine, 0);
}

// A row tile of a sequence and key head.
struct Item {
  int end;                 // 1: nothing left; 2: everyone says when all items before this one are done
  int ticket;
  int safe;                // maxima of every tile, all of them by one team
  int tiles;               // of keys
  int teams;               // bits: who has any of them
  int masked;              // the first of them that a mask cuts
  int head;                // key head
  int token, n;            // first token, tokens
  int key, keys;           // first token of the sequence; how many of its tokens any row sees
  int sees;                // how many the first token sees (causal: every token one more)
  int len;                 // tokens of the sequence
  long long o;             // the first token and query head in o
};

// 32 of the planned sequences, one a lane, from number `base` on.  A thread block's tickets ascend, so that most of them fall among those that the loading
// warp holds already: a search in memory is three loads one after the other, which cost 2,400 of an item's 5,500 clk where items are short.
struct Window {
  int4 seq;
  int base;
};

// Row tile number `ticket` (a whole warp calls it): sequence by sequence, the ones with most keys first, all key heads of a place after each other.
__device__ inline void make_item(const Params& p, int sequences, int ticket, Window& win, Item& im, int lane) {
  const int u = ticket / p.kv_heads;
  im.end = 0, im.safe = 0, im.ticket = ticket;
  im.head = ticket - u * p.kv_heads;
  // the last sequence that begins at u or in front of it
  uint32_t in = __ballot_sync(0xffffffffu, win.base + lane < sequences && win.seq.z <= u);
  if (in == 0 || (in == 0xffffffffu && win.base + 32 < sequences)) {
    // (every step cuts the range to a 32nd)
    int lo = 0, hi = sequences;
#pragma unroll 1
    while (hi - lo > 1) {
      const int step = ceil_div(hi - lo, 32), at = lo + lane * step;
      const int last = 31 - __clz(__ballot_sync(0xffffffffu, at < hi && __ldcg(&p.plan.seq[at].z) <= u));
      hi = min(hi, lo + (last + 1) * step);
      lo += last * step;
    }
    win.base = lo;
    win.seq = __ldcg(p.plan.seq + min(lo + lane, sequences - 1));
    in = 1;
  }
  const int from = 31 - __clz(in);
  const int4 q = make_int4(__shfl_sync(0xffffffffu, win.seq.x, from), __shfl_sync(0xffffffffu, win.seq.y, from), __shfl_sync(0xffffffffu, win.seq.z, from), 0);
  const int first = (ceil_div(q.y, p.tq) - 1 - (u - q.z)) * p.tq;
  im.n = min(p.tq, q.y - first);
  im.token = q.x + first;
  im.key = q.x, im.len = q.y;
  im.keys = p.causal ? first + im.n : q.y;
  im.sees = p.causal ? first + 1 : q.y;
  im.tiles = ceil_div(im.keys, kTile);
  im.masked = im.sees / kTile;
  im.o = (long long)im.head * p.group * p.o_stride_h + (long long)im.token * p.o_stride_t;
}

// ------------------------------------------------------------------ kernel

struct Ctx {
  volatile int* abort_smem;
  int* dev_status;
  long long limit;
};

// bounded wait; false = gave up (this CTA is leaving)
__device__ __noinline__ bool wait_slow(const Ctx& c, uint32_t bar, uint32_t parity, int site) {
  const long long t0 = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*c.abort_smem) return false;
    if (clock64() - t0 > c.limit) {
      *c.abort_smem = 1;
      report(c.dev_status, WAVEAL_ERR_TIMEOUT, site, blockIdx.x, threadIdx.x);
      return false;
    }
  }
}
__device__ __forceinline__ bool warp_wait(const Ctx& c, uint32_t bar, uint32_t parity, int site) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, wait_slow(c, bar, parity, site));
}

// Two numbers in the tensors' type: the results, and the probabilities, because one product of 16-bit types takes both operands in the
// same type and V is stored in this one.  Either is off by half a step of its own; the sums are taken before the rounding, in fp32.
template <class T> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <class T> __device__ __forceinline__ float2 unpack2(uint32_t x) {
  if constexpr (std::is_same_v<T, __half>) {
    return __half22float2(*reinterpret_cast<__half2*>(&x));
  } else {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
}
// two 16-bit numbers: is one of them infinite or NaN (all bits of its exponent set)
template <class T> __device__ __forceinline__ bool not_finite2(uint32_t x) {
  constexpr uint32_t m = std::is_same_v<T, __half> ? 0x7c00u : 0x7f80u;
  return (x & m) == m || (x & m << 16) == m << 16;
}

constexpr int kBuffers = 3;                          // of S
enum {
  B_ITEM_FULL = 0, B_ITEM_EMPTY = B_ITEM_FULL + kItems, B_Q_FULL = B_ITEM_EMPTY + kItems, B_Q_EMPTY = B_Q_FULL + 2,
  B_S_FULL = B_Q_EMPTY + 2,                          // twice as many as buffers: a barrier's phases are waited for by one team, in turn
  B_S_FREE = B_S_FULL + 2 * kBuffers, B_P = B_S_FREE + kBuffers, B_O_EMPTY = B_P + kBuffers, B_O_FULL = B_O_EMPTY + 2,
  B_REF = B_O_FULL + 2, B_PV_DONE = B_REF + kItems, B_PAIR = B_PV_DONE + 2, B_CHECK = B_PAIR + 8, B_FINAL = B_CHECK + 2 * kChecks, B_DONE = B_FINAL + 2,
  B_K_FULL
};
template <int D> constexpr int kBars = B_K_FULL + 2 * (Geo<D>::NKS + Geo<D>::NVS);

// Where P of 16 keys lies among the columns of its S: keys 0-31 at 48, 32-63 at 32, 64 on at 64.  It covers scores that its own threads have
// read (the second half of keys 0-63 first); columns 0-31 keep theirs, which all threads take the reference from.
__device__ __forceinline__ int p_column(int group) { return group < 4 ? 32 + (group ^ 2) * 8 : 32 + group * 8; }

// what lies behind the tiles in shared memory
template <int D> struct Small {
  unsigned long long bar[kBars<D>];
  Item items[kItems];
  float ref[kItems][kTile];                          // of the rows, from the team of the first tile
  float sums[kItems][2][2][kTile];                   // [item][team][half][row]
  float pair[2][2][2][kTile];                        // [team][turn][half][row]: maxima, from a row's one thread to its other
  int verdict[2][kChecks];                           // not every value of the team's masked tile is finite
  uint32_t tmem;
  int abort;
  int again;                                         // row tiles to be computed again: the last one of the chain
  int chained[kItems];                               // the row tile that a warp of the results has put into the chain from here, so that no other does
};

// a ring of tiles as one of its users walks it
template <int STAGES> struct Ring {
  uint32_t stage = 0, phase = 0;
  __device__ void next() {
    if (++stage == (uint32_t)STAGES) stage = 0, phase ^= 1;
  }
};

// A masked tile some of whose values are not finite: the row's sum over the keys that it sees, added to its accumulator (first: written).
// P is read back from tensor memory, as the products would take it.
template <int D, class T>
__device__ __noinline__ void add_visible(uint32_t p_addr, uint32_t o_addr, uint32_t v_smem, int visible, int first) {
  using G = Geo<D>;
#pragma unroll 1
  for (int c = 0; c < D; c += 8) {
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll 1
    for (int k = 0; k < kTile; k += 2) {
      uint32_t pk;
      asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(pk) : "r"(p_addr + p_column(k / 16) + k % 16 / 2) : "memory");
      asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(pk)::"memory");
      const float2 pr = unpack2<T>(pk);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int key = k + x;
        // (128-byte swizzle: 16-byte chunk i of row r lies at chunk i ^ (r & 7))
        const uint32_t a = v_smem + c / 64 * G::SLAB_BYTES + key * 128 + ((c % 64 / 8) ^ (key & 7)) * 16;
        uint32_t w[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a));
        if (key < visible) {
          const float pv = x ? pr.y : pr.x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 v = unpack2<T>(w[i]);
            acc[2 * i] += pv * v.x, acc[2 * i + 1] += pv * v.y;
          }
        }
      }
    }
    uint32_t o[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]) : "r"(o_addr + c) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(o[0]), "+r"(o[1]), "+r"(o[2]), "+r"(o[3]), "+r"(o[4]), "+r"(o[5]), "+r"(o[6]), "+r"(o[7])::"memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(first ? acc[i] : __uint_as_float(o[i]) + acc[i]);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]), "r"(o_addr + c) : "memory");
  }
  tc_wait_st();
}

// two products with A in tensor memory, 8 columns further, and B 16 keys further
__device__ __forceinline__ void umma2_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .b32 rx, a;\n\t.reg .pred e, p, t;\n\t.reg .b64 b;\n\t"
      "elect.sync rx|e, 0xFFFFFFFF;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, %3, %3;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "add.u32 a, %1, 8;\n\tadd.s64 b, %2, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// O of this thread's row times `scale`
template <int D> __device__ __noinline__ void rescale(uint32_t o_addr, float scale) {
#pragma unroll 1
  for (int c = 0; c < D; c += 16) {
    uint32_t v[16];
    WAVEAL_TMEM_LD16(o_addr + c, v, 0);
    WAVEAL_TMEM_WAIT_LD16(v, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * scale);
    WAVEAL_TMEM_ST16(o_addr + c, v, 0);
  }
  tc_wait_st();
}

template <int D, class T>
__global__ void __launch_bounds__(kThreads, 1)
k_prompt_attn(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              const __grid_constant__ Params p) {
  using G = Geo<D>;
  constexpr int B_K_EMPTY = B_K_FULL + G::NKS, B_V_FULL = B_K_EMPTY + G::NKS, B_V_EMPTY = B_V_FULL + G::NVS;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  Small<D>& sm = *reinterpret_cast<Small<D>*>(smem + G::OFF_END);
  const uint32_t bars = smem_u32(sm.bar);
  auto BAR = [&](int i) { return bars + 8 * i; };
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;

  if (warp == 1) {
    tmem_alloc(smem_u32(&sm.tmem), 512);
    tmem_relinquish();
  } else if (warp == 2) {
#pragma unroll 1
    for (int i = lane; i < kBars<D>; i += 32) {
      auto within = [&](int from, int to) { return i >= from && i < to; };
      int arrivals = 1;
      if (within(B_ITEM_EMPTY, B_Q_FULL)) arrivals = kItemReaders;
      else if (i == B_DONE) arrivals = 20;                                                   // softmax and results
      else if (within(B_P, B_O_EMPTY)) arrivals = 8;                                         // a team
      else if (within(B_REF, B_PV_DONE) || within(B_O_EMPTY, B_O_FULL)) arrivals = 4;        // half a team; results
      else if (within(B_PAIR, B_CHECK)) arrivals = 2;                                        // the two warps of 32 rows
      mbar_init(BAR(i), arrivals);
    }
    if (lane == 0) sm.abort = 0, sm.again = -1;
    if (lane < kItems) sm.chained[lane] = -1;
    fence_mbar_init();
  } else if (warp == 3 && lane == 0) {
    prefetch_tmap(&tmQ), prefetch_tmap(&tmK), prefetch_tmap(&tmV);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const Ctx ctx = {&sm.abort, p.dev_status, p.wait_limit};
  bool ok = true;

  // the next item, for everyone but the loader: false when there is none or a wait gave up
  uint32_t item_no = 0;
  const Item* im;
  auto next_item = [&] {
    const uint32_t at = item_no % kItems;
    if (!warp_wait(ctx, BAR(B_ITEM_FULL + at), item_no / kItems & 1, 110)) return ok = false;
    im = &sm.items[at];
    return im->end != 1;
  };
  auto item_done = [&] {
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(B_ITEM_EMPTY + item_no % kItems));
    ++item_no;
  };

  if (warp >= kLoadWarp) {
    auto landed = [&](uint32_t bar, uint32_t ph) {   // (no copy is left in flight, also where another warp has given up)
      const long long t0 = clock64();
#pragma unroll 1
      while (!mbar_try_wait(bar, ph) && clock64() - t0 < p.wait_limit / 4) {}
    };
    if (warp == kLoadWarp) {
      // ================================================================ items, Q, K
      Ring<G::NKS> ring;
      uint32_t k_no = 0, q_no = 0;
      waveal::wait_for_previous_kernel();
      Window win;
      win.base = 0;
      int row_tiles, sequences;
      if (p.direct) {
        win.seq = plan_few(p, lane, row_tiles);
        sequences = p.batch;
      } else {
        win.seq = __ldcg(p.plan.seq + min(lane, p.batch - 1));
        row_tiles = __ldcg(p.plan.head), sequences = __ldcg(p.plan.head + 2);
      }
      const long long tickets = (long long)row_tiles * p.kv_heads;
      // first every row tile, then a word to say that these were all, then those that are to be computed again, then the end
      int id = blockIdx.x < tickets ? (int)blockIdx.x : -1;
      bool again = false;
      uint32_t g2 = 0;                               // team of the next tile
      Item next;
      next.tiles = 0, next.end = 0;
#pragma unroll 1
      while (ok && next.end != 1) {
        int asked = 0;
        if (id >= 0) {
          if (lane == 0 && !again && !p.direct) asked = atomicAdd(p.plan.head + 1, 1);   // (used when this item's tiles have been asked for)
          make_item(p, sequences, id, win, next, lane);
          next.safe = again;
          next.teams = next.tiles > 1 && !again ? 3 : 1 << g2;
          if (!again) g2 = (g2 + next.tiles) & 1;
        } else {
          next.end = again ? 1 : 2, next.tiles = 0;
        }
        const uint32_t at = item_no % kItems;
        if (item_no >= kItems && !(ok = warp_wait(ctx, BAR(B_ITEM_EMPTY + at), (item_no / kItems & 1) ^ 1, 113))) break;
        if (lane == 0) {
          sm.items[at] = next;
          mbar_arrive(BAR(B_ITEM_FULL + at));
        }
        __syncwarp();
        ++item_no;
        if (next.tiles) {
          const uint32_t qb = q_no % 2, q_full = BAR(B_Q_FULL + qb);
          if (q_no >= 2 && !(ok = warp_wait(ctx, BAR(B_Q_EMPTY + qb), (q_no / 2 & 1) ^ 1, 112))) break;
          ++q_no;
          if (lane == 0) {
            mbar_expect_tx(q_full, p.tq * p.group * 128 * G::SLABS);
#pragma unroll
            for (int i = 0; i < G::SLABS; ++i)
              tma_load_3d(sbase + G::OFF_Q + qb * G::TILE_BYTES + i * G::SLAB_BYTES, &tmQ, i * 64, next.head * p.group, next.token, q_full);
          }
          __syncwarp();
        }
#pragma unroll 1
        for (int j = 0; j < next.tiles; ++j) {
          if (k_no >= (uint32_t)G::NKS && !(ok = warp_wait(ctx, BAR(B_K_EMPTY + ring.stage), ring.phase ^ 1, 111))) break;
          if (lane == 0 && !(p.drop_tile && blockIdx.x == 0 && k_no == 0)) {
            mbar_expect_tx(BAR(B_K_FULL + ring.stage), G::TILE_BYTES);
#pragma unroll
            for (int i = 0; i < G::SLABS; ++i)
              tma_load_3d(sbase + G::OFF_K + ring.stage * G::TILE_BYTES + i * G::SLAB_BYTES, &tmK, i * 64, next.head, next.key + j * kTile, BAR(B_K_FULL + ring.stage));
          }
          __syncwarp();
          ++k_no, ring.next();
        }
        if (next.end == 2) {
          if (!(ok = warp_wait(ctx, BAR(B_DONE), 0, 129))) break;
          again = true;
          id = *reinterpret_cast<volatile int*>(&sm.again);
        } else if (id >= 0) {
          const long long ticket = (long long)gridDim.x + __shfl_sync(0xffffffffu, asked, 0);
          id = again ? __ldcg(p.plan.again + id) : ticket < tickets && !p.direct ? (int)ticket : -1;
        }
      }
#pragma unroll 1
      for (uint32_t i = 0; i < (uint32_t)G::NKS && i < k_no; ++i) {
        const uint32_t n = k_no - 1 - i;
        if (!(p.drop_tile && blockIdx.x == 0 && n == 0)) landed(BAR(B_K_FULL + n % G::NKS), n / G::NKS & 1);
      }
#pragma unroll 1
      for (uint32_t i = 0; i < 2 && i < q_no; ++i) landed(BAR(B_Q_FULL + (q_no - 1 - i & 1)), (q_no - 1 - i) >> 1 & 1);
    } else if (warp <= kProductWarp) {
      // ================================================================ products
      // Two warps issue, one S = Q K^T, the other O += P V: what they do around the products (waits, ring positions) is a chain of 250 clk
      // and more for each group of them, and four products (256 clk) are all that the tensor pipe has queued.
      // (operands of the products come from shuffles, so that the compiler knows them to be the same in all lanes)
      constexpr uint32_t kTypeBits = (1u << 7) | (1u << 10), kType = std::is_same_v<T, __half> ? 0u : kTypeBits;
      constexpr uint32_t kQK = (make_idesc(128, 128, false) & ~kTypeBits) | kType, kPV = (make_idesc(128, D, true) & ~kTypeBits) | kType;
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      uint32_t b = 0, g2 = 0;                        // the tile's buffer, its number's last bit
      uint32_t uses = 0;                             // bits: how often each buffer has been used, modulo 2
      if (warp == kScoreWarp) {
        const uint64_t q_desc0 = make_desc(sbase + G::OFF_Q, 16, 1024), k_desc0 = make_desc(sbase + G::OFF_K, 16, 1024);
        Ring<G::NKS> ring;
        uint32_t items = 0, used = 0;
#pragma unroll 1
        while (ok && next_item()) {
          const int tiles = __shfl_sync(0xffffffffu, im->tiles, 0), safe = __shfl_sync(0xffffffffu, im->safe, 0);
          item_done();
          if (tiles == 0) continue;
          if (!(ok = warp_wait(ctx, BAR(B_Q_FULL + (items & 1)), items >> 1 & 1, 115))) break;
          const uint64_t qd = q_desc0 + (uint64_t)((items & 1) * (G::TILE_BYTES >> 4));
#pragma unroll 1
          for (int j = 0; j < tiles; ++j) {
            if (!(ok = warp_wait(ctx, BAR(B_K_FULL + ring.stage), ring.phase, 116))) break;
            const uint64_t kd = k_desc0 + (uint64_t)(ring.stage * (G::TILE_BYTES >> 4));
            const uint32_t s_col = tm + G::S_COL + b * kTile;
            // (S lies over an earlier tile's P: its P V is over)
            if ((used >> b & 1) && !(ok = warp_wait(ctx, BAR(B_S_FREE + b), (uses >> b & 1) ^ 1, 114))) break;
            used |= 1u << b, uses ^= 1u << b;
            tc_fence_after();
#pragma unroll
            for (int slab = 0; slab < G::SLABS; ++slab)
              umma4_ss(s_col, qd + (uint64_t)(slab * G::SLAB_BYTES >> 4), kd + (uint64_t)(slab * G::SLAB_BYTES >> 4), kQK, slab > 0);
            tc_commit(BAR(B_S_FULL + 2 * b + g2));
            tc_commit(BAR(B_K_EMPTY + ring.stage));
            ring.next();
            b = b == kBuffers - 1 ? 0 : b + 1;
            if (safe) b = b == kBuffers - 1 ? 0 : b + 1;
            else g2 ^= 1;
          }
          tc_commit(BAR(B_Q_EMPTY + (items & 1)));
          ++items;
        }
      } else {
        const uint64_t v_desc0 = make_desc(sbase + G::OFF_V, G::SLAB_BYTES, 1024);
        Ring<G::NVS> ring;
        uint32_t items = 0, checks[2] = {0, 0};
#pragma unroll 1
        while (ok && next_item()) {
          const int tiles = __shfl_sync(0xffffffffu, im->tiles, 0), safe = __shfl_sync(0xffffffffu, im->safe, 0);
          const int keys = __shfl_sync(0xffffffffu, im->keys, 0), masked = __shfl_sync(0xffffffffu, safe ? im->masked : INT_MAX, 0);
          item_done();
          if (tiles == 0) continue;
          const uint32_t ob = items % G::OS, o_col = tm + G::O_COL + ob * D;
#pragma unroll 1
          for (int j = 0; j < tiles; ++j) {
            if (!(ok = warp_wait(ctx, BAR(B_V_FULL + ring.stage), ring.phase, 117))) break;
            if (j == 0 && items >= G::OS && !(ok = warp_wait(ctx, BAR(B_O_EMPTY + ob), (items / G::OS & 1) ^ 1, 118))) break;
            const uint32_t s_col = tm + G::S_COL + b * kTile;
            const uint64_t vd = v_desc0 + (uint64_t)(ring.stage * (G::TILE_BYTES >> 4));
            int groups = min(kTile / 16, (keys - j * kTile + 15) / 16);   // of 16 keys that some row sees
            if (j >= masked) {
              const uint32_t c = checks[g2] % kChecks;
              if (!(ok = warp_wait(ctx, BAR(B_CHECK + g2 * kChecks + c), checks[g2] / kChecks & 1, 119))) break;
              if (__shfl_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&sm.verdict[g2][c]), 0)) groups = 0;
              ++checks[g2];
            }
            if (!(ok = warp_wait(ctx, BAR(B_P + b), uses >> b & 1, 120))) break;
            uses ^= 1u << b;
            tc_fence_after();
            if (groups == 8) {
              umma2_ts(o_col, s_col + 48, vd, kPV, j > 0);
              umma2_ts(o_col, s_col + 32, vd + 2 * 128, kPV, 1);
              umma4_ts(o_col, s_col + 64, vd + 4 * 128, kPV, 1);
            } else {
#pragma unroll 1
              for (int c = 0; c < groups; ++c) umma_bf16_ts(o_col, s_col + p_column(c), vd + (uint64_t)(c * 128), kPV, j > 0 || c > 0);
            }
            tc_commit(BAR(B_S_FREE + b));
            tc_commit(BAR(B_V_EMPTY + ring.stage));
            if (safe && j < tiles - 1) tc_commit(BAR(B_PV_DONE + g2));   // (waited for in front of the next tile)
            if (j == tiles - 1) tc_commit(BAR(B_O_FULL + ob));
            ring.next();
            b = b == kBuffers - 1 ? 0 : b + 1;
            if (safe) b = b == kBuffers - 1 ? 0 : b + 1;
            else g2 ^= 1;
          }
          ++items;
        }
      }
      // no product is still running when tensor memory is given back
      tc_commit(BAR(B_FINAL + warp - kScoreWarp));
      __syncwarp();
      landed(BAR(B_FINAL + warp - kScoreWarp), 0);
    } else if (warp == kValueWarp) {
      // ================================================================ V
      Ring<G::NVS> ring;
      uint32_t v_no = 0, g2 = 0, checks[2] = {0, 0};
#pragma unroll 1
      while (ok && next_item()) {
        const Item it = *im;
        item_done();
#pragma unroll 1
        for (int j = 0; j < it.tiles; ++j) {
          const uint32_t full = BAR(B_V_FULL + ring.stage), v = sbase + G::OFF_V + ring.stage * G::TILE_BYTES;
          if (v_no >= (uint32_t)G::NVS && !(ok = warp_wait(ctx, BAR(B_V_EMPTY + ring.stage), ring.phase ^ 1, 128))) break;
          if (lane == 0) {
            mbar_expect_tx(full, G::TILE_BYTES);
#pragma unroll
            for (int i = 0; i < G::SLABS; ++i) tma_load_3d(v + i * G::SLAB_BYTES, &tmV, i * 64, it.head, it.key + j * kTile, full);
          }
          __syncwarp();
          ++v_no;
          if (it.safe && j >= it.masked) {
            if (!(ok = warp_wait(ctx, full, ring.phase, 121))) break;
            const int len = it.len - j * kTile;      // rows of the tile that are the sequence's
            bool bad = false;
            if (p.causal) {
#pragma unroll 1
              for (int i = lane; i < min(len, kTile) * 8; i += 32) {
#pragma unroll
                for (int slab = 0; slab < G::SLABS; ++slab) {
                  uint32_t w[4];
                  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(v + slab * G::SLAB_BYTES + i * 16));
#pragma unroll
                  for (int k = 0; k < 4; ++k) bad |= not_finite2<T>(w[k]);
                }
              }
            }
            if (len < kTile) {
#pragma unroll
              for (int slab = 0; slab < G::SLABS; ++slab)
#pragma unroll 1
                for (int i = len * 8 + lane; i < kTile * 8; i += 32) st_shared_v4(v + slab * G::SLAB_BYTES + i * 16, 0, 0, 0, 0);
              fence_proxy_async();
            }
            const int verdict = __any_sync(0xffffffffu, bad);
            __syncwarp();
            if (lane == 0) {
              sm.verdict[g2][checks[g2] % kChecks] = verdict;
              mbar_arrive(BAR(B_CHECK + g2 * kChecks + checks[g2] % kChecks));
            }
            __syncwarp();
            ++checks[g2];
          }
          ring.next();
          if (!it.safe) g2 ^= 1;
        }
      }
#pragma unroll 1
      for (uint32_t i = 0; i < (uint32_t)G::NVS && i < v_no; ++i) landed(BAR(B_V_FULL + (v_no - 1 - i) % G::NVS), (v_no - 1 - i) / G::NVS & 1);
    } else {
      // ================================================================ results: a thread a row
      const int quad = warp & 3, r = quad * 32 + lane, tok = r / p.group, g = r - tok * p.group;
      T* const o0 = static_cast<T*>(p.o) + g * p.o_stride_h + tok * p.o_stride_t;
      uint32_t items = 0;
#pragma unroll 1
      while (ok && next_item()) {
        const int tiles = im->tiles, safe = im->safe, ticket = im->ticket;
        if (tiles == 0) {
          if (im->end == 2 && lane == 0) mbar_arrive(BAR(B_DONE));
          item_done();
          continue;
        }
        const uint32_t at = item_no % kItems, ob = items % G::OS, o_addr = tmem + ((uint32_t)(quad * 32) << 16) + G::O_COL + ob * D;
        const bool live = tok < im->n;
        T* const o = o0 + im->o;
        float* const lse = live && p.lse ? p.lse + (long long)(im->head * p.group + g) * p.tokens + im->token + tok : nullptr;
        if (!(ok = warp_wait(ctx, BAR(B_O_FULL + ob), items / G::OS & 1, 123))) break;
        ++items;
        tc_fence_after();
        // (of each team and half; safe: one team alone, by the number of the items' tiles in front; one tile: its team alone)
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (im->teams >> i & 1) sum += sm.sums[at][i][0][r] + sm.sums[at][i][1][r];
        const float ref = sm.ref[at][r], inv = sum == 0.f ? 0.f : __fdividef(1.0f, sum);
        float none0 = 0.f, none1 = 0.f;              // zero, NaN where something in O is not finite
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t u[32], w[16];
          WAVEAL_TMEM_LD32(o_addr + c, u, 0);
          WAVEAL_TMEM_WAIT_LD32(u, 0);
          if (c == D - 32) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(B_O_EMPTY + ob));
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x, y;
            ffma2(none0, none1, __uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]), 0.f, 0.f, none0, none1);
            ffma2(x, y, __uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]), inv, inv, 0.f, 0.f);
            w[i] = sum == 0.f ? 0u : pack2<T>(x, y);   // (O may be 0 times something)
          }
          // (a warp's rows lie far apart: every store is 32 lines to the memory pipe, so the fewer the better)
          if (live) {
            if (p.wide_o) {
              st_global_v8(o + c, w);
              st_global_v8(o + c + 16, w + 8);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(o + c + 8 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
            }
          }
        }
        if (lse) *lse = sum == 0.f ? -INFINITY : (ref * p.sl2 + __log2f(sum)) * 0.69314718055994531f;
        // O outgrew fp32 (V is very large), or met a value that the row does not see: neither happens in the other way
        const bool bad = !(sum < kSumLimit) || ref == -INFINITY || !(none0 + none1 == 0.f);
        // (once: the four warps may be several items apart, so every item's place has its own mark)
        if (__any_sync(0xffffffffu, bad && live && !safe) && lane == 0 && atomicExch(&sm.chained[at], ticket) != ticket)
          p.plan.again[ticket] = atomicExch(&sm.again, ticket);
        __syncwarp();
        item_done();
      }
    }
  } else {
    // ================================================================ softmax
    const uint32_t team = warp / 8;
    const int half = warp / 4 & 1, quad = warp & 3, r = quad * 32 + lane, tok = r / p.group;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16, tm = tmem + lanes;
    const float sl2 = p.sl2;
    uint32_t b = 0, g2 = 0;                          // buffer and number (its last bit) of the item's first tile
    uint32_t s_ph = 0;                               // bits: phases of this team's barriers of the buffers
    uint32_t items = 0, pairs = 0, checks = 0, done = 0, v_no = 0;
    // what the row's other thread has
    auto exchange = [&](float mine) {
      sm.pair[team][pairs & 1][half][r] = mine;
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_PAIR + team * 4 + quad));
      ok = warp_wait(ctx, BAR(B_PAIR + team * 4 + quad), pairs & 1, 122);
      return sm.pair[team][pairs++ & 1][half ^ 1][r];
    };
#pragma unroll 1
    while (ok && next_item()) {
      const int tiles = im->tiles, safe = im->safe;
      if (tiles == 0) {
        if (im->end == 2 && lane == 0) mbar_arrive(BAR(B_DONE));
        item_done();
        continue;
      }
      const uint32_t at = item_no % kItems, step = safe ? 2 : 1;
      const int keys = im->keys, first_sees = im->sees, masked = im->masked;
      const bool live = tok < im->n;
      const int sees = min(p.causal ? first_sees + tok : keys, keys) - half * 64;
      float ref = -INFINITY, minus = 0.f, s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
      const int plain = safe ? tiles : 2;            // from this tile on there is nothing to do but the exponentials, up to the first that a mask cuts
      const int j0 = g2 == team ? 0 : safe ? tiles : 1;
      uint32_t buf = (b + j0 * step) % kBuffers;
#pragma unroll 1
      for (int j = j0; j < tiles; j += 3 - step) {
        const uint32_t s_addr = tm + G::S_COL + buf * kTile, h_addr = s_addr + half * 64;
        if (!(ok = warp_wait(ctx, BAR(B_S_FULL + 2 * buf + team), s_ph >> buf & 1, 124))) break;
        s_ph ^= 1u << buf;
        tc_fence_after();
        int chunks = 2;                              // of this thread's 64 keys
        uint32_t u[32], w[16];
        const bool cut = j >= masked;
        if (j < plain || cut) {
          if (cut) {
            chunks = min(2, (keys - j * kTile - half * 64 + 31) / 32);   // (what is behind the last key is not used)
            // scores that the row does not see, 16 columns at a time from the first that some row does not see.  (Code that runs once or twice an
            // item is short: each 128 bytes of it come from beyond the instruction caches.)
            const int visible = sees - j * kTile, from = max(0, first_sees - j * kTile - half * 64) / 16 * 16;
#pragma unroll 1
            for (int c = from; c < 32 * chunks; c += 16) {
              uint32_t t[16];
              WAVEAL_TMEM_LD16(h_addr + c, t, 0);
              WAVEAL_TMEM_WAIT_LD16(t, 0);
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (i >= visible - c) t[i] = 0xff800000u;
              WAVEAL_TMEM_ST16(h_addr + c, t, 0);
            }
            tc_wait_st();
          }
          if (safe) {
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
              WAVEAL_TMEM_LD32(h_addr + 32 * c, u, 0);
              WAVEAL_TMEM_WAIT_LD32(u, 0);
              top = fmaxf(top, row_max32(u));
            }
            top = fmaxf(top, exchange(top));
            if (!ok) break;
            if (j == 0) {
              ref = top;
            } else {
              if (!(ok = warp_wait(ctx, BAR(B_PV_DONE + team), done++ & 1, 130))) break;   // of the last tile
              tc_fence_after();
              const bool grown = live && (top - ref) * sl2 > kGrowth;
              if (__any_sync(0xffffffffu, grown)) {
                const float scale = grown ? ex2((ref - top) * sl2) : 1.0f;
                if (grown) ref = top;
                s0 *= scale, s1 *= scale, s2 *= scale, s3 *= scale;
                rescale<D / 2>(tm + G::O_COL + items % G::OS * D + half * (D / 2), scale);
              }
            }
          } else if (j == 0) {
            // the largest of the first 16 scores: both threads of a row find the same
            uint32_t t[16];
            WAVEAL_TMEM_LD16(s_addr, t, 0);
            WAVEAL_TMEM_WAIT_LD16(t, 0);
            const int visible = sees + half * 64;
            ref = __uint_as_float(t[0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) ref = fmaxf(ref, i < visible ? __uint_as_float(t[i]) : -INFINITY);
            if (half == 0) {
              sm.ref[at][r] = ref;
              __syncwarp();
              if (lane == 0) mbar_arrive(BAR(B_REF + at));
            }
          } else if (j == 1) {
            if (!(ok = warp_wait(ctx, BAR(B_REF + at), item_no / kItems & 1, 131))) break;
            ref = sm.ref[at][r];
          }
          minus = ref == -INFINITY ? 0.f : -ref * sl2;
        }
#pragma unroll 1
        for (int n = 0; n < chunks; ++n) {
          const int c = half ? n : chunks - 1 - n;
          WAVEAL_TMEM_LD32(h_addr + 32 * c, u, 0);
          WAVEAL_TMEM_WAIT_LD32(u, 0);
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            float a, b, d, e;
            ffma2(a, b, __uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]), sl2, sl2, minus, minus);
            ffma2(d, e, __uint_as_float(u[2 * i + 2]), __uint_as_float(u[2 * i + 3]), sl2, sl2, minus, minus);
            a = ex2(a), b = ex2(b), d = ex2(d), e = ex2(e);
            fadd2(s0, s1, s0, s1, a, b);
            fadd2(s2, s3, s2, s3, d, e);
            w[i] = pack2<T>(a, b), w[i + 1] = pack2<T>(d, e);
          }
          WAVEAL_TMEM_ST16(s_addr + p_column(4 * half + 2 * c), w, 0);
        }
        tc_wait_st();
        if (cut && safe) {
          if (!(ok = warp_wait(ctx, BAR(B_CHECK + team * kChecks + checks % kChecks), checks / kChecks & 1, 125))) break;
          if (*reinterpret_cast<volatile int*>(&sm.verdict[team][checks % kChecks])) {
            // the row's first thread adds for both, when both have written P
            tc_fence_before();
            exchange(0.f);
            if (!ok) break;
            if (half == 0) {
              if (j == 0 && items >= G::OS && !(ok = warp_wait(ctx, BAR(B_O_EMPTY + items % G::OS), (items / G::OS & 1) ^ 1, 127))) break;
              tc_fence_after();
              add_visible<D, T>(s_addr, tm + G::O_COL + items % G::OS * D, sbase + G::OFF_V + (v_no + j) % G::NVS * G::TILE_BYTES, sees - j * kTile, j == 0);
            }
          }
          ++checks;
        }
        // (read once the products of the last tile are done)
        if (j + 3 - (int)step >= tiles) {
          sm.sums[at][team][half][r] = (s0 + s1) + (s2 + s3);
          if (safe && half == 0) sm.ref[at][r] = ref;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_P + buf));
        buf = buf == 0 ? kBuffers - 1 : buf - 1;     // two on
      }
      if (!ok) break;
      item_done();
      b = (b + tiles * step) % kBuffers;
      if (!safe) g2 = (g2 + tiles) & 1;
      v_no += tiles;
      ++items;
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------ host

// A dimension with one entry: its stride says nothing.
bool one_entry(const waveal_prompt_desc* d, int heads, int dim) { return (dim ? d->tokens : heads) <= 1; }

// [tokens][heads][channels] in boxes of 64 channels
waveal_status make_map(CUtensorMap* tm, const waveal_prompt_desc* d, const void* base, int heads, const int64_t* stride, int box_heads, int box_tokens,
                       const char* what) {
  const auto enc = waveal::tensor_map_encoder();
  if (!enc) return waveal::fail(WAVEAL_ERR_CUDA, "cuTensorMapEncodeTiled entry point not available");
  const cuuint64_t dims[3] = {(cuuint64_t)d->head_dim, (cuuint64_t)heads, (cuuint64_t)d->tokens};
  cuuint64_t bytes[2];
  for (int i = 0; i < 2; ++i) bytes[i] = (cuuint64_t)(one_entry(d, heads, i) ? d->head_dim : stride[i]) * 2;
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, one[3] = {1, 1, 1};
  const CUresult r = enc(tm, d->dtype == WAVEAL_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base),
                         dims, bytes, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return waveal::fail(WAVEAL_ERR_CUDA, "tensor map for %s rejected (CUresult %d)", what, (int)r);
  return WAVEAL_OK;
}

using Wide = __int128;                               // (strides may be any 64-bit numbers)

// Does any of low .. high steps bring a row at `at` onto one at 0, both `dim` elements long?  (The distance falls and then rises.)
bool lands(Wide at, Wide step, Wide low, Wide high, Wide dim) {
  if (low > high) return false;
  Wide n = step ? -at / step : low;
  if (step && n * step > -at) --n;
  for (const Wide k : {n, n + 1}) {
    const Wide gap = at + std::min(std::max(k, low), high) * step;
    if (gap < dim && -gap < dim) return true;
  }
  return false;
}

// Does o share an element with an input of `heads` heads?  Exact where their strides agree along one dimension, so that o may lie between an input's elements
// (one row a token for all tensors, an input's heads repeated by a stride of 0); otherwise the bytes from the first to the last element decide.
bool meets(const waveal_prompt_desc* d, const void* o, const void* x, int heads, const int64_t* stride) {
  const Wide D = d->head_dim, T = d->tokens, H = d->q_heads;
  const Wide ot = T > 1 ? d->o_stride[1] : 0, xt = T > 1 ? stride[1] : 0;
  const Wide oh = H > 1 ? d->o_stride[0] : 0, xh = heads > 1 ? stride[0] : oh;
  const Wide apart = ((Wide) reinterpret_cast<intptr_t>(o) - (Wide) reinterpret_cast<intptr_t>(x)) / 2;   // elements (both are aligned to eight)
  if (apart >= (heads - 1) * xh + (T - 1) * xt + D || -apart >= (H - 1) * oh + (T - 1) * ot + D) return false;
  if (ot != xt && oh != xh) return true;
  if (ot == xt && oh == xh) {
    // two rows that are i heads and k tokens apart, 1 - heads <= i < H, -T < k < T: the fewer of them one by one (at most 2 x 31,623: 10^9 rows)
    if (H + heads <= 2 * T) {
      for (Wide i = 1 - heads; i < H; ++i)
        if (lands(apart + i * oh, ot, 1 - T, T - 1, D)) return true;
    } else {
      for (Wide k = 1 - T; k < T; ++k)
        if (lands(apart + k * ot, oh, 1 - heads, H - 1, D)) return true;
    }
    return false;
  }
  // `step` is common; for each distance along it that can matter, o's rows along the other dimension one by one
  const bool by_token = ot == xt;
  const Wide step = by_token ? ot : oh, on = by_token ? H : T, xn = by_token ? (Wide)heads : T, os = by_token ? oh : ot, xs = by_token ? xh : xt;
  Wide low = by_token ? 1 - T : 1 - (Wide)heads, high = by_token ? T - 1 : H - 1;
  if (step) {
    low = std::max(low, (-(on - 1) * os - D - apart) / step - 1), high = std::min(high, ((xn - 1) * xs + D - apart) / step + 1);
  } else {
    low = high = 0;
  }
  if (low <= high && (high - low + 1) * on > 1 << 20) return true;   // (some ms of the host's time; the bytes' ranges overlap)
  for (Wide k = low; k <= high; ++k)
    for (Wide i = 0; i < on; ++i)
      if (lands(-(apart + k * step + i * os), xs, 0, xn - 1, D)) return true;
  return false;
}

// Do two of o's own rows share an element?
bool folds(const waveal_prompt_desc* d) {
  const Wide D = d->head_dim;
  Wide n = d->q_heads, step = n > 1 ? d->o_stride[0] : 0, more = d->tokens, far = more > 1 ? d->o_stride[1] : 0;
  if (more <= 1 || (n > 1 && far < step)) std::swap(n, more), std::swap(step, far);
  if ((n <= 1 || step >= D) && (more <= 1 || far >= (n - 1) * step + D)) return false;   // one dimension inside the other's steps
  if (n > more) std::swap(n, more), std::swap(step, far);
  for (Wide i = 0; i < n; ++i)
    if (lands(i * step, far, i ? 1 - more : 1, more - 1, D)) return true;
  return false;
}

// row tiles of all key heads that there can be
long long most_tickets(const waveal_prompt_desc* d) {
  const long long tq = kTile / (d->q_heads / d->kv_heads);
  return (d->tokens / tq + d->batch) * d->kv_heads;
}

struct Layout { size_t seq, again, bytes; };
Layout layout(const waveal_prompt_desc* d) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  Layout l;
  l.seq = 256;
  l.again = l.seq + up((size_t)d->batch * sizeof(int4));
  l.bytes = l.again + up((size_t)most_tickets(d) * sizeof(int));
  return l;
}

waveal_status check(const waveal_prompt_desc* d) {
  if (!d) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "desc is NULL");
  if (d->batch < 0 || d->tokens < 0) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "batch and tokens must not be negative");
  if (d->dtype != WAVEAL_BF16 && d->dtype != WAVEAL_FP16) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "dtype %d (WAVEAL_BF16 or WAVEAL_FP16)", d->dtype);
  if (d->head_dim != 64 && d->head_dim != 128) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->head_dim);
  if (d->kv_heads <= 0 || d->q_heads <= 0 || d->q_heads % d->kv_heads || d->q_heads / d->kv_heads > kTile)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q_heads %d: a multiple of kv_heads (%d), at most %d times as many", d->q_heads, d->kv_heads, kTile);
  if (d->flags & ~(WAVEAL_PROMPT_CAUSAL | WAVEAL_PROMPT_SELFTEST_LOST_TILE)) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "unknown flags 0x%x", d->flags);
  if (most_tickets(d) > 1000000000ll) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 10^9 row tiles (of every sequence and key head)");
  if ((long long)d->tokens * d->q_heads > 1000000000ll) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 10^9 rows (tokens * q_heads)");
  // (one item takes all keys of its sequence: every wait for its end stays far below the limit)
  if (d->tokens > 1 << 25) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^25 tokens");
  const int64_t* strides[4] = {d->q_stride, d->k_stride, d->v_stride, d->o_stride};
  for (int t = 0; t < 4; ++t)
    for (int i = 0; i < 2; ++i)
      if (!one_entry(d, t == 1 || t == 2 ? d->kv_heads : d->q_heads, i) && (strides[t][i] % 8 || strides[t][i] < 0))
        return waveal::fail(WAVEAL_ERR_INVALID_ARG, "strides must be multiples of 8 elements (16 bytes) and not negative");
  if (d->tokens && folds(d)) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "o's strides let its rows overlap each other");
  return WAVEAL_OK;
}

template <int D, class T>
waveal_status launch(const CUtensorMap* tm, const Params& p, unsigned grid, cudaStream_t st) {
  constexpr size_t smem = Geo<D>::OFF_END + sizeof(Small<D>);
  static_assert(smem <= 232448, "shared memory of an SM");
  static bool set[64] = {};
  int dev = 0;
  WAVEAL_CUDA_OK(cudaGetDevice(&dev));
  if (dev >= 64 || !set[dev]) {
    WAVEAL_CUDA_OK(cudaFuncSetAttribute(k_prompt_attn<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (dev < 64) set[dev] = true;
  }
  if (p.direct) {
    k_prompt_attn<D, T><<<grid, kThreads, smem, st>>>(tm[0], tm[1], tm[2], p);
    WAVEAL_CUDA_OK(cudaGetLastError());
  } else {
    k_prompt_plan<<<1, kPlanThreads, 0, st>>>(p);
    WAVEAL_CUDA_OK(cudaGetLastError());
    WAVEAL_CUDA_OK(waveal::launch_chained(k_prompt_attn<D, T>, dim3(grid), kThreads, smem, st, tm[0], tm[1], tm[2], p));
  }
  waveal::launch_counter() = p.direct ? 1 : 2;
  return WAVEAL_OK;
}

}  // namespace

extern "C" waveal_status waveal_prompt_attn_workspace_bytes(const waveal_prompt_desc* desc, size_t* bytes) {
  if (!bytes) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "bytes is NULL");
  if (waveal_status e = check(desc)) return e;
  *bytes = layout(desc).bytes;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_prompt_attn(const waveal_prompt_desc* d, const void* q, const void* k, const void* v, void* o, float* lse,
                                            const int32_t* seq_start, const int32_t* seq_len, float scale, void* ws, size_t ws_bytes,
                                            int32_t* dev_status, void* cuda_stream) {
  if (waveal_status e = check(d)) return e;
  if (d->tokens == 0 || d->batch == 0) {
    waveal::launch_counter() = 0;
    return WAVEAL_OK;
  }
  if (!q || !k || !v || !o || !seq_start) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q, k, v, o and seq_start are required");
  if (!waveal::aligned(q, 16) || !waveal::aligned(k, 16) || !waveal::aligned(v, 16) || !waveal::aligned(o, 16))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q, k, v and o must be 16-byte aligned");
  const Layout l = layout(d);
  if (!ws || ws_bytes < l.bytes) return waveal::fail(WAVEAL_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? ws_bytes : 0, l.bytes);
  if (!waveal::aligned(ws, 256)) return waveal::fail(WAVEAL_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (meets(d, o, q, d->q_heads, d->q_stride) || meets(d, o, k, d->kv_heads, d->k_stride) || meets(d, o, v, d->kv_heads, d->v_stride))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "o must not overlap q, k or v");
  const int sms = waveal::sm_count();
  if (sms <= 0) return waveal::fail(WAVEAL_ERR_CUDA, "number of SMs not available");

  Params p = {};
  p.batch = d->batch, p.tokens = d->tokens, p.kv_heads = d->kv_heads, p.group = d->q_heads / d->kv_heads, p.tq = kTile / p.group;
  p.causal = d->flags & WAVEAL_PROMPT_CAUSAL ? 1 : 0;
  char* w = static_cast<char*>(ws);
  p.plan.head = reinterpret_cast<int*>(w);
  p.plan.seq = reinterpret_cast<int4*>(w + l.seq);
  p.plan.again = reinterpret_cast<int*>(w + l.again);
  p.seq_start = seq_start, p.seq_len = seq_len;
  p.o = o, p.lse = lse, p.o_stride_h = d->o_stride[0], p.o_stride_t = d->o_stride[1];
  p.wide_o = waveal::aligned(o, 32);
  for (int i = 0; i < 2; ++i) p.wide_o = p.wide_o && (one_entry(d, d->q_heads, i) || d->o_stride[i] % 16 == 0);
  p.dev_status = dev_status;
  p.drop_tile = d->flags & WAVEAL_PROMPT_SELFTEST_LOST_TILE ? 1 : 0;
  p.wait_limit = p.drop_tile ? kSelfTestCycles : kTimeoutCycles;
  p.sl2 = (scale > 0.f ? scale : 1.0f / std::sqrt((float)d->head_dim)) * 1.4426950408889634f;

  CUtensorMap tm[3];
  if (waveal_status e = make_map(&tm[0], d, q, d->q_heads, d->q_stride, p.group, p.tq, "q")) return e;
  if (waveal_status e = make_map(&tm[1], d, k, d->kv_heads, d->k_stride, 1, kTile, "k")) return e;
  if (waveal_status e = make_map(&tm[2], d, v, d->kv_heads, d->v_stride, 1, kTile, "v")) return e;
  const unsigned grid = (unsigned)std::min((long long)sms, most_tickets(d));   // a thread block an SM
  // Few row tiles need no order and no tickets: every thread block plans for itself.  77 tokens, 8 query and 2 key heads: 7.6 us on
  // the GPU and 16.9 a call from Python instead of 9.0 and 19.8.
  p.direct = d->batch <= 32 && most_tickets(d) <= sms;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (d->dtype == WAVEAL_FP16) return d->head_dim == 128 ? launch<128, __half>(tm, p, grid, st) : launch<64, __half>(tm, p, grid, st);
  return d->head_dim == 128 ? launch<128, __nv_bfloat16>(tm, p, grid, st) : launch<64, __nv_bfloat16>(tm, p, grid, st);
}
