// Attention of a batch over a prefix that all sequences share and over each sequence's own keys, both in a paged cache.
//
//   o = sum_j exp(x_j) v_j / sum_j exp(x_j),  x_j = scale * q k_j,  j over the prefix and the row's own keys.
//
// The sum splits at will: a part keeps its reference m (a maximum so far), its sum l = sum 2^(x_j log2 e - m) and its unscaled
// output; parts join as sum_p 2^(m_p - m) (.)_p.  So the work is laid out by what it has to read:
//   * prefix units: the query rows of ALL sequences that read a key head, 256 at a time, against the prefix's keys;
//   * own units: a sequence's rows of a key head, 256 at a time, against its own keys.
// A row tile holds floor(128 / G) tokens with their G query heads each (G = query heads a key head), token by token, which
// is one TMA box of Q.
//
// One persistent CTA per SM.  Where there are at least as many prefix units as CTAs, whole ones are dealt out in turn, head by
// head (concurrent CTAs then read the same keys, through L2).  All the rest (prefix units left over, own units) is laid end to end in
// a line of key tiles, weighted by what they cost, and cut into equal pieces, one a CTA: no SM waits for another whatever
// the lengths are.  A unit that a cut goes through leaves a part on either side; k_join_parts adds them up.  The line
// is worked out from the lengths by every CTA itself at its start (a scan over the batch), so the lengths may live on the device.
//
// Inside a CTA (384 threads) there are two slots, each with its own S and O accumulators in tensor memory, its own issuing
// warp and its own four softmax warps:
//   warp 0   items (pieces of units), Q tiles and K tiles by TMA        warp 3   V tiles by TMA
//   warp 1, 2  slot 0, 1: S = Q K^T, O += P V (tcgen05, P in tensor memory over the columns of S)
//   warps 4-7, 8-11  slot 0, 1: online softmax, one thread a row; the epilogue
// With more than 128 rows the slots have a row tile each and share every K and V tile; with at most 128 they take the key tiles
// in turn and join their accumulators in the epilogue (both slots' warps reach the same lanes of tensor memory).  Either
// way one slot's products run while the other's softmax does.  O is rescaled only when a row's maximum has grown by more than 2^8.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "host_common.h"
#include "sm100.h"

namespace {

using namespace waveal::sm100;

constexpr int kThreads = 384;
constexpr int kVLoadWarp = 3, kSoftmaxWarp0 = 4;
constexpr int kTile = 128;                           // keys of a tile, rows of a slot
constexpr int kItems = 4;                            // items in flight between the loader and the others
constexpr int kItemReaders = 11;                     // V loader, two issuers, eight softmax warps
constexpr long long kTimeoutCycles = 4000000000ll;   // ~2 s at boost clock
constexpr long long kSelfTestCycles = 4000000ll;     // ~2 ms
constexpr float kGrowth = 8.0f;                      // log2 of how far a row's maximum may outgrow its reference

// Costs on the line of tiles: a key tile of a unit of up to 128 rows, of up to 256, and the start and end of a unit.
constexpr int kCostNarrow = 1, kCostWide = 2, kCostUnit = 1;
// a piece is not made shorter than this (below it the joining costs more than the tiles)
constexpr int kMinPiece = 2;

template <int D> struct Geo {
  static constexpr int SLABS = D / 64;               // 128-byte-swizzled slabs of 64 channels
  static constexpr int SLAB_BYTES = kTile * 128;
  static constexpr int TILE_BYTES = SLABS * SLAB_BYTES;
  static constexpr int NKS = D == 128 ? 3 : 6, NVS = D == 128 ? 2 : 6;
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + NKS * TILE_BYTES, OFF_END = OFF_V + NVS * TILE_BYTES;
  static constexpr int S_COL = 0, O_COL = 256;       // tensor memory: S 0-127, 128-255, O 256.., 384..
};

// ------------------------------------------------------------------ the line of tiles

struct Shape {
  int batch, tokens, kv_heads, group, tq;            // tq: tokens of a row tile
  int prefix_len, max_pages, page_shift, n_pages, causal;
  long long table_stride;
  const int* seq_start;
  const int* kv_len;
  int ctas;
};

struct Parts {
  float* o;                // [row][D], unscaled
  float2* ml;              // [row] {reference (log2), sum}
  long long* own_base;     // [batch] where a sequence's units begin on the line, from the first own unit on
  long long* total;        // cost of all own units
};

__host__ __device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// prefix units: 0 .. n on a head, all alike but the last
struct PrefixLine {
  int per_head, units, whole;     // units of a head; of all heads; dealt out whole
  int tiles, last_weight;
  long long cost, last_cost;      // of a unit, of a head's last

  __device__ explicit PrefixLine(const Shape& s) {
    tiles = ceil_div(s.prefix_len, kTile);
    per_head = tiles ? ceil_div(s.tokens, 2 * s.tq) : 0;
    units = per_head * s.kv_heads;
    whole = units / s.ctas * s.ctas;
    last_weight = s.tokens - (per_head - 1) * 2 * s.tq > s.tq ? kCostWide : kCostNarrow;
    cost = (long long)tiles * kCostWide + kCostUnit;
    last_cost = (long long)tiles * last_weight + kCostUnit;
  }
  __device__ long long before(int u) const {         // cost of units 0 .. u - 1
    const int h = u / max(per_head, 1), i = u - h * per_head;
    return h * ((per_head - 1) * cost + last_cost) + i * cost;
  }
  __device__ long long at(int u) const { return before(u) - before(whole); }
  __device__ long long total() const { return at(units); }
  __device__ int weight(int i) const { return i == per_head - 1 ? last_weight : kCostWide; }
  __device__ int find(long long x) const {           // the unit that position x of the line lies in
    x += before(whole);
    const long long head = (per_head - 1) * cost + last_cost;
    const int h = (int)(x / head);
    return h * per_head + min((int)((x - h * head) / cost), per_head - 1);
  }
};

struct Sequence { int start, n, len; };              // first token, new tokens, own keys

// bad (may be NULL): {site, value} of what is malformed
__device__ inline Sequence read_sequence(const Shape& s, int b, int* bad) {
  Sequence q = {s.seq_start[b], 0, 0};
  const int end = s.seq_start[b + 1], len = s.kv_len[b];
  if (q.start < 0 || end < q.start || end > s.tokens) {
    if (bad) bad[0] = 50, bad[1] = q.start < 0 ? q.start : end;
    q.start = 0;
    return q;
  }
  q.n = end - q.start;
  if (len < 0 || len > ((long long)s.max_pages << s.page_shift)) {
    if (bad) bad[0] = 51, bad[1] = len;
    return q;
  }
  q.len = len;
  return q;
}

// unit i of a sequence's own keys: tokens [first, first + n0 + n1) of its new ones, keys [0, keys)
struct OwnUnit { int first, n0, n1, keys, tiles, weight, cost; };
__device__ inline OwnUnit own_unit(const Shape& s, const Sequence& q, int i) {
  OwnUnit u;
  u.first = i * 2 * s.tq;
  u.n0 = min(s.tq, q.n - u.first);
  u.n1 = min(s.tq, q.n - u.first - u.n0);
  u.keys = s.causal ? max(0, q.len - q.n + u.first + u.n0 + u.n1) : q.len;
  u.tiles = ceil_div(u.keys, kTile);
  u.weight = u.n1 ? kCostWide : kCostNarrow;
  u.cost = u.tiles ? u.tiles * u.weight + kCostUnit : 0;
  return u;
}
__device__ inline long long own_head_cost(const Shape& s, const Sequence& q) {
  const int m = ceil_div(q.n, 2 * s.tq);
  long long c = 0;
  if (s.causal) {
    for (int i = 0; i < m; ++i) c += own_unit(s, q, i).cost;
  } else if (m) {
    c = (long long)(m - 1) * own_unit(s, q, 0).cost + own_unit(s, q, m - 1).cost;
  }
  return c;
}

// the line cut into pieces
struct Cuts {
  long long total;
  int pieces;
  __device__ Cuts(long long total_, int ctas) : total(total_) {
    pieces = (int)min((long long)ctas, max(1ll, total / kMinPiece));
  }
  __device__ long long begin(int c) const { return c * total / pieces; }
  __device__ int piece(long long x) const { return (int)(((x + 1) * pieces - 1) / total); }
  // tiles [from, to) of a unit at `at` that begin in piece c
  __device__ int first_tile(int c, long long at, int tiles, int weight) const {
    const long long d = begin(c) - at;
    return d <= 0 ? 0 : (int)min((long long)tiles, (d + weight - 1) / weight);
  }
};

// Where the parts of a row lie.  Units follow each other on the line in the order of their rows (prefix: head, token, query head
// of the group; own: sequence, key head, token, query head), and so do pieces: row + piece * (rows of the largest unit) is
// a place that no other part has.
__device__ inline long long part_row(const Shape& s, long long row, int piece) { return row + (long long)piece * 2 * s.tq * s.group; }
__device__ inline long long prefix_row(const Shape& s, int h, int token) { return ((long long)h * s.tokens + token) * s.group; }
__device__ inline long long own_row(const Shape& s, const Sequence& q, int h, int token) {   // token: from the sequence's first new one
  return (long long)s.tokens * s.kv_heads * s.group + ((long long)q.start * s.kv_heads + (long long)h * q.n + token) * s.group;
}

// ------------------------------------------------------------------ kernel

constexpr int kMaxKeys = 1 << 30;                    // of a list
constexpr int kAll = kMaxKeys + kTile;               // sees every list whole

struct Item {
  int tiles;               // 0: the end
  int wide;                // the slots have a row tile each
  int head, token;         // key head; first token of the call's tensors
  int n0, n1;              // tokens of the row tiles
  int first_key, keys;     // keys [first_key, keys) of the list, tile by tile
  int list;                // -1: the prefix, else the sequence
  int sees;                // keys that the first token sees (below 1: none); every token sees one more. kAll: all of them see all
  int direct;              // 1: no other part of these rows exists, o is written at once
  int row;                 // of the parts
};

struct Params {
  Shape s;
  Parts parts;
  const int* page_table;
  const int* prefix_pages;
  void* o;
  float* lse;
  long long o_stride_h, o_stride_t;
  int* dev_status;
  long long wait_limit;
  int drop_tile;
  float sl2;               // scale * log2(e)
};

struct Ctx {
  volatile int* abort_smem;
  int* dev_status;
  long long limit;
};

__device__ __noinline__ void report(int* status, int code, int site, int where, int value) {
  if (status && atomicCAS(status, 0, code) == 0) {
    status[1] = site;
    status[2] = where;
    status[3] = value;
  }
}

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
  return __all_sync(0xffffffffu, mbar_try_wait(bar, parity) || wait_slow(c, bar, parity, site));
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}

// D[tmem] (+)= A[smem] * B[smem]; both operands of the tensors' type
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if (elect_one())
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

template <class T> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

enum {
  B_ITEM_FULL = 0, B_ITEM_EMPTY = B_ITEM_FULL + kItems, B_Q_FULL = B_ITEM_EMPTY + kItems, B_Q_EMPTY = B_Q_FULL + 2,
  B_K_FULL = B_Q_EMPTY + 2, B_K_EMPTY = B_K_FULL + 6, B_V_FULL = B_K_EMPTY + 6, B_V_EMPTY = B_V_FULL + 6,
  B_S_FULL = B_V_EMPTY + 6, B_P_FULL = B_S_FULL + 2, B_PV_DONE = B_P_FULL + 4, B_O_EMPTY = B_PV_DONE + 2, B_SUMS = B_O_EMPTY + 2,
  B_FINAL = B_SUMS + 2, B_COUNT = B_FINAL + 2
};

// what lies behind the tiles in shared memory
struct Small {
  unsigned long long bar[B_COUNT];
  Item items[kItems];
  float2 sums[2][kTile];   // slot 1's references and sums of an item whose key tiles the slots share out (two: slot 1 may be an item ahead)
  long long warp_sum[kThreads / 32];
  long long own_total, start_base;
  int start_seq;
  uint32_t tmem;
  int abort;
};

// One K or V tile into its ring stage (a whole warp): boxes of up to 128 slots of a page, one lane each and slab.
// (the page of tile j's box was read while tile j - 1 waited for its stage)
template <int D>
struct TileLoader {
  using G = Geo<D>;
  uint32_t it = 0, armed = 0, parity = 0;
  int page = 0;

  __device__ int read_page(const Params& p, const Item& im, int key, int lane) const {
    const int shift = p.s.page_shift, box = min(1 << shift, kTile);
    const int nb = ceil_div(min(kTile, im.keys - key), box);
    const int k = key + (lane % max(nb, 1)) * box;
    if (lane >= nb * G::SLABS || key >= im.keys) return 0;
    const int* list = im.list < 0 ? p.prefix_pages : p.page_table + im.list * p.s.table_stride;
    return __ldg(list + (k >> shift));
  }
  template <int STAGES>
  __device__ bool load(const Ctx& c, const Params& p, const Item& im, int key, bool last, bool drop, int lane, uint32_t smem,
                       uint32_t full, uint32_t empty, const CUtensorMap* tm, int site) {
    const uint32_t st = it % STAGES, ph = it / STAGES & 1;
    const int shift = p.s.page_shift, box = min(1 << shift, kTile);
    const int nb = ceil_div(min(kTile, im.keys - key), box);
    int pg = page;
    if (!last) page = read_page(p, im, key + kTile, lane);
    if (it >= STAGES && !warp_wait(c, empty + 8 * st, ph ^ 1, site)) return false;
    ++it;
    if (drop) return true;
    if (lane == 0) mbar_expect_tx(full + 8 * st, nb * G::SLABS * box * 128);
    armed |= 1u << st;
    parity = (parity & ~(1u << st)) | ph << st;
    __syncwarp();
    if (lane < nb * G::SLABS) {
      const int slab = lane / nb, i = lane - slab * nb;
      if (pg < 0 || pg >= p.s.n_pages) {
        report(p.dev_status, WAVEAL_ERR_BAD_MASK, 52, im.list, pg);
        pg = p.s.n_pages;                            // beyond the cache: the copy engine fills in zeros
      }
      tma_load_4d(smem + st * G::TILE_BYTES + slab * G::SLAB_BYTES + i * box * 128, tm, slab * 64, (key + i * box) & ((1 << shift) - 1),
                  im.head, pg, full + 8 * st);
    }
    __syncwarp();
    return true;
  }
  // (after a wait gave up) leaves no copy in flight
  __device__ void drain(const Params& p, uint32_t full) const {
    for (int st = 0; st < 6; ++st)
      if (armed >> st & 1) {
        const long long t0 = clock64();
        while (!mbar_try_wait(full + 8 * st, parity >> st & 1) && clock64() - t0 < p.wait_limit / 4) {}
      }
  }
};

template <int D, class T>
__global__ void __launch_bounds__(kThreads, 1)
k_prefix_attn(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmQ1, const __grid_constant__ CUtensorMap tmK,
              const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Params p) {
  using G = Geo<D>;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  Small& sm = *reinterpret_cast<Small*>(smem + G::OFF_END);
  const uint32_t bars = smem_u32(sm.bar);
  auto BAR = [&](int i) { return bars + 8 * i; };
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const Shape& s = p.s;
  waveal::let_next_kernel_start();

  if (warp == 1) {
    tmem_alloc(smem_u32(&sm.tmem), 512);
    tmem_relinquish();
  } else if (warp == 2 && lane == 0) {
    for (int i = 0; i < kItems; ++i) mbar_init(BAR(B_ITEM_FULL + i), 1), mbar_init(BAR(B_ITEM_EMPTY + i), kItemReaders);
    for (int i = 0; i < 6; ++i) {
      mbar_init(BAR(B_K_FULL + i), 1), mbar_init(BAR(B_K_EMPTY + i), 2);
      mbar_init(BAR(B_V_FULL + i), 1), mbar_init(BAR(B_V_EMPTY + i), 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(BAR(B_Q_FULL + i), 1), mbar_init(BAR(B_Q_EMPTY + i), 2);
      mbar_init(BAR(B_S_FULL + i), 1), mbar_init(BAR(B_P_FULL + 2 * i), 4), mbar_init(BAR(B_P_FULL + 2 * i + 1), 4);
      mbar_init(BAR(B_PV_DONE + i), 1), mbar_init(BAR(B_O_EMPTY + i), 4), mbar_init(BAR(B_FINAL + i), 1);
      mbar_init(BAR(B_SUMS + i), 4);
    }
    sm.abort = 0;
    sm.start_seq = s.batch;
    fence_mbar_init();
  } else if (warp == 3 && lane == 0) {
    prefetch_tmap(&tmQ), prefetch_tmap(&tmQ1), prefetch_tmap(&tmK), prefetch_tmap(&tmV);
  }

  // ---- the line of tiles: every thread takes a run of sequences, the block scans their costs
  const PrefixLine line(s);
  const int per = ceil_div(s.batch, kThreads);
  const int b0 = min((int)threadIdx.x * per, s.batch), b1 = min(b0 + per, s.batch);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    int bad[2] = {0, 0};
    mine += own_head_cost(s, read_sequence(s, b, bad)) * s.kv_heads;
    if (bad[0] && blockIdx.x == 0) report(p.dev_status, WAVEAL_ERR_BAD_MASK, bad[0], b, bad[1]);
  }
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long x = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sm.warp_sum[warp] = upto;
  __syncthreads();
  long long own_total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) upto += sm.warp_sum[w];
    own_total += sm.warp_sum[w];
  }
  const Cuts cuts(max(line.total() + own_total, 1ll), s.ctas);
  const int piece = blockIdx.x;
  const bool has_piece = piece < cuts.pieces && line.total() + own_total > 0;
  const long long w0 = has_piece ? cuts.begin(piece) : 0, w1 = has_piece ? cuts.begin(piece + 1) : 0;
  {
    const long long from = max(w0 - line.total(), 0ll);
    long long base = upto - mine;
    if (blockIdx.x == 0 || (base <= from && from < upto))
      for (int b = b0; b < b1; ++b) {
        const long long c = own_head_cost(s, read_sequence(s, b, nullptr)) * s.kv_heads;
        if (base <= from && from < base + c) sm.start_seq = b, sm.start_base = base;
        if (blockIdx.x == 0) p.parts.own_base[b] = base;
        base += c;
      }
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.parts.total = own_total;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const Ctx ctx = {&sm.abort, p.dev_status, p.wait_limit};
  bool ok = true;

  // the next item, for everyone but the loader: false when there is none or a wait gave up
  uint32_t item_no = 0;
  auto next_item = [&](Item& im) {
    const uint32_t slot = item_no % kItems;
    if (!warp_wait(ctx, BAR(B_ITEM_FULL + slot), item_no / kItems & 1, 60)) return ok = false;
    im = sm.items[slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(B_ITEM_EMPTY + slot));
    ++item_no;
    return im.tiles > 0;
  };

  if (warp == 0) {
    // ================================================================ items, Q, K
    TileLoader<D> loader;
    uint32_t q_it = 0, q_armed = 0, q_parity = 0;
    auto load_q = [&](const CUtensorMap* tm, int token, int head, int n) {
      const uint32_t st = q_it & 1, ph = q_it >> 1 & 1;
      if (q_it >= 2 && !warp_wait(ctx, BAR(B_Q_EMPTY + st), ph ^ 1, 61)) return false;
      ++q_it;
      if (lane == 0) {
        mbar_expect_tx(BAR(B_Q_FULL + st), n * s.group * 128 * G::SLABS);
#pragma unroll
        for (int i = 0; i < G::SLABS; ++i)
          tma_load_3d(sbase + G::OFF_Q + st * G::TILE_BYTES + i * G::SLAB_BYTES, tm, i * 64, head, token, BAR(B_Q_FULL + st));
      }
      q_armed |= 1u << st, q_parity = (q_parity & ~(1u << st)) | ph << st;
      __syncwarp();
      return true;
    };
    auto publish = [&](const Item& im) {
      const uint32_t slot = item_no % kItems;
      if (item_no >= kItems && !warp_wait(ctx, BAR(B_ITEM_EMPTY + slot), (item_no / kItems & 1) ^ 1, 62)) return false;
      if (lane == 0) {
        sm.items[slot] = im;
        mbar_arrive(BAR(B_ITEM_FULL + slot));
      }
      __syncwarp();
      ++item_no;
      return true;
    };
    auto emit = [&](Item im) {
      loader.page = loader.read_page(p, im, im.first_key, lane);
      if (!publish(im)) return false;
      if (!load_q(im.n0 == 1 ? &tmQ1 : &tmQ, im.token, im.head * s.group, im.n0 == 1 ? 1 : s.tq)) return false;
      if (im.wide && !load_q(im.n1 == 1 ? &tmQ1 : &tmQ, im.token + s.tq, im.head * s.group, im.n1 == 1 ? 1 : s.tq)) return false;
      for (int j = 0; j < im.tiles; ++j)
        if (!loader.template load<G::NKS>(ctx, p, im, im.first_key + j * kTile, j == im.tiles - 1, p.drop_tile && blockIdx.x == 0 && loader.it == 0,
                                          lane, sbase + G::OFF_K, BAR(B_K_FULL), BAR(B_K_EMPTY), &tmK, 63))
          return false;
      return true;
    };
    auto prefix_item = [&](int u, int j0, int j1, int at_piece) {
      const int h = u / line.per_head, i = u - h * line.per_head;
      Item im;
      im.tiles = j1 - j0;
      im.head = h, im.token = i * 2 * s.tq;
      im.n0 = min(s.tq, s.tokens - im.token), im.n1 = min(s.tq, s.tokens - im.token - im.n0);
      im.wide = im.n1 > 0;
      im.first_key = j0 * kTile, im.keys = min(s.prefix_len, j1 * kTile);
      im.list = -1, im.sees = kAll;
      im.direct = 0;
      im.row = (int)part_row(s, prefix_row(s, h, im.token), at_piece);
      return emit(im);
    };
    // whole units
    for (int u = blockIdx.x; ok && u < line.whole; u += s.ctas) ok = prefix_item(u, 0, line.tiles, 0);
    // this CTA's piece of the line: prefix units ...
    if (ok && has_piece && w0 < line.total()) {
      for (int u = line.find(w0); ok && u < line.units; ++u) {
        const long long at = line.at(u);
        if (at >= w1) break;
        const int wt = line.weight(u % line.per_head);
        const int j0 = cuts.first_tile(piece, at, line.tiles, wt), j1 = cuts.first_tile(piece + 1, at, line.tiles, wt);
        if (j0 < j1) ok = prefix_item(u, j0, j1, piece);
      }
    }
    // ... and own units
    long long base = sm.start_base;
    for (int b = sm.start_seq; ok && has_piece && b < s.batch; ++b) {
      if (line.total() + base >= w1) break;
      const Sequence q = read_sequence(s, b, nullptr);
      const long long head_cost = own_head_cost(s, q);
      const int m = ceil_div(q.n, 2 * s.tq);
      const long long skip = w0 - line.total() - base;
      int h = head_cost && skip > 0 ? (int)min((long long)s.kv_heads, skip / head_cost) : 0;
      for (; ok && head_cost && h < s.kv_heads; ++h) {
        long long at = line.total() + base + h * head_cost;
        if (at >= w1) break;
        for (int i = 0; ok && i < m && at < w1; ++i) {
          const OwnUnit u = own_unit(s, q, i);
          const int j0 = cuts.first_tile(piece, at, u.tiles, u.weight), j1 = cuts.first_tile(piece + 1, at, u.tiles, u.weight);
          at += u.cost;
          if (j0 >= j1) continue;
          Item im;
          im.tiles = j1 - j0;
          im.head = h, im.token = q.start + u.first;
          im.n0 = u.n0, im.n1 = u.n1, im.wide = u.n1 > 0;
          im.first_key = j0 * kTile, im.keys = min(u.keys, j1 * kTile);
          im.list = b;
          im.sees = s.causal ? q.len - q.n + u.first + 1 : kAll;
          im.direct = line.tiles == 0 && j0 == 0 && j1 == u.tiles;
          im.row = (int)part_row(s, own_row(s, q, h, u.first), piece);
          ok = emit(im);
        }
      }
      base += head_cost * s.kv_heads;
    }
    if (ok) {
      Item im = {};
      publish(im);
    }
    if (*ctx.abort_smem) {
      loader.drain(p, BAR(B_K_FULL));
      for (int st = 0; st < 2; ++st)
        if (q_armed >> st & 1) {
          const long long t0 = clock64();
          while (!mbar_try_wait(BAR(B_Q_FULL + st), q_parity >> st & 1) && clock64() - t0 < p.wait_limit / 4) {}
        }
    }
  } else if (warp == kVLoadWarp) {
    // ================================================================ V
    TileLoader<D> loader;
    Item im;
    while (ok && next_item(im)) {
      loader.page = loader.read_page(p, im, im.first_key, lane);
      for (int j = 0; ok && j < im.tiles; ++j)
        ok = loader.template load<G::NVS>(ctx, p, im, im.first_key + j * kTile, j == im.tiles - 1, false, lane, sbase + G::OFF_V, BAR(B_V_FULL),
                                          BAR(B_V_EMPTY), &tmV, 64);
    }
    if (*ctx.abort_smem) loader.drain(p, BAR(B_V_FULL));
  } else if (warp < kVLoadWarp) {
    // ================================================================ products of a slot
    // Each slot has an issuing warp: what one waits for (its softmax, its last product) never holds up the other.  S and P share
    // columns, so a slot's next S = Q K^T waits for the end of its last P V.
    constexpr uint32_t kType = std::is_same_v<T, __half> ? 0u : (1u << 7) | (1u << 10);
    constexpr uint32_t IDESC_QK = (make_idesc(128, kTile, false) & ~((1u << 7) | (1u << 10))) | kType;
    constexpr uint32_t IDESC_PV = (make_idesc(128, D, true) & ~((1u << 7) | (1u << 10))) | kType;
    const int slot = warp - 1;
    const uint32_t d_s = tmem + G::S_COL + slot * kTile, d_o = tmem + G::O_COL + slot * kTile;
    const uint64_t q_desc0 = make_desc(sbase + G::OFF_Q, 16, 1024), k_desc0 = make_desc(sbase + G::OFF_K, 16, 1024);
    const uint64_t v_desc0 = make_desc(sbase + G::OFF_V, G::SLAB_BYTES, 1024);
    // A barrier of the rings is told from the one before last only by a parity, so every issuer waits for every Q, K and V tile in
    // turn, its own or not, and each is given back by both (its own when the products on it have ended).
    uint32_t g0 = 0, q_it = 0, done = 0, uses = 0;   // tiles of the CTA so far; Q tiles; tiles and items of this slot
    auto pass_on = [&](uint32_t full, uint32_t empty, uint32_t parity, int site) {
      if (!warp_wait(ctx, full, parity, site)) return false;
      if (lane == 0) mbar_arrive(empty);
      __syncwarp();
      return true;
    };
    Item im;
    while (ok && next_item(im)) {
      const int wide = __shfl_sync(0xffffffffu, im.wide, 0), tiles = __shfl_sync(0xffffffffu, im.tiles, 0);
      const int keys = __shfl_sync(0xffffffffu, im.keys - im.first_key, 0);
      const int from = wide ? 0 : slot;
      const int last = wide ? tiles - 1 : (tiles - 1 - slot) / 2 * 2 + slot;
      uint32_t qb = 0;
      for (int i = 0; ok && i <= wide; ++i, ++q_it) {
        const uint32_t b = q_it & 1, ph = q_it >> 1 & 1;
        if (from < tiles && (!wide || i == slot)) {
          qb = b;
          ok = warp_wait(ctx, BAR(B_Q_FULL + b), ph, 65);
        } else {
          ok = pass_on(BAR(B_Q_FULL + b), BAR(B_Q_EMPTY + b), ph, 65);
        }
      }
      for (int j = 0; ok && j < tiles; ++j) {
        const uint32_t g = g0 + j, ks = g % G::NKS, vs = g % G::NVS;
        if (!wide && (j & 1) != slot) {
          ok = pass_on(BAR(B_K_FULL + ks), BAR(B_K_EMPTY + ks), g / G::NKS & 1, 66) &&
               pass_on(BAR(B_V_FULL + vs), BAR(B_V_EMPTY + vs), g / G::NVS & 1, 68);
          continue;
        }
        if (!(ok = warp_wait(ctx, BAR(B_K_FULL + ks), g / G::NKS & 1, 66))) break;
        if (done && !(ok = warp_wait(ctx, BAR(B_PV_DONE + slot), (done - 1) & 1, 67))) break;
        tc_fence_after();
        {
          const uint64_t qd = q_desc0 + (uint64_t)(qb * (G::TILE_BYTES >> 4)), kd = k_desc0 + (uint64_t)(ks * (G::TILE_BYTES >> 4));
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint64_t at = (uint64_t)((c / 4 * G::SLAB_BYTES + c % 4 * 32) >> 4);
            umma_ss(d_s, qd + at, kd + at, IDESC_QK, c > 0);
          }
          tc_commit(BAR(B_K_EMPTY + ks));
          tc_commit(BAR(B_S_FULL + slot));
          if (j == last) tc_commit(BAR(B_Q_EMPTY + qb));
        }
        if (!(ok = warp_wait(ctx, BAR(B_V_FULL + vs), g / G::NVS & 1, 68))) break;
        const int valid = min(kTile, keys - j * kTile), steps = (valid + 15) / 16;
        if (valid < steps * 16) {
          // the last keys of a list: what lies behind them in the page (or was never loaded) must not meet the zeros of P
          const int chunks = (steps * 16 - valid) * 8;
#pragma unroll
          for (int slab = 0; slab < G::SLABS; ++slab)
            for (int i = lane; i < chunks; i += 32)
              st_shared_v4(sbase + G::OFF_V + vs * G::TILE_BYTES + slab * G::SLAB_BYTES + valid * 128 + i * 16, 0, 0, 0, 0);
          fence_proxy_async();
          __syncwarp();
        }
        if (j == from && uses && !(ok = warp_wait(ctx, BAR(B_O_EMPTY + slot), (uses - 1) & 1, 69))) break;
        const uint64_t vd = v_desc0 + (uint64_t)(vs * (G::TILE_BYTES >> 4));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(ok = warp_wait(ctx, BAR(B_P_FULL + 2 * slot + half), done & 1, 70))) break;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int k = half * 4 + c;
            if (k < steps) umma_bf16_ts(d_o, d_s + k * 8, vd + (uint64_t)((k * 16 * 128) >> 4), IDESC_PV, (j != from || k > 0) ? 1u : 0u);
          }
        }
        if (!ok) break;
        tc_commit(BAR(B_V_EMPTY + vs));
        tc_commit(BAR(B_PV_DONE + slot));
        ++done;
      }
      g0 += tiles;
      if (from < tiles) ++uses;
    }
    // no product is still running when tensor memory is given back
    tc_commit(BAR(B_FINAL + slot));
    __syncwarp();
    const long long t0 = clock64();
    while (!mbar_try_wait(BAR(B_FINAL + slot), 0) && clock64() - t0 < p.wait_limit / 4) {}
  } else {
    // ================================================================ softmax, epilogue
    const int slot = (warp - kSoftmaxWarp0) / 4, quad = warp & 3, r = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const uint32_t s_addr = tmem + lanes + G::S_COL + slot * kTile, o_addr = tmem + lanes + G::O_COL + slot * kTile;
    uint32_t done = 0, done1 = 0, joined = 0;        // tiles of this slot, of slot 1; items whose slots were joined
    Item im;
    while (ok && next_item(im)) {
      const bool wide = im.wide;
      const int step = wide ? 1 : 2, from = wide ? 0 : slot;
      const int tok = (wide && slot ? im.token + im.n0 : im.token) , n = wide && slot ? im.n1 : im.n0;
      const int rows = n * s.group;
      const bool live = r < rows, idle = quad * 32 >= rows;
      const int row_tok = r / s.group, row_sub = r - row_tok * s.group;
      // keys of this row, from the item's first; and those that every row of the tile sees
      const int all = im.keys - im.first_key;
      const int sees0 = im.sees - im.first_key + (wide && slot ? im.n0 : 0);
      const int sees = min(all, sees0 + row_tok);
      const int unmasked = min(all, sees0);
      float ref = -INFINITY, l0 = 0.f, l1 = 0.f;
      const uint32_t done1_new = done1 + (wide ? im.tiles : im.tiles / 2);
      for (int j = from; j < im.tiles; j += step) {
        if (!(ok = warp_wait(ctx, BAR(B_S_FULL + slot), done & 1, 71))) break;
        ++done;
        if (idle) {
          if (lane == 0) mbar_arrive(BAR(B_P_FULL + 2 * slot)), mbar_arrive(BAR(B_P_FULL + 2 * slot + 1));
          continue;
        }
        tc_fence_after();
        // 64 columns at a time, loaded once for the maximum and once more for the exponentials: a whole row in registers spills
        uint32_t sv[64];
        const int lim = sees - j * kTile;
        const bool masked = unmasked < (j + 1) * kTile;
        auto load_s = [&](int half) {
          WAVEAL_TMEM_LD32(s_addr + half * 64, sv, 0);
          WAVEAL_TMEM_LD32(s_addr + half * 64 + 32, sv, 32);
          WAVEAL_TMEM_WAIT_LD32(sv, 0);
          WAVEAL_TMEM_WAIT_LD32(sv, 32);
          if (masked) {
#pragma unroll
            for (int c = 0; c < 64; ++c) sv[c] = half * 64 + c < lim ? sv[c] : 0xff800000u;
          }
        };
        float mx = -INFINITY;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          load_s(half);
          float mx4[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) mx4[i] = __uint_as_float(sv[i]);
#pragma unroll
          for (int c = 4; c < 60; c += 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mx4[i] = fmax3(mx4[i], __uint_as_float(sv[c + 2 * i]), __uint_as_float(sv[c + 2 * i + 1]));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) mx4[i] = fmaxf(mx4[i], __uint_as_float(sv[60 + i]));
          mx = fmaxf(mx, fmaxf(fmax3(mx4[0], mx4[1], mx4[2]), mx4[3]));
        }
        mx *= p.sl2;
        const bool grows = live && mx > ref + kGrowth;
        if (__any_sync(0xffffffffu, grows)) {
          float a = 1.0f;
          if (grows) {
            a = ex2(ref - mx);
            ref = mx;
            l0 *= a, l1 *= a;
          }
          if (j != from) {
            // the rows' accumulators: not while a product still adds to them
            if (!(ok = warp_wait(ctx, BAR(B_PV_DONE + slot), (done - 2) & 1, 72))) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              WAVEAL_TMEM_LD32(o_addr + c, sv, 0);
              WAVEAL_TMEM_WAIT_LD32(sv, 0);
#pragma unroll
              for (int i = 0; i < 32; ++i) sv[i] = __float_as_uint(__uint_as_float(sv[i]) * a);
              WAVEAL_TMEM_ST32(o_addr + c, sv, 0);
            }
            tc_wait_st();
          }
        }
        const float b = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          load_s(half);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float x0, x1;
              ffma2(x0, x1, __uint_as_float(sv[q * 32 + 2 * i]), __uint_as_float(sv[q * 32 + 2 * i + 1]), p.sl2, p.sl2, b, b);
              x0 = ex2(x0), x1 = ex2(x1);
              fadd2(l0, l1, l0, l1, x0, x1);
              pk[i] = pack2<T>(x0, x1);
            }
            // P of a half of the keys lies over S columns that have been read by then
            WAVEAL_TMEM_ST16(s_addr + half * 32 + q * 16, pk, 0);
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(B_P_FULL + 2 * slot + half));
        }
      }
      if (!ok) break;
      const uint32_t last_done = done - 1;
      done1 = slot ? done : done1_new;

      // ---- epilogue
      float l = l0 + l1;
      const bool join = !wide && im.tiles > 1;
      if (!wide && slot) {
        if (join) {
          if (!idle) sm.sums[joined & 1][r] = make_float2(ref, l);
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(B_SUMS + (joined & 1)));
          ++joined;
        }
        continue;
      }
      float a0 = 1.0f, a1 = 0.0f;
      if (join) {
        if (!(ok = warp_wait(ctx, BAR(B_SUMS + (joined & 1)), joined >> 1 & 1, 73))) break;
        if (!(ok = warp_wait(ctx, BAR(B_PV_DONE + 1), (done1 - 1) & 1, 74))) break;
        const float2 other = idle ? make_float2(0.f, 0.f) : sm.sums[joined & 1][r];
        ++joined;
        const float m = fmaxf(ref, other.x);
        a0 = ref == -INFINITY ? 0.f : ex2(ref - m);
        a1 = other.x == -INFINITY ? 0.f : ex2(other.x - m);
        ref = m;
        l = l * a0 + other.y * a1;
      }
      if (!(ok = warp_wait(ctx, BAR(B_PV_DONE + slot), last_done & 1, 75))) break;
      tc_fence_after();
      if (!idle) {
        const long long out_row = im.row + (long long)(wide && slot ? im.n0 * s.group : 0) + r;
        float scale_o = 1.0f;
        T* o_ptr = nullptr;
        if (im.direct) {
          scale_o = l == 0.f ? 0.f : 1.0f / l;
          const int head = im.head * s.group + row_sub;
          o_ptr = static_cast<T*>(p.o) + head * p.o_stride_h + (long long)(tok + row_tok) * p.o_stride_t;
          if (live && p.lse) p.lse[(long long)head * s.tokens + tok + row_tok] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.69314718055994531f;
        } else if (live) {
          p.parts.ml[out_row] = make_float2(ref, l);
        }
        a0 *= scale_o, a1 *= scale_o;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t v[32], w[32];
          WAVEAL_TMEM_LD32(o_addr + c, v, 0);
          if (join) {
            WAVEAL_TMEM_LD32(o_addr + kTile + c, w, 0);
            WAVEAL_TMEM_WAIT_LD32(w, 0);
          }
          WAVEAL_TMEM_WAIT_LD32(v, 0);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float x = __uint_as_float(v[i]) * a0;
            if (join) x += __uint_as_float(w[i]) * a1;
            v[i] = __float_as_uint(x);
          }
          if (live) {
            if (im.direct) {
#pragma unroll
              for (int i = 0; i < 16; ++i) w[i] = pack2<T>(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
#pragma unroll
              for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(o_ptr + c + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
              float* dst = p.parts.o + out_row * D + c;
#pragma unroll
              for (int i = 0; i < 32; i += 8) st_global_v8(dst + i, v + i);
            }
          }
        }
        tc_fence_before();
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(BAR(B_O_EMPTY + slot));
        if (join) mbar_arrive(BAR(B_O_EMPTY + 1));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------ parts -> output

// WARPS warps a row (a token's query head), each with every WARPS-th part.
template <int D, class T, int WARPS>
__global__ void __launch_bounds__(128) k_join_parts(const __grid_constant__ Params p) {
  constexpr int C = D / 32;                          // channels of a lane
  const Shape& s = p.s;
  const int heads = s.kv_heads * s.group, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const long long id = (long long)blockIdx.x * (4 / WARPS) + warp / WARPS;
  const int token = (int)(id / heads), head = (int)(id - (long long)token * heads), h = head / s.group, g = head - h * s.group;
  const int part0 = WARPS > 1 ? warp : 0;
  __shared__ float2 ml_sh[4];
  __shared__ float o_sh[WARPS > 1 ? 3 : 1][D];
  waveal::wait_for_previous_kernel();
  bool mine = token < s.tokens;

  // whose token is it (a token of no sequence is left alone)
  Sequence q = {0, 0, 0};
  int b = 0;
  if (mine) {
    b = (int)min((long long)token * s.batch / s.tokens, (long long)s.batch - 1);
    q = read_sequence(s, b, nullptr);
    if (token < q.start || token >= q.start + q.n) {
      int l = 0, r = s.batch - 1;
      while (l < r) {
        const int m = (l + r + 1) >> 1;
        if (s.seq_start[m] <= token) l = m; else r = m - 1;
      }
      b = l;
      q = read_sequence(s, b, nullptr);
    }
    mine = token >= q.start && token < q.start + q.n;
  }

  float m = -INFINITY, l = 0.f, acc[C];
#pragma unroll
  for (int i = 0; i < C; ++i) acc[i] = 0.f;
  bool written = false;
  if (mine) {
    const PrefixLine line(s);
    const long long own_total = *p.parts.total;
    const Cuts cuts(max(line.total() + own_total, 1ll), s.ctas);
    int seen = 0;                                    // parts so far, over all warps
    auto add_unit = [&](long long row, bool whole, long long at, int tiles, int weight) {
      if (!tiles) return;
      const int c0 = whole ? 0 : cuts.piece(at), c1 = whole ? 0 : cuts.piece(at + (long long)(tiles - 1) * weight);
      for (int c = c0; c <= c1; ++c) {
        if (!whole && cuts.first_tile(c, at, tiles, weight) >= cuts.first_tile(c + 1, at, tiles, weight)) continue;
        if (WARPS > 1 && seen++ % WARPS != part0) continue;
        const long long at_row = part_row(s, row, c);
        const float2 ml = p.parts.ml[at_row];
        float v[C];
        const float* src = p.parts.o + at_row * D + lane * C;
        if constexpr (C == 4) {
          const float4 x = *reinterpret_cast<const float4*>(src);
          v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(src);
          v[0] = x.x, v[1] = x.y;
        }
        const float to = fmaxf(m, ml.x);
        const float a = m == -INFINITY ? 0.f : ex2(m - to), e = ml.x == -INFINITY ? 0.f : ex2(ml.x - to);
        m = to;
        l = l * a + ml.y * e;
#pragma unroll
        for (int i = 0; i < C; ++i) acc[i] = acc[i] * a + v[i] * e;
      }
    };
    if (line.tiles) {
      const int u = h * line.per_head + token / (2 * s.tq);
      add_unit(prefix_row(s, h, token) + g, u < line.whole, u < line.whole ? 0 : line.at(u), line.tiles, line.weight(token / (2 * s.tq)));
    }
    if (q.len) {
      const int i = (token - q.start) / (2 * s.tq);
      long long at = line.total() + p.parts.own_base[b] + h * own_head_cost(s, q);
      if (s.causal) {
        for (int k = 0; k < i; ++k) at += own_unit(s, q, k).cost;
      } else {
        at += (long long)i * own_unit(s, q, 0).cost;
      }
      const OwnUnit u = own_unit(s, q, i);
      written = line.tiles == 0 && u.tiles && cuts.piece(at) == cuts.piece(at + (long long)(u.tiles - 1) * u.weight);
      if (!written) add_unit(own_row(s, q, h, token - q.start) + g, false, at, u.tiles, u.weight);
    }
  }
  if constexpr (WARPS > 1) {
    if (lane == 0) ml_sh[warp] = make_float2(m, l);
    if (warp) {
#pragma unroll
      for (int i = 0; i < C; ++i) o_sh[warp - 1][lane * C + i] = acc[i];
    }
    __syncthreads();
    if (warp) return;
    float to = m;
    for (int w = 1; w < 4; ++w) to = fmaxf(to, ml_sh[w].x);
    const float a = m == -INFINITY ? 0.f : ex2(m - to);
    l *= a;
#pragma unroll
    for (int i = 0; i < C; ++i) acc[i] *= a;
    for (int w = 1; w < 4; ++w) {
      const float e = ml_sh[w].x == -INFINITY ? 0.f : ex2(ml_sh[w].x - to);
      l += ml_sh[w].y * e;
#pragma unroll
      for (int i = 0; i < C; ++i) acc[i] += o_sh[w - 1][lane * C + i] * e;
    }
    m = to;
  }
  if (!mine || written) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  T* o = static_cast<T*>(p.o) + head * p.o_stride_h + (long long)token * p.o_stride_t + lane * C;
  if constexpr (C == 4)
    *reinterpret_cast<uint2*>(o) = make_uint2(pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv));
  else
    *reinterpret_cast<uint32_t*>(o) = pack2<T>(acc[0] * inv, acc[1] * inv);
  if (p.lse && lane == 0) p.lse[(long long)head * s.tokens + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// ------------------------------------------------------------------ host

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn get_encode() {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

waveal_status make_map(CUtensorMap* tm, int dtype, const void* base, int rank, const cuuint64_t* dims, const long long* strides,
                       const cuuint32_t* box, const char* what) {
  EncodeTiledFn enc = get_encode();
  if (!enc) return waveal::fail(WAVEAL_ERR_CUDA, "cuTensorMapEncodeTiled entry point not available");
  cuuint64_t bytes[3];
  for (int i = 0; i + 1 < rank; ++i) bytes[i] = (cuuint64_t)strides[i] * 2;
  const cuuint32_t one[4] = {1, 1, 1, 1};
  const CUresult r = enc(tm, dtype == WAVEAL_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank,
                         const_cast<void*>(base), dims, bytes, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return waveal::fail(WAVEAL_ERR_CUDA, "tensor map for %s rejected (CUresult %d)", what, (int)r);
  return WAVEAL_OK;
}

// SMs of the current device (looked up once a device)
int sm_count() {
  static int counts[64] = {};
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev < 64 && counts[dev]) return counts[dev];
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev < 64) counts[dev] = n;
  return n;
}

// pieces of the line that room is made for, whatever the device (more SMs than this are not used)
constexpr int kMaxCtas = 192;

struct Layout { size_t total, own_base, ml, o, bytes; };

Layout layout(const waveal_cache_desc* c, const waveal_batch_desc* b) {
  const int group = b->q_heads / c->kv_heads;
  const size_t rows = (size_t)b->tokens * b->q_heads * 2 + (size_t)kMaxCtas * 2 * (kTile / group) * group;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Layout l;
  l.total = 0;
  l.own_base = 256;
  l.ml = l.own_base + up((size_t)b->batch * sizeof(long long));
  l.o = l.ml + up(rows * sizeof(float2));
  l.bytes = l.o + up(rows * c->head_dim * sizeof(float));
  return l;
}

waveal_status check_attn(const waveal_cache_desc* c, const waveal_batch_desc* b) {
  if (!c || !b) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "cache and batch are required");
  if (waveal_status e = waveal::check_cache(c)) return e;
  if (waveal_status e = waveal::check_batch(b)) return e;
  if (c->head_dim != 64 && c->head_dim != 128)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", c->head_dim);
  if (b->q_heads <= 0 || b->q_heads % c->kv_heads || b->q_heads / c->kv_heads > kTile)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q_heads %d: a multiple of kv_heads (%d), at most %d times as many", b->q_heads, c->kv_heads, kTile);
  if (b->flags & ~(WAVEAL_PREFIX_CAUSAL | WAVEAL_PREFIX_SELFTEST_LOST_TILE))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "unknown flags 0x%x", b->flags);
  if ((long long)b->tokens * b->q_heads > 1000000000ll)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 10^9 rows (tokens * q_heads)");
  if (b->prefix_len > kMaxKeys || (long long)b->max_pages * c->page_size > kMaxKeys)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^30 keys in a list (prefix_len, max_pages * page_size)");
  for (int i = 0; i < 3; ++i)
    if (c->k_stride[i] % 8 || c->v_stride[i] % 8 || c->k_stride[i] < 0 || c->v_stride[i] < 0)
      return waveal::fail(WAVEAL_ERR_INVALID_ARG, "cache strides must be multiples of 8 elements (16 bytes) and not negative");
  return WAVEAL_OK;
}

template <int D, class T>
waveal_status launch(const CUtensorMap* tm, const Params& p, cudaStream_t st) {
  constexpr size_t smem = Geo<D>::OFF_END + sizeof(Small);
  static_assert(smem <= 232448, "shared memory of an SM");
  static bool set[64] = {};
  int dev = 0;
  WAVEAL_CUDA_OK(cudaGetDevice(&dev));
  if (dev >= 64 || !set[dev]) {
    WAVEAL_CUDA_OK(cudaFuncSetAttribute(k_prefix_attn<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (dev < 64) set[dev] = true;
  }
  k_prefix_attn<D, T><<<p.s.ctas, kThreads, smem, st>>>(tm[0], tm[1], tm[2], tm[3], p);
  WAVEAL_CUDA_OK(cudaGetLastError());
  const long long rows = (long long)p.s.tokens * p.s.kv_heads * p.s.group;
  // few rows have many parts each: four warps a row
  if (rows <= 148 * 16)
    WAVEAL_CUDA_OK(waveal::launch_chained(k_join_parts<D, T, 4>, dim3((unsigned)rows), 128, 0, st, p));
  else
    WAVEAL_CUDA_OK(waveal::launch_chained(k_join_parts<D, T, 1>, dim3((unsigned)((rows + 3) / 4)), 128, 0, st, p));
  waveal::launch_counter() = 2;
  return WAVEAL_OK;
}

}  // namespace

extern "C" waveal_status waveal_prefix_attn_workspace_bytes(const waveal_cache_desc* cache, const waveal_batch_desc* batch, size_t* bytes) {
  if (!bytes) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "bytes is NULL");
  if (waveal_status e = check_attn(cache, batch)) return e;
  *bytes = layout(cache, batch).bytes;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_prefix_attn(const waveal_cache_desc* c, const waveal_batch_desc* b, const void* q, const int64_t* q_stride,
                                            const void* k_cache, const void* v_cache, void* o, const int64_t* o_stride, float* lse,
                                            const int32_t* seq_start, const int32_t* kv_len, const int32_t* page_table,
                                            const int32_t* prefix_pages, float scale, void* ws, size_t ws_bytes, int32_t* dev_status,
                                            void* cuda_stream) {
  if (waveal_status e = check_attn(c, b)) return e;
  if (b->tokens == 0 || b->batch == 0) {
    waveal::launch_counter() = 0;
    return WAVEAL_OK;
  }
  if (!q || !q_stride || !k_cache || !v_cache || !o || !o_stride || !seq_start || !kv_len || (b->max_pages && !page_table) ||
      (b->prefix_len && !prefix_pages))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q, k_cache, v_cache, o, their strides, seq_start and kv_len are required, page_table with "
                                                "max_pages, prefix_pages with prefix_len");
  if (!waveal::aligned(q, 16) || !waveal::aligned(o, 16) || !waveal::aligned(k_cache, 16) || !waveal::aligned(v_cache, 16))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q, o and the caches must be 16-byte aligned");
  for (int i = 0; i < 2; ++i)
    if (q_stride[i] % 8 || o_stride[i] % 8 || q_stride[i] < 0 || o_stride[i] < 0)
      return waveal::fail(WAVEAL_ERR_INVALID_ARG, "strides of q and o must be multiples of 8 elements (16 bytes) and not negative");
  const Layout l = layout(c, b);
  if (!ws || ws_bytes < l.bytes) return waveal::fail(WAVEAL_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? ws_bytes : 0, l.bytes);
  if (!waveal::aligned(ws, 256)) return waveal::fail(WAVEAL_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const int sms = sm_count();
  if (sms <= 0) return waveal::fail(WAVEAL_ERR_CUDA, "number of SMs not available");

  Params p = {};
  p.s.batch = b->batch, p.s.tokens = b->tokens, p.s.kv_heads = c->kv_heads;
  p.s.group = b->q_heads / c->kv_heads, p.s.tq = kTile / p.s.group;
  p.s.prefix_len = b->prefix_len, p.s.max_pages = b->max_pages, p.s.page_shift = __builtin_ctz((unsigned)c->page_size);
  p.s.n_pages = c->n_pages, p.s.causal = b->flags & WAVEAL_PREFIX_CAUSAL ? 1 : 0;
  p.s.table_stride = b->table_stride;
  p.s.seq_start = seq_start, p.s.kv_len = kv_len;
  p.s.ctas = std::min(sms, kMaxCtas);
  char* w = static_cast<char*>(ws);
  p.parts.total = reinterpret_cast<long long*>(w + l.total);
  p.parts.own_base = reinterpret_cast<long long*>(w + l.own_base);
  p.parts.ml = reinterpret_cast<float2*>(w + l.ml);
  p.parts.o = reinterpret_cast<float*>(w + l.o);
  p.page_table = page_table, p.prefix_pages = prefix_pages;
  p.o = o, p.lse = lse, p.o_stride_h = o_stride[0], p.o_stride_t = o_stride[1];
  p.dev_status = dev_status;
  p.drop_tile = b->flags & WAVEAL_PREFIX_SELFTEST_LOST_TILE ? 1 : 0;
  p.wait_limit = p.drop_tile ? kSelfTestCycles : kTimeoutCycles;
  p.sl2 = (scale > 0.f ? scale : 1.0f / std::sqrt((float)c->head_dim)) * 1.4426950408889634f;

  CUtensorMap tm[4];
  const cuuint64_t q_dims[3] = {(cuuint64_t)c->head_dim, (cuuint64_t)b->q_heads, (cuuint64_t)b->tokens};
  const long long q_strides[2] = {q_stride[0], q_stride[1]};
  const cuuint32_t box_q[3] = {64, (cuuint32_t)p.s.group, (cuuint32_t)p.s.tq}, box_q1[3] = {64, (cuuint32_t)p.s.group, 1};
  if (waveal_status e = make_map(&tm[0], c->dtype, q, 3, q_dims, q_strides, box_q, "q")) return e;
  if (waveal_status e = make_map(&tm[1], c->dtype, q, 3, q_dims, q_strides, box_q1, "q")) return e;
  const cuuint64_t kv_dims[4] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->page_size, (cuuint64_t)c->kv_heads, (cuuint64_t)c->n_pages};
  const cuuint32_t box_kv[4] = {64, (cuuint32_t)std::min(c->page_size, kTile), 1, 1};
  const long long k_strides[3] = {c->k_stride[2], c->k_stride[1], c->k_stride[0]}, v_strides[3] = {c->v_stride[2], c->v_stride[1], c->v_stride[0]};
  if (waveal_status e = make_map(&tm[2], c->dtype, k_cache, 4, kv_dims, k_strides, box_kv, "the key cache")) return e;
  if (waveal_status e = make_map(&tm[3], c->dtype, v_cache, 4, kv_dims, v_strides, box_kv, "the value cache")) return e;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (c->dtype == WAVEAL_FP16) return c->head_dim == 128 ? launch<128, __half>(tm, p, st) : launch<64, __half>(tm, p, st);
  return c->head_dim == 128 ? launch<128, __nv_bfloat16>(tm, p, st) : launch<64, __nv_bfloat16>(tm, p, st);
}
