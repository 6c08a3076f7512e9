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
// Inside a CTA (640 threads) there are two slots, each with two S buffers of 64 columns and an O accumulator in tensor memory and
// eight softmax warps:
//   warp 0   items (pieces of units), Q tiles and K tiles by TMA        warp 3   V tiles by TMA
//   warp 1   S = Q K^T of both slots     warp 2   O += P V (tcgen05, P in tensor memory over the columns of S)
//   warps 4-7 and 12-15, 8-11 and 16-19  slot 0, 1: online softmax, four warps an S buffer; the epilogue
// Three kinds of items, by their rows:
//   up to 256  wide: the slots have a row tile each and share every K and V tile, half a tile (64 keys) at a time;
//   up to 128  narrow: the slots take the key tiles in turn and join their accumulators in the epilogue;
//   up to 16   few: keys are the rows of S and query rows its columns, an item has one slot and its two buffers take the tiles in turn.
// O is rescaled only when a row's maximum has grown by more than 2^8.
//
// What bounds it (1 SM, 1.9 GHz; MMA at 64 clk for 128 x 128 x 16): few and narrow items are bound by memory: 16 / 64 / 128 rows a
// key head over 65,536 keys of 37 heads take 200 / 201 / 207 us at a floor of 193 (6.45 TB/s).  Wide items: 3,500 to 3,900 clk a
// key tile, of which the products take 2,530 (64-column products of Q K^T 47 clk instead of 32: both operands come out of
// shared memory) and the exponentials 2,050; 1,024 rows a head over 65,536 keys 1,085 us = 1.17 PFLOP/s, 0.71 of cuBLAS's 1.65
// (in bursts; 65 % of it with the ends of units: 6,240 rows a head over 32,760 keys and their own, 535 us).  The softmax loop is bound by issue
// and by how its instructions arrive: a quarter of the exponentials on the FMA pipe cost 11 %, a row of S in registers 37 % (spills),
// exponentials first and a maximum only where the sum asks for it 3 to 5 %.  head_dim 64: 863 us for half the flops, the same
// exponentials.  A call costs ~8 us before the first tile is there (cold instructions, lengths, the first item) and ~5 us behind the
// last one (epilogue, join): 18.8 us for three tokens over 500 keys.  (Long calls in a row run under the power cap: 64 tokens over 131,072 keys
// 164 us at 1,965 MHz and 189 us at 1,660, the same cycles.)
// Registers: 640 threads leave 96 each, and all four variants spill (268 bytes of stores, 468 of loads a thread by -Xptxas -v).  The form with eight
// softmax warps and more registers took 773 us for four frames, its successor with sixteen 750, today's 535.
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

constexpr int kThreads = 640;
constexpr int kVLoadWarp = 3, kSoftmaxWarp0 = 4;
constexpr int kTile = 128;                           // keys of a tile, rows of a slot
constexpr int kItems = 16;                           // items between the loader and the others
constexpr int kBatch = 8;                            // of them worked out at a time, a lane each
constexpr int kItemReaders = 19;                     // V loader, two issuers, sixteen softmax warps
constexpr long long kTimeoutCycles = 4000000000ll;   // ~2 s at boost clock
constexpr long long kSelfTestCycles = 4000000ll;     // ~2 ms
constexpr int kColumns = 16;                         // rows of an item that is computed with its keys as rows (below), at most
constexpr float kGrowth = 8.0f;                      // log2 of how far a row's maximum may outgrow its reference

// Costs on the line of tiles, about 1,000 clk each: a key tile of a unit of up to 16 rows, of up to 128, of up to 256; what a
// sequence's own tile costs more where its rows are many (its keys come from memory for this unit alone, the prefix's through L2);
// and the start and end of such a unit.
constexpr int kTileFew = 2, kTileNarrow = 3, kTileWide = 4, kOwn = 2, kUnitFew = 5, kUnitNarrow = 8, kUnitWide = 16;
// a piece is not made shorter than this (below it the joining costs more than the tiles)
constexpr int kMinPiece = 8;

template <int D> struct Geo {
  static constexpr int SLABS = D / 64;               // 128-byte-swizzled slabs of 64 channels
  static constexpr int SLAB_BYTES = kTile * 128;
  static constexpr int TILE_BYTES = SLABS * SLAB_BYTES;
  static constexpr int NKS = D == 128 ? 2 : 4, NVS = NKS;
  // P of items of few rows: two halves of 64 keys for each of the four S buffers
  static constexpr int P_HALF = kColumns * 128, P_TILE = 2 * P_HALF;
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + NKS * TILE_BYTES, OFF_P = OFF_V + NVS * TILE_BYTES;
  static constexpr int OFF_END = OFF_P + 4 * P_TILE;
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
  int2* pieces;            // [row / group] of a unit's first row: the first and the last piece that has tiles of it (left by the CTAs that
                           // work on its first and last tile)
  int4* sequences;         // [batch] {first token, new tokens, own keys}, malformed ones with 0 new tokens and starts that ascend; left by thread block 0
};

__host__ __device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// a unit of n0 and n1 tokens in its row tiles: 2 wide, 1 narrow, 0 few rows
__device__ inline int unit_kind(int n0, int n1, int group) { return n1 ? 2 : n0 * group > kColumns ? 1 : 0; }
__device__ inline int tile_cost(int kind) { return kind == 2 ? kTileWide : kind ? kTileNarrow : kTileFew; }
__device__ inline int unit_cost(int kind) { return kind == 2 ? kUnitWide : kind ? kUnitNarrow : kUnitFew; }

// prefix units: 0 .. n on a head, all alike (wide) but the last
struct PrefixLine {
  int per_head, units, whole;     // units of a head; of all heads; dealt out whole
  int tiles, last_weight;
  long long cost, last_cost;      // of a unit, of a head's last

  __device__ explicit PrefixLine(const Shape& s) {
    tiles = ceil_div(s.prefix_len, kTile);
    per_head = tiles ? ceil_div(s.tokens, 2 * s.tq) : 0;
    units = per_head * s.kv_heads;
    whole = units / s.ctas * s.ctas;
    const int rest = s.tokens - (per_head - 1) * 2 * s.tq, kind = unit_kind(min(rest, s.tq), max(rest - s.tq, 0), s.group);
    last_weight = tile_cost(kind);
    cost = (long long)tiles * kTileWide + kUnitWide;
    last_cost = (long long)tiles * last_weight + unit_cost(kind);
  }
  __device__ long long before(int u) const {         // cost of units 0 .. u - 1
    const int h = u / max(per_head, 1), i = u - h * per_head;
    return h * ((per_head - 1) * cost + last_cost) + i * cost;
  }
  __device__ long long at(int u) const { return before(u) - before(whole); }
  __device__ long long total() const { return at(units); }
  __device__ int weight(int i) const { return i == per_head - 1 ? last_weight : kTileWide; }
  __device__ int find(long long x) const {           // the unit that position x of the line lies in
    x += before(whole);
    const long long head = (per_head - 1) * cost + last_cost;
    const int h = x >> 32 ? (int)(x / head) : (int)((unsigned)x / (unsigned)min(head, 0xffffffffll));
    const long long in = x - h * head;
    return h * per_head + min(in >> 32 ? (int)(in / cost) : (int)((unsigned)in / (unsigned)min(cost, 0xffffffffll)), per_head - 1);
  }
};

struct Sequence { int start, n, len; };              // first token, new tokens, own keys

// Starts that decrease would let two sequences claim the same tokens, whose parts would then share their places.  So a sequence whose start lies
// below an earlier one has no new tokens.  `top`: the largest start in front of sequence b of those inside the tensors; where no
// start is malformed they ascend, and 0 does as well.
__device__ inline int raise_top(const Shape& s, int top, int start) { return start <= s.tokens ? max(top, start) : top; }
// bad (may be NULL): {site, value} of what is malformed
__device__ inline Sequence read_sequence(const Shape& s, int b, int top, int* bad) {
  Sequence q = {s.seq_start[b], 0, 0};
  const int end = s.seq_start[b + 1], len = s.kv_len[b];
  if (q.start < top || end < q.start || end > s.tokens) {
    if (bad) bad[0] = 50, bad[1] = q.start < 0 ? q.start : end;
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
  const int kind = unit_kind(u.n0, u.n1, s.group);
  u.weight = tile_cost(kind) + (kind ? kOwn : 0);
  u.cost = u.tiles ? u.tiles * u.weight + unit_cost(kind) : 0;
  return u;
}
// (Causal units differ, and one thread adds them up: ceil(new tokens / (2 tq)) steps at the start of every CTA, one or two for decoding and drafts,
// 3,125 for a prompt of 100,000 tokens at 8 query heads a key head.)
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

// the line cut into pieces: piece c begins at floor(c * total / pieces)
struct Cuts {
  long long each;          // total / pieces
  int rest, pieces;        // total % pieces
  __device__ Cuts(long long total, int ctas) {
    pieces = (int)min((long long)ctas, max(1ll, total / kMinPiece));
    if (total >> 32) {
      each = total / pieces;
    } else {
      each = (unsigned)total / (unsigned)pieces;               // (a 64-bit division takes 1,000 clk)
    }
    rest = (int)(total - each * pieces);
  }
  __device__ long long begin(int c) const { return each * c + (unsigned)(rest * c) / (unsigned)pieces; }
};
// of a unit at `at`: its first tile that begins at x or behind
__device__ inline int first_tile(long long x, long long at, int tiles, int weight) {
  const long long d = x - at;
  if (d <= 0 || d >= (long long)tiles * weight) return d <= 0 ? 0 : tiles;
  return ((unsigned)d + weight - 1) / (unsigned)weight;
}
static_assert(kMinPiece >= kTileWide + kOwn, "a piece between two others of a unit has a tile of it");

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
  int few;                 // 0: both slots, rows of S are query rows; 1: at most kColumns rows, which are its columns, and its keys the rows,
  int slot;                // all in this slot
};

// How far a CTA is on its way through its units: whole ones, its piece's prefix units, its piece's own units.
struct Walk {
  PrefixLine line;
  long long w0, w1;        // its piece of the line
  long long base, at;      // where the sequence, the next unit begin
  Sequence q;
  OwnUnit own;             // its first unit
  int piece, whole, unit;
  int top;                 // of seq (read_sequence)
  int seq, head, i, units; // head -1: the sequence has not been looked at; units: of a head
};

// The next items, up to kBatch, a lane each (a whole warp calls it): 3,000 clk of index arithmetic, for one item or for all of them.
// Returns the lanes that have one; none at the end.
__device__ __noinline__ unsigned next_units(const Shape& s, const Parts& parts, Walk& w, Item& im, int lane) {
  const PrefixLine& line = w.line;
  for (;;) {
    bool have = false;
    __syncwarp();
    if (w.whole < line.whole || w.unit < line.units) {
      const bool whole = w.whole < line.whole;
      const int u = whole ? w.whole + lane * s.ctas : w.unit + lane;
      int j0 = 0, j1 = line.tiles;
      const int h = u / line.per_head, i = u - h * line.per_head;
      bool past = false;                             // behind this CTA's piece
      if (whole) {
        have = lane < kBatch && u < line.whole;
      } else {
        const long long at = line.at(u);
        past = u >= line.units || at >= w.w1;
        j0 = first_tile(w.w0, at, line.tiles, line.weight(i)), j1 = first_tile(w.w1, at, line.tiles, line.weight(i));
        have = lane < kBatch && !past && j0 < j1;
      }
      if (have) {
        im.tiles = j1 - j0;
        im.head = h, im.token = i * 2 * s.tq;
        im.n0 = min(s.tq, s.tokens - im.token), im.n1 = min(s.tq, s.tokens - im.token - im.n0);
        im.first_key = j0 * kTile, im.keys = min(s.prefix_len, j1 * kTile);
        im.list = -1, im.sees = kAll;
        im.direct = 0;
        const long long row = prefix_row(s, h, im.token);
        const int piece = whole ? 0 : w.piece;
        im.row = (int)part_row(s, row, piece);
        int2& pieces = parts.pieces[h * s.tokens + im.token];
        if (j0 == 0) pieces.x = piece;
        if (j1 == line.tiles) pieces.y = piece;
      }
      const bool end = __any_sync(0xffffffffu, past && lane <= kBatch);
      if (lane == 0) {
        if (whole) w.whole += kBatch * s.ctas;
        else w.unit = end ? line.units : w.unit + kBatch;
      }
    } else if (w.seq < s.batch) {
      if (w.head < 0) {
        if (w.base >= w.w1) return 0;
        const Sequence q = read_sequence(s, w.seq, w.top, nullptr);
        const int units = ceil_div(q.n, 2 * s.tq);
        const OwnUnit own = own_unit(s, q, 0);
        const long long cost = units == 0 ? 0 : units == 1 ? own.cost : own_head_cost(s, q);
        const long long skip = w.w0 - w.base;
        const int head = cost && skip > 0 ? (int)min((long long)s.kv_heads, skip / cost) : 0;
        __syncwarp();
        if (lane == 0) {
          w.top = raise_top(s, w.top, q.start);
          w.q = q, w.own = own, w.units = units;
          w.at = w.base + head * cost;
          w.base += cost * s.kv_heads;
          w.head = head, w.i = 0;
          if (cost == 0) ++w.seq, w.head = -1;
        }
        continue;
      }
      // a sequence of one unit: its next heads; else the next units of the head
      const Sequence q = w.q;
      const bool one = w.units == 1;
      const int h = one ? w.head + lane : w.head, i = one ? 0 : w.i + lane;
      OwnUnit u = w.own;
      if (!one) u = own_unit(s, q, min(i, w.units - 1));
      const bool real = lane < kBatch && (one ? h < s.kv_heads : i < w.units);
      long long to = real ? u.cost : 0;
#pragma unroll
      for (int d = 1; d < kBatch; d *= 2) {
        const long long x = __shfl_up_sync(0xffffffffu, to, d);
        if (lane >= d) to += x;
      }
      const long long at = w.at + to - (real ? u.cost : 0), last = w.at + __shfl_sync(0xffffffffu, to, kBatch - 1);
      const int j0 = first_tile(w.w0, at, u.tiles, u.weight), j1 = first_tile(w.w1, at, u.tiles, u.weight);
      have = real && at < w.w1 && j0 < j1;
      if (have) {
        im.tiles = j1 - j0;
        im.head = h, im.token = q.start + u.first;
        im.n0 = u.n0, im.n1 = u.n1;
        im.first_key = j0 * kTile, im.keys = min(u.keys, j1 * kTile);
        im.list = w.seq;
        im.sees = s.causal ? q.len - q.n + u.first + 1 : kAll;
        im.direct = line.tiles == 0 && j0 == 0 && j1 == u.tiles;
        im.row = (int)part_row(s, own_row(s, q, h, u.first), w.piece);
        int2& pieces = parts.pieces[(s.tokens + q.start) * s.kv_heads + h * q.n + u.first];
        if (j0 == 0) pieces.x = w.piece;
        if (j1 == u.tiles) pieces.y = w.piece;
      }
      __syncwarp();
      if (lane == 0) {
        w.at = last;
        if (one) {
          w.head += kBatch;
        } else if ((w.i += kBatch) >= w.units) {
          w.i = 0, ++w.head;
        }
        if (last >= w.w1) w.seq = s.batch;
        else if (w.head >= s.kv_heads) ++w.seq, w.head = -1;
      }
    } else {
      return 0;
    }
    if (have) {
      im.wide = im.n1 > 0;
      im.few = !im.wide && im.n0 * s.group <= kColumns;
    }
    const unsigned who = __ballot_sync(0xffffffffu, have);
    __syncwarp();
    if (who) return who;
  }
}

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

// Two numbers in the tensors' type: the results, and the probabilities, because one product of 16-bit types takes both operands in the same
// type and V is stored in this one.  (Probabilities in two terms would double the second product.)  A probability is off by half a step
// of its own, as the result is: against 64 bits o is off by 0.0023 of its size in bf16 and 0.00029 in fp16, where probabilities in
// fp32 give 0.0017 and 0.00021.  Their sums are taken before the rounding, in fp32.
template <class T> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

constexpr int kStages = 4;                            // of a ring, at most
enum {
  B_ITEM_FULL = 0, B_ITEM_EMPTY = B_ITEM_FULL + kItems, B_Q_FULL = B_ITEM_EMPTY + kItems, B_Q_EMPTY = B_Q_FULL + 2,
  B_K_FULL = B_Q_EMPTY + 2, B_K_EMPTY = B_K_FULL + kStages, B_V_FULL = B_K_EMPTY + kStages, B_V_EMPTY = B_V_FULL + kStages,
  B_S_FULL = B_V_EMPTY + kStages, B_P_FULL = B_S_FULL + 4, B_PV_DONE = B_P_FULL + 4, B_O_EMPTY = B_PV_DONE + 4, B_SUMS = B_O_EMPTY + 2,
  B_SUMS_READ, B_COLS, B_COLS_READ = B_COLS + 2, B_VOTE = B_COLS_READ + 2, B_PAIR = B_VOTE + 4, B_REF = B_PAIR + 8, B_FINAL = B_REF + 8, B_COUNT = B_FINAL + 2
};

// 8 consecutive columns of this thread's lane of tensor memory
#define WAVEAL_TMEM_LD8(taddr, v)                                                                                      \
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"                         \
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])        \
               : "r"(taddr) : "memory")
#define WAVEAL_TMEM_WAIT_LD8(v)                                                                                        \
  asm volatile("tcgen05.wait::ld.sync.aligned;"                                                                        \
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7])::"memory")
#define WAVEAL_TMEM_ST8(taddr, v)                                                                                      \
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"                         \
               ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(taddr) : "memory")
// 8 or 16 columns by the array's length
__device__ __forceinline__ void tmem_load(uint32_t a, uint32_t (&v)[8]) { WAVEAL_TMEM_LD8(a, v); }
__device__ __forceinline__ void tmem_load(uint32_t a, uint32_t (&v)[16]) { WAVEAL_TMEM_LD16(a, v, 0); }
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[8]) { WAVEAL_TMEM_WAIT_LD8(v); }
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[16]) { WAVEAL_TMEM_WAIT_LD16(v, 0); }
__device__ __forceinline__ void tmem_store(uint32_t a, const uint32_t (&v)[8]) { WAVEAL_TMEM_ST8(a, v); }
__device__ __forceinline__ void tmem_store(uint32_t a, const uint32_t (&v)[16]) { WAVEAL_TMEM_ST16(a, v, 0); }
__device__ __forceinline__ void st_shared_u16(uint32_t addr, uint32_t x) {
  asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"((unsigned short)x) : "memory");
}

// what lies behind the tiles in shared memory
struct Small {
  unsigned long long bar[B_COUNT];
  Item items[kItems];
  float ref[2][kTile];                               // [slot][row]: the reference, from one half tile's owner to the next one's
  float pair[2][2][kTile];                           // [slot][owner][row]: sums
  float warp_max[4][4][kColumns];                    // few rows: [buffer][warp]
  float warp_l[2][4][kColumns];                      // few rows, sums: [slot][warp]
  struct { float sum[4][kColumns], ref[kColumns]; } cols[2];   // few rows: what the second half's owners leave for the first's
  float2 sums[kTile];                                // what slot 1 leaves of an item whose key tiles the slots share out: references and sums
  int vote[2][2][2];
  long long warp_sum[kThreads / 32];
  alignas(16) unsigned char walk_space[sizeof(Walk)];
  __device__ Walk& walk() { return *reinterpret_cast<Walk*>(walk_space); }
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

  // boxes of a tile: log2 of the box's rows, how many, and which one (and which slab of it) is this lane's
  __device__ static int box_shift(const Params& p) { return min(p.s.page_shift, 7); }
  __device__ static int boxes(const Params& p, const Item& im, int key) {
    return (min(kTile, im.keys - key) + (1 << box_shift(p)) - 1) >> box_shift(p);
  }
  __device__ int read_page(const Params& p, const Item& im, int key, int lane) const {
    if (key >= im.keys) return 0;
    const int nb = boxes(p, im, key), i = lane < nb ? lane : lane - nb;
    if (lane >= nb * G::SLABS) return 0;
    const int* list = im.list < 0 ? p.prefix_pages : p.page_table + im.list * p.s.table_stride;
    return __ldg(list + ((key + (i << box_shift(p))) >> p.s.page_shift));
  }
  template <int STAGES>
  __device__ bool load(const Ctx& c, const Params& p, const Item& im, int key, bool last, bool drop, int lane, uint32_t smem,
                       uint32_t full, uint32_t empty, const CUtensorMap* tm, int site) {
    const uint32_t st = it % STAGES, ph = it / STAGES & 1;
    const int shift = p.s.page_shift, box = 1 << box_shift(p), nb = boxes(p, im, key);
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
      const int slab = lane >= nb, i = lane - slab * nb;
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
  // leaves no copy in flight, also where another warp gives up once this one has nothing left to load (otherwise its tiles' readers have waited for them)
  __device__ void drain(const Params& p, uint32_t full) const {
    for (int st = 0; st < kStages; ++st)
      if (armed >> st & 1) {
        const long long t0 = clock64();
        while (!mbar_try_wait(full + 8 * st, parity >> st & 1) && clock64() - t0 < p.wait_limit / 4) {}
      }
  }
};

// up to and including this lane
template <class X, class Op> __device__ __forceinline__ X scan_warp(X x, int lane, Op op) {
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const X y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x = op(x, y);
  }
  return x;
}

// Where this thread block's piece of the line begins.  A thread has the costs of its run of sequences [b0, b1) and of its warp up to it; the
// warps' are in sm.warp_sum.  top: of b0 (read_sequence), where ORDERED is false.
template <bool ORDERED>
__device__ __forceinline__ void begin_walk(const Shape& s, Small& sm, const PrefixLine& line, int b0, int b1, long long mine, long long upto, int top) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const long long sums = scan_warp(lane < kThreads / 32 ? sm.warp_sum[lane] : 0, lane, [](long long a, long long b) { return a + b; });
  const long long own_total = __shfl_sync(0xffffffffu, sums, 31), before = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
  if (warp) upto += before;
  const Cuts cuts(max(line.total() + own_total, 1ll), s.ctas);
  const int piece = blockIdx.x;
  const bool has_piece = piece < cuts.pieces;
  const long long w0 = has_piece ? cuts.begin(piece) : 0, w1 = has_piece ? cuts.begin(piece + 1) : 0;
  const long long from = max(w0 - line.total(), 0ll);
  long long base = upto - mine;
  if (has_piece && base <= from && from < upto)
    for (int b = b0; b < b1; ++b) {
      const Sequence q = read_sequence(s, b, ORDERED ? 0 : top, nullptr);
      const long long c = own_head_cost(s, q) * s.kv_heads;
      if (base <= from && from < base + c) sm.walk().seq = b, sm.walk().base = line.total() + base, sm.walk().top = ORDERED ? 0 : top;
      if (!ORDERED) top = raise_top(s, top, q.start);
      base += c;
    }
  if (threadIdx.x == 0) {
    Walk& w = sm.walk();
    w.w0 = w0, w.w1 = w1;
    w.piece = piece, w.whole = blockIdx.x, w.unit = has_piece && w0 < line.total() ? line.find(w0) : line.units;
    w.head = -1;
    w.line = line;
  }
}

// All of that where a start is malformed: the costs once more, now that every thread learns of the starts in front of its run.  (All threads of
// the block call it, behind a barrier.)
__device__ __noinline__ void begin_out_of_order(const Params& p, Small& sm, int b0, int b1) {
  const Shape& s = p.s;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  int m = 0;
  for (int b = b0; b < b1; ++b) m = raise_top(s, m, s.seq_start[b]);
  m = scan_warp(m, lane, [](int a, int b) { return max(a, b); });
  if (lane == 31) sm.warp_sum[warp] = m;
  int top0 = __shfl_up_sync(0xffffffffu, m, 1);
  if (lane == 0) top0 = 0;
  __syncthreads();
  for (int w = 0; w < warp; ++w) top0 = max(top0, (int)sm.warp_sum[w]);
  int top = top0;
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    const Sequence q = read_sequence(s, b, top, nullptr);
    mine += own_head_cost(s, q) * s.kv_heads;
    top = raise_top(s, top, q.start);
    if (blockIdx.x == 0) p.parts.sequences[b] = make_int4(top, q.n, q.len, 0);
  }
  const long long upto = scan_warp(mine, lane, [](long long a, long long b) { return a + b; });
  __syncthreads();                                   // (every warp has read the others' largest starts)
  if (lane == 31) sm.warp_sum[warp] = upto;
  __syncthreads();
  begin_walk<false>(s, sm, PrefixLine(s), b0, b1, mine, upto, top0);
}

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
  } else if (warp == 2) {
    for (int i = lane; i < B_COUNT; i += 32) {
      const bool item = i >= B_ITEM_EMPTY && i < B_ITEM_EMPTY + kItems, warps4 = (i >= B_P_FULL && i < B_P_FULL + 4) || (i >= B_COLS && i < B_VOTE + 4);
      const bool warps8 = (i >= B_O_EMPTY && i < B_O_EMPTY + 2) || i == B_SUMS || i == B_SUMS_READ, warps2 = i >= B_PAIR && i < B_PAIR + 8;
      mbar_init(BAR(i), item ? kItemReaders : warps4 ? 4 : warps8 ? 8 : warps2 ? 2 : 1);
    }
    if (lane < 8) (&sm.vote[0][0][0])[lane] = 0;
    if (lane == 0) sm.abort = 0, sm.walk().seq = s.batch;
    fence_mbar_init();
  } else if (warp == 3 && lane == 0) {
    prefetch_tmap(&tmQ), prefetch_tmap(&tmQ1), prefetch_tmap(&tmK), prefetch_tmap(&tmV);
  }

  // ---- the line of tiles: every thread takes a run of sequences, the block scans their costs
  const PrefixLine line(s);
  const int per = ceil_div(s.batch, kThreads);
  const int b0 = min((int)threadIdx.x * per, s.batch), b1 = min(b0 + per, s.batch);
  long long mine = 0;
  bool bad_start = false;
  for (int b = b0; b < b1; ++b) {
    int bad[2] = {0, 0};
    const Sequence q = read_sequence(s, b, 0, bad);
    mine += own_head_cost(s, q) * s.kv_heads;
    bad_start |= bad[0] == 50;
    if (blockIdx.x == 0) {
      p.parts.sequences[b] = make_int4(q.start, q.n, q.len, 0);
      if (bad[0]) report(p.dev_status, WAVEAL_ERR_BAD_MASK, bad[0], b, bad[1]);
    }
  }
  long long upto = scan_warp(mine, lane, [](long long a, long long b) { return a + b; });
  if (lane == 31) sm.warp_sum[warp] = upto;
  if (!__syncthreads_or(bad_start)) begin_walk<true>(s, sm, line, b0, b1, mine, upto, 0);
  else begin_out_of_order(p, sm, b0, b1);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const Ctx ctx = {&sm.abort, p.dev_status, p.wait_limit};
  bool ok = true;

  // the next item, for everyone but the loader: false when there is none or a wait gave up
  uint32_t item_no = 0;
  // (it stays in shared memory: the softmax warps have no registers to spare for it)
  auto next_item = [&](const Item*& im) {
    const uint32_t slot = item_no % kItems;
    if (!warp_wait(ctx, BAR(B_ITEM_FULL + slot), item_no / kItems & 1, 60)) return ok = false;
    im = &sm.items[slot];
    return im->tiles > 0;
  };
  auto item_done = [&] {
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(B_ITEM_EMPTY + item_no % kItems));
    ++item_no;
  };

  if (warp == 0) {
    // ================================================================ items, Q, K
    TileLoader<D> loader;
    uint32_t q_it = 0, q_armed = 0, q_parity = 0, few_items = 0;
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
    Item next;
    bool more = true;
    while (ok && more) {
      const unsigned who = next_units(s, p.parts, sm.walk(), next, lane);
      const int count = max(__popc(who), 1), nth = __popc(who & ((1u << lane) - 1));   // (at the end: one item without tiles)
      more = who != 0;
      const uint32_t first = item_no;
      for (int i = 0; ok && i < count; ++i, ++item_no)
        if (item_no >= kItems) ok = warp_wait(ctx, BAR(B_ITEM_EMPTY + item_no % kItems), (item_no / kItems & 1) ^ 1, 62);
      if (!ok) break;
      // items of few rows take the slots in turn: one's epilogue runs beside the next one's tiles
      const unsigned few_lanes = __ballot_sync(0xffffffffu, (who >> lane & 1) && next.few);
      if (more ? who >> lane & 1 : lane == 0) {
        const uint32_t slot = (first + nth) % kItems;
        if (!more) next.tiles = 0, next.few = 0;
        next.slot = (few_items + __popc(few_lanes & ((1u << lane) - 1))) & 1;
        sm.items[slot] = next;
        mbar_arrive(BAR(B_ITEM_FULL + slot));
      }
      __syncwarp();
      few_items += __popc(few_lanes);
      for (int i = 0; ok && more && i < count; ++i) {
        const Item im = sm.items[(first + i) % kItems];
        loader.page = loader.read_page(p, im, im.first_key, lane);
        if (!(ok = load_q(im.n0 == 1 ? &tmQ1 : &tmQ, im.token, im.head * s.group, im.n0 == 1 ? 1 : s.tq))) break;
        if (im.wide && !(ok = load_q(im.n1 == 1 ? &tmQ1 : &tmQ, im.token + s.tq, im.head * s.group, im.n1 == 1 ? 1 : s.tq))) break;
        for (int j = 0; ok && j < im.tiles; ++j)
          ok = loader.template load<G::NKS>(ctx, p, im, im.first_key + j * kTile, j == im.tiles - 1, p.drop_tile && blockIdx.x == 0 && loader.it == 0,
                                            lane, sbase + G::OFF_K, BAR(B_K_FULL), BAR(B_K_EMPTY), &tmK, 63);
      }
    }
    // (a wait gave up: the rest is planned all the same.  The joining kernel reads the words that say which pieces hold a unit's parts,
    // and the workspace need not hold anything sensible before)
    while (!ok && more) more = next_units(s, p.parts, sm.walk(), next, lane) != 0;
    loader.drain(p, BAR(B_K_FULL));
    for (int st = 0; st < 2; ++st)
      if (q_armed >> st & 1) {
        const long long t0 = clock64();
        while (!mbar_try_wait(BAR(B_Q_FULL + st), q_parity >> st & 1) && clock64() - t0 < p.wait_limit / 4) {}
      }
  } else if (warp == kVLoadWarp) {
    // ================================================================ V
    TileLoader<D> loader;
    const Item* item;
    while (ok && next_item(item)) {
      const Item im = *item;
      item_done();
      loader.page = loader.read_page(p, im, im.first_key, lane);
      for (int j = 0; ok && j < im.tiles; ++j)
        ok = loader.template load<G::NVS>(ctx, p, im, im.first_key + j * kTile, j == im.tiles - 1, false, lane, sbase + G::OFF_V, BAR(B_V_FULL),
                                          BAR(B_V_EMPTY), &tmV, 64);
    }
    loader.drain(p, BAR(B_V_FULL));
  } else if (warp < kVLoadWarp) {
    // ================================================================ products
    // Two warps issue, one S = Q K^T, the other O += P V: what they do around the products (waits, ring positions,
    // descriptors) takes as long as the products when one warp has it all (2,690 clk a row tile and key tile;
    // with a warp for each slot's products 2,930; the softmax warps leave
    // them few issue slots).  S comes in half tiles of 64 keys, two buffers a slot: one is in its products while the other is in its
    // softmax.  (A product of 64 columns takes 47 clk, not 32: its operands come out of shared memory at that pace.  Whole tiles, one
    // buffer a slot: products and softmax of a slot take turns, 5,210 clk for two row tiles and a key tile.)  S and P of a half tile share columns, so
    // a buffer's next S waits for the end of its last P V.
    // (operands of the products come from shuffles, so that the compiler knows them to be the same in all lanes: otherwise
    // each one is brought from vector registers and the products are issued at half the rate)
    constexpr uint32_t kTypeBits = (1u << 7) | (1u << 10), kType = std::is_same_v<T, __half> ? 0u : kTypeBits;
    constexpr auto typed = [](uint32_t idesc) constexpr { return (idesc & ~kTypeBits) | kType; };
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const Item* im;
    if (warp == 1) {
      const uint64_t q_desc0 = make_desc(sbase + G::OFF_Q, 16, 1024), k_desc0 = make_desc(sbase + G::OFF_K, 16, 1024);
      uint32_t k_st = 0, k_ph = 0, qb = 0, q_ph = 0, used = 0, free_ph = 0;
      // buffer b's last product has ended
      auto buffer_free = [&](int b) {
        if ((used >> b & 1) && !(ok = warp_wait(ctx, BAR(B_PV_DONE + b), (free_ph >> b & 1) ^ 1, 67))) return false;
        used |= 1u << b;
        free_ph ^= 1u << b;
        return true;
      };
      while (ok && next_item(im)) {
        const int wide = __shfl_sync(0xffffffffu, im->wide, 0), tiles = __shfl_sync(0xffffffffu, im->tiles, 0);
        const int keys = __shfl_sync(0xffffffffu, im->keys - im->first_key, 0), few = __shfl_sync(0xffffffffu, im->few, 0), item_slot = __shfl_sync(0xffffffffu, im->slot, 0);
        item_done();
        const uint32_t qb0 = qb;
        if (!(ok = warp_wait(ctx, BAR(B_Q_FULL + qb), q_ph, 65))) break;
        q_ph ^= qb, qb ^= 1;
        if (wide) {
          if (!(ok = warp_wait(ctx, BAR(B_Q_FULL + qb), q_ph, 65))) break;
          q_ph ^= qb, qb ^= 1;
        }
        const uint64_t qd = q_desc0 + (uint64_t)(qb0 * (G::TILE_BYTES >> 4)), qd1 = q_desc0 + (uint64_t)((qb0 ^ 1) * (G::TILE_BYTES >> 4));
        for (int j = 0; ok && j < tiles; ++j) {
          if (!(ok = warp_wait(ctx, BAR(B_K_FULL) + 8 * k_st, k_ph, 66))) break;
          const uint64_t kd = k_desc0 + (uint64_t)(k_st * (G::TILE_BYTES >> 4));
          const bool two = keys - j * kTile > 64;
          if (few) {
            const int b = 2 * item_slot + (j & 1);
            if (!buffer_free(b)) break;
            tc_fence_after();
#pragma unroll
            for (int slab = 0; slab < G::SLABS; ++slab)
              umma4_ss(tm + G::S_COL + b * 64, kd + (uint64_t)(slab * G::SLAB_BYTES >> 4), qd + (uint64_t)(slab * G::SLAB_BYTES >> 4),
                       typed(make_idesc(128, kColumns, false)), slab > 0);
            tc_commit(BAR(B_S_FULL + b));
          } else {
            // (one copy of the code for the four buffers: eight copies did not stay in the instruction caches)
            const int count = (two ? 2 : 1) << wide;
#pragma unroll 1
            for (int x = 0; ok && x < count; ++x) {
              const int b = wide ? (x & 1) * 2 + x / 2 : (j & 1) * 2 + x;
              if (!buffer_free(b)) break;
              tc_fence_after();
              const uint64_t q = wide && (x & 1) ? qd1 : qd;
#pragma unroll
              for (int slab = 0; slab < G::SLABS; ++slab)
                umma4_ss(tm + G::S_COL + b * 64, q + (uint64_t)(slab * G::SLAB_BYTES >> 4), kd + (uint64_t)((slab * G::SLAB_BYTES + (b & 1) * 64 * 128) >> 4),
                         typed(make_idesc(128, 64, false)), slab > 0);
              tc_commit(BAR(B_S_FULL + b));
            }
          }
          if (!ok) break;
          tc_commit(BAR(B_K_EMPTY) + 8 * k_st);
          if (++k_st == (uint32_t)G::NKS) k_st = 0, k_ph ^= 1;
        }
        tc_commit(BAR(B_Q_EMPTY + qb0));
        if (wide) tc_commit(BAR(B_Q_EMPTY + (qb0 ^ 1)));
      }
    } else {
      const uint64_t v_desc0 = make_desc(sbase + G::OFF_V, G::SLAB_BYTES, 1024);
      // V^T as the first operand (head_dim 64: its rows twice, for a product of 128 rows)
      const uint64_t vt_desc0 = make_desc(sbase + G::OFF_V, D == 128 ? G::SLAB_BYTES : 0, 1024);
      uint32_t v_st = 0, v_ph = 0, used = 0, o_ph = 0, p_ph = 0;
      // the accumulator of the slot's last item has been read
      auto accumulator_free = [&](int slot) {
        if ((used >> slot & 1) && !(ok = warp_wait(ctx, BAR(B_O_EMPTY + slot), (o_ph >> slot & 1) ^ 1, 69))) return false;
        used |= 1u << slot;
        o_ph ^= 1u << slot;
        return true;
      };
      auto p_ready = [&](int b) {
        if (!(ok = warp_wait(ctx, BAR(B_P_FULL + b), p_ph >> b & 1, 70))) return false;
        p_ph ^= 1u << b;
        return true;
      };
      while (ok && next_item(im)) {
        const int wide = __shfl_sync(0xffffffffu, im->wide, 0), tiles = __shfl_sync(0xffffffffu, im->tiles, 0);
        const int keys = __shfl_sync(0xffffffffu, im->keys - im->first_key, 0), few = __shfl_sync(0xffffffffu, im->few, 0), item_slot = __shfl_sync(0xffffffffu, im->slot, 0);
        item_done();
        if (few ? !accumulator_free(item_slot) : !accumulator_free(0) || ((wide || tiles > 1) && !accumulator_free(1))) break;
        for (int j = 0; ok && j < tiles; ++j) {
          if (!(ok = warp_wait(ctx, BAR(B_V_FULL) + 8 * v_st, v_ph, 68))) break;
          const int valid = min(kTile, keys - j * kTile), groups = (valid + 15) / 16;
          if (valid < groups * 16) {
            // the last keys of a list: what lies behind them in the page (or was never loaded) must not meet the zeros of P
            const int chunks = (groups * 16 - valid) * 8;
#pragma unroll
            for (int slab = 0; slab < G::SLABS; ++slab)
              for (int i = lane; i < chunks; i += 32)
                st_shared_v4(sbase + G::OFF_V + v_st * G::TILE_BYTES + slab * G::SLAB_BYTES + valid * 128 + i * 16, 0, 0, 0, 0);
            fence_proxy_async();
            __syncwarp();
          }
          const uint64_t vd = v_desc0 + (uint64_t)(v_st * (G::TILE_BYTES >> 4));
          if (few) {
            const int b = 2 * item_slot + (j & 1);
            // (bit 15: the first operand's rows are contiguous)
            const uint32_t idesc = typed(make_idesc(128, kColumns, false)) | 1u << 15;
            const uint64_t vt = vt_desc0 + (uint64_t)(v_st * (G::TILE_BYTES >> 4)), pd = make_desc(sbase + G::OFF_P + b * G::P_TILE, 16, 1024);
            if (!p_ready(b)) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < 8; ++c)
              if (c < groups)
                umma_ss(tm + G::O_COL + b * 64, vt + (uint64_t)(c * 16 * 128 >> 4), pd + (uint64_t)((c / 4 * G::P_HALF + c % 4 * 32) >> 4), idesc,
                        j >= 2 || c > 0);
            tc_commit(BAR(B_PV_DONE + b));
          } else {
            const int count = (groups > 4 ? 2 : 1) << wide;
#pragma unroll 1
            for (int x = 0; ok && x < count; ++x) {
              const int b = wide ? (x & 1) * 2 + x / 2 : (j & 1) * 2 + x, half = b & 1, here = groups - 4 * half;
              if (!p_ready(b)) break;
              tc_fence_after();
              const bool first = half == 0 && (wide ? j == 0 : j < 2);
              const uint32_t d = tm + G::O_COL + b / 2 * kTile, a = tm + G::S_COL + b * 64;
              const uint64_t v = vd + (uint64_t)(half * 64 * 128 >> 4);
              if (here >= 4) {
                umma4_ts(d, a, v, typed(make_idesc(128, D, true)), !first);
              } else {
#pragma unroll 1
                for (int c = 0; c < here; ++c) umma_bf16_ts(d, a + c * 8, v + (uint64_t)(c * 16 * 128 >> 4), typed(make_idesc(128, D, true)), !first || c > 0);
              }
              tc_commit(BAR(B_PV_DONE + b));
            }
          }
          if (!ok) break;
          tc_commit(BAR(B_V_EMPTY) + 8 * v_st);
          if (++v_st == (uint32_t)G::NVS) v_st = 0, v_ph ^= 1;
        }
      }
    }
    // no product is still running when tensor memory is given back
    tc_commit(BAR(B_FINAL + warp - 1));
    __syncwarp();
    const long long t0 = clock64();
    while (!mbar_try_wait(BAR(B_FINAL + warp - 1), 0) && clock64() - t0 < p.wait_limit / 4) {}
  } else {
    // ================================================================ softmax, epilogue
    // Eight warps a slot, four for each of its two half tiles (a warp reaches only the 32 lanes of its quadrant): four softmax warps a
    // scheduler hide each other's latencies.  A row has the same reference in both: the owner of a half tile takes it over
    // from that of the one before, as soon as that one has its maximum.
    const int sw = warp - kSoftmaxWarp0, slot = sw / 4 & 1, half = sw / 8, quad = warp & 3, r = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const uint32_t s_addr = tmem + lanes + G::S_COL + slot * kTile, o_addr = tmem + lanes + G::O_COL + slot * kTile;
    uint32_t uses[4] = {0, 0, 0, 0};                 // of the four S buffers, in the items before this one
    uint32_t joined = 0, joined_few = 0, votes = 0, pairs = 0, refs = 0;

    // Items of up to 16 rows: with query rows as rows of S one warp would have all the exponentials, so there the keys are the rows:
    // S^T = K Q^T has a key a thread and a query row a column.  The slot's two groups of four warps take the tiles in turn, each with its
    // own accumulator, references and sums, and the first joins them.  P^T goes through shared memory, O^T = V^T P^T has a
    // channel a thread.  The four warps of a tile have the same references: they agree at a barrier whether any row has outgrown
    // its own, and only then (in the first tile, seldom afterwards) exchange their maxima.
    const int buffer = slot * 2 + half;
    auto agree = [&] {                               // all four warps have come here
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_VOTE + buffer));
      ok = warp_wait(ctx, BAR(B_VOTE + buffer), votes & 1, 77);
      ++votes;
      return ok;
    };
    // (N: columns that are computed, at least the item's rows: a warp that runs alone pays some 6 clk for each instruction)
    auto few_rows = [&](auto columns, const Item& im, uint32_t use0, uint32_t other0) {
      constexpr int N = decltype(columns)::value, NL = N < 8 ? 8 : N;   // NL: columns loaded
      const int tiles = im.tiles, rows = im.n0 * s.group, all = im.keys - im.first_key, sees0 = im.sees - im.first_key;
      const int unmasked = min(all, sees0), mine = (tiles + 1 - half) / 2;
      float ref[N], l[N];
#pragma unroll
      for (int c = 0; c < N; ++c) ref[c] = -INFINITY, l[c] = 0.f;
      // this thread's key in P: chunk 0 of a row, moved by the row's number mod 8 (128-byte swizzle)
      const uint32_t p_base = sbase + G::OFF_P + buffer * G::P_TILE + r / 64 * G::P_HALF + r % 8 * 2, chunk = r / 8 % 8;
      const uint32_t acc = tmem + lanes + G::O_COL + buffer * 64;
      for (int i = 0; i < mine; ++i) {
        if (!(ok = warp_wait(ctx, BAR(B_S_FULL + buffer), (use0 + i) & 1, 71))) return false;
        tc_fence_after();
        uint32_t sv[NL];
        tmem_load(tmem + lanes + G::S_COL + buffer * 64, sv);
        // the rows that see this thread's key
        const int key = (2 * i + half) * kTile + r;
        unsigned seen = (1u << rows) - 1;
        if (unmasked < (2 * i + half + 1) * kTile) {
          int g = 0, lim = sees0;                    // a token's group of rows after the other
          seen = 0;
#pragma unroll 1
          for (int c = 0; c < rows; ++c) {
            if (key < min(all, lim)) seen |= 1u << c;
            if (++g == s.group) g = 0, ++lim;
          }
        }
        tmem_wait(sv);
        float x[N], over = -INFINITY;
#pragma unroll
        for (int c = 0; c < N; ++c) {
          x[c] = seen >> c & 1 ? __uint_as_float(sv[c]) * p.sl2 : -INFINITY;
          over = fmaxf(over, x[c] - ref[c]);         // (-inf - -inf: NaN, which fmaxf leaves out)
        }
        volatile int* vote = &sm.vote[slot][half][i & 1];
        bool grow = i == 0;
        if (!grow) {
          if (__any_sync(0xffffffffu, over > kGrowth) && lane == 0) *vote = (int)(use0 + i) + 1;
          if (!agree()) return false;
          grow = *vote == (int)(use0 + i) + 1;
        }
        if (grow) {
          float m[N];
#pragma unroll
          for (int c = 0; c < N; ++c) asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m[c]) : "f"(x[c]));
          if (lane == 0) {
#pragma unroll
            for (int c = 0; c < N; c += 4) *reinterpret_cast<float4*>(&sm.warp_max[buffer][quad][c]) = make_float4(m[c], m[c + 1], m[c + 2], m[c + 3]);
          }
          if (!agree()) return false;
#pragma unroll
          for (int c = 0; c < N; c += 4) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float4 y = *reinterpret_cast<const float4*>(&sm.warp_max[buffer][w][c]);
              m[c] = fmaxf(m[c], y.x), m[c + 1] = fmaxf(m[c + 1], y.y), m[c + 2] = fmaxf(m[c + 2], y.z), m[c + 3] = fmaxf(m[c + 3], y.w);
            }
          }
#pragma unroll
          for (int c = 0; c < N; ++c) {
            const float to = m[c] > ref[c] + kGrowth ? m[c] : ref[c];
            m[c] = to == ref[c] ? 1.0f : ex2(ref[c] - to);
            ref[c] = to;
            l[c] *= m[c];
          }
          if (i) {
            // (the last product into this accumulator has ended: this tile's S was issued behind it)
            tmem_load(acc, sv);
            tmem_wait(sv);
#pragma unroll
            for (int c = 0; c < N; ++c) sv[c] = __float_as_uint(__uint_as_float(sv[c]) * m[c]);
            tmem_store(acc, sv);
            tc_wait_st();
          }
        }
#pragma unroll
        for (int c = 0; c < N; c += 2) {
          const float e0 = ex2(x[c] - (ref[c] == -INFINITY ? 0.f : ref[c])), e1 = ex2(x[c + 1] - (ref[c + 1] == -INFINITY ? 0.f : ref[c + 1]));
          l[c] += e0, l[c + 1] += e1;
          const uint32_t pk = pack2<T>(e0, e1);
          st_shared_u16(p_base + c * 128 + ((chunk ^ (c & 7)) << 4), pk);
          st_shared_u16(p_base + (c + 1) * 128 + ((chunk ^ ((c + 1) & 7)) << 4), pk >> 16);
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_P_FULL + buffer));
      }

      // ---- epilogue: sums over the warp's keys
      const bool join = tiles > 1;
      if (half && !join) return true;
#pragma unroll
      for (int w = N / 2, d = 16; w >= 1; w /= 2, d /= 2) {
#pragma unroll
        for (int i = 0; i < w; ++i) {
          const float give = lane & d ? l[i] : l[i + w], keep = lane & d ? l[i + w] : l[i];
          l[i] = keep + __shfl_xor_sync(0xffffffffu, give, d);
        }
      }
#pragma unroll
      for (int d = 16 / N; d >= 1; d /= 2) l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
      constexpr int kLanes = 32 / N;                 // that end up with a row's sum
      auto& cols = sm.cols[slot];
      if (half) {
        if (joined_few && !(ok = warp_wait(ctx, BAR(B_COLS_READ + slot), (joined_few - 1) & 1, 76))) return false;
        cols.sum[quad][lane / kLanes] = l[0];
        if (quad == 0 && lane == 0) {
#pragma unroll
          for (int c = 0; c < N; c += 4) *reinterpret_cast<float4*>(&cols.ref[c]) = make_float4(ref[c], ref[c + 1], ref[c + 2], ref[c + 3]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_COLS + slot));
        ++joined_few;
        return true;
      }
      sm.warp_l[slot][quad][lane / kLanes] = l[0];
      if (!agree()) return false;
      const int row = lane % N;
      float my_ref = ref[0], my_l = 0.f, a0 = 1.0f, a1 = 0.f;
#pragma unroll
      for (int c = 1; c < N; ++c) my_ref = row == c ? ref[c] : my_ref;
#pragma unroll
      for (int w = 0; w < 4; ++w) my_l += sm.warp_l[slot][w][row];
      if (join) {
        if (!(ok = warp_wait(ctx, BAR(B_COLS + slot), joined_few & 1, 73))) return false;
        float other = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) other += cols.sum[w][row];
        const float other_ref = cols.ref[row], m = fmaxf(my_ref, other_ref);
        ++joined_few;
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_COLS_READ + slot));
        a0 = my_ref == -INFINITY ? 0.f : ex2(my_ref - m);
        a1 = other_ref == -INFINITY ? 0.f : ex2(other_ref - m);
        my_ref = m;
        my_l = my_l * a0 + other * a1;
      }
      const bool direct = im.direct;
      if (direct) {
        const float inv = my_l == 0.f ? 0.f : 1.0f / my_l;
        a0 *= inv, a1 *= inv;
      }
      const int head0 = im.head * s.group;
      if (quad == 0 && lane < rows) {
        if (!direct)
          p.parts.ml[im.row + lane] = make_float2(my_ref, my_l);
        else if (p.lse)
          p.lse[(long long)(head0 + lane % s.group) * s.tokens + im.token + lane / s.group] =
              my_l == 0.f ? -INFINITY : (my_ref + log2f(my_l)) * 0.69314718055994531f;
      }
      if (!(ok = warp_wait(ctx, BAR(B_PV_DONE + buffer), (use0 + mine - 1) & 1, 75))) return false;
      if (join && !(ok = warp_wait(ctx, BAR(B_PV_DONE + buffer + 1), (other0 + tiles / 2 - 1) & 1, 74))) return false;
      tc_fence_after();
      uint32_t v[NL], w[NL];
      tmem_load(acc, v);
      tmem_load(acc + 64, w);                        // (of one tile alone: not used)
      tmem_wait(v);
      tmem_wait(w);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_O_EMPTY + slot)), mbar_arrive(BAR(B_O_EMPTY + slot));
      float* part = p.parts.o + (long long)im.row * D + r;
      T* out = static_cast<T*>(p.o) + head0 * p.o_stride_h + im.token * p.o_stride_t + r;
      const long long next_token = p.o_stride_t - (s.group - 1) * p.o_stride_h;
      int g = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float b0 = __shfl_sync(0xffffffffu, a0, i), b1 = __shfl_sync(0xffffffffu, a1, i);
        float y = __uint_as_float(v[i]) * b0;
        if (join) y += __uint_as_float(w[i]) * b1;
        if (i < rows && r < D) {
          if (direct) *reinterpret_cast<unsigned short*>(out) = (unsigned short)pack2<T>(y, 0.f);
          else *part = y;
        }
        part += D;
        if (++g == s.group) g = 0, out += next_token;
        else out += p.o_stride_h;
      }
      return true;
    };

    // a row's other owner has come here too
    auto pair = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_PAIR + slot * 4 + quad));
      ok = warp_wait(ctx, BAR(B_PAIR + slot * 4 + quad), pairs & 1, 78);
      ++pairs;
      return ok;
    };
    const Item* im;
    while (ok && next_item(im)) {
      const bool wide = im->wide;
      const int tiles = im->tiles, all = im->keys - im->first_key;
      if (im->few) {
        const int in = im->slot;
        if (in == slot) {
          const int rows = im->n0 * s.group;
          const uint32_t use0 = slot ? uses[2 + half] : uses[half], other0 = slot ? uses[3] : uses[1];
          if (rows <= 4) few_rows(std::integral_constant<int, 4>{}, *im, use0, other0);
          else if (rows <= 8) few_rows(std::integral_constant<int, 8>{}, *im, use0, other0);
          else few_rows(std::integral_constant<int, 16>{}, *im, use0, other0);
          if (!ok) break;
        }
        (in ? uses[2] : uses[0]) += (tiles + 1) / 2, (in ? uses[3] : uses[1]) += tiles / 2;
        item_done();
        continue;
      }
      // uses of the buffers by this item: every tile has a first half, and but for the last one of a list a second
      uint32_t n[4];
      {
        const int seconds = (all + 63) / 64 - tiles;           // tiles with a second half (all, or all but the last)
        n[0] = wide ? tiles : (tiles + 1) / 2, n[2] = wide ? tiles : tiles / 2;
        n[1] = wide ? seconds : (seconds + 1) / 2, n[3] = wide ? seconds : seconds / 2;
      }
      const uint32_t mine = slot ? n[2 + half] : n[half], others = slot ? n[3 - half] : n[1 - half], halves = mine + others;
      const uint32_t use0 = slot ? uses[2 + half] : uses[half], other0 = slot ? uses[3 - half] : uses[1 - half];
      const int rows = (wide && slot ? im->n1 : im->n0) * s.group;
      const bool idle = quad * 32 >= rows, live = r < rows;
      // keys of this row, from the item's first; and those that every row of the tile sees
      const int sees0 = im->sees - im->first_key + (wide && slot ? im->n0 : 0);
      const int sees = min(all, sees0 + r / s.group), unmasked = min(all, sees0);
      const uint32_t my_s = s_addr + half * 64;
      float ref = -INFINITY, l0 = 0.f, l1 = 0.f;
      for (uint32_t i = 0; i < mine; ++i) {
        if (!(ok = warp_wait(ctx, BAR(B_S_FULL + 2 * slot + half), (use0 + i) & 1, 71))) break;
        // half tile u of the slot: its owner goes on from the reference that u - 1's owner left
        const uint32_t u = 2 * i + half;
        if (idle) {
          // a warp without rows hands the reference on all the same: the chain of hand-overs is what keeps a warp that owns no half tile of an
          // item from testing a phase whose predecessor is not complete, which would pass by its parity and free the accumulators early
          if (u && !(ok = warp_wait(ctx, BAR(B_REF + slot * 4 + quad), (refs + u - 1) & 1, 72))) break;
          sm.ref[slot][r] = ref;
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(B_REF + slot * 4 + quad)), mbar_arrive(BAR(B_P_FULL + 2 * slot + half));
          continue;
        }
        tc_fence_after();
        const int key0 = (wide ? (int)i : 2 * (int)i + slot) * kTile + half * 64, lim = sees - key0;
        const bool masked = unmasked < key0 + 64;
        if (masked) {
          // keys that the row does not see, once and in S itself (in the passes below it would be instructions for every tile)
#pragma unroll 1
          for (int c0 = 0; c0 < 64; c0 += 8) {
            uint32_t v[8];
            WAVEAL_TMEM_LD8(my_s + c0, v);
            WAVEAL_TMEM_WAIT_LD8(v);
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = c < lim - c0 ? v[c] : 0xff800000u;
            WAVEAL_TMEM_ST8(my_s + c0, v);
          }
          tc_wait_st();
        }
        // S is loaded twice, for the maximum and for the exponentials (a row of it in registers spills), 16 columns at a time, the next ones
        // on their way while these are computed
        float mx;
        uint32_t w[2][16];
        {
          WAVEAL_TMEM_LD16(my_s, w[0], 0);
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t (&x)[16] = w[q & 1];
            WAVEAL_TMEM_WAIT_LD16(x, 0);
            if (q < 3) WAVEAL_TMEM_LD16(my_s + (q + 1) * 16, w[(q + 1) & 1], 0);
#pragma unroll
            for (int c = 0; c < 16; c += 8) {
#pragma unroll
              for (int k = 0; k < 4; ++k) m4[k] = fmax3(m4[k], __uint_as_float(x[c + 2 * k]), __uint_as_float(x[c + 2 * k + 1]));
            }
          }
          mx = fmaxf(fmax3(m4[0], m4[1], m4[2]), m4[3]);
        }
        mx *= p.sl2;
        float now = -INFINITY;
        if (u) {
          if (!(ok = warp_wait(ctx, BAR(B_REF + slot * 4 + quad), (refs + u - 1) & 1, 72))) break;
          now = sm.ref[slot][r];
        }
        const bool grows = live && mx > now + kGrowth;
        const float to = grows ? mx : now;
        sm.ref[slot][r] = to;
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_REF + slot * 4 + quad));
        if (to != ref) {
          const float a = ex2(ref - to);
          l0 *= a, l1 *= a;
          ref = to;
        }
        if (__any_sync(0xffffffffu, grows) && u) {
          // the accumulators, between the product before this one and this one's
          if (!(ok = warp_wait(ctx, BAR(B_PV_DONE + 2 * slot + (half ^ 1)), (other0 + i - (half ^ 1)) & 1, 73))) break;
          tc_fence_after();
          const float a = grows ? ex2(now - to) : 1.0f;
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            WAVEAL_TMEM_LD16(o_addr + c, w[0], 0);
            WAVEAL_TMEM_WAIT_LD16(w[0], 0);
#pragma unroll
            for (int k = 0; k < 16; ++k) w[0][k] = __float_as_uint(__uint_as_float(w[0][k]) * a);
            WAVEAL_TMEM_ST16(o_addr + c, w[0], 0);
          }
          tc_wait_st();
        }
        const float b = ref == -INFINITY ? 0.f : -ref;
        {
          WAVEAL_TMEM_LD16(my_s, w[0], 0);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t (&x)[16] = w[q & 1];
            WAVEAL_TMEM_WAIT_LD16(x, 0);
            if (q < 3) WAVEAL_TMEM_LD16(my_s + (q + 1) * 16, w[(q + 1) & 1], 0);
            uint32_t pk[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float x0, x1;
              ffma2(x0, x1, __uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]), p.sl2, p.sl2, b, b);
              x0 = ex2(x0), x1 = ex2(x1);
              fadd2(l0, l1, l0, l1, x0, x1);
              pk[k] = pack2<T>(x0, x1);
            }
            WAVEAL_TMEM_ST8(my_s + q * 8, pk);
          }
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_P_FULL + 2 * slot + half));
      }
      if (!ok) break;

      // ---- epilogue: the sums of a row's owners
      const bool join = !wide && tiles > 1;
      float l = l0 + l1;
      // the slot's last product
      const uint32_t last_bar = B_PV_DONE + 2 * slot + (mine > others || (mine == others && half) ? half : half ^ 1);
      const uint32_t last_ph = (mine > others || (mine == others && half) ? use0 + mine : other0 + others) - 1;
      if (halves) {
        if (!(ok = warp_wait(ctx, BAR(B_REF + slot * 4 + quad), (refs + halves - 1) & 1, 72))) break;
        const float to = sm.ref[slot][r];
        if (to != ref) l *= ex2(ref - to), ref = to;
        refs += halves;
        sm.pair[slot][half][r] = l;
        if (!pair()) break;
        l += sm.pair[slot][half ^ 1][r];
        if (!pair()) break;                          // (read: the next item's may be left there)
      }
      // slot 1's last product of a narrow item
      const uint32_t join_bar = B_PV_DONE + 2 + (n[2] == n[3] ? 1 : 0), join_ph = (n[2] == n[3] ? uses[3] + n[3] : uses[2] + n[2]) - 1;
#pragma unroll
      for (int k = 0; k < 4; ++k) uses[k] += n[k];
      if (!wide && slot) {
        if (join) {
          if (joined && !(ok = warp_wait(ctx, BAR(B_SUMS_READ), (joined - 1) & 1, 76))) break;
          if (!idle && half == 0) sm.sums[r] = make_float2(ref, l);
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(B_SUMS));
          ++joined;
        }
        item_done();
        continue;
      }
      float a0 = 1.0f, a1 = 0.0f;
      if (join) {
        if (!(ok = warp_wait(ctx, BAR(B_SUMS), joined & 1, 73))) break;
        const float2 other = idle ? make_float2(0.f, 0.f) : sm.sums[r];
        ++joined;
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_SUMS_READ));
        if (!(ok = warp_wait(ctx, BAR(join_bar), join_ph & 1, 74))) break;
        const float m = fmaxf(ref, other.x);
        a0 = ref == -INFINITY ? 0.f : ex2(ref - m);
        a1 = other.x == -INFINITY ? 0.f : ex2(other.x - m);
        ref = m;
        l = l * a0 + other.y * a1;
      }
      if (!(ok = warp_wait(ctx, BAR(last_bar), last_ph & 1, 75))) break;
      tc_fence_after();
      if (!idle) {
        const bool second = wide && slot, direct = im->direct;
        const long long out_row = im->row + (long long)(second ? im->n0 * s.group : 0) + r;
        float scale_o = 1.0f;
        T* o_ptr = nullptr;
        if (direct) {
          scale_o = l == 0.f ? 0.f : 1.0f / l;
          const int head = im->head * s.group + r % s.group, tok = im->token + (second ? im->n0 : 0) + r / s.group;
          o_ptr = static_cast<T*>(p.o) + head * p.o_stride_h + tok * p.o_stride_t;
          if (live && half == 0 && p.lse)
            p.lse[(long long)head * s.tokens + tok] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.69314718055994531f;
        } else if (live && half == 0) {
          p.parts.ml[out_row] = make_float2(ref, l);
        }
        a0 *= scale_o, a1 *= scale_o;
#pragma unroll 1
        for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 16) {
          uint32_t v[16], w[16];
          WAVEAL_TMEM_LD16(o_addr + c, v, 0);
          if (join) {
            WAVEAL_TMEM_LD16(o_addr + kTile + c, w, 0);
            WAVEAL_TMEM_WAIT_LD16(w, 0);
          }
          WAVEAL_TMEM_WAIT_LD16(v, 0);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x = __uint_as_float(v[i]) * a0;
            if (join) x += __uint_as_float(w[i]) * a1;
            v[i] = __float_as_uint(x);
          }
          if (live) {
            if (direct) {
#pragma unroll
              for (int i = 0; i < 8; ++i) w[i] = pack2<T>(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
#pragma unroll
              for (int i = 0; i < 8; i += 4) *reinterpret_cast<uint4*>(o_ptr + c + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
              float* dst = p.parts.o + out_row * D + c;
              st_global_v8(dst, v);
              st_global_v8(dst + 8, v + 8);
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
      item_done();
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------ parts -> output

// WARPS warps a row (a token's query head), with every WARPS-th part each.  The parts' references and sums are read a lane each, so that
// only one round trip stands before the loads of the parts themselves, which do not wait for each other.
template <int D, class T, int WARPS>
__global__ void __launch_bounds__(128) k_join_parts(const __grid_constant__ Params p) {
  constexpr int C = D / 32;                          // channels of a lane
  const Shape& s = p.s;
  const unsigned heads = s.kv_heads * s.group, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const unsigned id = blockIdx.x * (4 / WARPS) + warp / WARPS;
  const int token = id / heads, head = id - token * heads, h = head / s.group, g = head - h * s.group;
  __shared__ float o_sh[WARPS > 1 ? 3 : 1][D];
  waveal::wait_for_previous_kernel();
  bool mine = token < s.tokens;

  // whose token is it (a token of no sequence is left alone)
  Sequence q = {0, 0, 0};
  if (mine) {
    auto sequence = [&](int b) {
      const int4 x = p.parts.sequences[b];
      return Sequence{x.x, x.y, x.z};
    };
    q = sequence((int)((unsigned long long)token * s.batch / s.tokens));
    if (token < q.start || token >= q.start + q.n) {
      int l = 0, r = s.batch - 1;
      while (l < r) {
        const int m = (l + r + 1) >> 1;
        if (p.parts.sequences[m].x <= token) l = m; else r = m - 1;
      }
      q = sequence(l);
    }
    mine = token >= q.start && token < q.start + q.n;
  }

  float m = -INFINITY, l = 0.f, acc[C];
#pragma unroll
  for (int i = 0; i < C; ++i) acc[i] = 0.f;
  bool written = false;
  if (mine) {
    int2 shared = {0, -1}, own = {0, -1};            // pieces
    if (s.prefix_len) shared = p.parts.pieces[h * s.tokens + token / (2 * s.tq) * 2 * s.tq];
    const int first = (token - q.start) / (2 * s.tq) * 2 * s.tq;
    if ((s.causal ? q.len - q.n + min(q.n, first + 2 * s.tq) : q.len) > 0) own = p.parts.pieces[(s.tokens + q.start) * s.kv_heads + h * q.n + first];
    const int n0 = shared.y - shared.x + 1, n = n0 + own.y - own.x + 1;
    written = s.prefix_len == 0 && n == 1;
    const long long row0 = part_row(s, prefix_row(s, h, token) + g, shared.x), row1 = part_row(s, own_row(s, q, h, token - q.start) + g, own.x);
    for (int base = 0; base < n && !written; base += 32) {
      const int k = base + lane;
      const long long at = k < n0 ? part_row(s, row0, k) : part_row(s, row1, k - n0);
      const float2 ml = k < n ? p.parts.ml[at] : make_float2(-INFINITY, 0.f);
      float to = fmaxf(m, ml.x);
#pragma unroll
      for (int d = 16; d >= 1; d /= 2) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, d));
      const float scale = m == -INFINITY ? 0.f : ex2(m - to), weight = ml.x == -INFINITY ? 0.f : ex2(ml.x - to);
      float sum = ml.y * weight;
#pragma unroll
      for (int d = 16; d >= 1; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      m = to;
      l = l * scale + sum;
#pragma unroll
      for (int i = 0; i < C; ++i) acc[i] *= scale;
      const int count = min(32, n - base);
#pragma unroll 4
      for (int j = WARPS > 1 ? warp : 0; j < count; j += WARPS) {
        const float w = __shfl_sync(0xffffffffu, weight, j);
        const float* src = p.parts.o + __shfl_sync(0xffffffffu, at, j) * D + lane * C;
        if constexpr (C == 4) {
          const float4 x = *reinterpret_cast<const float4*>(src);
          acc[0] += x.x * w, acc[1] += x.y * w, acc[2] += x.z * w, acc[3] += x.w * w;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(src);
          acc[0] += x.x * w, acc[1] += x.y * w;
        }
      }
    }
  }
  if constexpr (WARPS > 1) {
    if (warp) {
#pragma unroll
      for (int i = 0; i < C; ++i) o_sh[warp - 1][lane * C + i] = acc[i];
    }
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
#pragma unroll
      for (int i = 0; i < C; ++i) acc[i] += o_sh[w - 1][lane * C + i];
    }
  }
  if (!mine || written) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  T* o = static_cast<T*>(p.o) + head * p.o_stride_h + token * p.o_stride_t + lane * C;
  if constexpr (C == 4)
    *reinterpret_cast<uint2*>(o) = make_uint2(pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv));
  else
    *reinterpret_cast<uint32_t*>(o) = pack2<T>(acc[0] * inv, acc[1] * inv);
  if (p.lse && lane == 0) p.lse[(long long)head * s.tokens + token] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// ------------------------------------------------------------------ host

waveal_status make_map(CUtensorMap* tm, int dtype, const void* base, int rank, const cuuint64_t* dims, const long long* strides,
                       const cuuint32_t* box, const char* what) {
  const auto enc = waveal::tensor_map_encoder();
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

// pieces of the line that room is made for, whatever the device (more SMs than this are not used)
constexpr int kMaxCtas = 192;

struct Layout { size_t pieces, sequences, ml, o, bytes; };

Layout layout(const waveal_cache_desc* c, const waveal_batch_desc* b) {
  const int group = b->q_heads / c->kv_heads;
  const size_t rows = (size_t)b->tokens * b->q_heads * 2 + (size_t)kMaxCtas * 2 * (kTile / group) * group;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Layout l;
  l.pieces = 0;
  l.sequences = up((size_t)b->tokens * c->kv_heads * 2 * sizeof(int2));
  l.ml = l.sequences + up((size_t)b->batch * sizeof(int4));
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
  const int sms = waveal::sm_count();
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
  p.parts.pieces = reinterpret_cast<int2*>(w + l.pieces);
  p.parts.sequences = reinterpret_cast<int4*>(w + l.sequences);
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
