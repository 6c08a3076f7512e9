// Rotary positions, and new keys and values into a paged cache with the rotation applied on the way.
//
// Pair (a, b) of a token at position p becomes amplitude * (a cos - b sin, b cos + a sin) with
// angle = 2 pi * frac(p * f).  f is given in units of 2^-64 turns, so p * f cut to 64 bits IS the fraction; its top 32
// bits, as a signed number of half turns in [-1, 1), go to sincospi: no rounding grows with the position, and
// the gradient is the same with the sine negated.
//
// Bound by memory: every channel is read once and written once (6 flops for each 8 bytes).  A thread has one
// (token, two vectors of VEC channels) and walks the heads with the cosines and sines of its VEC pairs in
// registers: they cost ~50 instructions a pair, shared by all heads of the token.  The two vectors stand half of
// rot_dim apart in both layouts, so that a warp's loads are contiguous either way.  Where the tokens alone do not fill the
// GPU the heads are split over as many blocks as are resident at once (kBlocksWanted).
//
// Measured (GPU time, 6.45 TB/s is a plain copy's rate): 80 heads of 32,760 tokens, three axes, 217 us = 6.19 TB/s; fp32 gradients of
// 16 heads of 4,099 tokens 9.6 us = 5.2 TB/s; four frames of 1,560 tokens into the cache, 40 + 80 heads, 71 us = 5.4 TB/s; 7,275
// tokens of ragged prompts, 28 + 8 heads of 64 in fp16, 15 us = 4.5 TB/s; 8 tokens of 40 heads 2.2 us.
// Four blocks an SM (64 registers) carry it: with three of 80 registers the clip takes 283 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cmath>
#include "host_common.h"

namespace {

constexpr int kThreads = 256;
// blocks to aim at by splitting the heads: the 4 that are resident on each of 148 SMs (the four frames above: 8 an SM 71.3 us, 4 an
// SM 70.9, 2 an SM 114; the ragged fp16 prompts 16.0 / 14.9 / 15.9: every block works out its angles again)
constexpr int kBlocksWanted = 148 * 4;
constexpr int kMaxHeadDim = 512;

struct Strides { long long h, t; };

struct RotateParams {
  const void* src[3];          // q, k, v (v is copied, never rotated)
  void* dst[3];
  Strides in[3], out[3];       // elements; `out` of k and v in a cache: {head, slot}
  long long out_page[3];
  int heads[3];
  int tokens, head_dim, rot_dim, slots;   // slots: threads a token
  int tokens_per_block, heads_per_block;
  int in_place;                // bits 0, 1: that output is its input, the channels behind rot_dim stay
  const int* positions;        // [axes][tokens] or NULL
  const long long* freqs;
  int axis_end0, axis_end1;    // pairs below end0 turn with axis 0, below end1 with axis 1, the others with axis 2
  float amplitude, sign;
  // cache
  const int* seq_start;
  const int* kv_len;
  const int* page_table;
  long long table_stride;
  int batch, max_pages, page_shift, n_pages, prefix_len;
  int* dev_status;
};

template <class T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }

// (a, b) turned.  Written out as one product and one multiply-add each, so that every width of vector gives the same bits.
__device__ __forceinline__ float turn_a(float a, float b, float c, float s) { return __fmaf_rn(a, c, -__fmul_rn(b, s)); }
__device__ __forceinline__ float turn_b(float a, float b, float c, float s) { return __fmaf_rn(b, c, __fmul_rn(a, s)); }

template <class T, int VEC> struct alignas(sizeof(T) * VEC) Vec { T v[VEC]; };

// Where a token of the batch belongs.
struct Place {
  int live;      // its queries are written
  int slot;      // place inside its page, or -1: keys and values are not written
  long long page;
  long long position;  // prefix_len + place among the own keys (two numbers of 31 bits)
};

__device__ void report(int* status, int site, int seq, int value) {
  if (status && atomicCAS(status, 0, (int)WAVEAL_ERR_BAD_MASK) == 0) {
    status[1] = site;
    status[2] = seq;
    status[3] = value;
  }
}

__device__ Place find_place(const RotateParams& p, int t) {
  Place w = {0, -1, 0, 0};
  // Which sequence: where all have as many new tokens, the guess is right (one round trip to memory instead of log2(batch)).
  int b = (int)((long long)t * p.batch / p.tokens);
  int lo = p.seq_start[b], hi = p.seq_start[b + 1];
  if (t < lo || t >= hi) {
    int l = 0, r = p.batch;                       // last b with seq_start[b] <= t
    while (l < r) {
      const int m = (l + r + 1) >> 1;
      if (p.seq_start[m] <= t) l = m; else r = m - 1;
    }
    b = l;
    if (b >= p.batch) return w;                   // behind the last sequence's tokens
    lo = p.seq_start[b], hi = p.seq_start[b + 1];
  }
  // not in front of the first sequence's tokens, nor in a malformed one (check_starts reports those)
  if (lo < 0 || t < lo || t >= hi || hi > p.tokens) return w;
  w.live = 1;
  const int len = p.kv_len[b];
  const long long place = (long long)len - (hi - lo) + (t - lo);
  w.position = p.prefix_len + place;
  if (len < hi - lo || len > ((long long)p.max_pages << p.page_shift)) {
    report(p.dev_status, 41, b, len);
    return w;
  }
  const int page = p.page_table[b * p.table_stride + (place >> p.page_shift)];
  if (page < 0 || page >= p.n_pages) {
    report(p.dev_status, 42, b, page);
    return w;
  }
  w.page = page;
  w.slot = (int)(place & ((1 << p.page_shift) - 1));
  return w;
}

// Starts that decrease or leave the tensors, each of them looked at by one thread of the grid: a token's way to its sequence passes a few
// only.  The threads of a block that find places have the lowest numbers, those that look here first the highest.
__device__ __forceinline__ void check_starts(const RotateParams& p) {
  if (blockIdx.y) return;
  for (long long b = (long long)blockIdx.x * kThreads + kThreads - 1 - threadIdx.x; b < p.batch; b += (long long)gridDim.x * kThreads) {
    const int lo = p.seq_start[b], hi = p.seq_start[b + 1];
    if (lo < 0 || hi < lo || hi > p.tokens) report(p.dev_status, 40, (int)b, lo < 0 ? lo : hi);
  }
}

template <class T, int VEC, bool INTERLEAVED, bool CACHE>
__global__ void __launch_bounds__(kThreads, 4) k_rotate(const __grid_constant__ RotateParams p) {
  using V = Vec<T, VEC>;
  __shared__ Place places[CACHE ? kThreads : 1];
  const int local = threadIdx.x / p.slots, slot = threadIdx.x - local * p.slots;
  const long long t0 = (long long)blockIdx.x * p.tokens_per_block;
  if constexpr (CACHE) {
    if (threadIdx.x < p.tokens_per_block && t0 + threadIdx.x < p.tokens) places[threadIdx.x] = find_place(p, (int)t0 + threadIdx.x);
    check_starts(p);
    __syncthreads();
  }
  if (local >= p.tokens_per_block || t0 + local >= p.tokens) return;
  const int t = (int)t0 + local;
  Place place = {1, 0, 0, 0};
  if constexpr (CACHE) place = places[local];

  // this thread's channels: rotated pairs, or two vectors behind them
  const int half = p.rot_dim / 2, rot_slots = half / VEC;
  const bool turns = slot < rot_slots;
  int e0, e1;
  float c[VEC], s[VEC];
  int first = blockIdx.y * p.heads_per_block, left = p.heads_per_block;
  if (turns) {
    e0 = INTERLEAVED && VEC == 1 ? 2 * slot : slot * VEC;
    e1 = INTERLEAVED && VEC == 1 ? 2 * slot + 1 : e0 + half;
    if (!CACHE || first < p.heads[0] + p.heads[1])   // (a block of values alone needs no angles)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      // halves: pair e0 + i is (e0 + i, e1 + i); interleaved: the pairs of the first vector, then those of the second
      const int pair = !INTERLEAVED ? e0 + i : VEC == 1 ? slot : i < VEC / 2 ? e0 / 2 + i : e1 / 2 + i - VEC / 2;
      const int axis = pair < p.axis_end0 ? 0 : pair < p.axis_end1 ? 1 : 2;
      const long long pos = !CACHE || p.positions ? __ldg(p.positions + (long long)axis * p.tokens + t) : place.position;
      const unsigned long long turn = (unsigned long long)pos * (unsigned long long)__ldg(p.freqs + pair);
      sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s[i], &c[i]);
      s[i] *= p.sign * p.amplitude;
      c[i] *= p.amplitude;
    }
  } else {
    e0 = p.rot_dim + (slot - rot_slots) * 2 * VEC;
    e1 = e0 + VEC;
  }

#pragma unroll
  for (int k = 0; k < (CACHE ? 3 : 2); ++k) {
    if (left <= 0) break;
    if (first >= p.heads[k]) {
      first -= p.heads[k];
      continue;
    }
    const int n = min(left, p.heads[k] - first);
    const T* src = static_cast<const T*>(p.src[k]) + (long long)first * p.in[k].h + (long long)t * p.in[k].t;
    T* dst = static_cast<T*>(p.dst[k]) + (long long)first * p.out[k].h;
    bool live = place.live;
    if (CACHE && k > 0) {
      live = place.slot >= 0;
      dst += place.page * p.out_page[k] + (long long)place.slot * p.out[k].t;
    } else {
      dst += (long long)t * p.out[k].t;
    }
    const bool turn_here = turns && (!CACHE || k < 2);
    // v has no rotated part: its vectors are taken two by two from the front
    const int a0 = CACHE && k == 2 ? slot * 2 * VEC : e0, a1 = CACHE && k == 2 ? a0 + VEC : e1;
    if (!turn_here && (a0 >= p.head_dim || (k < 2 && (p.in_place >> k & 1)))) live = false;
    if (live) {
      const bool two = a1 < p.head_dim;
#pragma unroll 2
      for (int h = 0; h < n; ++h) {
        const V x = *reinterpret_cast<const V*>(src + a0);
        V y = x;
        if (two) y = *reinterpret_cast<const V*>(src + a1);
        V u = x, w = y;
        if (turn_here) {
          if constexpr (INTERLEAVED && VEC > 1) {
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) {
              const float xa = to_float(x.v[2 * i]), xb = to_float(x.v[2 * i + 1]);
              const float ya = to_float(y.v[2 * i]), yb = to_float(y.v[2 * i + 1]);
              u.v[2 * i] = from_float<T>(turn_a(xa, xb, c[i], s[i]));
              u.v[2 * i + 1] = from_float<T>(turn_b(xa, xb, c[i], s[i]));
              w.v[2 * i] = from_float<T>(turn_a(ya, yb, c[VEC / 2 + i], s[VEC / 2 + i]));
              w.v[2 * i + 1] = from_float<T>(turn_b(ya, yb, c[VEC / 2 + i], s[VEC / 2 + i]));
            }
          } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const float a = to_float(x.v[i]), b = to_float(y.v[i]);
              u.v[i] = from_float<T>(turn_a(a, b, c[i], s[i]));
              w.v[i] = from_float<T>(turn_b(a, b, c[i], s[i]));
            }
          }
        }
        *reinterpret_cast<V*>(dst + a0) = u;
        if (two) *reinterpret_cast<V*>(dst + a1) = w;
        src += p.in[k].h;
        dst += p.out[k].h;
      }
    }
    left -= n;
    first = 0;
  }
}

// ------------------------------------------------------------------ host

int dtype_size(int dtype) { return dtype == WAVEAL_FP32 ? 4 : 2; }

waveal_status check_rotation(const waveal_rotation& r, int head_dim) {
  if (r.rot_dim < 2 || r.rot_dim % 2 || r.rot_dim > head_dim)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "rot_dim %d: even, 2 .. head_dim (%d)", r.rot_dim, head_dim);
  if (r.pairs != WAVEAL_PAIRS_HALVES && r.pairs != WAVEAL_PAIRS_INTERLEAVED)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "pairs %d: WAVEAL_PAIRS_HALVES or WAVEAL_PAIRS_INTERLEAVED", r.pairs);
  if (r.axes < 1 || r.axes > 3) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "axes %d: 1 .. 3", r.axes);
  long long sum = 0;
  for (int a = 0; a < 3; ++a) {
    if (r.axis_pairs[a] < 0 || (a >= r.axes && r.axis_pairs[a] != 0))
      return waveal::fail(WAVEAL_ERR_INVALID_ARG, "axis_pairs[%d] = %d with %d axes", a, r.axis_pairs[a], r.axes);
    sum += r.axis_pairs[a];
  }
  if (sum != r.rot_dim / 2)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "axis_pairs add up to %lld, rot_dim/2 is %d", sum, r.rot_dim / 2);
  if (!std::isfinite(r.amplitude)) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "amplitude is not finite");
  return WAVEAL_OK;
}

void set_rotation(RotateParams& p, const waveal_rotation& r) {
  p.rot_dim = r.rot_dim;
  p.axis_end0 = r.axis_pairs[0];
  p.axis_end1 = r.axis_pairs[0] + r.axis_pairs[1];
  p.amplitude = r.amplitude;
  p.sign = r.inverse ? -1.0f : 1.0f;
}

// the widest vector (16 bytes, 8, one element) that divides the channels' parts, the strides and the addresses
int widest(const RotateParams& p, int size, bool cache) {
  for (int vec : {16 / size, 8 / size}) {
    if (vec < 2 || (p.rot_dim / 2) % vec || p.head_dim % vec) continue;
    bool fits = true;
    for (int k = 0; k < 3; ++k) {
      if (!p.heads[k]) continue;
      for (long long s : {p.in[k].h, p.in[k].t, p.out[k].h, p.out[k].t, p.out_page[k]}) fits = fits && s % vec == 0;
      fits = fits && waveal::aligned(p.src[k], (size_t)vec * size) && waveal::aligned(p.dst[k], (size_t)vec * size);
    }
    if (fits) return vec;
  }
  return 1;
}

template <class T, int VEC, bool CACHE>
void launch_layout(const RotateParams& p, dim3 grid, int pairs, cudaStream_t st) {
  if (pairs == WAVEAL_PAIRS_INTERLEAVED)
    k_rotate<T, VEC, true, CACHE><<<grid, kThreads, 0, st>>>(p);
  else
    k_rotate<T, VEC, false, CACHE><<<grid, kThreads, 0, st>>>(p);
}

template <bool CACHE>
waveal_status launch(RotateParams& p, int dtype, int pairs, cudaStream_t st) {
  const int size = dtype_size(dtype), vec = widest(p, size, CACHE);
  const int rest = p.head_dim - p.rot_dim;
  p.slots = p.rot_dim / 2 / vec + (rest + 2 * vec - 1) / (2 * vec);
  p.tokens_per_block = kThreads / p.slots;
  const long long blocks = ((long long)p.tokens + p.tokens_per_block - 1) / p.tokens_per_block;
  const int heads = p.heads[0] + p.heads[1] + p.heads[2];
  const long long split = std::min<long long>(std::max<long long>(kBlocksWanted / blocks, 1), std::min(heads, 65535));
  p.heads_per_block = (int)((heads + split - 1) / split);
  const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
  if (dtype == WAVEAL_FP32) {
    if constexpr (!CACHE) {
      if (vec == 4) launch_layout<float, 4, false>(p, grid, pairs, st);
      else if (vec == 2) launch_layout<float, 2, false>(p, grid, pairs, st);
      else launch_layout<float, 1, false>(p, grid, pairs, st);
    }
  } else if (dtype == WAVEAL_BF16) {
    if (vec == 8) launch_layout<__nv_bfloat16, 8, CACHE>(p, grid, pairs, st);
    else if (vec == 4) launch_layout<__nv_bfloat16, 4, CACHE>(p, grid, pairs, st);
    else launch_layout<__nv_bfloat16, 1, CACHE>(p, grid, pairs, st);
  } else {
    if (vec == 8) launch_layout<__half, 8, CACHE>(p, grid, pairs, st);
    else if (vec == 4) launch_layout<__half, 4, CACHE>(p, grid, pairs, st);
    else launch_layout<__half, 1, CACHE>(p, grid, pairs, st);
  }
  WAVEAL_CUDA_OK(cudaGetLastError());
  waveal::launch_counter() = 1;
  return WAVEAL_OK;
}

}  // namespace

extern "C" waveal_status waveal_rope_freqs(int32_t rot_dim, double base, waveal_rope_scaling scaling, double factor,
                                           int64_t trained_len, int64_t* freqs, float* amplitude) {
  if (!freqs) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "freqs is NULL");
  if (rot_dim < 2 || rot_dim % 2) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "rot_dim %d: even and positive", rot_dim);
  if (!(base > 1.0) || !std::isfinite(base)) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "base must be above 1");
  if (scaling < WAVEAL_ROPE_NONE || scaling > WAVEAL_ROPE_PARTS)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "scaling %d: a waveal_rope_scaling", (int)scaling);
  if (scaling != WAVEAL_ROPE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "factor must be at least 1");
  if (scaling == WAVEAL_ROPE_PARTS && trained_len <= 0)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "trained_len must be positive for WAVEAL_ROPE_PARTS");
  const double two_pi = 6.283185307179586476925;
  if (scaling == WAVEAL_ROPE_NTK && rot_dim > 2) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double theta = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == WAVEAL_ROPE_LINEAR) theta /= factor;
    if (scaling == WAVEAL_ROPE_PARTS) {
      const double turns = (double)trained_len * theta / two_pi;
      const double keep = std::fmin(1.0, std::fmax(0.0, (turns - 1.0) / 31.0));
      theta = theta * keep + theta / factor * (1.0 - keep);
    }
    freqs[i] = (int64_t)(theta / two_pi * 0x1p64);        // theta <= 1 radian: below 2^62
  }
  if (amplitude) *amplitude = scaling == WAVEAL_ROPE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return WAVEAL_OK;
}

extern "C" waveal_status waveal_rope(const waveal_rope_desc* d, const void* q, void* q_out, const void* k, void* k_out,
                                     const int32_t* positions, const int64_t* freqs, void* cuda_stream) {
  if (!d) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "desc is NULL");
  if (d->tokens < 0 || d->q_heads <= 0 || d->k_heads < 0)
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "tokens and k_heads must not be negative, q_heads positive");
  if (d->q_heads > (1 << 20) || d->k_heads > (1 << 20)) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^20 heads");
  if (d->head_dim < 2 || d->head_dim > kMaxHeadDim)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "head_dim %d (supported: 2 .. %d)", d->head_dim, kMaxHeadDim);
  if (d->dtype < WAVEAL_BF16 || d->dtype > WAVEAL_FP32) return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "dtype %d", d->dtype);
  if (waveal_status e = check_rotation(d->rot, d->head_dim)) return e;
  if (d->tokens == 0) {
    waveal::launch_counter() = 0;
    return WAVEAL_OK;
  }
  if (!q || !q_out || !positions || !freqs || (d->k_heads && (!k || !k_out)))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q, q_out, positions and freqs are required, k and k_out with k_heads");
  const size_t size = dtype_size(d->dtype);
  RotateParams p = {};
  p.tokens = d->tokens;
  p.head_dim = d->head_dim;
  set_rotation(p, d->rot);
  p.positions = positions;
  p.freqs = reinterpret_cast<const long long*>(freqs);
  const void* src[2] = {q, k};
  void* dst[2] = {q_out, k_out};
  const int64_t* in[2] = {d->q_stride, d->k_stride};
  const int64_t* out[2] = {d->q_out_stride, d->k_out_stride};
  const int heads[2] = {d->q_heads, d->k_heads};
  for (int i = 0; i < 2; ++i) {
    if (!heads[i]) continue;
    if (!waveal::aligned(src[i], size) || !waveal::aligned(dst[i], size))
      return waveal::fail(WAVEAL_ERR_INVALID_ARG, "a tensor is not aligned to its element");
    p.src[i] = src[i];
    p.dst[i] = dst[i];
    p.in[i] = {in[i][0], in[i][1]};
    p.out[i] = {out[i][0], out[i][1]};
    p.heads[i] = heads[i];
    if (src[i] == dst[i]) {
      if (in[i][0] != out[i][0] || in[i][1] != out[i][1])
        return waveal::fail(WAVEAL_ERR_INVALID_ARG, "an output over its input needs the same strides");
      p.in_place |= 1 << i;
    }
  }
  return launch<false>(p, d->dtype, d->rot.pairs, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" waveal_status waveal_cache_append(const waveal_cache_desc* cache, const waveal_batch_desc* b, const waveal_rotation* rot,
                                             const waveal_append_strides* strides, const void* k, const void* v, const void* q,
                                             void* q_out, void* k_cache, void* v_cache, const int32_t* seq_start,
                                             const int32_t* kv_len, const int32_t* page_table, const int32_t* positions,
                                             const int64_t* freqs, int32_t* dev_status, void* cuda_stream) {
  if (!cache || !b || !strides) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "cache, batch and strides are required");
  if (waveal_status e = waveal::check_cache(cache)) return e;
  if (waveal_status e = waveal::check_batch(b)) return e;
  if (cache->head_dim < 2 || cache->head_dim > kMaxHeadDim)
    return waveal::fail(WAVEAL_ERR_UNSUPPORTED, "head_dim %d (supported: 2 .. %d)", cache->head_dim, kMaxHeadDim);
  if (b->q_heads < 0 || b->q_heads > (1 << 20)) return waveal::fail(WAVEAL_ERR_INVALID_ARG, "q_heads %d", b->q_heads);
  if (rot) {
    if (waveal_status e = check_rotation(*rot, cache->head_dim)) return e;
  } else if (b->q_heads) {
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "queries are passed to be rotated, but rot is NULL");
  }
  if (b->tokens == 0 || b->batch == 0) {
    waveal::launch_counter() = 0;
    return WAVEAL_OK;
  }
  if (!k || !v || !k_cache || !v_cache || !seq_start || !kv_len || !page_table || (rot && !freqs) || (b->q_heads && (!q || !q_out)))
    return waveal::fail(WAVEAL_ERR_INVALID_ARG, "k, v, k_cache, v_cache, seq_start, kv_len and page_table are required, freqs with a "
                                                "rotation, q and q_out with q_heads");
  RotateParams p = {};
  p.tokens = b->tokens;
  p.head_dim = cache->head_dim;
  waveal_rotation none = {};
  none.axes = 1;
  set_rotation(p, rot ? *rot : none);
  p.positions = positions;
  p.freqs = reinterpret_cast<const long long*>(freqs);
  const void* src[3] = {q, k, v};
  void* dst[3] = {q_out, k_cache, v_cache};
  const int64_t* in[3] = {strides->q, strides->k, strides->v};
  for (int i = b->q_heads ? 0 : 1; i < 3; ++i) {
    if (!waveal::aligned(src[i], 2) || !waveal::aligned(dst[i], 2))
      return waveal::fail(WAVEAL_ERR_INVALID_ARG, "a tensor is not aligned to its element");
    p.src[i] = src[i];
    p.dst[i] = dst[i];
    p.in[i] = {in[i][0], in[i][1]};
    p.heads[i] = i ? cache->kv_heads : b->q_heads;
  }
  p.out[0] = {strides->q_out[0], strides->q_out[1]};
  p.out[1] = {cache->k_stride[1], cache->k_stride[2]};
  p.out[2] = {cache->v_stride[1], cache->v_stride[2]};
  p.out_page[1] = cache->k_stride[0];
  p.out_page[2] = cache->v_stride[0];
  if (b->q_heads && q == q_out) {
    if (strides->q[0] != strides->q_out[0] || strides->q[1] != strides->q_out[1])
      return waveal::fail(WAVEAL_ERR_INVALID_ARG, "an output over its input needs the same strides");
    p.in_place = 1;
  }
  p.seq_start = seq_start;
  p.kv_len = kv_len;
  p.page_table = page_table;
  p.table_stride = b->table_stride;
  p.batch = b->batch;
  p.max_pages = b->max_pages;
  p.page_shift = __builtin_ctz((unsigned)cache->page_size);
  p.n_pages = cache->n_pages;
  p.prefix_len = b->prefix_len;
  p.dev_status = dev_status;
  return launch<true>(p, cache->dtype, rot ? rot->pairs : WAVEAL_PAIRS_HALVES, static_cast<cudaStream_t>(cuda_stream));
}
