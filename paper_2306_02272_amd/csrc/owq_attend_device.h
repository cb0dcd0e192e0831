// Attention over the 4-bit cache: what its kernels share.
//
// Scores come as S^T = K Q^T and outputs as O^T = V^T P^T on the 16x16x32 fp16 matrix instruction, so
// that the codes are the A operand of both products straight from the cache's words and the softmax
// weights go from the first product's result registers into the second's B operand without leaving
// the lane: lane (q = lane / 16, n = lane % 16) holds query row n and keys 16 h + 4 q + r, which are
// the eight keys of its value words.
//
// A code is not converted: (w >> 4 j) & 0x00f000f0 is a pair of fp16 subnormals c 2^-20, exact operands of the
// matrix cores.  Sums come out as if products were aligned by the operands' exponents, a subnormal's being the
// smallest normal number's, and cut below 2^-24 of the largest: six bits are lost there, ten with codes c 2^-24,
// which w & 0x000f000f would give one shift cheaper.  (Pairs of both scales, 243 us instead of 257 for a prompt
// of 2048 tokens behind 4100: the log-sum 1e-5 off instead of 6e-7, and results of single tokens behind 18 000
// others 2.7e-4 instead of 2.2e-4, growing with the length.)
// With q' = q 2^k of a row whose largest element lies in [2^10, 2^11), sum c q = acc 2^(20 - k), and
//     y = s (sum c q) + lo (sum q)      (times scale log2 e)
// The values' least parts need no product, and the weights' rounding to fp16 should act on codes
// measured from their middle: out = sum w (c - 8) + sum p (lo + 8 s) with w the rounded p s; the second
// sum is one number per row, and sum w 8 the product with a word of codes 8.  (With the rounding acting on
// c in 0..15, values of mean 0 come out almost three times as far off; with the sum of w taken by the
// packed dot product instead, 15 000 tokens came out at 3.4e-4 of 64 bits' result instead of 2.7e-4.)
// Where the keys are read for few rows and the result is fp16, what the rounding of w takes away is multiplied as
// well (SPLIT): 2.1e-4 of the result instead of 2.9e-4, 2.07e-4 being the result's own rounding; 64 sequences of
// 300 to 8192 tokens take 2% longer so.  Prompts stay with w, where that would be 27% of the time.
//
// Softmax with a running reference: weights are p = 2^(y - ref), and ref is raised (sums and products
// so far scaled down) only where some p s would leave fp16's range, above 2^11: to 2^4 of the largest.  It
// begins so low that a row's first visible key raises it.  Weights times step sizes therefore stay between
// 2^4 and 2^11 at the top, whatever the magnitude of the values.  Sums are fp32.
#pragma once
#include <hip/hip_runtime.h>

#include "owq_cache_device.h"
#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

constexpr int kWaves = 4;
constexpr float kNoRef = -3.402823466e38f;   // below every score, finite, so that differences with -infinity stay defined
constexpr float kRoom = 4.f;          // log2 of the largest p s where the reference has just been raised
constexpr float kLimit = 2048.f;      // of p s before the reference moves, far inside fp16's range

struct AttendArgs {
  CacheView c;
  const u32 *q;
  u32 *out;
  float *lse;
  float *part;           // partial results [slot][row][P]: sums of p s (c - 8) + p (lo + 8 s)
  float *part_sums;      // [slot][row][2]: reference, sum of p
  int64_t q_row, q_head;
  int32_t q_heads, group, max_new, window, sinks, max_len, bf16;
  int32_t *places;       // few rows: [sequence][2], its first workgroup and its ranges per head
  int32_t slot_rows, blocks, least_tiles, ranges, whole;
  float scale;           // log2 e included
};

// Tiles that rows at positions [pa, pb] may see: the sinks' first ones, then a run.
struct Span {
  int sink_tiles, low, count;
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : low + (i - sink_tiles); }
};

// Tiles that hold the tokens below `end`; end + 31 may be past the largest int.
__device__ __forceinline__ int tiles_up_to(int end) { return end > 0 ? (end - 1) / 32 + 1 : 0; }

__device__ __forceinline__ Span visible_tiles(const AttendArgs &a, int pa, int pb) {
  Span s;
  int end = pb + 1;                                                   // no key from here on
  end = end > a.max_len ? a.max_len : end;
  const int64_t room = (int64_t)a.c.table_stride << (a.c.page_shift + 5);
  end = end > room ? (int)room : end;
  int low = 0;
  if (a.window > 0 && pa >= a.window) low = pa - a.window + 1;
  s.low = low / 32;
  const int sink_end = tiles_up_to(a.sinks);
  s.sink_tiles = a.window > 0 && sink_end < s.low ? sink_end : s.low;
  const int last = tiles_up_to(end);
  if (end <= 0) {
    s.sink_tiles = 0;
    s.count = 0;
  } else if (a.window > 0) {
    s.sink_tiles = s.sink_tiles < last ? s.sink_tiles : last;
    s.count = s.sink_tiles + (last > s.low ? last - s.low : 0);
  } else {
    s.sink_tiles = 0;
    s.count = last;
  }
  return s;
}

// A tile's words and pairs as one lane holds them: keys 16 h + 4 quad + r in km[h][r], vm[h][r].
template <int STEPS>
struct Tile {
  u32x2 k[STEPS], v[STEPS];
  u32x4 km[2], vm[2];
};

template <int STEPS>
__device__ __forceinline__ void load_keys(const uint8_t *p, u32 lane8, Tile<STEPS> &t) {
#pragma unroll
  for (int s = 0; s < STEPS; ++s) t.k[s] = *reinterpret_cast<const u32x2 *>(p + lane8 + 512 * s);
}

template <int STEPS>
__device__ __forceinline__ void load_values(const uint8_t *p, u32 lane8, Tile<STEPS> &t) {
#pragma unroll
  for (int s = 0; s < STEPS; ++s) t.v[s] = *reinterpret_cast<const u32x2 *>(p + lane8 + 512 * (STEPS + s));
}

template <int STEPS>
__device__ __forceinline__ void load_pairs(const uint8_t *p, u32 quad16, Tile<STEPS> &t) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    t.km[h] = *reinterpret_cast<const u32x4 *>(p + quad16 + 1024 * STEPS + 64 * h);
    t.vm[h] = *reinterpret_cast<const u32x4 *>(p + quad16 + 1024 * STEPS + 128 + 64 * h);
  }
}

// The eight codes of a word as fp16 numbers c 2^-20.
__device__ __forceinline__ h8_t operand(u32 w) {
  const u32x4 v = {(w << 4) & 0x00f000f0u, w & 0x00f000f0u, (w >> 4) & 0x00f000f0u, (w >> 8) & 0x00f000f0u};
  return __builtin_bit_cast(h8_t, v);
}

template <int STEPS, int NQ>
struct Rows {
  h8_t q[NQ][STEPS];
  float c1[NQ], x1[NQ];           // factors of s acc and of lo
  float ref[NQ], l[NQ], low[NQ];  // reference, sum of p, sum of p (lo + 8 s), of this lane's keys
  int pos[NQ];
  f32x4 acc[NQ][2 * STEPS], mid[NQ];   // sums of w c 2^-20, and of w 8 2^-20 in every register
};

// Scores to weights for one column tile: s = the products of this lane's eight keys, EDGE: some of them are masked, those
// with index (16 h + r) above `hi`, and those not above `lo` unless below `sink`.  SPLIT: *rest = what their rounding takes away.
template <bool EDGE, bool SPLIT, int STEPS, int NQ>
__device__ __forceinline__ h8_t weights(const f32x4 (&s)[2], const Tile<STEPS> &t, int hi, int lo, int sink, int n,
                                        Rows<STEPS, NQ> &w, h8_t *rest) {
  float p[8], pv[8], most = 0.f;
  bool on[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = 16 * (i >> 2) + (i & 3);
    on[i] = !EDGE || (at <= hi && (at > lo || at < sink));
    const u32 km = t.km[i >> 2][i & 3], vm = t.vm[i >> 2][i & 3];
    const float y = __builtin_fmaf(half_lo(km), s[i >> 2][i & 3] * w.c1[n], __builtin_fmaf(half_hi(km), w.x1[n], -w.ref[n]));
    p[i] = __builtin_amdgcn_exp2f(y);
    pv[i] = p[i] * half_lo(vm);
    if (EDGE) {
      p[i] = on[i] ? p[i] : 0.f;
      pv[i] = on[i] ? pv[i] : 0.f;
    }
    most = fmaxf(most, pv[i]);
  }
  if (__any(most > kLimit)) {
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32 km = t.km[i >> 2][i & 3], vm = t.vm[i >> 2][i & 3];
      const float y = __builtin_fmaf(half_lo(km), s[i >> 2][i & 3] * w.c1[n], half_hi(km) * w.x1[n]);
      const float z = fmaxf(top, y + __builtin_amdgcn_logf(half_lo(vm)));
      top = on[i] ? z : top;
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // rows that need it only: what other rows of the wave hold must not show in a row's rounding
    const float ref = most > kLimit ? fmaxf(w.ref[n], top - kRoom) : w.ref[n];
    const float alpha = __builtin_amdgcn_exp2f(w.ref[n] - ref);
    w.ref[n] = ref;
    w.l[n] *= alpha;
    w.low[n] *= alpha;
#pragma unroll
    for (int d = 0; d < 2 * STEPS; ++d) w.acc[n][d] *= alpha;
    w.mid[n] *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32 km = t.km[i >> 2][i & 3];          // as above, bit for bit
      const float y = __builtin_fmaf(half_lo(km), s[i >> 2][i & 3] * w.c1[n], __builtin_fmaf(half_hi(km), w.x1[n], -ref));
      p[i] = __builtin_amdgcn_exp2f(y);
      pv[i] = p[i] * half_lo(t.vm[i >> 2][i & 3]);
      if (EDGE) {
        p[i] = on[i] ? p[i] : 0.f;
        pv[i] = on[i] ? pv[i] : 0.f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w.l[n] += p[i];
    const u32 vm = t.vm[i >> 2][i & 3];
    const float lo8 = __builtin_fmaf(8.f, half_lo(vm), half_hi(vm));
    w.low[n] = __builtin_fmaf(p[i], EDGE ? (on[i] ? lo8 : 0.f) : lo8, w.low[n]);
  }
  const u32x4 b = {F16::pack(pv[0], pv[1]), F16::pack(pv[2], pv[3]), F16::pack(pv[4], pv[5]), F16::pack(pv[6], pv[7])};
  const h8_t rounded = __builtin_bit_cast(h8_t, b);
  if (SPLIT) {
#pragma unroll
    for (int i = 0; i < 8; ++i) pv[i] -= (float)rounded[i];
    const u32x4 r = {F16::pack(pv[0], pv[1]), F16::pack(pv[2], pv[3]), F16::pack(pv[4], pv[5]), F16::pack(pv[6], pv[7])};
    *rest = __builtin_bit_cast(h8_t, r);
  }
  return rounded;
}

template <int STEPS, int NQ>
__device__ __forceinline__ void scores(const Tile<STEPS> &t, const Rows<STEPS, NQ> &w, f32x4 (&s)[NQ][2]) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) s[n][0] = s[n][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < STEPS; ++st)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const h8_t k = operand(t.k[st][h]);
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, w.q[n][st], s[n][h], 0, 0, 0);
    }
}

template <bool SPLIT, int STEPS, int NQ>
__device__ __forceinline__ void products(const Tile<STEPS> &t, const h8_t (&pb)[NQ], const h8_t (&rest)[NQ], Rows<STEPS, NQ> &w) {
  auto add = [&](f32x4 &acc, h8_t v, int n) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pb[n], acc, 0, 0, 0);
    if (SPLIT) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, rest[n], acc, 0, 0, 0);
  };
#pragma unroll
  for (int n = 0; n < NQ; ++n) add(w.mid[n], operand(0x88888888u), n);
#pragma unroll
  for (int st = 0; st < STEPS; ++st)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const h8_t v = operand(t.v[st][j]);
#pragma unroll
      for (int n = 0; n < NQ; ++n) add(w.acc[n][2 * st + j], v, n);
    }
}

// A tile of the wave's walk: its address, and whether it lies on a page.
struct Place {
  const uint8_t *p;
  int tile;
  bool there;
};
__device__ __forceinline__ Place place_of(const CacheView &c, int page, int head, int tile) {
  Place x;
  const uint8_t *p = tile_in_page(c, page, head, tile);
  x.there = p != nullptr;
  x.p = x.there ? p : c.pages;             // some page, not used
  x.tile = tile;
  return x;
}
template <int STEPS>
__device__ __forceinline__ void load_tile(const Place &x, int lane, Tile<STEPS> &t) {
  load_keys(x.p, lane * 8, t);
  load_pairs(x.p, (lane >> 4) * 16, t);
  load_values(x.p, lane * 8, t);
}

// Tiles from, from + STEP, ... below `to` of a span, the first of them loaded.  The next tile's words are asked for where this
// one's are used up (keys behind the first product, pairs behind the weights, values behind the second product); behind the
// last tile every lane asks for the same 16 bytes.
template <bool EDGE, bool SPLIT, int STEP, int STEPS, int NQ>
__device__ __forceinline__ void attend_tiles(const AttendArgs &a, const Span &span, int b, int head, int from, int to, int lane, Place now,
                                             Tile<STEPS> &t, Rows<STEPS, NQ> &w) {
  const CacheView &c = a.c;
  const int quad = lane >> 4;
  int i = from, next = i + STEP < to ? span.tile(i + STEP) : now.tile;
  int next_page = page_of_tile(c, b, next);
  while (true) {
    i += STEP;
    const bool more = i < to;
    const Place then = place_of(c, next_page, head, next);
    next = i + STEP < to ? span.tile(i + STEP) : next;
    next_page = page_of_tile(c, b, next);
    const u32 lane8 = more ? lane * 8 : 0, quad16 = more ? quad * 16 : 0;
    f32x4 s[NQ][2];
    scores(t, w, s);
    __builtin_amdgcn_sched_barrier(0);
    load_keys(then.p, lane8, t);
    h8_t pb[NQ], rest[NQ];
    if (now.there) {
      const int at = now.tile * 32 + 4 * quad;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int hi = (w.pos[n] < a.max_len ? w.pos[n] : a.max_len - 1) - at;
        const int lo = a.window == 0 ? -1 : w.pos[n] - a.window - at;
        pb[n] = weights<EDGE, SPLIT>(s[n], t, hi, lo, a.sinks - at, n, w, &rest[n]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load_pairs(then.p, quad16, t);
    if (now.there) products<SPLIT>(t, pb, rest, w);
    __builtin_amdgcn_sched_barrier(0);
    load_values(then.p, lane8, t);
    if (!more) break;
    now = then;
  }
}

// Over the wave, in every lane, in a fixed order.
__device__ __forceinline__ float wave_sum(float v) {
  v = lanes_sum<16>(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float wave_max(float v) {
  v = lanes_max<16>(v);
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quads_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A sequence as an attention call sees it.
struct Sequence {
  int row0, n_rows, p0;      // first row of q, rows x query heads per key/value head, position of the first row
};
__device__ __forceinline__ Sequence sequence_of(const AttendArgs &a, int b) {
  Sequence s;
  s.row0 = a.c.starts[b];
  const int n = a.c.starts[b + 1] - s.row0;
  s.p0 = a.c.lengths[b] - n;
  s.n_rows = n <= 0 ? 0 : (n < a.max_new ? n : a.max_new) * a.group;
  return s;
}

// Query rows first .. first + 16 NQ - 1 of a sequence and head into a wave's registers; sums at zero.
template <int STEPS, int NQ>
__device__ __forceinline__ void load_rows(const AttendArgs &a, const Sequence &sq, int head, int first, int lane, Rows<STEPS, NQ> &w) {
  const CacheView &c = a.c;
  const int quad = lane >> 4, col = lane & 15;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = first + 16 * n + col;
    const int clamped = row < sq.n_rows ? row : sq.n_rows - 1;
    const int token = clamped / a.group;
    w.pos[n] = sq.p0 + token;
    const int64_t at = (int64_t)sq.row0 + token;
    const bool on = row < sq.n_rows && at >= 0 && at < c.n_rows;
    const u32 *q = a.q + ((on ? at : 0) * a.q_row + (head * a.group + clamped - token * a.group) * a.q_head) / 2;
    u32x4 raw[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int d = 32 * st + 8 * quad;
      raw[st] = *reinterpret_cast<const u32x4 *>(q + (d < c.head_dim ? d / 2 : 0));
    }
    float top = 0.f, sum = 0.f;
    u32 keep[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      keep[st] = on && 32 * st + 8 * quad < c.head_dim ? 0xffffffffu : 0u;
      raw[st] &= (u32x4){keep[st], keep[st], keep[st], keep[st]};
      float f[8];
      if (a.bf16) unpack8<BF16>(raw[st], f);
      else unpack8<F16>(raw[st], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, __builtin_fabsf(f[e]));
        sum += f[e];
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    sum = quads_sum(sum);
    const int k = 11 - __builtin_amdgcn_frexp_expf(top);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      float f[8];
      if (a.bf16) unpack8<BF16>(raw[st], f);
      else unpack8<F16>(raw[st], f);
      h8_t h;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = (_Float16)__builtin_ldexpf(f[e], k);
      w.q[n][st] = h;
    }
    w.c1[n] = __builtin_ldexpf(a.scale, 20 - k);
    // an infinity makes every score NaN here: by itself it could make them all -infinity, which is a row that sees nothing
    w.x1[n] = top < __builtin_inff() ? a.scale * sum : __builtin_nanf("");
    w.ref[n] = kNoRef;
    w.l[n] = w.low[n] = 0.f;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < 2 * STEPS; ++d) w.acc[n][d] = zero;
    w.mid[n] = zero;
  }
}

// The run [w0, w1) of a span's indices whose tiles every row at positions [pa, pb] sees whole.
__device__ __forceinline__ void whole_tiles(const AttendArgs &a, const Span &span, int pa, int pb, int *w0, int *w1) {
  const int low = a.window > 0 && pb >= a.window ? (pb - a.window + 32) / 32 : 0;     // first tile inside every row's window
  const int seen = pa + 1 < a.max_len ? pa + 1 : a.max_len;
  const int end = seen > 0 ? seen / 32 : 0;                                           // first tile with a key that some row does not see
  *w0 = span.sink_tiles + (low > span.low ? low - span.low : 0);
  *w1 = span.sink_tiles + (end > span.low ? end - span.low : 0);
  *w1 = *w1 < *w0 ? *w0 : *w1;
}

// Indices i0 .. i1 of a span, every STEP-th from `offset` on: whole tiles, then the few that are masked key by key.  The first
// tile is asked for before the rows.
template <bool SPLIT, int STEP, int STEPS, int NQ>
__device__ __forceinline__ void attend_span(const AttendArgs &a, const Sequence &sq, const Span &span, int b, int head, int first, int pa, int pb,
                                            int i0, int i1, int offset, int lane, Rows<STEPS, NQ> &w) {
  int w0, w1;
  whole_tiles(a, span, pa, pb, &w0, &w1);
  const int from0 = (i0 > w0 ? i0 : w0) + offset, to0 = i1 < w1 ? i1 : w1;
  const int from1 = i0 + offset, to1 = i1 < w0 ? i1 : w0;
  const int from2 = (i0 > w1 ? i0 : w1) + offset, to2 = i1;
  const int begin = from0 < to0 ? from0 : from1 < to1 ? from1 : from2;
  Tile<STEPS> t;
  Place now = {a.c.pages, 0, false};
  if (begin < i1) {
    const int tile = span.tile(begin);
    now = place_of(a.c, page_of_tile(a.c, b, tile), head, tile);
    load_tile(now, lane, t);
  }
  load_rows(a, sq, head, first, lane, w);
  if (from0 < to0) attend_tiles<false, SPLIT, STEP>(a, span, b, head, from0, to0, lane, now, t, w);
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const int from = part ? from2 : from1, to = part ? to2 : to1;
    if (from >= to) continue;
    if (from != begin) {
      const int tile = span.tile(from);
      now = place_of(a.c, page_of_tile(a.c, b, tile), head, tile);
      load_tile(now, lane, t);
    }
    attend_tiles<true, SPLIT, STEP>(a, span, b, head, from, to, lane, now, t, w);
  }
}

__device__ __forceinline__ float lse_of(float ref, float total) {
  return total == 0.f ? -__builtin_inff() : (ref + __builtin_log2f(total)) * 0.69314718056f;
}

// Many rows per sequence and head (owq_attend_many.hip).
template <int STEPS>
void launch_attend_many(const AttendArgs &a, hipStream_t stream);

}  // namespace owq
