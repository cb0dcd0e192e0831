// Attention over the 4-bit cache.
//
// Scores come as S^T = K Q^T and outputs as O^T = V^T P^T on the 16x16x32 fp16 matrix instruction, so
// that the codes are the A operand of both products straight from the cache's words and the softmax
// weights go from the first product's result registers into the second's B operand without leaving
// the lane: lane (q = lane / 16, n = lane % 16) holds query row n and keys 16 h + 4 q + r, which are
// the eight keys of its value words.
//
// A code is not converted: w & 0x000f000f is a pair of fp16 subnormals c 2^-24, w & 0x00f000f0 a pair
// c 2^-20, exact operands of the matrix cores.  The queries (and the weights) of the first pairs are
// taken 16 times as large to even that out, the rest is undone in fp32: with q' = q 2^k of a row whose
// largest element lies in [2^10, 2^11), sum c q = acc 2^(20 - k), and
//     y = s (sum c q) + lo (sum q)      (times scale log2 e)
// The values' least parts need no product, and the weights' rounding to fp16 should act on codes
// measured from their middle: out = sum w (c - 8) + sum p (lo + 8 s) with w the rounded p s; the second
// sum is one number per row, and sum w 8 the product with a word of codes 8 (without it the rounding of
// weights errs on c in 0..15, and on values of mean 0 almost three times as far).
//
// Softmax with a running reference: weights are p = 2^(y - ref), and ref is raised (sums and products
// so far scaled down) only where some p s would leave fp16's range, above 2^11; it begins so low that
// a row's first visible key raises it to max(y + log2 s).  Weights times step sizes therefore stay
// within 2^11 of 1 at the top, whatever the magnitude of the values.  Sums are fp32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "owq_cache_device.h"
#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

constexpr int kWaves = 4;
constexpr float kNoRef = -1e30f;      // finite, so that differences with -infinity stay defined
constexpr float kLimit = 2048.f;      // of p s before the reference moves; 16 times that is an fp16 number

struct AttendArgs {
  CacheView c;
  const u32 *q;
  u32 *out;
  float *lse;
  float *part;           // [sequence, head, row][split][P]: sums of p s (c - 8) + p (lo + 8 s)
  float *part_sums;      // [sequence, head, row][split][2]: reference, sum of p
  int64_t q_row, q_head;
  int32_t q_heads, group, rows, row_blocks, splits, tiles_per_split, window, sinks, max_len, bf16;
  float scale;           // log2 e included
};

// Tiles that rows at positions [pa, pb] may see: the sinks' first ones, then a run.
struct Span {
  int sink_tiles, low, count;
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : low + (i - sink_tiles); }
};

__device__ __forceinline__ Span visible_tiles(const AttendArgs &a, int pa, int pb) {
  Span s;
  int end = pb + 1;                                                   // no key from here on
  end = end > a.max_len ? a.max_len : end;
  const int64_t room = (int64_t)a.c.table_stride << (a.c.page_shift + 5);
  end = end > room ? (int)room : end;
  int low = 0;
  if (a.window > 0 && pa >= a.window) low = pa - a.window + 1;
  s.low = low / 32;
  const int sink_end = (a.sinks + 31) / 32;
  s.sink_tiles = a.window > 0 && sink_end < s.low ? sink_end : s.low;
  const int last = (end + 31) / 32;
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

// The eight codes of a word as fp16 numbers: c 2^-24 at elements 0, 1, 4, 5, c 2^-20 at the others.
__device__ __forceinline__ h8_t operand(u32 w) {
  const u32x4 v = {w & 0x000f000fu, w & 0x00f000f0u, (w >> 8) & 0x000f000fu, (w >> 8) & 0x00f000f0u};
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
// with index (16 h + r) above `hi`, and those not above `lo` unless below `sink`.
template <bool EDGE, int STEPS, int NQ>
__device__ __forceinline__ h8_t weights(const f32x4 (&s)[2], const Tile<STEPS> &t, int hi, int lo, int sink, int n,
                                        Rows<STEPS, NQ> &w) {
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
    float y[8], top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32 km = t.km[i >> 2][i & 3], vm = t.vm[i >> 2][i & 3];
      y[i] = __builtin_fmaf(half_lo(km), s[i >> 2][i & 3] * w.c1[n], half_hi(km) * w.x1[n]);
      const float z = fmaxf(top, y[i] + __builtin_amdgcn_logf(half_lo(vm)));
      top = on[i] ? z : top;
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float ref = fmaxf(w.ref[n], top);
    const float alpha = __builtin_amdgcn_exp2f(w.ref[n] - ref);
    w.ref[n] = ref;
    w.l[n] *= alpha;
    w.low[n] *= alpha;
#pragma unroll
    for (int d = 0; d < 2 * STEPS; ++d) w.acc[n][d] *= alpha;
    w.mid[n] *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(y[i] - ref);
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
  const u32x4 b = {F16::pack(16.f * pv[0], 16.f * pv[1]), F16::pack(pv[2], pv[3]), F16::pack(16.f * pv[4], 16.f * pv[5]),
                   F16::pack(pv[6], pv[7])};
  return __builtin_bit_cast(h8_t, b);
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

template <int STEPS, int NQ>
__device__ __forceinline__ void products(const Tile<STEPS> &t, const h8_t (&pb)[NQ], Rows<STEPS, NQ> &w) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) w.mid[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(0x88888888u), pb[n], w.mid[n], 0, 0, 0);
#pragma unroll
  for (int st = 0; st < STEPS; ++st)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const h8_t v = operand(t.v[st][j]);
#pragma unroll
      for (int n = 0; n < NQ; ++n) w.acc[n][2 * st + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pb[n], w.acc[n][2 * st + j], 0, 0, 0);
    }
}

// Tiles from, from + STEP, ... below `to` of a span.  The next tile's words are asked for where this one's are used up (keys
// behind the first product, pairs behind the weights, values behind the second product); behind the last tile every lane
// asks for the same 16 bytes.
template <bool EDGE, int STEP, int STEPS, int NQ>
__device__ __forceinline__ void attend_tiles(const AttendArgs &a, const Span &span, int b, int head, int from, int to, int lane,
                                             Rows<STEPS, NQ> &w) {
  if (from >= to) return;
  const CacheView &c = a.c;
  const int quad = lane >> 4;
  Tile<STEPS> t;
  int i = from, tile = span.tile(i);
  const uint8_t *p = tile_in_page(c, page_of_tile(c, b, tile), head, tile);
  bool there = p != nullptr;
  p = there ? p : c.pages;             // some page, not used
  load_keys(p, lane * 8, t);
  load_pairs(p, quad * 16, t);
  load_values(p, lane * 8, t);
  int next = i + STEP < to ? span.tile(i + STEP) : tile;
  int next_page = page_of_tile(c, b, next);
  while (true) {
    i += STEP;
    const bool more = i < to;
    const uint8_t *pn = tile_in_page(c, next_page, head, next);
    const int after = i + STEP < to ? span.tile(i + STEP) : next;
    next_page = page_of_tile(c, b, after);
    const bool next_there = pn != nullptr;
    pn = next_there ? pn : c.pages;
    const u32 lane8 = more ? lane * 8 : 0, quad16 = more ? quad * 16 : 0;
    f32x4 s[NQ][2];
    scores(t, w, s);
    __builtin_amdgcn_sched_barrier(0);
    load_keys(pn, lane8, t);
    h8_t pb[NQ];
    if (there) {
      const int at = tile * 32 + 4 * quad;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int hi = (w.pos[n] < a.max_len ? w.pos[n] : a.max_len - 1) - at;
        const int lo = a.window == 0 ? -1 : w.pos[n] - a.window - at;
        pb[n] = weights<EDGE>(s[n], t, hi, lo, a.sinks - at, n, w);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load_pairs(pn, quad16, t);
    if (there) products(t, pb, w);
    __builtin_amdgcn_sched_barrier(0);
    load_values(pn, lane8, t);
    if (!more) break;
    tile = next;
    next = after;
    there = next_there;
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

// SHARE: the waves of a workgroup take other rows of the same keys.  Else: other keys of the same rows.
template <int STEPS, int NQ, bool SHARE>
__global__ __launch_bounds__(64 * kWaves, NQ >= 4 ? 1 : NQ == 2 ? 2 : 4) void owq_attend_kernel(AttendArgs a) {
  constexpr int P = 32 * STEPS;
  __shared__ float red[SHARE ? 1 : kWaves][16][P + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quad = lane >> 4, col = lane & 15;
  const int split = blockIdx.x % a.splits, block = blockIdx.x / a.splits;
  const int head = blockIdx.y, b = blockIdx.z;
  const CacheView &c = a.c;
  const int row0 = c.starts[b];
  const int n_new = c.starts[b + 1] - row0, len = c.lengths[b];
  const int n_rows = (n_new * a.group < a.rows ? n_new * a.group : a.rows);     // rows of this sequence and head
  const int first = (SHARE ? block * kWaves + wave : block) * 16 * NQ;          // first row of this wave
  if (first >= n_rows) return;                                                  // uniform over the workgroup unless SHARE, which has no barriers
  const int p0 = len - n_new;
  const int pa = p0 + first / a.group;
  const int last = (first + 16 * NQ < n_rows ? first + 16 * NQ : n_rows) - 1;
  const int pb_pos = p0 + last / a.group;
  const Span span = visible_tiles(a, pa, pb_pos);
  int i0 = split * a.tiles_per_split, i1 = i0 + a.tiles_per_split;
  i1 = i1 < span.count ? i1 : span.count;
  if (a.splits > 1 && i0 >= i1 && split > 0) return;                            // the sum over ranges does not look here

  Rows<STEPS, NQ> w;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = first + 16 * n + col;
    const int clamped = row < n_rows ? row : n_rows - 1;
    w.pos[n] = p0 + clamped / a.group;
    const int64_t at = (int64_t)row0 + clamped / a.group;
    const bool on = row < n_rows && at >= 0 && at < c.n_rows;
    const u32 *q = a.q + ((on ? at : 0) * a.q_row + (head * a.group + clamped % a.group) * a.q_head) / 2;
    float f[STEPS][8], top = 0.f, sum = 0.f;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int d = 32 * st + 8 * quad;
      u32x4 v = {0, 0, 0, 0};
      if (on && d < c.head_dim) v = *reinterpret_cast<const u32x4 *>(q + d / 2);
      if (a.bf16) unpack8<BF16>(v, f[st]);
      else unpack8<F16>(v, f[st]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, __builtin_fabsf(f[st][e]));
        sum += f[st][e];
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    sum = quads_sum(sum);
    const int k = 11 - __builtin_amdgcn_frexp_expf(top);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      h8_t h;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = (_Float16)__builtin_ldexpf(f[st][e], (e & 2) ? k : k + 4);
      w.q[n][st] = h;
    }
    w.c1[n] = __builtin_ldexpf(a.scale, 20 - k);
    w.x1[n] = a.scale * sum;
    w.ref[n] = kNoRef;
    w.l[n] = w.low[n] = 0.f;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < 2 * STEPS; ++d) w.acc[n][d] = zero;
    w.mid[n] = zero;
  }

  // Tiles that every row sees whole lie in one run of the span; the few others are masked key by key.
  constexpr int kStep = SHARE ? 1 : kWaves;
  int w0 = span.sink_tiles, w1 = span.sink_tiles;
  {
    const int low = a.window > 0 && pb_pos >= a.window ? (pb_pos - a.window + 32) / 32 : 0;       // first tile inside every row's window
    const int end = (pa + 1 < a.max_len ? pa + 1 : a.max_len) / 32;                               // first tile with a key that some row does not see
    w0 += low > span.low ? low - span.low : 0;
    w1 += end > span.low ? end - span.low : 0;
    w1 = w1 < w0 ? w0 : w1;
  }
  {
    const int from = i0 > w0 ? i0 : w0, to = i1 < w1 ? i1 : w1;
    attend_tiles<false, kStep>(a, span, b, head, from + (SHARE ? 0 : wave), to, lane, w);
    attend_tiles<true, kStep>(a, span, b, head, i0 + (SHARE ? 0 : wave), i1 < w0 ? i1 : w0, lane, w);
    attend_tiles<true, kStep>(a, span, b, head, (i0 > w1 ? i0 : w1) + (SHARE ? 0 : wave), i1, lane, w);
  }

  // results: column sums of a row lie in the lanes of its column
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float l = quads_sum(w.l[n]), low = quads_sum(w.low[n]);
    if (SHARE) {
      const int row = first + 16 * n + col;
      const int64_t at = (int64_t)row0 + row / a.group;
      if (row < n_rows && at >= 0 && at < c.n_rows) {
        const int h = head * a.group + row % a.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        u32 *out = a.out + (at * a.q_heads + h) * (c.head_dim / 2);
#pragma unroll
        for (int d = 0; d < 2 * STEPS; ++d) {
          const int dim = 16 * d + 4 * quad;
          if (dim >= c.head_dim) continue;
          float o[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) o[r] = __builtin_fmaf(w.acc[n][d][r] - w.mid[n][r], 0x1p20f, low) * inv;
          const u32x2 packed = a.bf16 ? (u32x2){BF16::pack(o[0], o[1]), BF16::pack(o[2], o[3])} : (u32x2){F16::pack(o[0], o[1]), F16::pack(o[2], o[3])};
          *reinterpret_cast<u32x2 *>(out + dim / 2) = packed;
        }
        if (a.lse != nullptr && quad == 0) a.lse[at * a.q_heads + h] = l == 0.f ? -__builtin_inff() : (w.ref[n] + __builtin_log2f(l)) * 0.69314718056f;
      }
      continue;
    }
    if (n > 0) __syncthreads();
#pragma unroll
    for (int d = 0; d < 2 * STEPS; ++d) {
      f32x4 o;
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] = __builtin_fmaf(w.acc[n][d][r] - w.mid[n][r], 0x1p20f, low);
      *reinterpret_cast<f32x4 *>(&red[wave][col][16 * d + 4 * quad]) = o;
    }
    if (quad == 0) {
      red[wave][col][P] = w.ref[n];
      red[wave][col][P + 1] = l;
    }
    __syncthreads();
    const int r = threadIdx.x >> 4, part = threadIdx.x & 15;      // row, columns part * 2 STEPS and on
    const int row = first + 16 * n + r;
    if (row >= n_rows) continue;
    float ref = red[0][r][P];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) ref = fmaxf(ref, red[v][r][P]);
    float total = 0.f, o[2 * STEPS];
#pragma unroll
    for (int e = 0; e < 2 * STEPS; ++e) o[e] = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float f = __builtin_amdgcn_exp2f(red[v][r][P] - ref);
      total = __builtin_fmaf(f, red[v][r][P + 1], total);
#pragma unroll
      for (int e = 0; e < 2 * STEPS; ++e) o[e] = __builtin_fmaf(f, red[v][r][part * 2 * STEPS + e], o[e]);
    }
    const int64_t at = (int64_t)row0 + row / a.group;
    if (at < 0 || at >= c.n_rows) continue;
    if (a.splits > 1) {
      const int64_t slot = (((int64_t)b * c.kv_heads + head) * a.rows + row) * a.splits + split;
      float *dst = a.part + slot * P + part * 2 * STEPS;
#pragma unroll
      for (int e = 0; e < 2 * STEPS; ++e) dst[e] = o[e];
      if (part == 0) {
        a.part_sums[2 * slot] = ref;
        a.part_sums[2 * slot + 1] = total;
      }
    } else {
      const int h = head * a.group + row % a.group;
      const float inv = total == 0.f ? 0.f : 1.f / total;
      u32 *out = a.out + (at * a.q_heads + h) * (c.head_dim / 2);
#pragma unroll
      for (int e = 0; e < 2 * STEPS; e += 2) {
        const int dim = part * 2 * STEPS + e;
        if (dim < c.head_dim) out[dim / 2] = a.bf16 ? BF16::pack(o[e] * inv, o[e + 1] * inv) : F16::pack(o[e] * inv, o[e + 1] * inv);
      }
      if (a.lse != nullptr && part == 0) a.lse[at * a.q_heads + h] = total == 0.f ? -__builtin_inff() : (ref + __builtin_log2f(total)) * 0.69314718056f;
    }
  }
}

// The ranges of a row joined: one wave per row, two columns per lane, 16 ranges in flight.
__global__ __launch_bounds__(256) void owq_attend_join_kernel(AttendArgs a, int block_rows, int P) {
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, b = blockIdx.z;
  const int row0 = c.starts[b];
  const int n_new = c.starts[b + 1] - row0, len = c.lengths[b];
  const int n_rows = (n_new * a.group < a.rows ? n_new * a.group : a.rows);
  if (row >= n_rows) return;
  const int64_t at = (int64_t)row0 + row / a.group;
  if (at < 0 || at >= c.n_rows) return;
  const int first = row / block_rows * block_rows;
  const int last = (first + block_rows < n_rows ? first + block_rows : n_rows) - 1;
  const Span span = visible_tiles(a, len - n_new + first / a.group, len - n_new + last / a.group);
  int used = (span.count + a.tiles_per_split - 1) / a.tiles_per_split;
  used = used < 1 ? 1 : used;
  const int64_t slot = (((int64_t)b * c.kv_heads + head) * a.rows + row) * a.splits;
  const float *sums = a.part_sums + 2 * slot, *src = a.part + slot * P;
  float ref = kNoRef;
  for (int s = lane; s < used; s += 64) ref = fmaxf(ref, sums[2 * s]);
  ref = wave_max(ref);
  float total = 0.f, o0 = 0.f, o1 = 0.f;
  const int col = 2 * lane < P ? 2 * lane : 0;
  for (int base = 0; base < used; base += 64) {
    const int mine = base + lane;
    const float f = mine < used ? __builtin_amdgcn_exp2f(sums[2 * mine] - ref) : 0.f;
    total = __builtin_fmaf(f, mine < used ? sums[2 * mine + 1] : 0.f, total);
    const int n = used - base < 64 ? used - base : 64;
    for (int s = 0; s < n; s += 16) {
      float2 v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at_s = base + (s + i < n ? s + i : n - 1);
        v[i] = *reinterpret_cast<const float2 *>(src + (int64_t)at_s * P + col);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        // lanes past the last range have f = 0
        const float g = s + i < n ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (s + i) & 63)) : 0.f;
        o0 = s + i < n ? __builtin_fmaf(g, v[i].x, o0) : o0;
        o1 = s + i < n ? __builtin_fmaf(g, v[i].y, o1) : o1;
      }
    }
  }
  total = wave_sum(total);
  const int h = head * a.group + row % a.group;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  if (2 * lane < c.head_dim) a.out[(at * a.q_heads + h) * (c.head_dim / 2) + lane] = a.bf16 ? BF16::pack(o0 * inv, o1 * inv) : F16::pack(o0 * inv, o1 * inv);
  if (a.lse != nullptr && lane == 0) a.lse[at * a.q_heads + h] = total == 0.f ? -__builtin_inff() : (ref + __builtin_log2f(total)) * 0.69314718056f;
}

AttendPlan attend_plan(const owq_cache_desc_t &d, const owq_attention_desc_t &a) {
  AttendPlan p;
  p.group = a.q_heads / d.kv_heads;
  p.rows = (int)std::min<int64_t>((int64_t)a.max_new * p.group, 0x7fffffff);
  p.share_keys = p.rows > 64;
  p.col_tiles = p.rows <= 16 ? 1 : p.rows <= 32 || p.share_keys ? 2 : 4;
  const int block = 16 * p.col_tiles * (p.share_keys ? kWaves : 1);
  p.row_blocks = (p.rows + block - 1) / block;
  int64_t seen = std::min<int64_t>(a.max_len, (int64_t)d.table_stride * d.page_size);
  if (a.window > 0) seen = std::min<int64_t>(seen, (int64_t)a.window + a.max_new + a.sinks + 96);
  const int tiles = (int)((seen + 31) / 32);
  p.splits = 1;
  p.tiles_per_split = tiles > 0 ? tiles : 1;
  if (!p.share_keys) {
    // enough workgroups for every compute unit, two tiles per wave at least
    const int64_t base = (int64_t)d.n_seqs * d.kv_heads * p.row_blocks;
#ifndef WGS
#define WGS 2048
#define TPW 2
#endif
    const int64_t want = std::max<int64_t>(1, WGS / std::max<int64_t>(1, base));
    const int most = std::max(1, tiles / (TPW * kWaves));
    const int splits = (int)std::min<int64_t>(want, most);
    p.tiles_per_split = std::max(1, (tiles + splits - 1) / splits);
    p.splits = std::max(1, (tiles + p.tiles_per_split - 1) / p.tiles_per_split);
  }
  const int P = (d.head_dim + 31) / 32 * 32;
  p.slots = (size_t)d.n_seqs * d.kv_heads * p.rows * p.splits;
  p.workspace = p.splits > 1 ? p.slots * (P + 2) * 4 : 0;
  return p;
}

template <int STEPS>
static void launch_steps(const AttendArgs &a, const AttendPlan &p, dim3 grid, hipStream_t s) {
  if (p.share_keys) owq_attend_kernel<STEPS, 2, true><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (p.col_tiles == 1) owq_attend_kernel<STEPS, 1, false><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (p.col_tiles == 2) owq_attend_kernel<STEPS, 2, false><<<grid, 64 * kWaves, 0, s>>>(a);
  else owq_attend_kernel<STEPS, 4, false><<<grid, 64 * kWaves, 0, s>>>(a);
}

int launch_attend(const CacheView &c, const owq_attention_desc_t &d, const AttendPlan &p, const void *q, void *out, float *lse,
                  void *workspace, void *stream) {
  AttendArgs a;
  a.c = c;
  a.q = static_cast<const u32 *>(q);
  a.out = static_cast<u32 *>(out);
  a.lse = lse;
  a.part = static_cast<float *>(workspace);
  a.part_sums = a.part + p.slots * ((c.head_dim + 31) / 32 * 32);
  a.q_row = d.q_row, a.q_head = d.q_head;
  a.q_heads = d.q_heads, a.group = p.group, a.rows = p.rows, a.row_blocks = p.row_blocks, a.splits = p.splits;
  a.tiles_per_split = p.tiles_per_split, a.window = d.window, a.sinks = d.sinks, a.max_len = d.max_len;
  a.bf16 = d.type == OWQ_TYPE_BF16;
  a.scale = d.scale * 1.44269504089f;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)(p.row_blocks * p.splits), (unsigned)c.kv_heads, (unsigned)c.n_seqs);
  const int steps = (c.head_dim + 31) / 32;
  switch (steps) {
    case 1: launch_steps<1>(a, p, grid, s); break;
    case 2: launch_steps<2>(a, p, grid, s); break;
    case 3: launch_steps<3>(a, p, grid, s); break;
    default: launch_steps<4>(a, p, grid, s); break;
  }
  if (p.splits > 1)
    owq_attend_join_kernel<<<dim3((unsigned)((p.rows + 3) / 4), (unsigned)c.kv_heads, (unsigned)c.n_seqs), 256, 0, s>>>(a, 16 * p.col_tiles, 32 * steps);
  return (int)hipGetLastError();
}

}  // namespace owq
