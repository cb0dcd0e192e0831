// Attention over the 4-bit cache, few rows: single tokens, drafts, short pieces.  The keys are what there is to read.  Every
// (sequence, head, block of 16 or 32 rows) has its tiles cut into ranges of equal length, one
// workgroup each; how long a range is at most goes by the sum of all sequences' tiles, so that the workgroups are as many
// as the compute units hold at once, whatever the lengths.  A workgroup finds its range by sums over the sequences.  Its
// waves take tiles in turn and are joined in LDS; ranges are joined by a second launch.  17 to 128 rows leave the most to join:
// 100 tokens of 3000, 32/8 heads, take 38 us, 30 in 520 workgroups that walk five tiles a wave, 6 to join 10 MB of partial
// results, where the operations take 4.2 and the bytes 1.0.
//
// Bound by memory where there is enough of it: one token each of 64 sequences of 300 to 8192, 32/8 heads of 128, in 76.6 us, 298 MB
// at 3.9 TB/s.  One token of 40/40 heads behind 4000 takes 17.3 us, 4 of them in the second launch: latency of what a
// workgroup reads one after the other (lengths, table, tiles).  Ranges by one length for all sequences: with the same
// number of ranges for each, 64 sequences of uneven lengths took 118 us where this took 74.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "owq_attend_device.h"

namespace owq {

constexpr int kResident = 3;      // workgroups of one column tile that a compute unit holds

// Tiles of each of a sequence's heads, at least one where there are rows, so that rows that see nothing are written.
__device__ __forceinline__ int tiles_of(const AttendArgs &a, const Sequence &sq) {
  if (sq.n_rows == 0) return 0;
  const int n = visible_tiles(a, sq.p0, sq.p0 + (sq.n_rows - 1) / a.group).count;
  return n < 1 ? 1 : n;
}
__device__ __forceinline__ int tiles_of(const AttendArgs &a, int b) { return b < a.c.n_seqs ? tiles_of(a, sequence_of(a, b)) : 0; }

__device__ __forceinline__ u64 add64(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ u64 last_lane(u64 v) {
  return (u64)(u32)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (u32)__builtin_amdgcn_readlane((int)v, 63);
}

// f(sequence's tiles) summed over all sequences, by every wave for itself: no barriers.  `mine` = the tiles of sequence `lane`.
template <class F>
__device__ __forceinline__ u64 sum_over(const AttendArgs &a, int mine, int lane, F &&f) {
  u64 v = f(mine);
  for (int b = lane + 64; b < a.c.n_seqs; b += 64) v += f(tiles_of(a, b));
  return last_lane(wave_scan(v, (u64)0, add64));
}

// Most tiles of a range: a.ranges of them over all heads, or as many more as it takes that every head has one.  Two
// corrections bring their number to a.ranges or below where that can be.
__device__ __forceinline__ int range_length(const AttendArgs &a, int mine, int lane) {
  const u64 want = (u64)a.ranges, heads = (u64)a.c.kv_heads * a.blocks;
  const u64 total = sum_over(a, mine, lane, [](int n) { return (u64)n; }) * heads;
  u64 length = (total + want - 1) / want;
  length = length > (u64)a.least_tiles ? length : (u64)a.least_tiles;
  if ((u64)a.c.n_seqs * heads * 2 <= want && a.c.n_seqs > 1)
    for (int k = 0; k < 2; ++k) {
      const int l = (int)length;
      const u64 n = sum_over(a, mine, lane, [&](int t) { return (u64)((t + l - 1) / l); }) * heads;
      if (n <= want) break;
      length = (length * n + want - 1) / want;
    }
  return length < 0x7fffffffull ? (int)length : 0x7fffffff;
}

// A finished row's eight, six, ... columns and its log-sum.
template <int STEPS>
__device__ __forceinline__ void store_row(const AttendArgs &a, const Sequence &sq, int head, int row, int part, const float *o, float ref, float total) {
  const int token = row / a.group;
  const int64_t at = (int64_t)sq.row0 + token;
  if (at < 0 || at >= a.c.n_rows) return;
  const int h = head * a.group + row - token * a.group;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  u32 *out = a.out + (at * a.q_heads + h) * (a.c.head_dim / 2);
#pragma unroll
  for (int e = 0; e < 2 * STEPS; e += 2) {
    const int dim = part * 2 * STEPS + e;
    if (dim < a.c.head_dim) out[dim / 2] = a.bf16 ? BF16::pack(o[e] * inv, o[e + 1] * inv) : F16::pack(o[e] * inv, o[e + 1] * inv);
  }
  if (a.lse != nullptr && part == 0) a.lse[at * a.q_heads + h] = lse_of(ref, total);
}

template <int STEPS, int NQ, bool SPLIT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, NQ == 2 || WAVES == 8 ? 2 : kResident) void owq_attend_few_kernel(AttendArgs a) {
  constexpr int P = 32 * STEPS;
  __shared__ float red[WAVES][16][P + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quad = lane >> 4, col = lane & 15;

  // this workgroup's sequence, head and range: every wave finds them for itself
  Sequence sq = {0, 0, 0};
  int b = -1, place = 0, ranges = 0;
  {
    Sequence mine = {0, 0, 0};
    if (lane < a.c.n_seqs) mine = sequence_of(a, lane);
    int tiles = tiles_of(a, mine);
    const int length = a.whole ? 0x7fffffff : range_length(a, tiles, lane);
    u64 before = 0;
    for (int base = 0; base < a.c.n_seqs; base += 64) {
      if (base > 0) {
        mine = base + lane < a.c.n_seqs ? sequence_of(a, base + lane) : Sequence{0, 0, 0};
        tiles = tiles_of(a, mine);
      }
      const int own = tiles > 0 ? (tiles - 1) / length + 1 : 0;
      const u64 cost = (u64)own * a.c.kv_heads * a.blocks;
      const u64 scan = wave_scan(cost, (u64)0, add64), from = before + scan - cost;
      const u64 here = __ballot(from <= blockIdx.x && blockIdx.x < from + cost);
      if (here != 0) {
        const int l = __ffsll(here) - 1;
        b = base + l;
        place = __builtin_amdgcn_readlane((int)(blockIdx.x - from), l);
        ranges = __builtin_amdgcn_readlane(own, l);
        sq.row0 = __builtin_amdgcn_readlane(mine.row0, l);
        sq.n_rows = __builtin_amdgcn_readlane(mine.n_rows, l);
        sq.p0 = __builtin_amdgcn_readlane(mine.p0, l);
        break;
      }
      before += last_lane(scan);
    }
  }
  if (b < 0) return;
  if (!a.whole && place == 0 && threadIdx.x == 0) {       // for the second launch
    a.places[2 * b] = (int)blockIdx.x;
    a.places[2 * b + 1] = ranges;
  }
  const int item = place / ranges, range = place - item * ranges;
  const int head = item / a.blocks, first = (item - head * a.blocks) * 16 * NQ;
  if (first >= sq.n_rows) return;
  const int last = (first + 16 * NQ < sq.n_rows ? first + 16 * NQ : sq.n_rows) - 1;
  const int pa = sq.p0 + first / a.group, pb = sq.p0 + last / a.group;
  const Span span = visible_tiles(a, pa, pb);
  const int i0 = (int)((int64_t)span.count * range / ranges), i1 = (int)((int64_t)span.count * (range + 1) / ranges);
  Rows<STEPS, NQ> w;
  attend_span<SPLIT, WAVES>(a, sq, span, b, head, first, pa, pb, i0, i1, wave, lane, w);

  // the waves joined: column sums of a row lie in the lanes of its column
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float l = quads_sum(w.l[n]), low = quads_sum(w.low[n]);
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
    if (r < 16 && row < sq.n_rows) {
      float ref = red[0][r][P];
#pragma unroll
      for (int v = 1; v < WAVES; ++v) ref = fmaxf(ref, red[v][r][P]);
      float total = 0.f, o[2 * STEPS];
#pragma unroll
      for (int e = 0; e < 2 * STEPS; ++e) o[e] = 0.f;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        const float f = __builtin_amdgcn_exp2f(red[v][r][P] - ref);
        total = __builtin_fmaf(f, red[v][r][P + 1], total);
#pragma unroll
        for (int e = 0; e < 2 * STEPS; ++e) o[e] = __builtin_fmaf(f, red[v][r][part * 2 * STEPS + e], o[e]);
      }
      if (ranges == 1) {
        store_row<STEPS>(a, sq, head, row, part, o, ref, total);
      } else {
        const int64_t slot = (int64_t)blockIdx.x * a.slot_rows + 16 * n + r;
        float *dst = a.part + slot * P + part * 2 * STEPS;
#pragma unroll
        for (int e = 0; e < 2 * STEPS; ++e) dst[e] = o[e];
        if (part == 0) {
          a.part_sums[2 * slot] = ref;
          a.part_sums[2 * slot + 1] = total;
        }
      }
    }
  }
}

// Rows of several ranges: one wave per row, two columns per lane, 16 ranges in flight.
__global__ __launch_bounds__(64 * kWaves) void owq_attend_join_kernel(AttendArgs a, int P) {
  const int lane = threadIdx.x & 63;
  const int head = blockIdx.y, b = blockIdx.z;
  const Sequence sq = sequence_of(a, b);
  const int row = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (row >= sq.n_rows) return;
  const int used = a.places[2 * b + 1];
  if (used == 1) return;
  const int block = row / a.slot_rows;
  const int64_t slot0 = (int64_t)(a.places[2 * b] + (head * a.blocks + block) * used) * a.slot_rows + row - block * a.slot_rows;
  auto slot_of = [&](int s) { return slot0 + (int64_t)s * a.slot_rows; };
  float ref = kNoRef;
  for (int s = lane; s < used; s += 64) ref = fmaxf(ref, a.part_sums[2 * slot_of(s)]);
  ref = wave_max(ref);
  float total = 0.f, o[2] = {0.f, 0.f};
  const int col = 2 * lane < P ? 2 * lane : 0;
  for (int base = 0; base < used; base += 64) {
    const int mine_s = base + lane < used ? base + lane : used - 1;
    const float f = base + lane < used ? __builtin_amdgcn_exp2f(a.part_sums[2 * slot_of(mine_s)] - ref) : 0.f;
    total = __builtin_fmaf(f, base + lane < used ? a.part_sums[2 * slot_of(mine_s) + 1] : 0.f, total);
    const int n = used - base < 64 ? used - base : 64;
    for (int s = 0; s < n; s += 16) {
      float2 v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = *reinterpret_cast<const float2 *>(a.part + slot_of(base + (s + i < n ? s + i : n - 1)) * P + col);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float g = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (s + i) & 63));
        o[0] = s + i < n ? __builtin_fmaf(g, v[i].x, o[0]) : o[0];
        o[1] = s + i < n ? __builtin_fmaf(g, v[i].y, o[1]) : o[1];
      }
    }
  }
  total = wave_sum(total);
  store_row<1>(a, sq, head, row, lane, o, ref, total);
}

AttendPlan attend_plan(const owq_cache_desc_t &d, const owq_attention_desc_t &a) {
  AttendPlan p{};
  p.group = a.q_heads / d.kv_heads;
  const int64_t rows = (int64_t)a.max_new * p.group;
  int64_t seen = std::min<int64_t>(a.max_len, (int64_t)d.table_stride * d.page_size);
  if (a.window > 0) seen = std::min<int64_t>(seen, (int64_t)a.window + a.max_new + a.sinks + 96);
  const int64_t tiles = std::max<int64_t>(1, (seen + 31) / 32);
  const int64_t heads = (int64_t)d.n_seqs * d.kv_heads;
  // Rows in blocks of 128 by whole spans read the keys least often; in blocks of 16 or 32 with the keys cut into ranges they
  // fill the machine with few of them.  Where the blocks of 128 are a workgroup per compute unit, the first is as fast or
  // faster (1 x 1000 of 1000 tokens, 32/8 heads, 256 blocks: 40 us, 49 with ranges); below that it is slower (300 of 2000,
  // 32/32 heads, 96 blocks: 72 us, 46 with ranges; 600 of 4000, 152 blocks: 132 us, 122), but for short spans of half a
  // machine's blocks, where a launch to join costs more (3 x 300 of 300, 204 blocks: 18 us, 28 with ranges).
  const int64_t wide = heads * ((rows + 127) / 128);
  p.fits = true;
  p.many = rows > 64 && (wide >= 256 || (wide >= 128 && tiles <= 16));
  if (p.many) return p;
  p.col_tiles = rows <= 16 ? 1 : 2;
  p.rows = (int)rows;
  p.slot_rows = (int)std::min<int64_t>(rows, 16 * p.col_tiles);
  p.blocks = (int)((rows + 16 * p.col_tiles - 1) / (16 * p.col_tiles));
  const int64_t items = heads * p.blocks;
  // As many workgroups as the compute units hold at once, two tiles per wave at least; whole spans and no second launch where
  // no sequence has more than four tiles per wave, or where the heads are many and the spans short (512 heads of 64 columns on
  // spans of 36 tiles, 8 waves: 14.5 us, 26 with ranges of 4 waves).  Whole spans of more than 16 tiles have 8 waves where the
  // compute units take all workgroups at once, one each with 68 KB of LDS, two up to 64 columns (256 heads of 128 columns on
  // spans of up to 47 tiles: 16 us, 19.3 with 4 waves; 512 heads on 19 tiles: 20 us, 16 with 4).
  const int64_t resident = 256 * (p.col_tiles == 2 ? 2 : kResident);
  p.waves = p.col_tiles == 1 && tiles > 16 && items <= (d.head_dim <= 64 ? 512 : 256) ? 8 : 4;
  p.whole = tiles <= 4 * p.waves || (items >= 256 && tiles <= 64);
  if (!p.whole) p.waves = 4;
  p.least_tiles = 2 * p.waves;
  // Items that fill the compute units by themselves come in turns, and twice the ranges even out their lengths.  More than 32
  // ranges of an item cost more to join than they gain (30 000 tokens of 32/8 heads: 21.3 us, 26.1 with 96).
  p.ranges = (int)(2 * items <= resident ? std::min(resident, 32 * items) : 2 * resident);
  // no more workgroups than p.ranges ranges and one more per item; nor than ranges of the least length
  const int64_t workgroups = p.whole ? items : std::min(p.ranges + items, items * ((tiles + p.least_tiles - 1) / p.least_tiles));
  p.fits = workgroups * 64 * p.waves < (1ll << 32);      // threads of a launch's axis
  p.workgroups = p.fits ? (int)workgroups : 0;
  p.slots = p.whole ? 0 : (size_t)p.workgroups * p.slot_rows;
  const int P = (d.head_dim + 31) / 32 * 32;
  p.workspace = p.whole ? 0 : p.slots * (P + 2) * 4 + (size_t)d.n_seqs * 8;
  return p;
}

template <int STEPS, int NQ, int WAVES>
static void launch_few(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  if (a.bf16) owq_attend_few_kernel<STEPS, NQ, false, WAVES><<<p.workgroups, 64 * WAVES, 0, s>>>(a);
  else owq_attend_few_kernel<STEPS, NQ, true, WAVES><<<p.workgroups, 64 * WAVES, 0, s>>>(a);
  if (!p.whole)
    owq_attend_join_kernel<<<dim3((unsigned)((p.rows + kWaves - 1) / kWaves), (unsigned)a.c.kv_heads, (unsigned)a.c.n_seqs), 64 * kWaves, 0, s>>>(
        a, 32 * STEPS);
}

template <int STEPS>
static void launch_steps(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  if (p.many) launch_attend_many<STEPS>(a, s);
  else if (p.col_tiles == 2) launch_few<STEPS, 2, 4>(a, p, s);
  else if (p.waves == 8) launch_few<STEPS, 1, 8>(a, p, s);
  else launch_few<STEPS, 1, 4>(a, p, s);
}

int launch_attend(const CacheView &c, const owq_attention_desc_t &d, const AttendPlan &p, const void *q, void *out, float *lse,
                  void *workspace, void *stream) {
  AttendArgs a;
  a.c = c;
  a.q = static_cast<const u32 *>(q);
  a.out = static_cast<u32 *>(out);
  a.lse = lse;
  const int steps = (c.head_dim + 31) / 32;
  a.part = static_cast<float *>(workspace);
  a.part_sums = a.part + p.slots * (32 * steps);
  a.q_row = d.q_row, a.q_head = d.q_head;
  a.q_heads = d.q_heads, a.group = p.group, a.max_new = d.max_new, a.window = d.window, a.sinks = d.sinks, a.max_len = d.max_len;
  a.bf16 = d.type == OWQ_TYPE_BF16;
  a.places = reinterpret_cast<int32_t *>(a.part_sums + 2 * p.slots);
  a.slot_rows = p.slot_rows, a.blocks = p.blocks, a.least_tiles = p.least_tiles, a.ranges = p.ranges, a.whole = p.whole;
  a.scale = d.scale * 1.44269504089f;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  switch (steps) {
    case 1: launch_steps<1>(a, p, s); break;
    case 2: launch_steps<2>(a, p, s); break;
    case 3: launch_steps<3>(a, p, s); break;
    default: launch_steps<4>(a, p, s); break;
  }
  return (int)hipGetLastError();
}

}  // namespace owq
