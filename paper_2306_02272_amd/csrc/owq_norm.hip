// Residual sum of a block with the norms around it, and the gradients.
//
// A team of waves takes a row (a token); a thread keeps CH pieces of eight elements of it in registers, so that each input is
// read once.  A norm needs the row's mean and squares: every wave takes them of its own elements about their own mean (no
// rounding of a large mean enters), and the waves' are joined as of sets of n_w elements:
//     mean = sum n_w mean_w / n,   M = sum M_w + n_w (mean_w - mean)^2
// which costs one barrier.  Without centring (rms) mean_w = 0 and the same code adds squares.
//
// Pieces past the row are 0, and so are weights there, so that products and sums need no further care.
//
// What bounds it, with the rows' bytes at the rate of a large copy (5.1 TB/s) in brackets: one row of 4096 3.3 us (a load, a
// reduction, a store behind each other); 4096 rows of 4096 fp16, layer norm, 24 to 28 us (26.3; reads and writes of memory); 1021
// rows of 9216 with both norms and the gate, fp32 residual, 26 to 32 (22.2; 165 registers: one workgroup of nine waves at work on a
// compute unit, vector instructions in 36 % of the cycles).  Gradients: 4096 rows of 4096 with dropout 34 + 4 us (32.9: memory, and 8 MB of partial sums written and read);
// 777 rows of 5003 with both norms and the gate 30 + 4 (9.2: 163 registers, ten waves per compute unit, one row behind the other in each;
// vector instructions in 42 % of the cycles).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "owq_norm_device.h"

namespace owq {

// Most threads of a team, by pieces of a thread: 64 registers for each, or as many as there are.  Fewest pieces first: 3640 rows of
// 4608 take 29 us with one piece and 45 with two (both norms 45 and 60), rows of 8192 29.4 and 30.5.  Past three pieces the rolled
// kernels: 1021 rows of 9216 19.4 us with two pieces and 19.7 in a rolled one (both norms 32.4 and 42.9),
// 1021 of 11 008 with two norms 32.7 with three and 43.0.
constexpr int norm_threads(int ch) { return ch == 1 ? 1024 : ch == 2 ? 640 : 512; }

// The inputs of a row as they lie in memory.
template <class E, class H, int CH>
struct ForwardRow {
  Piece<H> h[CH];
  Piece<E> o[CH], g[CH];
  __device__ __forceinline__ void load(const NormArgs &a, int64_t t, const RowPlace<CH> &at) {
    load_row<H, CH>(h, row_at<H>(a.h, t, a.h_row), at, a.width);
    load_row<E, CH>(o, a.branch ? row_at<E>(a.branch, t, a.branch_row) : nullptr, at, a.width);
    load_vector<E, CH>(g, a.gate ? row_at<E>(a.gate, t, a.gate_row) : nullptr, 1.f, at, a.width);
  }
};

template <class E, class H, int CH, bool POST>
__global__ __launch_bounds__(norm_threads(CH), CH > 1 ? 1 : (POST ? 6 : 8) - (Piece<H>::kSize == 4 ? 1 : 0)) void owq_norm_kernel(NormArgs a) {
  constexpr bool AHEAD = CH == 2 && !POST;      // where the registers hold the next row: 1021 rows of 9216 19.4 us, 25.4 by workgroups of a row
  __shared__ float2 part[2][kNormWaves];
  const RowPlace<CH> at(a.width, blockDim.x, true);
  TeamSum<float2> sums{part[0], 0};
  const DropKey key = drop_key(a.drop);
  const float inverse_width = 1.f / (float)a.width;
  const bool layer = a.norm == OWQ_NORM_LAYER, post_layer = a.post == OWQ_NORM_LAYER;
  ForwardRow<E, H, CH> now, next;
  if (AHEAD) next.load(a, blockIdx.x, at);
  for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    Piece<E> w[CH], b[CH];
    if (AHEAD) {
      now = next;
      if (t + gridDim.x < a.n_tokens) next.load(a, t + gridDim.x, at);
    } else {
      now.load(a, t, at);
    }
    float x[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) now.o[c].get(x[c]);
    if (POST) {
      load_vector<E, CH>(w, a.post_w, 1.f, at, a.width);
      load_vector<E, CH>(b, a.post_b, 0.f, at, a.width);
      const float2 p = sums.join(at, wave_stat<CH>(x, at, a.width, post_layer), make_float2(0.f, 0.f));
      apply_norm<E, CH>(x, joined_stat(p, at, inverse_width, post_layer, a.eps), w, b);
    }
    if (a.drop.threshold > 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const Stays on(a.drop, key, (u32)at.unit[c], (u32)t);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[c][j] = on(j) ? x[c][j] * a.drop.scale : 0.f;
      }
    }
    load_vector<E, CH>(w, a.w, 1.f, at, a.width);
    load_vector<E, CH>(b, a.b, 0.f, at, a.width);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float h[8], g[8];
      now.h[c].get(h);
      now.g[c].get(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[c][j] = __builtin_fmaf(a.h_scale, h[j], a.branch_scale * (x[c][j] * g[j]));
    }
    if (AHEAD) loads_done();
    if (a.total_out) store_row<H, CH>(x, row_at<H>(a.total_out, t, a.width), at, a.width);
    if (a.y) {
      const float2 p = sums.join(at, wave_stat<CH>(x, at, a.width, layer), make_float2(0.f, 0.f));
      apply_norm<E, CH>(x, joined_stat(p, at, inverse_width, layer, a.eps), w, b);
      store_row<E, CH>(x, row_at<E>(a.y, t, a.width), at, a.width);
    }
  }
}

// ---- gradients ----------------------------------------------------------------------------------------------------------------
// With q the gradient of a norm's output times its weight, c the wave's mean and n = (x - mean) size the normalised row, the
// input's is size (q - n mean(q n) - [layer] mean(q)).  A wave adds q (x - c) and q beside its squares, and the join moves them
// to the row's mean: sum q (x - mean) = sum_w (Q_w + (c_w - mean) q_w), so that one barrier serves the statistics and both means.
//
// A workgroup of at most 1024 threads is as many teams as fit; team i of workgroup k takes rows (k teams + i) + steps of all
// teams.  With one or two pieces a thread it asks for its next row before it works on this one, but where a norm of the branch meets a
// gate only with one piece and a residual in 16 bits.  With one piece what it adds up over its rows stays in registers, as a
// thread owns its columns; at the end the teams' are added through LDS and left as one row of the workspace, which a second
// kernel adds up in order.  Two and three pieces a thread leave no registers for that: their sums are kept in LDS, and those that it does
// not hold in the workspace's row from the start.

// Most threads of a workgroup: 128 registers for a thread, or 168 with the branch's side.  1021 rows of 8192 with both norms and the
// gate take 48.8 us with two pieces a thread, 76 in the rolled kernel; 1021 of 11 008 45 with three (rms before, no gate) and 58; 2048 of
// 8192 without the branch's side 38.0 with one piece and 1024 threads, 43.1 with two and 512.
constexpr int norm_backward_threads(int ch, bool branch) { return ch > 1 ? 512 : branch ? 640 : 1024; }

constexpr int kSumsLds = 38912;      // floats for the sums of two and three pieces a thread

template <int CH, bool REGISTERS>
struct ColumnSum;
template <int CH>
struct ColumnSum<CH, true> {
  float v[CH][8];
  __device__ __forceinline__ void start(float *, int, int, float *, const RowPlace<CH> &) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[c][j] = 0.f;
  }
  __device__ __forceinline__ void add(const RowPlace<CH> &, int c, const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[c][j] += x[j];
  }
  // store: the workgroup's [teams][columns] in LDS
  __device__ __forceinline__ void finish(float *mine, int k, int pitch, const RowPlace<CH> &at, int teams, float *store) {
    if (!mine || k < 0) return;            // the same for the whole workgroup
    float *to = mine + k * pitch;
    if (teams == 1) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (at.count[c] > 0) put8(to, at.unit[c], v[c]);
      return;
    }
    const int columns = at.threads * 8 * CH;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < CH; ++c) put8(store + at.team * columns, at.unit[c], v[c]);
    __syncthreads();
    for (int i = 4 * (int)threadIdx.x; i < pitch; i += 4 * (int)blockDim.x) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
      for (int j = 0; j < teams; ++j) s += *reinterpret_cast<const f32x4 *>(store + j * columns + i);
      *reinterpret_cast<f32x4 *>(to + i) = s;
    }
  }
};
template <int CH>
struct ColumnSum<CH, false> {
  float *to;
  __device__ __forceinline__ void start(float *mine, int k, int pitch, float *store, const RowPlace<CH> &at) {
    to = !mine || k < 0 ? nullptr : (k + 1) * pitch <= kSumsLds ? store + k * pitch : mine + k * pitch;
    if (!to) return;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.count[c] > 0) {
        f32x4 *p = reinterpret_cast<f32x4 *>(to) + 2 * at.unit[c];
        p[0] = p[1] = (f32x4){0.f, 0.f, 0.f, 0.f};
      }
  }
  __device__ __forceinline__ void add(const RowPlace<CH> &at, int c, const float (&x)[8]) {
    if (!to || at.count[c] == 0) return;
    f32x4 *p = reinterpret_cast<f32x4 *>(to) + 2 * at.unit[c];
    const f32x4 a = p[0], b = p[1];
    p[0] = (f32x4){a[0] + x[0], a[1] + x[1], a[2] + x[2], a[3] + x[3]};
    p[1] = (f32x4){b[0] + x[4], b[1] + x[5], b[2] + x[6], b[3] + x[7]};
  }
  __device__ __forceinline__ void finish(float *mine, int k, int pitch, const RowPlace<CH> &at, int, float *) {
    if (!mine || k < 0 || (k + 1) * pitch > kSumsLds) return;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.count[c] > 0) {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(to) + 2 * at.unit[c];
        f32x4 *out = reinterpret_cast<f32x4 *>(mine + k * pitch) + 2 * at.unit[c];
        out[0] = p[0];
        out[1] = p[1];
      }
  }
};

// Sums of a wave: c = its mean (0 without centring), squares of x - c, q (x - c), q.
template <int CH>
__device__ __forceinline__ float4 wave_back(const float (&x)[CH][8], const float (&q)[CH][8], const RowPlace<CH> &at, int width, bool layer) {
  const float2 s = wave_stat<CH>(x, at, width, layer);
  float qx = 0.f, qs = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) qx = __builtin_fmaf(q[c][j], x[c][j] - s.x, qx);
  if (layer) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) qs += q[c][j];
    qs = wave_sum(qs);
  }
  return make_float4(s.x, s.y, wave_sum(qx), qs);
}

template <class E, class H, int CH, bool POST, bool GATED>
struct BackwardRow {
  Piece<E> dy[CH], o[CH], g[CH];
  Piece<H> total[CH], d[CH];
  // what is not there: 0
  __device__ __forceinline__ void load(const NormArgs &a, int64_t t, bool on, const RowPlace<CH> &at) {
    load_row<E, CH>(dy, on && a.dy ? row_at<E>(a.dy, t, a.dy_row) : nullptr, at, a.width);
    load_row<H, CH>(total, on && a.dy ? row_at<H>(a.total, t, a.total_row) : nullptr, at, a.width);
    load_row<H, CH>(d, on && a.dtotal ? row_at<H>(a.dtotal, t, a.dtotal_row) : nullptr, at, a.width);
    if (POST || GATED) load_row<E, CH>(o, on && a.branch ? row_at<E>(a.branch, t, a.branch_row) : nullptr, at, a.width);
    if (GATED && CH < 3) load_row<E, CH>(g, on ? row_at<E>(a.gate, t, a.gate_row) : nullptr, at, a.width);
  }
};

template <class E, class H, int CH, bool POST, bool GATED>
__global__ __launch_bounds__(norm_backward_threads(CH, POST || GATED)) void owq_norm_backward_kernel(NormArgs a, int team_threads, int teams) {
  constexpr bool REG = CH == 1, AGAIN = CH > 1;
  constexpr bool AHEAD = CH < 3 && (!(POST && GATED) || (CH == 1 && Piece<H>::kSize == 2));      // where the registers hold it
  __shared__ float4 part[2][kNormWaves];
  __shared__ __attribute__((aligned(16))) float store[REG ? norm_backward_threads(CH, POST || GATED) * 8 : kSumsLds];
  const RowPlace<CH> at(a.width, team_threads, false);
  TeamSum<float4> sums{part[0], 0};
  const DropKey key = drop_key(a.drop);
  const float inverse_width = 1.f / (float)a.width;
  const bool layer = a.norm == OWQ_NORM_LAYER, post_layer = a.post == OWQ_NORM_LAYER;
  const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
  float *mine = a.partial ? a.partial + (int64_t)blockIdx.x * a.n_sums * a.pitch : nullptr;
  ColumnSum<CH, REG> sum_w, sum_b, sum_pw, sum_pb, sum_g;
  sum_w.start(mine, a.sum_w, a.pitch, store, at);
  sum_b.start(mine, a.sum_b, a.pitch, store, at);
  if (POST) sum_pw.start(mine, a.sum_post_w, a.pitch, store, at);
  if (POST) sum_pb.start(mine, a.sum_post_b, a.pitch, store, at);
  if (GATED) sum_g.start(mine, a.sum_gate, a.pitch, store, at);

  const int64_t stride = (int64_t)gridDim.x * teams;
  int64_t t = (int64_t)blockIdx.x * teams + at.team;
  BackwardRow<E, H, CH, POST, GATED> now, next;
  if (AHEAD) next.load(a, t, t < a.n_tokens, at);
  // in registers for all rows, or, with three pieces a thread, read again from the caches
  constexpr bool HELD = CH < 3;
  Piece<E> w[CH], pw[CH], pb[CH];
  if (HELD) {
    load_vector<E, CH>(w, a.w, 1.f, at, a.width);
    if (POST) load_vector<E, CH>(pw, a.post_w, 1.f, at, a.width);
    if (POST && GATED) load_vector<E, CH>(pb, a.post_b, 0.f, at, a.width);
  }
  auto shared = [&](Piece<E> &p, const void *v, float none, int c, float (&f)[8]) __attribute__((always_inline)) {
    if (HELD) {
      again<AGAIN>(p);
    } else {
      asm volatile("" : "+s"(v));      // keeps the load in the loop over rows
      load_shared<E>(p, v, none, at.unit[c], at.count[c], a.width);
    }
    p.get(f);
  };
  // as long as the workgroup's first team has a row
  for (int64_t first = (int64_t)blockIdx.x * teams; first < a.n_tokens; first += stride, t += stride) {
    const bool on_row = t < a.n_tokens;      // else a team without one: zeros, which without eps are no numbers once normalised
    if (AHEAD) {
      now = next;
      next.load(a, t + stride, t + stride < a.n_tokens, at);
    } else {
      now.load(a, t, on_row, at);
    }
    float d[CH][8], n[CH][8], o[CH][8];
    u32 kept[CH];
    if (a.dy) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float k[8];
        now.total[c].get(n[c]);
        now.dy[c].get(d[c]);
        if (on_row) sum_b.add(at, c, d[c]);
        shared(w[c], a.w, 1.f, c, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[c][j] *= k[j];
      }
      const void *total = row_at<H>(a.total, on_row ? t : 0, a.total_row);
      if (!HELD) asm volatile("" : "+s"(total));
      const float4 p = sums.join(at, wave_back<CH>(n, d, at, a.width, layer), none);
      const BackStat s = joined_back(p, at, inverse_width, layer, a.eps);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float g[8], y[8], k[8];
        again<AGAIN>(now.dy[c]);
        if (!HELD && POST && GATED && Piece<H>::kSize == 4) now.total[c].load(total, at.unit[c], a.width);
        else again<AGAIN>(now.total[c]);
        now.dy[c].get(y);
        now.total[c].get(n[c]);
        now.d[c].get(g);
        shared(w[c], a.w, 1.f, c, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          n[c][j] = (n[c][j] - s.mean) * s.size;
          d[c][j] = __builtin_fmaf(s.size, y[j] * k[j], g[j]) + __builtin_fmaf(s.along, n[c][j], s.all);
          y[j] *= n[c][j];
        }
        if (on_row) sum_w.add(at, c, y);
      }
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) now.d[c].get(d[c]);
    }
    if (AHEAD) loads_done();
    if (a.dh && on_row) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) n[c][j] = a.h_scale * d[c][j];
      store_row<H, CH>(n, row_at<H>(a.dh, t, a.width), at, a.width);
    }
    if (!a.branch_side) continue;
    // The branch's side.  n = branch_scale D times what dropping multiplies by, v = the gradient of the norm's output (or of the
    // branch), which is n gate where it stays.
    if (POST || GATED) {
#pragma unroll
      for (int c = 0; c < CH; ++c) now.o[c].get(o[c]);
    }
    const float scale = a.branch_scale * a.drop.scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      // past the row the norm's means still stand in d
      if (POST && !GATED && (a.width & 7) != 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) n[c][j] = j < at.count[c] ? scale * d[c][j] : 0.f;
      } else {
        const float f = POST && !GATED && at.count[c] == 0 ? 0.f : scale;
#pragma unroll
        for (int j = 0; j < 8; ++j) n[c][j] = f * d[c][j];
      }
      kept[c] = 255u;
      if (a.drop.threshold > 0) {
        const Stays on(a.drop, key, (u32)at.unit[c], (u32)t);
        kept[c] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (GATED) kept[c] |= on(j) ? 1u << j : 0u;
          else n[c][j] = on(j) ? n[c][j] : 0.f;
        }
      }
    }
    const void *gate = GATED && !HELD ? row_at<E>(a.gate, t, a.gate_row) : nullptr;      // one team: t is a row
    const void *branch = POST && GATED && !HELD ? row_at<E>(a.branch, t, a.branch_row) : nullptr;
    if (!HELD) asm volatile("" : "+s"(branch));
    auto gradient = [&](int c, float (&v)[8]) __attribute__((always_inline)) {
      if (GATED) {
        float g[8];
        shared(now.g[c], gate, 1.f, c, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = n[c][j] * g[j];
        if (a.drop.threshold > 0) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (kept[c] >> j) & 1u ? v[j] : 0.f;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = n[c][j];
      }
    };
    BackStat s = {0.f, 1.f, 0.f, 0.f};
    if (POST) {
      float q[CH][8];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float k[8];
        gradient(c, q[c]);
        if (on_row) sum_pb.add(at, c, q[c]);
        shared(pw[c], a.post_w, 1.f, c, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[c][j] *= k[j];
      }
      const float4 p = sums.join(at, wave_back<CH>(o, q, at, a.width, post_layer), none);
      s = joined_back(p, at, inverse_width, post_layer, a.eps);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float v[8], k[8], f[8];
      gradient(c, v);
      if (POST) {
        if (!HELD && GATED) now.o[c].load(branch, at.unit[c], a.width);
        else again<AGAIN>(now.o[c]);
        shared(pw[c], a.post_w, 1.f, c, k);
        now.o[c].get(o[c]);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[c][j] = (o[c][j] - s.mean) * s.size;
      }
      if (GATED) {
        if (POST) shared(pb[c], a.post_b, 0.f, c, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) n[c][j] *= POST ? __builtin_fmaf(o[c][j], k[j], f[j]) : o[c][j];
        if (a.drop.threshold > 0) {      // dropped: 0 whatever the branch holds
#pragma unroll
          for (int j = 0; j < 8; ++j) n[c][j] = (kept[c] >> j) & 1u ? n[c][j] : 0.f;
        }
        if (on_row) sum_g.add(at, c, n[c]);
      }
      if (POST) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[j] = v[j] * o[c][j];
          v[j] = __builtin_fmaf(s.size, v[j] * k[j], __builtin_fmaf(s.along, o[c][j], s.all));
        }
        if (on_row) sum_pw.add(at, c, f);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) d[c][j] = v[j];
    }
    if (GATED && a.dgate && on_row) store_row<E, CH>(n, row_at<E>(a.dgate, t, a.width), at, a.width);
    if (a.dbranch && on_row) store_row<E, CH>(d, row_at<E>(a.dbranch, t, a.width), at, a.width);
  }
  sum_w.finish(mine, a.sum_w, a.pitch, at, teams, store);
  sum_b.finish(mine, a.sum_b, a.pitch, at, teams, store);
  if (POST) sum_pw.finish(mine, a.sum_post_w, a.pitch, at, teams, store);
  if (POST) sum_pb.finish(mine, a.sum_post_b, a.pitch, at, teams, store);
  if (GATED) sum_g.finish(mine, a.sum_gate, a.pitch, at, teams, store);
}

struct NormSums {
  float *out[5];
};

// Column sums of partial [blocks][n_sums][pitch]: 64 columns per workgroup, four per thread, four rows of a thread in flight.  4.0 us for
// 8 MB of 256 workgroups' two sums of 4096, which lie in the last-level cache: the launch, two loads behind each other, a barrier.
// 32 columns or 16 per workgroup were no faster.
__global__ __launch_bounds__(1024) void owq_norm_sums_kernel(const float *partial, int blocks, int n_sums, int pitch, int width, NormSums sums) {
  constexpr int COLS = 64, kLanes = COLS / 4, kRows = 1024 / kLanes;
  __shared__ f32x4 part[kRows][kLanes];
  const int lane = threadIdx.x % kLanes, first = threadIdx.x / kLanes;
  const int col = blockIdx.x * COLS + 4 * lane, k = blockIdx.y;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (col < pitch) {
    const float *from = partial + (int64_t)k * pitch + col;
    const int64_t row = (int64_t)n_sums * pitch;
    for (int base = 0; base < blocks; base += 4 * kRows) {
      f32x4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = base + kRows * j + first;
        x[j] = *reinterpret_cast<const f32x4 *>(from + (i < blocks ? i : blocks - 1) * row);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (base + kRows * j + first < blocks) v += x[j];
    }
  }
  part[first][lane] = v;
  __syncthreads();
  if (threadIdx.x < 4 * COLS) {           // four threads add a quarter of the rows of a column each
    const int c = threadIdx.x >> 2, q = threadIdx.x & 3;
    const float *p = reinterpret_cast<const float *>(part);
    float total = 0.f;
#pragma unroll 16
    for (int i = 0; i < kRows / 4; ++i) total += p[(kRows / 4 * q + i) * COLS + c];
    total = lanes_sum<4>(total);
    float *out = sums.out[0];
#pragma unroll
    for (int i = 1; i < 5; ++i) out = k == i ? sums.out[i] : out;
    const int at = blockIdx.x * COLS + c;
    if (q == 0 && at < width) out[at] = total;
  }
}

// Pieces of a thread and threads of a team.
struct NormShape {
  int ch, threads;
};
template <class F>
static NormShape norm_shape(int width, int pieces, F &&most) {
  const int units = (width + 7) / 8;
  for (int ch = 1; ch <= pieces; ++ch)
    if (units <= ch * most(ch)) return NormShape{ch, ((units + ch - 1) / ch + 63) / 64 * 64};
  return NormShape{0, 0};      // too wide for the registers
}

template <class F>
static void for_types(int type, int h_type, F &&f) {
  if (type == OWQ_TYPE_F16) {
    if (h_type == OWQ_TYPE_F32) f(F16(), F32());
    else f(F16(), F16());
  } else {
    if (h_type == OWQ_TYPE_F32) f(BF16(), F32());
    else f(BF16(), BF16());
  }
}
template <class F>
static void for_bool(bool b, F &&f) {
  if (b) f(std::true_type());
  else f(std::false_type());
}
template <int MOST, class F>
static void for_pieces(int ch, F &&f) {
  if (ch == 1) f(std::integral_constant<int, 1>());
  else if (ch == 2) f(std::integral_constant<int, 2>());
  else if constexpr (MOST == 3) f(std::integral_constant<int, 3>());
}

int launch_norm(const NormArgs &args, int32_t type, int32_t h_type, void *stream) {
  NormArgs a = args;
  if (!a.branch) a.branch_scale = 0.f, a.post = OWQ_NORM_NONE;
  const NormShape n = norm_shape(a.width, 3, [](int ch) { return norm_threads(ch); });
  if (n.ch == 0) return launch_norm_wide(a, type, h_type, stream);
  // As many workgroups as the registers let be at work together, each of which takes several rows, where rows wait for a norm of the
  // branch or fill most of a compute unit: 3640 rows of 4608 with both norms 38.6 us, 45.2 with more workgroups than that; 2340 of
  // 7168 29.2 and 33.4.  Otherwise new workgroups as others end, whose loads run beside those: 5000 rows of 2560 24.3, 27.9 so.
  // With two or three pieces one workgroup per compute unit: 1021 rows of 9216 19.4 us, 21.0 with two.
  const int waves = 4 * ((a.post != OWQ_NORM_NONE ? 6 : 8) - (h_type == OWQ_TYPE_F32 ? 1 : 0)), per_row = n.threads / 64;
  const bool resident = a.post != OWQ_NORM_NONE || per_row >= 12;
  const int64_t most = n.ch > 1 ? 256 : resident ? 256 * (waves / per_row) : (1 << 20) / n.threads;
  const unsigned grid = (unsigned)(a.n_tokens < most ? a.n_tokens : most);
  for_types(type, h_type, [&](auto e, auto h) {
    for_pieces<3>(n.ch, [&](auto ch) {
      for_bool(a.post != OWQ_NORM_NONE, [&](auto post) {
        owq_norm_kernel<decltype(e), decltype(h), decltype(ch)::value, decltype(post)::value>
            <<<grid, n.threads, 0, static_cast<hipStream_t>(stream)>>>(a);
      });
    });
  });
  return (int)hipGetLastError();
}

// A workgroup per compute unit; as many teams in it as there are rows for, and the same number of rows for each.  8192 rows of 1024:
// 23.0 us with eight teams, 46.5 with one; 4096 of 4096 37.6 with two and 39.2.
static NormShape norm_backward_shape(int width, bool branch) {
  return norm_shape(width, 3, [=](int ch) { return norm_backward_threads(ch, branch); });
}
static int norm_teams(const NormShape &n, bool branch, int64_t n_tokens) {
  const int64_t fit = n.ch != 1 ? 1 : norm_backward_threads(1, branch) / n.threads, rows = (n_tokens + 255) / 256;
  return (int)(rows < 1 ? 1 : rows < fit ? rows : fit);
}

NormPlan norm_backward_plan(const owq_norm_desc_t &d) {
  const bool branch = d.post != OWQ_NORM_NONE || d.gate != OWQ_GATE_NONE;
  const int64_t teams = norm_teams(norm_backward_shape(d.width, branch), branch, d.n_tokens);
  const int64_t each = (d.n_tokens + 256 * teams - 1) / (256 * teams) * teams;      // rows of a workgroup
  return NormPlan{each == 0 ? 0 : (int32_t)((d.n_tokens + each - 1) / each), (d.width + 7) / 8 * 8};
}

int launch_norm_backward(const NormArgs &a, int32_t type, int32_t h_type, const NormPlan &p, float *const *sums, void *stream) {
  const bool branch = a.post != OWQ_NORM_NONE || a.gate != nullptr;
  const NormShape n = norm_backward_shape(a.width, branch);
  const int teams = norm_teams(n, branch, a.n_tokens);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.blocks > 0 && n.ch == 0) {
    launch_norm_backward_wide(a, type, h_type, p.blocks, stream);
  } else if (p.blocks > 0) for_types(type, h_type, [&](auto e, auto h) {
    for_pieces<3>(n.ch, [&](auto ch) {
      for_bool(a.post != OWQ_NORM_NONE && a.branch_side, [&](auto post) {
        for_bool(a.gate != nullptr && a.branch_side, [&](auto gated) {
          owq_norm_backward_kernel<decltype(e), decltype(h), decltype(ch)::value, decltype(post)::value, decltype(gated)::value>
              <<<p.blocks, n.threads * teams, 0, s>>>(a, n.threads, teams);
        });
      });
    });
  });
  if (a.n_sums > 0) {
    NormSums out{};
    for (int i = 0; i < a.n_sums; ++i) out.out[i] = sums[i];
    owq_norm_sums_kernel<<<dim3((unsigned)((a.width + 63) / 64), (unsigned)a.n_sums), 1024, 0, s>>>(a.partial, p.blocks, a.n_sums, p.pitch, a.width, out);
  }
  return (int)hipGetLastError();
}

}  // namespace owq
