// Residual sum of a block with the norms around it, and the gradients.
//
// A workgroup takes a row (a token); a thread keeps CH pieces of eight elements of it in registers, so that each input is read
// once.  A norm needs the row's mean and squares: every wave takes them of its own elements about their own mean (no rounding of
// a large mean enters), and the waves' are joined as of sets of n_w elements:
//     mean = sum n_w mean_w / n,   M = sum M_w + n_w (mean_w - mean)^2
// which costs one barrier.  Without centring (rms) mean_w = 0 and the same code adds squares.
#include <hip/hip_runtime.h>

#include <mutex>
#include <type_traits>

#include "owq_random_device.h"

namespace owq {

constexpr int kNormWaves = 16;

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  v = wave_scan(v, 0.f, [](float a, float b) { return a + b; });
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

template <int CH>
struct RowPlace {
  int unit[CH], count[CH];      // pieces of this thread and how many of their elements the row has
  int wave_count;               // elements of this wave
  __device__ __forceinline__ RowPlace(int width) {
    const int first = (threadIdx.x >> 6) * 64;
    wave_count = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      unit[c] = c * (int)blockDim.x + (int)threadIdx.x;
      const int n = width - 8 * unit[c], w = width - 8 * (c * (int)blockDim.x + first);
      count[c] = n < 0 ? 0 : n > 8 ? 8 : n;
      wave_count += w < 0 ? 0 : w > 512 ? 512 : w;
    }
  }
};

struct RowStat {
  float mean, size;      // size = 1 / sqrt(mean square + eps)
};

// What a wave knows of a row: mean and sum of squares about it.
template <int CH>
__device__ __forceinline__ void wave_stat(const float (&x)[CH][8], const RowPlace<CH> &at, bool layer, float *mean, float *squares) {
  float m = 0.f;
  if (layer) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) m += x[c][j];            // 0 past the row
    m = wave_sum(m) / (float)(at.wave_count > 0 ? at.wave_count : 1);
  }
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = j < at.count[c] ? x[c][j] - m : 0.f;
      s = __builtin_fmaf(d, d, s);
    }
  *mean = m;
  *squares = wave_sum(s);
}

// Sum over the workgroup's waves of what lane w of every 16 holds for wave w.
__device__ __forceinline__ float waves_sum(float v) { return lanes_sum<16>(v); }

__device__ __forceinline__ RowStat joined_stat(const float2 *part, int width, int ch, bool layer, float eps) {
  const int w = threadIdx.x & 15;
  const bool on = w < (int)(blockDim.x >> 6);
  const float2 p = on ? part[w] : make_float2(0.f, 0.f);
  float mean = 0.f, extra = 0.f;
  if (layer) {
    int n = 0;
    for (int c = 0; c < ch; ++c) {
      const int k = width - 8 * (c * (int)blockDim.x + 64 * w);
      n += k < 0 ? 0 : k > 512 ? 512 : k;
    }
    const float count = on ? (float)n : 0.f;
    mean = waves_sum(count * p.x) / (float)width;
    extra = count * (p.x - mean) * (p.x - mean);
  }
  const float squares = waves_sum(p.y + extra);
  return RowStat{mean, 1.f / __builtin_sqrtf(squares / (float)width + eps)};
}

// Statistics of a row over the whole workgroup.
template <int CH>
__device__ __forceinline__ RowStat row_stat(const float (&x)[CH][8], const RowPlace<CH> &at, float2 *part, int width, bool layer, float eps) {
  float m, s;
  wave_stat<CH>(x, at, layer, &m, &s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(m, s);
  __syncthreads();
  return joined_stat(part, width, CH, layer, eps);
}

template <class E, int CH>
__device__ __forceinline__ void load_row(Piece<E> (&p)[CH], const void *row, const RowPlace<CH> &at, int width) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (row && at.count[c] > 0) p[c].load(row, at.unit[c], width);
    else p[c].zero();
  }
}
template <class E, int CH>
__device__ __forceinline__ void store_row(const float (&x)[CH][8], void *row, const RowPlace<CH> &at, int width) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    Piece<E> p;
    p.put(x[c]);
    if (at.count[c] > 0) p.template store<true>(row, at.unit[c], width);
  }
}

// x of a norm's input -> its output; weight and bias as pieces, where there are any
template <class E, int CH>
__device__ __forceinline__ void apply_norm(float (&x)[CH][8], const RowStat &s, const Piece<E> (&w)[CH], bool has_w, const Piece<E> (&b)[CH],
                                           bool has_b) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float g[8];
    w[c].get(g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[c][j] = (x[c][j] - s.mean) * s.size;
      if (has_w) x[c][j] *= g[j];
    }
    if (has_b) {
      b[c].get(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[c][j] += g[j];
    }
  }
}

template <class E, class H, int CH>
__global__ __launch_bounds__(1024) void owq_norm_kernel(NormArgs a) {
  __shared__ float2 part[2][kNormWaves];
  const RowPlace<CH> at(a.width);
  const DropKey key = drop_key(a.drop);
  for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    Piece<H> ph[CH];
    Piece<E> po[CH], pg[CH], pw[CH], pb[CH];
    load_row<H, CH>(ph, row_at<H>(a.h, t, a.h_row), at, a.width);
    load_row<E, CH>(po, a.branch ? row_at<E>(a.branch, t, a.branch_row) : nullptr, at, a.width);
    load_row<E, CH>(pg, a.gate ? row_at<E>(a.gate, t, a.gate_row) : nullptr, at, a.width);
    float x[CH][8];
    if (a.branch) {
#pragma unroll
      for (int c = 0; c < CH; ++c) po[c].get(x[c]);
      if (a.post != OWQ_NORM_NONE) {
        load_row<E, CH>(pw, a.post_w, at, a.width);
        load_row<E, CH>(pb, a.post_b, at, a.width);
        const RowStat s = row_stat<CH>(x, at, part[0], a.width, a.post == OWQ_NORM_LAYER, a.eps);
        apply_norm<E, CH>(x, s, pw, a.post_w != nullptr, pb, a.post_b != nullptr);
      }
      if (a.drop.threshold > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const u32 bits = stays8(a.drop, key, (u32)at.unit[c], (u32)t);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[c][j] = (bits >> j) & 1u ? x[c][j] * a.drop.scale : 0.f;
        }
      }
    }
    load_row<E, CH>(pw, a.w, at, a.width);
    load_row<E, CH>(pb, a.b, at, a.width);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float h[8], g[8];
      ph[c].get(h);
      pg[c].get(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = a.branch ? a.branch_scale * (a.gate ? x[c][j] * g[j] : x[c][j]) : 0.f;
        x[c][j] = j < at.count[c] ? __builtin_fmaf(a.h_scale, h[j], u) : 0.f;      // 0 past the row, where a bias may stand
      }
    }
    if (a.total_out) store_row<H, CH>(x, row_at<H>(a.total_out, t, a.width), at, a.width);
    if (a.y) {
      const RowStat s = row_stat<CH>(x, at, part[1], a.width, a.norm == OWQ_NORM_LAYER, a.eps);
      apply_norm<E, CH>(x, s, pw, a.w != nullptr, pb, a.b != nullptr);
      store_row<E, CH>(x, row_at<E>(a.y, t, a.width), at, a.width);
    }
    __syncthreads();      // the next row writes `part` again
  }
}

// ---- gradients ----------------------------------------------------------------------------------------------------------------
// A workgroup takes rows blockIdx.x, + gridDim.x, ... and adds its part of the sums over tokens to columns that its threads own,
// in LDS or, where that does not hold them, in its row of the workspace; a second kernel adds the workgroups' in order.

// Two sums over the workgroup.
__device__ __forceinline__ float2 block_sums(float a, float b, float2 *part) {
  a = wave_sum(a), b = wave_sum(b);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  const int w = threadIdx.x & 15;
  const float2 p = w < (int)(blockDim.x >> 6) ? part[w] : make_float2(0.f, 0.f);
  return make_float2(waves_sum(p.x), waves_sum(p.y));
}

// acc[8 columns] += v
__device__ __forceinline__ void add_to(float *acc, const float *v) {
  f32x4 *p = reinterpret_cast<f32x4 *>(acc);
  const f32x4 a = p[0], b = p[1];
  p[0] = (f32x4){a[0] + v[0], a[1] + v[1], a[2] + v[2], a[3] + v[3]};
  p[1] = (f32x4){b[0] + v[4], b[1] + v[5], b[2] + v[6], b[3] + v[7]};
}

// Gradient through a norm: q = gradient of its output times the weight (0 past the row), n = normalised row; q becomes the
// gradient of its input.
template <int CH>
__device__ __forceinline__ void norm_back(float (&q)[CH][8], const float (&n)[CH][8], bool layer, float size, float width, float2 *part) {
  float qn = 0.f, qs = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      qn = __builtin_fmaf(q[c][j], n[c][j], qn);
      qs += q[c][j];
    }
  const float2 s = block_sums(qn, qs, part);
  const float mn = s.x / width, ms = layer ? s.y / width : 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) q[c][j] = size * (q[c][j] - n[c][j] * mn - ms);
}

template <class E, class H, int CH, bool LDS>
__global__ __launch_bounds__(1024) void owq_norm_backward_kernel(NormArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  __shared__ float2 part[4][kNormWaves];
  const RowPlace<CH> at(a.width);
  const DropKey key = drop_key(a.drop);
  const float width = (float)a.width;
  float *mine = a.partial ? a.partial + (int64_t)blockIdx.x * a.n_sums * a.pitch : nullptr;
  float *acc = LDS ? lds : mine;
  for (int k = 0; k < a.n_sums; ++k)
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.count[c] > 0) {
        f32x4 *p = reinterpret_cast<f32x4 *>(acc + k * a.pitch + 8 * at.unit[c]);
        p[0] = p[1] = (f32x4){0.f, 0.f, 0.f, 0.f};
      }
  auto add_row = [&](int k, const float (&v)[CH][8]) {
    if (k < 0) return;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.count[c] > 0) add_to(acc + k * a.pitch + 8 * at.unit[c], v[c]);
  };
  const bool branch_side = a.dbranch || a.dgate || a.sum_post_w >= 0 || a.sum_post_b >= 0 || a.sum_gate >= 0;
  const bool need_u = a.dgate || a.sum_gate >= 0, post = a.post != OWQ_NORM_NONE;
  for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    Piece<E> pdy[CH], po[CH], pg[CH], pw[CH];
    Piece<H> pd[CH], pt[CH];
    load_row<E, CH>(pdy, a.dy ? row_at<E>(a.dy, t, a.dy_row) : nullptr, at, a.width);
    load_row<H, CH>(pt, a.dy ? row_at<H>(a.total, t, a.total_row) : nullptr, at, a.width);
    load_row<H, CH>(pd, a.dtotal ? row_at<H>(a.dtotal, t, a.dtotal_row) : nullptr, at, a.width);
    load_row<E, CH>(po, branch_side && (post || need_u) ? row_at<E>(a.branch, t, a.branch_row) : nullptr, at, a.width);
    load_row<E, CH>(pg, a.gate && branch_side ? row_at<E>(a.gate, t, a.gate_row) : nullptr, at, a.width);
    float d[CH][8], n[CH][8], v[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) d[c][j] = 0.f;
    if (a.dy) {
      load_row<E, CH>(pw, a.w, at, a.width);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        pdy[c].get(d[c]);
        pt[c].get(n[c]);
      }
      const RowStat s = row_stat<CH>(n, at, part[0], a.width, a.norm == OWQ_NORM_LAYER, a.eps);
      add_row(a.sum_b, d);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float w[8];
        pw[c].get(w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          n[c][j] = (n[c][j] - s.mean) * s.size;
          v[c][j] = d[c][j] * n[c][j];
          if (a.w) d[c][j] *= w[j];
        }
      }
      add_row(a.sum_w, v);
      norm_back<CH>(d, n, a.norm == OWQ_NORM_LAYER, s.size, width, part[1]);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float g[8];
      pd[c].get(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d[c][j] = j < at.count[c] ? d[c][j] + g[j] : 0.f;
        v[c][j] = a.h_scale * d[c][j];
      }
    }
    if (a.dh) store_row<H, CH>(v, row_at<H>(a.dh, t, a.width), at, a.width);
    if (branch_side) {
      // d becomes the gradient of u, n the branch normalised
      RowStat s = {0.f, 1.f};
      if (post || need_u) {
#pragma unroll
        for (int c = 0; c < CH; ++c) po[c].get(n[c]);
        if (post) {
          s = row_stat<CH>(n, at, part[2], a.width, a.post == OWQ_NORM_LAYER, a.eps);
          load_row<E, CH>(pw, a.post_w, at, a.width);
        }
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const u32 bits = a.drop.threshold > 0 ? stays8(a.drop, key, (u32)at.unit[c], (u32)t) : 255u;
        float g[8], w[8], b[8];
        pg[c].get(g);
        pw[c].get(w);
        if (need_u && post && a.post_b) {
          Piece<E> pb;
          pb.zero();
          if (at.count[c] > 0) pb.load(a.post_b, at.unit[c], a.width);
          pb.get(b);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool on = (bits >> j) & 1u;
          const float e = a.branch_scale * d[c][j];
          if (post) n[c][j] = (n[c][j] - s.mean) * s.size;
          if (need_u) {
            float u = n[c][j];
            if (post && a.post_w) u *= w[j];
            if (post && a.post_b) u += b[j];
            v[c][j] = e * (on ? u * a.drop.scale : 0.f);
          }
          const float q = a.gate ? e * g[j] : e;
          d[c][j] = on ? q * a.drop.scale : 0.f;
        }
      }
      if (a.dgate) store_row<E, CH>(v, row_at<E>(a.dgate, t, a.width), at, a.width);
      add_row(a.sum_gate, v);
      if (post) {
        add_row(a.sum_post_b, d);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float w[8];
          pw[c].get(w);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[c][j] = d[c][j] * n[c][j];
            if (a.post_w) d[c][j] *= w[j];
          }
        }
        add_row(a.sum_post_w, v);
        if (a.dbranch) norm_back<CH>(d, n, a.post == OWQ_NORM_LAYER, s.size, width, part[3]);
      }
      if (a.dbranch) store_row<E, CH>(d, row_at<E>(a.dbranch, t, a.width), at, a.width);
    }
    __syncthreads();      // the next row writes `part` again
  }
  if (LDS && mine)
    for (int k = 0; k < a.n_sums; ++k)
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (at.count[c] > 0) {
          const int i = k * a.pitch + 8 * at.unit[c];
          const f32x4 *from = reinterpret_cast<const f32x4 *>(lds + i);
          f32x4 *to = reinterpret_cast<f32x4 *>(mine + i);
          to[0] = from[0];
          to[1] = from[1];
        }
}

struct NormSums {
  float *out[5];
};

// Column sums of partial [blocks][n_sums][pitch]: 64 columns per workgroup, 16 rows at a time.
__global__ __launch_bounds__(1024) void owq_norm_sums_kernel(const float *partial, int blocks, int n_sums, int pitch, int width, NormSums sums) {
  __shared__ float part[16][64];
  const int lane = threadIdx.x & 63, first = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane, k = blockIdx.y;
  float v = 0.f;
  if (col < width)
    for (int i = first; i < blocks; i += 16) v += partial[((int64_t)i * n_sums + k) * pitch + col];
  part[first][lane] = v;
  __syncthreads();
  if (first == 0 && col < width) {
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) total += part[i][lane];
    float *out = sums.out[0];
#pragma unroll
    for (int i = 1; i < 5; ++i) out = k == i ? sums.out[i] : out;
    out[col] = total;
  }
}

// Pieces of a thread and threads of a workgroup.
struct NormShape {
  int ch, threads;
};
static NormShape norm_shape(int width) {
  const int units = (width + 7) / 8;
  const int ch = units > 1024 ? 2 : 1;
  return NormShape{ch, ((units + ch - 1) / ch + 63) / 64 * 64};
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

int launch_norm(const NormArgs &a, int32_t type, int32_t h_type, void *stream) {
  const NormShape n = norm_shape(a.width);
  const unsigned grid = (unsigned)(a.n_tokens < (1 << 16) ? a.n_tokens : 1 << 16);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  for_types(type, h_type, [&](auto e, auto h) {
    if (n.ch == 1) owq_norm_kernel<decltype(e), decltype(h), 1><<<grid, n.threads, 0, s>>>(a);
    else owq_norm_kernel<decltype(e), decltype(h), 2><<<grid, n.threads, 0, s>>>(a);
  });
  return (int)hipGetLastError();
}

NormPlan norm_backward_plan(const owq_norm_desc_t &d) {
  const int64_t most = 512, each = (d.n_tokens + most - 1) / most;
  return NormPlan{each == 0 ? 0 : (int32_t)((d.n_tokens + each - 1) / each), (d.width + 7) / 8 * 8};
}

constexpr int kNormLds = 65536 - 1024;

int launch_norm_backward(const NormArgs &a, int32_t type, int32_t h_type, const NormPlan &p, float *const *sums, void *stream) {
  const NormShape n = norm_shape(a.width);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t bytes = (int64_t)a.n_sums * p.pitch * 4;
  const bool lds = bytes <= kNormLds;
  if (p.blocks > 0) for_types(type, h_type, [&](auto e, auto h) {
    auto go = [&](auto ch, auto in_lds) {
      owq_norm_backward_kernel<decltype(e), decltype(h), decltype(ch)::value, decltype(in_lds)::value>
          <<<p.blocks, n.threads, decltype(in_lds)::value ? (size_t)bytes : 0, s>>>(a);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    if (n.ch == 1 && lds) go(One(), std::true_type());
    else if (n.ch == 1) go(One(), std::false_type());
    else if (lds) go(Two(), std::true_type());
    else go(Two(), std::false_type());
  });
  if (a.n_sums > 0) {
    NormSums out{};
    for (int i = 0; i < a.n_sums; ++i) out.out[i] = sums[i];
    owq_norm_sums_kernel<<<dim3((unsigned)((a.width + 63) / 64), (unsigned)a.n_sums), 1024, 0, s>>>(a.partial, p.blocks, a.n_sums, p.pitch, a.width, out);
  }
  return (int)hipGetLastError();
}

}  // namespace owq
