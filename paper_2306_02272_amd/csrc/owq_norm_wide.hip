// Residual sum with norms, and the gradients, for rows that registers do not hold: a workgroup takes a row in rolled loops and
// keeps what it comes back to in LDS, where a thread's pieces are its own.  (With the pieces of such a row in registers and every
// loop over them unrolled the kernels are thousands of instructions that a row runs through once: fetching them bounds it.)
// The formulas and the join of the waves' statistics are those of owq_norm.hip.  1000 rows of 16 384 fp16 take 26 to 30 us (25.7 by their
// bytes at the rate of a large copy), 46 to 53 with both norms and a gate, their gradients 70 and 140 (32 and 39): the passes over a row stand
// behind each other, and a compute unit has one or two rows at work: LDS holds two of the forward's and one of the gradients', and the
// 132 to 134 registers of a forward with a norm of the branch let one workgroup of eight waves in; the gradients read and write the sums
// over tokens for every row.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "owq_norm_device.h"

namespace owq {

__device__ __forceinline__ void get8(const float *row, int unit, float (&x)[8]) {
  const f32x4 *p = reinterpret_cast<const f32x4 *>(row) + 2 * unit;
  const f32x4 a = p[0], b = p[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
}
__device__ __forceinline__ int count_of(int width, int unit) { return min(width - 8 * unit, 8); }

// Elements of wave w's pieces.
__device__ __forceinline__ int wave_elements(int width, int w) {
  int n = 0;
  for (int first = 64 * w; 8 * first < width; first += blockDim.x) n += min(width - 8 * first, 512);
  return n;
}

// The waves' numbers over the workgroup, in two sets in turn as in owq_norm.hip: those of wave (lane % 16).
struct WideJoin {
  float4 (*part)[kNormWaves];
  int turn;
  float join;          // elements of that wave
  __device__ __forceinline__ float4 operator()(const float4 &mine) {
    float4 *p = part[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = mine;
    __syncthreads();
    const int w = threadIdx.x & 15;
    return w < (int)(blockDim.x >> 6) ? p[w] : make_float4(0.f, 0.f, 0.f, 0.f);
  }
};

template <class F>
__device__ __forceinline__ void each_unit(int units, F &&f) {
#pragma unroll 2
  for (int u = threadIdx.x; u < units; u += blockDim.x) f(u);
}

// Mean (0 without centring) and squares about it of the wave's elements of a row in LDS; sum = its elements' sum over this lane.
__device__ __forceinline__ float2 wide_stat(const float *row, int width, int units, float inverse, float sum, float squares, bool layer) {
  if (!layer) return make_float2(0.f, wave_sum(squares));
  const float m = wave_sum(sum) * inverse;
  float s = 0.f;
  each_unit(units, [&](int u) {
    float x[8];
    get8(row, u, x);
    const int n = count_of(width, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = j < n ? x[j] - m : 0.f;
      s = __builtin_fmaf(d, d, s);
    }
  });
  return make_float2(m, wave_sum(s));
}

template <class E>
__device__ __forceinline__ void vector8(const void *v, int unit, int width, float none, float (&f)[8]) {
  if (v) {
    Piece<E> p;
    p.load(v, unit, width);
    p.get(f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 8 * unit + j < width ? none : 0.f;
  }
}

template <class E, class H, bool POST>
__global__ __launch_bounds__(512) void owq_norm_wide_kernel(NormArgs a) {
  __shared__ float4 part[2][kNormWaves];
  __shared__ __attribute__((aligned(16))) float row[OWQ_NORM_MAX_WIDTH];
  const int units = (a.width + 7) >> 3;
  const float inverse = 1.f / fmaxf((float)wave_elements(a.width, threadIdx.x >> 6), 1.f), inverse_width = 1.f / (float)a.width;
  WideJoin join{part, 0, (threadIdx.x & 15) < (blockDim.x >> 6) ? (float)wave_elements(a.width, threadIdx.x & 15) : 0.f};
  const DropKey key = drop_key(a.drop);
  const bool layer = a.norm == OWQ_NORM_LAYER, post_layer = a.post == OWQ_NORM_LAYER;
  for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    const void *h = row_at<H>(a.h, t, a.h_row), *o = a.branch ? row_at<E>(a.branch, t, a.branch_row) : nullptr;
    const void *gate = a.gate ? row_at<E>(a.gate, t, a.gate_row) : nullptr;
    RowStat post = {0.f, 1.f};
    if (POST) {
      float sum = 0.f, squares = 0.f;
      each_unit(units, [&](int u) {
        float x[8];
        vector8<E>(o, u, a.width, 0.f, x);
        put8(row, u, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j], squares = __builtin_fmaf(x[j], x[j], squares);
      });
      const float2 s = wide_stat(row, a.width, units, inverse, sum, squares, post_layer);
      const float4 p = join(make_float4(s.x, s.y, 0.f, 0.f));
      post = joined_stat(make_float2(p.x, p.y), join, inverse_width, post_layer, a.eps);
    }
    float sum = 0.f, squares = 0.f;
    void *total = a.total_out ? row_at<H>(a.total_out, t, a.width) : nullptr;
    each_unit(units, [&](int u) {
      Piece<H> ph;
      ph.load(h, u, a.width);
      float x[8], g[8], k[8], f[8];
      vector8<E>(gate, u, a.width, 1.f, g);
      if (POST) {
        vector8<E>(a.post_w, u, a.width, 1.f, k);
        vector8<E>(a.post_b, u, a.width, 0.f, f);
        get8(row, u, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf((x[j] - post.mean) * post.size, k[j], f[j]);
      } else {
        vector8<E>(o, u, a.width, 0.f, x);
      }
      if (a.drop.threshold > 0) {
        const Stays on(a.drop, key, (u32)u, (u32)t);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = on(j) ? x[j] * a.drop.scale : 0.f;
      }
      ph.get(f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = __builtin_fmaf(a.h_scale, f[j], a.branch_scale * (x[j] * g[j]));
        sum += x[j];
        squares = __builtin_fmaf(x[j], x[j], squares);
      }
      put8(row, u, x);
      if (total) {
        Piece<H> p;
        p.put(x);
        p.template store<true>(total, u, a.width);
      }
    });
    if (!a.y) continue;
    const float2 s = wide_stat(row, a.width, units, inverse, sum, squares, layer);
    const float4 p = join(make_float4(s.x, s.y, 0.f, 0.f));
    const RowStat norm = joined_stat(make_float2(p.x, p.y), join, inverse_width, layer, a.eps);
    void *y = row_at<E>(a.y, t, a.width);
    each_unit(units, [&](int u) {
      float x[8], k[8], f[8];
      vector8<E>(a.w, u, a.width, 1.f, k);
      vector8<E>(a.b, u, a.width, 0.f, f);
      get8(row, u, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf((x[j] - norm.mean) * norm.size, k[j], f[j]);
      Piece<E> p;
      p.put(x);
      p.template store<true>(y, u, a.width);
    });
  }
}

// Gradients.  x (the total, then the branch) and what the branch's side starts from lie in LDS; dy and the vectors are read again
// from the caches.  Sums over tokens are kept in the workgroup's row of the workspace, a thread's columns its own.
template <class E, class H, bool POST, bool GATED>
__global__ __launch_bounds__(1024) void owq_norm_backward_wide_kernel(NormArgs a) {
  __shared__ float4 part[2][kNormWaves];
  __shared__ __attribute__((aligned(16))) float xs[OWQ_NORM_MAX_WIDTH];
  __shared__ __attribute__((aligned(16))) float ns[POST ? OWQ_NORM_MAX_WIDTH : 4];
  __shared__ uint8_t keeps[POST && GATED ? OWQ_NORM_MAX_WIDTH / 8 : 4];
  const int units = (a.width + 7) >> 3;
  const float inverse = 1.f / fmaxf((float)wave_elements(a.width, threadIdx.x >> 6), 1.f), inverse_width = 1.f / (float)a.width;
  WideJoin join{part, 0, (threadIdx.x & 15) < (blockDim.x >> 6) ? (float)wave_elements(a.width, threadIdx.x & 15) : 0.f};
  const DropKey key = drop_key(a.drop);
  const bool layer = a.norm == OWQ_NORM_LAYER, post_layer = a.post == OWQ_NORM_LAYER;
  float *mine = a.partial ? a.partial + (int64_t)blockIdx.x * a.n_sums * a.pitch : nullptr;
  auto where = [&](int k) { return k >= 0 && mine ? mine + k * a.pitch : nullptr; };
  float *sum_w = where(a.sum_w), *sum_b = where(a.sum_b), *sum_pw = where(a.sum_post_w), *sum_pb = where(a.sum_post_b), *sum_g = where(a.sum_gate);
  for (int k = 0; k < a.n_sums && mine; ++k)
    each_unit(units, [&](int u) {
      const float zero[8] = {};
      put8(mine + k * a.pitch, u, zero);
    });
  auto add = [](float *to, int u, const float (&v)[8]) {
    if (!to) return;
    float x[8];
    get8(to, u, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += v[j];
    put8(to, u, x);
  };
  const float scale = a.branch_scale * a.drop.scale;
  for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    const void *dy = a.dy ? row_at<E>(a.dy, t, a.dy_row) : nullptr, *dtotal = a.dtotal ? row_at<H>(a.dtotal, t, a.dtotal_row) : nullptr;
    const void *branch = a.branch ? row_at<E>(a.branch, t, a.branch_row) : nullptr, *gate = GATED ? row_at<E>(a.gate, t, a.gate_row) : nullptr;
    // q(u) = gradient of a norm's output times its weight; the sums of one row about the wave's mean
    auto sums = [&](float sum, float squares, float qx, float qs, bool centred, auto &&q_of) {
      float2 s = make_float2(0.f, squares);
      if (centred) {
        const float m = wave_sum(sum) * inverse;
        s = make_float2(m, 0.f);
        qx = 0.f;
        each_unit(units, [&](int u) {
          float x[8], q[8];
          get8(xs, u, x);
          q_of(u, q);
          const int n = count_of(a.width, u);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float d = j < n ? x[j] - m : 0.f;
            s.y = __builtin_fmaf(d, d, s.y);
            qx = __builtin_fmaf(q[j], d, qx);
          }
        });
        qs = wave_sum(qs);
      }
      return join(make_float4(s.x, wave_sum(s.y), wave_sum(qx), qs));
    };
    BackStat s = {0.f, 1.f, 0.f, 0.f};
    if (a.dy) {
      const void *total = row_at<H>(a.total, t, a.total_row);
      auto q_of = [&](int u, float (&q)[8]) {
        float k[8];
        vector8<E>(dy, u, a.width, 0.f, q);
        vector8<E>(a.w, u, a.width, 1.f, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] *= k[j];
      };
      float sum = 0.f, squares = 0.f, qx = 0.f, qs = 0.f;
      each_unit(units, [&](int u) {
        float x[8], q[8];
        vector8<H>(total, u, a.width, 0.f, x);
        q_of(u, q);
        put8(xs, u, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum += x[j];
          squares = __builtin_fmaf(x[j], x[j], squares);
          qx = __builtin_fmaf(q[j], x[j], qx);
          qs += q[j];
        }
      });
      s = joined_back(sums(sum, squares, qx, qs, layer, q_of), join, inverse_width, layer, a.eps);
    }
    // gate and dropping, from e = branch_scale D / the share that stays
    auto side = [&](int u, u32 keep, const float (&n)[8], float (&v)[8]) {
      float g[8];
      if (GATED) vector8<E>(gate, u, a.width, 0.f, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (keep >> j) & 1u ? (GATED ? n[j] * g[j] : n[j]) : 0.f;
    };
    float sum = 0.f, squares = 0.f, qx = 0.f, qs = 0.f;
    each_unit(units, [&](int u) {
      float d[8], x[8], k[8];
      vector8<H>(dtotal, u, a.width, 0.f, d);
      if (a.dy) {
        float y[8];
        vector8<E>(dy, u, a.width, 0.f, y);
        vector8<E>(a.w, u, a.width, 1.f, k);
        get8(xs, u, x);
        add(sum_b, u, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = (x[j] - s.mean) * s.size;
          d[j] = __builtin_fmaf(s.size, y[j] * k[j], d[j]) + __builtin_fmaf(s.along, x[j], s.all);
          y[j] *= x[j];
        }
        add(sum_w, u, y);
      }
      if (a.dh) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = a.h_scale * d[j];
        Piece<H> p;
        p.put(x);
        p.template store<true>(row_at<H>(a.dh, t, a.width), u, a.width);
      }
      if (!a.branch_side) return;
      u32 keep = 255u;
      if (a.drop.threshold > 0) {
        const Stays on(a.drop, key, (u32)u, (u32)t);
        keep = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) keep |= on(j) ? 1u << j : 0u;
      }
      // past the row the norm's means still stand in d
      const int count = count_of(a.width, u);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = j < count ? scale * d[j] : 0.f;
      side(u, keep, d, v);
      if (POST) {
        if (!GATED) {
          put8(ns, u, v);
        } else {
          put8(ns, u, d);
          keeps[u] = (uint8_t)keep;
        }
        add(sum_pb, u, v);
        vector8<E>(branch, u, a.width, 0.f, x);
        vector8<E>(a.post_w, u, a.width, 1.f, k);
        put8(xs, u, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float q = v[j] * k[j];
          sum += x[j];
          squares = __builtin_fmaf(x[j], x[j], squares);
          qx = __builtin_fmaf(q, x[j], qx);
          qs += q;
        }
        return;
      }
      if (GATED) {
        vector8<E>(branch, u, a.width, 0.f, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (keep >> j) & 1u ? d[j] * x[j] : 0.f;
        add(sum_g, u, x);
        if (a.dgate) {
          Piece<E> p;
          p.put(x);
          p.template store<true>(row_at<E>(a.dgate, t, a.width), u, a.width);
        }
      }
      if (a.dbranch) {
        Piece<E> p;
        p.put(v);
        p.template store<true>(row_at<E>(a.dbranch, t, a.width), u, a.width);
      }
    });
    if (!POST) continue;
    auto v_of = [&](int u, float (&n)[8], u32 &keep, float (&v)[8]) {
      get8(ns, u, n);
      keep = 255u;
      if (GATED) {
        keep = keeps[u];
        side(u, keep, n, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = n[j];
      }
    };
    const float4 joined = sums(sum, squares, qx, qs, post_layer, [&](int u, float (&q)[8]) {
      float n[8], k[8];
      u32 keep;
      v_of(u, n, keep, q);
      vector8<E>(a.post_w, u, a.width, 1.f, k);
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] *= k[j];
    });
    s = joined_back(joined, join, inverse_width, post_layer, a.eps);
    each_unit(units, [&](int u) {
      float x[8], n[8], v[8], k[8], f[8];
      u32 keep;
      v_of(u, n, keep, v);
      vector8<E>(a.post_w, u, a.width, 1.f, k);
      get8(xs, u, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (x[j] - s.mean) * s.size;
      if (GATED) {
        vector8<E>(a.post_b, u, a.width, 0.f, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (keep >> j) & 1u ? n[j] * __builtin_fmaf(x[j], k[j], f[j]) : 0.f;
        add(sum_g, u, f);
        if (a.dgate) {
          Piece<E> p;
          p.put(f);
          p.template store<true>(row_at<E>(a.dgate, t, a.width), u, a.width);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = v[j] * x[j];
        v[j] = __builtin_fmaf(s.size, v[j] * k[j], __builtin_fmaf(s.along, x[j], s.all));
      }
      add(sum_pw, u, f);
      if (a.dbranch) {
        Piece<E> p;
        p.put(v);
        p.template store<true>(row_at<E>(a.dbranch, t, a.width), u, a.width);
      }
    });
  }
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

int launch_norm_wide(const NormArgs &a, int32_t type, int32_t h_type, void *stream) {
  const unsigned grid = (unsigned)(a.n_tokens < 512 ? a.n_tokens : 512);      // two a compute unit; with a norm of the branch the second waits for the first (registers)
  const hipStream_t s = static_cast<hipStream_t>(stream);
  for_types(type, h_type, [&](auto e, auto h) {
    if (a.post != OWQ_NORM_NONE) owq_norm_wide_kernel<decltype(e), decltype(h), true><<<grid, 512, 0, s>>>(a);
    else owq_norm_wide_kernel<decltype(e), decltype(h), false><<<grid, 512, 0, s>>>(a);
  });
  return (int)hipGetLastError();
}

void launch_norm_backward_wide(const NormArgs &a, int32_t type, int32_t h_type, int32_t blocks, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool post = a.post != OWQ_NORM_NONE && a.branch_side, gated = a.gate != nullptr && a.branch_side;
  for_types(type, h_type, [&](auto e, auto h) {
    using E = decltype(e);
    using H = decltype(h);
    if (post && gated) owq_norm_backward_wide_kernel<E, H, true, true><<<blocks, 1024, 0, s>>>(a);
    else if (post) owq_norm_backward_wide_kernel<E, H, true, false><<<blocks, 1024, 0, s>>>(a);
    else if (gated) owq_norm_backward_wide_kernel<E, H, false, true><<<blocks, 1024, 0, s>>>(a);
    else owq_norm_backward_wide_kernel<E, H, false, false><<<blocks, 1024, 0, s>>>(a);
  });
}

}  // namespace owq
