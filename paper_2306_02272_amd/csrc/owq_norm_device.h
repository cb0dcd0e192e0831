// Statistics of a row over a team of waves, and pieces of a row in registers: shared by the kernels of owq_norm.hip and owq_norm_wide.hip.
#pragma once
#include "owq_random_device.h"

namespace owq {

constexpr int kNormWaves = 16;      // of a workgroup

// Where a thread's pieces lie: team `team` of the workgroup, `threads` threads and `waves` waves each.
template <int CH>
struct RowPlace {
  int team, threads, waves, wave;
  int unit[CH], count[CH];      // pieces of this thread and how many of their elements the row has
  float inverse, join;          // 1 / elements of this wave; elements of wave (lane % 16) of the team
  __device__ __forceinline__ static int elements(int width, int threads, int w) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int k = width - 8 * (c * threads + 64 * w);
      n += k < 0 ? 0 : k > 512 ? 512 : k;
    }
    return n;
  }
  __device__ __forceinline__ RowPlace(int width, int team_threads, bool alone) : threads(team_threads), waves(team_threads >> 6) {
    team = alone ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / threads);      // whole waves
    const int i = (int)threadIdx.x - team * threads;
    wave = __builtin_amdgcn_readfirstlane(i >> 6);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      unit[c] = c * threads + i;
      const int n = width - 8 * unit[c];
      count[c] = n < 0 ? 0 : n > 8 ? 8 : n;
    }
    inverse = 1.f / fmaxf((float)elements(width, threads, wave), 1.f);
    const int w = threadIdx.x & 15;
    join = w < waves ? (float)elements(width, threads, w) : 0.f;
  }
};

// Sums over a team: every wave leaves its own in LDS.  Two sets in turn: who writes one has passed a barrier since it was read.
template <class T>
struct TeamSum {
  T *part;      // [2][kNormWaves]
  int turn;
  // g(sum over waves) of each of lane % 16's wave
  template <int CH>
  __device__ __forceinline__ T join(const RowPlace<CH> &at, const T &mine, const T &none) {
    T *p = part + turn * kNormWaves + at.team * at.waves;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) p[at.wave] = mine;
    __syncthreads();
    const int w = threadIdx.x & 15;
    return w < at.waves ? p[w] : none;
  }
};

struct RowStat {
  float mean, size;      // size = 1 / sqrt(mean square + eps)
};

// What a wave knows of a row: mean and sum of squares about it.
template <int CH>
__device__ __forceinline__ float2 wave_stat(const float (&x)[CH][8], const RowPlace<CH> &at, int width, bool layer) {
  float m = 0.f;
  if (layer) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) m += x[c][j];            // 0 past the row
    m = wave_sum(m) * at.inverse;
  }
  float s = 0.f;
  if (!layer) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) s = __builtin_fmaf(x[c][j], x[c][j], s);
  } else if ((width & 7) == 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const float mc = at.count[c] > 0 ? m : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s = __builtin_fmaf(x[c][j] - mc, x[c][j] - mc, s);
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = j < at.count[c] ? x[c][j] - m : 0.f;
        s = __builtin_fmaf(d, d, s);
      }
  }
  return make_float2(m, wave_sum(s));
}

// Joins lane % 16's wave's with the others'.
template <class At>
__device__ __forceinline__ RowStat joined_stat(float2 p, const At &at, float inverse_width, bool layer, float eps) {
  float mean = 0.f, extra = 0.f;
  if (layer) {
    mean = lanes_sum<16>(rounded(at.join * p.x)) * inverse_width;
    extra = at.join * (p.x - mean) * (p.x - mean);
  }
  return RowStat{mean, 1.f / __builtin_sqrtf(lanes_sum<16>(p.y + extra) * inverse_width + eps)};
}

// What is unpacked after this is unpacked again: between the passes over a row its pieces lie packed, not as the floats that the
// compiler would keep.  For rows whose floats the registers do not hold.
template <bool AGAIN>
__device__ __forceinline__ void again(u32x4 &v) {
  if (AGAIN) asm("" : "+v"(v));
}
template <bool AGAIN, class E>
__device__ __forceinline__ void again(Piece<E> &p) { again<AGAIN>(p.v); }
template <bool AGAIN>
__device__ __forceinline__ void again(Piece<F32> &p) {
  again<AGAIN>(p.v[0]);
  again<AGAIN>(p.v[1]);
}

template <class E, int CH>
__device__ __forceinline__ void load_row(Piece<E> (&p)[CH], const void *row, const RowPlace<CH> &at, int width) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (row) p[c].load(row, at.unit[c], width);
    else p[c].zero();
  }
}
// The next row's loads are waited for here, ahead of the first store of this row: later their wait would be one for the stores
// behind them too, as the counter of both goes down in order.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// A piece of a vector that all rows share; `none` where there is none.
template <class E>
__device__ __forceinline__ void load_shared(Piece<E> &p, const void *v, float none, int unit, int count, int width) {
  if (v) {
    p.load(v, unit, width);
  } else {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < count ? none : 0.f;
    p.put(f);
  }
}
template <class E, int CH>
__device__ __forceinline__ void load_vector(Piece<E> (&p)[CH], const void *v, float none, const RowPlace<CH> &at, int width) {
#pragma unroll
  for (int c = 0; c < CH; ++c) load_shared<E>(p[c], v, none, at.unit[c], at.count[c], width);
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

template <class E, int CH>
__device__ __forceinline__ void apply_norm(float (&x)[CH][8], const RowStat &s, const Piece<E> (&w)[CH], const Piece<E> (&b)[CH]) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float g[8], k[8];
    w[c].get(g);
    b[c].get(k);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[c][j] = __builtin_fmaf((x[c][j] - s.mean) * s.size, g[j], k[j]);
  }
}

// Piece `unit` of a row of floats in LDS or in the workspace.
__device__ __forceinline__ void put8(float *row, int unit, const float (&x)[8]) {
  f32x4 *p = reinterpret_cast<f32x4 *>(row) + 2 * unit;
  p[0] = (f32x4){x[0], x[1], x[2], x[3]};
  p[1] = (f32x4){x[4], x[5], x[6], x[7]};
}

// size, and the gradient as size q + along n + all
struct BackStat {
  float mean, size, along, all;
};
template <class At>
__device__ __forceinline__ BackStat joined_back(float4 p, const At &at, float inverse_width, bool layer, float eps) {
  const RowStat s = joined_stat(make_float2(p.x, p.y), at, inverse_width, layer, eps);
  float qx = p.z, all = 0.f;
  if (layer) {
    qx += (p.x - s.mean) * p.w;
    all = -lanes_sum<16>(p.w) * inverse_width * s.size;
  }
  return BackStat{s.mean, s.size, -lanes_sum<16>(qx) * inverse_width * s.size * s.size, all};
}

}  // namespace owq
