// Norm of every query and key head and the position rotation in one pass, and its gradients.
//
// A row (one head of one token) is cut into units of 16 elements that hold both partners of their
// eight pairs: pieces [8u, 8u + 8) and [R/2 + 8u, R/2 + 8u + 8) of the rotated part, or 16 elements
// in a row where neighbours are paired; what is not rotated follows in units of 16.  A lane takes a
// unit, L = 2^n >= units neighbouring lanes take a row: the rotation needs no exchange between
// lanes, the norm a sum over L <= 16 of them.  A thread keeps the cosines and sines of its unit
// (the same for all heads of a token) and walks down the heads.
//
// Bound by memory: 4096 tokens of 32 + 8 heads of 128 in 21.1 us, 86 MB at 4.1 TB/s (a copy of 1 GiB runs at 4.77);
// the gradients of 2048 tokens of 72 + 72 heads in 52.4 us, 4.3 TB/s, 6 of them for the weights' (sums left by every workgroup
// and their launch).  1021 tokens of 32 + 32 heads of 80 take 21.1 us, where the bytes take 6.6: 14.8 in the kernel, 9.6 where
// a workgroup, which has but one token, need not leave sums for the weights, and 3.9 in the second launch.  A single token is
// bound by its call (10.4 us, of them 2.8 in the kernel).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

struct RopeUnit {
  int off0, off1;        // first elements of the two pieces
  bool on, second, turned;
  int pair;              // first pair, for the tables
};

template <bool INTER>
__device__ __forceinline__ RopeUnit rope_unit(int u, int dim, int rot) {
  RopeUnit r;
  const int pairs = rot >> 4, tail = u - pairs;
  r.turned = u < pairs;
  r.off0 = r.turned ? (INTER ? 16 * u : 8 * u) : rot + 16 * tail;
  r.off1 = r.turned ? (INTER ? 16 * u + 8 : 8 * u + (rot >> 1)) : rot + 16 * tail + 8;
  r.on = r.off0 < dim;
  r.second = r.off1 < dim;
  r.pair = 8 * u;
  return r;
}

// y = R x (sign = 1) or its transpose (sign = -1) on the eight pairs of a unit
template <bool INTER>
__device__ __forceinline__ void rope_turn(float *f, const float *c, const float *s, float sign) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int a = INTER ? 2 * j : j, b = INTER ? 2 * j + 1 : j + 8;
    const float x = f[a], y = f[b], n = sign * s[j];
    f[a] = x * c[j] - y * n;
    f[b] = y * c[j] + x * n;
  }
}

template <class E>
__device__ __forceinline__ void load_unit(const u32 *row, const RopeUnit &r, float *f) {
  const u32x4 zero = {0, 0, 0, 0};
  const u32x4 a = r.on ? *reinterpret_cast<const u32x4 *>(row + (r.off0 >> 1)) : zero;
  const u32x4 b = r.second ? *reinterpret_cast<const u32x4 *>(row + (r.off1 >> 1)) : zero;
  unpack8<E>(a, f);
  unpack8<E>(b, f + 8);
}

// Results are not read again by this call: stores that leave the caches alone (4096 tokens of 40 heads: 20.9 us, 22.1 without).
template <class E>
__device__ __forceinline__ void store_unit(u32 *row, const RopeUnit &r, const float *f) {
  if (r.on) __builtin_nontemporal_store(pack8<E>(f), reinterpret_cast<u32x4 *>(row + (r.off0 >> 1)));
  if (r.second) __builtin_nontemporal_store(pack8<E>(f + 8), reinterpret_cast<u32x4 *>(row + (r.off1 >> 1)));
}

__device__ __forceinline__ void load_table(const float *cos, const float *sin, int p, int n_positions, int half_rot, const RopeUnit &r,
                                           float *c, float *s) {
  const bool inside = p >= 0 && p < n_positions;
  const int64_t at = (int64_t)(inside ? p : 0) * half_rot + r.pair;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float nan = __builtin_nanf("");
    c[j] = r.turned ? (inside ? cos[at + j] : nan) : 1.f;
    s[j] = r.turned ? (inside ? sin[at + j] : nan) : 0.f;
  }
}

struct RopeArgs {
  const u32 *q, *k, *wq, *wk;
  const u32 *dq_out, *dk_out;
  u32 *q_out, *k_out;
  const float *cos, *sin;
  const int32_t *positions;
  float *partial;
  int64_t q_token, q_head, k_token, k_head, dq_token, dq_head, dk_token, dk_head;
  int32_t n_tokens, q_heads, kv_heads, dim, rot, n_positions;
  float eps;
};

// One workgroup per (token, range of heads): heads slot, slot + slots, ... of its range.
template <class E, bool INTER, int L>
__global__ __launch_bounds__(256) void owq_rope_kernel(RopeArgs a) {
  const int slots = blockDim.x / L;
  const int slot = threadIdx.x / L;
  const RopeUnit r = rope_unit<INTER>(threadIdx.x % L, a.dim, a.rot);
  const int64_t t = blockIdx.x;
  float c[8], s[8];
  load_table(a.cos, a.sin, a.positions[t], a.n_positions, a.rot >> 1, r, c, s);
  const int heads = a.q_heads + a.kv_heads;
  for (int h = slot + (int)blockIdx.y * slots; h < heads; h += slots * (int)gridDim.y) {
    const bool is_k = h >= a.q_heads;
    const int hh = is_k ? h - a.q_heads : h;
    const u32 *row = is_k ? a.k + (t * a.k_token + hh * a.k_head) / 2 : a.q + (t * a.q_token + hh * a.q_head) / 2;
    const u32 *w = is_k ? a.wk : a.wq;
    float f[16];
    load_unit<E>(row, r, f);
    if (w != nullptr) {
      float g[16], sq = 0.f;
      load_unit<E>(w, r, g);
#pragma unroll
      for (int j = 0; j < 16; ++j) sq += f[j] * f[j];
      const float rs = 1.f / __builtin_sqrtf(lanes_sum<L>(sq) / (float)a.dim + a.eps);
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] = f[j] * rs * g[j];
    }
    if (r.turned) rope_turn<INTER>(f, c, s, 1.f);
    u32 *out = is_k ? a.k_out + (t * a.kv_heads + hh) * (a.dim / 2) : a.q_out + (t * a.q_heads + hh) * (a.dim / 2);
    store_unit<E>(out, r, f);
  }
}

// Gradients: a workgroup takes tokens blockIdx.x, + gridDim.x, ..., all heads, and leaves one row of
// sums for the weights (2 head_dim values) that owq_rope_weights_kernel adds up in order.
template <class E, bool INTER, int L>
__global__ __launch_bounds__(256) void owq_rope_backward_kernel(RopeArgs a) {
  __shared__ float sums[4][2][256];
  const int slots = blockDim.x / L;
  const int slot = threadIdx.x / L;
  const RopeUnit r = rope_unit<INTER>(threadIdx.x % L, a.dim, a.rot);
  float dw[2][16];
#pragma unroll
  for (int j = 0; j < 16; ++j) dw[0][j] = dw[1][j] = 0.f;
  for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    float c[8], s[8];
    bool tables = false;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const u32 *w = part ? a.wk : a.wq;
      const u32 *x = part ? a.k + t * a.k_token / 2 : a.q + t * a.q_token / 2;
      const u32 *dy = part ? a.dk_out + t * a.dk_token / 2 : a.dq_out + t * a.dq_token / 2;
      const int64_t xs = part ? a.k_head : a.q_head, ds = part ? a.dk_head : a.dq_head;
      const int heads = part ? a.kv_heads : a.q_heads;
      u32 *out = part ? a.k_out + t * heads * (a.dim / 2) : a.q_out + t * heads * (a.dim / 2);
      float g[16];
      for (int h = slot; h < heads; h += slots) {
        float d[16], f[16];
        load_unit<E>(dy + h * ds / 2, r, d);
        if (w != nullptr) load_unit<E>(x + h * xs / 2, r, f);
        // behind the first rows, which do not wait for the position
        if (h == slot && w != nullptr) load_unit<E>(w, r, g);
        if (!tables) load_table(a.cos, a.sin, a.positions[t], a.n_positions, a.rot >> 1, r, c, s);
        tables = true;
        if (w != nullptr) {
          float sq = 0.f, hx = 0.f;
          if (r.turned) rope_turn<INTER>(d, c, s, -1.f);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            sq += f[j] * f[j];
            hx += d[j] * g[j] * f[j];
          }
          const float rs = 1.f / __builtin_sqrtf(lanes_sum<L>(sq) / (float)a.dim + a.eps);
          const float mean = lanes_sum<L>(hx) / (float)a.dim * rs * rs;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            dw[part][j] += d[j] * f[j] * rs;
            d[j] = rs * (d[j] * g[j] - f[j] * mean);
          }
        } else if (r.turned) {
          rope_turn<INTER>(d, c, s, -1.f);
        }
        store_unit<E>(out + h * (a.dim / 2), r, d);
      }
    }
  }
  if (a.partial == nullptr) return;
  // rows of a wave: lanes that hold the same unit, L apart
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      float v = dw[part][j];
#pragma unroll
      for (int step = L; step < 64; step *= 2) v += __shfl_xor(v, step);
      dw[part][j] = v;
    }
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < L && r.on) {
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (j < 8 || r.second) sums[wave][part][j < 8 ? r.off0 + j : r.off1 + j - 8] = dw[part][j];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += blockDim.x) {
    const int part = i >= a.dim, e = part ? i - a.dim : i;
    float v = 0.f;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) v += sums[w][part][e];
    a.partial[(int64_t)blockIdx.x * 2 * a.dim + i] = v;
  }
}

// Column sums of partial [rows][2 dim]: 8 columns per workgroup, 128 rows at a time, eight of a thread's in flight.
__global__ __launch_bounds__(1024) void owq_rope_weights_kernel(const float *partial, int rows, int dim, float *dwq, float *dwk) {
  __shared__ float sums[128][9];
  const int lane = threadIdx.x & 7, first = threadIdx.x >> 3;
  const int col = blockIdx.x * 8 + lane;
  float v = 0.f;
  if (rows > 0)
    for (int base = 0; base < rows; base += 1024) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = base + 128 * j + first;
        x[j] = partial[(int64_t)(i < rows ? i : rows - 1) * 2 * dim + col];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v += base + 128 * j + first < rows ? x[j] : 0.f;
    }
  sums[first][lane] = v;
  __syncthreads();
  if (threadIdx.x < 64) {            // eight threads a column, 16 rows each
    const int c = threadIdx.x >> 3, part = threadIdx.x & 7;
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) total += sums[16 * part + i][c];
    total = lanes_sum<8>(total);
    const int at = blockIdx.x * 8 + c;
    float *out = at < dim ? dwq : dwk;
    if (part == 0 && out != nullptr) out[at < dim ? at : at - dim] = total;
  }
}

static RopeArgs rope_args(const owq_rope_desc_t &d, const RopePtrs &p) {
  RopeArgs a;
  a.q = static_cast<const u32 *>(p.q);
  a.k = static_cast<const u32 *>(p.k);
  a.wq = static_cast<const u32 *>(p.wq);
  a.wk = static_cast<const u32 *>(p.wk);
  a.dq_out = static_cast<const u32 *>(p.dq_out);
  a.dk_out = static_cast<const u32 *>(p.dk_out);
  a.q_out = static_cast<u32 *>(p.q_out);
  a.k_out = static_cast<u32 *>(p.k_out);
  a.cos = p.cos;
  a.sin = p.sin;
  a.positions = p.positions;
  a.partial = p.partial;
  a.q_token = d.q_token, a.q_head = d.q_head, a.k_token = d.k_token, a.k_head = d.k_head;
  a.dq_token = d.dq_token, a.dq_head = d.dq_head, a.dk_token = d.dk_token, a.dk_head = d.dk_head;
  a.n_tokens = d.n_tokens, a.q_heads = d.q_heads, a.kv_heads = d.kv_heads, a.dim = d.head_dim, a.rot = d.rotary_dim;
  a.n_positions = d.n_positions;
  a.eps = d.eps;
  return a;
}

// Lanes per row: the units of 16 elements, rounded up to a power of two (at most 16 for 256 elements).
static int rope_lanes(const owq_rope_desc_t &d) {
  const int units = d.rotary_dim / 16 + (d.head_dim - d.rotary_dim + 15) / 16;
  int lanes = 1;
  while (lanes < units) lanes *= 2;
  return lanes;
}

// Threads of a workgroup: whole waves for the heads of one token, 256 at most.
static int rope_threads(const owq_rope_desc_t &d, int lanes) {
  const int64_t n = ((int64_t)(d.q_heads + d.kv_heads) * lanes + 63) / 64 * 64;
  return n > 256 ? 256 : (int)n;
}

template <class F>
static void for_lanes(int lanes, F &&f) {
  switch (lanes) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    default: f(std::integral_constant<int, 16>()); break;
  }
}

template <class F>
static void for_kinds(int type, bool inter, F &&f) {
  if (type == OWQ_TYPE_F16) {
    if (inter) f(F16(), std::true_type());
    else f(F16(), std::false_type());
  } else {
    if (inter) f(BF16(), std::true_type());
    else f(BF16(), std::false_type());
  }
}

int launch_rope(const owq_rope_desc_t &d, const RopePtrs &p, void *stream) {
  const RopeArgs a = rope_args(d, p);
  const int lanes = rope_lanes(d), threads = rope_threads(d, lanes);
  const int slots = threads / lanes, heads = d.q_heads + d.kv_heads;
  // a thread takes one head where there are few tokens, all of its token's where there are many
  int ranges = (heads + slots - 1) / slots;
  while (ranges > 1 && (int64_t)d.n_tokens * (ranges / 2) >= 2048) ranges /= 2;
  const dim3 grid((unsigned)d.n_tokens, (unsigned)ranges);
  for_kinds(d.type, d.interleaved != 0, [&](auto e, auto inter) {
    for_lanes(lanes, [&](auto l) {
      owq_rope_kernel<decltype(e), decltype(inter)::value, decltype(l)::value><<<grid, threads, 0, static_cast<hipStream_t>(stream)>>>(a);
    });
  });
  return (int)hipGetLastError();
}

// The backward's workgroup: one to four waves, as many as leave the fewest idle lanes in the last round of heads.
static int rope_backward_threads(const owq_rope_desc_t &d, int lanes) {
  int best = 64;
  int64_t least = INT64_MAX;
  for (int threads = 64; threads <= 256; threads += 64) {
    const int slots = threads / lanes;
    const int64_t padded = ((int64_t)(d.q_heads + slots - 1) / slots + (d.kv_heads + slots - 1) / slots) * slots;
    if (padded <= least) {
      least = padded;
      best = threads;
    }
  }
  return best;
}

// 4096 waves at most (156 registers leave room for three per SIMD, 3072), and the same number of tokens for each workgroup, which
// has sums to leave.  2048 tokens of 144 heads, timed in turn on one set of tensors: 43.8 us with 1024 workgroups of two tokens and
// three waves, as here; 47.6 with 683 of three tokens, 47.6 with 512 of four, 50.0 with 2048 of one.
int32_t rope_backward_blocks(const owq_rope_desc_t &d) {
  const int64_t most = 4096 / (rope_backward_threads(d, rope_lanes(d)) / 64);
  const int64_t each = (d.n_tokens + most - 1) / most;       // tokens of a workgroup, the same for all but the last
  return each == 0 ? 0 : (int32_t)((d.n_tokens + each - 1) / each);
}

int launch_rope_backward(const owq_rope_desc_t &d, const RopePtrs &p, void *stream) {
  const RopeArgs a = rope_args(d, p);
  const int lanes = rope_lanes(d), threads = rope_backward_threads(d, lanes);
  const int blocks = rope_backward_blocks(d);
  if (blocks > 0) for_kinds(d.type, d.interleaved != 0, [&](auto e, auto inter) {
    for_lanes(lanes, [&](auto l) {
      owq_rope_backward_kernel<decltype(e), decltype(inter)::value, decltype(l)::value>
          <<<blocks, threads, 0, static_cast<hipStream_t>(stream)>>>(a);
    });
  });
  if (p.dwq != nullptr || p.dwk != nullptr)      // no tokens: zeros
    owq_rope_weights_kernel<<<2 * d.head_dim / 8, 1024, 0, static_cast<hipStream_t>(stream)>>>(a.partial, blocks, d.head_dim, p.dwq, p.dwk);
  return (int)hipGetLastError();
}

}  // namespace owq
