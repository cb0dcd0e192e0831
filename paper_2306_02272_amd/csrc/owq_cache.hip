// The cache of keys and values in 4 bits: new rows into it, and its contents back as fp16 or bf16.
// Layout and rounding: include/owq.h.
//
// A workgroup takes 32 tokens of one head (a tile).  Codes go through LDS as bytes [token][column]:
// rows of the cache's matrix-core words are gathered there (keys: 8 columns of a token, values: 8
// tokens of a column), so that both sides of the exchange are whole 16- and 8-byte accesses.
//
// Four prompts of 7269 tokens together, 40 heads of 128 (148 MB of fp16, 188 with the cache's bytes), in 58 us, 3.2 TB/s: a
// workgroup asks for its rows only behind lengths and table, and gathers the values' words by single bytes.  Back in 34 us,
// 5.5 TB/s: bound by memory.  One token each of 64 sequences, where a workgroup writes a 32nd of its tile: 6.7 us, back 7.2, the
// latency of reads that wait for each other (lengths, table, rows or tile).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "owq_cache_device.h"
#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

CacheView cache_view(const owq_cache_desc_t &d, const void *pages, const int32_t *table, const int32_t *starts,
                     const int32_t *lengths, int32_t n_rows) {
  CacheView c;
  c.pages = static_cast<uint8_t *>(const_cast<void *>(pages));
  c.table = table;
  c.starts = starts;
  c.lengths = lengths;
  c.tile_bytes = 32 * ((d.head_dim + 31) / 32 * 32) + 256;
  c.page_bytes = (int64_t)c.tile_bytes * (d.page_size / 32) * d.kv_heads;
  c.n_pages = d.n_pages;
  c.page_shift = 0;
  while ((32 << c.page_shift) < d.page_size) ++c.page_shift;
  c.kv_heads = d.kv_heads;
  c.head_dim = d.head_dim;
  c.table_stride = d.table_stride;
  c.n_seqs = d.n_seqs;
  c.n_rows = n_rows;
  return c;
}

// Codes of a row's 16 columns held by one of its 8 threads.  Returns (s, lo) as an fp16 pair.
template <class E>
__device__ __forceinline__ u32 quantise(u32x4 a, u32x4 b, bool on0, bool on1, u32 *codes) {
  float f[16];
  unpack8<E>(a, f);
  unpack8<E>(b, f + 8);
  float hi = -__builtin_inff(), lo = __builtin_inff(), bad = 0.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const bool on = j < 8 ? on0 : on1;
    hi = on ? fmaxf(hi, f[j]) : hi;
    lo = on ? fminf(lo, f[j]) : lo;
    bad = on && !(__builtin_fabsf(f[j]) < __builtin_inff()) ? 1.f : bad;
  }
  hi = lanes_max<8>(hi);
  lo = -lanes_max<8>(-lo);
  bad = lanes_max<8>(bad);
  const float third = 1.0f / 15.0f;
  const _Float16 s16 = (_Float16)fminf(fmaxf((hi - lo) * third, 0x1p-24f), 65504.f);
  const _Float16 l16 = (_Float16)fminf(fmaxf(lo, -65504.f), 65504.f);
  const float s = (float)s16, l = (float)l16;
  // rint of the rounded quotient, from a product with the reciprocal (1.5 units in the last place off, 3e-6 at 16): the two
  // differ only beside a half, where the division is done (it costs three times the rest of the element)
  const float inv = __builtin_amdgcn_rcpf(s);
  float q[16], beside = 0.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float x = (f[j] - l) * inv;
    q[j] = __builtin_rintf(x);
    beside = fmaxf(beside, __builtin_fabsf(x - q[j]));
  }
  if (beside > 0.4999f) {
#pragma unroll
    for (int j = 0; j < 16; ++j) q[j] = __builtin_rintf((f[j] - l) / s);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32 w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w |= (u32)(int)fminf(fmaxf(q[4 * i + j], 0.f), 15.f) << (8 * j);
    codes[i] = (bad != 0.f || (i < 2 ? !on0 : !on1)) ? 0u : w;
  }
  const h2_t pair = {s16, l16};
  return bad != 0.f ? 0x7e007e00u : __builtin_bit_cast(u32, pair);
}

struct AppendArgs {
  CacheView c;
  const u32 *k, *v;
  int64_t k_row, k_head, v_row, v_head;
  int32_t max_new;
};

constexpr int kCodePitch = 136;   // bytes of a token's codes in LDS: 128 columns, 8-byte units on other banks

template <class E>
__global__ __launch_bounds__(256) void owq_cache_append_kernel(AppendArgs a) {
  __shared__ __align__(16) uint8_t codes[2][32 * kCodePitch];
  const CacheView &c = a.c;
  const int b = blockIdx.z, head = blockIdx.y;
  const int row0 = c.starts[b], n_new = c.starts[b + 1] - row0, len = c.lengths[b];
  const int64_t first = (int64_t)len - n_new;      // position of row 0
  const int from = first < 0 ? 0 : (int)first;     // first position written
  if (n_new <= 0 || len <= from) return;
  const int tile = from / 32 + (int)blockIdx.x;
  const int64_t token0 = (int64_t)tile * 32;
  if (token0 >= len) return;
  int t0 = from > token0 ? (int)(from - token0) : 0;
  int t1 = len - token0 < 32 ? (int)(len - token0) : 32;            // tokens [t0, t1) of the tile are new
  const int64_t row_of_tile = row0 + token0 - first;
  if (first + a.max_new - token0 < t1) t1 = first + a.max_new > token0 ? (int)(first + a.max_new - token0) : 0;   // nor are rows past max_new
  if (row_of_tile + t0 < 0) t0 = row_of_tile > -32 ? (int)-row_of_tile : 32;             // rows outside the caller's tensors are not written
  if (row_of_tile + t1 > c.n_rows) t1 = c.n_rows > row_of_tile ? (int)(c.n_rows - row_of_tile) : 0;
  if (t1 <= t0) return;
  uint8_t *dst = cache_tile(c, b, head, tile);
  if (dst == nullptr) return;
  const int pad = (c.head_dim + 31) / 32 * 32;

  // rows in: thread = (token, 16 columns)
  const int token = threadIdx.x >> 3, col = (threadIdx.x & 7) * 16;
  const int64_t row = row_of_tile + token;
  const bool on = token >= t0 && token < t1;
  const bool on0 = on && col < c.head_dim, on1 = on && col + 8 < c.head_dim;
  const u32x4 zero = {0, 0, 0, 0};
  const u32 *kr = a.k + (row * a.k_row + head * a.k_head + col) / 2, *vr = a.v + (row * a.v_row + head * a.v_head + col) / 2;
  const u32x4 k0 = on0 ? *reinterpret_cast<const u32x4 *>(kr) : zero, k1 = on1 ? *reinterpret_cast<const u32x4 *>(kr + 4) : zero;
  const u32x4 v0 = on0 ? *reinterpret_cast<const u32x4 *>(vr) : zero, v1 = on1 ? *reinterpret_cast<const u32x4 *>(vr + 4) : zero;
  u32 w[4];
  const u32 km = quantise<E>(k0, k1, on0, on1, w);
  if (col < pad) *reinterpret_cast<u32x4 *>(&codes[0][token * kCodePitch + col]) = (u32x4){w[0], w[1], w[2], w[3]};
  const u32 vm = quantise<E>(v0, v1, on0, on1, w);
  if (col < pad) *reinterpret_cast<u32x4 *>(&codes[1][token * kCodePitch + col]) = (u32x4){w[0], w[1], w[2], w[3]};
  if (on && col == 0) {
    u32 *meta = reinterpret_cast<u32 *>(dst + 32 * pad);
    meta[token] = km;
    meta[32 + token] = vm;
  }
  __syncthreads();

  // words out: thread = (32 columns S, quad q, r), two words of keys and two of values
  const int i = threadIdx.x;
  if (i >= 2 * pad) return;
  const int r = i & 15, q = (i >> 4) & 3, S = i >> 6;
  u32 *kw = reinterpret_cast<u32 *>(dst) + 2 * i, *vw = reinterpret_cast<u32 *>(dst + 16 * pad) + 2 * i;
  u32x2 kk, vv;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u32x2 p = *reinterpret_cast<const u32x2 *>(&codes[0][(16 * h + r) * kCodePitch + 32 * S + 8 * q]);
    kk[h] = word_of_bytes(p.x, p.y);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    u32 word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      word |= (u32)codes[1][(16 * (e >> 2) + 4 * q + (e & 3)) * kCodePitch + 32 * S + 16 * j + r] << (4 * ((e >> 1) + 4 * (e & 1)));
    vv[j] = word;
  }
  if (t0 == 0 && t1 == 32) {         // the whole tile is new
    *reinterpret_cast<u32x2 *>(kw) = kk;
    *reinterpret_cast<u32x2 *>(vw) = vv;
    return;
  }
  u32 mask = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = 16 * (e >> 2) + 4 * q + (e & 3);
    mask |= t >= t0 && t < t1 ? 15u << (4 * ((e >> 1) + 4 * (e & 1))) : 0u;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int t = 16 * h + r;
    if (t >= t0 && t < t1) kw[h] = kk[h];
    if (mask != 0) vw[h] = (vw[h] & ~mask) | (vv[h] & mask);
  }
}

struct ReadArgs {
  CacheView c;
  u32 *k_out, *v_out;
  int32_t max_len;
};

template <class E>
__global__ __launch_bounds__(256) void owq_cache_read_kernel(ReadArgs a) {
  __shared__ __align__(16) uint8_t codes[2][32 * kCodePitch];
  const CacheView &c = a.c;
  const int b = blockIdx.z, head = blockIdx.y, tile = blockIdx.x;
  const int64_t row0 = c.starts[b];
  const int64_t all = c.starts[b + 1] - row0;
  const int64_t n = (all < a.max_len ? all : a.max_len) - (int64_t)tile * 32;    // tokens wanted from this tile on
  if (n <= 0) return;
  const uint8_t *src = cache_tile(c, b, head, tile);
  const int pad = (c.head_dim + 31) / 32 * 32;
  const int i = threadIdx.x, r = i & 15, q = (i >> 4) & 3, S = i >> 6;
  if (src != nullptr && i < 2 * pad) {
    const u32x2 kw = reinterpret_cast<const u32x2 *>(src)[i], vw = reinterpret_cast<const u32x2 *>(src + 16 * pad)[i];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      *reinterpret_cast<u32x2 *>(&codes[0][(16 * h + r) * kCodePitch + 32 * S + 8 * q]) = bytes_of_word(kw[h]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        codes[1][(16 * (e >> 2) + 4 * q + (e & 3)) * kCodePitch + 32 * S + 16 * j + r] = (vw[j] >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u;
  }
  __syncthreads();
  const int token = threadIdx.x >> 3, col = (threadIdx.x & 7) * 16;
  const int64_t row = row0 + (int64_t)tile * 32 + token;
  if (token >= n || row < 0 || row >= c.n_rows) return;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const u32 m = src ? reinterpret_cast<const u32 *>(src + 32 * pad)[32 * x + token] : 0u;
    const float s = half_lo(m), lo = half_hi(m);
    u32 *out = (x ? a.v_out : a.k_out) + (row * c.kv_heads + head) * (c.head_dim / 2);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int at = col + 8 * half;
      if (at >= c.head_dim) continue;
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = src ? __builtin_fmaf(s, (float)codes[x][token * kCodePitch + at + j], lo) : 0.f;
        asm("" : "+v"(f[j]));      // a binary32 value: not to be fused with the rounding to 16 bits
      }
      *reinterpret_cast<u32x4 *>(out + at / 2) = pack8<E>(f);
    }
  }
}

int launch_cache_append(const CacheView &c, const void *k, const void *v, int32_t type, int32_t max_new, int64_t k_row,
                        int64_t k_head, int64_t v_row, int64_t v_head, void *stream) {
  const AppendArgs a{c, static_cast<const u32 *>(k), static_cast<const u32 *>(v), k_row, k_head, v_row, v_head, max_new};
  // so many tokens touch at most this many tiles, wherever the first of them lies
  const int64_t most = std::min(max_new, c.n_rows);
  const dim3 grid((unsigned)((most + 30) / 32 + 1), (unsigned)c.kv_heads, (unsigned)c.n_seqs);
  if (type == OWQ_TYPE_F16) owq_cache_append_kernel<F16><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  else owq_cache_append_kernel<BF16><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  return (int)hipGetLastError();
}

int launch_cache_read(const CacheView &c, void *k_out, void *v_out, int32_t type, int32_t max_len, void *stream) {
  const ReadArgs a{c, static_cast<u32 *>(k_out), static_cast<u32 *>(v_out), max_len};
  const dim3 grid((unsigned)(((int64_t)std::min(max_len, c.n_rows) + 31) / 32), (unsigned)c.kv_heads, (unsigned)c.n_seqs);
  if (type == OWQ_TYPE_F16) owq_cache_read_kernel<F16><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  else owq_cache_read_kernel<BF16><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  return (int)hipGetLastError();
}

}  // namespace owq
