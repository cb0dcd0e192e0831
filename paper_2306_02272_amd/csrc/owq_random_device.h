// Random bits by counter: Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011), 16 bits for an element, so that one call serves the eight elements of a 16-byte piece.
#pragma once
#include "owq_ends.h"
#include "owq_step_device.h"

namespace owq {

// A product as it is rounded.  Ahead of a sum over lanes: there the compiler may fuse a lane's own product with the addition,
// but not its neighbour's, so that lanes would differ in the last bit of a sum that they share.
__device__ __forceinline__ float rounded(float v) {
  asm("" : "+v"(v));
  return v;
}

// Sum and maximum over the wave, in every lane, in a fixed order.
template <class F>
__device__ __forceinline__ float across_rows(float v, F &&f) {
  const u32 a = __builtin_bit_cast(u32, v);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  v = f(__builtin_bit_cast(float, (u32)r[0]), __builtin_bit_cast(float, (u32)r[1]));
  const u32 b = __builtin_bit_cast(u32, v);
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return f(__builtin_bit_cast(float, (u32)q[0]), __builtin_bit_cast(float, (u32)q[1]));
}
__device__ __forceinline__ float wave_sum(float v) {
  return across_rows(lanes_sum<16>(v), [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
  return across_rows(lanes_max<16>(v), [](float a, float b) { return fmaxf(a, b); });
}

// Halves of the key and the step, read once by a kernel.
struct DropKey {
  u32 k0, k1, step;
};
__device__ __forceinline__ DropKey drop_key(const Dropping &d) {
  if (d.threshold == 0) return DropKey{0, 0, 0};
  const u64 seed = d.rng[0], step = d.rng[1];
  return DropKey{(u32)seed, (u32)(seed >> 32), (u32)step};
}

__device__ __forceinline__ u32x4 philox(u32x4 c, u32 k0, u32 k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const u64 a = (u64)0xD2511F53u * c.x, b = (u64)0xCD9E8D57u * c.z;
    c = (u32x4){(u32)(b >> 32) ^ c.y ^ k0, (u32)b, (u32)(a >> 32) ^ c.w ^ k1, (u32)a};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// Which of the elements 8 unit .. 8 unit + 7 of a row stay.
struct Stays {
  u32x4 bits;
  u32 threshold;
  __device__ __forceinline__ Stays(const Dropping &d, const DropKey &k, u32 unit, u32 row)
      : bits(philox((u32x4){unit, row, k.step, (u32)d.site}, k.k0, k.k1)), threshold(d.threshold) {}
  __device__ __forceinline__ bool operator()(int j) const {
    const u32 w = bits[j >> 1];
    return ((j & 1) ? w >> 16 : w & 0xffffu) >= threshold;
  }
};

// ---- pieces of eight elements of rows that may begin anywhere -----------------------------------------------------------------
// The vector loads and stores take addresses on any boundary of the element; the last piece of a row may be cut.

typedef u32x4 u32x4_any2 __attribute__((aligned(2)));
typedef u32 u32_any2 __attribute__((aligned(2)));
typedef u32x4 u32x4_any4 __attribute__((aligned(4)));

// The eight elements of a piece as they lie in memory.
template <class E>
struct Piece {
  static constexpr int kSize = 2;
  u32x4 v;
  __device__ __forceinline__ void zero() { v = (u32x4){0, 0, 0, 0}; }
  // a row of less than 2^32 bytes: its address and a lane's offset in 32 bits
  __device__ __forceinline__ void load(const void *row, int unit, int width) {
    load(static_cast<const char *>(row) + (u32)unit * 16u, width - 8 * unit);
  }
  template <bool KEEP>
  __device__ __forceinline__ void store(void *row, int unit, int width) const {
    store<KEEP>(static_cast<char *>(row) + (u32)unit * 16u, width - 8 * unit);
  }
  // the piece itself, n elements of the row from there on
  __device__ __forceinline__ void load(const void *piece, int n) {
    const uint16_t *p = static_cast<const uint16_t *>(piece);
    if (n >= 8) {
      v = *reinterpret_cast<const u32x4_any2 *>(p);
    } else {       // four, two and one
      const bool four = n > 0 && (n & 4), two = n > 0 && (n & 2), one = n > 0 && (n & 1);
      u32 a = 0, b = 0, c = 0, d = 0;
      if (four) a = reinterpret_cast<const u32_any2 *>(p)[0], b = reinterpret_cast<const u32_any2 *>(p)[1];
      if (two) c = *reinterpret_cast<const u32_any2 *>(p + (four ? 4 : 0));
      if (one) d = p[(four ? 4 : 0) + (two ? 2 : 0)];
      const u32 first = two ? c : d, second = two ? d : 0;      // behind the four
      v = (u32x4){four ? a : first, four ? b : second, four ? first : 0, four ? second : 0};
    }
  }
  __device__ __forceinline__ void get(float *f) const { unpack8<E>(v, f); }
  __device__ __forceinline__ void put(const float *f) { v = pack8<E>(f); }
  template <bool KEEP>
  __device__ __forceinline__ void store(void *piece, int n) const {
    uint16_t *p = static_cast<uint16_t *>(piece);
    if (n >= 8) {
      if (KEEP) *reinterpret_cast<u32x4_any2 *>(p) = v;
      else __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any2 *>(p));
    } else {
      const bool four = n > 0 && (n & 4), two = n > 0 && (n & 2), one = n > 0 && (n & 1);
      const u32 first = four ? v[2] : v[0], second = four ? v[3] : v[1];
      if (four) reinterpret_cast<u32_any2 *>(p)[0] = v[0], reinterpret_cast<u32_any2 *>(p)[1] = v[1];
      if (two) *reinterpret_cast<u32_any2 *>(p + (four ? 4 : 0)) = first;
      if (one) p[(four ? 4 : 0) + (two ? 2 : 0)] = (uint16_t)(two ? second : first);
    }
  }
};

struct F32 {};
template <>
struct Piece<F32> {
  static constexpr int kSize = 4;
  u32x4 v[2];
  __device__ __forceinline__ void zero() { v[0] = v[1] = (u32x4){0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const void *row, int unit, int width) {
    load(static_cast<const char *>(row) + (u32)unit * 32u, width - 8 * unit);
  }
  template <bool KEEP>
  __device__ __forceinline__ void store(void *row, int unit, int width) const {
    store<KEEP>(static_cast<char *>(row) + (u32)unit * 32u, width - 8 * unit);
  }
  __device__ __forceinline__ void load(const void *piece, int n) {
    const u32 *p = static_cast<const u32 *>(piece);
    if (n >= 8) {
      v[0] = reinterpret_cast<const u32x4_any4 *>(p)[0];
      v[1] = reinterpret_cast<const u32x4_any4 *>(p)[1];
    } else {       // four, two and one
      const bool four = n > 0 && (n & 4), two = n > 0 && (n & 2), one = n > 0 && (n & 1);
      const u32x4 none = {0, 0, 0, 0};
      u32x4 a = none;
      u32 c0 = 0, c1 = 0, d = 0;
      if (four) a = *reinterpret_cast<const u32x4_any4 *>(p);
      if (two) c0 = p[four ? 4 : 0], c1 = p[four ? 5 : 1];
      if (one) d = p[(four ? 4 : 0) + (two ? 2 : 0)];
      const u32x4 rest = {two ? c0 : d, c1, two ? d : 0, 0};      // behind the four
      v[0] = four ? a : rest;
      v[1] = four ? rest : none;
    }
  }
  __device__ __forceinline__ void get(float *f) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const u32 w = v[j >> 2][j & 3];
      f[j] = __builtin_bit_cast(float, w);
    }
  }
  __device__ __forceinline__ void put(const float *f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j >> 2][j & 3] = __builtin_bit_cast(u32, f[j]);
  }
  template <bool KEEP>
  __device__ __forceinline__ void store(void *piece, int n) const {
    u32 *p = static_cast<u32 *>(piece);
    if (n >= 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (KEEP) reinterpret_cast<u32x4_any4 *>(p)[i] = v[i];
        else __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4_any4 *>(p) + i);
      }
    } else {
      const bool four = n > 0 && (n & 4), two = n > 0 && (n & 2), one = n > 0 && (n & 1);
      const u32x4 rest = four ? v[1] : v[0];
      if (four) *reinterpret_cast<u32x4_any4 *>(p) = v[0];
      if (two) p[four ? 4 : 0] = rest[0], p[four ? 5 : 1] = rest[1];
      if (one) p[(four ? 4 : 0) + (two ? 2 : 0)] = two ? rest[2] : rest[0];
    }
  }
};

template <class E>
__device__ __forceinline__ const void *row_at(const void *base, int64_t row, int64_t stride) {
  return static_cast<const char *>(base) + row * stride * Piece<E>::kSize;
}
template <class E>
__device__ __forceinline__ void *row_at(void *base, int64_t row, int64_t stride) {
  return static_cast<char *>(base) + row * stride * Piece<E>::kSize;
}

}  // namespace owq
