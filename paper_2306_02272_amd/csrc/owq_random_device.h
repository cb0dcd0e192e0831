// Random bits by counter: Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011), 16 bits for an element, so that one call serves the eight elements of a 16-byte piece.
#pragma once
#include "owq_ends.h"
#include "owq_step_device.h"

namespace owq {

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

// Which of the elements 8 unit .. 8 unit + 7 of a row stay, one bit each.
__device__ __forceinline__ u32 stays8(const Dropping &d, const DropKey &k, u32 unit, u32 row) {
  const u32x4 w = philox((u32x4){unit, row, k.step, (u32)d.site}, k.k0, k.k1);
  u32 bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bits |= (w[i] & 0xffffu) >= d.threshold ? 1u << (2 * i) : 0u;
    bits |= (w[i] >> 16) >= d.threshold ? 2u << (2 * i) : 0u;
  }
  return bits;
}

// ---- pieces of eight elements of rows that may begin anywhere -----------------------------------------------------------------
// The vector loads and stores take addresses on any boundary of the element; the last piece of a row may be cut.

typedef u32x4 u32x4_any2 __attribute__((aligned(2)));
typedef u32x4 u32x4_any4 __attribute__((aligned(4)));

// The eight elements of a piece as they lie in memory.
template <class E>
struct Piece {
  static constexpr int kSize = 2;
  u32x4 v;
  __device__ __forceinline__ void zero() { v = (u32x4){0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const void *row, int unit, int width) {
    const uint16_t *p = static_cast<const uint16_t *>(row) + 8 * unit;
    const int n = width - 8 * unit;
    if (n >= 8) {
      v = *reinterpret_cast<const u32x4_any2 *>(p);
    } else {
      zero();
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < n) v[j >> 1] |= (u32)p[j] << (16 * (j & 1));
    }
  }
  __device__ __forceinline__ void get(float *f) const { unpack8<E>(v, f); }
  __device__ __forceinline__ void put(const float *f) { v = pack8<E>(f); }
  template <bool KEEP>
  __device__ __forceinline__ void store(void *row, int unit, int width) const {
    uint16_t *p = static_cast<uint16_t *>(row) + 8 * unit;
    const int n = width - 8 * unit;
    if (n >= 8) {
      if (KEEP) *reinterpret_cast<u32x4_any2 *>(p) = v;
      else __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any2 *>(p));
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < n) p[j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
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
    const u32 *p = static_cast<const u32 *>(row) + 8 * unit;
    const int n = width - 8 * unit;
    if (n >= 8) {
      v[0] = reinterpret_cast<const u32x4_any4 *>(p)[0];
      v[1] = reinterpret_cast<const u32x4_any4 *>(p)[1];
    } else {
      zero();
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < n) v[j >> 2][j & 3] = p[j];
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
  __device__ __forceinline__ void store(void *row, int unit, int width) const {
    u32 *p = static_cast<u32 *>(row) + 8 * unit;
    const int n = width - 8 * unit;
    if (n >= 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (KEEP) reinterpret_cast<u32x4_any4 *>(p)[i] = v[i];
        else __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4_any4 *>(p) + i);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < n) p[j] = v[j >> 2][j & 3];
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
