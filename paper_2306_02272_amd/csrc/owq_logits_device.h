// A row of logits in memory and the order of its entries: shared by sampling and by log-probabilities.
#pragma once
#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

constexpr int kSampleThreads = 1024;
constexpr float kLog2e = 1.44269504089f, kLn2 = 0.69314718056f;

// Key order = logit order; -0 sorts with 0.
__device__ __forceinline__ u32 key_of(float x) {
  const u32 b = __builtin_bit_cast(u32, x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(u32 key) {
  return __builtin_bit_cast(float, (key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

// Half of what x lies above `from`: no infinity however far that is, as the small scales and large temperatures that make numbers of
// it take any logits.  One rounding, of which no more is left than of the difference's.
__device__ __forceinline__ float apart(float x, float from) { return __builtin_fmaf(0.5f, x, -0.5f * from); }

template <int TYPE>
__device__ __forceinline__ float logit_at(const void *row, int i) {
  if (TYPE == OWQ_TYPE_F32) return static_cast<const float *>(row)[i];
  const u32 w = static_cast<const uint16_t *>(row)[i];
  return TYPE == OWQ_TYPE_F16 ? F16::lo(w) : BF16::lo(w);
}

// A row as whole 16-byte units between its first and its last boundary, and up to 2 (kPer - 1) logits beside them.
template <int TYPE>
struct RowView {
  static constexpr int kPer = TYPE == OWQ_TYPE_F32 ? 4 : 8;
  static constexpr int kUnroll = 16 / kPer;      // units of a thread in flight: 16 logits
  const void *row;
  const u32x4 *units;
  int first, n_units, n_rest;                    // index of unit 0's first logit
  __device__ __forceinline__ RowView(const void *r, int vocab) : row(r) {
    const int size = 16 / kPer;
    const int skip = (int)((16 - (reinterpret_cast<uintptr_t>(r) & 15u)) & 15u) / size;
    first = skip < vocab ? skip : vocab;
    n_units = (vocab - first) / kPer;
    n_rest = vocab - n_units * kPer;
    units = reinterpret_cast<const u32x4 *>(static_cast<const char *>(r) + (int64_t)first * size);
  }
  __device__ __forceinline__ int rest(int j) const { return j < first ? j : j + n_units * kPer; }
  static __device__ __forceinline__ float get(const u32x4 &v, int e) {
    const u32 w = v[TYPE == OWQ_TYPE_F32 ? e & 3 : (e >> 1) & 3];
    if (TYPE == OWQ_TYPE_F32) return __builtin_bit_cast(float, w);
    if (TYPE == OWQ_TYPE_F16) return (e & 1) ? F16::hi(w) : F16::lo(w);
    return (e & 1) ? BF16::hi(w) : BF16::lo(w);
  }
  // g(values, indices' first per unit, units that exist) for 16 logits at a time; all threads make the same number of calls
  template <class G>
  __device__ __forceinline__ void batches(G &&g) const {
    const u32 low = TYPE == OWQ_TYPE_F32 ? 0xff800000u : TYPE == OWQ_TYPE_F16 ? 0xfc00fc00u : 0xff80ff80u;   // -infinity past the end
    // the logits beside the units come last, one per thread: one copy of g's code, not two
    for (int base = 0;; base += kSampleThreads * kUnroll) {
      const bool in_units = base < n_units;
      float x[16];
      if (in_units) {
        u32x4 v[kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) v[j] = units[min(base + j * kSampleThreads + (int)threadIdx.x, n_units - 1)];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
          const bool on = base + j * kSampleThreads + (int)threadIdx.x < n_units;
          v[j] = on ? v[j] : (u32x4){low, low, low, low};
#pragma unroll
          for (int e = 0; e < kPer; ++e) x[j * kPer + e] = get(v[j], e);
        }
      } else {
        if (n_rest == 0) break;
#pragma unroll
        for (int i = 1; i < 16; ++i) x[i] = -__builtin_inff();
        x[0] = (int)threadIdx.x < n_rest ? logit_at<TYPE>(row, rest(threadIdx.x)) : -__builtin_inff();
      }
      g(x, [&](int i) {
        return in_units ? first + (base + (i / kPer) * kSampleThreads + (int)threadIdx.x) * kPer + i % kPer
                        : (int)threadIdx.x < n_rest ? rest(threadIdx.x) : 0;
      });
      if (!in_units) break;
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F &&f) const {
    batches([&](const float (&x)[16], auto &&) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f(x[i]);
    });
  }
};

__device__ __forceinline__ u64 entry_of(float v, u32 at) { return (u64)key_of(v) << 32 | (0xffffffffu - at); }
__device__ __forceinline__ float entry_logit(u64 e) { return logit_of((u32)(e >> 32)); }
__device__ __forceinline__ u32 entry_at(u64 e) { return 0xffffffffu - (u32)e; }

}  // namespace owq
