// What a workgroup of 1024 threads does with a row of logits: passes over it, reductions, candidates listed and ranked in LDS, and
// the general way to its k largest.  Shared by sampling and by log-probabilities.
#pragma once
#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

constexpr int kSampleThreads = 1024;
constexpr float kMassUnit = 0x1p31f;
constexpr int kList = 1024;         // candidates that are ranked against each other
constexpr int kBins = 1024;         // of 1/16 in log2 of the probability, for counts
constexpr int kMassBins = 4096;     // of 1/128, for masses: what lies 2^-32 below the largest has none
constexpr float kLog2e = 1.44269504089f, kLn2 = 0.69314718056f;

struct SampleShared {
  u64 mass[kMassBins];
  u32 count[kBins];
  u64 list[kList], sure[kList];   // key << 32 | ~index: larger comes first
  u32 n_list, n_sure;
  u64 wave_mass[16];
  u32 wave_count[16];
  u64 best[16];
  float sum[16];
  u32 digit;
  u64 cut;
  u64 total;
};

// Key order = logit order; -0 sorts with 0.
__device__ __forceinline__ u32 key_of(float x) {
  const u32 b = __builtin_bit_cast(u32, x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(u32 key) {
  return __builtin_bit_cast(float, (key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

template <int TYPE>
__device__ __forceinline__ float logit_at(const void *row, int i) {
  if (TYPE == OWQ_TYPE_F32) return static_cast<const float *>(row)[i];
  const u32 w = static_cast<const uint16_t *>(row)[i];
  return TYPE == OWQ_TYPE_F16 ? F16::lo(w) : BF16::lo(w);
}

template <class T, class F>
__device__ __forceinline__ T block_reduce(T v, T none, T *part, F &&f) {
  v = wave_scan(v, none, f);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < kSampleThreads / 64; ++i) v = f(v, part[i]);
  return v;
}
__device__ __forceinline__ u64 block_max(u64 v, SampleShared &sh) {
  return block_reduce(v, (u64)0, sh.best, [](u64 a, u64 b) { return a > b ? a : b; });
}
__device__ __forceinline__ u64 block_add(u64 v, SampleShared &sh) {
  return block_reduce(v, (u64)0, sh.best, [](u64 a, u64 b) { return a + b; });
}
__device__ __forceinline__ float block_top(float v, SampleShared &sh) {
  return block_reduce(v, -__builtin_inff(), sh.sum, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float block_sum(float v, SampleShared &sh) {
  return block_reduce(v, 0.f, sh.sum, [](float a, float b) { return a + b; });
}

// The instruction takes subnormal numbers for 0; scaled by 2^32 (exactly) they are normal.
__device__ __forceinline__ float log2_of(float x) {
  const bool small = x < 0x1p-126f;
  return __builtin_amdgcn_logf(small ? x * 0x1p32f : x) - (small ? 32.f : 0.f);
}

__device__ __forceinline__ u32 mass_of(float x, float top, float rate) {
  return (u32)(__builtin_amdgcn_exp2f((x - top) * rate) * kMassUnit);
}

// Descends the keys by eight bits at a time.  By count: the key of the `want`-th largest.  By mass: the largest key
// with mass(keys >= it) >= want.  What lies above the key is left in *count_above and *mass_above.
template <int TYPE, bool MASS>
__device__ u32 select_key(const void *row, int vocab, float top, float rate, u32 floor_key, double want, u32 *count_above,
                          u64 *mass_above, SampleShared &sh) {
  u32 prefix = 0, n_above = 0;
  u64 m_above = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += kSampleThreads) {
      sh.mass[i] = 0;
      sh.count[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < vocab; i += kSampleThreads) {
      const float x = logit_at<TYPE>(row, i);
      const u32 key = key_of(x);
      if (key < floor_key || (shift < 24 && (key >> (shift + 8)) != (prefix >> (shift + 8)))) continue;
      const u32 d = (key >> shift) & 255u;
      atomicAdd(&sh.count[d], 1u);
      if (MASS) atomicAdd(&sh.mass[d], (u64)mass_of(x, top, rate));
    }
    __syncthreads();
    // sums over the bins above, bin 255 - t at thread t
    if (threadIdx.x < 256) {
      const int d = 255 - (int)threadIdx.x, lane = threadIdx.x & 63;
      u64 m = MASS ? sh.mass[d] : 0;
      u32 n = sh.count[d];
      const u64 m0 = m;
      const u32 n0 = n;
      m = wave_scan(m, (u64)0, [](u64 a, u64 b) { return a + b; });
      n = wave_scan(n, 0u, [](u32 a, u32 b) { return a + b; });
      if (lane == 63) {
        sh.wave_mass[threadIdx.x >> 6] = m;
        sh.wave_count[threadIdx.x >> 6] = n;
      }
      sh.mass[d] = m - m0;       // of the bins above it within the wave's 64
      sh.count[d] = n - n0;
      if (threadIdx.x == 0) sh.digit = 0;
    }
    __syncthreads();
    if (threadIdx.x < 256) {
      const int d = 255 - (int)threadIdx.x, wave = threadIdx.x >> 6;
      u64 m = m_above + sh.mass[d];
      u32 n = n_above + sh.count[d];
      for (int w = 0; w < wave; ++w) {
        m += sh.wave_mass[w];
        n += sh.wave_count[w];
      }
      // the lowest bin whose sum above still falls short of what is wanted holds the key
      const bool shortfall = MASS ? (double)m < want : (double)n < want;
      if (shortfall) atomicMax(&sh.digit, (u32)threadIdx.x);
      sh.mass[d] = m;
      sh.count[d] = n;
    }
    __syncthreads();
    const u32 d = 255u - sh.digit;
    m_above = sh.mass[d];
    n_above = sh.count[d];
    prefix |= d << shift;
  }
  *count_above = n_above;
  *mass_above = m_above;
  return prefix;
}

// The cut of a row: logits with a larger key stay, of those with this key the ones up to this index.
struct Cut {
  u32 key, at;
};

// The general way, from the row in memory.
template <int TYPE>
__device__ Cut general_cut(const void *row, int vocab, int k, float p, float top, float rate, SampleShared &sh) {
  u32 key = key_of(-__builtin_inff()) + 1u, ties = 0xffffffffu, n_above = 0;
  u64 m_above = 0;
  if (k >= 1 && k < vocab) {
    const u32 found = select_key<TYPE, false>(row, vocab, top, rate, key, (double)k, &n_above, &m_above, sh);
    if (found >= key) {       // else fewer than k finite logits
      key = found;
      ties = (u32)k - n_above;
    }
  }
  if (p < 1.f) {
    // mass of what stayed: all of it above the threshold, and its ties
    u64 m = 0;
    for (int i = threadIdx.x; i < vocab; i += kSampleThreads) {
      const float x = logit_at<TYPE>(row, i);
      const u32 kk = key_of(x);
      if (kk > key || (kk == key && ties == 0xffffffffu)) m += mass_of(x, top, rate);
    }
    u64 all = block_add(m, sh);
    if (ties != 0xffffffffu) all += (u64)ties * mass_of(logit_of(key), top, rate);
    const double want = fmax((double)p * (double)all, 1.0);
    const u32 found = select_key<TYPE, true>(row, vocab, top, rate, key, want, &n_above, &m_above, sh);
    const u32 each = mass_of(logit_of(found), top, rate);
    u32 need = 0xffffffffu;
    if (each > 0) {
      const double n = __builtin_ceil((want - (double)m_above) / (double)each);
      need = n < 1.0 ? 1u : n < 4e9 ? (u32)n : 0xffffffffu;
    }
    ties = found == key && ties < need ? ties : need;
    key = found;
  }
  // the index of the last tie that stays
  Cut c = {key, 0xffffffffu};
  if (ties != 0xffffffffu) {
    u32 before = 0;
    __syncthreads();
    if (threadIdx.x == 0) sh.digit = 0xffffffffu;
    for (int base = 0; base < vocab && before < ties; base += kSampleThreads) {
      const int i = base + threadIdx.x;
      const bool tie = i < vocab && key_of(logit_at<TYPE>(row, i)) == key;
      const u64 ballot = __ballot(tie);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.wave_count[threadIdx.x >> 6] = (u32)__popcll(ballot);
      __syncthreads();
      u32 rank = before, all = 0;
      for (int w = 0; w < kSampleThreads / 64; ++w) {
        if (w < (int)(threadIdx.x >> 6)) rank += sh.wave_count[w];
        all += sh.wave_count[w];
      }
      rank += (u32)__popcll(ballot & ((1ull << (threadIdx.x & 63)) - 1ull));
      if (tie && rank + 1 == ties) sh.digit = (u32)i;
      before += all;
    }
    __syncthreads();
    c.at = sh.digit;
  }
  return c;
}

// Threads' counts to their first places; *all = the sum.
__device__ __forceinline__ u32 block_places(u32 n, u32 *all, SampleShared &sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const u32 sum = wave_scan(n, 0u, [](u32 a, u32 b) { return a + b; });
  __syncthreads();
  if (lane == 63) sh.wave_count[wave] = sum;
  __syncthreads();
  u32 before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kSampleThreads / 64; ++w) {
    before += w < wave ? sh.wave_count[w] : 0u;
    total += sh.wave_count[w];
  }
  *all = total;
  return before + sum - n;
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

// A list of logits in LDS, in no order.
struct List {
  u64 *entry;
  u32 *n;
  // the logits of `bits` behind the entries that are there, read again as they are few; entries past kList are counted only
  template <int TYPE, class I>
  __device__ __forceinline__ void add(const RowView<TYPE> &x, u32 bits, I &&index) {
    if (!__any(bits != 0)) return;
    const int lane = threadIdx.x & 63;
    const u32 mine = (u32)__popc(bits);
    const u32 sum = wave_scan(mine, 0u, [](u32 a, u32 b) { return a + b; });
    u32 base = 0;
    if (lane == 63) base = atomicAdd(n, sum);
    u32 place = (u32)__builtin_amdgcn_readlane((int)base, 63) + sum - mine;
    for (; bits != 0 && place < (u32)kList; bits &= bits - 1, ++place) {
      const int i = index(__ffs(bits) - 1);
      entry[place] = entry_of(logit_at<TYPE>(x.row, i), (u32)i);
    }
  }
};

__device__ __forceinline__ void clear_lists(SampleShared &sh) {
  if (threadIdx.x == 0) sh.n_sure = sh.n_list = 0;
  sh.list[threadIdx.x] = 0;
}

// What precedes a logit in a list of n: how many, and their mass.
__device__ __forceinline__ void precede(const u64 *list, const u32 *list_mass, u32 n, u64 me, u32 *rank, u64 *mass) {
  u32 c = 0;
  u64 m = 0;
  for (u32 j = 0; j < n; j += 8) {
    u64 e[8];
    u32 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = list[j + i];           // past n: entries of 0, before nothing
      w[i] = list_mass[j + i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool before = e[i] > me;
      c += before ? 1u : 0u;
      m += before ? w[i] : 0u;
    }
  }
  *rank = c;
  *mass = m;
}

}  // namespace owq
