// One token per row of logits: temperature, top-k, top-p, min-p, and the largest z - ln e of what is left.
//
// A workgroup takes a row.  Filters are thresholds on the logit itself (a monotone 32-bit key) and, among
// equal logits at the threshold, on the index: the k-th largest key by four histograms of eight bits each,
// the nucleus' key by the same search over probability mass.  Masses are 2^38 e^(z - max z) as integers, so
// that the histograms' order of additions does not show.
#include <hip/hip_runtime.h>

#include "owq_step.h"
#include "owq_step_device.h"

namespace owq {

typedef unsigned long long u64;

constexpr int kSampleThreads = 1024;
constexpr float kMassUnit = 0x1p38f;
constexpr float kLog2e = 1.44269504089f;

struct SampleShared {
  u64 mass[256];
  u32 count[256];
  u64 wave_mass[4];
  u32 wave_count[4];
  u64 best[16];
  float sum[16];
  u32 digit, n_below;
  u64 m_below;
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

__device__ __forceinline__ u64 block_max(u64 v, SampleShared &sh) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const u64 o = __shfl_xor(v, s);
    v = o > v ? o : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh.best[0];
  for (int i = 1; i < kSampleThreads / 64; ++i) v = sh.best[i] > v ? sh.best[i] : v;
  return v;
}

__device__ __forceinline__ float block_sum(float v, SampleShared &sh) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) v += __shfl_xor(v, s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.sum[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
  for (int i = 0; i < kSampleThreads / 64; ++i) v += sh.sum[i];
  return v;
}

__device__ __forceinline__ u64 mass_of(float x, float top, float rate) {
  return (u64)(__builtin_amdgcn_exp2f((x - top) * rate) * kMassUnit);
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
      if (MASS) atomicAdd(&sh.mass[d], mass_of(x, top, rate));
    }
    __syncthreads();
    // sums over the bins above, bin 255 - t at thread t
    if (threadIdx.x < 256) {
      const int d = 255 - (int)threadIdx.x, lane = threadIdx.x & 63;
      u64 m = MASS ? sh.mass[d] : 0;
      u32 n = sh.count[d];
      const u64 m0 = m;
      const u32 n0 = n;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) {
        const u64 mo = __shfl_up(m, s);
        const u32 no = __shfl_up(n, s);
        if (lane >= s) {
          m += mo;
          n += no;
        }
      }
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

template <int TYPE>
__global__ __launch_bounds__(kSampleThreads) void owq_sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int r = blockIdx.x;
  const size_t size = TYPE == OWQ_TYPE_F32 ? 4 : 2;
  const void *row = static_cast<const char *>(a.logits) + (int64_t)r * a.logits_row * size;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  const float rate = kLog2e / (t > 0.f ? t : 1.f);

  u64 best = 0;
  float bad = 0.f;
  for (int i = threadIdx.x; i < a.vocab; i += kSampleThreads) {
    const float x = logit_at<TYPE>(row, i);
    if (x != x) bad = 1.f;
    const u64 v = (u64)key_of(x) << 32 | (0xffffffffu - (u32)i);
    best = v > best ? v : best;
  }
  bad = block_sum(bad, sh);
  best = block_max(best, sh);
  const float top = logit_of((u32)(best >> 32));
  const int greedy = (int)(0xffffffffu - (u32)best);
  if (bad != 0.f || !(__builtin_fabsf(top) < __builtin_inff()) || !(t >= 0.f) || (t > 0.f && a.noise == nullptr)) {
    if (threadIdx.x == 0) {
      a.token[r] = -1;
      if (a.logprob) a.logprob[r] = __builtin_nanf("");
    }
    return;
  }
  float total = 0.f;
  if (a.logprob) {
    for (int i = threadIdx.x; i < a.vocab; i += kSampleThreads) total += __builtin_amdgcn_exp2f((logit_at<TYPE>(row, i) - top) * rate);
    total = block_sum(total, sh);
  }
  int token = greedy;
  if (t > 0.f) {
    // the threshold (key, of its ties the first `ties`)
    u32 key = key_of(-__builtin_inff()) + 1u, ties = 0xffffffffu, n_above = 0;
    u64 m_above = 0;
    const int k = a.top_k ? a.top_k[r] : 0;
    if (k >= 1 && k < a.vocab) {
      const u32 found = select_key<TYPE, false>(row, a.vocab, top, rate, key, (double)k, &n_above, &m_above, sh);
      if (found >= key) {
        key = found;
        ties = (u32)k - n_above;
      }
    }
    const float p = a.top_p ? a.top_p[r] : 1.f;
    if (p < 1.f) {
      // mass of what stayed: all of it above the threshold, and its ties
      u64 m = 0;
      __syncthreads();
      if (threadIdx.x == 0) {
        sh.m_below = 0;
        sh.n_below = 0;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < a.vocab; i += kSampleThreads) {
        const float x = logit_at<TYPE>(row, i);
        const u32 kk = key_of(x);
        if (kk > key || (kk == key && ties == 0xffffffffu)) m += mass_of(x, top, rate);
      }
      atomicAdd(&sh.m_below, m);
      __syncthreads();
      u64 all = sh.m_below;
      if (ties != 0xffffffffu) all += (u64)ties * mass_of(logit_of(key), top, rate);
      const double want = fmax((double)p * (double)all, 1.0);
      const u32 found = select_key<TYPE, true>(row, a.vocab, top, rate, key, want, &n_above, &m_above, sh);
      const u64 each = mass_of(logit_of(found), top, rate);
      u32 need = 0xffffffffu;
      if (each > 0) {
        const double n = __builtin_ceil((want - (double)m_above) / (double)each);
        need = n < 1.0 ? 1u : n < 4e9 ? (u32)n : 0xffffffffu;
      }
      ties = found == key && ties < need ? ties : need;
      key = found;
    }
    const float mp = a.min_p ? a.min_p[r] : 0.f;
    const float z_top = top / t;
    const float least = mp > 0.f ? z_top + __builtin_logf(mp) : -__builtin_inff();
    // the last index that ties may have
    u32 cut = 0xffffffffu;
    if (ties != 0xffffffffu) {
      u32 before = 0;
      for (int base = 0; base < a.vocab; base += kSampleThreads) {
        const int i = base + threadIdx.x;
        const bool tie = i < a.vocab && key_of(logit_at<TYPE>(row, i)) == key;
        const u64 ballot = __ballot(tie);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh.count[threadIdx.x >> 6] = (u32)__popcll(ballot);
        __syncthreads();
        u32 rank = before, all = 0;
        for (int w = 0; w < kSampleThreads / 64; ++w) {
          if (w < (int)(threadIdx.x >> 6)) rank += sh.count[w];
          all += sh.count[w];
        }
        rank += (u32)__popcll(ballot & ((1ull << (threadIdx.x & 63)) - 1ull));
        if (threadIdx.x == 0 && base == 0) sh.digit = 0xffffffffu;
        __syncthreads();
        if (tie && rank + 1 == ties) sh.digit = (u32)i;
        before += all;
        if (before >= ties) break;       // uniform
      }
      __syncthreads();
      cut = sh.digit;
    }
    best = 0;
    const float *noise = a.noise + (int64_t)r * a.noise_row;
    for (int i = threadIdx.x; i < a.vocab; i += kSampleThreads) {
      const float x = logit_at<TYPE>(row, i);
      const u32 kk = key_of(x);
      if (kk < key || (kk == key && (u32)i > cut)) continue;
      const float z = x / t;
      if (!(z >= least) && x < top) continue;
      const u64 v = (u64)key_of(z - __builtin_logf(noise[i])) << 32 | (0xffffffffu - (u32)i);
      best = v > best ? v : best;
    }
    best = block_max(best, sh);
    token = (int)(0xffffffffu - (u32)best);
  }
  if (threadIdx.x == 0) {
    a.token[r] = token;
    const float d = t > 0.f ? t : 1.f;
    if (a.logprob) a.logprob[r] = (logit_at<TYPE>(row, token) - top) / d - __builtin_logf(total);
  }
}

size_t sample_workspace(int32_t, int32_t, int32_t) { return 0; }

int launch_sample(const SampleArgs &a, int32_t type, void *, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == OWQ_TYPE_F16) owq_sample_kernel<OWQ_TYPE_F16><<<a.n_rows, kSampleThreads, 0, s>>>(a);
  else if (type == OWQ_TYPE_BF16) owq_sample_kernel<OWQ_TYPE_BF16><<<a.n_rows, kSampleThreads, 0, s>>>(a);
  else owq_sample_kernel<OWQ_TYPE_F32><<<a.n_rows, kSampleThreads, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace owq
