// Log-probabilities of given tokens, entropy and the likeliest tokens of every row of logits, and the gradient to the logits.
//
// Forward: a workgroup of 1024 threads takes a row in one pass.  With m the largest logit so far and d = scale (x - m), a thread
// holds S = sum e^d and W = sum e^d d; when m grows to m', both are scaled: S' = f S, W' = f (W + (m - m') scale S), f = e^((m - m') scale).
//     ln p = d - ln S,   entropy = ln S - W / S
// Nothing is measured from anything but the largest logit, so that an offset of all logits costs no digits.
// Alternatives: the K-th of the threads' largest logits lies at or below the row's K-th; threads whose largest does not lie
// below that list their logits that do not either, and those are ranked.
// Backward: element by element, with p from the forward's m and ln S.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "owq_ends.h"
#include "owq_logits_device.h"
#include "owq_random_device.h"

namespace owq {

constexpr float kLowest = -3.402823466e38f;
constexpr float kVanishes = -200.f;      // 2^-200 is 0 in binary32; keeps 0 times infinity out of the sums

struct LogprobShared {
  float sum[16];
};

template <int TYPE, bool TOP>
__global__ __launch_bounds__(kSampleThreads) void owq_logprob_kernel(LogprobArgs a) {
  using Shared = typename std::conditional<TOP, SampleShared, LogprobShared>::type;
  __shared__ Shared sh;
  for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const size_t size = TYPE == OWQ_TYPE_F32 ? 4 : 2;
    const void *row = static_cast<const char *>(a.logits) + r * a.logits_row * size;
    const RowView<TYPE> x(row, a.vocab);
    const float rate = kLog2e * a.scale;
    const int target = a.targets ? a.targets[r] : -1;
    float at_target = 0.f;
    if ((uint32_t)target < (uint32_t)a.vocab) at_target = logit_at<TYPE>(row, target);

    float m = kLowest, s = 0.f, w = 0.f;
    auto raise = [&](float to) {
      const float d = fmaxf((m - to) * rate, kVanishes), f = __builtin_amdgcn_exp2f(d);
      w = f * __builtin_fmaf(s, d, w);
      s *= f;
      m = to;
    };
    x.batches([&](const float (&v)[16], auto &&) {
      float top = m;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, v[i]);
      raise(top);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float d = (v[i] - m) * rate, e = __builtin_amdgcn_exp2f(d);
        s += e;
        w = __builtin_fmaf(e, fmaxf(d, kVanishes), w);
      }
    });
    const float mine = m;
    auto all = [&](float v, float none, auto &&f) { return block_reduce(v, none, sh.sum, f); };
    auto add = [](float p, float q) { return p + q; };
    raise(all(m, kLowest, [](float p, float q) { return fmaxf(p, q); }));
    s = all(s, 0.f, add);
    w = all(w, 0.f, add);
    const float nan = __builtin_nanf("");
    const bool good = s > 0.f && m < __builtin_inff();       // not with a NaN in the row, nor if all is -infinity
    const float log_s = good ? __builtin_logf(s) : nan;
    if (threadIdx.x == 0) {
      a.stats[r] = good ? m : nan;
      a.stats[(int64_t)a.n_rows + r] = log_s;
      a.stats[2 * (int64_t)a.n_rows + r] = good ? log_s - kLn2 * (w / s) : nan;
      if (a.targets) a.logprob[r] = (uint32_t)target < (uint32_t)a.vocab ? (at_target - m) * a.scale - log_s : 0.f;
    }
    if constexpr (TOP) {
      const int64_t out = r * a.top;
      if (!good) {
        if ((int)threadIdx.x < a.top) {
          a.top_token[out + threadIdx.x] = -1;
          a.top_logprob[out + threadIdx.x] = nan;
        }
        continue;
      }
      // the least candidate: the threads' largest counted by bins of 1/16 in log2 of the probability
      sh.count[threadIdx.x] = 0;
      clear_lists(sh);
      __syncthreads();
      const float d = (m - mine) * rate * 16.f;
      atomicAdd(&sh.count[d < (float)(kBins - 1) ? (int)d : kBins - 1], 1u);
      __syncthreads();
      u32 n;
      const u32 own = sh.count[threadIdx.x];
      const u32 before = block_places(own, &n, sh);
      if (threadIdx.x == 0) sh.digit = kBins - 1;
      __syncthreads();
      if (before < (u32)a.top && before + own >= (u32)a.top) sh.digit = threadIdx.x;
      __syncthreads();
      // a little below the bin's edge, so that rounding leaves none of its logits out; the last bin is open
      const u32 bin = sh.digit;
      const float lo = bin >= kBins - 1 ? kLowest : fmaxf(m - ((float)(bin + 1) * 0.0625f / rate) * 1.00001f, kLowest);
      List list = {sh.list, &sh.n_list};
      if (__any(mine >= lo))
        x.batches([&](const float (&v)[16], auto &&index) {
          u32 bits = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) bits |= v[i] >= lo ? 1u << i : 0u;
          list.add(x, bits, index);
        });
      __syncthreads();
      if (sh.n_list > (u32)kList) {       // many equal logits: the general way
        const Cut cut = general_cut<TYPE>(row, a.vocab, a.top, 1.f, m, rate, sh);
        __syncthreads();
        clear_lists(sh);
        __syncthreads();
        x.batches([&](const float (&v)[16], auto &&index) {
          u32 bits = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const u32 k = key_of(v[i]);
            bits |= k > cut.key || (k == cut.key && (u32)index(i) <= cut.at) ? 1u << i : 0u;
          }
          list.add(x, bits, index);
        });
        __syncthreads();
      }
      const u32 found = sh.n_list;
      const u64 me = sh.list[threadIdx.x];
      if (threadIdx.x < found) {
        u32 rank = 0;
        for (u32 j = 0; j < found; j += 8)
#pragma unroll
          for (int i = 0; i < 8; ++i) rank += sh.list[j + i] > me ? 1u : 0u;      // past the end: 0, before nothing
        if (rank < (u32)a.top) {
          a.top_token[out + rank] = (int32_t)entry_at(me);
          a.top_logprob[out + rank] = (entry_logit(me) - m) * a.scale - log_s;
        }
      }
      if (threadIdx.x >= found && (int)threadIdx.x < a.top) {
        a.top_token[out + threadIdx.x] = -1;
        a.top_logprob[out + threadIdx.x] = -__builtin_inff();
      }
    }
  }
}

template <int TYPE>
static void launch_type(const LogprobArgs &a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20);
  if (a.top > 0) owq_logprob_kernel<TYPE, true><<<grid, kSampleThreads, 0, s>>>(a);
  else owq_logprob_kernel<TYPE, false><<<grid, kSampleThreads, 0, s>>>(a);
}

int launch_logprobs(const LogprobArgs &a, int32_t type, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == OWQ_TYPE_F16) launch_type<OWQ_TYPE_F16>(a, s);
  else if (type == OWQ_TYPE_BF16) launch_type<OWQ_TYPE_BF16>(a, s);
  else launch_type<OWQ_TYPE_F32>(a, s);
  return (int)hipGetLastError();
}

// A workgroup takes pieces blockIdx.x 256 + thread, ... of rows blockIdx.y, ...
template <class E>
__global__ __launch_bounds__(256) void owq_logprob_backward_kernel(LogprobBackwardArgs a) {
  const float rate = kLog2e * a.scale;
  const int units = (a.vocab + 7) >> 3;
  for (int64_t r = blockIdx.y; r < a.n_rows; r += gridDim.y) {
    const void *row = row_at<E>(a.logits, r, a.logits_row);
    void *out = row_at<E>(a.dlogits, r, a.vocab);
    const int target = a.targets ? a.targets[r] : -1;
    const bool counted = (uint32_t)target < (uint32_t)a.vocab;
    const float dlp = a.dlogprob && counted ? a.dlogprob[r] : 0.f, dh = a.dentropy ? a.dentropy[r] : 0.f;
    const float m = a.stats[r], log_s = a.stats[(int64_t)a.n_rows + r], entropy = a.stats[2 * (int64_t)a.n_rows + r];
    const bool none = dlp == 0.f && dh == 0.f;
    const float log2_s = log_s * kLog2e;
    const float c0 = -a.scale * __builtin_fmaf(dh, entropy, dlp), c1 = -a.scale * dh * kLn2;      // dz = p (c0 + c1 log2 p)
    for (int u = (int)blockIdx.x * 256 + threadIdx.x; u < units; u += (int)gridDim.x * 256) {
      Piece<E> p;
      float f[8];
      if (none) {
        p.zero();
      } else {
        p.load(row, u, a.vocab);
        p.get(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float l = __builtin_fmaf(f[j] - m, rate, -log2_s);
          f[j] = __builtin_amdgcn_exp2f(l) * __builtin_fmaf(c1, fmaxf(l, kVanishes), c0);
        }
        if (counted && u == target >> 3) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] += j == (target & 7) ? a.scale * dlp : 0.f;
        }
        p.put(f);
      }
      p.template store<false>(out, u, a.vocab);
    }
  }
}

int launch_logprobs_backward(const LogprobBackwardArgs &a, int32_t type, void *stream) {
  const int units = (a.vocab + 7) / 8;
  const dim3 grid((unsigned)((units + 511) / 512), (unsigned)(a.n_rows < 65535 ? a.n_rows : 65535));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == OWQ_TYPE_F16) owq_logprob_backward_kernel<F16><<<grid, 256, 0, s>>>(a);
  else if (type == OWQ_TYPE_BF16) owq_logprob_backward_kernel<BF16><<<grid, 256, 0, s>>>(a);
  else owq_logprob_backward_kernel<F32><<<grid, 256, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace owq
