// One token per row of logits: temperature, top-k, top-p, min-p, and the largest z - ln e of what is left.
//
// A workgroup of 1024 threads takes a row.  Every filter is a threshold on (logit, index) in the order "larger logit
// first, lower index first":
//   top-k up to 512: the k-th of the 1024 threads' largest logits lies at or below the row's k-th, so that a little more
//     than k logits are candidates; they are listed in LDS and each counts what precedes it, and the mass of that, which
//     decides top-k and top-p at once.  Two passes over the row;
//   a longer top-k, and top-p without a short one: counts, or masses, are added up by bins of 1/128 in log2; the logits of
//     the bin in which the wanted sum is reached are listed and ranked in the same way.  Three passes for either.
// A bin with more than 1024 logits, as in flat rows, takes the general way: keys by four histograms of eight bits each.  Passes are rolled loops of 16 logits per thread: with the row in registers every pass is
// straight-line code that a launch runs through once, and its instructions come from memory more slowly than the row does
// (179 us for 256 rows of 50 272 fp32 logits so, 36 now).
//
// Bound by the passes: those 256 rows with top-p take three, the first from memory, the others from the last-level cache:
// 36.5 us for 51.5 MB of logits, which one pass at a copy's rate would read in 10.8 (of the variates only those of the tokens
// that stay are read, some 70 a row); one row of 32 000 fp16 logits 11.0 us, 10.7 of them in the kernel.
// Masses are 2^31 e^(z - max z) as integers, so that no order of additions shows.
#include <hip/hip_runtime.h>

#include "owq_logits_device.h"

namespace owq {

// The first bin with which the sum over sh.mass reaches `want` (left in sh.digit; sh.total = the sum before it), or
// 0xffffffff if there is none.
__device__ __forceinline__ u32 find_bin(double want, SampleShared &sh) {
  constexpr int kEach = kMassBins / kSampleThreads;
  u64 own[kEach], sum = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) sum += own[j] = sh.mass[threadIdx.x * kEach + j];
  const u64 mine = sum;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  sum = wave_scan(sum, (u64)0, [](u64 a, u64 b) { return a + b; });
  if (lane == 63) sh.wave_mass[wave] = sum;
  if (threadIdx.x == 0) sh.digit = 0xffffffffu;
  __syncthreads();
  u64 ahead = sum - mine;
  for (int w = 0; w < wave; ++w) ahead += sh.wave_mass[w];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if ((double)ahead < want && (double)(ahead + own[j]) >= want) {
      sh.digit = threadIdx.x * kEach + j;
      sh.total = ahead;
    }
    ahead += own[j];
  }
  __syncthreads();
  return sh.digit;
}
__device__ __forceinline__ void clear_bins(SampleShared &sh) {
#pragma unroll
  for (int j = 0; j < kMassBins / kSampleThreads; ++j) sh.mass[j * kSampleThreads + threadIdx.x] = 0;
}

template <int TYPE>
__global__ __launch_bounds__(kSampleThreads) void owq_sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int r = blockIdx.x;
  const size_t size = TYPE == OWQ_TYPE_F32 ? 4 : 2;
  const void *row = static_cast<const char *>(a.logits) + (int64_t)r * a.logits_row * size;
  const RowView<TYPE> x(row, a.vocab);
  const float bottom = -__builtin_inff();
  float mine = bottom;
  x.each([&](float v) { mine = fmaxf(mine, v); });
  const float t = a.temperature ? a.temperature[r] : 1.f;
  const float rate = kLog2e / (t > 0.f ? t : 1.f);
  const int k = a.top_k ? a.top_k[r] : 0;
  const float p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f;
  const float top = block_top(mine, sh);
  const bool by_k = t > 0.f && k >= 1 && k < a.vocab, short_k = by_k && k <= kList / 2, long_k = by_k && !short_k, by_p = t > 0.f && !by_k && p < 1.f;
  // Everything is measured from the largest logit, in log2 of the probability: sums with a logit itself would round at its size,
  // not at the difference's, and overflow at small temperatures.
  auto below = [&](float v) { return (top - v) * rate; };
  const float reach = mp > 0.f ? -log2_of(mp) : __builtin_inff();       // z >= max z + ln min_p
  auto likely = [&](float v) { return below(v) <= reach || v == top; };
  clear_lists(sh);

  // what the second pass needs: the least candidate for a short top-k, empty bins for a long one and for top-p
  float lo = __builtin_inff();
  if (short_k) {
    sh.count[threadIdx.x] = 0;
    __syncthreads();
    const float d = below(mine) * 16.f;
    if (mine > bottom) atomicAdd(&sh.count[d < (float)(kBins - 1) ? (int)d : kBins - 1], 1u);
    __syncthreads();
    u32 all;
    const u32 own = sh.count[threadIdx.x];
    const u32 before = block_places(own, &all, sh);
    if (threadIdx.x == 0) sh.digit = kBins - 1;
    __syncthreads();
    if (before < (u32)k && before + own >= (u32)k) sh.digit = threadIdx.x;
    __syncthreads();
    // a little below the bin's edge, so that rounding leaves none of its logits out; the last bin is open
    const u32 bin = sh.digit;
    lo = bin >= kBins - 1 || all < (u32)k ? -3.402823466e38f : top - ((float)(bin + 1) * 0.0625f / rate) * 1.00001f;
  } else if (by_p || long_k) {
    clear_bins(sh);
  }
  __syncthreads();

  auto bin_at = [](float d) { return (u32)(int)(d * 128.f); };       // d in log2 below the largest, under 32
  auto bin_of = [&](float v) { return bin_at(fminf(below(v), 31.995f)); };
  List list = {sh.list, &sh.n_list}, sure = {sh.sure, &sh.n_sure};
  float total = 0.f;
  u64 m = 0;
  x.batches([&](const float (&v)[16], auto &&index) {
    u32 bits = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float d = below(v[i]), e = __builtin_amdgcn_exp2f(-d);
      total += e;
      bits |= v[i] >= lo ? 1u << i : 0u;
      if (by_p) {
        const u32 w = (u32)(e * kMassUnit);
        if (w > 0) atomicAdd(&sh.mass[bin_at(d)], (u64)w);
        m += w;
      }
    }
    if (short_k) list.add(x, bits, index);
  });
  total = block_sum(total, sh);           // NaN if a logit is (or the top infinite)
  // the temperature by itself: 1 / t of a subnormal one may still be finite, that of an infinite one is 0 and gives finite sums
  const bool warm = t >= 0x1p-126f && t < __builtin_inff();
  if (!(__builtin_fabsf(top) < __builtin_inff()) || total != total || !(t == 0.f || (warm && a.noise != nullptr))) {
    if (threadIdx.x == 0) {
      a.token[r] = -1;
      if (a.logprob) a.logprob[r] = __builtin_nanf("");
    }
    return;
  }

  const float *noise = a.noise + (int64_t)r * a.noise_row;
  auto score = [&](u64 e) {
    return entry_of(__builtin_fmaf(entry_logit(e) - top, rate, -log2_of(noise[entry_at(e)])), entry_at(e));
  };
  u64 best = 0;
  Cut cut = {key_of(bottom) + 1u, 0xffffffffu};
  u32 bin = 0xffffffffu;                  // top-p: the bin that the cut lies in
  bool done = false, general = false;     // general: one copy of that code

  if (t == 0.f) {
    x.batches([&](const float (&v)[16], auto &&index) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u64 o = v[i] == top ? (u64)(0xffffffffu - (u32)index(i)) : 0ull;
        best = o > best ? o : best;
      }
    });
    done = true;
  } else if (short_k && sh.n_list <= (u32)kList) {
    const u32 n = sh.n_list;
    const bool on = threadIdx.x < n;
    const u64 me = sh.list[threadIdx.x];
    const float v = entry_logit(me);
    const u32 w = on ? mass_of(v, top, rate) : 0u;
    sh.count[threadIdx.x] = w;
    __syncthreads();
    u32 rank;
    u64 ahead;
    precede(sh.list, sh.count, on ? n : 0u, me, &rank, &ahead);
    bool stays = on && rank < (u32)k;
    if (p < 1.f) {
      const u64 mass = block_add(stays ? (u64)w : 0ull, sh);
      stays = stays && (double)ahead < fmax((double)p * (double)mass, 1.0);
    }
    if (stays && likely(v)) best = score(me);
    done = true;
  } else if (short_k) {
    general = true;
  }
  // what the cut so far leaves
  float edge = bottom;
  u32 edge_at = 0;
  auto kept = [&](float v, u32 at) { return v > edge || (v == edge && v > bottom && at <= edge_at); };
  bool search_p = by_p;
  if (long_k) {
    x.batches([&](const float (&v)[16], auto &&) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (v[i] > bottom) atomicAdd(&sh.mass[bin_of(v[i])], 1ull);
    });
    __syncthreads();
    const u32 b = find_bin((double)k, sh);
    search_p = p < 1.f;
    if (b != 0xffffffffu) {               // else fewer than k finite logits
      const u32 above = (u32)sh.total;
      x.batches([&](const float (&v)[16], auto &&index) {
        u32 bits = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) bits |= v[i] > bottom && bin_of(v[i]) == b ? 1u << i : 0u;
        list.add(x, bits, index);
      });
      __syncthreads();
      const u32 n = sh.n_list;
      if (n > (u32)kList) {
        general = true;
        search_p = false;
      } else {
        const u64 me = sh.list[threadIdx.x];
        sh.count[threadIdx.x] = 0;
        __syncthreads();
        u32 rank;
        u64 none;
        precede(sh.list, sh.count, threadIdx.x < n ? n : 0u, me, &rank, &none);
        if (threadIdx.x < n && above + rank + 1 == (u32)k) sh.cut = me;
        __syncthreads();
        cut = Cut{(u32)(sh.cut >> 32), entry_at(sh.cut)};
        edge = logit_of(cut.key);
        edge_at = cut.at;
      }
    }
    if (search_p) {                       // masses of what stayed
      clear_bins(sh);
      clear_lists(sh);
      __syncthreads();
      x.batches([&](const float (&v)[16], auto &&index) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float d = below(v[i]);
          const u32 w = kept(v[i], (u32)index(i)) && d < 32.f ? (u32)(__builtin_amdgcn_exp2f(-d) * kMassUnit) : 0u;
          if (w > 0) atomicAdd(&sh.mass[bin_at(d)], (u64)w);
          m += w;
        }
      });
    }
  }
  if (search_p) {
    // the bin in which the wanted mass is reached
    m = block_add(m, sh);
    const double want = fmax((double)p * (double)m, 1.0);
    bin = find_bin(want, sh);
    const u64 above = sh.total;
    // its logits into one list, those before it into another: only what min_p leaves, which changes no order and no mass before
    x.batches([&](const float (&v)[16], auto &&index) {
      u32 inside = 0, before = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u32 b = bin_of(v[i]);
        const bool on = kept(v[i], (u32)index(i)) && likely(v[i]);
        inside |= on && b == bin ? 1u << i : 0u;
        before |= on && b < bin ? 1u << i : 0u;
      }
      list.add(x, inside, index);
      sure.add(x, before, index);
    });
    __syncthreads();
    const u32 n = sh.n_list, n_sure = sh.n_sure;
    if (n > (u32)kList) {
      general = true;
    } else {
      const bool on = threadIdx.x < n;
      const u64 me = sh.list[threadIdx.x];
      sh.count[threadIdx.x] = on ? mass_of(entry_logit(me), top, rate) : 0u;
      __syncthreads();
      u32 rank;
      u64 mass;
      precede(sh.list, sh.count, on ? n : 0u, me, &rank, &mass);
      const bool stays = on && (double)(above + mass) < want;
      if (n_sure <= (u32)kList) {
        if (stays) best = score(me);
        if (threadIdx.x < n_sure) {
          const u64 o = score(sh.sure[threadIdx.x]);
          best = o > best ? o : best;
        }
        done = true;
      } else {
        // the last that stays is the cut (above all of the bin if none does)
        const u64 last = block_max(stays ? (u64)rank + 1 : 0ull, sh);
        if (threadIdx.x == 0) sh.cut = ~0ull;
        __syncthreads();
        if (stays && (u64)rank + 1 == last) sh.cut = me;
        __syncthreads();
        cut = Cut{(u32)(sh.cut >> 32), entry_at(sh.cut)};
      }
    }
  }
  if (general) cut = general_cut<TYPE>(row, a.vocab, k, p, top, rate, sh);
  if (!done) {
    // many, or none left out: the random numbers of what stays by logit and, at the cut, by index.  Before the cut's bin
    // nothing is left out but by min_p.
    const bool binned = cut.key == 0xffffffffu;
    const float last = binned ? __builtin_inff() : logit_of(cut.key);
    x.batches([&](const float (&v)[16], auto &&index) {
      u32 bits = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool in = binned ? bin_of(v[i]) < bin : v[i] > last || (v[i] == last && (u32)index(i) <= cut.at);
        bits |= v[i] > bottom && in && likely(v[i]) ? 1u << i : 0u;
      }
      if (bits == 0) return;
      float u[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) u[i] = noise[min(index(i), a.vocab - 1)];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u64 o = entry_of(__builtin_fmaf(v[i] - top, rate, -log2_of(u[i])), (u32)index(i));
        best = ((bits >> i) & 1u) && o > best ? o : best;
      }
    });
  }
  best = block_max(best, sh);
  if (threadIdx.x == 0) {
    const int token = (int)(0xffffffffu - (u32)best);
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = (logit_at<TYPE>(row, token) - top) * (rate * kLn2) - __builtin_logf(total);
  }
}

int launch_sample(const SampleArgs &a, int32_t type, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == OWQ_TYPE_F16) owq_sample_kernel<OWQ_TYPE_F16><<<a.n_rows, kSampleThreads, 0, s>>>(a);
  else if (type == OWQ_TYPE_BF16) owq_sample_kernel<OWQ_TYPE_BF16><<<a.n_rows, kSampleThreads, 0, s>>>(a);
  else owq_sample_kernel<OWQ_TYPE_F32><<<a.n_rows, kSampleThreads, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace owq
