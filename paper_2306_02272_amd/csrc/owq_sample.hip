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

constexpr float kMassUnit = 0x1p31f;
constexpr int kList = 1024;         // candidates that are ranked against each other
constexpr int kBins = 1024;         // of 1/16 in log2 of the probability, for counts
constexpr int kMassBins = 4096;     // of 1/128, for masses: what lies 2^-32 below the largest has none

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
  return (u32)(__builtin_amdgcn_exp2f(apart(x, top) * rate) * kMassUnit);
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
__device__ __forceinline__ void clear_lists(SampleShared &sh) {
  if (threadIdx.x == 0) sh.n_sure = sh.n_list = 0;
  sh.list[threadIdx.x] = 0;
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
  const float rate = 2.f * kLog2e / (t > 0.f ? t : 1.f);      // of what lies between logits by halves
  const int k = a.top_k ? a.top_k[r] : 0;
  const float p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f;
  const float top = block_top(mine, sh);
  const bool by_k = t > 0.f && k >= 1 && k < a.vocab, short_k = by_k && k <= kList / 2, long_k = by_k && !short_k, by_p = t > 0.f && !by_k && p < 1.f;
  // Everything is measured from the largest logit, in log2 of the probability: sums with a logit itself would round at its size,
  // not at the difference's, and overflow at small temperatures.
  const float half_top = 0.5f * top;
  auto below = [&](float v) { return __builtin_fmaf(-0.5f, v, half_top) * rate; };      // apart(top, v)
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
    constexpr float kLowest = -3.402823466e38f;      // not -infinity: what stands past the row's end is no candidate
    lo = bin >= kBins - 1 || all < (u32)k ? kLowest : fmaxf(top - ((float)(bin + 1) * 0.125f / rate) * 1.00001f, kLowest);
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
    return entry_of(__builtin_fmaf(apart(entry_logit(e), top), rate, -log2_of(noise[entry_at(e)])), entry_at(e));
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
        const u64 o = entry_of(__builtin_fmaf(apart(v[i], top), rate, -log2_of(u[i])), (u32)index(i));
        best = ((bits >> i) & 1u) && o > best ? o : best;
      }
    });
  }
  best = block_max(best, sh);
  if (threadIdx.x == 0) {
    const int token = (int)(0xffffffffu - (u32)best);
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = apart(logit_at<TYPE>(row, token), top) * (rate * kLn2) - __builtin_logf(total);
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
