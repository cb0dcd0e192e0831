// Log-probabilities of given tokens, entropy and the likeliest tokens of every row of logits, and the gradient to the logits.
//
// Forward: a workgroup takes a row in one pass.  With m the largest logit so far and d = scale (x - m), a thread
// holds S = sum e^d and W = sum e^d d; when m grows to m', both are scaled: S' = f S, W' = f (W + (m - m') scale S), f = e^((m - m') scale).
//     ln p = d - ln S,   entropy = ln S - W / S
// Nothing is measured from anything but the largest logit, so that an offset of all logits costs no digits.
// Alternatives: the K-th of the threads' largest logits lies at or below the row's K-th; threads whose largest does not lie
// below that list their logits that do not either, and those are ranked.
// Backward: element by element, with p from the forward's m and ln S.
//
// A thread adds a batch's terms by themselves before they join its sums, so that ln S of a row of 131 077 equal terms on 128 threads is off
// by 74 steps of 2^-24 at most, where one sum was by 947.
//
// 2048 rows of 50 272 bf16 logits take 38 to 43 us (206 MB at 5.1 TB/s, the rate of a large copy, are 40.4, at 6.05, that of a large
// sum, 34): memory, with vector instructions in 88 % of the cycles; 333 rows of 50 272 fp32 ones with five alternatives 18 (13.1
// and 11.1; 333 workgroups do not divide by 256 compute units, and the list is made after the pass); one row of 32 000 with 20
// alternatives 7.3, 4.3 without them: one workgroup's loads, exponentials and join, then counts, winners, list and ranks, each behind a
// barrier; 32 rows of 120 000 11.5, one workgroup a row: 32 of 256 compute units at work.  Gradients of 2048 rows of 50 272 74 to 78 us
// (80.8 by the copy).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "owq_ends.h"
#include "owq_logits_device.h"
#include "owq_random_device.h"

namespace owq {

constexpr float kLowest = -3.402823466e38f;
constexpr float kVanishes = -200.f;      // 2^-200 is 0 in binary32; keeps 0 times infinity out of the sums

// Largest logit of a set, S and W about it.  rate: 2 scale / ln 2, of what lies between logits by halves.
struct Mass {
  float m, s, w;
  __device__ __forceinline__ void raise(float to, float rate) {
    const float d = fmaxf(apart(m, to) * rate, kVanishes), f = __builtin_amdgcn_exp2f(d);
    w = f * __builtin_fmaf(s, d, w);
    s *= f;
    m = to;
  }
  __device__ __forceinline__ void add(float v, float rate) {
    const float d = apart(v, m) * rate, e = __builtin_amdgcn_exp2f(d);
    s += e;
    w = __builtin_fmaf(e, fmaxf(d, kVanishes), w);
  }
};

// A row by THREADS threads: LOGITS each at a time, the next ones asked for before; what lies beside the row's 16-byte units is
// one logit of some threads.
template <int TYPE, int THREADS, int LOGITS = 16>
struct RowPass {
  typedef RowView<TYPE> View;
  static constexpr int kPer = View::kPer, kUnits = LOGITS / kPer, kStep = THREADS * kUnits;
  static __device__ __forceinline__ void fetch(const View &x, int base, u32x4 (&v)[kUnits]) {
#pragma unroll
    for (int j = 0; j < kUnits; ++j) v[j] = x.units[min(base + j * THREADS + (int)threadIdx.x, x.n_units - 1)];
  }
  static __device__ __forceinline__ Mass run(const View &x, float rate) {
    Mass a = {kLowest, 0.f, 0.f};
    u32x4 next[kUnits];
    if (x.n_units > 0) fetch(x, 0, next);
    if ((int)threadIdx.x < x.n_rest) {
      const float v = logit_at<TYPE>(x.row, x.rest(threadIdx.x));
      a.m = fmaxf(v, kLowest);
      a.add(v, rate);
    }
    const u32 low = TYPE == OWQ_TYPE_F32 ? 0xff800000u : TYPE == OWQ_TYPE_F16 ? 0xfc00fc00u : 0xff80ff80u;   // -infinity past the end
    for (int base = 0; base < x.n_units; base += kStep) {
      u32x4 now[kUnits];
#pragma unroll
      for (int j = 0; j < kUnits; ++j) now[j] = next[j];
      const bool last = base + kStep >= x.n_units;         // the same for the whole workgroup
      if (last) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j)
          if (base + j * THREADS + (int)threadIdx.x >= x.n_units) now[j] = (u32x4){low, low, low, low};
      } else {
        fetch(x, base + kStep, next);
      }
      float v[LOGITS], top = a.m;
#pragma unroll
      for (int i = 0; i < LOGITS; ++i) {
        v[i] = View::get(now[i / kPer], i % kPer);
        top = fmaxf(top, v[i]);
      }
      a.raise(top, rate);
      // these by themselves first: a sum of 16 and as many additions as batches, not 16 times as many, stand behind each other
      Mass b = {a.m, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < LOGITS; ++i) b.add(v[i], rate);
      a.s += b.s;
      a.w += b.w;
    }
    return a;
  }
  // over the workgroup, in every thread; part: [THREADS / 64]
  static __device__ __forceinline__ Mass join(Mass a, float rate, Mass *part) {
    a.raise(wave_max(a.m), rate);
    a.s = wave_sum(rounded(a.s));
    a.w = wave_sum(rounded(a.w));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
    __syncthreads();
    const int w = threadIdx.x & 15;
    a = w < THREADS / 64 ? part[w] : Mass{kLowest, 0.f, 0.f};
    a.raise(lanes_max<16>(a.m), rate);
    a.s = lanes_sum<16>(rounded(a.s));
    a.w = lanes_sum<16>(rounded(a.w));
    return a;
  }
};

template <int TYPE>
__device__ __forceinline__ const void *logits_row(const LogprobArgs &a, int64_t r) {
  return static_cast<const char *>(a.logits) + r * a.logits_row * (TYPE == OWQ_TYPE_F32 ? 4 : 2);
}

// What the row's numbers are made of; false where there is no distribution (a NaN, an infinity, nothing above -infinity).
template <int TYPE>
__device__ __forceinline__ bool store_row(const LogprobArgs &a, int64_t r, const Mass &all, const void *row, float *log_s) {
  const float nan = __builtin_nanf("");
  const bool good = all.s > 0.f && all.m < __builtin_inff();
  *log_s = good ? __builtin_logf(all.s) : nan;
  if (threadIdx.x == 0) {
    a.stats[r] = good ? all.m : nan;
    a.stats[(int64_t)a.n_rows + r] = *log_s;
    a.stats[2 * (int64_t)a.n_rows + r] = good ? *log_s - kLn2 * (all.w / all.s) : nan;
    if (a.targets) {
      const int target = a.targets[r];
      a.logprob[r] = (uint32_t)target < (uint32_t)a.vocab ? apart(logit_at<TYPE>(row, target), all.m) * (2.f * a.scale) - *log_s : 0.f;
    }
  }
  return good;
}

template <int TYPE, int THREADS>
__global__ __launch_bounds__(THREADS) void owq_logprob_kernel(LogprobArgs a) {
  __shared__ Mass part[THREADS / 64];
  const float rate = 2.f * kLog2e * a.scale;
  for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const void *row = logits_row<TYPE>(a, r);
    const RowView<TYPE> x(row, a.vocab);
    const Mass all = RowPass<TYPE, THREADS>::join(RowPass<TYPE, THREADS>::run(x, rate), rate, part);
    float log_s;
    store_row<TYPE>(a, r, all, row, &log_s);
    __syncthreads();       // the next row writes `part`
  }
}

// Tokens that are candidates, in LDS, in no order; entries past CAP are counted only.
template <int CAP>
struct Candidates {
  u64 entry[CAP];
  u32 n;
  __device__ __forceinline__ void clear() {
    entry[threadIdx.x] = 0;
    if (threadIdx.x == 0) n = 0;
  }
  // the logits at first + j for the set bits j; by whole waves
  template <int TYPE>
  __device__ __forceinline__ void add(const void *row, u32 bits, int first) {
    if (!__any(bits != 0)) return;
    const u32 mine = (u32)__popc(bits);
    const u32 sum = wave_scan(mine, 0u, [](u32 a, u32 b) { return a + b; });
    u32 base = 0;
    if ((threadIdx.x & 63) == 63) base = atomicAdd(&n, sum);
    u32 place = (u32)__builtin_amdgcn_readlane((int)base, 63) + sum - mine;
#pragma unroll 1
    for (; bits != 0 && place < (u32)CAP; bits &= bits - 1, ++place) {
      const int i = first + __ffs(bits) - 1;
      entry[place] = entry_of(logit_at<TYPE>(row, i), (u32)i);
    }
  }
};

// The row's k largest logits, lower indices first of equal ones, into an empty list, where k of them lie above -infinity: the k-th's
// key by four histograms of eight bits.  For rows with many equal logits.
template <int TYPE, int THREADS>
__device__ void list_largest(const void *row, int vocab, u32 k, Candidates<THREADS> &list, u32 *bins, u32 *found) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));      // what follows from it is not kept in registers through the pass above
  u32 key = 0, above = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = tid; i < 256; i += THREADS) bins[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < vocab; i += THREADS) {
      const u32 o = key_of(logit_at<TYPE>(row, i));
      if (shift == 24 || (o >> (shift + 8)) == (key >> (shift + 8))) atomicAdd(&bins[(o >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 64) {            // four bins a lane, the largest first
      u32 own[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += own[j] = bins[255 - 4 * tid - j];
      u32 before = above + wave_scan(sum, 0u, [](u32 a, u32 b) { return a + b; }) - sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < k && before + own[j] >= k) {
          found[0] = 255u - 4u * (u32)tid - (u32)j;
          found[1] = before;
        }
        before += own[j];
      }
    }
    __syncthreads();
    key |= found[0] << shift;
    above = found[1];
  }
  // those above it, and as many equal ones as are left, counted in the order of indices
  u32 left = k - above;
#pragma unroll 1
  for (int base = 0; base < vocab; base += THREADS) {
    const int i = base + tid;
    const u32 o = i < vocab ? key_of(logit_at<TYPE>(row, i)) : 0u;
    list.template add<TYPE>(row, o > key ? 1u : 0u, i);
    if (left == 0) continue;
    const u64 equal = __ballot(o == key);
    __syncthreads();
    if ((tid & 63) == 0) bins[tid >> 6] = (u32)__popcll(equal);
    __syncthreads();
    u32 rank = (u32)__popcll(equal & ((1ull << (tid & 63)) - 1ull)), sum = 0;
#pragma unroll 1
    for (int w = 0; w < THREADS / 64; ++w) {
      rank += w < (int)(tid >> 6) ? bins[w] : 0u;
      sum += bins[w];
    }
    list.template add<TYPE>(row, o == key && rank < left ? 1u : 0u, i);
    left = sum < left ? left - sum : 0;
  }
  __syncthreads();
}

template <int TYPE>
__device__ __forceinline__ void no_tokens(const LogprobArgs &a, int64_t out, int from, float lp) {
  for (int i = from + (int)threadIdx.x; i < a.top; i += blockDim.x) {
    a.top_token[out + i] = -1;
    a.top_logprob[out + i] = lp;
  }
}

// With alternatives.  The K-th of the threads' largest logits lies at or below the row's K-th; it is counted by bins of 1/16 in log2
// of the probability.  The logits of threads whose largest does not lie below that bin, and that do not either, are listed, 64 lanes a
// thread's, and the list is ranked.
template <int TYPE, int THREADS>
__global__ __launch_bounds__(THREADS, 8) void owq_logprob_top_kernel(LogprobArgs a) {
  constexpr int kPer = RowView<TYPE>::kPer;
  constexpr u32 kBins = 1024;
  __shared__ Mass part[THREADS / 64];
  __shared__ __attribute__((aligned(16))) u32 bins[kBins];
  __shared__ u32 winners[THREADS], n_winners, found[2];
  __shared__ Candidates<THREADS> list;
  const float rate = 2.f * kLog2e * a.scale;
  const int lane = threadIdx.x & 63;
  for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const void *row = logits_row<TYPE>(a, r);
    const RowView<TYPE> x(row, a.vocab);
    list.clear();
    if (threadIdx.x == 0) n_winners = 0;
    for (u32 i = threadIdx.x; i < kBins; i += THREADS) bins[i] = 0;
    typedef RowPass<TYPE, THREADS, TYPE == OWQ_TYPE_F32 ? 8 : 16> Pass;      // 64 registers: two workgroups of 1024 threads
    Mass all = Pass::run(x, rate);
    const float mine = all.m;
    all = Pass::join(all, rate, part);
    const float m = all.m;
    float log_s;
    const bool good = store_row<TYPE>(a, r, all, row, &log_s);
    const int64_t out = r * a.top;
    if (!good) {
      no_tokens<TYPE>(a, out, 0, __builtin_nanf(""));
      __syncthreads();
      continue;
    }
    const float d = apart(m, mine) * rate * 16.f;
    atomicAdd(&bins[d < (float)(kBins - 1) ? (u32)(int)d : kBins - 1], 1u);
    __syncthreads();
    u32 bin;
    {      // every wave for itself: 16 bins a lane
      u32x4 own[4];
      u32 sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        own[j] = reinterpret_cast<const u32x4 *>(bins)[4 * lane + j];
        sum += own[j].x + own[j].y + own[j].z + own[j].w;
      }
      u32 before = wave_scan(sum, 0u, [](u32 p, u32 q) { return p + q; }) - sum;
      const u64 is = __ballot(before < (u32)a.top && before + sum >= (u32)a.top);
      u32 at = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        before += own[j >> 2][j & 3];
        at += before < (u32)a.top ? 1u : 0u;
      }
      const int who = __builtin_ctzll(is);
      bin = (u32)who * 16u + (u32)__builtin_amdgcn_readlane((int)at, who);
    }
    // a little below the bin's edge, so that rounding leaves none of its logits out; the last bin is open
    const float lo = bin >= kBins - 1 ? kLowest : fmaxf(m - ((float)(bin + 1) * 0.125f / rate) * 1.00001f, kLowest);
    if (mine >= lo) winners[atomicAdd(&n_winners, 1u)] = threadIdx.x;
    __syncthreads();
    const u32 n_won = n_winners;
#pragma unroll 1
    for (u32 i = threadIdx.x >> 6; i < n_won; i += THREADS / 64) {
      const int who = __builtin_amdgcn_readfirstlane((int)winners[i]);
#pragma unroll 1
      for (int first = who; first < x.n_units; first += THREADS * 64) {
        const int u = first + THREADS * lane;
        const bool on = u < x.n_units;
        const u32x4 v = x.units[on ? u : first];
        u32 bits = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) bits |= on && RowView<TYPE>::get(v, j) >= lo ? 1u << j : 0u;
        list.template add<TYPE>(row, bits, x.first + u * kPer);
      }
      if (who < x.n_rest) {
        const int at = x.rest(who);
        list.template add<TYPE>(row, lane == 0 && logit_at<TYPE>(row, at) >= lo ? 1u : 0u, at);
      }
    }
    __syncthreads();
    if (list.n > (u32)THREADS) {
      __syncthreads();
      list.clear();
      list_largest<TYPE, THREADS>(row, a.vocab, (u32)a.top, list, bins, found);
    }
    const u32 n = list.n < (u32)THREADS ? list.n : (u32)THREADS;
    if (threadIdx.x < n) {
      const u64 me = list.entry[threadIdx.x];
      u32 rank = 0;
#pragma unroll 1
      for (u32 j = 0; j < n; j += 4)
#pragma unroll
        for (int i = 0; i < 4; ++i) rank += list.entry[j + i] > me ? 1u : 0u;      // past the end: 0, before nothing
      if (rank < (u32)a.top) {
        a.top_token[out + rank] = (int32_t)entry_at(me);
        a.top_logprob[out + rank] = apart(entry_logit(me), m) * (2.f * a.scale) - log_s;
      }
    }
    no_tokens<TYPE>(a, out, (int)n, -__builtin_inff());
    __syncthreads();
  }
}

// Threads of a row: 2^18 over all rows, so that the chip is full and the waves of a workgroup have several batches to read ahead
// in, but 16 logits for each at least.  Times in us by threads: 32000 bf16 logits, 768 rows: 12.1 with 1024, 11.7 with 512, 10.9 with
// 256, 12.7 with 128; 2048 rows of 50 272: 50.1, 48.2, 45.6, 43.5; 32 rows of 120 000: 11.0, 10.6, 13.0, 23.0.
template <int TYPE>
static void launch_type(const LogprobArgs &a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20);
  if (a.top > 0) {
    // Many rows, few alternatives: with 2048 rows of 32 000 bf16 logits 33.2 us for five by 256 threads a row, 38.4 by 1024, and 54.6
    // and 58.4 for 64; fp32 logits 55.3 and 54.6, 82.3 and 70.9; one row 7.3 and 6.3; 2048 rows of 1000 32.0 and 49.6 for 64.
    if (a.n_rows > 512 && a.top <= (a.vocab <= 8192 ? 64 : 16)) owq_logprob_top_kernel<TYPE, 256><<<grid, 256, 0, s>>>(a);
    else owq_logprob_top_kernel<TYPE, kSampleThreads><<<grid, kSampleThreads, 0, s>>>(a);
    return;
  }
  int threads = kSampleThreads;
  while (threads > 64 && (threads * 16 > a.vocab || (threads > 128 && (int64_t)threads * a.n_rows > (1 << 18)))) threads /= 2;
  switch (threads) {
    case 64: owq_logprob_kernel<TYPE, 64><<<grid, 64, 0, s>>>(a); break;
    case 128: owq_logprob_kernel<TYPE, 128><<<grid, 128, 0, s>>>(a); break;
    case 256: owq_logprob_kernel<TYPE, 256><<<grid, 256, 0, s>>>(a); break;
    case 512: owq_logprob_kernel<TYPE, 512><<<grid, 512, 0, s>>>(a); break;
    default: owq_logprob_kernel<TYPE, kSampleThreads><<<grid, kSampleThreads, 0, s>>>(a);
  }
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
  const float rate = 2.f * kLog2e * a.scale;
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
          const float l = __builtin_fmaf(apart(f[j], m), rate, -log2_s);
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
