// Dropout whose mask is a function of (seed, step, site, row, column) and is never stored; with the residual sum.
//
// A thread takes pieces of eight elements: one Philox call (ten rounds, two 32 x 32 -> 64 products each) for their 128 bits.
// Memory bounds it: 2048 rows of 16 384 bf16 take 24 us (134 MB, 5.5 TB/s; vector instructions, most of them Philox's, four fifths
// of the cycles), 40 rows of 768 2.4 us, most of it the launch.
#include <hip/hip_runtime.h>

#include "owq_random_device.h"

namespace owq {

// A workgroup is `across` pieces wide and 256 / across rows high.
template <class E>
__global__ __launch_bounds__(256) void owq_dropout_kernel(DropoutArgs a, int across_log2) {
  const int across = 1 << across_log2, down = 256 >> across_log2;
  const DropKey key = drop_key(a.drop);
  const int units = ((a.width - 1) >> 3) + 1;
  for (int64_t r = (int64_t)blockIdx.y * down + (threadIdx.x >> across_log2); r < a.n_rows; r += (int64_t)gridDim.y * down) {
    const void *x = row_at<E>(a.x, r, a.x_row);
    const void *res = a.residual ? row_at<E>(a.residual, r, a.residual_row) : nullptr;
    void *out = row_at<E>(a.out, r, a.width);
    for (int u = (int)blockIdx.x * across + (threadIdx.x & (across - 1)); u < units; u += (int)gridDim.x * across) {
      Piece<E> px, pr;
      const int64_t at = (int64_t)u * (8 * Piece<E>::kSize);      // a row may be 2^31 elements long
      const int left = a.width - 8 * u;
      px.load(static_cast<const char *>(x) + at, left);
      if (res) pr.load(static_cast<const char *>(res) + at, left);
      float f[8], g[8];
      px.get(f);
      if (a.drop.threshold > 0) {
        const Stays on(a.drop, key, (u32)u, (u32)r);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = on(j) ? f[j] * a.drop.scale : 0.f;
      }
      if (res) {
        pr.get(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] += g[j];
      }
      px.put(f);
      px.template store<false>(static_cast<char *>(out) + at, left);
    }
  }
}

int launch_dropout(const DropoutArgs &a, int32_t type, void *stream) {
  const int units = (a.width - 1) / 8 + 1;
  int across_log2 = 0;
  while (across_log2 < 8 && (1 << across_log2) < units) ++across_log2;
  const int64_t down = 256 >> across_log2, tall = (a.n_rows + down - 1) / down;
  const int wide = (units - 1) / (1 << across_log2) + 1;
  const dim3 grid((unsigned)(wide < 65536 ? wide : 65536), (unsigned)(tall < 8192 ? tall : 8192));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == OWQ_TYPE_F16) owq_dropout_kernel<F16><<<grid, 256, 0, s>>>(a, across_log2);
  else if (type == OWQ_TYPE_BF16) owq_dropout_kernel<BF16><<<grid, 256, 0, s>>>(a, across_log2);
  else owq_dropout_kernel<F32><<<grid, 256, 0, s>>>(a, across_log2);
  return (int)hipGetLastError();
}

}  // namespace owq
