// Attention over the 4-bit cache, many rows per sequence and key/value head: prompts.  The waves of a workgroup take other
// rows of the same keys, whose words they find in the caches.
//
// Bound by the vector instructions around the matrix ones: some 370 for 32 rows and 32 keys of 128 columns beside 34, twelve
// per score and lane, the rest to unpack 16 words.  2048 tokens of 32/8 heads behind 4100 others in 258 us, 667 TFLOP/s (a
// product of 8192 x 8192 x 8192: 1156).  32 rows per wave: with 16, in four waves per SIMD, 265 us where this took 243, with
// 64, which do not fit the registers, 931; with operands unpacked once per workgroup and passed through LDS, 264.
#include <hip/hip_runtime.h>

#include "owq_attend_device.h"

namespace owq {

constexpr int kCols = 2;       // 16-row tiles of a wave

template <int STEPS>
__global__ __launch_bounds__(64 * kWaves, 2) void owq_attend_many_kernel(AttendArgs a, bool paired) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quad = lane >> 4, col = lane & 15;
  // Causal rows see ever more keys: of the workgroups that share a compute unit (256 apart, where there are two), one comes
  // from the front and one from the back.
  int block_x = blockIdx.x, head = blockIdx.y, b = blockIdx.z;
  if (paired) {
    u32 id = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
    if ((id & 256u) && (id | 255u) < gridDim.x * gridDim.y * gridDim.z) id ^= 255u;
    block_x = id % gridDim.x, head = id / gridDim.x % gridDim.y, b = id / gridDim.x / gridDim.y;
  }
  const Sequence sq = sequence_of(a, b);
  const int first = (block_x * kWaves + wave) * 16 * kCols;
  if (first >= sq.n_rows) return;
  const int last = (first + 16 * kCols < sq.n_rows ? first + 16 * kCols : sq.n_rows) - 1;
  const int pa = sq.p0 + first / a.group, pb = sq.p0 + last / a.group;
  const Span span = visible_tiles(a, pa, pb);
  Rows<STEPS, kCols> w;
  attend_span<false, 1>(a, sq, span, b, head, first, pa, pb, 0, span.count, 0, lane, w);
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    const float l = quads_sum(w.l[n]), low = quads_sum(w.low[n]);
    const int row = first + 16 * n + col;
    const int token = row / a.group;
    const int64_t at = (int64_t)sq.row0 + token;
    if (row >= sq.n_rows || at < 0 || at >= a.c.n_rows) continue;
    const int h = head * a.group + row - token * a.group;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    u32 *out = a.out + (at * a.q_heads + h) * (a.c.head_dim / 2);
#pragma unroll
    for (int d = 0; d < 2 * STEPS; ++d) {
      const int dim = 16 * d + 4 * quad;
      if (dim >= a.c.head_dim) continue;
      float o[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] = __builtin_fmaf(w.acc[n][d][r] - w.mid[n][r], 0x1p20f, low) * inv;
      *reinterpret_cast<u32x2 *>(out + dim / 2) =
          a.bf16 ? (u32x2){BF16::pack(o[0], o[1]), BF16::pack(o[2], o[3])} : (u32x2){F16::pack(o[0], o[1]), F16::pack(o[2], o[3])};
    }
    if (a.lse != nullptr && quad == 0) a.lse[at * a.q_heads + h] = lse_of(w.ref[n], l);
  }
}

template <int STEPS>
void launch_attend_many(const AttendArgs &a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.max_new * a.group;
  constexpr int block = 16 * kCols * kWaves;
  const dim3 grid((unsigned)((rows + block - 1) / block), (unsigned)a.c.kv_heads, (unsigned)a.c.n_seqs);
  const bool paired = (int64_t)grid.x * grid.y * grid.z < (1ll << 31);
  owq_attend_many_kernel<STEPS><<<grid, 64 * kWaves, 0, stream>>>(a, paired);
}
template void launch_attend_many<1>(const AttendArgs &, hipStream_t);
template void launch_attend_many<2>(const AttendArgs &, hipStream_t);
template void launch_attend_many<3>(const AttendArgs &, hipStream_t);
template void launch_attend_many<4>(const AttendArgs &, hipStream_t);

}  // namespace owq
