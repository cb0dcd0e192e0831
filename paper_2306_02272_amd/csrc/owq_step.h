// Launchers of the operators between two layers (owq_rope.hip, owq_cache.hip, owq_attend.hip,
// owq_sample.hip), called by the checked entry points in owq_step.cpp.  All return a hipError_t as int.
#pragma once
#include <cstddef>
#include <cstdint>

#include "owq.h"

namespace owq {

struct RopePtrs {
  const void *q, *k, *wq, *wk;
  const float *cos, *sin;
  const int32_t *positions;
  const void *dq_out, *dk_out;   // backward only
  void *q_out, *k_out;           // the gradients of q and k in the backward
  float *dwq, *dwk;              // backward only
  float *partial;                // backward only: one row of 2 head_dim sums per workgroup
};

int launch_rope(const owq_rope_desc_t &d, const RopePtrs &p, void *stream);
int32_t rope_backward_blocks(const owq_rope_desc_t &d);
int launch_rope_backward(const owq_rope_desc_t &d, const RopePtrs &p, void *stream);

// Where the tokens of a ragged batch of sequences lie in the cache.
struct CacheView {
  uint8_t *pages;
  const int32_t *table, *starts, *lengths;
  int64_t page_bytes;
  int32_t n_pages, page_shift;    // log2 of the 32-token tiles of a page
  int32_t kv_heads, head_dim;
  int32_t table_stride, tile_bytes;
  int32_t n_seqs, n_rows;
};
CacheView cache_view(const owq_cache_desc_t &d, const void *pages, const int32_t *table, const int32_t *starts,
                     const int32_t *lengths, int32_t n_rows);

int launch_cache_append(const CacheView &c, const void *k, const void *v, int32_t type, int32_t max_new, int64_t k_row,
                        int64_t k_head, int64_t v_row, int64_t v_head, void *stream);
int launch_cache_read(const CacheView &c, void *k_out, void *v_out, int32_t type, int32_t max_len, void *stream);

// The work split of an attention call: everything that follows from the description alone.
struct AttendPlan {
  int32_t group;        // query heads per key/value head
  bool fits;            // a launch can hold it
  bool many;            // whole spans of keys for 128 rows; else ranges of them for 16 or 32, and:
  int32_t rows;         // most rows (new tokens x group) of a sequence and key/value head
  int32_t col_tiles;    // 16-row tiles of a wave
  int32_t waves;        // of a workgroup
  int32_t blocks, slot_rows;   // blocks of so many rows
  bool whole;           // one workgroup per sequence, head and block
  int32_t ranges, least_tiles, workgroups;
  size_t slots;         // rows of partial results
  size_t workspace;
};
AttendPlan attend_plan(const owq_cache_desc_t &d, const owq_attention_desc_t &a);
int launch_attend(const CacheView &c, const owq_attention_desc_t &a, const AttendPlan &p, const void *q, void *out, float *lse,
                  void *workspace, void *stream);

struct SampleArgs {
  const void *logits;
  const float *noise, *temperature, *top_p, *min_p;
  const int32_t *top_k;
  int32_t *token;
  float *logprob;
  int64_t logits_row, noise_row;
  int32_t n_rows, vocab;
};
int launch_sample(const SampleArgs &a, int32_t type, void *stream);

}  // namespace owq
