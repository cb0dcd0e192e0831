// extern "C" entry points of the operators between two layers: argument checks only; see include/owq.h.
#include "owq_step.h"

#include <algorithm>

using namespace owq;

static bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
static bool rows16(const void *p, int64_t a, int64_t b) { return aligned(p, 16) && a % 8 == 0 && b % 8 == 0; }

static owq_status_t check_rope(const owq_rope_desc_t *d) {
  if (!d) return OWQ_ERR_NULL;
  if (d->n_tokens < 0 || d->q_heads < 1 || d->kv_heads < 0 || d->n_positions < 1) return OWQ_ERR_SHAPE;
  if ((int64_t)d->q_heads + d->kv_heads > 65536) return OWQ_ERR_SHAPE;
  if (d->type != OWQ_TYPE_F16 && d->type != OWQ_TYPE_BF16) return OWQ_ERR_TYPE;
  if (d->head_dim < 16 || d->head_dim > 256 || d->head_dim % 8 != 0) return OWQ_ERR_UNSUPPORTED;
  if (d->rotary_dim < 16 || d->rotary_dim > d->head_dim || d->rotary_dim % 16 != 0) return OWQ_ERR_UNSUPPORTED;
  if (!(d->eps >= 0.f)) return OWQ_ERR_SHAPE;
  return OWQ_OK;
}

extern "C" {

owq_status_t owq_qk_norm_rope(const owq_rope_desc_t *d, const void *q, const void *k, const void *wq, const void *wk,
                              const float *cos, const float *sin, const int32_t *positions, void *q_out, void *k_out,
                              void *stream) {
  const owq_status_t st = check_rope(d);
  if (st != OWQ_OK) return st;
  if (d->n_tokens == 0) return OWQ_OK;
  if (!q || !q_out || !cos || !sin || !positions || (d->kv_heads > 0 && (!k || !k_out))) return OWQ_ERR_NULL;
  if (!rows16(q, d->q_token, d->q_head) || !aligned(q_out, 16) || !aligned(wq, 16) || !aligned(wk, 16)) return OWQ_ERR_BUFFER;
  if (d->kv_heads > 0 && (!rows16(k, d->k_token, d->k_head) || !aligned(k_out, 16))) return OWQ_ERR_BUFFER;
  if (!aligned(cos, 4) || !aligned(sin, 4) || !aligned(positions, 4)) return OWQ_ERR_BUFFER;
  RopePtrs p{};
  p.q = q, p.k = k, p.wq = wq, p.wk = wk, p.cos = cos, p.sin = sin, p.positions = positions, p.q_out = q_out, p.k_out = k_out;
  return launch_rope(*d, p, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

owq_status_t owq_qk_norm_rope_backward_workspace_bytes(const owq_rope_desc_t *d, size_t *bytes) {
  const owq_status_t st = check_rope(d);
  if (st != OWQ_OK) return st;
  if (!bytes) return OWQ_ERR_NULL;
  *bytes = (size_t)rope_backward_blocks(*d) * 2 * d->head_dim * sizeof(float);
  return OWQ_OK;
}

owq_status_t owq_qk_norm_rope_backward(const owq_rope_desc_t *d, const void *dq_out, const void *dk_out, const void *q,
                                       const void *k, const void *wq, const void *wk, const float *cos, const float *sin,
                                       const int32_t *positions, void *dq, void *dk, float *dwq, float *dwk,
                                       void *workspace, size_t workspace_bytes, void *stream) {
  const owq_status_t st = check_rope(d);
  if (st != OWQ_OK) return st;
  if (!wq) dwq = nullptr;
  if (!wk) dwk = nullptr;
  if (d->n_tokens > 0) {
    if (!dq_out || !dq || !cos || !sin || !positions || (wq && !q)) return OWQ_ERR_NULL;
    if (d->kv_heads > 0 && (!dk_out || !dk || (wk && !k))) return OWQ_ERR_NULL;
    if (!rows16(dq_out, d->dq_token, d->dq_head) || !aligned(dq, 16)) return OWQ_ERR_BUFFER;
    if (wq && !rows16(q, d->q_token, d->q_head)) return OWQ_ERR_BUFFER;
    if (d->kv_heads > 0 && (!rows16(dk_out, d->dk_token, d->dk_head) || !aligned(dk, 16))) return OWQ_ERR_BUFFER;
    if (d->kv_heads > 0 && wk && !rows16(k, d->k_token, d->k_head)) return OWQ_ERR_BUFFER;
    if (!aligned(cos, 4) || !aligned(sin, 4) || !aligned(positions, 4)) return OWQ_ERR_BUFFER;
  }
  if (!aligned(wq, 16) || !aligned(wk, 16) || !aligned(dwq, 4) || !aligned(dwk, 4)) return OWQ_ERR_BUFFER;
  RopePtrs p{};
  p.q = q, p.k = k, p.wq = wq, p.wk = wk, p.cos = cos, p.sin = sin, p.positions = positions;
  p.dq_out = dq_out, p.dk_out = dk_out, p.q_out = dq, p.k_out = dk, p.dwq = dwq, p.dwk = dwk;
  if (dwq || dwk) {
    size_t need = 0;
    (void)owq_qk_norm_rope_backward_workspace_bytes(d, &need);
    if (need > 0 && !workspace) return OWQ_ERR_NULL;
    if (!aligned(workspace, 16) || workspace_bytes < need) return OWQ_ERR_BUFFER;
    p.partial = static_cast<float *>(workspace);
  }
  return launch_rope_backward(*d, p, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

static owq_status_t check_cache(const owq_cache_desc_t *d) {
  if (!d) return OWQ_ERR_NULL;
  if (d->n_pages < 1 || d->kv_heads < 1 || d->kv_heads > 65535 || d->n_seqs < 0 || d->n_seqs > 65535 || d->table_stride < 1) return OWQ_ERR_SHAPE;
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8 != 0) return OWQ_ERR_UNSUPPORTED;
  if (d->page_size < 32 || d->page_size > 65536 || (d->page_size & (d->page_size - 1)) != 0) return OWQ_ERR_UNSUPPORTED;
  return OWQ_OK;
}

owq_status_t owq_cache_page_bytes(const owq_cache_desc_t *d, size_t *bytes) {
  if (!d || !bytes) return OWQ_ERR_NULL;
  owq_cache_desc_t one = *d;       // the table's fields do not matter
  one.n_pages = 1, one.n_seqs = 1, one.table_stride = 1;
  const owq_status_t st = check_cache(&one);
  if (st != OWQ_OK) return st;
  *bytes = (size_t)cache_view(one, nullptr, nullptr, nullptr, nullptr, 0).page_bytes;
  return OWQ_OK;
}

static owq_status_t check_cache_pointers(const void *pages, const int32_t *table, const int32_t *starts) {
  if (!pages || !table || !starts) return OWQ_ERR_NULL;
  return aligned(pages, 16) && aligned(table, 4) && aligned(starts, 4) ? OWQ_OK : OWQ_ERR_BUFFER;
}

owq_status_t owq_cache_append(const owq_cache_desc_t *d, void *pages, const int32_t *page_table, const int32_t *starts,
                              const int32_t *lengths, const void *k, const void *v, int32_t type, int32_t n_rows,
                              int32_t max_new, int64_t k_row, int64_t k_head, int64_t v_row, int64_t v_head, void *stream) {
  owq_status_t st = check_cache(d);
  if (st != OWQ_OK) return st;
  if (type != OWQ_TYPE_F16 && type != OWQ_TYPE_BF16) return OWQ_ERR_TYPE;
  if (n_rows < 0 || max_new < 0) return OWQ_ERR_SHAPE;
  if (n_rows == 0 || max_new == 0 || d->n_seqs == 0) return OWQ_OK;
  st = check_cache_pointers(pages, page_table, starts);
  if (st != OWQ_OK) return st;
  if (!lengths || !k || !v) return OWQ_ERR_NULL;
  if (!aligned(lengths, 4) || !rows16(k, k_row, k_head) || !rows16(v, v_row, v_head)) return OWQ_ERR_BUFFER;
  const CacheView c = cache_view(*d, pages, page_table, starts, lengths, n_rows);
  return launch_cache_append(c, k, v, type, max_new, k_row, k_head, v_row, v_head, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

owq_status_t owq_cache_read(const owq_cache_desc_t *d, const void *pages, const int32_t *page_table, const int32_t *starts,
                            void *k_out, void *v_out, int32_t type, int32_t n_rows, int32_t max_len, void *stream) {
  owq_status_t st = check_cache(d);
  if (st != OWQ_OK) return st;
  if (type != OWQ_TYPE_F16 && type != OWQ_TYPE_BF16) return OWQ_ERR_TYPE;
  if (n_rows < 0 || max_len < 0) return OWQ_ERR_SHAPE;
  if (n_rows == 0 || max_len == 0 || d->n_seqs == 0) return OWQ_OK;
  st = check_cache_pointers(pages, page_table, starts);
  if (st != OWQ_OK) return st;
  if (!k_out || !v_out) return OWQ_ERR_NULL;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return OWQ_ERR_BUFFER;
  const CacheView c = cache_view(*d, pages, page_table, starts, nullptr, n_rows);
  return launch_cache_read(c, k_out, v_out, type, max_len, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

static owq_status_t check_attention(const owq_cache_desc_t *d, const owq_attention_desc_t *a) {
  const owq_status_t st = check_cache(d);
  if (st != OWQ_OK) return st;
  if (!a) return OWQ_ERR_NULL;
  if (a->type != OWQ_TYPE_F16 && a->type != OWQ_TYPE_BF16) return OWQ_ERR_TYPE;
  if (a->q_heads < 1 || a->q_heads % d->kv_heads != 0 || a->n_rows < 0 || a->max_new < 0 || a->max_len < 0 || a->window < 0 || a->sinks < 0)
    return OWQ_ERR_SHAPE;
  if ((int64_t)std::min(a->max_new, a->n_rows) * (a->q_heads / d->kv_heads) > (1 << 30)) return OWQ_ERR_SHAPE;
  if (a->scale != a->scale) return OWQ_ERR_SHAPE;
  return OWQ_OK;
}

// The work split goes by the least bounds that hold.
static owq_attention_desc_t tightened(const owq_attention_desc_t *a) {
  owq_attention_desc_t t = *a;
  t.max_new = std::min(a->max_new, a->n_rows);
  return t;
}

owq_status_t owq_cache_attention_workspace_bytes(const owq_cache_desc_t *d, const owq_attention_desc_t *a, size_t *bytes) {
  const owq_status_t st = check_attention(d, a);
  if (st != OWQ_OK) return st;
  if (!bytes) return OWQ_ERR_NULL;
  *bytes = 0;
  if (a->n_rows == 0 || a->max_new == 0 || d->n_seqs == 0) return OWQ_OK;
  const AttendPlan plan = attend_plan(*d, tightened(a));
  *bytes = plan.workspace;
  return plan.fits ? OWQ_OK : OWQ_ERR_SHAPE;
}

owq_status_t owq_cache_attention(const owq_cache_desc_t *d, const owq_attention_desc_t *a, const void *q, const void *pages,
                                 const int32_t *page_table, const int32_t *starts, const int32_t *lengths, void *out,
                                 float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  owq_status_t st = check_attention(d, a);
  if (st != OWQ_OK) return st;
  if (a->n_rows == 0 || a->max_new == 0 || d->n_seqs == 0) return OWQ_OK;
  st = check_cache_pointers(pages, page_table, starts);
  if (st != OWQ_OK) return st;
  if (!q || !lengths || !out) return OWQ_ERR_NULL;
  if (!rows16(q, a->q_row, a->q_head) || !aligned(out, 16) || !aligned(lengths, 4) || !aligned(lse, 4)) return OWQ_ERR_BUFFER;
  const owq_attention_desc_t t = tightened(a);
  const AttendPlan plan = attend_plan(*d, t);
  if (!plan.fits) return OWQ_ERR_SHAPE;
  if (plan.workspace > 0 && !workspace) return OWQ_ERR_NULL;
  if (plan.workspace > 0 && (!aligned(workspace, 256) || workspace_bytes < plan.workspace)) return OWQ_ERR_BUFFER;
  const CacheView c = cache_view(*d, pages, page_table, starts, lengths, a->n_rows);
  return launch_attend(c, t, plan, q, out, lse, workspace, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

static owq_status_t check_sample(int32_t n_rows, int32_t vocab, int32_t type) {
  if (n_rows < 0 || vocab < 1 || vocab > (1 << 24)) return OWQ_ERR_SHAPE;
  if (type != OWQ_TYPE_F16 && type != OWQ_TYPE_BF16 && type != OWQ_TYPE_F32) return OWQ_ERR_TYPE;
  return OWQ_OK;
}

owq_status_t owq_sample(const void *logits, int32_t type, int32_t n_rows, int32_t vocab, int64_t logits_row, const float *noise,
                        int64_t noise_row, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                        int32_t *token, float *logprob, void *stream) {
  const owq_status_t st = check_sample(n_rows, vocab, type);
  if (st != OWQ_OK) return st;
  if (n_rows == 0) return OWQ_OK;
  if (!logits || !token || (!noise && !temperature)) return OWQ_ERR_NULL;
  if (!aligned(logits, type == OWQ_TYPE_F32 ? 4 : 2) || !aligned(noise, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
      !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(token, 4) || !aligned(logprob, 4))
    return OWQ_ERR_BUFFER;
  const SampleArgs a{logits, noise, temperature, top_p, min_p, top_k, token, logprob, logits_row, noise_row, n_rows, vocab};
  return launch_sample(a, type, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

}  // extern "C"
