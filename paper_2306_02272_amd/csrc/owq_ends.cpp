// extern "C" entry points of the operators at the ends of a block and of a tuning step: argument checks only; see
// include/owq.h.
#include "owq_ends.h"

#include <cmath>

using namespace owq;

static bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
static uintptr_t size_of(int32_t type) { return type == OWQ_TYPE_F32 ? 4 : 2; }

// p as 16 bits; false if it is none
static bool dropping(const uint64_t *rng, float p, int32_t site, Dropping *d) {
  if (!(p >= 0.f && p <= 65535.f / 65536.f)) return false;
  const uint32_t t = (uint32_t)std::rint((double)p * 65536.0);
  *d = Dropping{rng, t, (float)(65536.0 / (65536.0 - t)), site};
  return true;
}

extern "C" {

owq_status_t owq_dropout(const void *x, const void *residual, int32_t type, int32_t n_rows, int32_t width, int64_t x_row,
                         int64_t residual_row, const uint64_t *rng, float p, int32_t site, void *out, void *stream) {
  if (n_rows < 0 || width < 0) return OWQ_ERR_SHAPE;
  if (type != OWQ_TYPE_F16 && type != OWQ_TYPE_BF16 && type != OWQ_TYPE_F32) return OWQ_ERR_TYPE;
  Dropping drop;
  if (!dropping(rng, p, site, &drop)) return OWQ_ERR_SHAPE;
  if (n_rows == 0 || width == 0) return OWQ_OK;
  if (!x || !out || (drop.threshold > 0 && !rng)) return OWQ_ERR_NULL;
  if (!aligned(x, size_of(type)) || !aligned(residual, size_of(type)) || !aligned(out, size_of(type)) || !aligned(rng, 8)) return OWQ_ERR_BUFFER;
  const DropoutArgs a{x, residual, out, x_row, residual_row, n_rows, width, drop};
  return launch_dropout(a, type, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

static owq_status_t check_norm(const owq_norm_desc_t *d) {
  if (!d) return OWQ_ERR_NULL;
  if (d->n_tokens < 0 || d->width < 1) return OWQ_ERR_SHAPE;
  if (d->type != OWQ_TYPE_F16 && d->type != OWQ_TYPE_BF16) return OWQ_ERR_TYPE;
  if (d->h_type != d->type && d->h_type != OWQ_TYPE_F32) return OWQ_ERR_TYPE;
  if (d->width > OWQ_NORM_MAX_WIDTH) return OWQ_ERR_UNSUPPORTED;
  if (d->post < OWQ_NORM_NONE || d->post > OWQ_NORM_LAYER || d->norm < OWQ_NORM_NONE || d->norm > OWQ_NORM_LAYER) return OWQ_ERR_SHAPE;
  if (d->gate < OWQ_GATE_NONE || d->gate > OWQ_GATE_TOKEN) return OWQ_ERR_SHAPE;
  if (!(d->eps >= 0.f) || d->h_scale != d->h_scale || d->branch_scale != d->branch_scale) return OWQ_ERR_SHAPE;
  Dropping drop;
  return dropping(nullptr, d->p, d->site, &drop) ? OWQ_OK : OWQ_ERR_SHAPE;
}

static NormArgs norm_args(const owq_norm_desc_t *d, const uint64_t *rng) {
  NormArgs a{};
  a.h_row = d->h_row, a.branch_row = d->branch_row, a.gate_row = d->gate == OWQ_GATE_TOKEN ? d->gate_row : 0;
  a.total_row = d->total_row, a.dy_row = d->dy_row, a.dtotal_row = d->dtotal_row;
  a.n_tokens = d->n_tokens, a.width = d->width, a.post = d->post, a.norm = d->norm;
  a.eps = d->eps, a.h_scale = d->h_scale, a.branch_scale = d->branch_scale;
  (void)dropping(rng, d->p, d->site, &a.drop);
  a.sum_w = a.sum_b = a.sum_post_w = a.sum_post_b = a.sum_gate = -1;
  return a;
}

owq_status_t owq_residual_norm(const owq_norm_desc_t *d, const void *h, const void *branch, const void *gate,
                               const void *post_weight, const void *post_bias, const void *weight, const void *bias,
                               const uint64_t *rng, void *total, void *y, void *stream) {
  const owq_status_t st = check_norm(d);
  if (st != OWQ_OK) return st;
  if (d->n_tokens == 0) return OWQ_OK;
  if (!branch && (d->gate != OWQ_GATE_NONE || d->post != OWQ_NORM_NONE || d->p != 0.f)) return OWQ_ERR_NULL;
  NormArgs a = norm_args(d, rng);
  if (!h || (d->gate != OWQ_GATE_NONE && !gate) || (a.drop.threshold > 0 && !rng) || (d->norm != OWQ_NORM_NONE && !y)) return OWQ_ERR_NULL;
  const uintptr_t hs = size_of(d->h_type);
  if (!aligned(h, hs) || !aligned(total, hs) || !aligned(branch, 2) || !aligned(gate, 2) || !aligned(post_weight, 2) || !aligned(post_bias, 2) ||
      !aligned(weight, 2) || !aligned(bias, 2) || !aligned(y, 2) || !aligned(rng, 8))
    return OWQ_ERR_BUFFER;
  a.h = h, a.branch = branch, a.gate = d->gate != OWQ_GATE_NONE ? gate : nullptr;
  a.post_w = post_weight, a.post_b = post_bias, a.w = weight, a.b = bias;
  a.total_out = total, a.y = d->norm != OWQ_NORM_NONE ? y : nullptr;
  if (!a.total_out && !a.y) return OWQ_OK;
  return launch_norm(a, d->type, d->h_type, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

owq_status_t owq_residual_norm_backward_workspace_bytes(const owq_norm_desc_t *d, size_t *bytes) {
  const owq_status_t st = check_norm(d);
  if (st != OWQ_OK) return st;
  if (!bytes) return OWQ_ERR_NULL;
  const NormPlan p = norm_backward_plan(*d);
  const size_t sums = (d->norm != OWQ_NORM_NONE ? 2 : 0) + (d->post != OWQ_NORM_NONE ? 2 : 0) + (d->gate == OWQ_GATE_ROW ? 1 : 0);
  *bytes = (size_t)p.blocks * p.pitch * sums * sizeof(float);
  return OWQ_OK;
}

owq_status_t owq_residual_norm_backward(const owq_norm_desc_t *d, const void *dy, const void *dtotal, const void *total,
                                        const void *branch, const void *gate, const void *post_weight, const void *post_bias,
                                        const void *weight, const uint64_t *rng, void *dh, void *dbranch, void *dgate,
                                        float *dpost_weight, float *dpost_bias, float *dweight, float *dbias, void *workspace,
                                        size_t workspace_bytes, void *stream) {
  const owq_status_t st = check_norm(d);
  if (st != OWQ_OK) return st;
  if (d->norm == OWQ_NORM_NONE) dy = nullptr, dweight = dbias = nullptr;
  if (d->post == OWQ_NORM_NONE) dpost_weight = dpost_bias = nullptr;
  if (d->gate == OWQ_GATE_NONE) gate = dgate = nullptr;
  NormArgs a = norm_args(d, rng);
  const bool row_gate = d->gate == OWQ_GATE_ROW;
  const bool branch_side = dbranch || dgate || dpost_weight || dpost_bias;
  if (d->n_tokens > 0) {
    if ((dy && !total) || (d->gate != OWQ_GATE_NONE && !gate) || (a.drop.threshold > 0 && !rng)) return OWQ_ERR_NULL;
    if (!branch && branch_side && (dgate || d->post != OWQ_NORM_NONE)) return OWQ_ERR_NULL;
  }
  const uintptr_t hs = size_of(d->h_type);
  if (!aligned(dtotal, hs) || !aligned(total, hs) || !aligned(dh, hs) || !aligned(dy, 2) || !aligned(branch, 2) || !aligned(gate, 2) ||
      !aligned(post_weight, 2) || !aligned(post_bias, 2) || !aligned(weight, 2) || !aligned(rng, 8) || !aligned(dbranch, 2) ||
      !aligned(dgate, row_gate ? 4 : 2) || !aligned(dpost_weight, 4) || !aligned(dpost_bias, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
    return OWQ_ERR_BUFFER;
  a.dy = dy, a.dtotal = dtotal, a.total = total, a.gate = gate;
  a.branch = branch_side && (dgate || d->post != OWQ_NORM_NONE) ? branch : nullptr;      // read only where it is needed
  a.branch_side = branch_side;
  a.post_w = post_weight, a.post_b = post_bias, a.w = weight;
  a.dh = dh, a.dbranch = dbranch, a.dgate = row_gate ? nullptr : dgate;
  float *sums[5] = {};
  auto want = [&](float *p) {
    if (!p) return -1;
    sums[a.n_sums] = p;
    return a.n_sums++;
  };
  a.sum_w = want(dweight);
  a.sum_b = want(dbias);
  a.sum_post_w = want(dpost_weight);
  a.sum_post_b = want(dpost_bias);
  a.sum_gate = want(row_gate ? static_cast<float *>(dgate) : nullptr);
  const NormPlan p = norm_backward_plan(*d);
  a.pitch = p.pitch;
  if (a.n_sums > 0 && p.blocks > 0) {
    if (!workspace) return OWQ_ERR_NULL;
    size_t need = 0;
    (void)owq_residual_norm_backward_workspace_bytes(d, &need);
    if (!aligned(workspace, 16) || workspace_bytes < need) return OWQ_ERR_BUFFER;
    a.partial = static_cast<float *>(workspace);
  }
  return launch_norm_backward(a, d->type, d->h_type, p, sums, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

static owq_status_t check_logits(int32_t type, int32_t n_rows, int32_t vocab, float scale) {
  if (n_rows < 0 || vocab < 1 || vocab > (1 << 24)) return OWQ_ERR_SHAPE;
  if (type != OWQ_TYPE_F16 && type != OWQ_TYPE_BF16 && type != OWQ_TYPE_F32) return OWQ_ERR_TYPE;
  return scale >= 0x1p-126f && scale <= 0x1p126f ? OWQ_OK : OWQ_ERR_SHAPE;
}

owq_status_t owq_token_logprobs(const void *logits, int32_t type, int32_t n_rows, int32_t vocab, int64_t logits_row,
                                const int32_t *targets, float scale, int32_t top, float *logprob, int32_t *top_token,
                                float *top_logprob, float *stats, void *stream) {
  const owq_status_t st = check_logits(type, n_rows, vocab, scale);
  if (st != OWQ_OK) return st;
  if (top < 0 || top > 512) return OWQ_ERR_SHAPE;
  if (n_rows == 0) return OWQ_OK;
  if (!logits || !stats || (targets && !logprob) || (top > 0 && (!top_token || !top_logprob))) return OWQ_ERR_NULL;
  if (!aligned(logits, size_of(type)) || !aligned(targets, 4) || !aligned(logprob, 4) || !aligned(top_token, 4) || !aligned(top_logprob, 4) ||
      !aligned(stats, 4))
    return OWQ_ERR_BUFFER;
  const LogprobArgs a{logits, targets, logprob, top_logprob, stats, top_token, logits_row, n_rows, vocab, top, scale};
  return launch_logprobs(a, type, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

owq_status_t owq_token_logprobs_backward(const void *logits, int32_t type, int32_t n_rows, int32_t vocab, int64_t logits_row,
                                         const int32_t *targets, float scale, const float *stats, const float *dlogprob,
                                         const float *dentropy, void *dlogits, void *stream) {
  const owq_status_t st = check_logits(type, n_rows, vocab, scale);
  if (st != OWQ_OK) return st;
  if (n_rows == 0) return OWQ_OK;
  if (!logits || !stats || !dlogits || (dlogprob && !targets)) return OWQ_ERR_NULL;
  if (!aligned(logits, size_of(type)) || !aligned(dlogits, size_of(type)) || !aligned(targets, 4) || !aligned(stats, 4) || !aligned(dlogprob, 4) ||
      !aligned(dentropy, 4))
    return OWQ_ERR_BUFFER;
  const LogprobBackwardArgs a{logits, targets, stats, dlogprob, dentropy, dlogits, logits_row, n_rows, vocab, scale};
  return launch_logprobs_backward(a, type, stream) == 0 ? OWQ_OK : OWQ_ERR_HIP;
}

}  // extern "C"
