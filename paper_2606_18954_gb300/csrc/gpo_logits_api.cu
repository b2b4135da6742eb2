// Host side of the adjusted logits (gpo_logits_*): argument checks and the launch of gpo_logits.cu.
#include <cmath>
#include <cstring>

#include "gpo_stages.cuh"

using namespace gpo;

namespace {

bool id_size(int32_t n) { return n == 4 || n == 8; }

// The checks of either direction, and the arguments that both share.
gpo_status logits_args(gpo_ctx* c, const gpo_logits* l, LogitsArgs& a) {
  if (!l) return set_msg(c, "logits arguments NULL"), GPO_ERR_INVALID_ARG;
  if (l->num_rows < 0 || l->vocab < 1 || l->history_len < 0 || l->bias_len < 0)
    return set_msg(c, "negative size, or vocab < 1"), GPO_ERR_INVALID_ARG;
  // (the kernel's places in a row are 32-bit, with room for a CTA's step past the end)
  if (l->num_rows > kMaxCount || l->vocab > (int64_t)1 << 30)
    return set_msg(c, "more than 2^31 - 1024 rows or 2^30 tokens"), GPO_ERR_UNSUPPORTED;
  if (l->logits_stride < l->vocab) return set_msg(c, "row stride < vocab"), GPO_ERR_INVALID_ARG;
  if (l->logits_stride >= kMaxMatrix || (double)l->num_rows * (double)l->logits_stride >= (double)kMaxMatrix ||
      l->history_len >= kMaxMatrix || l->bias_len >= kMaxMatrix)
    return set_msg(c, "matrix or list too large"), GPO_ERR_UNSUPPORTED;
  if (l->dtype != GPO_DT_BF16 && l->dtype != GPO_DT_F16 && l->dtype != GPO_DT_F32)
    return set_msg(c, "unknown dtype %d", l->dtype), GPO_ERR_INVALID_ARG;
  if (l->num_rows > 0 && !l->logits) return set_msg(c, "logits NULL"), GPO_ERR_INVALID_ARG;
  if ((l->spans && l->history_len > 0 && (!l->history || !id_size(l->history_bytes))) ||
      (l->bias && l->bias_len > 0 && (!l->bias_ids || !id_size(l->bias_bytes))) || (l->target && !id_size(l->target_bytes)))
    return set_msg(c, "history or bias_ids NULL, or bytes of an id other than 4 or 8"), GPO_ERR_INVALID_ARG;
  if ((!l->scale && !(l->scale_all >= 1e-4 && l->scale_all <= 1e4)) ||
      (!l->repetition && !((float)l->repetition_all > 0.f && std::isfinite((float)l->repetition_all))) ||
      (!l->presence && !std::isfinite((float)l->presence_all)) || (!l->frequency && !std::isfinite((float)l->frequency_all)))
    return set_msg(c, "scale outside [1e-4, 1e4], repetition not a positive number, or a penalty not finite"), GPO_ERR_INVALID_ARG;
  if (l->mask && (l->mask_rows < 1 || l->mask_stride < 0 || (l->mask_rows > 1 && l->mask_stride < (l->vocab + 31) / 32) ||
                  l->mask_stride >= kMaxMatrix || (!l->mask_row && l->mask_rows != 1 && l->mask_rows != l->num_rows)))
    return set_msg(c, "masks need rows of ceil(vocab / 32) words, one for all rows or one each or mask_row"), GPO_ERR_INVALID_ARG;
  if (l->mask && (double)l->mask_rows * (double)l->mask_stride >= (double)kMaxMatrix)
    return set_msg(c, "masks too large"), GPO_ERR_UNSUPPORTED;
  if (!aligned(l->logits, l->dtype == GPO_DT_F32 ? 4 : 2) || !aligned(l->scale, 4) || !aligned(l->repetition, 4) ||
      !aligned(l->presence, 4) || !aligned(l->frequency, 4) || !aligned(l->spans, 8) || !aligned(l->bias, 4) ||
      !aligned(l->bias_spans, 8) || !aligned(l->mask, 4) || !aligned(l->mask_row, 4) ||
      (l->spans && l->history_len > 0 && !aligned(l->history, (size_t)l->history_bytes)) ||
      (l->bias && l->bias_len > 0 && !aligned(l->bias_ids, (size_t)l->bias_bytes)) ||
      (l->target && !aligned(l->target, (size_t)l->target_bytes)))
    return set_msg(c, "arrays must be aligned to their elements"), GPO_ERR_UNSUPPORTED;
  memset(&a, 0, sizeof a);
  a.R = l->num_rows;
  a.V = l->vocab;
  a.z = l->logits;
  a.z_stride = l->logits_stride;
  a.scale = l->scale;
  a.rep = l->repetition;
  a.pres = l->presence;
  a.freq = l->frequency;
  a.scale1 = (float)l->scale_all;
  a.rep1 = (float)l->repetition_all;
  a.pres1 = (float)l->presence_all;
  a.freq1 = (float)l->frequency_all;
  if (l->spans) {
    a.hist = l->history;
    a.hist_len = l->history_len;
    a.spans = l->spans;
    a.hist8 = l->history_bytes == 8;
  }
  if (l->bias && l->bias_len > 0) {
    a.bias = l->bias;
    a.bias_ids = l->bias_ids;
    a.bias_len = l->bias_len;
    a.bias_spans = l->bias_spans;
    a.bias8 = l->bias_bytes == 8;
  }
  if (l->mask) {
    a.mask = l->mask;
    a.mask_rows = l->mask_rows;
    a.mask_stride = l->mask_stride;
    a.mask_row = l->mask_row;
  }
  a.target = l->target;
  a.target8 = l->target_bytes == 8;
  return GPO_OK;
}

// Two matrices of R rows that share memory, but are not one and the same.
bool overlap(const void* p, int64_t ps, size_t pe, const void* q, int64_t qs, size_t qe, int64_t R, int64_t V) {
  if (R == 0 || (p == q && ps == qs && pe == qe)) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  const uintptr_t step = (uintptr_t)ps * pe, off = (b > a ? b - a : a - b) % (step ? step : 1);
  if (R > 1 && step == (uintptr_t)qs * qe) {  // (columns of one buffer, side by side)
    const uintptr_t lower = (uintptr_t)V * (b > a ? pe : qe), upper = (uintptr_t)V * (b > a ? qe : pe);
    if (off >= lower && step - off >= upper) return false;
  }
  const uintptr_t a1 = a + pe * (size_t)((R - 1) * ps + V), b1 = b + qe * (size_t)((R - 1) * qs + V);
  return a < b1 && b < a1;
}

}  // namespace

extern "C" {

gpo_status gpo_logits_adjust(gpo_ctx* ctx, const gpo_logits* l, const gpo_logits_outputs* out, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  LogitsArgs a;
  gpo_status s = logits_args(ctx, l, a);
  if (s != GPO_OK) return s;
  if (!out || (l->num_rows > 0 && !out->logits && !out->logp && !out->lse && !out->entropy))
    return set_msg(ctx, "no output is given"), GPO_ERR_INVALID_ARG;
  if (out->logp && l->num_rows > 0 && !l->target) return set_msg(ctx, "logp needs target"), GPO_ERR_INVALID_ARG;
  if (out->logits && (out->logits_stride < l->vocab || (out->dtype != l->dtype && out->dtype != GPO_DT_F32)))
    return set_msg(ctx, "adjusted logits: row stride < vocab, or neither fp32 nor the raw ones' type"), GPO_ERR_INVALID_ARG;
  if (out->logits && (double)l->num_rows * (double)out->logits_stride >= (double)kMaxMatrix)
    return set_msg(ctx, "adjusted logits too large"), GPO_ERR_UNSUPPORTED;
  if (!aligned(out->logp, 4) || !aligned(out->lse, 4) || !aligned(out->entropy, 4) ||
      !aligned(out->logits, out->dtype == GPO_DT_F32 ? 4 : 2))
    return set_msg(ctx, "outputs must be aligned to their elements"), GPO_ERR_UNSUPPORTED;
  if (out->logits && overlap(l->logits, l->logits_stride, l->dtype == GPO_DT_F32 ? 4 : 2, out->logits, out->logits_stride,
                             out->dtype == GPO_DT_F32 ? 4 : 2, l->num_rows, l->vocab))
    return set_msg(ctx, "adjusted and raw logits overlap"), GPO_ERR_INVALID_ARG;
  s = check_device(ctx);
  if (s != GPO_OK) return s;
  if (l->num_rows == 0) return ctx->nstages = 0, GPO_OK;
  a.out = out->logits;
  a.out_stride = out->logits_stride;
  a.out32 = out->logits && out->dtype == GPO_DT_F32;
  a.logp = out->logp;
  a.lse = out->lse;
  a.ent = out->entropy;
  Stages stage(ctx, stream);
  stage("logits_adjust", [&] { return launch_logits(stage.lc, a, l->dtype, stage.st); });
  return stage.done();
}

gpo_status gpo_logits_grad(gpo_ctx* ctx, const gpo_logits* l, const gpo_logits_grad_inputs* in, void* d_logits,
                           int64_t d_stride, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  LogitsArgs a;
  gpo_status s = logits_args(ctx, l, a);
  if (s != GPO_OK) return s;
  if (!in || (l->num_rows > 0 && (!d_logits || !l->target || !in->lse || !in->logp || !in->grad_logp ||
                                  (in->grad_entropy && !in->entropy))))
    return set_msg(ctx, "d_logits, target, lse, logp, grad_logp or (with grad_entropy) entropy NULL"), GPO_ERR_INVALID_ARG;
  if (d_stride < l->vocab) return set_msg(ctx, "row stride of the gradient < vocab"), GPO_ERR_INVALID_ARG;
  if ((double)l->num_rows * (double)d_stride >= (double)kMaxMatrix) return set_msg(ctx, "gradient too large"), GPO_ERR_UNSUPPORTED;
  const size_t e = l->dtype == GPO_DT_F32 ? 4 : 2;
  if (!aligned(d_logits, e) || !aligned(in->lse, 4) || !aligned(in->logp, 4) || !aligned(in->grad_logp, 4) ||
      !aligned(in->entropy, 4) || !aligned(in->grad_entropy, 4))
    return set_msg(ctx, "arrays must be aligned to their elements"), GPO_ERR_UNSUPPORTED;
  if (overlap(l->logits, l->logits_stride, e, d_logits, d_stride, e, l->num_rows, l->vocab))
    return set_msg(ctx, "gradient and raw logits overlap"), GPO_ERR_INVALID_ARG;
  s = check_device(ctx);
  if (s != GPO_OK) return s;
  if (l->num_rows == 0) return ctx->nstages = 0, GPO_OK;
  a.out = d_logits;
  a.out_stride = d_stride;
  a.lse_in = in->lse;
  a.logp_in = in->logp;
  a.g = in->grad_logp;
  a.ent_in = in->entropy;
  a.ge = in->grad_entropy;
  Stages stage(ctx, stream);
  stage("logits_grad", [&] { return launch_logits(stage.lc, a, l->dtype, stage.st); });
  return stage.done();
}

}  // extern "C"
