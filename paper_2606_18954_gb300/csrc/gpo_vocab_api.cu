// Host side of the vocabulary ends (gpo_vocab_*, gpo_embed*): argument checks, workspace layout,
// tensor maps and the launch sequences of gpo_vocab.cu, gpo_teach.cu and gpo_embed.cu.
#include <atomic>
#include <cmath>
#include <cstring>

#include <algorithm>

#include "gpo_stages.cuh"

using namespace gpo;

namespace {

struct VocabLayout {
  size_t marks, head, idx, hc, by_target, tile_first, rest, pm, ps, pu, tz, dz, acc, total;
  bool few;           // forward in one launch
  bool listed;        // only the tokens that take part are multiplied
  int64_t tp, hc_stride, piece, acc_stride;
  int splits;
};

int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// The workspace of either direction; no pointers are read.  (taught: of a distillation, which always goes in tiles.)
void vocab_layout(const gpo_vocab& v, bool grad, VocabLayout& L, bool taught = false) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = workspace_up(o + bytes);
    return at;
  };
  const int64_t T = v.num_tokens;
  L = VocabLayout();
  L.tp = up_to(T, kPairM);
  L.hc_stride = up_to(v.d, 64);  // rows of whole 128-byte lines
  L.few = !grad && !taught && T <= kVocabFew;
  L.listed = grad || (!L.few && (double)T * (double)v.vocab * (double)v.d >= (double)kVocabListed);
  if (T > 0 && L.few) L.marks = take(sizeof(uint64_t) * kVocabFewCtas);
  L.head = take(sizeof(VocabHead));
  if (T > 0 && L.listed) {
    L.idx = take(sizeof(int) * (size_t)T);
    L.hc = take(2 * (size_t)(up_to(T, 64) * L.hc_stride));
  }
  if (T > 0 && !grad) {
    const size_t parts = sizeof(float) * (size_t)(L.few ? kVocabFewCtas * kVocabFew : vocab_parts(v.vocab) * L.tp);
    L.pm = take(parts);
    L.ps = take(parts);
    L.pu = take(parts);
    L.tz = take(sizeof(float) * (size_t)L.tp);
  }
  if (T > 0 && grad) {
    L.by_target = take(sizeof(int) * (size_t)T);
    L.tile_first = take(sizeof(int) * (size_t)((v.vocab + kPairM - 1) / kPairM + 1));
    L.rest = take(sizeof(float) * (size_t)L.tp);
    // pieces of about equal size, a whole number of column tiles each
    const int64_t cols = std::max<int64_t>(1, kVocabPieceBytes / (2 * L.tp) / kPairN) * kPairN;
    const int64_t n = (v.vocab + cols - 1) / cols;
    L.piece = up_to((v.vocab + n - 1) / n, kPairN);
    L.acc_stride = up_to(v.d, 32);
    L.dz = take(2 * (size_t)(L.tp * L.piece));
    L.splits = vocab_splits(T, std::min(L.piece, v.vocab), v.d);
    if (L.piece < v.vocab || L.splits > 1) L.acc = take(sizeof(float) * (size_t)(L.splits * L.tp * L.acc_stride));
  }
  L.total = o;
}

gpo_status check_sizes(gpo_ctx* c, const gpo_vocab* v, bool targets = true) {
  if (!v) return set_msg(c, "vocab arguments NULL"), GPO_ERR_INVALID_ARG;
  if (v->num_tokens < 0 || v->vocab < 1 || v->d < 1) return set_msg(c, "negative size, or vocab or d < 1"), GPO_ERR_INVALID_ARG;
  if (v->num_tokens > kMaxCount || v->vocab > kMaxCount || v->d > kMaxCount)
    return set_msg(c, "more than 2^31 - 1024 tokens, vocabulary rows or columns"), GPO_ERR_UNSUPPORTED;
  if (v->hidden_stride < v->d || v->weight_stride < v->d) return set_msg(c, "row stride < d"), GPO_ERR_INVALID_ARG;
  if (v->hidden_stride >= kMaxMatrix || v->weight_stride >= kMaxMatrix ||
      (double)v->num_tokens * (double)v->hidden_stride >= (double)kMaxMatrix ||
      (double)v->vocab * (double)v->weight_stride >= (double)kMaxMatrix)
    return set_msg(c, "matrix too large"), GPO_ERR_UNSUPPORTED;
  const double tiles = ((double)v->num_tokens / kPairM + 1) * ((double)v->vocab / kPairN + 1);
  if (tiles >= 1e9) return set_msg(c, "too many logits"), GPO_ERR_UNSUPPORTED;
  if (v->dtype != GPO_DT_BF16 && v->dtype != GPO_DT_F16)
    return set_msg(c, "hidden and weight must be bf16 or fp16"), v->dtype == GPO_DT_F32 ? GPO_ERR_UNSUPPORTED : GPO_ERR_INVALID_ARG;
  if (targets && v->id_bytes != 4 && v->id_bytes != 8) return set_msg(c, "id_bytes must be 4 or 8"), GPO_ERR_INVALID_ARG;
  return GPO_OK;
}

gpo_status check_vocab(gpo_ctx* c, const gpo_vocab* v, bool targets = true) {
  gpo_status s = check_sizes(c, v, targets);
  if (s != GPO_OK) return s;
  if (!(v->scale >= 1e-4 && v->scale <= 1e4)) return set_msg(c, "scale outside [1e-4, 1e4]"), GPO_ERR_INVALID_ARG;
  if (!v->weight || (v->num_tokens > 0 && (!v->hidden || (targets && !v->target))))
    return set_msg(c, "hidden, weight or target NULL"), GPO_ERR_INVALID_ARG;
  if (v->hidden_stride % 8 != 0 || v->weight_stride % 8 != 0)
    return set_msg(c, "row bytes of hidden and weight must be a multiple of 16"), GPO_ERR_UNSUPPORTED;
  if (!aligned(v->weight, 16) || !aligned(v->hidden, 16) || (targets && !aligned(v->target, (size_t)v->id_bytes)))
    return set_msg(c, "hidden and weight must be 16-byte aligned, targets to their size"), GPO_ERR_UNSUPPORTED;
  return GPO_OK;
}

// (Fetching 256 bytes for a box's 128 takes rows that straddle lines 20 % longer: dz of 4000 tokens, 30000 x
// 1000, 144 us against 125.)
bool encode_map(CUtensorMap* m, EncodeTiledFn enc, const void* base, int64_t cols, int64_t rows, int64_t stride, int f16,
                int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(stride * 2)};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return enc(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
             strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix in blocks of 64 columns: cols a multiple of them, boxes of 64 rows of two blocks.
bool encode_blocks(CUtensorMap* m, EncodeTiledFn enc, const void* base, int64_t cols, int64_t rows, int64_t stride, int f16) {
  const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(cols / 64)};
  const cuuint64_t strides[2] = {(cuuint64_t)(stride * 2), 128};
  const cuuint32_t box[3] = {64, 64, 2}, estr[3] = {1, 1, 1};
  return enc(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims,
             strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Words of captured calls: the library's, as a graph may be replayed after its context is gone.  (A process that captures
// more calls than there are gives words out again: a call may then return another's error, or stop at it.)
__device__ __align__(256) uint32_t g_captured_words[kCapturedWords * kStatusWords];

template <class P>
P* at(void* base, size_t off) { return reinterpret_cast<P*>(static_cast<unsigned char*>(base) + off); }

// scale log2(e) for logits whose products the tensor cores add up `k` at a time: their fp32 additions, one per 16
// products, drop what lies below the running sum's last bit, always towards zero, which takes 0.10 to 0.13 (bf16) or
// 0.14 to 0.24 (fp16) of an ulp per addition from the sum, whether its terms lean one way or not.  The
// mean of that is given back here; what is left is about as large as the rounding of 32-bit sums (on dense rows lse is off
// by 1e-8 of itself in the mean).  Where products add without a loss, in rows that are zeros but for a few entries or
// of small integers, it is the error instead: 4.6e-7 (bf16) or 6.5e-7 (fp16) of a logit, 1.2e-7 or 1.7e-7 up to 16 tokens.
float logit_scale(const gpo_vocab& v, int k) {
  const double additions = (double)std::min<int64_t>(up_to(v.d, 16), k) / 16.0;
  const double lost = (v.dtype == GPO_DT_F16 ? 0.17 : 0.12) * additions * 0x1p-23;
  return (float)(v.scale * 1.4426950408889634 * (1.0 + lost));
}

// What both directions share; T > 0.
gpo_status vocab_args(gpo_ctx* ctx, const gpo_vocab& v, const VocabLayout& L, void* ws, VocabArgs& a, VocabMaps& m) {
  memset(&a, 0, sizeof a);
  memset(&m, 0, sizeof m);
  a.T = v.num_tokens;
  a.V = v.vocab;
  a.D = (int)v.d;
  a.target = v.target;
  a.id8 = v.id_bytes == 8;
  a.f16 = v.dtype == GPO_DT_F16;
  a.scale = (float)v.scale;
  a.hidden = v.hidden;
  a.hidden_stride = v.hidden_stride;
  a.head = at<VocabHead>(ws, L.head);
  a.idx = L.listed ? at<int>(ws, L.idx) : nullptr;
  a.hc = L.listed ? at<uint16_t>(ws, L.hc) : nullptr;
  a.hc_stride = L.hc_stride;
  a.debug_timeout = (ctx->params.flags & GPO_FLAG_DEBUG_TIMEOUT) != 0;
  EncodeTiledFn enc = encode_fn();
  if (!enc) return set_msg(ctx, "cuTensorMapEncodeTiled unavailable"), GPO_ERR_CUDA;
  const int64_t T64 = up_to(v.num_tokens, 64);
  bool ok = encode_map(&m.w, enc, v.weight, v.d, v.vocab, v.weight_stride, a.f16, L.few ? 32 : 128);
  if (!L.dz) ok = ok && encode_map(&m.h, enc, v.hidden, v.d, v.num_tokens, v.hidden_stride, a.f16, L.few ? kVocabFew : 128);
  if (L.few) ok = ok && encode_map(&m.wb, enc, v.weight, v.d, v.vocab, v.weight_stride, a.f16, 128);
  if (L.listed) ok = ok && encode_map(&m.hc, enc, a.hc, v.d, T64, L.hc_stride, a.f16, 128);
  if (L.dz) {
    void* dz = at<void>(ws, L.dz);
    a.w_blocks = v.d % 64 == 0;
    ok = ok && encode_map(&m.dz, enc, dz, L.piece, L.tp, L.piece, a.f16, 128) &&
         encode_blocks(&m.dzb, enc, dz, L.piece, L.tp, L.piece, a.f16) &&
         encode_blocks(&m.hb, enc, a.hc, L.hc_stride, T64, L.hc_stride, a.f16) &&
         (a.w_blocks ? encode_blocks(&m.wb, enc, v.weight, v.d, v.vocab, v.weight_stride, a.f16)
                     : encode_map(&m.wb, enc, v.weight, v.d, v.vocab, v.weight_stride, a.f16, 64));
  }
  if (!ok) return set_msg(ctx, "cuTensorMapEncodeTiled failed"), GPO_ERR_UNSUPPORTED;
  return GPO_OK;
}

// The checks of either gradient's outputs.
gpo_status check_grads(gpo_ctx* ctx, const gpo_vocab& v, const gpo_vocab_grads& out) {
  if (!out.d_weight && !out.d_hidden) return set_msg(ctx, "neither d_hidden nor d_weight is given"), GPO_ERR_INVALID_ARG;
  if ((out.d_hidden && out.d_hidden_stride < v.d) || (out.d_weight && out.d_weight_stride < v.d))
    return set_msg(ctx, "row stride of a gradient < d"), GPO_ERR_INVALID_ARG;
  if (!aligned(out.d_hidden, 2) || !aligned(out.d_weight, 2)) return set_msg(ctx, "gradients must be 2-byte aligned"), GPO_ERR_UNSUPPORTED;
  if ((out.d_hidden && (double)v.num_tokens * (double)out.d_hidden_stride >= (double)kMaxMatrix) ||
      (out.d_weight && (double)v.vocab * (double)out.d_weight_stride >= (double)kMaxMatrix))
    return set_msg(ctx, "gradient too large"), GPO_ERR_UNSUPPORTED;
  return GPO_OK;
}

// Gradients of no tokens.
gpo_status no_tokens(gpo_ctx* ctx, const gpo_vocab& v, const gpo_vocab_grads& out, void* stream) {
  ctx->nstages = 0;
  if (out.d_weight && !out.accumulate) {
    const cudaError_t e = cudaMemset2DAsync(out.d_weight, 2 * (size_t)out.d_weight_stride, 0, 2 * (size_t)v.d, (size_t)v.vocab,
                                            static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return set_msg(ctx, "memset failed: %s", cudaGetErrorString(e)), GPO_ERR_CUDA;
  }
  return GPO_OK;
}

// The arguments that either gradient has.
void grad_args(const gpo_vocab& v, const gpo_vocab_grads& out, const VocabLayout& L, void* workspace, VocabArgs& a) {
  a.sl2 = logit_scale(v, 64 * kVocabDzSeg);
  a.weight = v.weight;
  a.weight_stride = v.weight_stride;
  a.by_target = at<int>(workspace, L.by_target);
  a.tile_first = at<int>(workspace, L.tile_first);
  a.rest = at<float>(workspace, L.rest);
  a.dz = at<uint16_t>(workspace, L.dz);
  a.dz_stride = L.piece;
  a.acc = L.acc ? at<float>(workspace, L.acc) : nullptr;
  a.acc_rows = L.tp;
  a.acc_stride = L.acc_stride;
  a.splits = out.d_hidden ? L.splits : 1;
  a.dh = out.d_hidden;
  a.dh_stride = out.d_hidden_stride;
  a.dw = out.d_weight;
  a.dw_stride = out.d_weight_stride;
  a.accumulate = out.accumulate != 0;
}

// Whether d_weight's rows leave as bulk stores, and their tensor map.
// (a bulk store leaves out what lies past the matrix, but not to the element: of an odd width it wrote one more)
bool bulk_rows(const gpo_vocab& v, const VocabArgs& a, VocabMaps& m) {
  return a.dw && !a.accumulate && v.d % 8 == 0 && a.dw_stride % 8 == 0 && aligned(a.dw, 16) &&
         encode_map(&m.dw, encode_fn(), a.dw, v.d, v.vocab, a.dw_stride, a.f16, 32);
}

}  // namespace

namespace gpo {

int captured_place() {
  static std::atomic<uint32_t> next{0};
  return (int)(next.fetch_add(1, std::memory_order_relaxed) % kCapturedWords);
}

cudaError_t make_call_words(gpo_ctx* c) {
  constexpr size_t bytes = sizeof(uint32_t) * kStatusWords * kCallWords;
  c->calls = 0;
  c->call_words = c->host_words = nullptr;
  memset(c->returned, 0, sizeof c->returned);
  cudaError_t e = cudaMalloc(&c->call_words, bytes);
  if (e == cudaSuccess) e = cudaMallocHost(&c->host_words, bytes);
  if (e == cudaSuccess) e = cudaMemset(c->call_words, 0, bytes);
  if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  void* p = nullptr;
  if (e == cudaSuccess) e = cudaGetSymbolAddress(&p, g_captured_words);
  c->captured_words = static_cast<uint32_t*>(p);
  return e;
}

void free_call_words(gpo_ctx* c) {
  if (c->call_words) cudaFree(c->call_words);
  if (c->host_words) cudaFreeHost(c->host_words);
}

gpo_status read_call_words(gpo_ctx* c, cudaStream_t stream) {
  auto failed = [&](cudaError_t e) { return set_msg(c, "status read failed: %s", cudaGetErrorString(e)), GPO_ERR_CUDA; };
  auto error = [&](const uint32_t* w) { return (uint64_t)w[kStError + 1] << 32 | w[kStError]; };
  auto result = [&](const uint32_t* w) {
    const gpo_status code = (gpo_status)(error(w) & 0xFFFFu);
    set_msg(c, "%s (kernel %u, index %u)", gpo_status_string(code), w[kStWhere], w[kStDetail]);
    return code;
  };
  if (c->calls > 0) {
    cudaError_t e = cudaMemcpy(c->host_words, c->call_words, sizeof(uint32_t) * kStatusWords * kCallWords, cudaMemcpyDeviceToHost);
    if (e != cudaSuccess) return failed(e);
    uint64_t first = 0;
    for (int i = 0; i < kCallWords; ++i) {
      const uint64_t word = error(c->host_words + i * kStatusWords), call = word >> 16;
      if ((word & 0xFFFFu) == 0 || call == c->returned[i]) continue;
      c->returned[i] = call;
      if (first == 0 || call < first) first = call;
    }
    if (first != 0) return result(c->host_words + first % kCallWords * kStatusWords);
  }
  for (int i0 = 0; c->captured.any() && i0 < kCapturedWords; i0 += kCallWords) {  // as many at a time as host_words holds
    bool copied = false;
    for (int i = i0; i < i0 + kCallWords; ++i) {
      if (!c->captured[i]) continue;
      cudaError_t e = copied ? cudaSuccess : cudaMemcpy(c->host_words, c->captured_words + i0 * kStatusWords,
                                                        sizeof(uint32_t) * kStatusWords * kCallWords, cudaMemcpyDeviceToHost);
      if (e != cudaSuccess) return failed(e);
      copied = true;
      const uint32_t* w = c->host_words + (i - i0) * kStatusWords;
      if ((error(w) & 0xFFFFu) == 0) continue;
      e = cudaMemsetAsync(c->captured_words + i * kStatusWords + kStError, 0, sizeof(uint64_t), stream);  // (returned)
      return e == cudaSuccess ? result(w) : failed(e);
    }
  }
  return GPO_OK;
}

}  // namespace gpo

extern "C" {

gpo_status gpo_vocab_workspace_size(const gpo_vocab* v, int gradient, size_t* bytes) {
  if (!bytes) return GPO_ERR_INVALID_ARG;
  const gpo_status s = check_sizes(nullptr, v);
  if (s != GPO_OK) return s;
  VocabLayout L;
  vocab_layout(*v, gradient != 0, L);
  *bytes = L.total;
  return GPO_OK;
}

gpo_status gpo_vocab_logp(gpo_ctx* ctx, const gpo_vocab* v, const gpo_vocab_outputs* out, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  gpo_status s = check_vocab(ctx, v);
  if (s != GPO_OK) return s;
  if (!out || (v->num_tokens > 0 && !out->logp)) return set_msg(ctx, "logp output is NULL"), GPO_ERR_INVALID_ARG;
  if (!aligned(out->logp, 4) || !aligned(out->lse, 4) || !aligned(out->entropy, 4))
    return set_msg(ctx, "outputs must be 4-byte aligned"), GPO_ERR_UNSUPPORTED;
  VocabLayout L;
  vocab_layout(*v, false, L);
  s = check_call(ctx, workspace, workspace_bytes, L.total);
  if (s != GPO_OK) return s;
  if (v->num_tokens == 0) return ctx->nstages = 0, GPO_OK;
  VocabArgs a;
  VocabMaps m;
  s = vocab_args(ctx, *v, L, workspace, a, m);
  if (s != GPO_OK) return s;
  a.pm = at<float>(workspace, L.pm);
  a.ps = at<float>(workspace, L.ps);
  a.pu = at<float>(workspace, L.pu);
  a.tz = at<float>(workspace, L.tz);
  const bool by_row = v->num_tokens <= kPairM;  // the parts of a row side by side: one CTA joins them
  a.part_row = by_row ? vocab_parts(v->vocab) : 1;
  a.part_col = by_row ? 1 : L.tp;
  a.logp = out->logp;
  a.lse_out = out->lse;
  a.ent_out = out->entropy;
  a.sl2 = logit_scale(*v, 64 * (L.few ? kVocabFewSeg : kVocabSeg));
  const bool ent = out->entropy != nullptr;
  if (L.few) {
    Stages stage(ctx, stream);
    uint64_t* marks = at<uint64_t>(workspace, L.marks);
    // (replays share the call's mark)
    const uint64_t mark = stage.captured ? 1 : fresh_tag();
    if (stage.captured && stage.e == cudaSuccess)
      stage.e = cudaMemsetAsync(marks, 0, sizeof(uint64_t) * kVocabFewCtas, stage.lc.stream);
    stage("vocab_few", [&] { return launch_vocab_few(stage.lc, m, a, stage.st, ent, marks, mark); });
    return stage.done();
  }
  Stages stage(ctx, stream);
  if (L.listed) stage("vocab_rows", [&] { return launch_vocab_rows(stage.lc, a, stage.st); });
  stage("vocab_lse", [&] { return launch_vocab_lse(stage.lc, m, a, stage.st, ent); });
  stage("vocab_join", [&] { return launch_vocab_join(stage.lc, a, stage.st, ent); });
  return stage.done();
}

gpo_status gpo_vocab_grad(gpo_ctx* ctx, const gpo_vocab* v, const gpo_vocab_grad_inputs* in, const gpo_vocab_grads* out,
                          void* workspace, size_t workspace_bytes, void* stream) {
  return gpo_vocab_grad_logp(ctx, v, in, nullptr, out, workspace, workspace_bytes, stream);
}

gpo_status gpo_vocab_grad_logp(gpo_ctx* ctx, const gpo_vocab* v, const gpo_vocab_grad_inputs* in, const float* logp,
                               const gpo_vocab_grads* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  gpo_status s = check_vocab(ctx, v);
  if (s != GPO_OK) return s;
  const int64_t T = v->num_tokens;
  if (!in || !out) return set_msg(ctx, "inputs or outputs NULL"), GPO_ERR_INVALID_ARG;
  if (T > 0 && (!in->lse || !in->grad_logp || (in->grad_entropy && !in->entropy)))
    return set_msg(ctx, "lse, grad_logp or (with grad_entropy) entropy NULL"), GPO_ERR_INVALID_ARG;
  if (!aligned(in->lse, 4) || !aligned(in->grad_logp, 4) || !aligned(in->entropy, 4) || !aligned(in->grad_entropy, 4) ||
      !aligned(logp, 4))
    return set_msg(ctx, "inputs must be 4-byte aligned"), GPO_ERR_UNSUPPORTED;
  s = check_grads(ctx, *v, *out);
  if (s != GPO_OK) return s;
  VocabLayout L;
  vocab_layout(*v, true, L);
  s = check_call(ctx, workspace, workspace_bytes, L.total);
  if (s != GPO_OK) return s;
  if (T == 0) return no_tokens(ctx, *v, *out, stream);
  VocabArgs a;
  VocabMaps m;
  s = vocab_args(ctx, *v, L, workspace, a, m);
  if (s != GPO_OK) return s;
  a.lse = in->lse;
  a.g = in->grad_logp;
  a.ent = in->entropy;
  a.ge = in->grad_entropy;
  a.lp = logp;
  grad_args(*v, *out, L, workspace, a);
  a.dw_bulk = bulk_rows(*v, a, m);
  Stages stage(ctx, stream);
  stage("vocab_order", [&] { return launch_vocab_order(stage.lc, a, stage.st); });
  for (int64_t v0 = 0; v0 < v->vocab; v0 += L.piece) {
    a.v0 = v0;
    a.vn = std::min(L.piece, v->vocab - v0);
    a.first = v0 == 0;
    a.last = v0 + L.piece >= v->vocab;
    stage("vocab_dz", [&] { return launch_vocab_dz(stage.lc, m, a, stage.st); });
    stage("vocab_products", [&] { return launch_vocab_products(stage.lc, m, a, stage.st); });
  }
  return stage.done();
}

}  // extern "C"

namespace {

// The workspace of a distillation: that of the products, then the teacher's.
struct TeachLayout {
  VocabLayout v;
  size_t id, first, place, q, lq, z, n, qr, target;  // forward
  size_t none, dense, dense_lse;                     // gradient (and target)
  size_t total;
  int64_t stride, first_stride;
};

void teach_layout(const gpo_vocab& v, int64_t k, bool grad, TeachLayout& L) {
  L = TeachLayout();
  vocab_layout(v, grad, L.v, true);
  size_t o = L.v.total;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = workspace_up(o + bytes);
    return at;
  };
  const size_t T = (size_t)v.num_tokens;
  L.stride = up_to(k, 8);
  L.first_stride = up_to(vocab_parts(v.vocab) + 1, 2);
  const size_t all = T * (size_t)L.stride;
  if (T > 0) L.target = take(4 * T);
  if (T > 0 && !grad) {
    L.id = take(4 * all);
    L.first = take(2 * T * (size_t)L.first_stride);
    L.place = take(2 * all);
    L.q = take(4 * all);
    L.lq = take(4 * all);
    L.z = take(4 * all);
    L.n = take(4 * T);
    L.qr = take(4 * T);
  }
  if (T > 0 && grad) {
    L.none = take(4 * T);
    L.dense = take(4 * T);
    L.dense_lse = take(4 * T);
  }
  L.total = o;
}

gpo_status check_teacher_sizes(gpo_ctx* c, const gpo_vocab& v, const gpo_teacher* t, bool grad) {
  if (!t) return set_msg(c, "teacher arguments NULL"), GPO_ERR_INVALID_ARG;
  if (t->k < 1) return set_msg(c, "k < 1"), GPO_ERR_INVALID_ARG;
  if (t->k > GPO_MAX_TEACHER) return set_msg(c, "more than %d entries of a teacher", GPO_MAX_TEACHER), GPO_ERR_UNSUPPORTED;
  if (t->ids_stride < t->k || (!grad && t->logits_stride < t->k)) return set_msg(c, "row stride < k"), GPO_ERR_INVALID_ARG;
  const double rows = (double)std::max<int64_t>(v.num_tokens, 1);
  if (rows * (double)t->ids_stride >= (double)kMaxMatrix || (!grad && rows * (double)t->logits_stride >= (double)kMaxMatrix))
    return set_msg(c, "teacher too large"), GPO_ERR_UNSUPPORTED;
  if (t->id_bytes != 4 && t->id_bytes != 8) return set_msg(c, "id_bytes must be 4 or 8"), GPO_ERR_INVALID_ARG;
  return GPO_OK;
}

gpo_status check_teacher(gpo_ctx* c, const gpo_vocab& v, const gpo_teacher* t, bool grad) {
  const gpo_status s = check_teacher_sizes(c, v, t, grad);
  if (s != GPO_OK) return s;
  if (!grad) {
    if (t->dtype != GPO_DT_BF16 && t->dtype != GPO_DT_F16 && t->dtype != GPO_DT_F32)
      return set_msg(c, "unknown dtype %d of the teacher", t->dtype), GPO_ERR_INVALID_ARG;
    if (!(t->scale >= 1e-4 && t->scale <= 1e4)) return set_msg(c, "teacher's scale outside [1e-4, 1e4]"), GPO_ERR_INVALID_ARG;
    if (t->tail && t->scale != 1.0) return set_msg(c, "log-probabilities have no scale"), GPO_ERR_INVALID_ARG;
  }
  if (v.num_tokens > 0 && (!t->ids || (!grad && !t->logits))) return set_msg(c, "teacher's ids or logits NULL"), GPO_ERR_INVALID_ARG;
  if (!aligned(t->ids, (size_t)t->id_bytes) || (!grad && !aligned(t->logits, t->dtype == GPO_DT_F32 ? 4 : 2)))
    return set_msg(c, "teacher's arrays must be aligned to their elements"), GPO_ERR_UNSUPPORTED;
  return GPO_OK;
}

void teach_args(const gpo_vocab& v, const gpo_teacher& t, const TeachLayout& L, void* ws, TeachArgs& a) {
  memset(&a, 0, sizeof a);
  a.T = v.num_tokens;
  a.V = v.vocab;
  a.k = (int)t.k;
  a.ids = t.ids;
  a.ids_stride = t.ids_stride;
  a.id8 = t.id_bytes == 8;
  a.logits = t.logits;
  a.logits_stride = t.logits_stride;
  a.dtype = t.dtype;
  a.scale = (float)t.scale;
  a.tail = t.tail != 0;
  a.stride = L.stride;
  a.first_stride = L.first_stride;
  a.target = at<int>(ws, L.target);
}

}  // namespace

extern "C" {

gpo_status gpo_vocab_distill_workspace_size(const gpo_vocab* v, const gpo_teacher* t, int gradient, size_t* bytes) {
  if (!bytes) return GPO_ERR_INVALID_ARG;
  gpo_status s = check_sizes(nullptr, v, false);
  if (s == GPO_OK) s = check_teacher_sizes(nullptr, *v, t, gradient != 0);
  if (s != GPO_OK) return s;
  TeachLayout L;
  teach_layout(*v, t->k, gradient != 0, L);
  *bytes = L.total;
  return GPO_OK;
}

gpo_status gpo_vocab_distill(gpo_ctx* ctx, const gpo_vocab* v, const gpo_teacher* t, const gpo_distill_outputs* out, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  gpo_status s = check_vocab(ctx, v, false);
  if (s == GPO_OK) s = check_teacher(ctx, *v, t, false);
  if (s != GPO_OK) return s;
  if (!out || (v->num_tokens > 0 && (!out->loss || !out->delta || !out->rest || !out->rest_lse)))
    return set_msg(ctx, "loss, delta, rest or rest_lse NULL"), GPO_ERR_INVALID_ARG;
  if (out->delta_stride < t->k) return set_msg(ctx, "row stride of delta < k"), GPO_ERR_INVALID_ARG;
  if ((double)v->num_tokens * (double)out->delta_stride >= (double)kMaxMatrix) return set_msg(ctx, "delta too large"), GPO_ERR_UNSUPPORTED;
  if (!aligned(out->loss, 4) || !aligned(out->delta, 4) || !aligned(out->rest, 4) || !aligned(out->rest_lse, 4) || !aligned(out->lse, 4))
    return set_msg(ctx, "outputs must be 4-byte aligned"), GPO_ERR_UNSUPPORTED;
  TeachLayout L;
  teach_layout(*v, t->k, false, L);
  s = check_call(ctx, workspace, workspace_bytes, L.total);
  if (s != GPO_OK) return s;
  if (v->num_tokens == 0) return ctx->nstages = 0, GPO_OK;
  VocabArgs a;
  VocabMaps m;
  s = vocab_args(ctx, *v, L.v, workspace, a, m);
  if (s != GPO_OK) return s;
  TeachArgs ta;
  teach_args(*v, *t, L, workspace, ta);
  ta.id = at<int>(workspace, L.id);
  ta.first = at<uint16_t>(workspace, L.first);
  ta.place = at<int16_t>(workspace, L.place);
  ta.q = at<float>(workspace, L.q);
  ta.lq = at<float>(workspace, L.lq);
  ta.n = at<int>(workspace, L.n);
  ta.qr = at<float>(workspace, L.qr);
  ta.loss = out->loss;
  ta.lse = out->lse;
  ta.rest = out->rest;
  ta.rest_lse = out->rest_lse;
  ta.delta = out->delta;
  ta.delta_stride = out->delta_stride;
  a.target = ta.target;
  a.id8 = 0;
  a.pm = at<float>(workspace, L.v.pm);
  a.ps = at<float>(workspace, L.v.ps);
  a.pu = at<float>(workspace, L.v.pu);
  a.tz = at<float>(workspace, L.v.tz);
  a.part_row = 1;
  a.part_col = L.v.tp;
  a.logp = out->loss;  // (launch_vocab_rows: zeros of the tokens that take no part)
  // (of few tokens shorter sums, as in their log-probabilities: there no other tokens' errors average one row's out)
  a.top_seg = v->num_tokens <= 16 ? kVocabFewSeg : kVocabSeg;
  a.sl2 = logit_scale(*v, 64 * a.top_seg);
  a.top_id = ta.id;
  a.top_first = ta.first;
  a.first_stride = L.first_stride;
  a.top_z = at<float>(workspace, L.z);
  a.top_stride = L.stride;
  Stages stage(ctx, stream);
  stage("teach_sort", [&] { return launch_teach_sort(stage.lc, ta, stage.st); });
  if (L.v.listed) stage("vocab_rows", [&] { return launch_vocab_rows(stage.lc, a, stage.st); });
  stage("vocab_taught", [&] { return launch_vocab_taught(stage.lc, m, a, stage.st); });
  stage("teach_join", [&] { return launch_teach_join(stage.lc, ta, a, stage.st); });
  return stage.done();
}

gpo_status gpo_vocab_distill_grad(gpo_ctx* ctx, const gpo_vocab* v, const gpo_teacher* t, const gpo_distill_grad_inputs* in,
                                  const gpo_vocab_grads* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  gpo_status s = check_vocab(ctx, v, false);
  if (s == GPO_OK) s = check_teacher(ctx, *v, t, true);
  if (s != GPO_OK) return s;
  const int64_t T = v->num_tokens;
  if (!in || !out) return set_msg(ctx, "inputs or outputs NULL"), GPO_ERR_INVALID_ARG;
  if (T > 0 && (!in->grad_loss || !in->delta || !in->rest || !in->rest_lse))
    return set_msg(ctx, "grad_loss, delta, rest or rest_lse NULL"), GPO_ERR_INVALID_ARG;
  if (in->delta_stride < t->k) return set_msg(ctx, "row stride of delta < k"), GPO_ERR_INVALID_ARG;
  if ((double)T * (double)in->delta_stride >= (double)kMaxMatrix) return set_msg(ctx, "delta too large"), GPO_ERR_UNSUPPORTED;
  if (!aligned(in->grad_loss, 4) || !aligned(in->delta, 4) || !aligned(in->rest, 4) || !aligned(in->rest_lse, 4))
    return set_msg(ctx, "inputs must be 4-byte aligned"), GPO_ERR_UNSUPPORTED;
  s = check_grads(ctx, *v, *out);
  if (s != GPO_OK) return s;
  TeachLayout L;
  teach_layout(*v, t->k, true, L);
  s = check_call(ctx, workspace, workspace_bytes, L.total);
  if (s != GPO_OK) return s;
  if (T == 0) return no_tokens(ctx, *v, *out, stream);
  VocabArgs a;
  VocabMaps m;
  s = vocab_args(ctx, *v, L.v, workspace, a, m);
  if (s != GPO_OK) return s;
  TeachArgs ta;
  teach_args(*v, *t, L, workspace, ta);
  ta.g = in->grad_loss;
  ta.delta_in = in->delta;
  ta.delta_stride = in->delta_stride;
  ta.rest_in = in->rest;
  ta.rest_lse_in = in->rest_lse;
  ta.none = at<int>(workspace, L.none);
  ta.dense = at<float>(workspace, L.dense);
  ta.dense_lse = at<float>(workspace, L.dense_lse);
  grad_args(*v, *out, L.v, workspace, a);
  a.id8 = 0;
  a.dw_bulk = bulk_rows(*v, a, m);
  Stages stage(ctx, stream);
  stage("teach_grad", [&] { return launch_teach_grad(stage.lc, ta, stage.st); });
  a.target = ta.target;
  a.g = in->grad_loss;
  stage("vocab_order", [&] { return launch_vocab_order(stage.lc, a, stage.st); });
  a.target = ta.none;  // (dz: of no target)
  a.g = ta.dense;
  a.lse = ta.dense_lse;
  for (int64_t v0 = 0; v0 < v->vocab; v0 += L.v.piece) {
    a.v0 = v0;
    a.vn = std::min(L.v.piece, v->vocab - v0);
    a.first = v0 == 0;
    a.last = v0 + L.v.piece >= v->vocab;
    stage("vocab_dz", [&] { return launch_vocab_dz(stage.lc, m, a, stage.st); });
    stage("teach_entries", [&] { return launch_teach_entries(stage.lc, ta, a, stage.st); });
    stage("vocab_products", [&] { return launch_vocab_products(stage.lc, m, a, stage.st); });
  }
  return stage.done();
}

}  // extern "C"

namespace {

struct EmbedLayout {
  size_t perm, sid, start, part, total;
  int64_t part_stride;
};

void embed_layout(const gpo_embedding& e, bool grad, EmbedLayout& L) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = workspace_up(o + bytes);
    return at;
  };
  L = EmbedLayout();
  if (!grad) take(1);  // (the lookup needs none; a workspace has at least one byte)
  if (grad) {
    L.part_stride = up_to(e.d, 4);
    L.perm = take(sizeof(int) * (size_t)e.num_tokens);
    L.sid = take(sizeof(int) * (size_t)e.num_tokens);
    L.start = take(sizeof(int) * (size_t)(e.vocab + 1));
    const int piece = embed_piece(e.num_tokens);
    L.part = take(sizeof(float) * 2 * (size_t)((e.num_tokens + piece - 1) / piece * L.part_stride));
  }
  L.total = o;
}

gpo_status check_embed_sizes(gpo_ctx* c, const gpo_embedding* e) {
  if (!e) return set_msg(c, "embedding arguments NULL"), GPO_ERR_INVALID_ARG;
  if (e->num_tokens < 0 || e->vocab < 1 || e->d < 1) return set_msg(c, "negative size, or vocab or d < 1"), GPO_ERR_INVALID_ARG;
  if (e->num_tokens > kMaxCount || e->vocab > kMaxCount || e->d > kMaxCount)
    return set_msg(c, "more than 2^31 - 1024 tokens, table rows or columns"), GPO_ERR_UNSUPPORTED;
  if (e->table_stride < e->d || e->row_stride < e->d) return set_msg(c, "row stride < d"), GPO_ERR_INVALID_ARG;
  if ((double)e->num_tokens * (double)e->row_stride >= (double)kMaxMatrix ||
      (double)e->vocab * (double)e->table_stride >= (double)kMaxMatrix)
    return set_msg(c, "matrix too large"), GPO_ERR_UNSUPPORTED;
  if (e->dtype != GPO_DT_BF16 && e->dtype != GPO_DT_F16 && e->dtype != GPO_DT_F32)
    return set_msg(c, "unknown dtype %d", e->dtype), GPO_ERR_INVALID_ARG;
  if (e->id_bytes != 4 && e->id_bytes != 8) return set_msg(c, "id_bytes must be 4 or 8"), GPO_ERR_INVALID_ARG;
  return GPO_OK;
}

// The checks of either direction, and the arguments that both share.
gpo_status embed_args(gpo_ctx* ctx, const gpo_embedding* e, const void* table, const void* rows, bool grad, void* ws,
                      size_t bytes, EmbedLayout& L, EmbedArgs& a) {
  gpo_status s = check_embed_sizes(ctx, e);
  if (s != GPO_OK) return s;
  if (!std::isfinite((float)e->scale)) return set_msg(ctx, "scale is not a finite fp32 number"), GPO_ERR_INVALID_ARG;
  if (!table || (e->num_tokens > 0 && (!rows || !e->ids))) return set_msg(ctx, "table, rows or ids NULL"), GPO_ERR_INVALID_ARG;
  const uintptr_t esz = e->dtype == GPO_DT_F32 ? 4 : 2;
  if (!aligned(table, esz) || !aligned(rows, esz) || !aligned(e->ids, (size_t)e->id_bytes))
    return set_msg(ctx, "table, rows or ids not aligned to their elements"), GPO_ERR_UNSUPPORTED;
  embed_layout(*e, grad, L);
  s = check_call(ctx, ws, bytes, L.total);
  if (s != GPO_OK) return s;
  memset(&a, 0, sizeof a);
  a.T = e->num_tokens;
  a.V = e->vocab;
  a.D = e->d;
  a.ids = e->ids;
  a.id8 = e->id_bytes == 8;
  a.dtype = e->dtype;
  a.scale = (float)e->scale;
  return GPO_OK;
}

}  // namespace

extern "C" {

gpo_status gpo_embed_workspace_size(const gpo_embedding* e, int gradient, size_t* bytes) {
  if (!bytes) return GPO_ERR_INVALID_ARG;
  const gpo_status s = check_embed_sizes(nullptr, e);
  if (s != GPO_OK) return s;
  EmbedLayout L;
  embed_layout(*e, gradient != 0, L);
  *bytes = L.total;
  return GPO_OK;
}

gpo_status gpo_embed(gpo_ctx* ctx, const gpo_embedding* e, const void* table, void* out, void* workspace,
                     size_t workspace_bytes, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  EmbedLayout L;
  EmbedArgs a;
  const gpo_status s = embed_args(ctx, e, table, out, false, workspace, workspace_bytes, L, a);
  if (s != GPO_OK) return s;
  if (a.T == 0) return ctx->nstages = 0, GPO_OK;
  a.src = table;
  a.src_stride = e->table_stride;
  a.dst = out;
  a.dst_stride = e->row_stride;
  Stages stage(ctx, stream);
  stage("embed", [&] { return launch_embed(stage.lc, a, stage.st); });
  return stage.done();
}

gpo_status gpo_embed_grad(gpo_ctx* ctx, const gpo_embedding* e, const void* grad, void* d_table, int accumulate,
                          void* workspace, size_t workspace_bytes, void* stream) {
  if (!ctx) return GPO_ERR_INVALID_ARG;
  ctx->msg[0] = 0;
  EmbedLayout L;
  EmbedArgs a;
  const gpo_status s = embed_args(ctx, e, d_table, grad, true, workspace, workspace_bytes, L, a);
  if (s != GPO_OK) return s;
  a.src = grad;
  a.src_stride = e->row_stride;
  a.dst = d_table;
  a.dst_stride = e->table_stride;
  a.accumulate = accumulate != 0;
  a.perm = at<int>(workspace, L.perm);
  a.sid = at<int>(workspace, L.sid);
  a.start = at<int>(workspace, L.start);
  a.part = at<float>(workspace, L.part);
  a.part_stride = L.part_stride;
  Stages stage(ctx, stream);
  stage("embed_grad", [&] { return launch_embed_grad(stage.lc, a, stage.st); });
  return stage.done();
}

}  // extern "C"
