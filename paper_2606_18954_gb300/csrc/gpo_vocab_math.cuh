// Sums of exponentials over parts of the vocabulary, shared by the kernels of gpo_vocab.cu and
// gpo_vocab_few.cu.  Logits are in units of log 2 here: scale log2(e) <h, w>.
#pragma once

#include "gpo_internal.cuh"

namespace gpo {

// A logit that is left out (a column past the vocabulary, the target) and the maximum of a part without
// logits: for every scale in [1e-4, 1e4] the first, scaled, is finite and far below the second
constexpr float kNone = -1e33f, kLow = -1e28f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ int64_t load_id(const void* ids, int id8, int64_t t) {
  return id8 ? static_cast<const int64_t*>(ids)[t] : (int64_t)static_cast<const int32_t*>(ids)[t];
}

struct Part {
  float m, s, u;
};
// Two parts of a row as one: sums relative to the larger maximum.
template <bool kEnt>
__device__ __forceinline__ Part join(const Part& x, const Part& y) {
  const float m = fmaxf(x.m, y.m);
  const float a = x.m - m, b = y.m - m, ca = exp2f(a), cb = exp2f(b);
  Part r;
  r.m = m;
  r.s = ca * x.s + cb * y.s;
  r.u = kEnt ? ca * (x.u + a * x.s) + cb * (y.u + b * y.s) : 0.f;
  return r;
}

template <bool kEnt>
__device__ __forceinline__ void finish(const VocabArgs& a, int64_t tok, float zy, const Part& p) {
  const float top = fmaxf(p.m, zy), y = zy - top, c = p.m - top, ec = exp2f(c);
  const float others = ec * p.s, total = others + exp2f(y);
  const float ln2 = 0.6931471805599453f;
  const float lt = y == 0.f ? log1pf(others) : logf(total);
  a.logp[tok] = fmaf(y, ln2, -lt);
  if (a.lse_out) a.lse_out[tok] = fmaf(top, ln2, lt);
  if (kEnt) a.ent_out[tok] = lt - ln2 * (ec * (p.u + c * p.s) + exp2f(y) * y) / total;
}

}  // namespace gpo
