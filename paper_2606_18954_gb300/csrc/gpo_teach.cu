// Distillation from a teacher's top tokens: what goes before and after the products of gpo_vocab.cu (formulas in
// include/graphpo.h).  Times of 2048 tokens (1434 with a teacher) of 65536 x 2048 with up to 32 entries.
//
// Forward:  teach_sort_kernel   a warp per token puts the teacher's entries in the order of their ids (by counting the smaller
//                               ones: k^2 / 32 comparisons a lane, four ids of every load against up to four of the lane's own)
//                               with their probabilities and a tail's remainder, and counts those before every 128 columns of the vocabulary.  14 us
//                               between events, of 256 entries a token 38 (one comparison a load, and the columns one search
//                               after another 17 and 81): the instructions of both loops
//           vocab_pair_kernel   <kLseTop>: logits tiles that stay in tensor memory; a row's entries are taken out of its
//                               maximum and sum, which are then those of the other tokens.  214 to 225 us, 1710 to 1800 TFLOP/s,
//                               tensor pipe busy 86 % of the time (93 % of its SMs' active cycles).  Every entry among a warp's 32 rows and 32 columns is a pass over the 32
//                               (100 instructions): of narrow states, whose tiles' products are short, that shows (8192 tokens of
//                               131072 x 256 with 48 entries 545 us, log-probabilities 461)
//           teach_join_kernel   the parts of a row joined, divergence and p - q from them and the entries' logits.  12 us
// Gradient: outside the entries dz is g (p - q of all others together) times the softmax over the others, for either form of the
//           loss; inside it is g (p - q).  So vocab_pair_kernel's dz of a token without a target, with the others' log-sum-exp,
//           is right for all but the entries, which teach_entries_kernel writes over it, rounded once (6 us); then the products.
//           The largest entry (teach_grad_kernel, 6 us) takes the place that a target has there: the tokens are in the
//           order of those, and what its rounding takes is added to both products.  That brings the gradients' error from 1.4
//           times that of their own rounding to 1.0 to 1.2.
// Keeping the entries out of the sum over the others keeps the digits of both: where the student is nearly certain of one
// of the teacher's tokens, 1 - p is a sum of small terms here, and so is the others' share p_r.  1 - q comes from the teacher's
// log-probability by expm1, and of two numbers p - q or 1 - q less 1 - p is taken, whichever are smaller.
#define GPO_REPORT __noinline__
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gpo_vocab_math.cuh"

namespace gpo {

namespace {

constexpr int kSortWarps = 4;
constexpr int kNoId = 0x7fffffff;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float load_value(const void* p, int dtype, int64_t i) {
  if (dtype == GPO_DT_F32) return static_cast<const float*>(p)[i];
  if (dtype == GPO_DT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}

template <class F>
__device__ __forceinline__ float over_warp(float x, F f) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = f(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float warp_max(float x) { return over_warp(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float warp_sum(float x) { return over_warp(x, [](float a, float b) { return a + b; }); }
// The lowest index (below 2^31) of any lane.
__device__ __forceinline__ int warp_first(int x) { return (int)__reduce_min_sync(0xffffffffu, (unsigned)x); }

// The entries of a warp's token by their ids: calls f(j, id, rank) for every entry j that is one, kOwn of a lane at a time.
// ids: k of them, then kNoId up to a multiple of 4.  Equal ids get equal ranks.
template <int kOwn, class F>
__device__ __forceinline__ void rank_entries(const int* ids, int k, F f) {
#pragma unroll 1
  for (int j0 = threadIdx.x & 31; j0 < k; j0 += 32 * kOwn) {
    int id[kOwn], rank[kOwn];
#pragma unroll
    for (int u = 0; u < kOwn; ++u) id[u] = j0 + 32 * u < k ? ids[j0 + 32 * u] : kNoId, rank[u] = 0;
#pragma unroll 4
    for (int i = 0; i < k; i += 4) {
      const int4 x = *reinterpret_cast<const int4*>(ids + i);
#pragma unroll
      for (int u = 0; u < kOwn; ++u) rank[u] += (x.x < id[u]) + (x.y < id[u]) + (x.z < id[u]) + (x.w < id[u]);
    }
#pragma unroll
    for (int u = 0; u < kOwn; ++u)
      if (id[u] != kNoId) f(j0 + 32 * u, id[u], rank[u]);
  }
}

__global__ void __launch_bounds__(32 * kSortWarps) teach_sort_kernel(TeachArgs t, Status st) {
  __shared__ __align__(16) int s_id[kSortWarps][kTeachMax];
  __shared__ int s_sorted[kSortWarps][2 * kTeachMax];
  __shared__ float s_v[kSortWarps][kTeachMax];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  let_next_start();
  const int64_t tok = (int64_t)blockIdx.x * kSortWarps + warp;
  if (tok >= t.T) return;
  int *ids = s_id[warp], n = 0;
  float *v = s_v[warp], m = -INFINITY;
  bool bad = false;
  for (int j = lane; j < t.k; j += 32) {
    const int64_t id = load_id(t.ids, t.id8, tok * t.ids_stride + j);
    const bool in = id >= 0 && id < t.V;
    if (id >= t.V) report(st, GPO_ERR_SHAPE, 50, (int)tok);
    ids[j] = in ? (int)id : kNoId;
    const float x = in ? load_value(t.logits, t.dtype, tok * t.logits_stride + j) : -INFINITY;
    v[j] = x * t.scale;
    bad |= !(v[j] < INFINITY);  // (and so x)
    m = fmaxf(m, v[j]);
    n += in;
  }
  if (lane < (-t.k & 3)) ids[t.k + lane] = kNoId;  // (kTeachMax is a multiple of 4)
  n = __reduce_add_sync(0xffffffffu, n);
  m = warp_max(m);
  if (__any_sync(0xffffffffu, bad)) {
    if (lane == 0) report(st, GPO_ERR_NONFINITE, 51, (int)tok);
    n = 0;
  }
  if (!t.tail && m == -INFINITY) n = 0;  // (no distribution)
  const int step = n > 0 ? 1 << (31 - __clz(n)) : 0;  // the largest power of two that is not above n
  for (int j = lane; j < 2 * step; j += 32) s_sorted[warp][j] = kNoId;
  __syncwarp();
  float shift = 0.f, qr = 0.f;  // log q = v - shift
  if (n > 0) {
    // the largest apart: log q of a nearly certain token has its digits, and 1 - q of it
    int first = kNoId;
    for (int j = lane; j < t.k; j += 32)
      if (v[j] == m) first = min(first, j);
    first = warp_first(first);
    if (!t.tail || m > 0.f) {
      float others = 0.f;
      for (int j = lane; j < t.k; j += 32)
        if (j != first) others += expf(v[j] - m);
      shift = log1pf(warp_sum(others));
    } else {
      // 1 - the sum, in 64 bits: it may be small beside the others, too.  (1 - q of the largest from exp, not expm1, was off by
      // 6e-8, 1 % of a remainder of 1e-5)
      double others = 0.0;
      for (int j = lane; j < t.k; j += 32)
        if (j != first) others += (double)expf(v[j]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) others += __shfl_xor_sync(0xffffffffu, others, o);
      const double left = -(double)expm1f(m) - others;
      m = 0.f;
      if (left < 0.0) shift = log1pf((float)-left);  // (probabilities rounded to fewer bits)
      else qr = (float)left;
    }
  }
  float* delta = t.delta + tok * t.delta_stride;
  for (int j = lane; j < t.k; j += 32)
    if (n == 0 || ids[j] == kNoId) delta[j] = 0.f;
  if (n > 0) {
    auto put = [&](int j, int id, int rank) {
      const int64_t at = tok * t.stride + rank;
      const float lq = v[j] - m - shift;
      t.id[at] = s_sorted[warp][rank] = id;
      t.place[at] = (int16_t)j;
      t.lq[at] = lq;
      t.q[at] = expf(lq);
    };
    if (t.k <= 32) rank_entries<1>(ids, t.k, put);
    else if (t.k <= 64) rank_entries<2>(ids, t.k, put);
    else rank_entries<4>(ids, t.k, put);
    __syncwarp();
    bool twice = false;  // of equal ranks one place stays empty
    for (int j = lane; j < n; j += 32) twice |= s_sorted[warp][j] == kNoId;
    if (__any_sync(0xffffffffu, twice)) {
      if (lane == 0) report(st, GPO_ERR_SHAPE, 52, (int)tok);
      n = 0;
    }
  }
  // The entries below 128 p, by steps of powers of two; four places a lane are looked for at a time.
  const int parts = (int)vocab_parts(t.V);
  for (int p = lane; p <= parts; p += 128) {
    int first[4] = {0, 0, 0, 0};
    for (int s = n > 0 ? step : 0; s > 0; s >>= 1)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if ((uint32_t)s_sorted[warp][first[u] + s - 1] < 128u * (uint32_t)(p + 32 * u)) first[u] += s;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (p + 32 * u <= parts) t.first[tok * t.first_stride + p + 32 * u] = (uint16_t)first[u];
  }
  if (lane == 0) {
    t.n[tok] = n;
    t.qr[tok] = qr;
    t.target[tok] = n > 0 ? 0 : -1;
    if (n == 0) {
      t.loss[tok] = 0.f;
      t.rest[tok] = 0.f;
      t.rest_lse[tok] = 0.f;
      if (t.lse) t.lse[tok] = 0.f;
    }
  }
}

// A CTA takes 32 rows: their parts by its warps in turn, then a row each.
__global__ void __launch_bounds__(1024) teach_join_kernel(TeachArgs t, VocabArgs a, int parts) {
  __shared__ Part red[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  after_previous();
  const int rows = a.idx ? a.head->rows : (int)a.T, row0 = blockIdx.x * 32;
  if (row0 >= rows) return;
  Part p = {kLow, 0.f, 0.f};
  if (row0 + lane < rows) {
#pragma unroll 8
    for (int i = warp; i < parts; i += 32) {
      const int64_t at = (row0 + lane) * a.part_row + (int64_t)i * a.part_col;
      p = join<false>(p, Part{a.pm[at], a.ps[at], 0.f});
    }
  }
  red[warp][lane] = p;
  __syncthreads();
  if (row0 + warp >= rows) return;
  const int64_t tok = a.idx ? a.idx[row0 + warp] : row0 + warp;
  const int n = t.n[tok];
  if (n == 0) return;
  p = red[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    p = join<false>(p, Part{__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o), 0.f});
  // logits in units of log 2; the largest entry apart
  const float *z = a.top_z + tok * t.stride, *q = t.q + tok * t.stride, *lq = t.lq + tok * t.stride;
  float most = -INFINITY;
  for (int j = lane; j < n; j += 32) most = fmaxf(most, z[j]);
  most = warp_max(most);
  int first = kNoId;
  for (int j = lane; j < n; j += 32)
    if (z[j] == most) first = min(first, j);
  first = warp_first(first);  // (none where they are NaN)
  const bool some = n < t.V;  // tokens other than the entries (whose sum may be NaN, or 0 where every logit of theirs is -inf)
  const float top = some ? fmaxf(p.m, most) : most, er = some ? p.s * exp2f(p.m - top) : 0.f, ef = exp2f(most - top);
  float mine = 0.f, q_mine = 0.f;  // of the entries but the largest
  for (int j = lane; j < n; j += 32) {
    if (j == first) continue;
    mine += exp2f(z[j] - top);
    q_mine += q[j];
  }
  mine = warp_sum(mine);
  q_mine = warp_sum(q_mine);
  const float left = t.qr[tok], qr = some ? left : 0.f;  // (of no tokens: what the teacher's probabilities were rounded by)
  const float others = mine + er, q_others = q_mine + left, qf = first < n ? q[first] : 0.f;
  const float total = others + ef, lt = top == most ? log1pf(others) : logf(total), inv = 1.f / total;
  // p - q of the largest entry and of the others together: of numbers whose sum is above 1, 1 - q less 1 - p, whose digits p and q
  // do not have; else p - q, whose digits 1 - p and 1 - q do not have
  const float pf = ef * inv, pr = er * inv, p_entries = (mine + ef) * inv, q_entries = q_mine + qf;
  const float df = pf + qf > 1.f ? q_others - others * inv : pf - qf;
  const float dr = pr + qr > 1.f ? q_entries - p_entries : pr - qr;
  float loss = 0.f;
  float* delta = t.delta + tok * t.delta_stride;
  for (int j = lane; j < n; j += 32) {
    const float y = z[j] - top, qj = q[j];
    if (qj > 0.f) loss = fmaf(qj, lq[j] - fmaf(y, kLn2, -lt), loss);
    delta[t.place[tok * t.stride + j]] = j == first ? df : fmaf(exp2f(y), inv, -qj);
  }
  loss = warp_sum(loss);
  if (lane == 0) {
    const float log_others = some ? fmaf(p.m, kLn2, logf(p.s)) : -INFINITY;
    if (qr > 0.f) {
      const float log_q = qr > 0.5f ? log1pf(-q_entries) : logf(qr);
      loss = fmaf(qr, log_q - (pr > 0.5f ? log1pf(-p_entries) : fmaf(p.m - top, kLn2, logf(p.s)) - lt), loss);
    }
    t.loss[tok] = loss;
    t.rest[tok] = dr;
    t.rest_lse[tok] = log_others;
    if (t.lse) t.lse[tok] = fmaf(top, kLn2, lt);
  }
}

// What vocab_pair_kernel's dz takes of a token, and whether it has a gradient.
__global__ void __launch_bounds__(256) teach_grad_kernel(TeachArgs t, Status st) {
  const int lane = threadIdx.x & 31;
  let_next_start();
  const int64_t tok = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (tok >= t.T) return;
  int top = -1;  // the entry of the largest |delta|, of equal ones that of the lowest id
  float most = -1.f;
  bool learns = !(t.rest_in[tok] == 0.f);  // (a NaN is not 0)
  for (int j = lane; j < t.k; j += 32) {
    const int64_t id = load_id(t.ids, t.id8, tok * t.ids_stride + j);
    if (id >= t.V) report(st, GPO_ERR_SHAPE, 53, (int)tok);
    if (id < 0 || id >= t.V) continue;
    const float x = fabsf(t.delta_in[tok * t.delta_stride + j]);
    learns |= !(x == 0.f);
    if (top < 0 || x > most || (x == most && id < top)) top = (int)id, most = x;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const int id = __shfl_xor_sync(0xffffffffu, top, o);
    const float x = __shfl_xor_sync(0xffffffffu, most, o);
    if (id >= 0 && (top < 0 || x > most || (x == most && id < top))) top = id, most = x;
  }
  // Without any p - q that is not 0 every dz is 0: of a token whose teacher gives nothing a probability, rest_lse is a 0 that is
  // none, and its hidden row may hold anything, which would reach d_weight as 0 times that.
  learns = __any_sync(0xffffffffu, learns);
  if (lane != 0) return;
  const float lse = t.rest_lse_in[tok];
  t.target[tok] = learns ? top : -1;
  t.none[tok] = -1;
  t.dense[tok] = -t.g[tok] * t.rest_in[tok];
  t.dense_lse[tok] = lse == -INFINITY ? INFINITY : lse;  // (no other tokens: their p is 0)
}

__global__ void __launch_bounds__(256) teach_entries_kernel(TeachArgs t, VocabArgs a, Status st) {
  const int lane = threadIdx.x & 31;
  let_next_start();
  after_previous();
  const int64_t warp = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), nwarps = (int64_t)gridDim.x * 8;
  const int rows = a.head->rows;
  const float gs = a.head->dz_scale;
  for (int64_t r = warp; r < rows; r += nwarps) {
    const int64_t tok = a.idx[r];
    const float g = t.g[tok] * gs;
    for (int j = lane; j < t.k; j += 32) {
      const int64_t id = load_id(t.ids, t.id8, tok * t.ids_stride + j);
      if (id < a.v0 || id >= a.v0 + a.vn || id >= t.V) continue;
      const float x = g * t.delta_in[tok * t.delta_stride + j];
      if (!GPO_BOUNDS(st, id - a.v0, a.dz_stride, kWhereVocabRow)) continue;
      uint16_t* dst = a.dz + r * a.dz_stride + (id - a.v0);
      float rounded;
      if (a.f16) {
        const __half h = __float2half_rn(x);
        *reinterpret_cast<__half*>(dst) = h;
        rounded = __half2float(h);
      } else {
        const __nv_bfloat16 h = __float2bfloat16_rn(x);
        *reinterpret_cast<__nv_bfloat16*>(dst) = h;
        rounded = __bfloat162float(h);
      }
      if (id == a.by_target[r]) a.rest[r] = x - rounded;
    }
  }
}

}  // namespace

cudaError_t launch_teach_sort(const LaunchCtx& lc, const TeachArgs& t, const Status& st) {
  teach_sort_kernel<<<(unsigned)((t.T + kSortWarps - 1) / kSortWarps), 32 * kSortWarps, 0, lc.stream>>>(t, st);
  return cudaGetLastError();
}

cudaError_t launch_teach_join(const LaunchCtx& lc, const TeachArgs& t, const VocabArgs& a, const Status&) {
  return launch_after(teach_join_kernel, (unsigned)((t.T + 31) / 32), 1024, 0, lc.stream, t, a, (int)vocab_parts(t.V));
}

cudaError_t launch_teach_grad(const LaunchCtx& lc, const TeachArgs& t, const Status& st) {
  teach_grad_kernel<<<(unsigned)((t.T + 7) / 8), 256, 0, lc.stream>>>(t, st);
  return cudaGetLastError();
}

cudaError_t launch_teach_entries(const LaunchCtx& lc, const TeachArgs& t, const VocabArgs& a, const Status& st) {
  return launch_after(teach_entries_kernel, (unsigned)std::min<int64_t>((t.T + 7) / 8, (int64_t)lc.num_sms * 8), 256, 0, lc.stream, t, a, st);
}

}  // namespace gpo
