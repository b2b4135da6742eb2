// Logits as a sampler takes them, their log-probabilities, and the gradient of the raw ones (formulas in
// include/graphpo.h): penalties for the tokens of a row's history, biases, a mask, a scale.
//
// One launch, no workspace.  A row is the work of a cluster of 1 to 8 CTAs (as many as few rows leave SMs for), which take
// slices of it in turn: kThreads x kVecs accesses of 16 bytes, fetched one slice ahead into registers.  What makes an
// entry special, a token of the history or a bias, is found per slice: every CTA reads the row's whole history (a few
// thousand tokens, from L1 after the first slice) and counts those of the slice in shared memory, a word per entry and one bit in
// a bitmap; the mask's bits of the slice are another bitmap.  So the pass over the logits looks at two bytes per 8 of them, and at
// the counts of special ones only, of which 4096 consecutive logits have a few.  Sums of exponentials run with the
// pass, relative to a maximum of each thread's own; threads, warps and CTAs of a row are joined in a fixed order.
#define GPO_REPORT __noinline__
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gpo_pair.cuh"
#include "gpo_vocab_math.cuh"

namespace gpo {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kCtas = 4;                         // on one SM
constexpr int kVecs = 2;                         // accesses of 32 bytes of a thread that are in flight
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr uint32_t kSeen = 1u << 31, kBiased = 1u << 30, kCount = kBiased - 1;  // an entry's word: flags, occurrences
enum Op { kAdjust, kScore, kGrad };              // write the adjusted logits, only their statistics, the gradient

// A vector of 32 bytes of logits.
struct Vec {
  uint32_t w[8];
};
// (streamed: nothing reads a row again but the few special entries)
__device__ __forceinline__ Vec load_global(const void* p) {
  Vec r;
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
               : "l"(p)
               : "memory");
  return r;
}
// The same where `take` says so, else r stays as it is.
__device__ __forceinline__ void load_global_if(Vec& r, const void* p, bool take) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.s32 q, %9, 0;\n\t"
      "@q ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t}"
      : "+r"(r.w[0]), "+r"(r.w[1]), "+r"(r.w[2]), "+r"(r.w[3]), "+r"(r.w[4]), "+r"(r.w[5]), "+r"(r.w[6]), "+r"(r.w[7])
      : "l"(p), "r"((int)take)
      : "memory");
}
__device__ __forceinline__ void store_global(void* p, const Vec& x) {
  asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x.w[0]), "r"(x.w[1]), "r"(x.w[2]),
               "r"(x.w[3]), "r"(x.w[4]), "r"(x.w[5]), "r"(x.w[6]), "r"(x.w[7])
               : "memory");
}

template <int kType>
struct Raw;
template <>
struct Raw<GPO_DT_F32> {
  using T = float;
  static constexpr int kPer = 8;
  static constexpr bool kFloors = false;
  // the entries of `take`, `other` in the place of the rest; those of `b` in the places `of_b`
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t other) {
    Vec x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = take >> i & 1u ? r.w[i] : other;
    return x;
  }
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take) { return keep(r, take, 0xFF800000u); }  // -inf
  static __device__ __forceinline__ Vec choose(const Vec& a, const Vec& b, uint32_t of_b) {
    Vec x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = of_b >> i & 1u ? b.w[i] : a.w[i];
    return x;
  }
  static __device__ __forceinline__ Vec floor(const Vec& r) { return r; }
  static __device__ __forceinline__ float top(const Vec& r) {
    float t = __uint_as_float(r.w[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) t = fmaxf(t, __uint_as_float(r.w[i]));
    return t;
  }
  static __device__ __forceinline__ void widen(const Vec& r, float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(r.w[i]);
  }
  static __device__ __forceinline__ Vec narrow(const float (&y)[8]) {
    Vec r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(y[i]);
    return r;
  }
  static __device__ __forceinline__ float get(const Vec& r, int i) { return __uint_as_float(r.w[i]); }
  static __device__ __forceinline__ float get1(T x) { return x; }
  static __device__ __forceinline__ T put(float x) { return x; }
};
// (two 16-bit entries per word)
struct Raw16 {
  static constexpr int kPer = 16;
  template <uint32_t kSel>
  static __device__ __forceinline__ uint32_t spread(uint32_t x) {
    uint32_t r;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(r) : "r"(x), "n"(kSel));
    return r;
  }
  // Sixteen ones in the half of word i / 2 for every bit i.  A nibble's bits go to the sign bits of four bytes (i + 7 (j + 1) is
  // different for every bit i and factor bit j, so that nothing carries), which prmt spreads.
  static __device__ __forceinline__ Vec mask(uint32_t take) {
    Vec m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = (take >> 4 * i & 15u) * 0x10204080u & 0x80808080u;
      m.w[2 * i] = spread<0x9988>(a);
      m.w[2 * i + 1] = spread<0xBBAA>(a);
    }
    return m;
  }
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t other) {
    Vec m = mask(take);
#pragma unroll
    for (int i = 0; i < 8; ++i) m.w[i] = (r.w[i] & m.w[i]) | (other & ~m.w[i]);
    return m;
  }
  static __device__ __forceinline__ Vec choose(const Vec& a, const Vec& b, uint32_t of_b) {
    Vec m = mask(of_b);
#pragma unroll
    for (int i = 0; i < 8; ++i) m.w[i] = (a.w[i] & ~m.w[i]) | (b.w[i] & m.w[i]);
    return m;
  }
};
template <>
struct Raw<GPO_DT_BF16> : Raw16 {
  using T = __nv_bfloat16;
  using Raw16::keep;
  static constexpr bool kFloors = true;
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take) { return Raw16::keep(r, take, 0xFF80FF80u); }
  static __device__ __forceinline__ __nv_bfloat162 h2(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  // -1e33 for -inf and what is below it, which for every scale is left out of a row all the same; a NaN stays one
  static __device__ __forceinline__ Vec floor(const Vec& r) {
    Vec x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __nv_bfloat162 t = __hmax2_nan(h2(r.w[i]), h2(0xF645F645u));
      x.w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    return x;
  }
  static __device__ __forceinline__ float top(const Vec& r) {
    __nv_bfloat162 t = h2(r.w[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) t = __hmax2(t, h2(r.w[i]));
    return fmaxf(__low2float(t), __high2float(t));
  }
  static __device__ __forceinline__ void widen(const Vec& r, float (&y)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[2 * i] = __uint_as_float(r.w[i] << 16);
      y[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ Vec narrow(const float (&y)[16]) {
    Vec r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
      r.w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return r;
  }
  static __device__ __forceinline__ float get(const Vec& r, int i) {
    return __uint_as_float(i & 1 ? r.w[i / 2] & 0xFFFF0000u : r.w[i / 2] << 16);
  }
  static __device__ __forceinline__ float get1(T x) { return __bfloat162float(x); }
  static __device__ __forceinline__ T put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Raw<GPO_DT_F16> : Raw16 {
  using T = __half;
  using Raw16::keep;
  static constexpr bool kFloors = false;  // (fp16 has no number that is below all that counts)
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take) { return Raw16::keep(r, take, 0xFC00FC00u); }
  static __device__ __forceinline__ __half2 h2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
  static __device__ __forceinline__ Vec floor(const Vec& r) { return r; }
  static __device__ __forceinline__ float top(const Vec& r) {
    __half2 t = h2(r.w[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) t = __hmax2(t, h2(r.w[i]));
    return fmaxf(__low2float(t), __high2float(t));
  }
  static __device__ __forceinline__ void widen(const Vec& r, float (&y)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = __half22float2(h2(r.w[i]));
      y[2 * i] = f.x;
      y[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ Vec narrow(const float (&y)[16]) {
    Vec r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __half2 h = __floats2half2_rn(y[2 * i], y[2 * i + 1]);
      r.w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return r;
  }
  static __device__ __forceinline__ float get(const Vec& r, int i) {
    return __half2float(__ushort_as_half((unsigned short)(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2])));
  }
  static __device__ __forceinline__ float get1(T x) { return __half2float(x); }
  static __device__ __forceinline__ T put(float x) { return __float2half_rn(x); }
};

// A row, read by one warp.
struct Row {
  const void* z;
  void* out;
  int shift;                  // elements between the 32-byte boundary before the row and the row
  int vecs;                   // accesses of 32 bytes that hold the row
  int live;                   // has a target, or a gradient, or needs none
  int vec;                    // the output's accesses of a whole vector are aligned
  int special;                // some entry may be special
  float scale, sl2;           // and times log2(e)
  float rep, inv, pres, freq; // repetition and 1 / it
  int64_t h0, hg, h1;         // the history, from where on generated
  int64_t b0, b1;             // biases
  const uint32_t* mask;       // null: every token is allowed
  int64_t target;             // -1: none
  float g, e, lse, logp, ent; // gradient
};

struct Shared {
  Row row;
  Part part[kWarps];
  float at;                   // the target's adjusted logit
  Part cluster[8];
  float cluster_at;
  int before[kWarps];         // special entries of each warp's words
};

constexpr int kSpan = 131072;         // entries of which it is known at one time which are special
constexpr int kWords = kSpan / 32;
constexpr int kGroups = kWords / 4;   // groups of four words, whose special entries are counted together
constexpr int kOwn = kGroups / kWarps;  // groups of a warp, side by side
constexpr int kCap = 2048;            // special entries that are looked at in one round
struct Smem {
  Shared sh;
  alignas(16) uint32_t special[kWords];
  alignas(16) uint32_t allow[kWords];
  uint32_t before[kGroups];           // special entries in the groups before
  union {
    struct {
      uint32_t list[kCap];            // the round's special entries, in their order,
      uint32_t count[kCap];           // and their flags and occurrences
    };
    float stage[kWarps][512];         // values of each warp on their way out
  };
};

// The bias of v among the row's (ascending).
__device__ __forceinline__ float bias_of(const LogitsArgs& a, const Row& w, int64_t v) {
  int64_t lo = w.b0, hi = w.b1;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (load_id(a.bias_ids, a.bias8, mid) < v) lo = mid + 1;
    else hi = mid;
  }
  return lo < w.b1 && load_id(a.bias_ids, a.bias8, lo) == v ? a.bias[lo] : 0.f;
}

// A special entry's logit before the scale, and its derivative.
__device__ __forceinline__ float adjusted(const LogitsArgs& a, const Row& w, uint32_t slot, float z, int v, float& slope) {
  const uint32_t n = slot & kCount;
  slope = slot & ~kBiased ? (z > 0.f ? w.inv : w.rep) : 1.f;
  float y = z * slope;
  if (n != 0) y -= fmaf(w.freq, (float)n, w.pres);
  if (slot & kBiased) y += bias_of(a, w, v);
  return y;
}

// One warp reads a row's arguments, a lane each, and checks them.
template <int kType, int kOp>
__device__ __forceinline__ void read_row(const LogitsArgs& a, const Status& st, int64_t r, Row& out, int lane, bool first) {
  using E = Raw<kType>;
  using T = typename E::T;
  const char* p = nullptr;
  bool wide = false;
  auto from = [&](const void* base, int64_t i, bool is8) {
    if (base) p = static_cast<const char*>(base) + (is8 ? 8 : 4) * i;
    wide = is8;
  };
  switch (lane) {
    case 0: from(a.scale, r, false); break;
    case 1: from(a.rep, r, false); break;
    case 2: from(a.pres, r, false); break;
    case 3: from(a.freq, r, false); break;
    case 4:
    case 5:
    case 6: from(a.spans, 3 * r + lane - 4, true); break;
    case 7:
    case 8: from(a.bias_spans, 2 * r + lane - 7, true); break;
    case 9: from(a.mask_row, r, false); break;
    case 10: from(a.target, r, a.target8 != 0); break;
    case 11: from(kOp == kGrad ? a.g : nullptr, r, false); break;
    case 12: from(kOp == kGrad ? a.ge : nullptr, r, false); break;
    case 13: from(kOp == kGrad && a.ge ? a.ent_in : nullptr, r, false); break;
    case 14: from(kOp == kGrad ? a.lse_in : nullptr, r, false); break;
    case 15: from(kOp == kGrad ? a.logp_in : nullptr, r, false); break;
    default: break;
  }
  const uint32_t lo = p ? *reinterpret_cast<const uint32_t*>(p) : 0u;
  const uint32_t hi = p && wide ? *reinterpret_cast<const uint32_t*>(p + 4) : (uint32_t)((int32_t)lo >> 31);
  auto f32 = [&](int l, const void* given, float all) {
    const float x = __uint_as_float(__shfl_sync(0xffffffffu, lo, l));
    return given ? x : all;
  };
  auto i64 = [&](int l) {
    const uint32_t x = __shfl_sync(0xffffffffu, lo, l), y = __shfl_sync(0xffffffffu, hi, l);
    return (int64_t)((uint64_t)y << 32 | x);
  };
  auto bad = [&](int code, int what) {
    if (first && lane == 0) report(st, code, 40 + what, (int)r);
  };
  Row w;
  const T* z = static_cast<const T*>(a.z) + r * a.z_stride;
  w.z = z;
  w.shift = (int)((reinterpret_cast<uintptr_t>(z) & 31) / sizeof(T));
  w.vecs = (int)((a.V + w.shift + E::kPer - 1) / E::kPer);
  const size_t osz = a.out32 ? 4 : sizeof(T);
  w.out = kOp == kScore ? nullptr : static_cast<char*>(a.out) + r * a.out_stride * osz;
  w.vec = kOp == kScore || ((reinterpret_cast<uintptr_t>(w.out) - w.shift * osz) & 31) == 0;
  w.scale = f32(0, a.scale, a.scale1);
  w.rep = f32(1, a.rep, a.rep1);
  w.pres = f32(2, a.pres, a.pres1);
  w.freq = f32(3, a.freq, a.freq1);
  if (!(w.scale >= 1e-4f && w.scale <= 1e4f) || !(w.rep > 0.f && w.rep < INFINITY) || !isfinite(w.pres) || !isfinite(w.freq)) {
    bad(GPO_ERR_INVALID_ARG, 1);
    w.scale = w.rep = 1.f;
    w.pres = w.freq = 0.f;
  }
  w.sl2 = w.scale * kLog2e;
  w.inv = 1.f / w.rep;
  const int64_t h0 = i64(4), hg = i64(5), h1 = i64(6);
  w.h0 = w.hg = w.h1 = 0;
  if (h0 < 0 || hg < h0 || h1 < hg || h1 > a.hist_len || h1 - h0 > (int64_t)kCount) bad(GPO_ERR_SHAPE, 2);  // (without spans: zeros)
  else if (w.rep != 1.f || w.pres != 0.f || w.freq != 0.f) w.h0 = h0, w.hg = hg, w.h1 = h1;
  w.b0 = i64(7);
  w.b1 = i64(8);
  if (!a.bias_spans) w.b1 = a.bias_len;
  if (w.b0 < 0 || w.b1 < w.b0 || w.b1 > a.bias_len) {
    bad(GPO_ERR_SHAPE, 3);
    w.b0 = w.b1 = 0;
  }
  w.special = w.h1 > w.h0 || w.b1 > w.b0;
  const int64_t m = a.mask_row ? i64(9) : a.mask_rows == 1 ? 0 : r;
  w.mask = a.mask && m >= 0 && m < a.mask_rows ? a.mask + m * a.mask_stride : nullptr;
  if (a.mask && m >= a.mask_rows) bad(GPO_ERR_SHAPE, 4);
  w.target = a.target ? i64(10) : -1;
  if (w.target >= a.V) {
    bad(GPO_ERR_SHAPE, 5);
    w.target = -1;
  }
  w.live = kOp == kAdjust || w.target >= 0;
  w.g = f32(11, a.g, 0.f);
  w.e = f32(12, a.ge, 0.f);
  w.ent = f32(13, a.ge, 0.f);
  w.lse = f32(14, a.g, 0.f);
  w.logp = f32(15, a.g, 0.f);
  // (a row that nothing was left of has no gradient)
  if (kOp == kGrad && ((w.g == 0.f && w.e == 0.f) || w.lse == -INFINITY)) w.live = 0;
  if (lane == 0) out = w;
}

// Calls f(id - lo, i) for the ids of the history in the n entries from lo on, i their place.
template <class F>
__device__ __forceinline__ void for_history(const LogitsArgs& a, const Row& w, int lo, int64_t n, F f) {
  for (int64_t i = w.h0 + threadIdx.x; i < w.h1; i += 4 * kThreads) {
    int64_t id[4];
    // (one branch around the loads of a thread, which are then in flight together)
    if (a.hist8) {
#pragma unroll
      for (int k = 0; k < 4; ++k) id[k] = i + k * kThreads < w.h1 ? static_cast<const int64_t*>(a.hist)[i + k * kThreads] : -1;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) id[k] = i + k * kThreads < w.h1 ? static_cast<const int32_t*>(a.hist)[i + k * kThreads] : -1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t rel = id[k] - lo;
      if (id[k] >= 0 && rel >= 0 && rel < n) f(rel, i + k * kThreads);
    }
  }
}

// Marks the special entries of a span of n from entry lo on (below 0: before the row) in their bitmap, which was zeros, and
// writes that of the allowed ones where the row has a mask.
// (last: of the row; ids past the vocabulary are found there)
__device__ __forceinline__ void mark_span(const LogitsArgs& a, const Status& st, const Row& w, int lo, int n, bool last, Smem& sm) {
  const int V = (int)a.V;
  if (w.mask) {
    const int words = (V + 31) >> 5, sh = lo & 31, at0 = lo >> 5;
    for (int j = threadIdx.x; j < (n + 31) / 32; j += kThreads) {
      const int at = at0 + j;
      const uint32_t x0 = at >= 0 && at < words ? __ldg(w.mask + at) : 0u, x1 = at + 1 < words ? __ldg(w.mask + at + 1) : 0u;
      sm.allow[j] = __funnelshift_r(x0, x1, (uint32_t)sh);
    }
  }
  if (!w.special) return;
  for_history(a, w, lo, last ? INT64_MAX : n, [&](int64_t rel, int64_t i) {
    if (lo + rel >= V) report(st, GPO_ERR_SHAPE, 46, (int)i);
    else atomicOr(sm.special + (rel >> 5), 1u << (rel & 31u));
  });
  for (int64_t i = w.b0 + threadIdx.x; i < w.b1; i += kThreads) {
    const int64_t id = load_id(a.bias_ids, a.bias8, i), rel = id - lo;
    if (id < 0 || id >= V || (i > w.b0 && load_id(a.bias_ids, a.bias8, i - 1) >= id)) report(st, GPO_ERR_SHAPE, 47, (int)i);
    else if (rel >= 0 && rel < n) atomicOr(sm.special + (rel >> 5), 1u << (rel & 31u));
  }
}

// The number of special entries of the span, and of those before each group of words; these leave the allowed ones.
__device__ __forceinline__ int rank_span(int n, bool masked, Smem& sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, groups = (n + 127) / 128;
  int sum = 0;
#pragma unroll 1
  for (int g0 = warp * kOwn; g0 < min(groups, (warp + 1) * kOwn); g0 += 32) {
    const int g = g0 + lane;
    const uint4 x = reinterpret_cast<const uint4*>(sm.special)[g];
    uint4& al = reinterpret_cast<uint4*>(sm.allow)[g];
    al = masked ? make_uint4(al.x & ~x.x, al.y & ~x.y, al.z & ~x.z, al.w & ~x.w) : make_uint4(~x.x, ~x.y, ~x.z, ~x.w);
    const int own = __popc(x.x) + __popc(x.y) + __popc(x.z) + __popc(x.w);
    int upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    sm.before[g] = sum + upto - own;
    sum += __shfl_sync(0xffffffffu, upto, 31);
  }
  if (lane == 0) sm.sh.before[warp] = sum;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < kWarps; ++k) {
    const int y = sm.sh.before[k];
    if (k < warp) before += y;
    all += y;
  }
  for (int g = warp * kOwn + lane; g < min(groups, (warp + 1) * kOwn); g += 32) sm.before[g] += before;
  return all;
}

// The round's special entries, those of ranks [first, first + kCap), and their flags and counts.  Between barriers of the caller.
__device__ __forceinline__ void list_special(const LogitsArgs& a, const Row& w, int lo, int n, int first, int total, Smem& sm) {
  for (int g = threadIdx.x; g < (n + 127) / 128; g += kThreads) {
    const uint4 x = reinterpret_cast<const uint4*>(sm.special)[g];
    int k = (int)sm.before[g] - first;
    auto put = [&](uint32_t bits, int rel) {
      for (; bits; bits &= bits - 1, ++k)
        if (k >= 0 && k < kCap) sm.list[k] = rel + __ffs(bits) - 1;
    };
    put(x.x, 128 * g);
    put(x.y, 128 * g + 32);
    put(x.z, 128 * g + 64);
    put(x.w, 128 * g + 96);
  }
  for (int c = threadIdx.x; c < min(kCap, total - first); c += kThreads) sm.count[c] = 0;
  __syncthreads();
  auto at = [&](uint32_t rel) {
    const uint32_t word = rel >> 5 & 3u, low = (1u << (rel & 31u)) - 1u;
    const uint4 x = reinterpret_cast<const uint4*>(sm.special)[rel >> 7];
    const uint32_t own = word == 0 ? x.x : word == 1 ? x.y : word == 2 ? x.z : x.w;
    return (int)sm.before[rel >> 7] - first + __popc(own & low) + (word > 0 ? __popc(x.x) : 0) + (word > 1 ? __popc(x.y) : 0) +
           (word > 2 ? __popc(x.z) : 0);
  };
  for_history(a, w, lo, min((int64_t)n, a.V - lo), [&](int64_t rel, int64_t i) {
    const int k = at((uint32_t)rel);
    if (k < 0 || k >= kCap) return;
    if (i >= w.hg) atomicAdd(sm.count + k, 1u);
    else atomicOr(sm.count + k, kSeen);
  });
  for (int64_t i = w.b0 + threadIdx.x; i < w.b1; i += kThreads) {
    const int64_t id = load_id(a.bias_ids, a.bias8, i), rel = id - lo;
    if (id < 0 || id >= a.V || rel < 0 || rel >= n || !(sm.special[rel >> 5] >> (rel & 31) & 1u)) continue;
    const int k = at((uint32_t)rel);
    if (k >= 0 && k < kCap) atomicOr(sm.count + k, kBiased);
  }
}

// Which entries of the vector at v are in the row.
template <int kPer>
__device__ __forceinline__ uint32_t in_row(int v, int V) {
  uint32_t in = (1u << kPer) - 1u;
  if (v < 0) in &= v <= -kPer ? 0u : in << -v;
  if (v + kPer > V) in &= v >= V ? 0u : in >> (v + kPer - V);
  return in;
}

// A vector of the row, whose first entry is v; entries outside the row are 0.
template <int kType>
__device__ __forceinline__ Vec load_vec(const void* row, int v, int V) {
  using E = Raw<kType>;
  using T = typename E::T;
  const T* z = static_cast<const T*>(row);
  if (v >= 0 && v + E::kPer <= V) return load_global(z + v);
  float y[E::kPer];
#pragma unroll
  for (int i = 0; i < E::kPer; ++i) y[i] = v + i >= 0 && v + i < V ? E::get1(z[v + i]) : 0.f;
  return E::narrow(y);
}

// kPer values of every lane to the row, by a whole warp: lane 0's first entry is v0, `in` says which of a lane's are to be written (none from `end` on).
// In an aligned row a lane's are one or two accesses; in others the warp's go through shared memory, so that an access
// takes 32 entries side by side.
template <int kType>
__device__ __forceinline__ void store_vec(bool wide, const Row& w, const float (&y)[Raw<kType>::kPer], const Vec& narrow, int v0, uint32_t in,
                                          int end, float* stage, int lane) {
  using E = Raw<kType>;
  using T = typename E::T;
  constexpr int kPer = E::kPer;
  const int v = v0 + lane * kPer;
  const bool whole = in == (1u << kPer) - 1u;
  if (w.vec && whole) {
    if (wide) {
      float* p = static_cast<float*>(w.out) + v;
#pragma unroll
      for (int i = 0; i < kPer / 8; ++i) {
        Vec x;
#pragma unroll
        for (int k = 0; k < 8; ++k) x.w[k] = __float_as_uint(y[8 * i + k]);
        store_global(p + 8 * i, x);
      }
    } else {
      store_global(static_cast<T*>(w.out) + v, narrow);
    }
  }
  if (w.vec && __all_sync(0xffffffffu, whole)) return;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPer; ++i) stage[lane * kPer + i] = wide || sizeof(T) == 4 ? y[i] : E::get(narrow, i);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int x = v0 + i * 32 + lane;
    const float f = stage[i * 32 + lane];
    if (x < 0 || x >= end) continue;
    if (wide) static_cast<float*>(w.out)[x] = f;
    else static_cast<T*>(w.out)[x] = E::put(f);
  }
  __syncwarp();
}

// The statistics of a row from its joined parts; zy: the target's logit in units of log 2, which is in no part.
__device__ __forceinline__ void finish_row(const LogitsArgs& a, int64_t r, bool has, float zy, const Part& p) {
  const bool at = has && !(zy <= kLow);  // (a NaN is one)
  const float top = at ? fmaxf(p.m, zy) : p.m;
  const float c = p.m - top, ec = exp2f(c);
  const float y = at ? zy - top : -INFINITY, ey = at ? exp2f(y) : 0.f;
  const float others = ec * p.s, total = others + ey;
  const bool none = total == 0.f;
  const float lt = y == 0.f ? log1pf(others) : logf(total);
  if (a.logp) a.logp[r] = !has ? 0.f : at ? fmaf(y, kLn2, -lt) : -INFINITY;
  if (a.lse) a.lse[r] = none ? -INFINITY : fmaf(top, kLn2, lt);
  if (a.ent) a.ent[r] = none ? 0.f : lt - kLn2 * (ec * (p.u + c * p.s) + (at ? ey * y : 0.f)) / total;
}

__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_remote(uint32_t addr, float x) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(x) : "memory");
}

// Sums of exponentials so far, in two chains, relative to m.
struct Running {
  float m, s[2], u[2];
};
template <bool kEnt>
__device__ __forceinline__ void raise(Running& p, float top) {
  if (!(top > p.m)) return;
  const float c = p.m - top, e = ex2(c);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (kEnt) p.u[k] = e * fmaf(c, p.s[k], p.u[k]);
    p.s[k] *= e;
  }
  p.m = top;
}

template <int kType, int kOp, bool kEnt>
__global__ void __launch_bounds__(kThreads, kCtas) logits_kernel(LogitsArgs a, int cluster, Status st) {
  using E = Raw<kType>;
  using T = typename E::T;
  constexpr int kPer = E::kPer, kSpanVecs = kSpan / kPer, kBatch = kThreads * kVecs;
  constexpr uint32_t kAll = (1u << kPer) - 1u;
  extern __shared__ __align__(16) unsigned char smem[];
  Smem& sm = *reinterpret_cast<Smem*>(smem);
  Shared& sh = sm.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = (int)a.V;
  float* stage = sm.stage[warp];
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t r = blockIdx.x / cluster;
  const bool wide = a.out32 && sizeof(T) == 2;
  if (warp == 0) read_row<kType, kOp>(a, st, r, sh.row, lane, rank == 0);
  if (a.spans || a.bias)
    for (int g = tid; g < kGroups; g += kThreads) reinterpret_cast<uint4*>(sm.special)[g] = make_uint4(0u, 0u, 0u, 0u);
  if (blockIdx.x == 0 && tid == 32) next_tag(st);
  __syncthreads();
  const Row& w = sh.row;
  // this CTA's share of the row's vectors (in whole words of the bitmaps)
  const int share = (w.vecs + cluster * 4 - 1) / (cluster * 4) * 4, v0 = min(w.vecs, rank * share), v1 = min(w.vecs, v0 + share);
  if (!w.live) {
    if (kOp == kGrad) {  // zeros
      float d[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j) d[j] = 0.f;
      const int end = min(V, v1 * kPer - w.shift);
#pragma unroll 1
      for (int b = v0 + tid; b - lane < v1; b += kThreads) {
        const int v = b * kPer - w.shift;
        store_vec<kType>(false, w, d, E::narrow(d), v - lane * kPer, b < v1 ? in_row<kPer>(v, V) : 0u, end, stage, lane);
      }
    } else if (rank == 0 && tid == 0) {
      if (a.logp) a.logp[r] = 0.f;
      if (a.lse) a.lse[r] = 0.f;
      if (a.ent) a.ent[r] = 0.f;
    }
    return;
  }
  const bool marked = w.special || w.mask;
  const float scale = w.scale, sl2 = w.sl2;
  const float gs = kOp == kGrad ? w.g * scale : 0.f, es = kOp == kGrad ? w.e * scale : 0.f;
  const float w_lse = kOp == kGrad ? w.lse : 0.f, w_ent = kOp == kGrad ? w.ent : 0.f;
  const Vec* base = reinterpret_cast<const Vec*>(static_cast<const char*>(w.z) - w.shift * sizeof(T)) + tid;
  // vectors that are full of the row's entries
  const int whole0 = w.shift ? 1 : 0, whole1 = min(v1, (V + w.shift) / kPer);
  // whether the warp's 32 vectors, the first at b + i kThreads + 32 warp, are all whole and before `end`
  auto full = [&](int b, int i, int end) {
    const int n = end - 32 - whole0, at = b + i * kThreads + warp * 32 - whole0;
    return (uint32_t)at <= (uint32_t)n && n >= 0;
  };
  Vec raw[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
#pragma unroll
    for (int k = 0; k < 8; ++k) raw[i].w[k] = 0u;
    load_global_if(raw[i], base + v0 + i * kThreads, full(v0, i, whole1));
  }
  Running p = {kLow, {0.f, 0.f}, {0.f, 0.f}};
#pragma unroll 1
  for (int s0 = v0; s0 < v1; s0 += kSpanVecs) {
      const int s1 = min(v1, s0 + kSpanVecs), lo = s0 * kPer - w.shift, n = (s1 - s0) * kPer;
      if (marked) {
        mark_span(a, st, w, lo, n, s1 == w.vecs, sm);
        __syncthreads();
      }
      const int total = w.special ? rank_span(n, w.mask != nullptr, sm) : 0;
      const int trel = w.target >= 0 && w.target >= lo && w.target < (int64_t)lo + n ? (int)w.target - lo : -1, tvec = trel < 0 ? -1 : trel / kPer;
      // a special entry, or the target: rel its place in the span
      auto single = [&](int rel, uint32_t slot) {
        const int v = lo + rel;
        const bool may = !w.mask || (__ldg(w.mask + (v >> 5)) >> (v & 31) & 1u);
        const float z = may ? E::get1(static_cast<const T*>(w.z)[v]) : 0.f;
        float slope = 1.f;
        const float y = !may ? -INFINITY : slot ? adjusted(a, w, slot, z, v, slope) : z;
        if (kOp != kGrad && rel == trel) sh.at = y;
        if (kOp == kGrad) {
          float d = 0.f;
          if (may && rel == trel) {  // (p from its log-probability, which has the digits of 1 - p)
            const float pe = expf(w.logp);
            d = -gs * expm1f(w.logp) - (kEnt && pe > 0.f ? es * pe * (w.logp + w.ent) : 0.f);
          } else if (may) {
            const float x = fmaxf(fmaf(y, scale, -w.lse), -200.f), pe = ex2(x * kLog2e);
            d = w.lse == w.lse ? -gs * pe - (kEnt ? es * pe * (x + w.ent) : 0.f) : w.lse;
          }
          static_cast<T*>(w.out)[v] = E::put(d * slope);
        } else {
          if (kOp == kAdjust) {
            if (wide) static_cast<float*>(w.out)[v] = y * scale;
            else static_cast<T*>(w.out)[v] = E::put(y * scale);
          }
          if (!may || rel == trel) return;
          raise<kEnt>(p, y * sl2);
          const float d = fmaf(y, sl2, -p.m), x = ex2(d);
          p.s[0] += x;
          if (kEnt) p.u[0] = fmaf(x, fmaxf(d, -200.f), p.u[0]);
        }
      };
      // a warp's 32 vectors, idx this lane's; edge: some may be outside the row or the span
      auto dense = [&](const Vec& z, int idx, bool edge) {
        const int v = idx * kPer - w.shift, at = idx - s0;
        uint32_t take = kAll, sp = 0u, in = kAll;
        if (edge) in = idx >= s1 ? 0u : in_row<kPer>(v, V) & kAll;
        if (marked) {
          const int k = edge ? min(at, kSpan / kPer - 1) : at;
          auto bits = [&](const uint32_t* p) -> uint32_t {
            return kPer == 16 ? reinterpret_cast<const uint16_t*>(p)[k] : reinterpret_cast<const uint8_t*>(p)[k];
          };
          take = bits(sm.allow);
          if (kOp != kScore && total) sp = bits(sm.special);
        }
        if (edge) take &= in;
        if (at == tvec) {
          const uint32_t bit = 1u << (uint32_t)trel % kPer;
          sp |= bit;
          take &= ~bit;
        }
        if (kOp == kGrad) {
          // d y_j = -gs p_j - es p_j (log p_j + H)
          float y[kPer];
          E::widen(z, y);
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            float d = fmaf(y[j], scale, -w_lse);
            if (kEnt) d = fmaxf(d, -200.f);
            const float x = ex2(d * kLog2e);
            y[j] = kEnt ? x * fmaf(-es, d + w_ent, -gs) : -gs * x;
          }
          Vec o = E::narrow(y);
          if (take != kAll) o = E::keep(o, take, 0u);
          if (sp) o = E::choose(o, z, sp);  // (special ones keep theirs: `out` may be the logits, and they are read once more)
          if (sizeof(T) == 4) E::widen(o, y);
          store_vec<kType>(false, w, y, o, v - lane * kPer, in, min(V, s1 * kPer - w.shift), stage, lane);
        } else {
          Vec x = z;
          if (take != kAll) x = E::keep(x, take);
          if (kEnt && kOp == kScore) x = E::floor(x);
          const float top = E::top(x) * sl2;
          float y[kPer];
          if (kOp == kAdjust) {
            E::widen(x, y);
            float o[kPer];
            Vec q = x;
#pragma unroll
            for (int j = 0; j < kPer; ++j) o[j] = y[j] * scale;
            if (scale != 1.f && !wide) q = E::narrow(o);
            if (sp && !wide) q = E::choose(q, z, sp);
            if (sizeof(T) == 4) E::widen(q, o);
            store_vec<kType>(wide, w, o, q, v - lane * kPer, in, min(V, s1 * kPer - w.shift), stage, lane);
          } else {
            E::widen(x, y);
          }
          raise<kEnt>(p, top);
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            const float d = fmaf(y[j], sl2, -p.m), e = ex2(d);
            p.s[j & 1] += e;
            // (0 times -inf is 0 here)
            if (kEnt) p.u[j & 1] = fmaf(e, kOp == kScore && E::kFloors ? d : fmaxf(d, -200.f), p.u[j & 1]);
          }
        }
      };
#pragma unroll 1
      for (int b = s0; b < s1; b += kBatch) {
        const int next = b + kBatch < s1 ? b + kBatch : s1;  // (of the span, or the next span's first)
        uint32_t rest = 0u;                                  // vectors at the ends
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          if (full(b, i, min(s1, whole1))) dense(raw[i], b + i * kThreads + tid, false);
          else rest |= 1u << i;
          load_global_if(raw[i], base + next + i * kThreads, full(next, i, whole1));
        }
#pragma unroll 1
        for (; rest; rest &= rest - 1) {
          const int idx = b + (__ffs(rest) - 1) * kThreads + tid;
          if (idx - lane < s1) dense(load_vec<kType>(w.z, idx * kPer - w.shift, V), idx, true);
        }
      }
      if (total) {
        for (int first = 0; first < total; first += kCap) {
          __syncthreads();
          list_special(a, w, lo, n, first, total, sm);
          __syncthreads();
          for (int k = tid; k < min(kCap, total - first); k += kThreads) single((int)sm.list[k], sm.count[k]);
        }
      }
      if (trel >= 0 && !(total && (sm.special[trel >> 5] >> (trel & 31) & 1u))) {
        __syncthreads();
        if (tid == 0) single(trel, 0u);
      }
      if (s1 < v1 && marked) {
        __syncthreads();
        if (total)
          for (int g = tid; g < kGroups; g += kThreads) reinterpret_cast<uint4*>(sm.special)[g] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
      }
  }
  if (kOp == kGrad) return;
  Part x = {p.m, p.s[0] + p.s[1], p.u[0] + p.u[1]};
  auto join_lanes = [&](int from) {
    for (int o = from; o > 0; o >>= 1) {
      const Part y = {__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.s, o),
                      __shfl_xor_sync(0xffffffffu, x.u, o)};
      x = join<kEnt>(x, y);
    }
  };
  join_lanes(16);
  if (lane == 0) sh.part[warp] = x;
  __syncthreads();
  if (warp == 0) {
    x = lane < kWarps ? sh.part[lane] : Part{kLow, 0.f, 0.f};
    join_lanes(kWarps / 2);
    if (lane == 0 && cluster > 1) {
      st_remote(remote(&sh.cluster[rank].m, 0), x.m);
      st_remote(remote(&sh.cluster[rank].s, 0), x.s);
      st_remote(remote(&sh.cluster[rank].u, 0), x.u);
      // (who has the target's logit passes it on)
      const int64_t tv = w.target < 0 ? -1 : (w.target + w.shift) / kPer;
      if (tv >= v0 && tv < v1) st_remote(remote(&sh.cluster_at, 0), sh.at);
    }
    __syncwarp();
  }
  if (cluster > 1) cluster_sync();
  if (rank != 0 || tid != 0) return;
  float at = sh.at;
  if (cluster > 1) {
    at = sh.cluster_at;
    x = sh.cluster[0];
    for (int c = 1; c < cluster; ++c) x = join<kEnt>(x, sh.cluster[c]);
  }
  finish_row(a, r, w.target >= 0, w.target >= 0 ? at * w.sl2 : 0.f, x);
}

template <int kType, int kOp, bool kEnt>
cudaError_t setup_one() {
  return cudaFuncSetAttribute(logits_kernel<kType, kOp, kEnt>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
}
template <int kType>
cudaError_t setup_type() {
  cudaError_t e = setup_one<kType, kAdjust, false>();
  if (e == cudaSuccess) e = setup_one<kType, kAdjust, true>();
  if (e == cudaSuccess) e = setup_one<kType, kScore, false>();
  if (e == cudaSuccess) e = setup_one<kType, kScore, true>();
  if (e == cudaSuccess) e = setup_one<kType, kGrad, false>();
  if (e == cudaSuccess) e = setup_one<kType, kGrad, true>();
  return e;
}

template <int kType, int kOp, bool kEnt>
cudaError_t launch_one(const LaunchCtx& lc, const LogitsArgs& a, const Status& st) {
  // a row of few gets a cluster, each of whose CTAs has a batch of its vectors or more
  const int64_t ctas = kCtas * (int64_t)lc.num_sms, batches = (a.V / Raw<kType>::kPer + kThreads * kVecs - 1) / (kThreads * kVecs);
  int cluster = 1;
  while (cluster < 8 && 2 * cluster * a.R <= ctas && 2 * cluster <= batches) cluster *= 2;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)cluster;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(cluster * a.R));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem);
  cfg.stream = lc.stream;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logits_kernel<kType, kOp, kEnt>, a, cluster, st);
}
template <int kType>
cudaError_t launch_type(const LaunchCtx& lc, const LogitsArgs& a, const Status& st) {
  if (a.g) return a.ge ? launch_one<kType, kGrad, true>(lc, a, st) : launch_one<kType, kGrad, false>(lc, a, st);
  if (a.out) return a.ent ? launch_one<kType, kAdjust, true>(lc, a, st) : launch_one<kType, kAdjust, false>(lc, a, st);
  return a.ent ? launch_one<kType, kScore, true>(lc, a, st) : launch_one<kType, kScore, false>(lc, a, st);
}

}  // namespace

cudaError_t setup_logits() {
  cudaError_t e = setup_type<GPO_DT_BF16>();
  if (e == cudaSuccess) e = setup_type<GPO_DT_F16>();
  if (e == cudaSuccess) e = setup_type<GPO_DT_F32>();
  return e;
}

cudaError_t launch_logits(const LaunchCtx& lc, const LogitsArgs& a, int dtype, const Status& st) {
  switch (dtype) {
    case GPO_DT_BF16: return launch_type<GPO_DT_BF16>(lc, a, st);
    case GPO_DT_F16: return launch_type<GPO_DT_F16>(lc, a, st);
    default: return launch_type<GPO_DT_F32>(lc, a, st);
  }
}

}  // namespace gpo
