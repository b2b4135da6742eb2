// Logits as a sampler takes them, their log-probabilities, and the gradient of the raw ones (formulas in
// include/graphpo.h): penalties for the tokens of a row's history, biases, a mask, a scale.
//
// One launch, no workspace.  A CTA takes a row (of few rows a cluster of 2 to 8 a row), four of them on an SM.
//   fetch    Each warp fetches its own 1 KB pieces of the row by bulk copies, two at a time, in a ring of its own: no warp waits
//            for another, and the first of them are under way before the row's arguments are known.
//   special  What the history or a bias changes: a bitmap of the span (up to 81920 entries at a time), ranks by counting its
//            bits, a list of them in their order with flags and occurrences.  Three barriers; the history is read once, of what was
//            generated twice (the second time from L1).
//   dense    One pass over all others, 32 bytes a lane: two bytes of a bitmap say which of 16 count (allowed, not special).
//            Sums of exponentials run with the pass, relative to a maximum of each thread's own.  The entries are rounded
//            and stored as whole vectors; of rows of other alignment through shared memory.
//   ends     Special entries, the target, and what lies before the row's first and behind its last boundary of 32 bytes: a
//            thread each, their logits from L2, where the pass has just been.
// Threads, warps and CTAs of a row are joined in a fixed order, and no float is added atomically: the same bits on every run.
//
// What bounds it: without penalties and masks HBM and the issue of instructions together (us, calls in a row in a graph):
// gradient of 4096 x 65536 bf16 (2870 live) 141, 5.8 TB/s of the bytes needed; log-probabilities and entropies of the same 92,
// of which the exponentials alone take 41 of the special-function units' time and 10 instructions an entry at 2.8 of 4 a
// cycle the rest; 256 x 131072 adjusted 28, 4.8 TB/s.  With histories of 1300 tokens, penalties and masks 188, 144; with 4000 tokens 52: the
// bitmaps' bits spread over 16-bit lanes (2 instructions an entry), then the special entries (3 to 4).  Longer histories and
// vocabularies: beside kSpan.  Where a row has many times kCap special entries the lists are read as many times: a bias for each of 131072
// tokens takes 8.7 ms for 256 rows, 1.6 ms for one.
// Tried when those three were 187, 144 and 48 (gradient, log-probabilities, step): loads to registers in place of the rings 233,
// 151, 69; 3 CTAs and 2 KB pieces 190, 147, 66; 2 CTAs of 512 threads 207, 175, 69; the special entries' sums before the pass,
// whose scattered reads come from HBM then, 290, 170, 97; every warp reading the row's arguments itself 190, 153, 49;
// the bits spread by a product and byte permutations 188, 149, 48.
#define GPO_REPORT __noinline__
#define GPO_TAG_ADVANCES 1
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gpo_pair.cuh"
#include "gpo_vocab_math.cuh"

namespace gpo {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kCtas = 4;                         // on one SM
constexpr int kChunk = 1024;                     // bytes of a row that a warp fetches at a time,
constexpr int kChunkVecs = kChunk / 32;          // of 32 for a lane,
constexpr int kDeep = 2;                         // and how many of them are in flight
constexpr int kLead = 16;                        // bits of the bitmaps before a span's first whole 32 bytes
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr uint32_t kSeen = 1u << 31, kBiased = 1u << 30, kCount = kBiased - 1;  // an entry's word: flags, occurrences
// the adjusted logits (in fp32, of 16-bit ones), only their statistics, the gradient, the statistics with entropies without targets
enum Op { kAdjust, kAdjust32, kScore, kGrad, kScoreAll };
__host__ __device__ constexpr bool writes(int op) { return op == kAdjust || op == kAdjust32; }
__host__ __device__ constexpr bool scores(int op) { return op == kScore || op == kScoreAll; }
// entropies of rows that may have no target (see raise)
__host__ __device__ constexpr bool holds_out(int op, bool ent) { return ent && (writes(op) || op == kScoreAll); }

// 32 bytes of logits, a lane's.
struct Vec {
  uint32_t w[8];
};

template <int kType>
struct Raw;
template <>
struct Raw<GPO_DT_F32> {
  using T = float;
  static constexpr int kPer = 8;
  static constexpr bool kFloors = false;
  // the entries of `take`, `other` in the place of the rest; those of `b` in the places `of_b`
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t other, uint32_t) {
    Vec x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = take >> i & 1u ? r.w[i] : other;
    return x;
  }
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t) { return keep(r, take, 0xFF800000u, 0u); }  // -inf
  static __device__ __forceinline__ Vec choose(const Vec& a, const Vec& b, uint32_t of_b, uint32_t) {
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
  // leaves out the entries that are `top`; returns how many they were
  static __device__ __forceinline__ int take_out(Vec& r, float top) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (__uint_as_float(r.w[i]) == top) r.w[i] = 0xFF800000u, ++n;
    return n;
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
  // Sixteen ones in the half of word i / 2 for every bit i: two words at a time from a table of a nibble's, whose 16 entries of 8
  // bytes lie in all banks once (three instructions a nibble; a product and two byte permutations took six).
  static __device__ __forceinline__ Vec mask(uint32_t take, uint32_t table) {
    Vec m;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(m.w[2 * i]), "=r"(m.w[2 * i + 1]) : "r"((take << 3 >> 4 * i & 0x78u) | table));
    return m;
  }
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t other, uint32_t table) {
    Vec m = mask(take, table);
#pragma unroll
    for (int i = 0; i < 8; ++i) m.w[i] = (r.w[i] & m.w[i]) | (other & ~m.w[i]);
    return m;
  }
  // (same: ones in the 16-bit lanes that leave)
  static __device__ __forceinline__ int leave(uint32_t& w, uint32_t same, uint32_t other) {
    w = (w & ~same) | (other & same);
    return __popc(same);
  }
  static __device__ __forceinline__ Vec choose(const Vec& a, const Vec& b, uint32_t of_b, uint32_t table) {
    Vec m = mask(of_b, table);
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
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t table) { return Raw16::keep(r, take, 0xFF80FF80u, table); }
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
  static __device__ __forceinline__ int take_out(Vec& r, float top) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) n += leave(r.w[i], __heq2_mask(h2(r.w[i]), __float2bfloat162_rn(top)), 0xF645F645u);
    return n / 16;
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
  static __device__ __forceinline__ Vec keep(const Vec& r, uint32_t take, uint32_t table) { return Raw16::keep(r, take, 0xFC00FC00u, table); }
  static __device__ __forceinline__ __half2 h2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
  static __device__ __forceinline__ Vec floor(const Vec& r) { return r; }
  static __device__ __forceinline__ float top(const Vec& r) {
    __half2 t = h2(r.w[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) t = __hmax2(t, h2(r.w[i]));
    return fmaxf(__low2float(t), __high2float(t));
  }
  static __device__ __forceinline__ int take_out(Vec& r, float top) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) n += leave(r.w[i], __heq2_mask(h2(r.w[i]), __float2half2_rn(top)), 0xFC00FC00u);
    return n / 16;
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

// A row's arguments, read by one warp.
struct Row {
  const void* z;
  void* out;
  int live;                   // has a target, or a gradient, or needs none
  int vec;                    // the output's vectors are on boundaries of 32 bytes where the row's are
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
  float held[kWarps];
  float at;                   // the target's adjusted logit
  Part cluster[8];
  float cluster_held[8];
  float cluster_at;
  int before[kWarps];         // special entries of each warp's words
};

// Entries of which it is known at one time which are special, and special entries that are looked at in one round: as many as four
// CTAs on an SM have memory for (57344 bytes each; a span's bitmaps and ranks take 9 bytes for 32 entries, a round's 8 for one).  The
// history is read anew for every span and every round (us: log-probabilities of 4096 x 65536 with histories to 1824, to 8992, of
// 1500 x 151936 to 9500, 256 x 151936 adjusted with histories to 16384): spans of 36864 with rounds twice as long 163, 200, 203, 99;
// 69632 and 768 146, 195, 187, 120; 69632 and 1536 146, 178, 181, 99; these 146, 178, 164, 82.
constexpr int kSpan = 81920;
constexpr int kWords = kSpan / 32;
constexpr int kGroups = kWords / 4;   // groups of four words, whose special entries are counted together
static_assert((kWarps & (kWarps - 1)) == 0 && kGroups % 32 == 0, "a join in halves, whole accesses of a warp");
constexpr int kCap = 1536;
constexpr int kIds = 4;               // ids of the history of a thread in flight
struct Smem {
  Shared sh;
  alignas(16) uint32_t special[kWords];
  alignas(16) uint32_t allow[kWords];
  uint32_t before[kGroups];           // special entries in the groups before
  uint32_t list[kCap];                // the round's special entries, in their order,
  uint32_t count[kCap];               // and their flags and occurrences
  uint32_t stage[kWarps][128];        // words of each warp on their way out
  alignas(128) uint2 nibble[16];      // ones in the 16-bit lanes of a nibble's bits (Raw16::mask)
  uint64_t full[kWarps][kDeep];
  alignas(128) unsigned char ring[kWarps][kDeep][kChunk];
};
static_assert(kCtas * (sizeof(Smem) + 1024) <= 228 * 1024, "kCtas CTAs on an SM");

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

// A row: `head` entries before the first boundary of 32 bytes, `vecs` whole vectors, then less than one.
template <class T>
struct Edges {
  int head, vecs;
  __device__ __forceinline__ Edges(const T* z, int64_t V) {
    constexpr int kPer = 32 / sizeof(T);
    head = (int)min(V, (int64_t)((0 - (int)(reinterpret_cast<uintptr_t>(z) / sizeof(T))) & (kPer - 1)));
    vecs = (int)(V - head) / kPer;
  }
};

// One warp reads a row's arguments, a lane each, and checks them.
template <int kType, int kOp>
__device__ __forceinline__ void read_row(const LogitsArgs& a, const Status& st, int64_t r, Row& out, int lane, bool first) {
  using T = typename Raw<kType>::T;
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
  const size_t osz = kOp == kAdjust32 ? 4 : sizeof(T);
  w.out = scores(kOp) ? nullptr : static_cast<char*>(a.out) + r * a.out_stride * osz;
  w.vec = scores(kOp) || ((reinterpret_cast<uintptr_t>(w.out) + Edges<T>(z, a.V).head * osz) & 31) == 0;
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
  w.live = writes(kOp) || !a.target || w.target >= 0;  // (the gradient has targets)
  w.g = f32(11, a.g, 0.f);
  w.e = f32(12, a.ge, 0.f);
  w.ent = f32(13, a.ge, 0.f);
  w.lse = f32(14, a.g, 0.f);
  w.logp = f32(15, a.g, 0.f);
  // (a row that nothing was left of has no gradient)
  if (kOp == kGrad && ((w.g == 0.f && w.e == 0.f) || w.lse == -INFINITY)) w.live = 0;
  if (lane == 0) out = w;
}

// Calls f(id - lo, place in the history) for the ids of the row's history from place `from` on that are in [lo + r0, lo + r1); returns
// whether this thread met one past the vocabulary.
template <class F>
__device__ __forceinline__ bool each_id(const LogitsArgs& a, const Row& w, int from, int lo, int r0, int r1, F f) {
  const int len = (int)(w.h1 - w.h0), V = (int)a.V;
  bool bad = false;
#pragma unroll 1
  for (int i = from + threadIdx.x; i < len; i += kIds * kThreads) {
    int id[kIds];
    // (one branch around the loads, which are then in flight together)
    if (a.hist8) {
      const int64_t* ids = static_cast<const int64_t*>(a.hist) + w.h0 + i;
#pragma unroll
      for (int k = 0; k < kIds; ++k) {
        const int64_t x = i + k * kThreads < len ? ids[k * kThreads] : -1;
        id[k] = x < 0 ? -1 : (int)min(x, a.V);
      }
    } else {
      const int32_t* ids = static_cast<const int32_t*>(a.hist) + w.h0 + i;
#pragma unroll
      for (int k = 0; k < kIds; ++k) id[k] = i + k * kThreads < len ? max(ids[k * kThreads], -1) : -1;
    }
#pragma unroll
    for (int k = 0; k < kIds; ++k) {
      const int rel = id[k] - lo;  // (-1 is no entry of the row: it is below r0)
      bad |= id[k] >= V;
      if ((uint32_t)(rel - r0) < (uint32_t)(r1 - r0)) f((uint32_t)rel, i + k * kThreads);
    }
  }
  return bad;
}

// A span of a row: bit j of the bitmaps is entry lo + j; [r0, r1) of them are the span's, r1 <= kSpan.
struct Span {
  int lo, r0, r1;
};

// Marks the special entries of a span in their bitmap, which was zeros, and writes that of the allowed ones where the row has a
// mask.
__device__ __forceinline__ void mark_span(const LogitsArgs& a, const Status& st, const Row& w, const Span& s, Smem& sm) {
  const int V = (int)a.V;
  auto mark = [&](uint32_t rel) { atomicOr(sm.special + (rel >> 5), 1u << (rel & 31u)); };
  if (w.special) {
    if (each_id(a, w, 0, s.lo, s.r0, s.r1, [&](uint32_t rel, int) { mark(rel); })) report(st, GPO_ERR_SHAPE, 46, (int)w.h0);
    for (int64_t i = w.b0 + threadIdx.x; i < w.b1; i += kThreads) {
      const int64_t x = load_id(a.bias_ids, a.bias8, i), rel = x - s.lo;
      if (x < 0 || x >= V || (i > w.b0 && load_id(a.bias_ids, a.bias8, i - 1) >= x)) report(st, GPO_ERR_SHAPE, 47, (int)i);
      else if (rel >= s.r0 && rel < s.r1) mark((uint32_t)rel);
    }
  }
  if (w.mask) {
    const int words = (V + 31) >> 5, sh = s.lo & 31, at0 = s.lo >> 5;
    for (int j = threadIdx.x; j < (s.r1 + 31) / 32; j += kThreads) {
      const int at = at0 + j;
      const uint32_t x0 = at >= 0 && at < words ? __ldg(w.mask + at) : 0u, x1 = at + 1 < words ? __ldg(w.mask + at + 1) : 0u;
      sm.allow[j] = __funnelshift_r(x0, x1, (uint32_t)sh);
    }
  }
}

// The special entries of group g, the first of which comes to place k.
__device__ __forceinline__ void list_group(const uint4& x, int g, int k, Smem& sm) {
  auto put = [&](uint32_t bits, int rel) {
    for (; bits; bits &= bits - 1, ++k)
      if (k >= 0 && k < kCap) sm.list[k] = rel + __ffs(bits) - 1;
  };
  put(x.x, 128 * g);
  put(x.y, 128 * g + 32);
  put(x.z, 128 * g + 64);
  put(x.w, 128 * g + 96);
}

// The special entries of the span that are allowed, which alone stay special and leave the allowed ones; returns their number, with
// the first kCap of them in the list.  Behind a barrier of the caller's; another comes before the list is read.
__device__ __forceinline__ int rank_span(int n, bool masked, uint32_t flags, Smem& sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, groups = (n + 127) / 128;
  const int own = (groups + 32 * kWarps - 1) / (32 * kWarps) * 32, end = min(groups, (warp + 1) * own);  // of a warp, side by side
  uint4* special = reinterpret_cast<uint4*>(sm.special);
  int sum = 0;
#pragma unroll 1
  for (int g0 = warp * own; g0 < end; g0 += 32) {
    const int g = g0 + lane;
    uint4& al = reinterpret_cast<uint4*>(sm.allow)[g];
    uint4 x = special[g];
    if (masked) special[g] = x = make_uint4(x.x & al.x, x.y & al.y, x.z & al.z, x.w & al.w);
    al = masked ? make_uint4(al.x & ~x.x, al.y & ~x.y, al.z & ~x.z, al.w & ~x.w) : make_uint4(~x.x, ~x.y, ~x.z, ~x.w);
    const int mine = __popc(x.x) + __popc(x.y) + __popc(x.z) + __popc(x.w);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    sm.before[g] = sum + upto - mine;
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
#pragma unroll 1
  for (int g = warp * own + lane; g < end; g += 32) {
    const int k = sm.before[g] += before;
    list_group(special[g], g, k, sm);
  }
  for (int c = threadIdx.x; c < min(kCap, all); c += kThreads) sm.count[c] = flags;
  return all;
}

// The list of a later round, of ranks [first, first + kCap).  Between barriers of the caller's.
__device__ __forceinline__ void list_span(int n, int first, int total, uint32_t flags, Smem& sm) {
  for (int g = threadIdx.x; g < (n + 127) / 128; g += kThreads)
    list_group(reinterpret_cast<const uint4*>(sm.special)[g], g, (int)sm.before[g] - first, sm);
  for (int c = threadIdx.x; c < min(kCap, total - first); c += kThreads) sm.count[c] = flags;
}

// The flags and counts of the entries in the list, whose first is of rank `first`.  Between barriers of the caller's.
__device__ __forceinline__ void count_span(const LogitsArgs& a, const Row& w, const Span& s, int first, Smem& sm) {
  // the place of a special entry in the list, of others far above its end
  auto at = [&](uint32_t rel) {
    const uint32_t word = rel >> 5 & 3u, bit = 1u << (rel & 31u);
    const uint4 x = reinterpret_cast<const uint4*>(sm.special)[rel >> 7];
    const uint32_t own = word == 0 ? x.x : word == 1 ? x.y : word == 2 ? x.z : x.w;
    const int k = (int)sm.before[rel >> 7] - first + __popc(own & (bit - 1u)) + (word > 0 ? __popc(x.x) : 0) + (word > 1 ? __popc(x.y) : 0) +
                  (word > 2 ? __popc(x.z) : 0);
    return own & bit ? (uint32_t)k : 0xFFFFFFFFu;
  };
  // (without biases every one of them is of the history: flags says so already, and only what was generated is looked at)
  const int generated = (int)(w.hg - w.h0);
  if (w.b1 > w.b0 || w.pres != 0.f || w.freq != 0.f)
    each_id(a, w, w.b1 > w.b0 ? 0 : generated, s.lo, s.r0, s.r1, [&](uint32_t rel, int i) {
      const uint32_t to = at(rel);
      if (to >= (uint32_t)kCap) return;
      if (i >= generated) atomicAdd(sm.count + to, 1u);
      else atomicOr(sm.count + to, kSeen);
    });
  for (int64_t i = w.b0 + threadIdx.x; i < w.b1; i += kThreads) {
    const int64_t rel = load_id(a.bias_ids, a.bias8, i) - s.lo;
    if (rel < s.r0 || rel >= s.r1) continue;
    const uint32_t to = at((uint32_t)rel);
    if (to < (uint32_t)kCap) atomicOr(sm.count + to, kBiased);
  }
}

// A warp's ring by 32-bit addresses in shared memory (through generic pointers every chunk takes 30 instructions more).
__device__ __forceinline__ Vec load_shared(uint32_t at) {
  Vec r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "r"(at) : "memory");
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4 + 16];" : "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ bool has_arrived(uint32_t bar, uint32_t phase) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(phase)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void store_global(void* p, const Vec& x) {
  asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x.w[0]), "r"(x.w[1]), "r"(x.w[2]),
               "r"(x.w[3]), "r"(x.w[4]), "r"(x.w[5]), "r"(x.w[6]), "r"(x.w[7])
               : "memory");
}
// Bytes (a multiple of 16, as are the addresses) to this CTA's shared memory, counted on a barrier that expects them.
__device__ __forceinline__ void bulk_load(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "mbarrier.arrive.expect_tx.shared::cta.b64 _, [%3], %2;\n\t"
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to),
      "l"(from), "r"(bytes), "r"(bar)
      : "memory");
}

// Four words of every lane to a row of any alignment, by a whole warp: entries of 4 or 2 bytes, lane 0's first v0, the next lane's
// `stride` after it, none from `end` on.  Through shared memory, so that an access takes 32 words side by side.  (A call of its own:
// few rows need it, and its registers are the others' spills.)
__device__ __noinline__ void store_ragged(void* out, bool four, uint4 x, int v0, int stride, int end, uint32_t* stage) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  reinterpret_cast<uint4*>(stage)[lane] = x;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = i * 32 + lane, v = v0 + at / 4 * stride + (four ? at % 4 : 2 * (at % 4));
    const uint32_t y = stage[at];
    if (four) {
      if (v < end) static_cast<uint32_t*>(out)[v] = y;
    } else {
      if (v < end) static_cast<uint16_t*>(out)[v] = (uint16_t)y;
      if (v + 1 < end) static_cast<uint16_t*>(out)[v + 1] = (uint16_t)(y >> 16);
    }
  }
  __syncwarp();
}

// A vector of every lane to the row, by a whole warp: lane 0's first entry is v0, none from `end` on, which lies between two lanes'.
// y: the same in fp32, for rows of those.
template <int kType, bool kWide>
__device__ __forceinline__ void store_vec(const Row& w, const float (&y)[Raw<kType>::kPer], const Vec& x, int v0, int end, uint32_t* stage, int lane) {
  using T = typename Raw<kType>::T;
  constexpr int kPer = Raw<kType>::kPer;
  const int v = v0 + lane * kPer;
  if (kWide) {
#pragma unroll
    for (int i = 0; i < kPer; i += 8) {
      Vec o;
#pragma unroll
      for (int k = 0; k < 8; ++k) o.w[k] = __float_as_uint(y[i + k]);
      if (!w.vec) {
        store_ragged(w.out, true, make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]), v0 + i, kPer, end, stage);
        store_ragged(w.out, true, make_uint4(o.w[4], o.w[5], o.w[6], o.w[7]), v0 + i + 4, kPer, end, stage);
      } else if (v < end) {
        store_global(static_cast<float*>(w.out) + v + i, o);
      }
    }
  } else if (!w.vec) {
    store_ragged(w.out, sizeof(T) == 4, make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]), v0, kPer, end, stage);
    store_ragged(w.out, sizeof(T) == 4, make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]), v0 + kPer / 2, kPer, end, stage);
  } else if (v < end) {
    store_global(static_cast<T*>(w.out) + v, x);
  }
}

// The statistics of a row from its joined parts; zy: the target's logit in units of log 2, which is in no part; held: how many
// entries equal to the maximum are not (0 with a target).
__device__ __forceinline__ void finish_row(const LogitsArgs& a, int64_t r, bool has, float zy, const Part& p, float held) {
  const bool at = has && !(zy <= kLow);  // (a NaN is one)
  const float top = at ? fmaxf(p.m, zy) : p.m;
  const float c = p.m - top, ec = exp2f(c);
  const float y = at ? zy - top : -INFINITY, ey = at ? exp2f(y) : 0.f;
  const float others = ec * p.s, total = others + (ey + held);
  const bool none = total == 0.f;
  const float lt = y == 0.f || held != 0.f ? log1pf(others) : logf(total);
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

// Two numbers in one register pair, which the packed instructions take.
__device__ __forceinline__ float lo_f2(uint64_t a) { return __uint_as_float((uint32_t)a); }
__device__ __forceinline__ float hi_f2(uint64_t a) { return __uint_as_float((uint32_t)(a >> 32)); }
__device__ __forceinline__ uint64_t make_f2(float a, float b) { return pack_f2(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ uint64_t ex2_f2(uint64_t a) { return make_f2(ex2(lo_f2(a)), ex2(hi_f2(a))); }
__device__ __forceinline__ uint64_t max_f2(uint64_t a, float b) { return make_f2(fmaxf(lo_f2(a), b), fmaxf(hi_f2(a), b)); }
template <int kN>
__device__ __forceinline__ void pairs_of(const float (&x)[kN], uint64_t (&y)[kN / 2]) {
#pragma unroll
  for (int j = 0; j < kN / 2; ++j) y[j] = make_f2(x[2 * j], x[2 * j + 1]);
}
template <int kN>
__device__ __forceinline__ void of_pairs(const uint64_t (&y)[kN / 2], float (&x)[kN]) {
#pragma unroll
  for (int j = 0; j < kN / 2; ++j) x[2 * j] = lo_f2(y[j]), x[2 * j + 1] = hi_f2(y[j]);
}

// Sums of exponentials so far, in two chains, relative to m; held: how many (0 or 1) of the entries that are m are not in them.
struct Running {
  float m;
  uint64_t s, u;
  float held;
};
template <bool kB>
struct Bool {
  static constexpr bool value = kB;
};

// Takes `top` as the maximum if it is larger; returns whether that entry then stays out of the sums.
// The entropy of a row that is nearly certain of one token is a sum of small terms, of which a sum that holds the largest, 1,
// keeps 6e-8 (an entropy of 1e-6 was off by 10 %).  A target's logit is out of the sums; in a row without one (apart) an entry more
// than kApart above all before it stays out until a larger one comes: where others are nearer than that, the entropy is above 0.2.
// (256 x 131072 adjusted 52 us for 50; 53 with every new maximum out.)
constexpr float kApart = 4.f;
template <bool kEnt, bool kHolds>
__device__ __forceinline__ bool raise(Running& p, float top, bool apart) {
  if (!(top > p.m)) return false;
  const float c = p.m - top;
  const uint64_t e = f2splat(ex2(c));
  if (kHolds) p.s = f2add(p.s, make_f2(p.held, 0.f));
  if (kEnt) p.u = f2mul(e, f2fma(f2splat(c), p.s, p.u));
  p.s = f2mul(e, p.s);
  p.m = top;
  if (kHolds) p.held = apart && c < -kApart ? 1.f : 0.f;
  return kHolds && p.held != 0.f;
}
// Two parts of a row as one, of which the one with the larger maximum keeps what it holds out.
template <bool kEnt, bool kHolds>
__device__ __forceinline__ Part join_held(Part x, float& held, Part y, float held_y) {
  if (kHolds) {
    if (x.m >= y.m) y.s += held_y;
    else x.s += held, held = held_y;
  }
  return join<kEnt>(x, y);
}

// All CTAs of the cluster have started once the wait, behind everyone's arrival, is over: only then is there shared memory of theirs.
__device__ __forceinline__ void cluster_started() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <int kType, int kOp, bool kEnt>
__global__ void __launch_bounds__(kThreads, kCtas) logits_kernel(LogitsArgs a, int cluster, Status st) {
  using E = Raw<kType>;
  using T = typename E::T;
  constexpr int kPer = E::kPer, kSpanVecs = (kSpan - 3 * kLead) / kPer / kChunkVecs * kChunkVecs;
  constexpr uint32_t kAll = (1u << kPer) - 1u;
  constexpr bool wide = kOp == kAdjust32, kHolds = holds_out(kOp, kEnt);
  extern __shared__ __align__(128) unsigned char smem[];
  Smem& sm = *reinterpret_cast<Smem*>(smem);
  Shared& sh = sm.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = (int)a.V;
  uint32_t* stage = sm.stage[warp];
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  const bool joins = kOp != kGrad && cluster > 1;
  if (joins) cluster_started();
  const int64_t r = blockIdx.x / cluster;
  const T* z0 = static_cast<const T*>(a.z) + r * a.z_stride;
  const Edges<T> row(z0, V);
  // this CTA's share of the row's accesses, in chunks; the warps take them in turn
  const int chunks = (row.vecs + kChunkVecs - 1) / kChunkVecs, share = (chunks + cluster - 1) / cluster;
  const int c0 = min(chunks, rank * share), c1 = min(chunks, c0 + share);
  const uint32_t full = smem_u32(sm.full[warp]), ring = smem_u32(sm.ring[warp]);
  // the chunks of this warp: the next to fetch, the vectors from it to the end of the share; how many are fetched, and done
  const char* ahead = reinterpret_cast<const char*>(z0 + row.head) + (int64_t)(c0 + warp) * kChunk;
  int left = min(row.vecs, c1 * kChunkVecs) - (c0 + warp) * kChunkVecs;
  uint32_t fetched = 0, taken = 0;
  auto fetch = [&]() {
    if (left <= 0) return;
    const uint32_t slot = fetched % kDeep;
    if (lane == 0) bulk_load(ring + slot * kChunk, ahead, 32u * (uint32_t)min(kChunkVecs, left), full + slot * 8);
    ++fetched;
    ahead += kWarps * kChunk;
    left -= kWarps * kChunkVecs;
  };
  // The row's first bytes are on their way before anything else is known of it but that it is read
  // (bounded waits for them are below, for every chunk that is fetched).
  const int64_t wanted = a.target && !writes(kOp) ? load_id(a.target, a.target8, r) : 0;
  if (lane == 0) {
    for (int k = 0; k < kDeep; ++k) mbar_init(sm.full[warp] + k, 1);
    fence_mbar_init();
  }
  __syncwarp();
  const bool early = wanted >= 0 && wanted < V;
  if (early)
    for (int k = 0; k < kDeep; ++k) fetch();
  if (warp == 0) read_row<kType, kOp>(a, st, r, sh.row, lane, rank == 0);
  if (a.spans || a.bias)
    for (int g = tid; g < kGroups; g += kThreads) reinterpret_cast<uint4*>(sm.special)[g] = make_uint4(0u, 0u, 0u, 0u);
  if (blockIdx.x == 0 && tid == 32) next_tag(st);
  if (tid >= 64 && tid < 80) {
    auto lanes = [&](int bit) { return (tid >> bit & 1 ? 0xFFFFu : 0u) | (tid >> (bit + 1) & 1 ? 0xFFFF0000u : 0u); };
    sm.nibble[tid - 64] = make_uint2(lanes(0), lanes(2));
  }
  __syncthreads();
  uint32_t nibble = smem_u32(sm.nibble);
  asm volatile("" : "+r"(nibble));  // (so that no load from the table comes before the barrier)
  const Row& w = sh.row;
  bool ok = true;  // (of the whole warp)
  auto arrived = [&]() {
    const uint32_t slot = taken % kDeep, phase = taken / kDeep & 1u;
    if (__all_sync(0xffffffffu, has_arrived(full + slot * 8, phase))) return true;
    ok = __all_sync(0xffffffffu, mbar_wait(sm.full[warp] + slot, phase, st, 48));
    return ok;
  };
  // every copy that was asked for lands before the shared memory goes
  auto drain = [&]() {
    for (; taken < fetched; ++taken) mbar_wait(sm.full[warp] + taken % kDeep, taken / kDeep & 1u, st, 48, 200000000ull, false);
  };
  if (!w.live) {
    drain();
    if (joins) cluster_wait();
    if (kOp == kGrad) {  // zeros
      const float none[kPer] = {};
      const Vec zero = E::narrow(none);
      const int from = row.head + min(row.vecs, c0 * kChunkVecs) * kPer, whole = row.head + min(row.vecs, c1 * kChunkVecs) * kPer;
      const int first = rank == 0 ? 0 : from, end = rank == cluster - 1 ? V : whole;
      T* out = static_cast<T*>(w.out);
      for (int v = first + tid; v < from; v += kThreads) out[v] = E::put(0.f);
#pragma unroll 1
      for (int v = from + warp * 32 * kPer; v < whole; v += kThreads * kPer) store_vec<kType, false>(w, none, zero, v, whole, stage, lane);
      for (int v = whole + tid; v < end; v += kThreads) out[v] = E::put(0.f);
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
  if (!early)
    for (int k = 0; k < kDeep; ++k) fetch();
  bool holds = false;  // the target
  const uint32_t flags = w.b1 > w.b0 ? 0u : kSeen;  // of every special entry
  Running p = {kLow, 0ull, 0ull, 0.f};
  const bool apart = kHolds && w.target < 0;
#pragma unroll 1
  for (int s0 = min(row.vecs, c0 * kChunkVecs);; s0 += kSpanVecs) {
    const int end = min(row.vecs, c1 * kChunkVecs), s1 = min(end, s0 + kSpanVecs);
    const bool head = rank == 0 && s0 == 0, last = s1 == end, tail = last && rank == cluster - 1;
    // bit kLead of the bitmaps is the span's first whole vector's, what is before or behind those its ends
    Span span;
    span.lo = row.head + s0 * kPer - kLead;
    span.r0 = head ? kLead - row.head : kLead;
    span.r1 = tail ? V - span.lo : (s1 - s0) * kPer + kLead;
    const int trel = w.target >= (int64_t)span.lo + span.r0 && w.target < (int64_t)span.lo + span.r1 ? (int)w.target - span.lo : -1;
    holds |= trel >= 0;
    int total = 0;
    if (marked) {
      mark_span(a, st, w, span, sm);
      __syncthreads();
      if (w.special) {
        total = rank_span(span.r1, w.mask != nullptr, flags, sm);
        __syncthreads();
        if (total) count_span(a, w, span, 0, sm);  // (complete after the dense pass's barrier)
      }
    }
    // d y_j = -gs p_j - es p_j (log p_j + H), without the target's gs
    auto gradient = [&](float (&y)[kPer]) {
      uint64_t y2[kPer / 2];
      pairs_of(y, y2);
      const uint64_t s2 = f2splat(scale), n2 = f2splat(-w_lse), k2 = f2splat(kLog2e), g2 = f2splat(-gs), e2 = f2splat(-es), h2 = f2splat(w_ent);
#pragma unroll
      for (int j = 0; j < kPer / 2; ++j) {
        uint64_t d = f2fma(y2[j], s2, n2);
        if (kEnt) d = max_f2(d, -200.f);
        const uint64_t x = ex2_f2(f2mul(d, k2));
        y2[j] = f2mul(x, kEnt ? f2fma(e2, f2add(d, h2), g2) : g2);
      }
      of_pairs(y2, y);
    };
    // the entries that are left in x enter the sums
    auto sums = [&](Vec& x) {
      const float top = E::top(x);
      if (raise<kEnt, kHolds>(p, top * sl2, apart)) p.s = f2add(p.s, make_f2((float)(E::take_out(x, top) - 1), 0.f));
      float y[kPer];
      uint64_t y2[kPer / 2];
      E::widen(x, y);
      pairs_of(y, y2);
      const uint64_t s2 = f2splat(sl2), n2 = f2splat(-p.m);
#pragma unroll
      for (int j = 0; j < kPer / 2; ++j) {
        const uint64_t d = f2fma(y2[j], s2, n2), e = ex2_f2(d);
        p.s = f2add(p.s, e);
        // (0 times -inf is 0 here)
        if (kEnt) p.u = f2fma(e, E::kFloors ? d : max_f2(d, -200.f), p.u);
      }
    };
    // What an allowed entry becomes (rel: its place in the span, z: its raw logit); it enters the sums.
    auto single = [&](int rel, uint32_t slot, float z) {
      float slope;
      const float y = adjusted(a, w, slot, z, span.lo + rel, slope);
      if (kOp == kGrad) {
        float d;
        if (rel == trel) {  // (p from its log-probability, which has the digits of 1 - p)
          const float pe = expf(w.logp);
          d = -gs * expm1f(w.logp) - (kEnt && pe > 0.f ? es * pe * (w.logp + w.ent) : 0.f);
        } else {
          const float x = fmaxf(fmaf(y, scale, -w.lse), -200.f), pe = ex2(x * kLog2e);
          d = w.lse == w.lse ? -gs * pe - (kEnt ? es * pe * (x + w.ent) : 0.f) : w.lse;
        }
        return d * slope;
      }
      if (rel == trel) {
        sh.at = y;
      } else if (!raise<kEnt, kHolds>(p, y * sl2, apart)) {
        const float d = fmaf(y, sl2, -p.m), x = ex2(d);
        p.s = f2add(p.s, make_f2(x, 0.f));
        if (kEnt) p.u = f2fma(make_f2(x, 0.f), make_f2(fmaxf(d, -200.f), 0.f), p.u);
      }
      return y * scale;
    };
    auto put = [&](int rel, float x) {
      if (!GPO_BOUNDS(st, span.lo + rel, V, kWhereLogits)) return;
      if (wide) static_cast<float*>(w.out)[span.lo + rel] = x;
      else static_cast<T*>(w.out)[span.lo + rel] = E::put(x);
    };
    // the bits of the span's k-th vector
    auto bits_at = [&](const uint32_t* p, int k) -> uint32_t {
      return kPer == 16 ? reinterpret_cast<const uint16_t*>(p)[k + kLead / 16] : reinterpret_cast<const uint8_t*>(p)[k + kLead / 8];
    };
    const int stop = s1 - s0, tvec = trel < kLead ? -1 : (trel - kLead) / kPer;  // the span's vectors, the target's
    // Each lane's vector, the span's k-th.  kMarked: some entries may be masked or special, or none of the span; kKeep: special
    // ones are written as they were, to be read once more.
    auto dense = [&](Vec& x, int k, auto is_marked, auto keeps) {
      constexpr bool kMarked = decltype(is_marked)::value, kKeep = decltype(keeps)::value;
      uint32_t take = kAll, sp = 0u;
      if (kMarked) {
        if (marked) take = bits_at(sm.allow, k);
        if (kKeep && total) sp = bits_at(sm.special, k);
        if (k == tvec) {  // (a special one, too)
          const uint32_t bit = 1u << (trel - kLead) % kPer;
          take &= ~bit;
          sp |= bit;
        }
        if (k >= stop) take = 0u;
      }
      const int first = span.lo + kLead + (k - lane) * kPer, from = span.lo + kLead + stop * kPer;
      float y[kPer];
      if (kOp == kGrad) {
        E::widen(x, y);
        gradient(y);
        Vec o = E::narrow(y);
        if (kMarked) o = E::keep(o, take, 0u, nibble);
        if (kMarked && kKeep) o = E::choose(o, x, sp, nibble);
        store_vec<kType, false>(w, y, o, first, from, stage, lane);
      } else {
        if (writes(kOp)) {
          Vec q = x;
          if (kMarked) q = E::keep(q, take, nibble);
          E::widen(q, y);
#pragma unroll
          for (int j = 0; j < kPer; ++j) y[j] *= scale;
          if (!wide) q = E::narrow(y);
          if (!wide && kMarked && kKeep) q = E::choose(q, x, sp, nibble);
          store_vec<kType, wide>(w, y, q, first, from, stage, lane);
        }
        if (kMarked) x = E::keep(x, take, nibble);
        if (kEnt) x = E::floor(x);
        sums(x);
      }
    };
    auto pass = [&](auto keeps) {
      // the chunks of the span, of which those that end by `whole` have nothing special in them, but for the target's
      const int whole = marked ? 0 : stop - kChunkVecs + 1, taught = tvec < 0 ? -1 : tvec / kChunkVecs * kChunkVecs;
      int at = (c0 + (int)taken * kWarps + warp) * kChunkVecs - s0;  // (the span's at-th vector)
#pragma unroll 1
      for (; at < stop && ok; at += kWarps * kChunkVecs, ++taken) {
        if (!arrived()) break;
        const uint32_t from = ring + taken % kDeep * kChunk + lane * 32;
#pragma unroll
        for (int u = 0; u < kChunkVecs; u += 32) {
          Vec x = load_shared(from + 32 * u);
          if (at < whole && at != taught) dense(x, at + u + lane, Bool<false>(), Bool<false>());
          else dense(x, at + u + lane, Bool<true>(), keeps);
        }
        __syncwarp();  // (all lanes have read the chunk)
        fetch();
      }
    };
    const bool keep = !scores(kOp) && !wide && w.out == w.z;
    if (scores(kOp) || wide) pass(Bool<false>());
    else if (keep) pass(Bool<true>());
    else pass(Bool<false>());
    // the entries that need more than the dense pass: special ones, the target, the row's ends
    const T* zs = z0 + span.lo;
    auto raw_at = [&](int rel) { return GPO_BOUNDS(st, span.lo + rel, V, kWhereLogits) ? E::get1(zs[rel]) : 0.f; };
    if (total || w.target >= 0 || marked) __syncthreads();
    for (int first = 0; first < total; first += kCap) {
      if (first > 0) {
        __syncthreads();
        list_span(span.r1, first, total, flags, sm);
        __syncthreads();
        count_span(a, w, span, first, sm);
        __syncthreads();
      }
      const int m = min(kCap, total - first);
#pragma unroll 1
      for (int k0 = tid; k0 < m; k0 += 4 * kThreads) {
        float z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = k0 + k * kThreads < m ? raw_at((int)sm.list[k0 + k * kThreads]) : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k0 + k * kThreads < m) {
            const int rel = (int)sm.list[k0 + k * kThreads];
            const float x = single(rel, sm.count[k0 + k * kThreads], z[k]);
            if (!scores(kOp)) put(rel, x);
          }
      }
    }
    // (ends: less than a vector before the first whole one and behind the last; then a target among no special entries)
    const int behind = stop * kPer + kLead;
    int rel = -1;
    if (tid < 16) rel = tid < kLead - span.r0 ? span.r0 + tid : -1;
    else if (tid < 32) rel = behind + tid - 16 < span.r1 ? behind + tid - 16 : -1;
    else if (tid == 32 && trel >= kLead && trel < behind) rel = trel;
    if (rel >= 0 && !(total && (sm.special[rel >> 5] >> (rel & 31) & 1u))) {
      // (rank_span has taken the special ones out of the allowed)
      if (!marked || (sm.allow[rel >> 5] >> (rel & 31) & 1u)) {
        const float x = single(rel, 0u, raw_at(rel));
        if (!scores(kOp)) put(rel, x);
      } else {
        if (!scores(kOp)) put(rel, kOp == kGrad ? 0.f : -INFINITY);
        if (kOp != kGrad && rel == trel) sh.at = -INFINITY;
      }
    }
    if (last) break;
    if (marked) {
      __syncthreads();
      if (total)
        for (int g = tid; g < kGroups; g += kThreads) reinterpret_cast<uint4*>(sm.special)[g] = make_uint4(0u, 0u, 0u, 0u);
      __syncthreads();
    }
  }
  if (!ok) drain();
  if (kOp == kGrad) return;
  Part x = {p.m, lo_f2(p.s) + hi_f2(p.s), lo_f2(p.u) + hi_f2(p.u)};
  float held = p.held;
  auto join_lanes = [&](int from) {
    for (int o = from; o > 0; o >>= 1) {
      const Part y = {__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.s, o),
                      __shfl_xor_sync(0xffffffffu, x.u, o)};
      x = join_held<kEnt, kHolds>(x, held, y, kHolds ? __shfl_xor_sync(0xffffffffu, held, o) : 0.f);
    }
  };
  join_lanes(16);
  if (lane == 0) {
    sh.part[warp] = x;
    if (kHolds) sh.held[warp] = held;
  }
  __syncthreads();
  if (joins) cluster_wait();
  if (warp == 0) {
    x = lane < kWarps ? sh.part[lane] : Part{kLow, 0.f, 0.f};
    held = kHolds && lane < kWarps ? sh.held[lane] : 0.f;
    join_lanes(kWarps / 2);
    if (lane == 0 && cluster > 1) {
      st_remote(remote(&sh.cluster[rank].m, 0), x.m);
      st_remote(remote(&sh.cluster[rank].s, 0), x.s);
      st_remote(remote(&sh.cluster[rank].u, 0), x.u);
      if (kHolds) st_remote(remote(&sh.cluster_held[rank], 0), held);
      // (who has the target's logit passes it on)
      if (holds) st_remote(remote(&sh.cluster_at, 0), sh.at);
    }
    __syncwarp();
  }
  if (cluster > 1) cluster_sync();
  if (rank != 0 || tid != 0) return;
  float at = sh.at;
  if (cluster > 1) {
    at = sh.cluster_at;
    x = sh.cluster[0];
    held = kHolds ? sh.cluster_held[0] : 0.f;
    for (int c = 1; c < cluster; ++c) x = join_held<kEnt, kHolds>(x, held, sh.cluster[c], kHolds ? sh.cluster_held[c] : 0.f);
  }
  finish_row(a, r, w.target >= 0, w.target >= 0 ? at * w.sl2 : 0.f, x, held);
}

template <int kType, int kOp, bool kEnt>
cudaError_t setup_one() {
  return cudaFuncSetAttribute(logits_kernel<kType, kOp, kEnt>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
}
template <int kType>
cudaError_t setup_type() {
  cudaError_t e = setup_one<kType, kAdjust, false>();
  if (e == cudaSuccess) e = setup_one<kType, kAdjust, true>();
  if (kType != GPO_DT_F32 && e == cudaSuccess) e = setup_one<kType, kType == GPO_DT_F32 ? kAdjust : kAdjust32, false>();
  if (kType != GPO_DT_F32 && e == cudaSuccess) e = setup_one<kType, kType == GPO_DT_F32 ? kAdjust : kAdjust32, true>();
  if (e == cudaSuccess) e = setup_one<kType, kScore, false>();
  if (e == cudaSuccess) e = setup_one<kType, kScore, true>();
  if (e == cudaSuccess) e = setup_one<kType, kScoreAll, true>();
  if (e == cudaSuccess) e = setup_one<kType, kGrad, false>();
  if (e == cudaSuccess) e = setup_one<kType, kGrad, true>();
  return e;
}

template <int kType, int kOp, bool kEnt>
cudaError_t launch_one(const LaunchCtx& lc, const LogitsArgs& a, const Status& st) {
  // a row of few gets a cluster, each of whose CTAs has a chunk for every warp or more
  const int64_t ctas = kCtas * (int64_t)lc.num_sms, batches = a.V / (kWarps * kChunkVecs * Raw<kType>::kPer);
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
  if (a.out && a.out32 && kType != GPO_DT_F32) {
    constexpr int kOp = kType == GPO_DT_F32 ? kAdjust : kAdjust32;
    return a.ent ? launch_one<kType, kOp, true>(lc, a, st) : launch_one<kType, kOp, false>(lc, a, st);
  }
  if (a.out) return a.ent ? launch_one<kType, kAdjust, true>(lc, a, st) : launch_one<kType, kAdjust, false>(lc, a, st);
  if (a.ent && !a.target) return launch_one<kType, kScoreAll, true>(lc, a, st);
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
