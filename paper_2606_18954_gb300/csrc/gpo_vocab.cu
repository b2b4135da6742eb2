// Per-token log-probabilities from hidden states and the vocabulary matrix, and their gradients,
// on the tcgen05 tensor cores (the formulas are in include/graphpo.h).
//
// Forward, two launches, and one more before them for large products (kVocabListed; up to 16 tokens:
// gpo_vocab_few.cu):
//   rows     vocab_rows_kernel lists the tokens with a target and copies their hidden rows together
//            (not where every token has one): the others then cost no product.  Bound by the reads: every CTA looks at
//            every target; 12 us for 4096 tokens, of which 2867 take part, 2048 wide
//   lse      vocab_pair_kernel<kLse>: logits tiles of 256 tokens x 256 vocabulary rows that stay in tensor
//            memory; the epilogue reduces each row's 128 columns to a maximum and a sum (and the entropy's
//            sum), the target's logit kept apart.  Bound by the tensor cores, in long runs by the power that they may
//            take: 2867 x 100003 x 2048 600 us, 1960 TFLOP/s; 8192 x 131072 x 2048 2.1 to 2.4 ms, 1830 to 2060
//   join     vocab_join_kernel, up to 256 tokens vocab_join_row_kernel: the parts of a row joined in a fixed order.
//            Bound by HBM and latency: 26 MB in 14 us
// Gradient, piece by piece of the vocabulary (dz of a piece takes at most 512 MiB):
//   order    vocab_order_kernel, from 4097 tokens on vocab_sort_kernel and vocab_gather_kernel: the tokens with a gradient
//            that is not 0, in the order of their targets, and their rows.  Bound by latency: 12 to 22 us up to 16384
//            tokens, 66 for 65536
//   dz       vocab_pair_kernel<kDz>: the logits again, dz in the epilogue, written in 16 bits.  Bound by the tensor
//            cores: 1434 x 65536 x 2048 230 us, 1670 TFLOP/s
//   products vocab_pair_kernel<kProducts>: d_hidden += dz W and d_weight = dz^T hidden in one launch;
//            with few tokens the k of d_hidden in parts (vocab_splits) that vocab_parts_kernel adds.  Bound by the
//            tensor cores and what feeds them: a step of 64 k takes 0.32 us, where its MMAs take 0.27; 1434 x 65536 x
//            2048 465 us, 1650 TFLOP/s.  (Six stages in place of five, boxes fetched into L2 ahead, a second loading
//            thread: none of them faster.)
// The tiles are as large as tensor memory allows with two accumulators of fp32, one for the MMAs and one for the epilogue:
// each operand byte is used 128 times from shared memory, which both CTAs of a pair fill half and half.
// Keeping the sum over the other tokens of the vocabulary apart from the target's term keeps the
// digits of a nearly certain token's log-probability -log(1 + sum), which is a small number.
#define GPO_REPORT __noinline__
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gpo_pair.cuh"
#include "gpo_sort.cuh"
#include "gpo_vocab_math.cuh"

namespace gpo {

namespace {

// Ent: with the entropy; Wide: dz of logits that are several accumulations (see kVocabDzSeg); Rows: products whose results
// have rows of any alignment (see store_rows)
enum Mode { kLse, kLseEnt, kDz, kDzEnt, kDzWide, kDzWideEnt, kProducts, kProductsRows };
__host__ __device__ constexpr bool is_products(int mode) { return mode == kProducts || mode == kProductsRows; }
__host__ __device__ constexpr bool is_lse(int mode) { return mode == kLse || mode == kLseEnt; }
__host__ __device__ constexpr bool is_wide(int mode) { return mode == kDzWide || mode == kDzWideEnt; }
__host__ __device__ constexpr bool has_ent(int mode) { return mode == kLseEnt || mode == kDzEnt || mode == kDzWideEnt; }
__host__ __device__ constexpr bool keeps_logits(int mode) { return is_lse(mode) || is_wide(mode); }  // 128 of them per epilogue thread

constexpr int kTile16 = 64;                        // elements of one 128-byte swizzle row
constexpr int kVStages = 6;                        // of the logits
constexpr int kPStages = 5;                        // of the products (with 4, 4000 x 30000 x 1000 take 6 % longer)
constexpr int kVThreads = 384;                     // warps: 0 loads, 1 MMAs, 2 rests, 3 idle, 4..11 epilogue
constexpr int kVEpiWarps = 8, kLoadWarp = 0, kMmaWarp = 1, kRestWarp = 2, kIdleWarp = 3;
// The epilogue of the logits keeps 128 of them per thread: its warps take registers that the other four
// give back.  The shares add up to no more than the launch brings (setup_mode checks that).
// The split of each mode is one without spills: the loads' and the MMAs' lane would find theirs in an L1
// that the epilogue's stores sweep, and fall behind the tensor cores.
constexpr int kRegsLaunch = 168;
__host__ __device__ constexpr int regs_few(int mode) { return is_wide(mode) ? 120 : 88; }
__host__ __device__ constexpr int regs_many(int mode) { return is_wide(mode) ? 192 : 208; }
static_assert(128 * regs_few(kDzWide) + 256 * regs_many(kDzWide) <= kVThreads * kRegsLaunch &&
              128 * regs_few(kLse) + 256 * regs_many(kLse) <= kVThreads * kRegsLaunch, "register split");
constexpr int kVBox = kTile16 * 128;               // one 64 x 64 box
constexpr int kVStage = 4 * kVBox;                 // A and B halves of one k-step, per CTA
constexpr int kVCols = 512;                        // two accumulators of 256 columns
// Logits: after kVocabSeg (dz: kVocabDzSeg) steps of 64 k the tensor cores' sum is taken over into registers.  Their
// fp32 additions drop the bits below the sum's last one, always towards zero, so that a sum of d products
// shrinks by about d / 130 ulps: 4e-6 of a logit at d = 4096, too much for the log-probability of
// a nearly certain token.  Shorter sums, added in registers with rounding, keep that down (the mean of what is left
// is given back by logit_scale on the host), but reading tensor memory holds up the MMAs: 8192 tokens, 131072 x 2048
// take 2175 us in one sum, 2230 by 512 products, 2435 by 384, 2645 by 256.
template <int kMode>
__device__ __forceinline__ constexpr int segment_of() {
  return is_lse(kMode) ? kVocabSeg : is_wide(kMode) ? kVocabDzSeg : 1 << 30;
}
constexpr int kNoKey = 0x7fffffff;                 // above every target: a token without a gradient
constexpr int kRaster = 32;                        // row tiles that share one pass over the columns

struct __align__(8) VocabCtl {
  uint64_t full[kVStages];
  uint64_t empty[kVStages];
  uint64_t tfull[2];
  uint64_t tempty[2];
  uint64_t rfull[2];   // products: the operands of write_rests
  uint64_t rempty[2];
  uint64_t drain;
  uint32_t tmem_base;
};

// Shared memory of the products beside their ring: two operands of write_rests, and per epilogue warp 32 rows of 128
// bytes on their way out.
constexpr int kRestBytes = 2 * kVBox;
constexpr int kWarpBytes = 4 * 1024;
constexpr size_t kVCtl = (sizeof(VocabCtl) + 15) & ~size_t(15);
constexpr size_t kVSmem = kVCtl + 1023 + (size_t)kVStages * kVStage;
constexpr size_t kPSmem = kVCtl + 1023 + (size_t)kPStages * kVStage + 2 * (size_t)kRestBytes + (size_t)kVEpiWarps * kWarpBytes;
__host__ __device__ constexpr size_t smem_of(int mode) { return is_products(mode) ? kPSmem : kVSmem; }

__device__ __forceinline__ uint32_t pack16(float a, float b, int f16) {
  if (f16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint16_t round16(float a, int f16) { return (uint16_t)(pack16(a, 0.f, f16) & 0xFFFFu); }
__device__ __forceinline__ float widen16(uint16_t x, int f16) {
  return f16 ? __half2float(__ushort_as_half(x)) : __uint_as_float((uint32_t)x << 16);
}

// One tile of a pair: the rows of A from m0, the columns (rows of B) from n0, steps [ka, ka + kb) of 64 of k.
struct Tile {
  int job;    // kProducts: 0 d_hidden, 1 d_weight
  int split;  // d_hidden: which part of k
  int m0, n0, ka, kb;
};

// The tiles of one launch and which pair takes which, in what order.
struct Plan {
  int p, np;           // this pair of np
  int mt, nt, kb;      // kLse, kDz: row tiles, column tiles, k-steps
  int dt;              // kProducts: column tiles of d
  int n_dh, kb_dh, splits, own_dh, n_dw, kb_dw;
  int light0, nlight, extra;  // pairs from light0 on take `extra` d_weight tiles more, for the d_hidden tile they lack
};

constexpr int kEpiSteps = 6;  // k-steps that a tile's epilogue in the products takes the time of
template <int kMode>
__device__ __forceinline__ Plan make_plan(const VocabArgs& a, int rows) {
  Plan q;
  q.p = (int)blockIdx.x >> 1;
  q.np = (int)gridDim.x >> 1;
  q.mt = (rows + kPairM - 1) / kPairM;
  const int64_t cols = is_lse(kMode) ? a.V : a.vn;
  q.nt = (int)((cols + kPairN - 1) / kPairN);
  q.kb = (a.D + kTile16 - 1) / kTile16;
  q.dt = (a.D + kPairN - 1) / kPairN;
  // the longer d_hidden tiles first, round robin; the pairs that get one less take as much work in
  // d_weight tiles, the rest of which go round robin too.  (A d_weight tile takes an eighth more than its steps,
  // for those of write_rests and its ends: 700 tokens of 65536 x 1024 137 us instead of 144; a fourth is too much for
  // 4000 of 30000 x 1000, 226 instead of 213.  kEpiSteps 8 instead of 6: 60 of 30000 x 1024 44.5 us instead of 39.)
  q.splits = a.splits;
  q.n_dh = a.dh ? q.mt * q.dt * q.splits : 0;
  q.n_dw = a.dw ? q.nt * q.dt : 0;
  q.kb_dh = (int)((a.vn + kTile16 - 1) / kTile16);
  q.kb_dw = (rows + kTile16 - 1) / kTile16;
  q.own_dh = q.n_dh / q.np + (q.p < q.n_dh % q.np ? 1 : 0);
  q.light0 = q.n_dh % q.np;
  q.nlight = q.np - q.light0;
  q.extra = q.light0 > 0 ? min(max(q.kb_dh / q.splits, kEpiSteps) / max(q.kb_dw + q.kb_dw / 8, kEpiSteps), q.n_dw / q.nlight) : 0;
  return q;
}

// The pair's s-th tile; false after the last.
template <int kMode>
__device__ __forceinline__ bool next_tile(const Plan& q, int s, Tile& t) {
  if (!is_products(kMode)) {
    const int64_t i = q.p + (int64_t)s * q.np;
    if (i >= (int64_t)q.mt * q.nt) return false;
    // kRaster row tiles take the columns together: what the pairs work on at one time is few columns of
    // all those rows, whose hidden states stay in L2 while the vocabulary matrix streams through once
    const int64_t per = (int64_t)kRaster * q.nt;
    const int g = (int)(i / per);
    const int r = (int)(i - g * per);
    const int gm = min(kRaster, q.mt - g * kRaster);
    t.job = t.split = t.ka = 0;
    t.m0 = (g * kRaster + r % gm) * kPairM;
    t.n0 = r / gm * kPairN;
    t.kb = q.kb;
    return true;
  }
  if (s < q.own_dh) {
    const int i = q.p + s * q.np, mn = q.mt * q.dt, o = i % mn;
    t.job = 0;
    t.split = i / mn;
    t.m0 = o / q.dt * kPairM;
    t.n0 = o % q.dt * kPairN;
    t.ka = (int)((int64_t)q.kb_dh * t.split / q.splits);
    t.kb = (int)((int64_t)q.kb_dh * (t.split + 1) / q.splits) - t.ka;
    return true;
  }
  s -= q.own_dh;
  int j;
  if (q.p >= q.light0 && s < q.extra) {
    j = q.p - q.light0 + s * q.nlight;
  } else {
    if (q.p >= q.light0) s -= q.extra;
    j = q.extra * q.nlight + q.p + s * q.np;
  }
  if (j >= q.n_dw) return false;
  t.job = 1;
  t.split = t.ka = 0;
  t.m0 = j / q.dt * kPairM;
  t.n0 = j % q.dt * kPairN;
  t.kb = q.kb_dw;
  return true;
}

// 32 bytes, 32-byte aligned: one whole sector.
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&x)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]),
               "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
               : "memory");
}

// Rows of whole, aligned 16 bytes.
__host__ __device__ __forceinline__ bool vec_rows(const void* p, int64_t stride) { return ((stride & 7) | (reinterpret_cast<uintptr_t>(p) & 15)) == 0; }

// 16 bits of 32 consecutive columns of a row to memory (add: added to what it holds), 16-byte aligned, those below `cols`.
__device__ __forceinline__ void store16(uint16_t* dst, const float (&x)[32], int cols, int f16, bool add) {
#pragma unroll
  for (int c = 0; c < 32; c += 8) {
    uint32_t o[4] = {0u, 0u, 0u, 0u};
    const bool whole = c + 8 <= cols;
    if (add && whole) {
      const uint4 u = *reinterpret_cast<const uint4*>(dst + c);
      o[0] = u.x, o[1] = u.y, o[2] = u.z, o[3] = u.w;
    } else if (add) {
      for (int i = 0; i < 8 && c + i < cols; ++i) o[i >> 1] |= (uint32_t)dst[c + i] << (16 * (i & 1));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = add ? widen16((uint16_t)(o[i] & 0xFFFFu), f16) : 0.f, hi = add ? widen16((uint16_t)(o[i] >> 16), f16) : 0.f;
      o[i] = pack16(x[c + 2 * i] + lo, x[c + 2 * i + 1] + hi, f16);
    }
    if (whole) {
      *reinterpret_cast<uint4*>(dst + c) = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) dst[c + i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
    }
  }
}

// The same of a warp's 32 rows, a lane each (its row in memory: row, or none below 0), for rows of any alignment:
// through `own`, 4 KB of shared memory, so that the warp takes row by row.  (2048 tokens of 30000 x 1001: the products
// in 205 us; 480 with a lane for each row and its stores of 2 bytes.)
__device__ __forceinline__ void store_rows(float* own, const float (&x)[32], uint16_t* dst, int64_t stride, int64_t row, int cols,
                                           int f16, bool add, int lane) {
#pragma unroll
  for (int c = 0; c < 32; ++c) own[lane * 32 + (c ^ lane)] = x[c];
  __syncwarp();
  const bool in = lane < cols;
#pragma unroll 8
  for (int r = 0; r < 32; ++r) {
    const int64_t to = __shfl_sync(0xffffffffu, row, r);
    if (to >= 0 && in) {
      uint16_t* at = dst + to * stride + lane;
      const float y = own[r * 32 + (lane ^ r)];
      *at = round16(add ? y + widen16(*at, f16) : y, f16);
    }
  }
  __syncwarp();
}

// Brings `cols` 16-bit columns of a row into L1, for add_row.
__device__ __forceinline__ void prefetch_row(const uint16_t* x, int cols) {
  for (int c = 0; c < cols; c += 64) asm volatile("prefetch.global.L1 [%0];" ::"l"(x + c));
}
// y[j] += w x[j] for 32 columns of a row of hidden or weight, those below `cols` rounded up to 8 (the
// row has them; what lies past its width is not used).
__device__ __forceinline__ void add_row(const uint16_t* x, float w, int cols, int f16, float (&y)[32]) {
#pragma unroll
  for (int c = 0; c < 32; c += 8) {
    if (c < cols) {
      const uint4 u = *reinterpret_cast<const uint4*>(x + c);
      const uint32_t h[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[c + 2 * i] = fmaf(w, widen16((uint16_t)(h[i] & 0xFFFFu), f16), y[c + 2 * i]);
        y[c + 2 * i + 1] = fmaf(w, widen16((uint16_t)(h[i] >> 16), f16), y[c + 2 * i + 1]);
      }
    }
  }
}

// What the roles of a CTA share.
struct Cta {
  VocabCtl* ctl;
  unsigned char* smem;  // the dynamic shared memory
  uint32_t tiles;       // the ring, the same offset in both CTAs
  uint32_t tmem, rank;
  int rows;             // tokens that are multiplied
};
// Where a role is in the ring and among the accumulations; it goes on from one pass over tiles to the next.
struct Pipe {
  int stage = 0;
  uint32_t phase = 0;
  uint32_t issued = 0;  // loads: stages filled
  int sum = 0;          // accumulations: one per tile, or per segment of a logits tile

  template <int kS>
  __device__ __forceinline__ void next() {
    if (++stage == kS) {
      stage = 0;
      phase ^= 1u;
    }
  }
};

// The tokens whose targets are rows of a d_weight tile: [ra, rb) of the list.
__device__ __forceinline__ void tokens_of(const VocabArgs& a, const Tile& t, int& ra, int& rb) {
  const int* first = a.tile_first + ((int)a.v0 + t.m0) / kPairM;
  ra = __ldcg(first);
  rb = __ldcg(first + 1);
}

// Of a token's dz the target's entry is the largest part, unless the policy is sure of another token.  Its rounding to 16
// bits would add 40 % to the error that the gradients' own rounding leaves, so what that rounding takes away
// (a.rest) is added to both products.  The other entries' rounding stays: it adds 1 % to the whole error (1.0016 and 1.0004
// of one rounding, 2048 tokens of 65536 x 2048), but 41 % in rows of d_weight that are no token's target, and up to 26 %
// to both gradients where every token is sure of another.  A second product of those rests would double the products' time.
// The rest goes to d_hidden in the epilogue, a row of the vocabulary matrix per
// token (add_row); to d_weight as steps of its own after those of dz: the tokens whose targets are rows of the tile are
// one run of the list, which is in the order of the targets, and 64 of them at a time are a step whose A is zeros but
// for each token's rest in its target's row.  The rests are rounded to 16 bits there, 2^-17 (bf16) of the
// entry of dz.  All tiles together take T / 64 such steps and one more each, however often a token occurs.
// Here one warp of either CTA writes these A, two steps ahead of the MMAs, as a load of dz would leave them: 128 bytes
// per k for 64 rows of the tile, swizzled.  A lane takes two k, and clears what it wrote two steps before.
__device__ __forceinline__ bool write_rests(const VocabArgs& a, const Status& st, const Cta& c, int ring, int lane) {
  const Plan plan = make_plan<kProducts>(a, c.rows);
  unsigned char* buf = c.smem + (c.tiles - smem_u32(c.smem)) + ring;
  for (int j = lane; j < 2 * kRestBytes / 16; j += 32) *reinterpret_cast<uint4*>(buf + 16 * j) = make_uint4(0u, 0u, 0u, 0u);
  __syncwarp();
  int was[2][2] = {{-1, -1}, {-1, -1}};
  uint32_t n = 0;
  Tile t;
  for (int s = plan.own_dh; next_tile<kProducts>(plan, s, t); ++s) {
    const int v = (int)a.v0 + t.m0 + (int)c.rank * (kPairM / 2);
    int ra, rb;
    tokens_of(a, t, ra, rb);
    for (int r0 = ra; r0 < rb; r0 += kTile16, ++n) {
      int at[2];
      float rest[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + 32 * h + lane;
        at[h] = r < rb ? __ldcg(a.by_target + r) - v : -1;
        rest[h] = r < rb ? __ldcg(a.rest + r) : 0.f;
      }
      const uint32_t b = n & 1u;
      if (!__all_sync(0xffffffffu, mbar_wait(&c.ctl->rempty[b], ((n >> 1) & 1u) ^ 1u, st, 28))) return false;
      unsigned char* to = buf + b * kRestBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int& old = b ? was[1][h] : was[0][h];
        if (old >= 0) *reinterpret_cast<uint16_t*>(to + old) = 0;
        old = -1;
        const int k = 32 * h + lane, col = at[h] & 63;
        if (at[h] >= 0 && at[h] < kPairM / 2) {
          old = (at[h] >> 6) * kVBox + k * 128 + (((col >> 3) ^ (k & 7)) << 4) + 2 * (col & 7);
          *reinterpret_cast<uint16_t*>(to + old) = round16(rest[h], a.f16);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_release_cluster(leader_addr(&c.ctl->rfull[b]));
    }
  }
  return true;
}

// Loads of all tiles of this pair, by one thread of either CTA: its halves of the operands.  False after a timeout.
template <int kMode, int kS>
__device__ __forceinline__ bool load_tiles(const VocabMaps& maps, const VocabArgs& a, const Status& st, const Cta& c,
                                           Pipe& p) {
  constexpr bool kLogits = is_lse(kMode);
  const Plan plan = make_plan<kMode>(a, c.rows);
  const CUtensorMap* hmap = a.idx && (!kLogits || c.rows < a.T) ? &maps.hc : &maps.h;
  Tile t;
  for (int s = 0; next_tile<kMode>(plan, s, t); ++s) {
    const int am = t.m0 + (int)c.rank * (kPairM / 2), bn = t.n0 + (int)c.rank * (kPairN / 2);
    const int v0 = kLogits ? 0 : (int)a.v0;
    int ra = 0, rb = 0;
    if (is_products(kMode) && t.job == 1) tokens_of(a, t, ra, rb);
    // (few and large boxes: what this one thread issues for a step counts in the step's time)
    for (int k = 0; k < t.kb; ++k) {
      if (!mbar_wait(&c.ctl->empty[p.stage], p.phase ^ 1u, st, 20)) return false;
      const uint32_t sa = c.tiles + (uint32_t)p.stage * kVStage, sb = sa + 2 * kVBox;
      const uint32_t bar = leader_addr(&c.ctl->full[p.stage]);
      if (c.rank == 0) mbar_arrive_expect_tx(&c.ctl->full[p.stage], 2 * kVStage);
      ++p.issued;
      const int kx = (t.ka + k) * kTile16;
      if (!is_products(kMode)) {
        tma_load_2d_pair(sa, hmap, bar, kx, am);
        tma_load_2d_pair(sb, &maps.w, bar, kx, v0 + bn);
      } else if (t.job == 0) {
        tma_load_2d_pair(sa, &maps.dz, bar, kx, am);
        if (a.w_blocks) {
          tma_load_3d_pair(sb, &maps.wb, bar, v0 + kx, bn / kTile16);
        } else {
          tma_load_2d_pair(sb, &maps.wb, bar, bn, v0 + kx);
          tma_load_2d_pair(sb + kVBox, &maps.wb, bar, bn + kTile16, v0 + kx);
        }
      } else {
        tma_load_3d_pair(sa, &maps.dzb, bar, kx, am / kTile16);
        tma_load_3d_pair(sb, &maps.hb, bar, kx, bn / kTile16);
      }
      p.next<kS>();
    }
    for (int r = ra; r < rb; r += kTile16) {  // the hidden rows of write_rests
      if (!mbar_wait(&c.ctl->empty[p.stage], p.phase ^ 1u, st, 20)) return false;
      const uint32_t bar = leader_addr(&c.ctl->full[p.stage]);
      if (c.rank == 0) mbar_arrive_expect_tx(&c.ctl->full[p.stage], kVStage);
      ++p.issued;
      tma_load_3d_pair(c.tiles + (uint32_t)p.stage * kVStage + 2 * kVBox, &maps.hb, bar, r, bn / kTile16);
      p.next<kS>();
    }
  }
  return true;
}

// Their MMAs, by one thread of the leader.
template <int kMode, int kS>
__device__ __forceinline__ bool mma_tiles(const VocabArgs& a, const Status& st, const Cta& c, Pipe& p) {
  constexpr int seg = segment_of<kMode>();
  const Plan plan = make_plan<kMode>(a, c.rows);
  uint32_t rest = 0;  // steps of write_rests so far
  Tile t;
  for (int s = 0; next_tile<kMode>(plan, s, t); ++s) {
    const bool a_mn = is_products(kMode) && t.job == 1, b_mn = is_products(kMode);
    const uint32_t idesc = idesc_16_f32(kPairM, kPairN, a.f16 != 0, a_mn, b_mn);
    int ra = 0, rb = 0;
    if (is_products(kMode) && t.job == 1) tokens_of(a, t, ra, rb);
    // whole steps, and the instructions (16 k each) of the one that the operands end in
    const int ends = !is_products(kMode) ? a.D : t.job == 1 ? c.rows : (int)a.vn - t.ka * kTile16;
    const int whole = min(t.kb, ends / kTile16), last = whole < t.kb ? (ends - whole * kTile16 + 15) / 16 : 0;
    // (of the ring's first stage; addresses are in units of 16 bytes there)
    const uint64_t a0 = a_mn ? smem_desc_mn128(c.tiles, kVBox) : smem_desc_k128(c.tiles);
    const uint64_t b0 = (b_mn ? smem_desc_mn128(c.tiles, kVBox) : smem_desc_k128(c.tiles)) + (2 * kVBox >> 4);
    // 16 k: 32 bytes of a K-major row, 16 rows of 128 bytes otherwise
    const uint32_t as = a_mn ? 128u : 2u, bs = b_mn ? 128u : 2u;
    for (int64_t k0 = 0; k0 < t.kb || k0 == 0; k0 += seg, ++p.sum) {
      const int buf = p.sum & 1;
      if (!mbar_wait_cluster(&c.ctl->tempty[buf], ((uint32_t)(p.sum >> 1) & 1u) ^ 1u, st, 22)) return false;
      tc_fence_after();
      const uint32_t dt = c.tmem + (uint32_t)(buf * kPairN);
      const int k1 = (int)min((int64_t)t.kb, k0 + seg), kw = min(whole, k1);
      uint32_t add = 0;
      // (what this thread does between two steps' instructions shows in the time: whole steps by themselves)
      for (int k = (int)k0; k < kw; ++k) {
        if (!mbar_wait(&c.ctl->full[p.stage], p.phase, st, 23)) return false;
        tc_fence_after();
        const uint32_t at = (uint32_t)p.stage * (kVStage >> 4);
#pragma unroll
        for (uint32_t kk = 0; kk < kTile16 / 16; ++kk) mma_f16_pair(dt, a0 + at + as * kk, b0 + at + bs * kk, idesc, add | kk);
        add = 1;
        mma_commit_pair(&c.ctl->empty[p.stage]);
        p.next<kS>();
      }
      if (kw < k1) {
        if (!mbar_wait(&c.ctl->full[p.stage], p.phase, st, 23)) return false;
        tc_fence_after();
        const uint32_t at = (uint32_t)p.stage * (kVStage >> 4);
#pragma unroll 1
        for (int kk = 0; kk < last; ++kk, add = 1) mma_f16_pair(dt, a0 + at + as * kk, b0 + at + bs * kk, idesc, add);
        mma_commit_pair(&c.ctl->empty[p.stage]);
        p.next<kS>();
      }
      if constexpr (is_products(kMode)) {
#pragma unroll 1
        for (int r = ra; r < rb; r += kTile16, ++rest) {  // the steps of write_rests
          if (!mbar_wait(&c.ctl->full[p.stage], p.phase, st, 23)) return false;
          if (!mbar_wait_cluster(&c.ctl->rfull[rest & 1u], (rest >> 1) & 1u, st, 29)) return false;
          tc_fence_after();
          const uint32_t aa = (kS * kVStage + (rest & 1u) * kRestBytes) >> 4, at = (uint32_t)p.stage * (kVStage >> 4);
          const int n = min(kTile16 / 16, (rb - r + 15) / 16);
#pragma unroll 1
          for (int kk = 0; kk < n; ++kk) mma_f16_pair(dt, a0 + aa + as * kk, b0 + at + bs * kk, idesc, 1);
          mma_commit_pair(&c.ctl->empty[p.stage]);
          mma_commit_pair(&c.ctl->rempty[rest & 1u]);
          p.next<kS>();
        }
      }
      mma_commit_pair(&c.ctl->tfull[buf]);
    }
  }
  return true;
}

// What a row's token brings to its dz.
struct DzRow {
  float l2, g, e, ent;  // lse in units of log 2, d loss / d logp and d entropy (times the scale of an fp16 dz), entropy
  float at;             // dz at the target from the row's logp; NaN without one: then as every other column's
};
// (1 - p of a nearly certain token as a difference would be the error of its logit and of lse, 1e-7 of them, not 1 - p.
// logp, the forward pass's log1p of the sum over the other columns, still has its digits.)
template <bool kEnt>
__device__ __forceinline__ float dz_at_target(const DzRow& w, float lp) {
  const float v = -w.g * expm1f(lp);
  return kEnt ? fmaf(-w.e * expf(lp), lp + w.ent, v) : v;
}
// dz of 32 columns from their logits z, rounded to 16 bits and stored: those below `cols`, zeros past them (p of a
// padding row or column is no probability, and its row may hold anything).  tgt: the target's place; its dz into vt.
template <bool kEnt>
__device__ __forceinline__ void dz_columns(const VocabArgs& a, const DzRow& w, const float* z, int cols, int tgt, float& vt,
                                           uint16_t* dst) {
#pragma unroll
  for (int c = 0; c < 32; c += 16) {
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      float y[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = c + i + h;
        const float d = fmaf(z[j], a.sl2, -w.l2);  // log2 p
        const float p = ex2(d);
        float v = (j == tgt ? w.g : 0.f) - w.g * p;
        if (kEnt) v = fmaf(-w.e * p, fmaf(d, 0.6931471805599453f, w.ent), v);
        if (j == tgt) {
          if (w.at == w.at) v = w.at;
          vt = v;
        }
        y[h] = j < cols ? v : 0.f;
      }
      o[i / 2] = pack16(y[0], y[1], a.f16);
    }
    st_global_32(dst + c, o);
  }
}

// Their epilogues, by warps 4..11 of either CTA.  False (for the whole warp) after a timeout.
// (dz of logits that are one accumulation goes 32 columns at a time: a fourth of the code, which a call of few
// tiles runs cold.)
template <int kMode, int kS>
__device__ __forceinline__ bool finish_tiles(const VocabMaps& maps, const VocabArgs& a, const Status& st, const Cta& c, Pipe& p) {
  constexpr bool kLogits = is_lse(kMode);
  constexpr int seg = segment_of<kMode>();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = c.rows;
  const Plan plan = make_plan<kMode>(a, rows);
  const int q = warp & 3, half = (warp - 4) >> 2;  // tensor memory lanes 32 q .., columns 128 half ..
  const int r = (int)c.rank * (kPairM / 2) + q * 32 + lane;  // row in the tile
  const uint32_t lanes = c.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * (kPairN / 2));
  const uint32_t te = leader_addr(&c.ctl->tempty[0]);
  // waits for the n-th accumulation; false (for the whole warp) when that gave up
  auto ready = [&](int n) {
    const bool got = __all_sync(0xffffffffu, mbar_wait(&c.ctl->tfull[n & 1], (uint32_t)(n >> 1) & 1u, st, 25));
    tc_fence_after();
    return got;
  };
  // this warp has read its part of the n-th accumulation
  auto release = [&](int n) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive_cluster(te + 8u * (uint32_t)(n & 1));
  };
  unsigned char* own = c.smem + (c.tiles - smem_u32(c.smem)) + kS * kVStage + 2 * kRestBytes + (warp - 4) * kWarpBytes;  // (products)
  Tile t;
  for (int s = 0; next_tile<kMode>(plan, s, t); ++s) {
    const int row = t.m0 + r;
    const int n0 = t.n0 + half * (kPairN / 2);  // first column of this warp
    if constexpr (!is_products(kMode)) {
      const bool live = row < rows;
      // what the row's token brings
      int64_t tok = 0;
      int tgt = -1;
      DzRow w = {0.f, 0.f, 0.f, 0.f, __int_as_float(0x7fffffff)};
      if (live) {
        tok = a.idx ? __ldcg(a.idx + row) : row;
        const int64_t id = load_id(a.target, a.id8, tok);
        if (id >= 0 && id < a.V) tgt = (int)(id - (kLogits ? 0 : a.v0)) - n0;  // its column, from n0 on
        if (!kLogits) {
          const float gs = __ldcg(&a.head->dz_scale);
          w.l2 = a.lse[tok] * 1.4426950408889634f;
          w.g = a.g[tok] * gs;
          if (has_ent(kMode)) {
            w.e = a.ge[tok] * gs;
            w.ent = a.ent[tok];
          }
          // (kDzWideEnt takes it once its logits are summed: here, four of its registers would be spilled)
          if (kMode != kDzWideEnt && a.lp && tgt >= 0 && tgt < kPairN / 2) w.at = dz_at_target<has_ent(kMode)>(w, a.lp[tok]);
        }
      }
      if constexpr (kMode == kDz || kMode == kDzEnt) {
        uint16_t* dst = a.dz + (int64_t)row * a.dz_stride + n0;
        float vt = 0.f;
        if (!ready(p.sum)) return false;
#pragma unroll 1
        for (int ch = 0; ch < kPairN / 2; ch += 32) {
          uint32_t x[32];
          __syncwarp();
          tmem_ld_32x32b_x32(lanes + (uint32_t)((p.sum & 1) * kPairN + ch), x);
          tmem_wait_ld();
          if (ch + 32 == kPairN / 2) release(p.sum);
          float z[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) z[j] = __uint_as_float(x[j]);
          dz_columns<has_ent(kMode)>(a, w, z, (live ? (int)a.vn - n0 : 0) - ch, tgt - ch, vt, dst + ch);
        }
        ++p.sum;
        if (live && tgt >= 0 && tgt < kPairN / 2) a.rest[row] = vt - widen16(round16(vt, a.f16), a.f16);
      } else {
        uint64_t zz[kPairN / 4];  // two logits each
#pragma unroll
        for (int c = 0; c < kPairN / 4; ++c) zz[c] = 0ull;
        bool ok = true;
        const bool any = __any_sync(0xffffffffu, live);
        for (int k0 = 0; k0 < t.kb; k0 += seg, ++p.sum) {
          ok = ready(p.sum);
          if (!ok) break;
          const uint32_t src = lanes + (uint32_t)((p.sum & 1) * kPairN);
          if (any) {
#pragma unroll
            for (int c = 0; c < kPairN / 2; c += 32) {
              uint32_t x[32];
              tmem_ld_32x32b_x32(src + (uint32_t)c, x);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; j += 2) zz[(c + j) / 2] = f2add(zz[(c + j) / 2], pack_f2(x[j], x[j + 1]));
            }
          }
          release(p.sum);
        }
        if (!ok) return false;
        if (kLogits && !any) continue;  // no row of this warp is a token's
        float z[kPairN / 2];
#pragma unroll
        for (int c = 0; c < kPairN / 4; ++c) {
          uint32_t lo, hi;
          unpack_f2(zz[c], lo, hi);
          z[2 * c] = __uint_as_float(lo);
          z[2 * c + 1] = __uint_as_float(hi);
        }
        if constexpr (kLogits) {
          const int cols = (int)a.V - n0;
          if (cols < kPairN / 2) {
#pragma unroll
            for (int j = 0; j < kPairN / 2; ++j)
              if (j >= cols) z[j] = kNone;
          }
          const bool here = tgt >= 0 && tgt < kPairN / 2;
          if (__any_sync(0xffffffffu, here)) {  // the target's logit leaves the sums
            float tz = 0.f;
#pragma unroll
            for (int j = 0; j < kPairN / 2; ++j)
              if (j == tgt) {
                tz = z[j];
                z[j] = kNone;
              }
            if (here) a.tz[row] = tz * a.sl2;
          }
          float top[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
          for (int j = 4; j < kPairN / 2; ++j) top[j & 3] = fmaxf(top[j & 3], z[j]);
          const float m = fmaxf(kLow, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.sl2);
          float s4[4] = {0.f, 0.f, 0.f, 0.f}, u4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < kPairN / 2; ++j) {
            const float d = fmaf(z[j], a.sl2, -m);
            const float p = ex2(d);
            s4[j & 3] += p;
            if (has_ent(kMode)) u4[j & 3] = fmaf(p, d, u4[j & 3]);
          }
          if (live) {
            const int64_t at = (int64_t)row * a.part_row + (int64_t)(n0 / (kPairN / 2)) * a.part_col;
            a.pm[at] = m;
            a.ps[at] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            if (has_ent(kMode)) a.pu[at] = (u4[0] + u4[1]) + (u4[2] + u4[3]);
          }
        } else {
          uint16_t* dst = a.dz + (int64_t)row * a.dz_stride + n0;
          const int cols = live ? (int)a.vn - n0 : 0;
          float vt = 0.f;
          if (kMode == kDzWideEnt && a.lp && live && tgt >= 0 && tgt < kPairN / 2) w.at = dz_at_target<true>(w, a.lp[tok]);
#pragma unroll
          for (int ch = 0; ch < kPairN / 2; ch += 32) dz_columns<has_ent(kMode)>(a, w, z + ch, cols - ch, tgt - ch, vt, dst + ch);
          // what the rounding takes from dz at the target, by far the row's largest part: the products' epilogues add it
          if (live && tgt >= 0 && tgt < kPairN / 2) a.rest[row] = vt - widen16(round16(vt, a.f16), a.f16);
        }
      }
    } else {
      const bool live = row < (t.job == 1 ? (int)a.vn : rows);
      float rest = 0.f;  // d_hidden: what rounding took at the row's target, and the target's row
      const uint16_t* wrow = nullptr;
      if (t.job == 0 && live && t.split == 0) {
        const int y = __ldcg(a.by_target + row);
        if (y >= a.v0 && y < a.v0 + a.vn) {
          rest = __ldcg(a.rest + row);
          wrow = static_cast<const uint16_t*>(a.weight) + (int64_t)y * a.weight_stride;
        }
      }
      // (it is fetched while the sums are still being made)
      if (wrow) prefetch_row(wrow + n0, min(kPairN / 2, a.D - n0));
      const int tok = t.job == 0 && live ? __ldcg(a.idx + row) : 0;
      const bool bulk = t.job == 1 && a.dw_bulk != 0;
      const bool vec = t.job == 1 ? vec_rows(a.dw, a.dw_stride) : vec_rows(a.dh, a.dh_stride);
      const bool by_rows = kMode == kProductsRows && !vec && (t.job == 1 || (a.last && a.splits == 1));
      if (lane == 0) bulk_read();  // (the last tile's rows have left)
      __syncwarp();
      if (!ready(p.sum)) return false;
      const float f = a.scale / __ldcg(&a.head->dz_scale);
#pragma unroll 1
      for (int ch = 0; ch < kPairN / 2 / 32; ++ch) {
        uint32_t x[32];
        __syncwarp();
        tmem_ld_32x32b_x32(lanes + (uint32_t)((p.sum & 1) * kPairN + ch * 32), x);
        tmem_wait_ld();
        if (ch == kPairN / 2 / 32 - 1) release(p.sum);
        const int c0 = n0 + ch * 32;
        const int cols = a.D - c0;
        float y[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) y[j] = t.kb > 0 ? __uint_as_float(x[j]) : 0.f;  // (no tokens, or a short last piece's empty part of k: no product ran)
        if (rest != 0.f) add_row(wrow + c0, rest, cols, a.f16, y);
#pragma unroll
        for (int j = 0; j < 32; ++j) y[j] *= f;
        if (live && cols > 0 && t.job == 0) {
          const bool out = a.last && a.splits == 1;  // the whole sum
          if (!(a.first && out)) {  // several pieces or parts of k: the sums so far in fp32
            // (rows of whole 128-byte lines: what lies past the width is written, and never used)
            float* acc = a.acc + ((int64_t)t.split * a.acc_rows + row) * a.acc_stride + c0;
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              if (!a.first) {
                const float4 o0 = __ldcg(reinterpret_cast<const float4*>(acc + i)), o1 = __ldcg(reinterpret_cast<const float4*>(acc + i + 4));
                y[i] += o0.x, y[i + 1] += o0.y, y[i + 2] += o0.z, y[i + 3] += o0.w;
                y[i + 4] += o1.x, y[i + 5] += o1.y, y[i + 6] += o1.z, y[i + 7] += o1.w;
              }
              if (!out) {
                const uint32_t o[8] = {__float_as_uint(y[i]), __float_as_uint(y[i + 1]), __float_as_uint(y[i + 2]),
                                       __float_as_uint(y[i + 3]), __float_as_uint(y[i + 4]), __float_as_uint(y[i + 5]),
                                       __float_as_uint(y[i + 6]), __float_as_uint(y[i + 7])};
                st_global_32(acc + i, o);
              }
            }
          }
          if (out && vec && GPO_BOUNDS(st, tok, a.T, kWhereVocabToken))
            store16(static_cast<uint16_t*>(a.dh) + (int64_t)tok * a.dh_stride + c0, y, cols, a.f16, false);
        } else if (bulk && cols > 0) {
          // 64 columns of the warp's 32 rows, 128 bytes each with the 128-byte swizzle, go out as one bulk copy, which
          // leaves out what lies past the matrix: with a store per lane and row a tile's took 4 us of the load and store unit
          if ((ch & 1) == 0 && ch > 0) {
            if (lane == 0) bulk_read();
            __syncwarp();
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(own + lane * 128 + ((((ch & 1) * 4 + i) ^ (lane & 7)) << 4)) =
                make_uint4(pack16(y[8 * i], y[8 * i + 1], a.f16), pack16(y[8 * i + 2], y[8 * i + 3], a.f16),
                           pack16(y[8 * i + 4], y[8 * i + 5], a.f16), pack16(y[8 * i + 6], y[8 * i + 7], a.f16));
          if ((ch & 1) == 1 || cols <= 32) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bulk_store_2d(&maps.dw, own, n0 + (ch & ~1) * 32, (int)a.v0 + row);
          }
        } else if (vec && live && cols > 0 && GPO_BOUNDS(st, a.v0 + row, a.V, kWhereVocabRow)) {
          store16(static_cast<uint16_t*>(a.dw) + (a.v0 + row) * a.dw_stride + c0, y, cols, a.f16, a.accumulate != 0);
        }
        if (kMode == kProductsRows && by_rows && cols > 0) {
          const int64_t at = t.job == 1 ? a.v0 + row : tok;
          const bool put = live && GPO_BOUNDS(st, at, t.job == 1 ? a.V : a.T, t.job == 1 ? kWhereVocabRow : kWhereVocabToken);
          store_rows(reinterpret_cast<float*>(own), y, static_cast<uint16_t*>(t.job == 1 ? a.dw : a.dh) + c0,
                     t.job == 1 ? a.dw_stride : a.dh_stride, put ? at : -1, cols, a.f16, t.job == 1 && a.accumulate != 0, lane);
        }
      }
      ++p.sum;
    }
  }
  if constexpr (is_products(kMode)) {
    if (lane == 0) bulk_done();
    __syncwarp();
  }
  return true;
}

// Barriers and tensor memory of a pair.
template <int kS>
__device__ __forceinline__ Cta begin_pair(unsigned char* smem) {
  Cta c;
  c.smem = smem;
  c.ctl = reinterpret_cast<VocabCtl*>(smem);
  constexpr uint32_t kCtlBytes = (sizeof(VocabCtl) + 15) & ~15u;
  c.tiles = (smem_u32(smem) + kCtlBytes + 1023u) & ~1023u;
  c.rank = cluster_rank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kS; ++s) {
      mbar_init(&c.ctl->full[s], 1);
      mbar_init(&c.ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&c.ctl->tfull[b], 1);
      mbar_init(&c.ctl->tempty[b], 2 * kVEpiWarps);
      mbar_init(&c.ctl->rfull[b], 2);
      mbar_init(&c.ctl->rempty[b], 1);
    }
    mbar_init(&c.ctl->drain, 1);
    fence_mbar_init();
  }
  if (threadIdx.x >> 5 == kMmaWarp) {
    tmem_alloc_pair(&c.ctl->tmem_base, kVCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  c.tmem = c.ctl->tmem_base;
  return c;
}

__device__ __forceinline__ void end_pair(const Status& st, const Cta& c) {
  // after a timeout: every copy that either CTA issued lands before the shared memory goes
  if (threadIdx.x == 0 && aborted(st)) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 1000000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  if (threadIdx.x >> 5 == kMmaWarp) tmem_dealloc_pair(c.tmem, kVCols);
}

// Wind-down of the loading lane: the leader's barriers count both CTAs' copies, which land before the CTAs may exit.
template <int kS>
__device__ __forceinline__ void end_loads(const Status& st, const Cta& c, const Pipe& p) {
  if (c.rank == 0)
    for (uint32_t s = 0; s < kS; ++s)
      if (s < p.issued) mbar_wait(&c.ctl->full[s], (p.issued - 1 - s) / kS & 1u, st, 21, 200000000ull, false);
}
// Of the MMA lane: all issued MMAs complete before tensor memory is released.
__device__ __forceinline__ void end_mmas(const Status& st, const Cta& c) {
  mma_commit_pair(&c.ctl->drain);
  mbar_wait(&c.ctl->drain, 0, st, 24, 200000000ull, false);
}

template <int kMode>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kVThreads, 1)
    vocab_pair_kernel(const __grid_constant__ VocabMaps maps, VocabArgs a, Status st) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  constexpr int kS = is_products(kMode) ? kPStages : kVStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  Cta c = begin_pair<kS>(smem_raw);
  after_previous();
  // (as the call's first kernel; in the idle warp's own branch below, kLse and kLseEnt spill 100 bytes)
  if (is_lse(kMode) && !a.idx && blockIdx.x == 0 && threadIdx.x == 32 * kIdleWarp) next_tag(st);
  __syncwarp();
  c.rows = a.idx ? a.head->rows : (int)a.T;
  Pipe p;
  if (warp < 4) {
    if (keeps_logits(kMode)) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(regs_few(kMode)));
    if (warp == kLoadWarp && lane == 0) {
      load_tiles<kMode, kS>(maps, a, st, c, p);
      end_loads<kS>(st, c, p);
    } else if (is_products(kMode) && warp == kRestWarp) {
      if (a.dw) write_rests(a, st, c, kS * kVStage, lane);
    } else if (warp == kMmaWarp && lane == 0 && c.rank == 0) {
      if (a.debug_timeout) mbar_wait(&c.ctl->drain, 0, st, 27, kDebugTimeoutNs);  // reports GPO_ERR_TIMEOUT
      else mma_tiles<kMode, kS>(a, st, c, p);
      end_mmas(st, c);
    }
    __syncwarp();
  } else {
    if (keeps_logits(kMode)) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(regs_many(kMode)));
    finish_tiles<kMode, kS>(maps, a, st, c, p);
  }
  end_pair(st, c);
}

// ------------------------------------------------------------------ tokens that take part

// Tokens up to which their order is found by comparing all with all, in one launch; beyond, by the sort and a
// gathering launch (vocabulary 32000 x 512: 14.5 against 17.2 us for 2048 tokens, as long for 4096,
// 36 against 19 for 8192; for 65536 890 against 66).
constexpr int kVocabOrder = 4096;
constexpr int kRowThreads = 1024;
constexpr int kRowAhead = 8;  // tokens of a thread in flight

// Forward: the list of the tokens with a target, in their order, their number, their hidden rows copied
// together (where some token is left out), and the zeros of the others' results.  Every CTA looks
// at all tokens (a few bytes each) to know how many take part, and how many before its own share of
// them: one launch and no exchange.
// (Id: a template, so that the loads of one thread need no branch between them.)
template <class Id>
__global__ void __launch_bounds__(kRowThreads) vocab_rows_kernel(VocabArgs a, Status st) {
  constexpr int kW = kRowThreads / 32;
  __shared__ int s_before[kW], s_all[kW], s_cnt[kW];
  __shared__ int s_list[kRowThreads];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  let_next_start();
  const int64_t ta = a.T * blockIdx.x / gridDim.x, tb = a.T * (blockIdx.x + 1) / gridDim.x;
  const Id* target = static_cast<const Id*>(a.target);
  int before = 0, all = 0;
  for (int64_t t0 = threadIdx.x; t0 < a.T; t0 += kRowAhead * kRowThreads) {
    Id id[kRowAhead];
#pragma unroll
    for (int k = 0; k < kRowAhead; ++k) id[k] = t0 + k * kRowThreads < a.T ? target[t0 + k * kRowThreads] : (Id)-1;
#pragma unroll
    for (int k = 0; k < kRowAhead; ++k) {
      const int64_t t = t0 + k * kRowThreads;
      const bool in = id[k] >= 0 && id[k] < a.V;
      if (id[k] >= a.V && blockIdx.x == 0) report(st, GPO_ERR_SHAPE, 26, (int)t);
      all += in;
      before += in && t < ta;
    }
  }
  all = __reduce_add_sync(0xffffffffu, all);
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) {
    s_all[warp] = all;
    s_before[warp] = before;
  }
  __syncthreads();
  all = __reduce_add_sync(0xffffffffu, s_all[lane]);
  int base = __reduce_add_sync(0xffffffffu, s_before[lane]);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.head->rows = all;
    a.head->dz_scale = 1.f;
  }
  const bool gather = all < a.T;
  const int chunks = (a.D + 7) / 8;  // 16 bytes each (rows hold a multiple of them)
  for (int64_t t0 = ta; t0 < tb; t0 += kRowThreads) {
    const int64_t t = t0 + threadIdx.x;
    const Id id = t < tb ? target[t] : (Id)-1;
    const bool in = id >= 0 && id < a.V;
    const uint32_t m = __ballot_sync(0xffffffffu, in);
    if (lane == 0) s_cnt[warp] = __popc(m);
    __syncthreads();
    const int n = __reduce_add_sync(0xffffffffu, s_cnt[lane]);
    const int lower = __reduce_add_sync(0xffffffffu, lane < warp ? s_cnt[lane] : 0);
    if (in) {
      const int r = lower + __popc(m & ((1u << lane) - 1u));
      s_list[r] = (int)t;
      if (GPO_BOUNDS(st, base + r, a.T, kWhereVocabRow)) a.idx[base + r] = (int)t;
    } else if (t < tb) {
      a.logp[t] = 0.f;
      if (a.lse_out) a.lse_out[t] = 0.f;
      if (a.ent_out) a.ent_out[t] = 0.f;
    }
    __syncthreads();
    if (gather) {
      for (int r = warp; r < n; r += kW) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.hidden) + (int64_t)s_list[r] * a.hidden_stride);
        uint4* dst = reinterpret_cast<uint4*>(a.hc + (int64_t)(base + r) * a.hc_stride);
#pragma unroll 8
        for (int c = lane; c < chunks; c += 32) dst[c] = src[c];
      }
    }
    base += n;
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) next_tag(st);
}

// A power of two that brings an fp16 dz, |dz| <= bound, into the type's range; 1 for bf16.  (|dz| is at most
// |g| + |e| max p |log p + H|, whose last factor is below log V + 1 < 24.)
__device__ __forceinline__ float scale_of_dz(const VocabArgs& a, float bound) {
  if (!a.f16 || !(bound > 0.f) || !isfinite(bound)) return 1.f;
  int ex;
  frexpf(bound, &ex);  // bound <= 2^ex: |dz| up to 2^14, within fp16's 65504
  return ldexpf(1.f, min(max(14 - ex, -100), 100));
}
// A token without a gradient gets a d_hidden of zeros, from one warp.
__device__ __forceinline__ void no_d_hidden(const VocabArgs& a, int64_t t, bool vec, int lane) {
  uint16_t* dst = static_cast<uint16_t*>(a.dh) + t * a.dh_stride;
  const int whole = vec ? a.D / 8 : 0;
  for (int c = lane; c < whole; c += 32) reinterpret_cast<uint4*>(dst)[c] = make_uint4(0u, 0u, 0u, 0u);
  for (int c = whole * 8 + lane; c < a.D; c += 32) dst[c] = 0;
}
// One hidden row to its place in hc, by one warp (rows hold a multiple of 16 bytes); t < 0: zeros, in the rows
// behind the last that the steps of the d_weight product meet: those of dz end at a multiple of 64, those of the
// rests less than 64 behind the last row (what lies past the tensor map's end reads as zeros).
__device__ __forceinline__ int64_t rows_behind(const VocabArgs& a, int64_t rows) {
  return min((rows + kTile16 - 1) / kTile16 + 1, (a.T + kTile16 - 1) / kTile16) * kTile16;
}
__device__ __forceinline__ void gather_row(const VocabArgs& a, int64_t r, int64_t t, int lane) {
  const int chunks = (a.D + 7) / 8;
  uint4* dst = reinterpret_cast<uint4*>(a.hc + r * a.hc_stride);
  if (t < 0) {
    for (int c = lane; c < chunks; c += 32) dst[c] = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.hidden) + t * a.hidden_stride);
#pragma unroll 8
  for (int c = lane; c < chunks; c += 32) dst[c] = src[c];
}
// Gradient: the tokens with a target and a gradient that is not 0, in the order of their targets and, for one
// target, their own; their number, the scale of an fp16 dz, the number of tokens before each tile's targets, their hidden
// rows in that order with zeros behind them (see gather_row), and the zeros of the others' d_hidden.
// A token's place is the number of those before it in that order: every CTA counts, for its share of the
// tokens, through all of them (T^2 / 152 comparisons in shared memory), with no exchange between CTAs and no
// second launch.
__global__ void __launch_bounds__(kRowThreads) vocab_order_kernel(VocabArgs a, Status st) {
  constexpr int kW = kRowThreads / 32, kPer = kVocabOrder / kRowThreads;
  __shared__ int s_key[kVocabOrder];
  __shared__ int s_all[kW];
  __shared__ float s_big[kW];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, T = (int)a.T;
  let_next_start();
  int64_t id[kPer];
  float g[kPer], e[kPer];
  // (one branch around the loads of a thread, which are then in flight together)
  if (a.id8) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int u = k * kRowThreads + threadIdx.x;
      id[k] = u < T ? static_cast<const int64_t*>(a.target)[u] : -1;
    }
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int u = k * kRowThreads + threadIdx.x;
      id[k] = u < T ? static_cast<const int32_t*>(a.target)[u] : -1;
    }
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int u = k * kRowThreads + threadIdx.x;
    g[k] = u < T ? a.g[u] : 0.f;
    e[k] = 0.f;
  }
  if (a.ge) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k * kRowThreads + threadIdx.x < T) e[k] = a.ge[k * kRowThreads + threadIdx.x];
  }
  int all = 0;
  float bound = 0.f;  // of |dz| (see scale_of_dz)
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int u = k * kRowThreads + threadIdx.x;
    const bool in = id[k] >= 0 && id[k] < a.V && (g[k] != 0.f || e[k] != 0.f);
    if (in) {
      ++all;
      bound = fmaxf(bound, fabsf(g[k]) + 24.f * fabsf(e[k]));
    }
    if (id[k] >= a.V && blockIdx.x == 0) report(st, GPO_ERR_SHAPE, 26, u);
    s_key[u] = in ? (int)id[k] : kNoKey;
  }
  all = __reduce_add_sync(0xffffffffu, all);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) bound = fmaxf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
  if (lane == 0) {
    s_all[warp] = all;
    s_big[warp] = bound;
  }
  __syncthreads();
  all = __reduce_add_sync(0xffffffffu, s_all[lane]);
  const bool vec = vec_rows(a.dh, a.dh_stride);
  const int ta = (int)(a.T * blockIdx.x / gridDim.x), tb = (int)(a.T * (blockIdx.x + 1) / gridDim.x);
  for (int t = ta + warp; t < tb; t += kW) {
    const int key = s_key[t];
    if (key != kNoKey) {
      int r = 0;
#pragma unroll 4
      for (int u = lane; u < T; u += 32) r += s_key[u] < key + (u < t ? 1 : 0);
      r = __reduce_add_sync(0xffffffffu, r);
      if (!GPO_BOUNDS(st, r, a.T, kWhereVocabRow)) continue;
      if (lane == 0) {
        a.idx[r] = t;
        a.by_target[r] = key;
      }
      gather_row(a, r, t, lane);
    } else if (a.dh) {
      no_d_hidden(a, t, vec, lane);
    }
  }
  const int64_t tiles = (a.V + kPairM - 1) / kPairM;
  for (int64_t j = blockIdx.x + (int64_t)gridDim.x * (kW - 1 - warp); j <= tiles; j += (int64_t)gridDim.x * kW) {
    const int key = (int)min(j * kPairM, a.V);
    int n = 0;
#pragma unroll 4
    for (int u = lane; u < T; u += 32) n += s_key[u] < key;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) a.tile_first[j] = n;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    for (int w = 0; w < kW; ++w) bound = fmaxf(bound, s_big[w]);
    a.head->rows = all;
    a.head->dz_scale = scale_of_dz(a, bound);
  }
  if (blockIdx.x == gridDim.x - 1)
    for (int64_t r = all + warp; r < rows_behind(a, all); r += kW) gather_row(a, r, -1, lane);
  if (blockIdx.x == 0 && threadIdx.x == 0) next_tag(st);
}

// The same for more than kVocabOrder tokens, whose comparisons would grow with T^2: the sort's work grows with T.
template <class Id>
struct VocabKeys {
  using Key = Id;
  const VocabArgs& a;
  float bound = 0.f;  // of |dz| (see scale_of_dz)
  __device__ explicit VocabKeys(const VocabArgs& args) : a(args) {}
  __device__ __forceinline__ void load(int64_t t0, int64_t tb, Id (&id)[kSortAhead]) {
    const Id* target = static_cast<const Id*>(a.target);
    float g[kSortAhead], e[kSortAhead];
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      const bool in = t0 + 32 * k < tb;
      id[k] = in ? target[t0 + 32 * k] : (Id)-1;
      g[k] = in ? a.g[t0 + 32 * k] : 0.f;
      e[k] = 0.f;
    }
    if (a.ge) {
#pragma unroll
      for (int k = 0; k < kSortAhead; ++k)
        if (t0 + 32 * k < tb) e[k] = a.ge[t0 + 32 * k];
    }
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      if (id[k] < 0 || id[k] >= a.V) continue;
      if (g[k] != 0.f || e[k] != 0.f) bound = fmaxf(bound, fabsf(g[k]) + 24.f * fabsf(e[k]));
      else id[k] = (Id)-1;
    }
  }
};

template <class Id>
__global__ void __launch_bounds__(kSortThreads, 1) vocab_sort_kernel(VocabArgs a, int per, Status st) {
  extern __shared__ int hist[];
  __shared__ float s_big[kSortWarps];
  let_next_start();
  VocabKeys<Id> keys(a);
  sort_tokens<26, kWhereVocabRow>(
      keys, a.T, a.V, per, hist, st,
      [&](int64_t row, int first) {
        if (row % kPairM == 0 || row == a.V) a.tile_first[(row + kPairM - 1) / kPairM] = first;
        if (row == a.V) a.head->rows = first;
      },
      [&](int place, int64_t t, Id id) {
        a.idx[place] = (int)t;
        a.by_target[place] = (int)id;
      });
  float bound = keys.bound;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) bound = fmaxf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
  if ((threadIdx.x & 31) == 0) s_big[threadIdx.x >> 5] = bound;
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    for (int w = 0; w < kSortWarps; ++w) bound = fmaxf(bound, s_big[w]);
    a.head->dz_scale = scale_of_dz(a, bound);
    next_tag(st);
  }
}

__global__ void __launch_bounds__(256) vocab_gather_kernel(VocabArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), nwarps = (int64_t)gridDim.x * 8;
  let_next_start();
  after_previous();
  const int64_t rows = a.head->rows, pad = rows_behind(a, rows);
  for (int64_t r = warp; r < pad; r += nwarps) gather_row(a, r, r < rows ? a.idx[r] : -1, lane);
  if (!a.dh) return;
  const bool vec = vec_rows(a.dh, a.dh_stride);
  for (int64_t t = warp; t < a.T; t += nwarps) {
    const int64_t id = load_id(a.target, a.id8, t);
    if (id >= 0 && id < a.V && (a.g[t] != 0.f || (a.ge && a.ge[t] != 0.f))) continue;
    no_d_hidden(a, t, vec, lane);
  }
}

// d_hidden from the sums of its parts of k, added in order, by threads i0, i0 + step, ..
__device__ __forceinline__ void add_parts(const VocabArgs& a, int rows, int64_t i0, int64_t step) {
  const int quads = (a.D + 3) / 4;
  const bool vec = ((a.dh_stride & 3) | (reinterpret_cast<uintptr_t>(a.dh) & 7)) == 0;
  for (int64_t i = i0; i < (int64_t)rows * quads; i += step) {
    const int row = (int)(i / quads), c = (int)(i - (int64_t)row * quads) * 4;
    const float* p = a.acc + (int64_t)row * a.acc_stride + c;
    float4 s = __ldcg(reinterpret_cast<const float4*>(p));
#pragma unroll 4
    for (int k = 1; k < a.splits; ++k) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p + k * a.acc_rows * a.acc_stride));
      s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
    uint16_t* dst = static_cast<uint16_t*>(a.dh) + (int64_t)__ldcg(a.idx + row) * a.dh_stride + c;
    const uint2 o = make_uint2(pack16(s.x, s.y, a.f16), pack16(s.z, s.w, a.f16));
    if (vec && c + 4 <= a.D) {
      *reinterpret_cast<uint2*>(dst) = o;
    } else {
      const uint16_t h[4] = {(uint16_t)o.x, (uint16_t)(o.x >> 16), (uint16_t)o.y, (uint16_t)(o.y >> 16)};
      for (int j = 0; j < 4 && c + j < a.D; ++j) dst[j] = h[j];
    }
  }
}

__global__ void __launch_bounds__(256) vocab_parts_kernel(VocabArgs a) {
  after_previous();
  add_parts(a, a.head->rows, (int64_t)blockIdx.x * blockDim.x + threadIdx.x, (int64_t)gridDim.x * blockDim.x);
}

// ------------------------------------------------------------------ joining the parts of a row

constexpr int kJoinThreads = 256;

// Parts of a row side by side: a CTA per row (few tokens).  Where the tokens are listed, a row is one of the list: its
// parts and its target's logit are at the row's number, its target and its results at the token's.
template <bool kEnt>
__global__ void __launch_bounds__(kJoinThreads) vocab_join_row_kernel(VocabArgs a, int parts, Status st) {
  __shared__ Part red[kJoinThreads / 32];
  const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  after_previous();
  if (a.idx && row >= a.head->rows) return;  // (vocab_rows_kernel has written the others' zeros)
  const int64_t tok = a.idx ? a.idx[row] : row;
  const int64_t id = load_id(a.target, a.id8, tok);
  if (id < 0 || id >= a.V) {
    if (threadIdx.x == 0) {
      if (id >= a.V) report(st, GPO_ERR_SHAPE, 26, row);
      a.logp[tok] = 0.f;
      if (a.lse_out) a.lse_out[tok] = 0.f;
      if (kEnt) a.ent_out[tok] = 0.f;
    }
    return;
  }
  Part p = {kLow, 0.f, 0.f};
  const int64_t at = (int64_t)row * a.part_row;
  for (int i = threadIdx.x; i < parts; i += kJoinThreads)
    p = join<kEnt>(p, Part{a.pm[at + i], a.ps[at + i], kEnt ? a.pu[at + i] : 0.f});
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Part y = {__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                    __shfl_xor_sync(0xffffffffu, p.u, o)};
    p = join<kEnt>(p, y);
  }
  if (lane == 0) red[warp] = p;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kJoinThreads / 32; ++w) p = join<kEnt>(p, red[w]);
    finish<kEnt>(a, tok, a.tz[row], p);
  }
}

// Rows side by side: a CTA takes 32 rows, its warps the parts in turn.
template <bool kEnt>
__global__ void __launch_bounds__(1024) vocab_join_kernel(VocabArgs a, int parts, Status st) {
  __shared__ Part red[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  after_previous();
  const int row = blockIdx.x * 32 + lane, rows = a.idx ? a.head->rows : (int)a.T;
  if (blockIdx.x * 32 >= rows) return;
  Part p = {kLow, 0.f, 0.f};
  if (row < rows) {
#pragma unroll 4
    for (int i = warp; i < parts; i += 32) {
      const int64_t at = row + (int64_t)i * a.part_col;
      p = join<kEnt>(p, Part{a.pm[at], a.ps[at], kEnt ? a.pu[at] : 0.f});
    }
  }
  red[warp][lane] = p;
  __syncthreads();
  if (warp == 0 && row < rows) {
    const int64_t tok = a.idx ? a.idx[row] : row;
    const int64_t id = load_id(a.target, a.id8, tok);
    if (id >= 0 && id < a.V) {
      for (int w = 1; w < 32; ++w) p = join<kEnt>(p, red[w][lane]);
      finish<kEnt>(a, tok, a.tz[row], p);
    } else {  // (every token is multiplied)
      if (id >= a.V) report(st, GPO_ERR_SHAPE, 26, row);
      a.logp[tok] = 0.f;
      if (a.lse_out) a.lse_out[tok] = 0.f;
      if (kEnt) a.ent_out[tok] = 0.f;
    }
  }
}

int g_pairs = 0;  // CTA pairs resident at one time

template <int kMode>
cudaError_t setup_mode() {
  cudaFuncAttributes at;
  const cudaError_t e = cudaFuncGetAttributes(&at, vocab_pair_kernel<kMode>);
  if (e != cudaSuccess) return e;
  // (a split that asks for more registers than the launch brings would wait for ever)
  if (keeps_logits(kMode) && at.numRegs < kRegsLaunch) return cudaErrorInvalidConfiguration;
  return cudaFuncSetAttribute(vocab_pair_kernel<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of(kMode));
}

template <int kMode>
cudaError_t launch_pair(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st, int64_t tiles) {
  const int64_t pairs = min((int64_t)g_pairs, max(tiles, (int64_t)1));
  return launch_after(vocab_pair_kernel<kMode>, (unsigned)(2 * pairs), kVThreads, smem_of(kMode), lc.stream, m, a, st);
}

int64_t tiles_of(int64_t rows, int64_t cols) { return ((rows + kPairM - 1) / kPairM) * ((cols + kPairN - 1) / kPairN); }

}  // namespace

cudaError_t setup_vocab() {
  cudaError_t e = setup_mode<kLse>();
  if (e == cudaSuccess) e = setup_mode<kLseEnt>();
  if (e == cudaSuccess) e = setup_mode<kDz>();
  if (e == cudaSuccess) e = setup_mode<kDzEnt>();
  if (e == cudaSuccess) e = setup_mode<kDzWide>();
  if (e == cudaSuccess) e = setup_mode<kDzWideEnt>();
  if (e == cudaSuccess) e = setup_mode<kProducts>();
  if (e == cudaSuccess) e = setup_mode<kProductsRows>();
  const int bytes = (int)sort_smem(kSortMaxRows);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(vocab_sort_kernel<int32_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(vocab_sort_kernel<int64_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kVThreads);
  cfg.dynamicSmemBytes = kPSmem;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 2;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  int n = 0;
  e = cudaOccupancyMaxActiveClusters(&n, vocab_pair_kernel<kProducts>, &cfg);
  if (e == cudaSuccess) g_pairs = n > 0 ? n : 1;
  return e;
}

cudaError_t launch_vocab_rows(const LaunchCtx& lc, const VocabArgs& a, const Status& st) {
  const int grid = (int)max((int64_t)1, min(a.T / 4, (int64_t)lc.num_sms));
  if (a.id8) vocab_rows_kernel<int64_t><<<grid, kRowThreads, 0, lc.stream>>>(a, st);
  else vocab_rows_kernel<int32_t><<<grid, kRowThreads, 0, lc.stream>>>(a, st);
  return cudaGetLastError();
}

cudaError_t launch_vocab_order(const LaunchCtx& lc, const VocabArgs& a, const Status& st) {
  if (a.T > kVocabOrder) {
    const int per = sort_rows(a.V, lc.num_sms);
    const unsigned ctas = (unsigned)((a.V + per - 1) / per);
    if (a.id8) vocab_sort_kernel<int64_t><<<ctas, kSortThreads, sort_smem(per), lc.stream>>>(a, per, st);
    else vocab_sort_kernel<int32_t><<<ctas, kSortThreads, sort_smem(per), lc.stream>>>(a, per, st);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_after(vocab_gather_kernel, (unsigned)min((a.T + 7) / 8, (int64_t)lc.num_sms * 8), 256, 0, lc.stream, a);
  }
  const int grid = (int)max((int64_t)1, min(a.T / 4, (int64_t)lc.num_sms));
  vocab_order_kernel<<<grid, kRowThreads, 0, lc.stream>>>(a, st);
  return cudaGetLastError();
}

cudaError_t launch_vocab_lse(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st, bool ent) {
  return ent ? launch_pair<kLseEnt>(lc, m, a, st, tiles_of(a.T, a.V)) : launch_pair<kLse>(lc, m, a, st, tiles_of(a.T, a.V));
}

cudaError_t launch_vocab_join(const LaunchCtx& lc, const VocabArgs& a, const Status& st, bool ent) {
  const int parts = (int)vocab_parts(a.V);
  if (a.part_col == 1)
    return launch_after(ent ? vocab_join_row_kernel<true> : vocab_join_row_kernel<false>, (unsigned)a.T, kJoinThreads, 0,
                        lc.stream, a, parts, st);
  return launch_after(ent ? vocab_join_kernel<true> : vocab_join_kernel<false>, (unsigned)((a.T + 31) / 32), 1024, 0,
                      lc.stream, a, parts, st);
}

cudaError_t launch_vocab_dz(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st) {
  const int64_t tiles = tiles_of(a.T, a.vn);
  if (a.D <= kTile16 * kVocabDzSeg) return a.ge ? launch_pair<kDzEnt>(lc, m, a, st, tiles) : launch_pair<kDz>(lc, m, a, st, tiles);
  return a.ge ? launch_pair<kDzWideEnt>(lc, m, a, st, tiles) : launch_pair<kDzWide>(lc, m, a, st, tiles);
}

// With few row tiles the k of d_hidden, the vocabulary, is cut into parts for as many pairs as its share of
// the work is worth (300 tokens, 8191 x 512: one pair's sum over 8191 rows took 35 of the call's 67 us).
int vocab_splits(int64_t T, int64_t vn, int64_t D) {
  const int64_t dt = (D + kPairN - 1) / kPairN, mt = (T + kPairM - 1) / kPairM, kb = (vn + kTile16 - 1) / kTile16;
  const int64_t work = mt * dt * kb + (vn + kPairN - 1) / kPairN * dt * max((T + kTile16 - 1) / kTile16, (int64_t)kEpiSteps);
  const int64_t share = max(work / kVocabPairs, (int64_t)kEpiSteps);  // k-steps of one pair
  if (kb <= 24) return 1;  // (less time than the launch that adds the parts)
  return (int)max((int64_t)1, min((kb + share - 1) / share, (int64_t)kVocabMaxSplits));
}

cudaError_t launch_vocab_products(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st) {
  const int64_t tiles = (a.dh ? tiles_of(a.T, a.D) * a.splits : 0) + (a.dw ? tiles_of(a.vn, a.D) : 0);
  const bool vec = (!a.dh || vec_rows(a.dh, a.dh_stride)) && (!a.dw || vec_rows(a.dw, a.dw_stride));
  const cudaError_t e = vec ? launch_pair<kProducts>(lc, m, a, st, tiles) : launch_pair<kProductsRows>(lc, m, a, st, tiles);
  if (e != cudaSuccess || !a.last || a.splits == 1) return e;
  const int64_t quads = a.T * ((a.D + 3) / 4);
  return launch_after(vocab_parts_kernel, (unsigned)min((quads + 255) / 256, (int64_t)lc.num_sms * 8), 256, 0, lc.stream, a);
}

}  // namespace gpo
