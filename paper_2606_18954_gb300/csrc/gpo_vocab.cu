// Per-token log-probabilities from hidden states and the vocabulary matrix, and their gradients,
// on the tcgen05 tensor cores (the formulas are in include/graphpo.h).
//
// Forward, two launches and for more than 256 tokens two more before them:
//   rows     vocab_index_kernel lists the tokens with a target, vocab_gather_kernel copies their
//            hidden rows together (skipped where every token has one): tokens without a target cost no
//            product, and what their rows hold reaches nothing
//   lse      vocab_pair_kernel<kLse>: logits tiles of 256 tokens x 256 vocabulary rows that stay in tensor
//            memory; the epilogue reduces each row's 128 columns to a maximum and a sum (and the entropy's
//            sum), the target's logit kept apart
//   join     vocab_join_kernel: the parts of a row joined in a fixed order
// Gradient, piece by piece of the vocabulary (dz of a piece takes at most 512 MiB):
//   rows     as above, for the tokens with a gradient that is not 0
//   dz       vocab_pair_kernel<kDz>: the logits again, dz in the epilogue, written in 16 bits
//   products vocab_pair_kernel<kProducts>: d_hidden += dz W and d_weight = dz^T hidden in one launch
// Keeping the sum over the other tokens of the vocabulary apart from the target's term keeps the
// digits of a nearly certain token's log-probability -log(1 + sum), which is a small number.
#define GPO_REPORT __noinline__
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gpo_pair.cuh"

namespace gpo {

namespace {

enum Mode { kLse, kLseEnt, kDz, kDzEnt, kProducts };

constexpr int kTile16 = 64;                        // elements of one 128-byte swizzle row
constexpr int kVStages = 6;
constexpr int kVThreads = 384;                     // warps: 0 loads, 1 MMAs, 2 tensor memory, 4..11 epilogue
constexpr int kVEpiWarps = 8;
constexpr int kVBox = kTile16 * 128;               // one 64 x 64 box
constexpr int kVStage = 4 * kVBox;                 // A and B halves of one k-step, per CTA
constexpr int kVCols = 512;                        // two accumulators of 256 columns
// Logits: steps of k after which the tensor cores' sum is taken over into registers.  Their fp32
// additions drop the bits below the sum's last one, always towards zero, so that a sum of d products
// shrinks by about d / 16 half ulps: 7e-6 of a logit at d = 4096, too much for the log-probability of
// a nearly certain token.  Sums of 256 products, added in registers with rounding, stay at fp32's own
// error.  (The gradients' sums are rounded to 16 bits, 1e3 times as much.)
constexpr int kSegment = 4;
constexpr int kRaster = 32;                        // row tiles that share one pass over the columns
// A logit that is left out (a column past the vocabulary, the target) and the maximum of a part without
// logits: for every scale in [1e-4, 1e4] the first, scaled, is finite and far below the second
constexpr float kNone = -1e33f, kLow = -1e28f;

struct __align__(8) VocabCtl {
  uint64_t full[kVStages];
  uint64_t empty[kVStages];
  uint64_t tfull[2];
  uint64_t tempty[2];
  uint64_t drain;
  uint32_t tmem_base;
};

constexpr size_t kVSmem = ((sizeof(VocabCtl) + 15) & ~size_t(15)) + 1023 + (size_t)kVStages * kVStage;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ int64_t load_id(const void* ids, int id8, int64_t t) {
  return id8 ? static_cast<const int64_t*>(ids)[t] : (int64_t)static_cast<const int32_t*>(ids)[t];
}

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

// One tile of a pair: the rows of A from m0, the columns (rows of B) from n0, kb steps of 64 of k.
struct Tile {
  int job;  // kProducts: 0 d_hidden, 1 d_weight
  int m0, n0, kb;
};

// The tiles of one launch and which pair takes which, in what order.
struct Plan {
  int p, np;           // this pair of np
  int mt, nt, kb;      // kLse, kDz: row tiles, column tiles, k-steps
  int dt;              // kProducts: column tiles of d
  int n_dh, kb_dh, own_dh, n_dw, kb_dw;
  int light0, nlight, extra;  // pairs from light0 on take `extra` d_weight tiles more, for the d_hidden tile they lack
};

template <int kMode>
__device__ __forceinline__ Plan make_plan(const VocabArgs& a, int rows) {
  Plan q;
  q.p = (int)blockIdx.x >> 1;
  q.np = (int)gridDim.x >> 1;
  q.mt = (rows + kPairM - 1) / kPairM;
  const int64_t cols = kMode == kLse || kMode == kLseEnt ? a.V : a.vn;
  q.nt = (int)((cols + kPairN - 1) / kPairN);
  q.kb = (a.D + kTile16 - 1) / kTile16;
  q.dt = (a.D + kPairN - 1) / kPairN;
  // the longer d_hidden tiles first, round robin; the pairs that get one less take as much work in
  // d_weight tiles, the rest of which go round robin too
  q.n_dh = a.dh ? q.mt * q.dt : 0;
  q.n_dw = a.dw ? q.nt * q.dt : 0;
  q.kb_dh = (int)((a.vn + kTile16 - 1) / kTile16);
  q.kb_dw = (rows + kTile16 - 1) / kTile16;
  q.own_dh = q.n_dh / q.np + (q.p < q.n_dh % q.np ? 1 : 0);
  q.light0 = q.n_dh % q.np;
  q.nlight = q.np - q.light0;
  q.extra = q.light0 > 0 && q.kb_dw > 0 ? min(q.kb_dh / q.kb_dw, q.n_dw / q.nlight) : 0;
  return q;
}

// The pair's s-th tile; false after the last.
template <int kMode>
__device__ __forceinline__ bool next_tile(const Plan& q, int s, Tile& t) {
  if (kMode != kProducts) {
    const int64_t i = q.p + (int64_t)s * q.np;
    if (i >= (int64_t)q.mt * q.nt) return false;
    // kRaster row tiles take the columns together: what the pairs work on at one time is few columns of
    // all those rows, whose hidden states stay in L2 while the vocabulary matrix streams through once
    const int64_t per = (int64_t)kRaster * q.nt;
    const int g = (int)(i / per);
    const int r = (int)(i - g * per);
    const int gm = min(kRaster, q.mt - g * kRaster);
    t.job = 0;
    t.m0 = (g * kRaster + r % gm) * kPairM;
    t.n0 = r / gm * kPairN;
    t.kb = q.kb;
    return true;
  }
  if (s < q.own_dh) {
    const int i = q.p + s * q.np;
    t.job = 0;
    t.m0 = i / q.dt * kPairM;
    t.n0 = i % q.dt * kPairN;
    t.kb = q.kb_dh;
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
  t.m0 = j / q.dt * kPairM;
  t.n0 = j % q.dt * kPairN;
  t.kb = q.kb_dw;
  return true;
}

// 16 bits of 32 consecutive columns of a row to memory, those below `cols`.
__device__ __forceinline__ void store16(uint16_t* dst, const float (&x)[32], int cols, bool vec, int f16, bool add) {
  if (vec && cols >= 32) {
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
      uint4* p = reinterpret_cast<uint4*>(dst + c);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[c + i];
      if (add) {
        const uint4 o = *p;
        const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[2 * i] += widen16((uint16_t)(w[i] & 0xFFFFu), f16);
          y[2 * i + 1] += widen16((uint16_t)(w[i] >> 16), f16);
        }
      }
      *p = make_uint4(pack16(y[0], y[1], f16), pack16(y[2], y[3], f16), pack16(y[4], y[5], f16), pack16(y[6], y[7], f16));
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < 32; ++c)
    if (c < cols) dst[c] = round16(add ? x[c] + widen16(dst[c], f16) : x[c], f16);
}

template <int kMode>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kVThreads, 1)
    vocab_pair_kernel(const __grid_constant__ VocabMaps maps, VocabArgs a, Status st) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  VocabCtl* ctl = reinterpret_cast<VocabCtl*>(smem_raw);
  const uint32_t sbase = smem_u32(smem_raw);
  constexpr uint32_t kCtlBytes = (sizeof(VocabCtl) + 15) & ~15u;
  const uint32_t tiles = (sbase + kCtlBytes + 1023u) & ~1023u;  // the same offset in both CTAs
  constexpr bool kLogits = kMode == kLse || kMode == kLseEnt;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int rows = a.idx ? a.head->rows : (int)a.T;
  const Plan plan = make_plan<kMode>(a, rows);
  const CUtensorMap* hmap = a.idx && rows < a.T ? &maps.hc : &maps.h;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kVStages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->tfull[b], 1);
      mbar_init(&ctl->tempty[b], 2 * kVEpiWarps);
    }
    mbar_init(&ctl->drain, 1);
    fence_mbar_init();
  }
  if (warp == 2) {
    tmem_alloc_pair(&ctl->tmem_base, kVCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;

  if (warp == 0) {
    // ------------------------------------------------------------ loads (lane 0 of either CTA: its halves)
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      Tile t;
      for (int s = 0; ok && next_tile<kMode>(plan, s, t); ++s) {
        const CUtensorMap* ma = kMode == kProducts ? &maps.dz : hmap;
        const CUtensorMap* mb = kMode == kProducts && t.job == 1 ? hmap : &maps.w;
        const bool a_mn = kMode == kProducts && t.job == 1, b_mn = kMode == kProducts;
        const int am = t.m0 + (int)rank * (kPairM / 2), bn = t.n0 + (int)rank * (kPairN / 2);
        const int v0 = kLogits ? 0 : (int)a.v0;
        for (int k = 0; k < t.kb; ++k) {
          if (!mbar_wait(&ctl->empty[stage], phase ^ 1u, st, 20)) {
            ok = false;
            break;
          }
          const uint32_t sa = tiles + (uint32_t)stage * kVStage, sb = sa + 2 * kVBox;
          const uint32_t bar = leader_addr(&ctl->full[stage]);
          if (rank == 0) mbar_arrive_expect_tx(&ctl->full[stage], 2 * kVStage);
          ++issued;
          const int kx = k * kTile16;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (a_mn) tma_load_2d_pair(sa + h * kVBox, ma, bar, am + h * kTile16, kx);
            else tma_load_2d_pair(sa + h * kVBox, ma, bar, kx, am + h * kTile16);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!b_mn) tma_load_2d_pair(sb + h * kVBox, mb, bar, kx, v0 + bn + h * kTile16);
            else tma_load_2d_pair(sb + h * kVBox, mb, bar, bn + h * kTile16, (t.job == 0 ? v0 : 0) + kx);
          }
          if (++stage == kVStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      // wind-down: the copies land before the CTAs may exit
      if (rank == 0)
        for (uint32_t s = 0; s < kVStages; ++s)
          if (s < issued) mbar_wait(&ctl->full[s], (issued - 1 - s) / kVStages & 1u, st, 21, 200000000ull, false);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs (lane 0 of the leader)
    if (lane == 0 && rank == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      if (a.debug_timeout) {
        mbar_wait(&ctl->drain, 0, st, 27, kDebugTimeoutNs);  // returns false: reports GPO_ERR_TIMEOUT
        ok = false;
      }
      Tile t;
      int sum = 0;  // accumulations so far: one per tile, or per segment of a logits tile
      for (int s = 0; ok && next_tile<kMode>(plan, s, t); ++s) {
        const bool a_mn = kMode == kProducts && t.job == 1, b_mn = kMode == kProducts;
        const uint32_t idesc = idesc_16_f32(kPairM, kPairN, a.f16 != 0, a_mn, b_mn);
        for (int k0 = 0; ok && (k0 < t.kb || k0 == 0); k0 += kMode == kProducts ? t.kb + 1 : kSegment, ++sum) {
        const int buf = sum & 1;
        if (!mbar_wait_cluster(&ctl->tempty[buf], ((uint32_t)(sum >> 1) & 1u) ^ 1u, st, 22)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t dt = tmem + (uint32_t)(buf * kPairN);
        const int k1 = kMode == kProducts ? t.kb : min(t.kb, k0 + kSegment);
        for (int k = k0; k < k1; ++k) {
          if (!mbar_wait(&ctl->full[stage], phase, st, 23)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sa = tiles + (uint32_t)stage * kVStage, sb = sa + 2 * kVBox;
          const uint64_t ad = a_mn ? smem_desc_mn128(sa, kVBox) : smem_desc_k128(sa);
          const uint64_t bd = b_mn ? smem_desc_mn128(sb, kVBox) : smem_desc_k128(sb);
          // 16 k: 32 bytes of a K-major row, 16 rows of 128 bytes otherwise (addresses >> 4)
          const uint32_t as = a_mn ? 128u : 2u, bs = b_mn ? 128u : 2u;
#pragma unroll
          for (uint32_t kk = 0; kk < kTile16 / 16; ++kk)
            mma_f16_pair(dt, ad + as * kk, bd + bs * kk, idesc, ((k - k0) | (int)kk) != 0);
          mma_commit_pair(&ctl->empty[stage]);
          if (++stage == kVStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (ok) mma_commit_pair(&ctl->tfull[buf]);
        }
      }
      // wind-down: all issued MMAs complete before tensor memory is released
      mma_commit_pair(&ctl->drain);
      mbar_wait(&ctl->drain, 0, st, 24, 200000000ull, false);
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ------------------------------------------------------------ epilogue
    const int q = warp & 3, half = (warp - 4) >> 2;  // tensor memory lanes 32 q .., columns 128 half ..
    const int r = (int)rank * (kPairM / 2) + q * 32 + lane;  // row in the tile
    const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * (kPairN / 2));
    const uint32_t te = leader_addr(&ctl->tempty[0]);
    // waits for the n-th accumulation; false (for the whole warp) when that gave up
    auto ready = [&](int n) {
      const bool got = __all_sync(0xffffffffu, mbar_wait(&ctl->tfull[n & 1], (uint32_t)(n >> 1) & 1u, st, 25));
      tc_fence_after();
      return got;
    };
    // this warp has read its part of the n-th accumulation
    auto release = [&](int n) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(te + 8u * (uint32_t)(n & 1));
    };
    Tile t;
    int sum = 0;
    for (int s = 0; next_tile<kMode>(plan, s, t); ++s) {
      const int row = t.m0 + r;
      const int n0 = t.n0 + half * (kPairN / 2);  // first column of this warp
      if constexpr (kMode != kProducts) {
        const bool live = row < rows;
        // what the row's token brings
        int64_t tok = 0;
        int tgt = -1;
        float l2 = 0.f, g = 0.f, e = 0.f, ent = 0.f;
        if (live) {
          tok = a.idx ? a.idx[row] : row;
          const int64_t id = load_id(a.target, a.id8, tok);
          if (id >= 0 && id < a.V) tgt = (int)(id - (kLogits ? 0 : a.v0)) - n0;  // its column, from n0 on
          if (!kLogits) {
            const float gs = a.head->dz_scale;
            l2 = a.lse[tok] * 1.4426950408889634f;
            g = a.g[tok] * gs;
            if (kMode == kDzEnt) {
              e = a.ge[tok] * gs;
              ent = a.ent[tok];
            }
          }
        }
        float z[kPairN / 2];
        bool ok = true;
        for (int k0 = 0; k0 < t.kb; k0 += kSegment, ++sum) {
          ok = ready(sum);
          if (!ok) break;
          const uint32_t src = lanes + (uint32_t)((sum & 1) * kPairN);
#pragma unroll
          for (int c = 0; c < kPairN / 2; c += 16) {
            uint32_t x[16];
            tmem_ld_32x32b_x16(src + (uint32_t)c, x);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) z[c + j] = k0 == 0 ? __uint_as_float(x[j]) : z[c + j] + __uint_as_float(x[j]);
          }
          release(sum);
        }
        if (!ok) break;
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
            if (kMode == kLseEnt) u4[j & 3] = fmaf(p, d, u4[j & 3]);
          }
          if (live) {
            const int64_t at = (int64_t)row * a.part_row + (int64_t)(n0 / (kPairN / 2)) * a.part_col;
            a.pm[at] = m;
            a.ps[at] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            if (kMode == kLseEnt) a.pu[at] = (u4[0] + u4[1]) + (u4[2] + u4[3]);
          }
        } else {
          uint4* dst = reinterpret_cast<uint4*>(a.dz + (int64_t)row * a.dz_stride + n0);
          const int cols = live ? (int)a.vn - n0 : 0;
#pragma unroll
          for (int c = 0; c < kPairN / 2; c += 8) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int j = c + i;
              const float d = fmaf(z[j], a.sl2, -l2);  // log2 p
              const float p = ex2(d);
              float v = (j == tgt ? g : 0.f) - g * p;
              if (kMode == kDzEnt) v = fmaf(-e * p, fmaf(d, 0.6931471805599453f, ent), v);
              // (p of a padding row or column is no probability, and its row may hold anything)
              y[i] = j < cols ? v : 0.f;
            }
            dst[c / 8] = make_uint4(pack16(y[0], y[1], a.f16), pack16(y[2], y[3], a.f16), pack16(y[4], y[5], a.f16),
                                    pack16(y[6], y[7], a.f16));
          }
        }
      } else {
        const bool live = row < (t.job == 1 ? (int)a.vn : rows);
        if (!ready(sum)) break;
        const float f = t.kb > 0 ? a.scale / a.head->dz_scale : 0.f;
#pragma unroll 1
        for (int ch = 0; ch < kPairN / 2 / 32; ++ch) {
          uint32_t x[32];
          __syncwarp();
          tmem_ld_32x32b_x32(lanes + (uint32_t)((sum & 1) * kPairN + ch * 32), x);
          tmem_wait_ld();
          if (ch == kPairN / 2 / 32 - 1) release(sum);
          const int c0 = n0 + ch * 32;
          float y[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) y[j] = t.kb > 0 ? __uint_as_float(x[j]) * f : 0.f;  // (no tokens: no product ran)
          const int cols = a.D - c0;
          if (live && cols > 0 && t.job == 0) {
            if (!(a.first && a.last)) {  // several pieces: sums so far in fp32
              float4* acc = reinterpret_cast<float4*>(a.acc + (int64_t)row * a.acc_stride + c0);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                if (4 * i < cols) {
                  if (!a.first) {
                    const float4 o = acc[i];
                    y[4 * i] += o.x;
                    y[4 * i + 1] += o.y;
                    y[4 * i + 2] += o.z;
                    y[4 * i + 3] += o.w;
                  }
                  if (!a.last) acc[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                }
              }
            }
            if (a.last) {
              uint16_t* dst = static_cast<uint16_t*>(a.dh) + (int64_t)a.idx[row] * a.dh_stride + c0;
              store16(dst, y, cols, ((a.dh_stride & 7) | (reinterpret_cast<uintptr_t>(a.dh) & 15)) == 0, a.f16, false);
            }
          } else if (live && cols > 0) {
            uint16_t* dst = static_cast<uint16_t*>(a.dw) + (a.v0 + row) * a.dw_stride + c0;
            store16(dst, y, cols, ((a.dw_stride & 7) | (reinterpret_cast<uintptr_t>(a.dw) & 15)) == 0, a.f16,
                    a.accumulate != 0);
          }
        }
        ++sum;
      }
    }
  }

  // after a timeout: every copy that either CTA issued lands before the shared memory goes
  if (threadIdx.x == 0 && aborted(st)) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 1000000ull) __nanosleep(1000);
  }
  if (kMode == kProducts && a.last && blockIdx.x == 0 && threadIdx.x == 0) sign_status(st);
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  if (warp == 2) tmem_dealloc_pair(tmem, kVCols);
}

// ------------------------------------------------------------------ tokens that take part

__device__ __forceinline__ bool takes_part(const VocabArgs& a, int64_t t, bool grad) {
  const int64_t id = load_id(a.target, a.id8, t);
  if (id < 0 || id >= a.V) return false;
  return !grad || a.g[t] != 0.f || (a.ge && a.ge[t] != 0.f);
}

constexpr int kIndexThreads = 1024;

// One CTA: the list of the tokens that take part, in order, their number, the forward outputs of
// the others and the scale of an fp16 dz.
template <bool kGrad>
__global__ void __launch_bounds__(kIndexThreads) vocab_index_kernel(VocabArgs a, Status st) {
  __shared__ int cnt[kIndexThreads / 32];
  __shared__ float big[kIndexThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int base = 0;
  float bound = 0.f;  // of |dz|: |g| + |e| max p |log p + H|, whose last factor is below log V + 1
  for (int64_t t0 = 0; t0 < a.T; t0 += kIndexThreads) {
    const int64_t t = t0 + threadIdx.x;
    bool in = false;
    if (t < a.T) {
      const int64_t id = load_id(a.target, a.id8, t);
      if (id >= a.V) report(st, GPO_ERR_SHAPE, 26, (int)t);
      in = takes_part(a, t, kGrad);
      if (kGrad && in) bound = fmaxf(bound, fabsf(a.g[t]) + (a.ge ? 24.f * fabsf(a.ge[t]) : 0.f));
      if (!kGrad && !in) {
        a.logp[t] = 0.f;
        if (a.lse_out) a.lse_out[t] = 0.f;
        if (a.ent_out) a.ent_out[t] = 0.f;
      }
    }
    const uint32_t m = __ballot_sync(0xffffffffu, in);
    if (lane == 0) cnt[warp] = __popc(m);
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kIndexThreads / 32; ++w) {
      if (w < warp) before += cnt[w];
      all += cnt[w];
    }
    if (in) a.idx[base + before + __popc(m & ((1u << lane) - 1u))] = (int)t;
    base += all;
    __syncthreads();
  }
  if (kGrad && a.f16) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) bound = fmaxf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
    if (lane == 0) big[warp] = bound;
    __syncthreads();
    for (int w = 0; w < kIndexThreads / 32; ++w) bound = fmaxf(bound, big[w]);
  }
  if (threadIdx.x == 0) {
    float s = 1.f;
    if (kGrad && a.f16 && bound > 0.f && isfinite(bound)) {
      int ex;
      frexpf(bound, &ex);  // bound <= 2^ex: |dz| up to 2^14, within fp16's 65504
      s = ldexpf(1.f, min(max(14 - ex, -100), 100));
    }
    a.head->rows = base;
    a.head->dz_scale = s;
  }
}

// Copies the listed rows together (where some token is left out), zeros up to the next k-step of the
// d_weight product, and zeros the d_hidden rows of the others.
template <bool kGrad>
__global__ void __launch_bounds__(256) vocab_gather_kernel(VocabArgs a) {
  const int rows = a.head->rows;
  const bool gather = rows < a.T;
  const int64_t pad = ((int64_t)rows + kTile16 - 1) / kTile16 * kTile16;
  const int chunks = (a.D + 7) / 8;  // 16 bytes each (rows hold a multiple of them)
  for (int64_t r = blockIdx.x; r < max(pad, a.T); r += gridDim.x) {
    if (gather && r < pad) {
      uint4* dst = reinterpret_cast<uint4*>(a.hc + r * a.hc_stride);
      if (r < rows) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.hidden) + (int64_t)a.idx[r] * a.hidden_stride);
        for (int c = threadIdx.x; c < chunks; c += blockDim.x) dst[c] = src[c];
      } else {
        for (int c = threadIdx.x; c < chunks; c += blockDim.x) dst[c] = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    if (kGrad && a.dh && r < a.T && !takes_part(a, r, true)) {
      uint16_t* dst = static_cast<uint16_t*>(a.dh) + r * a.dh_stride;
      for (int c = threadIdx.x; c < a.D; c += blockDim.x) dst[c] = 0;
    }
  }
}

// ------------------------------------------------------------------ joining the parts of a row

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

constexpr int kJoinThreads = 256;

// Parts of a row side by side: a CTA per row (few tokens).
template <bool kEnt>
__global__ void __launch_bounds__(kJoinThreads) vocab_join_row_kernel(VocabArgs a, int parts, Status st) {
  __shared__ Part red[kJoinThreads / 32];
  const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t id = load_id(a.target, a.id8, row);
  if (row == 0 && threadIdx.x == 0) sign_status(st);
  if (id < 0 || id >= a.V) {
    if (threadIdx.x == 0) {
      if (id >= a.V) report(st, GPO_ERR_SHAPE, 26, row);
      a.logp[row] = 0.f;
      if (a.lse_out) a.lse_out[row] = 0.f;
      if (kEnt) a.ent_out[row] = 0.f;
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
    finish<kEnt>(a, row, a.tz[row], p);
  }
}

// Rows side by side: a CTA takes 32 rows, its warps the parts in turn.
template <bool kEnt>
__global__ void __launch_bounds__(1024) vocab_join_kernel(VocabArgs a, int parts, Status st) {
  __shared__ Part red[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x * 32 + lane, rows = a.head->rows;
  if (blockIdx.x == 0 && threadIdx.x == 0) sign_status(st);
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
    for (int w = 1; w < 32; ++w) p = join<kEnt>(p, red[w][lane]);
    finish<kEnt>(a, a.idx[row], a.tz[row], p);
  }
}

int g_pairs = 0;  // CTA pairs resident at one time

template <int kMode>
cudaError_t setup_mode() {
  return cudaFuncSetAttribute(vocab_pair_kernel<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kVSmem);
}

template <int kMode>
cudaError_t launch_pair(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st, int64_t tiles) {
  const int64_t pairs = min((int64_t)g_pairs, max(tiles, (int64_t)1));
  vocab_pair_kernel<kMode><<<(unsigned)(2 * pairs), kVThreads, kVSmem, lc.stream>>>(m, a, st);
  return cudaGetLastError();
}

int64_t tiles_of(int64_t rows, int64_t cols) { return ((rows + kPairM - 1) / kPairM) * ((cols + kPairN - 1) / kPairN); }

}  // namespace

cudaError_t setup_vocab() {
  cudaError_t e = setup_mode<kLse>();
  if (e == cudaSuccess) e = setup_mode<kLseEnt>();
  if (e == cudaSuccess) e = setup_mode<kDz>();
  if (e == cudaSuccess) e = setup_mode<kDzEnt>();
  if (e == cudaSuccess) e = setup_mode<kProducts>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kVThreads);
  cfg.dynamicSmemBytes = kVSmem;
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

cudaError_t launch_vocab_rows(const LaunchCtx& lc, const VocabArgs& a, const Status& st, bool grad) {
  if (grad) vocab_index_kernel<true><<<1, kIndexThreads, 0, lc.stream>>>(a, st);
  else vocab_index_kernel<false><<<1, kIndexThreads, 0, lc.stream>>>(a, st);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int grid = (int)min(a.T, (int64_t)lc.num_sms * 8);
  if (grad) vocab_gather_kernel<true><<<grid, 256, 0, lc.stream>>>(a);
  else vocab_gather_kernel<false><<<grid, 256, 0, lc.stream>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_vocab_lse(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st, bool ent) {
  return ent ? launch_pair<kLseEnt>(lc, m, a, st, tiles_of(a.T, a.V)) : launch_pair<kLse>(lc, m, a, st, tiles_of(a.T, a.V));
}

cudaError_t launch_vocab_join(const LaunchCtx& lc, const VocabArgs& a, const Status& st, bool ent) {
  const int parts = (int)vocab_parts(a.V);
  if (!a.idx) {
    if (ent) vocab_join_row_kernel<true><<<(unsigned)a.T, kJoinThreads, 0, lc.stream>>>(a, parts, st);
    else vocab_join_row_kernel<false><<<(unsigned)a.T, kJoinThreads, 0, lc.stream>>>(a, parts, st);
  } else {
    const unsigned grid = (unsigned)((a.T + 31) / 32);
    if (ent) vocab_join_kernel<true><<<grid, 1024, 0, lc.stream>>>(a, parts, st);
    else vocab_join_kernel<false><<<grid, 1024, 0, lc.stream>>>(a, parts, st);
  }
  return cudaGetLastError();
}

cudaError_t launch_vocab_dz(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st) {
  return a.ge ? launch_pair<kDzEnt>(lc, m, a, st, tiles_of(a.T, a.vn)) : launch_pair<kDz>(lc, m, a, st, tiles_of(a.T, a.vn));
}

cudaError_t launch_vocab_products(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st) {
  return launch_pair<kProducts>(lc, m, a, st, (a.dh ? tiles_of(a.T, a.D) : 0) + (a.dw ? tiles_of(a.vn, a.D) : 0));
}

}  // namespace gpo
