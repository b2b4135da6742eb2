// Log-probabilities of up to 16 tokens (decoding) in one launch.
//
// With few tokens every weight is read once and the products are cheap, so the roles are turned
// round: 128 vocabulary rows at a time are the tensor cores' A operand, the tokens (16 columns) the B operand,
// which costs an MMA of few columns and little tensor memory to read.  A CTA
// per SM streams an equal share of the vocabulary, in units of 32 rows, through a ring of TMA boxes; a
// lane owns a vocabulary row and keeps the running maximum and sum of every token over its
// rows in registers, with no exchange until the end.  Then the CTA joins its 128 lanes, and the CTA that
// finds every other's mark joins the CTAs' parts: no second launch, no counter to reset.  (The marks are the
// call's own: a mark left by another call is none.  Every CTA publishes its part, fences, and
// then looks: whichever comes last sees all marks.  Two that both see them write the same results.)
// The accumulators are taken over into registers every 128 products (see gpo_vocab.cu).
// Bound by HBM: one token, 131072 x 4096, 1.074 GB read in 178 us, 6.0 TB/s; below some 30 MB by the chain of launch,
// first loads and join: 7 tokens, 1009 x 256, 10 us.
#define GPO_REPORT __noinline__
#include "gpo_vocab_math.cuh"

namespace gpo {

namespace {

constexpr int kFewThreads = 384;      // warps: 0 loads, 1 MMAs, 2 tensor memory, 4..11 epilogue
constexpr int kFewEpi = 256;          // epilogue threads
constexpr int kFewBar = 1;            // their named barrier
constexpr int kFewUnit = 32;          // vocabulary rows of one TMA box
constexpr int kFewTile = 128;
constexpr int kFewStages = 12;        // at most
constexpr int kFewRing = 200 * 1024;  // bytes
constexpr int kFewBufs = 4;           // accumulators of kN columns

struct __align__(8) FewCtl {
  uint64_t full[kFewStages];
  uint64_t empty[kFewStages];
  uint64_t tfull[kFewBufs];
  uint64_t tempty[kFewBufs];
  uint64_t drain;
  uint32_t tmem_base;
  int target[kVocabFew];
};
constexpr size_t kFewSmem = ((sizeof(FewCtl) + 15) & ~size_t(15)) + 1023 + kFewRing;

template <int kRegs>
__device__ __forceinline__ void tmem_ld(uint32_t addr, uint32_t (&r)[kRegs]) {
  static_assert(kRegs == 8, "columns of one load");
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(addr));
}

__device__ __forceinline__ bool few_any(bool flag) {
  uint32_t out;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(out)
      : "r"((uint32_t)flag), "n"(kFewBar), "n"(kFewEpi)
      : "memory");
  return out != 0;
}

template <bool kEnt>
__global__ void __launch_bounds__(kFewThreads, 1)
    vocab_few_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap tmap,
                     const __grid_constant__ CUtensorMap hmap, VocabArgs a, Status st, uint64_t* marks, uint64_t mark) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  FewCtl* ctl = reinterpret_cast<FewCtl*>(smem_raw);
  const uint32_t sbase = smem_u32(smem_raw);
  constexpr uint32_t kCtl = (sizeof(FewCtl) + 15) & ~15u;
  const uint32_t ring_off = ((sbase + kCtl + 1023u) & ~1023u) - sbase;
  unsigned char* ring = smem_raw + ring_off;
  constexpr int kN = kVocabFew, kA = kFewTile * 128, kB = kN * 128, kStage = kA + kB;
  constexpr int kStages = kFewRing / kStage < kFewStages ? kFewRing / kStage : kFewStages;
  constexpr int kCols = kN / 2;  // tokens of one epilogue thread
  constexpr uint32_t kTmem = kFewBufs * kN;
  static_assert(kTmem == 64 && kFewEpi % kN == 0, "tensor memory columns, threads of a token");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)blockIdx.x, nctas = (int)gridDim.x;
  const int64_t units = (a.V + kFewUnit - 1) / kFewUnit;
  const int u0 = (int)(units * cta / nctas), u1 = (int)(units * (cta + 1) / nctas);
  const int kb = (a.D + 63) / 64;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < kFewBufs; ++b) {
      mbar_init(&ctl->tfull[b], 1);
      mbar_init(&ctl->tempty[b], kFewEpi / 32);
    }
    mbar_init(&ctl->drain, 1);
    fence_mbar_init();
  }
  if (warp == 2) {
    tmem_alloc(&ctl->tmem_base, kTmem);
    tmem_relinquish();
  }
  if (threadIdx.x < kVocabFew) {
    int tgt = -1;
    if (threadIdx.x < a.T) {
      const int64_t id = load_id(a.target, a.id8, threadIdx.x);
      if (id >= a.V && cta == 0) report(st, GPO_ERR_SHAPE, 40, (int)threadIdx.x);
      if (id >= 0 && id < a.V) tgt = (int)id;
    }
    ctl->target[threadIdx.x] = tgt;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;

  if (warp == 0) {
    // ------------------------------------------------------------ loads (lane 0)
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int u = u0; ok && u < u1; u += kFewTile / kFewUnit) {
        const int boxes = min(kFewTile / kFewUnit, u1 - u);
        for (int k = 0; k < kb; ++k) {
          if (!mbar_wait(&ctl->empty[stage], phase ^ 1u, st, 41)) {
            ok = false;
            break;
          }
          unsigned char* sa = ring + stage * kStage;
          mbar_arrive_expect_tx(&ctl->full[stage], (uint32_t)(boxes * kFewUnit * 128 + kB));
          ++issued;
          // (a whole tile in one box: in four, one token of 131072 x 4096 took 184 us in place of 181)
          if (boxes == kFewTile / kFewUnit) tma_load_2d(sa, &tmap, &ctl->full[stage], k * 64, u * kFewUnit);
          else
            for (int b = 0; b < boxes; ++b)
              tma_load_2d(sa + b * kFewUnit * 128, &wmap, &ctl->full[stage], k * 64, (u + b) * kFewUnit);
          tma_load_2d(sa + kA, &hmap, &ctl->full[stage], k * 64, 0);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      // wind-down: every issued copy must land before the CTA may exit
      for (uint32_t s = 0; s < kStages; ++s)
        if (s < issued) mbar_wait(&ctl->full[s], (issued - 1 - s) / kStages & 1u, st, 42, 200000000ull, false);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs (lane 0)
    if (lane == 0) {
      int stage = 0, sum = 0;
      uint32_t phase = 0;
      bool ok = true;
      if (a.debug_timeout) {
        mbar_wait(&ctl->drain, 0, st, 47, kDebugTimeoutNs);  // returns false: reports GPO_ERR_TIMEOUT
        ok = false;
      }
      const uint32_t idesc = (1u << 4) | (a.f16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(kN >> 3) << 17) |
                             ((uint32_t)(kFewTile >> 4) << 24);
      for (int u = u0; ok && u < u1; u += kFewTile / kFewUnit) {
        for (int k0 = 0; ok && k0 < kb; k0 += kVocabFewSeg, ++sum) {
          const int buf = sum % kFewBufs;
          if (!mbar_wait(&ctl->tempty[buf], ((uint32_t)(sum / kFewBufs) & 1u) ^ 1u, st, 43)) {
            ok = false;
            break;
          }
          tc_fence_after();
          for (int k = k0; k < min(kb, k0 + kVocabFewSeg); ++k) {
            if (!mbar_wait(&ctl->full[stage], phase, st, 44)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t sa = smem_u32(ring + stage * kStage);
            const uint64_t ad = smem_desc_k128(sa), bd = smem_desc_k128(sa + kA);
#pragma unroll
            for (uint32_t kk = 0; kk < 4; ++kk)
              mma_bf16_ss(tmem + (uint32_t)(buf * kN), ad + 2u * kk, bd + 2u * kk, idesc, (k - k0 | (int)kk) != 0);
            mma_commit(&ctl->empty[stage]);
            if (++stage == kStages) {
              stage = 0;
              phase ^= 1u;
            }
          }
          if (ok) mma_commit(&ctl->tfull[buf]);
        }
      }
      mma_commit(&ctl->drain);  // wind-down: all issued MMAs complete before tensor memory is released
      mbar_wait(&ctl->drain, 0, st, 45, 200000000ull, false);
    }
    __syncwarp();
  } else if (warp == 3) {
    if (lane == 0 && cta == 0) next_tag(st);
    __syncwarp();
  } else if (warp >= 4) {
    // ------------------------------------------------------------ epilogue
    const int q = warp & 3, half = (warp - 4) >> 2, te = threadIdx.x - 128;
    const uint32_t src = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * kCols);
    float m[kCols], s[kCols], w[kEnt ? kCols : 1];
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      m[j] = kLow;
      s[j] = 0.f;
      if (kEnt) w[j] = 0.f;
    }
    bool ok = true;
    int sum = 0;
    for (int u = u0; ok && u < u1; u += kFewTile / kFewUnit) {
      float z[kCols];
#pragma unroll
      for (int j = 0; j < kCols; ++j) z[j] = 0.f;
      for (int k0 = 0; k0 < kb; k0 += kVocabFewSeg, ++sum) {
        const int buf = sum % kFewBufs;
        ok = __all_sync(0xffffffffu, mbar_wait(&ctl->tfull[buf], (uint32_t)(sum / kFewBufs) & 1u, st, 46));
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < kCols; c += 8) {
          uint32_t x[8];
          tmem_ld(src + (uint32_t)(buf * kN + c), x);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 8; ++j) z[c + j] += __uint_as_float(x[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl->tempty[buf]);
      }
      if (!ok) break;
      const int64_t v = (int64_t)(u + q) * kFewUnit + lane;
      if (u + q < u1 && v < a.V) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          const float x = z[j] * a.sl2;
          if (ctl->target[half * kCols + j] == (int)v) {
            a.tz[half * kCols + j] = x;  // the target's logit stays out of the sums
          } else {
            const float d = x - m[j], e = ex2(-fabsf(d));
            if (kEnt) w[j] = d > 0.f ? e * (w[j] - d * s[j]) : fmaf(e, d, w[j]);
            s[j] = d > 0.f ? fmaf(s[j], e, 1.f) : s[j] + e;
            m[j] = fmaxf(m[j], x);
          }
        }
      }
    }
    // the CTA's part of every token: the 128 lanes' through shared memory (the ring is free: every
    // accumulation is done), kPer threads a token
    if (!few_any(!ok)) {
      constexpr int kRow = kFewTile + 1, kPer = kFewEpi / kN;
      float* red = reinterpret_cast<float*>(ring);
#pragma unroll
      for (int j = 0; j < kCols; ++j) {
        const int at = (half * kCols + j) * kRow + q * 32 + lane;
        red[at] = m[j];
        red[kN * kRow + at] = s[j];
        if (kEnt) red[2 * kN * kRow + at] = w[j];
      }
      few_any(false);
      const int tok = te / kPer, part = te % kPer;
      Part p = {kLow, 0.f, 0.f};
      const float* mine = red + tok * kRow + part;
      for (int i = 0; i < kFewTile; i += kPer) p.m = fmaxf(p.m, mine[i]);
      for (int i = 0; i < kFewTile; i += kPer) {
        const float d = mine[i] - p.m, e = ex2(d), si = mine[kN * kRow + i];
        p.s = fmaf(e, si, p.s);
        if (kEnt) p.u = fmaf(e, fmaf(d, si, mine[2 * kN * kRow + i]), p.u);
      }
#pragma unroll
      for (int o = 1; o < kPer; o <<= 1) {
        const Part y = {__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                        __shfl_xor_sync(0xffffffffu, p.u, o)};
        p = join<kEnt>(p, y);
      }
      if (part == 0) {
        const int at = cta * kVocabFew + tok;
        a.pm[at] = p.m;
        a.ps[at] = p.s;
        if (kEnt) a.pu[at] = p.u;
      }
      few_any(false);
      if (te == 0) {
        __threadfence();
        asm volatile("st.release.gpu.global.b64 [%0], %1;" ::"l"(marks + cta), "l"(mark) : "memory");
      }
      few_any(false);
      asm volatile("fence.sc.gpu;" ::: "memory");
      bool missing = false;
      for (int i = te; i < nctas; i += kFewEpi) {
        uint64_t x;
        asm volatile("ld.acquire.gpu.global.b64 %0, [%1];" : "=l"(x) : "l"(marks + i) : "memory");
        missing |= x != mark;
      }
      if (!few_any(missing)) {
        for (int t = te >> 5; t < a.T; t += kFewEpi / 32) {
          Part p = {kLow, 0.f, 0.f};
          for (int i = lane; i < nctas; i += 32) {
            const int at = i * kVocabFew + t;
            p = join<kEnt>(p, Part{__ldcg(a.pm + at), __ldcg(a.ps + at), kEnt ? __ldcg(a.pu + at) : 0.f});
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            const Part y = {__shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
                            __shfl_xor_sync(0xffffffffu, p.u, o)};
            p = join<kEnt>(p, y);
          }
          if (lane == 0) {
            if (ctl->target[t] >= 0) {
              finish<kEnt>(a, t, __ldcg(a.tz + t), p);
            } else {
              a.logp[t] = 0.f;
              if (a.lse_out) a.lse_out[t] = 0.f;
              if (kEnt) a.ent_out[t] = 0.f;
            }
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_dealloc(tmem, kTmem);
}

}  // namespace

cudaError_t setup_vocab_few() {
  cudaError_t e = cudaFuncSetAttribute(vocab_few_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(vocab_few_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem);
}

cudaError_t launch_vocab_few(const LaunchCtx& lc, const VocabMaps& m, const VocabArgs& a, const Status& st, bool ent,
                             uint64_t* marks, uint64_t mark) {
  const int64_t units = (a.V + kFewUnit - 1) / kFewUnit;
  const unsigned grid = (unsigned)min(units, (int64_t)min(lc.num_sms, kVocabFewCtas));
  if (ent) vocab_few_kernel<true><<<grid, kFewThreads, kFewSmem, lc.stream>>>(m.w, m.wb, m.h, a, st, marks, mark);
  else vocab_few_kernel<false><<<grid, kFewThreads, kFewSmem, lc.stream>>>(m.w, m.wb, m.h, a, st, marks, mark);
  return cudaGetLastError();
}

}  // namespace gpo
