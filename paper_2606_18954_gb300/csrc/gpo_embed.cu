// Token embedding and the gradient of its table (formulas in include/graphpo.h).
//
//   embed      embed_kernel: a warp per token and 4 KB of its row, 16-byte accesses, eight in flight per
//              lane.  32768 tokens of 4096 values (16 bits) out of 131072 rows 73 us, 126 MB read and
//              210 written to HBM, 4.6 TB/s: DRAM is busy 58 % of the time, so it is not what bounds it (the reads of
//              scattered rows and their writes in one warp, most likely: the sums below reach 6.2)
//   gradient   embed_sort_kernel: the tokens in the order of their ids (gpo_sort.cuh): 17 us for 32768
//              embed_sum_kernel: the sorted tokens in pieces of equal length, a warp per piece and
//              512 bytes of the rows: runs of one id are summed in order in fp32, a run inside the
//              piece is a finished row, a run that the piece's ends cut leaves its sum in the
//              workspace.  So the work does not depend on how often a token occurs.  Rows
//              without tokens are zeroed by the same launch.  Bound by HBM: 32768 tokens of 4096 values into
//              131072 rows 206 us, 269 MB read and 1016 written, 6.2 TB/s
//              embed_join_kernel: the sums of cut runs, added in order: 15 us there
// Every sum has a fixed order: the results are the same on every run.
#define GPO_REPORT __noinline__
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gpo_internal.cuh"
#include "gpo_sort.cuh"

namespace gpo {

namespace {

template <int kType>
struct Elem;
template <>
struct Elem<GPO_DT_F32> {
  using T = float;
  static constexpr int kPer = 4;  // per 16 bytes
  static __device__ __forceinline__ float get(T x) { return x; }
  static __device__ __forceinline__ T put(float x) { return x; }
};
template <>
struct Elem<GPO_DT_BF16> {
  using T = __nv_bfloat16;
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float get(T x) { return __bfloat162float(x); }
  static __device__ __forceinline__ T put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Elem<GPO_DT_F16> {
  using T = __half;
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float get(T x) { return __half2float(x); }
  static __device__ __forceinline__ T put(float x) { return __float2half_rn(x); }
};

__device__ __forceinline__ int64_t id_of(const void* ids, int id8, int64_t t) {
  return id8 ? static_cast<const int64_t*>(ids)[t] : (int64_t)static_cast<const int32_t*>(ids)[t];
}

// A lane's kPer columns of a block of 32 kPer: with 16-byte accesses (kVec) side by side, else 32 apart.
template <int kType, bool kVec>
struct Cols {
  using E = Elem<kType>;
  using T = typename E::T;
  static constexpr int kPer = E::kPer;
  static __device__ __forceinline__ int64_t at(int64_t block, int lane, int i) {
    return block * 32 * kPer + (kVec ? lane * kPer + i : i * 32 + lane);
  }
  struct Raw {
    uint4 v;
  };
  // (a row's last block may end inside a lane's 16 bytes: those columns one by one)
  static __device__ __forceinline__ Raw load(const T* row, int64_t block, int lane, int64_t d) {
    Raw r;
    r.v = make_uint4(0u, 0u, 0u, 0u);
    if (kVec && at(block, lane, kPer) <= d) {
      r.v = __ldg(reinterpret_cast<const uint4*>(row + at(block, lane, 0)));
    } else {
      T* e = reinterpret_cast<T*>(&r.v);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (at(block, lane, i) < d) e[i] = row[at(block, lane, i)];
    }
    return r;
  }
  static __device__ __forceinline__ void add(const Raw& r, float (&s)[kPer]) {
    const T* e = reinterpret_cast<const T*>(&r.v);
#pragma unroll
    for (int i = 0; i < kPer; ++i) s[i] += E::get(e[i]);
  }
  // row = scale s (+ what it holds); stream: not to be kept in L2
  static __device__ __forceinline__ void store(T* row, int64_t block, int lane, int64_t d, const float (&s)[kPer],
                                               float scale, bool add, bool stream) {
    Raw r;
    T* e = reinterpret_cast<T*>(&r.v);
    const bool whole = kVec && at(block, lane, kPer) <= d;
    if (add && whole) r.v = *reinterpret_cast<const uint4*>(row + at(block, lane, 0));
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t c = at(block, lane, i);
      if (add && !whole && c < d) e[i] = row[c];
      e[i] = E::put(add ? fmaf(scale, s[i], E::get(e[i])) : scale * s[i]);
    }
    if (whole && stream) __stcs(reinterpret_cast<uint4*>(row + at(block, lane, 0)), r.v);
    else if (whole) *reinterpret_cast<uint4*>(row + at(block, lane, 0)) = r.v;
    else
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (at(block, lane, i) < d) row[at(block, lane, i)] = e[i];
  }
};

// ------------------------------------------------------------------ lookup

constexpr int kLookBlocks = 8;  // column blocks (512 bytes each) of one step of a warp

template <int kType, bool kVec>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, Status st) {
  using C = Cols<kType, kVec>;
  using T = typename C::T;
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t nwarps = (int64_t)gridDim.x * (blockDim.x >> 5);
  const int64_t blocks = (a.D + 32 * C::kPer - 1) / (32 * C::kPer);
  const int64_t steps = (blocks + kLookBlocks - 1) / kLookBlocks;
  for (int64_t it = warp; it < a.T * steps; it += nwarps) {
    const int64_t t = it / steps, b0 = (it - t * steps) * kLookBlocks;
    const int64_t id = id_of(a.ids, a.id8, t);
    if (id >= a.V && lane == 0) report(st, GPO_ERR_SHAPE, 30, (int)t);
    const bool in = id >= 0 && id < a.V;
    const T* src = static_cast<const T*>(a.src) + (in ? id : 0) * a.src_stride;
    T* dst = static_cast<T*>(a.dst) + t * a.dst_stride;
    typename C::Raw r[kLookBlocks];
#pragma unroll
    for (int b = 0; b < kLookBlocks; ++b) {
      if (in && b0 + b < blocks) r[b] = C::load(src, b0 + b, lane, a.D);
      else r[b].v = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int b = 0; b < kLookBlocks; ++b) {
      if (b0 + b >= blocks) break;
      float s[C::kPer];
#pragma unroll
      for (int i = 0; i < C::kPer; ++i) s[i] = 0.f;
      C::add(r[b], s);
      C::store(dst, b0 + b, lane, a.D, s, a.scale, false, false);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) next_tag(st);
}

// ------------------------------------------------------------------ sort

// The ids of a CTA's tokens as the sort's keys.  (Id: a template, so that the loads of one thread need no
// branch between them and are in flight together.)
template <class Id>
struct EmbedKeys {
  using Key = Id;
  const Id* ids;
  __device__ __forceinline__ void load(int64_t t0, int64_t tb, Id (&id)[kSortAhead]) {
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) id[k] = t0 + 32 * k < tb ? ids[t0 + 32 * k] : (Id)-1;
  }
};

template <class Id>
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(EmbedArgs a, int per, Status st) {
  extern __shared__ int hist[];
  let_next_start();
  EmbedKeys<Id> keys = {static_cast<const Id*>(a.ids)};
  sort_tokens<31, kWhereEmbedPlace>(
      keys, a.T, a.V, per, hist, st, [&](int64_t row, int first) { a.start[row] = first; },
      [&](int place, int64_t t, Id id) {
        a.perm[place] = (int)t;
        a.sid[place] = (int)id;
      });
  if (blockIdx.x == 0 && threadIdx.x == 0) next_tag(st);
}

// ------------------------------------------------------------------ sums of runs

constexpr int kSumThreads = 256;
constexpr int kSumAhead = 8;  // rows in flight per lane

template <int kType, bool kVec>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(EmbedArgs a, int piece, Status st) {
  using C = Cols<kType, kVec>;
  using T = typename C::T;
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);
  const int64_t nwarps = (int64_t)gridDim.x * (kSumThreads / 32);
  const int64_t blocks = (a.D + 32 * C::kPer - 1) / (32 * C::kPer);
  let_next_start();
  after_previous();
  const int n = a.start[a.V];
  const int64_t pieces = ((int64_t)n + piece - 1) / piece;
  const int64_t empties = a.accumulate ? 0 : (a.V + 31) / 32;  // groups of 32 rows that may have no token
  T* out = static_cast<T*>(a.dst);
  for (int64_t it = warp; it < (pieces + empties) * blocks; it += nwarps) {
    const int64_t unit = it / blocks, b = it - unit * blocks;
    float s[C::kPer];
#pragma unroll
    for (int i = 0; i < C::kPer; ++i) s[i] = 0.f;
    if (unit >= pieces) {
      const int64_t v = (unit - pieces) * 32 + lane;
      uint32_t m = __ballot_sync(0xffffffffu, v < a.V && a.start[min(v, a.V - 1)] == a.start[min(v, a.V - 1) + 1]);
      for (; m; m &= m - 1u)
        C::store(out + ((unit - pieces) * 32 + __ffs(m) - 1) * a.dst_stride, b, lane, a.D, s, 1.f, false, true);
      continue;
    }
    const int64_t p0 = unit * piece, p1 = min(p0 + piece, (int64_t)n);
    int run = a.sid[p0];                                      // the id being summed
    bool cut = p0 > 0 && a.sid[p0 - 1] == run;                // its run began before the piece
    const int after = p1 < n ? a.sid[p1] : -1;
    auto leave = [&](bool cut_after) {
      if (cut || cut_after) {
        float* part = a.part + (unit * 2 + (cut ? 0 : 1)) * a.part_stride;
#pragma unroll
        for (int i = 0; i < C::kPer; ++i)
          if (C::at(b, lane, i) < a.D) part[C::at(b, lane, i)] = s[i];
      } else if (GPO_BOUNDS(st, run, a.V, kWhereEmbedRow)) {
        C::store(out + (int64_t)run * a.dst_stride, b, lane, a.D, s, a.scale, a.accumulate != 0, true);
      }
#pragma unroll
      for (int i = 0; i < C::kPer; ++i) s[i] = 0.f;
    };
    for (int64_t q = p0; q < p1; q += 32) {
      const int64_t pos = q + lane;
      const int tok = pos < p1 ? a.perm[pos] : 0, id = pos < p1 ? a.sid[pos] : -1;
      const int cnt = (int)min((int64_t)32, p1 - q);
#pragma unroll 1
      for (int j0 = 0; j0 < cnt; j0 += kSumAhead) {
        typename C::Raw r[kSumAhead];
#pragma unroll
        for (int j = 0; j < kSumAhead; ++j) {
          const int tk = __shfl_sync(0xffffffffu, tok, (j0 + j) & 31);
          if (j0 + j < cnt) r[j] = C::load(static_cast<const T*>(a.src) + (int64_t)tk * a.src_stride, b, lane, a.D);
        }
#pragma unroll
        for (int j = 0; j < kSumAhead; ++j) {
          const int v = __shfl_sync(0xffffffffu, id, (j0 + j) & 31);
          if (j0 + j < cnt) {
            if (v != run) {
              leave(false);
              run = v;
              cut = false;
            }
            C::add(r[j], s);
          }
        }
      }
    }
    leave(after == run);
  }
}

// Cut runs: a warp takes kJoinPieces pieces and 32 x 4 columns; a run belongs to the piece it starts in.
constexpr int kJoinPieces = 2;
constexpr int kJoinAhead = 8;

template <int kType>
__global__ void __launch_bounds__(256) embed_join_kernel(EmbedArgs a, int piece) {
  using E = Elem<kType>;
  using T = typename E::T;
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t nwarps = (int64_t)gridDim.x * (blockDim.x >> 5);
  after_previous();
  const int n = a.start[a.V];
  const int64_t pieces = ((int64_t)n + piece - 1) / piece;
  const int64_t blocks = (a.D + 127) / 128, groups = (pieces + kJoinPieces - 1) / kJoinPieces;
  for (int64_t it = warp; it < groups * blocks; it += nwarps) {
    const int64_t g = it / blocks, b = it - g * blocks;
    // lane k: the run that the end of piece g * kJoinPieces + k cuts, if it starts in that piece
    const int64_t p = g * kJoinPieces + (lane & (kJoinPieces - 1));
    int row = -1;
    if (lane < kJoinPieces && (p + 1) * piece < n) {
      const int x = a.sid[(p + 1) * piece - 1];
      if (x == a.sid[(p + 1) * piece] && a.start[x] >= p * piece) row = x;
    }
    for (uint32_t m = __ballot_sync(0xffffffffu, row >= 0); m; m &= m - 1u) {
      const int k = __ffs(m) - 1;
      const int v = __shfl_sync(0xffffffffu, row, k);
      const int64_t pa = g * kJoinPieces + k, pz = ((int64_t)a.start[v + 1] - 1) / piece;
      const int64_t c = b * 128 + lane * 4;
      if (c >= a.D) continue;
      const float* part = a.part + c;  // (rows of the workspace have room for whole float4)
      float4 s = *reinterpret_cast<const float4*>(part + (pa * 2 + 1) * a.part_stride);
#pragma unroll 1
      for (int64_t q = pa + 1; q <= pz; q += kJoinAhead) {
        float4 x[kJoinAhead];
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j)
          if (q + j <= pz) x[j] = *reinterpret_cast<const float4*>(part + (q + j) * 2 * a.part_stride);
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j)
          if (q + j <= pz) s.x += x[j].x, s.y += x[j].y, s.z += x[j].z, s.w += x[j].w;
      }
      T* dst = static_cast<T*>(a.dst) + (int64_t)v * a.dst_stride + c;
      const float y[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < a.D) dst[i] = E::put(a.accumulate ? fmaf(a.scale, y[i], E::get(dst[i])) : a.scale * y[i]);
    }
  }
}

inline bool vec_rows(const void* p, int64_t stride, int esz) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride * esz % 16 == 0;
}

template <int kType>
cudaError_t look(const LaunchCtx& lc, const EmbedArgs& a, const Status& st) {
  const int esz = kType == GPO_DT_F32 ? 4 : 2;
  const int64_t per = (int64_t)kLookBlocks * 512 / esz;
  const int64_t warps = a.T * ((a.D + per - 1) / per);
  const int grid = (int)min((warps + 7) / 8, (int64_t)lc.num_sms * 8);
  if (vec_rows(a.src, a.src_stride, esz) && vec_rows(a.dst, a.dst_stride, esz))
    embed_kernel<kType, true><<<grid, 256, 0, lc.stream>>>(a, st);
  else embed_kernel<kType, false><<<grid, 256, 0, lc.stream>>>(a, st);
  return cudaGetLastError();
}

template <int kType>
cudaError_t sums(const LaunchCtx& lc, const EmbedArgs& a, const Status& st) {
  const int esz = kType == GPO_DT_F32 ? 4 : 2;
  const int piece = embed_piece(a.T);
  const int64_t blocks = (a.D * esz + 511) / 512, pieces = (a.T + piece - 1) / piece;
  const int64_t units = (pieces + (a.accumulate ? 0 : (a.V + 31) / 32)) * blocks;
  const unsigned grid = (unsigned)max((int64_t)1, min((units + 7) / 8, (int64_t)lc.num_sms * 16));
  const bool vec = vec_rows(a.src, a.src_stride, esz) && vec_rows(a.dst, a.dst_stride, esz);
  const cudaError_t e = launch_after(vec ? embed_sum_kernel<kType, true> : embed_sum_kernel<kType, false>, grid, kSumThreads,
                                     0, lc.stream, a, piece, st);
  if (e != cudaSuccess || pieces < 2) return e;
  const int64_t jobs = (pieces + kJoinPieces - 1) / kJoinPieces * ((a.D + 127) / 128);
  return launch_after(embed_join_kernel<kType>, (unsigned)min((jobs + 7) / 8, (int64_t)lc.num_sms * 8), 256, 0, lc.stream, a, piece);
}

}  // namespace

// Longer pieces leave fewer sums of a frequent token to join, shorter ones give more warps something to do.
int embed_piece(int64_t T) { return T <= 4096 ? 8 : T <= 16384 ? 32 : T <= 65536 ? 64 : 128; }

cudaError_t setup_embed() {
  const int bytes = (int)sort_smem(kSortMaxRows);
  const cudaError_t e = cudaFuncSetAttribute(embed_sort_kernel<int32_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(embed_sort_kernel<int64_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

cudaError_t launch_embed(const LaunchCtx& lc, const EmbedArgs& a, const Status& st) {
  if (a.dtype == GPO_DT_F32) return look<GPO_DT_F32>(lc, a, st);
  if (a.dtype == GPO_DT_F16) return look<GPO_DT_F16>(lc, a, st);
  return look<GPO_DT_BF16>(lc, a, st);
}

cudaError_t launch_embed_grad(const LaunchCtx& lc, const EmbedArgs& a, const Status& st) {
  const int per = sort_rows(a.V, lc.num_sms);
  const unsigned grid = (unsigned)((a.V + per - 1) / per);
  if (a.id8) embed_sort_kernel<int64_t><<<grid, kSortThreads, sort_smem(per), lc.stream>>>(a, per, st);
  else embed_sort_kernel<int32_t><<<grid, kSortThreads, sort_smem(per), lc.stream>>>(a, per, st);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (a.dtype == GPO_DT_F32) return sums<GPO_DT_F32>(lc, a, st);
  if (a.dtype == GPO_DT_F16) return sums<GPO_DT_F16>(lc, a, st);
  return sums<GPO_DT_BF16>(lc, a, st);
}

}  // namespace gpo
