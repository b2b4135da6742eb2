// A stable counting sort of tokens by their row of a table, for embed_sort_kernel and vocab_sort_kernel,
// without any exchange between CTAs.  CTA b owns the rows [b per, (b + 1) per), up to kSortMaxRows, and reads all
// keys twice from L2 (4 or 8 bytes a token, against the hundreds or thousands of a token's row): first it counts those
// of its rows, per warp and row, and those of the rows before its own, which gives its place in the
// sorted list; then every warp places its tokens in their order.
#pragma once

#include "gpo_internal.cuh"

namespace gpo {

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortAhead = 8;      // keys of a lane in flight
constexpr int kSortMaxRows = 1024;

inline size_t sort_smem(int rows) { return sizeof(int) * (size_t)(kSortWarps + 1) * rows; }
// Rows per CTA: one CTA per SM where that leaves it at least a warp's worth of them.
inline int sort_rows(int64_t V, int num_sms) {
  return (int)std::min<int64_t>(std::max<int64_t>((V + num_sms - 1) / num_sms, 32), kSortMaxRows);
}

// keys.load(t0, tb, id): the keys of tokens t0 + 32 k < tb, -1 for one that takes no part (a key from V on
// is reported and takes none either); begin(row, first): the first place of a row, and of row V the number
// of all that take part; put(place, token, key).  hist: sort_smem(per) bytes, [kSortWarps][per] counts, then places; [per]
// first place of a row.
template <int kCode, int kWhere, class Keys, class Begin, class Put>
__device__ __forceinline__ void sort_tokens(Keys& keys, int64_t T, int64_t V, int per, int* hist, const Status& st,
                                            Begin begin, Put put) {
  using Id = typename Keys::Key;
  __shared__ int wsum[kSortWarps];
  __shared__ int s_base;
  int* first = hist + kSortWarps * per;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Id r0 = (Id)blockIdx.x * per, r1 = (Id)min((int64_t)r0 + per, V);
  const int nr = (int)(r1 - r0);
  for (int i = threadIdx.x; i < kSortWarps * per; i += kSortThreads) hist[i] = 0;
  if (threadIdx.x == 0) s_base = 0;
  __syncthreads();
  const int64_t seg = ((T + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
  const int64_t ta = min(T, warp * seg), tb = min(T, ta + seg);
  int below = 0;
  for (int64_t t0 = ta + lane; t0 < tb; t0 += 32 * kSortAhead) {
    Id id[kSortAhead];
    keys.load(t0, tb, id);
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      if (id[k] >= r0 && id[k] < r1) atomicAdd(&hist[warp * per + (int)(id[k] - r0)], 1);
      below += id[k] >= 0 && id[k] < r0;
      if (id[k] >= V && blockIdx.x == 0) report(st, GPO_ERR_SHAPE, kCode, (int)(t0 + 32 * k));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) below += __shfl_xor_sync(0xffffffffu, below, o);
  if (lane == 0) atomicAdd(&s_base, below);
  __syncthreads();
  // thread i: row r0 + i (per <= kSortThreads)
  const int i = threadIdx.x;
  int total = 0;
  if (i < nr) {
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = hist[w * per + i];
      hist[w * per + i] = total;
      total += c;
    }
  }
  int incl = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) wsum[warp] = incl;
  __syncthreads();
  int before = s_base;
  for (int w = 0; w < warp; ++w) before += wsum[w];
  if (i < nr) {
    const int s = before + incl - total;
    first[i] = s;
    begin((int64_t)r0 + i, s);
    if ((int64_t)r0 + i == V - 1) begin(V, s + total);
  }
  __syncthreads();
  for (int64_t t0 = ta + lane; t0 - lane < tb; t0 += 32 * kSortAhead) {
    Id id[kSortAhead];
    keys.load(t0, tb, id);
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      const bool in = id[k] >= r0 && id[k] < r1;
      if (!__any_sync(0xffffffffu, in)) continue;
      const int row = in ? (int)(id[k] - r0) : -1;  // (few different values: match takes them one after another)
      const uint32_t same = __match_any_sync(0xffffffffu, row);
      int at = 0;
      if (in) at = hist[warp * per + row];
      __syncwarp();
      if (in) {
        const int place = first[row] + at + __popc(same & ((1u << lane) - 1u));
        if (GPO_BOUNDS(st, place, T, kWhere)) put(place, t0 + 32 * k, id[k]);
        if (lane == __ffs(same) - 1) hist[warp * per + row] = at + __popc(same);
      }
      __syncwarp();
    }
  }
}

}  // namespace gpo
