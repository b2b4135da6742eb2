// The context of the C ABI and what the translation units that implement its calls share.
// Host code.
#pragma once

#include <vector>

#include "gpo_internal.cuh"

struct gpo_ctx {
  gpo_params params;
  int device;
  int num_sms;
  uint32_t* host_status;      // pinned copy of the workspace status words
  const uint32_t* last_status; // device status words of the last gpo_compute
  char msg[512];
  bool timing;
  int nstages;                 // stages recorded by the last gpo_compute
  cudaEvent_t ev[gpo::kMaxStages + 1];
  const char* stage_name[gpo::kMaxStages];
  // gpo_compute_host: helper streams and events (created by its first pipelined call) and
  // the per-group state and token offsets of the last host batch
  bool pipe_ready;
  cudaStream_t pipe_in, pipe_out, pipe_comp[gpo::kPipeComputeStreams];
  cudaEvent_t pipe_ev[2 * gpo::kPipeMaxChunks + 2];
  std::vector<int64_t> pipe_s, pipe_t;
};

namespace gpo {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled of the driver; null where it is not to be had.
EncodeTiledFn encode_fn();

// Leaves a message for gpo_last_error (c may be null).
void set_msg(gpo_ctx* c, const char* fmt, ...);

// A tag of the status words that no other call of this process has.
uint64_t fresh_tag();

constexpr size_t kWorkspaceAlign = 256;
inline size_t workspace_up(size_t x) { return (x + kWorkspaceAlign - 1) & ~(kWorkspaceAlign - 1); }

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace gpo
