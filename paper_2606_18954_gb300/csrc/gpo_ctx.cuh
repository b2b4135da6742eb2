// The context of the C ABI and what the translation units that implement its calls share.
// Host code.
#pragma once

#include <bitset>
#include <vector>

#include "gpo_internal.cuh"

namespace gpo {
// Status words of the calls of the vocabulary ends (gpo_vocab_api.cu): a call's own, one of kCallWords in turn, and
// those of captured calls, which belong to the library and outlive the context.
constexpr int kCallWords = 256;
constexpr int kCapturedWords = 4096;
static_assert(kCapturedWords % kCallWords == 0, "read kCallWords at a time");
}  // namespace gpo

struct gpo_ctx {
  gpo_params params;
  int device;
  int num_sms;
  uint32_t* host_status;      // pinned copy of the workspace status words
  const uint32_t* last_status; // device status words of the last gpo_compute or loss call
  bool last_read;              // gpo_sync_status has returned what they say
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
  // the vocabulary ends' calls: the n-th signs its errors with n in words n % kCallWords
  uint64_t calls;
  uint32_t* call_words;        // [kCallWords][kStatusWords] on the device
  uint32_t* host_words;        // the same, pinned: the copy that is read
  uint64_t returned[gpo::kCallWords];  // the call whose error in these words has been returned
  uint32_t* captured_words;    // the library's, on this context's device
  std::bitset<gpo::kCapturedWords> captured;  // which of them this context's captured calls have
};

namespace gpo {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled of the driver; null where it is not to be had.
EncodeTiledFn encode_fn();

// Leaves a message for gpo_last_error (c may be null).
void set_msg(gpo_ctx* c, const char* fmt, ...);

// A tag that no other call of this process has.
uint64_t fresh_tag();

// The status words of the vocabulary ends' calls: memory for them, its release, and the first error that has not been
// returned yet (GPO_OK if none; `stream` has been waited for).
cudaError_t make_call_words(gpo_ctx* c);
void free_call_words(gpo_ctx* c);
gpo_status read_call_words(gpo_ctx* c, cudaStream_t stream);

// A call other than theirs is the last one.
inline void set_last_status(gpo_ctx* c, const uint32_t* words) {
  c->last_status = words;
  c->last_read = false;
}

constexpr size_t kWorkspaceAlign = 256;
inline size_t workspace_up(size_t x) { return (x + kWorkspaceAlign - 1) & ~(kWorkspaceAlign - 1); }

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace gpo
