// What the calls on a model's vocabulary share on the host (gpo_vocab_api.cu, gpo_logits_api.cu): checks, and the launches of a
// call with their status words.  Host code.
#pragma once

#include <nvtx3/nvToolsExt.h>

#include "gpo_ctx.cuh"

namespace gpo {

constexpr int64_t kMaxCount = ((int64_t)1 << 31) - 1024;  // tokens, vocabulary rows, width
constexpr int64_t kMaxMatrix = (int64_t)1 << 40;          // elements of a matrix

// The kernels run on the context's device.
inline gpo_status check_device(gpo_ctx* c) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != c->device)
    return set_msg(c, "current device differs from the context's"), GPO_ERR_INVALID_ARG;
  return GPO_OK;
}

inline gpo_status check_call(gpo_ctx* c, const void* workspace, size_t have, size_t need) {
  if (!workspace || !aligned(workspace, kWorkspaceAlign) || have < need)
    return set_msg(c, "workspace needs %zu bytes, 256-byte aligned", need), GPO_ERR_WORKSPACE;
  return check_device(c);
}

// The place of a captured call's words among the library's.
int captured_place();

// The launches of one call: an NVTX range around each and, with timing on, a CUDA event after it.
struct Stages {
  gpo_ctx* ctx;
  LaunchCtx lc;
  int n;
  cudaError_t e;
  Status st;
  bool captured;

  // The call's errors: in words and with a tag of its own; in a graph, whose replays share both, in words that no other
  // call has, with a tag that every replay advances (next_tag; a memset node before it took 0.7 us of each).
  Stages(gpo_ctx* c, void* stream) : ctx(c), n(0), e(cudaSuccess) {
    lc.stream = static_cast<cudaStream_t>(stream);
    lc.num_sms = c->num_sms;
    if (ctx->timing) e = cudaEventRecord(ctx->ev[0], lc.stream);
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    captured = cudaStreamIsCapturing(lc.stream, &cap) != cudaSuccess || cap != cudaStreamCaptureStatusNone;
    if (captured) {
      cudaGetLastError();
      const int i = captured_place();
      ctx->captured.set(i);
      st.p = ctx->captured_words + i * kStatusWords;
      st.tag = kStoredTag;
    } else {
      st.tag = ++ctx->calls;
      st.p = ctx->call_words + ctx->calls % kCallWords * kStatusWords;
    }
  }
  template <class F>
  void operator()(const char* name, F launch) {
    if (e != cudaSuccess) return;
    nvtxRangePushA(name);
    e = launch();
    nvtxRangePop();
    if (ctx->timing && e == cudaSuccess && n < kMaxStages) {
      ctx->stage_name[n] = name;
      e = cudaEventRecord(ctx->ev[++n], lc.stream);
    }
  }
  gpo_status done() {
    ctx->nstages = n;
    if (ctx->last_read) ctx->last_status = nullptr;
    if (e != cudaSuccess) return set_msg(ctx, "launch failed: %s", cudaGetErrorString(e)), GPO_ERR_CUDA;
    return GPO_OK;
  }
};

}  // namespace gpo
