"""What stops a wait in a kernel: an error of its own call, never one that an earlier replay of the same captured call left."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_18954_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#define GPO_TAG_ADVANCES 1
#include "gpo_internal.cuh"
using namespace gpo;
static uint32_t words[kStatusWords];
static void error_of(uint64_t tag, int code) {
  *reinterpret_cast<uint64_t*>(words + kStError) = tag << 16 | (uint64_t)code;
}
static const uint64_t kWaits[] = {0, 1000, 100000, 900000, 2000000, 1999000000};
static int failed = 0;
static void expect(bool got, bool want, const char* what, uint64_t ns) {
  if (got == want) return;
  std::printf("%s after %llu ns\n", what, (unsigned long long)ns);
  ++failed;
}
int main() {
  const Status replay = {words, kStoredTag}, call = {words, 77};
  uint64_t& tag = *reinterpret_cast<uint64_t*>(words + kStTag);
  tag = 41;
  for (uint64_t ns : kWaits) expect(GPO_STOPS_WAITING(replay, ns), false, "no error", ns);
  for (int code : {GPO_ERR_SHAPE, GPO_ERR_TIMEOUT, GPO_ERR_NONFINITE}) {
    // a replay before this one has left its error, and the first block's store has not been seen
    error_of(tag, code);
    for (uint64_t ns : kWaits)
      if (ns < 1000000) expect(GPO_STOPS_WAITING(replay, ns), false, "earlier error, tag not advanced", ns);
    next_tag(replay);
    for (uint64_t ns : kWaits) expect(GPO_STOPS_WAITING(replay, ns), false, "earlier error", ns);
    // an error of this replay: the others stop when they have waited long enough to know it for one
    error_of(tag, code);
    for (uint64_t ns : kWaits)
      if (ns > 1000000) expect(GPO_STOPS_WAITING(replay, ns), true, "own error", ns);
    next_tag(replay);
  }
  // a call with a tag of its own knows at once
  error_of(77, GPO_ERR_TIMEOUT);
  for (uint64_t ns : kWaits) expect(GPO_STOPS_WAITING(call, ns), true, "the call's error", ns);
  error_of(76, GPO_ERR_TIMEOUT);
  for (uint64_t ns : kWaits) expect(GPO_STOPS_WAITING(call, ns), false, "another call's error", ns);
  next_tag(call);
  expect(tag == 47, true, "a call's tag is its own", 0);
  std::printf("%d failed\n", failed);
}
"""


def test_what_stops_a_wait(tmp_path):
    from paper_2606_18954_gb300 import buildlib
    try:
        nvcc = buildlib._nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src = tmp_path / "waits.cu"
    src.write_text(PROGRAM)
    exe = tmp_path / "waits"
    subprocess.check_call([nvcc, *buildlib.FLAGS, *buildlib.ARCH, "-I", CSRC, str(src), "-o", str(exe)])
    out = subprocess.check_output([str(exe)], text=True)
    assert out == "0 failed\n", out


def test_waits_ask_the_rule():
    """No wait asks for the bare error word, and every file of waits in calls whose replays advance their tag says that they do."""
    text = {n: open(os.path.join(CSRC, n)).read() for n in os.listdir(CSRC) if n.endswith((".cu", ".cuh"))}
    assert text
    for name, t in text.items():
        for line in t.splitlines():
            assert not ("aborted(st)" in line and "return false" in line), (name, line)
        if name.endswith(".cu") and "next_tag(st)" in t and "mbar_wait" in t:
            assert t.index("#define GPO_TAG_ADVANCES 1") < t.index('#include "gpo_'), name
