"""The adjusted logits and the distillation under the debug build of libgraphpo (GPO_DEBUG: the places of special entries, the
rows of gathered tokens and the entries of dz are checked before they are used, and reported as GPO_ERR_BOUNDS).  A child process
loads that library and runs them against plain torch in 64 bits; each call must finish with no status."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import sys
import torch
sys.path.insert(0, ROOT)
sys.path.insert(0, ROOT + "/tests")
import paper_2606_18954_gb300 as P
import distill_ref
import logits_ref
from paper_2606_18954_gb300 import binding, buildlib
assert binding.lib_path() == buildlib.DEBUG_LIB, binding.lib_path()
gp = P.GraphPO()
for R, V, dt, kw in ((3, 140007, torch.bfloat16, dict(history=9000, biases=2000, masks=2, pad=3)), (700, 1001, torch.float16, dict(masks=3, masked=0.3, biases=9)),
                     (40, 9001, torch.float32, dict(history=300, pad=1, temperature=True)), (2, 30000, torch.bfloat16, dict(penalties=False, history=0))):
    z, y, how = logits_ref.inputs(R, V, dt, seed=R, **kw)
    g = torch.randn(R, device="cuda")
    ref = logits_ref.exact(z, y, how, g)
    f = gp.logits_adjust(z, y, **how)
    d = gp.logits_grad(z, y, f["lse"], f["logp"], g, **how)["d_logits"]
    s = gp.logits_adjust(z, write=torch.float32, **how)["logits"]
    gp.check()
    for k in f:
        logits_ref.near(f[k], ref[k], ref["t_" + k], k)
    logits_ref.near(d, torch.where(torch.isfinite(ref["d_logits"]), ref["d_logits"], 0.0), ref["t_d_logits"], "d_logits")
    every = logits_ref.exact(z, None, how)["logits"]
    assert torch.equal(torch.isinf(s), torch.isinf(every)) and s.shape == z.shape
    print("ok logits", R, V, flush=True)
for T, V, d, k, dt, kw in ((300, 3000, 264, 33, torch.float16, dict(masked=0.3)), (4500, 700, 64, 16, torch.bfloat16, dict(masked=0.5, short=True, tail=True)),
                           (5, 40, 72, 40, torch.bfloat16, {})):
    h, w, ids, t = distill_ref.inputs(T, V, d, k, dt, seed=T, **kw)
    g = torch.randn(T, device="cuda") * (512.0 if dt is torch.float16 else 1.0) / T
    ref = distill_ref.exact(h, w, ids, t, tail=kw.get("tail", False), g=g)
    f = gp.vocab_distill(h, w, ids, t, tail=kw.get("tail", False))
    r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
    gp.check()
    for n in ("loss", "delta", "rest", "rest_lse"):
        distill_ref.near(f[n], ref[n], ref["t_" + n], n)
    for n in r:
        distill_ref.near(r[n], ref[n], ref["t_" + n], n)
    print("ok distill", T, V, flush=True)
'''


def test_under_the_debug_build():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    from paper_2606_18954_gb300 import buildlib
    lib = buildlib.build(debug=True)
    r = subprocess.run([sys.executable, "-c", f"ROOT = {ROOT!r}\n" + CHILD], env=dict(os.environ, GRAPHPO_LIB=lib),
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert r.stdout.count("ok ") == 7, r.stdout
