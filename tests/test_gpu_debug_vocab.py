"""The vocabulary ends under the debug build of libgraphpo (GPO_DEBUG: every index of a list, a sorted place, a row of a
gradient is checked before it is used, and reported as GPO_ERR_BOUNDS).  A child process loads that library and runs
every kernel of theirs against plain torch in 64 bits; each call must finish with no status."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import math, sys
import torch
sys.path.insert(0, ROOT)
sys.path.insert(0, ROOT + "/tests")
import paper_2606_18954_gb300 as P
from paper_2606_18954_gb300 import binding, buildlib
from vocab_ref import close, head_exact, head_inputs
assert binding.lib_path() == buildlib.DEBUG_LIB, binding.lib_path()
assert b"GPO_DEBUG" in binding.load().gpo_version(), binding.load().gpo_version()
gp = P.GraphPO()

# one launch; tiles with a joining CTA per row, and per 32 rows; wide rows; the sort instead of the comparison; rows of any
# alignment, added; listed tokens of a short and of a long batch
for T, V, d, dtype, masked, entropy, any_rows in (
        (9, 20011, 136, "bf16", 0.3, True, False), (16, 40, 64, "f16", 0.0, False, False), (200, 3001, 264, "f16", 0.3, True, False),
        (700, 1025, 328, "bf16", 0.2, True, True), (300, 700, 2104, "bf16", 0.3, True, False), (300, 700, 2104, "f16", 0.0, False, True),
        (4500, 500, 72, "bf16", 0.3, False, False), (9000, 300, 40, "f16", 0.5, True, True)):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    h, w, y = head_inputs(T, V, d, dt, 0, masked, seed=T, id_dtype=torch.int64 if T % 2 else torch.int32, sure=8.0)
    f = gp.vocab_logp(h, w, y, entropy=entropy)
    gp.check()
    to = 512.0 if dtype == "f16" else 1.0
    g = torch.randn(T, device="cuda") * to / T
    g[::3] = 0.0
    e = torch.randn(T, device="cuda") * 0.05 * to / T if entropy else None
    extra = 3 if any_rows else 0
    base = torch.randn(V, d + extra, device="cuda").to(dt) * 1e-3
    out = {"d_hidden": torch.empty(T, d + extra, device="cuda", dtype=dt)[:, :d], "d_weight": base.clone()[:, :d]}
    gp.vocab_grad(h, w, y, f["lse"], g, entropy=f.get("entropy"), grad_entropy=e, out=out, accumulate=any_rows, logp=f["logp"])
    gp.check()
    ref = head_exact(h, w, y, 1.0, g, e)
    for k in f:
        close(f[k], ref[k], ref["t_" + k], k)
    close(out["d_hidden"], ref["d_hidden"], ref["t_d_hidden"], "d_hidden")
    want = ref["d_weight"] + (base[:, :d].double() if any_rows else 0)
    close(out["d_weight"], want, ref["t_d_weight"] + 2.0 ** -8 * want.abs(), "d_weight")
    print("ok head", T, V, d, dtype, flush=True)

# listed: 2^37 products
T, V, d = 256, 131072, 4096
h, w, y = head_inputs(T, V, d, torch.bfloat16, masked=0.4, seed=1)
f = gp.vocab_logp(h, w, y, entropy=True)
gp.check()
ref = head_exact(h, w, y, 1.0)
for k in f:
    close(f[k], ref[k], ref["t_" + k], k)
print("ok listed", flush=True)
del h, w, ref
h, w, y = head_inputs(9000, 30011, 520, torch.bfloat16, masked=0.4, seed=31)
f = gp.vocab_logp(h, w, y)
gp.check()
ref = head_exact(h[:2000], w, y[:2000], 1.0)
for k in f:
    close(f[k][:2000], ref[k], ref["t_" + k], k)
print("ok listed long", flush=True)
del h, w, ref

for dt, T, V, d, off in ((torch.float32, 5000, 900, 65, 0), (torch.bfloat16, 20000, 40000, 136, 0), (torch.float16, 1000, 300, 257, 1)):
    table = (torch.randn(V, d + off, device="cuda") / 4).to(dt)[:, off:]
    u = torch.rand(T, device="cuda", dtype=torch.float64)
    ids = torch.where(u < 0.1, -1, (torch.exp(u * math.log(V + 1)) - 1).long()).clamp(max=V - 1)
    x = gp.embed(table, ids)
    gp.check()
    keep = ids >= 0
    assert torch.equal(x, torch.where(keep[:, None], table[ids.clamp(min=0)], torch.zeros((), dtype=dt, device="cuda")))
    out = torch.zeros(V, d + off, device="cuda", dtype=dt)[:, off:]
    for _ in range(2):  # the second time added to the first
        gp.embed_grad(x, ids, V, out=out, accumulate=_ > 0)
    gp.check()
    want = 2 * torch.zeros(V, d, dtype=torch.float64, device="cuda").index_put_((ids[keep],), x[keep].double(), accumulate=True)
    assert float((out.double() - want).norm()) <= 2.0 ** -7 * float(want.norm())
    print("ok embed", T, V, d, dt, flush=True)
'''


def test_vocabulary_ends_under_the_debug_build():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    from paper_2606_18954_gb300 import buildlib
    lib = buildlib.build(debug=True)
    r = subprocess.run([sys.executable, "-c", f"ROOT = {ROOT!r}\n" + CHILD], env=dict(os.environ, GRAPHPO_LIB=lib),
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert r.stdout.count("ok ") == 13, r.stdout
