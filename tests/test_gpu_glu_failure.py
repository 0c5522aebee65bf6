"""A wait of the feed-forward kernels that runs out: the checked build leaves out one operand tile, in a child process (the record of
these calls belongs to the process's device and stays)."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


@pytest.mark.parametrize("load", [1, 2])
@pytest.mark.parametrize("direction,sizes", [("forward", (600, 512, 1024)), ("forward", (4096, 136, 4736)), ("backward", (6001, 520, 3000)),
                                             ("backward", (300, 264, 2056))])
def test_withheld_load(load, direction, sizes):
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    env = dict(os.environ, NSP_LIBRARY=str(ROOT / "paper_2609_22755_b200" / "libnsp_checked.so"))
    r = subprocess.run([sys.executable, str(ROOT / "tests" / "withheld_glu_load_case.py"), str(load), direction, *map(str, sizes)], env=env,
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "other calls after the timeout: ok" in r.stdout


@pytest.mark.parametrize("call", ["rope", "norm", "glu"])
def test_first_call_under_capture(call):
    """The first call of a process, made while a stream is being captured."""
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    code = f"""
import sys
sys.path.insert(0, {str(ROOT)!r})
import numpy as np, torch
from paper_2609_22755_b200 import binding as B
x = torch.randn(64, 4, 128, device="cuda").bfloat16()
w, y, h = torch.randn(256, 128, device="cuda").bfloat16(), torch.zeros_like(x), torch.zeros(256, 256, device="cuda", dtype=torch.bfloat16)
flat, out = x.view(256, 128), y.view(256, 128)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
def go():
    if {call!r} == "rope":
        B.nsp_rope(x, y, None, np.full(64, 0.1))
    elif {call!r} == "norm":
        B.nsp_norm_fwd(flat, None, None, out, None, None)
    else:
        B.nsp_glu_fwd(flat, w, w, h)
with torch.cuda.graph(graph):
    go()
graph.replay()
torch.cuda.synchronize()
got = (h if {call!r} == "glu" else y).clone()
assert got.abs().sum() > 0
go()
torch.cuda.synchronize()
assert torch.equal(got, h if {call!r} == "glu" else y)
print("ok")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
