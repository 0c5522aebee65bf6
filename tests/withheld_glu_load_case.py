"""Run by test_gpu_glu_failure.py with NSP_LIBRARY pointing at libnsp_checked.so: one operand tile of a feed-forward product never
arrives. The launch ends by itself, the record names the wait, later nsp_glu calls are refused with it, other calls go on."""
import sys
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
sys.path.insert(0, str(ROOT))
sys.path.insert(0, str(ROOT / "tests"))

import torch  # noqa: E402

import parity_util as P  # noqa: E402
from paper_2609_22755_b200 import binding as B  # noqa: E402
from paper_2609_22755_b200 import workloads as W  # noqa: E402

load, direction, rows, d, f = sys.argv[1], sys.argv[2], *map(int, sys.argv[3:])
rnd = lambda *s: torch.randn(*s, device="cuda").bfloat16()
x, wg, wu, dh, g, u = rnd(rows, d), rnd(f, d), rnd(f, d), rnd(rows, f), rnd(rows, f), rnd(rows, f)
h, dx, dwg, dwu = rnd(rows, f), rnd(rows, d), rnd(f, d), rnd(f, d)
ws = torch.empty(B.nsp_glu_bwd_ws_bytes(rows, d, f), dtype=torch.uint8, device="cuda")


def call():
    if direction == "forward":
        B.nsp_glu_fwd(x, wg, wu, h)
    else:
        B.nsp_glu_bwd(dh, x, wg, wu, g, u, dx, dwg, dwu, ws)


call()
assert B.nsp_glu_status() == (0, 0, 0, 0)
B.nsp_checked_withhold_glu_load(int(load))
call()
torch.cuda.synchronize()  # the launch ends by itself
code, tile, where, aux = B.nsp_glu_status()
print("withheld glu load:", (code, tile, where, aux))
assert (code, tile, where) == (B.NSP_ERR_DEVICE_TIMEOUT, 0, 52), (code, tile, where, aux)  # the issuer, waiting for operands
B.nsp_checked_withhold_glu_load(0)
try:
    call()
    raise SystemExit("a later call was not refused")
except B.NspError as e:
    assert e.code == B.NSP_ERR_DEVICE_TIMEOUT
run = P.GpuRun(W.config(1))  # attention is not concerned
run.forward()
run.backward()
assert run.status()[0] == 0
y = torch.empty_like(x)
B.nsp_norm_fwd(x, None, None, y, None, None)
torch.cuda.synchronize()
assert torch.isfinite(y).all()
print("other calls after the timeout: ok")
