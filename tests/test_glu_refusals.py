"""What the calls of the gated feed-forward block refuse before anything reaches a device. No GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2609_22755_b200 import build

    build.build_library()
    from paper_2609_22755_b200 import binding

    return binding


BUF = 1 << 20  # an address that is never dereferenced: every case is refused first, or has nothing to do


def _call(B, which, rows=4, d=64, f=128, act=0, ws=1 << 28, ws_bytes=1 << 30, **change):
    shape = {"x": d, "w_gate": d, "w_up": d, "h": f, "g": f, "u": f, "dh": f, "dx": d, "dw_gate": d, "dw_up": d}
    m = {}
    for i, (name, cols) in enumerate(shape.items()):
        v = change.get(name, {})
        m[name] = None if v is None else ctypes.byref(B.Matrix(v.get("data", BUF * (i + 1)), v.get("ld", cols)))
    if which == "fwd":
        return B.lib().nsp_glu_fwd(*[m[k] for k in ("x", "w_gate", "w_up", "h", "g", "u")], rows, d, f, act, None)
    return B.lib().nsp_glu_bwd(*[m[k] for k in ("dh", "x", "w_gate", "w_up", "g", "u", "dx", "dw_gate", "dw_up")], rows, d, f, act, ws, ws_bytes,
                               None)


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_refusals(B, which):
    inv, uns = B.NSP_ERR_INVALID_ARG, B.NSP_ERR_UNSUPPORTED
    call = lambda **k: _call(B, which, **k)
    assert call(rows=-1) == inv and call(d=0) == inv and call(f=0) == inv and call(act=2) == inv
    assert call(d=63) == uns and call(f=129) == uns and call(d=1048584) == uns
    assert call(rows=1 << 27, f=128) == uns
    out = "h" if which == "fwd" else "dx"
    for name in ("x", "w_gate", "w_up", out) + (() if which == "fwd" else ("g", "u", "dh", "dw_gate")):
        assert call(**{name: {"data": None}}) == inv
        assert call(**{name: {"data": BUF + 8}}) == inv  # not on 16 bytes
        assert call(**{name: {"ld": 56}}) == inv  # rows that overlap
        assert call(**{name: {"ld": 132}}) == inv  # rows not on 16 bytes
        assert call(**{name: {"ld": (1 << 31) + 8}}) == inv
    if which == "fwd":
        assert call(rows=0) == B.NSP_OK and call(rows=0, x=None) == B.NSP_OK
        assert call(x=None) == inv and call(h=None) == inv and call(u={"ld": 56}) == inv
    else:
        assert call(dw_gate=None) == inv and call(dw_up=None) == inv  # both or neither
        assert call(dw_gate=None, dw_up=None, dx=None) == B.NSP_OK  # nothing is wanted
        assert call(dh=None) == inv and call(g=None) == inv and call(x=None) == inv and call(w_up=None) == inv
        assert call(rows=0, dw_gate=None, dw_up=None) == B.NSP_OK
        need = B.nsp_glu_bwd_ws_bytes(4, 64, 128)
        assert call(ws=None) == B.NSP_ERR_WORKSPACE and call(ws=BUF + 16) == B.NSP_ERR_WORKSPACE
        assert call(ws_bytes=need - 1) == B.NSP_ERR_WORKSPACE


def test_workspace_and_status(B):
    assert B.nsp_glu_bwd_ws_bytes(0, 64, 128) == 0
    dg_du, partial = 4 * 16384 * 12288, B.nsp_glu_bwd_ws_bytes(1, 8, 8)
    assert dg_du < B.nsp_glu_bwd_ws_bytes(16384, 4096, 12288) <= dg_du + partial  # a bounded part beside dg and du
    assert partial < 1 << 26
    for bad in ((-1, 64, 128), (4, 60, 128), (4, 64, 0)):
        with pytest.raises(B.NspError):
            B.nsp_glu_bwd_ws_bytes(*bad)
    assert B.lib().nsp_glu_status(None) == B.NSP_ERR_INVALID_ARG


def test_binding_refusals(B):
    import torch

    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(B.NspError):
        B.nsp_glu_fwd(x, x, x, x)  # not on a device
    with pytest.raises(B.NspError):
        B.nsp_glu_bwd(x, x, x, x, x, x, x, x, x, None)
