"""What the rotary and norm calls refuse, before anything reaches a device, and the frequencies (host only). No GPU."""
import ctypes
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2609_22755_b200 import build

    build.build_library()
    from paper_2609_22755_b200 import binding

    return binding


BUF = 1 << 20  # an address that is never dereferenced: every case is refused first, or has nothing to do


def _rope(B, tensors=None, head_dim=128, rot=128, layout=0, freq="ok", magnitude=1.0, **change):
    t = dict(x=BUF, y=2 * BUF, positions=None, tokens=0, x_token_stride=1024, x_head_stride=128, y_token_stride=1024, y_head_stride=128,
             heads=8, dtype=B.NSP_BF16)
    t.update(change)
    n = 1 if tensors is None else tensors
    array = (B.RopeTensor * max(n, 1))(*[B.RopeTensor(**t) for _ in range(max(n, 1))])
    f = np.full(max(rot // 2, 1), 0.5) if isinstance(freq, str) else freq
    return B.lib().nsp_rope(array, n, head_dim, rot, layout, None if f is None else B._ptr(f), magnitude, 0, None)


def test_rope_refusals(B):
    inv, uns = B.NSP_ERR_INVALID_ARG, B.NSP_ERR_UNSUPPORTED
    assert _rope(B) == B.NSP_OK  # no tokens
    assert _rope(B, tensors=0) == B.NSP_OK
    assert _rope(B, x=None, y=None) == B.NSP_OK
    assert _rope(B, tensors=-1) == inv
    assert _rope(B, tensors=65) == uns
    assert _rope(B, freq=None) == inv
    assert _rope(B, rot=0) == inv and _rope(B, rot=3) == inv and _rope(B, rot=130) == inv
    assert _rope(B, head_dim=0, rot=2) == inv
    assert _rope(B, head_dim=2048, rot=514) == uns and _rope(B, head_dim=2048) == uns
    assert _rope(B, layout=2) == inv
    assert _rope(B, magnitude=math.inf) == inv and _rope(B, magnitude=math.nan) == inv
    assert _rope(B, freq=np.array([0.5] * 63 + [math.nan])) == inv
    assert _rope(B, freq=np.array([math.inf] + [0.5] * 63)) == inv
    assert _rope(B, tokens=-1) == inv
    one = dict(tokens=4)
    assert _rope(B, heads=0, **one) == inv
    assert _rope(B, dtype=5, **one) == inv
    assert _rope(B, x=None, **one) == inv and _rope(B, y=None, **one) == inv
    assert _rope(B, x=BUF + 1, **one) == inv  # not on an element
    assert _rope(B, positions=BUF + 4, **one) == inv
    assert _rope(B, x_token_stride=-1, **one) == inv and _rope(B, y_head_stride=2 ** 31 + 1, **one) == inv
    assert _rope(B, y_head_stride=127, **one) == inv  # heads that overlap
    assert _rope(B, y_token_stride=7 * 128 + 127, **one) == inv  # tokens that overlap
    assert _rope(B, y_token_stride=128, y_head_stride=3 * 128 + 127, **one) == inv  # heads in front
    assert _rope(B, y=BUF, x_token_stride=2048, **one) == inv  # in place, with other strides
    assert _rope(B, tokens=2 ** 31) == uns
    assert _rope(B, tokens=2 ** 20, heads=2 ** 11) == uns
    assert _rope(B, heads=65537, **one) == uns


def test_rope_frequencies(B):
    with pytest.raises(B.NspError):
        B.nsp_rope_frequencies(127)
    for bad in (dict(rot_dim=514), dict(rot_dim=0), dict(rot_dim=64, base=1.0), dict(rot_dim=64, base=math.inf), dict(rot_dim=64, kind=9),
                dict(rot_dim=64, kind=1, scale=0.5), dict(rot_dim=64, kind=3, scale=2.0),  # trained_tokens = 0
                dict(rot_dim=64, kind=3, scale=2.0, trained_tokens=4096, fast_turns=1.0, slow_turns=1.0),
                dict(rot_dim=64, kind=3, scale=2.0, trained_tokens=4096, slow_turns=0.0)):
        with pytest.raises(B.NspError):
            B.nsp_rope_frequencies(**bad)
    for rot, base in ((2, 1e4), (64, 1e4), (128, 5e5), (512, 1e6)):
        plain, m = B.nsp_rope_frequencies(rot, base)
        want = base ** (-np.arange(0, rot, 2) / rot)
        np.testing.assert_allclose(plain, want, rtol=1e-14)
        assert m == 1.0
        linear, m = B.nsp_rope_frequencies(rot, base, B.NSP_ROPE_LINEAR, scale=4.0)
        np.testing.assert_allclose(linear, want / 4, rtol=1e-14)
        assert m == 1.0
    stretched, _ = B.nsp_rope_frequencies(128, 1e4, B.NSP_ROPE_BASE, scale=8.0)
    plain, _ = B.nsp_rope_frequencies(128, 1e4)
    assert stretched[0] == 1.0 and abs(stretched[-1] * 8 / plain[-1] - 1) < 1e-12
    parts, m = B.nsp_rope_frequencies(128, 1e6, B.NSP_ROPE_PARTS, scale=8.0, trained_tokens=32768)
    plain, _ = B.nsp_rope_frequencies(128, 1e6)
    turns = 32768 * plain / (2 * math.pi)
    ratio = parts / plain
    assert abs(m - (0.1 * math.log(8.0) + 1)) < 1e-6
    assert (ratio[turns > 40] == 1.0).all() and np.allclose(ratio[turns < 0.8], 1 / 8, rtol=1e-14)
    assert (np.diff(ratio) <= 1e-15).all() and ((ratio > 0.13) & (ratio < 0.99)).any()  # a ramp in between


def _norm(B, which, **change):
    v = dict(x=BUF, y=2 * BUF, dy=4 * BUF, w=None, b=None, mean=8 * BUF, rstd=9 * BUF, dw=16 * BUF, db=None, outer=4, inner=1, dim=256,
             dtype=B.NSP_BF16, w_dtype=B.NSP_F32, kind=B.NSP_NORM_LAYER, eps=1e-5, ws=32 * BUF, ws_bytes=1 << 30, o=256, i=0, yo=256, yi=0)
    v.update(change)
    x, y, dy = B.Rows(v["x"], v["o"], v["i"]), B.Rows(v["y"], v["yo"], v["yi"]), B.Rows(v["dy"], v["o"], v["i"])
    ref = ctypes.byref
    shape = (v["outer"], v["inner"], v["dim"], v["dtype"], v["w_dtype"], v["kind"])
    if which == "fwd":
        return B.lib().nsp_norm_fwd(ref(x), v["w"], v["b"], ref(y), v["mean"], v["rstd"], *shape, v["eps"], None)
    return B.lib().nsp_norm_bwd(ref(x), ref(dy), v["w"], v["mean"], v["rstd"], ref(y), v["dw"], v["db"], *shape, v["ws"], v["ws_bytes"], None)


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_norm_refusals(B, which):
    inv, uns = B.NSP_ERR_INVALID_ARG, B.NSP_ERR_UNSUPPORTED
    call = lambda **k: _norm(B, which, **k)
    assert call(outer=0, dw=None) == B.NSP_OK  # nothing to do
    assert call(outer=-1) == inv and call(inner=0) == inv and call(dim=0) == inv
    assert call(dtype=3) == inv and call(w_dtype=3) == inv and call(kind=2) == inv
    assert call(dim=16385) == uns and call(outer=2 ** 31) == uns and call(outer=2 ** 20, inner=2 ** 11) == uns
    assert call(x=None) == inv and call(y=None) == inv and call(x=BUF + 1) == inv
    assert call(w=BUF + 2) == inv and call(mean=BUF + 2) == inv and call(rstd=BUF + 1) == inv
    assert call(o=-1) == inv and call(o=2 ** 31 + 1) == inv
    assert call(yo=255) == inv  # output rows that overlap
    assert call(inner=4, i=256, o=1024, yi=256, yo=1023) == inv
    assert call(inner=4, i=256, o=1024, yi=255, yo=1024) == inv
    assert call(y=BUF, o=512) == inv  # in place, with other strides
    if which == "fwd":
        assert call(eps=-1.0) == inv and call(eps=math.nan) == inv and call(b=BUF + 2) == inv
    else:
        assert call(dy=None) == inv and call(mean=None) == inv and call(rstd=None) == inv and call(dw=BUF + 2) == inv
        assert call(y=4 * BUF, o=512) == inv  # onto dy, with other strides
        assert call(ws=None) == B.NSP_ERR_WORKSPACE and call(ws=BUF + 8) == B.NSP_ERR_WORKSPACE
        assert call(ws_bytes=2 * 4 * 256 - 1) == B.NSP_ERR_WORKSPACE


def test_norm_workspace(B):
    for bad in ((-1, 8), (8, 0)):
        with pytest.raises(B.NspError):
            B.nsp_norm_bwd_ws_bytes(*bad)
    with pytest.raises(B.NspError):
        B.nsp_norm_bwd_ws_bytes(8, 16385)
    assert B.nsp_norm_bwd_ws_bytes(0, 4096) == 0
    assert B.nsp_norm_bwd_ws_bytes(1, 4096) == 2 * 4 * 4096
    for dim in (1, 64, 128, 1000, 4096, 8191, 16384):  # bounded, whatever the number of rows
        assert B.nsp_norm_bwd_ws_bytes(2 ** 31 - 1, dim) <= 2 * 4 * dim * 148 * 32


def test_binding_refuses_what_is_not_on_the_device(B):
    import torch

    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    f = np.full(64, 0.5)
    with pytest.raises(B.NspError):
        B.nsp_rope(x, x, None, f)
    with pytest.raises(B.NspError):
        B.nsp_rope([x], [x, x], None, f)
    with pytest.raises(B.NspError):
        B.nsp_rope([x], [x], [None], [])
    with pytest.raises(B.NspError):
        B.nsp_norm_fwd(x[:, 0], None, None, x[:, 0], None, None)
    with pytest.raises(B.NspError):
        B.nsp_norm_bwd(x[:, 0], x[:, 0], None, None, None, x[:, 0], None, None, None)
    B.nsp_rope([], [], None, f)
