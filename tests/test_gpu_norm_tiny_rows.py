"""Gradients of norms of rows so small that 1 / rstd^2 has no normal number in fp32 (eps = 0): rstd itself and the gradients have."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 136, 512, 1024, 4096, 8320, 16384, 129, 2051])
def test_gradients_of_tiny_rows(B, dim, dtype, kind):
    """Rows of order 2^-72 to 2^-40, of statistics in 64 bits rounded to fp32 (of tiny rows the sum of squares has few bits in fp32)."""
    import torch

    dt, layer = torch.float32 if dtype == "f32" else torch.bfloat16, kind == "layer"
    g = torch.Generator("cuda").manual_seed(dim)
    scale = 2.0 ** -torch.arange(40, 73, 4, device="cuda", dtype=torch.float32)
    x = (torch.randn(len(scale), dim, generator=g, device="cuda") * scale[:, None]).to(dt)
    dy, w = torch.randn(x.shape, generator=g, device="cuda").to(dt), torch.randn(dim, generator=g, device="cuda")
    v = x.double()
    mean = v.mean(-1).float() if layer else None
    m = mean.double()[:, None] if layer else 0.0
    rstd = ((v - m).square().mean(-1) ** -0.5).float()
    dx, dw = torch.empty_like(x), torch.empty(dim, device="cuda")
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(len(x), dim), dtype=torch.uint8, device="cuda")
    B.nsp_norm_bwd(x, dy, w, mean, rstd, dx, dw, None, ws, kind=B.NSP_NORM_LAYER if layer else B.NSP_NORM_RMS)
    r = rstd.double()[:, None]
    h, t = (v - m) * r, dy.double() * w.double()
    c1, c2 = (t * h).mean(-1, keepdim=True), t.mean(-1, keepdim=True) if layer else 0.0 * r
    want = r * (t - h * c1 - c2)
    # h has three roundings (the difference, its size and the product), t one, the means 48 additions one behind the other at most, of
    # products with four roundings; two sums and a product behind them
    e_h = 3 * U * (v.abs() + abs(m)) * r
    e_c1 = 54 * U * (t * h).abs().mean(-1, keepdim=True) + (t.abs() * e_h).mean(-1, keepdim=True)
    e_c2 = 52 * U * t.abs().mean(-1, keepdim=True)
    bound = r * (U * (4 * t.abs() + 4 * c2.abs() + 6 * (h * c1).abs()) + e_c2 + h.abs() * e_c1 + c1.abs() * e_h)
    off, half = (dx.double() - want).abs(), torch.finfo(dt).eps / 2
    assert bool((off <= bound + half * (want.abs() + bound)).all())
    g64 = dy.double()
    assert bool(((dw.double() - (g64 * h).sum(0)).abs() <= (len(x) * U * (g64 * h).abs() + g64.abs() * e_h).sum(0)).all())
