"""Norms of rows that lie far from zero: where every element is the row's mean, the centred row is zero, whatever the reciprocal of the
standard deviation makes of a rounding."""
import pytest

pytestmark = pytest.mark.gpu

# aligned rows of every number of lanes, warps and vectors, and unaligned ones of a warp and of a block
DIMS = [8, 64, 72, 128, 200, 256, 400, 512, 1000, 1024, 2048, 2056, 4096, 5504, 8192, 8320, 12288, 16384, 7, 129, 257, 2051, 5511, 16383]


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


def constant_rows(dim, dtype):
    """Constants of at most 8 significant bits: any number up to 16,384 of them adds up exactly in fp32 (22 bits), in any order, the
    quotient by that number is the constant, and so the mean has no rounding. Above 2^112 a row of at most 300 stays in fp32."""
    import torch

    values = [1000.0, -1000.0, 3.0, 0.0, -255.0, 2.0 ** 20, 129.0 * 2 ** 90]
    if dim <= 300:
        values += [2.0 ** 118, -(2.0 ** 119)]  # times 316 = 1 / sqrt(1e-5) they leave fp32
    return torch.tensor(values, device="cuda", dtype=dtype)[:, None].expand(-1, dim).contiguous()


def types(name):
    import torch

    return torch.float32 if name == "f32" else torch.bfloat16


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", DIMS)
def test_constant_rows_are_centred_to_zero(B, dim, dtype):
    import torch

    x = constant_rows(dim, types(dtype))
    g = torch.Generator("cuda").manual_seed(dim)
    w, b = (torch.randn(dim, generator=g, device="cuda") for _ in range(2))
    y, mean, rstd = torch.empty_like(x), torch.empty(len(x), device="cuda"), torch.empty(len(x), device="cuda")
    B.nsp_norm_fwd(x, w, b, y, mean, rstd)
    assert torch.equal(mean, x[:, 0].float())
    assert torch.equal(y, b.to(x.dtype).expand_as(y))  # 0 w + b
    # 1 / sqrt(eps) with the roundings of 1e-5 to fp32, of the root and of the quotient
    assert bool(((rstd.double() * 1e-5 ** 0.5 - 1).abs() <= 3 * 2.0 ** -24).all())


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", DIMS)
def test_gradients_of_constant_rows(B, dim, dtype, eps):
    """h = 0: such rows add nothing to dweight, and dx = rstd (t - mean(t)), also where mean * rstd leaves fp32 (2^110 * 10^6)."""
    import torch

    U, dt = 2.0 ** -24, types(dtype)
    x = torch.cat([constant_rows(dim, dt), torch.full((1, dim), 2.0 ** 110, device="cuda", dtype=dt)])
    g = torch.Generator("cuda").manual_seed(dim)
    dy, w = torch.randn(x.shape, generator=g, device="cuda").to(dt), torch.randn(dim, generator=g, device="cuda")
    mean, rstd = x[:, 0].float().contiguous(), torch.full((len(x),), eps ** -0.5, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(len(x), dim), dtype=torch.uint8, device="cuda")
    B.nsp_norm_bwd(x, dy, w, mean, rstd, dx, dw, db, ws)
    assert torch.equal(dw, torch.zeros_like(dw))
    t, r = dy.double() * w.double(), rstd.double()[:, None]
    c2 = t.mean(-1, keepdim=True)
    want = r * (t - c2)
    # t, its difference from the mean and the product with rstd are rounded once each; the mean is a sum of 48 additions one behind the
    # other at most (32 of a thread, 5 in a warp, 5 over the warps, and products)
    bound = r * U * (4 * t.abs() + 4 * c2.abs() + 52 * t.abs().mean(-1, keepdim=True))
    off, half = (dx.double() - want).abs(), torch.finfo(dt).eps / 2
    assert bool((off <= bound + half * (want.abs() + bound)).all())
    assert bool(((db.double() - dy.double().sum(0)).abs() <= len(x) * U * dy.double().abs().sum(0)).all())
