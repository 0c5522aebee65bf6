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
