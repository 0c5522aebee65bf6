"""Rotary positions against the definition in 64 bits: layouts, part of the head, types, strides, far positions, several tensors,
in place; what lies beside the outputs stays as it was."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


def reference(x, pos, freq, layout, magnitude, inverse):
    """(result, bound on a kernel's error) in 64 bits. The angle in fp32 turns is off by at most 2^-24 of half a turn (3.15 *
    2^-24 radians) and 2^-32 of a turn, sine and cosine by 2^-23 each, their factor and the two products and the sum by 2^-24
    each: together below 8 * 2^-24 * |magnitude| (|a| + |b|); then half a step of the output's type."""
    import torch

    rot = 2 * len(freq)
    f = torch.as_tensor(freq, dtype=torch.float64, device=x.device)
    p = torch.arange(x.shape[0], device=x.device) if pos is None else pos
    # p * f modulo whole turns in 128 bits: the product of doubles loses far positions
    turns = np.array([[(int(a) * b) % 1 for b in _exact_turns(freq)] for a in p.cpu().tolist()], dtype=np.float64).reshape(len(p), rot // 2)
    angle = 2 * np.pi * torch.as_tensor(turns, device=x.device)[:, None]
    del f
    c, s = magnitude * torch.cos(angle), magnitude * torch.sin(angle) * (-1 if inverse else 1)
    v = x.double()
    a, b = (v[..., :rot // 2], v[..., rot // 2:rot]) if layout == 0 else (v[..., 0:rot:2], v[..., 1:rot:2])
    u, w = a * c - b * s, b * c + a * s
    out, tol = v.clone(), torch.zeros_like(v)
    size = 8 * 2.0 ** -24 * abs(magnitude) * (a.abs() + b.abs())
    eps = torch.finfo(x.dtype).eps / 2
    for half, value in ((0, u), (1, w)):
        at = slice(half * rot // 2, (half + 1) * rot // 2) if layout == 0 else slice(half, rot, 2)
        out[..., at], tol[..., at] = value, size + eps * (value.abs() + size)
    return out, tol


def _exact_turns(freq):
    from fractions import Fraction

    # pi to 60 digits
    pi = Fraction(3141592653589793238462643383279502884197169399375105820974945, 10 ** 60)
    return [Fraction(float(f)) / (2 * pi) for f in freq]


def check(y, want):
    import torch

    out, tol = want
    off = (y.double() - out).abs()
    assert bool((off <= tol).all()), f"{(off - tol).max().item():.3g} over the bound"
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("head_dim,rot", [(128, 128), (64, 64), (128, 64), (128, 24), (96, 40), (72, 58), (2, 2), (80, 80), (256, 200), (5, 4)])
@pytest.mark.parametrize("tokens,heads,dtype", [(1, 1, "bf16"), (37, 9, "bf16"), (129, 4, "f32"), (3, 33, "f32")])
def test_against_the_definition(B, layout, head_dim, rot, tokens, heads, dtype):
    import torch

    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(tokens * 1000 + rot)
    x = torch.randn(tokens, heads, head_dim, generator=g, device="cuda").to(dt)
    pos = torch.randint(0, 400000, (tokens,), generator=g, device="cuda")
    freq, _ = B.nsp_rope_frequencies(rot, 1e6)
    for inverse in (False, True):
        guarded = torch.full((tokens * heads * head_dim + 128,), 7.0, dtype=dt, device="cuda")
        y = guarded[64:-64].view(x.shape)
        B.nsp_rope(x, y, pos, freq, layout=layout, magnitude=1.25, inverse=inverse)
        check(y, reference(x, pos, freq, layout, 1.25, inverse))
        assert torch.equal(y[..., rot:], x[..., rot:])  # the rest as it is, bit for bit
        assert bool((guarded[:64] == 7.0).all()) and bool((guarded[-64:] == 7.0).all())


@pytest.mark.parametrize("layout", [0, 1])
def test_far_positions(B, layout):
    import torch

    pos = torch.tensor([0, 1, -1, 393215, 2 ** 24 + 1, 2 ** 31 - 1, 2 ** 31, -2 ** 31, 2 ** 40 + 12345], device="cuda")
    x = torch.randn(len(pos), 3, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    freq = np.concatenate([B.nsp_rope_frequencies(60)[0], [0.0, -0.7]])
    y = torch.empty_like(x)
    B.nsp_rope(x, y, pos, freq, layout=layout)
    check(y, reference(x, pos, freq, layout, 1.0, False))


@pytest.mark.parametrize("dtype,off,token_more,head_more", [("bf16", 0, 0, 0), ("bf16", 4, 0, 0), ("bf16", 1, 8, 0), ("f32", 2, 3, 4), ("f32", 1, 0, 1),
                                                           ("bf16", 0, 4, 4), ("bf16", 0, 8, 8)])
def test_strides_and_alignment(B, dtype, off, token_more, head_more):
    import torch

    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    T, H, D = 41, 6, 128
    head = D + head_more
    token = H * head + token_more
    whole = torch.randn(off + T * token, device="cuda", generator=torch.Generator("cuda").manual_seed(off)).to(dt)
    x = whole.as_strided((T, H, D), (token, head, 1), off)
    into = torch.full_like(whole, 7.0)
    y = into.as_strided((T, H, D), (token, head, 1), off)
    freq, _ = B.nsp_rope_frequencies(96)
    B.nsp_rope(x, y, None, freq)
    want = reference(x, None, freq, 0, 1.0, False)
    check(y, want)
    y.fill_(7.0)
    assert bool((into == 7.0).all())  # nothing outside the view was written
    # heads in front of tokens, an input that every token shares, and in place
    z = torch.empty(H, T, D, dtype=dt, device="cuda").transpose(0, 1)
    B.nsp_rope(x, z, None, freq)
    check(z, want)
    B.nsp_rope(x[:1].expand(T, H, D), z, None, freq)
    check(z, reference(x[:1].expand(T, H, D), None, freq, 0, 1.0, False))
    before = whole.clone()
    B.nsp_rope(x, x, None, freq)
    check(x, want)
    x.copy_(before.as_strided((T, H, D), (token, head, 1), off))
    assert torch.equal(whole, before)


def test_many_tensors_in_one_launch(B):
    """64 tensors of a chain: other lengths (none, one), head counts and types, with positions of their own."""
    import torch

    g = torch.Generator("cuda").manual_seed(1)
    freq, _ = B.nsp_rope_frequencies(64)
    xs, ys, ps = [], [], []
    for i in range(64):
        T, H = [0, 1, 5, 130, 700][i % 5], [1, 2, 5, 32][i % 4]
        x = torch.randn(T, H, 64, generator=g, device="cuda").to([torch.bfloat16, torch.float32][i % 2])
        xs.append(x), ys.append(torch.empty_like(x)), ps.append(torch.randint(0, 9000, (T,), generator=g, device="cuda") if i % 3 else None)
    before = B.launch_count()
    B.nsp_rope(xs, ys, ps, freq, layout=B.NSP_ROPE_INTERLEAVED)
    assert B.launch_count() - before == 1
    for x, y, p in zip(xs, ys, ps):
        if x.numel():
            check(y, reference(x, p, freq, 1, 1.0, False))
    with pytest.raises(B.NspError):
        B.nsp_rope(xs + xs[1:2], ys + ys[1:2], ps + ps[1:2], freq)


def test_large_and_the_way_back(B):
    """Sizes that take several heads a thread; the inverse undoes the rotation and is its adjoint: <R x, z> = <x, R' z>."""
    import torch

    T, g = 20011, torch.Generator("cuda").manual_seed(9)
    freq, _ = B.nsp_rope_frequencies(128)
    for H, layout in ((32, 0), (5, 1), (7, 0)):
        x = torch.randn(T, H, 128, generator=g, device="cuda")
        z = torch.randn(T, H, 128, generator=g, device="cuda")
        y, back, zb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(z)
        B.nsp_rope(x, y, None, freq, layout=layout)
        B.nsp_rope(y, back, None, freq, layout=layout, inverse=True)
        # twice the bound of one rotation, on |a| + |b| <= 2 max
        assert (back - x).abs().max().item() <= 2 * 9 * 2.0 ** -24 * 2 * x.abs().max().item()
        B.nsp_rope(z, zb, None, freq, layout=layout, inverse=True)
        lhs, rhs = (y.double() * z).sum().item(), (x.double() * zb).sum().item()
        size = (y.double().abs() * z.abs()).sum().item()
        assert abs(lhs - rhs) <= 2 * 9 * 2.0 ** -24 * 2 * size
        at = torch.cat([torch.arange(40), torch.arange(T - 40, T)]).cuda()
        check(y[at], reference(x[at], at, freq, layout, 1.0, False))


def test_streams_and_graphs(B):
    import torch

    freq, _ = B.nsp_rope_frequencies(128)
    x = torch.randn(3000, 8, 128, device="cuda")
    want, y = torch.empty_like(x), torch.zeros_like(x)
    B.nsp_rope(x, want, None, freq)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.nsp_rope(x, y, None, freq)  # the current stream
    side.synchronize()
    assert torch.equal(y, want)
    y.zero_()
    torch.cuda.synchronize()
    B.nsp_rope(x, y, None, freq, stream=side)  # a named one
    side.synchronize()
    assert torch.equal(y, want)
    graph, other = torch.cuda.CUDAGraph(), freq.copy()
    with torch.cuda.graph(graph):
        B.nsp_rope(x, y, None, other)
        B.nsp_rope(y, y, None, other, inverse=True)
        B.nsp_rope(y, y, None, other)
    other[:] = 0.0  # the captured calls keep their values
    for k in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator("cuda").manual_seed(k), device="cuda"))
        graph.replay()
        B.nsp_rope(x, want, None, freq)
        # three rotations in a row
        assert (y - want).abs().max().item() <= 3 * 9 * 2.0 ** -24 * 2 * x.abs().max().item()


def test_values_that_are_not_finite_stay_in_their_pairs(B):
    import torch

    freq, _ = B.nsp_rope_frequencies(64)
    x = torch.ones(9, 5, 128, dtype=torch.bfloat16, device="cuda")
    x[4, 2, 7], x[5, 1, 100], x[0, 0, 40] = float("inf"), float("nan"), float("-inf")
    y = torch.empty_like(x)
    B.nsp_rope(x, y, None, freq)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[4, 2, [7, 39]] = True
    want[0, 0, [8, 40]] = True
    want[5, 1, 100] = True
    assert torch.equal(bad, want)
