"""Layer norm and RMS norm against the definition in 64 bits, there and back: short and long rows, odd sizes, strides, types, in
place, no parameters, no rows; gradients against differences as well."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32
CHAIN = 48  # additions one behind the other in a sum over a row: 32 of a thread, 5 in a warp, 5 over the warps, and products


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


def forward(x, w, b, eps, layer):
    """((y, its bound), (mean, bound), (rstd, bound)) in 64 bits, y before its rounding."""
    v = x.double()
    mu = v.mean(-1, keepdim=True) if layer else v.new_zeros(v.shape[:-1] + (1,))
    e_mu = CHAIN * U * v.abs().mean(-1, keepdim=True) if layer else 0 * mu
    d = v - mu
    var = (d * d).mean(-1, keepdim=True)
    r = (var + eps) ** -0.5
    # the sum of squares: each (x - mu) off by e_mu and a rounding; sum of 2 d e_mu vanishes with the exact mean, e_mu^2 stays
    e_var = (CHAIN + 4) * U * var + e_mu ** 2 + 2 * U * (v.abs() + mu.abs()).mean(-1, keepdim=True) * d.abs().mean(-1, keepdim=True)
    rel_r = 0.5 * e_var / (var + eps) + 4 * U
    hat = d * r
    w64 = 1.0 if w is None else w.double()
    b64 = 0.0 if b is None else b.double()
    y = hat * w64 + b64
    size = abs(w64) if w is None else w64.abs()
    e_y = size * (r * (e_mu + 2 * U * (v.abs() + mu.abs())) + hat.abs() * (rel_r + 4 * U)) + 2 * U * (y.abs() + (0 if b is None else b64.abs()))
    return (y, e_y), (mu[..., 0], (e_mu + 2 * U * mu.abs())[..., 0]), (r[..., 0], (r * rel_r)[..., 0])


def near(got, want, bound, what):
    """Within the bound and half a step of the output's type."""
    import torch

    half = torch.finfo(got.dtype).eps / 2
    off = (got.double() - want).abs()
    tol = bound + half * (want.abs() + bound)
    assert bool((off <= tol).all()), f"{what}: off by {off.max().item():.3g}, {(off / tol.clamp_min(1e-300)).max().item():.3g} of the bound"


def make(shape, dtype, seed, fused=False, scale=1.5, mean=0.25):
    import torch

    g = torch.Generator("cuda").manual_seed(seed)
    more = list(shape)
    if fused:
        more[-2 if len(shape) == 3 else -1] += 3 if len(shape) == 3 else 16 if fused == 16 else 3
    x = (torch.randn(more, generator=g, device="cuda") * scale + mean).to(dtype)
    return x[:, :shape[1]] if fused and len(shape) == 3 else x[:, :shape[-1]]


def types(name):
    import torch

    return torch.float32 if name == "f32" else torch.bfloat16


DIMS = [1, 7, 64, 72, 128, 136, 200, 256, 257, 500, 512, 520, 1000, 1024, 1032, 2048, 2051, 4096, 4104, 8192, 8200, 8193, 16376, 16384, 16383]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("kind,dtype,w_type,rows", [("layer", "bf16", "f32", 37), ("rms", "bf16", "bf16", 1), ("layer", "f32", "bf16", 5),
                                                    ("rms", "f32", "f32", 700)])
def test_both_ways(B, dim, kind, dtype, w_type, rows):
    one_case(B, (rows, dim), kind, dtype, w_type)


@pytest.mark.parametrize("shape,fused,kind,dtype", [((5, 36, 128), False, "rms", "bf16"), ((77, 10, 64), True, "layer", "bf16"), ((3000, 5, 128), True, "rms", "f32"),
                                                    ((1, 7, 96), True, "layer", "f32"), ((65, 3, 33), True, "rms", "bf16"), ((129, 2048), 16, "layer", "bf16"),
                                                    ((129, 2048), 3, "rms", "bf16"), ((2000, 256), 3, "layer", "f32"), ((20000, 128), False, "layer", "bf16")])
def test_strides_and_heads(B, shape, fused, kind, dtype):
    one_case(B, shape, kind, dtype, "f32", fused=fused)


@pytest.mark.parametrize("weight,bias,grads", [(False, False, False), (True, False, True), (False, True, True), (True, True, False)])
def test_without_parameters(B, weight, bias, grads):
    one_case(B, (33, 384), "layer", "bf16", "bf16", weight=weight, bias=bias, grads=grads)


def test_rows_far_from_zero(B):
    """The variance of rows whose mean is a thousand times their spread."""
    one_case(B, (64, 1536), "layer", "f32", "f32", scale=0.5, mean=600.0)


def one_case(B, shape, kind, dtype, w_type, fused=False, weight=True, bias=True, grads=True, scale=1.5, mean=0.25):
    import torch

    dt, wt, dim, layer = types(dtype), types(w_type), shape[-1], kind == "layer"
    code = B.NSP_NORM_LAYER if layer else B.NSP_NORM_RMS
    x = make(shape, dt, dim, fused, scale, mean)
    w = make((1, dim), wt, 2, scale=0.2, mean=1.0).view(-1) if weight else None
    b = make((1, dim), wt, 3, scale=0.1, mean=0.0).view(-1) if bias else None
    eps = 1e-5
    rows = x.numel() // dim
    guarded = torch.full((x.numel() + 128,), 7.0, dtype=dt, device="cuda")
    y = guarded[64:-64].view(shape)
    mu, r = torch.empty(shape[:-1], device="cuda"), torch.empty(shape[:-1], device="cuda")
    B.nsp_norm_fwd(x, w, b, y, mu if layer else None, r, eps=eps, kind=code)
    (want_y, e_y), (want_mu, e_mu), (want_r, e_r) = forward(x, w, b, eps, layer)
    near(y, want_y, e_y, "y")
    near(r, want_r, e_r, "rstd")
    if layer:
        near(mu, want_mu, e_mu, "mean")
    assert bool((guarded[:64] == 7.0).all()) and bool((guarded[-64:] == 7.0).all())

    # the way back, from the statistics as they are
    dy = make(shape, dt, dim + 1, fused, 1.0, 0.0)
    dx_all = torch.full((x.numel() + 128,), 7.0, dtype=dt, device="cuda")
    dx = dx_all[64:-64].view(shape)
    dw = torch.full((dim,), float("nan"), device="cuda") if grads and weight else None
    db = torch.full((dim,), float("nan"), device="cuda") if grads and bias else None
    ws = torch.empty(max(B.nsp_norm_bwd_ws_bytes(rows, dim), 16), dtype=torch.uint8, device="cuda")
    B.nsp_norm_bwd(x, dy, w, mu if layer else None, r, dx, dw, db, ws if grads else None, kind=code)
    v, g, r64 = x.double(), dy.double(), r.double()[..., None]
    m64 = mu.double()[..., None] if layer else 0 * r64
    h = (v - m64) * r64
    e_h = 3 * U * (v.abs() + m64.abs()) * r64
    t = g * w.double() if weight else g
    c1, c2 = (t * h).mean(-1, keepdim=True), t.mean(-1, keepdim=True) if layer else 0 * r64
    e_c1 = (CHAIN + 6) * U * (t * h).abs().mean(-1, keepdim=True) + (t.abs() * e_h).mean(-1, keepdim=True)
    e_c2 = (CHAIN + 4) * U * t.abs().mean(-1, keepdim=True)
    bound = r64 * (U * (4 * t.abs() + 4 * c2.abs() + 6 * (h * c1).abs()) + e_c2 + h.abs() * e_c1 + c1.abs() * e_h)
    near(dx, r64 * (t - h * c1 - c2), bound, "dx")
    assert bool((dx_all[:64] == 7.0).all()) and bool((dx_all[-64:] == 7.0).all())
    every = tuple(range(x.dim() - 1))
    chain = rows / 148 + 300  # of a team's rows, of a block's teams, of the blocks: each less than that many additions
    if dw is not None:
        near(dw, (g * h).sum(every), (chain * U * (g * h).abs() + g.abs() * e_h).sum(every), "dweight")
    if db is not None:
        near(db, g.sum(every), chain * U * g.abs().sum(every), "dbias")


@pytest.mark.parametrize("dim", [128, 1000, 2051])
def test_in_place_and_the_same_bits(B, dim):
    import torch

    x, dy = make((300, dim), torch.bfloat16, 1), make((300, dim), torch.bfloat16, 2)
    w, b = torch.randn(dim, device="cuda"), torch.randn(dim, device="cuda")
    y, mu, r = torch.empty_like(x), torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    B.nsp_norm_fwd(x, w, b, y, mu, r)
    z = x.clone()
    B.nsp_norm_fwd(z, w, b, z, None, None)
    assert torch.equal(y, z)
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(300, dim), dtype=torch.uint8, device="cuda")
    first = None
    for into in ("dx", "x", "dy", "dx"):
        xx, gg = x.clone(), dy.clone()
        dx = {"dx": torch.empty_like(x), "x": xx, "dy": gg}[into]
        dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
        ws.fill_(255)
        B.nsp_norm_bwd(xx, gg, w, mu, r, dx, dw, db, ws)
        got = (dx.clone(), dw, db)
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(got, first))


def test_no_rows(B):
    import torch

    x = torch.empty(0, 256, device="cuda")
    B.nsp_norm_fwd(x, None, None, x, None, None)
    dw, db = torch.full((256,), 5.0, device="cuda"), torch.full((256,), 5.0, device="cuda")
    B.nsp_norm_bwd(x, x, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), x, dw, db, None)
    assert not dw.any() and not db.any()  # sums over nothing


def test_zero_rows_and_values_that_are_not_finite(B):
    """Rows of zeros give zeros (and the bias); a row that is not finite spoils itself and, in the parameters' gradients, its columns."""
    import torch

    x = torch.randn(50, 640, device="cuda").bfloat16()
    x[7] = 0
    x[9, 3] = float("inf")
    x[11, 600] = float("nan")
    b = torch.randn(640, device="cuda")
    y, mu, r = torch.empty_like(x), torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    B.nsp_norm_fwd(x, None, b, y, mu, r)
    assert torch.equal(y[7], b.bfloat16())
    spoilt = ~torch.isfinite(y).all(1)
    assert spoilt.nonzero().flatten().tolist() == [9, 11]


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradients_against_differences(B, kind):
    """Along random directions of x, w and b: central differences of the definition in 64 bits, against the kernel's gradients."""
    import torch

    shape, dim, layer = (40, 352), 352, kind == "layer"
    code = B.NSP_NORM_LAYER if layer else B.NSP_NORM_RMS
    x, dy = make(shape, torch.float32, 5), make(shape, torch.float32, 6, scale=1.0, mean=0.0)
    w, b = make((1, dim), torch.float32, 7, scale=0.2, mean=1.0).view(-1), make((1, dim), torch.float32, 8).view(-1)
    y, mu, r = torch.empty_like(x), torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    B.nsp_norm_fwd(x, w, b, y, mu if layer else None, r, kind=code)
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(40, dim), dtype=torch.uint8, device="cuda")
    B.nsp_norm_bwd(x, dy, w, mu if layer else None, r, dx, dw, db, ws, kind=code)

    def loss(x64, w64, b64):
        m = x64.mean(-1, keepdim=True) if layer else 0.0
        d = x64 - m
        return ((d * ((d * d).mean(-1, keepdim=True) + 1e-5) ** -0.5 * w64 + b64) * dy.double()).sum().item()

    at = [t.double() for t in (x, w, b)]
    for k, grad in enumerate((dx, dw, db)):
        v = torch.randn(grad.shape, generator=torch.Generator("cuda").manual_seed(k), device="cuda", dtype=torch.float64)
        h = 1e-5
        plus, minus = [t.clone() for t in at], [t.clone() for t in at]
        plus[k] += h * v
        minus[k] -= h * v
        slope = (loss(*plus) - loss(*minus)) / (2 * h)
        # the difference: h^2 (third derivative, of order one per element) and 2^-52 / h of the loss; the gradient: fp32
        size = (grad.double().abs() * v.abs()).sum().item()
        assert abs(slope - (grad.double() * v).sum().item()) <= 1e-5 * size


def test_streams_and_graphs(B):
    import torch

    x, dy = make((500, 1024), torch.bfloat16, 1), make((500, 1024), torch.bfloat16, 2)
    w = torch.randn(1024, device="cuda")
    mk = lambda: (torch.empty_like(x), torch.empty(500, device="cuda"), torch.empty(500, device="cuda"), torch.empty_like(x),
                  torch.empty(1024, device="cuda"), torch.empty(1024, device="cuda"))
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(500, 1024), dtype=torch.uint8, device="cuda")

    def step(o, stream=None):
        B.nsp_norm_fwd(x, w, w, o[0], o[1], o[2], stream=stream)
        B.nsp_norm_bwd(x, dy, w, o[1], o[2], o[3], o[4], o[5], ws, stream=stream)

    want, got = mk(), mk()
    step(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(got, side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    for k in range(3):
        x.copy_(make((500, 1024), torch.bfloat16, 10 + k))
        graph.replay()
        step(want)
        assert all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("dim", [129, 300, 2051, 4104, 5511, 16383])
def test_in_place_with_many_rows_to_a_block(B, dim, kind):
    """Rows of 2,051 bf16 share their 16-byte pieces with neighbours that other blocks write."""
    import torch

    rows = 4000
    x, dy = make((rows, dim), torch.bfloat16, 1), make((rows, dim), torch.bfloat16, 2)
    w = torch.randn(dim, device="cuda")
    y, mu, r = torch.empty_like(x), torch.empty(rows, device="cuda") if kind == 0 else None, torch.empty(rows, device="cuda")
    B.nsp_norm_fwd(x, w, w, y, mu, r, kind=kind)
    z = x.clone()
    B.nsp_norm_fwd(z, w, w, z, None, None, kind=kind)
    assert torch.equal(y, z)
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(rows, dim), dtype=torch.uint8, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    B.nsp_norm_bwd(x, dy, w, mu, r, dx, dw, db, ws, kind=kind)
    for onto_x in (True, False):
        xx, gg, dw2, db2 = x.clone(), dy.clone(), torch.empty_like(dw), torch.empty_like(db)
        into = xx if onto_x else gg
        B.nsp_norm_bwd(xx, gg, w, mu, r, into, dw2, db2, ws, kind=kind)
        assert torch.equal(into, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_sizes_beyond_32_bits_are_refused(B):
    """A size that 32 bits cut to a small one must not become a call with that one."""
    import torch

    x = torch.zeros(1, 1, 8, device="cuda").expand(1, 2 ** 32 + 1, 8)
    w = torch.ones(8, device="cuda")
    for call in (lambda: B.nsp_norm_fwd(x, w, None, x, None, None), lambda: B.nsp_rope([x], [x], None, [0.5, 0.25]),
                 lambda: B.nsp_norm_fwd(x[0], w, None, x[0], None, None)):
        with pytest.raises(B.NspError):
            call()


@pytest.mark.parametrize("dim", [8320, 11000, 12288, 12296])
@pytest.mark.parametrize("kind,dtype,w_type,rows", [("layer", "bf16", "f32", 700), ("rms", "bf16", "bf16", 149), ("layer", "f32", "bf16", 300)])
def test_rows_between_two_and_four_vectors_of_a_thread(B, dim, kind, dtype, w_type, rows):
    one_case(B, (rows, dim), kind, dtype, w_type)
