"""The gated feed-forward block against the definition in 64 bits, there and back: one row to many tiles, odd sizes, strides,
outputs that are not wanted; what lies beside the outputs stays as it was."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    yield binding
    assert binding.nsp_glu_status() == (0, 0, 0, 0)


HALF = 2.0 ** -8  # half a step of bf16


def chain(n):
    """A sum of n products in fp32 on the tensor cores: 16 products are added to the accumulator at a time, each addition off by
    at most a whole step (2^-23) of the sum of magnitudes."""
    return (n / 16 + 16) * 2.0 ** -23


def act64(x, act):
    import math

    import torch

    if act == 0:
        p = torch.sigmoid(x)
        return x * p, p * (1 + x * (1 - p))
    p = 0.5 * torch.erfc(-x / math.sqrt(2))
    return x * p, p + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def near(got, want, bound, what):
    off = (got.double() - want).abs()
    tol = bound + HALF * (want.abs() + bound)
    assert bool((off <= tol).all()), f"{what}: off by {off.max().item():.3g}, {(off / tol.clamp_min(1e-300)).max().item():.3g} of the bound"


def normal(shape, seed, scale=1.0, ld=0):
    import torch

    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape[0], shape[1] + ld, generator=g, device="cuda") * scale).bfloat16()[:, :shape[1]]


class Guarded:
    """Outputs inside a buffer whose other elements must keep their value."""

    def __init__(self):
        self.all = []

    def new(self, rows, cols, more=0):
        import torch

        whole = torch.full((rows + 4, cols + more + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        view = whole[2:2 + rows, 8:8 + cols] if more else torch.as_strided(whole, (rows, cols), (cols, 1), 2 * (cols + 8) // 8 * 8)
        self.all.append((whole, view))
        return view

    def check(self):
        for whole, view in self.all:
            view.fill_(7.0)
            assert bool((whole == 7.0).all())


SIZES = [(1, 8, 8), (5, 128, 14336), (100, 264, 4000), (130, 392, 9480), (17, 2048, 264), (700, 128, 8200), (1, 64, 128), (2, 72, 136), (77, 1024, 2816), (127, 128, 256), (128, 64, 128), (129, 520, 264), (255, 200, 1032),
         (256, 256, 256), (257, 72, 136), (300, 2056, 520), (1000, 512, 1544), (513, 136, 8), (40, 8, 4096), (3, 4104, 24), (2500, 768, 2304),
         (4096, 136, 4736), (6001, 520, 3000), (9000, 136, 1160), (2560, 2568, 2056)]  # the last ones on tiles of 512 rows, one way or both


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("rows,d,f", SIZES)
def test_forward(B, rows, d, f, act):
    forward_case(B, rows, d, f, act, saved=(rows + d) % 3 > 0)


@pytest.mark.parametrize("more", [8, 24])
def test_forward_strides(B, more):
    forward_case(B, 300, 264, 392, 0, saved=True, more=more)


def forward_case(B, rows, d, f, act, saved, more=0):
    x, wg, wu = normal((rows, d), 1, ld=more), normal((f, d), 2, 1.5 * d ** -0.5, more), normal((f, d), 3, d ** -0.5, more)
    out = Guarded()
    h = out.new(rows, f, more)
    g, u = (out.new(rows, f, more), out.new(rows, f, more)) if saved else (None, None)
    B.nsp_glu_fwd(x, wg, wu, h, g, u, act=act)
    g64, u64 = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    e_g = chain(d) * (x.double().abs() @ wg.double().abs().t())
    e_u = chain(d) * (x.double().abs() @ wu.double().abs().t())
    a64, _ = act64(g64, act)
    # the slopes of both activations lie within 1.13; exp, erf and the quotient are good to 2^-20
    e_a = 1.13 * e_g + 2.0 ** -20 * (a64.abs() + g64.abs())
    near(h, a64 * u64, e_a * (u64.abs() + e_u) + a64.abs() * e_u + 2.0 ** -22 * (a64 * u64).abs(), "h")
    if saved:
        near(g, g64, e_g, "g")
        near(u, u64, e_u, "u")
    out.check()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("rows,d,f", SIZES)
def test_backward(B, rows, d, f, act):
    backward_case(B, rows, d, f, act)


@pytest.mark.parametrize("more,want", [(8, "xw"), (24, "xw"), (0, "x"), (0, "w")])
def test_backward_strides_and_outputs(B, more, want):
    backward_case(B, 300, 264, 392, 0, more, want)


def rounded(v, e):
    """(v in bf16, bound on how far the rounding of a value within e of v may be from that). Two roundings that differ are those
    of values at most e apart, each off by half a step at most: e + 2 * 2^-8 (|v| + e). Zero where all of v - e .. v + e rounds
    to the same."""
    r = v.bfloat16()
    differs = ((v + e).bfloat16() != r) | ((v - e).bfloat16() != r)
    return r.double(), differs * (e + 2 * HALF * (v.abs() + e))


def backward_case(B, rows, d, f, act, more=0, want="xw"):
    import torch

    x, wg, wu = normal((rows, d), 1, ld=more), normal((f, d), 2, d ** -0.5, more), normal((f, d), 3, d ** -0.5, more)
    dh, g, u = normal((rows, f), 4, ld=more), normal((rows, f), 5, 1.5, more), normal((rows, f), 6, ld=more)
    out = Guarded()
    dx = out.new(rows, d, more) if "x" in want else None
    dwg, dwu = (out.new(f, d, more), out.new(f, d, more)) if "w" in want else (None, None)
    ws = torch.empty(B.nsp_glu_bwd_ws_bytes(rows, d, f), dtype=torch.uint8, device="cuda")
    B.nsp_glu_bwd(dh, x, wg, wu, g, u, dx, dwg, dwu, ws, act=act)
    g64, u64, h64, x64 = (t.double() for t in (g, u, dh, x))
    value, slope = act64(g64, act)
    dg, mg = rounded(h64 * u64 * slope, 2.0 ** -20 * (h64 * u64).abs() * (1 + g64.abs()))
    du, mu = rounded(h64 * value, 2.0 ** -20 * h64.abs() * (value.abs() + g64.abs()))
    if dx is not None:
        a, b = wg.double(), wu.double()
        bound = chain(2 * f) * (dg.abs() @ a.abs() + du.abs() @ b.abs()) + (mg @ a.abs() + mu @ b.abs())
        near(dx, dg @ a + du @ b, bound, "dx")
    if dwg is not None:
        for got, v, m, what in ((dwg, dg, mg, "dw_gate"), (dwu, du, mu, "dw_up")):
            bound = chain(rows) * (v.abs().t() @ x64.abs()) + m.t() @ x64.abs()
            near(got, v.t() @ x64, bound, what)
    out.check()


def test_no_rows(B):
    import torch

    e = lambda *s: torch.full(s, 5.0, dtype=torch.bfloat16, device="cuda")
    wg, dwg, dwu = e(136, 72), e(136, 72), e(136, 96)[:, :72]
    B.nsp_glu_fwd(e(0, 72), wg, wg, e(0, 136))
    B.nsp_glu_bwd(e(0, 136), e(0, 72), wg, wg, e(0, 136), e(0, 136), e(0, 72), dwg, dwu, None)
    assert not dwg.any() and not dwu.any()
    assert bool((dwu.as_strided((136, 96), (96, 1))[:, 72:] == 5.0).all())


def test_gradients_against_differences(B):
    """Along random directions of x and the weights, in 64 bits: the whole block, from x to sum(h dh)."""
    import torch

    rows, d, f = 200, 136, 264
    x, wg, wu, dh = normal((rows, d), 1), normal((f, d), 2, d ** -0.5), normal((f, d), 3, d ** -0.5), normal((rows, f), 4)
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.nsp_glu_bwd_ws_bytes(rows, d, f), dtype=torch.uint8, device="cuda")
    for act in (0, 1):
        h, g, u, dx, dwg, dwu = e(rows, f), e(rows, f), e(rows, f), e(rows, d), e(f, d), e(f, d)
        B.nsp_glu_fwd(x, wg, wu, h, g, u, act=act)
        B.nsp_glu_bwd(dh, x, wg, wu, g, u, dx, dwg, dwu, ws, act=act)

        def loss(x64, a, b):
            return (act64(x64 @ a.t(), act)[0] * (x64 @ b.t()) * dh.double()).sum().item()

        at = [t.double() for t in (x, wg, wu)]
        for k, grad in enumerate((dx, dwg, dwu)):
            v = torch.randn(grad.shape, generator=torch.Generator("cuda").manual_seed(k), device="cuda", dtype=torch.float64)
            plus, minus = [t.clone() for t in at], [t.clone() for t in at]
            plus[k] += 1e-5 * v
            minus[k] -= 1e-5 * v
            slope = (loss(*plus) - loss(*minus)) / 2e-5
            # g, u, dg, du and the gradient itself are rounded to bf16: five errors of at most 2^-8 (the slope of the slope of
            # either activation lies within 0.8) on the sum of magnitudes of every element
            size = (grad.double().abs() * v.abs()).sum().item()
            inner = size  # their average magnitude is the rounded gradient's own
            assert abs(slope - (grad.double() * v).sum().item()) <= 5 * HALF * inner


def test_rows_keep_to_themselves(B):
    """A row that is not finite spoils its own outputs alone; the rows of the last tile that do not exist spoil nothing."""
    import torch

    x, wg, wu = normal((300, 128), 1), normal((256, 128), 2, 0.1), normal((256, 128), 3, 0.1)
    x[17, 5], x[299, 100] = float("nan"), float("inf")
    h = torch.empty(300, 256, dtype=torch.bfloat16, device="cuda")
    B.nsp_glu_fwd(x, wg, wu, h)
    spoilt = ~torch.isfinite(h).all(1)
    assert spoilt.nonzero().flatten().tolist() == [17, 299]


def test_streams_graphs_and_the_same_bits(B):
    import torch

    rows, d, f = 1300, 392, 1032
    x, wg, wu, dh = normal((rows, d), 1), normal((f, d), 2, 0.05), normal((f, d), 3, 0.05), normal((rows, f), 4)
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    mk = lambda: (e(rows, f), e(rows, f), e(rows, f), e(rows, d), e(f, d), e(f, d))
    ws = torch.empty(B.nsp_glu_bwd_ws_bytes(rows, d, f), dtype=torch.uint8, device="cuda")

    def step(o, stream=None):
        B.nsp_glu_fwd(x, wg, wu, o[0], o[1], o[2], stream=stream)
        B.nsp_glu_bwd(dh, x, wg, wu, o[1], o[2], o[3], o[4], o[5], ws, stream=stream)

    want, got = mk(), mk()
    step(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        step(got, side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    for k in range(3):
        x.copy_(normal((rows, d), 10 + k))
        graph.replay()
        step(want)
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_many_small_calls(B):
    """Launches that follow one another without a wait, of other tile counts and operand layouts."""
    import torch

    ws = torch.empty(B.nsp_glu_bwd_ws_bytes(700, 136, 328), dtype=torch.uint8, device="cuda")
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    sets = []
    for k in range(12):
        rows, d, f = 1 + 97 * k % 700, 8 * (1 + 5 * k % 17), 8 * (1 + 7 * k % 41)
        x, wg, wu, dh = normal((rows, d), k), normal((f, d), 20 + k, 0.1), normal((f, d), 40 + k, 0.1), normal((rows, f), 60 + k)
        sets.append((x, wg, wu, dh, e(rows, f), e(rows, f), e(rows, f), e(rows, d), e(f, d), e(f, d)))

    def go():
        for x, wg, wu, dh, h, g, u, dx, dwg, dwu in sets:
            B.nsp_glu_fwd(x, wg, wu, h, g, u)
            B.nsp_glu_bwd(dh, x, wg, wu, g, u, dx, dwg, dwu, ws)

    go()
    torch.cuda.synchronize()
    want = [[t.clone() for t in s[4:]] for s in sets]
    for _ in range(20):
        go()
    for s, w in zip(sets, want):
        assert all(torch.equal(p, q) for p, q in zip(s[4:], w))
