"""Token-wise operators called as no other test does: rows whose outer axis is the denser one, and two host threads with a stream each."""
import threading

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("outer,inner,dim", [(7, 36, 128), (130, 3, 64), (9, 5, 1024), (4, 300, 520), (3, 3, 16384), (50, 6, 33), (5, 40, 2051), (1, 9, 256), (9, 1, 256)])
def test_heads_in_front_of_tokens(B, outer, inner, dim, kind):
    """[outer, inner] rows that lie in memory as [inner, outer]: the bits are those of the same rows in order."""
    import torch

    g = torch.Generator("cuda").manual_seed(dim)
    rnd = lambda: torch.randn(outer, inner, dim, generator=g, device="cuda").bfloat16()
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    x, dy, w, rows = rnd(), rnd(), torch.randn(dim, generator=g, device="cuda"), outer * inner
    mean, rstd = torch.empty(rows, device="cuda") if kind == 0 else None, torch.empty(rows, device="cuda")
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(dim, device="cuda")
    ws = torch.empty(B.nsp_norm_bwd_ws_bytes(rows, dim), dtype=torch.uint8, device="cuda")
    B.nsp_norm_fwd(x, w, None, y, mean, rstd, kind=kind)
    B.nsp_norm_bwd(x, dy, w, mean, rstd, dx, dw, None, ws, kind=kind)
    x2, dy2, y2, dx2 = turned(x), turned(dy), turned(torch.zeros_like(x)), turned(torch.zeros_like(x))
    mean2, rstd2, dw2 = None if mean is None else torch.empty_like(mean), torch.empty_like(rstd), torch.empty_like(dw)
    B.nsp_norm_fwd(x2, w, None, y2, mean2, rstd2, kind=kind)
    B.nsp_norm_bwd(x2, dy2, w, mean2, rstd2, dx2, dw2, None, ws, kind=kind)
    assert torch.equal(y2, y) and torch.equal(rstd2, rstd) and torch.equal(dx2, dx) and torch.equal(dw2, dw)
    assert mean is None or torch.equal(mean2, mean)
    B.nsp_norm_bwd(x2, dy2, w, mean2, rstd2, x2, dw2, None, ws, kind=kind)  # in place
    assert torch.equal(x2, dx) and torch.equal(dw2, dw)


def test_two_threads_with_a_stream_each(B):
    """Feed-forward block, rotation and norm of two threads at once: the results of one after the other."""
    import torch

    freq, _ = B.nsp_rope_frequencies(128)
    sets = []
    for k, (rows, d, f) in enumerate(((700, 264, 1032), (1500, 512, 520))):
        g = torch.Generator("cuda").manual_seed(k)
        rnd = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).bfloat16()
        e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
        t = {"x": rnd(rows, d), "wg": rnd(f, d, scale=d ** -0.5), "wu": rnd(f, d, scale=d ** -0.5), "dh": rnd(rows, f), "q": rnd(rows, 4 + k, 128),
             "ws": e(B.nsp_glu_bwd_ws_bytes(rows, d, f), dtype=torch.uint8)}
        out = {"n": e(rows, d), "r": e(rows, dtype=torch.float32), "h": e(rows, f), "g": e(rows, f), "u": e(rows, f), "dx": e(rows, d),
               "dwg": e(f, d), "dwu": e(f, d), "q": e(rows, 4 + k, 128)}
        sets.append((t, out, torch.cuda.Stream()))

    def step(t, o, stream):
        B.nsp_rope(t["q"], o["q"], None, freq, stream=stream)
        B.nsp_norm_fwd(t["x"], None, None, o["n"], None, o["r"], kind=B.NSP_NORM_RMS, stream=stream)
        B.nsp_glu_fwd(o["n"], t["wg"], t["wu"], o["h"], o["g"], o["u"], stream=stream)
        B.nsp_glu_bwd(t["dh"], o["n"], t["wg"], t["wu"], o["g"], o["u"], o["dx"], o["dwg"], o["dwu"], t["ws"], stream=stream)

    torch.cuda.synchronize()
    wants = []
    for t, o, stream in sets:
        step(t, o, stream)
        torch.cuda.synchronize()
        wants.append({n: v.clone() for n, v in o.items()})
        for v in o.values():
            v.fill_(7.0)
    torch.cuda.synchronize()
    raised = []

    def go(*args):
        try:
            for _ in range(300):
                step(*args)
        except B.NspError as error:
            raised.append(error)

    threads = [threading.Thread(target=go, args=s) for s in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not raised and B.nsp_glu_status()[0] == 0
    for (_, o, _), want in zip(sets, wants):
        for n in o:
            assert torch.equal(o[n], want[n]), n
