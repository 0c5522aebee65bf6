"""The operators together, as a layer of a nested shard runs them: norm, projections (plain torch), norms of the heads, rotation,
packed attention, norm, gated feed-forward block, there and back, against the same layer in 64 bits with autograd."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

D, DM, FF = 128, 256, 520


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


class Layer:
    """One node of a chain: segments of one head structure, packed."""

    def __init__(self, lengths, hq, hkv, seed):
        import torch

        from paper_2609_22755_b200 import binding as B
        from paper_2609_22755_b200 import workloads as W
        from paper_2609_22755_b200.api import NspAttention, Rotary

        self.B, self.t, self.hq, self.hkv, self.lengths = B, torch, hq, hkv, lengths
        self.T = sum(lengths)
        g = torch.Generator("cuda").manual_seed(seed)
        rnd = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).bfloat16()
        self.x, self.dout = rnd(self.T, DM), rnd(self.T, FF)
        self.p = {"n1": rnd(DM, scale=0.1) + 1, "wqkv": rnd((hq + 2 * hkv) * D, DM, scale=DM ** -0.5), "nq": rnd(D, scale=0.1) + 1,
                  "nk": rnd(D, scale=0.1) + 1, "wo": rnd(DM, hq * D, scale=(hq * D) ** -0.5), "n2": rnd(DM, scale=0.1) + 1,
                  "wg": rnd(FF, DM, scale=DM ** -0.5), "wu": rnd(FF, DM, scale=DM ** -0.5)}
        self.att = NspAttention(W.custom(lengths, [hq] * len(lengths), [hkv] * len(lengths)), dkv_dtype="bf16", rope=Rotary(D, 1e4))

    def step(self):
        """Loss gradients by the library: (out, dx, gradients of the parameters)."""
        B, t, p, T, a = self.B, self.t, self.p, self.T, self.att
        e = lambda *s, dtype=t.bfloat16: t.empty(s, dtype=dtype, device="cuda")
        f32 = t.float32
        n1, r1 = e(T, DM), e(T, dtype=f32)
        B.nsp_norm_fwd(self.x, p["n1"], None, n1, None, r1, kind=B.NSP_NORM_RMS)
        qkv = (n1 @ p["wqkv"].t()).view(T, self.hq + 2 * self.hkv, D)
        q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]
        qn, kn = a.q.view(T, self.hq, D), a.k.view(T, self.hkv, D)
        rq, rk = e(T, self.hq, dtype=f32), e(T, self.hkv, dtype=f32)
        B.nsp_norm_fwd(q, p["nq"], None, qn, None, rq, kind=B.NSP_NORM_RMS)  # views into the joint projection
        B.nsp_norm_fwd(k, p["nk"], None, kn, None, rk, kind=B.NSP_NORM_RMS)
        a.v.view(T, self.hkv, D).copy_(v)
        a.forward()
        x2 = self.x + a.o.view(T, -1) @ p["wo"].t()
        n2, mu2, r2 = e(T, DM), e(T, dtype=f32), e(T, dtype=f32)
        B.nsp_norm_fwd(x2, p["n2"], None, n2, mu2, r2)
        h, gate, up = e(T, FF), e(T, FF), e(T, FF)
        B.nsp_glu_fwd(n2, p["wg"], p["wu"], h, gate, up)
        # back
        grads = {}
        ws = t.empty(max(B.nsp_glu_bwd_ws_bytes(T, DM, FF), B.nsp_norm_bwd_ws_bytes(T * self.hq, DM)), dtype=t.uint8, device="cuda")
        dn2, grads["wg"], grads["wu"] = e(T, DM), e(FF, DM), e(FF, DM)
        B.nsp_glu_bwd(self.dout, n2, p["wg"], p["wu"], gate, up, dn2, grads["wg"], grads["wu"], ws)
        dx2, grads["n2"] = e(T, DM), e(DM, dtype=f32)
        B.nsp_norm_bwd(x2, dn2, p["n2"], mu2, r2, dx2, grads["n2"], None, ws)
        a.do.view(T, -1).copy_(dx2 @ p["wo"])
        grads["wo"] = dx2.t() @ a.o.view(T, -1)
        a.backward()
        dqkv = e(T, self.hq + 2 * self.hkv, D)
        grads["nq"], grads["nk"] = e(D, dtype=f32), e(D, dtype=f32)
        B.nsp_norm_bwd(q, a.dq.view(T, self.hq, D), p["nq"], None, rq, dqkv[:, :self.hq], grads["nq"], None, ws, kind=B.NSP_NORM_RMS)
        B.nsp_norm_bwd(k, a.dk.view(T, self.hkv, D), p["nk"], None, rk, dqkv[:, self.hq:self.hq + self.hkv], grads["nk"], None, ws,
                       kind=B.NSP_NORM_RMS)
        dqkv[:, self.hq + self.hkv:].copy_(a.dv.view(T, self.hkv, D))
        dqkv = dqkv.view(T, -1)
        dn1, grads["wqkv"] = dqkv @ p["wqkv"], dqkv.t() @ n1
        dx, grads["n1"] = e(T, DM), e(DM, dtype=f32)
        B.nsp_norm_bwd(self.x, dn1, p["n1"], None, r1, dx, grads["n1"], None, ws, kind=B.NSP_NORM_RMS)
        return h, dx + dx2, grads

    def exact(self):
        t = self.t
        x = self.x.double().requires_grad_()
        p = {k: v.double().requires_grad_() for k, v in self.p.items()}
        rms = lambda z, w: z * (z.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w
        pos = t.cat([t.arange(n, device="cuda") for n in self.lengths]).double()
        angle = pos[:, None] * (1e4 ** (-t.arange(0, D, 2, device="cuda").double() / D))
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        turn = lambda z: t.cat([z[..., :D // 2] * c - z[..., D // 2:] * s, z[..., D // 2:] * c + z[..., :D // 2] * s], -1)
        qkv = (rms(x, p["n1"]) @ p["wqkv"].t()).view(self.T, -1, D)
        q, k, v = turn(rms(qkv[:, :self.hq], p["nq"])), turn(rms(qkv[:, self.hq:self.hq + self.hkv], p["nk"])), qkv[:, self.hq + self.hkv:]
        outs, at = [], 0
        for n in self.lengths:
            qs, ks, vs = (z[at:at + n].transpose(0, 1) for z in (q, k, v))
            ks, vs = (z.repeat_interleave(self.hq // self.hkv, 0) for z in (ks, vs))
            score = qs @ ks.transpose(1, 2) / math.sqrt(D)
            score = score.masked_fill(t.ones(n, n, dtype=t.bool, device="cuda").triu(1), -math.inf)
            outs.append((score.softmax(-1) @ vs).transpose(0, 1))
            at += n
        x2 = x + t.cat(outs).reshape(self.T, -1) @ p["wo"].t()
        m = x2 - x2.mean(-1, keepdim=True)
        n2 = m * (m.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * p["n2"]
        g = n2 @ p["wg"].t()
        h = g * t.sigmoid(g) * (n2 @ p["wu"].t())
        (h * self.dout.double()).sum().backward()
        return h.detach(), x.grad, {k: v.grad for k, v in p.items()}


# Of the ten to sixteen tensors between an input and a gradient each is rounded to bf16 once, by at most 2^-8 of its value; carried on
# by maps whose gain in the 2-norm is about one (norms, projections of random weights, the softmax of scores of order one), the
# rounding of every one of them adds at most that much of the result's norm.
BOUND = 16 * 2.0 ** -8


@pytest.mark.parametrize("lengths,hq,hkv", [([70, 1, 129, 300], 4, 2), ([513], 2, 1), ([16] * 20, 4, 4)])
def test_a_layer_there_and_back(B, lengths, hq, hkv):
    layer = Layer(lengths, hq, hkv, seed=len(lengths))
    out, dx, grads = layer.step()
    want_out, want_dx, want = layer.exact()
    far = lambda got, w: ((got.double() - w).norm() / w.norm()).item()
    assert far(out, want_out) <= BOUND
    assert far(dx, want_dx) <= BOUND
    for name, g in grads.items():
        assert far(g, want[name]) <= BOUND, name


def test_captured_and_on_another_stream(B):
    """The same bits from a replayed graph and from a side stream."""
    import torch

    layer = Layer([200, 57], 4, 2, seed=9)
    want = layer.step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer.step()  # warm-up of the capture's library calls
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.step()
    x = layer.x.clone()
    layer.x.zero_()
    graph.replay()
    layer.x.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    # dQ is a sum in arrival order (1e-5 in fp32, rounded to bf16 behind it): what lies behind it is compared within that
    assert torch.equal(got[0], want[0]) and torch.equal(got[2]["wg"], want[2]["wg"]) and torch.equal(got[2]["n2"], want[2]["n2"])
    assert ((got[1].double() - want[1].double()).norm() / want[1].double().norm()).item() <= 2.0 ** -8


@pytest.mark.parametrize("recompute", [False, True])
def test_attention_with_rope(B, recompute):
    """NspAttention(rope=...) over a chain of two nodes is the rotation, the attention and the rotation back by hand; positions of one's
    own shift nothing but the angles."""
    import torch

    from paper_2609_22755_b200 import workloads as W
    from paper_2609_22755_b200.api import NspAttention, Rotary

    w = W.custom([300, 128, 77, 1], [4, 4, 8, 8], [1, 1, 2, 2])
    rope = Rotary(64, 1e4, layout=B.NSP_ROPE_INTERLEAVED)
    g = torch.Generator("cuda").manual_seed(4)
    host = {n: torch.randn(k, generator=g, device="cuda").bfloat16() for n, k in (("q", w.q_elems()), ("k", w.kv_elems()), ("v", w.kv_elems()),
                                                                                 ("do", w.q_elems()))}
    flags = np.array([1, 0, 1, 0], np.uint8) if recompute else None
    shifted = torch.cat([torch.arange(n) + 1000 * i for i, n in enumerate(w.lengths)])
    results = []
    for a in (NspAttention(w, rope=rope, dq_dtype="f32"), NspAttention(w, dq_dtype="f32"), NspAttention(w, rope=rope, dq_dtype="f32", positions=shifted)):
        a.load(host)
        if a.rope is None:  # by hand
            at = [(300 + 128, 4, 1), (78, 8, 2)]
            pos = torch.cat([torch.arange(int(n)) for n in w.lengths]).cuda()
            pq, pk, pt = 0, 0, 0

            def turn(q, k, inverse):
                pq = pk = pt = 0
                for n, hq, hkv in at:
                    for z, o, h in ((q, pq, hq), (k, pk, hkv)):
                        view = z[o:o + n * h * 128].view(n, h, 128)
                        B.nsp_rope(view, view, pos[pt:pt + n], rope.inv_freq, layout=rope.layout, inverse=inverse)
                    pq, pk, pt = pq + n * hq * 128, pk + n * hkv * 128, pt + n

            turn(a.q, a.k, False)
            a.forward()
            a.backward(flags)
            turn(a.dq, a.dk, True)
        else:
            before = a.q.clone()
            a.forward()
            a.backward(flags)
            assert torch.equal(a.q, before)  # the caller's queries stay unrotated
        assert a.status()[0] == 0
        results.append({n: getattr(a, n).clone() for n in ("o", "lse", "dq", "dk", "dv")})
    one, two, moved = results
    for n in ("o", "lse", "dk", "dv"):
        assert torch.equal(one[n], two[n]), n
    near = lambda x, y, tol: ((x.double() - y.double()).norm() / y.double().norm()).item() <= tol
    assert near(one["dq"], two["dq"], 1e-5)
    # scores depend on differences of positions: the same attention up to the rounding of rotated queries and keys to bf16, which
    # scores of order one take on as they are, and everything behind them
    for n in ("o", "dq", "dk", "dv"):
        assert near(moved[n], one[n], BOUND), n


def test_node_layouts_with_rope(B):
    """A degree-1 node: prologue and epilogue with rope around the exchange, on the device."""
    import torch

    from paper_2609_22755_b200.api import Rotary
    from paper_2609_22755_b200.ulysses import NodeLayout, UlyssesExchange

    lay, rope = NodeLayout([96, 33], 1, 0, 8, 2, 128), Rotary(128)
    ex = UlyssesExchange(lay, [0])
    x = torch.randn(129, 8, 128, device="cuda")
    want = torch.empty_like(x)
    rope.rotate(x, want, torch.cat([torch.arange(96), torch.arange(33)]).cuda())
    got = ex.to_attention_layout(x, "q", rope=rope)
    assert torch.equal(got, want)
    back = ex.from_attention_layout(got, "q", rope=rope)
    assert (back - x).abs().max().item() <= 2 * 9 * 2.0 ** -24 * 2 * x.abs().max().item()  # twice the bound of a rotation
    into = [torch.empty(129, 8, 128, device="cuda")]
    ex.store_to_attention_layouts(x, "q", into, rope=rope)
    assert torch.equal(into[0], want)


def test_cost_table_times_the_token_operators(B):
    from paper_2609_22755_b200.measure_cost_table import measure_token_ops

    ops = measure_token_ops(256, 512, 4, 2, tokens=512, iters=1)
    assert set(ops) == {"norm", "rotation", "feed_forward"} and all(v > 0 for v in ops.values())


def test_node_layouts_with_rope_on_another_stream(B):
    """The rotated copy belongs to the stream that the calls are given: what the current stream allocates meanwhile is other memory."""
    import torch

    from paper_2609_22755_b200.api import Rotary
    from paper_2609_22755_b200.ulysses import NodeLayout, UlyssesExchange

    lay, rope, side = NodeLayout([9600, 3300], 1, 0, 8, 2, 128), Rotary(128), torch.cuda.Stream()
    ex = UlyssesExchange(lay, [0])
    x = torch.randn(12900, 8, 128, device="cuda")
    want = torch.empty_like(x)
    rope.rotate(x, want, torch.cat([torch.arange(9600), torch.arange(3300)]).cuda())
    for stream in (side, side.cuda_stream):
        into = [torch.zeros_like(x)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(10_000_000)  # the calls below run behind this
        ex.store_to_attention_layouts(x, "q", into, rope=rope, stream=stream)
        others = [torch.full_like(x, 7.0) for _ in range(4)]
        side.synchronize()
        assert torch.equal(into[0], want)
        del others
