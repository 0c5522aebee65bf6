"""NspAttention(rope=...) whose backward pass recomputes: the queries and keys that it reads are those of now, whether or not a forward pass has
been run on them. On the CPU the library's calls are stand-ins; on the GPU the gradients are compared with those behind a forward pass."""
import numpy as np
import pytest
import torch

from paper_2609_22755_b200 import binding as B
from paper_2609_22755_b200 import workloads as W
from paper_2609_22755_b200.api import NspAttention


class Turn:
    """Stand-in for a Rotary: 1 is added on the way in and taken off on the way back."""

    def rotate(self, xs, ys, positions, inverse=False, stream=None):
        for x, y in zip(xs, ys):
            y.copy_(x - 1 if inverse else x + 1)


def test_recomputation_reads_the_queries_and_keys_of_now(monkeypatch):
    a = NspAttention.__new__(NspAttention)
    a.torch, a.w, a.dev, a.stream, a.plan, a.scale = torch, W.custom([4, 3], [2, 2], [1, 1]), torch.device("cpu"), None, None, 1.0
    a.q, a.dq, a.do = (torch.zeros(a.w.q_elems()) for _ in range(3))
    a.k, a.v, a.dk, a.dv = (torch.zeros(a.w.kv_elems()) for _ in range(4))
    a.o, a.lse, a.ws, a.rope = None, None, torch.empty(0), Turn()
    a._prepare_rope(None)
    a.q_rot.fill_(-5.0), a.k_rot.fill_(-5.0)  # of another batch
    monkeypatch.setattr(B, "nsp_plan_recompute_ws_bytes", lambda plan: 0)
    seen = []
    monkeypatch.setattr(B, "nsp_attn_bwd_recompute", lambda plan, flags, q, k, *rest, **named: seen.append((q.clone(), k.clone())))
    a.q.fill_(2.0), a.k.fill_(3.0)
    a.backward(recompute=np.ones(2, np.uint8))
    assert bool((seen[0][0] == 3.0).all()) and bool((seen[0][1] == 4.0).all())


@pytest.mark.gpu
def test_recomputation_without_a_forward_pass():
    from paper_2609_22755_b200.api import Rotary

    w = W.custom([300, 128, 77], [4, 4, 8], [1, 1, 2])
    a = NspAttention(w, rope=Rotary(128), dq_dtype="f32")
    g = torch.Generator("cuda").manual_seed(5)
    sizes = (("q", w.q_elems()), ("k", w.kv_elems()), ("v", w.kv_elems()), ("do", w.q_elems()))
    batches = [{n: torch.randn(k, generator=g, device="cuda").bfloat16() for n, k in sizes} for _ in range(2)]
    flags = np.ones(3, np.uint8)
    a.load(batches[0])
    a.forward()
    a.backward(flags)
    want = {n: getattr(a, n).clone() for n in ("dq", "dk", "dv")}
    a.load(batches[1])
    a.forward()
    a.load(batches[0])
    a.backward(flags)
    assert a.status()[0] == 0
    assert torch.equal(a.dk, want["dk"]) and torch.equal(a.dv, want["dv"])
    # dQ is a sum in arrival order: 1e-5 in fp32
    assert ((a.dq.double() - want["dq"].double()).norm() / want["dq"].double().norm()).item() <= 1e-5
