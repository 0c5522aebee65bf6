"""The paths that rotate queries and keys, host side: runs of a packed batch, positions of a GPU's token slices, which tensors the
prologue and the epilogue hand to the rotation. No GPU: the rotation is a stand-in."""
import numpy as np
import pytest
import torch

from paper_2609_22755_b200 import binding as B
from paper_2609_22755_b200 import workloads as W
from paper_2609_22755_b200.api import NspAttention, packed_runs
from paper_2609_22755_b200.ulysses import NodeLayout, UlyssesExchange


class Turns:
    """Stand-in for the library's layout steps of a degree-1 node, where the exchange is a copy, and of the rotation."""

    def __init__(self):
        self.seen = []

    def gather(self, src, dst, tokens, heads, hpb, D, first, stream=None):
        dst.copy_(src.reshape(1, tokens, heads, D))

    def scatter(self, src, dst, tokens, heads, hpb, D, first, stream=None):
        dst.copy_(src.reshape(tokens, heads, D))

    def gather_to(self, src, dst_tensors, dst_row, sample_off, tokens, heads, hpb, D, first, stream=None):
        dst_tensors[0].copy_(src.reshape(dst_tensors[0].shape))

    def rotate(self, rope, x, y, positions, inverse, stream=None):
        self.seen.append((rope, positions.tolist(), inverse, x is y))
        y.copy_(x + (-rope if inverse else rope) * positions[:, None, None].to(x.dtype))


def test_positions_of_token_slices():
    lay = [NodeLayout([8, 0, 20], 4, r, 8, 4, 16) for r in range(4)]
    assert lay[0].positions().tolist() == [0, 1, 0, 1, 2, 3, 4]
    assert lay[3].positions().tolist() == [6, 7, 15, 16, 17, 18, 19]
    whole = [torch.cat([lay[r].positions()[a:b] for r in range(4)]).tolist() for a, b in ((0, 2), (2, 7))]
    assert whole == [list(range(8)), list(range(20))]
    assert NodeLayout([], 2, 0, 4, 2).positions().numel() == 0


def test_prologue_and_epilogue_rotate_the_token_slices():
    lay, ops = NodeLayout([3, 5], 1, 0, 4, 2, 8), Turns()
    ex = UlyssesExchange(lay, [0], ops=ops)
    x = torch.randn(8, 4, 8)
    pos = torch.tensor([0, 1, 2, 0, 1, 2, 3, 4.0])[:, None, None]
    before = x.clone()
    got = ex.to_attention_layout(x, "q", rope=2.0)
    assert torch.equal(got, x + 2 * pos) and torch.equal(x, before)  # the caller's tensor is left alone
    back = ex.from_attention_layout(got, "q", rope=2.0)
    assert torch.allclose(back, x, atol=1e-5)
    into = [torch.empty(8, 4, 8)]
    ex.store_to_attention_layouts(x, "q", into, rope=2.0)
    assert torch.equal(into[0], got)
    assert torch.equal(ex.to_attention_layout(x, "q"), x)  # without rope nothing changes
    assert [s[2:] for s in ops.seen] == [(False, False), (True, True), (False, False)]
    assert all(s[1] == [0, 1, 2, 0, 1, 2, 3, 4] for s in ops.seen)


def test_runs_of_a_packed_batch():
    w = W.custom([5, 0, 7, 3, 3, 9], [8, 8, 4, 4, 8, 8], [2, 2, 1, 1, 2, 2])
    assert packed_runs(w) == [(0, 2, 5, 8, 2), (2, 4, 10, 4, 1), (4, 6, 12, 8, 2)]
    assert packed_runs(W.custom([], [], [])) == []
    assert sum(n * hq for _, _, n, hq, _ in packed_runs(w)) * w.head_dim == w.q_elems()


def test_step_host_refuses_rope():
    a = NspAttention.__new__(NspAttention)
    a.rope = object()
    with pytest.raises(B.NspError) as e:
        a.step_host({}, {})
    assert e.value.code == B.NSP_ERR_UNSUPPORTED


def test_positions_are_checked():
    a = NspAttention.__new__(NspAttention)
    a.torch, a.w, a.dev = torch, W.custom([4, 3], [2, 2], [1, 1]), torch.device("cpu")
    a.q = a.dq = torch.zeros(a.w.q_elems())
    a.k = a.dk = torch.zeros(a.w.kv_elems())
    for bad in (torch.zeros(7), torch.zeros(6, dtype=torch.int64), torch.zeros(7, 1, dtype=torch.int64)):
        with pytest.raises(ValueError):
            a._prepare_rope(bad)
    a._prepare_rope(None)
    assert a.positions.tolist() == [0, 1, 2, 3, 0, 1, 2]
    assert [tuple(v.shape) for v in a._rope_in] == [(7, 2, 128), (7, 1, 128)] and len(a._run_positions) == 2
