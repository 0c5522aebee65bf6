"""Which positions every tensor of a rotary call is handed: lists that name a tensor of positions more than once, with None in between. On
the CPU the library is a stand-in that keeps what it is given; on the GPU one call is compared with single ones."""
import numpy as np
import pytest
import torch

from paper_2609_22755_b200 import binding as B

ORDERS = ["P-P", "P-", "-P-P", "PP-PQ-QP", "P-Q-P", "Q--Q"]


def positions_of(order, tensors):
    return [None if c == "-" else tensors[c] for c in order]


@pytest.mark.parametrize("order", ORDERS)
def test_every_tensor_gets_its_positions(monkeypatch, order):
    handed = []

    class Library:
        def nsp_rope(self, packed, n, *rest):
            handed.extend(B._ROPE_TENSOR.unpack_from(packed, i * B._ROPE_TENSOR.size)[2] for i in range(n))
            return B.NSP_OK

    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(B, "_on_device", lambda *a: None)
    monkeypatch.setattr(B, "_stream_on", lambda *a: 0)
    if not B._Torch.ready:
        B._Torch.fill()
    at = {"P": torch.arange(5), "Q": torch.arange(5) * 7}
    x = [torch.zeros(5, 2, 64) for _ in order]
    B.nsp_rope(x, x, positions_of(order, at), np.full(32, 0.5))
    assert handed == [0 if c == "-" else at[c].data_ptr() for c in order]


@pytest.mark.gpu
@pytest.mark.parametrize("order", ORDERS)
def test_one_call_is_as_many_single_ones(order):
    at = {"P": torch.arange(37, device="cuda") + 1000, "Q": torch.arange(37, device="cuda") * 7}
    pos = positions_of(order, at)
    freq, _ = B.nsp_rope_frequencies(64)
    g = torch.Generator("cuda").manual_seed(3)
    xs = [torch.randn(37, 1 + i % 3, 64, generator=g, device="cuda") for i in range(len(order))]
    ys, want = [torch.empty_like(x) for x in xs], [torch.empty_like(x) for x in xs]
    B.nsp_rope(xs, ys, pos, freq)
    for x, w, p in zip(xs, want, pos):
        B.nsp_rope(x, w, p, freq)
    assert all(torch.equal(y, w) for y, w in zip(ys, want))
