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


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [0, 1])
def test_angles_are_as_good_as_stated(layout):
    """Cosines and sines themselves, of pairs (1, 0), at positions of up to 2^36 and frequencies of up to a turn a position, and some of several
    turns: the angle within 2 pi (2^-32 + |p| 2^-63 max(1, |f| / 2 pi)), the polynomials within 1.7 * 2^-24, their factor and the sum
    of the two products 2^-24 each."""
    from fractions import Fraction

    pi = Fraction(3141592653589793238462643383279502884197169399375105820974945, 10 ** 60)
    rng = np.random.default_rng(4)
    pos = np.concatenate([[0, 1, -1, 2, 2 ** 36, -2 ** 36], (2.0 ** rng.uniform(0, 36, 200)).astype(np.int64) * rng.choice([-1, 1], 200)])
    freq = np.concatenate([rng.uniform(-2 * np.pi, 2 * np.pi, 20), [1.0, 1e-6, 3.14159, 6.28, 100.0, -1e4], 1e6 ** -rng.uniform(0, 1, 6)])
    x = torch.zeros(len(pos), 1, 2 * len(freq), device="cuda")
    first = (slice(0, len(freq)), slice(len(freq), None)) if layout == 0 else (slice(0, None, 2), slice(1, None, 2))
    x[..., first[0]] = 1.0
    y = torch.empty_like(x)
    B.nsp_rope(x, y, torch.as_tensor(pos).cuda(), freq, layout=layout)
    turns = np.array([[float((int(p) * Fraction(float(f)) / (2 * pi)) % 1) for f in freq] for p in pos])
    bound = 2 * np.pi * (2.0 ** -32 + np.abs(pos)[:, None] * 2.0 ** -63 * np.maximum(1, np.abs(freq) / (2 * np.pi))) + 3.7 * 2.0 ** -24
    for at, exact in ((first[0], np.cos), (first[1], np.sin)):
        off = np.abs(y[:, 0, at].double().cpu().numpy() - exact(2 * np.pi * turns))
        assert (off <= bound).all(), (off / bound).max()
