"""Gradients of the gated feed-forward block against differences of the definition in 64 bits, along the formula's own gradients. There the
derivative is as large as the gradient, several times what the roundings of the kernels can amount to; along a random direction it is
smaller than that, and a wrong gradient would pass. The CPU part shows that such ones do not pass here."""
import math

import pytest
import torch

HALF = 2.0 ** -8  # half a step of bf16
ROWS, D, F = 40, 72, 88


def act64(x, act):
    if act == 0:
        return x * torch.sigmoid(x)
    return x * 0.5 * torch.erfc(-x / math.sqrt(2))


def inputs(device):
    g = torch.Generator().manual_seed(11)
    rnd = lambda rows, cols, scale: (torch.randn(rows, cols, generator=g) * scale).bfloat16().to(device)
    return rnd(ROWS, D, 1.0), rnd(F, D, D ** -0.5), rnd(F, D, D ** -0.5), rnd(ROWS, F, 1.0)


def loss(x, wg, wu, dh, act):
    return (act64(x @ wg.t(), act) * (x @ wu.t()) * dh).sum()


def formula(x, wg, wu, dh, act):
    """(gradients of sum(h dh) with respect to x, w_gate, w_up, how far the kernel's may be from each), 64 bits. g and u are rounded to
    bf16 before the backward pass reads them, dg and du before the products: with |act'| <= 1.13 and |act''| <= 0.8
        |error of dg| <= |dh| 2^-8 (2 |u act'| + 0.8 |u g|),  |error of du| <= |dh| 2^-8 (|act| + 1.13 |g|)
    to first order (products of two such errors: 2^-7 of that, taken as 2^-6), the sums of products are in fp32 (2^-16 of their
    magnitudes), and the gradient is rounded once more."""
    leaf = [t.double().requires_grad_() for t in (x, wg, wu)]
    g, u = leaf[0] @ leaf[1].t(), leaf[0] @ leaf[2].t()
    g.retain_grad(), u.retain_grad()
    a = act64(g, act)
    (a * u * dh.double()).sum().backward()
    dg, du, g, u, a, size = g.grad.abs(), u.grad.abs(), g.detach().abs(), u.detach().abs(), a.detach().abs(), dh.double().abs()
    e_dg = (1 + 2.0 ** -6) * HALF * (2 * dg + 0.8 * size * u * g) + 2.0 ** -16 * dg
    e_du = (1 + 2.0 ** -6) * HALF * (du + 1.13 * size * g) + 2.0 ** -16 * du
    x, wg, wu = (t.double().abs() for t in (x, wg, wu))
    errors = [e_dg @ wg + e_du @ wu, e_dg.t() @ x, e_du.t() @ x]
    grads = [t.grad for t in leaf]
    return grads, [e + HALF * (k.abs() + e) for k, e in zip(grads, errors)]


def check(x, wg, wu, dh, act, got):
    """Assert that the gradients `got` are the derivatives of the loss along the formula's gradients."""
    grads, errors = formula(x, wg, wu, dh, act)
    at = [t.double() for t in (x, wg, wu)]
    for k, (have, want, error) in enumerate(zip(got, grads, errors)):
        v = want / want.norm()
        plus, minus = [t.clone() for t in at], [t.clone() for t in at]
        plus[k] += 1e-4 * v
        minus[k] -= 1e-4 * v
        slope = ((loss(*plus, dh.double(), act) - loss(*minus, dh.double(), act)) / 2e-4).item()
        bound = (error * v.abs()).sum().item()
        assert bound <= 0.2 * slope  # the check says something
        # the difference: h^2 times a third derivative of order one, 2^-52 / h times the loss
        assert abs(slope - (have.double() * v).sum().item()) <= bound + 1e-6 * slope, k


@pytest.mark.parametrize("act", [0, 1])
def test_the_check_tells_wrong_gradients(act):
    """The formula's gradients in bf16 pass; negated ones, ones without one of two terms, with rows in another order and of another
    activation do not."""
    args = inputs("cpu")
    good = [t.bfloat16() for t in formula(*args, act)[0]]
    check(*args, act, good)
    x, wg, wu, dh = (t.double() for t in args)
    dg = torch.autograd.functional.vjp(lambda g: act64(g, act) * (x @ wu.t()), x @ wg.t(), dh)[1]
    wrong = [[-t if i == k else t for i, t in enumerate(good)] for k in range(3)]
    wrong += [[t.flip(0) if i == k else t for i, t in enumerate(good)] for k in range(3)]
    wrong += [[good[0].double() - dg @ wg, good[1], good[2]], [dg @ wg, good[1], good[2]]]
    wrong += [[good[0], good[2], good[1]]]
    for bad in wrong:
        with pytest.raises(AssertionError):
            check(*args, act, bad)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [0, 1])
def test_gradients_along_the_formulas(act):
    from paper_2609_22755_b200 import binding as B

    x, wg, wu, dh = inputs("cuda")
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    h, g, u, got = e(ROWS, F), e(ROWS, F), e(ROWS, F), (e(ROWS, D), e(F, D), e(F, D))
    ws = torch.empty(B.nsp_glu_bwd_ws_bytes(ROWS, D, F), dtype=torch.uint8, device="cuda")
    B.nsp_glu_fwd(x, wg, wu, h, g, u, act=act)
    B.nsp_glu_bwd(dh, x, wg, wu, g, u, *got, ws, act=act)
    check(x, wg, wu, dh, act, got)
    assert B.nsp_glu_status()[0] == 0
