"""Gradients of the norms around a block on rows far from 1 in size, against 64 bits; bounds as in test_gpu_norms.  The rows' factors r go from 1e-16
to 1e15, whose third powers fp32 does not hold; their squares' sums it does."""
import pytest
import torch

import paper_2605_19945_amd as moe
from test_gpu_norms import BF16, F32, F64, ONCE, TWICE, U, close, dev, normal

pytestmark = pytest.mark.gpu

SIZES = [1e-14, 1e-13, 1e-12, 1.0, 1e12, 1e14, 1e16]


def rows_of(d, seed, dtype, sizes):
    """Rows of these sizes, and gradients that lie partly along them (otherwise the projection is a small share)."""
    x = normal((len(sizes), d), seed)
    dh = (normal((len(sizes), d), seed + 1) + x).to(dtype[1])
    return (x.double() * torch.tensor(sizes, dtype=F64)[:, None]).to(dtype[0]), dh


def gradient_of(x, w, dh, eps):
    """(gradient of x, of w, magnitude of the first) of x r w in 64 bits."""
    x, w, dh = x.double().requires_grad_(), w.double().requires_grad_(), dh.double()
    (x * (x.square().mean(1, keepdim=True) + eps).rsqrt() * w).backward(dh)
    xa, p = x.detach().abs(), (dh * w.detach()).abs()
    r = (xa.square().mean(1, keepdim=True) + eps).rsqrt()
    return x.grad, w.grad, r * (p + xa * r * (r * (p * xa).mean(1, keepdim=True))), (dh.abs() * xa * r).sum(0)


@pytest.mark.parametrize("d", [64, 1000, 2048, 4096, 8200, 16384])
@pytest.mark.parametrize("S,B", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("eps", [0.0, 1e-30])
def test_gradients_of_far_rows(d, S, B, eps):
    w = 1 + normal((d,), 9, 0.2)
    x, dh = rows_of(d, 1, (S, B), SIZES)
    gx, gw, mx, mw = gradient_of(x, w, dh, eps)
    dx, dw = moe.moe_rms_norm_backward(dev(dh), dev(x), dev(w), eps=eps)
    close(dx, gx, mx, ONCE)
    close(dw, gw, mw, ONCE + len(SIZES) * U)
    # the join: the same row as what the next norm took, ...
    y, _ = rows_of(d, 5, (B, B), [1.0] * len(SIZES))
    got = moe.moe_residual_norm_backward(None, dev(y), None, out=dev(x), dh=dev(dh), norm=False, next_weight=dev(w), eps=eps)
    close(got[0], gx, mx, ONCE)
    close(got[3], gw, mw, ONCE + len(SIZES) * U)
    # ... and as the block's output, behind a gate
    y, dout = rows_of(d, 7, (B, S), SIZES)
    gate = normal((len(SIZES),), 8)
    dn = dout.double() * gate.double()[:, None]
    gy, gw, my, mw = gradient_of(y, w, dn, eps)
    got = moe.moe_residual_norm_backward(dev(dout), dev(y), dev(w), gate=dev(gate), eps=eps)
    close(got[1], gy, my, TWICE)
    close(got[2], gw, mw, TWICE + len(SIZES) * U)


@pytest.mark.parametrize("d", [64, 4096, 16384])
def test_gradients_of_rows_of_zeros(d):
    """Without a projection: the gradient times the root of eps' reciprocal."""
    w, x = 1 + normal((d,), 9, 0.2), torch.zeros(3, d)
    dh = normal((3, d), 3)
    for eps in (1e-30, 1e-6):
        ref = dh.double() * w.double() * eps ** -0.5
        dx, dw = moe.moe_rms_norm_backward(dev(dh), dev(x), dev(w), eps=eps)
        close(dx, ref, ref.abs(), ONCE)
        assert not dw.any()
        got = moe.moe_residual_norm_backward(dev(dh), dev(x), dev(w), eps=eps)
        close(got[1], ref, ref.abs(), TWICE)
        assert not got[2].any()


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("d", [64, 2048, 16384])
@pytest.mark.parametrize("B", [BF16, F32])
def test_infinite_outputs_of_a_block_without_a_norm(d, B, gate):
    """dy = gate dout w holds no y."""
    y, dout, w = normal((4, d), 1).to(B), normal((4, d), 2), 1 + normal((d,), 3, 0.2)
    g = normal((4,), 4) if gate else None
    y[1, d // 3], y[2, 0] = float("inf"), float("nan")
    got = moe.moe_residual_norm_backward(dev(dout), dev(y), dev(w), norm=False, gate=None if g is None else dev(g))
    ref = dout.double() * w.double() * (1 if g is None else g.double()[:, None])
    close(got[1], ref, ref.abs(), ONCE)
    assert torch.equal(got[0].cpu(), dout)
