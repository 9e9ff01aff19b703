"""The example that trains a layer's experts and serves them in 4 bits, on a small layer."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("finetune_experts", os.path.join(ROOT, "examples", "finetune_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss_and_the_served_layers_agree():
    got = load().run(T=300, d=256, f=320, E=8, k=2, steps=25, log=lambda *_: None)
    # clipped steps against a fixed target: the loss falls by far more than its rounding
    assert got["losses"][-1] < 0.8 * got["losses"][0] and all(n > 0 for n in got["norms"])
    # bf16 against bf16: both round the intermediates and the result once or twice more than the other (2^-8 each)
    assert got["served"] < 2e-2
    # a 4-bit value is off by at most a third of itself where it is largest (between 4 and 6 a step of 2), about a tenth on average, rows
    # and weights alike, in two products in a row; a layer served with wrong scales or rows would be off by its own size
    assert 0.02 < got["served4"] < 0.4
    assert torch.isfinite(got["dx"]).all()


def test_gradients_of_the_layer_against_autograd():
    """One step's gradients against torch's own differentiation of the same layer in 64 bits on the CPU."""
    import paper_2605_19945_amd as moe
    ex = load()
    E, d, f, rows = 3, 64, 96, [17, 0, 40]
    g = torch.Generator().manual_seed(5)
    off = torch.tensor([0, 17, 17, 57], dtype=torch.int32)
    xp, dy = (torch.randn(57, n, generator=g).to(torch.bfloat16) for n in (d, d))
    w13, w2 = (torch.randn(s, generator=g).mul(0.1).to(torch.bfloat16) for s in ((E, d, 2 * f), (E, f, d)))
    o = off.cuda()
    y, gu, h = ex.experts_forward(xp.cuda(), w13.cuda(), w2.cuda(), o)
    dw13, dw2, dx = ex.experts_backward(dy.cuda(), xp.cuda(), gu, h, w13.cuda(), w2.cuda(), o)
    x64, a, b = (t.double().requires_grad_() for t in (xp, w13, w2))
    parts = []
    for e in range(E):
        p = x64[int(off[e]):int(off[e + 1])] @ a[e]
        parts.append((torch.nn.functional.silu(p[:, :f]) * p[:, f:]) @ b[e])
    out = torch.cat(parts)
    out.backward(dy.double())
    # at most four values on the way are rounded to bf16, by 2^-8 of each at most: 2^-6 of the result's norm
    for got, ref in ((y, out.detach()), (dx, x64.grad), (dw13, a.grad), (dw2, b.grad)):
        assert float((got.cpu().double() - ref).norm()) <= 2.0 ** -6 * float(ref.norm())
    assert (dw13[1] == 0).all() and (dw2[1] == 0).all()
