"""The operators around a block together, as the example's block runs them: norm, route, experts, combine, norm and residual, backward, clipping,
orthogonalised steps."""
import importlib.util
import os

import pytest
import torch

import paper_2605_19945_amd as moe

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F64 = torch.float64


def load():
    spec = importlib.util.spec_from_file_location("finetune_experts", os.path.join(ROOT, "examples", "finetune_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs():
    got = load().run_block(T=300, d=256, f=320, E=8, k=2, steps=3, log=lambda *_: None)
    assert len(got["losses"]) == 3 and torch.isfinite(got["dx"]).all() and all(n > 0 for n in got["norms"])


@pytest.fixture(scope="module")
def step():
    """One step of a small block on the GPU, and the same in 64 bits on the CPU by torch's own differentiation under the GPU's routing."""
    ex = load()
    T, d, f, E, k = 70, 128, 192, 4, 2
    g = torch.Generator().manual_seed(3)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g) * std).to(dtype)

    x, dout = normal(T, d), normal(T, d)
    w13, w2 = normal(E, d, 2 * f, std=d ** -0.5), normal(E, f, d, std=f ** -0.5)
    norms = [1 + normal(d, std=0.2, dtype=torch.float32) for _ in range(2)]
    ctx = moe.MoEContext(T, d, f, E, k)
    router = ctx.moe_pack_router(normal(d, E, std=d ** -0.5, dtype=torch.float32).cuda())
    dev = [t.cuda() for t in (w13, w2)], [n.cuda() for n in norms]
    out, kept = ex.block_forward(ctx, x.cuda(), router, *dev)
    grads = ex.block_backward(ctx, dout.cuda(), x.cuda(), *dev, kept)
    h = moe.moe_rms_norm(x.cuda(), dev[1][0])
    idx, w, _ = (t.cpu() if t is not None else None for t in ctx.moe_route(h, router))
    torch.cuda.synchronize()
    ctx.close()

    x64, a, b, n0, n1 = (t.double().requires_grad_() for t in (x, w13, w2, *norms))

    def norm(t, wt):
        return t / (t.square().mean(1, keepdim=True) + 1e-6).sqrt() * wt

    h64, c = norm(x64, n0), torch.zeros(T, d, dtype=F64)
    for e in range(E):
        weight = torch.where(idx == e, w.double(), 0.0).sum(1, keepdim=True)
        p = h64 @ a[e]
        c = c + weight * ((torch.nn.functional.silu(p[:, :f]) * p[:, f:]) @ b[e])
    ref = x64 + norm(c, n1)
    ref.backward(dout.double())
    return ex, [t.cpu() for t in (out, *grads)], [ref.detach(), x64.grad, a.grad, b.grad, n0.grad, n1.grad], f


def test_gradients_of_the_block(step):
    """On the way to any of them at most twelve values are rounded to bf16 (h, gate and up, hidden, y, c, their gradients, dy, dxp, dh, the results), by 2^-8
    of each at most, so the results are off by less than 2^-4 of their norm."""
    for got, ref in zip(step[1], step[2]):
        assert got.shape == ref.shape and float((got.double() - ref).norm()) <= 2.0 ** -4 * float(ref.norm())


def test_the_update_of_the_block(step):
    """The step that the gradients lead to: momentum from zeros, u = (1 + 0.95) g, each projection's matrices orthogonalised by themselves."""
    ex, got, _, f = step
    for grad, half in ((got[2], f), (got[3], 0)):
        momentum = torch.zeros_like(grad).cuda()
        u = ex.orthogonal_update(grad.cuda(), momentum, half).cpu()
        assert torch.equal(momentum.cpu(), grad)
        parts = [(0, half), (half, 2 * half)] if half else [(0, grad.shape[2])]
        for a, b in parts:
            for e in range(grad.shape[0]):
                X = 1.95 * grad[e, :, a:b].double()
                X = X / (X.norm() + 1e-7)
                for _ in range(5):
                    S = X @ X.t()
                    X = 3.4445 * X + (-4.7750 * S + 2.0315 * S @ S) @ X
                X = X * 0.2 * max(X.shape) ** 0.5
                # 1.95 g is rounded to 32 bits before; the steps carry 2^-24 on by at most 3.4445^5 < 2^9, and add as much a few times over
                assert float((u[e, :, a:b].double() - X).norm()) <= 2.0 ** -12 * float(X.norm())


def test_a_captured_step():
    """The whole step in a graph, replayed over other tokens with eager steps between, gives the eager step's bits."""
    ex = load()
    T, d, f, E, k = 96, 256, 128, 4, 2
    g = torch.Generator().manual_seed(9)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g) * std).to(dtype).cuda()

    x, dout = normal(T, d), normal(T, d)
    weights, norms = [normal(E, d, 2 * f, std=d ** -0.5), normal(E, f, d, std=f ** -0.5)], [1 + normal(d, std=0.2, dtype=torch.float32) for _ in range(2)]
    ctx = moe.MoEContext(T, d, f, E, k)
    router = ctx.moe_pack_router(normal(d, E, std=d ** -0.5, dtype=torch.float32))

    def step():
        out, kept = ex.block_forward(ctx, x, router, weights, norms)
        dx, *grads = ex.block_backward(ctx, dout, x, weights, norms, kept)
        length = moe.moe_clip_grad_norm(grads, 1.0)
        return [out, dx, length, *grads, *(ex.orthogonal_update(t, torch.zeros_like(t), h) for t, h in zip(grads[:2], (f, 0)))]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        x.copy_(normal(T, d))
        dout.copy_(normal(T, d))
        graph.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, want)) and all(torch.equal(a, b) for a, b in zip(held, want))
    ctx.close()
