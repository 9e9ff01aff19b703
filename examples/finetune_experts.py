#!/usr/bin/env python3
"""Fine-tunes the experts of one MoE layer and serves them in 4 bits.

    python examples/finetune_experts.py [--tokens T --width d --expert-width f --experts E --topk k --steps S] [--block]

A layer with random experts learns the outputs of another one with the same router.  Routing, dispatch and combine are the
context's calls; the experts run on row-major weights through the grouped products, whose gradients come from the same
calls; the gradients are clipped to a global norm and taken off 32-bit master weights.  Afterwards the trained experts are
packed for `moe_layer_forward` and quantised to 4 bits, and both ways of serving them are compared with the trained layer.

With --block the layer stands in a block on a residual stream: a norm before its router, a norm behind its combine and the residual, whose weights
are trained too, and the experts' matrices take orthogonalised steps with momentum.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_19945_amd as moe  # noqa: E402


def experts_forward(xp, w13, w2, offsets):
    """Rows through their experts; what the backward pass needs is returned with the result."""
    gu = moe.moe_grouped_gemm(xp, w13, offsets)      # gate and up projection side by side
    h = moe.moe_swiglu(gu, offsets)
    return moe.moe_grouped_gemm(h, w2, offsets), gu, h


def experts_backward(dy, xp, gu, h, w13, w2, offsets):
    """Gradients of both weight tensors (fp32) and of the rows."""
    dw2 = moe.moe_grouped_gemm_wgrad(h, dy, offsets)
    dh = moe.moe_grouped_gemm(dy, w2, offsets, transpose_w=True)
    dgu = moe.moe_swiglu_backward(dh, gu, offsets)
    dw13 = moe.moe_grouped_gemm_wgrad(xp, dgu, offsets)
    return dw13, dw2, moe.moe_grouped_gemm(dgu, w13, offsets, transpose_w=True)


def experts_forward_4bit(xp, w13, w2, offsets):
    """The same rows on quantised experts: w13 and w2 are (values, scales); rows are quantised on the way in."""
    gu = moe.moe_mxfp4_grouped_gemm(*moe.moe_mxfp4_quantize(xp, offsets), *w13, offsets)
    h = moe.moe_swiglu(gu, offsets)
    return moe.moe_mxfp4_grouped_gemm(*moe.moe_mxfp4_quantize(h, offsets), *w2, offsets)


def relative(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def run(T=2048, d=512, f=1024, E=8, k=2, steps=40, lr=0.3, max_norm=1.0, seed=0, log=print):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    ctx = moe.MoEContext(T, d, f, E, k)
    router = ctx.moe_pack_router(normal(d, E, std=d ** -0.5, dtype=torch.float32))
    teacher = ctx.moe_pack_weights(normal(E, d, f, std=d ** -0.5), normal(E, d, f, std=d ** -0.5), normal(E, f, d, std=f ** -0.5))
    master = [normal(E, d, 2 * f, std=d ** -0.5, dtype=torch.float32), normal(E, f, d, std=f ** -0.5, dtype=torch.float32)]
    weights = [m.to(torch.bfloat16) for m in master]
    x = normal(T, d, std=1.0)
    target = ctx.moe_layer_forward(x, router, None, teacher)

    idx, w, _ = ctx.moe_route(x, router)
    xp, offsets, row_of, tok_of = ctx.moe_permute(x, idx)
    w_row = torch.empty(xp.shape[0], device="cuda")
    w_row[row_of.flatten().long()] = w.flatten()      # gate weight of every row (all experts live here)
    ones = torch.ones_like(w)
    losses, norms = [], []
    for _ in range(steps):
        y, gu, h = experts_forward(xp, *weights, offsets)
        out = ctx.moe_combine(y, row_of, w)
        diff = out.float() - target.float()
        losses.append(diff.square().mean())
        dout = diff * (2.0 / T)                       # of the squared error, averaged over the tokens
        dy = (dout[tok_of.long()] * w_row[:, None]).to(torch.bfloat16)
        dw13, dw2, dxp = experts_backward(dy, xp, gu, h, *weights, offsets)
        dx = ctx.moe_combine(dxp, row_of, ones)       # what a layer below would get
        norms.append(moe.moe_clip_grad_norm([dw13, dw2], max_norm))
        for m, grad, wt in zip(master, (dw13, dw2), weights):
            m.sub_(grad, alpha=lr)
            wt.copy_(m)
    losses, norms = torch.stack(losses).tolist(), torch.stack(norms).tolist()
    log(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} steps, gradient norm {norms[0]:.3f} -> {norms[-1]:.3f}")

    out = ctx.moe_combine(experts_forward(xp, *weights, offsets)[0], row_of, w)
    w13, w2 = weights
    packed = ctx.moe_pack_weights(w13[:, :, :f].contiguous(), w13[:, :, f:].contiguous(), w2)
    served = relative(ctx.moe_layer_forward(x, router, None, packed), out)
    four = [moe.moe_mxfp4_quantize_weights(t) for t in weights]
    served4 = relative(ctx.moe_combine(experts_forward_4bit(xp, *four, offsets), row_of, w), out)
    size = sum(t.numel() for t in weights) * 2 / sum(v.numel() + s.numel() for v, s in four)
    log(f"served packed: {served:.4f} from the trained layer; in 4 bits: {served4:.4f}, weights {size:.2f} times smaller")
    ctx.close()
    return dict(losses=losses, norms=norms, served=served, served4=served4, dx=dx)


def block_forward(ctx, x, router, weights, norms):
    """The stream behind the block, and what the backward pass needs."""
    h = moe.moe_rms_norm(x, norms[0])
    idx, w, _ = ctx.moe_route(h, router)
    xp, offsets, row_of, tok_of = ctx.moe_permute(h, idx)
    y, gu, hidden = experts_forward(xp, *weights, offsets)
    c = ctx.moe_combine(y, row_of, w)
    out, _ = moe.moe_residual_norm(x, c, norms[1])
    return out, (xp, offsets, row_of, tok_of, w, gu, hidden, c)


def block_backward(ctx, dout, x, weights, norms, kept):
    """Gradients of x, of both weight tensors and of both norms' weights (the router is not trained, nor is anything through its weights)."""
    xp, offsets, row_of, tok_of, w, gu, hidden, c = kept
    dres, dc, dnorm1, _, _ = moe.moe_residual_norm_backward(dout, c, norms[1])
    w_row = torch.empty(xp.shape[0], device=x.device)
    w_row[row_of.flatten().long()] = w.flatten()
    dy = (dc[tok_of.long()].float() * w_row[:, None]).to(torch.bfloat16)
    dw13, dw2, dxp = experts_backward(dy, xp, gu, hidden, *weights, offsets)
    dh = ctx.moe_combine(dxp, row_of, torch.ones_like(w))
    dx, dnorm0 = moe.moe_rms_norm_backward(dh, x, norms[0], dres=dres)
    return dx, dw13, dw2, dnorm0, dnorm1


def orthogonal_update(grad, momentum, f=0, decay=0.95):
    """The step of a stack of matrices: Nesterov momentum, orthogonalised, gate and up projection (f > 0) each by itself; its values have a root mean
    square near that of 0.2 whatever the matrix's shape."""
    momentum.mul_(decay).add_(grad)
    u = grad.add(momentum, alpha=decay)
    for part in (u[:, :, :f], u[:, :, f:]) if f else (u,):
        moe.moe_orthogonalize(part, scale=0.2 * max(part.shape[1:]) ** 0.5, out=part)
    return u


def run_block(T=2048, d=512, f=1024, E=8, k=2, steps=40, lr=0.02, norm_lr=0.05, max_norm=1.0, seed=0, log=print):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    ctx = moe.MoEContext(T, d, f, E, k)
    router = ctx.moe_pack_router(normal(d, E, std=d ** -0.5, dtype=torch.float32))
    teacher = [normal(E, d, 2 * f, std=d ** -0.5), normal(E, f, d, std=f ** -0.5)]
    norms = [torch.ones(d, device="cuda"), torch.ones(d, device="cuda")]
    x = normal(T, d, std=1.0)
    target, _ = block_forward(ctx, x, router, teacher, [n + 0.2 * normal(d, std=1.0, dtype=torch.float32) for n in norms])
    master = [normal(E, d, 2 * f, std=d ** -0.5, dtype=torch.float32), normal(E, f, d, std=f ** -0.5, dtype=torch.float32)]
    weights, momenta = [m.to(torch.bfloat16) for m in master], [torch.zeros_like(m) for m in master]
    losses, lengths = [], []
    for _ in range(steps):
        out, kept = block_forward(ctx, x, router, weights, norms)
        diff = out.float() - target.float()
        losses.append(diff.square().mean())
        dx, dw13, dw2, dn0, dn1 = block_backward(ctx, (diff * (2.0 / T)).to(torch.bfloat16), x, weights, norms, kept)
        lengths.append(moe.moe_clip_grad_norm([dw13, dw2, dn0, dn1], max_norm))
        for m, grad, mom, wt, half in zip(master, (dw13, dw2), momenta, weights, (f, 0)):
            m.sub_(orthogonal_update(grad, mom, half), alpha=lr)
            wt.copy_(m)
        for n, grad in zip(norms, (dn0, dn1)):
            n.sub_(grad, alpha=norm_lr)
    losses, lengths = torch.stack(losses).tolist(), torch.stack(lengths).tolist()
    log(f"block: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} orthogonalised steps, gradient norm {lengths[0]:.3f} -> {lengths[-1]:.3f}")
    ctx.close()
    return dict(losses=losses, norms=lengths, dx=dx)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--expert-width", type=int, default=1024)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--topk", type=int, default=2)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--block", action="store_true", help="train the layer in a block, with norms and orthogonalised steps")
    a = ap.parse_args()
    (run_block if a.block else run)(a.tokens, a.width, a.expert_width, a.experts, a.topk, a.steps)


if __name__ == "__main__":
    main()
