"""Products grouped by expert on every kernel that they may run on (the cases of operator_plans.py, whose plans are checked
without a GPU), against 64 bits.

Bounds.  Products of whole numbers up to 2 have sums that 32 bits hold exactly, in any order, so bf16 operands give the exact
results, rounded once.  4-bit operands: a sum of K products in 32 bits is off by at most K 2^-23 times the sum of their magnitudes, the
rounding to bf16 by 2^-8 of the value."""
import numpy as np
import pytest
import torch

import paper_2605_19945_amd as moe
from operator_plans import CASES

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def whole(shape, seed, dtype=BF16):
    return torch.randint(-2, 3, shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16)


def offsets_of(rows):
    return torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32).cuda()


def experts(rows):
    ends = np.cumsum(rows).tolist()
    return [(e, end - n, end) for e, (n, end) in enumerate(zip(rows, ends)) if n]


def output(rows, N):
    """Rows of N among wider ones, and those wider ones."""
    wide = torch.full((rows, N + 16), 7.0, dtype=BF16, device="cuda")
    return wide[:, 8:8 + N], wide


def rest_untouched(wide, n, N):
    return bool((wide[n:] == 7).all() and (wide[:, :8] == 7).all() and (wide[:, 8 + N:] == 7).all())


def ids(cases):
    return [f"{c[0]}-{'+'.join(map(str, c[1]))}-{c[3]}-{c[4]}" for c in cases]


ROWS = [c for c in CASES if c[0] in ("fwd", "dx")]


@pytest.mark.parametrize("kind,rows,more,K,N,plan", ROWS, ids=ids(ROWS))
def test_rows_times_weights_exactly(kind, rows, more, K, N, plan):
    n, transpose = sum(rows), kind == "dx"
    x = whole((n + more, K), 1)
    x[n:] = float("nan")
    w = whole((len(rows), N, K) if transpose else (len(rows), K, N), 2)
    out, wide = output(n + more, N)
    moe.moe_grouped_gemm(x, w, offsets_of(rows), transpose_w=transpose, out=out)
    for e, a, b in experts(rows):
        m = w[e].t() if transpose else w[e]
        assert torch.equal(out[a:b], torch.mm(x[a:b].double(), m.contiguous().double()).to(BF16)), e
    assert rest_untouched(wide, n, N)


FOUR = [c for c in CASES if c[0] == "mx"]


@pytest.mark.parametrize("kind,rows,more,K,N,plan", FOUR, ids=ids(FOUR))
def test_rows_times_weights_in_4_bits(kind, rows, more, K, N, plan):
    """Scales differ by powers of two from block to block, in rows and in weights, so that a product under another block's scale
    would be off by its own size; the rows behind the last one hold no numbers."""
    n, E, blocks = sum(rows), len(rows), torch.arange(K // 32, device="cuda")
    turn = torch.exp2(((blocks + blocks // 4) % 5 - 2).float()).repeat_interleave(32)  # of neighbouring blocks, steps and pairs of steps
    x = normal((n + more, K), 3) * (turn * torch.exp2((torch.arange(n + more, device="cuda") % 7 - 3).float())[:, None]).to(BF16)
    w = normal((E, K, N), 4) * (turn.flip(0)[:, None] * torch.exp2((torch.arange(N, device="cuda") % 3).float())).to(BF16)
    xq, xs = moe.moe_mxfp4_quantize(x)
    wq, ws = moe.moe_mxfp4_quantize_weights(w)
    xv, wv = moe.moe_mxfp4_dequantize(xq, xs), moe.moe_mxfp4_dequantize(wq, ws)  # (exact)
    xs[n:] = 255
    out, wide = output(n + more, N)
    moe.moe_mxfp4_grouped_gemm(xq, xs, wq, ws, offsets_of(rows), out=out)
    for e, a, b in experts(rows):
        p, q = xv[a:b].double(), wv[e].double().t().contiguous()
        ref, size = torch.mm(p, q), torch.mm(p.abs(), q.abs())
        assert ((out[a:b].double() - ref).abs() <= 2.0 ** -8 * 1.01 * ref.abs() + K * 2.0 ** -23 * size).all(), e
    assert rest_untouched(wide, n, N)


GRADIENTS = [c for c in CASES if c[0] == "dw"]


@pytest.mark.parametrize("dtype,accumulate", [(F32, False), (BF16, False), (F32, True)], ids=["fp32", "bf16", "added"])
@pytest.mark.parametrize("kind,rows,more,M,N,plan", GRADIENTS, ids=ids(GRADIENTS))
def test_gradient_of_weights_exactly(kind, rows, more, M, N, plan, dtype, accumulate):
    """In memory of the result's own with something in front and behind; one that is added to keeps what experts without rows hold."""
    n, E = sum(rows), len(rows)
    x, dy = whole((n + more, M), 5), whole((n + more, N), 6)
    x[n:] = dy[n:] = float("nan")
    flat = whole((E * M * N + 128,), 7, dtype) * 50
    before = flat.clone()
    out = flat[64:-64].view(E, M, N)
    moe.moe_grouped_gemm_wgrad(x, dy, offsets_of(rows), out=out, accumulate=accumulate)
    old = before[64:-64].view(E, M, N)
    with_rows = set()
    for e, a, b in experts(rows):
        ref = torch.mm(x[a:b].double().t().contiguous(), dy[a:b].double())
        assert torch.equal(out[e], (ref + old[e].double() if accumulate else ref).to(dtype)), e
        with_rows.add(e)
    for e in set(range(E)) - with_rows:
        assert torch.equal(out[e], old[e] if accumulate else torch.zeros_like(out[e])), e
    assert torch.equal(flat[:64], before[:64]) and torch.equal(flat[-64:], before[-64:])
