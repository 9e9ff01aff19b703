"""How far orthogonalised updates are from 64 bits, beside the same steps with products in 32 bits.

Bounds.  fp32 results: products in 32 bits round 2^-24 of each sum as it grows, by chance about (k / 3)^1/2 2^-24 of the magnitudes of k terms; two parts of
fp16 hold 22 bits, off by 2^-23 of the value at most and 2^-23 / 3^1/2 in the mean square, of both operands, and their sums round as often as matrix instructions
add, k / 32 times, twice (two small products): for k of 64 and more that is within the mean square of the former, so the two errors are of one size; each
is one draw, carried on by five steps, and 2 leaves one draw that much room.  Below |g| = eps the steps are next to a factor and nothing is carried on: there an
fp32 result is held to 6 roundings of X to 22 bits and as many of products (12^1/2 2^-22 of its norm, and twice that).
bf16 results: one part holds 11 bits, a rounding by chance 2^-12 / 3^1/2 of the value, as often as 5 steps of 4 operands, but the result's own
rounding is 2^-9 / 3^1/2 2^1/2, five times as much as each: less than 2 of that in all."""
import pytest
import torch

import paper_2605_19945_amd as moe
from test_gpu_orthogonalize import ABC, BF16, F32, gradient, steps_of
from test_gpu_orthogonalize_schedules import DAMPED, RAISING

pytestmark = pytest.mark.gpu


def plain(G, coefficients, eps=1e-7):
    """The steps in 32 bits."""
    tall = G.shape[0] > G.shape[1]
    X = (G.t() if tall else G).float()
    X = X / (X.square().sum().sqrt() + eps)
    for a, b, c in coefficients:
        S = X @ X.t()
        X = a * X + (b * S + c * (S @ S)) @ X
    return (X.t() if tall else X).to(G.dtype)


def errors(G, coefficients):
    ref = steps_of(G, coefficients)
    got = moe.moe_orthogonalize(G, steps=len(coefficients), coefficients=coefficients)
    return tuple(float((t.double() - ref).norm() / ref.norm()) for t in (got, plain(G, coefficients)))


@pytest.mark.parametrize("rows,cols", [(64, 300), (100, 2000), (128, 256), (300, 400), (768, 2048), (2048, 512), (1024, 1024), (1100, 1300), (2048, 4096)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["gauss", "steep"])
def test_errors_beside_32_bit_products(rows, cols, dtype, kind):
    G = gradient((rows, cols), rows + cols, dtype, kind).cuda()
    for coefficients in ((ABC,) * 5, RAISING[:5], DAMPED[:5]):
        ours, theirs = errors(G, coefficients)
        print(rows, cols, dtype, kind, f"{coefficients[0][0]:.2f}: {ours:.3e}, of 32-bit products {theirs:.3e}, {ours / theirs:.2f} times", flush=True)
        assert ours <= 2 * theirs


@pytest.mark.parametrize("rows,cols", [(24, 83), (100, 500), (300, 400), (2048, 4096)])
def test_errors_far_below_eps(rows, cols):
    for share in (1e-4, 1e-6, 1e-12):
        G = gradient((rows, cols), 5, F32).cuda().double()
        G = (G / G.norm() * (share * 1e-7)).float()
        ours, _ = errors(G, (ABC,) * 5)
        assert ours <= 2 * 12 ** 0.5 * 2.0 ** -22


def test_errors_of_a_stack_in_pairs():
    """Steps in pairs with a pair at the end: its Q S Q is the last S there is."""
    G = gradient((128, 768, 2048), 768 + 2048, F32).cuda()
    for coefficients in (RAISING[:5], DAMPED[:5], RAISING[:6]):
        ref = steps_of(G[0], coefficients)
        got = moe.moe_orthogonalize(G, steps=len(coefficients), coefficients=coefficients)[0]
        ours, theirs = (float((t.double() - ref).norm() / ref.norm()) for t in (got, plain(G[0], coefficients)))
        assert ours <= 2 * theirs, (ours, theirs)
