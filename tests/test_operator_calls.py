"""What the binding refuses of the operators around the experts' weights beside types, shapes and places (no GPU needed)."""
import os

import pytest
import torch

import paper_2605_19945_amd as moe


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(moe.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return moe.load_library()


def test_nothing_that_needs_a_gradient_is_taken_without_a_word():
    """The calls record no graph.  A result through which torch would lose a gradient is refused, as torch's own calls with out= do
    (the message is looked at: these tensors would also be refused for their place)."""
    bf = torch.bfloat16
    x, w, off, dy = torch.zeros(4, 64, dtype=bf), torch.zeros(2, 64, 40, dtype=bf), torch.zeros(3, dtype=torch.int32), torch.zeros(4, 40, dtype=bf)
    gu, h = torch.zeros(4, 64, dtype=bf), torch.zeros(4, 32, dtype=bf)

    def learnt(t):
        return t.clone().requires_grad_()

    calls = [
        lambda: moe.moe_grouped_gemm(learnt(x), w, off),
        lambda: moe.moe_grouped_gemm(x, learnt(w), off),
        lambda: moe.moe_grouped_gemm(x, w, off, out=learnt(dy)),
        lambda: moe.moe_grouped_gemm_wgrad(learnt(x), dy, off),
        lambda: moe.moe_grouped_gemm_wgrad(x, learnt(dy), off),
        lambda: moe.moe_grouped_gemm_wgrad(x, dy, off, out=learnt(torch.zeros(2, 64, 40))),
        lambda: moe.moe_swiglu(learnt(gu)),
        lambda: moe.moe_swiglu(gu, out=learnt(h)),
        lambda: moe.moe_swiglu_backward(learnt(h), gu),
        lambda: moe.moe_swiglu_backward(h, learnt(gu)),
        lambda: moe.moe_swiglu_backward(h, gu, out=learnt(gu)),
        lambda: moe.moe_swiglu_backward(h, gu, h=learnt(h)),
        lambda: moe.moe_mxfp4_grouped_gemm(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 16, dtype=torch.uint8),
                                           torch.zeros(2, 40, 32, dtype=torch.uint8), torch.zeros(2, 40, 16, dtype=torch.uint8), off, out=learnt(dy)),
    ]
    for i, f in enumerate(calls):
        with pytest.raises(moe.MoEError, match="record no graph"):
            f()
            pytest.fail(f"call {i} was accepted")
        with torch.no_grad(), pytest.raises(moe.MoEError, match="on the GPU"):
            f()
