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


# ---- outputs that lie over something else ----
# In: two matrices as address, rows, bytes between rows and of a row.  Out: 1 where they share a byte.
OVERLAP = r"""
#include "moe_overlap.h"
#include <cstdio>
int main() {
    long long a[4], b[4];
    while (scanf("%lld %lld %lld %lld %lld %lld %lld %lld", a, a + 1, a + 2, a + 3, b, b + 1, b + 2, b + 3) == 8)
        printf("%d\n", overlap(Rows((void*)a[0], a[1], a[2], a[3]), Rows((void*)b[0], b[1], b[2], b[3])));
}
"""


def test_matrices_that_share_bytes_are_found(tmp_path):
    """Against the sets of their bytes, over small matrices in all positions to each other."""
    import random
    import sched_host
    exe = sched_host.compile_host(OVERLAP, str(tmp_path))
    rng, cases = random.Random(3), []
    for _ in range(20000):
        one = []
        for _ in range(2):
            n, width = rng.choice([0, 1, 1, 2, 3, 5, 9]), rng.randint(1, 6)
            one.append((rng.randint(1, 40), n, width + rng.randint(0, 9) if n > 1 else rng.randint(1, 50), width))
        if rng.random() < 0.4 and one[0][1] > 1 and one[1][1] > 1:  # views into the same rows
            ld = max(one[0][2], one[1][2])
            one = [(at, n, ld, width) for at, n, _, width in one]
        cases.append(one)
    got = sched_host.run(exe, "\n".join(" ".join(map(str, a + b)) for a, b in cases)).split()
    bytes_of = lambda at, n, ld, width: {at + i * ld + j for i in range(n) for j in range(width)}
    assert len(got) == len(cases)
    for (a, b), g in zip(cases, got):
        assert int(g) == bool(bytes_of(*a) & bytes_of(*b)), (a, b)
    assert 2000 < sum(map(int, got)) < 18000


INVALID, DEVICE = 1, 4


def at(n):
    import ctypes as C
    return C.c_void_p(n)


# C entry, its arguments in memory of their own, and changes that move an output over an input (or another output) by a part of it.
# Nothing is launched, so nothing lies at these addresses.
APART = [
    ("moe_grouped_gemm", dict(x=1 << 20, ldx=64, w=1 << 24, t=0, offsets=1 << 12, rows=9, E=2, K=64, N=40, y=1 << 28, ldy=40, ws=None, bytes=0, stream=None),
     [dict(y=1 << 20), dict(y=(1 << 20) + 128 * 8 + 112), dict(y=(1 << 20) - 80 * 9 + 16), dict(y=1 << 24), dict(y=(1 << 24) + 2 * 64 * 40 * 2 - 16),
      dict(y=(1 << 20) + 64, ldx=128, ldy=128), dict(y=(1 << 24) - 160 * 8 - 80 + 16, ldy=80)]),
    ("moe_grouped_gemm_wgrad", dict(x=1 << 20, ldx=64, dy=1 << 24, lddy=40, offsets=1 << 12, rows=9, E=2, K=64, N=40, dw=1 << 28, type=1, acc=0, ws=None, bytes=0,
                                    stream=None),
     [dict(dw=1 << 20), dict(dw=(1 << 20) - 2 * 64 * 40 * 4 + 16), dict(dw=1 << 24), dict(dw=(1 << 24) + 80 * 9 - 16), dict(dw=1 << 24, acc=1)]),
    ("moe_swiglu", dict(gu=1 << 20, ldgu=144, n=None, rows=9, f=72, h=1 << 24, ldh=72, stream=None),
     [dict(h=1 << 20), dict(h=(1 << 20) + 144), dict(h=(1 << 20) + 16, ldh=144), dict(h=(1 << 20) + 144 + 288 * 8, ldh=72), dict(h=(1 << 20) + 128, ldh=144)]),
    ("moe_swiglu_backward", dict(dh=1 << 20, lddh=72, gu=1 << 24, ldgu=144, n=None, rows=9, f=72, dgu=1 << 28, lddgu=144, h=1 << 30, ldh=72, stream=None),
     [dict(dgu=1 << 20), dict(dgu=(1 << 24) + 16), dict(dgu=(1 << 24), lddgu=152), dict(dgu=(1 << 24) + 144, lddgu=144), dict(h=1 << 28, ldh=144), dict(h=1 << 24),
      dict(h=(1 << 20) + 16), dict(dgu=1 << 24, h=1 << 24, ldh=144), dict(dgu=1 << 24, h=(1 << 24) + 144, ldh=144)]),
    ("moe_mxfp4_quantize", dict(x=1 << 20, type=0, ldx=64, n=None, rows=9, K=64, q=1 << 24, s=1 << 28, stream=None),
     [dict(q=1 << 20), dict(s=1 << 20), dict(q=1 << 28), dict(s=(1 << 24) + 32 * 9 - 16), dict(q=(1 << 20) + 256 * 8 + 240, type=1)]),
    ("moe_mxfp4_quantize_weights", dict(w=1 << 20, E=2, K=64, N=40, q=1 << 24, s=1 << 28, stream=None),
     [dict(q=1 << 20), dict(s=(1 << 20) + 2 * 64 * 40 * 2 - 16), dict(s=1 << 24)]),
    ("moe_mxfp4_dequantize", dict(q=1 << 20, s=1 << 24, rows=9, K=64, x=1 << 28, ldx=64, stream=None),
     [dict(x=1 << 20), dict(x=(1 << 20) - 128 * 9 + 16), dict(x=(1 << 24) + 16 * 8)]),
    ("moe_mxfp4_grouped_gemm", dict(xq=1 << 20, xs=1 << 22, wq=1 << 24, ws=1 << 26, offsets=1 << 12, rows=9, E=2, K=64, N=40, y=1 << 28, ldy=40, space=None, bytes=0,
                                    stream=None),
     [dict(y=1 << 20), dict(y=(1 << 22) + 16 * 8), dict(y=1 << 24), dict(y=(1 << 26) + 2 * 40 * 16 - 16)]),
]


# Side by side, in place, or with nothing in the bytes between.
ASIDE = {
    "moe_grouped_gemm": [dict(y=(1 << 20) + 128, ldx=104, ldy=104), dict(y=(1 << 20) - 80, ldx=104, ldy=104), dict(y=(1 << 20) + 128 * 9), dict(y=(1 << 24) - 80 * 9),
                         dict(y=(1 << 20) + 128, ldx=208, ldy=104), dict(y=(1 << 24) - 160 * 8 - 80, ldy=80)],
    "moe_grouped_gemm_wgrad": [dict(dw=(1 << 20) + 128 * 9), dict(x=1 << 24, ldx=104, dy=(1 << 24) + 128, lddy=104)],
    "moe_swiglu": [dict(h=1 << 20, ldh=144), dict(h=(1 << 20) + 144, ldh=144), dict(h=(1 << 20) + 288, ldgu=216, ldh=216), dict(rows=1, h=1 << 20)],
    "moe_swiglu_backward": [dict(dgu=1 << 24), dict(h=1 << 20), dict(h=None), dict(h=1 << 24, ldh=144), dict(h=(1 << 24) + 144, ldh=144), dict(dgu=1 << 20, lddh=144)],
    "moe_mxfp4_quantize": [dict(n=1 << 12), dict(s=(1 << 24) + 32 * 9)],
    "moe_mxfp4_dequantize": [dict(x=(1 << 20) + 32, ldx=72, rows=1)],
}


@pytest.mark.skipif(torch.cuda.is_available(), reason="for the host: made-up addresses")
@pytest.mark.parametrize("name,base,changes", APART, ids=[a[0] for a in APART])
def test_outputs_over_inputs_are_refused(lib, name, base, changes):
    pointers = {"x", "w", "offsets", "y", "dy", "dw", "gu", "h", "dh", "dgu", "n", "q", "s", "xq", "xs", "wq", "ws"}

    def call(**change):
        return getattr(lib, name)(*[at(v) if k in pointers and v is not None else v for k, v in dict(base, **change).items()])

    for change in changes:
        assert call(**change) == INVALID, change
    for change in ASIDE.get(name, []) + [{}]:  # as far as the launch, for which there is no device
        assert call(**change) == DEVICE, change
