"""What the operators around the experts' weights refuse, before anything is launched: status codes of the C entry points
and errors of the binding (no GPU needed)."""
import ctypes as C
import os

import pytest
import torch

import paper_2605_19945_amd as moe

P = C.c_void_p(4096)      # an aligned address that nothing looks behind
OFF = C.c_void_p(4100)    # aligned to 4 bytes only
INVALID, SHAPE, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(moe.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return moe.load_library()


def call(fn, base, **change):
    args = dict(base, **change)
    return fn(*args.values())


def test_grouped_gemm(lib):
    base = dict(x=P, ldx=64, w=P, t=0, offsets=P, rows=0, E=2, K=64, N=64, y=P, ldy=64, ws=None, bytes=0, stream=None)
    assert call(lib.moe_grouped_gemm, base) == 0          # no rows: nothing to do
    for change in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(E=0), dict(offsets=None), dict(offsets=C.c_void_p(4097)), dict(w=None),
                   dict(w=OFF), dict(x=None, rows=1), dict(x=OFF, rows=1), dict(y=None, rows=1), dict(y=OFF), dict(ldx=56), dict(ldx=68),
                   dict(ldy=60), dict(ldx=(1 << 21) + 8)):
        assert call(lib.moe_grouped_gemm, base, **change) == INVALID, change
    for change in (dict(E=257), dict(K=0), dict(K=60), dict(N=4), dict(N=-8), dict(K=(1 << 17) + 8, ldx=1 << 18)):
        assert call(lib.moe_grouped_gemm, base, **change) == SHAPE, change


def test_grouped_wgrad(lib):
    base = dict(x=P, ldx=64, dy=P, lddy=64, offsets=P, rows=1, E=2, K=64, N=64, dw=P, type=0, acc=0, ws=None, bytes=0, stream=None)
    for change in (dict(rows=-1), dict(E=0), dict(offsets=None), dict(dw=None), dict(dw=OFF), dict(x=None), dict(dy=OFF), dict(ldx=32),
                   dict(lddy=65), dict(type=2), dict(type=0, acc=1)):
        assert call(lib.moe_grouped_gemm_wgrad, base, **change) == INVALID, change
    for change in (dict(E=300), dict(K=12), dict(N=1 << 18)):
        assert call(lib.moe_grouped_gemm_wgrad, base, **change) == SHAPE, change


def test_workspaces_of_the_grouped_products(lib):
    """A long reduction of few tiles is cut and needs a workspace, which is checked; sizes that are none need none."""
    need = lib.moe_grouped_gemm_workspace_bytes(2, 1, 14336, 128, 0)
    assert need > 0 and need % (2 * 128 * 4) == 0
    base = dict(x=P, ldx=14336, w=P, t=0, offsets=P, rows=2, E=1, K=14336, N=128, y=P, ldy=128, ws=P, bytes=need - 1, stream=None)
    assert call(lib.moe_grouped_gemm, base) == WORKSPACE
    assert call(lib.moe_grouped_gemm, base, bytes=need, ws=None) == INVALID and call(lib.moe_grouped_gemm, base, bytes=need, ws=OFF) == INVALID
    need = lib.moe_grouped_gemm_wgrad_workspace_bytes(8192, 1, 64, 64)
    assert need > 0 and need % (64 * 64 * 4) == 0
    base = dict(x=P, ldx=64, dy=P, lddy=64, offsets=P, rows=8192, E=1, K=64, N=64, dw=P, type=0, acc=0, ws=P, bytes=need - 1, stream=None)
    assert call(lib.moe_grouped_gemm_wgrad, base) == WORKSPACE
    assert call(lib.moe_grouped_gemm_wgrad, base, bytes=need, ws=None) == INVALID
    need = lib.moe_mxfp4_grouped_gemm_workspace_bytes(2, 1, 14336, 64)
    assert need > 0
    base = dict(xq=P, xs=P, wq=P, wsc=P, offsets=P, rows=2, E=1, K=14336, N=64, y=P, ldy=64, ws=P, bytes=need - 1, stream=None)
    assert call(lib.moe_mxfp4_grouped_gemm, base) == WORKSPACE
    # enough tiles, or sizes that are refused
    assert lib.moe_grouped_gemm_workspace_bytes(8192, 8, 4096, 28672, 0) == 0
    assert lib.moe_grouped_gemm_workspace_bytes(-1, 8, 4096, 28672, 0) == 0 and lib.moe_grouped_gemm_workspace_bytes(2, 1, 14337, 128, 0) == 0
    assert lib.moe_mxfp4_grouped_gemm_workspace_bytes(2, 1, 48, 64) == 0
    # never past 64 MiB
    for rows in (1, 100, 5000, 1 << 20):
        for E, K, N in ((1, 131072, 8), (256, 131072, 8), (1, 131072, 4096), (8, 14336, 512)):
            assert lib.moe_grouped_gemm_workspace_bytes(rows, E, K, N, 0) <= 64 << 20
            assert lib.moe_grouped_gemm_wgrad_workspace_bytes(rows, E, K, N) <= 64 << 20


def test_swiglu(lib):
    base = dict(gu=P, ldgu=128, n=None, rows=0, f=64, h=P, ldh=64, stream=None)
    assert call(lib.moe_swiglu, base) == 0
    for change in (dict(rows=-1), dict(n=C.c_void_p(4098)), dict(gu=None, rows=1), dict(gu=OFF), dict(h=OFF), dict(ldgu=120), dict(ldgu=132),
                   dict(ldh=32)):
        assert call(lib.moe_swiglu, base, **change) == INVALID, change
    assert call(lib.moe_swiglu, base, f=12) == SHAPE and call(lib.moe_swiglu, base, f=0) == SHAPE
    base = dict(dh=P, lddh=64, gu=P, ldgu=128, n=None, rows=0, f=64, dgu=P, lddgu=128, h=None, ldh=0, stream=None)
    assert call(lib.moe_swiglu_backward, base) == 0
    for change in (dict(rows=-1), dict(dh=OFF), dict(gu=OFF), dict(dgu=OFF), dict(h=OFF), dict(h=P, ldh=32), dict(lddh=8), dict(lddgu=64),
                   dict(dgu=None, rows=1)):
        assert call(lib.moe_swiglu_backward, base, **change) == INVALID, change


def test_lists_of_gradients(lib):
    n = 3
    ptrs, counts, types = (C.c_void_p * n)(4096, 4100, 4104), (C.c_int64 * n)(5, 5, 5), (C.c_int32 * n)(0, 1, 0)
    need = lib.moe_grad_norm_workspace_bytes(n)
    assert need > 0 and lib.moe_grad_norm_workspace_bytes(-1) == 0
    assert lib.moe_grad_norm_workspace_bytes(1000) > need
    base = dict(grads=ptrs, counts=counts, types=types, n=n, ws=P, bytes=need, norm=P, stream=None)
    for change in (dict(n=-1), dict(grads=None), dict(counts=None), dict(types=None), dict(ws=None), dict(ws=OFF), dict(norm=None),
                   dict(norm=C.c_void_p(4098)), dict(types=(C.c_int32 * n)(0, 2, 0)), dict(counts=(C.c_int64 * n)(5, -1, 5)),
                   dict(grads=(C.c_void_p * n)(4096, 4098, 4104)), dict(grads=(C.c_void_p * n)(4096, None, 4104))):
        assert call(lib.moe_grad_norm, base, **change) == INVALID, change
    assert call(lib.moe_grad_norm, base, bytes=need - 1) == WORKSPACE
    base = dict(grads=ptrs, outs=ptrs, counts=counts, types=types, n=n, max_norm=1.0, ws=P, bytes=need, norm=P, stream=None)
    for change in (dict(outs=None), dict(outs=(C.c_void_p * n)(4096, 4100, 4105)), dict(max_norm=-1.0), dict(max_norm=float("nan"))):
        assert call(lib.moe_clip_grad_norm, base, **change) == INVALID, change
    assert call(lib.moe_clip_grad_norm, base, bytes=0) == WORKSPACE


def test_mxfp4(lib):
    assert [lib.moe_mxfp4_scale_cols(K) for K in (32, 512, 544, 14336, 1 << 17)] == [16, 16, 32, 448, 4096]
    assert [lib.moe_mxfp4_scale_cols(K) for K in (0, 16, 48, -32, (1 << 17) + 32)] == [0] * 5
    base = dict(x=P, type=0, ldx=64, n=None, rows=0, K=64, q=P, s=P, stream=None)
    assert call(lib.moe_mxfp4_quantize, base) == 0
    for change in (dict(rows=-1), dict(type=5), dict(ldx=32), dict(ldx=68), dict(x=OFF), dict(q=OFF), dict(s=OFF), dict(q=None, rows=1),
                   dict(n=C.c_void_p(4097))):
        assert call(lib.moe_mxfp4_quantize, base, **change) == INVALID, change
    assert call(lib.moe_mxfp4_quantize, base, K=48) == SHAPE
    base = dict(w=P, E=1, K=64, N=64, q=P, s=P, stream=None)
    for change in (dict(E=0), dict(w=None), dict(q=OFF), dict(s=None)):
        assert call(lib.moe_mxfp4_quantize_weights, base, **change) == INVALID, change
    for change in (dict(E=257), dict(K=40), dict(N=12)):
        assert call(lib.moe_mxfp4_quantize_weights, base, **change) == SHAPE, change
    base = dict(q=P, s=P, rows=0, K=64, x=P, ldx=64, stream=None)
    assert call(lib.moe_mxfp4_dequantize, base) == 0
    assert call(lib.moe_mxfp4_dequantize, base, rows=-1) == INVALID and call(lib.moe_mxfp4_dequantize, base, ldx=63) == INVALID
    assert call(lib.moe_mxfp4_dequantize, base, K=16) == SHAPE
    base = dict(xq=P, xs=P, wq=P, ws=P, offsets=P, rows=0, E=2, K=64, N=64, y=P, ldy=64, space=None, bytes=0, stream=None)
    assert call(lib.moe_mxfp4_grouped_gemm, base) == 0
    for change in (dict(rows=-1), dict(offsets=None), dict(xq=OFF), dict(xs=OFF), dict(wq=None), dict(ws=OFF), dict(y=OFF), dict(ldy=8)):
        assert call(lib.moe_mxfp4_grouped_gemm, base, **change) == INVALID, change
    assert call(lib.moe_mxfp4_grouped_gemm, base, K=40) == SHAPE and call(lib.moe_mxfp4_grouped_gemm, base, N=9) == SHAPE


def test_binding_refuses_what_it_cannot_pass_on(lib):
    bf = torch.bfloat16
    x, w, off = torch.zeros(4, 64, dtype=bf), torch.zeros(2, 64, 40, dtype=bf), torch.zeros(3, dtype=torch.int32)
    bad = [
        lambda: moe.moe_grouped_gemm(x, w, off),                               # not on a GPU
        lambda: moe.moe_grouped_gemm(x.float(), w, off),
        lambda: moe.moe_grouped_gemm(x, w.float(), off),
        lambda: moe.moe_grouped_gemm(x, w[0], off),
        lambda: moe.moe_grouped_gemm(x[:, :32], w, off),
        lambda: moe.moe_grouped_gemm(x.t(), w.transpose(1, 2), off),
        lambda: moe.moe_grouped_gemm(x, w, off[:2]),
        lambda: moe.moe_grouped_gemm(x, w, off.long()),
        lambda: moe.moe_grouped_gemm(x, w, off, transpose_w=True),
        lambda: moe.moe_grouped_gemm(x, w, off, out=torch.zeros(3, 40, dtype=bf)),
        lambda: moe.moe_grouped_gemm(x, w, off, out=torch.zeros(4, 40)),
        lambda: moe.moe_grouped_gemm_wgrad(x, x[:2], off),
        lambda: moe.moe_grouped_gemm_wgrad(x, x, off, accumulate=True),
        lambda: moe.moe_grouped_gemm_wgrad(x, x, off, dtype=torch.float16),
        lambda: moe.moe_grouped_gemm_wgrad(x, x, off, dtype=bf, out=torch.zeros(2, 64, 64)),
        lambda: moe.moe_grouped_gemm_wgrad(x, x, off, out=torch.zeros(2, 64, 63)),
        lambda: moe.moe_swiglu(x[:, :63]),
        lambda: moe.moe_swiglu(x, offsets=off.float()),
        lambda: moe.moe_swiglu(x),
        lambda: moe.moe_swiglu_backward(x, x),
        lambda: moe.moe_swiglu_backward(x[:2, :32], x),
        lambda: moe.moe_grad_norm([x.half()]),
        lambda: moe.moe_grad_norm([x.t()]),
        lambda: moe.moe_clip_grad_norm([x], 1.0),
        lambda: moe.moe_clip_grad_norm([x], 1.0, out=[x[:2]]),
        lambda: moe.moe_clip_grad_norm([x], 1.0, out=[]),
        lambda: moe.moe_mxfp4_quantize(x.half()),
        lambda: moe.moe_mxfp4_quantize(x),
        lambda: moe.moe_mxfp4_quantize_weights(w[0]),
        lambda: moe.moe_mxfp4_dequantize(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.uint8)),
        lambda: moe.moe_mxfp4_dequantize(torch.zeros(2, 20, dtype=torch.uint8), torch.zeros(2, 16, dtype=torch.uint8)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(moe.MoEError):
            f()
            pytest.fail(f"call {i} was accepted")
