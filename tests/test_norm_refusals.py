"""What the norms around a block refuse, before anything is launched (no GPU needed)."""
import ctypes as C
import os

import pytest
import torch

import paper_2605_19945_amd as moe

INVALID, SHAPE, WORKSPACE = 1, 2, 3
OFF = C.c_void_p(4100)    # aligned to 4 bytes only


def at(k):
    """Addresses far from each other that nothing looks behind."""
    return C.c_void_p((k + 1) << 32)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(moe.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return moe.load_library()


def call(fn, base, **change):
    return fn(*dict(base, **change).values())


def test_norm(lib):
    base = dict(x=at(0), xt=0, ldx=64, w=at(1), wt=1, eps=1e-6, n=at(2), rows=0, d=64, h=at(3), ht=0, ldh=64, stream=None)
    assert call(lib.moe_rms_norm, base) == 0
    for change in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(n=C.c_void_p(4097)), dict(xt=2),
                   dict(ht=-1), dict(wt=3), dict(ht=1), dict(w=OFF), dict(x=OFF), dict(h=OFF), dict(ldx=56), dict(ldx=68), dict(ldh=60), dict(x=None, rows=1),
                   dict(h=None, rows=1), dict(ldx=(1 << 21) + 8), dict(rows=4, h=C.c_void_p((1 << 32) + 16)), dict(rows=4, h=at(1)), dict(rows=4, h=at(2))):
        assert call(lib.moe_rms_norm, base, **change) == INVALID, change
    for d in (0, 4, 12, -8, 16392):
        assert call(lib.moe_rms_norm, base, d=d) == SHAPE, d


def test_norm_backward(lib):
    need = lib.moe_norm_backward_workspace_bytes(4, 64)
    assert need > 0 and lib.moe_norm_backward_workspace_bytes(-1, 64) == lib.moe_norm_backward_workspace_bytes(4, 60) == 0
    assert lib.moe_norm_backward_workspace_bytes(1 << 24, 16384) <= 128 << 20
    base = dict(dh=at(0), ht=0, lddh=64, x=at(1), xt=0, ldx=64, w=at(2), wt=1, eps=1e-6, dres=at(3), lddres=64, n=at(4), rows=4, d=64, dx=at(5), lddx=64,
                dw=at(6), ws=at(7), bytes=need, stream=None)
    assert call(lib.moe_rms_norm_backward, base, bytes=need - 1) == WORKSPACE
    for change in (dict(ws=None), dict(ws=OFF), dict(dh=None), dict(x=OFF), dict(dx=None), dict(dw=OFF), dict(dres=OFF), dict(lddres=63), dict(lddx=8),
                   dict(lddh=70), dict(ht=1), dict(dx=C.c_void_p((1 << 32) + 16)), dict(dx=at(2)), dict(dx=at(4)), dict(dw=at(1)), dict(dw=at(5)),
                   dict(ws=at(5)), dict(ws=at(6)), dict(ws=at(0)), dict(eps=-0.5), dict(rows=-4)):
        assert call(lib.moe_rms_norm_backward, base, **change) == INVALID, change
    assert call(lib.moe_rms_norm_backward, base, d=60) == SHAPE


def test_join(lib):
    base = dict(x=at(0), xt=0, ldx=64, y=at(1), yt=0, ldy=64, w=at(2), wt=1, norm=1, gate=at(3), ldgate=64, scale=1.0, nxt=at(4), eps=1e-6, n=at(5), rows=0,
                d=64, out=at(6), ldout=64, h=at(7), ldh=64, stream=None)
    assert call(lib.moe_residual_norm, base) == 0
    for change in (dict(h=None, rows=1), dict(gate=None), dict(gate=OFF), dict(gate=C.c_void_p(4098), ldgate=0), dict(ldgate=60), dict(y=OFF), dict(out=OFF), dict(ldy=32),
                   dict(yt=1), dict(xt=5), dict(nxt=OFF), dict(wt=2), dict(rows=4, y=None), dict(rows=4, out=at(7)), dict(rows=4, out=at(2)), dict(rows=4, h=at(4)),
                   dict(rows=4, out=C.c_void_p((1 << 32) + 128)), dict(rows=4, h=C.c_void_p((2 << 32) + 16)), dict(rows=4, out=at(3), ldgate=0), dict(rows=4, h=at(5))):
        assert call(lib.moe_residual_norm, base, **change) == INVALID, change
    assert call(lib.moe_residual_norm, base, d=20) == SHAPE


def test_join_backward(lib):
    need = lib.moe_norm_backward_workspace_bytes(4, 64)
    base = dict(dout=at(0), lddout=64, dh=at(1), lddh=64, o=at(2), xt=0, ldo=64, y=at(3), yt=0, ldy=64, w=at(4), wt=1, norm=1, gate=at(5), ldgate=64, scale=1.0,
                nxt=at(6), eps=1e-6, n=at(7), rows=4, d=64, dx=at(8), lddx=64, dy=at(9), lddy=64, dgate=at(10), lddgate=64, dw=at(11), dnext=at(12), ws=at(13),
                bytes=need, stream=None)
    assert call(lib.moe_residual_norm_backward, base, bytes=0) == WORKSPACE
    for change in (dict(ws=None), dict(dh=None), dict(dh=None, nxt=None), dict(o=None), dict(y=None), dict(dx=None), dict(dy=OFF), dict(gate=None), dict(gate=None, ldgate=0),
                   dict(dgate=OFF), dict(lddgate=56), dict(dw=OFF), dict(dnext=OFF), dict(dy=at(8)), dict(dgate=at(8)), dict(dgate=at(9)), dict(dx=at(4)), dict(dw=at(12)),
                   dict(dw=at(3)), dict(dnext=at(8)), dict(ws=at(12)), dict(ws=at(9)), dict(dx=C.c_void_p((1 << 32) + 8 * 16)), dict(dy=C.c_void_p((4 << 32) + 16)),
                   dict(ldgate=0, dgate=at(5)), dict(ldgate=0, dgate=at(9)), dict(yt=1), dict(ldo=0), dict(eps=float("nan"))):
        assert call(lib.moe_residual_norm_backward, base, **change) == INVALID, change
    assert call(lib.moe_residual_norm_backward, base, d=16400) == SHAPE


def refused(fn, *args, **kw):
    with pytest.raises(moe.MoEError):
        fn(*args, **kw)


def test_the_binding_refuses(lib):
    BF16, F32 = torch.bfloat16, torch.float32
    x, w = torch.ones(4, 64, dtype=BF16), torch.ones(64)
    refused(moe.moe_rms_norm, x, w)                                                     # not on the GPU
    for bad_x, bad_w in ((x.half(), w), (x[0], w), (x.t(), w), (x, w[:32]), (x, w.half()), (x, torch.ones(128)[::2]), (x.requires_grad_(False).float().requires_grad_(), w)):
        refused(moe.moe_rms_norm, bad_x, bad_w)
    refused(moe.moe_rms_norm, x, w, dtype=F32)                                          # a wider block than its stream
    refused(moe.moe_rms_norm, x, w, dtype=torch.float16)
    refused(moe.moe_rms_norm, x, w, offsets=torch.zeros(3))
    refused(moe.moe_rms_norm_backward, x[:3], x, w)
    refused(moe.moe_rms_norm_backward, x.float(), x, w)
    refused(moe.moe_rms_norm_backward, x, x, w, dres=x.float())
    refused(moe.moe_residual_norm, x, x.float(), w)
    refused(moe.moe_residual_norm, x, x, w, next_weight=w.to(BF16))                     # weights of two types
    refused(moe.moe_residual_norm, x, x, w, gate=torch.ones(4, dtype=BF16))
    refused(moe.moe_residual_norm, x, x, w, gate=torch.ones(5))
    refused(moe.moe_residual_norm, x, x, w, gate=torch.ones(4, 64))
    refused(moe.moe_residual_norm, x, x, w, h=x)
    refused(moe.moe_residual_norm_backward, x, x, w, dh=x, next_weight=w)               # without out
    refused(moe.moe_residual_norm_backward, x, x, w, next_weight=w)
    refused(moe.moe_residual_norm_backward, x, x, w, dh=x, out=x)
    refused(moe.moe_residual_norm_backward, None, x, w)
    refused(moe.moe_residual_norm_backward, x, x, w, gate=torch.ones(3))
