"""What the orthogonalised updates refuse, before anything is launched (no GPU needed)."""
import ctypes as C
import os

import pytest
import torch

import paper_2605_19945_amd as moe

INVALID, SHAPE, WORKSPACE = 1, 2, 3


def at(k, off=0):
    return C.c_void_p(((k + 1) << 36) + off)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(moe.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return moe.load_library()


def test_c_entry(lib):
    abc = (C.c_float * 6)(3.4445, -4.775, 2.0315, 1.5, -0.5, 0.0)
    need = lib.moe_orthogonalize_workspace_bytes(2, 64, 100)
    assert need > 0
    base = dict(g=at(0), type=1, sg=6400, ldg=100, E=2, rows=64, cols=100, abc=abc, steps=2, eps=1e-7, scale=1.0, out=at(1), ot=0, so=6400, ldo=100, ws=at(2),
                bytes=need, stream=None)

    def call(**change):
        return lib.moe_orthogonalize(*dict(base, **change).values())

    assert call(bytes=need - 1) == WORKSPACE
    nan = (C.c_float * 6)(1.0, float("nan"), 0, 0, 0, 0)
    for change in (dict(g=None), dict(out=None), dict(g=at(0, 2)), dict(out=at(1, 1)), dict(type=2), dict(ot=-1), dict(E=0), dict(rows=0), dict(cols=0), dict(abc=None),
                   dict(abc=nan), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(ldg=99), dict(ldo=64),
                   dict(sg=6399), dict(so=0), dict(sg=1 << 41), dict(ldg=(1 << 21) + 1), dict(ws=None), dict(ws=at(2, 16)), dict(out=at(0)), dict(out=at(0, 400)),
                   dict(out=at(0, 4), ot=1), dict(ws=at(0)), dict(ws=at(1)), dict(out=at(0), ot=1, so=6500)):
        assert call(**change) == INVALID, change
    for change in (dict(E=257), dict(rows=(1 << 17) + 1), dict(cols=(1 << 17) + 1), dict(rows=1 << 15, cols=(1 << 14) + 1)):
        assert call(**change) == SHAPE, change


def test_workspace(lib):
    ws = lib.moe_orthogonalize_workspace_bytes
    assert ws(0, 8, 8) == ws(257, 8, 8) == ws(1, 0, 8) == ws(1, 8, (1 << 17) + 1) == 0
    assert ws(8, 100, 50) == ws(8, 50, 100) <= 8 * ws(1, 100, 50)
    assert ws(256, 2048, 2048) <= 8 << 30 < 256 * ws(1, 2048, 2048)
    for rows, cols in ((1, 1), (4096, 14336), (7168, 2048)):   # about 8 bytes a value, whole tiles, sums of cut reductions
        assert ws(1, rows, cols) <= 8 * (rows + 256) * (cols + 256) + 12 * (min(rows, cols) + 256) ** 2 + (64 << 20)


def test_the_binding_refuses(lib):
    def refused(*args, **kw):
        with pytest.raises(moe.MoEError):
            moe.moe_orthogonalize(*args, **kw)

    g = torch.ones(2, 8, 16)
    refused(g)                                                      # not on the GPU
    refused(g.half())
    refused(g[0, 0])
    refused(g[None])
    refused(g.transpose(1, 2))
    refused(g[:, :, ::2])
    refused(g, dtype=torch.float16)
    refused(g, out=torch.ones(2, 8, 15))
    refused(g, out=torch.ones(2, 8, 16), dtype=torch.bfloat16)
    refused(g.clone().requires_grad_())
    for bad in ((1.0, 2.0), ((1.0, 2.0, 3.0),) * 4, (1.0, "x", 2.0), ((1.0, 2.0),) * 5, (1e300, 0.0, 0.0)):
        refused(g, coefficients=bad)
    for bad in (None, 1.0, [1.0, 2.0], torch.ones(2), ([1.0, 2.0, 3.0],) * 4, [[1.0, 2.0]] * 5, (torch.ones(3), 1.0, 2.0), "abc"):
        refused(g, coefficients=bad)
    for steps in (0, -1, 65, 10 ** 9, 5.0, "5", None):
        refused(g, steps=steps)


def test_coefficients_in_any_form():
    """Lists, tuples, arrays and tensors of numbers; a tensor whose values change is read again."""
    from paper_2605_19945_amd.binding import _coefficients
    one = _coefficients("", (3.0, -4.0, 2.0), 2)
    assert list(memoryview(one).cast("f")) == [3.0, -4.0, 2.0] * 2
    abc = torch.tensor([3.0, -4.0, 2.0])
    for same in ([3, -4, 2], abc, tuple(abc), abc.numpy(), [[3.0, -4.0, 2.0]] * 2, ([3.0, -4.0, 2.0], (3.0, -4.0, 2.0)), abc.expand(2, 3)):
        assert _coefficients("", same, 2) == one
    parts = tuple(abc)
    abc[0] = 1.0
    assert list(memoryview(_coefficients("", parts, 2)).cast("f")) == [1.0, -4.0, 2.0] * 2


def test_first_coefficients_that_no_scale_holds(lib):
    """Small singular values take Q's value at zero, which is the first coefficient."""
    need = lib.moe_orthogonalize_workspace_bytes(1, 8, 8)

    def call(*abc):
        return lib.moe_orthogonalize(at(0), 1, 64, 8, 1, 8, 8, (C.c_float * len(abc))(*abc), len(abc) // 3, 1e-7, 1.0, at(1), 1, 64, 8, at(2), need, None)

    for abc in ((4001.0, 0.0, 0.0), (-4001.0, 0.0, 0.0), (1.5, -0.5, 0.0, 1e6, 0.0, 0.0), (1.0, 1.1e6, 0.0), (1.0, 0.0, -1.1e6), (1.0, float("inf"), 0.0)):
        assert call(*abc) == INVALID, abc


def test_workspace_of_padded_sizes(lib):
    """What the header states, for small sides and stacks; and not less than X in two parts, twice, needs."""
    for E in (1, 3, 128):
        for rows, cols in ((1, 1), (1, 9), (1, 131072), (17, 8004), (33, 100), (65, 100), (128, 256), (129, 127), (129, 129), (200, 3000), (330, 826), (1024, 1024)):
            n, m = min(rows, cols), max(rows, cols)
            most = next((k for k in (32, 64, 128) if n <= k), -(-n // 256) * 256), (-(-m // 64) * 64 if n <= 128 else -(-m // 256) * 256) + 32
            bound = E * (8 * most[0] * most[1] + 12 * most[0] * (most[0] + 32) + 8 * most[0] + 4112) + (64 << 20)
            got = lib.moe_orthogonalize_workspace_bytes(E, rows, cols)
            assert 8 * E * n * m <= got <= min(bound, 8 << 30), (E, rows, cols)
            assert lib.moe_orthogonalize_workspace_bytes(E, cols, rows) == got
