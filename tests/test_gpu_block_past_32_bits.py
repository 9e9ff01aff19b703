"""The operators around a block on tensors of more than 2^31 values and stacks past the workspace: what lies behind that is looked at, with the
bounds of the small sizes."""
import pytest
import torch

import paper_2605_19945_amd as moe
import test_gpu_norms as norms
import test_gpu_orthogonalize as orth

pytestmark = pytest.mark.gpu

BF16, F32, LINE = torch.bfloat16, torch.float32, 1 << 31


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def normal(shape, seed, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("d", [16384, 512])
def test_long_streams(d):
    rows = LINE // d + 70
    x, y, w = normal((rows, d), 1), normal((rows, d), 2), normal((d,), 3, F32)
    pick = torch.tensor([0, 1, LINE // d - 1, LINE // d, LINE // d + 1, rows - 2, rows - 1])
    at = pick.cuda()
    out, h = moe.moe_residual_norm(x, y, w, next_weight=w, eps=norms.EPS)
    c = dict(x=x[at].cpu(), y=y[at].cpu(), w=w.cpu(), next=w.cpu(), gate=None, norm=True)
    ref = norms.ref_forward(c, 1.0)
    norms.close(out[at], ref[0], ref[1], norms.ONCE)
    norms.close(h[at], ref[2], ref[3], norms.TWICE)
    del h
    # gradients: rows in the middle of which nothing comes back but from those looked at, so the weights' sums are theirs
    dout = torch.zeros_like(x)
    dout[at] = normal((len(pick), d), 4)
    dx, dy, dw, _, _ = moe.moe_residual_norm_backward(dout, y, w, eps=norms.EPS)
    c.update(dout=dout[at].cpu(), dh=None, next=None)
    norms.check_backward((dx[at], dy[at], dw, None, None), c, 1.0)
    assert not dx[2:100].any() and not dy[2:100].any()


@pytest.mark.parametrize("rows,cols", [(60, 70), (300, 280), (1100, 70)])
def test_matrices_far_apart(rows, cols):
    """Matrices 2^30 values from each other, and rows 2^21 values from each other (of matrices beside each other in these rows)."""
    room = torch.zeros(1101 << 21, dtype=BF16, device="cuda")
    G = normal((3, rows, cols), 5)
    for size in ((1 << 30, cols), (cols, 1 << 21)):
        view = room.as_strided((3, rows, cols), (size[0], size[1], 1), 3)
        view.copy_(G)
        got = moe.moe_orthogonalize(view, out=view)
        assert got is view
        orth.check(got.contiguous(), G)
        view.zero_()
        assert not room[:1 << 22].any()


def test_flat_matrices_in_turns():
    """Stacks of matrices of up to 128 rows past the workspace's 8 GiB; the last turn has fewer matrices, and so more workgroups for each."""
    rows, cols = 100, 60000
    lib = moe.load_library()
    E = next(e for e in range(2, 257) if lib.moe_orthogonalize_workspace_bytes(e, rows, cols) == lib.moe_orthogonalize_workspace_bytes(256, rows, cols)) + 4
    assert 100 < E <= 252
    G = normal((E, rows, cols), 6)
    got = moe.moe_orthogonalize(G)
    for e in (0, E - 6, E - 5, E - 4, E - 2, E - 1):
        orth.check(got[e], G[e])
