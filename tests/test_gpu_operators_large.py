"""The memory-bound operators around the experts' weights at sizes where other variants of their kernels run (longer parts,
the non-temporal hint, several turns of a workgroup, bands), against 64 bits on the GPU."""
import math

import pytest
import torch

import paper_2605_19945_amd as moe
from test_gpu_operators import ref_quantize, unpack

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, seed, std=1.0, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=torch.Generator(device="cuda").manual_seed(seed))


# (values, type, values in front of the first one, of the output), in turn
MIXED = [(30_000_007, F32, 1, 1), (70_000_003, BF16, 3, 3), (4_099, BF16, 0, 1), (0, F32, 0, 0), (9_999_999, BF16, 5, 6), (1, F32, 2, 2), (6_000_001, F32, 0, 3)]
LISTS = {
    "long parts": [(12_000_001, BF16, 1, 1), (16_385, F32, 3, 3), (7_000_000, BF16, 0, 7)],   # above 16.8 M values
    "past the cache": MIXED,                                                                    # above 256 MB
    "past the cache, several launches": MIXED + [(333_333, BF16, 1, 1)] * 128 + MIXED[1:2],
}


def tensors_of(sizes, which, seed):
    """Gradients (which 2) or outputs (which 3) at their places."""
    out = []
    for i, size in enumerate(sizes):
        n, dtype, ahead = size[0], size[1], size[which]
        t = normal((ahead + n + 8,), seed + i, 1e-2, dtype) if which == 2 else torch.full((ahead + n + 8,), 9.0, dtype=dtype, device="cuda")
        out.append(t[ahead:ahead + n])
    return out


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("share", [0.25, 4.0])
def test_clip_grad_norm_of_long_lists(name, share):
    sizes = LISTS[name]
    grads, out = tensors_of(sizes, 2, 1), tensors_of(sizes, 3, 0)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    # squares and their sums are formed in 64 bits here and there; the norm is rounded to 32 once
    assert abs(float(moe.moe_grad_norm(grads)) - norm) <= 2.0 ** -23 * norm
    before = [g.clone() for g in grads]
    assert abs(float(moe.moe_clip_grad_norm(grads, share * norm, out=out)) - norm) <= 2.0 ** -23 * norm
    scale = min(1.0, share * norm / (norm + 1e-6))

    def right(g, o):  # the product in 32 bits with a scale of 32 bits, and one rounding to bf16
        rounding = 2.0 ** -8 * 1.01 if g.dtype == BF16 else 2.0 ** -22
        return bool(((o.double() - g.double() * scale).abs() <= rounding * g.double().abs() * scale + 1e-38).all())

    for g, b, o in zip(grads, before, out):
        assert torch.equal(g, b) and right(g, o)
        rest = torch.as_strided(o, (8,), (1,), o.storage_offset() + o.numel())
        assert (rest == 9).all()
    moe.moe_clip_grad_norm(grads, share * norm)
    for g, b, o in zip(grads, before, out):
        assert torch.equal(g, o) and (share < 1 or torch.equal(g, b))


def test_swiglu_and_its_gradient_past_the_cache():
    """More than 128 MB of results: the bounds are those of the small sizes."""
    rows, f, live = 4099, 16_392, 4097
    off = torch.tensor([0, 40, live], dtype=torch.int32).cuda()
    gu, dh = normal((rows, 2 * f), 11, 3.0), normal((rows, f), 12)
    gu[0, :8] = torch.tensor([0.0, -0.0, 100.0, -100.0, 1e30, -1e30, 88.0, -88.0], dtype=BF16)
    h, again = torch.full((rows, f), 3.0, dtype=BF16, device="cuda"), torch.full((rows, f), 3.0, dtype=BF16, device="cuda")
    dgu = torch.full((rows, 2 * f), 3.0, dtype=BF16, device="cuda")
    moe.moe_swiglu(gu, offsets=off, out=h)
    moe.moe_swiglu_backward(dh, gu, offsets=off, out=dgu, h=again)
    assert torch.equal(again, h) and (h[live:] == 3).all() and (dgu[live:] == 3).all()
    assert torch.equal(moe.moe_swiglu_backward(dh, gu)[:live], dgu[:live])
    small = 2.0 ** -19
    for a in range(0, live, 1024):
        b = min(a + 1024, live)
        g, u, d = gu[a:b, :f].double(), gu[a:b, f:].double(), dh[a:b].double()
        s = torch.sigmoid(g)
        assert ((h[a:b].double() - g * s * u).abs() <= (2.0 ** -8 * 1.01 + small) * (g * s * u).abs() + 1e-37).all()
        dg, du = d * u * s * (1 + g * (1 - s)), d * g * s
        terms = (d * u).abs() * s * (1 + g.abs() * (1 - s))
        assert ((dgu[a:b, :f].double() - dg).abs() <= 2.0 ** -8 * 1.01 * dg.abs() + small * terms + 1e-37).all()
        assert ((dgu[a:b, f:].double() - du).abs() <= (2.0 ** -8 * 1.01 + small) * du.abs() + 1e-37).all()
    moe.moe_swiglu_backward(dh, gu, offsets=off, out=gu)  # over gu itself
    assert torch.equal(gu[:live], dgu[:live])


@pytest.mark.parametrize("E,K,N", [(2, 1312, 264), (1, 2592, 136), (3, 1056, 392)])  # bands of 4 and 2, of 4, 4 and 3, of 4 and 1 stretches
def test_mxfp4_quantize_weights_in_bands(E, K, N):
    w = normal((E, K, N), 13, 0.02)
    values, scales = moe.moe_mxfp4_quantize_weights(w)
    for e in range(E):
        code, byte = ref_quantize(w[e].t().cpu().double().numpy())
        assert (unpack(values[e]) == code).all() and (scales[e].cpu().numpy()[:, :K // 32] == byte).all()
        assert (scales[e].cpu().numpy()[:, K // 32:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_mxfp4_rows_of_several_turns(dtype):
    """More rows than the workgroups take at once, there and back; a sample of them against the search for the nearest code, and all of
    them against the bound of half a step between neighbouring values."""
    rows, K = 5003, 4128
    x = normal((rows, K + 8), 14, dtype=dtype)[:, :K]
    values, scales = moe.moe_mxfp4_quantize(x)
    pick = torch.tensor([0, 1, 2500, 3640, 3641, rows - 2, rows - 1])
    code, byte = ref_quantize(x[pick.cuda()].cpu().double().numpy())
    assert (unpack(values[pick.cuda()]) == code).all() and (scales[pick.cuda()].cpu().numpy()[:, :K // 32] == byte).all()
    assert (scales[:, K // 32:] == 0).all()
    back = moe.moe_mxfp4_dequantize(values, scales).double().view(rows, -1, 32)
    unit = torch.exp2(scales[:, :K // 32].double() - 127)[..., None]
    a = x.double().reshape(rows, -1, 32)
    # in units: steps of 0.5 below 2, 1 below 4, 2 below 6, and nothing above 6 although the largest magnitude is below 8
    m = (a / unit).abs()
    half = torch.where(m < 2, 0.25, torch.where(m < 4, 0.5, torch.where(m < 6, 1.0, m - 6)))
    assert (m.amax(-1) < 8).all() and (m.amax(-1) >= 4).all()
    assert ((back - a).abs() <= half * unit).all()
