"""The operators around the experts' weights on tensors of more than 2^31 values: what lies behind that is looked at, against
64 bits.  Whole numbers up to 2 give exact sums, so products are compared by equality; the other bounds are those of the small sizes."""
import math

import pytest
import torch

import paper_2605_19945_amd as moe
from test_gpu_operators import ref_quantize, unpack

pytestmark = pytest.mark.gpu

BF16, F32, LINE = torch.bfloat16, torch.float32, 1 << 31


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def whole(shape, seed, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=torch.int8, device="cuda").random_(-2, 3, generator=g).to(dtype)


def normal(shape, seed, std=1.0):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(0.0, std, generator=torch.Generator(device="cuda").manual_seed(seed))


def offsets_of(rows):
    off = torch.zeros(len(rows) + 1, dtype=torch.int32)
    off[1:] = torch.tensor(rows).cumsum(0)
    return off.cuda()


def looked_at(rows, width):
    """The first rows, those around value 2^31 of a matrix of this width, the last ones."""
    mid = LINE // width
    return torch.tensor(sorted({0, 1, *range(mid - 3, mid + 3), *range(rows - 3, rows)} & set(range(rows)))).cuda()


@pytest.mark.parametrize("transpose_w", [False, True])
def test_long_rows_in_and_out(transpose_w):
    rows, wide, N = [900_000, 0, 200_001], 2048, 72
    n, off = sum(rows), offsets_of(rows)
    pick = looked_at(n, wide)
    expert = (pick >= rows[0]).long() * 2
    for K, M in ((wide, N), (N, wide)):  # rows that pass the line are read, then written
        x, w = whole((n, K), 1), whole((3, M, K) if transpose_w else (3, K, M), 2)
        y = moe.moe_grouped_gemm(x, w, off, transpose_w=transpose_w)
        m = (w.transpose(1, 2) if transpose_w else w).double()[expert].contiguous()
        assert torch.equal(y[pick], (x[pick].double()[:, :, None] * m).sum(1).to(BF16))
        del x, y


def test_gradient_of_weights_from_long_rows():
    rows, K, N = [900_000, 0, 200_001], 2048, 72
    x, dy = whole((sum(rows), K), 3), whole((sum(rows), N), 4)
    for a, b, M, L in ((x, dy, K, N), (dy, x, N, K)):
        got = moe.moe_grouped_gemm_wgrad(a, b, offsets_of(rows))
        at = 0
        for e, n in enumerate(rows):
            ref = torch.zeros(M, L, dtype=torch.float64, device="cuda")
            for lo in range(at, at + n, 1 << 17):
                hi = min(lo + (1 << 17), at + n)
                ref += torch.mm(a[lo:hi].double().t().contiguous(), b[lo:hi].double())
            at += n
            assert torch.equal(got[e], ref.to(F32)), e


def test_large_weights_and_their_gradients():
    E, K, N = 48, 4096, 14336
    rows = [0] * E
    rows[3], rows[40], rows[E - 1] = 5, 2, 37
    off = offsets_of(rows)
    x, dy, w = whole((44, K), 5), whole((44, N), 6), whole((E, K, N), 7)
    y, dx, dw = moe.moe_grouped_gemm(x, w, off), moe.moe_grouped_gemm(dy, w, off, transpose_w=True), moe.moe_grouped_gemm_wgrad(x, dy, off)
    for e, a, b in ((3, 0, 5), (40, 5, 7), (E - 1, 7, 44)):
        assert torch.equal(y[a:b], torch.mm(x[a:b].double(), w[e].double()).to(BF16))
        assert torch.equal(dx[a:b], torch.mm(dy[a:b].double(), w[e].double().t().contiguous()).to(BF16))
        assert torch.equal(dw[e], torch.mm(x[a:b].double().t().contiguous(), dy[a:b].double()).to(F32))
    assert not dw[:3].any() and not dw[4:40].any() and not dw[41:E - 1].any()


def test_swiglu_and_its_gradient_of_long_rows():
    rows, f = 300_000, 4096
    gu, dh = normal((rows, 2 * f), 8, 2.0), normal((rows, f), 9)
    h, dgu = moe.moe_swiglu(gu), moe.moe_swiglu_backward(dh, gu)
    pick = torch.cat([looked_at(rows, 2 * f), looked_at(rows, f)[-3:]])
    g, u, d = gu[pick, :f].double(), gu[pick, f:].double(), dh[pick].double()
    s, small = torch.sigmoid(g), 2.0 ** -19
    assert ((h[pick].double() - g * s * u).abs() <= (2.0 ** -8 * 1.01 + small) * (g * s * u).abs() + 1e-37).all()
    dg, du = d * u * s * (1 + g * (1 - s)), d * g * s
    assert ((dgu[pick, :f].double() - dg).abs() <= 2.0 ** -8 * 1.01 * dg.abs() + small * (d * u).abs() * s * (1 + g.abs() * (1 - s)) + 1e-37).all()
    assert ((dgu[pick, f:].double() - du).abs() <= (2.0 ** -8 * 1.01 + small) * du.abs() + 1e-37).all()


def test_a_long_gradient():
    n = LINE + 70_005
    flat, other = normal((n + 1,), 10, 1e-2), normal((1001,), 11, 1e-2)
    g = flat[1:]
    total = sum(float(c.double().square().sum()) for c in (*g.split(1 << 28), other))
    norm = math.sqrt(total)
    out = [torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros_like(other)]  # (of another 16-byte phase)
    assert abs(float(moe.moe_clip_grad_norm([g, other], 0.5 * norm, out=out)) - norm) <= 2.0 ** -23 * norm
    scale = 0.5 * norm / (norm + 1e-6)
    for at in (0, 1 << 30, LINE - 5000, LINE - 8, n - 70_000):
        a, b = g[at:at + 70_000].double(), out[0][at:at + 70_000].double()
        assert ((b - a * scale).abs() <= 2.0 ** -8 * 1.01 * a.abs() * scale).all()
    moe.moe_clip_grad_norm([g, other], 0.5 * norm)
    assert torch.equal(g, out[0]) and torch.equal(other, out[1])


def test_long_rows_in_4_bits():
    rows, K, N = 600_000, 4096, 40
    off = offsets_of([550_000, 50_000])
    x, w = normal((rows, K), 12), normal((2, K, N), 13, 0.02)
    q, s = moe.moe_mxfp4_quantize(x)
    pick = looked_at(rows, K)
    code, byte = ref_quantize(x[pick].cpu().double().numpy())
    assert (unpack(q[pick]) == code).all() and (s[pick].cpu().numpy()[:, :K // 32] == byte).all()
    back = moe.moe_mxfp4_dequantize(q, s)
    assert torch.equal(back[pick], moe.moe_mxfp4_dequantize(q[pick], s[pick]))
    wq = moe.moe_mxfp4_quantize_weights(w)
    y = moe.moe_mxfp4_grouped_gemm(q, s, *wq, off)
    p, m = back[pick].double(), moe.moe_mxfp4_dequantize(*wq).double()[(pick >= 550_000).long()]
    ref, size = (m * p[:, None]).sum(2), (m * p[:, None]).abs().sum(2)
    assert ((y[pick].double() - ref).abs() <= 2.0 ** -8 * 1.01 * ref.abs() + K * 2.0 ** -23 * size).all()


def test_large_weights_in_4_bits():
    E, K, N = 80, 14336, 8192  # 2^32 bytes of codes and more
    w = torch.empty(E, K, N, dtype=BF16, device="cuda")
    for e in range(E):
        w[e] = normal((K, N), 100 + e, 0.02)
    rows = [0] * E
    rows[0], rows[E - 1] = 3, 30
    x = normal((33, K), 14)
    wq, ws = moe.moe_mxfp4_quantize_weights(w)
    cols = torch.tensor([0, 127, 128, N - 1])
    code, byte = ref_quantize(w[E - 1][:, cols.cuda()].t().cpu().double().numpy())
    assert (unpack(wq[E - 1][cols.cuda()]) == code).all() and (ws[E - 1][cols.cuda()].cpu().numpy() == byte).all()
    xq, xs = moe.moe_mxfp4_quantize(x)
    y = moe.moe_mxfp4_grouped_gemm(xq, xs, wq, ws, offsets_of(rows))
    for e, a, b in ((0, 0, 3), (E - 1, 3, 33)):
        p, m = moe.moe_mxfp4_dequantize(xq[a:b], xs[a:b]).double(), moe.moe_mxfp4_dequantize(wq[e], ws[e]).double().t().contiguous()
        ref, size = torch.mm(p, m), torch.mm(p.abs(), m.abs())
        assert ((y[a:b].double() - ref).abs() <= 2.0 ** -8 * 1.01 * ref.abs() + K * 2.0 ** -23 * size).all()
    del w
    whole_back = moe.moe_mxfp4_dequantize(wq, ws)
    assert torch.equal(whole_back[E - 1], moe.moe_mxfp4_dequantize(wq[E - 1], ws[E - 1]))
