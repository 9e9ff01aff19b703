"""The norms around a block and their gradients against plain computations in 64 bits (torch float64 on the CPU, gradients by torch's own
differentiation).

Bounds.  With u = 2^-24: a row's sum is a chain of at most 32 additions a lane, 6 over the lanes and 8 over the wavefronts, each off by u
of the magnitudes, so a sum is off by less than 2^-18 of the sum of its terms' magnitudes; a factor 1 / sqrt(mean) by half of that and
2^-22; the few products behind it by u each.  A value that is a sum of terms is therefore off by at most 2^-17 of the sum of its terms'
magnitudes, one that takes such a value into a second row sum by 2^-16, a sum over R rows by R u more; and a result that is rounded to a type by
eps / 2 of itself.  The magnitudes are formed by the same formulas on absolute values."""
import pytest
import torch

import paper_2605_19945_amd as moe

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
ONCE, TWICE, U = 2.0 ** -17, 2.0 ** -16, 2.0 ** -24
EPS = 1e-5


def normal(shape, seed, std=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def close(got, ref, mag, rel):
    """|got - ref| <= eps / 2 |ref| + rel mag, value by value (rounding of a value that is itself off: eps / 2 of both)."""
    got, half = got.cpu().double(), torch.finfo(got.dtype).eps / 2
    bound = half * (ref.abs() + rel * mag) + rel * mag
    worst = float(((got - ref).abs() - bound).max()) if ref.numel() else 0.0
    assert got.shape == ref.shape and worst <= 0.0, (worst, float((got - ref).abs().max()))


def factor(x):
    return (x.square().mean(1, keepdim=True) + EPS).rsqrt()


def case(rows, d, S, B, W=F32, gate="row", norm=True, nxt=True, seed=0):
    c = dict(x=normal((rows, d), seed, dtype=S) * 3, y=normal((rows, d), seed + 1, dtype=B) * torch.logspace(-2, 1, rows)[:, None].to(B),
             w=(1 + normal((d,), seed + 2, 0.2)).to(W), gate=None, next=(1 + normal((d,), seed + 3, 0.2)).to(W) if nxt else None,
             dout=normal((rows, d), seed + 4, dtype=S), dh=normal((rows, d), seed + 5, dtype=B) if nxt else None, norm=norm)
    if gate == "row":
        c["gate"] = normal((rows,), seed + 6)
    elif gate == "full":
        c["gate"] = normal((rows, d), seed + 6, dtype=B)
    return c


def dev(t):
    return None if t is None else t.cuda()


def d64(t):
    return None if t is None else t.double()


def ref_forward(c, scale):
    x, y, w, nxt = map(d64, (c["x"], c["y"], c["w"], c["next"]))
    g = torch.ones(1, 1, dtype=F64) if c["gate"] is None else d64(c["gate"]) if c["gate"].dim() == 2 else d64(c["gate"])[:, None]
    n = (y * factor(y) if c["norm"] else y) * w
    out, mag = scale * x + g * n, abs(scale) * x.abs() + (g * n).abs()
    if nxt is None:
        return out, mag, None, None
    r = factor(out)
    # (the row's factor sees values that are off by 2^-17 of mag: a share of at most the same of the root of mag's squares)
    return out, mag, out * r * nxt, (mag + out.abs() * (mag.square().mean(1, keepdim=True) + EPS).sqrt() * r) * r * nxt.abs()


def ref_backward(c, scale):
    """(reference, magnitude) of the gradients of x, y, w, next, gate; c["x"] is the stream that the next norm took."""
    o, y, w, nxt, dout, dh = map(d64, (c["x"], c["y"], c["w"], c["next"], c["dout"], c["dh"]))
    g = None if c["gate"] is None else d64(c["gate"])
    leaves = [t.requires_grad_() if t is not None else None for t in (o, y, w, nxt, g)]
    with torch.enable_grad():
        D = dout
        if nxt is not None:
            (o * factor(o) * nxt).backward(dh)
            D = dout + o.grad
        n = (y * factor(y) if c["norm"] else y) * w
        (n if g is None else (g[:, None] if g.dim() == 1 else g) * n).backward(D)
    o, y, w, nxt, g = (t.detach() if t is not None else None for t in leaves)
    gy, gw, gn, gg = (t.grad if t is not None else None for t in leaves[1:])
    M, ro = dout.abs(), factor(o)
    if nxt is not None:
        p = (dh * nxt).abs()
        M = M + ro * (p + o.abs() * ro ** 2 * (p * o.abs()).mean(1, keepdim=True))
    ry = factor(y) if c["norm"] else torch.ones(len(y), 1, dtype=F64)
    ga = 1.0 if g is None else g.abs() if g.dim() == 2 else g.abs()[:, None]
    q, yr = ga * M * w.abs(), y.abs() * ry
    my = ry * (q + (yr * (q * yr).mean(1, keepdim=True) if c["norm"] else 0))
    mg = M * yr * w.abs()
    out = [(scale * D, abs(scale) * M), (gy, my), (gw, (ga * M * yr).sum(0))]
    out.append((gn, (dh * o * ro).abs().sum(0)) if nxt is not None else (None, None))
    return out + [(gg, (mg.sum(1) if g.dim() == 1 else mg)) if g is not None else (None, None)]


def run_backward(c, scale, **kw):
    return moe.moe_residual_norm_backward(dev(c["dout"]), dev(c["y"]), dev(c["w"]), out=dev(c["x"]), dh=dev(c["dh"]), norm=c["norm"], gate=dev(c["gate"]),
                                          scale=scale, next_weight=dev(c["next"]), eps=EPS, **kw)


def check_backward(got, c, scale):
    rows = c["y"].shape[0]
    for i, (t, (ref, mag)) in enumerate(zip(got, ref_backward(c, scale))):
        assert (t is None) == (ref is None), i
        if t is not None:
            close(t, ref, mag, TWICE + (rows * U if i in (2, 3) else 0))


TYPES = [(BF16, BF16), (F32, BF16), (F32, F32)]
SIZES = [(1, 8), (3, 64), (9, 512), (17, 520), (8, 1024), (7, 1032), (5, 2048), (77, 2056), (1, 4096), (4, 4104), (2, 8192), (3, 8200), (2, 16384)]


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("S,B", TYPES)
def test_norm(rows, d, S, B):
    for W in (F32, BF16, None):
        c = case(rows, d, S, B, W or F32, nxt=True, seed=rows + d)
        x, dh, w = c["x"], c["dh"], c["w"] if W else None
        got = moe.moe_rms_norm(dev(x), dev(w), eps=EPS, dtype=B)
        x64, w64 = x.double().requires_grad_(), (w.double() if W else torch.ones(d, dtype=F64)).requires_grad_()
        ref = x64 * factor(x64) * w64
        assert got.dtype is B
        close(got, ref.detach(), ref.detach().abs(), ONCE)
        ref.backward(dh.double())
        for dres in (None, c["dout"]):
            dx, dw = moe.moe_rms_norm_backward(dev(dh), dev(x), dev(w), eps=EPS, dres=dev(dres))
            xa, r, p = x.double(), factor(x.double()), (dh.double() * w64.detach()).abs()
            mag = r * (p + xa.abs() * r ** 2 * (p * xa.abs()).mean(1, keepdim=True)) + (0 if dres is None else dres.double().abs())
            assert dx.dtype is S
            close(dx, x64.grad + (0 if dres is None else dres.double()), mag, ONCE)
            assert (dw is None) == (W is None)
            if W:
                close(dw, w64.grad, (dh.double() * xa * r).abs().sum(0), ONCE + rows * U)


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("S,B", TYPES)
@pytest.mark.parametrize("gate", ["none", "row", "full"])
def test_join(rows, d, S, B, gate):
    for norm, nxt, scale, W in ((True, True, 0.7, F32), (False, True, 1.0, BF16), (True, False, 1.0, BF16), (False, False, -2.0, F32)):
        c = case(rows, d, S, B, W, gate, norm, nxt, seed=3 * rows + d)
        out, h = moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), dev(c["w"]), norm=norm, gate=dev(c["gate"]), scale=scale, next_weight=dev(c["next"]), eps=EPS)
        ro, mo, rh, mh = ref_forward(c, scale)
        assert out.dtype is S and (h is None) == (not nxt)
        close(out, ro, mo, ONCE)
        if nxt:
            assert h.dtype is B
            close(h, rh, mh, TWICE)
        check_backward(run_backward(c, scale), c, scale)


@pytest.mark.parametrize("rows,d", [(20000, 64), (17001, 512), (9001, 1000), (4099, 2048), (2500, 4096), (1100, 8192), (1030, 16384)])
def test_more_rows_than_one_launch_holds_at_once(rows, d):
    c = case(rows, d, BF16, BF16, seed=1)
    out, h = moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), dev(c["w"]), gate=dev(c["gate"]), next_weight=dev(c["next"]), eps=EPS)
    ro, mo, rh, mh = ref_forward(c, 1.0)
    close(out, ro, mo, ONCE)
    close(h, rh, mh, TWICE)
    got = run_backward(c, 1.0)
    check_backward(got, c, 1.0)
    again = run_backward(c, 1.0)      # fixed orders: the same bits
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_weights_absent_and_gradients_alone():
    c = case(6, 200, BF16, BF16, gate="none")
    ones = torch.ones(200)
    a = moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), None, next_weight=dev(c["next"]), eps=EPS)
    b = moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), ones.cuda(), next_weight=dev(c["next"]), eps=EPS)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    c["w"] = ones
    full = run_backward(c, 1.0)
    got = moe.moe_residual_norm_backward(dev(c["dout"]), dev(c["y"]), None, out=dev(c["x"]), dh=dev(c["dh"]), next_weight=dev(c["next"]), eps=EPS)
    assert got[2] is None and torch.equal(got[0], full[0]) and torch.equal(got[1], full[1]) and torch.equal(got[3], full[3])
    c["dout"] = torch.zeros_like(c["dout"])
    zero = run_backward(c, 1.0)
    got = moe.moe_residual_norm_backward(None, dev(c["y"]), ones.cuda(), out=dev(c["x"]), dh=dev(c["dh"]), next_weight=dev(c["next"]), eps=EPS)
    assert all(torch.equal(s, t) for s, t in zip(got[:4], zero[:4]))


@pytest.mark.parametrize("live", [0, 1, 5, 11, 40, -3])
@pytest.mark.parametrize("d", [64, 2048, 5000])
def test_rows_behind_the_last_one_stay_as_they_are(live, d):
    rows, n = 11, min(max(live, 0), 11)
    c = case(rows, d, F32, BF16, gate="full")
    off = torch.tensor([0, 3, live], dtype=torch.int32).cuda()
    mark = 7.0
    out, h, dx, dy = (torch.full((rows, d), mark, dtype=t, device="cuda") for t in (F32, BF16, F32, BF16))
    kw = dict(gate=dev(c["gate"]), next_weight=dev(c["next"]), eps=EPS)
    moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), dev(c["w"]), offsets=off, out=out, h=h, **kw)
    got = moe.moe_residual_norm_backward(dev(c["dout"]), dev(c["y"]), dev(c["w"]), out=dev(c["x"]), dh=dev(c["dh"]), offsets=off, dx=dx, dy=dy, **kw)
    part = {k: (v[:n] if isinstance(v, torch.Tensor) and v.dim() == 2 else v) for k, v in c.items()}
    for t in (out, h, dx, dy):
        assert (t[n:] == mark).all()
    if n:
        ro, mo, rh, mh = ref_forward(part, 1.0)
        close(out[:n], ro, mo, ONCE)
        close(h[:n], rh, mh, TWICE)
        check_backward([dx[:n], dy[:n], got[2], got[3], got[4][:n]], part, 1.0)
    else:
        assert not got[2].any() and not got[3].any()
    hh = torch.full((rows, d), mark, dtype=BF16, device="cuda")
    moe.moe_rms_norm(dev(c["x"]), dev(c["w"]), eps=EPS, offsets=off, out=hh)
    g = torch.full((rows, d), mark, dtype=F32, device="cuda")
    _, dw = moe.moe_rms_norm_backward(dev(c["dh"]), dev(c["x"]), dev(c["w"]), eps=EPS, offsets=off, out=g)
    assert (hh[n:] == mark).all() and (g[n:] == mark).all()
    whole = moe.moe_rms_norm(dev(c["x"])[:n], dev(c["w"]), eps=EPS, dtype=BF16)
    _, dw_part = moe.moe_rms_norm_backward(dev(c["dh"])[:n], dev(c["x"])[:n], dev(c["w"]), eps=EPS)
    assert torch.equal(hh[:n], whole)
    ref = dw_part.double().cpu()
    close(dw, ref, (c["dh"][:n].double() * c["x"][:n].double() * factor(c["x"][:n].double())).abs().sum(0) if n else ref.abs(), 2 * rows * U)


def test_no_rows():
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    w = torch.ones(64, device="cuda")
    assert moe.moe_rms_norm(x, w).shape == (0, 64)
    dx, dw = moe.moe_rms_norm_backward(x, x, w)
    assert dx.shape == (0, 64) and not dw.any()
    out, h = moe.moe_residual_norm(x, x, w, next_weight=w)
    assert out.shape == h.shape == (0, 64)
    got = moe.moe_residual_norm_backward(x, x, w, out=x, dh=x, next_weight=w)
    assert not got[2].any() and not got[3].any()


@pytest.mark.parametrize("d", [72, 1536, 4096])
def test_views_into_wider_rows(d):
    rows = 13
    c = case(rows, d, BF16, BF16, gate="full")
    flat = {k: dev(v) for k, v in c.items() if isinstance(v, torch.Tensor)}

    def wide(t, pad):
        w = torch.full((rows, d + pad), 9.0, dtype=t.dtype, device="cuda")
        w[:, 8:8 + d] = t
        return w[:, 8:8 + d], w

    views = {k: wide(v, 16 + 8 * i)[0] for i, (k, v) in enumerate(flat.items()) if v.dim() == 2}
    kw = dict(next_weight=flat["next"], eps=EPS)
    a = moe.moe_residual_norm(flat["x"], flat["y"], flat["w"], gate=flat["gate"], **kw)
    (ov, ow), (hv, hw) = wide(torch.zeros_like(flat["x"]), 24), wide(torch.zeros_like(flat["x"]), 40)
    b = moe.moe_residual_norm(views["x"], views["y"], flat["w"], gate=views["gate"], out=ov, h=hv, **kw)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    for t in (ow, hw):
        assert (t[:, :8] == 9).all() and (t[:, 8 + d:] == 9).all()
    a = moe.moe_residual_norm_backward(flat["dout"], flat["y"], flat["w"], out=flat["x"], dh=flat["dh"], gate=flat["gate"], **kw)
    b = moe.moe_residual_norm_backward(views["dout"], views["y"], flat["w"], out=views["x"], dh=views["dh"], gate=views["gate"], dx=ov, dy=hv, **kw)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    for t in (ow, hw):
        assert (t[:, :8] == 9).all() and (t[:, 8 + d:] == 9).all()
    assert torch.equal(moe.moe_rms_norm(flat["x"], flat["w"]), moe.moe_rms_norm(views["x"], flat["w"], out=ov))
    a, b = (moe.moe_rms_norm_backward(t["dh"], t["x"], flat["w"], dres=t["dout"]) for t in (flat, views))
    assert all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("d", [64, 2048, 6000])
def test_results_in_the_place_of_inputs(d):
    c = case(9, d, BF16, BF16, gate="full")
    kw = dict(next_weight=dev(c["next"]), eps=EPS)

    def forward(o, h):
        t = {k: dev(c[k]) for k in ("x", "y", "gate")}
        return moe.moe_residual_norm(t["x"], t["y"], dev(c["w"]), gate=t["gate"], out=t.get(o), h=t.get(h), **kw)

    want = forward(None, None)
    for o, h in (("x", "y"), ("y", "x"), ("gate", "x"), ("x", "gate"), ("x", None)):
        assert all(torch.equal(a, b) for a, b in zip(want, forward(o, h))), (o, h)

    def backward(gx, gy):
        t = {k: dev(c[k]) for k in ("dout", "dh", "x", "y", "gate")}
        return moe.moe_residual_norm_backward(t["dout"], t["y"], dev(c["w"]), out=t["x"], dh=t["dh"], gate=t["gate"], dx=t.get(gx), dy=t.get(gy), **kw)

    want = backward(None, None)
    for gx, gy in (("dout", "dh"), ("x", "y"), ("y", "x"), ("dh", "dout"), ("gate", "y")):
        assert all(torch.equal(a, b) for a, b in zip(want, backward(gx, gy))), (gx, gy)
    x, dh, dres = dev(c["x"]), dev(c["dh"]), dev(c["dout"])
    want = moe.moe_rms_norm_backward(dh, x, dev(c["w"]), dres=dres)
    for place in range(3):
        t = [dh.clone(), x.clone(), dres.clone()]
        got = moe.moe_rms_norm_backward(t[0], t[1], dev(c["w"]), dres=t[2], out=t[place])
        assert got[0] is t[place] and all(torch.equal(a, b) for a, b in zip(want, got))
    want = moe.moe_rms_norm(x, dev(c["w"]))
    assert torch.equal(want, moe.moe_rms_norm(x, dev(c["w"]), out=x))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 1536, 4096])
def test_a_spoilt_row_spoils_no_other(bad, d):
    c = case(12, d, BF16, BF16)
    clean = moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), dev(c["w"]), gate=dev(c["gate"]), next_weight=dev(c["next"]), eps=EPS)
    grads = run_backward(c, 1.0)
    for name in ("x", "y", "dh"):
        s = dict(c)
        s[name] = c[name].clone()
        s[name][5, d // 2] = bad
        others = [i for i in range(12) if i != 5]
        got = moe.moe_residual_norm(dev(s["x"]), dev(s["y"]), dev(s["w"]), gate=dev(s["gate"]), next_weight=dev(s["next"]), eps=EPS)
        assert all(torch.equal(a[others], b[others]) for a, b in zip(clean, got))
        if name != "dh":
            assert not torch.isfinite(got[1][5].float()).all()
        got = run_backward(s, 1.0)
        assert all(torch.equal(got[i][others], grads[i][others]) for i in (0, 1, 4))


def test_rows_of_zeros_and_far_values():
    x = torch.zeros(3, 64, dtype=F32)
    x[1, 3], x[2] = 3e18, 1e-20
    w = torch.ones(64)
    got = moe.moe_rms_norm(x.cuda(), w.cuda(), eps=1e-6).cpu()
    assert not got[0].any() and abs(float(got[1, 3]) - 8.0) <= 8.0 * ONCE    # one value: root of 64
    close(got[2:], x[2:].double() * 1e3, x[2:].double() * 1e3, ONCE)
    assert torch.isnan(moe.moe_rms_norm(x.cuda(), w.cuda(), eps=0.0)[0]).all()  # 0 / 0


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("gate", ["none", "row", "full"])
def test_gradients_against_differences(norm, gate):
    """Central differences of the kernel's own forward pass along one direction for each input follow those of 64 bits at the same step t, of which
    each side's results are off by 2^-16 of their magnitudes; and the gradients are what those of 64 bits come to at a step 2^-10 t, but for the two
    thirds of their change at twice that step (what a central difference misses grows with the square of the step) and their own bound."""
    rows, d, scale, t = 4, 136, 0.7, 2.0 ** -5
    c = case(rows, d, F32, F32, F32, gate, norm, True, seed=11)
    co, ch = normal((rows, d), 50), normal((rows, d), 51)

    def exact(p):
        o, mo, h, mh = ref_forward(p, scale)
        return float((o * co.double()).sum() + (h * ch.double()).sum()), float((mo * co.abs()).sum() + (mh * ch.abs()).sum())

    def kernel(p):
        o, h = moe.moe_residual_norm(dev(p["x"]), dev(p["y"]), dev(p["w"]), norm=norm, gate=dev(p["gate"]), scale=scale, next_weight=dev(p["next"]), eps=EPS)
        return float((o.cpu().double() * co).sum() + (h.cpu().double() * ch).sum())

    out = moe.moe_residual_norm(dev(c["x"]), dev(c["y"]), dev(c["w"]), norm=norm, gate=dev(c["gate"]), scale=scale, eps=EPS)[0]
    there = dict(c, x=out.cpu(), dout=co, dh=ch)
    for i, (name, grad) in enumerate(zip(("x", "y", "w", "next", "gate"), run_backward(there, scale))):
        if grad is None:
            continue
        v = normal(c[name].shape, 60)

        def difference(f, step, dtype):
            plus, minus = (f(dict(c, **{name: c[name].to(dtype) + sign * step * v.to(dtype)})) for sign in (1, -1))
            return (plus - minus) / (2 * step)

        ideal, mag = difference(lambda p: exact(p)[0], t, F32), exact(c)[1]
        assert abs(difference(kernel, t, F32) - ideal) <= 2 * TWICE * mag / t, name
        s = t * 2.0 ** -10
        limit, twice = (difference(lambda p: exact(p)[0], k * s, F64) for k in (1, 2))
        own = float((ref_backward(there, scale)[i][1] * v.abs()).sum())
        assert abs(float((grad.cpu().double() * v).sum()) - limit) <= TWICE * own + abs(twice - limit) * 2 / 3, name


def test_on_a_side_stream_and_in_a_graph():
    c = case(33, 1536, BF16, BF16)
    t = {k: dev(v) for k, v in c.items() if isinstance(v, torch.Tensor)}

    def step():
        out, h = moe.moe_residual_norm(t["x"], t["y"], t["w"], gate=t["gate"], next_weight=t["next"], eps=EPS)
        return (out, h, moe.moe_rms_norm(out, t["w"]), *moe.moe_residual_norm_backward(t["dout"], t["y"], t["w"], out=out, dh=t["dh"], gate=t["gate"],
                                                                                     next_weight=t["next"], eps=EPS),
                *moe.moe_rms_norm_backward(t["dh"], t["x"], t["w"], dres=t["dout"]))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        t["x"].copy_(dev(c["x"]) * (1 + k))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), k
