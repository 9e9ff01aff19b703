"""Three operators around one block's training step, as cases that can be timed and compared: plain forms in elementary torch
operations, and the calls of `paper_2605_19945_amd` that do the same.

A case is one call path on one size:

* op "norm": the norm of the residual stream that a block begins with, h = x / sqrt(mean(x^2) + eps) * w, a row at a time --
             dir "fwd", or "bwd": the gradients of x and w from that of h, the residual's own gradient added to x's;
* op "join": what a block ends with, out = scale * x + gate * n with n the norm of the block's output y times a weight
             (norm "rms") or y times a weight for each channel (norm "none"); gate a number for each row ("row"), for each
             value ("full") or absent ("none"); with the norm that the next block begins with in the same pass (next) --
             dir "fwd" (out and that norm) or "bwd" (the gradients of x, y, gate and both weights from those of out and of
             that norm);
* op "orth": a stack of matrices, each brought near the orthogonal matrix next to it by Newton-Schulz steps, as optimisers do
             with the update of a weight: X = G / (|G| + 1e-7), five times X = a X + (b S + c S S) X with S = X X^T (of a
             tall matrix: the same on its transpose), times a scale.

Widths are those of `workloads/gen.py` and the benchmark: the tiny layer (128, 256, 8 experts), the Mixtral shape
(4096, 14336, 8 experts), 128 fine-grained experts (2048, 768), one GPU's 32 experts of an expert-parallel layer
(7168, 2048).  Drawn cases add free sizes of the same ranges.  Streams are Gaussians whose rows differ in scale and whose few
strong channels stand out; gradients of weights are the sum of a few strong directions and Gaussian noise.
"""
import math

import torch

own = False

EPS = 1e-6
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
TINY = 1e-7
MAX_ROW_VALUES = 65536 * 4096     # values of the largest listed stream
MAX_MATRIX_VALUES = 8 * 4096 * 14336
W_STD = 0.1


def listed():
    return [
        # one user's decode step, the norm in front of the router: launch and host time only
        _norm("norm_decode_T1", "fwd", rows=1, d=4096),
        # a prefill batch of the widest model, odd number of tokens
        _norm("norm_ep_T8191", "fwd", rows=8191, d=7168),
        # training, a 32-bit residual stream under bf16 blocks: the norm's gradient added to the stream's
        _norm("norm_bwd_fine_T8192", "bwd", rows=8192, d=2048, stream="fp32"),
        # one token of the widest model behind its experts: norm, row gate, residual, and the next block's norm
        _join("join_decode_T1", "fwd", rows=1, d=7168, norm="rms", gate="row", next=True),
        # a decode batch without a norm behind the block, channels scaled
        _join("join_mixtral_T64", "fwd", rows=64, d=4096, norm="none", gate="none", next=True, scale=0.7),
        # a long prefill, everything at once
        _join("join_mixtral_T65536", "fwd", rows=65536, d=4096, norm="rms", gate="row", next=True),
        # a fine-tuning step on a short prompt, odd number of tokens
        _join("join_bwd_fine_T77", "bwd", rows=77, d=2048, norm="rms", gate="row", next=True),
        # the gradients of a training batch's block, a gate for every value
        _join("join_bwd_mixtral_T8192", "bwd", rows=8192, d=4096, norm="rms", gate="full", next=True, scale=0.7),
        # the update of a toy layer's experts: launches count
        _orth("orth_tiny", E=8, rows=128, cols=256, type="fp32"),
        # 128 fine-grained experts' down projection, gradients in bf16
        _orth("orth_fine", E=128, rows=768, cols=2048, type="bf16"),
        # tall matrices kept in 32 bits, one GPU's share of an expert-parallel layer's up projection
        _orth("orth_ep", E=32, rows=7168, cols=2048, type="fp32"),
        # one projection of the Mixtral shape, a view into the gradient of gate and up projection side by side
        _orth("orth_mixtral", E=8, rows=4096, cols=14336, type="bf16", pad=14336),
    ]


def _norm(name, dir, rows, d, stream="bf16", block="bf16", weight="fp32", pad=0):
    """stream: type of the residual stream, block: of what goes into the block and comes out of it, weight: of the weights;
    pad: values between the end of a row of the stream and the next one (a view into wider rows)."""
    return _named(name, dict(op="norm", dir=dir, rows=rows, d=d, stream=stream, block=block, weight=weight, pad=pad))


def _join(name, dir, rows, d, norm, gate, next, scale=1.0, stream="bf16", block="bf16", weight="fp32", pad=0):
    return _named(name, dict(op="join", dir=dir, rows=rows, d=d, norm=norm, gate=gate, next=next, scale=scale, stream=stream,
                             block=block, weight=weight, pad=pad))


def _orth(name, E, rows, cols, type, pad=0):
    return _named(name, dict(op="orth", E=E, rows=rows, cols=cols, type=type, pad=pad))


def _named(name, c):
    return dict(c, name=name) if name else c


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "join", "join", "orth", "orth"])
    if op == "orth":
        E = rng.choice([1, 1, 2, 4, 8, 16, 32, 60, 128])
        rows, cols = (_log_uniform(rng, 8, 14336) for _ in range(2))
        if rng.random() < 0.5:  # widths of models, rather than any
            rows, cols = (-(-n // 64) * 64 for n in (rows, cols))
        top = work(listed()[-1])["flops"]
        while E * rows * cols > MAX_MATRIX_VALUES or _orth_flops(E, rows, cols) > top:
            if E > 1:
                E //= 2
            else:
                rows, cols = max(8, rows // 2), max(8, cols // 2)
        return _orth("", E, rows, cols, rng.choice(["bf16", "fp32"]), rng.choice([0, 0, 8, cols]))
    d = 8 * _log_uniform(rng, 8, 2048)
    stream, block = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
    kind = dict(rows=_log_uniform(rng, 1, min(65536, MAX_ROW_VALUES // (2 * d if stream == "fp32" else d))), d=d, stream=stream,
                block=block, weight=rng.choice(["fp32", "bf16"]), pad=rng.choice([0, 0, 8, 64]), dir=rng.choice(["fwd", "bwd"]))
    if kind["dir"] == "bwd":
        kind["rows"] = min(kind["rows"], max(1, MAX_ROW_VALUES // (4 * d)))
    if op == "norm":
        return _norm("", **kind)
    return _join("", norm=rng.choice(["rms", "rms", "none"]), gate=rng.choice(["none", "row", "full"]), next=rng.random() < 0.7,
                 scale=rng.choice([1.0, 1.0, 0.7]), **kind)


# ---- inputs -------------------------------------------------------------------------------------------
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _normals(seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 29)

    def normal(*shape, dtype=torch.float32, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    return normal


def _stream(normal, rows, d, dtype, pad=0):
    """Rows of a residual stream: their scales differ by a factor of a few, some channels are ten times as strong."""
    x = normal(rows, d + pad, dtype=dtype)
    x *= torch.exp(0.5 * normal(rows, 1))
    x[:, 5::97] *= 10.0
    return x[:, :d]


def prepare(case, seed):
    c = case
    normal = _normals(seed)
    if c["op"] == "orth":
        E, rows, cols = c["E"], c["rows"], c["cols"]
        wide = torch.empty(E, rows, cols + c["pad"], dtype=TYPES[c["type"]], device="cuda")
        for e in range(E):  # a few directions carry most of the norm, scales differ from matrix to matrix
            top = normal(rows, 4) @ normal(4, cols + c["pad"])
            wide[e] = (top + 0.5 * normal(rows, cols + c["pad"])) * (1e-3 * (1 + e % 5))
        return dict(op="orth", g=wide[:, :, :cols], scale=max(1.0, rows / cols) ** 0.5)
    rows, d, S, B = c["rows"], c["d"], TYPES[c["stream"]], TYPES[c["block"]]

    def weight():
        return (1.0 + normal(d, std=W_STD)).to(TYPES[c["weight"]])

    s = dict(op=c["op"], dir=c["dir"], x=_stream(normal, rows, d, S, c["pad"]), block=B)
    if c["op"] == "norm":
        s["w"] = weight()
        if c["dir"] == "bwd":
            s.update(dh=normal(rows, d, dtype=B, std=0.1), dres=normal(rows, d, dtype=S, std=0.1))
        return s
    s.update(y=_stream(normal, rows, d, B), w=weight(), w_next=weight() if c["next"] else None, rms=c["norm"] == "rms",
             scale=c["scale"], gate=None)
    if c["gate"] == "row":
        s["gate"] = torch.sigmoid(normal(rows))
    elif c["gate"] == "full":
        s["gate"] = torch.sigmoid(normal(rows, d)).to(B)
    if c["dir"] == "bwd":  # x is then what the block left in its stream
        s.update(dout=normal(rows, d, dtype=S, std=0.1), dh=normal(rows, d, dtype=B, std=0.1) if c["next"] else None)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------
def _factor(x):
    """1 / sqrt(mean(x^2) + eps) of every row."""
    return torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)


def _norm_gradients(dh, x, w):
    """(gradient of x, of w) of x * factor * w; w None: ones."""
    r = _factor(x)
    p = dh if w is None else dh * w
    dx = r * (p - x * (r * r * (p * x).mean(1, keepdim=True)))
    return dx, (dh * x * r).sum(0)


def _plain_norm(s):
    x, w = s["x"].float(), s["w"].float()
    if s["dir"] == "fwd":
        return (x * _factor(x) * w).to(s["block"])
    dx, dw = _norm_gradients(s["dh"].float(), x, w)
    return (dx + s["dres"].float()).to(s["x"].dtype), dw


def _plain_join(s):
    y, w = s["y"].float(), s["w"].float()
    gate = 1.0 if s["gate"] is None else s["gate"].float() if s["gate"].dim() == 2 else s["gate"][:, None]
    if s["dir"] == "fwd":
        n = (y * _factor(y) if s["rms"] else y) * w
        out = s["scale"] * s["x"].float() + gate * n
        if s["w_next"] is None:
            return out.to(s["x"].dtype)
        return out.to(s["x"].dtype), (out * _factor(out) * s["w_next"].float()).to(s["block"])
    D, grads = s["dout"].float(), []
    if s["w_next"] is not None:
        dx, dw = _norm_gradients(s["dh"].float(), s["x"].float(), s["w_next"].float())
        D, grads = D + dx, [dw]
    dn = gate * D
    if s["rms"]:
        dy, dw = _norm_gradients(dn, y, w)
    else:
        dy, dw = dn * w, (dn * y).sum(0)
    grads = [(s["scale"] * D).to(s["x"].dtype), dy.to(s["block"]), dw] + grads
    if s["gate"] is not None:
        n = (y * _factor(y) if s["rms"] else y) * w
        dgate = D * n
        grads.append(dgate.sum(1) if s["gate"].dim() == 1 else dgate.to(s["block"]))
    return grads


def _plain_orth(s):
    g = s["g"]
    tall = g.shape[1] > g.shape[2]
    out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
    a, b, c = COEFFICIENTS
    for e in range(g.shape[0]):
        X = g[e].t().float().contiguous() if tall else g[e].float()
        X = X / (X.square().sum().sqrt() + TINY)
        for _ in range(STEPS):
            S = torch.mm(X, X.t())
            X = a * X + torch.mm(b * S + c * torch.mm(S, S), X)
        out[e] = s["scale"] * (X.t() if tall else X)
    return out


# ---- one pass -------------------------------------------------------------------------------------------
def run(s):
    if not own:
        return {"norm": _plain_norm, "join": _plain_join, "orth": _plain_orth}[s["op"]](s)
    import paper_2605_19945_amd as moe
    if s["op"] == "orth":
        return moe.moe_orthogonalize(s["g"], scale=s["scale"])
    if s["op"] == "norm":
        if s["dir"] == "fwd":
            return moe.moe_rms_norm(s["x"], s["w"], eps=EPS, dtype=s["block"])
        return moe.moe_rms_norm_backward(s["dh"], s["x"], s["w"], eps=EPS, dres=s["dres"])
    how = dict(norm=s["rms"], gate=s["gate"], scale=s["scale"], next_weight=s["w_next"], eps=EPS)
    if s["dir"] == "fwd":
        out, h = moe.moe_residual_norm(s["x"], s["y"], s["w"], **how)
        return out if h is None else (out, h)
    dx, dy, dw, dnext, dgate = moe.moe_residual_norm_backward(s["dout"], s["y"], s["w"], out=s["x"], dh=s["dh"], **how)
    return [t for t in (dx, dy, dw, dnext, dgate) if t is not None]


# ---- what a pass cannot do without ----------------------------------------------------------------------
def _orth_flops(E, rows, cols):
    n, m = float(min(rows, cols)), float(max(rows, cols))
    return E * STEPS * (n * n * m + n * n * n + 2 * n * n * m)  # the two symmetric products: one half of them


def work(case):
    c = case
    if c["op"] == "orth":
        values = float(c["E"]) * c["rows"] * c["cols"]
        return {"bytes": 2 * values * (4 if c["type"] == "fp32" else 2), "flops": _orth_flops(c["E"], c["rows"], c["cols"])}
    n, S, B = float(c["rows"]) * c["d"], 4 if c["stream"] == "fp32" else 2, 4 if c["block"] == "fp32" else 2
    small = c["d"] * 4.0
    if c["op"] == "norm":  # x in and h out; dh, x and the residual's gradient in and dx out
        return {"bytes": n * (S + B) + small, "flops": 4 * n} if c["dir"] == "fwd" else \
            {"bytes": n * (B + 3 * S) + 2 * small, "flops": 10 * n}
    gate = {"none": 0.0, "row": 4.0 * c["rows"], "full": n * B}[c["gate"]]
    if c["dir"] == "fwd":  # x, y and gate in, out and the next block's rows out
        return {"bytes": n * (2 * S + B + (B if c["next"] else 0)) + gate + 2 * small, "flops": 10 * n}
    # gradients of out and of the next rows, out, y and gate in; gradients of x, y and gate out
    return {"bytes": n * (S + (B + S if c["next"] else 0) + B + S + B) + 2 * gate + 4 * small, "flops": 25 * n}


# ---- the same results in 64 bits ------------------------------------------------------------------------
def _by_root(v, w):
    """v divided by the root of its rows' mean square (and eps), times w."""
    return v / (torch.linalg.vector_norm(v, dim=1, keepdim=True) ** 2 / v.shape[1] + EPS) ** 0.5 * w


def _exact_orth(case, s):
    a, b, c = COEFFICIENTS
    n, m = sorted((case["rows"], case["cols"]))
    if case["E"] * STEPS * (4.0 * n * n * m + 2.0 * n ** 3) > 5e14:
        return None
    out = torch.empty(s["g"].shape, dtype=torch.float64, device="cuda")
    eye = torch.eye(n, dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        M = s["g"][e].double()
        M = M / (torch.linalg.vector_norm(M) + TINY)
        wide = case["rows"] <= case["cols"]
        for _ in range(STEPS):
            A = M @ M.t() if wide else M.t() @ M
            poly = a * eye + (b * eye + c * A) @ A
            M = poly @ M if wide else M @ poly
        out[e] = M * s["scale"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orth":
        return _exact_orth(case, s)

    def leaf(t):
        return t.double().requires_grad_() if t is not None else None

    with torch.enable_grad():
        if case["op"] == "norm":
            x, w = leaf(s["x"]), leaf(s["w"])
            h = _by_root(x, w)
            if case["dir"] == "fwd":
                return h.detach()
            h.backward(s["dh"].double())
            return x.grad + s["dres"].double(), w.grad
        y, w, gate, w_next = leaf(s["y"]), leaf(s["w"]), leaf(s["gate"]), leaf(s["w_next"])
        branch = _by_root(y, w) if s["rms"] else y * w
        if gate is not None:
            branch = branch * (gate.unsqueeze(1) if gate.dim() == 1 else gate)
        if case["dir"] == "fwd":
            out = (s["x"].double() * s["scale"] + branch).detach()
            return out if w_next is None else (out, _by_root(out, w_next).detach())
        total, o = s["dout"].double(), leaf(s["x"])
        if w_next is not None:
            _by_root(o, w_next).backward(s["dh"].double())
            total = total + o.grad
        branch.backward(total)
        grads = [total * s["scale"], y.grad, w.grad, w_next.grad if w_next is not None else None, gate.grad if gate is not None else None]
        return [t for t in grads if t is not None]
