"""The cases that the operators around a layer's products are measured with: microscaled 4-bit quantisation, the layer's products
on such operands (forward, both gradients, a few tokens), and the orthogonalised update of its weight.

`run` computes them in plain torch (`own` false: 32 bits, elementary operations) or through paper_2508_04355_amd.ops."""
import torch

own = False

DEV = "cuda"
BLOCK = 32                                   # values that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # magnitudes of the 4-bit type, by code
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS, MU = 5, 1e-7, 0.95
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -------------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the activation of one token before a projection: launch latency
        {"name": "quantise token", "op": "quantise", "rows": 1, "cols": 4096, "dtype": "bf16", "both": False},
        # a small fp32 matrix with a short last block in each direction
        {"name": "quantise ragged", "op": "quantise", "rows": 1000, "cols": 777, "dtype": "f32", "both": True},
        # the activations of a training batch, for the forward product and for the weight's gradient
        {"name": "quantise batch", "op": "quantise", "rows": 16384, "cols": 4096, "dtype": "bf16", "both": True},
        # one token through a layer whose weight is kept in 4 bits
        {"name": "linear token", "op": "linear", "n": 1, "k": 4096, "m": 14336, "dtype": "bf16"},
        # a small batch of tokens through the layer that follows
        {"name": "linear few", "op": "linear", "n": 24, "k": 14336, "m": 4096, "dtype": "bf16"},
        # a prompt or training batch
        {"name": "linear batch", "op": "linear", "n": 16384, "k": 4096, "m": 14336, "dtype": "bf16"},
        # forward, gradient of the input and of the weight, sizes that fill no tile
        {"name": "train ragged", "op": "train", "n": 1000, "k": 777, "m": 1100, "dtype": "f32"},
        # the three products of a training step of a large layer, with all that they quantise
        {"name": "train layer", "op": "train", "n": 16384, "k": 4096, "m": 14336, "dtype": "bf16"},
        # the update of one small weight: latency of a chain of products
        {"name": "orthogonalise small", "op": "orth", "rows": 128, "cols": 128, "batch": 1, "dtype": "f32", "momentum": True},
        # many small weights (experts, heads) at once
        {"name": "orthogonalise many", "op": "orth", "rows": 512, "cols": 512, "batch": 256, "dtype": "bf16", "momentum": False},
        # a tall weight of odd size
        {"name": "orthogonalise tall", "op": "orth", "rows": 3001, "cols": 801, "batch": 1, "dtype": "f32", "momentum": True},
        # the weight of the large layer, with its momentum
        {"name": "orthogonalise layer", "op": "orth", "rows": 4096, "cols": 14336, "batch": 1, "dtype": "bf16", "momentum": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["quantise", "linear", "linear", "train", "orth", "orth"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "quantise":
        rows = _log(rng, 1, 16384)
        return {"op": op, "rows": rows, "cols": _log(rng, 32, 16384 * 4096 // max(rows, 4096)), "dtype": dtype, "both": rng.random() < 0.5}
    if op in ("linear", "train"):
        # few tokens as often as many; products no larger than the listed ones
        k, m = _log(rng, 64, 14336), _log(rng, 64, 14336)
        n = _log(rng, 1, 16384)
        while n * k * m > 16384 * 4096 * 14336 or (op == "train" and dtype == "f32" and n * k * m > 1 << 38):
            k, m = max(64, k // 2), max(64, m // 2)
        if rng.random() < 0.5:      # as widths usually are; the others stay odd
            k, m = max(64, k // 64 * 64), max(64, m // 64 * 64)
        return {"op": op, "n": n, "k": k, "m": m, "dtype": dtype}
    rows, cols = _log(rng, 16, 4096), _log(rng, 16, 8192)
    if rng.random() < 0.5:
        rows, cols = cols, rows
    small, large = min(rows, cols), max(rows, cols)
    most = min(256, (1 << 26) // (rows * cols), max(1, (1 << 37) // (small * small * large)))
    batch = _log(rng, 1, max(1, most)) if rng.random() < 0.6 else 1
    return {"op": op, "rows": rows, "cols": cols, "batch": batch, "dtype": dtype, "momentum": rng.random() < 0.5}


# ---- inputs ----------------------------------------------------------------------------------------------------------------------

def _activations(g, n, k, dtype):
    """N(0, 1) with a few channels twenty times as large, as a transformer's hidden states have; the last rows are padding."""
    x = torch.randn(n, k, device=DEV, generator=g)
    x[:, torch.rand(k, device=DEV, generator=g) < 0.01] *= 20.0
    if n >= 64:
        x[n - n // 64:] = 0.0
    return x.to(DTYPES[dtype])


def _out_gradient(g, n, m, dtype):
    """Small values, tokens of different weight, no gradient from the padded tokens."""
    dy = torch.randn(n, m, device=DEV, generator=g) * (1e-3 * torch.exp(torch.randn(n, 1, device=DEV, generator=g)))
    if n >= 64:
        dy[n - n // 64:] = 0.0
    return dy.to(DTYPES[dtype])


def _weight_gradient(g, batch, rows, cols, dtype):
    """A few strong directions over a floor of noise."""
    r = min(64, rows, cols)
    s = torch.rand(batch, r, 1, device=DEV, generator=g)
    u = torch.randn(batch, rows, r, device=DEV, generator=g)
    w = torch.randn(batch, r, cols, device=DEV, generator=g) * s * (r ** -0.5)
    return (1e-3 * (torch.matmul(u, w) + 0.5 * torch.randn(batch, rows, cols, device=DEV, generator=g))).to(DTYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case)
    if case["op"] == "quantise":
        s["x"] = _activations(g, case["rows"], case["cols"], case["dtype"])
    elif case["op"] in ("linear", "train"):
        s["x"] = _activations(g, case["n"], case["k"], case["dtype"])
        w = 0.02 * torch.randn(case["m"], case["k"], device=DEV, generator=g)
        if case["op"] == "linear":      # a weight kept in 4 bits, in the layout of include/gecc_ops.h
            codes, exps = _codes(w)
            s["w"] = _pack(codes, exps, case["m"], case["k"])
        else:
            s["w"] = w.to(DTYPES[case["dtype"]])
            s["dy"] = _out_gradient(g, case["n"], case["m"], case["dtype"])
    else:
        s["g"] = _weight_gradient(g, case["batch"], case["rows"], case["cols"], case["dtype"])
        s["m"] = 8.0 * _weight_gradient(g, case["batch"], case["rows"], case["cols"], "f32") if case["momentum"] else None
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------------------

def _codes(x):
    """[rows, cols] fp32 -> codes [rows, blocks, 32] (0..15) and exponents [rows, blocks] of their scales."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x, (0, nb * BLOCK - cols)).view(rows, nb, BLOCK)
    amax = x.abs().amax(dim=2)
    exps = torch.where(amax > 0, torch.frexp(amax)[1] - 3, -127).clamp(min=-127)      # floor(log2 amax) - 2
    v = torch.ldexp(x, -exps.unsqueeze(2))
    a = v.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return code | ((v < 0).to(torch.uint8) << 3), exps


def _values(codes, exps, cols):
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    v = torch.ldexp(grid[codes.long()], exps.unsqueeze(2))
    return v.reshape(v.shape[0], -1)[:, :cols]


def _rounded(x):
    return _values(*_codes(x.float()), x.shape[1])


def _pack(codes, exps, rows, cols):
    """(data, scales) as include/gecc_ops.h lays them out: data [rows][cols up to 256s / 2], the lower half of a byte first; scales in
    tiles of 16 rows x 16 blocks, in a tile [row][block % 4][block // 4], one byte each, exponent + 127."""
    kb = -(-cols // 256) * 8
    data = torch.zeros(rows, kb * BLOCK, dtype=torch.uint8, device=codes.device)
    data[:, :codes.shape[1] * BLOCK] = codes.reshape(rows, -1)
    data = data[:, 0::2] | (data[:, 1::2] << 4)
    r16, b16 = -(-rows // 16), -(-kb // 16)
    scales = torch.zeros(r16 * 16, b16 * 16, dtype=torch.uint8, device=codes.device)
    scales[:rows, :exps.shape[1]] = (exps + 127).to(torch.uint8)
    scales = scales.view(r16, 16, b16, 4, 4).permute(0, 2, 1, 4, 3).contiguous()
    return data.contiguous(), scales


def _unpack(data, scales, rows, cols):
    nb = -(-cols // BLOCK)
    codes = torch.stack((data & 15, data >> 4), dim=2).view(rows, -1, BLOCK)[:, :nb]
    r16, b16 = scales.shape[:2]
    exps = scales.permute(0, 2, 1, 4, 3).reshape(r16 * 16, b16 * 16)[:rows, :nb].int() - 127
    return codes, exps


def _orthogonalise(u, scale):
    a, b, c = COEFFICIENTS
    x = u / (u.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        p = torch.matmul(x, x.transpose(1, 2).contiguous())
        p = b * p + c * torch.matmul(p, p)
        x = a * x + torch.matmul(p, x)
    return scale * (x.transpose(1, 2) if tall else x)


def _scale(case):
    return max(1.0, case["rows"] / case["cols"]) ** 0.5


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    dt = DTYPES[s["dtype"]]
    if s["op"] == "quantise":
        q = _rounded(s["x"]).bfloat16()      # exact: 2 significant bits
        return (q, _rounded(s["x"].t()).bfloat16()) if s["both"] else q
    if s["op"] == "linear":
        w = _values(*_unpack(*s["w"], s["m"], s["k"]), s["k"])
        return torch.matmul(_rounded(s["x"]), w.t()).to(dt)
    if s["op"] == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        y = torch.matmul(_rounded(x), _rounded(w).t()).to(dt)
        dx = torch.matmul(_rounded(dy), _rounded(w.t()).t()).to(dt)
        dw = torch.matmul(_rounded(dy.t()), _rounded(x.t()).t())
        return {"y": y, "dx": dx, "dw": dw}
    u, m = s["g"].float(), s["m"]
    if m is not None:
        m.mul_(MU).add_(u)
        u = u + MU * m
    o = _orthogonalise(u, _scale(s)).bfloat16()
    return {"o": o} if m is None else {"o": o, "m": m}


def _run_own(s):
    from paper_2508_04355_amd import ops
    dt = DTYPES[s["dtype"]]
    if s["op"] == "quantise":
        if s["both"]:
            q, t = ops.mx4_quantize(s["x"], both=True)
            return ops.mx4_dequantize(q), ops.mx4_dequantize(t)
        return ops.mx4_dequantize(ops.mx4_quantize(s["x"]))
    if s["op"] == "linear":
        return ops.mx4_linear(s["x"], ops.Mx4(*s["w"], s["m"], s["k"]), dtype=dt)
    if s["op"] == "train":
        w, wt = ops.mx4_quantize(s["w"], both=True)
        x, xt = ops.mx4_quantize(s["x"], both=True)
        y = ops.mx4_gemm(x, w, dtype=dt)
        dx, dw = ops.mx4_linear_backward(s["dy"], wt, xt, dtype=dt)
        return {"y": y, "dx": dx, "dw": dw}
    o = ops.orthogonalize(s["g"], momentum=s["m"], mu=MU, nesterov=True, steps=STEPS, coefficients=COEFFICIENTS, eps=EPS, scale=_scale(s))
    return {"o": o} if s["m"] is None else {"o": o, "m": s["m"]}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    packed = 0.5 + 1.0 / BLOCK
    if case["op"] == "quantise":
        n = case["rows"] * case["cols"]
        # the packed form is written and read back; values come back in bf16
        return {"bytes": n * (size + (2 if case["both"] else 1) * (2 * packed + 2)), "flops": 0}
    if case["op"] == "linear":
        n, k, m = case["n"], case["k"], case["m"]
        return {"bytes": size * n * (k + m) + packed * k * m, "flops": 2.0 * n * k * m}
    if case["op"] == "train":
        n, k, m = case["n"], case["k"], case["m"]
        return {"bytes": size * (2 * n * k + 2 * n * m + k * m) + 4 * k * m, "flops": 6.0 * n * k * m}
    s, l = sorted((case["rows"], case["cols"]))
    n = case["batch"] * s * l
    # X X^T and A A are symmetric: half of each is enough
    return {"bytes": n * (size + 2 + (8 if case["momentum"] else 0)), "flops": case["batch"] * STEPS * (float(s) * (s + 1) * (l + s) + 2.0 * s * s * l)}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------------

def _exact_rounded(x):
    """Each value's nearest neighbour on the block's grid, ties to the even code, found by distance."""
    x = x.double()
    rows, cols = x.shape
    out = torch.empty_like(x)
    for c0 in range(0, cols, BLOCK * 64):          # in pieces, so that the table of distances stays small
        p = x[:, c0:c0 + BLOCK * 64]
        w = p.shape[1]
        p = torch.cat((p, p.new_zeros(rows, -w % BLOCK)), dim=1).view(rows, -1, BLOCK)
        top = p.abs().max(dim=2, keepdim=True).values
        unit = torch.exp2((torch.log2(torch.where(top > 0, top, torch.ones_like(top))) + 1e-12).floor() - 2)
        best = torch.full_like(p, float("inf"))
        got = torch.zeros_like(p)
        for code in (0, 2, 4, 6, 1, 3, 5, 7):      # even codes first: a tie does not replace them
            d = (p.abs() / unit - GRID[code]).abs()
            nearer = d < best
            best = torch.where(nearer, d, best)
            got = torch.where(nearer, torch.full_like(p, GRID[code]), got)
        out[:, c0:c0 + w] = (got * unit * torch.sign(p)).view(rows, -1)[:, :w]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantise":
        q = _exact_rounded(s["x"])
        return (q, _exact_rounded(s["x"].t().contiguous())) if case["both"] else q
    if case["op"] == "linear":
        codes, exps = _unpack(*s["w"], case["m"], case["k"])
        w = torch.tensor(GRID, device=DEV, dtype=torch.float64)[(codes & 7).long()] * torch.exp2(exps.double()).unsqueeze(2)
        w = torch.where(codes > 7, -w, w).view(case["m"], -1)[:, :case["k"]]
        return _exact_rounded(s["x"]) @ w.t()
    if case["op"] == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        y = _exact_rounded(x) @ _exact_rounded(w).t()
        dx = _exact_rounded(dy) @ _exact_rounded(w.t().contiguous()).t()
        dw = _exact_rounded(dy.t().contiguous()) @ _exact_rounded(x.t().contiguous()).t()
        return {"y": y, "dx": dx, "dw": dw}
    a, b, c = COEFFICIENTS
    g, m = s["g"].double(), s["m"]
    if m is not None:
        m = MU * m.double() + g
        g = g + MU * m
    outs = []
    for x in g:                                     # sigma -> a sigma + b sigma^3 + c sigma^5, five times, on each singular value
        x = x / (torch.linalg.vector_norm(x) + EPS)
        left = x.shape[0] <= x.shape[1]
        for _ in range(STEPS):
            gram = x @ x.t() if left else x.t() @ x
            poly = b * gram + c * (gram @ gram)
            poly.diagonal().add_(a)
            x = poly @ x if left else x @ poly
        outs.append(_scale(case) * x)
    o = torch.stack(outs)
    return {"o": o} if m is None else {"o": o, "m": m}
