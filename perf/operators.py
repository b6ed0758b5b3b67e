"""The matrix work of a training step that goes beyond the bf16 products and Adam, as cases that can be timed: products of 8-bit
floating point with a scale for every 128 of the contraction, the quantiser that feeds them, and the update of weight matrices by
their orthogonalised momentum.

A case is a dict of plain values:
  quant    rows x cols of type src (bf16, fp32) to 8-bit codes, along the columns and, transposed, along the rows; tile: one scale for
           128 x 128 (a weight) instead of 128 (an activation)
  linear   y = x W^T + bias: x [tokens, inp] bf16, quantised here, W [out, inp] quantised once per update, y bf16
  grads    dx = dy W and dW = dy^T x of that layer: dy [tokens, out] bf16, quantised here both ways, the codes of x along the tokens and of
           W^T kept from the forward pass and from the update; dx bf16, dW fp32
  orth     count matrices rows x cols orthogonalised, in and out of type src; products of 16 or 32 bits
  muon     one update of a stack of transformer layers: per layer four matrices hidden x hidden, one ffn x hidden and one hidden x ffn
"""
import math

import numpy as np
import torch

own = False

COEFF = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
# an update in the warm-up of a run, as the training loop makes it: sums of DENOM samples' gradients
MUON = dict(lr=1e-4, momentum=0.95, weight_decay=0.01, rms=0.2)
DENOM = 64.0


def listed():
    return [
        # a few odd rows: the smallest call of the quantiser, and the activations of 8192 tokens before a feed-forward product
        dict(kind="quant", rows=37, cols=200, src="fp32", tile=False, name="quant_small"),
        dict(kind="quant", rows=8192, cols=4096, src="bf16", tile=False, name="quant_tokens"),
        # one token through a feed-forward layer: launches and the read of the weight
        dict(kind="linear", tokens=1, inp=1024, out=4096, name="linear_one_token"),
        # a batch that ends anywhere, widths that are no multiple of anything
        dict(kind="linear", tokens=1237, inp=1000, out=2603, name="linear_ragged"),
        # the query, key and value projection of 64 x 128 tokens (base encoder)
        dict(kind="linear", tokens=8192, inp=768, out=2304, name="linear_base"),
        # a large generic product
        dict(kind="linear", tokens=8192, inp=8192, out=8192, name="linear_large"),
        # backward of a short ragged batch, and of a feed-forward layer of the large encoder over 16384 tokens
        dict(kind="grads", tokens=333, inp=520, out=1111, name="grads_ragged"),
        dict(kind="grads", tokens=16384, inp=1024, out=4096, name="grads_large"),
        # one odd matrix in 32 bits; a batch of square ones with 16-bit products
        dict(kind="orth", count=1, rows=130, cols=67, src="fp32", products=32, name="orth_small"),
        dict(kind="orth", count=24, rows=1024, cols=1024, src="bf16", products=16, name="orth_batch"),
        # the toy model in 32 bits; the 24 layers of the large encoder
        dict(kind="muon", layers=1, hidden=128, ffn=512, products=32, name="muon_toy"),
        dict(kind="muon", layers=24, hidden=1024, ffn=4096, products=16, name="muon_large"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call: products from one token to 16384 with widths from 64 to 8192 (odd ones included), matrices from 16 to 2048 a side, stacks of
    1 to 24 layers."""
    kind = rng.choice(["quant", "linear", "linear", "grads", "orth", "muon"])
    if kind == "quant":
        src, tile = rng.choice([("bf16", False), ("bf16", False), ("fp32", False), ("fp32", True), ("bf16", True)])
        return dict(kind=kind, rows=_log_int(rng, 1, 8192), cols=_log_int(rng, 16, 8192), src=src, tile=tile)
    if kind in ("linear", "grads"):
        widths = [rng.choice([64 * _log_int(rng, 1, 64), _log_int(rng, 64, 4096)]) for _ in range(2)]
        return dict(kind=kind, tokens=_log_int(rng, 1, 16384), inp=widths[0], out=widths[1])
    if kind == "orth":
        src, products = rng.choice([("bf16", 16), ("bf16", 16), ("fp32", 32)])
        return dict(kind=kind, count=_log_int(rng, 1, 16), rows=_log_int(rng, 16, 2048), cols=_log_int(rng, 16, 2048), src=src, products=products)
    hidden = 64 * _log_int(rng, 1, 16)
    return dict(kind=kind, layers=rng.randint(1, 12), hidden=hidden, ffn=hidden * rng.choice([2, 4]), products=rng.choice([16, 16, 32]))


# ---- the 8-bit format ---------------------------------------------------------------------------
def _blocks(n):
    return -(-n // 128)


def _wide(n):
    """Bytes of a row of n codes: whole blocks, zeros behind the last code."""
    return 128 * _blocks(n)


def _scale_ld(n):
    return 4 * -(-_blocks(n) // 4)


def _exponent(amax):
    """The least e with amax <= 448 2^e, as the byte e + 127."""
    f, x = torch.frexp(amax)
    e = torch.where(f <= 0.875, x - 9, x - 8)
    return (torch.where(amax == 0, torch.zeros_like(e), e) + 127).clamp(0, 254)


def _power(byte):
    """2^(byte - 127) in 32 bits, from its bits."""
    return torch.where(byte == 0, 1 << 22, byte << 23).to(torch.int32).view(torch.float32)


def _codes(x, tile):
    """Codes [R, whole blocks] (float8) and scale bytes [R, blocks] of x [R, C] along its columns."""
    R, C = x.shape
    g = torch.nn.functional.pad(x.float(), (0, _wide(C) - C)).reshape(R, -1, 128)
    amax = g.abs().amax(2)
    if tile:
        amax = torch.nn.functional.pad(amax, (0, 0, 0, _wide(R) - R)).view(-1, 128, amax.shape[1]).amax(1).repeat_interleave(128, 0)[:R]
    byte = _exponent(amax)
    q = (g * _power(254 - byte)[:, :, None]).to(torch.float8_e4m3fn).view(R, -1)
    return q, byte.to(torch.uint8)


def _values(q, s):
    """The values, in 32 bits, that codes and scale bytes stand for."""
    return (q.float().view(q.shape[0], -1, 128) * _power(s.int())[:, :, None]).view(q.shape[0], -1)


def _keep(x, tile):
    """Codes as a program keeps them: bytes in rows of whole blocks, scale bytes in rows of whole words."""
    q, s = _codes(x, tile)
    return q.view(torch.uint8), torch.nn.functional.pad(s, (0, _scale_ld(x.shape[1]) - s.shape[1]))


def _empty(rows, n, dev):
    return torch.empty(rows, _wide(n), dtype=torch.uint8, device=dev), torch.zeros(rows, _scale_ld(n), dtype=torch.uint8, device=dev)


# ---- inputs ---------------------------------------------------------------------------------------
def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _tokens(gen, rows, cols):
    """Activations: tokens of different size, and a few channels that are much larger than the others."""
    x = _rand(gen, rows, cols) * torch.exp(0.3 * _rand(gen, rows, 1))
    return x * (1 + 20 * (torch.rand(cols, generator=gen, device="cuda") < 0.01))


def _gradients(gen, rows, cols):
    """Gradients of tokens: sizes over two orders of magnitude from token to token."""
    return _rand(gen, rows, cols) * 1e-3 * torch.exp(_rand(gen, rows, 1))


def _matrices(gen, count, rows, cols):
    """Gradients of weights: a few directions that the tokens share, and noise."""
    r = min(8, rows, cols)
    strong = torch.matmul(_rand(gen, count, rows, r), _rand(gen, count, r, cols)) * (2.0 / math.sqrt(r))
    return (strong + _rand(gen, count, rows, cols)) * 1e-3


def _stack(case):
    """(rows, cols) of a stack's matrices in the order of the flat buffer, and the number of its elements."""
    h, f = case["hidden"], case["ffn"]
    shapes = [(h, h)] * 4 + [(f, h), (h, f)]
    return shapes * case["layers"], case["layers"] * (4 * h * h + 2 * f * h)


def _offsets(shapes):
    return np.concatenate([[0], np.cumsum([r * c for r, c in shapes])]).tolist()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], dict(case)
    bf16 = torch.bfloat16
    if kind == "quant":
        R, C = case["rows"], case["cols"]
        x = 0.02 * _rand(gen, R, C) if case["tile"] else _tokens(gen, R, C)
        s["x"] = x.to(bf16 if case["src"] == "bf16" else torch.float32)
        s["q"], s["s"] = _empty(R, C, "cuda")
        s["qt"], s["st"] = _empty(C, R, "cuda")
    elif kind == "linear":
        T, K, N = case["tokens"], case["inp"], case["out"]
        s["x"] = _tokens(gen, T, K).to(bf16)
        s["bias"] = (0.02 * _rand(gen, N)).to(bf16)
        s["wq"], s["ws"] = _keep(0.02 * _rand(gen, N, K), True)
        s["q"], s["s"] = _empty(T, K, "cuda")
        s["y"] = torch.empty(T, N, dtype=bf16, device="cuda")
        s["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    elif kind == "grads":
        T, K, N = case["tokens"], case["inp"], case["out"]
        s["dy"] = _gradients(gen, T, N).to(bf16)
        s["xtq"], s["xts"] = _keep(_tokens(gen, T, K).to(bf16).t().contiguous(), False)
        s["wtq"], s["wts"] = _keep(0.02 * _rand(gen, K, N), True)
        s["q"], s["s"] = _empty(T, N, "cuda")
        s["qt"], s["st"] = _empty(N, T, "cuda")
        s["dx"] = torch.empty(T, K, dtype=bf16, device="cuda")
        s["dw"] = torch.empty(N, K, device="cuda")
        s["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    elif kind == "orth":
        x = _matrices(gen, case["count"], case["rows"], case["cols"])
        s["x"] = x.to(bf16 if case["src"] == "bf16" else torch.float32)
        s["y"] = torch.empty_like(s["x"])
        s["shapes"] = [(case["rows"], case["cols"])] * case["count"]
    else:
        s["shapes"], n = _stack(case)
        s["w"] = 0.02 * _rand(gen, n)
        s["lowp"] = s["w"].to(bf16)
        # the momentum of a run in progress, and this update's gradient sums, per layer and kind of matrix
        fields = [torch.cat([_matrices(gen, case["layers"], r, c).view(case["layers"], -1) for r, c in s["shapes"][:6]], 1).view(-1)
                  for _ in range(2)]
        s["m"], s["G"] = 4.0 * fields[0], DENOM * fields[1]
    if "shapes" in s:
        s["at"] = _offsets(s["shapes"])
        s["workspace"] = None
    return s


# ---- the plain forms ------------------------------------------------------------------------------
def _polynomial(x):
    """One step of X <- a X + (b A + c A A) X, A = X X^T, on a batch."""
    a, b, c = COEFF
    A = torch.matmul(x, x.transpose(1, 2).contiguous())
    return a * x + torch.matmul(b * A + c * torch.matmul(A, A), x)


def _orthogonal(x):
    """x [count, rows, cols] in 32 bits."""
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    x = x / (x.square().sum((1, 2), keepdim=True, dtype=torch.float64).sqrt().float() + EPS)
    x = _polynomial(_polynomial(_polynomial(_polynomial(_polynomial(x)))))
    return x.transpose(1, 2) if tall else x


def _factor(rows, cols):
    return MUON["rms"] * math.sqrt(max(rows, cols))


def _muon(s):
    """In 32 bits: the momentum, then per shape a batch of matrices, then the weights and their bf16 copy."""
    g = s["G"] / DENOM
    s["m"].mul_(MUON["momentum"]).add_(g)
    u = g + MUON["momentum"] * s["m"]
    L, h, f = s["layers"], s["hidden"], s["ffn"]
    u, w = u.view(L, -1), s["w"].view(L, -1)
    cut = [0, 4 * h * h, 4 * h * h + f * h, 4 * h * h + 2 * f * h]
    parts = [(u[:, i:j], r, c) for i, j, r, c in zip(cut, cut[1:], (h, f, h), (h, h, f))]
    step = torch.cat([(_factor(r, c) * _orthogonal(p.reshape(-1, r, c))).reshape(L, -1) for p, r, c in parts], 1)
    w.mul_(1 - MUON["lr"] * MUON["weight_decay"]).sub_(MUON["lr"] * step)
    s["lowp"].copy_(s["w"])
    return [s["w"], s["m"], s["lowp"]]


def _plain(s):
    kind = s["kind"]
    if kind == "quant":
        q, b = _codes(s["x"], s["tile"])
        qt, bt = _codes(s["x"].t(), s["tile"])
        return [q, b.view(torch.float8_e8m0fnu), qt, bt.view(torch.float8_e8m0fnu)]
    if kind == "linear":
        y = torch.matmul(_values(*_codes(s["x"], False)), _values(s["wq"].view(torch.float8_e4m3fn), s["ws"][:, :_blocks(s["inp"])]).t())
        return [(y + s["bias"].float()).to(torch.bfloat16)]
    if kind == "grads":
        f8 = torch.float8_e4m3fn
        dx = torch.matmul(_values(*_codes(s["dy"], False)), _values(s["wtq"].view(f8), s["wts"][:, :_blocks(s["out"])]).t())
        dw = torch.matmul(_values(*_codes(s["dy"].t(), False)), _values(s["xtq"].view(f8), s["xts"][:, :_blocks(s["tokens"])]).t())
        return [dx.to(torch.bfloat16), dw]
    if kind == "orth":
        return [_orthogonal(s["x"].float()).to(s["x"].dtype)]
    return _muon(s)


# ---- the framework's calls ------------------------------------------------------------------------
def _mats(hs, s):
    return [(at, c, r, c) for at, (r, c) in zip(s["at"], s["shapes"])]


def _calls(s):
    from paper_2009_14783_amd import binding as hs
    kind = s["kind"]
    types = {torch.bfloat16: hs.HS_BF16, torch.float32: hs.HS_FP32}
    f8 = torch.float8_e4m3fn
    if kind == "quant":
        x = s["x"]
        R, C = x.shape
        hs.hs_op_quantize_fp8(types[x.dtype], x, C, R, C, int(s["tile"]), s["q"], s["q"].shape[1], s["s"], s["s"].shape[1], s["qt"], s["qt"].shape[1],
                              s["st"], s["st"].shape[1])
        e8 = torch.float8_e8m0fnu
        return [s["q"].view(f8), s["s"].view(e8)[:, :_blocks(C)], s["qt"].view(f8), s["st"].view(e8)[:, :_blocks(R)]]
    if kind == "linear":
        T, K, N = s["tokens"], s["inp"], s["out"]
        hs.hs_op_quantize_fp8(hs.HS_BF16, s["x"], K, T, K, 0, s["q"], s["q"].shape[1], s["s"], s["s"].shape[1])
        hs.hs_op_gemm_fp8(T, N, K, s["q"], s["q"].shape[1], s["s"], s["s"].shape[1], s["wq"], s["wq"].shape[1], s["ws"], s["ws"].shape[1], s["y"], N,
                          bias=s["bias"], scratch=s["scratch"], scratch_bytes=s["scratch"].numel())
        return [s["y"]]
    if kind == "grads":
        T, K, N = s["tokens"], s["inp"], s["out"]
        hs.hs_op_quantize_fp8(hs.HS_BF16, s["dy"], N, T, N, 0, s["q"], s["q"].shape[1], s["s"], s["s"].shape[1], s["qt"], s["qt"].shape[1], s["st"],
                              s["st"].shape[1])
        hs.hs_op_gemm_fp8(T, K, N, s["q"], s["q"].shape[1], s["s"], s["s"].shape[1], s["wtq"], s["wtq"].shape[1], s["wts"], s["wts"].shape[1], s["dx"], K,
                          scratch=s["scratch"], scratch_bytes=s["scratch"].numel())
        hs.hs_op_gemm_fp8(N, K, T, s["qt"], s["qt"].shape[1], s["st"], s["st"].shape[1], s["xtq"], s["xtq"].shape[1], s["xts"], s["xts"].shape[1], s["dw"], K,
                          c_f32=1, scratch=s["scratch"], scratch_bytes=s["scratch"].numel())
        return [s["dx"], s["dw"]]
    products = hs.HS_BF16 if s["products"] == 16 else hs.HS_FP32
    if s["workspace"] is None:      # the plan that a program makes once: the list of its matrices and the workspace for it
        s["mats"] = hs.make_matrices(_mats(hs, s))
        s["workspace"] = torch.empty(hs.hs_orthogonalize_workspace_bytes(s["mats"], products), dtype=torch.uint8, device="cuda")
    ws, size = s["workspace"], s["at"][-1]
    if kind == "orth":
        hs.hs_op_orthogonalize(types[s["x"].dtype], s["x"], s["y"], size, s["mats"], products, STEPS, None, EPS, ws, ws.numel())
        return [s["y"]]
    hs.hs_muon_step(s["w"], s["m"], s["G"], s["lowp"], size, s["mats"], products, DENOM, MUON["lr"], MUON["momentum"], 1, MUON["weight_decay"],
                    MUON["rms"], STEPS, None, EPS, ws, ws.numel())
    return [s["w"], s["m"], s["lowp"]]


def run(state):
    """One pass: the codes and scales, the layer's output, its gradients, the orthogonal matrices, or the updated weights, momentum and bf16 copy."""
    return _calls(state) if own else _plain(state)


def work(case):
    """Inputs read once, outputs written once; operations of the products (a symmetric result has half of them)."""
    kind = case["kind"]
    if kind == "quant":
        R, C = case["rows"], case["cols"]
        return {"bytes": R * C * ((2 if case["src"] == "bf16" else 4) + 2) + R * _blocks(C) + C * _blocks(R), "flops": 0}
    if kind in ("linear", "grads"):
        T, K, N = case["tokens"], case["inp"], case["out"]
        if kind == "linear":
            return {"bytes": 2 * T * K + N * K + 2 * T * N, "flops": 2 * T * K * N}
        return {"bytes": 2 * T * N + T * K + N * K + 2 * T * K + 4 * N * K, "flops": 4 * T * K * N}
    shapes = [(case["rows"], case["cols"])] * case["count"] if kind == "orth" else _stack(case)[0]
    flops = sum(STEPS * (3.0 * min(r, c) ** 2 * max(r, c) + min(r, c) ** 3) for r, c in shapes)
    n = sum(r * c for r, c in shapes)
    return {"bytes": n * (22 if kind == "muon" else 4 if case["src"] == "bf16" else 8), "flops": flops}


# ---- from the definitions, in 64 bits ---------------------------------------------------------------
def _grid(x, axis, square):
    """x in 64 bits rounded to 8-bit codes along `axis`: the codes' values, and the exponents spread over x's elements.  Four bits of
    significand, steps of 2^-9 below 2^-6, the scale of a group the power of two that brings its largest value to 448 at most."""
    x = x.double()
    group = torch.arange(x.shape[axis], device=x.device) // 128
    m = x.abs()
    cells = torch.zeros(int(group[-1]) + 1, x.shape[1 - axis], dtype=torch.float64, device=x.device)
    cells.index_reduce_(0, group, m if axis == 0 else m.t(), "amax")
    if square:
        other = torch.arange(x.shape[1 - axis], device=x.device) // 128
        most = torch.zeros(int(other[-1]) + 1, cells.shape[0], dtype=torch.float64, device=x.device).index_reduce_(0, other, cells.t(), "amax")
        cells = most[other].t()
    # ceil(log2(largest / 448)), put right where the logarithm is a rounding off
    e = torch.ceil(torch.log2(cells / 448.0).clamp(-127, 127))
    e = e + (cells > 448.0 * torch.exp2(e)).double() - (cells <= 448.0 * torch.exp2(e - 1)).double()
    e = torch.where(cells == 0, torch.zeros_like(e), e).clamp(-127, 127)
    scale = e[group] if axis == 0 else e[group].t()
    y = x / torch.exp2(scale)
    ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))).clamp_min(-6.0) - 3.0)
    return torch.round(y / ulp) * ulp, scale, e


def _rounded(x, axis, square):
    code, scale, _ = _grid(x, axis, square)
    return code * torch.exp2(scale)


def _whole(q, s, n):
    """The values of kept codes, in 64 bits."""
    block = torch.arange(n, device=q.device) // 128
    return q.view(torch.float8_e4m3fn)[:, :n].double() * torch.exp2(s.double() - 127.0)[:, block]


def _limit(u):
    """u / (|u| + eps) through the polynomial in 64 bits, as X (a I + B (b I + c B)) with B the Gram matrix of the shorter side."""
    u = u / (torch.sqrt((u * u).sum()) + EPS)
    flip = u.shape[0] < u.shape[1]
    v = u.t().contiguous() if flip else u
    eye = torch.eye(v.shape[1], dtype=torch.float64, device=u.device)
    for _ in range(STEPS):
        B = v.t().contiguous() @ v
        v = v @ (COEFF[0] * eye + B @ (COEFF[1] * eye + COEFF[2] * B))
    return v.t() if flip else v


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quant":
        q, _, e = _grid(s["x"], 1, case["tile"])
        qt, _, et = _grid(s["x"], 0, case["tile"])
        pad = torch.nn.functional.pad
        return [pad(q, (0, _wide(case["cols"]) - case["cols"])), torch.exp2(e.t()), pad(qt.t(), (0, _wide(case["rows"]) - case["rows"])),
                torch.exp2(et.t())]
    if kind == "linear":
        return [_rounded(s["x"], 1, False) @ _whole(s["wq"], s["ws"], case["inp"]).t().contiguous() + s["bias"].double()]
    if kind == "grads":
        dx = _rounded(s["dy"], 1, False) @ _whole(s["wtq"], s["wts"], case["out"]).t().contiguous()
        dw = _rounded(s["dy"], 0, False).t().contiguous() @ _whole(s["xtq"], s["xts"], case["tokens"]).t().contiguous()
        return [dx, dw]
    if kind == "orth":
        return [torch.stack([_limit(x.double()) for x in s["x"]])]
    w, m, G = (s[k].double() for k in ("w", "m", "G"))
    m = MUON["momentum"] * m + G / DENOM
    u = G / DENOM + MUON["momentum"] * m
    for at, (r, c) in zip(s["at"], s["shapes"]):
        i = slice(at, at + r * c)
        w[i] = w[i] - MUON["lr"] * MUON["weight_decay"] * w[i] - (MUON["lr"] * _factor(r, c) * _limit(u[i].view(r, c))).reshape(-1)
    return [w, m, w]
