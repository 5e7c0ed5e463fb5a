"""Performance cases of the norm, microscaled and grouped operators.

A transformer layer with quantized linears normalizes its residual stream,
quantizes the result and multiplies it with quantized weights.  Each case
is one pass through one of these steps on buffers a program already holds:
RMS norm with the residual's addition and 8-bit or MXFP4 codes, MXFP4
quantization of activations or weights (and back to values), the MXFP4
product of a layer, and the product of routed experts with ragged row
counts.

MXFP4 here is the OCP Microscaling format: blocks of 32 values along a row
share a scale 2^e (a byte e + 127), values are E2M1 (0, 0.5, 1, 1.5, 2, 3,
4, 6 and a sign), two to a byte, the even element in the low half.

Quantized outputs are returned as the values they stand for, in bf16 (which
holds every MXFP4 value of these ranges exactly).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5

# most multiply-adds of one drawn product: those of the largest listed one
MAX_MACS = 16384 * 14336 * 4096
# most elements of one drawn norm or quantization
MAX_ROW_ELEMS = 8192 * 8192


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one decode token's norm in front of an 8-bit attention projection
        dict(name="norm8_decode_1", op="norm8", n=1, d=4096, dtype="bf16", residual=True),
        # the norm of a prefill at the stress width
        dict(name="norm8_prefill_8192", op="norm8", n=8192, d=8192, dtype="bf16", residual=True),
        # a decode batch in front of an MXFP4 projection
        dict(name="normmx_decode_48", op="normmx", n=48, d=4096, dtype="bf16", residual=True),
        # a ragged prefill in fp32 without a residual: the first layer's
        # norm, at the MLP-down width
        dict(name="normmx_f32_3001", op="normmx", n=3001, d=14336, dtype="f32", residual=False),
        # activations of a ragged prompt chunk in front of the MLP-down product
        dict(name="quant_chunk_257", op="quant", n=257, d=14336, dtype="bf16"),
        # the stress layer's weights, quantized once when a model is loaded
        dict(name="quant_weights_stress", op="quant", n=28672, d=8192, dtype="f32"),
        # one decode token through an attention projection
        dict(name="linear_decode_1", op="linear", n=1, d_in=4096, d_out=4096, out="f32"),
        # a decode batch through the MLP-up projection
        dict(name="linear_decode_48", op="linear", n=48, d_in=4096, d_out=14336, out="bf16"),
        # MLP-up prefill at the benchmark's shape
        dict(name="linear_prefill_8192", op="linear", n=8192, d_in=4096, d_out=14336, out="bf16"),
        # a decode batch of 32 tokens, four of 64 experts each, gathered by
        # token from the batch's codes
        dict(name="grouped_decode_32x4", op="grouped", tokens=32, topk=4, groups=64, d_in=2048,
             d_out=1024, gather=True, out="f32"),
        # a ragged prompt chunk, two of 16 experts a token, gathered
        dict(name="grouped_chunk_1003x2", op="grouped", tokens=1003, topk=2, groups=16, d_in=4096,
             d_out=4096, gather=True, out="f32"),
        # the MLP-down products of a prefill's routed rows, already sorted
        # by expert
        dict(name="grouped_prefill_8192x2", op="grouped", tokens=8192, topk=2, groups=8, d_in=14336,
             d_out=4096, gather=False, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm8"] * 3 + ["normmx"] * 3 + ["quant"] * 3 + ["linear"] * 6 + ["grouped"] * 5)
    if op in ("norm8", "normmx", "quant"):
        d = _log_int(rng, 128, 16384)
        if op != "norm8" or rng.random() < 0.7:     # 8-bit rows may have any length
            d = max(32, d // 32 * 32)
        case = dict(op=op, n=max(1, min(_log_int(rng, 1, 16384), MAX_ROW_ELEMS // d)), d=d,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
        if op != "quant":
            case["residual"] = rng.random() < 0.7
        return case
    d_in = max(4, _log_int(rng, 256, 14336) // 32) * 32
    if rng.random() < 0.6:
        d_in = max(256, d_in // 256 * 256)
    d_out = _log_int(rng, 100, 14336)
    if rng.random() < 0.6:
        d_out = max(64, d_out // 64 * 64)
    out = rng.choice(["f32", "bf16"])
    if op == "linear":
        n = max(1, min(_log_int(rng, 1, 8192), MAX_MACS // (d_in * d_out)))
        return dict(op=op, n=n, d_in=d_in, d_out=d_out, out=out)
    groups = rng.choice([2, 4, 8, 16, 32, 64, 128])
    # every expert's weights fit beside three states
    d_out = max(64, min(d_out, (1 << 29) // (groups * d_in)))
    topk = rng.choice([1, 2, 2, 4, 8])
    topk = min(topk, groups)
    tokens = max(1, min(_log_int(rng, 1, 8192), MAX_MACS // (4 * topk * d_in * d_out)))
    return dict(op=op, tokens=tokens, topk=topk, groups=groups, d_in=d_in, d_out=d_out,
                gather=rng.random() < 0.5, out=out)


# ------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(n, d, g):
    """Rows with a lognormal scale a channel and a few outlier channels."""
    scale = torch.exp(0.7 * _randn(g, d))
    scale[torch.randint(0, d, (8,), generator=g, device="cuda")] *= 30.0
    return _randn(g, n, d) * scale


def _encode(v):
    """MXFP4 codes and scale bytes of rows v [n, d]."""
    n, d = v.shape
    b = v.view(n, d // 32, 32)
    e = torch.floor(torch.log2(b.abs().amax(2).clamp(min=1e-30))) - 2.0
    a = b.abs() / torch.exp2(e).unsqueeze(2)
    idx = torch.zeros(a.shape, dtype=torch.uint8, device="cuda")
    for mid in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
        idx += a > mid
    idx = (idx + 8 * (b < 0).to(torch.uint8)).view(n, d)
    return idx[:, 0::2] + 16 * idx[:, 1::2], (e + 127.0).to(torch.uint8)


def _weights(rows, d, g):
    """Gaussian rows with a lognormal scale a row."""
    return _randn(g, rows, d) * (torch.exp(0.3 * _randn(g, rows, 1)) / math.sqrt(d))


def _routing(case, g):
    """Row order by expert, offsets [groups + 1] and the token of every
    row: each token takes its top-k experts by score, where experts differ
    in popularity, so counts are ragged and some experts may have no row."""
    t, k, e = case["tokens"], case["topk"], case["groups"]
    score = _randn(g, t, e) + 0.7 * _randn(g, e)
    expert = score.topk(k, dim=1).indices.reshape(-1)
    order = torch.argsort(expert, stable=True)
    counts = torch.bincount(expert, minlength=e)
    offsets = torch.zeros(e + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0).to(torch.int32)
    return order, expert[order], offsets, int(counts.max())


def prepare(case, seed):
    g = _gen(seed)
    op, s = case["op"], {"case": case}
    if op in ("norm8", "normmx", "quant"):
        n, d, dt = case["n"], case["d"], _dtype(case["dtype"])
        s["x"] = _activations(n, d, g).to(dt)
        s["values"] = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
        if op == "norm8":
            s["codes"] = torch.empty(n, d, dtype=torch.int8, device="cuda")
            s["s_x"] = torch.empty(n, dtype=torch.float32, device="cuda")
        else:
            s["codes"] = torch.empty(n, d // 2, dtype=torch.uint8, device="cuda")
            s["scales"] = torch.empty(n, d // 32, dtype=torch.uint8, device="cuda")
        if op != "quant":
            s["weight"] = (1.0 + 0.2 * _randn(g, d)).to(dt)
            s["res"] = _activations(n, d, g).to(dt) if case["residual"] else None
            s["res_out"] = torch.empty(n, d, dtype=dt, device="cuda") if case["residual"] else None
        return s
    d_in, d_out = case["d_in"], case["d_out"]
    if op == "linear":
        s["cx"], s["ex"] = _encode(_activations(case["n"], d_in, g))
        s["cw"], s["ew"] = _encode(_weights(d_out, d_in, g))
        s["y"] = torch.empty(case["n"], d_out, dtype=_dtype(case["out"]), device="cuda")
        return s
    e, m = case["groups"], case["tokens"] * case["topk"]
    order, s["expert"], s["offsets"], s["longest"] = _routing(case, g)
    s["cx"], s["ex"] = _encode(_activations(case["tokens"] if case["gather"] else m, d_in, g))
    s["row_ids"] = (order // case["topk"]).to(torch.int32) if case["gather"] else None
    s["cw"] = torch.empty(e, d_out, d_in // 2, dtype=torch.uint8, device="cuda")
    s["ew"] = torch.empty(e, d_out, d_in // 32, dtype=torch.uint8, device="cuda")
    for i in range(e):
        s["cw"][i], s["ew"][i] = _encode(_weights(d_out, d_in, g))
    s["y"] = torch.empty(m, d_out, dtype=_dtype(case["out"]), device="cuda")
    return s


# -------------------------------------------------------------- plain forms
def _mx4_values(v):
    """Values of v [n, d] after MXFP4 quantization, in fp32."""
    n, d = v.shape
    b = v.view(n, d // 32, 32)
    # floor(log2) of a block's largest magnitude from its exponent field, in
    # [-125, 125] after the format's largest exponent 2 is taken off
    e = (b.abs().amax(2, keepdim=True).view(torch.int32) >> 23) - 129
    scale = torch.exp2(e.clamp(min=-126).float())
    a = b.abs() / scale
    q = torch.where(a < 2, torch.round(a * 2) / 2,
                    torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2)).clamp(max=6.0)
    return (torch.copysign(q, b) * scale).view(n, d)


def _mx4_decode(codes, scales):
    """fp32 values of packed codes [..., d/2] and scale bytes [..., d/32]."""
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0,
                          -4.0, -6.0], device=codes.device)
    c = codes.to(torch.int32)
    v = torch.stack([level[c & 15], level[c >> 4]], dim=-1)
    v = v.view(*codes.shape[:-1], scales.shape[-1], 32)
    return (v * torch.exp2(scales.float() - 127.0).unsqueeze(-1)).flatten(-2)


def _norm(s):
    """fp32 y of a norm pass: the sum of squares in 64 bits (long rows, and
    codes are decided next to a border), and the updated residual."""
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    r = 1.0 / torch.sqrt(h.double().square().mean(1, keepdim=True) + EPS)
    return h, (h * s["weight"].float()) * r.float()


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "quant":
        return {"values": _mx4_values(s["x"].float()).to(torch.bfloat16)}
    if op in ("norm8", "normmx"):
        h, y = _norm(s)
        out = {} if s["res"] is None else {"residual": h.to(s["x"].dtype)}
        if op == "normmx":
            out["values"] = _mx4_values(y).to(torch.bfloat16)
            return out
        amax = y.abs().amax(1, keepdim=True)
        s_x = amax / 127.0
        # a division of tensors: a number over a tensor is formed through
        # the rounded reciprocal, which moves codes next to a border
        q = torch.round(y * torch.div(torch.full_like(amax, 127.0), amax)).clamp(-127, 127)
        return out | {"values": (q * s_x).to(torch.bfloat16), "s_x": s_x[:, 0]}
    x = _mx4_decode(s["cx"], s["ex"])
    w = _mx4_decode(s["cw"], s["ew"])
    dt = _dtype(case["out"])
    if op == "linear":
        return {"y": torch.matmul(x, w.t().contiguous()).to(dt)}
    # every expert's rows, padded to the longest, as one batch of products
    offsets, expert = s["offsets"].long(), s["expert"]
    m, longest = expert.shape[0], s["longest"]
    at = offsets[:-1, None] + torch.arange(longest, device="cuda")
    at = at.clamp(max=m - 1)
    if s["row_ids"] is not None:
        at = s["row_ids"].long()[at]
    y = torch.bmm(x[at], w.transpose(1, 2).contiguous())
    place = torch.arange(m, device="cuda") - offsets[expert]
    return {"y": y[expert, place].to(dt)}


# -------------------------------------------------------------------- pass
def run(s):
    if not own:
        return _run_plain(s)
    import paper_2603_04359_amd as cat
    op = s["case"]["op"]
    if op == "quant":
        cat.cat_mx4_quant(s["x"], s["codes"], s["scales"])
        cat.cat_mx4_dequant(s["codes"], s["scales"], s["values"])
        return {"values": s["values"]}
    if op == "normmx":
        cat.cat_rmsnorm_mx4(s["x"], s["weight"], s["codes"], s["scales"], residual=s["res"],
                            residual_out=s["res_out"], eps=EPS)
        cat.cat_mx4_dequant(s["codes"], s["scales"], s["values"])
        out = {"values": s["values"]}
    elif op == "norm8":
        cat.cat_rmsnorm_quant(s["x"], s["weight"], s["codes"], s["s_x"], residual=s["res"],
                              residual_out=s["res_out"], eps=EPS)
        torch.mul(s["codes"], s["s_x"][:, None], out=s["values"])
        out = {"values": s["values"], "s_x": s["s_x"]}
    elif op == "linear":
        cat.cat_mx4_linear(s["cx"], s["ex"], s["cw"], s["ew"], s["y"])
        return {"y": s["y"]}
    else:
        cat.cat_mx4_linear_grouped(s["cx"], s["ex"], s["offsets"], s["cw"], s["ew"], s["y"],
                                   row_ids=s["row_ids"])
        return {"y": s["y"]}
    if s["res"] is not None:
        out["residual"] = s["res_out"]
    return out


def work(case):
    """Each input read once, each output written once (quantized outputs as
    bf16 values); multiply-adds as two operations."""
    op = case["op"]
    if op in ("norm8", "normmx", "quant"):
        n, d, el = case["n"], case["d"], 2 if case["dtype"] == "bf16" else 4
        streams = 1 + (2 if case.get("residual") else 0)
        byts = n * d * (el * streams + 2) + (0 if op == "quant" else d * el) + (4 * n if op == "norm8" else 0)
        return {"bytes": byts, "flops": n * d * (4 if op == "quant" else 8)}
    d_in, d_out = case["d_in"], case["d_out"]
    row = d_in // 2 + d_in // 32
    out = 4 if case["out"] == "f32" else 2
    if op == "linear":
        n = case["n"]
        return {"bytes": (n + d_out) * row + n * d_out * out, "flops": 2 * n * d_in * d_out}
    m, e = case["tokens"] * case["topk"], case["groups"]
    rows = case["tokens"] if case["gather"] else m
    # with fewer rows than experts only the weights of the chosen ones
    byts = rows * row + min(m, e) * d_out * row + m * d_out * out + 4 * (e + 1) + (4 * m if case["gather"] else 0)
    return {"bytes": byts, "flops": 2 * m * d_in * d_out}


# --------------------------------------------------------- 64-bit reference
def _nearest_mx4(v):
    """MXFP4 values of v (fp64) by the distance to each level: the nearest
    level, of two equally near the one with the even code."""
    n, d = v.shape
    b = v.view(-1, 32)
    amax = b.abs().amax(1, keepdim=True)
    e = torch.frexp(amax)[1].double() - 1.0             # floor(log2 amax)
    scale = torch.exp2(e - 2.0)
    scale = torch.where(amax > 0, scale, torch.ones_like(scale))
    a = b.abs() / scale
    out = torch.zeros_like(a)
    levels = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
    for i in range(1, 8):
        mid = (levels[i - 1] + levels[i]) / 2
        # a tie goes to the even code: up to level i where i is even
        out = torch.where((a >= mid) if i % 2 == 0 else (a > mid), levels[i], out)
    return (torch.where(b < 0, -out, out) * scale).view(n, d)


def _decode64(codes, scales):
    half = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).to(torch.int64)
    mag, neg = half % 8, half >= 8
    val = torch.where(mag < 2, mag * 0.5, (1.0 + (mag % 2) * 0.5) * torch.exp2((mag // 2 - 1).double()))
    val = torch.where(neg, -val, val.double()).double()
    return val * torch.exp2(scales.double() - 127.0).repeat_interleave(32, dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        return {"values": _nearest_mx4(s["x"].double())}
    if op in ("norm8", "normmx"):
        h = s["x"].double()
        if s["res"] is not None:
            h = h + s["res"].double()
        y = h * s["weight"].double() / (h.pow(2).sum(1, keepdim=True) / h.shape[1] + EPS).sqrt()
        out = {} if s["res"] is None else {"residual": h}
        if op == "normmx":
            return out | {"values": _nearest_mx4(y)}
        step = y.abs().amax(1, keepdim=True) / 127.0
        return out | {"values": torch.round(y / step) * step, "s_x": step[:, 0]}
    x = _decode64(s["cx"], s["ex"])
    if op == "linear":
        y = torch.empty(case["n"], case["d_out"], dtype=torch.float64, device="cuda")
        for a in range(0, case["d_out"], 2048):
            y[:, a:a + 2048] = x @ _decode64(s["cw"][a:a + 2048], s["ew"][a:a + 2048]).t().contiguous()
        return {"y": y}
    ends = s["offsets"].tolist()
    y = torch.empty(ends[-1], case["d_out"], dtype=torch.float64, device="cuda")
    for i in range(case["groups"]):
        lo, hi = ends[i], ends[i + 1]
        if hi > lo:
            xi = x[lo:hi] if s["row_ids"] is None else x[s["row_ids"][lo:hi].long()]
            y[lo:hi] = xi @ _decode64(s["cw"][i], s["ew"][i]).t().contiguous()
    return {"y": y}
