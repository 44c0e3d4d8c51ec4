"""What is measured of the operators around the 8-bit products of a training or serving step: the
root-mean-square norm that takes the residual's addition in and writes the next product's packed
operand, the log probabilities of given tokens (with entropy and the most likely alternatives)
behind the last product, and the orthogonalised update of a weight.

Where `own` is false, `run` computes each operator in its plain form (elementary torch
operations in 32 bits); where it is true, it makes the calls of ``paper_1501_06633_b200``.
`exact` evaluates the definitions in 64 bits.

RMS norm:        h = x + r,  y = h gamma / sqrt(mean(h^2) + eps)       (r: the residual, may be absent)
Log probability: z = scale x,  lse = log sum exp z,  logprob = z[target] - lse,  entropy = -sum p log p,  p = exp(z - lse)
                 A target outside the row stands for no token: its logprob is 0 and has no gradient.  Alternatives are the
                 largest x, ties to the lowest index; a place for which no logit above -inf is left holds index -1.
Orthogonalised:  X = G / (|G| + eps);  five times  A = X X^T,  X = a X + (b A + c A A) X    (of the shorter side)

The 8-bit format: blocks of up to 128 values along a row ("row") or a column ("col").  With m the
largest finite magnitude of a block and V the largest number of the 8-bit type (448 for E4M3, 57344
for E5M2), the scale is 2^E, E the least integer with m <= V 2^E (0 for zeros), and the values are
x 2^-E rounded to the type.  Scales are E8M0 bytes, [block][row] for rows, [block][column] for columns.
"""
import math

import torch

own = False

BLOCK = 128
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": E4M3, "e5m2": E5M2}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
A, B, C = 3.4445, -4.7750, 2.0315


def listed():
    return [
        # one token of a decoder: the block's output joins the residual, the next projection's operand leaves packed
        dict(name="rms norm one token", op="rms_fprop", rows=1, cols=4096, type="bf16", residual=True, packed=True),
        # a training batch through the same norm
        dict(name="rms norm fprop", op="rms_fprop", rows=8192, cols=4096, type="bf16", residual=True, packed=True),
        # its backward pass from the sum as it was packed, with the gradient that came along the residual
        dict(name="rms norm bprop packed", op="rms_bprop", rows=8192, cols=4096, type="bf16", residual=True, packed=True),
        # a norm inside a layer, of a width that fits nothing, from the wide input
        dict(name="rms norm bprop ragged", op="rms_bprop", rows=1531, cols=2309, type="f16", residual=False, packed=False),
        # one token being decoded: its log probability among the twenty most likely
        dict(name="log probs one token", op="lp_fprop", rows=1, cols=131072, type="bf16", top=20, scale=1.0),
        # scoring a batch of given tokens
        dict(name="log probs fprop", op="lp_fprop", rows=2048, cols=131072, type="bf16", top=5, scale=1.0),
        # fp32 logits of a vocabulary of odd size at a temperature
        dict(name="log probs ragged", op="lp_fprop", rows=301, cols=49999, type="f32", top=1, scale=1.25),
        # the gradient of that batch's log probabilities and entropies, wide
        dict(name="log probs bprop", op="lp_bprop", rows=2048, cols=131072, type="bf16", packed=False, scale=1.0),
        # the same where 8-bit products follow: packed for the input gradient (rows) and the weight gradient (columns)
        dict(name="log probs bprop packed", op="lp_bprop", rows=4096, cols=32000, type="bf16", packed=True, scale=1.0),
        # the update of a square projection
        dict(name="orthogonalise 4096", op="ortho", batch=1, rows=4096, cols=4096, type="bf16", steps=5),
        # of a layer whose sizes fit no tile, from its fp32 gradient
        dict(name="orthogonalise ragged", op="ortho", batch=1, rows=1000, cols=2309, type="f32", steps=5),
        # of sixteen equal small layers at once, taller than wide
        dict(name="orthogonalise batch", op="ortho", batch=16, rows=512, cols=128, type="bf16", steps=5),
    ]


def draw(rng):
    def size(lo, hi, step=1):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, v // step * step))

    def width(lo, hi):  # widths are mostly multiples of 16, sometimes anything
        return size(lo, hi, rng.choice((1, 16, 16, 128)))

    op = rng.choice(("rms_fprop", "rms_bprop", "lp_fprop", "lp_bprop", "ortho", "ortho"))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op in ("rms_fprop", "rms_bprop"):
        cols = width(64, 8192)
        return dict(op=op, rows=size(1, min(8192, 8192 * 4096 // cols)), cols=cols, type=kind, residual=rng.random() < 0.6,
                    packed=rng.random() < 0.5)
    if op in ("lp_fprop", "lp_bprop"):
        cols = width(500, 200000)
        case = dict(op=op, rows=size(1, min(4096, (1 << 27) // cols)), cols=cols, type=kind, scale=rng.choice((1.0, 1.0, 0.5, 1.25)))
        case.update({"top": rng.choice((0, 1, 5, 20, 32))} if op == "lp_fprop" else {"packed": rng.random() < 0.4})
        return case
    rows, cols = width(16, 4096), width(16, 4096)
    return dict(op=op, batch=size(1, max(1, min(24, (1 << 22) // (rows * cols)))), rows=rows, cols=cols, type=kind,
                steps=rng.choice((5, 5, 5, 3, 6)))


def work(case):
    op = case["op"]
    blocks = lambda n: -(-n // BLOCK)  # noqa: E731
    if op == "ortho":
        n, m = sorted((case["rows"], case["cols"]))
        # A and B are symmetric: half of each is computed
        return {"bytes": case["batch"] * n * m * (BYTES[case["type"]] + 2.0),
                "flops": case["batch"] * case["steps"] * (3.0 * n * n * m + 1.0 * n * n * n)}
    r, c, e = case["rows"], case["cols"], BYTES[case["type"]]
    n, scales = r * c, r * blocks(c)
    if op == "rms_fprop":
        return {"bytes": e * n * (3 if case["residual"] else 1) + (n + scales + 4 * r if case["packed"] else e * n) + 4 * c, "flops": 6.0 * n}
    if op == "rms_bprop":
        return {"bytes": e * n * (3 if case["residual"] else 2) + (n + scales if case["packed"] else e * n) + 4 * r + 8 * c, "flops": 10.0 * n}
    if op == "lp_fprop":
        return {"bytes": e * n + r * (8 + 12 + 12 * case["top"]), "flops": 6.0 * n}
    return {"bytes": e * n + r * 24 + (2 * n + scales + blocks(r) * c if case["packed"] else e * n), "flops": 8.0 * n}


# ---------------------------------------------------------------- the plain form


def cut(x, block):
    """`x` in 32 bits as [row blocks][rows of a block][column blocks][columns of a block], zeros at the ends."""
    rows, cols = (1, BLOCK) if block == "row" else (BLOCK, 1)
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % cols, 0, -x.shape[0] % rows))
    return x.view(x.shape[0] // rows, rows, x.shape[1] // cols, cols)


def power(e):
    """2^e in 32 bits, for whole e in [-126, 127]."""
    return ((e + 127) << 23).view(torch.float32)


def pack(x, block, to):
    """(values, scales) of a matrix in 32 bits."""
    parts = cut(x, block)
    most = torch.where(torch.isfinite(parts), parts.abs(), 0.0).amax(dim=(1, 3))
    part, e = torch.frexp(most / LARGEST[to])
    e = torch.where(most == 0, 0, torch.where(part == 0.5, e - 1, e)).clamp(-126, 127).to(torch.int32)
    q = (parts * power(-e)[:, None, :, None]).reshape(parts.shape[0] * parts.shape[1], -1)[:x.shape[0], :x.shape[1]].to(to)
    scales = (e + 127).to(torch.uint8).view(E8M0)
    return q, scales.t().contiguous() if block == "row" else scales


def unpack(q, scales):
    """The values that a matrix packed in rows stands for."""
    return q.to(torch.float32) * scales.to(torch.float32).t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def largest(x, top):
    """Indices of the largest values of each row, ties to the lowest index."""
    bits = (x + 0.0).view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -(bits + (1 << 31)), bits)
    keys = (order << 32) + ((1 << 31) - torch.arange(x.shape[1], device=x.device))
    return (1 << 31) - (torch.topk(keys, top, dim=1).values & 0xFFFFFFFF)


def run_plain(s):
    case, op, f32 = s["case"], s["case"]["op"], torch.float32
    if op == "rms_fprop":
        h, got = s["x"].to(f32), {}
        if case["residual"]:
            h = h + s["r"].to(f32)
            got["sum"] = h.to(s["x"].dtype)
        rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        y = h * rstd * s["gamma"]
        if not case["packed"]:
            return {**got, "y": y.to(s["x"].dtype)}
        q, sq = pack(y, "row", E4M3)
        return {**got, "q": q, "sq": sq, "rstd": rstd[:, 0]}
    if op == "rms_bprop":
        h = unpack(s["c"], s["sc"]) if case["packed"] else s["x"].to(f32)
        dy, rstd = s["dy"].to(f32), s["rstd"][:, None]
        hh, g = h * rstd, dy * s["gamma"]
        dx = rstd * (g - hh * (g * hh).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + s["dsum"].to(f32)
        return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * hh).sum(0)}
    if op in ("lp_fprop", "lp_bprop"):
        x = s["x"].to(f32)
        z, t = x * case["scale"], s["target"]
        token = (t >= 0) & (t < x.shape[1])
        at = torch.where(token, t, 0)[:, None]
    if op == "lp_fprop":
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(1, keepdim=True)
        log_total = torch.log(total)
        got = {"lse": (m + log_total)[:, 0],
               "logprob": torch.where(token, (z.gather(1, at) - m - log_total)[:, 0], 0.0),
               "entropy": (log_total - torch.where(e > 0, e * (z - m), 0.0).sum(1, keepdim=True) / total)[:, 0]}
        if case["top"]:
            i = largest(x, case["top"])
            v = x.gather(1, i)
            got["top_logprob"] = v * case["scale"] - m - log_total
            got["top_index"] = torch.where(v == -math.inf, -1, i).to(torch.int32)
        return got
    if op == "lp_bprop":
        logp = z - s["lse"][:, None]
        p = torch.exp(logp)
        dx = -p * (s["dlogprob"] * token)[:, None] - s["dentropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]), 0.0)
        dx = dx.scatter_add_(1, at, (s["dlogprob"] * token)[:, None]) * case["scale"]
        if not case["packed"]:
            return {"dx": dx.to(s["x"].dtype)}
        (q, sq), (qc, sc) = pack(dx, "row", E5M2), pack(dx, "col", E5M2)
        return {"q_row": q, "s_row": sq, "q_col": qc, "s_col": sc}
    x = s["x"].to(f32)
    tall = case["rows"] > case["cols"]
    x = x.transpose(1, 2) if tall else x
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + 1e-7)
    for _ in range(case["steps"]):
        a = x @ x.transpose(1, 2)
        x = A * x + (B * a + C * (a @ a)) @ x
    return {"out": (x.transpose(1, 2) if tall else x).to(torch.bfloat16)}


# ---------------------------------------------------------------- what a program has in hand


def pitched(q):
    """The same 8-bit matrix in rows that start at multiples of 16 bytes."""
    wide = torch.zeros(q.shape[0], -(-q.shape[1] // 16) * 16, dtype=torch.uint8, device=q.device)
    wide[:, :q.shape[1]] = q.view(torch.uint8)
    return wide.view(q.dtype)[:, :q.shape[1]]


def inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    def hidden(rows, cols):
        """Activations: a few columns much larger than the rest, rows of different sizes, not quite centred."""
        big = torch.where(uniform(cols) < 0.01, 20.0, 1.0)
        return (normal(rows, cols) + 0.1) * big * torch.exp(0.5 * normal(rows, 1))

    def gradient(rows, cols):
        """Gradients: small, and of very different sizes from row to row."""
        return normal(rows, cols) * 1e-4 * torch.exp(normal(rows, 1))

    op, s, kind = case["op"], {"case": case}, TYPES[case["type"]]
    r, c = case["rows"], case["cols"]
    if op == "rms_fprop":
        s["x"], s["gamma"] = normal(r, c).to(kind), 1 + 0.2 * normal(c)
        if case["residual"]:
            s["r"] = hidden(r, c).to(kind)
    elif op == "rms_bprop":
        h = hidden(r, c).to(kind)
        wide = h.to(torch.float32)
        s["rstd"] = 1 / torch.sqrt((wide * wide).mean(1) + EPS)
        s["gamma"], s["dy"] = 1 + 0.2 * normal(c), gradient(r, c).to(kind)
        if case["residual"]:
            s["dsum"] = gradient(r, c).to(kind)
        if case["packed"]:
            q, s["sc"] = pack(wide, "row", E4M3)
            s["c"] = pitched(q)
        else:
            s["x"] = h
    elif op in ("lp_fprop", "lp_bprop"):
        # logits as a trained model gives them: most far below the largest, a few tokens and the end of the row masked
        x = normal(r, c).mul_(2.5).add_(normal(c)).add_(8 * (uniform(r, c) < 8 / c))
        x.masked_fill_(uniform(c) < 0.002, -math.inf)
        x[:, -(c // 100):] = -math.inf
        s["x"] = x.to(kind)
        token = (uniform(r) * (c - c // 100)).to(torch.int64)
        likely = s["x"].argmax(1)
        s["target"] = torch.where(uniform(r) < 0.1, -100, torch.where(uniform(r) < 0.5, likely, token))
        if op == "lp_bprop":
            z = s["x"].to(torch.float32) * case["scale"]
            logp = torch.log_softmax(z, 1)
            s["lse"] = torch.logsumexp(z, 1)
            s["entropy"] = -torch.where(logp > -math.inf, torch.exp(logp) * logp, 0.0).sum(1)
            s["dlogprob"], s["dentropy"] = normal(r) / r, 0.01 * normal(r) / r
    else:
        # the update of a weight: a few strong directions above many weak ones
        n, k = case["batch"], max(1, min(r, c) // 32)
        strong = torch.bmm(normal(n, r, k), normal(n, k, c)) / math.sqrt(k)
        s["x"] = (1e-3 * (strong + 0.3 * normal(n, r, c))).to(kind)
    return s


def prepare(case, seed):
    s = inputs(case, seed)
    if own:
        s["call"] = call(s)
    return s


def call(s):
    """The descriptor, results and workspace that a program keeps, and the call that it makes with them."""
    import paper_1501_06633_b200 as mx

    case, op = s["case"], s["case"]["op"]
    code = {"f32": mx.DTYPE_F32, "bf16": mx.DTYPE_BF16, "f16": mx.DTYPE_F16}[case["type"]]
    kind = TYPES[case["type"]]
    blocks = lambda n: -(-n // BLOCK)  # noqa: E731

    def values(rows, cols, to=E4M3):
        return pitched(torch.zeros(rows, cols, dtype=torch.uint8, device="cuda").view(to))

    def scales(*shape):
        return torch.zeros(*shape, dtype=torch.uint8, device="cuda").view(E8M0)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    r, c = case["rows"], case["cols"]
    if op == "rms_fprop":
        got = {"sum": empty(r, c, dtype=kind)} if case["residual"] else {}
        if case["packed"]:
            got.update(q=values(r, c), sq=scales(blocks(c), r), rstd=empty(r))
            more = dict(packed=(got["q"], got["sq"]), rstd=got["rstd"])
        else:
            got["y"] = empty(r, c, dtype=kind)
            more = dict(y=got["y"])
        d = mx.RmsNormDesc.make(r, c, eps=EPS, x_type=code, ldq=got["q"].stride(0) if case["packed"] else None)
        return lambda: (mx.rms_norm_fprop(d, s["x"], s["gamma"], residual=s.get("r"), sum=got.get("sum"), **more), got)[1]
    if op == "rms_bprop":
        h = s["c"] if case["packed"] else s["x"]
        d = mx.RmsNormDesc.make(r, c, eps=EPS, x_type=mx.DTYPE_E4M3 if case["packed"] else code, y_type=code, ldx=h.stride(0))
        got = {"dx": empty(r, c, dtype=kind), "dgamma": empty(c)}
        ws = empty(max(16, mx.rms_norm_bprop_workspace(d)), dtype=torch.uint8)
        return lambda: (mx.rms_norm_bprop(d, s["dy"], h, s["gamma"], s["rstd"], got["dx"], got["dgamma"], ws, dsum=s.get("dsum"),
                                          h_scale=s.get("sc")), got)[1]
    if op == "lp_fprop":
        got = {"lse": empty(r), "logprob": empty(r), "entropy": empty(r)}
        if case["top"]:
            got.update(top_logprob=empty(r, case["top"]), top_index=empty(r, case["top"], dtype=torch.int32))
        d = mx.LogprobDesc.make(r, c, top=case["top"], scale=case["scale"], x_type=code)
        return lambda: (mx.logprob_fprop(d, s["x"], s["target"], **got), got)[1]
    if op == "lp_bprop":
        if case["packed"]:
            row, col = (values(r, c, E5M2), scales(blocks(c), r)), (values(r, c, E5M2), scales(blocks(r), c))
            got, to = {"q_row": row[0], "s_row": row[1], "q_col": col[0], "s_col": col[1]}, dict(row=row, col=col)
            d = mx.LogprobDesc.make(r, c, scale=case["scale"], x_type=code, ldq=row[0].stride(0))
        else:
            got = to = {"dx": empty(r, c, dtype=kind)}
            d = mx.LogprobDesc.make(r, c, scale=case["scale"], x_type=code)
        return lambda: (mx.logprob_bprop(d, s["x"], s["target"], s["lse"], dlogprob=s["dlogprob"], entropy=s["entropy"],
                                         dentropy=s["dentropy"], **to), got)[1]
    d = mx.OrthoDesc.make(r, c, batch=case["batch"], steps=case["steps"], x_type=code)
    out = empty(case["batch"], r, c, dtype=torch.bfloat16)
    ws = empty(mx.orthogonalise_workspace(d), dtype=torch.uint8)
    return lambda: (mx.orthogonalise(d, s["x"], out, ws, coefficients=(A, B, C)), {"out": out})[1]


def run(s):
    return s["call"]() if own else run_plain(s)


# ---------------------------------------------------------------- 64 bits


def round8(v, to):
    """`v` in 64 bits, rounded to the nearest number of an 8-bit type, ties to even (|v| is in its range)."""
    bits, least = (3, -6) if to == E4M3 else (2, -14)
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=least) - bits)
    return torch.round(v / step) * step


def pack64(x, block, to):
    rows, cols = x.shape
    br, bc = (1, BLOCK) if block == "row" else (BLOCK, 1)
    wide = torch.zeros(-(-rows // br) * br, -(-cols // bc) * bc, dtype=torch.float64, device=x.device)
    wide[:rows, :cols] = x
    most = wide.abs().unflatten(1, (-1, bc)).amax(2).unflatten(0, (-1, br)).amax(1)
    e = torch.ceil(torch.log2(most.clamp(min=1e-300) / LARGEST[to]))
    e = e + (LARGEST[to] * torch.exp2(e) < most).double()  # a logarithm that was rounded down,
    e = e - (LARGEST[to] * torch.exp2(e - 1) >= most).double()  # or up
    scale = torch.where(most == 0, 1.0, torch.exp2(e.clamp(-126, 127)))
    each = scale.repeat_interleave(br, 0).repeat_interleave(bc, 1)[:rows, :cols]
    return round8(x / each, to), scale.t().contiguous() if block == "row" else scale


def exact(case, seed):
    s, op, f64 = inputs(case, seed), case["op"], torch.float64
    if op == "rms_fprop":
        h = s["x"].to(f64)
        got = {}
        if case["residual"]:
            h = got["sum"] = torch.add(h, s["r"].to(f64))
        rstd = (torch.linalg.vector_norm(h, dim=1).square() / h.shape[1] + EPS).rsqrt()
        y = torch.einsum("rc,r,c->rc", h, rstd, s["gamma"].to(f64))
        if not case["packed"]:
            return {**got, "y": y}
        q, sq = pack64(y, "row", E4M3)
        return {**got, "q": q, "sq": sq, "rstd": rstd}
    if op == "rms_bprop":
        if case["packed"]:
            k = torch.kron(s["sc"].to(torch.float32).to(f64).t().contiguous(), torch.ones(1, BLOCK, dtype=f64, device="cuda"))
            h = s["c"].to(torch.float32).to(f64) * k[:, :case["cols"]]
        else:
            h = s["x"].to(f64)
        dy, rstd, gamma = s["dy"].to(f64), s["rstd"].to(f64), s["gamma"].to(f64)
        inner = torch.mv(dy * h, gamma) * rstd ** 3 / h.shape[1]
        dx = torch.addcmul(dy * gamma * rstd[:, None], h, inner[:, None], value=-1)
        if case["residual"]:
            dx += s["dsum"].to(f64)
        return {"dx": dx, "dgamma": torch.einsum("rc,rc,r->c", dy, h, rstd)}
    if op == "lp_fprop":
        x, t = s["x"].to(f64), s["target"]
        logp = torch.log_softmax(x * case["scale"], 1)
        token = (t >= 0) & (t < x.shape[1])
        rows = torch.arange(x.shape[0], device="cuda")
        got = {"lse": torch.logsumexp(x * case["scale"], 1), "logprob": torch.where(token, logp[rows, t.clamp(0, x.shape[1] - 1)], 0.0),
               "entropy": torch.special.entr(torch.exp(logp)).sum(1)}
        if case["top"]:
            v, i = torch.sort(x, dim=1, descending=True, stable=True)
            v, i = v[:, :case["top"]], i[:, :case["top"]]
            got["top_logprob"] = logp.gather(1, i)
            got["top_index"] = i.masked_fill(v == -math.inf, -1).to(torch.int32)
        return got
    if op == "lp_bprop":
        x, t = s["x"].to(f64), s["target"]
        z = (x * case["scale"]).sub_(s["lse"].to(f64)[:, None])
        p = torch.exp(z)
        token = ((t >= 0) & (t < x.shape[1])).to(f64) * s["dlogprob"].to(f64)
        dx = z.nan_to_num_(neginf=0.0).add_(s["entropy"].to(f64)[:, None]).mul_(s["dentropy"].to(f64)[:, None]).add_(token[:, None]).mul_(p).neg_()
        dx[torch.arange(x.shape[0], device="cuda"), t.clamp(0, x.shape[1] - 1)] += token
        dx *= case["scale"]
        if not case["packed"]:
            return {"dx": dx}
        (q, sq), (qc, sc) = pack64(dx, "row", E5M2), pack64(dx, "col", E5M2)
        return {"q_row": q, "s_row": sq, "q_col": qc, "s_col": sc}
    x = s["x"].to(f64)
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + 1e-7)
    eye = torch.eye(min(case["rows"], case["cols"]), dtype=f64, device="cuda")
    for _ in range(case["steps"]):
        if case["rows"] <= case["cols"]:
            gram = torch.einsum("nij,nkj->nik", x, x)
            x = torch.bmm(torch.baddbmm(A * eye + B * gram, gram, gram, alpha=C), x)
        else:
            gram = torch.einsum("nji,njk->nik", x, x)
            x = torch.bmm(x, torch.baddbmm(A * eye + B * gram, gram, gram, alpha=C))
    return {"out": x}
