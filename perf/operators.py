"""What is measured of the 8-bit training operators: matrix product with block scales, layer
norm, packing of activations, and the gated activation that works from packed activations.

Where `own` is false, `run` computes each operator in its plain form (elementary torch
operations in 32 bits); where it is true, it makes the calls of ``paper_1501_06633_b200``.
`exact` evaluates the definitions in 64 bits.

The 8-bit format.  A matrix is cut into blocks of up to 128 values along a row ("row"), along
a column ("col"), or of 128 x 128 ("tile").  With m the largest finite magnitude of a block and
V the largest number of the 8-bit type (448 for E4M3, 57344 for E5M2), the block's scale is 2^E,
E the least integer with m <= V 2^E (0 for a block of zeros), and its values are x 2^-E rounded
to the type.  Scales are E8M0 bytes, laid out [block][row] for rows, [block][column] for columns,
[row block][column block] for tiles.  Rows of packed values start at multiples of 16 bytes.
"""
import math

import torch

own = False

BLOCK = 128
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": E4M3, "e5m2": E5M2}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "e5m2": 1}
EPS = 1e-5


def listed():
    return [
        # one token of a decoder through a square projection: every weight is read once
        dict(name="gemm8 one token", op="gemm8", way="fprop", tokens=1, inner=4096, outer=4096, grad="e4m3", out="bf16"),
        # a prompt, or a small batch of a training step, through the same projection
        dict(name="gemm8 fprop 2048", op="gemm8", way="fprop", tokens=2048, inner=4096, outer=4096, grad="e4m3", out="bf16"),
        # gradient of the inputs where no size fits a tile: the weights are read as they were stored for the forward pass
        dict(name="gemm8 dgrad ragged", op="gemm8", way="dgrad", tokens=1531, inner=1000, outer=2309, grad="e5m2", out="bf16"),
        # gradient of the weights of a wide layer over a whole training batch: the largest product
        dict(name="gemm8 wgrad 16384", op="gemm8", way="wgrad", tokens=16384, inner=4096, outer=8192, grad="e4m3", out="f32"),
        # three tokens being decoded: nothing but the normalised values is wanted
        dict(name="layer norm 3 tokens", op="ln_fprop", rows=3, cols=2048, type="bf16", packed=False),
        # a training batch: the product's packed operand, the statistics and the packed input for the backward pass
        dict(name="layer norm fprop", op="ln_fprop", rows=8192, cols=4096, type="bf16", packed=True),
        # its backward pass, which has the input only as it was packed
        dict(name="layer norm bprop packed", op="ln_bprop", rows=8192, cols=4096, type="bf16", packed=True),
        # an output gradient, packed once for the input gradient (rows) and once for the weight gradient (columns)
        dict(name="pack rows and columns", op="pack", rows=8192, cols=4096, type="bf16", to="e5m2", blocks="row+col"),
        # the forward pass's operand, packed again along the tokens for the weight gradient; no multiple of 128
        dict(name="repack ragged", op="repack", rows=5000, cols=2056, to="e4m3"),
        # the maps in front of the 5x5 layer (96 channels of 27 x 27, 128 images), unpacked for its filter gradient
        dict(name="unpack maps", op="unpack", rows=96 * 27 * 27, cols=128, type="bf16", to="e4m3"),
        # gated activation of a training batch: operand of the next product, and the packed inputs for the backward pass
        dict(name="act8 fprop", op="act_fprop", rows=8192, cols=4096, act="silu", gated=True, type="bf16", packed=True),
        # its backward pass from packed inputs; columns that end inside a block
        dict(name="act8 bprop packed", op="act_bprop", rows=4097, cols=2736, act="gelu", gated=True, type="bf16", packed=True),
    ]


def draw(rng):
    def size(lo, hi, step=1):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, v // step * step))

    def width(lo, hi):  # widths are mostly multiples of 16, sometimes anything
        return size(lo, hi, rng.choice((1, 16, 16, 128)))

    op = rng.choice(("gemm8", "gemm8", "gemm8", "ln_fprop", "ln_bprop", "pack", "repack", "unpack", "act_fprop", "act_bprop"))
    if op == "gemm8":
        way = rng.choice(("fprop", "dgrad", "wgrad"))
        return dict(op=op, way=way, tokens=size(1, 16384), inner=width(128, 6144), outer=width(128, 8192),
                    grad=rng.choice(("e4m3", "e5m2")), out="f32" if way == "wgrad" else rng.choice(("bf16", "f16", "f32")))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    case = dict(op=op, rows=size(1, 8192), cols=width(128, 4096))
    if op in ("ln_fprop", "ln_bprop"):
        case.update(type=kind, packed=rng.random() < 0.5)
    elif op == "pack":
        case.update(type=kind, to=rng.choice(("e4m3", "e5m2")), blocks=rng.choice(("row", "col", "tile", "row+col")))
    elif op == "repack":
        case.update(to=rng.choice(("e4m3", "e5m2")))
    elif op == "unpack":
        case.update(type=kind, to=rng.choice(("e4m3", "e5m2")))
    else:
        case.update(act=rng.choice(("silu", "gelu", "gelu_tanh")), gated=rng.random() < 0.75, type=kind, packed=rng.random() < 0.7)
    return case


def work(case):
    op = case["op"]
    blocks = lambda n: -(-n // BLOCK)  # noqa: E731
    if op == "gemm8":
        t, i, o = case["tokens"], case["inner"], case["outer"]
        out = {"fprop": t * o, "dgrad": t * i, "wgrad": o * i}[case["way"]] * BYTES[case["out"]]
        read = {"fprop": t * i + o * i, "dgrad": t * o + o * i, "wgrad": t * o + t * i}[case["way"]]
        scales = {"fprop": t * blocks(i) + blocks(o) * blocks(i), "dgrad": t * blocks(o) + blocks(o) * blocks(i),
                  "wgrad": blocks(t) * (o + i)}[case["way"]]
        return {"bytes": read + scales + out, "flops": 2.0 * t * i * o}
    r, c = case["rows"], case["cols"]
    n, scales = r * c, r * blocks(c)
    if op == "ln_fprop":
        e = BYTES[case["type"]]
        return {"bytes": e * n + 8 * c + (2 * n + 2 * scales + 8 * r if case["packed"] else e * n), "flops": 8.0 * n}
    if op == "ln_bprop":
        e = BYTES[case["type"]]
        return {"bytes": 2 * e * n + (n + scales if case["packed"] else e * n) + 8 * r + 12 * c, "flops": 14.0 * n}
    if op == "pack":
        forms = case["blocks"].split("+")
        per = {"row": scales, "col": blocks(r) * c, "tile": blocks(r) * blocks(c)}
        return {"bytes": BYTES[case["type"]] * n + sum(n + per[f] for f in forms), "flops": 3.0 * n * len(forms)}
    if op == "repack":
        return {"bytes": 2 * n + scales + blocks(r) * c, "flops": 4.0 * n}
    if op == "unpack":
        return {"bytes": n + scales + BYTES[case["type"]] * n, "flops": 1.0 * n}
    e, halves = BYTES[case["type"]], 2 if case["gated"] else 1
    if op == "act_fprop":
        return {"bytes": halves * e * n + n + scales + (halves * (n + scales) if case["packed"] else 0), "flops": 12.0 * n}
    return {"bytes": e * n + halves * (n + scales if case["packed"] else e * n) + halves * e * n, "flops": 16.0 * n}


# ---------------------------------------------------------------- the plain form


def cut(x, block):
    """`x` in 32 bits as [row blocks][rows of a block][column blocks][columns of a block], zeros at the ends."""
    rows = 1 if block == "row" else BLOCK
    cols = 1 if block == "col" else BLOCK
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


def spread(scales, block, rows, cols):
    """The scale of each value in 32 bits, as a matrix that broadcasts to [rows][cols]."""
    s = scales.to(torch.float32)
    if block == "row":
        return s.t().repeat_interleave(BLOCK, 1)[:, :cols]
    s = s.repeat_interleave(BLOCK, 0)[:rows]
    return s if block == "col" else s.repeat_interleave(BLOCK, 1)[:, :cols]


def unpack(q, scales, block):
    return q.to(torch.float32) * spread(scales, block, *q.shape)


def act(name, g):
    """The activation and its derivative."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def halves(s, case, packed):
    """Gate and, where there is one, up half of act8's inputs in 32 bits."""
    c, n = case["cols"], -(-case["cols"] // BLOCK)
    if not packed:
        h = s["h"].to(torch.float32)
        return h[:, :c], h[:, c:]
    up = unpack(s["c"][:, c:], s["sc"][n:], "row") if case["gated"] else None
    return unpack(s["c"][:, :c], s["sc"][:n], "row"), up


def run_plain(s):
    case, op, f32 = s["case"], s["case"]["op"], torch.float32
    if op == "gemm8":
        a, b = unpack(s["a"], s["sa"], s["block_a"]), unpack(s["b"], s["sb"], s["block_b"])
        a, b = {"fprop": (a, b.t()), "dgrad": (a, b), "wgrad": (a.t(), b)}[case["way"]]
        return {"c": (a @ b).to(TYPES[case["out"]])}
    if op == "ln_fprop":
        x = s["x"].to(f32)
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        y = d * rstd * s["gamma"] + s["beta"]
        if not case["packed"]:
            return {"y": y.to(s["x"].dtype)}
        q, sq = pack(y, "row", E4M3)
        c, sc = pack(x, "row", E4M3)
        return {"q": q, "sq": sq, "c": c, "sc": sc, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "ln_bprop":
        x = unpack(s["c"], s["sc"], "row") if case["packed"] else s["x"].to(f32)
        dy, rstd = s["dy"].to(f32), s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        g = dy * s["gamma"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    if op == "pack":
        x, got = s["x"].to(f32), {}
        for form in case["blocks"].split("+"):
            got["q_" + form], got["s_" + form] = pack(x, form, TYPES[case["to"]])
        return got
    if op == "repack":
        q, sq = pack(unpack(s["c"], s["sc"], "row"), "col", TYPES[case["to"]])
        return {"q_col": q, "s_col": sq}
    if op == "unpack":
        return {"x": unpack(s["c"], s["sc"], "row").to(TYPES[case["type"]])}
    if op == "act_fprop":
        g, u = halves(s, case, False)
        f, _ = act(case["act"], g)
        q, sq = pack(f * u if case["gated"] else f, "row", E4M3)
        if not case["packed"]:
            return {"q": q, "sq": sq}
        parts = [pack(x, "row", E4M3) for x in ((g, u) if case["gated"] else (g,))]
        c = torch.cat([x.view(torch.uint8) for x, _ in parts], 1).view(E4M3)
        sc = torch.cat([x.view(torch.uint8) for _, x in parts], 0).view(E8M0)
        return {"q": q, "sq": sq, "c": c, "sc": sc}
    g, u = halves(s, case, case["packed"])
    f, df = act(case["act"], g)
    da = s["da"].to(f32)
    dh = torch.cat((da * u * df, da * f), 1) if case["gated"] else da * df
    return {"dh": dh.to(s["da"].dtype)}


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

    def hidden(rows, cols):
        """Activations: a few columns much larger than the rest, rows of different sizes, not quite centred."""
        big = torch.where(torch.rand(cols, device="cuda", generator=gen) < 0.01, 20.0, 1.0)
        return (normal(rows, cols) + 0.1) * big * torch.exp(0.5 * normal(rows, 1))

    def gradient(rows, cols):
        """Gradients: small, and of very different sizes from row to row."""
        return normal(rows, cols) * 1e-4 * torch.exp(normal(rows, 1))

    def packed(x, block, to):
        q, scales = pack(x, block, to)
        return pitched(q), scales

    op, s = case["op"], {"case": case}
    if op == "gemm8":
        t, i, o, way, grad = case["tokens"], case["inner"], case["outer"], case["way"], TYPES[case["grad"]]
        if way == "fprop":
            s["a"], s["sa"] = packed(hidden(t, i), "row", E4M3)
        else:
            s["a"], s["sa"] = packed(gradient(t, o), "row" if way == "dgrad" else "col", grad)
        if way == "wgrad":
            s["b"], s["sb"] = packed(hidden(t, i), "col", E4M3)
        else:
            s["b"], s["sb"] = packed(normal(o, i) * 0.02, "tile", E4M3)
        s["block_a"] = "col" if way == "wgrad" else "row"
        s["block_b"] = "col" if way == "wgrad" else "tile"
        return s
    r, c = case["rows"], case["cols"]
    kind = TYPES.get(case.get("type"))
    if op in ("ln_fprop", "ln_bprop"):
        x = hidden(r, c).to(kind)
        s["gamma"] = 1 + 0.2 * normal(c)
        s["beta"] = 0.1 * normal(c)
        if op == "ln_fprop":
            s["x"] = x
            return s
        x = x.to(torch.float32)
        s["mean"] = x.mean(1)
        s["rstd"] = 1 / torch.sqrt(x.var(1, unbiased=False) + EPS)
        s["dy"] = gradient(r, c).to(kind)
        if case["packed"]:
            s["c"], s["sc"] = packed(x, "row", E4M3)
        else:
            s["x"] = x.to(kind)
    elif op == "pack":
        s["x"] = (gradient(r, c) if case["to"] == "e5m2" else hidden(r, c)).to(kind)
    elif op in ("repack", "unpack"):
        s["c"], s["sc"] = packed(hidden(r, c), "row", TYPES[case["to"]])
    else:
        many = 2 if case["gated"] else 1
        h = (normal(r, many * c) * 1.5).to(kind)
        if op == "act_bprop":
            s["da"] = gradient(r, c).to(kind)
        if op == "act_fprop" or not case["packed"]:
            s["h"] = h
        else:
            parts = [pack(x, "row", E4M3) for x in h.to(torch.float32).split(c, 1)]
            s["c"] = pitched(torch.cat([x.view(torch.uint8) for x, _ in parts], 1).view(E4M3))
            s["sc"] = torch.cat([x.view(torch.uint8) for _, x in parts], 0).view(E8M0)
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
    code = {"f32": mx.DTYPE_F32, "bf16": mx.DTYPE_BF16, "f16": mx.DTYPE_F16, "e4m3": mx.DTYPE_E4M3, "e5m2": mx.DTYPE_E5M2}
    form = {"row": mx.BLOCK_ROW, "col": mx.BLOCK_COL, "tile": mx.BLOCK_TILE}
    blocks = lambda n: -(-n // BLOCK)  # noqa: E731

    def values(rows, cols, to=E4M3):
        return pitched(torch.zeros(rows, cols, dtype=torch.uint8, device="cuda").view(to))

    def scales(*shape):
        return torch.zeros(*shape, dtype=torch.uint8, device="cuda").view(E8M0)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if op == "gemm8":
        t, i, o = case["tokens"], case["inner"], case["outer"]
        m, n, k = {"fprop": (t, o, i), "dgrad": (t, i, o), "wgrad": (o, i, t)}[case["way"]]
        across = {"fprop": (mx.MAJOR_K, mx.MAJOR_K), "dgrad": (mx.MAJOR_K, mx.MAJOR_MN), "wgrad": (mx.MAJOR_MN, mx.MAJOR_MN)}[case["way"]]
        c = empty(m, n, dtype=TYPES[case["out"]])
        d = mx.Gemm8Desc.make(m, n, k, a_type=code["e4m3" if case["way"] == "fprop" else case["grad"]], b_type=mx.DTYPE_E4M3,
                              c_type=code[case["out"]], a_major=across[0], b_major=across[1], a_block=form[s["block_a"]],
                              b_block=form[s["block_b"]], lda=s["a"].stride(0), ldb=s["b"].stride(0), ldc=n)
        return lambda: (mx.gemm8(d, s["a"], s["sa"], s["b"], s["sb"], c), {"c": c})[1]
    r, c = case["rows"], case["cols"]
    kind = TYPES.get(case.get("type"))
    if op == "ln_fprop":
        q = values(r, c)
        d = mx.LayerNormDesc.make(r, c, eps=EPS, x_type=code[case["type"]], ldq=q.stride(0))
        if not case["packed"]:
            y = empty(r, c, dtype=kind)
            return lambda: (mx.layer_norm_fprop(d, s["x"], s["gamma"], s["beta"], y=y), {"y": y})[1]
        got = {"q": q, "sq": scales(blocks(c), r), "c": values(r, c), "sc": scales(blocks(c), r), "mean": empty(r), "rstd": empty(r)}
        return lambda: (mx.layer_norm_fprop(d, s["x"], s["gamma"], s["beta"], mean=got["mean"], rstd=got["rstd"], packed=(q, got["sq"]),
                                            checkpoint=(got["c"], got["sc"])), got)[1]
    if op == "ln_bprop":
        x, sx = (s["c"], s["sc"]) if case["packed"] else (s["x"], None)
        d = mx.LayerNormDesc.make(r, c, eps=EPS, x_type=mx.DTYPE_E4M3 if case["packed"] else code[case["type"]], ldx=x.stride(0),
                                  y_type=code[case["type"]])
        got = {"dx": empty(r, c, dtype=kind), "dgamma": empty(c), "dbeta": empty(c)}
        ws = empty(max(16, mx.layer_norm_bprop_workspace(d)), dtype=torch.uint8)
        return lambda: (mx.layer_norm_bprop(d, s["dy"], x, s["gamma"], s["mean"], s["rstd"], got["dx"], got["dgamma"], got["dbeta"], ws,
                                            x_scale=sx), got)[1]
    if op == "pack":
        forms, got = case["blocks"].split("+"), {}
        size = {"row": (blocks(c), r), "col": (blocks(r), c), "tile": (blocks(r), blocks(c))}
        for f in forms:
            got["q_" + f], got["s_" + f] = values(r, c, TYPES[case["to"]]), scales(*size[f])
        d = mx.Quant8Desc.make(r, c, x_type=code[case["type"]], q_type=code[case["to"]], ldq=got["q_" + forms[0]].stride(0))
        to = {f: (got["q_" + f], got["s_" + f]) for f in forms}
        return lambda: (mx.quant8(d, s["x"], **to), got)[1]
    if op == "repack":
        got = {"q_col": values(r, c, TYPES[case["to"]]), "s_col": scales(blocks(r), c)}
        d = mx.Quant8Desc.make(r, c, x_type=code[case["to"]], q_type=code[case["to"]], ldx=s["c"].stride(0), ldq=got["q_col"].stride(0))
        return lambda: (mx.quant8(d, s["c"], col=(got["q_col"], got["s_col"]), x_scale=s["sc"]), got)[1]
    if op == "unpack":
        x = empty(r, c, dtype=kind)
        d = mx.Quant8Desc.make(r, c, x_type=code[case["type"]], q_type=code[case["to"]], ldq=s["c"].stride(0))
        return lambda: (mx.dequant8(d, s["c"], s["sc"], x, mx.BLOCK_ROW), {"x": x})[1]
    many = 2 if case["gated"] else 1
    kinds = {"silu": mx.ACT_SILU, "gelu": mx.ACT_GELU, "gelu_tanh": mx.ACT_GELU_TANH}
    if op == "act_fprop":
        got = {"q": values(r, c), "sq": scales(blocks(c), r)}
        more = {}
        if case["packed"]:
            got.update(c=values(r, many * c), sc=scales(many * blocks(c), r))
            more = {"checkpoint": (got["c"], got["sc"])}
        d = mx.Act8Desc.make(r, c, act=kinds[case["act"]], gated=case["gated"], x_type=code[case["type"]], ldq=got["q"].stride(0),
                             ldc=got["c"].stride(0) if case["packed"] else None)
        return lambda: (mx.act8_fprop(d, s["h"], packed=(got["q"], got["sq"]), **more), got)[1]
    dh = empty(r, many * c, dtype=kind)
    h, sh = (s["c"], s["sc"]) if case["packed"] else (s["h"], None)
    d = mx.Act8Desc.make(r, c, act=kinds[case["act"]], gated=case["gated"], x_type=code[case["type"]],
                         h_type=mx.DTYPE_E4M3 if case["packed"] else None, ldc=h.stride(0) if case["packed"] else None)
    return lambda: (mx.act8_bprop(d, s["da"], h, dh, h_scale=sh), {"dh": dh})[1]


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
    br, bc = {"row": (1, BLOCK), "col": (BLOCK, 1), "tile": (BLOCK, BLOCK)}[block]
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

    def values(q, scales, block):
        x = q.to(torch.float32).to(f64)
        k = scales.to(torch.float32).to(f64)
        k = k.t() if block == "row" else k
        k = k if block == "row" else k.repeat_interleave(BLOCK, 0)[:x.shape[0]]
        return x * (k if block == "col" else k.repeat_interleave(BLOCK, 1)[:, :x.shape[1]])

    if op == "gemm8":
        a, b = values(s["a"], s["sa"], s["block_a"]), values(s["b"], s["sb"], s["block_b"])
        return {"c": torch.einsum({"fprop": "ti,oi->to", "dgrad": "to,oi->ti", "wgrad": "to,ti->oi"}[case["way"]], a, b)}
    if op == "ln_fprop":
        x = s["x"].to(f64)
        mean, var = x.mean(1), x.var(1, unbiased=False)
        rstd = (var + EPS).rsqrt()
        y = torch.addcmul(s["beta"].to(f64), (x - mean[:, None]) * rstd[:, None], s["gamma"].to(f64))
        if not case["packed"]:
            return {"y": y}
        (q, sq), (c, sc) = pack64(y, "row", E4M3), pack64(x, "row", E4M3)
        return {"q": q, "sq": sq, "c": c, "sc": sc, "mean": mean, "rstd": rstd}
    if op == "ln_bprop":
        x = values(s["c"], s["sc"], "row") if case["packed"] else s["x"].to(f64)
        dy, gamma, rstd = s["dy"].to(f64), s["gamma"].to(f64), s["rstd"].to(f64)
        xh = (x - s["mean"].to(f64)[:, None]) * rstd[:, None]
        s1 = torch.mv(dy, gamma) / x.shape[1]
        s2 = torch.mv(dy * xh, gamma) / x.shape[1]
        dx = (dy * gamma - s1[:, None] - xh * s2[:, None]) * rstd[:, None]
        return {"dx": dx, "dgamma": torch.einsum("rc,rc->c", dy, xh), "dbeta": dy.sum(0)}
    if op == "pack":
        got = {}
        for form in case["blocks"].split("+"):
            got["q_" + form], got["s_" + form] = pack64(s["x"].to(f64), form, TYPES[case["to"]])
        return got
    if op == "repack":
        q, sq = pack64(values(s["c"], s["sc"], "row"), "col", TYPES[case["to"]])
        return {"q_col": q, "s_col": sq}
    if op == "unpack":
        return {"x": values(s["c"], s["sc"], "row")}

    def f_df(g):
        if case["act"] == "silu":
            s = torch.sigmoid(g)
            return g * s, s + g * s * torch.sigmoid(-g)
        if case["act"] == "gelu":
            p = torch.special.ndtr(g)
            return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        z = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)  # (1 + tanh(z / 2)) / 2 is the sigmoid of z
        p = torch.sigmoid(z)
        return g * p, p + g * p * torch.sigmoid(-z) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)

    c, n, gated = case["cols"], -(-case["cols"] // BLOCK), case["gated"]
    if op == "act_fprop":
        h = s["h"].to(f64)
        f = f_df(h[:, :c])[0]
        q, sq = pack64(f * h[:, c:] if gated else f, "row", E4M3)
        if not case["packed"]:
            return {"q": q, "sq": sq}
        parts = [pack64(x, "row", E4M3) for x in h.split(c, 1)]
        return {"q": q, "sq": sq, "c": torch.cat([x for x, _ in parts], 1), "sc": torch.cat([x for _, x in parts], 0)}
    if case["packed"]:
        h = torch.cat([values(s["c"][:, k * c:(k + 1) * c], s["sc"][k * n:(k + 1) * n], "row") for k in range(2 if gated else 1)], 1)
    else:
        h = s["h"].to(f64)
    f, df = f_df(h[:, :c])
    da = s["da"].to(f64)
    return {"dh": torch.cat((da * df * h[:, c:], da * f), 1) if gated else da * df}
