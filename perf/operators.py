"""Timing cases of the library's decoder operators: the normalisation that hands its rows on in 8 bits, the
products with 4-bit weights, and the mixture-of-experts layer.

``run`` computes them in plain torch operations while ``own`` is false, and through the library's binding while it
is true.  Sizes are those of the repository's own layers (1000, 1024, 2048, 4096, 8192, 9216) and generic ones.
"""
import math

import torch

own = False

F = torch.float32
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8,
         "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "int8": 1, "e4m3": 1}
TOP = {"int8": 127.0, "e4m3": 448.0}
EPS = 1e-6


def _binding():
    from paper_1712_01084_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------- cases
def listed():
    norm = dict(op="norm8", dtype="bf16", codes="e4m3", group=0)
    q4 = dict(op="q4", group=128, zeros=False, x="bf16", y="f32", batch=1)
    moe = dict(op="moe", weights="bf16", x="bf16", y="bf16", group=128)
    return [
        # one decoding step of one sequence: all latency
        dict(norm, name="norm8 1x4096", rows=1, cols=4096),
        # a decoding step of a small batch, integer codes with a scale per 128 columns
        dict(norm, name="norm8 33x9216 int8", rows=33, cols=9216, dtype="f16", codes="int8", group=128),
        # a prompt of 2,000 odd tokens, a width that leaves rows off the 16-byte boundary
        dict(norm, name="norm8 2047x4095", rows=2047, cols=4095, dtype="f16", group=128),
        # a batch of prompts: all bandwidth
        dict(norm, name="norm8 8192x8192", rows=8192, cols=8192),
        # the output layer of the repository's chain in 4 bits: rows that fill no whole tile, fine groups
        dict(q4, name="q4 1000x4096", rows=1000, cols=4096, group=32, x="f16"),
        # the chain's first layer for eight vectors, zero points, wide x
        dict(q4, name="q4 4096x9216 b8", rows=4096, cols=9216, group=64, zeros=True, batch=8, y="bf16"),
        # a projection fed by the norm's 8-bit rows
        dict(q4, name="q4 4096x4096 e4m3", rows=4096, cols=4096, x="e4m3", y="bf16"),
        # the repository's largest layer, one vector
        dict(q4, name="q4 8192x8192", rows=8192, cols=8192, x="f16"),
        # the same for a batch that takes two column tiles, exact float input
        dict(q4, name="q4 8192x8192 b16 f32", rows=8192, cols=8192, x="f32", zeros=True, batch=16),
        # a small layer of eight experts, one token
        dict(moe, name="moe e8k2 1024 t1", experts=8, top_k=2, cols=1024, inner=1024, tokens=1),
        # fine-grained experts in 4 bits, a small batch of single tokens
        dict(moe, name="moe e64k8 2048 t4 q4", experts=64, top_k=8, cols=2048, inner=1024, tokens=4, weights="q4"),
        # wide experts, a batch that reaches most of them
        dict(moe, name="moe e64k8 4096 t16", experts=64, top_k=8, cols=4096, inner=2048, tokens=16),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    """A length on a logarithmic scale: mostly multiples of 64, one in four any whole number."""
    n = _log(rng, low, high)
    n = n if rng.random() < 0.25 else min(high, max(low, 64 * round(n / 64)))
    return n if n % 1024 or n in (1024, 2048, 4096, 8192, 9216) else n - 64


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("norm8", "q4", "moe"))
        if op == "norm8":
            c = dict(op=op, rows=_log(rng, 1, 8192), cols=_size(rng, 256, 9216), dtype=rng.choice(("bf16", "f16", "f32")),
                     codes=rng.choice(("e4m3", "e4m3", "int8")), group=rng.choice((0, 128)))
        elif op == "q4":
            c = dict(op=op, rows=_size(rng, 512, 9216), cols=_size(rng, 512, 9216), group=rng.choice((32, 64, 128, 128, 256, 0)),
                     zeros=rng.random() < 0.5, x=rng.choice(("f16", "bf16", "f32", "int8", "e4m3")),
                     y=rng.choice(("f32", "f16", "bf16")), batch=_log(rng, 1, 16))
        else:
            c = dict(op=op, experts=rng.choice((4, 8, 16, 32, 60, 64)), top_k=rng.randint(1, 8), cols=_size(rng, 512, 4096),
                     inner=_size(rng, 256, 2048), tokens=_log(rng, 1, 16), weights=rng.choice(("bf16", "f16", "q4")),
                     group=128, x="bf16", y=rng.choice(("bf16", "f32")))
            if c["weights"] == "f16":
                c["x"] = "f16"
            if c["top_k"] > c["experts"] // 2:
                continue
        if _cost(c) <= most:
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _groups(c):
    return -(-c["cols"] // c["group"]) if c["group"] else 1


def _weight_bytes(rows, cols, kind, group, zeros):
    if kind != "q4":
        return rows * cols * 2
    return rows * cols / 2 + rows * -(-cols // (group or cols)) * (2.5 if zeros else 2)


def work(c):
    if c["op"] == "norm8":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (3 * SIZE[c["dtype"]] + 1) + c["cols"] * SIZE[c["dtype"]] + c["rows"] * _groups(c) * 4,
                "flops": 8 * n}
    if c["op"] == "q4":
        m, n, b = c["rows"], c["cols"], c["batch"]
        return {"bytes": _weight_bytes(m, n, "q4", c["group"], c["zeros"]) + b * n * SIZE[c["x"]] + b * m * SIZE[c["y"]],
                "flops": 2 * m * n * b}
    e, k, h, f, t = c["experts"], c["top_k"], c["cols"], c["inner"], c["tokens"]
    used = e * (1 - (1 - k / e) ** t)  # experts that t tokens reach, on average
    one = _weight_bytes(2 * f, h, c["weights"], c["group"], False) + _weight_bytes(h, f, c["weights"], c["group"], False)
    return {"bytes": used * one + e * h * 2 + t * h * (2 + SIZE[c["y"]]), "flops": 2 * t * (k * 3 * f * h + e * h)}


# ------------------------------------------------------------------------------------------------ inputs
def _quantised(w, group, zeros):
    """4-bit codes (two to a byte, the even column in the low half), f16 scales and zero points of rounded weights."""
    rows, cols = w.shape
    g = group or cols
    n = -(-cols // g)
    v = torch.nn.functional.pad(w, (0, n * g - cols)).view(rows, n, g)
    if zeros:
        low, high = v.amin(2).clamp(max=0), v.amax(2).clamp(min=0)
        s = ((high - low) / 15).clamp(min=1e-6).half()
        z = (-low / s.float()).round().clamp(0, 15)
    else:
        s = (v.abs().amax(2) / 7.5).clamp(min=1e-6).half()
        z = torch.full_like(s, 8.0, dtype=F)
    q = (v / s.float()[..., None] + z[..., None]).round_().clamp_(0, 15).to(torch.uint8).view(rows, n * g)[:, :cols]
    if cols % 2:
        q = torch.nn.functional.pad(q, (0, 1))
    return (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), s, z.to(torch.uint8) if zeros else None


def _activations(shape, gen, dtype):
    """Hidden states: unit scale, a few channels that stand out."""
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * (1 + 7 * (torch.rand(shape[-1], generator=gen, device="cuda") > 0.99))).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    s = dict(case)
    if case["op"] == "norm8":
        t = TYPES[case["dtype"]]
        s["x"], s["r"] = _activations((case["rows"], case["cols"]), gen, t), _activations((case["rows"], case["cols"]), gen, t)
        s["w"] = (1 + 0.2 * normal(case["cols"])).to(t)
    elif case["op"] == "q4":
        m, n = case["rows"], case["cols"]
        s["codes"], s["scales"], s["points"] = _quantised(normal(m, n) / math.sqrt(n), case["group"], case["zeros"])
        s["bias"] = 0.1 * normal(m)
        x = _activations((case["batch"], n), gen, F)
        s["x_scales"] = None
        if case["x"] in TOP:
            s["x_scales"] = (x.abs().amax(1) / TOP[case["x"]]).contiguous()
            x = x / s["x_scales"][:, None]
            x = x.round().to(torch.int8) if case["x"] == "int8" else x.to(torch.float8_e4m3fn)
        s["x"] = x.to(TYPES[case["x"]])
        if own:
            s["layer"] = _binding().Q4Layer(m, n, case["group"], s.pop("codes"), s.pop("scales"), s.pop("points"), s.pop("bias"))
    else:
        e, h, f = case["experts"], case["cols"], case["inner"]
        t = TYPES["f16" if case["weights"] == "f16" else "bf16"]
        s["x"] = _activations((case["tokens"], h), gen, TYPES[case["x"]])
        s["router"] = (normal(e, h) / math.sqrt(h)).to(t)
        up, down = [], []
        for _ in range(e):
            a, b = normal(2 * f, h) / math.sqrt(h), normal(h, f) / math.sqrt(f)
            q4 = case["weights"] == "q4"
            up.append(_quantised(a, case["group"], False)[:2] if q4 else (a.to(t),))
            down.append(_quantised(b, case["group"], False)[:2] if q4 else (b.to(t),))
        s["up"], s["down"] = ([torch.stack(p) for p in zip(*w)] for w in (up, down))
        if own:
            make = _binding().MoELayer.q4 if case["weights"] == "q4" else _binding().MoELayer
            more = {"group": case["group"]} if case["weights"] == "q4" else {}
            s["layer"] = make(s.pop("router"), *s.pop("up"), *s.pop("down"), inner=f, top_k=case["top_k"], max_tokens=case["tokens"], **more)
    return s


# ----------------------------------------------------------------------------------------- the operators
def _norm8(s):
    h = s["x"].to(F) + s["r"].to(F)
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["w"].to(F)
    rows, cols = n.shape
    g = s["group"] or cols
    k = -(-cols // g)
    v = torch.nn.functional.pad(n, (0, k * g - cols)).view(rows, k, g)
    scales = v.abs().amax(2) / TOP[s["codes"]]
    v = v / torch.where(scales > 0, scales, 1.0)[..., None]
    v = v.view(rows, k * g)[:, :cols]
    codes = v.round().to(torch.int8) if s["codes"] == "int8" else v.to(torch.float8_e4m3fn)
    return codes, scales, h.to(s["x"].dtype)


def _unpacked(codes, cols):
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return q[..., :cols].to(F)


def _floats(codes, scales, points, group, cols):
    """The weights that 4-bit codes stand for."""
    g = group or cols
    spread = lambda v: v.to(F).repeat_interleave(g, -1)[..., :cols]  # noqa: E731
    return (_unpacked(codes, cols) - (8.0 if points is None else spread(points))) * spread(scales)


def _q4(s):
    x = s["x"].to(F)
    if s["x_scales"] is not None:
        x = x * s["x_scales"][:, None]
    w = _floats(s["codes"], s["scales"], s["points"], s["group"], s["cols"])
    return (x @ w.T + s["bias"]).to(TYPES[s["y"]])


def _moe(s):
    x, k = s["x"].to(F), s["top_k"]
    p = torch.softmax(x @ s["router"].to(F).T, 1)
    p, picked = torch.sort(p, dim=1, descending=True, stable=True)
    p, picked = p[:, :k], picked[:, :k]
    p = p / p.sum(1, keepdim=True)
    of = lambda w, cols: (_floats(*(v[picked] for v in w), None, s["group"], cols) if len(w) == 2 else w[0][picked].to(F))  # noqa: E731
    gu = torch.matmul(of(s["up"], s["cols"]), x[:, None, :, None]).squeeze(-1)
    gate, up = gu.split(s["inner"], -1)
    a = gate / (1 + torch.exp(-gate)) * up
    y = torch.matmul(of(s["down"], s["inner"]), a[..., None]).squeeze(-1)
    return (y * p[..., None]).sum(1).to(TYPES[s["y"]])


def run(s):
    if s["op"] == "norm8":
        if own:
            codes, scales, hidden = _binding().pp_rmsnorm_q8(s["x"], s["w"], residual=s["r"], eps=EPS, codes=s["codes"], group=s["group"])
        else:
            codes, scales, hidden = _norm8(s)
        # 8-bit integers are returned as the values they stand for, in units of their scale
        return {"codes": codes.to(torch.float16) if s["codes"] == "int8" else codes, "scales": scales, "hidden": hidden}
    if s["op"] == "q4":
        if own:
            return _binding().pp_q4_forward(s["layer"], s["x"], x_scales=s["x_scales"], out_dtype=TYPES[s["y"]])
        return _q4(s)
    if own:
        return _binding().pp_moe_forward(s["layer"], s["x"], out_dtype=TYPES[s["y"]])
    return _moe(s)


# ---------------------------------------------------------------------------- the definitions in 64 bits
def _exact_weights(w, e, rows, cols, group):
    """Expert e's matrix in 64 bits: element by element from its code, its scale and the middle code 8."""
    if len(w) == 1:
        return w[0][e].double()
    column = torch.arange(cols, device="cuda")
    code = (w[0][e].int()[:, column // 2] >> (4 * (column % 2))) & 15
    return (code - 8).double() * w[1][e].double()[:, column // (group or cols)]


def exact(case, seed):
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    x = s["x"].double()
    if case["op"] == "norm8":
        h = x + s["r"].double()
        n = h / (h.pow(2).sum(1, keepdim=True) / case["cols"] + EPS).sqrt() * s["w"].double()
        g = case["group"] or case["cols"]
        parts = n.abs().split(g, 1)
        scales = torch.stack([p.max(1).values for p in parts], 1) / TOP[case["codes"]]
        # the codes stand for n / scale: that value itself, which no 8 bits can hold
        codes = torch.cat([p / scales[:, i:i + 1] for i, p in enumerate(n.split(g, 1))], 1)
        return {"codes": codes, "scales": scales, "hidden": h}
    if case["op"] == "q4":
        n, g = case["cols"], case["group"] or case["cols"]
        if s["x_scales"] is not None:
            x = x * s["x_scales"].double()[:, None]
        y = s["bias"].double().expand(case["batch"], -1).clone()
        for i, lo in enumerate(range(0, n, g)):  # group after group
            column = torch.arange(lo, min(n, lo + g), device="cuda")
            code = ((s["codes"].int()[:, column // 2] >> (4 * (column % 2))) & 15).double()
            z = 8.0 if s["points"] is None else s["points"][:, i:i + 1].double()
            y += (x[:, column] @ (code - z).T) * s["scales"][:, i].double()
        return y
    e, h, f, k = case["experts"], case["cols"], case["inner"], case["top_k"]
    logits = torch.einsum("th,eh->te", x, s["router"].double())
    y = torch.zeros_like(x)
    logits = logits.cpu().tolist()
    ranked = [sorted(range(e), key=lambda i, row=row: (-row[i], i))[:k] for row in logits]
    for i in range(e):
        rows = [t for t, r in enumerate(ranked) if i in r]
        if not rows:
            continue
        up = x[rows] @ _exact_weights(s["up"], i, 2 * f, h, case["group"]).T
        act = up[:, :f] * torch.sigmoid(up[:, :f]) * up[:, f:]
        down = act @ _exact_weights(s["down"], i, h, f, case["group"]).T
        for j, t in enumerate(rows):
            share = math.exp(logits[t][i]) / sum(math.exp(logits[t][m]) for m in ranked[t])
            y[t] += share * down[j]
    return y
