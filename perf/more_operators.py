"""Timing cases of the library's paged-cache operators: the plan of a step (block tables and slots from request lengths), the
append of new keys and values (with rotary embedding) to the cache, and the attention of one new token over it.

``run`` computes them in plain torch operations while ``own`` is false, and through the library's binding while it is
true.  Head counts, widths and lengths are generic ones.
"""
import math

import torch

own = False

F = torch.float32
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8,
         "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "int8": 1, "e4m3": 1}
TOP = {"int8": 127.0, "e4m3": 448.0}
THETA = 500000.0


def _binding():
    from paper_1712_01084_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------- cases
def listed():
    # lengths (plan, attention) are drawn from half of `length` to `length`; heads are those of queries
    plan = dict(op="plan", new=1)
    append = dict(op="append", dtype="bf16", cache="bf16", heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False,
                  page=16, heads_first=False)
    attn = dict(op="attn", dtype="bf16", cache="bf16", heads=32, kv_heads=8, dim=128, page=16, heads_first=False, window=0)
    return [
        # one sequence, one token: all latency
        dict(plan, name="plan b1", batch=1, length=4000, width=512, page=16),
        # a decoding step of a full batch
        dict(plan, name="plan b256", batch=256, length=8000, width=512, page=16),
        # prompts of a batch that is being filled, pieces of up to 8,000 tokens
        dict(plan, name="plan b48 prompts", batch=48, length=2000, width=160, page=64, new=8000),
        # one decoding step of one sequence: all latency
        dict(append, name="append 1", tokens=1),
        # a decoding step of a batch into an 8-bit cache
        dict(append, name="append 64 e4m3", tokens=64, cache="e4m3", heads=64, page=64),
        # a prompt of odd length, wide heads of which a quarter turns, neighbouring pairs, pages head by head
        dict(append, name="append 4095 f16 d256", tokens=4095, dtype="f16", cache="f16", heads=16, kv_heads=2, dim=256, rotary=64,
             interleaved=True, page=32, heads_first=True),
        # prompts of a batch: all bandwidth
        dict(append, name="append 16384", tokens=16384, heads=64),
        # one sequence at its beginning: all latency
        dict(attn, name="attn b1 513", batch=1, length=513),
        # exact numbers, a key-value head for each query head, short sequences
        dict(attn, name="attn b6 1000 f32 d64", batch=6, length=1000, dtype="f32", cache="f32", heads=16, kv_heads=16, dim=64),
        # one long sequence: the cache's length is all there is to split
        dict(attn, name="attn b1 131072", batch=1, length=131072),
        # a serving batch with an 8-bit cache
        dict(attn, name="attn b33 12000 e4m3", batch=33, length=12000, cache="e4m3", heads=64, page=64, heads_first=True),
        # a serving batch: all bandwidth
        dict(attn, name="attn b64 8192", batch=64, length=8192, page=32),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("plan", "append", "attn")}
    while True:
        op = rng.choice(("plan", "append", "attn", "attn"))
        page = rng.choice((1, 8, 16, 16, 32, 64, 100, 128))
        if op == "plan":
            c = dict(op=op, batch=_log(rng, 1, 1024), length=_log(rng, 1, 32768), page=page, new=rng.choice((1, 1, _log(rng, 1, 8192))))
            c["width"] = -(-(c["length"] + c["new"]) // page) + rng.randint(0, 7)
            if c["batch"] * c["width"] > 1 << 20 or c["batch"] * c["new"] > 400000:
                continue
        else:
            kv = rng.choice((1, 2, 4, 8, 8, 16))
            group = rng.choice((1, 2, 4, 5, 7, 8, 16))
            dim = rng.choice((64, 72, 80, 96, 128, 128, 192, 256))
            dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
            c = dict(op=op, dtype=dtype, cache=rng.choice((dtype, dtype, "e4m3", "int8")), heads=kv * group, kv_heads=kv, dim=dim,
                     page=page, heads_first=rng.random() < 0.5)
            if kv * group > 128:
                continue
            if op == "append":
                c.update(tokens=_log(rng, 1, 16384), rotary=rng.choice((dim, dim, 32)), interleaved=rng.random() < 0.5)
            else:
                c.update(batch=_log(rng, 1, 256), length=_log(rng, 1, 131072), window=rng.choice((0, 0, 0, 1000)))
                if c["batch"] * c["length"] * kv * dim > 1 << 29:     # values a cache holds of keys
                    continue
        if _cost(c) <= most[op]:
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def work(c):
    if c["op"] == "plan":
        added = c["batch"] * (c["new"] + 1) / 2 if c["new"] > 1 else c["batch"]
        return {"bytes": c["batch"] * 16 + added * 12 + added / c["page"] * 8, "flops": 4 * added}
    el, stored = SIZE[c["dtype"]], c["dim"] * SIZE[c["cache"]] + (4 if c["cache"] in TOP else 0)
    if c["op"] == "append":
        return {"bytes": c["tokens"] * ((2 * c["heads"] + 2 * c["kv_heads"]) * c["dim"] * el + 2 * c["kv_heads"] * stored + 12),
                "flops": 3 * c["tokens"] * (c["heads"] + c["kv_heads"]) * c["rotary"]}
    mean = c["length"] * (1 + 0.75 * (c["batch"] - 1)) / c["batch"]        # the first is `length` long
    if c["window"]:
        mean = min(mean, c["window"])
    return {"bytes": c["batch"] * (mean * 2 * c["kv_heads"] * stored + 2 * c["heads"] * c["dim"] * el + mean / c["page"] * 4),
            "flops": c["batch"] * mean * 4 * c["heads"] * c["dim"]}


# ------------------------------------------------------------------------------------------------ inputs
def _between(gen, low, high, shape):
    return torch.randint(low, high + 1, shape, generator=gen, device="cuda", dtype=torch.int32)


def _stored(values, kind):
    """Rows of values as the cache holds them: rounded, or codes with a scale per row."""
    if kind not in TOP:
        return values.to(TYPES[kind]), None
    scales = values.abs().amax(-1).to(F) / TOP[kind]
    codes = values.to(F) / torch.where(scales > 0, scales, 1.0)[..., None]
    return (codes.round().to(torch.int8) if kind == "int8" else codes.to(TYPES[kind])), scales


def _pages(case, gen, count):
    """A cache of `count` pages that other requests have used before: (k, v, their scales), token by token or head by head."""
    page, h, d = case["page"], case["kv_heads"], case["dim"]
    shape = (count, h, page, d) if case["heads_first"] else (count, page, h, d)
    out, scales = [], []
    for _ in range(2):
        if case["cache"] in TOP:
            codes = torch.empty(shape, dtype=TYPES[case["cache"]], device="cuda")
            sc = torch.empty(count, page, h, device="cuda")
            step = max(1, (1 << 26) // (page * h * d))
            for i in range(0, count, step):
                part = torch.randn((min(step, count - i),) + shape[1:], generator=gen, device="cuda", dtype=torch.float16)
                q, s = _stored(part, case["cache"])
                codes[i:i + step] = q
                sc[i:i + step] = s.transpose(1, 2) if case["heads_first"] else s
            out.append(codes)
            scales.append(sc)
        else:
            out.append(torch.randn(shape, generator=gen, device="cuda", dtype=TYPES[case["cache"]]))
            scales.append(None)
    if case["heads_first"]:
        out = [t.transpose(1, 2) for t in out]
    return out + scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    page = case["page"]
    if case["op"] == "plan":
        b, w = case["batch"], case["width"]
        s["lengths"] = _between(gen, case["length"] // 2, case["length"], (b,))
        s["added"] = _between(gen, 1, case["new"], (b,))
        order = torch.randperm(b * w + 64, generator=gen, device="cuda").to(torch.int32)
        held = -(-s["lengths"] // page)
        column = torch.arange(w, device="cuda", dtype=torch.int32)
        before = torch.cumsum(held, 0, dtype=torch.int32) - held
        s["table"] = torch.where(column < held[:, None], order[(before[:, None] + column).clamp(max=b * w).long()], -1).contiguous()
        s["free"], s["taken"] = order, held.sum(dtype=torch.int32).reshape(1)
        s["rows"] = -(-b * case["new"] // 8) * 8           # a multiple of 8, as programs pad their steps
        if own:
            s["plan"] = _binding().PagedPlan(b, s["rows"])
    elif case["op"] == "append":
        n, h, g, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        t = TYPES[case["dtype"]]
        # the three in one row, as one projection hands them on; a few channels of the keys stand out
        qkv = torch.randn(n, (h + 2 * g) * d, generator=gen, device="cuda")
        qkv[:, h * d:(h + g) * d] *= 1 + 7 * (torch.rand(g * d, generator=gen, device="cuda") > 0.98)
        qkv = qkv.to(t)
        s["q"], s["k"], s["v"] = (p.unflatten(1, (-1, d)) for p in qkv.split([h * d, g * d, g * d], 1))
        count = -(-n // page) + 3
        s["cache_k"], s["cache_v"], s["scales_k"], s["scales_v"] = _pages(case, gen, count)
        order = torch.randperm(count, generator=gen, device="cuda")
        slots = (order[:, None] * page + torch.arange(page, device="cuda")).flatten()[:n].clone()
        rest = n // 50                                     # a padded step: the last rows are nobody's
        if rest:
            slots[-rest:] = -1
        s["slots"] = slots
        first = _between(gen, 0, 1 << 20, (1,))
        s["positions"] = first + torch.arange(n, device="cuda", dtype=torch.int32) % 4096
        s["inv_freq"] = (THETA ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])).to(F).cuda()
        if own:
            s["paged"] = _binding().PagedCache(s["cache_k"], s["cache_v"], s["scales_k"], s["scales_v"])
    else:
        b, h, d = case["batch"], case["heads"], case["dim"]
        lengths = _between(gen, max(1, case["length"] // 2), case["length"], (b,))
        lengths[0] = case["length"]
        width = -(-case["length"] // page)
        held = -(-lengths // page)
        count = int(held.sum()) + 2
        s["cache_k"], s["cache_v"], s["scales_k"], s["scales_v"] = _pages(case, gen, count)
        order = torch.randperm(count, generator=gen, device="cuda").to(torch.int32)
        column = torch.arange(width, device="cuda", dtype=torch.int32)
        before = torch.cumsum(held, 0, dtype=torch.int32) - held
        at = (before[:, None] + column).clamp(max=count - 1).long()
        s["table"] = torch.where(column < held[:, None], order[at], -1).contiguous()
        s["lengths"] = lengths
        s["q"] = (1.5 * torch.randn(b, h, d, generator=gen, device="cuda")).to(TYPES[case["dtype"]])
        if own:
            s["paged"] = _binding().PagedCache(s["cache_k"], s["cache_v"], s["scales_k"], s["scales_v"])
    return s


# ----------------------------------------------------------------------------------------- the operators
def _plan(s):
    page, rows, table = s["page"], s["rows"], s["table"]
    b, w = table.shape
    have = s["lengths"].clamp(0, w * page)
    add = s["added"].clamp(min=0)
    total = torch.minimum(have + add, torch.full_like(have, w * page))
    first, last = (have + page - 1) // page, (total + page - 1) // page
    need = last - first
    base = torch.cumsum(need, 0, dtype=torch.int32) - need
    column = torch.arange(w, device=table.device, dtype=torch.int32)
    new = (column >= first[:, None]) & (column < last[:, None])
    at = s["taken"] + base[:, None] + column - first[:, None]
    there = (at >= 0) & (at < s["free"].numel())
    given = torch.where(there, s["free"][torch.where(there, at, 0).long()], -1)
    table.copy_(torch.where(new, given, table))
    ends = torch.cumsum(add, 0, dtype=torch.int32)
    starts = torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=rows)
    row = torch.arange(rows, device=table.device, dtype=torch.int32)
    of = torch.searchsorted(ends, row, right=True)
    mine = of < b
    of = of.clamp(max=b - 1)
    position = have[of] + row - (ends - add)[of]
    column = position // page
    inside = mine & (column < w)
    number = table.view(-1)[of * w + column.clamp(max=w - 1)].long()
    slots = torch.where(inside & (number >= 0), number * page + position % page, -1)
    return {"table": table, "slots": slots, "positions": torch.where(mine, position, 0), "starts": starts, "lengths": total,
            "taken": s["taken"] + need.sum(dtype=torch.int32)}


def _turned(x, angle, interleaved):
    """Rows x [tokens][heads][dim] in 32 bits with the pairs of their first dimensions turned by angle [tokens][pairs]."""
    r = 2 * angle.shape[1]
    cos, sin = angle.cos().to(F)[:, None], angle.sin().to(F)[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    pair = (a * cos - b * sin, a * sin + b * cos)
    turned = torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)
    return torch.cat([turned, x[..., r:]], -1)


def _append(s):
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    q = _turned(s["q"].to(F), angle, s["interleaved"]).to(s["q"].dtype)
    rows = (_turned(s["k"].to(F), angle, s["interleaved"]), s["v"].to(F))
    count = s["cache_k"].shape[0] * s["page"]
    live = s["slots"] >= 0
    # a slot that nobody writes gets back what it holds
    owner = torch.full((count + 1,), -1, device="cuda", dtype=torch.long)
    owner[torch.where(live, s["slots"], count)] = torch.arange(s["tokens"], device="cuda")
    owner = owner[:count].view(-1, s["page"])
    written = owner >= 0
    owner = owner.clamp(min=0)
    for x, name in zip(rows, "kv"):
        codes, scales = _stored(x, s["cache"])
        for values, buffer in ((codes, s["cache_" + name]), (scales, s["scales_" + name])):
            if values is None:
                continue
            mask = written.reshape(written.shape + (1,) * (buffer.dim() - 2))
            if buffer.dtype == torch.float8_e4m3fn:        # no selection of 8-bit floats: by their bits
                buffer.view(torch.uint8).copy_(torch.where(mask, values.view(torch.uint8)[owner], buffer.view(torch.uint8)))
            else:
                buffer.copy_(torch.where(mask, values[owner], buffer))
    return q


def _attn(s):
    page, table, lengths = s["page"], s["table"], s["lengths"]
    b, w = table.shape
    g = s["kv_heads"]
    heads, d = s["q"].shape[1:]
    position = torch.arange(w * page, device=table.device)
    out = torch.empty_like(s["q"])
    step = max(1, (1 << 28) // (w * page * g * d))
    for i in range(0, b, step):
        number = table[i:i + step].clamp(min=0).long()
        n = number.shape[0]
        inside = position < lengths[i:i + step, None]
        if s["window"]:
            inside &= position >= lengths[i:i + step, None] - s["window"]
        held = []
        for name in ("k", "v"):
            x = s["cache_" + name][number].to(F)
            if s["scales_" + name] is not None:
                x *= s["scales_" + name][number][..., None]
            held.append(x.reshape(n, w * page, g, d))
        k, v = held
        q = s["q"][i:i + step].to(F).view(n, g, heads // g, d)
        score = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
        score.masked_fill_(~inside[:, None, None], -math.inf)
        score -= score.amax(-1, keepdim=True)
        p = torch.exp(score)
        p /= p.sum(-1, keepdim=True)
        v.masked_fill_(~inside[:, :, None, None], 0.0)
        out[i:i + step] = torch.matmul(p, v.permute(0, 2, 1, 3)).view(n, heads, d).to(out.dtype)
    return out


def _cache_values(kind, k, v, scales_k, scales_v):
    """What a cache holds, the 8-bit integers as the values they stand for (in units of their scale)."""
    k, v = (t.to(torch.float16) if kind == "int8" else t for t in (k, v))
    out = {"cache_k": k, "cache_v": v}
    if kind in TOP:
        out.update(scales_k=scales_k, scales_v=scales_v)
    return out


def run(s):
    if s["op"] == "plan":
        if not own:
            return _plan(s)
        p = _binding().pp_paged_plan(s["lengths"], s["added"], s["table"], s["free"], s["taken"], s["page"], out=s["plan"])
        return {"table": s["table"], "slots": p.slots, "positions": p.positions, "starts": p.starts, "lengths": p.lengths, "taken": p.taken}
    if s["op"] == "append":
        if own:
            q = _binding().pp_kv_append(s["paged"], s["k"], s["v"], s["slots"], q=s["q"], positions=s["positions"],
                                        inv_freq=s["inv_freq"], interleaved=s["interleaved"])
        else:
            q = _append(s)
        return {"q": q, **_cache_values(s["cache"], s["cache_k"], s["cache_v"], s["scales_k"], s["scales_v"])}
    if own:
        return _binding().pp_paged_attention(s["paged"], s["q"], s["table"], s["lengths"], window=s["window"])
    return _attn(s)


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    page = case["page"]
    if case["op"] == "plan":
        return _exact_plan(s)
    if case["op"] == "append":
        return _exact_append(s, case["cache"])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["lengths"].tolist()):
        low = max(0, n - case["window"]) if case["window"] else 0
        at = torch.arange(low, n, device="cuda")
        number, offset = s["table"][r].long()[at // page], at % page
        for g in range(case["kv_heads"]):                  # head after head: a long sequence in 64 bits is large
            k, v = (s[name][number, offset, g].double() for name in ("cache_k", "cache_v"))
            if case["cache"] in TOP:
                k, v = k * s["scales_k"][number, offset, g].double()[:, None], v * s["scales_v"][number, offset, g].double()[:, None]
            of = slice(g * case["heads"] // case["kv_heads"], (g + 1) * case["heads"] // case["kv_heads"])
            score = (s["q"][r, of].double() @ k.T) * case["dim"] ** -0.5
            out[r, of] = torch.softmax(score, 1) @ v
    return out


def _exact_plan(s):
    page, rows = s["page"], s["rows"]
    table, free, taken = s["table"].tolist(), s["free"].tolist(), int(s["taken"])
    slots, positions, starts, lengths = [], [], [0], []
    for r, (have, add) in enumerate(zip(s["lengths"].tolist(), s["added"].tolist())):
        for position in range(have, have + add):
            column = position // page
            if position % page == 0 and column < len(table[r]):
                table[r][column] = free[taken] if taken < len(free) else -1
                taken += 1
            number = table[r][column] if column < len(table[r]) else -1
            slots.append(number * page + position % page if number >= 0 else -1)
            positions.append(position)
        starts.append(min(rows, len(positions)))
        lengths.append(min(have + add, page * len(table[r])))
    slots, positions = slots[:rows], positions[:rows]
    slots, positions = slots + [-1] * (rows - len(slots)), positions + [0] * (rows - len(positions))
    of = lambda x, t: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    return {"table": of(table, torch.int32), "slots": of(slots, torch.int64), "positions": of(positions, torch.int32),
            "starts": of(starts, torch.int32), "lengths": of(lengths, torch.int32), "taken": of([taken], torch.int32)}


def _exact_append(s, kind):
    half = s["rotary"] // 2
    turn = torch.exp(1j * s["positions"].double()[:, None] * s["inv_freq"].double()[None])[:, None]

    def rotate(x):
        x = x.double().clone()
        first = slice(0, 2 * half, 2) if s["interleaved"] else slice(0, half)
        second = slice(1, 2 * half, 2) if s["interleaved"] else slice(half, 2 * half)
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    live = torch.nonzero(s["slots"] >= 0)[:, 0]
    number, offset = s["slots"][live] // s["page"], s["slots"][live] % s["page"]
    out = {"q": rotate(s["q"])}
    for name, x in (("k", rotate(s["k"])), ("v", s["v"].double())):
        x = x[live]
        cache = s["cache_" + name].double()
        if kind in TOP:
            scales = s["scales_" + name].double()
            top = x.abs().max(-1).values / TOP[kind]
            scales[number, offset] = top
            # the codes stand for x / scale: that value itself, which no 8 bits can hold
            x = x / torch.where(top > 0, top, 1.0)[..., None]
            out["scales_" + name] = scales
        cache[number, offset] = x
        out["cache_" + name] = None if kind == "int8" else cache           # integers: rounded or not, no value between
    return {k: out[k] for k in ("q", "cache_k", "cache_v", "scales_k", "scales_v") if k in out}
