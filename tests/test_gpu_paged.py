"""The operators of the paged key-value cache against plain implementations in 64 bits: the plan of a step, the append of keys
and values, the attention of one new token.

Tolerances.  Whole numbers are equal.  Rotary embedding: the angle is within pi 2^-24 (rounded to 32 bits within half a turn), cosine
and sine within 2 units of 2^-24 besides, products and sum round three times: 4 + 2 + 2 units of 2^-24 of |x| + |y|, 8e-7 with room
for the float product of a scale.  Attention: see _bound.
"""
import math

import pytest
import torch

from paper_1712_01084_b200 import binding as pb

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"int8": 127.0, "e4m3": 448.0}
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
FLOOR = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}   # half a step among the subnormals
TURN = 8e-7


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


# ------------------------------------------------------------------------------------------------------ plan
def _plan_reference(lengths, added, table, free, taken, page, rows):
    width = len(table[0]) if table else 1
    cap = width * page
    table = [list(r) for r in table]
    slots, positions, starts, out = [], [], [0], []
    total = 0
    for r, (have, add) in enumerate(zip(lengths, added)):
        have, add = min(max(have, 0), cap), max(add, 0)
        end = min(have + add, cap)
        for column in range(-(-have // page), -(-end // page)):
            table[r][column] = free[taken] if 0 <= taken < len(free) else -1
            taken += 1
        total += add
        for position in range(have, have + min(add, max(0, rows - len(slots)))):
            number = table[r][position // page] if position < cap else -1
            slots.append(number * page + position % page if number >= 0 else -1)
            positions.append(position)
        starts.append(min(rows, total))
        out.append(end)
    rest = rows - len(slots)
    return table, slots + [-1] * rest, positions + [0] * rest, starts, out, taken


def _plan_case(seed, requests, width, page, most_have, most_add, rows=None, spare=8, idle=0.2):
    g = torch.Generator().manual_seed(seed)
    draw = lambda low, high, n: torch.randint(low, high + 1, (n,), generator=g).tolist()  # noqa: E731
    lengths, added = draw(0, most_have, requests), draw(0, most_add, requests)
    added = [0 if u < idle else a for u, a in zip(torch.rand(requests, generator=g).tolist(), added)]
    free = torch.randperm(requests * width + spare, generator=g).tolist()
    table, taken = [[-1] * width for _ in range(requests)], 0
    for r in range(requests):
        for c in range(min(width, -(-lengths[r] // page))):
            table[r][c] = free[taken]
            taken += 1
    return lengths, added, table, free, taken, sum(added) if rows is None else rows


def _check_plan(lengths, added, table, free, taken, page, rows, in_place=False, ld=0):
    want = _plan_reference(lengths, added, table, free, taken, page, rows)
    width = len(table[0]) if table else 1
    store = torch.full((len(table), width + ld), 77, dtype=torch.int32, device="cuda")
    t = store[:, :width]
    t.copy_(_ints(table).view(len(table), width))
    out = pb.PagedPlan(len(lengths), rows)
    a, b = _ints(lengths), _ints([taken])
    if in_place:
        out.lengths, out.taken = a, b
    got = pb.pp_paged_plan(a, _ints(added), t, _ints(free), b, page, out=out)
    assert got is out
    assert t.tolist() == want[0] and bool((store[:, width:] == 77).all())
    assert got.slots.tolist() == want[1] and got.positions.tolist() == want[2] and got.starts.tolist() == want[3]
    assert got.lengths.tolist() == want[4] and got.taken.tolist() == [want[5]]
    if not in_place:
        assert a.tolist() == lengths and b.tolist() == [taken]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("requests,width,page,have,add", [(1, 1, 1, 0, 1), (1, 4, 16, 17, 1), (3, 5, 7, 20, 9), (256, 12, 16, 150, 1), (257, 3, 100, 200, 60),
                                                          (1000, 2, 64, 60, 3), (40, 30, 128, 1000, 2000), (8192, 2, 8, 9, 2)])
def test_plan_matches_definition(requests, width, page, have, add, in_place):
    case = _plan_case(requests, requests, width, page, have, add)
    _check_plan(*case[:5], page, case[5], in_place, ld=requests % 3)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_at_its_edges(in_place):
    _check_plan([], [], [], [3, 1], 1, 16, 5, in_place)                                      # no request: rows are nobody's
    _check_plan([0, 0], [0, 0], [[-1], [-1]], [5], 0, 4, 0, in_place)                        # nothing to do, no rows
    _check_plan([0, 3], [4, 2], [[9], [8]], [], 0, 4, 8, in_place)                           # no page to give, and past the capacity
    _check_plan([2, 0, 6], [9, 5, 1], [[4, -1], [-1, -1], [6, 7]], [0, 1, 2, 3], 3, 4, 20, in_place)   # the list ends in between
    _check_plan([-5, 100, 4], [3, -2, 2], [[-1, -1], [1, 2], [3, -1]], list(range(10)), 4, 4, 6, in_place)   # outside the ranges
    _check_plan([1, 1, 1], [700, 800, 900], [[2, -1], [1, -1], [0, -1]], list(range(9)), 3, 8, 1100, in_place)   # fewer rows than tokens
    _check_plan([5], [4], [[-1, -1]], [4, 4], 0, 8, 4, in_place)                             # an old page is missing
    _check_plan([0], [3], [[-1, -1]], [4, 6], -1, 2, 3, in_place)                            # a position before the list


@pytest.mark.gpu
def test_plan_counts_past_32_bits():
    big = 2 ** 31 - 1
    # rows end long before the tokens do
    _check_plan([0, 1, 0], [big, big, 5], [[-1, -1], [0, -1], [-1, -1]], list(range(9)), 1, 4, 1200)
    # slots beyond 2^31: page * page_size
    page = 1 << 20
    p = pb.pp_paged_plan(_ints([3]), _ints([2]), _ints([[5000]]), _ints([0]), _ints([0]), page, rows=2)
    assert p.slots.tolist() == [5000 * page + 3, 5000 * page + 4]


@pytest.mark.gpu
def test_plan_steps_in_a_graph():
    """A captured step that goes on from its own lengths: replays are the steps of a loop."""
    page, width, requests = 4, 6, 3
    free = [7, 3, 9, 1, 0, 2, 4, 5, 6, 8] + list(range(10, 30))
    table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
    plan = pb.PagedPlan(requests, 4)
    plan.lengths.copy_(_ints([0, 3, 8]))
    table.copy_(_ints([[-1] * 6, [7] + [-1] * 5, [3, 9] + [-1] * 4]))
    plan.taken.copy_(_ints([3]))
    added, f = _ints([1, 1, 1]), _ints(free)
    state = ([0, 3, 8], table.tolist(), 3)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pb.pp_paged_plan(plan.lengths, added, table, f, plan.taken, page, out=plan)
    for _ in range(7):
        graph.replay()
        torch.cuda.synchronize()
        t, slots, positions, starts, lengths, taken = _plan_reference(state[0], [1, 1, 1], state[1], free, state[2], page, 4)
        assert table.tolist() == t and plan.slots.tolist() == slots and plan.lengths.tolist() == lengths and plan.taken.tolist() == [taken]
        state = (lengths, t, taken)


@pytest.mark.gpu
def test_plan_refuses_arrays_that_meet():
    a, b, t, f, k = _ints([1, 2]), _ints([1, 1]), _ints([[0], [1]]), _ints([2, 3]), _ints([0])
    for name, other in (("lengths", b), ("taken", a[:1]), ("positions", t.view(-1)), ("lengths", f)):
        out = pb.PagedPlan(2, 2)
        setattr(out, name, other)
        with pytest.raises(pb.PPError, match="INVALID_ARG"):
            pb.pp_paged_plan(a, b, t, f, k, 4, out=out)
    both = torch.zeros(5, dtype=torch.int32, device="cuda")
    out = pb.PagedPlan(2, 2)
    out.starts, out.positions = both[:3], both[2:4]
    with pytest.raises(pb.PPError, match="INVALID_ARG"):
        pb.pp_paged_plan(a, b, t, f, k, 4, out=out)


# ---------------------------------------------------------------------------------------------------- append
def _cache(g, pages, page, heads, dim, kind, heads_first=False, fill=None):
    """(k, v, scales or None twice) with random contents, in views of either order."""
    shape = (pages, heads, page, dim) if heads_first else (pages, page, heads, dim)
    out = []
    for _ in range(2):
        x = torch.randn(shape, generator=g, device="cuda") if fill is None else torch.full(shape, fill, device="cuda")
        x = (x * 40).round().clamp(-127, 127).to(torch.int8) if kind == "int8" else x.to(TYPES[kind])
        out.append(x.transpose(1, 2) if heads_first else x)
    if kind in TOP:
        out += [0.01 + 0.02 * torch.rand(pages, page, heads, generator=g, device="cuda") for _ in range(2)]
    else:
        out += [None, None]
    return out


def _rotated(x, positions, inv_freq, interleaved):
    """Rows in 64 bits, turned, and |x| + |y| of each pair."""
    x = x.double()
    mass = x.abs()
    if inv_freq is None:
        return x, mass
    n = inv_freq.numel()
    angle = (positions.double()[:, None] * inv_freq.double())[:, None]
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., first], x[..., second]
    out, mass = x.clone(), mass.clone()
    out[..., first], out[..., second] = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
    mass[..., first] = mass[..., second] = a.abs() + b.abs()
    return out, mass


def _check_append(c, before, k, v, slots, q, positions, inv_freq, interleaved, q_in, got, kind):
    page = c.page_size
    live = [(t, s) for t, s in enumerate(slots.tolist()) if 0 <= s < c.pages * page]
    tokens = torch.tensor([t for t, _ in live], dtype=torch.long, device="cuda")
    at = torch.tensor([s for _, s in live], dtype=torch.long, device="cuda")
    touched = torch.zeros(c.pages * page, dtype=torch.bool, device="cuda")
    touched[at] = True
    if q is not None:
        want, mass = _rotated(q_in, positions, inv_freq, interleaved)
        bound = (TURN if inv_freq is not None else 0) * mass + ROUND[q.dtype] * want.abs() * (1 + 1e-6) + FLOOR[q.dtype]
        assert bool(((got.double() - want).abs() <= bound).all())
    for x, buffer, old, scales, old_scales, turned in ((k, c.k, before[0], c.k_scales, before[2], True), (v, c.v, before[1], c.v_scales, before[3], False)):
        new = buffer.reshape(c.pages * page, *buffer.shape[2:])
        old = old.reshape(new.shape)
        bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[new.element_size()]
        assert torch.equal(new[~touched].view(bits), old[~touched].view(bits))
        want, mass = _rotated(x, positions, inv_freq if turned else None, interleaved)
        want, mass, have = want[tokens], mass[tokens], new[at].double()
        err = (TURN if turned and inv_freq is not None else 0) * mass
        if kind in TOP:
            s = scales.reshape(c.pages * page, -1)
            assert torch.equal(s[~touched], old_scales.reshape(s.shape)[~touched])
            s = s[at].double()
            top = want.abs().amax(-1)
            assert bool(((s - top / TOP[kind]).abs() <= err.amax(-1) / TOP[kind] + top / TOP[kind] * 2.0 ** -24 * 1.01 + 2.0 ** -149).all())
            value = torch.where(s[..., None] > 0, want / s[..., None].clamp(min=1e-300), 0.0)
            err = err / s[..., None].clamp(min=1e-300) * (s[..., None] > 0) + value.abs() * 2.0 ** -23
            half = 0.5 if kind == "int8" else torch.clamp(value.abs() * 2.0 ** -4, min=2.0 ** -10)
            # an error that carries a value over the border of two steps leaves it within half a step and the error
            assert bool(((have - value).abs() <= half + err * 1.1).all())
        else:
            assert bool(((have - want).abs() <= err + ROUND[new.dtype] * want.abs() * (1 + 1e-6) + FLOOR[new.dtype]).all())


def _append_case(seed, dtype, kind, heads, kv_heads, dim, tokens, pairs, interleaved, page=8, heads_first=False, skip=(), first=0, shift=0):
    g, t = _gen(seed), TYPES[dtype]
    pages = -(-tokens // page) + 2
    k_buf, v_buf, ks, vs = _cache(g, pages, page, kv_heads, dim, kind, heads_first)
    c = pb.PagedCache(k_buf, v_buf, ks, vs)
    before = [None if x is None else x.clone() for x in (k_buf, v_buf, ks, vs)]
    wide = torch.randn(tokens, (heads + 2 * kv_heads) * dim + shift, generator=g, device="cuda").to(t)[:, shift:]
    q, k, v = (p.unflatten(1, (-1, dim)) if p.shape[1] else None for p in wide.split([heads * dim, kv_heads * dim, kv_heads * dim], 1))
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens]
    for i in skip:
        slots[i % tokens] = -1 if i % 2 else pages * page + i
    positions = (first + torch.arange(tokens, device="cuda", dtype=torch.int64) * 37).clamp(max=2 ** 31 - 1).to(torch.int32)
    inv_freq = None
    if pairs:
        inv_freq = (10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float()
    return c, before, q, k, v, slots, positions if pairs else None, inv_freq, interleaved


APPENDS = [(h, g, d, t, p, i, kw) for h, g, d, t, p, i, kw in [
    (4, 1, 64, 1, 32, False, {}), (8, 2, 128, 3, 64, False, {}), (3, 3, 128, 70, 32, True, {"heads_first": True}), (5, 1, 80, 9, 40, False, {}),
    (2, 2, 256, 5, 32, True, {"page": 3}), (2, 1, 96, 17, 0, False, {}), (0, 4, 64, 6, 16, False, {}), (7, 1, 72, 11, 36, False, {"page": 1}),
    (7, 1, 72, 11, 30, True, {}), (2, 1, 1, 4, 0, False, {}), (3, 1, 5, 4, 2, False, {}), (3, 1, 5, 4, 2, True, {}), (2, 2, 33, 8, 16, True, {"shift": 1}),
    (4, 2, 64, 8, 32, False, {"shift": 3}), (64, 8, 128, 300, 64, False, {"first": 1 << 20}), (1, 1, 200, 2, 100, False, {"first": 2 ** 31 - 30})]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "e4m3"), ("f16", "int8"), ("f32", "e4m3"), ("f32", "int8")])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_matches_definition(dtype, kind, case):
    heads, kv, dim, tokens, pairs, interleaved, kw = APPENDS[case]
    c, before, q, k, v, slots, positions, inv_freq, interleaved = _append_case(case, dtype, kind, heads, kv, dim, tokens, pairs, interleaved,
                                                                              skip=(2, 5) if tokens > 5 else (), **kw)
    got = pb.pp_kv_append(c, k, v, slots, q=q, positions=positions, inv_freq=inv_freq, interleaved=interleaved)
    _check_append(c, before, k, v, slots, q, positions, inv_freq, interleaved, q, got, kind)


# from 16 tokens to an SM on a CTA takes several of them: one fewer than that, ragged ends, heads that two CTAs share, no q, no turn
MANY = [(2, 1, 64, 2367, 32, False, {}), (2, 1, 64, 2368, 32, False, {}), (4, 2, 128, 4099, 32, True, {"page": 3}), (1, 1, 72, 16411, 36, False, {"page": 16}),
        (6, 2, 256, 5003, 128, False, {"heads_first": True}), (0, 2, 96, 9001, 48, False, {}), (256, 8, 16, 2500, 8, False, {}), (2, 2, 80, 7001, 0, False, {})]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "int8"), ("f32", "e4m3")])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_append_of_many_tokens(dtype, kind, case):
    heads, kv, dim, tokens, pairs, interleaved, kw = MANY[case]
    c, before, q, k, v, slots, positions, inv_freq, interleaved = _append_case(100 + case, dtype, kind, heads, kv, dim, tokens, pairs, interleaved,
                                                                              skip=(0, 3, 8, tokens - 1), **kw)
    got = pb.pp_kv_append(c, k, v, slots, q=q, positions=positions, inv_freq=inv_freq, interleaved=interleaved)
    _check_append(c, before, k, v, slots, q, positions, inv_freq, interleaved, q, got, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind,dim,shift", [("bf16", "bf16", 128, 0), ("f16", "int8", 96, 0), ("f32", "f32", 10, 1), ("bf16", "e4m3", 64, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_turns_q_in_its_place(dtype, kind, dim, shift, interleaved):
    c, before, q, k, v, slots, positions, inv_freq, _ = _append_case(3, dtype, kind, 6, 2, dim, 21, dim // 2, interleaved, shift=shift)
    q_in, k_in, v_in = q.clone(), k.clone(), v.clone()
    got = pb.pp_kv_append(c, k, v, slots, q=q, positions=positions, inv_freq=inv_freq, interleaved=interleaved, out=q)
    assert got is q and torch.equal(k, k_in) and torch.equal(v, v_in)
    _check_append(c, before, k_in, v_in, slots, q, positions, inv_freq, interleaved, q_in, q, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dim,shift", [(64, 0), (64, 1), (20, 0)])
def test_append_of_rows_that_are_not_finite_or_zero(kind, dim, shift):
    c, before, q, k, v, slots, _, _, _ = _append_case(5, "f32", kind, 2, 2, dim, 6, 0, False, shift=shift)
    k[1, 0, 3], k[2, 1, 5], v[3, 0, 0], k[4, 0], v[4, 1], k[5, 0] = math.nan, math.inf, -math.inf, 0.0, 0.0, 1e-44
    pb.pp_kv_append(c, k, v, slots)
    at = lambda scales, t, h: float(scales.reshape(-1, 2)[slots[t], h])  # noqa: E731
    row = lambda x, t, h: x.reshape(-1, 2, dim)[slots[t], h].float()  # noqa: E731
    for scales, t, h in ((c.k_scales, 1, 0), (c.k_scales, 2, 1), (c.v_scales, 3, 0)):
        assert math.isnan(at(scales, t, h))
    for x, scales, t, h in ((c.k, c.k_scales, 4, 0), (c.v, c.v_scales, 4, 1), (c.k, c.k_scales, 5, 0)):
        assert at(scales, t, h) == 0.0 and bool((row(x, t, h) == 0).all())
    for t, h in ((1, 1), (2, 0), (0, 0)):                                                    # neighbours are untouched by it
        want = k[t, h].double()
        step = 0.5 if kind == "int8" else (want.abs().amax() / at(c.k_scales, t, h) * 2.0 ** -4)
        assert bool(((row(c.k, t, h).double() * at(c.k_scales, t, h) - want).abs() <= step * at(c.k_scales, t, h) * 1.001).all())


@pytest.mark.gpu
def test_append_of_nothing_and_refusals():
    c = pb.PagedCache.empty(2, 4, 2, 16)
    e = torch.empty(0, 2, 16, dtype=torch.bfloat16, device="cuda")
    assert pb.pp_kv_append(c, e, e, _ints([], torch.int64)) is None
    assert pb.pp_kv_append(c, e, e, _ints([], torch.int64), q=e).shape == (0, 2, 16)
    x = torch.randn(3, 2, 16, device="cuda").bfloat16()
    slots, positions, f = _ints([0, 1, 2], torch.int64), _ints([0, 1, 2]), torch.ones(8, device="cuda")
    call = lambda **kw: pb.pp_kv_append(c, **{**dict(k=x, v=x, slots=slots, q=x, positions=positions, inv_freq=f), **kw})  # noqa: E731
    call()
    for kw in ({"k": x[:2]}, {"v": x[:, :1]}, {"slots": slots[:2]}, {"positions": None}, {"inv_freq": None}, {"inv_freq": torch.ones(9, device="cuda")},
               {"inv_freq": f.double()}, {"q": x[:2]}, {"k": x[..., :8]}, {"q": None, "out": x}, {"out": x[:2]}, {"k": x.cpu()}, {"q": x[0]}):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in ({"v": x.float()}, {"q": x.half()}, {"slots": slots.int()}, {"positions": positions.long()}):
        with pytest.raises(TypeError):
            call(**kw)
    h = x.half()
    with pytest.raises(pb.PPError, match="UNSUPPORTED"):                                     # no rounding to another 16-bit type
        call(k=h, v=h, q=h)
    row = torch.randn(3, 8, 16, device="cuda").bfloat16()                                    # out beside q, k and v in their rows
    got = pb.pp_kv_append(c, row[:, 2:4], row[:, 4:6], slots, q=row[:, :2], positions=positions, inv_freq=f, out=row[:, 6:])
    assert torch.equal(got, pb.pp_kv_append(c, row[:, 2:4], row[:, 4:6], slots, q=row[:, :2], positions=positions, inv_freq=f))
    with pytest.raises(pb.PPError, match="INVALID_ARG"):                                     # out across k in its rows
        pb.pp_kv_append(c, row[:, 2:4], row[:, 4:6], slots, q=row[:, :2], positions=positions, inv_freq=f, out=row[:, 3:5])
    wide = torch.zeros(4, 2, 16, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pb.PPError, match="INVALID_ARG"):                                     # out across q
        call(q=wide[:3], out=wide[1:])
    with pytest.raises(pb.PPError, match="INVALID_ARG"):                                     # out across k
        call(k=wide[:3], out=wide[:3])
    with pytest.raises(pb.PPError, match="INVALID_ARG"):                                     # rows of out on one another
        call(out=torch.zeros(1, 2, 16, dtype=torch.bfloat16, device="cuda").expand(3, 2, 16))


# ------------------------------------------------------------------------------------------------- attention
def _attention_case(seed, dtype, kind, heads, kv_heads, dim, page, lengths, heads_first=False, width=None, spread=1.0, order=None):
    """A cache whose unused places hold NaN (8 bits: NaN scales), its table, and q."""
    g, t = _gen(seed), TYPES[dtype]
    held = [-(-n // page) for n in lengths]
    width = max(held + [1]) if width is None else width
    pages = sum(held) + 2
    shape = (pages, heads_first and kv_heads or page, page if heads_first else kv_heads, dim)
    values = [torch.randn(shape, generator=g, device="cuda") * s for s in (spread, 1.0)]
    if heads_first:
        values = [x.transpose(1, 2) for x in values]
    perm = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
    used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    at = 0
    for r, n in enumerate(lengths):
        mine = perm[at:at + held[r]]
        at += held[r]
        if mine:
            table[r, :held[r]] = _ints(mine)
            for i, p in enumerate(mine):
                used[p, :n - i * page] = True
    scales = [None, None]
    if kind in TOP:
        scales = [x.abs().amax(-1) / TOP[kind] * (0.5 + torch.rand(x.shape[:3], generator=g, device="cuda")) for x in values]
        values = [x / s[..., None] for x, s in zip(values, scales)]
        values = [x.round().clamp(-127, 127).to(torch.int8) if kind == "int8" else x.clamp(-448, 448).to(TYPES[kind]) for x in values]
        for s in scales:
            s[~used] = math.nan
        scales = [s.contiguous() for s in scales]
    else:
        values = [x.to(TYPES[kind]) for x in values]
        for x in values:
            x[~used] = math.nan
    q = torch.randn(len(lengths), heads, dim, generator=g, device="cuda").to(t)
    return pb.PagedCache(*values, *scales), q, table, _ints(lengths)


def _attention_reference(c, q, table, lengths, scale, window=0):
    """(out, log of the sum, what the bound is made of) in 64 bits, request by request."""
    heads, g = q.shape[1], c.kv_heads
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    mass, slack = torch.zeros_like(out), torch.zeros_like(lse)
    for r, n in enumerate(lengths.tolist()):
        n = min(max(n, 0), table.shape[1] * c.page_size)
        at = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        number = table[r].long()[at // c.page_size]
        there = (number >= 0) & (number < c.pages)
        at, number = at[there], number[there]
        if not at.numel():
            continue
        k, v = c.k[number, at % c.page_size].double(), c.v[number, at % c.page_size].double()
        if c.k_scales is not None:
            k = k * c.k_scales[number, at % c.page_size].double()[..., None]
            v = v * c.v_scales[number, at % c.page_size].double()[..., None]
        k, v = (x.repeat_interleave(heads // g, 1) for x in (k, v))
        s = torch.einsum("hd,nhd->hn", q[r].double(), k) * scale
        p = torch.softmax(s, 1)
        out[r] = torch.einsum("hn,nhd->hd", p, v)
        mass[r] = torch.einsum("hn,nhd->hd", p, v.abs())
        lse[r] = torch.logsumexp(s, 1)
        most = torch.einsum("hd,nhd->hn", q[r].double().abs(), k.abs()).amax(1) * abs(scale)
        slack[r] = most * (c.head_dim + 8) * 2.0 ** -23 + (s.amax(1) - s.amin(1)) * 2.0 ** -22
    return out, lse, mass, slack


def _bound(out, mass, slack, positions, dtype, kind):
    """A score is a sum of head_dim exact products held in 32 bits, whose additions err by 2^-23 of the largest partial sum at most, and a
    few roundings of the factors; the exponential's argument rounds by 2^-24 of itself; p and the sum of p then err by `slack` and
    2^-21 (exponential, factors of a running maximum), p enters the second product rounded to 16 bits (bf16 caches: 2^-17; else
    less, but for a bf16 output over 8 bits, where it is one f16 number: half a step is 2^-11 of p, and only the numerator has it,
    since the sum of p is taken before: sum |dp v| <= 2^-11 sum p |v|), and a sum over n positions in 32 bits passes at most n / 8 + 600 additions (two instructions a tile of 16; four warps;
    some 300 parts, and their joining).  All errors of p count twice: above and below the fraction."""
    grow = 2 * (slack + 2.0 ** -21 + 2.0 ** -17) + (positions / 8 + 600) * 2.0 ** -23
    if dtype == torch.bfloat16 and kind in (torch.int8, torch.float8_e4m3fn):
        grow = grow + 2.0 ** -11
    return ROUND[dtype] * out.abs() * (1 + 1e-6) + FLOOR[dtype] + grow[..., None] * mass


def _check_attention(c, q, table, lengths, window=0, scale=None, got=None):
    used = 1 / math.sqrt(c.head_dim) if scale is None else scale
    want, lse, mass, slack = _attention_reference(c, q, table, lengths, used, window)
    if got is None:
        got = pb.pp_paged_attention(c, q, table, lengths, window=window, scale=scale, lse=True)
    o, e = got
    assert o.shape == q.shape and o.dtype == q.dtype and e.dtype == torch.float32
    most = float(lengths.max()) if lengths.numel() else 0.0
    most = min(most, window) if window else most
    err, bound = (o.double() - want).abs(), _bound(want, mass, slack, most, q.dtype, c.k.dtype)
    assert bool((err <= bound).all()), float((err / bound).max())
    none = torch.isinf(lse)
    assert torch.equal(torch.isinf(e) & (e < 0), none) and bool((o[none] == 0).all())
    d = (e.double() - lse).abs()[~none]
    assert bool((d <= 2 * slack[~none] + (most / 8 + 600) * 2.0 ** -23 + 2.0 ** -20 + lse[~none].abs() * 2.0 ** -22).all())
    return o


SOME = [0, 1, 15, 16, 17, 63, 64, 65, 130, 500, 1000, 3000]
KINDS = [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "e4m3"), ("f16", "int8"), ("f32", "e4m3"), ("bf16", "int8"), ("f32", "int8")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads,kv_heads,dim,page,heads_first", [
    (8, 1, 128, 16, False), (8, 8, 64, 16, True), (32, 2, 128, 32, False), (6, 2, 96, 1, True), (10, 2, 80, 7, False), (16, 1, 256, 64, False), (4, 4, 192, 128, True),
    (40, 2, 64, 16, False), (5, 1, 72, 100, False), (9, 3, 100, 16, True), (14, 2, 112, 5, False), (2, 1, 33, 16, False), (3, 3, 1, 8, True), (12, 1, 250, 16, False),
    (33, 1, 256, 9, True), (7, 1, 130, 4, False)])
def test_attention_matches_definition(dtype, kind, heads, kv_heads, dim, page, heads_first):
    case = _attention_case(dim + heads, dtype, kind, heads, kv_heads, dim, page, SOME, heads_first)
    _check_attention(*case)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("window", [1, 16, 63, 64, 65, 200, 5000])
def test_attention_windows(dtype, kind, window):
    _check_attention(*_attention_case(window, dtype, kind, 8, 2, 64, 16, SOME), window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("lengths", [[40000], [1], [0], [0, 0, 0], [20000, 1, 1, 30000], [64] * 300, [130] * 700])
def test_attention_over_few_and_many(dtype, kind, lengths):
    _check_attention(*_attention_case(len(lengths), dtype, kind, 8, 2, 64, 16, lengths))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads,kv_heads,dim,page,heads_first", [(8, 4, 128, 16, False), (32, 8, 64, 32, True), (12, 12, 96, 16, False), (80, 4, 64, 8, False), (16, 16, 72, 48, False),
                                                                 (36, 4, 256, 16, False), (12, 6, 64, 16, False)])
def test_attention_long_and_short_at_once(dtype, kind, heads, kv_heads, dim, page, heads_first):
    """Lengths that no even division fits: all heads in a row, cut into equal parts, four heads at a time where their number allows it."""
    case = _attention_case(dim, dtype, kind, heads, kv_heads, dim, page, [9000, 1, 0, 5000, 64, 17000, 333], heads_first, width=17000 // page + 400)
    _check_attention(*case)
    _check_attention(*case, window=3001)
    c, q, table, lengths = case
    got, lse = pb.pp_paged_attention(c, q, table, lengths, lse=True)
    again, lse2 = pb.pp_paged_attention(c, q, table, lengths, lse=True)
    assert torch.equal(got, again) and torch.equal(lse, lse2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
def test_attention_with_large_scores(dtype, kind):
    # one key far above the others, and a scale that makes most p vanish
    c, q, table, lengths = _attention_case(4, dtype, kind, 4, 2, 64, 16, [300, 2000], spread=3.0)
    _check_attention(c, q, table, lengths, scale=1.0)
    _check_attention(c, q, table, lengths, scale=-0.25)
    _check_attention(c, q, table, lengths, scale=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
def test_attention_skips_what_is_no_page(dtype, kind):
    c, q, table, lengths = _attention_case(6, dtype, kind, 8, 2, 64, 8, [300, 40, 16, 700])
    table[0, 3], table[0, 10], table[1, :], table[2, 1], table[3, 40:] = -1, c.pages, -1, 2 ** 31 - 1, -7
    o = _check_attention(c, q, table, lengths)
    assert bool((o[1] == 0).all())


@pytest.mark.gpu
def test_attention_lengths_outside_the_table():
    c, q, table, lengths = _attention_case(7, "bf16", "bf16", 4, 1, 64, 16, [64, 30, 64])
    _check_attention(c, q, table, _ints([1000, -3, 2 ** 31 - 1]))


@pytest.mark.gpu
@pytest.mark.parametrize("kv_heads", [1, 4])
@pytest.mark.parametrize("page", [16, 1])
def test_attention_at_the_end_of_the_longest_table(kv_heads, page):
    """Positions just below 2^31 - 2^13: looking ahead of the last one stays within the numbers."""
    width = (2 ** 31 - 1 - 8192) // page
    if page == 1:
        width = 2 ** 20                                                      # a table of 8 GB is not worth it: the same tail, far from the limit
    c, q, _, _ = _attention_case(15, "bf16", "e4m3", 4 * kv_heads, kv_heads, 64, page, [60])
    c.k_scales.fill_(0.01)
    c.v_scales.fill_(0.02)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    last = -(-60 // page)
    table[0, -last:] = torch.arange(last, dtype=torch.int32, device="cuda")
    n = width * page
    for length, window in ((n, 50), (n - 3, 41), (2 ** 31 - 1, 33)):
        _check_attention(c, q, table, _ints([length]), window=window)
    if page == 16:
        with pytest.raises(pb.PPError, match="UNSUPPORTED"):
            pb.pp_paged_attention(c, q, torch.full((1, 2 ** 27), -1, dtype=torch.int32, device="cuda"), _ints([5]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
def test_attention_hands_on_what_is_not_finite(dtype, kind):
    c, q, table, lengths = _attention_case(8, dtype, kind, 4, 2, 64, 16, [100, 100, 100, 100])
    q[1, 0, 3] = math.nan                                                                    # one head of one request
    if kind in TOP:
        c.v_scales[int(table[2, 1]), 4, 1] = math.nan                                        # one key-value head
    else:
        c.v[int(table[2, 1]), 4, 1, 7] = math.nan
    o = pb.pp_paged_attention(c, q, table, lengths)
    bad = torch.isnan(o)
    assert bool(bad[1, 0].all()) and not bool(bad[0].any()) and not bool(bad[3].any()) and not bool(bad[1, 1:].any()) and not bool(bad[2, :2].any())
    assert bool(bad[2, 2:, 7].all()) and (kind in TOP or int(bad[2].sum()) == 2)


@pytest.mark.gpu
def test_attention_where_every_score_is_minus_infinity():
    c, q, table, lengths = _attention_case(9, "f32", "f32", 2, 1, 64, 16, [100])
    k = c.k.clone()
    k[..., 0] = -math.inf
    c2 = pb.PagedCache(k, c.v)
    q[..., 0] = 1.0
    o, lse = pb.pp_paged_attention(c2, q, table, lengths, lse=True)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("shift", [1, 2, 4, 8])
def test_attention_of_rows_at_any_alignment(dtype, kind, shift):
    """Keys, values and q whose rows start `shift` elements off, keys and values in one tensor."""
    c, q, table, lengths = _attention_case(10, dtype, kind, 6, 2, 64, 16, [70, 1, 333])
    pages, page, g, d = c.k.shape
    both = torch.zeros(pages, 2, page, g, d + 8 + shift, dtype=torch.uint8 if kind == "e4m3" else c.k.dtype, device="cuda")
    both = both.view(c.k.dtype)
    k, v = both[:, 0, :, :, shift:shift + d], both[:, 1, :, :, shift:shift + d]
    k.copy_(c.k)
    v.copy_(c.v)
    row = torch.zeros(q.shape[0], q.shape[1] + 1, d + shift, dtype=q.dtype, device="cuda")[:, 1:, shift:]
    row.copy_(q)
    wide = torch.full((3, table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")[:, :table.shape[1]]
    wide.copy_(table)
    _check_attention(pb.PagedCache(k, v, c.k_scales, c.v_scales), row, wide, lengths)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f16", "int8")])
def test_cache_past_32_bits(dtype, kind):
    """Pages more than 2^32 bytes apart: append to the last, attend over all."""
    d, g, page = 64, 2, 16
    t = TYPES[kind]
    far = 2 ** 32 // t.itemsize + 4096
    pages = 3
    store = torch.empty(((pages - 1) * far + 2 * page * g * d) * t.itemsize, dtype=torch.uint8, device="cuda").view(t)
    strides = (far, g * d, d, 1)
    k = torch.as_strided(store, (pages, page, g, d), strides, 0)
    v = torch.as_strided(store, (pages, page, g, d), strides, page * g * d)
    scales = [torch.ones(pages, page, g, device="cuda") for _ in range(2)] if kind in TOP else [None, None]
    c = pb.PagedCache(k, v, *scales)
    gen = _gen(1)
    x = torch.randn(pages * page, 3 * g, d, generator=gen, device="cuda").to(TYPES[dtype])
    pb.pp_kv_append(c, x[:, :g], x[:, g:2 * g], torch.arange(pages * page, device="cuda"))
    q = torch.randn(1, 4, d, generator=gen, device="cuda").to(TYPES[dtype])
    _check_attention(c, q, _ints([[2, 0, 1]]), _ints([47]))
    if kind not in TOP:
        assert torch.equal(k[2], x[2 * page:, :g])


@pytest.mark.gpu
def test_attention_repeats_bit_for_bit_and_calls_overlap():
    """The same bits alone, on several streams at once, and in two graphs that are replayed at once."""
    case = _attention_case(11, "bf16", "bf16", 32, 8, 128, 16, [5000, 37, 9000, 1])
    other = _attention_case(12, "bf16", "e4m3", 16, 2, 128, 32, [7000, 3])
    want, want2 = pb.pp_paged_attention(*case), pb.pp_paged_attention(*other)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(20):
        with torch.cuda.stream(a):
            got.append((pb.pp_paged_attention(*case), want))
        got.append((pb.pp_paged_attention(*other, stream=b), want2))
        with torch.cuda.stream(b):
            got.append((pb.pp_paged_attention(*case), want))
    graphs = []
    for c, w in ((case, want), (other, want2)):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = pb.pp_paged_attention(*c)
        graphs.append((graph, o, w))
    for _ in range(10):
        for s, (graph, _, _) in zip((a, b), graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for o, w in got + [(o, w) for _, o, w in graphs]:
        assert torch.equal(o, w)


@pytest.mark.gpu
def test_attention_in_a_graph_follows_its_lengths():
    c, q, table, lengths = _attention_case(13, "f16", "f16", 8, 2, 64, 16, [900, 400])
    graph = torch.cuda.CUDAGraph()
    pb.pp_paged_attention(c, q, table, lengths)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = pb.pp_paged_attention(c, q, table, lengths, lse=True)
    for n in ([900, 400], [0, 400], [1, 64], [65, 399]):
        lengths.copy_(_ints(n))
        graph.replay()
        torch.cuda.synchronize()
        _check_attention(c, q, table, lengths, got=got)


@pytest.mark.gpu
def test_attention_refusals():
    c, q, table, lengths = _attention_case(14, "bf16", "bf16", 4, 2, 64, 16, [30, 20])
    call = lambda **kw: pb.pp_paged_attention(c, **{**dict(q=q, table=table, lengths=lengths), **kw})  # noqa: E731
    call(out=torch.empty_like(q))
    for kw in ({"q": q[0]}, {"q": q[:, :3]}, {"q": q[:1]}, {"q": q[..., :32]}, {"table": table[:1]}, {"table": table.t()}, {"lengths": lengths[:1]},
               {"table": table.cpu()}, {"out": torch.empty_like(q)[:1]}, {"out": q.float()}, {"q": q[:, :0]}):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in ({"table": table.long()}, {"lengths": lengths.long()}, {"q": q.to(torch.int8).double()}):
        with pytest.raises(TypeError):
            call(**kw)
    for kw in ({"q": q.half()}, {"q": q.float()}):
        with pytest.raises(pb.PPError, match="UNSUPPORTED"):
            call(**kw)
    for kw in ({"window": -1}, {"scale": math.inf}, {"scale": math.nan}, {"out": q}):
        with pytest.raises(pb.PPError, match="INVALID_ARG"):
            call(**kw)
    e = q[:0]
    assert pb.pp_paged_attention(c, e, table[:0], lengths[:0]).shape == (0, 4, 64)
    o, lse = pb.pp_paged_attention(c, e, table[:0], lengths[:0], lse=True)
    assert lse.shape == (0, 4)


@pytest.mark.gpu
def test_cache_refusals():
    k = torch.zeros(3, 4, 2, 16, dtype=torch.bfloat16, device="cuda")
    v, s = torch.zeros_like(k), torch.ones(3, 4, 2, device="cuda")
    codes = torch.zeros(3, 4, 2, 16, dtype=torch.int8, device="cuda")
    pb.PagedCache(k, v)
    pb.PagedCache(codes, codes.clone(), s, s.clone())
    for args in ((k, v[:2]), (k, v, s, s.clone()), (codes, codes.clone()), (codes, codes.clone(), s, s[:2]), (k, v.float()), (k[..., ::2], v[..., ::2]),
                 (k[0], v[0]), (k[:0], v[:0]), (k, v.cpu())):
        with pytest.raises(ValueError):
            pb.PagedCache(*args)
    with pytest.raises(TypeError):
        pb.PagedCache(k.double(), v.double())
    for args in ((k, k), (k[:1].expand(3, 4, 2, 16), v), (k, v[:, :1].expand(3, 4, 2, 16)), (codes, codes.clone(), s, s)):
        with pytest.raises(pb.PPError, match="INVALID_ARG"):
            pb.PagedCache(*args)
    with pytest.raises(pb.PPError, match="UNSUPPORTED"):
        pb.PagedCache(*(torch.zeros(1, 1, 1, 257, device="cuda") for _ in range(2)))
