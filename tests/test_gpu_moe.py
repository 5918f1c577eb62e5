"""The mixture-of-experts layer against its definition in 64 bits.

Tolerances.  Gate and up are sums of exact products in fp32, within 1e-5 of sum |w x| (the library's tolerance for fp32
layers, see the 4-bit products).  silu(g) u then errs by at most 1.1 |dg| |u| + |silu(g)| |du| (|silu'| < 1.1) and a few
fp32 roundings, the chosen weights p by the logits' error (2e-6 of sum |r x|, sums of a hundred fp32 additions per lane at
most) and expf; the down product carries that through |D| and adds 1e-5 of its own.  The bound is evaluated in 64 bits
element by element.  A result in f16 or bf16 is rounded once more.
"""
import pytest
import torch

from paper_1712_01084_b200 import binding as pb

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _codes(g, E, rows, cols, group, zeros):
    q = torch.randint(0, 16, (E, rows, cols), generator=g, device="cuda", dtype=torch.uint8)
    n = -(-cols // group) if group else 1
    s = ((0.5 + torch.rand(E, rows, n, generator=g, device="cuda")) * 0.2 / cols ** 0.5).half()
    z = torch.randint(5, 11, (E, rows, n), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    p = torch.nn.functional.pad(q, (0, cols % 2))
    col = torch.arange(cols, device="cuda") // (group or cols)
    w = (q.double() - (z.double()[..., col] if zeros else 8.0)) * s.double()[..., col]
    return (p[..., 0::2] | (p[..., 1::2] << 4)).contiguous(), s, z, w


class Case:
    """A layer and its weights in 64 bits."""

    def __init__(self, seed, E, k, H, F, weights, max_tokens, group=128, zeros=False, renorm=True):
        g = _gen(seed)
        self.E, self.k, self.H, self.F, self.renorm = E, k, H, F, renorm
        r = torch.randn(E, H, generator=g, device="cuda") / H ** 0.5
        r = r if weights == "q4" else r.to(TYPES[weights])
        self.r = r.double()
        more = dict(inner=F, top_k=k, max_tokens=max_tokens, renormalize=renorm)
        if weights == "q4":
            uc, us, uz, self.u = _codes(g, E, 2 * F, H, group, zeros)
            dc, ds, dz, self.d = _codes(g, E, H, F, group, zeros)
            self.layer = pb.MoELayer.q4(r, uc, us, dc, ds, uz, dz, group=group, **more)
        else:
            u = (torch.randn(E, 2 * F, H, generator=g, device="cuda") / H ** 0.5).to(TYPES[weights])
            d = (torch.randn(E, H, F, generator=g, device="cuda") / F ** 0.5).to(TYPES[weights])
            self.u, self.d = u.double(), d.double()
            self.layer = pb.MoELayer(r, u, d, **more)

    def reference(self, x):
        """y, its error bound, and the routing, in 64 bits."""
        x = x.double()
        logits = x @ self.r.T
        e_logit = 2e-6 * (x.abs() @ self.r.abs().T).amax(1)
        order = torch.argsort(logits, dim=1, descending=True, stable=True)[:, :self.k]
        p = torch.softmax(logits, 1)
        p = torch.gather(p, 1, order)
        if self.renorm:
            p = p / p.sum(1, keepdim=True)
        y, bound = torch.zeros_like(x), torch.zeros_like(x)
        for t in range(x.shape[0]):
            for j in range(self.k):
                e, pj = int(order[t, j]), p[t, j]
                gu, mass = self.u[e] @ x[t], 1e-5 * (self.u[e].abs() @ x[t].abs())
                g, u, dg, du = gu[:self.F], gu[self.F:], mass[:self.F], mass[self.F:]
                silu = g * torch.sigmoid(g)
                act = pj * silu * u
                d_act = pj * (1.1 * dg * u.abs() + (silu.abs() + 1.1 * dg) * du) + act.abs() * (2 * e_logit[t] + 4e-6)
                D = self.d[e]
                y[t] += D @ act
                bound[t] += D.abs() @ (d_act + 1e-5 * act.abs() + 3e-11)
        return y, bound, order, p

    def check(self, x, out_dtype=None):
        y, ids, gates = pb.pp_moe_forward(self.layer, x, out_dtype=out_dtype, routing=True)
        x = x.reshape(-1, self.H)
        want, bound, order, p = self.reference(x)
        assert torch.equal(ids.long(), order)
        assert bool(((gates.double() - p).abs() <= p * (4e-6 * (x.double().abs() @ self.r.abs().T).amax(1, keepdim=True) + 4e-6)).all())
        err = (y.double() - want).abs()
        full = bound + ROUND[y.dtype] * (want.abs() + bound) * 1.001 + (2.0 ** -24 if y.dtype == torch.float16 else 1e-30)
        assert bool((err <= full).all()), float((err / full).max())
        assert self.layer.status() == pb.PP_OK
        return y


@pytest.mark.gpu
@pytest.mark.parametrize("weights,xt", [("bf16", "bf16"), ("bf16", "f16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "bf16"), ("f16", "f32"),
                                        ("q4", "bf16"), ("q4", "f16"), ("q4", "f32")])
@pytest.mark.parametrize("E,k,H,F", [(1, 1, 1, 1), (4, 2, 64, 32), (8, 2, 256, 96), (5, 5, 130, 33), (16, 3, 1000, 129), (64, 8, 512, 256)])
def test_moe_matches_definition(weights, xt, E, k, H, F):
    c = Case(E * 100 + H, E, k, H, F, weights, 8, renorm=E != 8)
    for T in (1, 2, 8):
        x = torch.randn(T, H, generator=_gen(T), device="cuda").to(TYPES[xt])
        c.check(x, torch.float32)
        c.check(x)


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "q4"])
@pytest.mark.parametrize("T", [1, 3, 5, 6, 11, 16, 31, 32])
@pytest.mark.parametrize("E,k", [(2, 1), (2, 2), (40, 6), (256, 16)])
def test_moe_token_counts(weights, T, E, k):
    """Experts with no token, with one, and with more than one pass takes."""
    c = Case(T + E, E, k, 192, 64, weights, 32)
    x = torch.randn(T, 192, generator=_gen(T), device="cuda").bfloat16()
    y = c.check(x, torch.float32)
    assert torch.equal(y, pb.pp_moe_forward(c.layer, x, out_dtype=torch.float32))     # the same bits every time


@pytest.mark.gpu
@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, False), (64, True), (128, True), (256, False), (0, False), (0, True)])
def test_moe_four_bit_groups(group, zeros):
    c = Case(group + zeros, 6, 2, 700, 301, "q4", 4, group=group, zeros=zeros)
    c.check(torch.randn(3, 700, generator=_gen(1), device="cuda").half(), torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "f16", "q4"])
def test_moe_larger(weights):
    c = Case(3, 16, 4, 2048, 1024, weights, 16)
    for T in (1, 7, 16):
        c.check(torch.randn(T, 2048, generator=_gen(T), device="cuda").bfloat16(), torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("weights,E,k,H,F,T", [
    ("bf16", 2, 1, 4096, 80, 1),         # 10 strips of 128 units: every strip on several CTAs
    ("f16", 2, 2, 4096, 1000, 1),        # 250 strips: one and a half to a CTA
    ("bf16", 4, 2, 2800, 600, 3),        # 88 units to a strip, just more than a join costs; several tokens
    ("f16", 16, 4, 4100, 200, 16),       # two tiles of columns, a last unit of four columns
    ("q4", 2, 1, 11008, 80, 1),          # 86 units of 128 columns
    ("q4", 8, 2, 11000, 72, 5),
    ("bf16", 2, 2, 4096, 14336, 1)])     # wide experts of an ordinary size: 3,584 strips, 32 over
def test_moe_strips_of_gate_and_up_that_several_ctas_share(weights, E, k, H, F, T):
    c = Case(E * H + F, E, k, H, F, weights, T)
    x = torch.randn(T, H, generator=_gen(T), device="cuda").bfloat16()
    y = c.check(x, torch.float32)
    for _ in range(3):
        assert torch.equal(y, pb.pp_moe_forward(c.layer, x, out_dtype=torch.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "f16", "q4"])
def test_moe_strides_and_alignment(weights):
    c = Case(5, 8, 2, 333, 80, weights, 4)
    big = torch.randn(4, 1000, generator=_gen(2), device="cuda").bfloat16()
    for off in (0, 1, 4, 7):
        c.check(big[:, off:off + 333], torch.float32)
    c.check(big[0, :333], torch.float32)                                    # one token as a vector


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "f16", "q4"])
def test_moe_range_of_inputs(weights):
    c = Case(6, 8, 2, 256, 64, weights, 4)
    x = torch.randn(4, 256, generator=_gen(3), device="cuda").bfloat16()
    x[0] *= 1000.0
    x[1] *= 0.05
    x[2] = 0.0
    y = c.check(x, torch.float32)
    assert bool((y[2] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 6])
@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_moe_four_bit_tokens_with_elements_that_stand_out(xt, T):
    """Elements of a token ten thousand times the rest where router, gate and up have zeros: the tolerance is the rest's."""
    E, k, H, F = 4, 2, 512, 64
    g = _gen(13)
    out = torch.arange(60, H, 128, device="cuda")
    c = object.__new__(Case)
    c.E, c.k, c.H, c.F, c.renorm = E, k, H, F, True
    r = torch.randn(E, H, generator=g, device="cuda") / H ** 0.5
    r[:, out] = 0.0
    uc, us, _, c.u = _codes(g, E, 2 * F, H, 128, False)
    uc[..., out // 2] = (uc[..., out // 2] & 0xF0) | 0x08                     # even columns: the low half, the zero point 8
    c.u[..., out] = 0.0
    dc, ds, _, c.d = _codes(g, E, H, F, 128, False)
    c.r = r.double()
    c.layer = pb.MoELayer.q4(r, uc, us, dc, ds, group=128, inner=F, top_k=k, max_tokens=T)
    x = torch.randn(T, H, generator=g, device="cuda")
    x[:, out] = 1e4 * (1 + torch.rand(T, len(out), generator=g, device="cuda"))
    c.check(x.to(TYPES[xt]), torch.float32)


@pytest.mark.gpu
def test_moe_ties_go_to_the_lowest_index():
    E, H = 12, 64
    r = torch.zeros(E, H, device="cuda")
    r[:, 0] = torch.tensor([0, 3, 1, 3, 3, 1, 0, 3, 2, 2, 1, 0.0], device="cuda")
    w = torch.zeros(E, 64, H, device="cuda").bfloat16()
    L = pb.MoELayer(r, w, torch.zeros(E, H, 32, device="cuda").bfloat16(), inner=32, top_k=6, max_tokens=2)
    x = torch.zeros(2, H, device="cuda")
    x[0, 0] = 1.0                                                           # the second token: every logit is 0
    _, ids, gates = pb.pp_moe_forward(L, x, routing=True)
    assert ids.tolist() == [[1, 3, 4, 7, 8, 9], [0, 1, 2, 3, 4, 5]]
    assert float((gates[1] - 1 / 6).abs().max()) < 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("weights,xt", [("bf16", "f32"), ("f16", "f32"), ("f16", "bf16"), ("q4", "f32"), ("q4", "bf16")])
@pytest.mark.parametrize("T", [1, 16])
def test_moe_tokens_of_any_size(weights, xt, T):
    """Tokens from 1e-15 to 1e15 in one call: act goes from 1e-30 to 1e30, far out of binary16 on both sides.  One expert, so
    that its weight is 1.  act enters the down products with an absolute error of at most 2^-59 |x|^2 |G row| |U row|."""
    c = Case(14, 1, 1, 320, 72, weights, T)
    u, d = c.u[0], c.d[0]
    scales = torch.logspace(-15, 15, 16, device="cuda")
    for i in range(0, 16, T):
        x = (torch.randn(T, c.H, generator=_gen(i), device="cuda") * scales[i:i + T, None]).to(TYPES[xt])
        y, x = pb.pp_moe_forward(c.layer, x, out_dtype=torch.float32).double(), x.double()
        gu, mass = x @ u.T, 1e-5 * (x.abs() @ u.abs().T)
        g, v, dg, dv = gu[:, :c.F], gu[:, c.F:], mass[:, :c.F], mass[:, c.F:]
        silu = g * torch.sigmoid(g)
        act = silu * v
        d_act = 1.1 * dg * v.abs() + (silu.abs() + 1.1 * dg) * dv + act.abs() * 1.4e-5
        norms = u.norm(dim=1)
        floor = 2.0 ** -59 * (x * x).sum(1, keepdim=True) * norms[:c.F].max() * norms[c.F:].max()
        err, bound = (y - act @ d.T).abs(), (d_act + floor) @ d.abs().T
        assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.gpu
def test_moe_act_bound_leaves_out_rows_that_are_not_finite():
    """An infinite weight in one expert must not cost the others their bits."""
    c = Case(15, 4, 1, 256, 64, "f16", 4)
    g = _gen(15)
    r = torch.randn(4, 256, generator=g, device="cuda") / 16
    r[3] = 0.0
    u, d = (c.u.clone().half(), c.d.half())
    u[3, 5, 7], u[3, 64 + 9, 3] = float("inf"), float("nan")
    x = torch.randn(4, 256, generator=g, device="cuda").half()
    r[3] = -100 * x[0].float()                                               # never chosen by any token like the first
    x = x[:1].expand(4, -1).contiguous()
    c.r, c.u, c.d = r.half().double(), u.double(), d.double()
    c.layer = pb.MoELayer(r.half(), u, d, inner=64, top_k=1, max_tokens=4)
    c.check(x, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "q4"])
def test_moe_not_finite_tokens_stay_alone(weights):
    c = Case(7, 8, 2, 256, 64, weights, 4)
    x = torch.randn(4, 256, generator=_gen(4), device="cuda")
    good = x[[0, 3]].clone()
    x[1, 9] = float("nan")
    x[2, 200] = float("inf")
    y, ids, _ = pb.pp_moe_forward(c.layer, x, routing=True)
    assert int(ids.min()) >= 0 and int(ids.max()) < 8
    assert not bool(torch.isfinite(y[1]).any()) and not bool(torch.isfinite(y[2]).any())
    want, bound, _, _ = c.reference(good)
    assert bool(((y[[0, 3]].double() - want).abs() <= bound).all())


@pytest.mark.gpu
def test_moe_sequence_stream_and_graph():
    c = Case(8, 16, 4, 512, 128, "bf16", 4)
    x0 = torch.randn(2, 512, generator=_gen(5), device="cuda").bfloat16()

    def chain(x):
        for _ in range(20):
            x = pb.pp_moe_forward(c.layer, x)
        return x

    want = chain(x0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = chain(x0)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    xs = x0.clone()
    with torch.cuda.graph(graph):
        z = chain(xs)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(z, want) and c.layer.status() == pb.PP_OK


@pytest.mark.gpu
def test_moe_grid_wait_runs_out():
    """A barrier limit of one poll: the kernel gives up, says so and ends by itself; then it works again."""
    c = Case(9, 16, 4, 2048, 256, "bf16", 16)
    x = torch.randn(16, 2048, generator=_gen(6), device="cuda").bfloat16()
    pb.pp_set_tuning(15, 1)
    try:
        raised = 0
        for _ in range(20):
            pb.pp_moe_forward(c.layer, x)
            raised += c.layer.status() == 7
        assert raised > 0
    finally:
        pb.pp_set_tuning(15, 0)
    assert c.layer.status() == pb.PP_OK
    c.check(x, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("E,k,H,F,T", [(2, 1, 4096, 80, 1),       # step 1 is cut inside strips: 10 of 128 units
                                       (256, 16, 192, 64, 32)],   # step 2: 12 strips of about 440 units
                         ids=["gate_up", "down"])
def test_moe_recovers_after_a_wait_ran_out_at_divided_strips(E, k, H, F, T):
    """A CTA that gave up never arrives at the strips it shares; the next call must not count those that did."""
    c = Case(E + H, E, k, H, F, "bf16", T)
    x = torch.randn(T, H, generator=_gen(12), device="cuda").bfloat16()
    want = c.check(x, torch.float32)
    raised = 0
    for polls in (1, 2, 3, 4, 6, 8, 12, 16, 24, 32):
        pb.pp_set_tuning(15, polls)
        try:
            for _ in range(4):
                pb.pp_moe_forward(c.layer, x, out_dtype=torch.float32)
                raised += c.layer.status() == 7
        finally:
            pb.pp_set_tuning(15, 0)
        for _ in range(3):
            assert torch.equal(pb.pp_moe_forward(c.layer, x, out_dtype=torch.float32), want)
        assert c.layer.status() == pb.PP_OK
    assert raised > 0
    c.check(x, torch.float32)


@pytest.mark.gpu
def test_moe_refusals():
    E, H, F = 4, 64, 32
    r = torch.zeros(E, H, device="cuda")
    u, d = torch.zeros(E, 2 * F, H, device="cuda").half(), torch.zeros(E, H, F, device="cuda").half()
    ok = dict(inner=F, top_k=2, max_tokens=4)
    for bad, status in ((dict(top_k=5), 1), (dict(top_k=0), 1), (dict(max_tokens=0), 1), (dict(max_tokens=33), 6)):
        with pytest.raises(pb.PPError) as e:
            pb.MoELayer(r, u, d, **{**ok, **bad})
        assert e.value.status == status
    with pytest.raises(TypeError):
        pb.MoELayer(r, u, d.bfloat16(), **ok)
    with pytest.raises(TypeError):
        pb.MoELayer(r, u.float(), d.float(), **ok)
    with pytest.raises(ValueError):
        pb.MoELayer(r, u[:, :-1], d, **ok)
    with pytest.raises(ValueError):
        pb.MoELayer(r.cpu(), u, d, **ok)
    with pytest.raises(pb.PPError) as e:
        pb.MoELayer(torch.zeros(300, 16, device="cuda"), torch.zeros(300, 16, 16, device="cuda").half(),
                    torch.zeros(300, 16, 8, device="cuda").half(), inner=8, top_k=2, max_tokens=1)
    assert e.value.status == 6
    c, s = torch.zeros(E, 2 * F, H // 2, device="cuda", dtype=torch.uint8), torch.ones(E, 2 * F, 1, device="cuda").half()
    dc, ds = torch.zeros(E, H, F // 2, device="cuda", dtype=torch.uint8), torch.ones(E, H, 1, device="cuda").half()
    with pytest.raises(pb.PPError) as e:
        pb.MoELayer.q4(r, c, s, dc, ds, gate_up_zeros=torch.zeros(E, 2 * F, 1, device="cuda", dtype=torch.uint8), group=0, **ok)
    assert e.value.status == 1
    with pytest.raises(TypeError):
        pb.MoELayer.q4(r, c, s, dc, ds.bfloat16(), group=0, **ok)
    L = pb.MoELayer(r, u, d, **ok)
    for x in (torch.zeros(5, H, device="cuda"), torch.zeros(0, H, device="cuda")):
        with pytest.raises(pb.PPError) as e:
            pb.pp_moe_forward(L, x)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        pb.pp_moe_forward(L, torch.zeros(1, H + 1, device="cuda"))
    with pytest.raises(TypeError):
        pb.pp_moe_forward(L, torch.zeros(1, H, device="cuda").double())
    with pytest.raises(pb.PPError) as e:
        pb.pp_moe_forward(L, torch.zeros(1, H, device="cuda").to(torch.int8), out_dtype=torch.float32)
    assert e.value.status == 6


def test_moe_c_interface_refuses_null():
    L = pb.lib()
    h = pb.ctypes.c_void_p()
    assert L.pp_moe_create(pb.ctypes.byref(h), 4, 64, 32, 2, 1, 4, None, pb.PP_F16, None, None, pb.PP_F16, None) == 1 and not h
    assert L.pp_moe_create(None, 4, 64, 32, 2, 1, 4, 16, pb.PP_F16, 16, 16, pb.PP_F16, None) == 1
    assert L.pp_moe_create_q4(pb.ctypes.byref(h), 4, 64, 32, 2, 1, 4, 16, pb.PP_F16, 48, 16, 16, None, 16, 16, None, pb.PP_F16, None) == 6
    assert L.pp_moe_forward(None, 16, 64, pb.PP_F16, 16, pb.PP_F16, 1, None, None, None) == 1
    assert L.pp_moe_destroy(None) == 1 and L.pp_moe_status(None, None) == 1
