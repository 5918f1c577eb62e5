"""The example block: its four calls in sequence against the same steps in 64 bits.

Each step is compared with the definition applied to what the step before it really handed on, so that a code that rounds
the other way, or a choice of experts that hangs on it, does not spread: the bounds are those of the single operators.
"""
import pytest
import torch

from paper_1712_01084_b200 import binding as pb
from paper_1712_01084_b200 import decode_block

SUM = 1e-5


def _floats(codes, scales, cols, group=128):
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)[..., :cols].double()
    return (q - 8) * scales.double().repeat_interleave(group, -1)[..., :cols]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 700), (2, 5, 256)])
def test_quantize_q4_rounds_to_the_nearest_code(shape):
    w = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    codes, scales = decode_block.quantize_q4(w)
    err = (_floats(codes, scales, shape[-1]) - w.double()).abs()
    step = scales.double().repeat_interleave(128, -1)[..., :shape[-1]]
    assert bool((err <= step * 0.5 * 1.01 + step * 0.51 * (w.double().abs() >= 7.49 * step)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("experts", ["q4", "bf16"])
@pytest.mark.parametrize("tokens", [1, 3])
def test_block_steps(experts, tokens):
    H, F = 512, 256
    gen = torch.Generator(device="cuda").manual_seed(2)
    b = decode_block.DecodeBlock(H, F, 16, 4, 4, experts, generator=gen)
    # the projection's weights again, from the same stream of random numbers
    gen2 = torch.Generator(device="cuda").manual_seed(2)
    for _ in range(2):
        torch.randn(H, generator=gen2, device="cuda")
    w = _floats(*decode_block.quantize_q4(torch.randn(H, H, generator=gen2, device="cuda") / H ** 0.5), H)
    a = torch.randn(tokens, H, generator=gen, device="cuda").bfloat16()
    h = torch.randn(tokens, H, generator=gen, device="cuda").bfloat16()
    h0 = h.clone()
    y, h1 = b.step(a, h)
    assert h1 is h and y.shape == a.shape and bool(torch.isfinite(y).all()) and b.moe.status() == 0
    # the same calls one by one
    q, s, ha = pb.pp_rmsnorm_q8(a, b.norm1, residual=h0, group=128)
    assert torch.equal(ha, (a.float() + h0.float()).bfloat16())
    x = q.double() * s.double().repeat_interleave(128, 1)
    p = pb.pp_q4_forward(b.dense, q, x_scales=s, out_dtype=torch.bfloat16)
    err, mass = (p.double() - x @ w.T).abs(), x.abs() @ w.abs().T
    assert bool((err <= SUM * mass + 2.0 ** -8 * (x @ w.T).abs() * 1.001).all())
    _, _, hb, n = pb.pp_rmsnorm_q8(p, b.norm2, residual=ha, group=128, normed=True)
    assert torch.equal(h, hb)
    assert torch.equal(y, pb.pp_moe_forward(b.moe, n))


@pytest.mark.gpu
def test_block_in_a_graph_repeats():
    b = decode_block.DecodeBlock(256, 128, 8, 2, 2, "q4", generator=torch.Generator(device="cuda").manual_seed(3))
    a = torch.randn(2, 256, device="cuda").bfloat16()
    h = torch.zeros_like(a)
    want, _ = b.step(a, h)
    h_want = h.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.zero_()
        y = b.step(a, h)[0]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(h, h_want)


def _norm64(x, w, eps=1e-6):
    """n of the definition, and codes' scales per 128 columns."""
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    return n, torch.stack([p.abs().amax(-1) for p in n.split(128, -1)], -1) / 448.0


def _codes_match(q, s, n, scales):
    """e4m3 codes within half a step of n / s, the scales within the norm's fp32 error (see the single operator's test)."""
    tol = 6e-6
    assert bool(((s.double() - scales).abs() <= tol * scales).all())
    v = n / scales.repeat_interleave(128, 1)
    assert bool(((q.double() - v).abs() <= v.abs() * 2.0 ** -4 * (1 + 1e-4) + 2.0 ** -10 + 448 * 2 * tol * 2.0 ** -3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("experts", ["q4", "bf16"])
@pytest.mark.parametrize("tokens", [1, 3])
def test_block_steps_against_the_definitions(experts, tokens):
    """Norms, routing and experts of a step in 64 bits, with the weights drawn again from the same random numbers."""
    H, F, E, k = 512, 256, 16, 4
    b = decode_block.DecodeBlock(H, F, E, k, 4, experts, generator=torch.Generator(device="cuda").manual_seed(5))
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    w1, w2 = ((1 + 0.1 * rand(H)).bfloat16() for _ in range(2))
    rand(H, H)                                                               # the projection, checked by test_block_steps
    router = (rand(E, H) / H ** 0.5).bfloat16().double()
    up, down = rand(E, 2 * F, H) / H ** 0.5, rand(E, H, F) / F ** 0.5
    if experts == "q4":
        up, down = _floats(*decode_block.quantize_q4(up), H), _floats(*decode_block.quantize_q4(down), F)
    else:
        up, down = up.bfloat16().double(), down.bfloat16().double()
    a, h0 = rand(tokens, H).bfloat16(), rand(tokens, H).bfloat16()
    h = h0.clone()
    y, _ = b.step(a, h)

    n64, scales = _norm64(a.double() + h0.double(), w1)
    q, s, ha = pb.pp_rmsnorm_q8(a, b.norm1, residual=h0, group=128)
    _codes_match(q, s, n64, scales)
    p = pb.pp_q4_forward(b.dense, q, x_scales=s, out_dtype=torch.bfloat16)
    assert torch.equal(h, (p.float() + ha.float()).bfloat16())
    n64, scales = _norm64(p.double() + ha.double(), w2)
    q, s, _, n = pb.pp_rmsnorm_q8(p, b.norm2, residual=ha, group=128, normed=True)
    _codes_match(q, s, n64, scales)
    assert bool(((n.double() - n64).abs() <= n64.abs() * (2.0 ** -8 + 6e-6)).all())

    x = n.double()                                                           # what the experts really get
    logits = x @ router.T
    order = torch.argsort(logits, dim=1, descending=True, stable=True)[:, :k]
    gates = torch.softmax(logits.gather(1, order), 1)
    e_logit = 2e-6 * (x.abs() @ router.abs().T).amax(1)
    _, ids, got = pb.pp_moe_forward(b.moe, n, routing=True)
    assert torch.equal(ids.long(), order)
    assert bool(((got.double() - gates).abs() <= gates * (2 * e_logit[:, None] + 4e-6)).all())
    want, bound = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(tokens):
        for e, g in zip(order[t].tolist(), gates[t]):
            gu, mass = up[e] @ x[t], SUM * (up[e].abs() @ x[t].abs())
            gate, u, dg, du = gu[:F], gu[F:], mass[:F], mass[F:]
            silu = gate * torch.sigmoid(gate)
            act = g * silu * u
            d_act = g * (1.1 * dg * u.abs() + (silu.abs() + 1.1 * dg) * du) + act.abs() * (2 * e_logit[t] + 4e-6)
            want[t] += down[e] @ act
            bound[t] += down[e].abs() @ (d_act + SUM * act.abs() + 3e-11)
    assert bool(((y.double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound) * 1.001).all())


@pytest.mark.gpu
def test_normalised_rows_feed_a_pruned_layer_and_back():
    """f16 rows of the norm into a pruned layer, its f32 result into the next norm."""
    from paper_1712_01084_b200 import synth
    import numpy as np
    from oracle import pp_oracle as po
    wl = synth.config5(k=16, batch=2, scale=0.25)
    lay = wl.layers[0]
    L = pb.Layer.from_synth(lay)
    x = torch.from_numpy(wl.x).cuda()
    w = torch.ones(x.shape[1], device="cuda").half()
    n = pb.pp_rmsnorm_q8(x, w, normed=True)[3]
    y = pb.pp_forward(L, n, lay.act)
    want, _, mass = po.layer_forward(lay, n.double().cpu().numpy())
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= 2e-3 * mass + 1e-4)
    ones = torch.ones(y.shape[1], device="cuda")
    q, s, _ = pb.pp_rmsnorm_q8(y, ones, group=128)
    cols = y.shape[1]
    assert cols % 128 == 0
    _codes_match(q, s, *_norm64(y.double(), ones))
