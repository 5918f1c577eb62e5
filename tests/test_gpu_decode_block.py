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
