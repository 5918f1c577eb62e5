"""Attention over a paged cache with scores so large that the steps of floats between them are no small part of a power of two."""
import math

import pytest
import torch

from paper_1712_01084_b200 import binding as pb
from test_gpu_paged import KINDS, ROUND, TOP, TYPES, _attention_case


def _one_key(dtype, kind, size, dim=64, heads=16, kv_heads=2, page=16, length=200):
    """Key 77 is like q of each head, and size^2 long; the others point away from it: its value is the answer."""
    c, q, table, n = _attention_case(1, dtype, kind, heads, kv_heads, dim, page, [length, 100])
    away = torch.full((length, kv_heads, dim), -1.0, device="cuda")
    away[77] = 1.0
    for r, m in ((0, length), (1, 100)):
        at = torch.arange(m, device="cuda")
        number, place = table[r].long()[at // page], at % page
        if kind in TOP:
            c.k[number, place] = (away[:m] * 100).to(TYPES[kind])
            c.k_scales[number, place] = size / 100
        else:
            c.k[number, place] = (away[:m] * size).to(TYPES[kind])
    step = torch.arange(heads, device="cuda")[None, :, None] / 100
    q.copy_((size * (1 + step)).expand_as(q))
    want, key = [], []
    for r in range(2):
        page77, place77 = int(table[r, 77 // page]), 77 % page
        v = c.v[page77, place77].double()
        k = c.k[page77, place77].double()
        if kind in TOP:
            v, k = v * c.v_scales[page77, place77].double()[:, None], k * c.k_scales[page77, place77].double()[:, None]
        key.append(k.repeat_interleave(heads // kv_heads, 0))
        want.append(v.repeat_interleave(heads // kv_heads, 0))
    return c, q, table, n, torch.stack(want), (torch.stack(key) * q.double()).sum(-1) / math.sqrt(dim)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("size", [300.0, 3000.0, 9000.0, 30000.0, 1e6, 1e9])
def test_attention_with_scores_past_the_steps_of_floats(dtype, kind, size):
    """A score of size^2 * 8: its step may be thousands, and the largest one still takes all the weight."""
    if size > 50000 and "f16" in (dtype, kind):
        pytest.skip("f16 ends at 65504")
    c, q, table, n, want, score = _one_key(dtype, kind, size)
    assert bool(torch.isfinite(q).all())
    got, lse = pb.pp_paged_attention(c, q, table, n, lse=True)
    # one value, weight 1: the product of its code and scale, rounded to floats, and the output's rounding; for a bf16 output over 8 bits p
    # is one f16 number in the sum of values and a float in that of weights, half a step of 2^-11 apart, since its logarithm is the
    # product of the score that 32 bits do not hold less what they do
    one = 2.0 ** -11 if q.dtype == torch.bfloat16 and kind in TOP else 0.0
    assert bool(((got.double() - want).abs() <= (ROUND[q.dtype] + one + 2.0 ** -20) * want.abs()).all())
    assert bool(((lse.double() - score).abs() <= score * (c.head_dim + 8) * 2.0 ** -23).all())
