"""Attention over a paged cache with infinities in q and in values, whatever the rows' alignment."""
import math

import pytest
import torch

from paper_1712_01084_b200 import binding as pb
from test_gpu_paged import KINDS, TOP, _attention_case


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("shift", [0, 1])
def test_attention_of_an_infinite_q(dtype, kind, shift):
    """An element of q that is infinite makes a head's scores infinite: 0 where all of them are minus infinity, else NaN.  Large elements
    beside it change nothing, nor does the alignment of q."""
    c, q, table, n = _attention_case(2, dtype, kind, 4, 2, 64, 16, [100, 40])
    c.k.copy_(torch.where(c.k.float() == 0, torch.ones_like(c.k.float()), c.k.float()).to(c.k.dtype))      # no 0 * inf
    for r, m in enumerate([100, 40]):
        at = torch.arange(m, device="cuda")
        number, place = table[r].long()[at // 16], at % 16
        x = c.k[number, place].float()
        x[..., 5] = x[..., 5].abs()
        c.k[number, place] = x.to(c.k.dtype)
    big = 60000.0 if dtype == "f16" else 1e6
    q[0, 0, 5], q[0, 1, 5], q[1, 3, 5] = -math.inf, math.inf, -math.inf
    q[0, 0, 6], q[1, 3, 9] = big, -big
    row = torch.zeros(2, 4, 64 + shift, dtype=q.dtype, device="cuda")[..., shift:]
    row.copy_(q)
    o, lse = pb.pp_paged_attention(c, row, table, n, lse=True)
    for r, h in ((0, 0), (1, 3)):
        assert bool((o[r, h] == 0).all()) and float(lse[r, h]) == -math.inf
    assert bool(torch.isnan(o[0, 1]).all())
    rest = torch.ones(2, 4, dtype=torch.bool, device="cuda")
    rest[0, 0] = rest[0, 1] = rest[1, 3] = False
    assert bool(torch.isfinite(o[rest]).all()) and bool(torch.isfinite(lse[rest]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [k for k in KINDS if k[1] not in TOP])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("sign", [1, -1])
def test_attention_over_an_infinite_value(dtype, kind, shift, sign):
    """A dimension in which a value is infinite is not finite, whatever the alignment; the other dimensions and heads are as without it."""
    c, q, table, n = _attention_case(4, dtype, kind, 4, 2, 64, 16, [100, 40])
    pages, page, g, d = c.k.shape
    k, v = (torch.zeros(pages, page, g, d + 8 * shift + shift, dtype=c.k.dtype, device="cuda")[..., shift:shift + d] for _ in range(2))
    k.copy_(c.k)
    v.copy_(c.v)
    c = pb.PagedCache(k, v)
    want = pb.pp_paged_attention(c, q, table, n)
    v[int(table[0, 2]), 3, 1, 7] = sign * math.inf
    v[int(table[1, 0]), 0, 0, 20] = sign * math.inf
    got = pb.pp_paged_attention(c, q, table, n)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 2:, 7] = bad[1, :2, 20] = True
    assert not bool(torch.isfinite(got[bad]).any()) and torch.equal(got[~bad], want[~bad])
