"""Attention over 8-bit caches whose value scales lie far apart, against the definition in 64 bits.

Tolerance: that of test_gpu_paged._bound, and what the second product cannot hold.  p times the scale of its value enters as one or
two f16 numbers relative to the largest such product that the warp has met, which stands at 2^6 at least; half the last step of f16
is 2^-25, so each position may be off by 2^-31 of the largest product times its code, which is Q at most."""
import math

import pytest
import torch

from paper_1712_01084_b200 import binding as pb
from test_gpu_paged import KINDS, TOP, _attention_case, _attention_reference, _bound

EIGHT = [k for k in KINDS if k[1] in TOP] + [("f16", "e4m3")]


def _heaviest(c, q, table, lengths):
    """The largest p * |scale of the value| of each request and head, and the positions that it holds."""
    out = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    for r, n in enumerate(lengths.tolist()):
        at = torch.arange(n, device="cuda")
        number = table[r].long()[at // c.page_size]
        k = c.k[number, at % c.page_size].double() * c.k_scales[number, at % c.page_size].double()[..., None]
        v = c.v_scales[number, at % c.page_size].double().abs()
        k, v = (x.repeat_interleave(q.shape[1] // c.kv_heads, 1) for x in (k, v))
        p = torch.softmax(torch.einsum("hd,nhd->hn", q[r].double(), k) / math.sqrt(c.head_dim), 1)
        out[r] = (p * v.T).amax(1)
    return out


def _check(c, q, table, lengths):
    want, lse, mass, slack = _attention_reference(c, q, table, lengths, 1 / math.sqrt(c.head_dim))
    got, e = pb.pp_paged_attention(c, q, table, lengths, lse=True)
    top = 127.0 if c.k.dtype == torch.int8 else 448.0
    lost = lengths.double()[:, None] * 2.0 ** -31 * top * _heaviest(c, q, table, lengths)
    err = (got.double() - want).abs()
    bound = _bound(want, mass, slack, float(lengths.max()), q.dtype, c.k.dtype) + lost[..., None]
    # an f16 output ends at 65504: what is past it, or may be within the bound, rounds to an infinity of its sign
    past = torch.isinf(got) & (got.double().sign() == want.sign()) & (want.abs() + bound > 65504.0) if q.dtype == torch.float16 else torch.zeros_like(got, dtype=torch.bool)
    assert bool(((err <= bound) | past).all()), float((err / bound)[~past].max())
    none = torch.isinf(lse)
    assert torch.equal(torch.isinf(e) & (e < 0), none)
    assert bool(((e.double() - lse).abs()[~none] <= 2 * slack[~none] + (float(lengths.max()) / 8 + 600) * 2.0 ** -23 + 2.0 ** -20 + lse[~none].abs() * 2.0 ** -22).all())


def _set(c, table, r, position, k0=None, scale=None):
    """Gives one position of request r a key that is k0 in its first dimension and 0 else, and a scale of its values."""
    page, place = int(table[r, position // c.page_size]), position % c.page_size
    if k0 is not None:
        top = 127.0 if c.k.dtype == torch.int8 else 448.0
        row = torch.zeros(c.kv_heads, c.head_dim, device="cuda")
        row[:, 0] = math.copysign(top, k0)
        c.k[page, place] = row.to(c.k.dtype)
        c.k_scales[page, place] = abs(k0) / top
    if scale is not None:
        c.v_scales[page, place] = scale


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", EIGHT)
@pytest.mark.parametrize("ratio", [10, 20, 34])
@pytest.mark.parametrize("place", ["first", "last", "alone"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths", [(8, 1, 64, 16, [10, 100]), (32, 2, 128, 16, [300, 17]), (16, 4, 96, 1, [40, 2000]), (8, 2, 192, 32, [1000] * 3),
                                                             (8, 8, 128, 16, [20000, 9000])])
def test_attention_beside_a_large_value_of_no_weight(dtype, kind, ratio, place, heads, kv_heads, dim, page, lengths):
    """One value 2^ratio above the others (of the requests before it too), at a score that leaves it next to no weight: the others keep their bits."""
    c, q, table, n = _attention_case(ratio + dim, dtype, kind, heads, kv_heads, dim, page, lengths)
    q[..., 0] = 4.0
    # "alone": in front of the positions that its warp reads with it
    for r, length in enumerate(lengths):
        at = {"first": 0, "last": length - 1, "alone": min(64, length - 1)}[place]
        _set(c, table, r, at, k0=-20.0 * math.sqrt(dim), scale=float(c.v_scales[~torch.isnan(c.v_scales)].max()) * 2.0 ** ratio)
    _check(c, q, table, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", EIGHT)
@pytest.mark.parametrize("ratio", [6, 12, 20, 30])
def test_attention_beside_a_large_value_that_counts_as_much(dtype, kind, ratio):
    """The score of the large value is as far below the others' as its scale is above theirs."""
    for at in (0, 5, 150):
        c, q, table, n = _attention_case(ratio, dtype, kind, 8, 1, 64, 16, [200, 151])
        q[..., 0] = 1.0
        for r in range(2):
            _set(c, table, r, at, k0=-ratio * math.log(2.0) * 8, scale=0.01 * 2.0 ** ratio)
        _check(c, q, table, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", EIGHT)
@pytest.mark.parametrize("spread", [8, 24, 60])
@pytest.mark.parametrize("order", ["random", "rising", "falling"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths", [(8, 2, 64, 16, [700, 33]), (16, 1, 128, 8, [400]), (4, 4, 256, 16, [200] * 4), (8, 8, 128, 16, [12000, 700])])
def test_attention_over_scales_of_every_size(dtype, kind, spread, order, heads, kv_heads, dim, page, lengths):
    """Scales of values over 2^spread, and scores over tens, in any order: maxima and largest products move time and again."""
    c, q, table, n = _attention_case(spread, dtype, kind, heads, kv_heads, dim, page, lengths)
    q[..., 0] = 2.0
    g = torch.Generator().manual_seed(spread)
    for r, length in enumerate(lengths):
        at = torch.arange(length)
        rise = {"random": torch.rand(length, generator=g), "rising": at / length, "falling": 1 - at / length}[order]
        number, place = table[r].cpu().long()[at // page].cuda(), (at % page).cuda()
        c.v_scales[number, place] = (2.0 ** (spread * (torch.rand(length, kv_heads, generator=g) - 0.5)) * 0.01).cuda()
        codes = c.k[number, place].float() / 16
        codes[..., 0] = ((2 * rise.cuda() - 1) * TOP[kind])[:, None]       # a part of the score that goes over +-20
        c.k[number, place] = (codes.round() if kind == "int8" else codes).to(c.k.dtype)
        c.k_scales[number, place] = 10 * math.sqrt(dim) / TOP[kind]
    _check(c, q, table, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [("bf16", "e4m3"), ("f16", "int8"), ("f32", "e4m3"), ("f32", "int8")])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -118, 2.0 ** -110, 2.0 ** -20, 2.0 ** 100])
def test_attention_over_scales_near_the_ends(dtype, kind, scale):
    """All values at one far scale, and then one of ordinary size among them."""
    if scale > 1 and dtype == "f16":
        scale = 1.0                                          # f16 outputs end at 65504
    c, q, table, n = _attention_case(3, dtype, kind, 8, 2, 64, 16, [300, 20])
    c.v_scales[~torch.isnan(c.v_scales)] = scale
    _check(c, q, table, n)
    for r, at in ((0, 299), (1, 3)):
        _set(c, table, r, at, scale=0.01)
    _check(c, q, table, n)
