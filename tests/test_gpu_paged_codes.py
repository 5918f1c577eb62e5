"""8-bit codes and scales that an append stores, bit for bit: scale = max / Q and code = value / scale, each quotient rounded to a
float, the code then to nearest, ties to even.  The values are not turned, so nothing else rounds; torch's division on the CPU is
that of IEEE."""
import pytest
import torch

from paper_1712_01084_b200 import binding as pb

TOP = {"int8": 127.0, "e4m3": 448.0}
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def _rows(kind, dim, count, dtype, seed):
    """Rows whose values lie at, or next to, the borders of two codes, in units of the scale that the row's largest value makes."""
    g = torch.Generator().manual_seed(seed)
    most = (0.5 + torch.rand(count, 1, generator=g)) * 2.0 ** torch.randint(-20, 12, (count, 1), generator=g)
    most[0::3] = (most[0::3] * 64).round() / 64 + 1 / 64                  # few bits, for ties that floats hold
    most = most.to(TYPES[dtype]).float()
    scale = most / TOP[kind]
    if kind == "int8":
        border = torch.randint(0, 126, (count, dim), generator=g) + 0.5
    else:
        codes = torch.arange(0, 126, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
        borders = (codes[1:] + codes[:-1]) / 2
        border = borders[torch.randint(0, borders.numel(), (count, dim), generator=g)]
    x = (border.double() * scale.double()).float()
    x = x.view(torch.int32).add(torch.randint(-1, 2, x.shape, generator=g).int()).view(torch.float32)
    x = torch.where(torch.rand(x.shape, generator=g) < 0.5, x, -x)
    x = torch.minimum(x.abs(), most).copysign(x)
    x[torch.arange(count), torch.randint(0, dim, (count,), generator=g)] = most[:, 0]
    return x.to(TYPES[dtype])


def _codes(x, kind):
    x = x.float()
    scale = x.abs().amax(-1) / TOP[kind]
    q = x / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]
    q = torch.where(scale[..., None] > 0, q, torch.zeros_like(q)).clamp(-TOP[kind], TOP[kind])
    return (q.round().to(torch.int8) if kind == "int8" else q.to(torch.float8_e4m3fn)).float(), scale


def _check(x, kind, shift=0):
    """x on the CPU, [tokens][2][dim], stored as keys and (in another order) as values."""
    n, g, d = x.shape
    pages = -(-n // 16)
    buffers = [torch.zeros(pages, 16, g, d + shift, dtype=torch.uint8, device="cuda").view(TYPES[kind])[..., shift:] for _ in range(2)]
    scales = [torch.zeros(pages, 16, g, device="cuda") for _ in range(2)]
    c = pb.PagedCache(*buffers, *scales)
    rows = [x.cuda(), x.flip(0).cuda()]
    pb.pp_kv_append(c, *rows, torch.arange(n, device="cuda"))
    for buffer, s, row in zip(buffers, scales, (x, x.flip(0))):
        codes, scale = _codes(row, kind)
        assert torch.equal(s.reshape(-1, g)[:n].cpu(), scale)
        got = buffer.float().reshape(-1, g, d)[:n].cpu()
        assert torch.equal(got, codes), int((got != codes).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,shift", [(128, 0), (72, 0), (64, 1), (33, 0)])
@pytest.mark.parametrize("tokens", [1, 64, 3000])
def test_codes_are_the_rounded_quotients(kind, dtype, dim, shift, tokens):
    _check(_rows(kind, dim, 2 * tokens, dtype, dim + tokens).view(tokens, 2, dim), kind, shift)


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0, 1])
def test_a_code_at_a_tie(shift):
    """6.5 scales exactly, which is 6, and its neighbours."""
    scale = torch.tensor(15.625) / 127
    tie = 6.5 * scale
    assert float(tie.double() / scale.double()) == 6.5
    x = torch.zeros(2, 2, 64)
    x[..., 0], x[..., 1], x[..., 2], x[..., 3] = 15.625, tie, -tie, torch.nextafter(tie, torch.tensor(9.0))
    assert _codes(x, "int8")[0][0, 0, :4].tolist() == [127, 6, -6, 7]
    _check(x, "int8", shift)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shift", [0, 1])
def test_codes_of_the_smallest_rows(kind, shift):
    """Rows down to the smallest subnormal numbers, and zeros."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 2, 64, generator=g)
    x = x / x.abs().amax(-1, keepdim=True)
    x = (x.double() * 2.0 ** torch.linspace(-149, -90, 40, dtype=torch.float64)[:, None, None]).float()
    x[3, 1] = 0.0
    _check(x, kind, shift)
