"""The decoder operators against plain implementations in 64 bits: normalisation to 8 bits and 4-bit products.

Tolerances.  Sums of exact products held in fp32: each addition errs by at most 2^-23 of the partial sum (the
tensor-core instruction cuts instead of rounding), a weight passes fewer than 84 additions, so an element is within
84 * 2^-23 = 1e-5 of sum |w x|, the library's tolerance for fp32 layers; a result in f16 or bf16 is rounded once more,
by 2^-11 or 2^-8 of itself at most.
"""
import numpy as np
import pytest
import torch

from paper_1712_01084_b200 import binding as pb

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SUM = 1e-5


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ------------------------------------------------------------------------------------------ normalisation
def _norm64(x, r, w, eps, top, group):
    h = x.double() + (0 if r is None else r.double())
    n = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * w.double()
    parts = n.split(group or n.shape[-1], -1)
    scales = torch.stack([p.abs().amax(-1) for p in parts], -1) / top
    spread = torch.cat([scales[:, i:i + 1].expand(-1, p.shape[-1]) for i, p in enumerate(parts)], -1)
    return h, n, scales, spread


def _check_norm(x, r, w, eps, codes, group, got):
    top = 448.0 if codes == "e4m3" else 127.0
    h, n, scales, spread = _norm64(x, r, w, eps, top, group)
    q, s, hidden = got[:3]
    assert q.shape == x.shape and s.shape == scales.shape
    # n: a sum of squares (its relative error is that of one addition chain, at most 1e-5 / 2 after the root) and four roundings
    tol = 6e-6
    assert bool(((s.double() - scales).abs() <= tol * scales).all())
    if hidden is not None:
        want = (x.float() + r.float()).to(x.dtype) if r is not None else x
        assert torch.equal(hidden, want)
    v = torch.where(spread > 0, n / spread.clamp(min=1e-300), torch.zeros_like(n))
    err = (q.double() - v).abs()
    if codes == "int8":
        bound = 0.5 + 127 * 2 * tol
    else:       # half a step: 2^-4 of the value, 2^-10 among the subnormals
        bound = v.abs() * 2.0 ** -4 * (1 + 1e-4) + 2.0 ** -10 + 448 * 2 * tol * 2.0 ** -3
    assert bool((err <= bound).all()), float((err - bound).max())
    if len(got) > 3:
        assert bool(((got[3].double() - n).abs() <= n.abs() * (ROUND[x.dtype] + tol)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("codes,group", [("e4m3", 0), ("e4m3", 128), ("int8", 0), ("int8", 128)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 7), (1, 128), (3, 129), (5, 1000), (4, 4096), (3, 4095), (2, 9216), (3, 8200),
                                       (2, 20001), (1, 32768), (300, 264)])
def test_norm_matches_definition(dtype, codes, group, rows, cols):
    g, t = _gen(rows * 40000 + cols), TYPES[dtype]
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").to(t) for _ in range(2))
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(t)
    got = pb.pp_rmsnorm_q8(x, w, residual=r, eps=1e-5, codes=codes, group=group, normed=True)
    _check_norm(x, r, w, 1e-5, codes, group, got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("codes,group", [("e4m3", 0), ("int8", 128)])
@pytest.mark.parametrize("rows,cols", [(1300, 8192), (2500, 4096), (9600, 136), (1190, 10240), (5000, 1000)])
def test_norm_many_rows(dtype, codes, group, rows, cols):
    g, t = _gen(rows + cols), TYPES[dtype]
    big = torch.randn(2, rows, cols + 8, generator=g, device="cuda").to(t)
    x, r = big[0, :, :cols], big[1, :, 8:]
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(t)
    keep = r.clone()
    got = pb.pp_rmsnorm_q8(x, w, residual=r, eps=1e-5, codes=codes, group=group, hidden_out=r, normed=True)
    _check_norm(x, keep, w, 1e-5, codes, group, (got[0], got[1], got[2].clone()))
    n = _norm64(x, keep, w, 1e-5, 1.0, group)[1]                             # among millions of values some are f16 subnormals,
    least = 2.0 ** -25 if dtype == "f16" else 0.0                            # whose rounding is up to half of 2^-24
    assert bool(((got[3].double() - n).abs() <= n.abs() * (ROUND[t] + 6e-6) + least).all())
    q, s, _ = pb.pp_rmsnorm_q8(x, w, eps=1e-5, codes=codes, group=group)     # without a residual
    _check_norm(x, None, w, 1e-5, codes, group, (q, s, None))


@pytest.mark.gpu
@pytest.mark.parametrize("cols,off", [(1024, 0), (1024, 3), (1001, 1), (512, 8)])
@pytest.mark.parametrize("in_place", ["residual", "x"])
def test_norm_strided_rows_in_place(cols, off, in_place):
    g = _gen(cols + off)
    big = torch.randn(2, 6, cols + 40, generator=g, device="cuda").bfloat16()
    x, r = (b[:, off:off + cols] for b in big)
    w = torch.randn(cols, generator=g, device="cuda")                       # float32 weight beside bf16 rows
    x0, r0, rest = x.clone(), r.clone(), big[:, :, cols + off:].clone()
    out = r if in_place == "residual" else x
    q, s, h = pb.pp_rmsnorm_q8(x, w, residual=r, group=128, hidden_out=out)
    assert h is out
    _check_norm(x0, r0, w, 1e-6, "e4m3", 128, (q, s, h.clone()))
    assert torch.equal(big[:, :, cols + off:], rest)


@pytest.mark.gpu
def test_norm_without_residual_and_empty():
    g = _gen(1)
    x, w = torch.randn(3, 640, generator=g, device="cuda").half(), torch.ones(640, device="cuda").half()
    q, s, h = pb.pp_rmsnorm_q8(x, w)
    assert h is None
    _check_norm(x, None, w, 1e-6, "e4m3", 0, (q, s, None))
    out = torch.empty_like(x)
    assert torch.equal(pb.pp_rmsnorm_q8(x, w, hidden_out=out)[2], x)
    q, s, _ = pb.pp_rmsnorm_q8(x[:0], w)
    assert q.shape == (0, 640) and s.shape == (0, 1)
    q, s, _ = pb.pp_rmsnorm_q8(x[0], w)                                     # a single row as a vector
    assert q.shape == (640,) and s.shape == (1,)


@pytest.mark.gpu
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("group", [0, 128])
def test_norm_rows_of_zeros_nan_inf_and_tiny(codes, group):
    cols = 512
    x = torch.randn(6, cols, generator=_gen(2), device="cuda")
    w = torch.ones(cols, device="cuda")
    x[0] = 0.0
    x[1, 5] = float("nan")
    x[2, 300] = float("inf")
    x[3, 128:256] = 0.0                     # one group of zeros among others
    x[4] *= 1e-30                           # eps rules: scales near the smallest normal numbers
    w2 = w.clone()
    w2[0:128] = 1e-12
    q, s, _ = pb.pp_rmsnorm_q8(x, w2, codes=codes, group=group, eps=1e-6)
    assert bool((s[0] == 0).all()) and bool((q[0].float() == 0).all())
    assert bool(torch.isnan(s[1]).all()) and bool(torch.isnan(s[2]).any())
    keep = [3, 4, 5]
    if group:
        assert float(s[3, 1]) == 0.0 and bool((q[3, 128:256].float() == 0).all())
    top = 448.0 if codes == "e4m3" else 127.0
    _, n, scales, spread = _norm64(x[keep], None, w2, 1e-6, top, group)
    assert bool(((s[keep].double() - scales).abs() <= 6e-6 * scales + 1e-44).all())
    big = spread > 1e-36
    v = torch.where(big, n / spread.clamp(min=1e-300), torch.zeros_like(n))
    err = torch.where(big, (q[keep].double() - v).abs(), torch.zeros_like(v))
    assert bool((err <= (0.51 if codes == "int8" else v.abs() / 16 * 1.001 + 2.0 ** -9)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("rows,cols,off", [(3, 512, 0), (3, 509, 1), (1600, 4096, 0)], ids=["few", "odd", "many"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_rows_that_are_not_finite_have_nan_scales(dtype, rows, cols, off, codes, group):
    """All of a row's scales are NaN, whatever the weight at the odd element, and no other row is touched."""
    t = TYPES[dtype]
    x = torch.randn(rows, cols + off, generator=_gen(20), device="cuda").to(t)[:, off:]
    w = (1 + 0.3 * torch.randn(cols, generator=_gen(21), device="cuda")).to(t)
    w[300] = 0.0                                                             # infinity times 0
    clean = pb.pp_rmsnorm_q8(x, w, codes=codes, group=group, normed=True)
    for at, value in ((5, float("inf")), (300, float("inf")), (300, float("-inf")), (300, float("nan")), (130, 3e19)):
        bad = x.clone()
        bad[1, at] = value                                                   # the last: finite, its square is not
        got = pb.pp_rmsnorm_q8(bad, w, codes=codes, group=group, normed=True)
        assert bool(torch.isnan(got[1][1]).all()) and bool(torch.isnan(got[3][1]).all())
        keep = [0, rows - 1]
        for a, b in zip(got, clean):
            if a is not None:
                assert torch.equal(a[keep].view(torch.uint8), b[keep].view(torch.uint8))
    odd = w.clone()
    odd[200] = float("nan")
    scales = pb.pp_rmsnorm_q8(x, odd, codes=codes, group=group)[1]
    nan = torch.isnan(scales)
    assert bool(nan[:, 1 if group else 0].all()) and int(nan.sum()) == rows


@pytest.mark.gpu
def test_norm_of_nearly_all_rows_that_an_int_counts():
    """The kernel for many rows asks for rows ahead of the one it works on: their numbers pass 2^31."""
    rows, cols = 2 ** 31 - 1, 8
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 * 2 ** 30:
        pytest.skip("takes 60 GB of device memory")
    x = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    ends = [slice(0, 5000), slice(rows - 20000, rows)]
    for i, e in enumerate(ends):
        x[e] = torch.randn(x[e].shape, generator=_gen(30 + i), device="cuda").bfloat16()
    w = (1 + 0.3 * torch.randn(cols, generator=_gen(32), device="cuda")).bfloat16()
    q, s, _ = pb.pp_rmsnorm_q8(x, w, eps=1e-5)
    for e in ends:
        _check_norm(x[e], None, w, 1e-5, "e4m3", 0, (q[e], s[e], None))
    del x, q, s
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_norm_refusals():
    x, w = torch.zeros(2, 256, device="cuda"), torch.zeros(256, device="cuda")
    with pytest.raises(ValueError):
        pb.pp_rmsnorm_q8(x, w[:255])
    with pytest.raises(ValueError):
        pb.pp_rmsnorm_q8(x.t(), torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError):
        pb.pp_rmsnorm_q8(x.cpu(), w)
    with pytest.raises(TypeError):
        pb.pp_rmsnorm_q8(x.double(), w)
    with pytest.raises(TypeError):
        pb.pp_rmsnorm_q8(x, w, residual=x.half())
    with pytest.raises(ValueError):
        pb.pp_rmsnorm_q8(x, w, codes="int4")
    for bad in (dict(group=64), dict(group=-128)):
        with pytest.raises(pb.PPError) as e:
            pb.pp_rmsnorm_q8(x, w, **bad)
        assert e.value.status == 6
    with pytest.raises(pb.PPError) as e:
        pb.pp_rmsnorm_q8(x, w.half())
    assert e.value.status == 6
    with pytest.raises(pb.PPError) as e:
        pb.pp_rmsnorm_q8(x, w, eps=float("nan"))
    assert e.value.status == 1
    with pytest.raises(pb.PPError) as e:
        pb.pp_rmsnorm_q8(torch.zeros(1, 32776, device="cuda"), torch.zeros(32776, device="cuda"))
    assert e.value.status == 6


# --------------------------------------------------------------------------------------- 4-bit products
def _q4_data(seed, M, N, group, zeros, scale_type=torch.float16):
    g = _gen(seed)
    q = torch.randint(0, 16, (M, N), generator=g, device="cuda", dtype=torch.uint8)
    groups = -(-N // group) if group else 1
    s = ((0.5 + torch.rand(M, groups, generator=g, device="cuda")) * 0.01).to(scale_type)
    z = torch.randint(0, 16, (M, groups), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    p = torch.nn.functional.pad(q, (0, N % 2), value=15)                     # the spare half byte holds anything
    codes = (p[:, 0::2] | (p[:, 1::2] << 4)).contiguous()
    col = torch.arange(N, device="cuda") // (group or N)
    w = (q.double() - (z.double()[:, col] if zeros else 8.0)) * s.double()[:, col]
    return codes, s, z, w


def _x8(x, kind, per_group):
    """x in 8 bits with scales per row or per 128 columns, and the values they stand for."""
    b, N = x.shape
    n = -(-N // 128) if per_group else 1
    width = 128 if per_group else N
    v = torch.nn.functional.pad(x, (0, n * width - N)).view(b, n, width)
    s = v.abs().amax(2) / (127.0 if kind == "int8" else 448.0) + 1e-9
    q = v / s[..., None]
    q = q.round().to(torch.int8) if kind == "int8" else q.to(torch.float8_e4m3fn)
    val = (q.double() * s.double()[..., None]).view(b, -1)[:, :N]
    return q.view(b, -1)[:, :N].contiguous(), s.contiguous(), val


def _check_y(y, w, x64, bias=None, relu=False):
    ref = x64 @ w.T
    mass = x64.abs() @ w.abs().T
    if bias is not None:
        ref = ref + bias.double()
        mass = mass + bias.double().abs()
    if relu:
        ref = ref.clamp(min=0)
    err = (y.double() - ref).abs()
    bound = SUM * mass + ROUND[y.dtype] * ref.abs() * 1.001 + 1e-30 + (2.0 ** -24 if y.dtype == torch.float16 else 0)
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 128, 256, 0])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,N", [(1, 1), (16, 128), (17, 33), (5, 300), (1000, 4096), (257, 1001), (2100, 640)])
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
def test_q4_matches_definition(M, N, group, zeros, xt):
    codes, s, z, w = _q4_data(M * 7 + N + group, M, N, group, zeros, torch.bfloat16 if zeros else torch.float16)
    g = _gen(5)
    bias = torch.randn(M, generator=g, device="cuda") if zeros else None
    L = pb.Q4Layer(M, N, group, codes, s, z, bias)
    for batch in (1, 3):
        x = torch.randn(batch, N, generator=g, device="cuda").to(TYPES[xt])
        _check_y(pb.pp_q4_forward(L, x), w, x.double(), bias)
        _check_y(pb.pp_q4_forward(L, x, pb.PP_ACT_RELU, out_dtype=x.dtype), w, x.double(), bias, relu=True)
    L.close()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("per_group", [False, True])
@pytest.mark.parametrize("M,N,group,batch", [(130, 515, 32, 1), (96, 4096, 128, 5), (1000, 2048, 64, 33), (40, 1000, 0, 9)])
def test_q4_eight_bit_inputs(kind, per_group, M, N, group, batch):
    codes, s, z, w = _q4_data(M + N, M, N, group, True)
    L = pb.Q4Layer(M, N, group, codes, s, z)
    x = torch.randn(batch, N, generator=_gen(6), device="cuda") * torch.linspace(0.1, 5, N, device="cuda")
    q, xs, val = _x8(x, kind, per_group)
    _check_y(pb.pp_q4_forward(L, q, x_scales=xs), w, val)


@pytest.mark.gpu
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch", [1, 2, 4, 5, 8, 9, 16, 17, 32, 33, 70])
def test_q4_batches(xt, batch):
    M, N = 333, 1152
    codes, s, z, w = _q4_data(9, M, N, 128, False)
    L = pb.Q4Layer(M, N, 128, codes, s)
    x = torch.randn(batch, N, generator=_gen(batch), device="cuda").to(TYPES[xt])
    y = pb.pp_q4_forward(L, x)
    _check_y(y, w, x.double())
    assert torch.equal(y, pb.pp_q4_forward(L, x))                            # the same bits every time


@pytest.mark.gpu
@pytest.mark.parametrize("group,zeros", [(0, False), (0, True), (32, False), (32, True), (64, True), (128, False)])
@pytest.mark.parametrize("N", [2 ** 18, 2 ** 18 - 129, 158720 + 128, 120000])
def test_q4_widest_layers_take_every_input(N, group, zeros):
    M = 37
    codes, s, z, w = _q4_data(N + group, M, N, group, zeros)
    L = pb.Q4Layer(M, N, group, codes, s, z)
    for batch in (1, 2, 3, 9):
        x = torch.randn(batch, N, generator=_gen(41), device="cuda")
        for t in TYPES.values():
            _check_y(pb.pp_q4_forward(L, x.to(t)), w, x.to(t).double())
        for kind in ("int8", "e4m3"):
            q, xs, val = _x8(x, kind, True)
            _check_y(pb.pp_q4_forward(L, q, x_scales=xs), w, val)
    L.close()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,batch", [(8192, 8192, 1), (8192, 8192, 16), (4096, 9216, 8), (20000, 256, 3), (64, 70000, 2), (48, 200000, 16)])
def test_q4_large(M, N, batch):
    codes, s, z, w = _q4_data(11, M, N, 128, True)
    L = pb.Q4Layer(M, N, 128, codes, s, z)
    for xt in (torch.bfloat16, torch.float32):
        x = torch.rand(batch, N, generator=_gen(3), device="cuda").to(xt)    # all of one sign
        ref, mass = x.double() @ w.T, x.double().abs() @ w.abs().T
        err = (pb.pp_q4_forward(L, x).double() - ref).abs()
        assert bool((err <= SUM * mass).all())


@pytest.mark.gpu
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
def test_q4_strides_alignment_and_range(xt):
    M, N, t = 70, 389, TYPES[xt]
    codes, s, z, w = _q4_data(12, M, N, 64, True)
    L = pb.Q4Layer(M, N, 64, codes, s, z)
    big = torch.randn(4, 1000, generator=_gen(4), device="cuda").to(t)
    for off in (0, 1, 2, 3, 5, 8):
        x = big[:, off:off + N]
        _check_y(pb.pp_q4_forward(L, x), w, x.double())
    x = big[:, :N].clone()
    x[0] *= 1e4                                                              # magnitudes far apart inside a block
    x[0, ::3] *= 1e-7 if xt != "f16" else 1e-3
    if xt != "f16":
        x[1] *= 1e30
        x[2] *= 1e-30
    x[3] = 0
    y = pb.pp_q4_forward(L, x)
    _check_y(y, w, x.double())
    assert bool((y[3] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128, 0])
@pytest.mark.parametrize("ratio", [1e3, 1e4])
def test_q4_elements_that_stand_out_beside_zero_weights(xt, group, ratio):
    """One element of 128 a thousand or ten thousand times the rest, in columns where every other row's weight is 0: in those
    rows the tolerance is that of the rest alone, 0.8 SUM |w| on average.  Fixed point of 31 bits errs by up to 2^-31 * 2e4 =
    0.93 SUM of |w| where the errors of 127 elements agree, by a tenth of that where they are independent."""
    M, N = 64, 1000
    codes, s, _, w = _q4_data(50 + group, M, N, group, False)
    out = torch.arange(60, N, 128, device="cuda")
    for c in out.tolist():                                                   # the zero point, 8: a weight of 0
        low = c % 2 == 0
        codes[::2, c // 2] = (codes[::2, c // 2] & (0xF0 if low else 0x0F)) | (0x08 if low else 0x80)
    w[::2, out] = 0.0
    L = pb.Q4Layer(M, N, group, codes, s)
    for batch in (1, 2, 3):
        x = torch.randn(batch, N, generator=_gen(51), device="cuda")
        x[:, out] = ratio * (1 + torch.rand(batch, len(out), generator=_gen(52), device="cuda"))
        x = x.to(TYPES[xt])
        _check_y(pb.pp_q4_forward(L, x), w, x.double())


@pytest.mark.gpu
def test_q4_not_finite_inputs_stay_in_their_row():
    M, N = 64, 512
    codes, s, z, w = _q4_data(13, M, N, 128, False)
    L = pb.Q4Layer(M, N, 128, codes, s)
    for t in TYPES.values():
        x = torch.randn(3, N, generator=_gen(8), device="cuda").to(t)
        x[1, 77] = float("inf")
        x[2, 300] = float("nan")
        y = pb.pp_q4_forward(L, x)
        _check_y(y[:1], w, x[:1].double())
        assert not bool(torch.isfinite(y[1:]).any())


@pytest.mark.gpu
def test_q4_extreme_codes_are_exact():
    M, N = 32, 256
    q = torch.tensor([0, 15], device="cuda", dtype=torch.uint8).repeat(M, N // 2)
    codes = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
    for zp in (0, 7, 15):
        z = torch.full((M, N // 32), zp, dtype=torch.uint8, device="cuda")
        L = pb.Q4Layer(M, N, 32, codes, torch.ones(M, N // 32, device="cuda").half(), z)
        x = torch.randint(-8, 9, (2, N), generator=_gen(9), device="cuda").to(torch.bfloat16)
        want = x.double() @ (q.double() - zp).T                              # whole numbers: no rounding anywhere
        assert torch.equal(pb.pp_q4_forward(L, x).double(), want)


@pytest.mark.gpu
def test_decode_operators_on_another_stream_and_in_sequence():
    """norm -> product -> norm on a side stream, many times without waiting, each step reading the one before."""
    N = 2048
    codes, s, _, w = _q4_data(14, N, N, 128, False)
    L = pb.Q4Layer(N, N, 128, codes, s)
    wt = torch.ones(N, device="cuda").bfloat16()
    x0 = torch.randn(2, N, generator=_gen(10), device="cuda").bfloat16()

    def chain():
        h, y = x0.clone(), torch.zeros_like(x0)
        for _ in range(12):
            q, sc, h = pb.pp_rmsnorm_q8(y, wt, residual=h, group=128)
            y = pb.pp_q4_forward(L, q, x_scales=sc, out_dtype=torch.bfloat16)
        return h, y

    want = chain()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            got = chain()
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_a_failed_launch_is_not_reported_by_the_next_call():
    """Launches into a stream capture that is no longer valid fail on the host; a layer made after them does not."""
    L, driver = pb.lib(), pb.ctypes.CDLL("libcuda.so.1")
    x, w = torch.randn(2, 256, device="cuda"), torch.ones(256, device="cuda")
    codes, s, _, _ = _q4_data(40, 64, 256, 64, False)
    layer = pb.Q4Layer(64, 256, 64, codes, s)
    q, scales, y = torch.empty(2, 256, device="cuda", dtype=torch.int8), torch.empty(2, device="cuda"), torch.empty(2, 64, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    handle = pb.ctypes.c_void_p(side.cuda_stream)
    p = lambda t: pb.ctypes.c_void_p(t.data_ptr())  # noqa: E731
    calls = (lambda: L.pp_rmsnorm_q8(p(x), 256, None, 0, p(w), pb.PP_F32, pb.PP_F32, 2, 256, 1e-6, pb.PP_I8, 0, p(q), p(scales), None, 0, None, handle),
             lambda: L.pp_q4_forward(layer._h, p(x), 256, pb.PP_F32, None, 0, p(y), pb.PP_F32, 2, 0, handle))
    for call in calls:
        assert driver.cuStreamBeginCapture_v2(handle, 2) == 0
        assert driver.cuStreamSynchronize(handle) != 0                       # not allowed there: the capture is invalid from now on
        status = call()
        graph = pb.ctypes.c_void_p()
        assert driver.cuStreamEndCapture(handle, pb.ctypes.byref(graph)) != 0 and not graph
        assert status == 5
        pb.Q4Layer(64, 256, 64, codes, s).close()
        assert call() == 0
    side.synchronize()
    _check_y(y, _q4_data(40, 64, 256, 64, False)[3], x.double())


@pytest.mark.gpu
def test_q4_in_a_graph():
    codes, s, _, w = _q4_data(15, 512, 1024, 64, False)
    L = pb.Q4Layer(512, 1024, 64, codes, s)
    x = torch.randn(1, 1024, device="cuda").half()
    y = pb.pp_q4_forward(L, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = pb.pp_q4_forward(L, x)
    x.copy_(torch.randn(1, 1024, generator=_gen(11), device="cuda").half())
    graph.replay()
    torch.cuda.synchronize()
    _check_y(z, w, x.double())
    assert y.shape == z.shape


@pytest.mark.gpu
def test_outputs_that_cross_inputs_are_refused():
    """Other CTAs still read what one writes.  Matrices in each other's gaps, and hidden_out in the place of an input, pass."""
    big = torch.randn(9, 1024, device="cuda")
    w = torch.ones(256, device="cuda")
    x = big[:8, :256]
    for out in (big[1:, :256], big[:8, 128:384], big[:8, 1:257]):
        for args in (dict(x=x, hidden_out=out), dict(x=big[:8, 512:768], residual=x, hidden_out=out)):
            with pytest.raises(pb.PPError) as e:
                pb.pp_rmsnorm_q8(weight=w, **args)
            assert e.value.status == 1
    for out in (big[:8, 256:512], big[1:, 768:], x):
        pb.pp_rmsnorm_q8(x, w, hidden_out=out)
    codes, s, _, m = _q4_data(60, 96, 256, 64, False)
    L = pb.Q4Layer(96, 256, 64, codes, s)
    flat = torch.randn(8 * 1024, device="cuda")
    x = flat.view(8, 1024)[:, :256]
    for start in (0, 255, 1024 - 96 * 8 + 1, 1000, 7 * 1024 + 255):
        with pytest.raises(pb.PPError) as e:
            pb.pp_q4_forward(L, x, out=flat[start:start + 96 * 8].view(8, 96))
        assert e.value.status == 1
    keep = x.clone()
    y = pb.pp_q4_forward(L, x, out=flat[256:256 + 96 * 8].view(8, 96))      # just fits between two rows
    assert torch.equal(x, keep)
    _check_y(y, m, keep.double())


@pytest.mark.gpu
def test_matrices_the_wrong_way_round_are_refused():
    """They hold as many elements as the right ones."""
    codes, s, _, _ = _q4_data(60, 96, 256, 64, False)
    L = pb.Q4Layer(96, 256, 64, codes, s)
    q = torch.zeros(4, 256, device="cuda", dtype=torch.int8)
    with pytest.raises(ValueError, match="x_scales"):
        pb.pp_q4_forward(L, q, x_scales=torch.ones(2, 4, device="cuda"))
    for scales in (torch.ones(4, 2, device="cuda"), torch.ones(4, 1, device="cuda"), torch.ones(4, device="cuda")):
        assert pb.pp_q4_forward(L, q, x_scales=scales).shape == (4, 96)
    pb.pp_q4_forward(L, q[0], x_scales=torch.ones(2, device="cuda"))
    x = torch.zeros(4, 256, device="cuda")
    with pytest.raises(ValueError, match="out"):
        pb.pp_q4_forward(L, x, out=torch.empty(96, 4, device="cuda"))
    for shape in ((4, 96), (4 * 96,)):
        assert pb.pp_q4_forward(L, x, out=torch.empty(shape, device="cuda")).shape == shape


@pytest.mark.gpu
def test_q4_refusals():
    codes, s, z, _ = _q4_data(16, 64, 256, 64, True)
    for bad in (dict(group=16), dict(group=96), dict(group=-64)):
        groups = -(-256 // bad["group"]) if bad["group"] > 0 else 1
        with pytest.raises(pb.PPError) as e:
            pb.Q4Layer(64, 256, bad["group"], codes, s[:, :1].expand(-1, groups).contiguous())
        assert e.value.status in (1, 6)
    with pytest.raises(ValueError):
        pb.Q4Layer(64, 256, 64, codes[:, :-1], s)
    with pytest.raises(TypeError):
        pb.Q4Layer(64, 256, 64, codes, s.float())
    with pytest.raises(TypeError):
        pb.Q4Layer(64, 256, 64, codes.to(torch.int8), s)
    with pytest.raises(ValueError):
        pb.Q4Layer(64, 256, 64, codes, s, z[:, :2])
    L = pb.Q4Layer(64, 256, 64, codes, s, z)
    x = torch.zeros(2, 256, device="cuda")
    with pytest.raises(ValueError):
        pb.pp_q4_forward(L, x[:, :255])
    with pytest.raises(ValueError):
        pb.pp_q4_forward(L, x.cpu())
    with pytest.raises(TypeError):
        pb.pp_q4_forward(L, x.double())
    for bad in (dict(x=x, x_scales=torch.ones(2, 1, device="cuda")), dict(x=x.to(torch.int8)), dict(x=x[:0])):
        with pytest.raises(pb.PPError) as e:
            pb.pp_q4_forward(L, **bad)
        assert e.value.status == 1
    with pytest.raises(pb.PPError) as e:
        pb.pp_q4_forward(L, x, out_dtype=torch.int8)
    assert e.value.status == 6
    with pytest.raises(pb.PPError):
        pb.pp_q4_forward(L, x, act=7)


def test_c_interface_refuses_null():
    L = pb.lib()
    h = pb.ctypes.c_void_p()
    assert L.pp_q4_create(pb.ctypes.byref(h), 16, 128, 64, None, None, pb.PP_F16, None, None, None) == 1 and not h
    assert L.pp_q4_create(None, 16, 128, 64, 16, 16, pb.PP_F16, None, None, None) == 1
    assert L.pp_q4_forward(None, 16, 128, pb.PP_F16, None, 0, 16, pb.PP_F32, 1, 0, None) == 1
    assert L.pp_q4_destroy(None) == 1
    assert L.pp_rmsnorm_q8(None, 0, None, 0, None, pb.PP_F16, pb.PP_F16, 1, 8, 1e-6, pb.PP_I8, 0, None, None, None, 0, None, None) == 1
    assert L.pp_rmsnorm_q8(16, 8, None, 0, 16, pb.PP_I8, pb.PP_I8, 1, 8, 1e-6, pb.PP_I8, 0, 16, 16, None, 0, None, None) == 6
