"""The `stream` argument: what a call writes lies in memory of the stream it runs on.

Two ways in which memory of the current stream would show: a block that was just freed there, while a kernel that reads it
still waits in the queue, is handed to the call and overwritten; or the call's result is dropped, its block handed out
again on the current stream, and the call, still waiting on its own, writes over the new owner."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CYCLES = 100_000_000            # of a kernel that only waits: some 50 ms


@pytest.fixture(scope="module")
def pb():
    from paper_1712_01084_b200 import binding
    return binding


def _gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def _norm(pb):
    x, r = (torch.randn(700, 2048, generator=_gen(1), device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(2048, device="cuda").bfloat16()
    return lambda stream=None: pb.pp_rmsnorm_q8(x, w, residual=r, group=128, normed=True, stream=stream)


def _q4(pb):
    codes = torch.randint(0, 256, (30000, 64), generator=_gen(2), device="cuda", dtype=torch.uint8)
    layer = pb.Q4Layer(30000, 128, 128, codes, torch.ones(30000, 1, device="cuda").half())
    x = torch.randn(16, 128, generator=_gen(3), device="cuda")
    return lambda stream=None: (pb.pp_q4_forward(layer, x, stream=stream),)


def _moe(pb):
    g = _gen(4)
    layer = pb.MoELayer(torch.randn(8, 1024, generator=g, device="cuda"), torch.randn(8, 128, 1024, generator=g, device="cuda").half() / 32,
                        torch.randn(8, 1024, 64, generator=g, device="cuda").half() / 8, inner=64, top_k=2, max_tokens=16)
    x = torch.randn(16, 1024, generator=g, device="cuda")
    return lambda stream=None: pb.pp_moe_forward(layer, x, routing=True, stream=stream)


OPERATORS = {"norm": _norm, "q4": _q4, "moe": _moe}


def _check_stream_argument(call):
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    # freed blocks of the outputs' sizes, their readers still waiting
    held = [torch.full((t.numel() * t.element_size(),), 7, device="cuda", dtype=torch.uint8) for t in want for _ in range(2)]
    at = {h.data_ptr() for h in held}
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(CYCLES)
    read = [h + 1 for h in held]
    del held
    got = call(stream=side)
    assert not at & {t.data_ptr() for t in got}
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    assert all(bool((r == 8).all()) for r in read)

    # outputs dropped while the call waits
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
    got = call(stream=side)
    del got
    mine = [torch.full((t.numel() * t.element_size(),), 9, device="cuda", dtype=torch.uint8) for t in want for _ in range(2)]
    torch.cuda.synchronize()
    assert all(bool((m == 9).all()) for m in mine)


@pytest.mark.parametrize("operator", list(OPERATORS))
def test_decoder_operators_allocate_on_the_given_stream(pb, operator):
    _check_stream_argument(OPERATORS[operator](pb))


@pytest.mark.parametrize("operator", list(OPERATORS))
def test_decoder_operators_take_the_default_stream(pb, operator):
    """The default stream's handle is 0."""
    call = OPERATORS[operator](pb)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()) as _:
        current = torch.cuda.current_stream()
        got = call(stream=torch.cuda.default_stream())
        assert torch.cuda.current_stream() == current
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))


def _layer(pb, batch=8):
    from paper_1712_01084_b200 import synth
    wl = synth.config5(k=16, batch=batch, scale=0.25)
    return pb.Layer.from_synth(wl.layers[0]), torch.from_numpy(wl.x).cuda()


def _forward(pb):
    L, x = _layer(pb)
    return lambda stream=None: (pb.pp_forward(L, x, stream=stream),)


def _pivoted(pb):
    L, x = _layer(pb)
    return lambda stream=None: (pb.pp_forward_pivoted(L, x, stream=stream),)


def _chain(pb):
    L, x = _layer(pb)
    C = pb.pp_chain_create([L], [0], 8)
    return lambda stream=None: (pb.pp_chain_forward(C, x, stream=stream),)


def _layout(pb):
    import numpy as np
    rng = np.random.default_rng(5)
    perm = np.arange(1024, dtype=np.int32)
    S = pb.LayoutStudy(1024, 32, pb.PP_LAYOUT_BRC, pb.PP_MAP_ROWS_PER_LANE, perm, perm, rng.standard_normal(32 * 32 * 32).astype(np.float32))
    x = torch.randn(1024, generator=_gen(6), device="cuda")
    return lambda stream=None: (S.forward(x, stream=stream),)


@pytest.mark.parametrize("make", [_forward, _pivoted, _chain, _layout], ids=["layer", "pivoted", "chain", "layout"])
def test_layers_allocate_on_the_given_stream(pb, make):
    _check_stream_argument(make(pb))
