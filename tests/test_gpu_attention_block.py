"""The example's attention half: plan, norm, projections, append and attention in sequence over several steps.

Each call is compared with the definition applied to what the call before it really handed on; the bounds are those of the
single operators' tests (norm and 4-bit products: 1e-5 of the sum of magnitudes; attention: see test_gpu_paged.py).
"""
import math
import sys

import pytest
import torch

from paper_1712_01084_b200 import binding as pb
from paper_1712_01084_b200 import decode_block

SUM = 1e-5


def _floats(codes, scales, cols, group=128):
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)[..., :cols].double()
    return (q - 8) * scales.double().repeat_interleave(group, -1)[..., :cols]


def _product(y, x, w):
    """bfloat16 rows y against W x in 64 bits."""
    want, mass = x @ w.T, x.abs() @ w.abs().T
    assert bool(((y.double() - want).abs() <= SUM * mass + 2.0 ** -8 * want.abs() * 1.001).all())


def _turned(x, positions, inv_freq):
    angle = (positions.double()[:, None] * inv_freq.double())[:, None]
    n = inv_freq.numel()
    a, b = x[..., :n].double(), x[..., n:].double()
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(8, 2, 64, 16), (6, 3, 32, 5)])
def test_attention_half_steps(kind, heads, kv_heads, dim, page):
    H, requests, width = 256, 3, 24
    seed = lambda: torch.Generator(device="cuda").manual_seed(9)  # noqa: E731
    x = decode_block.DecodeAttention(H, heads, kv_heads, dim, requests * width, page, kind, generator=seed())
    gen = seed()                                                             # the weights again, from the same stream of random numbers
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    rand(H)
    rows = (heads + 2 * kv_heads) * dim
    w_qkv = _floats(*decode_block.quantize_q4(rand(rows, H) / H ** 0.5), H)
    w_out = _floats(*decode_block.quantize_q4(rand(H, heads * dim) / (heads * dim) ** 0.5), heads * dim)

    # prompts of 37, 0 and 60 tokens, in one call with padding
    held = [37, 0, 60]
    prompts = decode_block.PagedRequests(requests, width, requests * width, page, 100)
    plan = prompts.begin(torch.tensor(held, dtype=torch.int32, device="cuda"))
    k, v = (rand(100, kv_heads, dim).bfloat16() for _ in range(2))
    pb.pp_kv_append(x.cache, k, v, plan.slots, positions=plan.positions, inv_freq=x.inv_freq)
    keys = [_turned(k, plan.positions, x.inv_freq)[s:s + n] for s, n in zip(plan.starts.tolist(), held)]
    values = [v[s:s + n].double() for s, n in zip(plan.starts.tolist(), held)]

    state = decode_block.PagedRequests(requests, width, requests * width, page, requests)
    state.table, state.free = prompts.table, prompts.free
    state.plan.lengths.copy_(plan.lengths)
    state.plan.taken.copy_(plan.taken)
    h = torch.randn(requests, H, generator=gen, device="cuda").bfloat16()
    one = torch.ones(requests, dtype=torch.int32, device="cuda")
    for step in range(20):
        a = torch.randn(requests, H, generator=gen, device="cuda").bfloat16()
        state.begin(one)
        assert state.plan.positions.tolist() == [n + step for n in held] and state.plan.lengths.tolist() == [n + step + 1 for n in held]
        before = h.clone()
        y, _ = x.step(a, h, state)
        # the same calls one by one, each against its definition
        q8, s, hidden = pb.pp_rmsnorm_q8(a, x.norm, residual=before, group=128)
        assert torch.equal(h, hidden)
        qkv = pb.pp_q4_forward(x.qkv, q8, x_scales=s, out_dtype=torch.bfloat16)
        _product(qkv, q8.double() * s.double().repeat_interleave(128, 1), w_qkv)
        q, new_k, new_v = qkv.view(requests, -1, dim).split([heads, kv_heads, kv_heads], 1)
        turned = pb.pp_kv_append(x.cache, new_k, new_v, torch.full((requests,), -1, device="cuda"), q=q, positions=state.plan.positions, inv_freq=x.inv_freq)
        want = _turned(q, state.plan.positions, x.inv_freq)
        assert bool(((turned.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6 * q.double().abs().amax()).all())
        k_rows = _turned(new_k, state.plan.positions, x.inv_freq)
        o = pb.pp_paged_attention(x.cache, turned, state.table, state.plan.lengths)
        assert torch.equal(y, pb.pp_q4_forward(x.out, o.flatten(1), out_dtype=torch.bfloat16))
        _product(y, o.flatten(1).double(), w_out)
        for r in range(requests):
            keys[r], values[r] = torch.cat([keys[r], k_rows[r:r + 1]]), torch.cat([values[r], new_v[r:r + 1].double()])
            n = keys[r].shape[0]
            at = torch.arange(n, device="cuda")
            number = state.table[r].long()[at // page]
            ck, cv = (t[number, at % page].double() for t in (x.cache.k, x.cache.v))
            if x.cache.k_scales is not None:
                ck, cv = ck * x.cache.k_scales[number, at % page].double()[..., None], cv * x.cache.v_scales[number, at % page].double()[..., None]
            # what the cache holds is the keys and values, within the rounding of its type: half a step of the value, or of the row's scale
            for got, true in ((ck, keys[r]), (cv, values[r])):
                top = true.abs().amax(-1, keepdim=True)
                half = 2.0 ** -8 * true.abs() if kind == torch.bfloat16 else top / 254 if kind == torch.int8 else 2.0 ** -4 * true.abs() + top / 448 * 2.0 ** -10
                assert bool(((got - true).abs() <= half * 1.001 + 2e-6 * top).all())
            ck, cv = (t.repeat_interleave(heads // kv_heads, 1) for t in (ck, cv))
            p = torch.softmax(torch.einsum("hd,nhd->hn", turned[r].double(), ck) / math.sqrt(dim), 1)
            want, mass = torch.einsum("hn,nhd->hd", p, cv), torch.einsum("hn,nhd->hd", p, cv.abs())
            # p as one f16 number (8 bits) errs by 2^-11 at most, with the score's and the sums' errors below 2^-12 here
            assert bool(((o[r].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -10 if kind != torch.bfloat16 else 2.0 ** -12) * mass).all())


@pytest.mark.gpu
def test_attention_half_in_a_graph_goes_on_from_step_to_step():
    """Replays are steps: each finds its own slots, and the caches and outputs are those of the same steps called one by one."""
    def run(captured):
        gen = torch.Generator(device="cuda").manual_seed(4)
        x = decode_block.DecodeAttention(256, 4, 2, 64, 40, 8, generator=gen)
        for t in (x.cache.k, x.cache.v):
            t.view(torch.uint8).zero_()
        for t in (x.cache.k_scales, x.cache.v_scales):
            t.zero_()
        state = decode_block.PagedRequests(2, 20, 40, 8, 2)
        a = torch.randn(2, 256, generator=gen, device="cuda").bfloat16()
        h = torch.zeros_like(a)
        one = torch.ones(2, dtype=torch.int32, device="cuda")
        out = []

        def step():
            state.begin(one)
            return x.step(a, h, state)[0]
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                y = step()
            for _ in range(30):
                graph.replay()
                out.append(y.clone())
        else:
            out = [step() for _ in range(30)]
        torch.cuda.synchronize()
        return out, x.cache, state
    (a, ca, sa), (b, cb, sb) = run(False), run(True)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    assert torch.equal(ca.k.view(torch.uint8), cb.k.view(torch.uint8)) and torch.equal(ca.v_scales, cb.v_scales)
    assert torch.equal(sa.table, sb.table) and sa.plan.lengths.tolist() == sb.plan.lengths.tolist() == [30, 30]


@pytest.mark.gpu
@pytest.mark.parametrize("more", [[], ["--heads", "8", "--kv-heads", "2", "--head-dim", "64", "--context", "100", "--page", "16"]])
def test_the_command_runs(monkeypatch, capsys, more):
    monkeypatch.setattr(sys, "argv", ["decode_block", "--hidden", "256", "--inner", "128", "--experts", "8", "--top-k", "2", "--tokens", "2", "--layers", "2",
                                      "--steps", "3"] + more)
    decode_block.main()
    out = capsys.readouterr().out
    assert "finite: True" in out and "status 0" in out and (not more or "100 to 107 tokens" in out)
