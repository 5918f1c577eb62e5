"""Example: a decoding step, on the library's decoder operators.

    python -m paper_1712_01084_b200.decode_block --hidden 2048 --tokens 1 --layers 8 --steps 20
    python -m paper_1712_01084_b200.decode_block --heads 16 --context 4000       # with attention

A block's feed-forward half adds its input to the residual stream, normalises it to 8 bits, multiplies the 8-bit rows with a 4-bit matrix, adds
and normalises again, and runs a mixture-of-experts layer on the result:

    q, s, h    = pp_rmsnorm_q8(a, w1, residual=h)              # h += a
    p          = pp_q4_forward(dense, q, x_scales=s)
    q, s, h, n = pp_rmsnorm_q8(p, w2, residual=h, normed=True) # h += p
    a          = pp_moe_forward(moe, n)

and its attention half (``--heads``) does the same with attention over a paged cache of past keys and values:

    plan       = pp_paged_plan(lengths, ...)                   # once a step: pages and slots of the new tokens
    q, s, h    = pp_rmsnorm_q8(a, w, residual=h)
    q, k, v    = pp_q4_forward(qkv, q, x_scales=s)
    q          = pp_kv_append(cache, k, v, plan.slots, q=q)    # rotary embedding; k and v into the cache
    o          = pp_paged_attention(cache, q, table, plan.lengths)
    a          = pp_q4_forward(out, o)

Nothing waits for the host; the command captures a step over all layers in a CUDA graph and prints its time.  Weights are random; ``quantize_q4`` rounds float weights to codes and scales in plain torch operations,
as a checkpoint in 4 bits would bring them.
"""
from __future__ import annotations

import argparse


def quantize_q4(w, group: int = 128):
    """(codes, scales) of rounded weights [..., rows, cols], every zero point 8: the arrays Q4Layer and MoELayer.q4 take."""
    import torch
    *lead, cols = w.shape
    n = -(-cols // group)
    v = torch.nn.functional.pad(w.float(), (0, n * group - cols)).view(*lead, n, group)
    scales = (v.abs().amax(-1) / 7.5).clamp(min=1e-6).half()
    q = (v / scales.float().unsqueeze(-1) + 8).round().clamp(0, 15).to(torch.uint8).view(*lead, n * group)[..., :cols]
    if cols % 2:
        q = torch.nn.functional.pad(q, (0, 1))
    return (q[..., 0::2] | (q[..., 1::2] << 4)).contiguous(), scales.contiguous()


class DecodeBlock:
    """One block: two norms, a 4-bit projection [hidden][hidden] and a mixture of experts.  ``experts`` in "q4" or "bf16"."""

    def __init__(self, hidden: int, inner: int, n_experts: int, top_k: int, max_tokens: int, experts: str = "q4", group: int = 128,
                 generator=None):
        import torch
        from . import binding as pb
        self._pb = pb
        rand = lambda *shape: torch.randn(shape, generator=generator, device="cuda")  # noqa: E731
        self.norm1, self.norm2 = ((1 + 0.1 * rand(hidden)).bfloat16() for _ in range(2))
        self.dense = pb.Q4Layer(hidden, hidden, group, *quantize_q4(rand(hidden, hidden) / hidden ** 0.5, group))
        router = (rand(n_experts, hidden) / hidden ** 0.5).bfloat16()
        up, down = rand(n_experts, 2 * inner, hidden) / hidden ** 0.5, rand(n_experts, hidden, inner) / inner ** 0.5
        more = dict(inner=inner, top_k=top_k, max_tokens=max_tokens)
        if experts == "q4":
            self.moe = pb.MoELayer.q4(router, *quantize_q4(up, group), *quantize_q4(down, group), group=group, **more)
        else:
            self.moe = pb.MoELayer(router, up.bfloat16(), down.bfloat16(), **more)

    def step(self, a, h, eps: float = 1e-6):
        """(a, h) -> (a, h): a, what the block before (or attention) hands on, and h, the residual stream (updated in place);
        bfloat16 [tokens][hidden]."""
        pb = self._pb
        q, s, _ = pb.pp_rmsnorm_q8(a, self.norm1, residual=h, eps=eps, group=128, hidden_out=h)
        p = pb.pp_q4_forward(self.dense, q, x_scales=s, out_dtype=a.dtype)
        _, _, _, n = pb.pp_rmsnorm_q8(p, self.norm2, residual=h, eps=eps, group=128, hidden_out=h, normed=True)
        return pb.pp_moe_forward(self.moe, n), h


class PagedRequests:
    """Requests that share the pages of one or more caches: the block table, the free list and the plan of the current step, for
    ``rows`` new tokens a step at most.  ``begin(added)`` takes int32 [requests], tokens to come (none for an idle request), and
    goes on from the lengths that the step before left; it may be captured into a graph, whose replays then are the steps."""

    def __init__(self, requests: int, width: int, pages: int, page_size: int, rows: int):
        import torch
        from . import binding as pb
        self._pb, self.page_size = pb, page_size
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.plan = pb.PagedPlan(requests, rows)
        self.plan.lengths.zero_()
        self.plan.taken.zero_()

    def begin(self, added):
        p = self.plan
        return self._pb.pp_paged_plan(p.lengths, added, self.table, self.free, p.taken, self.page_size, out=p)


class DecodeAttention:
    """The attention half of a block: norm, 4-bit projections [(heads + 2 kv_heads) head_dim][hidden] and [hidden][heads head_dim], and
    a paged cache (e4m3 with a scale for each token and head, unless cache_dtype says another 8-bit type or bfloat16)."""

    def __init__(self, hidden: int, heads: int, kv_heads: int, head_dim: int, pages: int, page_size: int, cache_dtype=None, group: int = 128,
                 theta: float = 500000.0, generator=None):
        import torch
        from . import binding as pb
        self._pb, self.heads, self.kv_heads, self.head_dim = pb, heads, kv_heads, head_dim
        rand = lambda *shape: torch.randn(shape, generator=generator, device="cuda")  # noqa: E731
        self.norm = (1 + 0.1 * rand(hidden)).bfloat16()
        rows, width = (heads + 2 * kv_heads) * head_dim, heads * head_dim
        self.qkv = pb.Q4Layer(rows, hidden, group, *quantize_q4(rand(rows, hidden) / hidden ** 0.5, group))
        self.out = pb.Q4Layer(hidden, width, group, *quantize_q4(rand(hidden, width) / width ** 0.5, group))
        self.inv_freq = (theta ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).float().cuda()
        self.cache = pb.PagedCache.empty(pages, page_size, kv_heads, head_dim, torch.float8_e4m3fn if cache_dtype is None else cache_dtype)

    def step(self, a, h, requests: PagedRequests, eps: float = 1e-6):
        """(a, h) -> (a, h) for one new token of each request, planned by requests.begin; bfloat16 [requests][hidden], h in place."""
        pb, plan = self._pb, requests.plan
        q, s, _ = pb.pp_rmsnorm_q8(a, self.norm, residual=h, eps=eps, group=128, hidden_out=h)
        qkv = pb.pp_q4_forward(self.qkv, q, x_scales=s, out_dtype=a.dtype).view(a.shape[0], -1, self.head_dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        pb.pp_kv_append(self.cache, k, v, plan.slots, q=q, positions=plan.positions, inv_freq=self.inv_freq, out=q)
        o = pb.pp_paged_attention(self.cache, q, requests.table, plan.lengths)
        return pb.pp_q4_forward(self.out, o.flatten(1), out_dtype=a.dtype), h


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--inner", type=int, default=1024)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--top-k", type=int, default=8)
    ap.add_argument("--weights", default="q4", choices=["q4", "bf16"])
    ap.add_argument("--tokens", type=int, default=1)
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--heads", type=int, default=0, help="query heads of an attention half in front of each block (0: none)")
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--context", type=int, default=1000, help="tokens that each request's cache holds at the start")
    ap.add_argument("--page", type=int, default=16)
    args = ap.parse_args()

    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    blocks = [DecodeBlock(args.hidden, args.inner, args.experts, args.top_k, args.tokens, args.weights, generator=gen)
              for _ in range(args.layers)]
    a0 = torch.randn(args.tokens, args.hidden, generator=gen, device="cuda").bfloat16()
    h = torch.zeros_like(a0)

    attention, requests = [], None
    if args.heads:
        # one token of each request a step: the warm-up, the capture's replays, and the caches' tokens before them
        width = -(-(args.context + args.steps + 8) // args.page)
        requests = PagedRequests(args.tokens, width, args.tokens * width, args.page, args.tokens)
        attention = [DecodeAttention(args.hidden, args.heads, args.kv_heads, args.head_dim, args.tokens * width, args.page, generator=gen) for _ in blocks]
        some = torch.randn(args.context, args.kv_heads, args.head_dim, generator=gen, device="cuda").bfloat16()
        fill = PagedRequests(args.tokens, width, args.tokens * width, args.page, args.tokens * args.context)
        fill.table, fill.free = requests.table, requests.free
        plan = fill.begin(torch.full((args.tokens,), args.context, dtype=torch.int32, device="cuda"))
        requests.plan.lengths.copy_(plan.lengths)
        requests.plan.taken.copy_(plan.taken)
        for x in attention:
            for slots in plan.slots.split(args.context):
                blocks[0]._pb.pp_kv_append(x.cache, some, some, slots)
        one = torch.ones(args.tokens, dtype=torch.int32, device="cuda")

    def step():
        h.zero_()
        a = a0
        if requests is not None:
            requests.begin(one)
        for i, b in enumerate(blocks):
            if attention:
                a, _ = attention[i].step(a, h, requests)
            a, _ = b.step(a, h)
        return a

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        graph.replay()
    begin.record()
    for _ in range(args.steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    bad = [b.moe.status() for b in blocks if b.moe.status()]
    if attention:
        print(f"attention of {args.heads} heads over {args.kv_heads} of {args.head_dim}, {args.context} to {int(requests.plan.lengths.max())} tokens a request in "
              f"pages of {args.page}")
    print(f"{args.layers} blocks of {args.hidden} ({args.experts} experts of {args.inner}, {args.top_k} a token, {args.weights}), "
          f"{args.tokens} token(s): {begin.elapsed_time(end) * 1e3 / args.steps:.1f} us a step, "
          f"{begin.elapsed_time(end) * 1e3 / args.steps / args.layers:.1f} us a block; finite: {bool(torch.isfinite(out).all())}; "
          f"status {bad[0] if bad else 0}")


if __name__ == "__main__":
    main()
