"""Example: the feed-forward half of a decoding step, on the library's decoder operators.

    python -m paper_1712_01084_b200.decode_block --hidden 2048 --tokens 1 --layers 8 --steps 20

A block adds its input to the residual stream, normalises it to 8 bits, multiplies the 8-bit rows with a 4-bit matrix, adds
and normalises again, and runs a mixture-of-experts layer on the result:

    q, s, h    = pp_rmsnorm_q8(a, w1, residual=h)              # h += a
    p          = pp_q4_forward(dense, q, x_scales=s)
    q, s, h, n = pp_rmsnorm_q8(p, w2, residual=h, normed=True) # h += p
    a          = pp_moe_forward(moe, n)

Four kernels a block, none of which waits for the host; the command captures a step over all layers in a CUDA graph and
prints its time.  Weights are random; ``quantize_q4`` rounds float weights to codes and scales in plain torch operations,
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
    args = ap.parse_args()

    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    blocks = [DecodeBlock(args.hidden, args.inner, args.experts, args.top_k, args.tokens, args.weights, generator=gen)
              for _ in range(args.layers)]
    a0 = torch.randn(args.tokens, args.hidden, generator=gen, device="cuda").bfloat16()
    h = torch.zeros_like(a0)

    def step():
        h.zero_()
        a = a0
        for b in blocks:
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
    print(f"{args.layers} blocks of {args.hidden} ({args.experts} experts of {args.inner}, {args.top_k} a token, {args.weights}), "
          f"{args.tokens} token(s): {begin.elapsed_time(end) * 1e3 / args.steps:.1f} us a step, "
          f"{begin.elapsed_time(end) * 1e3 / args.steps / args.layers:.1f} us a block; finite: {bool(torch.isfinite(out).all())}; "
          f"status {bad[0] if bad else 0}")


if __name__ == "__main__":
    main()
