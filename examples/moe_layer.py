"""A mixture-of-experts layer over P ranks, one expert a rank, and its decode step.

Prefill: every rank routes its tokens; the rows travel to their experts through the
non-uniform all-to-all (gathered from token order on the way); the experts run on them in
8-bit products; the rows travel back and are summed with their weights.

    route -> update_counts_device, set_row_maps -> rows_alltoallv -> expert_rows -> alltoallv -> combine

Decode: the same layer for a handful of tokens in one launch (``few``).

    python examples/moe_layer.py [--ranks 64] [--tokens 512] [--hidden 4096] [--inter 2048] [--k 2]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_02581_b200 import binding as B  # noqa: E402
from paper_2411_02581_b200 import moe  # noqa: E402


class Layer:
    """Weights in 8 bits, a router in bf16, and the two exchanges' plans."""

    def __init__(self, ranks, hidden, inter, k, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape: torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5  # noqa: E731
        self.ranks, self.hidden, self.inter, self.k = ranks, hidden, inter, k
        self.router = new(ranks, hidden).to(torch.bfloat16)
        tiles = lambda m: moe.fp8_quantize(m, "tiles")  # noqa: E731
        up = [tiles(new(inter, hidden)) for _ in range(2 * ranks)]
        down = [tiles(new(hidden, inter)) for _ in range(ranks)]
        stack = lambda parts: torch.stack([p.contiguous().view(torch.uint8) for p in parts]).view(torch.float8_e4m3fn)  # noqa: E731
        self.w13 = stack([q for q, _ in up]).view(ranks, 2, inter, hidden)
        self.s13 = torch.stack([s for _, s in up]).view(ranks, 2, *up[0][1].shape)
        self.w2, self.s2 = stack([q for q, _ in down]), torch.stack([s for _, s in down])
        zero = np.zeros((ranks, ranks), dtype=np.int64)
        # radix `ranks`: one hop; rows are the exchanges' elements
        self.there, self.back = (B.Plan(ranks, max(2, ranks), elem_size=2 * hidden, sendcounts=zero) for _ in range(2))

    def prefill(self, x):
        """x: [ranks * tokens, hidden] bf16, rank after rank."""
        r = moe.route(x.float() @ self.router.float().t(), self.k, renormalize=True, ranks=self.ranks)
        rows = r.rows.numel()
        self.there.update_counts_device(r.counts)
        self.there.set_row_maps(r.rows, None, x.shape[0], rows)
        arrived = torch.empty(rows, self.hidden, dtype=torch.bfloat16, device=x.device)
        self.there.rows_alltoallv(x, arrived)
        offsets = torch.zeros(self.ranks + 1, dtype=torch.int64, device=x.device)
        offsets[1:] = r.counts.sum(0).cumsum(0)
        y = moe.expert_rows(arrived, offsets, self.w13, self.s13, self.w2, self.s2)
        self.back.update_counts_device(r.counts.t().contiguous())
        self.back.alloc_workspace()
        home = torch.empty_like(y)
        self.back.alltoallv(y, home)
        return moe.combine(home, r.weights, r.pos), r

    def decode(self, x):
        """x: [at most 64 tokens, hidden] bf16."""
        return moe.few(x, self.router, self.k, self.w13, self.w2, s13=self.s13, s2=self.s2, renormalize=True)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("ranks", 64), ("tokens", 512), ("hidden", 4096), ("inter", 2048), ("k", 2)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    layer = Layer(a.ranks, a.hidden, a.inter, a.k)
    x = torch.randn(a.ranks * a.tokens, a.hidden, device="cuda").to(torch.bfloat16)
    out, r = layer.prefill(x)
    same = moe.experts(x, r.ids, r.weights, layer.w13, layer.s13, layer.w2, layer.s2)
    few = layer.decode(x[:8])
    near = float((few.float() - out[:8].float()).norm() / out[:8].float().norm())
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    times = []
    for f in (lambda: layer.prefill(x), lambda: layer.decode(x[:8])):
        f()
        start.record()
        for _ in range(5):
            f()
        end.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(end) / 5)
    print(f"prefill of {a.ranks} x {a.tokens} tokens {times[0]:.3f} ms, decode of 8 tokens {times[1]:.3f} ms; "
          f"dispatched rows give {'the same' if torch.equal(out, same) else 'ANOTHER'} result as the experts in place; "
          f"8-bit rows against 16-bit ones differ by {near:.3f}")
    return torch.equal(out, same), near


if __name__ == "__main__":
    main()
