"""The mixture-of-experts half of a decoder layer on the device path, behind the attention half
(attention_block.py): the norm between them with the residual sum, the router, the experts and the norm
before the next layer.

    y, r -> prq_block_norm        (r + y, and its norm h)
         -> prq_moe_route         (experts and weights of every token)
         -> prq_moe_layer         (all experts, 64 tokens at a time)
         -> prq_block_norm        (the residual again, and the next layer's input)

Everything that a call needs is allocated beforehand, so a step can be captured into a HIP graph.

``python -m paper_2609_22106_amd.moe_block`` runs a Qwen3-30B-A3B-shaped decoder layer with random
weights: steps of one and of 64 sequences, as captured graphs.  One JSON line each.
"""
from __future__ import annotations

import json
import sys

import numpy as np
import torch

from . import attention_block, inputs, prq

STEP = 64                                      # tokens of one prq_moe_layer call


class MoEBlock:
    """router [E, hidden] bf16; gate_up: PackedWeight of E weights [2 I, hidden]; down: of E weights
    [hidden, I + k_tail]; norm_weight and next_weight [hidden]: of the norms before this half and before
    the next layer.  Further keywords go to prq_moe_route (scoring, bias, renormalize, scale)."""

    def __init__(self, router, gate_up, down, k, k_tail, norm_weight, next_weight, max_rows, eps=1e-6, **routing):
        self.router, self.gate_up, self.down, self.k, self.k_tail = router, gate_up, down, k, k_tail
        self.norm_weight, self.next_weight, self.eps, self.routing = norm_weight, next_weight, eps, routing
        E, hidden = router.shape
        new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")       # noqa: E731
        self.h, self.out, self.next = (new(max_rows, hidden) for _ in range(3))
        self.ids, self.weights = new(max_rows, k, dtype=torch.int32), new(max_rows, k, dtype=torch.float32)
        I = down.K_aug - k_tail
        # One workspace for both calls, at the largest that any number of rows asks for.
        self.ws = torch.zeros(max([prq.prq_moe_route_workspace_bytes(m, E, hidden) for m in range(1, max_rows + 1)]
                                  + [prq.prq_moe_layer_workspace_bytes(m, k, E, hidden, I, k_tail, down.N)
                                     for m in range(1, min(max_rows, STEP) + 1)]), dtype=torch.uint8, device="cuda")

    def experts(self, h):
        """h [M, hidden] bf16 -> the experts' weighted sum [M, hidden] bf16 (the block's own buffer)."""
        M = h.shape[0]
        ids, weights = prq.prq_moe_route(h, self.router, self.k, ids=self.ids[:M], weights=self.weights[:M],
                                         workspace=self.ws, **self.routing)
        for i in range(0, M, STEP):
            rows = slice(i, min(i + STEP, M))
            prq.prq_moe_layer(h[rows], ids[rows], weights[rows], self.gate_up, self.down, k_tail=self.k_tail,
                              out=self.out[rows], workspace=self.ws)
        return self.out[:M]

    def __call__(self, y, residual):
        """y [M, hidden], the attention half's output, and the residual, updated in place -> the next
        layer's input [M, hidden] bf16 (the block's own buffer)."""
        M = y.shape[0]
        h, _ = prq.prq_block_norm(y, residual, self.norm_weight, eps=self.eps, out=self.h[:M])
        return prq.prq_block_norm(self.experts(h), residual, self.next_weight, eps=self.eps, out=self.next[:M])[0]


def random_experts(rng, E, N, K):
    """PackedWeight of E weights [N, K] of random MXFP4 values of a spread near K^-1/2."""
    code = 127 - int(round(np.log2(K) / 2)) - 1
    q, s = inputs.random_mxfp4(rng, (E, N), K, code - 1, code)
    return prq.prq_pack_weight(torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda())


def random_block(rng, hidden, E, k, I, k_tail, max_rows, **routing):
    weight = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).cuda()       # noqa: E731
    return MoEBlock((weight(E, hidden) * hidden ** -0.5).bfloat16(), random_experts(rng, E, 2 * I, hidden),
                    random_experts(rng, E, hidden, I + k_tail), k, k_tail, 1 + 0.1 * weight(hidden),
                    1 + 0.1 * weight(hidden), max_rows, **routing)


def main(argv=None):
    rng = np.random.default_rng(0)
    hidden, heads, kv_heads, D, page_size, B, longest = 2048, 32, 4, 128, 64, 64, 2048
    E, k, I, k_tail = 128, 8, 768, 64
    per = longest // page_size
    attention = attention_block.random_block(rng, hidden, heads, kv_heads, D, B * per, page_size, [16, 8], B, B, longest)
    moe = random_block(rng, hidden, E, k, I, k_tail, B)
    pages = rng.permutation(B * per).astype(np.int32).reshape(B, per)
    cached = [int(n) for n in rng.integers(100, longest - 1, B)]
    adapter = [int(a) for a in rng.integers(-1, 2, B)]
    for n in (1, B):
        batch = attention_block.Batch([(c, [-1]) for c in cached[:n]], pages[:n], page_size, adapter[:n])
        x = torch.randn((n, hidden), device="cuda").bfloat16()
        residual = torch.randn((n, hidden), device="cuda")
        # (one sequence's rows and 64's take other kernels: both before a capture)
        moe(attention(x, batch), residual)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = moe(attention(x, batch), residual)
        events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        graph.replay()
        events[0].record()
        for _ in range(20):
            graph.replay()
        events[1].record()
        events[1].synchronize()
        assert torch.isfinite(out).all()
        print(json.dumps({"step": "decode", "sequences": n, "experts": E, "cached_tokens": sum(cached[:n]),
                          "us": round(events[0].elapsed_time(events[1]) / 20 * 1e3, 1)}), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
