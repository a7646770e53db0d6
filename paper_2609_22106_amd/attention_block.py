"""The attention half of a decoder layer on the device path: one fused q/k/v projection and
the output projection in MXFP4, each with the requests' own low-rank adapters beside it, the
norm and rotation of the heads, the paged cache and the attention over it.

    x -> prq_quant_act, prq_gemm, prq_lora        (q, k, v of all rows, float32)
      -> prq_qk_norm_rope                         (q in bf16, k and v into the cache)
      -> prq_tree_attention
      -> prq_quant_act, prq_gemm, prq_lora

A batch's rows may be a chunk of a prompt, a single token or a tree of drafted tokens of
each request, mixed.  Everything that a call needs is allocated beforehand, so a step can be
captured into a HIP graph.

``python -m paper_2609_22106_amd.attention_block`` runs a Qwen3-4B-shaped block: the prompts
of eight requests, then steps that each check a tree of drafted tokens a request, as a
captured graph.  One JSON line each.
"""
from __future__ import annotations

import json
import sys

import numpy as np
import torch

from . import inputs, prq


class Projection:
    """W [N, K] (bf16 bits) in MXFP4 with a residual tail, and the adapters beside it."""

    def __init__(self, W, Xcal, alpha, k_tail, adapters, max_rows, max_requests):
        art = prq.prq_prepare(W, Xcal, alpha, k_tail)
        dev = {k: torch.from_numpy(art[k]).cuda() for k in ("inv_scale_pos", "perm", "Wq", "Wsc")}
        (self.N, self.K), self.k_tail, self.adapters = W.shape, k_tail, adapters
        self.inv_scale, self.perm = dev["inv_scale_pos"], dev["perm"]
        self.W = prq.prq_pack_weight(dev["Wq"], dev["Wsc"])
        K_aug = self.K + k_tail
        self.Aq = torch.empty((max_rows, K_aug // 2), dtype=torch.uint8, device="cuda")
        self.Asc = torch.empty((max_rows, K_aug // 32), dtype=torch.uint8, device="cuda")
        self.Y = torch.empty((max_rows, self.N), dtype=torch.float32, device="cuda")
        # Both workspaces at the largest that any number of rows asks for.
        rows = range(1, max_rows + 1)
        self.ws = torch.zeros(max(prq.prq_gemm_workspace_bytes(m, self.N, K_aug) for m in rows),
                              dtype=torch.uint8, device="cuda")
        self.lora_ws = torch.empty(max(prq.prq_lora_workspace_bytes(m, s, self.N, self.K, adapters.max_rank)
                                       for m in rows for s in range(1, max_requests + 1)),
                                   dtype=torch.uint8, device="cuda")

    def __call__(self, x, batch):
        M = x.shape[0]
        Aq, Asc = prq.prq_quant_act(x, self.K, self.k_tail, self.inv_scale, self.perm, Aq=self.Aq[:M],
                                    Asc=self.Asc[:M])
        Y = prq.prq_gemm(Aq, Asc, self.W, Y=self.Y[:M], workspace=self.ws)
        return prq.prq_lora(x, self.adapters, batch.offsets, batch.adapter, Y, workspace=self.lora_ws)


class Batch:
    """What one call works on: the requests' rows, where they are and what they see.

    requests: [(cached tokens, parents), ...]: row i of a request is the child of its row
    parents[i] (< i; -1: of the last cached token) and sits at that one's position plus one.
    page_table: int32 [requests, pages] (host).  adapter: one per request, -1 for none."""

    def __init__(self, requests, page_table, page_size, adapter):
        rows = [len(parents) for _, parents in requests]
        M, widest = sum(rows), max(rows + [1])
        position, slot = np.zeros(M, np.int32), np.zeros(M, np.int64)
        mask = np.zeros((M, widest), bool)
        row = 0
        for b, (cached, parents) in enumerate(requests):
            for i, parent in enumerate(parents):
                position[row + i] = (position[row + parent] if parent >= 0 else cached - 1) + 1
                at = cached + i
                slot[row + i] = int(page_table[b, at // page_size]) * page_size + at % page_size
                if parent >= 0:
                    mask[row + i] = mask[row + parent]
                mask[row + i, i] = True
            row += rows[b]
        chains = all(list(parents) == list(range(-1, len(parents) - 1)) for _, parents in requests)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()     # noqa: E731
        self.M, self.position, self.slot = M, dev(position), dev(slot)
        self.mask = None if chains else dev(mask)
        self.pages = dev(np.asarray(page_table, np.int32))
        self.cached = dev(np.array([c for c, _ in requests], np.int32))
        self.offsets = dev(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))
        self.adapter = dev(np.asarray(adapter, np.int32))


class AttentionBlock:
    """heads query heads of the cache's size over the cache's kv heads."""

    def __init__(self, qkv, o, heads, cache, table, q_weight, k_weight, max_rows, max_requests, max_kv_len):
        self.qkv, self.o, self.heads, self.cache, self.table = qkv, o, heads, cache, table
        self.q_weight, self.k_weight, self.max_kv_len = q_weight, k_weight, max_kv_len
        self.scale = cache.D ** -0.5
        self.q = torch.empty((max_rows, heads, cache.D), dtype=torch.bfloat16, device="cuda")
        self.attended = torch.empty_like(self.q)
        self.lse = torch.empty((max_rows, heads), dtype=torch.float32, device="cuda")
        self.ws = torch.zeros(max(prq.prq_tree_attention_workspace_bytes(m, b, heads, cache.heads, cache.D, max_kv_len)
                                  for m in range(1, max_rows + 1) for b in range(1, max_requests + 1)),
                              dtype=torch.uint8, device="cuda")

    def __call__(self, x, batch):
        """x [M, hidden] bf16 -> [M, hidden] float32 (the block's own buffer)."""
        M, q_wide, kv_wide = batch.M, self.heads * self.cache.D, self.cache.heads * self.cache.D
        y = self.qkv(x, batch)
        q = prq.prq_qk_norm_rope(y[:, :q_wide], y[:, q_wide:q_wide + kv_wide], y[:, q_wide + kv_wide:],
                                 batch.position, self.table, self.cache, batch.slot, self.q_weight, self.k_weight,
                                 out=self.q[:M])
        a, _ = prq.prq_tree_attention(q, self.cache, batch.pages, batch.cached, batch.offsets, self.scale, batch.mask,
                                      max_kv_len=self.max_kv_len, out=self.attended[:M], lse=self.lse[:M],
                                      workspace=self.ws)
        return self.o(a.reshape(M, q_wide), batch)


def random_block(rng, hidden, heads, kv_heads, D, pages, page_size, ranks, max_rows, max_requests, positions):
    """A block with random weights and adapters of the given ranks."""
    def projection(N, K):
        W = inputs.f32_to_bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * K ** -0.5)
        Xcal = inputs.f32_to_bf16_bits(rng.standard_normal((32, K), dtype=np.float32))
        pairs = [(torch.from_numpy(rng.standard_normal((r, K), dtype=np.float32) * K ** -0.5),
                  torch.from_numpy(rng.standard_normal((N, r), dtype=np.float32) * r ** -0.5)) for r in ranks]
        return Projection(W, Xcal, 0.5, inputs.tail_width(K), prq.prq_lora_adapters(pairs, [0.5] * len(ranks)),
                          max_rows, max_requests)
    weight = lambda: torch.from_numpy((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)).cuda()  # noqa: E731
    return AttentionBlock(projection((heads + 2 * kv_heads) * D, hidden), projection(hidden, heads * D), heads,
                          prq.prq_paged_kv(pages, kv_heads, page_size, D),
                          prq.prq_rope_table(positions, D, theta=1e6), weight(), weight(), max_rows, max_requests,
                          positions)


def main(argv=None):
    rng = np.random.default_rng(0)
    hidden, heads, kv_heads, D, page_size, B, longest = 2560, 32, 8, 128, 64, 8, 4096
    per = longest // page_size
    tree = [-1, 0, 1, 2, 0, 4, 1, 0]                # the first four: the likeliest path
    prompts = [int(n) for n in rng.integers(100, 500, B)]
    block = random_block(rng, hidden, heads, kv_heads, D, B * per, page_size, [16, 8, 64, 32], sum(prompts), B,
                         longest)
    pages = rng.permutation(B * per).astype(np.int32).reshape(B, per)
    adapter = [int(a) for a in rng.integers(-1, 4, B)]
    x = torch.randn((sum(prompts), hidden), device="cuda").to(torch.bfloat16)

    def timed(run, n=10):
        run()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(n):
            run()
        end.record()
        end.synchronize()
        return round(start.elapsed_time(end) / n * 1e3, 1)

    first = Batch([(0, range(-1, n - 1)) for n in prompts], pages, page_size, adapter)
    us = timed(lambda: block(x, first))
    print(json.dumps({"step": "prompts", "rows": first.M, "us": us}), flush=True)

    # A step's tables are static, so that one graph serves all steps: each takes its first
    # four tokens as accepted, whose keys and values are in the cache already.
    cached = list(prompts)
    batch = Batch([(c, tree) for c in cached], pages, page_size, adapter)
    x = x[:batch.M].clone()
    block(x, batch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block(x, batch)
    for step in range(20):
        now = Batch([(c, tree) for c in cached], pages, page_size, adapter)
        for name in ("position", "slot", "cached"):
            getattr(batch, name).copy_(getattr(now, name))
        x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        cached = [c + 4 for c in cached]
    assert torch.isfinite(y).all()
    print(json.dumps({"step": "trees", "requests": B, "rows": batch.M, "cached_tokens": sum(cached),
                      "us": timed(graph.replay)}), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
