"""Agents decoding on long histories: projection, head norms and rotation, append,
attention over selected pages, eviction.

    python examples/sparse_decode.py [--agents 16] [--tokens 60000] [--steps 20] [--top 64] [--layers 4]

A stack of attention layers with random weights stands in for a model.  Every agent's history goes into
the cache in turns of a thousand tokens; then a token per agent and step is decoded, once with every page
attended and once with `--top` pages per layer and KV head, and both runs evict back to the same budget."""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_10582_gb300 as md  # noqa: E402

HQ, HKV, D = 16, 2, 128
HIDDEN = 1024


class Model:
    """Attention layers over one cache."""

    def __init__(self, agents, layers, tokens, page=32, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return torch.randn(shape, generator=g, device="cuda").bfloat16() / shape[0] ** 0.5

        self.agents, self.layers = agents, layers
        self.qkv = [weight(HIDDEN, (HQ + 2 * HKV) * D) for _ in range(layers)]
        self.proj = [weight(HQ * D, HIDDEN) for _ in range(layers)]
        self.norm = torch.ones((layers, 2, D), device="cuda") * 1.5
        self.table = md.md_rope_table(np.exp(np.arange(D // 2) * (-np.log(1e6) / (D // 2))), tokens + 4096)
        pages = tokens // page + 160
        self.cache = md.Cache(layers, HQ, HKV, page, agents, pages, agents * pages)
        self.cache.set_region_params(md.MD_REGION_SYSTEM, 1.0, 160.0, True)
        for r in range(1, md.MD_NUM_REGIONS):
            self.cache.set_region_params(r, 1.0 - 0.12 * r, 20.0 * r, False)
        self.labels = np.full(agents, md.MD_REGION_SCRATCHPAD, np.uint8)
        self.seen = 0

    def rows(self, layer, x, positions, q, k, v):
        """The layer's query, key and value rows of x, from one projection."""
        qkv = (x @ self.qkv[layer]).view(x.shape[0], HQ + 2 * HKV, D)
        md.md_norm_rope(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], q, k, v, positions=positions,
                        table=self.table, q_weight=self.norm[layer, 0], k_weight=self.norm[layer, 1])

    def read(self, agent, x, region, first):
        """Appends a turn (a prompt, a tool's output) of one agent, at positions first, first + 1, ...
        Its hidden states are taken as they are at every layer: a prompt's own attention is the
        model's business."""
        T = x.shape[0]
        k, v = (torch.empty((self.layers, HKV, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q = torch.empty((T, HQ, D), dtype=torch.bfloat16, device="cuda")
        positions = torch.arange(first, first + T, dtype=torch.int32, device="cuda")
        for l in range(self.layers):
            self.rows(l, x, positions, q, k[l].transpose(0, 1), v[l].transpose(0, 1))
        self.cache.append_tokens(agent, np.full(T, region, np.uint8), k, v)

    def step(self, x):
        """One new token per agent through all layers."""
        B = self.agents
        positions = torch.full((B,), self.seen, dtype=torch.int32, device="cuda")
        q, o = (torch.empty((B, HQ, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        k, v = (torch.empty((B, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for l in range(self.layers):
            self.rows(l, x, positions, q, k, v)
            self.cache.decode_layer(l, B, q, k, v, self.labels, o)
            x = torch.addmm(x, o.view(B, HQ * D), self.proj[l])
        self.seen += 1
        return torch.nn.functional.layer_norm(x, (HIDDEN,))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--agents", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=60000, help="history of each agent")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--top", type=int, default=64, help="pages attended per layer and KV head")
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args(argv)
    result = {}
    for top in (0, a.top):
        model = Model(a.agents, a.layers, a.tokens)
        model.cache.sparse_enable(top)
        g = torch.Generator(device="cuda").manual_seed(1)
        for agent in range(a.agents):
            for turn, first in enumerate(range(0, a.tokens, 1000)):
                x = torch.randn((min(1000, a.tokens - first), HIDDEN), generator=g, device="cuda").bfloat16()
                model.read(agent, x, md.MD_REGION_SYSTEM if turn == 0 else 1 + turn % 5, first)
        model.seen = a.tokens
        budget = np.array([model.cache.query(md.MD_QUERY_PAGES, b) for b in range(a.agents)], np.int32)
        x = torch.randn((a.agents, HIDDEN), generator=g, device="cuda").bfloat16()
        for i in range(a.steps + 3):
            if i == 3:
                torch.cuda.synchronize()
                t = time.perf_counter()
            x = model.step(x)
            model.cache.evict(budget)
        assert model.cache.sync() == md.MD_OK
        result[top] = (time.perf_counter() - t) / a.steps
        cached = sum(model.cache.query(md.MD_QUERY_TOKENS, b) for b in range(a.agents))
        print(f"{'all pages' if top == 0 else f'{top} pages':>10}: {1e6 * result[top]:8.1f} us per step, "
              f"{cached} tokens cached, |x| {float(x.float().norm()):.3f}")
        model.cache.close()
    return result


if __name__ == "__main__":
    main()
