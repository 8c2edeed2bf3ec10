"""An agent's decode loop on a long history: projection, head norms and rotation,
append, attention over selected pages, eviction.

    python examples/sparse_decode.py [--tokens 60000] [--steps 20] [--top 64] [--layers 4]

A stack of attention layers with random weights stands in for a model.  The history goes into the
cache in turns of a thousand tokens; then the same tokens are decoded with every page attended and with
`--top` pages per layer and KV head, and both runs evict to the same budget."""
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


class Agent:
    """Attention layers over one cache of one sequence."""

    def __init__(self, layers, tokens, page=32, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return torch.randn(shape, generator=g, device="cuda").bfloat16() / shape[0] ** 0.5

        self.layers = layers
        self.qkv = [weight(HIDDEN, (HQ + 2 * HKV) * D) for _ in range(layers)]
        self.proj = [weight(HQ * D, HIDDEN) for _ in range(layers)]
        self.norm = torch.ones((layers, 2, D), device="cuda") * 1.5
        self.table = md.md_rope_table(np.exp(np.arange(D // 2) * (-np.log(1e6) / (D // 2))), tokens + 4096)
        pages = tokens // page + 160
        self.cache = md.Cache(layers, HQ, HKV, page, 1, pages, pages)
        self.cache.set_region_params(md.MD_REGION_SYSTEM, 1.0, 160.0, True)
        for r in range(1, md.MD_NUM_REGIONS):
            self.cache.set_region_params(r, 1.0 - 0.12 * r, 20.0 * r, False)
        self.seen = 0

    def rows(self, layer, x, q, k, v):
        """The layer's query, key and value rows of x, at the next positions."""
        T = x.shape[0]
        qkv = (x @ self.qkv[layer]).view(T, HQ + 2 * HKV, D)
        pos = torch.arange(self.seen, self.seen + T, dtype=torch.int32, device="cuda")
        md.md_norm_rope(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], q, k, v, positions=pos, table=self.table,
                        q_weight=self.norm[layer, 0], k_weight=self.norm[layer, 1])

    def read(self, x, region):
        """Appends a turn (a prompt, a tool's output) to the cache.  Its hidden states are taken as
        they are at every layer: a prompt's own attention is the model's business."""
        T = x.shape[0]
        k, v = (torch.empty((self.layers, HKV, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q = torch.empty((T, HQ, D), dtype=torch.bfloat16, device="cuda")
        for l in range(self.layers):
            self.rows(l, x, q, k[l].transpose(0, 1), v[l].transpose(0, 1))
        self.cache.append_tokens(0, np.full(T, region, np.uint8), k, v)
        self.seen += T

    def step(self, x):
        """One new token through all layers."""
        label = np.array([md.MD_REGION_SCRATCHPAD], np.uint8)
        q, o = (torch.empty((1, HQ, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        k, v = (torch.empty((1, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for l in range(self.layers):
            self.rows(l, x, q, k, v)
            self.cache.decode_layer(l, 1, q, k, v, label, o)
            x = x + o.view(1, HQ * D) @ self.proj[l]
        self.seen += 1
        return x / x.float().square().mean().sqrt().bfloat16()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=60000)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--top", type=int, default=64, help="pages attended per layer and KV head")
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args(argv)
    result = {}
    for top in (0, a.top):
        agent = Agent(a.layers, a.tokens)
        agent.cache.sparse_enable(top)
        g = torch.Generator(device="cuda").manual_seed(1)
        turn = 0
        while agent.seen < a.tokens:
            n = min(1000, a.tokens - agent.seen)
            agent.read(torch.randn((n, HIDDEN), generator=g, device="cuda").bfloat16(),
                       md.MD_REGION_SYSTEM if turn == 0 else 1 + turn % 5)
            turn += 1
        budget = [agent.cache.query(md.MD_QUERY_PAGES)]
        x = torch.randn((1, HIDDEN), generator=g, device="cuda").bfloat16()
        for i in range(a.steps + 3):
            if i == 3:
                torch.cuda.synchronize()
                t = time.perf_counter()
            x = agent.step(x)
            agent.cache.evict(budget)
        assert agent.cache.sync() == md.MD_OK
        result[top] = (time.perf_counter() - t) / a.steps
        print(f"{'all pages' if top == 0 else f'{top} pages':>10}: {1e6 * result[top]:8.1f} us per step, "
              f"{agent.cache.query(md.MD_QUERY_TOKENS)} tokens cached, |x| {float(x.float().norm()):.4f}")
        agent.cache.close()
    return result


if __name__ == "__main__":
    main()
