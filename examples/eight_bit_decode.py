"""Agents decoding on caches in eight bits, every other layer under a sliding window: projection, head
norms and rotation, quantised append, attention.

    python examples/eight_bit_decode.py [--agents 16] [--tokens 60000] [--steps 20] [--layers 4] [--window 4096]

A stack of attention layers with random weights stands in for a model.  The caller owns the cache: a pool of
pages, their scales and a block table.  Histories go in as prompts; then a token per agent and step is decoded, and
in the end the last tokens are read back from the cache and compared with the rows that went in."""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_10582_gb300 as md  # noqa: E402

HQ, HKV, D = 16, 2, 128
HIDDEN, PAGE, SINKS = 1024, 32, 4


class Model:
    """Attention layers over one cache in eight bits."""

    def __init__(self, agents, layers, tokens, window, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return torch.randn(shape, generator=g, device="cuda").bfloat16() / shape[0] ** 0.5

        self.agents, self.layers, self.window = agents, layers, window
        self.qkv = [weight(HIDDEN, (HQ + 2 * HKV) * D) for _ in range(layers)]
        self.proj = [weight(HQ * D, HIDDEN) for _ in range(layers)]
        self.norm = torch.ones((layers, 2, D), device="cuda") * 1.5
        self.rope = md.md_rope_table(np.exp(np.arange(D // 2) * (-np.log(1e6) / (D // 2))), tokens)
        pages = -(-tokens // PAGE)
        self.table = torch.randperm(agents * pages, generator=g, device="cuda").int().view(agents, pages)
        self.pool = torch.empty((layers, agents * pages, HKV, 2, PAGE, D), dtype=torch.float8_e4m3fn, device="cuda")
        self.scales = torch.empty((layers, agents * pages, HKV, 2, PAGE // md.MD_SCALE_TOKENS), device="cuda")
        self.workspace = torch.empty(md.MD_ATTEND_WORKSPACE, dtype=torch.uint8, device="cuda")
        self.n = np.zeros(agents, np.int32)                      # cached tokens per agent

    def rows(self, layer, x, positions):
        """The layer's query, key and value rows of x, from one projection."""
        T = x.shape[0]
        q = torch.empty((T, HQ, D), dtype=torch.bfloat16, device="cuda")
        k, v = (torch.empty((T, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        qkv = (x @ self.qkv[layer]).view(T, HQ + 2 * HKV, D)
        md.md_norm_rope(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], q, k, v, positions=positions,
                        table=self.rope, q_weight=self.norm[layer, 0], k_weight=self.norm[layer, 1])
        return q, k, v

    def write(self, layer, k, v, count):
        one = slice(layer, layer + 1)
        md.md_write_cache8(k[:, None], v[:, None], self.pool[one], self.scales[one], self.table, self.n, count)

    def read(self, x, count):
        """Appends a prompt per agent: x holds their tokens one after the other.  Its hidden states are taken
        as they are at every layer: a prompt's own attention is the model's business."""
        positions = np.concatenate([np.arange(n, n + c) for n, c in zip(self.n, count)]).astype(np.int32)
        positions = torch.from_numpy(positions).cuda()
        for l in range(self.layers):
            _, k, v = self.rows(l, x, positions)
            self.write(l, k, v, count)
        self.n = self.n + count

    def step(self, x):
        """One new token per agent through all layers; the new rows of the last one."""
        positions, count = torch.from_numpy(self.n).cuda(), np.ones(self.agents, np.int32)
        for l in range(self.layers):
            q, k, v = self.rows(l, x, positions)
            self.write(l, k, v, count)
            o = torch.empty_like(q)
            md.md_attend_cache(q[:, None], self.pool[l:l + 1], self.table, self.n + count, o[:, None],
                               scales=self.scales[l:l + 1], window=self.window if l % 2 else None, sinks=SINKS,
                               workspace=self.workspace)
            x = torch.addmm(x, o.view(self.agents, HQ * D), self.proj[l])
        self.n = self.n + count
        return torch.nn.functional.layer_norm(x, (HIDDEN,)), k, v


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--agents", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=60000, help="history of the longest agent")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--window", type=int, default=4096)
    a = ap.parse_args(argv)
    model = Model(a.agents, a.layers, a.tokens + a.steps + 3, a.window)
    g = torch.Generator(device="cuda").manual_seed(1)
    left = np.linspace(a.tokens, a.tokens // 2, a.agents).astype(np.int32)     # agents' histories differ
    while left.any():
        count = np.minimum(left, 1000).astype(np.int32)
        model.read(torch.randn((int(count.sum()), HIDDEN), generator=g, device="cuda").bfloat16(), count)
        left = left - count
    x = torch.randn((a.agents, HIDDEN), generator=g, device="cuda").bfloat16()
    for i in range(a.steps + 3):
        if i == 3:
            torch.cuda.synchronize()
            t = time.perf_counter()
        x, k, v = model.step(x)
    torch.cuda.synchronize()
    per_step = (time.perf_counter() - t) / a.steps
    # the last tokens' rows of the last layer, back from the cache
    back = [torch.empty_like(y) for y in (k, v)]
    last = slice(a.layers - 1, a.layers)
    md.md_read_cache8(back[0][:, None], back[1][:, None], model.pool[last], model.scales[last], model.table, model.n - 1,
                      np.ones(a.agents, np.int32))
    off = max(float((b.float() - y.float()).norm() / y.float().norm()) for b, y in zip(back, (k, v)))
    print(f"{1e6 * per_step:8.1f} us per step, {int(model.n.sum())} tokens in {model.pool.nbytes + model.scales.nbytes} bytes, "
          f"rows off by {off:.4f}, |x| {float(x.float().norm()):.3f}")
    return off


if __name__ == "__main__":
    main()
