"""Both ends of a split model's hand-over, with the cache's operators: the sender prefills prompts of several lengths into
its own 8-bit caches (one a layer), reads the keys and values back, compresses them (TS + TAB-Q, one blob for all layers)
and sends the blob; the receiver restores it, stores the rows in caches of its own - other blocks, another block size -
and goes on with single tokens, next to the sender doing the same, so that the two can be compared.

    python -m paper_2511_04002_amd.serve [--requests 8] [--prompt 700] [--layers 4] [--steps 32] [--dtype bf16]

The layers are attention blocks with random weights (norm of queries and keys, rotation, attention, output projection,
residual): what is measured is the operators, not a model's answers.
"""
from __future__ import annotations

import argparse
import json
from typing import Dict, List


class Side:
    """One end: a cache for each layer, which share one block table, and the steps over them."""

    def __init__(self, model: "Layers", requests: int, longest: int, block: int):
        from . import cache
        self.m, self.requests = model, requests
        each = -(-longest // block)
        self.c = cache.Cache(requests * each, block, model.q_heads, model.kv_heads, model.dim, model.dtype, each)
        self.memory = [self.c.new_memory() for _ in model.qkv]
        self.table, self.ring = self.c.new_table(requests), self.c.new_ring()
        self.lengths, self.counters = self.c.new_lengths(requests), self.c.new_counters()

    def schedule(self, new: List[int]):
        """Places for new[r] more tokens of each request."""
        import torch
        s = self.c.new_schedule(self.requests, max(1, sum(new)))
        self.c.schedule(torch.tensor(new, dtype=torch.int32, device="cuda"), self.lengths, self.table, self.ring, self.counters, s)
        self.lengths, self.counters = s.lengths, s.counters
        return s

    def step(self, x, s, max_new: int, max_length: int):
        """x [tokens, hidden]: the tokens that were scheduled as s, through all layers."""
        m, c = self.m, self.c
        for memory, w_qkv, w_out in zip(self.memory, m.qkv, m.out):
            qkv = x @ w_qkv
            q, k = qkv[:, :m.q_width], qkv[:, m.q_width:m.q_width + m.kv_width]
            q, k = c.norm_rotate(q, k, s.positions, m.angles, m.weight, m.weight)
            c.append(memory, k, qkv[:, m.q_width + m.kv_width:], s.slots)
            x = x + c.attend(memory, q, self.table, s.starts, s.lengths, max_new, max_length).flatten(1) @ w_out
        return x

    def rows(self, s, tokens: int):
        """Keys and values of the tokens scheduled as s, layer after layer, as the compressor takes them."""
        import torch
        out = []
        for memory in self.memory:
            k, v = (torch.empty((tokens, self.m.kv_width), dtype=self.c.kind, device="cuda") for _ in range(2))
            self.c.gather(memory, self.table, s.starts, s.lengths, k, v)
            out += [k, v]
        return out

    def store(self, rows, s) -> None:
        for i, memory in enumerate(self.memory):
            self.c.append(memory, rows[2 * i], rows[2 * i + 1], s.slots)


class Layers:
    """Random weights of the attention blocks."""

    def __init__(self, layers: int, q_heads: int, kv_heads: int, dim: int, dtype: str, longest: int, seed: int = 0):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        kind = torch.float16 if dtype == "f16" else torch.bfloat16
        self.q_heads, self.kv_heads, self.dim, self.dtype = q_heads, kv_heads, dim, dtype
        self.q_width, self.kv_width = q_heads * dim, kv_heads * dim
        hidden = self.q_width

        def randn(*shape, scale):
            return (torch.randn(shape, device="cuda", generator=g) * scale).to(kind)

        self.qkv = [randn(hidden, hidden + 2 * self.kv_width, scale=hidden ** -0.5) for _ in range(layers)]
        self.out = [randn(hidden, hidden, scale=hidden ** -0.5) for _ in range(layers)]
        self.weight = (1 + randn(dim, scale=0.1).float()).to(kind)
        rate = 10000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * rate
        self.angles = torch.cat((angle.cos(), angle.sin()), 1).float()
        self.generator, self.randn = g, randn


def run(requests: int = 8, prompt: int = 700, layers: int = 4, steps: int = 32, q_heads: int = 32, kv_heads: int = 8,
        dim: int = 128, dtype: str = "bf16", bits=(4, 6, 8), budget: float = 0.01, seed: int = 0) -> Dict[str, float]:
    """-> what was sent, and how far the receiver's steps are from the sender's."""
    import torch

    from . import tsq
    longest = prompt + steps
    prompts = [max(1, prompt * (r + 1) // requests) for r in range(requests)]
    total = sum(prompts)
    m = Layers(layers, q_heads, kv_heads, dim, dtype, longest, seed)
    sender, receiver = Side(m, requests, longest, 16), Side(m, requests, longest, 32)

    s = sender.schedule(prompts)
    sender.step(m.randn(total, m.q_width, scale=1.0), s, max(prompts), max(prompts))
    rows = sender.rows(s, total)
    plan = tsq.Plan(2 * layers * total, m.kv_width, dtype, 8.0, bits, budget)
    blob, _ = plan.compress_batch(rows)
    restored = [torch.empty_like(x) for x in rows]
    plan.decompress_batch(blob, restored)
    receiver.store(restored, receiver.schedule(prompts))
    sent = plan.info(blob).compressed_bytes

    worst, times = 0.0, []
    for i in range(steps):
        x = m.randn(requests, m.q_width, scale=1.0)
        want = sender.step(x, sender.schedule([1] * requests), 1, longest)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        got = receiver.step(x, receiver.schedule([1] * requests), 1, longest)
        end.record()
        worst = max(worst, float((got.float() - want.float()).norm() / (want - x).float().norm()))
        times.append(begin.elapsed_time(end) * 1e3)
    assert torch.equal(sender.lengths, receiver.lengths)
    return {"requests": requests, "tokens_sent": total, "layers": layers, "cache_bytes": 2 * layers * total * m.kv_width * 2, "sent_bytes": int(sent),
            "relative_difference": worst, "step_us": sorted(times)[len(times) // 2] if times else 0.0}


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("requests", 8), ("prompt", 700), ("layers", 4), ("steps", 32), ("q-heads", 32), ("kv-heads", 8), ("dim", 128)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--dtype", choices=("f16", "bf16"), default="bf16")
    a = p.parse_args()
    print(json.dumps(run(a.requests, a.prompt, a.layers, a.steps, a.q_heads, a.kv_heads, a.dim, a.dtype)))


if __name__ == "__main__":
    main()
