#!/usr/bin/env python3
"""A model instance's step on the card, and the profile that the placer decides from.

A small decoder of random weights serves `level` requests behind one prompt: the prompt's pages are shared (fork), each
step grows the rows by a token (extend, copy on write), writes its keys and values with the heads' norms and the rotation
(append), attends (the shared beginning read once for all), and chooses tokens (penalties, temperature).  A step is
captured into a graph and replayed; nothing goes through the host between steps.  The seconds per step against the load
are what maaso_profile_fit makes the table from that maaso_profile_tables_load takes.

    python examples/measure_instance.py [--layers 4] [--levels 1,2,4,8,16,32,64] [--prompt 900] [--steps 32]
"""
from __future__ import annotations

import argparse
import json
import sys
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

import numpy as np
import torch

from paper_2509_06362_amd import binding, instance as I


class Decoder:
    """Weights of a decoder with grouped heads, head norms and rotation; plain products are torch's."""

    def __init__(self, layers=4, heads=16, kv_heads=4, dim=128, vocab=32000, max_len=4096, dtype=torch.bfloat16, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.layers, self.heads, self.kv_heads, self.dim, self.vocab, self.dtype = layers, heads, kv_heads, dim, vocab, dtype
        self.hidden = hidden = heads * dim

        def weight(out, into):
            return (torch.randn(out, into, generator=g) * into ** -0.5).to(dtype).cuda()

        self.embedding = torch.randn(vocab, hidden, generator=g).to(dtype).cuda()
        self.qkv = [weight((heads + 2 * kv_heads) * dim, hidden) for _ in range(layers)]
        self.out = [weight(hidden, hidden) for _ in range(layers)]
        self.up = [weight(2 * hidden, hidden) for _ in range(layers)]
        self.down = [weight(hidden, 2 * hidden) for _ in range(layers)]
        self.q_norm = [(1 + 0.1 * torch.randn(dim, generator=g)).to(dtype).cuda() for _ in range(layers)]
        self.k_norm = [(1 + 0.1 * torch.randn(dim, generator=g)).to(dtype).cuda() for _ in range(layers)]
        angle = torch.arange(max_len, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()

    def normed(self, x):
        x = x.float()
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)).to(self.dtype)


class Serving:
    """What a program keeps for a running instance: the pages, the cache, and the tensors of a step."""

    def __init__(self, model, rows, pages, page_size=64, width=64):
        m, cuda = model, dict(device="cuda")
        self.model, self.inst = model, I.maaso_instance_create(torch.cuda.current_device())
        self.pages = I.KvPages(torch.zeros(pages, dtype=torch.int32, **cuda), torch.full((rows, width), -1, dtype=torch.int32, **cuda),
                               torch.zeros(rows, dtype=torch.int32, **cuda), page_size)
        self.cache = I.KvCache(torch.zeros(m.layers, pages, m.kv_heads, page_size, m.dim, dtype=m.dtype, **cuda),
                               torch.zeros(m.layers, pages, m.kv_heads, m.dim, page_size, dtype=m.dtype, **cuda))
        self.max_len = width * page_size

    def buffers(self, rows, tokens):
        """The tensors of a step of these rows (a list) with `tokens` new ones each."""
        m, n, cuda = self.model, len(rows), dict(device="cuda")
        total = n * tokens
        return dict(rows=torch.tensor(rows, dtype=torch.int32, **cuda), q_start=torch.arange(0, total + 1, tokens, dtype=torch.int32, **cuda),
                    slot=torch.empty(total, dtype=torch.int64, **cuda), pos=torch.empty(total, dtype=torch.int32, **cuda),
                    copies=torch.empty(n, 2, dtype=torch.int32, **cuda), q=torch.empty(total, m.heads, m.dim, dtype=m.dtype, **cuda),
                    o=torch.empty(total, m.heads, m.dim, dtype=m.dtype, **cuda), last=torch.arange(tokens - 1, total, tokens, **cuda),
                    chosen=torch.empty(n, dtype=torch.int32, **cuda), tokens=tokens)

    def step(self, ids, b, group=None, adjust=None):
        """Logits behind the rows' new tokens `ids`, the chosen tokens in b["chosen"]; group: (group_start, shared, most)."""
        m, inst = self.model, self.inst
        start, shared, most = group or (None, None, 0)
        I.maaso_kv_extend(inst, self.pages, rows=b["rows"], q_start=b["q_start"], slot=b["slot"], pos=b["pos"], copies=b["copies"])
        I.maaso_kv_copy(inst, self.cache, pairs=b["copies"])
        x, wide, side = m.embedding[ids], m.heads * m.dim, m.kv_heads * m.dim
        for layer in range(m.layers):
            qkv = m.normed(x) @ m.qkv[layer].T
            q, k, v = (t.unflatten(1, (-1, m.dim)) for t in (qkv[:, :wide], qkv[:, wide:wide + side], qkv[:, wide + side:]))
            I.maaso_kv_append(inst, self.cache, layer=layer, q=q, k=k, v=v, q_out=b["q"], slot=b["slot"], pos=b["pos"], cos_sin=m.cos_sin,
                              q_weight=m.q_norm[layer], k_weight=m.k_norm[layer])
            I.maaso_kv_attention(inst, self.cache, self.pages, layer=layer, q=b["q"], out=b["o"], q_start=b["q_start"], rows=b["rows"], scale=m.dim ** -0.5,
                                 max_q=b["tokens"], max_len=self.max_len, group_start=start, shared=shared, max_shared=most)
            x = x + b["o"].flatten(1) @ m.out[layer].T
            x = x + torch.relu(m.normed(x) @ m.up[layer].T) @ m.down[layer].T
        logits = m.normed(x[b["last"]]) @ m.embedding.T
        I.maaso_logits_adjust(inst, logits=logits, chosen=b["chosen"], **(adjust or {}))
        return logits


def measure(model, level, prompt, steps, page_size=64):
    """Seconds per step of `level` requests behind one prompt of that many tokens."""
    width = -(-(prompt + steps + 8) // page_size)
    s = Serving(model, level + 1, width + level * (2 + -(-(steps + 8) // page_size)), page_size, width)
    ids = torch.randint(model.vocab, (prompt,), device="cuda", generator=torch.Generator("cuda").manual_seed(level))
    b = s.buffers([0], prompt)
    s.step(ids, b)
    rows = list(range(1, level + 1))
    first, at = b["chosen"], s.buffers(rows, 1)
    I.maaso_kv_fork(s.inst, s.pages, parents=torch.zeros(level, dtype=torch.int32, device="cuda"), children=at["rows"])
    whole = prompt // page_size * page_size
    group = (torch.tensor([0, level], dtype=torch.int32, device="cuda"), torch.tensor([whole], dtype=torch.int32, device="cuda"), whole) if whole else None
    said = ids.int().repeat(level)
    adjust = dict(history=said, history_start=torch.arange(0, level * prompt + 1, prompt, dtype=torch.int32, device="cuda"),
                  frequency=torch.full((level,), 0.1, device="cuda"), temperature=torch.full((level,), 0.8, device="cuda"))
    tokens = first.repeat(level)

    def one():
        s.step(tokens, at, group, adjust)
        tokens.copy_(at["chosen"])

    side = torch.cuda.Stream()  # (a captured step's libraries are set up by one that is not)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
        one()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    graph.replay()
    begin, end = torch.cuda.Event(True), torch.cuda.Event(True)
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    bits = I.maaso_instance_status(s.inst)
    if bits:
        raise RuntimeError(f"the instance reports {bits}")
    seconds = begin.elapsed_time(end) / steps / 1e3
    s.inst.close()
    return seconds


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--levels", default="1,2,4,8,16,32,64")
    p.add_argument("--prompt", type=int, default=900)
    p.add_argument("--steps", type=int, default=32)
    a = p.parse_args(argv)
    levels = [int(x) for x in a.levels.split(",")]
    model = Decoder(layers=a.layers)
    seconds = [measure(model, level, a.prompt, a.steps) for level in levels]
    # a request's tokens per second against the load, as the profiler's fit takes them
    params, tbt = binding.maaso_profile_fit([0, len(levels)], np.array(levels), 1.0 / np.array(seconds), b_cap=max(levels))
    print(json.dumps({"levels": levels, "us_per_step": [round(s * 1e6, 1) for s in seconds], "tokens_per_s": [round(n / s) for n, s in zip(levels, seconds)],
                      "fit": {"T0": params[0, 0], "delta": params[0, 1], "eps": params[0, 2]}, "tbt_at_cap": float(tbt[0, -1])}))


if __name__ == "__main__":
    main()
