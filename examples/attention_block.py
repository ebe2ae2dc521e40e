#!/usr/bin/env python3
"""The attention half of a transformer block on compressed weights and a 4-bit
key/value cache: ragged prompts, then generated tokens in a captured HIP graph.

For each token: query, key and value projections from entropy-coded weights
(eq_decode_gemm for prompts, eq_decode_gemv_multi for single tokens), the norm of
each query and key head with its rotation (eq_qk_norm_rope), the new keys and
values into the paged cache (eq_kv_append), attention over it (eq_attn_kv4), and
the output projection.  The result is held against plain attention in 64 bits on
the cache's values as eq_kv_read returns them.

    python examples/attention_block.py [--hidden 1024] [--heads 16] [--kv-heads 4] [--steps 16]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2601_22787_amd as eq  # noqa: E402
import synth  # noqa: E402
from synth.configs import small_spec  # noqa: E402

DIM, PAGE = 128, 64


def layer(rows, cols, seed, device):
    """A version-2 container of synthetic weights at about 3 bits a weight."""
    spec = small_spec(rows, cols, bits=3.0, seed=seed)
    w = synth.weights(spec)
    alpha, _ = eq.eqe_alpha_search(w, 3.0, sample_rows=min(rows, 256))
    return eq.Layer(eq.eqe_encode2(w, alpha, tile_rows=64, tile_cols=128), device)


class Attention:
    """Projections, norms and rotation tables of one block."""

    def __init__(self, hidden, heads, kv_heads, max_len, device="cuda"):
        self.hidden, self.heads, self.kv_heads, self.max_len = hidden, heads, kv_heads, max_len
        rows = (heads * DIM, kv_heads * DIM, kv_heads * DIM)
        self.qkv = [layer(r, hidden, 10 + i, device) for i, r in enumerate(rows)]
        self.out = layer(hidden, heads * DIM, 20, device)
        g = torch.Generator(device=device)
        g.manual_seed(3)
        w = 1 + 0.2 * torch.randn(2, DIM, device=device, generator=g)
        self.q_weight, self.k_weight = w.to(torch.bfloat16)
        a = torch.arange(max_len, device=device).double()[:, None] * \
            10000.0 ** (-torch.arange(0, DIM, 2, device=device).double() / DIM)
        self.rope = eq.Rope(a.cos().float(), a.sin().float())

    def buffers(self, tokens, cache, batch):
        """What a call over `tokens` rows writes, kept between calls."""
        dev = self.qkv[0].dev_blob.device

        def room(*shape, kind=torch.float32):
            return torch.empty(*shape, dtype=kind, device=dev)

        few = tokens <= 8
        return {
            "y": [room(tokens, layer.rows) for layer in self.qkv],
            "ws": eq.multi_workspace(self.qkv, tokens) if few else
            room(max(eq.eq_gemm_workspace_bytes(x, tokens) for x in self.qkv), kind=torch.uint8),
            "q": room(tokens, self.heads, DIM, kind=torch.bfloat16),
            "k": room(tokens, self.kv_heads, DIM, kind=torch.bfloat16),
            "attn": room(tokens, self.heads, DIM, kind=torch.bfloat16),
            "attn_ws": eq.attn_workspace(cache, batch, self.heads),
            "out": room(tokens, self.hidden),
            "out_ws": self.out.gemm_workspace(tokens),
        }

    def __call__(self, x, positions, cache, batch, b):
        """x [tokens, hidden] BF16 -> b["out"] [tokens, hidden] fp32."""
        n = x.shape[0]
        if n <= 8:
            eq.eq_decode_gemv_multi(self.qkv, x, n, None, b["y"], b["ws"])
        else:
            for layer, y in zip(self.qkv, b["y"]):
                eq.eq_decode_gemm(layer, x, n, None, y, b["ws"])
        q, k, v = (y.view(n, -1, DIM) for y in b["y"])
        eq.eq_qk_norm_rope(q, k, b["q"], b["k"], q_weight=self.q_weight, k_weight=self.k_weight,
                           rope=self.rope, positions=positions)
        eq.eq_kv_append(cache, batch, b["k"], v)
        eq.eq_attn_kv4(cache, batch, b["q"], DIM ** -0.5, b["attn"], b["attn_ws"])
        eq.eq_decode_gemm(self.out, b["attn"].view(n, -1), n, None, b["out"], b["out_ws"])
        return b["out"]


def plain(q, keys, values, places):
    """Attention in 64 bits of q [n, heads, D], row i at places[i]."""
    group = q.shape[1] // keys.shape[1]
    k = keys.double().repeat_interleave(group, dim=1).permute(1, 2, 0).contiguous()
    v = values.double().repeat_interleave(group, dim=1).transpose(0, 1).contiguous()
    s = torch.bmm(q.double().transpose(0, 1).contiguous(), k) / math.sqrt(DIM)
    at = torch.arange(keys.shape[0], device=q.device)
    s.masked_fill_(at[None, None, :] > places[None, :, None], -math.inf)
    return torch.bmm(torch.softmax(s, dim=-1), v).transpose(0, 1)


def error(block, cache, b, starts, lens, news, table):
    """Largest relative error of b["attn"] over the sequences."""
    dev = b["q"].device
    total, worst = sum(lens), 0.0
    whole = eq.KvBatch(torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device=dev),
                       torch.tensor(lens, dtype=torch.int32, device=dev), table, n_tokens=total,
                       max_new=max(lens), max_len=block.max_len)
    kv = torch.empty(2, total, block.kv_heads, DIM, dtype=torch.bfloat16, device=dev)
    eq.eq_kv_read(cache, whole, kv[0], kv[1])
    at = 0
    for i, (t, n) in enumerate(zip(lens, news)):
        rows = slice(starts[i], starts[i] + n)
        ref = plain(b["q"][rows], kv[0, at:at + t], kv[1, at:at + t],
                    torch.arange(t - n, t, device=dev))
        worst = max(worst, float((b["attn"][rows].double() - ref).norm() / ref.norm()))
        at += t
    return worst


def run(hidden=1024, heads=16, kv_heads=4, prompts=(37, 150, 5), steps=16, say=print):
    dev = torch.device("cuda:0")
    n = len(prompts)
    max_len = -(-(max(prompts) + steps + 1) // PAGE) * PAGE
    block = Attention(hidden, heads, kv_heads, max_len, dev)
    pages = max_len // PAGE
    cache = eq.KvCache.empty(n * pages, page_tokens=PAGE, kv_heads=kv_heads, head_dim=DIM, device=dev)
    table = torch.randperm(n * pages, device=dev).int().view(n, pages).contiguous()
    lens = torch.tensor(prompts, dtype=torch.int32, device=dev)

    # the prompts, all in one ragged call
    starts = [0] + list(np.cumsum(prompts))
    batch = eq.KvBatch(torch.tensor(starts, dtype=torch.int32, device=dev), lens, table,
                       n_tokens=starts[-1], max_new=max(prompts), max_len=max_len)
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    x = torch.randn(starts[-1], hidden, device=dev, generator=g).to(torch.bfloat16)
    places = torch.cat([torch.arange(t, dtype=torch.int32, device=dev) for t in prompts])
    b = block.buffers(starts[-1], cache, batch)
    block(x, places, cache, batch, b)
    errors = [error(block, cache, b, starts, list(prompts), list(prompts), table)]
    say(f"prompts {prompts}: relative error of attention {errors[0]:.2e}")

    # generated tokens: one a sequence, captured once, lengths on the device
    step = eq.KvBatch(torch.arange(n + 1, dtype=torch.int32, device=dev), lens, table, n_tokens=n,
                      max_new=1, max_len=max_len)
    xs = torch.randn(n, hidden, device=dev, generator=g).to(torch.bfloat16)
    place = torch.empty(n, dtype=torch.int32, device=dev)
    b = block.buffers(n, cache, step)

    def advance():
        place.copy_(lens)
        lens.add_(1)
        block(xs, place, cache, step, b)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        advance()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        advance()
    now = [t + 1 for t in prompts]
    for i in range(steps):
        xs.normal_(generator=g)
        graph.replay()
        now = [t + 1 for t in now]
        if i in (0, steps - 1):
            errors.append(error(block, cache, b, list(range(n)), now, [1] * n, table))
            say(f"step {i + 1}, lengths {now}: relative error {errors[-1]:.2e}")
    for layer in block.qkv + [block.out]:
        if eq.eq_get_status(layer) != eq.EQ_OK:
            raise RuntimeError("a projection's stream is damaged")
    keep = lens.clone()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(50):
        lens.copy_(keep)
        lens.sub_(1)
        graph.replay()
    torch.cuda.synchronize()
    say(f"{n} tokens a step: {(time.perf_counter() - t0) / 50 * 1e6:.1f} us a step (graph replay)")
    return errors


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    errors = run(a.hidden, a.heads, a.kv_heads, steps=a.steps)
    return 0 if max(errors) < 1e-2 else 1


if __name__ == "__main__":
    sys.exit(main())
