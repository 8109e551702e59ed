"""One decoder layer's attention block served from a paged cache.

Every step runs, for all sequences at once,

    qkv = x . W_qkv                         nj.matmul (fp16 weights, fp32 result)
    q, cache <- turned q; k, v appended     nj.kv_append
    o = attention(q, cache)                 nj.paged_attention
    y = o . W_out                           nj.matmul

first on the prompts, taken in chunks, then token by token.  Pages are handed
out as sequences grow; the page table on the GPU is all that the kernels see
of it.  Weights and inputs are random (the layer's shapes are a 7B decoder's
unless given); --check compares every output row with the same block computed in
fp64 without a cache.

    python examples/serve_layer.py [--prompts 300,37,1] [--steps 8] [--check]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2309_08978_amd as nj


class Layer:
    """Weights, rotary table and paged cache of one attention block."""

    def __init__(self, width, q_heads, kv_heads, dim, page_size, pages, positions, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.q_heads, self.kv_heads, self.dim, self.page_size = q_heads, kv_heads, dim, page_size
        self.w_qkv = (torch.randn(width, (q_heads + 2 * kv_heads) * dim, device="cuda", generator=g) * width ** -0.5).half()
        self.w_out = (torch.randn(q_heads * dim, width, device="cuda", generator=g) * (q_heads * dim) ** -0.5).half()
        self.table = nj.rotary_table(positions, dim)
        shape = (pages, page_size, kv_heads, dim)
        self.cache = nj.PagedCache(*(torch.empty(shape, dtype=torch.float16, device="cuda") for _ in range(2)))
        self.free = list(range(pages))
        self.pages = []                    # per sequence

    def grow(self, lengths):
        """Pages for sequences of these lengths; the page table."""
        for s, n in enumerate(lengths):
            if s == len(self.pages):
                self.pages.append([])
            while len(self.pages[s]) * self.page_size < n:
                self.pages[s].append(self.free.pop())
        cols = max(len(p) for p in self.pages)
        return torch.tensor([p + [0] * (cols - len(p)) for p in self.pages], dtype=torch.int32, device="cuda")

    def step(self, x, new, lengths):
        """x [sum of new, width] fp16: the rows of `new` tokens per sequence, whose lengths become `lengths`."""
        start = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
        batch = nj.PagedBatch(start, torch.tensor(lengths, dtype=torch.int32, device="cuda"), self.grow(lengths),
                              tokens=x.shape[0], max_q=max(new), max_kv=max(lengths))
        hq, hk = self.q_heads, self.kv_heads
        qkv = nj.matmul(x, self.w_qkv).view(x.shape[0], hq + 2 * hk, self.dim)
        q = nj.kv_append(self.cache, batch, qkv[:, hq:hq + hk], qkv[:, hq + hk:], self.table, qkv[:, :hq])
        o = nj.paged_attention(q, self.cache, batch)
        return nj.matmul(o.view(x.shape[0], -1), self.w_out)

    def plain(self, x):
        """The same block in fp64 on one whole sequence x [tokens, width]."""
        n, hq, hk, d = x.shape[0], self.q_heads, self.kv_heads, self.dim
        qkv = (x.double() @ self.w_qkv.double()).view(n, hq + 2 * hk, d)
        cos, sin = self.table.table[:n, None, :d // 2].double(), self.table.table[:n, None, d // 2:].double()
        a, b = qkv[:, :hq + hk, :d // 2], qkv[:, :hq + hk, d // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        q, k, v = turned[:, :hq], turned[:, hq:], qkv[:, hq + hk:]
        out = torch.empty(n, hq, d, dtype=torch.float64, device=x.device)
        later = torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1)
        for h in range(hq):
            logits = (q[:, h] @ k[:, h * hk // hq].t()) * d ** -0.5
            out[:, h] = torch.softmax(logits.masked_fill(later, float("-inf")), dim=1) @ v[:, h * hk // hq]
        return out.reshape(n, -1) @ self.w_out.double()


def serve(prompts, steps, width=4096, q_heads=32, kv_heads=32, dim=128, page_size=16, chunk=256, check=False, seed=0):
    """-> (ms of the prompts, ms of a decode step, largest relative error of a sequence, or None)."""
    total = [n + steps for n in prompts]
    layer = Layer(width, q_heads, kv_heads, dim, page_size, sum(-(-n // page_size) for n in total) + 1, max(total), seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = [torch.randn(n, width, device="cuda", generator=g).half() for n in total]
    outs = [[] for _ in prompts]
    done = [0] * len(prompts)

    def run(new):
        rows = torch.cat([x[s][done[s]:done[s] + n] for s, n in enumerate(new)])
        for s, n in enumerate(new):
            done[s] += n
        for s, y in enumerate(layer.step(rows, new, done).split(new)):
            outs[s].append(y)

    torch.cuda.synchronize()
    t0 = time.perf_counter()
    while any(d < n for d, n in zip(done, prompts)):       # sequences whose prompt is done wait with no new token
        run([min(chunk, n - d) for d, n in zip(done, prompts)])
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    for _ in range(steps):
        run([1] * len(prompts))
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    error = None
    if check:
        error = 0.0
        for s, n in enumerate(total):
            want, got = layer.plain(x[s]), torch.cat(outs[s]).double()
            error = max(error, float((got - want).norm() / want.norm()))
    return (t1 - t0) * 1e3, (t2 - t1) * 1e3 / max(steps, 1), error


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", default="300,37,1", help="prompt lengths, comma separated")
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=32)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=16)
    ap.add_argument("--chunk", type=int, default=256)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    prompts = [int(n) for n in a.prompts.split(",")]
    serve(prompts, 1, a.width, a.heads, a.kv_heads, a.dim, a.page, a.chunk)     # first launches
    prompt_ms, step_ms, error = serve(prompts, a.steps, a.width, a.heads, a.kv_heads, a.dim, a.page, a.chunk, a.check)
    print(f"prompts {prompts} in chunks of {a.chunk}: {prompt_ms:.2f} ms, decode step {step_ms:.3f} ms"
          + (f", relative error {error:.1e}" if error is not None else ""))
    return 0


if __name__ == "__main__":
    sys.exit(main())
