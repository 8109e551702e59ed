"""Greedy decoding with drafted trees over a paged cache: one decoder layer
between an embedding and an LM head.

A drafter that looks at one token only proposes a tree of next tokens for every
sequence; one step runs all nodes; the longest path along which the layer agrees
is kept.  Every step runs, for all sequences at once,

    arrays of the step from the lengths     nj.paged_step (pages given back and taken on the GPU)
    qkv = x . W_qkv                         nj.matmul
    q, cache <- normed, turned q; k, v      nj.kv_append_slots
    o = attention along the trees           nj.tree_attention
    logits = (x + o . W_out) . W_lm         nj.matmul
    penalties, biases, allowed tokens       nj.adjust_logits
    accepted nodes to their places          nj.kv_move

Prompts are taken by the same steps, as trees that are chains.  Weights are random;
--check walks the generated sequences in fp64 without a cache and tells how far
below the best allowed logit the chosen ones lie (0 up to rounding).

    python examples/speculate.py [--prompts 40,7,1] [--tokens 32] [--nodes 12] [--check]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2309_08978_amd as nj

EPS = 1e-6


class Model:
    """Embedding, one attention block with head norms, LM head; the drafter's table."""

    def __init__(self, vocab, width, q_heads, kv_heads, dim, positions, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.width, self.q_heads, self.kv_heads, self.dim = vocab, width, q_heads, kv_heads, dim

        def normal(*shape, scale):
            return (torch.randn(*shape, device="cuda", generator=g) * scale).half()

        self.embed = normal(vocab, width, scale=1.0)
        self.w_qkv = normal(width, (q_heads + 2 * kv_heads) * dim, scale=width ** -0.5)
        self.w_out = normal(q_heads * dim, width, scale=0.5 * (q_heads * dim) ** -0.5)
        self.w_lm = normal(width, vocab, scale=width ** -0.5)
        self.q_weight, self.k_weight = (1 + 0.1 * torch.randn(dim, device="cuda", generator=g) for _ in range(2))
        self.norm = nj.HeadNorm(self.q_weight, self.k_weight, EPS)
        self.table = nj.rotary_table(positions, dim)
        # what the drafter knows: the two likeliest tokens after each one, without attention
        self.next = nj.matmul(self.embed, self.w_lm).topk(2, dim=1).indices.cpu().tolist()

    def rules_of(self, histories, penalties, banned):
        """The rules of rows with these histories (lists of tokens)."""
        rows, longest = len(histories), max(1, max(len(h) for h in histories))
        history = torch.tensor([h + [-1] * (longest - len(h)) for h in histories], dtype=torch.int32, device="cuda")
        allowed = torch.ones(-(-self.vocab // 32) * 32, dtype=torch.int64)
        allowed[torch.tensor(banned, dtype=torch.int64)] = 0
        words = (allowed.view(-1, 32) << torch.arange(32)).sum(1)
        mask = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)[None].cuda()
        each = {k: torch.full((rows,), float(v), device="cuda") for k, v in penalties.items()}
        return nj.LogitRules(history=history, length=torch.tensor([len(h) for h in histories], dtype=torch.int32, device="cuda"),
                             mask=mask, mask_row=torch.zeros(rows, dtype=torch.int32, device="cuda"), **each)

    def plain(self, tokens):
        """Logits [tokens, vocab] of a whole sequence in fp64, without rules."""
        n, hq, hk, d = len(tokens), self.q_heads, self.kv_heads, self.dim
        x = self.embed[torch.tensor(tokens, device="cuda")].double()
        qkv = (x @ self.w_qkv.double()).view(n, hq + 2 * hk, d)
        cos, sin = self.table.table[:n, None, :d // 2].double(), self.table.table[:n, None, d // 2:].double()

        def turned(h, w):
            h = h / ((h * h).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
            a, b = h[..., :d // 2], h[..., d // 2:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)

        q, k, v = turned(qkv[:, :hq], self.q_weight), turned(qkv[:, hq:hq + hk], self.k_weight), qkv[:, hq + hk:]
        out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
        later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        for h in range(hq):
            w = torch.softmax(((q[:, h] @ k[:, h * hk // hq].t()) * d ** -0.5).masked_fill(later, float("-inf")), dim=1)
            out[:, h] = w @ v[:, h * hk // hq]
        return (x + out.reshape(n, -1) @ self.w_out.double()) @ self.w_lm.double()


class Server:
    """The cache, its free pages and the sequences in it."""

    def __init__(self, model, sequences, page_size, pages, columns, rows, words):
        self.model = model
        shape = (pages, page_size, model.kv_heads, model.dim)
        self.cache = nj.PagedCache(*(torch.empty(shape, dtype=torch.float16, device="cuda") for _ in range(2)))
        self.pool = nj.PagePool(torch.arange(pages, dtype=torch.int32, device="cuda"), torch.tensor([pages], dtype=torch.int32, device="cuda"))
        self.held = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        table = torch.zeros((sequences, columns), dtype=torch.int32, device="cuda")
        self.step = nj.PagedStep(table, page_size, rows, mask_words=words, kv_len=self.held)
        self.most_keys = columns * page_size

    def run(self, keep, trees, penalties, banned, histories):
        """One step: keep cached tokens, then trees [(tokens, parents)] of new ones -> logits [rows, vocab]."""
        m, step = self.model, self.step
        counts = [len(t) for t, _ in trees]
        rows = sum(counts)
        pad = [0] * (step.tokens - rows)
        tokens = torch.tensor([t for tree, _ in trees for t in tree] + pad, device="cuda")
        parent = torch.tensor([p for _, up in trees for p in up] + pad, dtype=torch.int32, device="cuda")
        nj.paged_step(step, self.pool, self.held, torch.tensor(counts, dtype=torch.int32, device="cuda"),
                      keep=torch.tensor(keep, dtype=torch.int32, device="cuda"), parent=parent)
        x = m.embed[tokens]
        hq, hk = m.q_heads, m.kv_heads
        qkv = nj.matmul(x, m.w_qkv).view(step.tokens, hq + 2 * hk, m.dim)
        q = torch.zeros((step.tokens, hq, m.dim), dtype=torch.float16, device="cuda")
        nj.kv_append_slots(self.cache, step.slots, qkv[:, hq:hq + hk], qkv[:, hq + hk:], step.positions, m.table, qkv[:, :hq], q, m.norm)
        self.batch = step.batch(max_q=max(counts), max_kv=self.most_keys)
        o = nj.tree_attention(q, self.cache, self.batch, step.mask, torch.zeros_like(q))
        y = x[:rows] + nj.matmul(o[:rows].reshape(rows, -1), m.w_out).half()
        logits = nj.matmul(y, m.w_lm)
        if int(step.status[0]):
            raise RuntimeError(f"the step was refused: {step.status.tolist()}")
        return nj.adjust_logits(logits, m.rules_of(histories, penalties, banned), logits)

    def accept(self, paths):
        """Each sequence's accepted nodes go to the places behind what it kept."""
        most = max(1, max(len(p) for p in paths))
        nj.kv_move(self.cache, self.batch, torch.tensor([p + [0] * (most - len(p)) for p in paths], dtype=torch.int32, device="cuda"),
                   torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda"))


def draft(model, root, nodes):
    """A tree of `nodes` tokens below and with `root`: the likeliest chain first, then second choices along it."""
    tokens, parents = [root], [-1]
    while len(tokens) < (nodes + 1) // 2:
        parents.append(len(tokens) - 1)
        tokens.append(model.next[tokens[-1]][0])
    for i in range(len(tokens)):
        if len(tokens) < nodes:
            parents.append(i)
            tokens.append(model.next[tokens[i]][1])
    return tokens, parents


def path_to(parents, node):
    up = []
    while node >= 0:
        up.append(node)
        node = parents[node]
    return up[::-1]


def generate(prompts, new, nodes=12, vocab=512, width=256, q_heads=4, kv_heads=2, dim=64, page_size=16, chunk=32, check=False, seed=0,
             penalties=(("frequency", 0.2), ("presence", 0.1), ("repetition", 1.05)), banned=(3, 7)):
    """-> (generated tokens per sequence, steps, largest shortfall of a chosen logit in fp64, or None)."""
    penalties = dict(penalties)
    n, longest = len(prompts), max(prompts) + new + nodes
    model = Model(vocab, width, q_heads, kv_heads, dim, longest + 1, seed)
    columns = -(-(longest + 1) // page_size)
    words = max(1, -(-max(nodes, chunk) // 32))
    server = Server(model, n, page_size, n * columns, columns, n * max(nodes, chunk), words)
    g = torch.Generator().manual_seed(seed + 1)
    said = [torch.randint(0, vocab, (p,), generator=g).tolist() for p in prompts]      # prompt, then what was generated
    done = [0] * n                                                                     # tokens of it in the cache
    want = [p + new for p in prompts]
    steps = 0
    while any(len(s) < w for s, w in zip(said, want)):
        trees = []
        for b in range(n):
            rest = said[b][done[b]:]
            if len(said[b]) >= want[b]:
                trees.append(([], []))                                                 # done: its pages go back
                done[b] = 0
            elif len(rest) > 1:                                                        # a prompt: a chain of its next tokens
                part = rest[:chunk]
                trees.append((part, list(range(-1, len(part) - 1))))
            else:
                trees.append(draft(model, rest[0], nodes))
        histories = []
        for b, (tokens, parents) in enumerate(trees):
            seen = said[b][:done[b]]
            histories += [seen + [tokens[i] for i in path_to(parents, node)] for node in range(len(tokens))]
        logits = server.run(done, trees, penalties, banned, histories)
        best = logits.argmax(dim=1).cpu().tolist()
        at, paths = 0, []
        for b, (tokens, parents) in enumerate(trees):
            choice = best[at:at + len(tokens)]
            at += len(tokens)
            if not tokens:
                paths.append([])
                continue
            rest = said[b][done[b]:]
            if len(rest) > 1:
                path = list(range(len(tokens)))
                if len(tokens) == len(rest):
                    said[b].append(choice[-1])
            else:
                path = [0]                                                             # the root is what was said last
                said[b].append(choice[0])
                while len(said[b]) < want[b]:
                    child = [i for i, p in enumerate(parents) if p == path[-1] and tokens[i] == said[b][-1]]
                    if not child:
                        break
                    path.append(child[0])
                    said[b].append(choice[child[0]])
            paths.append(path)
            done[b] += len(path)
        server.accept(paths)
        steps += 1
    worst = None
    if check:
        worst = 0.0
        for s, p in zip(said, prompts):
            z = model.plain(s)
            for i in range(p - 1, len(s) - 1):
                row, before = z[i].clone(), torch.tensor(s[:i + 1], device="cuda")
                count = torch.bincount(before, minlength=vocab).double()
                rho = torch.where(row > 0, 1 / penalties.get("repetition", 1.0), penalties.get("repetition", 1.0))
                row = torch.where(count > 0, row * rho, row) - penalties.get("frequency", 0.0) * count
                row = torch.where(count > 0, row - penalties.get("presence", 0.0), row)
                row[list(banned)] = float("-inf")
                worst = max(worst, float(row.max() - row[s[i + 1]]))
    return [s[p:] for s, p in zip(said, prompts)], steps, worst


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", default="40,7,1", help="prompt lengths, comma separated")
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--nodes", type=int, default=12)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    prompts = [int(p) for p in a.prompts.split(",")]
    said, steps, worst = generate(prompts, a.tokens, a.nodes, check=a.check)
    print(f"{sum(map(len, said))} tokens in {steps} steps" + (f", chosen logits at most {worst:.1e} below the best" if a.check else ""))
    return 0


if __name__ == "__main__":
    sys.exit(main())
