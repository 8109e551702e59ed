"""Measured cases: the operators around the layers when drafted tokens are
served from a paged cache -- one step from the requests' lengths to the
logits and on to the next step.

Kinds of case

``step``    the arrays of one step from the requests' lengths: sequence b holds
            ``held`` tokens, of which ``keep`` stay, and gets ``added`` new
            ones; pages go back to a stack of free pages or are taken from it; row
            starts, key counts, page table, slots and positions come out, with
            ``tree`` > 0 (nodes a sequence at most) also which new tokens each one
            sees: its ancestors and itself
``append``  queries and keys of new rows, each head scaled to a mean square of 1
            and by a weight a dim, turned by rotary angles; keys and values go
            to the rows' slots in a paged cache.  q, k and v are column ranges of
            one tensor of type ``src``; cache and queries have type ``dtype``;
            ``pad`` rows behind the last sequence are left alone
``train``   the same norm and turn without a cache and its gradients: y from x,
            dx and the weight's gradient from dy; ``per_head``: a weight a head
``tree``    attention of drafted tokens: every row sees its sequence's cached
            keys (with ``window`` > 0 the last of them) and its ancestors
            among the new ones
``move``    the keys and values of accepted nodes move to the places behind
            the cached ones
``logits``  repetition, presence and frequency penalties, biases of single
            tokens and bit masks of allowed tokens on rows of logits

Values: activations, keys, values and gradients N(0, 1), queries of attention
N(0, 2) (logits of a trained layer spread wider than those of random vectors),
weights of norms N(1, 0.1), logits N(0, 3).  Trees: the first nodes are the
likeliest chain, the others hang from random earlier nodes, as a drafter adds
them.  Histories: most tokens from a few hundred that repeat.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16}


def _step(name, sequences, context, ragged, tree, page):
    return {"name": name, "kind": "step", "sequences": sequences, "context": context, "ragged": ragged, "tree": tree, "page": page}


def _append(name, sequences, chunk, context, ragged, pad, q_heads, kv_heads, dim, rot, layout, src, dtype, page):
    return {"name": name, "kind": "append", "sequences": sequences, "chunk": chunk, "context": context, "ragged": ragged,
            "pad": pad, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "layout": layout, "src": src,
            "dtype": dtype, "page": page}


def _train(name, tokens, heads, dim, rot, layout, dtype, per_head=False):
    return {"name": name, "kind": "train", "tokens": tokens, "heads": heads, "dim": dim, "rot": rot, "layout": layout,
            "dtype": dtype, "per_head": per_head}


def _tree(name, sequences, chunk, context, ragged, q_heads, kv_heads, dim, dtype, page, window=0):
    return {"name": name, "kind": "tree", "sequences": sequences, "chunk": chunk, "context": context, "ragged": ragged,
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page, "window": window}


def _move(name, sequences, chunk, context, ragged, accepted, kv_heads, dim, dtype, page):
    return {"name": name, "kind": "move", "sequences": sequences, "chunk": chunk, "context": context, "ragged": ragged,
            "accepted": accepted, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page}


def _logits(name, rows, vocab, history, biases, masked, src, dst):
    return {"name": name, "kind": "logits", "rows": rows, "vocab": vocab, "history": history, "biases": biases,
            "masked": masked, "src": src, "dst": dst}


def listed():
    return [
        # a decode step of eight requests, one new token each
        _step("step_decode", 8, 2000, 0.9, 0, 16),
        # a full serving batch: requests that come, go and shrink to what was accepted, trees of up to 48 drafted tokens
        _step("step_trees", 256, 8192, 0.95, 48, 16),
        # the smallest append: one decoded token
        _append("append_token_f16", 1, 1, 1000, 0.0, 0, 32, 8, 128, 128, "half", "f16", "f16", 16),
        # ragged prompts as an fp32 qkv linear gives them, in a batch padded to whole hundreds
        _append("append_prompts_f32", 5, 900, 900, 0.8, 37, 32, 8, 128, 128, "half", "f32", "f16", 16),
        # queries of a training step, forward and backward
        _train("train_f16", 4096, 32, 128, 128, "half", "f16"),
        # one drafted tree of a base-size fp32 decoder
        _tree("tree_one_f32", 1, 24, 1023, 0.0, 12, 12, 64, "f32", 16),
        # trees of a serving batch, four query heads to a key head
        _tree("tree_batch_f16", 16, 32, 4096, 0.9, 32, 8, 128, "f16", 64),
        # a wide tree behind one long document
        _tree("tree_long_f16", 1, 64, 65536, 0.0, 32, 8, 128, "f16", 128),
        # accepted tokens of a few requests
        _move("move_f16", 4, 32, 1000, 0.9, 6, 8, 128, "f16", 16),
        # accepted tokens of a large batch of fp32 requests
        _move("move_batch_f32", 64, 64, 1000, 0.9, 16, 12, 64, "f32", 32),
        # one request's logits, fp32 as the LM head gives them, no grammar
        _logits("logits_row", 1, 32000, 1000, 20, False, "f32", "f32"),
        # logits of a batch with long histories and grammars
        _logits("logits_batch", 64, 128000, 4000, 100, True, "f32", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one to 512 sequences, trees of one to
    128 nodes, contexts to 65536, heads of 64, 96 and 128 dims, one to eight query
    heads to a key head, pages of any size, vocabularies from 1000 to 256000."""
    pick = rng.random()
    dim = rng.choice([64, 96, 128, 128])
    rot = dim if rng.random() < 0.7 else dim // 2
    layout = rng.choice(["half", "interleaved"])
    dtype = rng.choice(["f32", "f16", "f16"])
    page = rng.choice([16, 16, 32, 64, 128, _log_int(rng, 1, 200)])
    ragged = round(rng.uniform(0, 0.95), 3)
    kv_heads = rng.choice([4, 8, 12, 16, 32])
    q_heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8) if kv_heads * g <= 32])
    if pick < 0.15:
        return {"kind": "step", "sequences": _log_int(rng, 1, 512), "context": _log_int(rng, 100, 8192), "ragged": ragged,
                "tree": rng.choice([0, _log_int(rng, 2, 128)]), "page": max(page, 8)}
    if pick < 0.3:
        sequences = _log_int(rng, 1, 32)
        chunk = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(2, 3600 // sequences))
        return {"kind": "append", "sequences": sequences, "chunk": chunk, "context": chunk + _log_int(rng, 1, 2000),
                "ragged": ragged, "pad": rng.choice([0, rng.randint(1, 100)]), "q_heads": q_heads, "kv_heads": kv_heads,
                "dim": dim, "rot": rot, "layout": layout, "src": rng.choice(["f32", "f16"]), "dtype": dtype, "page": page}
    if pick < 0.4:
        return {"kind": "train", "tokens": _log_int(rng, 1, 4096), "heads": rng.choice([8, 12, 16, 32]), "dim": dim, "rot": rot,
                "layout": layout, "dtype": dtype, "per_head": rng.random() < 0.3}
    if pick < 0.5:
        chunk = _log_int(rng, 2, 128)
        return {"kind": "move", "sequences": _log_int(rng, 1, 64), "chunk": chunk, "context": chunk + _log_int(rng, 1, 1000),
                "ragged": ragged, "accepted": rng.randint(1, max(1, chunk // 2)), "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
                "page": page}
    if pick < 0.65:
        while True:
            rows, vocab, history = _log_int(rng, 1, 256), _log_int(rng, 1000, 256000), _log_int(rng, 1, 32000)
            if rows * vocab <= 64 * 128000 and rows * history <= 64 * 16000:
                break
        return {"kind": "logits", "rows": rows, "vocab": vocab, "history": history, "biases": rng.choice([0, rng.randint(1, 300)]),
                "masked": rng.random() < 0.5, "src": rng.choice(["f32", "f32", "f16"]), "dst": rng.choice(["f32", "f32", "f16"])}
    while True:
        sequences = _log_int(rng, 1, 32)
        chunk = _log_int(rng, 1, 128)
        context = chunk + _log_int(rng, 1, 65536 - chunk)
        # no more keys, scores and products than the largest listed case has
        if (sequences * context * kv_heads * dim <= 65536 * 8 * 128
                and sequences * chunk * context * q_heads <= 64 * 65536 * 32 * (0.9 if dtype == "f16" else 0.25)):
            break
    return {"kind": "tree", "sequences": sequences, "chunk": chunk, "context": context, "ragged": ragged, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "window": _log_int(rng, chunk, context) if rng.random() < 0.2 else 0}


def _lengths(case):
    """New tokens and keys of every sequence: spread over the range, the first sequence the longest."""
    new, keys = [], []
    for i in range(case["sequences"]):
        n = max(1, int(case["chunk"] * (1.0 - case["ragged"] * ((i * 0.6180339887) % 1.0))))
        past = int((case["context"] - case["chunk"]) * (1.0 - case["ragged"] * ((i * 0.7548776662) % 1.0)))
        new.append(n)
        keys.append(past + n)
    return new, keys


def _requests(case):
    """held, keep and added tokens of every sequence of a step: most go on, some
    have just come, some are done, some are taken whole into a smaller tree."""
    held, keep, added = [], [], []
    for i in range(case["sequences"]):
        n = max(1, int(case["context"] * (1.0 - case["ragged"] * ((i * 0.7548776662) % 1.0))))
        tree = max(1, int(case["tree"] * (1.0 - 0.7 * ((i * 0.6180339887) % 1.0)))) if case["tree"] else 1
        if i % 11 == 5:      # new
            held, keep, added = held + [0], keep + [0], added + [min(tree, 32 * _words(case)) if case["tree"] else 1 + i % 40]
        elif i % 11 == 9:    # done
            held, keep, added = held + [n], keep + [0], added + [0]
        else:
            drafted = min(n, tree)
            held, keep, added = held + [n], keep + [n - drafted + min(drafted, 1 + i % 5) if case["tree"] else n], added + [tree]
    return held, keep, added


def _words(case):
    return -(-case["tree"] // 32)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1) + 31)
    return g


def _table(positions, rot):
    """[positions][cos of rot / 2 pairs, sin of rot / 2 pairs]."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float().cuda()


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype).cuda()


def _starts(counts):
    return [0] + torch.tensor(counts).cumsum(0).tolist()


def _pages(held, page, columns, spare, g):
    """Page table of sequences that hold these tokens, pages in random order; the ids that are left."""
    need = torch.tensor([-(-n // page) for n in held])
    total = int(need.sum())
    order = torch.randperm(total + spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(held), columns), -1, dtype=torch.int32, device="cuda")
    used = (torch.arange(columns)[None, :] < need[:, None]).cuda()
    table[used] = order[:total]
    return table, order[total:].contiguous(), total + spare


def _parents(counts, g):
    """Parents within each sequence: a chain of about a third of the nodes, the others below random earlier ones."""
    tokens = sum(counts)
    start = torch.tensor(_starts(counts))
    seq = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts), output_size=tokens)
    i = (torch.arange(tokens) - start[seq]).cuda()
    chain = (torch.tensor(counts)[seq] // 3).cuda()
    u = torch.rand(tokens, generator=g, device="cuda")
    other = torch.minimum((u * i).long(), (i - 1).clamp(min=0))
    return torch.where(i == 0, -1, torch.where(i <= chain, i - 1, other)).to(torch.int32), seq.cuda(), i


def _seen(parent, seq, i, start, nodes):
    """bool [tokens, nodes]: the ancestors of every token and itself; its depth."""
    tokens = parent.shape[0]
    up = torch.where(parent >= 0, parent.long() + start.long()[seq], tokens)    # row `tokens`: above every root
    up = torch.cat([up, up.new_tensor([tokens])])
    seen = torch.zeros((tokens + 1, nodes), dtype=torch.bool, device="cuda")
    seen[:tokens] = torch.arange(nodes, device="cuda") == i[:, None]
    for _ in range(max(1, nodes - 1).bit_length()):      # twice as far up each time
        seen = seen | seen[up]
        up = up[up]
    seen = seen[:tokens]
    return seen, seen.sum(dim=1) - 1


def _bits(seen):
    """int32 words of 32 bits, the lowest first."""
    words = -(-seen.shape[1] // 32)
    padded = torch.zeros((seen.shape[0], 32 * words), dtype=torch.int64, device="cuda")
    padded[:, :seen.shape[1]] = seen
    w = (padded.view(-1, words, 32) << torch.arange(32, device="cuda")).sum(dim=-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _inputs(case, seed):
    g = _generator(seed)
    kind = case["kind"]

    def normal(*shape, dtype=torch.float32, scale=1.0, mean=0.0):
        t = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
        return t.mul_(scale).add_(mean).to(dtype)

    if kind == "step":
        held, keep, added = _requests(case)
        page = case["page"]
        columns = max(-(-max(h, k + a) // page) for h, k, a in zip(held, keep, added)) + 1
        table, free, pages = _pages(held, page, columns, sum(-(-a // page) + 1 for a in added) + 5, g)
        s = {"held": _ints(held), "keep": _ints(keep), "added": _ints(added), "page_table": table, "tokens": sum(added) + 3,
             "free": torch.zeros(pages, dtype=torch.int32, device="cuda"), "count": _ints([free.numel()])}
        s["free"][:free.numel()] = free
        if case["tree"]:
            parent = torch.full((s["tokens"],), -1, dtype=torch.int32, device="cuda")
            parent[:sum(added)] = _parents(added, g)[0]
            s["parent"] = parent
        return s
    if kind == "train":
        rows, dt = max(2048, 2 * case["tokens"]), _DT[case["dtype"]]
        first = int(torch.randint(0, rows - case["tokens"] + 1, (1,), generator=g, device="cuda"))
        shape = (case["tokens"], case["heads"], case["dim"])
        return {"x": normal(*shape, dtype=dt), "dy": normal(*shape, dtype=dt), "table": _table(rows, case["rot"]),
                "weight": normal(*(shape[1:] if case["per_head"] else shape[2:]), scale=0.1, mean=1.0),
                "positions": torch.arange(first, first + case["tokens"], dtype=torch.int32, device="cuda")}
    if kind == "logits":
        rows, vocab, most = case["rows"], case["vocab"], case["history"]
        spread = [1.0 - 0.9 * ((i * 0.6180339887) % 1.0) for i in range(rows)]
        length = [max(1, int(most * u)) for u in spread]
        few = torch.randint(0, vocab, (rows, 300), generator=g, device="cuda")
        pick = torch.randint(0, 300, (rows, most), generator=g, device="cuda")
        anything = torch.randint(0, vocab, (rows, most), generator=g, device="cuda")
        repeat = torch.rand((rows, most), generator=g, device="cuda") < 0.7
        s = {"logits": normal(rows, vocab, dtype=_DT[case["src"]], scale=3.0),
             "history": torch.where(repeat, few.gather(1, pick), anything).to(torch.int32), "length": _ints(length),
             "prompt": _ints([n // 3 for n in length]),
             "repetition": torch.rand(rows, generator=g, device="cuda") * 0.4 + 1.0,
             "presence": torch.rand(rows, generator=g, device="cuda") - 0.3,
             "frequency": torch.rand(rows, generator=g, device="cuda") * 0.3}
        if case["biases"]:
            n = case["biases"]
            first = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
            s["bias_token"] = ((first + torch.arange(n, device="cuda") * (vocab // n)) % vocab).to(torch.int32)
            s["bias_value"] = normal(rows, n, scale=5.0)
        if case["masked"]:      # two grammars share the rows, every fourth row has none
            words = -(-vocab // 32)
            s["mask"] = torch.randint(-(1 << 31), 1 << 31, (2, words), generator=g, device="cuda").to(torch.int32)
            s["mask_row"] = _ints([i % 4 - 1 if i % 4 < 3 else 0 for i in range(rows)])
        return s

    new, keys = _lengths(case)
    hk, d, dt, page = case["kv_heads"], case["dim"], _DT[case["dtype"]], case["page"]
    table, _, pages = _pages(keys, page, max(-(-n // page) for n in keys), 3, g)
    tokens = sum(new)
    start = _ints(_starts(new))
    s = {"start": start, "keys": _ints(keys), "page_table": table,
         "k_cache": normal(pages, page, hk, d, dtype=dt), "v_cache": normal(pages, page, hk, d, dtype=dt)}
    if kind == "append":
        seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new), output_size=tokens).cuda()
        pos = torch.arange(tokens, device="cuda") - start.long()[seq] + (s["keys"] - _ints(new)).long()[seq]
        rows = tokens + case["pad"]
        s["slots"] = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
        s["slots"][:tokens] = table[seq, pos // page].long() * page + pos % page
        s["positions"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s["positions"][:tokens] = pos
        s["qkv"] = normal(rows, (case["q_heads"] + 2 * hk) * d, dtype=_DT[case["src"]])
        s["table"] = _table(case["context"], case["rot"])
        s["q_weight"], s["k_weight"] = normal(d, scale=0.1, mean=1.0), normal(d, scale=0.1, mean=1.0)
        return s
    parent, seq, i = _parents(new, g)
    seen, depth = _seen(parent, seq, i, start, case["chunk"])
    if kind == "tree":
        s["q"] = normal(tokens, case["q_heads"], d, dtype=dt, scale=2.0)
        s["mask"] = _bits(seen)
        s["positions"] = ((s["keys"] - _ints(new)).long()[seq] + depth).to(torch.int32)
        return s
    # accepted: the likeliest chain's first nodes, then nodes behind the chain
    count = [min(n, max(1, int(case["accepted"] * (1.0 - 0.6 * ((j * 0.4142135623) % 1.0))))) for j, n in enumerate(new)]
    path = torch.zeros((len(new), case["accepted"]), dtype=torch.int32)
    for j, (n, a) in enumerate(zip(new, count)):
        along = (a + 1) // 2
        later = torch.arange(a - along) + max(along, a)
        step = max(1, (n - a) // max(1, a - along))
        path[j, :along] = torch.arange(along)
        path[j, along:a] = torch.minimum(later + torch.arange(a - along) * (step - 1), torch.tensor(n - 1)) if n > a + a else torch.arange(along, a)
    s["path"], s["accepted"] = path.cuda(), _ints(count)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "append":
        hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
        rows = s["qkv"].view(-1, hq + 2 * hk, d)
        s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        s["out"] = torch.zeros(s["q"].shape, dtype=_DT[case["dtype"]], device="cuda")
    elif kind == "train":
        s["out"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["dw"] = torch.empty_like(s["weight"])
    elif kind == "tree":
        s["out"] = torch.empty_like(s["q"])
    elif kind == "logits":
        s["out"] = torch.empty(s["logits"].shape, dtype=_DT[case["dst"]], device="cuda")
    if own:
        # what a serving program keeps: the handles of cache, table, weights, pool and rules; the arrays of the step
        import paper_2309_08978_amd as nj
        if "table" in s:
            s["rotary"] = nj.RotaryTable(s["table"], layout=case["layout"])
        if "k_cache" in s:
            s["cache"] = nj.PagedCache(s["k_cache"], s["v_cache"])
        if kind == "append":
            s["norm"] = nj.HeadNorm(s["q_weight"], s["k_weight"], eps=1e-6)
        elif kind in ("tree", "move"):
            s["batch"] = nj.PagedBatch(s["start"], s["keys"], s["page_table"], tokens=int(s["start"][-1]),
                                       max_q=case["chunk"], max_kv=case["context"])
        elif kind == "step":
            s["left"] = torch.zeros_like(s["count"])
            s["pool"] = nj.PagePool(s["free"], s["count"], s["left"])
            s["step"] = nj.PagedStep(s["page_table"], case["page"], s["tokens"], mask_words=_words(case))
        elif kind == "logits":
            s["rules"] = nj.LogitRules(**{k: s[k] for k in ("history", "length", "prompt", "repetition", "presence", "frequency",
                                                            "bias_token", "bias_value", "mask", "mask_row") if k in s})
    return s


def _normed(x, weight):
    """fp32 rows of heads times the weight, and the scale of each row."""
    x = x.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6)
    return x * r * weight, r


def _turn(x, cos, sin, layout):
    """The plain rotation in 32 bits: x [tokens, heads, dim], cos and sin [tokens, 1, rot / 2]."""
    n = cos.shape[-1]
    a, b = (x[..., :n], x[..., n:2 * n]) if layout == "half" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, w], dim=-1) if layout == "half" else torch.stack([u, w], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., 2 * n:]], dim=-1)


def _plain_step(s, case):
    held, keep, added, table, page = s["held"].long(), s["keep"].long(), s["added"].long(), s["page_table"], case["page"]
    old, length = -(-held // page), keep + added
    need = -(-length // page)
    back, more = (old - need).clamp(min=0), (need - old).clamp(min=0)
    col, capacity = torch.arange(table.shape[1], device="cuda"), s["free"].numel()
    count = s["count"].long()
    top = count + back.sum()
    # what comes back lies above the stack in order, what is taken comes from its new top
    stack = torch.cat([s["free"], s["free"].new_zeros(1)])
    at = count + (back.cumsum(0) - back)[:, None] + col - need[:, None]
    stack[torch.where((col >= need[:, None]) & (col < old[:, None]), at, capacity)] = table
    at = top - 1 - ((more.cumsum(0) - more)[:, None] + col - old[:, None])
    table.copy_(torch.where((col >= old[:, None]) & (col < need[:, None]), stack[at.clamp(0, capacity)], table))
    left = top - more.sum()
    s["free"].copy_(torch.where(torch.arange(capacity, device="cuda") < left, stack[:-1], s["free"]))
    q_start = torch.cat([added.new_zeros(1), added.cumsum(0)])
    t = torch.arange(s["tokens"], device="cuda")
    live = t < q_start[-1]
    seq = (q_start[1:, None] <= t).sum(dim=0).clamp(max=held.numel() - 1)
    i = t - q_start[seq]
    pos = keep[seq] + i
    slot = table[seq, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    out = {"q_start": q_start.to(torch.int32), "kv_len": length.to(torch.int32), "page_table": table, "free": s["free"],
           "left": left.to(torch.int32), "slots": torch.where(live, slot, -1)}
    if case["tree"]:
        seen, depth = _seen(torch.where(live, s["parent"], -1), seq, torch.where(live, i, -1), q_start, 32 * _words(case))
        pos = keep[seq] + depth
        out["mask"] = _bits(seen)
    out["positions"] = torch.where(live, pos, 0).to(torch.int32)
    return out


def _plain_append(s, case):
    live = s["slots"] >= 0
    n, page = case["rot"] // 2, case["page"]
    t = s["table"][s["positions"].long()]
    cos, sin = t[:, None, :n], t[:, None, n:]
    q = _turn(_normed(s["q"], s["q_weight"])[0], cos, sin, case["layout"]).to(s["out"].dtype)
    s["out"].copy_(torch.where(live[:, None, None], q, s["out"]))
    k = _turn(_normed(s["k"], s["k_weight"])[0], cos, sin, case["layout"])
    rows = s["slots"].numel() - case["pad"]             # padding is behind all rows
    slot = s["slots"][:rows]
    s["k_cache"][slot // page, slot % page] = k[:rows].to(s["k_cache"].dtype)
    s["v_cache"][slot // page, slot % page] = s["v"][:rows].to(s["v_cache"].dtype)
    return s["out"], s["k_cache"], s["v_cache"]


def _plain_train(s, case):
    n = case["rot"] // 2
    t = s["table"][s["positions"].long()]
    cos, sin = t[:, None, :n], t[:, None, n:]
    y, r = _normed(s["x"], s["weight"])
    s["out"].copy_(_turn(y, cos, sin, case["layout"]))
    g = _turn(s["dy"].float(), cos, -sin, case["layout"])
    unit = s["x"].float() * r
    s["dw"].copy_((g * unit).double().sum(dim=(0,) if case["per_head"] else (0, 1)))
    g = g * s["weight"]
    s["dx"].copy_(r * (g - unit * (g * unit).mean(dim=-1, keepdim=True)))
    return s["out"], s["dx"], s["dw"]


def _plain_tree(s, case):
    """All sequences at once, padded to the longest; rows and keys past a sequence's end are masked."""
    q, hk, d, page = s["q"], case["kv_heads"], case["dim"], case["page"]
    tokens, hq = q.shape[:2]
    bs, mq, mk = case["sequences"], case["chunk"], case["context"]
    start, keys = s["start"].long(), s["keys"].long()
    past = keys - (start[1:] - start[:-1])
    i, j = torch.arange(mq, device="cuda"), torch.arange(mk, device="cuda")
    row = (start[:-1, None] + i).clamp(max=tokens - 1)
    # [sequence, key head, query head of it, row, dim]
    qp = q[row].float().view(bs, mq, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(bs, hk, -1, d)
    there = j < keys[:, None]
    at = s["page_table"][:, (j // page).clamp(max=s["page_table"].shape[1] - 1)].long()
    at = torch.where(there, at, 0)
    k = s["k_cache"][at, j % page].float().permute(0, 2, 3, 1).contiguous()
    x = torch.matmul(qp, k).mul_(1.0 / math.sqrt(d)).view(bs, hk, hq // hk, mq, mk)
    del k
    node = (j - past[:, None]).clamp(0, 32 * s["mask"].shape[1] - 1)
    word = s["mask"].long()[row].gather(2, (node // 32)[:, None, :].expand(-1, mq, -1))
    drafted = (word >> (node % 32)[:, None, :]) & 1 > 0
    cached = (j < past[:, None])[:, None, :]
    if case["window"]:
        seen = torch.where(cached, j > s["positions"].long()[row][:, :, None] - case["window"], drafted)
    else:
        seen = cached | drafted
    seen = seen & there[:, None, :]
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    x.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = x.sum(dim=-1, keepdim=True)
    v = s["v_cache"][at, j % page].float().permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(x.view(bs, hk, -1, mk), v).view(bs, hk, hq // hk, mq, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(bs, mq, hq, d)
    t = torch.arange(tokens, device="cuda")
    seq = (start[1:, None] <= t).sum(dim=0)
    s["out"].copy_(o[seq, t - start[seq]])
    return s["out"]


def _plain_move(s, case):
    page, n = case["page"], s["path"].shape[1]
    start, keys = s["start"].long(), s["keys"].long()
    past = (keys - (start[1:] - start[:-1]))[:, None]
    i = torch.arange(n, device="cuda")
    at_to = torch.minimum(i, s["accepted"][:, None] - 1)     # places past the accepted ones repeat the last of these
    at_from, at_to = past + s["path"].long().gather(1, at_to), past + at_to
    table = s["page_table"].long()
    source = table.gather(1, at_from // page) * page + at_from % page
    target = table.gather(1, at_to // page) * page + at_to % page
    for cache in (s["k_cache"], s["v_cache"]):
        flat = cache.view(-1, *cache.shape[2:])
        flat[target] = flat[source]
    return s["k_cache"], s["v_cache"]


def _plain_logits(s, case):
    x = s["logits"].float()
    rows, vocab = x.shape
    place = torch.arange(s["history"].shape[1], device="cuda")
    there = place < s["length"][:, None]
    token = torch.where(there, s["history"].long(), vocab)
    counts = torch.zeros((2, rows, vocab + 1), device="cuda")
    counts[0].scatter_add_(1, token, torch.ones_like(token, dtype=torch.float32))
    counts[1].scatter_add_(1, torch.where(place < s["prompt"][:, None], vocab, token), torch.ones_like(token, dtype=torch.float32))
    seen, c = counts[0, :, :vocab] > 0, counts[1, :, :vocab]
    rho = s["repetition"][:, None]
    z = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
    z = z - s["frequency"][:, None] * c - torch.where(c > 0, s["presence"][:, None], 0.0)
    if "bias_token" in s:
        z.scatter_add_(1, s["bias_token"].long(), s["bias_value"])
    if "mask" in s:
        v = torch.arange(vocab, device="cuda")
        allowed = (s["mask"][:, v // 32] >> (v % 32)) & 1 > 0
        pick = s["mask_row"].long()
        z = torch.where(allowed[pick.clamp(min=0)] | (pick < 0)[:, None], z, float("-inf"))
    s["out"].copy_(z)
    return s["out"]


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"step": _plain_step, "append": _plain_append, "train": _plain_train, "tree": _plain_tree, "move": _plain_move,
                "logits": _plain_logits}[kind](state, case)
    import paper_2309_08978_amd as nj
    if kind == "step":
        step = nj.paged_step(state["step"], state["pool"], state["held"], state["added"], keep=state["keep"],
                             parent=state.get("parent"))
        out = {"q_start": step.q_start, "kv_len": step.kv_len, "page_table": step.page_table, "free": state["free"],
               "left": state["left"], "slots": step.slots, "positions": step.positions}
        return {**out, "mask": step.mask} if case["tree"] else out
    if kind == "append":
        nj.kv_append_slots(state["cache"], state["slots"], state["k"], state["v"], positions=state["positions"],
                           rotary=state["rotary"], q=state["q"], q_out=state["out"], norm=state["norm"])
        return state["out"], state["k_cache"], state["v_cache"]
    if kind == "train":
        nj.norm_rotary(state["x"], state["weight"], state["positions"], state["rotary"], eps=1e-6, out=state["out"])
        nj.norm_rotary_grad(state["dy"], state["x"], state["weight"], state["positions"], state["rotary"], eps=1e-6,
                            dx=state["dx"], dweight=state["dw"])
        return state["out"], state["dx"], state["dw"]
    if kind == "tree":
        return nj.tree_attention(state["q"], state["cache"], state["batch"], state["mask"], state["out"],
                                 positions=state["positions"], window=case["window"])
    if kind == "move":
        nj.kv_move(state["cache"], state["batch"], state["path"], state["accepted"])
        return state["k_cache"], state["v_cache"]
    return nj.adjust_logits(state["logits"], state["rules"], state["out"])


def _bytes_of(dtype):
    return 2 if dtype == "f16" else 4


def work(case):
    kind = case["kind"]
    if kind == "step":
        held, keep, added = _requests(case)
        page, n, rows = case["page"], case["sequences"], sum(added)
        moved = sum(abs(-(-(k + a) // page) - -(-h // page)) for h, k, a in zip(held, keep, added))
        words = _words(case)
        return {"bytes": 4 * (3 * n + 2 * n + 1) + 8 * moved + rows * (8 + 4 + (4 + 4 * words if words else 0)), "flops": 0}
    if kind == "logits":
        rows, vocab = case["rows"], case["vocab"]
        seen = sum(max(1, int(case["history"] * (1.0 - 0.9 * ((i * 0.6180339887) % 1.0)))) for i in range(rows))
        masks = 2 * 4 * -(-vocab // 32) if case["masked"] else 0
        return {"bytes": rows * vocab * (_bytes_of(case["src"]) + _bytes_of(case["dst"])) + 4 * seen + 8 * rows * case["biases"] + masks,
                "flops": 4 * rows * vocab}
    if kind == "train":
        n = case["tokens"] * case["heads"]
        return {"bytes": 4 * n * case["dim"] * _bytes_of(case["dtype"]) + 8 * case["tokens"] * (case["rot"] + 1),
                "flops": n * (6 * case["rot"] + 16 * case["dim"])}
    new, keys = _lengths(case)
    hk, d, e = case["kv_heads"], case["dim"], _bytes_of(case["dtype"])
    if kind == "append":
        t, hq = sum(new), case["q_heads"]
        return {"bytes": t * (hq + 2 * hk) * d * (_bytes_of(case["src"]) + e) + t * (4 * (case["rot"] + 1) + 8),
                "flops": t * (hq + hk) * (3 * case["rot"] + 4 * d)}
    if kind == "move":
        moved = sum(min(n, max(1, int(case["accepted"] * (1.0 - 0.6 * ((j * 0.4142135623) % 1.0))))) for j, n in enumerate(new))
        return {"bytes": moved * 4 * hk * d * e + 4 * moved, "flops": 0}
    hq = case["q_heads"]
    pairs = read = 0
    for n, m in zip(new, keys):
        w = min(case["window"] or m, m)
        pairs += n * min(m - n, w) + n * (1 + n // 6)       # about a third of the nodes of a chain a row
        read += min(m, n + w)
    pages = sum(-(-m // case["page"]) for m in keys)
    return {"bytes": (2 * sum(new) * hq + 2 * read * hk) * d * e + 4 * pages + 4 * sum(new) * -(-case["chunk"] // 32),
            "flops": 4 * pairs * hq * d}


def exact(case, seed):
    kind = case["kind"]
    if kind == "step":
        return None           # whole numbers only
    s = _inputs(case, seed)

    def normed(x, weight):
        x = x.double()
        return x / ((x ** 2).sum(dim=-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * weight.double()

    def turned(x, angle_rows, sign):
        out, n = x.clone(), case["rot"] // 2
        c, w = s["table"][angle_rows, :n].double()[:, None], sign * s["table"][angle_rows, n:].double()[:, None]
        first = torch.arange(n, device="cuda") * (1 if case["layout"] == "half" else 2)
        second = first + (n if case["layout"] == "half" else 1)
        a, b = x[..., first], x[..., second]
        out[..., first], out[..., second] = a * c - b * w, a * w + b * c
        return out

    if kind == "append":
        hq, hk, d, tokens = case["q_heads"], case["kv_heads"], case["dim"], s["slots"].numel() - case["pad"]
        x = s["qkv"].view(-1, hq + 2 * hk, d)
        at, where = s["positions"].long(), s["slots"][:tokens]
        q = turned(normed(x[:, :hq], s["q_weight"]), at, 1.0)
        q[tokens:] = 0.0
        k, v = s["k_cache"].double(), s["v_cache"].double()
        k.view(-1, hk, d)[where] = turned(normed(x[:, hq:hq + hk], s["k_weight"]), at, 1.0)[:tokens]
        v.view(-1, hk, d)[where] = x[:tokens, hq + hk:].double()
        return q, k, v
    if kind == "train":
        at = s["positions"].long()
        x, w = s["x"].double(), s["weight"].double()
        g = turned(s["dy"].double(), at, -1.0)
        size = ((x ** 2).mean(dim=-1, keepdim=True) + 1e-6).sqrt()
        # the norm's derivative: of x / size along each dim
        h = g * w / size
        dx = h - x * (h * x).sum(dim=-1, keepdim=True) / (case["dim"] * size ** 2)
        dw = g * x / size
        return turned(normed(s["x"], s["weight"]), at, 1.0), dx, dw.sum(dim=0) if case["per_head"] else dw.sum(dim=0).sum(dim=0)
    if kind == "logits":
        rows, vocab = case["rows"], case["vocab"]
        out = s["logits"].double()
        for r in range(rows):
            n, p = int(s["length"][r]), int(s["prompt"][r])
            seen = torch.bincount(s["history"][r, :n].long(), minlength=vocab) > 0
            c = torch.bincount(s["history"][r, p:n].long(), minlength=vocab).double()
            rho = s["repetition"][r].double()
            z = out[r].clone()
            z[seen & (out[r] > 0)] /= rho
            z[seen & ~(out[r] > 0)] *= rho
            z -= c * s["frequency"][r].double()
            z[c > 0] -= s["presence"][r].double()
            if "bias_token" in s:
                z[s["bias_token"][r].long()] += s["bias_value"][r].double()
            if "mask" in s and int(s["mask_row"][r]) >= 0:
                words = s["mask"][int(s["mask_row"][r])]
                bits = torch.stack([(words >> b) & 1 for b in range(32)], dim=1).flatten()[:vocab]
                z[bits == 0] = float("-inf")
            out[r] = z
        return out
    new, keys = _lengths(case)
    hk, d, page = case["kv_heads"], case["dim"], case["page"]
    pages = s["page_table"].cpu().tolist()
    if kind == "move":
        k, v = s["k_cache"].double(), s["v_cache"].double()
        path, count = s["path"].cpu().tolist(), s["accepted"].cpu().tolist()
        source, target = [], []
        for b, (n, m) in enumerate(zip(new, keys)):
            for i in range(count[b]):
                a, z = m - n + path[b][i], m - n + i
                source.append(pages[b][a // page] * page + a % page)
                target.append(pages[b][z // page] * page + z % page)
        source, target = torch.tensor(source, device="cuda"), torch.tensor(target, device="cuda")
        for c in (k, v):
            c.view(-1, hk, d)[target] = c.view(-1, hk, d)[source].clone()
        return k, v
    hq = case["q_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    begin = 0
    for b, (count, m) in enumerate(zip(new, keys)):
        slot = torch.tensor([pages[b][p // page] * page + p % page for p in range(m)], device="cuda")
        hidden = torch.zeros((count, m), dtype=torch.bool, device="cuda")
        words = s["mask"][begin:begin + count]
        bits = torch.stack([(words >> e) & 1 for e in range(32)], dim=2).flatten(1)[:, :count]
        hidden[:, m - count:] = bits == 0
        if case["window"]:
            j = torch.arange(m - count, device="cuda")[None, :]
            hidden[:, :m - count] = j <= s["positions"][begin:begin + count, None].long() - case["window"]
        for h in range(hk):
            k = s["k_cache"].view(-1, hk, d)[slot, h].double()
            v = s["v_cache"].view(-1, hk, d)[slot, h].double()
            for g in range(h * (hq // hk), (h + 1) * (hq // hk)):
                logits = (s["q"][begin:begin + count, g].double() @ k.t()) / math.sqrt(d)
                out[begin:begin + count, g] = torch.softmax(logits.masked_fill(hidden, float("-inf")), dim=1) @ v
        begin += count
    return out
