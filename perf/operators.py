"""Measured cases: the operators between a decoder layer's qkv linear and its
output linear when the layer is served from a paged cache.

Kinds of case

``rotary``     rotary positions on one tensor of rows: x[tokens, heads, dim],
               the first ``rot`` dims of every head turned by the angles of the
               row's position (``layout`` half: pairs (i, i + rot / 2);
               interleaved: pairs (2 i, 2 i + 1)); ``transpose``: the transposed
               turn, which takes a gradient back.  ``src`` and ``dst`` types
``append``     new keys (turned) and values go to their slots in a paged cache
               and the queries of the same rows are turned, all from the rows
               that a qkv linear gives: q, k and v are column ranges of one
               tensor [tokens, (q_heads + 2 kv_heads) dim] of type ``src``;
               cache and turned queries have type ``dtype``
``attention``  attention of every sequence's new tokens over its cached keys
               and values: causal (key j is seen from position j on) or not,
               ``window`` > 0: only the last ``window`` keys

A batch has ``sequences`` sequences of up to ``chunk`` new tokens each and up
to ``context`` keys with these; ``ragged`` = 0: all alike, towards 1: from
almost none to the largest.  Pages of ``page`` tokens lie in a pool in random
order.

Values: queries, keys and values N(0, 1), queries of attention N(0, 2) (logits
of a trained layer spread wider than those of random vectors), cos and sin of
base 10000, ``scaled``: for four times the trained length, the low
frequencies slowed down.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16}


def _rotary(name, tokens, heads, dim, rot, layout, src, dst, scaled=False, transpose=False):
    return {"name": name, "kind": "rotary", "tokens": tokens, "heads": heads, "dim": dim, "rot": rot, "layout": layout,
            "src": src, "dst": dst, "scaled": scaled, "transpose": transpose}


def _append(name, sequences, chunk, context, ragged, q_heads, kv_heads, dim, rot, layout, src, dtype, page, scaled=False):
    return {"name": name, "kind": "append", "sequences": sequences, "chunk": chunk, "context": context, "ragged": ragged,
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "layout": layout, "src": src,
            "dtype": dtype, "page": page, "scaled": scaled}


def _attention(name, sequences, chunk, context, ragged, q_heads, kv_heads, dim, dtype, page, causal=True, window=0):
    return {"name": name, "kind": "attention", "sequences": sequences, "chunk": chunk, "context": context,
            "ragged": ragged, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "causal": causal, "window": window}


def listed():
    return [
        # the smallest call: the query heads of one decoded token
        _rotary("rotary_token_f16", 1, 32, 128, 128, "half", "f16", "f16"),
        # the queries of a long prompt as its fp32 qkv linear gives them, rounded for the fp16 attention
        _rotary("rotary_prompt_f32", 4096, 32, 128, 128, "half", "f32", "f16", scaled=True),
        # decode step of eight sequences, four query heads to a key head
        _append("append_decode_f16", 8, 1, 2000, 0.9, 32, 8, 128, 128, "half", "f32", "f16", 16),
        # ragged prompts of an fp32 layer, interleaved pairs, half of each head turned
        _append("append_prompts_f32", 5, 777, 777, 0.9, 16, 16, 64, 32, "interleaved", "f32", "f32", 33),
        # decode attention of one sequence, every head with keys of its own
        _attention("decode_f16", 1, 1, 1023, 0.0, 32, 32, 128, "f16", 16),
        # decode step of a full serving batch of very different lengths
        _attention("decode_batch_f16", 32, 1, 4096, 0.95, 32, 8, 128, "f16", 64),
        # decode over one long document
        _attention("decode_long_f16", 1, 1, 65536, 0.0, 32, 8, 128, "f16", 128),
        # decode step of a base-size fp32 decoder
        _attention("decode_f32", 4, 1, 500, 0.5, 12, 12, 64, "f32", 16),
        # the next 512 tokens of a prompt that is taken in pieces
        _attention("chunk_f16", 1, 512, 2048, 0.0, 32, 32, 128, "f16", 16),
        # ragged prompts of small heads, all new, in one call
        _attention("prompts_f16", 6, 777, 777, 0.9, 12, 12, 64, "f16", 16),
        # the encoder's keys seen by every decoder position, fp32, four sequences of 256
        _attention("cross_f32", 4, 256, 256, 0.0, 16, 16, 64, "f32", 32, causal=False),
        # the largest call: 2048 new tokens at the end of 16384
        _attention("chunk_long_f16", 1, 2048, 16384, 0.0, 32, 8, 128, "f16", 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: single tokens to prompts of thousands,
    contexts to 65536, one to 32 sequences, heads of 64, 96 and 128 dims, one
    to eight query heads to a key head, pages of any size, both types."""
    pick = rng.random()
    dim = rng.choice([64, 96, 128, 128])
    rot = dim if rng.random() < 0.7 else dim // 2
    layout = rng.choice(["half", "interleaved"])
    dtype = rng.choice(["f32", "f16", "f16"])
    if pick < 0.15:
        return {"kind": "rotary", "tokens": _log_int(rng, 1, 4096), "heads": rng.choice([8, 12, 16, 32]), "dim": dim,
                "rot": rot, "layout": layout, "src": rng.choice(["f32", "f16"]), "dst": dtype,
                "scaled": rng.random() < 0.5, "transpose": rng.random() < 0.3}
    kv_heads = rng.choice([4, 8, 12, 16, 32])
    q_heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8) if kv_heads * g <= 32])
    page = rng.choice([16, 16, 32, 64, 128, _log_int(rng, 1, 200)])
    if pick < 0.3:
        sequences = _log_int(rng, 1, 32)
        chunk = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, 4096 // sequences))
        return {"kind": "append", "sequences": sequences, "chunk": chunk, "context": chunk + _log_int(rng, 1, 2000),
                "ragged": round(rng.uniform(0, 0.95), 3), "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
                "layout": layout, "src": rng.choice(["f32", "f16"]), "dtype": dtype, "page": page,
                "scaled": rng.random() < 0.5}
    decode = pick < 0.65
    while True:
        sequences = _log_int(rng, 1, 32)
        chunk = rng.choice([1, 1, 1, rng.randint(2, 5)]) if decode else _log_int(rng, 6, 2048)
        context = chunk + (_log_int(rng, 1, 65536 - chunk) if decode or rng.random() < 0.6 else 0)
        # no more keys, scores and products than the largest listed cases have
        if (sequences * context * kv_heads * dim <= 65536 * 8 * 128
                and sequences * chunk * context * q_heads <= 2048 * 16384 * 32 * (0.9 if dtype == "f16" else 0.1)):
            break
    causal = decode or rng.random() < 0.8
    window = _log_int(rng, 1, context) if causal and rng.random() < 0.2 else 0
    return {"kind": "attention", "sequences": sequences, "chunk": chunk, "context": context,
            "ragged": round(rng.uniform(0, 0.95), 3), "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "page": page, "causal": causal, "window": window}


def _lengths(case):
    """New tokens and keys of every sequence: spread over the range, the first sequence the longest."""
    new, keys = [], []
    for i in range(case["sequences"]):
        n = max(1, int(case["chunk"] * (1.0 - case["ragged"] * ((i * 0.6180339887) % 1.0))))
        past = int((case["context"] - case["chunk"]) * (1.0 - case["ragged"] * ((i * 0.7548776662) % 1.0)))
        new.append(n)
        keys.append(past + n)
    return new, keys


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1) + 29)
    return g


def _table(positions, rot, scaled):
    """[positions][cos of rot / 2 pairs, sin of rot / 2 pairs]."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaled:   # four times the trained 1024 positions: what turns less than once over these goes four times slower
        turns = 1024 * f / (2 * math.pi)
        keep = ((turns - 1) / 31).clamp(0, 1)
        f = f * keep + f / 4 * (1 - keep)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * f
    m = 0.1 * math.log(4) + 1.0 if scaled else 1.0
    return (torch.cat([a.cos(), a.sin()], dim=1) * m).float().cuda()


def _batch(case, g):
    """Starts, key counts and page table on the GPU; pages of the pool."""
    new, keys = _lengths(case)
    page = case["page"]
    need = [-(-n // page) for n in keys]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(keys), max(need)), -1, dtype=torch.int32)
    cols = torch.arange(max(need))
    used = cols[None, :] < torch.tensor(need)[:, None]
    table = table.cuda()
    table[used.cuda()] = order[:sum(need)]
    start = torch.zeros(len(new) + 1, dtype=torch.int32)
    start[1:] = torch.tensor(new).cumsum(0)
    return start.cuda(), torch.tensor(keys, dtype=torch.int32).cuda(), table, pages, sum(new)


def _inputs(case, seed):
    g = _generator(seed)

    def normal(*shape, dtype, scale=1.0):
        t = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
        return t.mul_(scale).to(dtype)

    if case["kind"] == "rotary":
        rows = max(2048, 2 * case["tokens"])
        first = int(torch.randint(0, rows - case["tokens"] + 1, (1,), generator=g, device="cuda"))
        return {"x": normal(case["tokens"], case["heads"], case["dim"], dtype=_DT[case["src"]]),
                "positions": torch.arange(first, first + case["tokens"], dtype=torch.int32, device="cuda"),
                "table": _table(rows, case["rot"], case["scaled"])}
    start, keys, table, pages, tokens = _batch(case, g)
    hq, hk, d, dt = case["q_heads"], case["kv_heads"], case["dim"], _DT[case["dtype"]]
    s = {"start": start, "keys": keys, "page_table": table,
         "k_cache": normal(pages, case["page"], hk, d, dtype=dt), "v_cache": normal(pages, case["page"], hk, d, dtype=dt)}
    if case["kind"] == "append":
        s["qkv"] = normal(tokens, (hq + 2 * hk) * d, dtype=_DT[case["src"]])
        s["table"] = _table(case["context"], case["rot"], case["scaled"])
    else:
        s["q"] = normal(tokens, hq, d, dtype=dt, scale=2.0)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "rotary":
        s["out"] = torch.empty(s["x"].shape, dtype=_DT[case["dst"]], device="cuda")
    elif case["kind"] == "append":
        hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
        rows = s["qkv"].view(-1, hq + 2 * hk, d)
        s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        s["out"] = torch.empty(s["q"].shape, dtype=_DT[case["dtype"]], device="cuda")
    else:
        s["out"] = torch.empty_like(s["q"])
    if own:
        # what a serving program keeps: the cache's and the table's handles, and the batch's, which every layer of a step shares
        import paper_2309_08978_amd as nj
        if "table" in s:
            s["rotary"] = nj.RotaryTable(s["table"], layout=case["layout"])
        if "k_cache" in s:
            s["cache"] = nj.PagedCache(s["k_cache"], s["v_cache"])
            s["batch"] = nj.PagedBatch(s["start"], s["keys"], s["page_table"], tokens=s["out"].shape[0],
                                       max_q=case["chunk"], max_kv=case["context"])
    return s


def _turn(x, cos, sin, layout):
    """The plain rotation in 32 bits: x [tokens, heads, dim], cos and sin [tokens, 1, rot / 2]."""
    n = cos.shape[-1]
    x = x.float()
    a, b = (x[..., :n], x[..., n:2 * n]) if layout == "half" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, w], dim=-1) if layout == "half" else torch.stack([u, w], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., 2 * n:]], dim=-1)


def _rows(start, keys, tokens):
    """Sequence and position of every new token."""
    new = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new, output_size=tokens)
    return seq, torch.arange(tokens, device="cuda") - start[seq] + (keys - new)[seq]


def _plain_append(s, case):
    q, k, v = s["q"], s["k"], s["v"]
    seq, pos = _rows(s["start"], s["keys"], q.shape[0])
    n = case["rot"] // 2
    cos, sin = s["table"][pos, None, :n], s["table"][pos, None, n:]
    s["out"].copy_(_turn(q, cos, sin, case["layout"]))
    page, slot = s["page_table"][seq, pos // case["page"]].long(), pos % case["page"]
    s["k_cache"][page, slot] = _turn(k, cos, sin, case["layout"]).to(s["k_cache"].dtype)
    s["v_cache"][page, slot] = v.to(s["v_cache"].dtype)
    return s["out"], s["k_cache"], s["v_cache"]


def _plain_attention(s, case):
    """All sequences at once, padded to the longest; rows and keys past a sequence's end are masked."""
    q, hk, d, page = s["q"], case["kv_heads"], case["dim"], case["page"]
    tokens, hq = q.shape[:2]
    bs, mq, mk = case["sequences"], case["chunk"], case["context"]
    start, keys = s["start"].long(), s["keys"].long()
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
    seen = there[:, None, :]
    if case["causal"]:
        pos = (keys - (start[1:] - start[:-1]))[:, None] + i
        seen = seen & (j <= pos[:, :, None])
        if case["window"]:
            seen = seen & (j > pos[:, :, None] - case["window"])
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    x.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = x.sum(dim=-1, keepdim=True)
    v = s["v_cache"][at, j % page].float().permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(x.view(bs, hk, -1, mk), v).view(bs, hk, hq // hk, mq, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(bs, mq, hq, d)
    seq, pos = _rows(s["start"], s["keys"], tokens)
    s["out"].copy_(o[seq, torch.arange(tokens, device="cuda") - start[seq]])
    return s["out"]


def run(state):
    case = state["case"]
    if own:
        import paper_2309_08978_amd as nj
        if case["kind"] == "rotary":
            return nj.rotary(state["x"], state["positions"], state["rotary"], state["out"], transpose=case["transpose"])
        if case["kind"] == "append":
            nj.kv_append(state["cache"], state["batch"], state["k"], state["v"], state["rotary"], state["q"], state["out"])
            return state["out"], state["k_cache"], state["v_cache"]
        return nj.paged_attention(state["q"], state["cache"], state["batch"], state["out"], causal=case["causal"],
                                  window=case["window"])
    if case["kind"] == "rotary":
        n = case["rot"] // 2
        t = state["table"][state["positions"].long()]
        cos, sin = t[:, None, :n], t[:, None, n:]
        state["out"].copy_(_turn(state["x"], cos, -sin if case["transpose"] else sin, case["layout"]))
        return state["out"]
    return _plain_append(state, case) if case["kind"] == "append" else _plain_attention(state, case)


def _bytes_of(dtype):
    return 2 if dtype == "f16" else 4


def work(case):
    if case["kind"] == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": n * case["dim"] * (_bytes_of(case["src"]) + _bytes_of(case["dst"])) + case["tokens"] * 4 * (case["rot"] + 1),
                "flops": 3 * n * case["rot"]}
    new, keys = _lengths(case)
    hq, hk, d, e = case["q_heads"], case["kv_heads"], case["dim"], _bytes_of(case["dtype"])
    if case["kind"] == "append":
        t = sum(new)
        return {"bytes": t * (hq + 2 * hk) * d * (_bytes_of(case["src"]) + e) + t * 4 * (case["rot"] + 1),
                "flops": 3 * t * (hq + hk) * case["rot"]}
    pairs = read = 0
    for n, m in zip(new, keys):
        if not case["causal"]:
            pairs, read = pairs + n * m, read + m
            continue
        w = case["window"] or m
        first = m - n + 1    # keys that the first new token sees without a window; the last one sees m
        full = max(0, min(n, w - first))      # rows that the window does not cut
        pairs += full * first + full * (full - 1) // 2 + (n - full) * w
        read += min(m, n - 1 + w)
    pages = sum(-(-m // case["page"]) for m in keys)
    return {"bytes": (2 * sum(new) * hq + 2 * read * hk) * d * e + 4 * pages, "flops": 4 * pairs * hq * d}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] != "attention":
        n = case["rot"] // 2

        def turned(x, angle_rows, sign):
            out = x.double().clone()
            c, w = s["table"][angle_rows, :n].double()[:, None], sign * s["table"][angle_rows, n:].double()[:, None]
            first = torch.arange(n, device="cuda") * (1 if case["layout"] == "half" else 2)
            second = first + (n if case["layout"] == "half" else 1)
            a, b = x[..., first].double(), x[..., second].double()
            out[..., first], out[..., second] = a * c - b * w, a * w + b * c
            return out

    if case["kind"] == "rotary":
        return turned(s["x"], s["positions"].long(), -1.0 if case["transpose"] else 1.0)
    new, keys = _lengths(case)
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    pages = s["page_table"].cpu().tolist()
    if case["kind"] == "append":
        where, rows = [], []
        for b, (count, m) in enumerate(zip(new, keys)):
            for p in range(m - count, m):
                where.append(pages[b][p // page] * page + p % page)
                rows.append(p)
        where, rows = torch.tensor(where, device="cuda"), torch.tensor(rows, device="cuda")
        x = s["qkv"].view(-1, hq + 2 * hk, d)
        k, v = s["k_cache"].double(), s["v_cache"].double()
        k.view(-1, hk, d)[where] = turned(x[:, hq:hq + hk], rows, 1.0)
        v.view(-1, hk, d)[where] = x[:, hq + hk:].double()
        return turned(x[:, :hq], rows, 1.0), k, v
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    begin = 0
    for b, (count, m) in enumerate(zip(new, keys)):
        slot = torch.tensor([pages[b][p // page] * page + p % page for p in range(m)], device="cuda")
        pos = torch.arange(m - count, m, device="cuda")[:, None]
        j = torch.arange(m, device="cuda")[None, :]
        hidden = torch.zeros((count, m), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = j > pos
            if case["window"]:
                hidden |= j <= pos - case["window"]
        for h in range(hk):
            k = s["k_cache"].view(-1, hk, d)[slot, h].double()
            v = s["v_cache"].view(-1, hk, d)[slot, h].double()
            for g in range(h * (hq // hk), (h + 1) * (hq // hk)):
                logits = (s["q"][begin:begin + count, g].double() @ k.t()) / math.sqrt(d)
                out[begin:begin + count, g] = torch.softmax(logits.masked_fill(hidden, float("-inf")), dim=1) @ v
        begin += count
    return out
