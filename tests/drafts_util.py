"""Plain forms of the operators of a step of drafted tokens: lists and 64 bits."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import torch

import paper_2309_08978_amd as nj
from tests.serving_util import U16, U32, turn

MISSING, LENGTHS, ROWS, POOL = 1, 2, 4, 8


def plain_step(held, keep, added, table, stack, count, capacity, page, tokens, parent=None, words=0):
    """The arrays of a step, sequence by sequence and page by page.  table: list of lists (changed), stack: list (changed).
    -> dict of q_start, kv_len, positions, slots, mask, status, count."""
    n, columns = len(held), len(table[0]) if table else 0
    need = lambda t: -(-t // page)  # noqa: E731
    bad = 0
    for h, k, a in zip(held, keep, added):
        if h < 0 or k < 0 or k > h or a < 0 or max(h, k + a) > min(columns * page, 1 << 30):
            bad |= LENGTHS
        elif parent is not None and a > 32 * words:
            bad |= ROWS
    fine = [h >= 0 and 0 <= k <= h and a >= 0 and max(h, k + a) <= min(columns * page, 1 << 30) for h, k, a in zip(held, keep, added)]
    if sum(a for a, ok in zip(added, fine) if ok) > tokens:
        bad |= ROWS
    back = [(b, c) for b in range(n) if fine[b] for c in range(need(keep[b] + added[b]), need(held[b]))]
    more = [(b, c) for b in range(n) if fine[b] for c in range(need(held[b]), need(keep[b] + added[b]))]
    if not 0 <= count <= capacity or count + len(back) > capacity:
        bad |= POOL
    missing = 0 if bad & (LENGTHS | POOL) else max(0, len(more) - len(back) - count)
    if missing:
        bad |= MISSING
    out = {"positions": [0] * tokens, "slots": [-1] * tokens, "mask": [[0] * words for _ in range(tokens)]}
    if bad:
        return {**out, "q_start": [0] * (n + 1), "kv_len": list(held), "status": [bad, missing, 0, count], "count": count}
    free = stack[:count] + [table[b][c] for b, c in back]
    for b, c in more:
        table[b][c] = free.pop()
    stack[count:len(free)] = free[count:]
    starts, t = [0], 0
    for b in range(n):
        seen = []
        for i in range(added[b]):
            place = keep[b] + i
            pg = table[b][place // page]
            out["slots"][t] = pg * page + place % page if pg >= 0 else -1
            out["positions"][t] = place
            if parent is not None:
                p = parent[t]
                mine = {i} | (seen[p] if 0 <= p < i else set())
                seen.append(mine)
                out["positions"][t] = keep[b] + len(mine) - 1
                for j in mine:
                    out["mask"][t][j // 32] |= 1 << j % 32
            t += 1
        starts.append(t)
    return {**out, "q_start": starts, "kv_len": [k + a for k, a in zip(keep, added)], "status": [0, 0, t, len(free)], "count": len(free)}


def signed(word):
    return word - (1 << 32) if word >= 1 << 31 else word


def normed(x, weight, eps):
    """x [..., dim] fp64 normed and its bound.  The sum of n squares, each rounded, in any order is off by n U32 of itself; its
    mean and eps round twice more; the root of a relative error e is off by e / 2, rsqrt by an ulp (2 U32); two products."""
    n = x.shape[-1]
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    return y, ((n + 2) / 2 + 4) * U32 * np.abs(y)


def turned_with_bound(x, bound, cos, sin, layout, sign=1.0):
    """turn() of values that are off by `bound`."""
    y, b = turn(x, cos, sin, layout, sign)
    carried, _ = turn(bound, np.abs(cos), -np.abs(sin), layout)     # |a c| + |b s| for the first side ...
    other, _ = turn(bound, np.abs(cos), np.abs(sin), layout)        # ... and for the second
    return y, 1.01 * b + np.maximum(np.abs(carried), np.abs(other))


def norm_grad(x, dy, weight, eps, cos, sin, layout):
    """(dx, dw per head and dim, bounds) in fp64 for x, dy [tokens, heads, dim].

    Of dx = r (h - u m), h = g w: r is off by (n / 2 + 4) U32 of itself, g by 3 U32 of the sides' sizes, u = x r by n / 2 + 5, m,
    a sum of n products times r / n, by n + 4 and r's; dx adds three roundings: less than (2 n + 20) U32 of the sizes together.
    dw: a sum over the rows of products of that g and u."""
    n = x.shape[-1]
    g, gb = turn(dy, cos, sin, layout, -1.0) if cos is not None else (dy, np.zeros_like(dy))
    size = np.abs(g) + gb / U32           # what g's roundings are relative to: three times its sides
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u, h = x * r, g * weight
    m = (h * u).mean(-1, keepdims=True)
    dx = r * (h - u * m)
    sizes = r * (size * np.abs(weight) + np.abs(u) * (size * np.abs(weight) * np.abs(u)).mean(-1, keepdims=True))
    rows = x.shape[0]
    dw = (g * u).sum(0)
    dwb = (rows + n / 2 + 12) * U32 * (size * np.abs(u)).sum(0)
    return dx, dw, (2 * n + 20) * U32 * sizes, dwb


def tree_seen(B, mask, window=0, positions=None):
    """What every new token of a serving_util.Batch sees: a bool [new, keys] a sequence."""
    words = mask.shape[1]
    out = []
    for b, (n, m) in enumerate(zip(B.news, B.keys)):
        seen = np.zeros((n, m), dtype=bool)
        past = m - n
        for i in range(n):
            t = B.start[b] + i
            lo = 0
            if window:
                p = min(max(int(positions[t]), past), past + n - 1)
                lo = max(p - window + 1, 0)
            seen[i, lo:max(past, 0)] = True
            for j in range(max(0, -past), min(n, 32 * words)):
                if int(mask[t, j // 32]) >> j % 32 & 1:
                    seen[i, past + j] = True
        out.append(seen)
    return out


def attention_of(B, seen, scale=None):
    """(out, bound) in fp64 of a serving_util.Batch whose rows see `seen`; bounds as serving_util.attention derives them."""
    scale = B.dim ** -0.5 if scale is None else scale
    out = np.full((B.tokens, B.hq, B.dim), np.nan)
    bound = np.zeros_like(out)
    q, group = B.q.double().numpy(), B.hq // B.hk
    for b, (n, m) in enumerate(zip(B.news, B.keys)):
        slots = B.key_slots(b)
        k = np.stack([B.k[s].double().numpy() for s in slots]) if slots else np.zeros((0, B.hk, B.dim))
        v = np.stack([B.v[s].double().numpy() for s in slots]) if slots else np.zeros((0, B.hk, B.dim))
        rows, sees = slice(B.start[b], B.start[b] + n), seen[b]
        some = sees.any(1)[:, None]
        for h in range(B.hq if n else 0):
            qq, kk, vv = q[rows, h], k[:, h // group], v[:, h // group]
            out[rows, h] = 0.0
            if not some.any():
                continue
            with np.errstate(all="ignore"):
                x = np.where(sees, scale * (qq @ kk.T), -np.inf)
                top = x.max(1, keepdims=True)
                w = np.where(sees, np.exp(x - top), 0.0)
                fine = np.isfinite(vv).all()
                # (a sum of values that are not finite is left to the formula, row by row, over what the row sees)
                o = w @ vv if fine else np.stack([(w[i, sees[i]][:, None] * vv[sees[i]]).sum(0) for i in range(n)])
                o = o / w.sum(1, keepdims=True)
                size = abs(scale) * np.linalg.norm(qq, axis=1) * np.where(sees, np.linalg.norm(kk, axis=1), 0.0).max(1)
                e = (B.dim + 4) * U32 * size + 2 * U32 * np.where(sees, np.abs(x - top), 0.0).max(1) + 4 * U32
                most = np.where(sees, np.abs(vv).max(1), 0.0).max(1)
                bd = (most * (2 * e + 2 * sees.sum(1) * U32))[:, None] * np.ones((1, B.dim))
                if B.dtype == "f16":
                    bd = bd + most[:, None] * U16 + np.abs(o) * U16 + 2.0 ** -24
            out[rows, h], bound[rows, h] = np.where(some, o, 0.0), np.where(some, bd, 0.0)
    return out, np.where(np.isfinite(bound), bound, np.inf)


class Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("tile_rows", "row_tiles", "splits", "split_keys", "waves")] + [("ws_floats", ctypes.c_int64)]


def tree_plan(dtype, news, keys, hq, hk, dim, window=0, cus=256) -> Plan:
    """nnjit::tree_plan (csrc/serving.h) for a batch whose max_q and max_kv are its longest."""
    f = nj.load(build_if_missing=True)._ZN5nnjit9tree_planEilliiillli
    i, n = ctypes.c_int, ctypes.c_int64
    f.restype, f.argtypes = Plan, [i, n, n, i, i, i, n, n, n, i]
    return f(nj.NNJIT_F16 if dtype == "f16" else nj.NNJIT_F32, sum(news), len(news), hq, hk, dim, max(news), max(keys),
             window + max(news) if window else 0, cus)


# (dtype, new tokens, keys, query heads, key heads, dim, tile rows, split over the keys, waves): every tile height, split and
# unsplit, for each class of head dims of either type
TREE_COVER = [
    ("f16", [4, 1], [24, 14], 1, 1, 64, 16, False, 4),
    ("f16", [4, 1], [204, 134], 1, 1, 64, 16, False, 8),
    ("f16", [4, 1], [1004, 667], 1, 1, 64, 16, True, 4),
    ("f16", [40, 7, 1], [60, 20, 21], 64, 16, 64, 64, False, 4),
    ("f16", [40, 7, 1], [3040, 2007, 3001], 4, 4, 64, 64, True, 4),
    ("f16", [128, 1, 100, 90, 77, 128], [148, 14, 120, 96, 90, 148], 64, 16, 64, 128, False, 4),
    ("f16", [40, 7, 1], [2040, 1340, 2001], 32, 8, 64, 128, True, 4),
    ("f16", [4, 1], [24, 14], 1, 1, 96, 16, False, 4),
    ("f16", [4, 1], [204, 134], 1, 1, 96, 16, False, 8),
    ("f16", [4, 1], [504, 334], 1, 1, 96, 16, True, 4),
    ("f16", [40, 7, 1], [60, 20, 21], 64, 16, 96, 64, False, 4),
    ("f16", [40, 7, 1], [2040, 1340, 2001], 4, 4, 96, 64, True, 4),
    ("f16", [128, 1, 100, 90, 77, 128], [148, 14, 120, 96, 90, 148], 64, 16, 96, 128, False, 4),
    ("f16", [40, 7, 1], [2040, 1340, 2001], 32, 8, 96, 128, True, 4),
    ("f16", [4, 1], [24, 14], 1, 1, 128, 16, False, 4),
    ("f16", [4, 1], [304, 201], 1, 1, 128, 16, True, 4),
    ("f16", [40, 7, 1], [60, 20, 21], 64, 16, 128, 64, False, 4),
    ("f16", [40, 7, 1], [2040, 1340, 2001], 4, 4, 128, 64, True, 4),
    ("f16", [128, 1, 100, 90, 77, 128], [148, 14, 120, 96, 90, 148], 64, 16, 128, 128, False, 4),
    ("f16", [40, 7, 1], [3040, 2007, 3001], 64, 16, 128, 128, True, 4),
    ("f16", [4, 1], [24, 14], 1, 1, 200, 16, False, 4),
    ("f16", [4, 1], [304, 201], 1, 1, 200, 16, True, 4),
    ("f16", [40, 7, 1], [60, 20, 21], 64, 16, 200, 128, False, 4),
    ("f16", [40, 7, 1], [540, 340, 501], 16, 4, 200, 128, True, 4),
    ("f32", [4, 1], [24, 14], 1, 1, 64, 16, False, 4),
    ("f32", [4, 1], [204, 134], 1, 1, 64, 16, False, 8),
    ("f32", [4, 1], [504, 334], 1, 1, 64, 16, True, 4),
    ("f32", [100, 3], [120, 16], 64, 16, 64, 64, False, 4),
    ("f32", [40, 7, 1], [1040, 673, 1001], 16, 4, 64, 64, True, 4),
    ("f32", [100, 31, 77, 90], [120, 44, 97, 96], 64, 16, 64, 128, False, 4),
    ("f32", [40, 33, 40, 1], [540, 366, 540, 167], 32, 8, 64, 128, True, 4),
    ("f32", [4, 1], [24, 14], 1, 1, 96, 16, False, 4),
    ("f32", [4, 1], [204, 134], 1, 1, 96, 16, False, 8),
    ("f32", [4, 1], [304, 201], 1, 1, 96, 16, True, 4),
    ("f32", [100, 3], [120, 16], 64, 16, 96, 64, False, 4),
    ("f32", [40, 7, 1], [1040, 673, 1001], 16, 4, 96, 64, True, 4),
    ("f32", [100, 31, 77, 90], [120, 44, 97, 96], 64, 16, 96, 128, False, 4),
    ("f32", [100, 3], [1100, 669], 16, 4, 96, 128, True, 4),
    ("f32", [4, 1], [24, 14], 1, 1, 128, 16, False, 4),
    ("f32", [4, 1], [204, 134], 1, 1, 128, 16, True, 4),
    ("f32", [100, 3], [120, 16], 64, 16, 128, 64, False, 4),
    ("f32", [128, 1, 100, 90, 77, 128], [1128, 667, 1100, 423, 743, 1128], 2, 1, 128, 64, True, 4),
    ("f32", [100, 31, 77, 90], [120, 44, 97, 96], 64, 16, 128, 128, False, 4),
    ("f32", [100, 3], [1100, 669], 16, 4, 128, 128, True, 4),
    ("f32", [4, 1], [24, 14], 1, 1, 200, 16, False, 4),
    ("f32", [4, 1], [204, 134], 1, 1, 200, 16, True, 4),
    ("f32", [100, 31, 77, 90], [120, 44, 97, 96], 64, 16, 200, 128, False, 4),
    ("f32", [128, 1, 100, 90, 77, 128], [2128, 1334, 2100, 756, 1410, 2128], 2, 1, 200, 128, True, 4),
]


def cover_name(case) -> str:
    dtype, news, keys, hq, hk, dim, rows, split, waves = case
    return f"{dtype}-{dim}-{rows}rows-{'split' if split else 'whole'}-{waves}waves"


def random_mask(B, words, rng, density=0.4):
    """Random words: bits of tokens that a sequence does not have among them."""
    bits = rng.random((B.tokens, words, 32)) < density
    return (bits.astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)


def tree_mask(B, words, rng):
    """Ancestors of random trees; (mask, depth of every row)."""
    mask, depth = np.zeros((B.tokens, words), dtype=np.uint32), np.zeros(B.tokens, dtype=np.int64)
    for b, n in enumerate(B.news):
        for i in range(n):
            t = B.start[b] + i
            p = int(rng.integers(-1, i)) if i else -1
            if p >= 0:
                mask[t] = mask[B.start[b] + p]
                depth[t] = depth[B.start[b] + p] + 1
            mask[t, i // 32] |= np.uint32(1 << i % 32)
    return mask, depth


def plain_logits(x, history=None, length=None, prompt=None, repetition=None, presence=None, frequency=None, bias=None, allowed=None):
    """Rows of logits under the rules in fp64, and the bound of fp32 arithmetic (an operation each rounds to U32 of its size).
    history: a list of tokens a row; bias: a list of (token, value) a row; allowed: bool [rows, vocab]."""
    z = x.astype(np.float64).copy()
    rows, vocab = z.shape
    size = np.abs(z)
    for r in range(rows):
        if history is not None:
            n = len(history[r]) if length is None else min(max(length[r], 0), len(history[r]))
            tokens = history[r][:n]
            made = tokens[max(0, prompt[r]) if prompt is not None else 0:]
            seen = {t for t in tokens if 0 <= t < vocab}
            for t in seen:
                if repetition is not None:
                    z[r, t] = z[r, t] / float(repetition[r]) if z[r, t] > 0 else z[r, t] * float(repetition[r])
                c = made.count(t)
                size[r, t] += abs(z[r, t])
                if c:
                    f, p = float(frequency[r]) if frequency is not None else 0.0, float(presence[r]) if presence is not None else 0.0
                    z[r, t] = z[r, t] - f * c - p
                    size[r, t] += abs(f * c) * 2 + abs(p)
        if bias is not None:
            last = {t: float(v) for t, v in bias[r] if 0 <= t < vocab}
            for t, v in last.items():
                z[r, t] += v
                size[r, t] += abs(v)
    bound = 4 * U32 * size
    if allowed is not None:
        z = np.where(allowed, z, -math.inf)
        bound = np.where(allowed, bound, 0.0)
    return z, bound


def words_of(allowed):
    """int32 words of bool [rows, vocab]."""
    rows, vocab = allowed.shape
    padded = np.zeros((rows, -(-vocab // 32) * 32), dtype=np.uint64)
    padded[:, :vocab] = allowed
    w = (padded.reshape(rows, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32))


class LogitPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("threads", "quads", "narrow")]


def logit_plan(rows, vocab, history, biases=60, cus=256) -> LogitPlan:
    """nnjit::logit_plan (csrc/serving.h)."""
    f = nj.load(build_if_missing=True)._ZN5nnjit10logit_planElllli
    f.restype, f.argtypes = LogitPlan, [ctypes.c_int64] * 4 + [ctypes.c_int]
    return f(rows, vocab, history, biases, cus)


# (rows, vocab, history, threads, groups of four tokens a thread, one word of LDS a token): every kernel of the logit rules,
# rows of one segment and of several, with last segments that hold little
LOGIT_COVER = [
    (5, 4097, 64, 512, 1, True),
    (2, 130, 4096, 512, 1, True),
    (3, 9001, 5000, 1024, 1, True),
    (130, 4099, 90, 1024, 2, True),
    (3, 9001, 33000, 1024, 1, False),
    (300, 9001, 50, 1024, 2, True),
    (130, 9000, 33000, 1024, 2, False),
    (256, 16390, 90, 1024, 4, True),
    (400, 9001, 50, 1024, 4, True),
    (2100, 701, 20, 1024, 4, True),
]
