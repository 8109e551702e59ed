"""Plain 64-bit forms of the serving operators, and batches to test them on.

Pools are poisoned: every slot that no sequence uses holds NaN or infinities,
and page table entries past the used pages hold ids outside the pool."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2309_08978_amd as nj

U32, U16 = 2.0 ** -24, 2.0 ** -11      # half a unit in the last place, relative
DT = {"f32": torch.float32, "f16": torch.float16}


class Batch:
    """Ragged sequences in a paged cache: host copies (exact) and device tensors.

    news, keys: new tokens and keys (with the new ones) per sequence; a
    sequence whose keys are fewer than its new tokens has rows without a key.
    order 'nhd': pool [page, slot, head, dim]; 'hnd': [page, head, slot, dim].
    pad: rows behind the last sequence.  shift: the pool and head rows begin
    that many elements into their buffers (unaligned)."""

    def __init__(self, news, keys, q_heads, kv_heads, dim, page, dtype, seed=0, order="nhd", pad=0, shift=0, extra_dim=0,
                 q_scale=1.0, row_gap=0):
        self.news, self.keys, self.hq, self.hk, self.dim, self.page, self.dtype = news, keys, q_heads, kv_heads, dim, page, dtype
        rng = np.random.default_rng([seed, len(news), dim, page])
        dt = DT[dtype]
        need = [-(-n // page) for n in keys]
        pages = sum(need) + 2
        order_of_pages = rng.permutation(pages)
        cols = max(need + [1])
        self.table = np.full((len(keys), cols + 1), 1 << 30, dtype=np.int32)
        self.table[:, 1::2] = -7
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order_of_pages[at:at + n]
            at += n
        self.tokens = sum(news) + pad
        self.start = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        width = dim + extra_dim
        shape = (pages, page, kv_heads, width) if order == "nhd" else (pages, kv_heads, page, width)

        def pool(poison):
            flat = torch.full((math.prod(shape) + shift,), poison, dtype=dt)
            t = flat[shift:].view(shape)[..., :dim]
            return t if order == "nhd" else t.transpose(1, 2)

        self.k, self.v = pool(float("nan")), pool(float("inf"))
        self.v[..., ::2] = float("nan")
        for b, n in enumerate(keys):
            for j in range(n):
                pg, slot = self.table[b, j // page], j % page
                self.k[pg, slot] = torch.from_numpy(rng.standard_normal((kv_heads, dim))).to(dt)
                self.v[pg, slot] = torch.from_numpy(rng.standard_normal((kv_heads, dim))).to(dt)
        rows = torch.zeros((self.tokens * (q_heads * dim + row_gap) + shift,), dtype=dt)
        self.q = rows[shift:].view(self.tokens, q_heads * dim + row_gap)[:, :q_heads * dim].view(self.tokens, q_heads, dim) \
            if row_gap == 0 else torch.as_strided(rows, (self.tokens, q_heads, dim), (q_heads * dim + row_gap, dim, 1), shift)
        self.q.copy_(torch.from_numpy(rng.standard_normal((self.tokens, q_heads, dim)) * q_scale).to(dt))

    @staticmethod
    def _to_device(t):
        """The tensor on the GPU with the same strides and alignment."""
        base = t._base if t._base is not None else t
        while base._base is not None:
            base = base._base
        return torch.as_strided(base.cuda(), t.shape, t.stride(), t.storage_offset())

    def device(self, max_q=None, max_kv=None):
        d = self
        d.dq, d.dk, d.dv = self._to_device(self.q), self._to_device(self.k), self._to_device(self.v)
        d.cache = nj.PagedCache(d.dk, d.dv)
        d.batch = nj.PagedBatch(torch.from_numpy(self.start).cuda(), torch.tensor(self.keys, dtype=torch.int32, device="cuda"),
                                torch.from_numpy(self.table).cuda(), tokens=self.tokens,
                                max_q=max(self.news) if max_q is None else max_q,
                                max_kv=max(self.keys) if max_kv is None else max_kv)
        return d

    def key_slots(self, b):
        n = self.keys[b]
        return [(int(self.table[b, j // self.page]), j % self.page) for j in range(n)]


def attention(B: Batch, scale=None, causal=True, window=0):
    """(out [tokens, heads, dim] in fp64, elementwise error bound of an fp32 or fp16 kernel); rows of no sequence are NaN.

    Bound: logits are sums of dim fp32 products, off by at most (dim + 4) U32 scale |q| |k|; a logit off by e changes its weight
    by a factor 1 +- e, so all of them move the result by at most 2 max(e) max|v|; sums of n weights and n products round
    2 n times; exp2 of an argument x rounds it by |x| U32 and gives 2 ulp.  fp16: weights rounded to 11 bits, and the result."""
    scale = B.dim ** -0.5 if scale is None else scale
    out = np.full((B.tokens, B.hq, B.dim), np.nan)
    bound = np.zeros_like(out)
    q, group = B.q.double().numpy(), B.hq // B.hk
    for b, (n, m) in enumerate(zip(B.news, B.keys)):
        slots = B.key_slots(b)
        k = np.stack([B.k[s].double().numpy() for s in slots]) if slots else np.zeros((0, B.hk, B.dim))
        v = np.stack([B.v[s].double().numpy() for s in slots]) if slots else np.zeros((0, B.hk, B.dim))
        pos = np.arange(m - n, m)[:, None]
        j = np.arange(m)[None, :]
        seen = (j <= pos) if causal else np.ones((n, m), dtype=bool)
        if causal and window:
            seen &= j > pos - window
        rows = slice(B.start[b], B.start[b] + n)
        some = seen.any(1)
        for h in range(B.hq if n else 0):
            out[rows, h] = 0.0
            if not some.any():
                continue
            kk, vv, qq = k[:, h // group], v[:, h // group], q[rows, h]
            with np.errstate(all="ignore"):
                # masked places are taken out before any arithmetic: their logits are -inf, their values met by no weight
                x = np.where(seen, scale * (qq @ kk.T), -np.inf)
                top = x.max(1, keepdims=True)
                w = np.where(seen, np.exp(x - top), 0.0)
                # (a sum of nothing but infinities and NaN is left to the formula, row by row)
                fine = np.isfinite(vv).all()
                if fine:
                    o = w @ vv
                else:
                    o = np.stack([(w[i, seen[i]][:, None] * vv[seen[i]]).sum(0) for i in range(n)])
                o = o / w.sum(1, keepdims=True)
                size = abs(scale) * np.linalg.norm(qq, axis=1) * np.where(seen, np.linalg.norm(kk, axis=1), 0.0).max(1)
                spread = np.where(seen, np.abs(x - top), 0.0).max(1)
                e = (B.dim + 4) * U32 * size + 2 * U32 * spread + 4 * U32
                most = np.where(seen[:, :, None], np.abs(vv)[None], 0.0).max((1, 2)) if not fine else \
                    np.where(seen, np.abs(vv).max(1)[None], 0.0).max(1)
                bd = (most * (2 * e + 2 * seen.sum(1) * U32))[:, None] * np.ones((1, B.dim))
                if B.dtype == "f16":
                    bd = bd + most[:, None] * U16 + np.abs(o) * U16 + 2.0 ** -24
            out[rows, h] = np.where(some[:, None], o, 0.0)
            bound[rows, h] = np.where(some[:, None], bd, 0.0)
    return out, np.where(np.isfinite(bound), bound, np.inf)


def check_attention(B: Batch, got, scale=None, causal=True, window=0):
    """Every element inside its bound, infinities and NaN where the formula has them; the whole within the relative norm
    that roundings of independent sign leave (fp32: 1e-5, the bar of this library's products; fp16: two roundings to 11
    bits, whose mean square is U16 / sqrt(3) times at most 1, so below 2 U16)."""
    ref, bound = attention(B, scale, causal, window)
    rows = sum(B.news)
    got, ref, bound = got[:rows].double().cpu().numpy(), ref[:rows], bound[:rows]
    assert np.array_equal(np.isnan(got), np.isnan(ref)), "NaN in other places"
    inf = np.isinf(ref)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], ref[inf]), "infinities in other places"
    fine = np.isfinite(ref)
    off = got[fine] - ref[fine]
    worst = (np.abs(off) - bound[fine]).max() if fine.any() else 0.0
    assert worst <= 0, f"an element is {worst} beyond its bound"
    norm = np.linalg.norm(ref[fine])
    if norm > 0:
        rel = np.linalg.norm(off) / norm
        assert rel <= (1e-5 if B.dtype == "f32" else 2 * U16), rel


def turn(x, cos, sin, layout, sign=1.0):
    """x [tokens, heads, dim] fp64 turned; cos, sin [tokens, pairs]; and the error bound of fp32 arithmetic."""
    n = cos.shape[1]
    y, bound = x.copy(), np.zeros_like(x)
    i = np.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    c, s = cos[:, None, :], sign * sin[:, None, :]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size = 3 * U32 * (np.abs(x[..., a]) + np.abs(x[..., b])) * np.maximum(np.abs(c), np.abs(s))
    bound[..., a], bound[..., b] = size, size
    return y, bound


def rounded(y, bound, dtype):
    """The bound after rounding to dtype."""
    u, tiny = (U16, 2.0 ** -25) if dtype == "f16" else (U32, 2.0 ** -149)
    return bound + (np.abs(y) + bound) * u + tiny
