"""Shapes that reach every attention kernel, the plan that the library makes
of a shape, and a check of every element against the formula."""
from __future__ import annotations

import ctypes

import numpy as np

import paper_2309_08978_amd as nj
from tests.serving_util import U16, U32, Batch


class Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("tile_rows", "row_tiles", "splits", "split_keys", "waves")] + [("ws_floats", ctypes.c_int64)]


def plan(dtype, news, keys, hq, hk, dim, causal=True, window=0, cus=256) -> Plan:
    """nnjit::attention_plan (csrc/serving.h) for a batch whose max_q and max_kv are its longest."""
    f = nj.load(build_if_missing=True)._ZN5nnjit14attention_planEilliiillili
    i, n = ctypes.c_int, ctypes.c_int64
    f.restype, f.argtypes = Plan, [i, n, n, i, i, i, n, n, i, n, i]
    return f(nj.NNJIT_F16 if dtype == "f16" else nj.NNJIT_F32, sum(news), len(news), hq, hk, dim, max(news), max(keys), int(causal), window, cus)


# (dtype, new tokens, keys, query heads, key heads, dim, tile rows, split over the keys, waves): every tile height, split and
# unsplit, for each class of head dims of either type
COVER = [
    ("f16", [40, 7, 1], [40, 30, 90], 1, 1, 64, 16, False, 4), ("f16", [100, 3], [400, 9], 1, 1, 64, 16, True, 4),
    ("f16", [40, 33, 40, 1], [40, 33, 38, 7], 32, 8, 64, 64, False, 4), ("f16", [100, 1, 77, 90, 100, 64], [1100, 600, 77, 900, 1050, 1], 1, 1, 64, 64, True, 4),
    ("f16", [100, 31, 77, 90, 100, 64], [100, 90, 77, 100, 50, 64], 64, 16, 64, 128, False, 4),
    ("f16", [100, 1, 77, 90, 100, 64], [2600, 600, 77, 900, 99, 1050], 16, 4, 64, 128, True, 4),
    ("f16", [40, 33, 40, 1], [40, 33, 38, 7], 32, 8, 96, 64, False, 4), ("f16", [500, 60], [800, 400], 1, 1, 96, 64, True, 4),
    ("f16", [100, 31, 77, 90, 100, 64], [100, 90, 77, 100, 50, 64], 64, 16, 96, 128, False, 4),
    ("f16", [100, 1, 77, 90, 100, 64], [2600, 600, 77, 900, 99, 1050], 16, 8, 96, 128, True, 4),
    ("f16", [40, 33, 40, 1, 40, 40], [40, 33, 38, 7, 40, 40], 16, 4, 128, 64, False, 4), ("f16", [500, 60], [800, 400], 1, 1, 128, 64, True, 4),
    ("f16", [320, 1], [2620, 54], 16, 4, 128, 64, True, 4), ("f16", [100, 31, 77, 90, 100, 64], [100, 90, 77, 100, 50, 64], 64, 16, 128, 128, False, 4),
    ("f16", [500, 480, 300], [3000, 900, 2000], 8, 2, 128, 128, True, 4),
    ("f16", [40, 33, 40, 1, 40, 40], [40, 33, 38, 7, 40, 40], 16, 4, 200, 128, False, 4), ("f16", [40, 1, 33, 12], [1040, 700, 33, 9], 8, 8, 200, 128, True, 4),
    ("f32", [40, 7, 1], [40, 30, 90], 1, 1, 64, 16, False, 4), ("f32", [40, 7, 1], [340, 30, 90], 1, 1, 64, 16, True, 4),
    ("f32", [200, 180, 33, 200], [200, 220, 33, 150], 16, 4, 64, 64, False, 4), ("f32", [500, 1, 400, 500, 500, 300], [800, 700, 500, 10, 777, 300], 1, 1, 64, 64, True, 4),
    ("f32", [100, 31, 77, 90, 100, 64], [100, 90, 77, 100, 50, 64], 32, 8, 64, 128, False, 4),
    ("f32", [200, 1, 177, 190, 200, 64], [1200, 600, 177, 900, 199, 1050], 2, 1, 64, 128, True, 4), ("f32", [320, 1], [4020, 54], 16, 16, 64, 128, True, 4),
    ("f32", [200, 180, 33, 200], [200, 220, 33, 150], 16, 16, 96, 64, False, 4), ("f32", [500, 60], [3000, 400], 1, 1, 96, 64, True, 4),
    ("f32", [100, 31, 77, 90], [100, 90, 77, 120], 64, 16, 96, 128, False, 4), ("f32", [320, 300], [2820, 400], 2, 1, 96, 128, True, 4),
    ("f32", [320, 300, 33, 320, 1, 320], [320, 310, 33, 200, 9, 320], 8, 2, 128, 64, False, 4),
    ("f32", [100, 31, 77, 90], [100, 90, 77, 120], 64, 16, 128, 128, False, 4), ("f32", [320, 300, 33, 320, 1, 320], [1320, 310, 33, 900, 9, 320], 2, 1, 128, 128, True, 4),
    ("f32", [100, 31, 77, 90], [100, 90, 77, 120], 64, 16, 200, 128, False, 4), ("f32", [500, 400, 33, 500], [3000, 410, 33, 2000], 1, 1, 200, 128, True, 4),
    # single tokens: four and eight waves
    ("f16", [1] * 3, [60, 1, 33], 2, 2, 64, 16, False, 4), ("f16", [1] * 3, [1000, 1, 333], 2, 1, 64, 16, True, 4), ("f16", [1] * 24, [500] * 12 + [1] * 12, 8, 8, 64, 16, False, 8),
    ("f16", [1] * 24, [500] * 12 + list(range(1, 13)), 8, 4, 96, 16, False, 8), ("f16", [1] * 32, [500] * 16 + list(range(1, 17)), 16, 8, 128, 16, False, 8),
    ("f16", [1] * 2, [500, 70], 8, 2, 128, 16, True, 4), ("f16", [1] * 2, [500, 70], 2, 2, 200, 16, True, 4), ("f16", [1] * 2, [60, 7], 2, 2, 200, 16, False, 4),
    ("f32", [1] * 3, [60, 1, 33], 2, 2, 64, 16, False, 4), ("f32", [1] * 3, [500, 1, 333], 2, 1, 64, 16, True, 4), ("f32", [1] * 24, [500] * 12 + [1] * 12, 4, 4, 64, 16, False, 8),
    ("f32", [1] * 24, [500] * 12 + list(range(1, 13)), 16, 8, 96, 16, False, 8), ("f32", [1] * 24, [500] * 12 + list(range(1, 13)), 8, 8, 128, 16, False, 8),
    ("f32", [1] * 2, [200, 70], 8, 2, 128, 16, True, 4), ("f32", [1] * 2, [200, 70], 2, 2, 200, 16, True, 4), ("f32", [1] * 2, [60, 7], 2, 2, 200, 16, False, 4),
]


def name(case) -> str:
    dtype, news, keys, hq, hk, dim, rows, split, waves = case
    return f"{dtype}-{dim}-{rows}rows-{'split' if split else 'whole'}-{waves}waves-{len(news)}x{max(news)}on{max(keys)}"


def strict(B: Batch, got, scale=None, causal=True, window=0):
    """Every element of got [tokens, heads, dim] inside a bound of its own dim; keys must be finite, queries and values need not.

    In units of the mean of |v| by weight, dim by dim: a logit is off by (dim + 4) U32 |scale| |q| |k| (sums of dim products; in
    three parts a product by U32), once in the numerator and once in the denominator; its weight by 6 U32 of the row's spread of
    logits (differences, scale, product, along two references), 4 U32 of an exp2 and as much for every move of a reference (one
    in 16 keys at most); sums of n terms by n U32 each.  fp16: weights by U16 and 2^-35 of the largest, the result by U16 and
    half of the smallest half."""
    scale = B.dim ** -0.5 if scale is None else scale
    got = got.double().cpu().numpy()
    q, group = B.q.double().numpy(), B.hq // B.hk
    for b, (n, m) in enumerate(zip(B.news, B.keys)):
        if n == 0:
            continue
        rows = slice(int(B.start[b]), int(B.start[b]) + n)
        if m == 0:
            assert (got[rows] == 0).all()
            continue
        pg, slot = np.array([B.table[b, j // B.page] for j in range(m)]), np.arange(m) % B.page
        k, v = B.k[pg, slot].double().numpy(), B.v[pg, slot].double().numpy()
        pos, j = np.arange(m - n, m)[:, None], np.arange(m)[None]
        seen = (j <= pos) | (not causal)
        if causal and window:
            seen &= j > pos - window
        some, count = seen.any(1), seen.sum(1)[:, None]
        for h in range(B.hq):
            kk, vv, qq = k[:, h // group], v[:, h // group], q[rows, h]
            good = np.isfinite(qq).all(1)
            qq = np.where(good[:, None], qq, 0.0)
            x = np.where(seen, scale * (qq @ kk.T), -np.inf)
            top = np.where(some, x.max(1), 0.0)[:, None]
            w = np.where(seen, np.exp(x - top), 0.0)
            total = np.where(some[:, None], w.sum(1, keepdims=True), 1.0)
            vf = np.where(np.isfinite(vv), vv, 0.0)
            ref, mean = (w @ vf) / total, (w @ np.abs(vf)) / total
            most = np.abs(vf).max(0)[None]
            size = abs(scale) * np.linalg.norm(qq, axis=1) * np.where(seen, np.linalg.norm(kk, axis=1)[None], 0.0).max(1)
            spread = np.where(seen, top - x, 0.0).max(1)
            e = ((B.dim + 4) * size + 6 * spread + 4)[:, None] * U32 + (count / 4) * U32
            bound = mean * (2 * e + 2 * count * U32)
            if B.dtype == "f16":
                bound = bound + mean * U16 + count * 2.0 ** -35 * most + np.abs(ref) * U16 + 2.0 ** -25
            if not np.isfinite(vv).all():
                s = seen.astype(np.float64)
                plus, minus, nan = s @ (vv == np.inf), s @ (vv == -np.inf), s @ np.isnan(vv)
                ref = np.where(plus > 0, np.inf, np.where(minus > 0, -np.inf, ref))
                ref = np.where((nan > 0) | ((plus > 0) & (minus > 0)), np.nan, ref)
            ref = np.where((good | ~some)[:, None], ref, np.nan)
            ref, bound = np.where(some[:, None], ref, 0.0), np.where(some[:, None], bound, 0.0)
            g = got[rows, h]
            assert np.array_equal(np.isnan(g), np.isnan(ref)), (b, h, "NaN in other places")
            inf = np.isinf(ref)
            assert np.array_equal(np.isinf(g), inf) and np.array_equal(g[inf], ref[inf]), (b, h, "infinities in other places")
            fine = np.isfinite(ref)
            off = np.abs(g[fine] - ref[fine]) - bound[fine]
            assert off.max(initial=0.0) <= 0, (b, h, off.max(), bound[fine][off.argmax()])
