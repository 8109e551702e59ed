"""Serving operators on the GPU at the ends of their arguments' ranges: against
the 64-bit forms, with bounds derived where they are used."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.serving_util import DT, U16, U32, Batch, attention, check_attention

pytestmark = pytest.mark.gpu


def _attend(B, **kw):
    out = torch.full(B.q.shape, 7.0, dtype=DT[B.dtype], device="cuda")
    nj.paged_attention(B.dq, B.cache, B.batch, out, **kw)
    torch.cuda.synchronize()
    return out


# enough rows for tall tiles as well, some before the first key
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys,heads", [([12], [9], 2), ([3, 1], [2, 3000], 2), ([320] * 5, [317, 40, 9, 320, 500], 16)])
@pytest.mark.parametrize("window", [(1 << 31) - 1, 1 << 40])
def test_window_past_every_key(dtype, news, keys, heads, window):
    """A window larger than any context is no window, for sequences with fewer keys than new tokens too."""
    B = Batch(news, keys, heads, heads, 64, 16, dtype, seed=31).device()
    got = _attend(B, window=window)
    check_attention(B, got)
    assert torch.equal(got, _attend(B))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys,columns,hq,hk", [([8, 1], [20, 33], 1, 4, 2), ([40, 5], [50, 70], 2, 2, 2), ([1], [3000], 100, 2, 1),
                                                     ([320, 40], [500, 330], 20, 16, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 6), (False, 0)])
def test_lengths_past_the_page_table(dtype, news, keys, columns, hq, hk, causal, window):
    """Keys past the table's columns do not exist; positions stay those of kv_len, as an append takes them.

    Bound: see tests.serving_util.attention, here with all sizes taken as the largest of the case."""
    dim, page = 64, 16
    B = Batch(news, keys, hq, hk, dim, page, dtype, seed=32).device()
    table = torch.from_numpy(B.table[:, :columns].copy()).cuda()
    B.batch = nj.PagedBatch(B.batch.q_start, B.batch.kv_len, table, tokens=B.tokens, max_q=max(news), max_kv=max(keys))
    got = _attend(B, causal=causal, window=window).double().cpu().numpy()
    q, group = B.q.double().numpy(), hq // hk
    for b, (n, m) in enumerate(zip(news, keys)):
        slots = B.key_slots(b)[:columns * page]
        k, v = (np.stack([t[s].double().numpy() for s in slots]) for t in (B.k, B.v))
        pos, j = np.arange(m - n, m)[:, None], np.arange(len(slots))[None]
        seen = (j <= pos) | (not causal)
        if window:
            seen &= j > pos - window
        for h in range(hq):
            qq = q[B.start[b]:B.start[b] + n, h]
            x = np.where(seen, dim ** -0.5 * (qq @ k[:, h // group].T), -np.inf)
            top = x.max(1, keepdims=True)
            w = np.where(seen, np.exp(x - np.where(seen.any(1, keepdims=True), top, 0.0)), 0.0)
            total = w.sum(1, keepdims=True)
            ref = np.where(total > 0, w @ v[:, h // group] / np.where(total > 0, total, 1.0), 0.0)
            size = dim ** -0.5 * np.linalg.norm(qq, axis=1).max() * np.linalg.norm(k[:, h // group], axis=1).max()
            e = (dim + 4) * U32 * size + 4 * U32 * size + 4 * U32
            bound = np.abs(v).max() * (2 * e + 2 * len(slots) * U32 + (2 * U16 if dtype == "f16" else 0.0))
            off = np.abs(got[B.start[b]:B.start[b] + n, h] - ref)
            assert off.max() <= bound, (b, h, off.max(), bound)
            assert (off[~seen.any(1)] == 0).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("window", [0, 5])
def test_lengths_near_2_to_the_31(dtype, rows, window):
    """A kv_len that passes every limit is no key index past 32 bits: keys from 2^30 on do not exist.  (Pages of 2^30
    tokens that all lie in one place, which only the C entry point takes; a non-causal or unwindowed call would walk all keys.)"""
    page, dt = 1 << 30, DT[dtype]
    k, v = torch.randn(2, 1, 1, 64, device="cuda").to(dt)
    q = torch.randn(rows, 1, 64, device="cuda").to(dt)
    out = torch.full_like(q, 7.0)
    i32 = dict(dtype=torch.int32, device="cuda")
    table, start = torch.zeros(1, 3, **i32), torch.tensor([0, rows], **i32)
    cache = nj.PagedKvDesc(k.data_ptr(), v.data_ptr(), 0, 0, 64, 0, 0, 64, 1, page, 1, 64, nj.NNJIT_F16 if dtype == "f16" else nj.NNJIT_F32)
    for length in ((1 << 30) + 2, (1 << 31) - 3, (1 << 31) - 1):
        lengths = torch.tensor([length], **i32)
        # without a window only the rows' first 64 keys are asked for
        batch = nj.PagedBatchDesc(1, rows, start.data_ptr(), lengths.data_ptr(), table.data_ptr(), 3, 3, rows, 1 << 30 if window else 64)
        nj.check(nj.nnjit_paged_attention(cache, batch, 1, q, 64, 64, out, 64, 64, 0.125, 1, window))
        torch.cuda.synchronize()
        first = torch.arange(rows, device="cuda") + length - rows - window + 1     # first key that a row sees
        sees = (first < 1 << 30) if window else first > 0
        assert torch.equal(out[~sees], torch.zeros_like(out[~sees]))
        # all keys are alike: the value itself, up to the rounding of a mean of equal values
        assert torch.allclose(out[sees].float(), v.float().expand(rows, 1, 64)[sees], rtol=2e-3 if dtype == "f16" else 1e-5, atol=0)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys,max_q,hq,hk,tile", [([3, 40], [3000, 2000], 3, 4, 2, 16), ([1, 17, 1], [900, 5000, 3000], 1, 3, 3, 16),
                                                        ([320, 700], [3000, 1500], 320, 16, 4, 128)])
def test_rows_past_max_q(dtype, news, keys, max_q, hq, hk, tile):
    """Rows that a too small max_q leaves out keep what they held, also where keys are split: scratch of an earlier call is
    not taken for their sums.  (Rows that share the last tile may be computed, and are right then.)"""
    other = Batch([1], [20000], 32, 32, 64, 16, dtype, seed=33).device()
    B = Batch(news, keys, hq, hk, 64, 16, dtype, seed=34).device(max_q=max_q)
    _attend(other)                                           # fills the stream's scratch
    got = _attend(B)
    left = (got == 7.0).flatten(1).all(1).cpu()
    for b, n in enumerate(news):
        r = left[B.start[b]:B.start[b] + n]
        assert not bool(r[:max_q].any())
        assert bool(r[max_q + -(-tile * hk // hq):].all())
    # the rows that were computed, as with a large enough max_q (another plan: other roundings)
    B.batch.desc.max_q = max(news)
    full = _attend(B)
    check_attention(B, full)
    diff = (got[~left].double() - full[~left].double()).norm() / full[~left].double().norm()
    assert float(diff) <= (4 * U16 if dtype == "f16" else 2e-5), float(diff)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys,hq,hk,dim", [([1], [700], 2, 2, 64), ([1] * 32, [700] * 32, 8, 8, 64), ([3], [2000], 4, 2, 128),
                                                 ([320], [700], 16, 16, 64), ([320], [700], 4, 4, 128), ([320], [2500], 16, 4, 128),
                                                 ([320], [700], 16, 16, 200)])
def test_references_of_any_size(dtype, news, keys, hq, hk, dim):
    """Large logits that grow along the keys, so that every row's reference moves again and again, with values that shrink as the
    weights grow: all steps count alike.  The logits are exact (multiples of 1/16), so only the weights' own roundings are left.

    Bound on an element, in units of the mean of |v| by weight: an exponent is a difference of logits, times a rounded scale,
    rounded: 3 U32 of the row's spread in all, along every chain of references; an exp2 is off by 2 ulp, once a key and once
    a move (of at most one in 16 keys); the sums of n terms by n U32 each.  fp16: weights rounded to 11 bits, and the result."""
    step, most = (6.0, 11) if dtype == "f32" else (6.0, 1)
    B = Batch(news, keys, hq, hk, dim, 16, dtype, seed=35)
    rng = np.random.default_rng(36)
    B.q.zero_()
    B.q[..., 0], B.q[..., 1] = 256.0, 1.0
    rows = []
    for b, m in enumerate(keys):
        level = np.minimum(np.arange(m) * 16 // max(m, 1), most)
        small = np.round((step * level + rng.normal(0, 0.5, m)) * 16) / 16
        value = rng.uniform(0.5, 1.5, (m, hk, dim)) * (np.where(level % 2, -1.0, 1.0) * np.exp(step * (most - level)))[:, None, None]
        for j, s in enumerate(B.key_slots(b)):
            B.k[s][:, 0], B.k[s][:, 1] = 512.0, float(small[j])
            B.v[s] = torch.from_numpy(value[j]).to(DT[dtype])
        rows.append((small, np.stack([B.v[s].double().numpy() for s in B.key_slots(b)])))
    got = _attend(B.device(), scale=1.0).double().cpu().numpy()
    for b, (n, m) in enumerate(zip(news, keys)):
        small, v = rows[b]
        for i in range(n):
            x = small[:m - n + i + 1]
            w = np.exp(x - x.max())
            vv = v[:len(x)]
            ref, mean = np.tensordot(w, vv, 1) / w.sum(), np.tensordot(w, np.abs(vv), 1) / w.sum()
            spread = x.max() - x.min()
            bound = mean * (2 * (3 * spread + 4 + len(x) / 4) + 2 * len(x)) * U32
            if dtype == "f16":
                bound = bound + mean * U16 + np.abs(ref) * U16 + 2.0 ** -25
            off = np.abs(got[B.start[b] + i] - np.repeat(ref, hq // hk, 0))
            worst = (off / np.repeat(bound, hq // hk, 0)).max()
            assert worst <= 1, (b, i, worst)


@pytest.mark.parametrize("news,keys,hq,hk,dim,page", [([1] * 2, [700, 60], 2, 2, 64, 16), ([1] * 16, [900] * 16, 8, 8, 64, 16), ([2], [5000], 4, 2, 128, 5),
                                                      ([1], [700], 2, 1, 256, 16), ([320], [700], 16, 16, 64, 16), ([320], [700], 4, 4, 128, 5),
                                                      ([320], [2500], 16, 4, 128, 16), ([600], [600], 32, 32, 64, 16), ([200], [700], 16, 16, 200, 16)])
@pytest.mark.parametrize("bits", [12.3, 20.6, 23.5, 25.0])
def test_small_weights_fp16(news, keys, hq, hk, dim, page, bits):
    """A first key that takes nearly all weight but has values of zero: the result is the sum of the others, whose weights
    (about 2^-bits of the largest) must have kept their bits."""
    B = Batch(news, keys, hq, hk, dim, page, "f16", seed=37)
    rng = np.random.default_rng(38)
    B.q.zero_()
    B.q[..., 0] = 1.0
    for b, m in enumerate(keys):
        for j, s in enumerate(B.key_slots(b)):
            B.k[s][:, 0] = bits * float(np.log(2.0)) + 1.0 if j == 0 else float(rng.normal(1.0, 0.3))
            B.v[s] = 0.0 if j == 0 else B.v[s] * 512.0
    check_attention(B, _attend(B.device(), scale=1.0), scale=1.0)


@pytest.mark.parametrize("news,keys,heads", [([1] * 3, [700, 60, 3000], 2), ([320], [700], 16)])
@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 20, 2.0 ** 25])
def test_large_logits_fp16(news, keys, heads, size):
    """Logits whose last bit in fp32 is worth up to 2: nearly one-hot rows, finite, and right where the largest logit is clear."""
    B = Batch(news, keys, heads, heads, 64, 16, "f16", seed=39)
    B.q *= size ** 0.5 / 8
    B.k *= size ** 0.5 / 8
    got = _attend(B.device(), scale=1.0).double().cpu().numpy()
    assert np.isfinite(got).all()
    for b, (n, m) in enumerate(zip(news, keys)):
        k, v = (np.stack([t[s].double().numpy() for s in B.key_slots(b)]) for t in (B.k, B.v))
        for i in range(n):
            x = np.einsum("hd,jhd->hj", B.q[int(B.start[b]) + i].double().numpy(), k[:m - n + i + 1])
            order = np.sort(x, 1)
            clear = order[:, -1] - order[:, -2] > 30 + 68 * U32 * size * 8 if x.shape[1] > 1 else np.ones(heads, dtype=bool)
            want = v[x.argmax(1), np.arange(heads)]
            assert (np.abs(got[B.start[b] + i] - want)[clear] <= 2 * U16 * np.abs(want)[clear] + 1e-6).all()


def test_capture_that_needs_scratch():
    """A captured call whose stream lacks the scratch is refused with what to do; lengths of the run that readies it are free."""
    B = Batch([1], [5000], 4, 1, 128, 16, "f16", seed=40).device()
    want = _attend(B)
    # a stream of its own: torch hands its streams out again and again, with the scratch of earlier calls
    handle = ctypes.c_void_p()
    assert nj.load().hipStreamCreateWithFlags(ctypes.byref(handle), 1) == 0
    s, out = torch.cuda.ExternalStream(handle.value), torch.empty_like(B.dq)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(nj.NnjitError, match="^NNJIT_EHIP: scratch of .* being captured; run a call of the same sizes once"):
            nj.paged_attention(B.dq, B.cache, B.batch, out)
    B.batch.kv_len.fill_(3)
    nj.paged_attention(B.dq, B.cache, B.batch, out, stream=s)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph(), stream=s):
        nj.paged_attention(B.dq, B.cache, B.batch, out)
    B.batch.kv_len.fill_(5000)
    torch.cuda.synchronize()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_append_behind_the_table():
    """Positions behind the rotary table are clamped to it, as nnjit_rotary clamps them; slots are not."""
    cache = nj.PagedCache(torch.zeros(2, 16, 1, 8, device="cuda"), torch.zeros(2, 16, 1, 8, device="cuda"))
    i32 = dict(dtype=torch.int32, device="cuda")
    batch = nj.PagedBatch(torch.tensor([0, 3], **i32), torch.tensor([12], **i32), torch.tensor([[1, 0]], **i32), tokens=3)
    table = nj.rotary_table(11, 8)
    x = torch.randn(3, 1, 8, device="cuda")
    q = nj.kv_append(cache, batch, x, x, table, x)
    want = nj.rotary(x, torch.tensor([9, 10, 10], **i32), table)
    assert torch.equal(q, want) and torch.equal(cache.k[1, 9:12], want) and torch.equal(cache.v[1, 9:12], x)


@pytest.mark.parametrize("count,keys,heads,dim", [(4, 500, 12, 64), (2, 300, 8, 128), (1, 700, 8, 256), (24, 500, 8, 64), (1, 3000, 4, 96)])
def test_rounding_of_single_rows_fp32(count, keys, heads, dim):
    """The error that roundings of independent sign leave, in U32 relative to the result.

    A logit is a sum of dim products of keys N(0, 1) and queries N(0, 4): a chain of m sums with steps of size 2 rounds m / sqrt(6)
    times that off (each partial sum by U32 / sqrt(3) of its size 2 sqrt(j)), four chains of dim / 4 are off by half of what one
    chain over all is.  That error of a weight is the result's (values N(0, 1): sums of w_j d_j v_j against sums of w_j v_j).
    Weights, sums over the keys and the division leave about 3 more; a factor of 1.4 (one chain has 2) for all that is estimated."""
    B = Batch([1] * count, [keys - 7 * i for i in range(count)], heads, heads, dim, 16, "f32", seed=41, q_scale=2.0).device()
    ref, _ = attention(B)
    off = _attend(B).double().cpu().numpy() - ref
    logit = dim ** -0.5 * 2 * 2.0 * (dim / 4) / 6 ** 0.5
    rel = np.linalg.norm(off) / np.linalg.norm(ref) / U32
    assert rel <= (1.4 ** 2 * logit ** 2 + 9) ** 0.5, (rel, logit)
