"""The serving operators on the GPU against plain forms in 64 bits: rotary
positions, appends to a paged cache, attention over it."""
import math

import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.serving_util import DT, U16, U32, Batch, attention, check_attention, rounded, turn

pytestmark = pytest.mark.gpu


def _attend(B, **kw):
    out = torch.full(B.q.shape, 7.0, dtype=DT[B.dtype], device="cuda")
    nj.paged_attention(B.dq, B.cache, B.batch, out, **kw)
    torch.cuda.synchronize()
    return out


def _case(news, keys, hq, hk, dim, page, dtype, **kw):
    how = {k: kw.pop(k) for k in ("scale", "causal", "window") if k in kw}
    limits = {k: kw.pop(k) for k in ("max_q", "max_kv") if k in kw}
    B = Batch(news, keys, hq, hk, dim, page, dtype, **kw).device(**limits)
    got = _attend(B, **how)
    check_attention(B, got, **how)
    assert bool((got[sum(news):] == 7.0).all()), "rows of no sequence are left alone"
    return B, got


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(4, 4, 64), (8, 2, 128), (6, 2, 96), (16, 1, 64), (5, 1, 256)])
@pytest.mark.parametrize("page", [16, 5])
def test_decode(dtype, hq, hk, dim, page):
    """Single tokens: lengths of one, around tile and page ends, long ones."""
    _case([1] * 7, [1, 2, 31, 32, 33, 130, 517], hq, hk, dim, page, dtype, seed=1)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(3, 3, 64), (4, 2, 128), (8, 1, 96), (2, 1, 256)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 37), (False, 0)])
def test_chunks(dtype, hq, hk, dim, causal, window):
    """New tokens at the end of cached ones, all lengths in one call."""
    _case([70, 1, 33, 5, 128], [70, 90, 200, 5, 150], hq, hk, dim, 16, dtype, seed=2, causal=causal, window=window)


def _many(count, longest, past):
    """Ragged sequences: 1, `longest` and what lies between, with 0 .. past cached keys."""
    news = [longest, 1] + [1 + (37 * i * i + 11 * i) % longest for i in range(2, count)]
    return news, [n + (53 * i) % (past + 1) for i, n in enumerate(news)]


# enough rows for the tall tiles, in 64 and in 128 rows, unsplit and (few heads, long caches) split over the keys
TALL = [(17, 200, 90, 16, 16, 64, {}), (17, 250, 50, 16, 16, 128, {}), (17, 250, 50, 32, 16, 96, dict(window=40)),
        (20, 200, 60, 16, 8, 128, dict(causal=False)), (17, 250, 60, 16, 16, 40, {}), (32, 160, 40, 16, 16, 256, {}),
        (4, 256, 0, 16, 16, 64, dict(causal=False)), (1, 512, 0, 32, 32, 128, {}), (2, 320, 3700, 16, 16, 64, {}),
        (2, 320, 2300, 16, 4, 128, {}), (2, 320, 2300, 16, 4, 128, dict(window=700))]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("count,longest,past,hq,hk,dim,how", TALL)
@pytest.mark.parametrize("page", [16, 5])
def test_many_rows(dtype, count, longest, past, hq, hk, dim, how, page):
    news, keys = _many(count, longest, past)
    _case(news, keys, hq, hk, dim, page, dtype, seed=21, **how)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("dim,shift,row_gap,extra", [(64, 1, 3, 1), (96, 0, 1, 0), (77, 0, 0, 0), (128, 2, 0, 0), (200, 1, 0, 0)])
def test_many_rows_of_any_alignment(dtype, dim, shift, row_gap, extra):
    news, keys = _many(16, 190, 70)
    _case(news, keys, 16, 16, dim, 16, dtype, seed=22, shift=shift, row_gap=row_gap, extra_dim=extra, order="hnd")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("count,longest,past,hq,hk", [(17, 200, 90, 16, 16), (2, 320, 3000, 16, 4)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_many_rows_masked_places(dtype, count, longest, past, hq, hk, bad):
    """As test_masked_places, where tiles of rows share keys; keys and queries that are not finite spoil their own rows."""
    news, keys = _many(count, longest, past)
    B = Batch(news, keys, hq, hk, 64, 16, dtype, seed=23)
    late = B.key_slots(0)
    B.v[late[keys[0] - 40]][1, 5] = bad
    B.v[late[keys[0] - 40]][2, 9] = -bad
    B.v[late[keys[0] - 1]][2, 9] = bad
    if bad != bad:      # (a logit of +inf gives NaN, one of -inf no weight: both by the sign of the query; NaN always NaN)
        B.k[late[keys[0] - 33]][3, 7] = bad
        B.q[int(B.start[1]), 0, 0] = bad
    B.device()
    check_attention(B, _attend(B))


@pytest.mark.parametrize("count,longest,past,hq,hk,dim", [(17, 200, 90, 16, 16, 64), (17, 120, 90, 16, 16, 128), (2, 320, 3000, 16, 4, 64)])
def test_values_of_any_size_f32(count, longest, past, hq, hk, dim):
    """fp32 values that round to an infinity in bf16, and tiny and zero ones."""
    news, keys = _many(count, longest, past)
    B = Batch(news, keys, hq, hk, dim, 16, "f32", seed=24)
    s = B.key_slots(0)
    B.v[s[3]][0, 1] = 3.395e38
    B.v[s[keys[0] - 2]][1, 2] = -3.395e38
    B.v[s[5]][2] = 0.0
    B.v[s[6]][2] = 1e-30
    B.device()
    check_attention(B, _attend(B))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("page,order", [(1, "nhd"), (3, "hnd"), (32, "hnd"), (48, "nhd"), (64, "nhd"), (1000, "hnd")])
def test_pages(dtype, page, order):
    """Pages of any size in both pool layouts, ends inside tiles."""
    _case([40, 3], [140, 77], 4, 2, 64, page, dtype, seed=3, order=order)
    _case([1, 1, 1], [140, 77, 300], 4, 2, 64, page, dtype, seed=4, order=order)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("dim,shift,row_gap,extra", [(1, 0, 0, 0), (17, 0, 0, 0), (33, 1, 5, 3), (64, 1, 0, 0), (80, 0, 8, 8),
                                                     (128, 0, 3, 0), (129, 0, 0, 0), (200, 0, 0, 0), (255, 2, 1, 0)])
def test_any_alignment(dtype, dim, shift, row_gap, extra):
    """Odd head dimensions, strides with gaps, tensors that begin anywhere."""
    _case([35, 1], [60, 41], 4, 2, dim, 16, dtype, seed=5, shift=shift, row_gap=row_gap, extra_dim=extra)
    _case([1, 1], [60, 41], 4, 2, dim, 16, dtype, seed=6, shift=shift, row_gap=row_gap, extra_dim=extra)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rows_without_keys(dtype):
    """Fewer keys than new tokens (the first ones see nothing), no key at all, no new token, rows behind the batch."""
    B, got = _case([5, 0, 40, 3, 1], [2, 9, 17, 0, 0], 4, 2, 64, 16, dtype, seed=7, pad=3)
    assert bool((got[:3] == 0).all()) and bool((got[45:49] == 0).all())
    B, got = _case([1, 1], [0, 0], 2, 2, 64, 16, dtype, seed=8)
    assert bool((got == 0).all())
    B, got = _case([0, 0], [3, 4], 2, 2, 64, 16, dtype, seed=8, pad=2, max_q=1)
    # split over the keys
    B, got = _case([3, 1], [2, 3000], 2, 1, 64, 16, dtype, seed=9)
    assert bool((got[:1] == 0).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys", [([50], [90]), ([4], [90]), ([2], [1500])])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_masked_places(dtype, news, keys, bad):
    """A value that is not finite reaches the rows that see it, and no other."""
    B = Batch(news, keys, 4, 2, 64, 16, dtype, seed=10)
    late = B.key_slots(0)[keys[0] - 2]           # the last two rows see it
    B.v[late][1, 5] = bad
    B.v[late][1, 40] = -bad
    B.v[B.key_slots(0)[keys[0] - 1]][1, 40] = bad
    B.device()
    check_attention(B, _attend(B))
    # a key of such values: their logits are what the formula makes of them
    B = Batch(news, keys, 4, 2, 64, 16, dtype, seed=11)
    B.k[B.key_slots(0)[keys[0] - 1]][0, 3] = bad
    B.device()
    check_attention(B, _attend(B))
    # with a window that has passed a bad value by
    B = Batch(news, keys, 4, 2, 64, 16, dtype, seed=12)
    B.v[B.key_slots(0)[keys[0] - news[0] - 3]][:, :] = bad
    B.k[B.key_slots(0)[keys[0] - news[0] - 3]][:, :] = bad
    B.device()
    check_attention(B, _attend(B, window=4), window=4)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("keys", [20, 2000])
def test_logits_of_minus_infinity(dtype, keys):
    """Seen keys whose logits are all -inf give 0 / 0; one finite logit among them takes all the weight."""
    B = Batch([1, 1], [keys, keys], 2, 1, 64, 16, dtype, seed=13)
    B.q.abs_()
    for b in range(2):
        for j, s in enumerate(B.key_slots(b)):
            if b == 0 or j != keys // 2:
                B.k[s] = -float("inf")
    B.device()
    got = _attend(B)
    check_attention(B, got)
    assert bool(torch.isnan(got[0]).all()) and bool(torch.isfinite(got[1]).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys", [([1, 1], [100, 700]), ([60, 9], [100, 700])])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 4.0, 60.0])
def test_scales(dtype, news, keys, scale):
    """Negative and zero scales, and logits in the thousands."""
    B = Batch(news, keys, 4, 4, 64, 16, dtype, seed=14).device()
    got = _attend(B, scale=scale)
    ref, _ = attention(B, scale)
    assert bool(torch.isfinite(got).all())
    if scale < 10:
        check_attention(B, got, scale=scale)
    else:
        # a logit of size 60 |q| |k| is known to 3e-3 only: nearly one-hot rows, compared where the largest weight is clear
        rel = np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        assert rel < 2e-2, rel


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys,hq,hk", [([1], [6000], 2, 2), ([1, 1], [4097, 33], 8, 1), ([7], [3001], 4, 1), ([64], [2500], 2, 1)])
def test_keys_split_over_workgroups(dtype, news, keys, hq, hk):
    """Long contexts of few rows; limits far above the lengths change nothing beyond rounding, and runs repeat bit for bit."""
    B, got = _case(news, keys, hq, hk, 128, 32, dtype, seed=15)
    again = _attend(B)
    assert torch.equal(got, again)
    _case(news, keys, hq, hk, 128, 32, dtype, seed=15, max_kv=50000, max_q=max(news) + 100)
    if len(news) == 1:
        _case(news, keys, hq, hk, 128, 32, dtype, seed=16, window=1000)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("count,hq,hk,dim", [(2, 3, 3, 64), (5, 2, 1, 128), (8, 8, 8, 64), (9, 10, 5, 96), (13, 4, 4, 128)])
def test_splits_of_many_sequences(dtype, count, hq, hk, dim):
    """Every (split, sequence, head) is taken once, whatever their numbers: lengths from one to thousands."""
    keys = [3000 if i % 3 == 0 else 1 + (971 * i) % 2500 for i in range(count)]
    B, got = _case([1] * count, keys, hq, hk, dim, 16, dtype, seed=19)
    assert torch.equal(got, _attend(B))
    _case([2] * count, [k + 1 for k in keys], hq, hk, dim, 33, dtype, seed=20)


def test_offsets_past_32_bits():
    """Pages beyond the 2^32nd byte and the 2^31st element of the pool."""
    page, hk, dim = 64, 8, 128
    pages = (1 << 31) // (page * hk * dim) + 40
    k = torch.empty((pages, page, hk, dim), dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    B = Batch([1, 20], [150, 90], 16, hk, dim, page, "f16", seed=17).device()
    used = [int(x) for b in range(2) for x in B.table[b, :-(-B.keys[b] // page)]]
    moved = {x: pages - 1 - i for i, x in enumerate(used)}
    for x, y in moved.items():
        k[y], v[y] = B.dk[x], B.dv[x]
    table = torch.tensor([[moved.get(int(x), int(x)) for x in row] for row in B.table], dtype=torch.int32, device="cuda")
    batch = nj.PagedBatch(B.batch.q_start, B.batch.kv_len, table, tokens=B.tokens, max_q=20, max_kv=150)
    cache = nj.PagedCache(k, v)
    got = nj.paged_attention(B.dq, cache, batch)
    check_attention(B, got)
    new = torch.randn(21, hk, dim, device="cuda")
    nj.kv_append(cache, batch, new, 2 * new)
    last = moved[int(B.table[0, 149 // page])]
    assert torch.equal(k[last, 149 % page], new[0].half()) and torch.equal(v[last, 149 % page], (2 * new[0]).half())


def test_streams_and_graph():
    """Calls on a stream of their own; a captured call follows the lengths that the device holds at each replay."""
    B = Batch([1, 1, 1], [900, 40, 333], 8, 2, 64, 16, "f16", seed=18).device(max_kv=1000)
    want = _attend(B)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(B.dq)
    nj.paged_attention(B.dq, B.cache, B.batch, out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        nj.paged_attention(B.dq, B.cache, B.batch, out, stream=s)
    for keys in ([900, 40, 333], [17, 1, 200], [0, 40, 320], [899, 2, 331]):
        B.keys = keys
        B.batch.kv_len.copy_(torch.tensor(keys, dtype=torch.int32))
        out.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _attend(B)), keys
        check_attention(B, out)


def test_two_streams_share_no_scratch():
    """Split calls on two streams at once."""
    cases = [Batch([1], [5000], 4, 1, 128, 16, "f16", seed=19 + i).device() for i in range(2)]
    want = [_attend(B) for B in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.empty_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for B, s, o in zip(cases, streams, outs):
            nj.paged_attention(B.dq, B.cache, B.batch, o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


# --------------------------------------------------------------------- rotary

def _table(positions, rot, seed=0):
    rng = np.random.default_rng(seed)
    a = rng.uniform(-3, 3, (positions, rot // 2))
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("f32", "f16"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("tokens,heads,dim,rot", [(1, 32, 128, 128), (7, 5, 64, 32), (33, 3, 96, 96), (2, 1, 2, 2), (19, 2, 33, 10),
                                                  (5, 40, 256, 64), (1500, 2, 80, 80)])
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary(layout, src, dst, tokens, heads, dim, rot, transpose):
    rng = np.random.default_rng([tokens, dim])
    table = _table(50, rot)
    pos = rng.integers(0, 50, tokens).astype(np.int32)
    wide = torch.from_numpy(rng.standard_normal((tokens, heads + 2, dim))).to(DT[src]).cuda()
    x = wide[:, 1:heads + 1]                                     # columns of a wider result
    out = torch.full((tokens, heads, dim), 9.0, dtype=DT[dst], device="cuda")
    nj.rotary(x, torch.from_numpy(pos).cuda(), nj.RotaryTable(table, layout), out, transpose=transpose)
    t = table.double().cpu().numpy()[pos]
    y, bound = turn(x.double().cpu().numpy(), t[:, :rot // 2], t[:, rot // 2:], layout, -1.0 if transpose else 1.0)
    bound[..., rot:] = 0
    assert (np.abs(out.double().cpu().numpy() - y) <= rounded(y, bound, dst)).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", [(64, 64), (48, 20)])
def test_rotary_gradient(layout, dim, rot):
    """The transposed turn is the gradient: against differences of the turn (exact up to rounding, it is linear), and in place."""
    table = nj.RotaryTable(_table(20, rot, seed=1), layout)
    pos = torch.tensor([3, 19, 0], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    x, up = torch.randn(3, 2, dim, device="cuda", generator=g), torch.randn(3, 2, dim, device="cuda", generator=g)
    grad = nj.rotary(up, pos, table, transpose=True)
    for i in range(dim):
        step = torch.zeros_like(x)
        step[..., i] = 0.5
        diff = (nj.rotary(x + step, pos, table).double() - nj.rotary(x - step, pos, table).double())
        want = (diff * up.double()).sum(-1)
        # the two sides round 4 times each, of values up to |x| + 1
        assert torch.allclose(grad[..., i].double(), want, rtol=0, atol=8 * U32 * 6 * float(up.abs().sum(-1).max()))
    same = x.clone()
    nj.rotary(same, pos, table, same)
    assert torch.equal(same, nj.rotary(x, pos, table))


def test_rotary_positions_are_clamped():
    table = nj.RotaryTable(_table(10, 8), "half")
    x = torch.randn(3, 1, 8, device="cuda")
    got = nj.rotary(x, torch.tensor([-5, 10, 1 << 30], dtype=torch.int32, device="cuda"), table)
    assert torch.equal(got, nj.rotary(x, torch.tensor([0, 9, 9], dtype=torch.int32, device="cuda"), table))
    assert nj.rotary(x[:0], torch.empty(0, dtype=torch.int32, device="cuda"), table).shape == (0, 1, 8)


def _frequencies(rot, base, s):
    i = np.arange(rot // 2, dtype=np.float64)
    if s is not None and s.kind == nj.NNJIT_ROTARY_BASE and rot > 2:   # a single pair has frequency 1 for any base
        base = base * s.factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if s is None or s.kind in (nj.NNJIT_ROTARY_PLAIN, nj.NNJIT_ROTARY_BASE):
        return f
    if s.kind == nj.NNJIT_ROTARY_LINEAR:
        return f / s.factor
    if s.kind == nj.NNJIT_ROTARY_TURNS:
        keep = np.clip((s.original * f / (2 * np.pi) - s.slow) / (s.fast - s.slow), 0, 1)
    else:
        index = [rot * np.log(s.original / (n * 2 * np.pi)) / (2 * np.log(base)) for n in (s.fast, s.slow)]
        lo, hi = max(np.floor(index[0]), 0), min(np.ceil(index[1]), rot - 1)
        keep = 1 - np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
    return f * keep + f / s.factor * (1 - keep)


@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (2, 10000.0), (34, 1234.5)])
@pytest.mark.parametrize("kind", [None, nj.NNJIT_ROTARY_LINEAR, nj.NNJIT_ROTARY_BASE, nj.NNJIT_ROTARY_TURNS, nj.NNJIT_ROTARY_INDEX])
def test_rotary_table(rot, base, kind):
    """Angles to 10^5 positions: the table is cos and sin of 64-bit angles, rounded once (angles of 10^5 known to 2^-36)."""
    s = None if kind is None else nj.RotaryScaling(kind, 4.0, 2048.0, 32.0, 1.0, 1.25)
    positions = 100003
    t = nj.rotary_table(positions, rot, base, scaling=s)
    p = np.concatenate([np.arange(300), np.arange(positions - 300, positions)])
    a = p[:, None] * _frequencies(rot, base, s)[None]
    want = np.concatenate([np.cos(a), np.sin(a)], 1) * (1.0 if s is None else 1.25)
    got = t.table.double().cpu().numpy()[p]
    assert np.abs(got - want).max() <= 1.25 * U32 + 2.0 ** -34


# --------------------------------------------------------------------- append

@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 32), (None, 0), ("half", 10)])
@pytest.mark.parametrize("src,dst", [("f32", "f16"), ("f32", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("page,order,shift", [(16, "nhd", 0), (5, "hnd", 0), (16, "nhd", 1)])
def test_append(layout, rot, src, dst, page, order, shift):
    """Every slot of the pool: the new tokens' where they belong, all others untouched; queries turned."""
    news, keys, hq, hk, dim = [3, 0, 17, 1, 4], [3, 8, 40, 65, 2], 6, 2, 64
    B = Batch(news, keys, hq, hk, dim, page, dst, seed=20, order=order, pad=2, shift=shift).device()
    g = torch.Generator(device="cuda").manual_seed(6)
    qkv = torch.randn(B.tokens, (hq + 2 * hk) * dim + shift, device="cuda", generator=g).to(DT[src])[:, shift:]
    rows = torch.as_strided(qkv, (B.tokens, hq + 2 * hk, dim), (qkv.stride(0), dim, 1), qkv.storage_offset())
    q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
    table = nj.RotaryTable(_table(80, rot, seed=2), layout) if rot else None
    before = [B.dk.cpu().clone(), B.dv.cpu().clone()]
    out = torch.full((B.tokens, hq, dim), 5.0, dtype=DT[dst], device="cuda")
    nj.kv_append(B.cache, B.batch, k, v, table, q, out)
    got = [B.dk.cpu(), B.dv.cpu()]
    t = table.table.double().cpu().numpy() if rot else np.ones((80, 2))
    done = np.zeros(before[0].shape[:2], dtype=bool)
    for b, (n, m) in enumerate(zip(news, keys)):
        for i in range(n):
            pos, row = m - n + i, int(B.start[b]) + i

            def turned(x):
                x = x[row].double().cpu().numpy()[None]
                if not rot:
                    return x[0], rounded(x[0], 0 * x[0], dst)
                at = t[max(pos, 0)][None]
                y, bound = turn(x, at[:, :rot // 2], at[:, rot // 2:], layout)
                bound[..., rot:] = 0
                return y[0], rounded(y[0], bound[0], dst)

            y, bound = turned(q)
            assert (np.abs(out[row].double().cpu().numpy() - y) <= bound).all()
            if pos < 0:
                continue
            pg, slot = int(B.table[b, pos // page]), pos % page
            done[pg, slot] = True
            y, bound = turned(k)
            assert (np.abs(got[0][pg, slot].double().numpy() - y) <= bound).all()
            assert torch.equal(got[1][pg, slot], v[row].to(DT[dst]).cpu())
    for x, y in zip(got, before):
        left = torch.from_numpy(~done)
        assert torch.equal(x[left].nan_to_num(3.0, 4.0), y[left].nan_to_num(3.0, 4.0))
    assert bool((out[sum(news):] == 5.0).all())


def test_append_many_sequences_and_bad_pages():
    """More sequences than a wave has lanes; page ids outside the pool and positions past the table are not written."""
    n, page = 200, 4
    cache = nj.PagedCache(torch.zeros(n, page, 1, 8, device="cuda"), torch.zeros(n, page, 1, 8, device="cuda"))
    keys = torch.arange(n, dtype=torch.int32) % page + 1
    table = torch.arange(n, dtype=torch.int32).flip(0)[:, None].contiguous()
    table[7], table[8], keys[9] = -1, n, page + 1
    start = torch.arange(n + 1, dtype=torch.int32).cuda()
    x = torch.randn(n, 1, 8, device="cuda")
    nj.kv_append(cache, nj.PagedBatch(start, keys.cuda(), table.cuda(), tokens=n), x, -x)
    want = torch.zeros(n, page, 1, 8)
    for b in range(n):
        if b not in (7, 8, 9):
            want[int(table[b]), int(keys[b]) - 1] = x[b].cpu()
    assert torch.equal(cache.k.cpu(), want) and torch.equal(cache.v.cpu(), -want)


def test_append_in_a_graph():
    """A captured append follows the lengths on the device, with eager work between the replays."""
    cache = nj.PagedCache(torch.zeros(4, 16, 2, 64, device="cuda"), torch.zeros(4, 16, 2, 64, device="cuda"))
    keys = torch.tensor([1], dtype=torch.int32, device="cuda")
    batch = nj.PagedBatch(torch.tensor([0, 1], dtype=torch.int32, device="cuda"), keys,
                          torch.tensor([[3, 1, 0, 2]], dtype=torch.int32, device="cuda"), tokens=1)
    table = nj.rotary_table(64, 64)
    k, v = torch.randn(1, 2, 64, device="cuda"), torch.randn(1, 2, 64, device="cuda")
    s = torch.cuda.Stream()
    nj.kv_append(cache, batch, k, v, table, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        nj.kv_append(cache, batch, k, v, table, stream=s)
    for n in (5, 17, 64):
        keys.fill_(n)
        k.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        page = [3, 1, 0, 2][(n - 1) // 16]
        want = nj.rotary(k, torch.tensor([n - 1], dtype=torch.int32, device="cuda"), table)
        assert torch.equal(cache.k[page, (n - 1) % 16], want[0]) and torch.equal(cache.v[page, (n - 1) % 16], v[0])


# -------------------------------------------------------------------- example

@pytest.mark.parametrize("kv_heads,dim,page,chunk", [(4, 64, 16, 50), (2, 128, 7, 1000), (1, 32, 64, 17)])
def test_example_serves_a_layer(kv_heads, dim, page, chunk):
    """Chunked prompts and decode steps through the whole block against fp64 without a cache.  Roundings to fp16 of q, k, v
    and o (one each, below U16 relative; those of q and k move logits of size 1) and of the weights of the softmax: below 8 U16."""
    from examples import serve_layer
    _, _, error = serve_layer.serve([130, 1, 64, 17], 5, width=256, q_heads=4, kv_heads=kv_heads, dim=dim, page_size=page,
                                    chunk=chunk, check=True)
    assert error < 8 * U16, error
