"""The operators of a step of drafted tokens where their descriptions allow more
than a plain step does: batches with fewer rows than their starts say, handles
used in turn, the longest lists, calls of many rows."""
import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.drafts_util import LOGIT_COVER, attention_of, normed, signed, tree_seen, turned_with_bound
from tests.serving_util import DT, Batch, rounded
from tests.test_gpu_drafts import _angles, _inside, _logits_case, _np, _rows

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# ------------------------------------------------------------ the step's arrays

def _chain(i, words):
    bits = (2 << min(i, 32 * words - 1)) - 1
    return [signed(bits >> 32 * w & 0xffffffff) for w in range(words)]


@pytest.mark.parametrize("words", [1, 2, 32])
@pytest.mark.parametrize("added", [[1, 1], [70, 3], [0, 33], [64, 31], [1200, 1]])
@pytest.mark.parametrize("in_place", [False, True])
def test_masks_of_a_step_without_trees(added, words, in_place):
    """A step that was a tree's and is filled without parents has the masks of chains, not its last step's; rows behind the last
    sequence, and all rows of a refused step, see nothing."""
    tokens, pages = 1300, 200
    held = _i32([0, 0])
    pool = nj.PagePool(torch.arange(pages, dtype=torch.int32, device="cuda"), _i32([pages]))
    step = nj.PagedStep(torch.zeros((2, 100), dtype=torch.int32, device="cuda"), 16, tokens, words, kv_len=held if in_place else None)
    nj.paged_step(step, pool, held, _i32([20, 32]), parent=_i32([-1] + [0] * (tokens - 1)))
    assert step.status.tolist()[0] == 0 and step.mask[19, 0].tolist() == signed(1 | 1 << 19)
    held = held if in_place else step.kv_len
    nj.paged_step(step, pool, held, _i32(added), keep=_i32([10, 10]))
    want = [_chain(i, words) for n in added for i in range(n)]
    assert step.status.tolist()[0] == 0
    assert step.mask.tolist() == want + [[0] * words] * (tokens - len(want))
    nj.paged_step(step, pool, step.kv_len, _i32([1 << 20, 1]))
    assert step.status.tolist()[0] != 0 and not step.mask.any()


def test_chain_masks_serve_tree_attention():
    """... so that a step of up to 32 mask_words new tokens a sequence may use either attention."""
    B = Batch([20, 1, 33], [120, 9, 33], 4, 2, 64, 16, "f32", seed=6).device()
    pages = int(B.table[B.table < 1 << 29].max()) + 1
    step = nj.PagedStep(B.batch.page_table.clone(), 16, B.tokens, 2)
    pool = nj.PagePool(torch.zeros(pages, dtype=torch.int32, device="cuda"), _i32([0]))
    nj.paged_step(step, pool, _i32(B.keys), _i32(B.news), keep=_i32([m - n for n, m in zip(B.news, B.keys)]))
    assert step.status.tolist()[0] == 0 and step.kv_len.tolist() == B.keys
    got = nj.tree_attention(B.dq, B.cache, step.batch(), step.mask)
    want, bound = attention_of(B, tree_seen(B, step.mask.cpu().numpy().view(np.uint32)))
    causal = [np.tril(np.ones((n, m), dtype=bool), m - n) for n, m in zip(B.news, B.keys)]
    assert all(np.array_equal(a, b) for a, b in zip(causal, tree_seen(B, step.mask.cpu().numpy().view(np.uint32))))
    assert (np.abs(got.double().cpu().numpy() - want) <= bound + 2.0 ** -24 * np.abs(want)).all()


def test_a_step_of_almost_all_the_pages_that_a_pool_can_hold():
    """Sequences that end give back 2^31 - 8192 pages in their order; the next step's rows take the last of them."""
    n, columns, rows = 8192, (1 << 18) - 1, (1 << 24) - 1
    given = n * columns
    table = torch.arange(given, dtype=torch.int32, device="cuda").view(n, columns)
    free, count = torch.full(((1 << 31) - 1,), -3, dtype=torch.int32, device="cuda"), _i32([0])
    pool, step = nj.PagePool(free, count), nj.PagedStep(table, 1, rows)
    none = torch.zeros(n, dtype=torch.int32, device="cuda")
    nj.paged_step(step, pool, torch.full_like(none, columns), none, keep=none)
    assert step.status.tolist() == [0, 0, 0, given] and count.tolist() == [given]
    assert torch.equal(free[:given].view(n, columns), table) and bool((free[given:] == -3).all())
    nj.paged_step(step, pool, step.kv_len, torch.full_like(none, 2047))
    assert step.status.tolist() == [0, 0, 2047 * n, given - 2047 * n]
    want = free[given - 2047 * n:given].flip(0)
    assert torch.equal(table[:, :2047].reshape(-1), want) and torch.equal(step.slots[:2047 * n], want.long())


# ------------------------------------------------- norms: memory read and written

def _qkv(dtype=torch.float16, heads=10, dim=64, tokens=70):
    return torch.randn(tokens, heads, dim, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)


def test_norms_that_overlap_are_refused():
    """Results over their operands with another type, stride or begin; nothing is launched."""
    w, rows, slots = torch.ones(64, device="cuda"), _qkv(torch.float32), torch.arange(70, device="cuda")
    kept = rows.clone()
    x, halves = rows[:, :4], rows.view(torch.float16).view(70, 10, 2, 64)
    cache = nj.PagedCache(*(torch.zeros(5, 16, 2, 64, dtype=torch.float16, device="cuda") for _ in range(2)))
    other = nj.PagedCache(cache.k.float(), cache.v.float())
    fp16 = torch.as_strided(rows.view(torch.float16), (70, 4, 64), (640, 64, 1))
    bad = [
        lambda: nj.norm_rotary(x, w, out=fp16), lambda: nj.norm_rotary(x, w, out=rows[:, 1:5]), lambda: nj.norm_rotary(x[1:], w, out=x[:-1]),
        lambda: nj.norm_rotary(x, w, out=halves[:, :4, 0]), lambda: nj.norm_rotary(x, w, out=torch.as_strided(rows, (70, 4, 64), (512, 64, 1))),
        lambda: nj.kv_append_slots(cache, slots, rows[:, 4:6], rows[:, 6:8], q=x, q_out=fp16),
        lambda: nj.kv_append_slots(other, slots, rows[:, 4:6], rows[:, 6:8], q=x, q_out=rows[:, 1:5]),
        lambda: nj.kv_append_slots(other, slots, rows[:, 4:6], rows[:, 8:10], q=x, q_out=rows[:, 5:9]),
        lambda: nj.kv_append_slots(other, slots, rows[:, 8:10], rows[:, 4:6], q=x, q_out=rows[:, 5:9]),
        lambda: nj.norm_rotary_grad(x, rows[:, 6:], w, dx=rows[:, 3:7]), lambda: nj.norm_rotary_grad(fp16, kept[:, :4], w, dx=x),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(nj.NnjitError, match="overlap"):
            call()
            raise AssertionError(f"call {i} was not refused")
    torch.cuda.synchronize()
    assert torch.equal(rows, kept)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_norms_in_place_and_side_by_side(dtype):
    """Operands and results that are column ranges of one tensor; queries turned in place in a packed projection."""
    w, table, pos = torch.rand(64, device="cuda") + 0.5, nj.rotary_table(100, 64), torch.arange(70, dtype=torch.int32, device="cuda")
    rows = _qkv(dtype)
    want = nj.norm_rotary(rows[:, :4], w, pos, table)
    side = rows.clone()
    nj.norm_rotary(side[:, :4], w, pos, table, out=side[:, 4:8])
    assert torch.equal(side[:, 4:8], want) and torch.equal(side[:, :4], rows[:, :4]) and torch.equal(side[:, 8:], rows[:, 8:])
    slots = torch.randperm(80, device="cuda")[:70]
    slots[[3, 69]] = -1
    made = []
    for in_place in (False, True):
        cache = nj.PagedCache(*(torch.zeros(5, 16, 2, 64, dtype=dtype, device="cuda") for _ in range(2)))
        qkv = rows.clone()
        q = qkv[:, :4]
        out = q if in_place else q.clone()
        nj.kv_append_slots(cache, slots, qkv[:, 4:6], qkv[:, 6:8], pos, table, q, out, nj.HeadNorm(w, w))
        assert torch.equal(qkv[:, 4:], rows[:, 4:]) and torch.equal(out[[3, 69]], rows[[3, 69], :4])
        made.append((out.clone(), cache.k, cache.v))
    assert all(torch.equal(a, b) for a, b in zip(*made))
    keep = slots >= 0
    assert torch.equal(made[0][0][keep], want[keep])


# ------------------------------------------------------- norms of many rows

# (tokens, query heads, key heads, dim, rotary dims, layout, elements before the first row, a weight a head, source, cache): 1024
# tokens and more have workgroups of several tokens, whose last one may hold fewer; groups with several rows of a
# token, of queries or of keys and values; rows from any address
MANY = [
    (1024, 32, 8, 128, 128, "half", 0, False, "f16", "f16"), (1025, 32, 8, 128, 128, "half", 0, True, "f32", "f16"),
    (2051, 32, 8, 64, 64, "interleaved", 0, False, "f32", "f32"), (2051, 5, 1, 256, 256, "half", 0, True, "f16", "f16"),
    (1025, 5, 1, 64, 32, "half", 0, True, "f16", "f32"), (2051, 5, 1, 128, 0, "half", 0, False, "f32", "f16"),
    (1030, 32, 8, 96, 96, "interleaved", 0, False, "f16", "f16"), (1025, 1, 16, 64, 64, "half", 0, False, "f16", "f16"),
    (3001, 2, 1, 8, 8, "half", 0, True, "f32", "f32"), (1027, 40, 1, 136, 8, "half", 0, False, "f32", "f16"),
    (1025, 5, 2, 77, 30, "half", 3, False, "f16", "f16"), (1025, 6, 1, 128, 64, "interleaved", 1, True, "f32", "f16"),
    (2051, 1, 3, 255, 254, "half", 0, False, "f32", "f32"),
]


@pytest.mark.parametrize("tokens,hq,hk,dim,rot,layout,shift,per_head,src,dtype", MANY)
def test_norms_and_appends_of_many_rows(tokens, hq, hk, dim, rot, layout, shift, per_head, src, dtype):
    """Element by element; skipped rows -- the last ones among them -- and slots that no row names stay as they were."""
    rng = np.random.default_rng([tokens, dim])
    qkv = _rows(rng, tokens, hq + 2 * hk, dim, src, 0, shift)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    weights = [torch.from_numpy(rng.standard_normal((h, dim) if per_head else dim) * 0.2 + 1).to(DT[src]).cuda() for h in (hq, hk)]
    table, kw, cos, sin = None, {}, None, None
    if rot:
        t, pos, cos, sin = _angles(rng, tokens, rot)
        table, pos = nj.RotaryTable(torch.from_numpy(t).cuda(), layout), torch.from_numpy(pos).cuda()
        kw = dict(positions=pos, table=table)

    def expected(x, w):
        y, b = normed(_np(x), _np(w), 1e-5)
        return turned_with_bound(y, b, cos, sin, layout) if rot else (y, b)

    want_q, bound_q = expected(q, weights[0])
    out = _rows(rng, tokens, hq, dim, dtype, 0, shift)
    nj.norm_rotary(q, weights[0], eps=1e-5, out=out, **kw)
    _inside(_np(out), want_q, rounded(want_q, bound_q, dtype))
    again = nj.norm_rotary(q, weights[0], eps=1e-5, **kw) if shift == 0 else None
    if again is not None:
        packed = qkv.clone()
        nj.norm_rotary(packed[:, :hq], weights[0], eps=1e-5, out=packed[:, :hq], **kw)
        assert torch.equal(packed[:, :hq], again) and torch.equal(packed[:, hq:], qkv[:, hq:])

    page, pages = 7, -(-tokens // 7) + 3
    flat = torch.full((2, pages * page * hk * dim + shift), 3.0, dtype=DT[dtype], device="cuda")
    cache = nj.PagedCache(*(f[shift:].view(pages, hk, page, dim).transpose(1, 2) for f in flat))
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    slots[rng.random(tokens) < 0.05] = -1
    slots[[tokens - 1, tokens - 3]], slots[5] = -1, pages * page
    live = (slots >= 0) & (slots < pages * page)
    out = torch.full((tokens, hq, dim), 3.0, dtype=DT[dtype], device="cuda")
    nj.kv_append_slots(cache, torch.from_numpy(slots).cuda(), k, v, kw.get("positions"), table, q, out, nj.HeadNorm(*weights, eps=1e-5))
    _inside(_np(out)[live], want_q[live], rounded(want_q, bound_q, dtype)[live])
    assert bool((out.cpu()[~torch.from_numpy(live)] == 3.0).all())
    want_k, bound_k = expected(k, weights[1])
    got_k, got_v = (_np(c).reshape(pages * page, hk, dim) for c in (cache.k, cache.v))
    _inside(got_k[slots[live]], want_k[live], rounded(want_k, bound_k, dtype)[live])
    assert np.array_equal(got_v[slots[live]], _np(v.to(DT[dtype]))[live])
    named = np.zeros(pages * page, bool)
    named[slots[live]] = True
    assert (got_k[~named] == 3.0).all() and (got_v[~named] == 3.0).all()


@pytest.mark.parametrize("heads,dim,shift", [(1, 64, 0), (3, 128, 0), (8, 64, 0), (32, 128, 0), (5, 256, 0), (40, 8, 0), (6, 64, 1), (33, 16, 3)])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_weight_gradients_to_the_last_row(heads, dim, shift, per_head, dtype):
    """Whole numbers, so that a row left out or taken twice shows: x = +-1 and eps = 0 in dims of a power of two make r = 1 exactly
    (the mean of the squares is 1), and dy whole and up to 8 makes every partial sum of g x r a whole number below 2^24."""
    for tokens in (1, 2, 3, 31, 33, 127, 500, 1025, 4000, 4099, 8191):
        if tokens * heads * dim > 1 << 24:
            continue
        rng = np.random.default_rng([tokens, heads])
        x, dy = _rows(rng, tokens, heads, dim, dtype, 0, shift), _rows(rng, tokens, heads, dim, dtype, 0, shift)
        x.copy_(torch.from_numpy(rng.choice([-1.0, 1.0], (tokens, heads, dim))))
        dy.copy_(torch.from_numpy(rng.integers(-8, 9, (tokens, heads, dim)).astype(np.float64)))
        w = torch.ones((heads, dim) if per_head else dim, device="cuda")
        dw = nj.norm_rotary_grad(dy, x, w, eps=0.0)[1]
        want = (dy.double() * x.double()).sum(0) if per_head else (dy.double() * x.double()).sum((0, 1))
        assert torch.equal(dw.double(), want), tokens


# ---------------------------------------------------------------- moves

@pytest.mark.parametrize("rows", [14, 11, 7, 5])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_move_with_fewer_rows_than_the_starts_say(rows, dtype):
    """Places follow kv_len and the starts, as they do for appends and attention, though the last rows are not in the batch:
    entries that name those are skipped, the others go where an append of the same batch puts its rows."""
    news, keys, path, accepted = [5, 9], [30, 25], [[1, 3, 3, 4], [2, 4, 7, 8]], [3, 4]
    B = Batch(news, keys, 2, 2, 64, 16, dtype, seed=4).device()
    batch = nj.PagedBatch(B.batch.q_start, B.batch.kv_len, B.batch.page_table, tokens=rows)
    nj.kv_move(B.cache, batch, _i32(path), _i32(accepted))
    torch.cuda.synchronize()
    for before, after in ((B.k, B.dk.cpu()), (B.v, B.dv.cpu())):
        for b, (n, m) in enumerate(zip(news, keys)):
            slots = B.key_slots(b)
            want = [before[s] for s in slots]
            there = min(n, max(rows - sum(news[:b]), 0))
            for i, p in enumerate(path[b][:accepted[b]]):
                if i < p < there:
                    want[m - n + i] = before[slots[m - n + p]]
            for s, w in zip(slots, want):
                assert torch.equal(after[s], w)


def test_moves_along_the_longest_path():
    """A path of as many entries as a call takes, all accepted, says the lengths; those that the sequence has move."""
    n = (1 << 31) - 1
    path = torch.zeros((1, n), dtype=torch.int32, device="cuda")
    path[0, :4] = _i32([1, 3, 4, 6])
    B = Batch([7], [30], 2, 2, 64, 16, "f16", seed=4).device()
    rows = [B.k[s].clone() for s in B.key_slots(0)]
    batch = nj.PagedBatch(_i32([0, 7]), _i32(B.keys), B.batch.page_table, tokens=7)
    nj.kv_move(B.cache, batch, path, _i32([n]))
    want = list(rows)
    want[23], want[24], want[25], want[26] = rows[24], rows[26], rows[27], rows[29]
    torch.cuda.synchronize()
    for s, w in zip(B.key_slots(0), want):
        assert torch.equal(B.dk[s].cpu(), w)


# ---------------------------------------------------------------- logits

def test_logits_of_the_longest_lists():
    """Histories and biases of as many entries as a call takes: their last ones count, and the walk ends there."""
    n, vocab = (1 << 31) - 1, 8
    x = torch.full((1, vocab), 2.0, device="cuda")
    history = torch.full((1, n), -1, dtype=torch.int32, device="cuda")
    history[0, 0], history[0, n // 2], history[0, n - 1], history[0, n - 2] = 3, 3, 3, 5
    ones = torch.ones(1, device="cuda")
    y = nj.adjust_logits(x, nj.LogitRules(history=history, prompt=_i32([1]), frequency=ones, presence=ones)).cpu()
    assert y.tolist() == [[2.0, 2.0, 2.0, -1.0, 2.0, 0.0, 2.0, 2.0]]
    tokens, values = history[:, :n - 1], torch.zeros((1, n), device="cuda")[:, :n - 1]
    values[0, 0], values[0, n // 2], values[0, n - 2] = 1.0, 4.0, 8.0
    y = nj.adjust_logits(x, nj.LogitRules(bias_token=tokens, bias_value=values)).cpu()
    assert y.tolist() == [[2.0, 2.0, 2.0, 6.0, 2.0, 10.0, 2.0, 2.0]]


@pytest.mark.parametrize("case", LOGIT_COVER, ids=str)
@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("f32", "f16"), ("f16", "f32"), ("f16", "f16")])
def test_every_kernel_of_logits(case, src, dst):
    """Rows that are taken four tokens at a time and rows of no alignment, with a mask a row and with grammars; in place."""
    rows, vocab, history = case[:3]
    gap = -vocab % 4
    length = [history] + list(range(1, rows)) if history > 4096 else None          # (one long one: the plain form counts slowly)
    _logits_case(rows, vocab, history, src, dst, gap=gap, mask_rows=5, length=length, seed=2)
    _logits_case(rows, vocab, history, src, dst, gap=gap + 1, shift=1, length=length, seed=3)
    if src == dst:
        _logits_case(rows, vocab, history, src, dst, gap=gap, length=length, in_place=True, seed=4)


# ------------------------------------------------------------- far and shared memory

def _far(shape, stride, dtype):
    """A tensor whose first dimension's stride passes 2^31 elements (memory of its own)."""
    size = (shape[0] - 1) * stride + int(np.prod(shape[1:]))
    inner = torch.empty(shape[1:], device="meta").stride()
    return torch.as_strided(torch.empty(size, dtype=dtype, device="cuda"), shape, (stride, *inner))


FAR = (1 << 31) + 64


def test_caches_past_31_bits():
    """Pages more than 2^31 elements apart: appends, moves and trees as on a cache whose pages lie together."""
    g = torch.Generator("cuda").manual_seed(2)
    r = lambda *shape: torch.randn(*shape, device="cuda", generator=g).half()  # noqa: E731
    near = nj.PagedCache(r(3, 16, 2, 64), r(3, 16, 2, 64))
    far = nj.PagedCache(*(_far((3, 16, 2, 64), FAR, torch.float16) for _ in range(2)))
    far.k.copy_(near.k)
    far.v.copy_(near.v)
    k, v, q, w = r(9, 2, 64), r(9, 2, 64), r(9, 8, 64), r(64).float() + 2
    slots, table = _i32([40, 41, 47, 0, 1, 30, 31, -1, 44]).long(), nj.rotary_table(64, 64)
    pos, pages = torch.arange(9, dtype=torch.int32, device="cuda"), _i32([[2, 0, 1]])
    mask = _i32([[(2 << i) - 1] for i in range(9)])
    got = []
    for cache in (near, far):
        turned = nj.kv_append_slots(cache, slots, k, v, pos, table, q, torch.zeros_like(q), nj.HeadNorm(w, w))
        batch = nj.PagedBatch(_i32([0, 9]), _i32([44]), pages, tokens=9)
        out = nj.tree_attention(turned, cache, batch, mask)
        nj.kv_move(cache, batch, _i32([[1, 3, 5, 8]]), _i32([4]))
        got.append((turned, out, nj.tree_attention(turned, cache, batch, mask), cache.k.clone(), cache.v.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dim", [64, 63])
def test_rows_past_31_bits(dim):
    """Tokens more than 2^31 elements apart: norms and their gradients, element by element as side by side."""
    x, dy = torch.randn(3, 2, dim, device="cuda").half(), torch.randn(3, 2, dim, device="cuda").half()
    w = torch.rand(dim, device="cuda") + 0.5
    fx, fy = _far(x.shape, FAR, torch.float16), _far(x.shape, FAR, torch.float16)
    fx.copy_(x)
    fy.copy_(dy)
    y, (dx, dw) = nj.norm_rotary(x, w), nj.norm_rotary_grad(dy, x, w)
    assert torch.equal(nj.norm_rotary(fx, w), y)
    got = nj.norm_rotary_grad(fy, fx, w, dx=fy)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    assert torch.equal(nj.norm_rotary(fx, w, out=fx), y)


def test_logits_past_31_bits():
    x = torch.randn(3, 5000, device="cuda").half()
    far = _far(x.shape, FAR, torch.float16)
    far.copy_(x)
    rules = nj.LogitRules(history=_i32([[1, 2, 4999]] * 3), frequency=torch.ones(3, device="cuda"), mask=_i32([[-5] * 157] * 3))
    want = nj.adjust_logits(x, rules)
    assert torch.equal(nj.adjust_logits(far, rules, far), want) and torch.equal(far, want)


@pytest.mark.parametrize("dim,tokens", [(64, 40), (128, 1100), (77, 33)])
def test_norms_of_shared_rows(dim, tokens):
    """x and dy that are one row, one token or one head for all: as of their copies."""
    table, w = nj.rotary_table(2000, dim // 2 * 2), torch.rand(3, dim, device="cuda") + 0.5
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    full = torch.randn(tokens, 3, dim, device="cuda")
    for x in (full[:1].expand_as(full), full[:, :1].expand_as(full), full[:1, :1].expand_as(full)):
        # (of the alignment that a copy has: it picks the kernel)
        y, (dx, dw) = nj.norm_rotary(x.contiguous(), w, pos, table), nj.norm_rotary_grad(x.contiguous(), full, w, pos, table)
        assert torch.equal(nj.norm_rotary(x, w, pos, table), y)
        for a, b in zip(nj.norm_rotary_grad(x, full, w, pos, table), (dx, dw)):
            assert torch.equal(a, b)
        for a, b in zip(nj.norm_rotary_grad(full, x, w, pos, table), nj.norm_rotary_grad(full, x.contiguous(), w, pos, table)):
            assert torch.equal(a, b)
