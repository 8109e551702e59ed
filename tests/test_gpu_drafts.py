"""A step of drafted tokens on the GPU against plain forms: the step's arrays,
norms of heads with turn and append and their gradients, attention of trees,
moves of accepted tokens, logit rules."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.drafts_util import (LENGTHS, MISSING, POOL, ROWS, TREE_COVER, attention_of, cover_name, norm_grad, normed, plain_logits, plain_step,
                               random_mask, signed, tree_mask, tree_seen, turned_with_bound, words_of)
from tests.serving_util import DT, U16, Batch, rounded

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _host(t):
    torch.cuda.synchronize()
    return t.cpu()


# ------------------------------------------------------------ the step's arrays

class Steps:
    """A page table and pool on the GPU with their plain counterparts."""

    def __init__(self, held, page, columns, spare, seed=0, capacity=None):
        rng = np.random.default_rng(seed)
        need = [-(-h // page) for h in held]
        ids = rng.permutation(sum(need) + spare).tolist()
        self.page, self.held, self.columns = page, list(held), columns
        self.table = [[ids.pop() for _ in range(n)] + [-5] * (columns - n) for n in need]
        self.count = len(ids)
        self.capacity = sum(need) + spare if capacity is None else capacity
        self.stack = ids + [-9] * (self.capacity - len(ids))
        self.d_table = _i32(self.table).view(len(held), columns)
        self.d_stack, self.d_count = _i32(self.stack), _i32([self.count])

    def check(self, added, tokens, keep=None, parent=None, words=0, in_place=False, tensors=None):
        keep_ = self.held if keep is None else keep
        want = plain_step(self.held, keep_, added, self.table, self.stack, self.count, self.capacity, self.page, tokens, parent, words)
        held = _i32(self.held)
        out = torch.full((1,), 77, dtype=torch.int32, device="cuda")
        pool = nj.PagePool(self.d_stack, self.d_count, None if in_place else out)
        step = nj.PagedStep(self.d_table, self.page, tokens, words, kv_len=held if in_place else None)
        for t in (step.q_start, step.positions, step.slots):
            t.fill_(99)
        nj.paged_step(step, pool, held, _i32(added), None if keep is None else _i32(keep), None if parent is None else _i32(parent))
        for name in ("q_start", "kv_len", "positions", "slots", "status"):
            assert _host(getattr(step, name)).tolist() == want[name], name
        assert _host(pool.count_out).tolist() == [want["count"]]
        if not in_place:
            self.d_count = out
        assert _host(self.d_table).tolist() == self.table
        assert _host(self.d_stack).tolist() == self.stack
        if parent is not None:
            assert _host(step.mask).tolist() == [[signed(w) for w in row] for row in want["mask"]]
        self.count = want["count"]
        self.held = list(want["kv_len"])
        return want


def _requests(rng, n, longest, tree):
    """Lengths of every kind: empty, just come, done, shrinking, going on."""
    held = [int(x) for x in rng.integers(0, longest + 1, n)]
    keep = [h if k > 1 else 0 if k == 0 else int(rng.integers(0, h + 1)) for h, k in zip(held, rng.integers(0, 5, n))]
    added = [0 if k == 0 and rng.random() < 0.5 else int(rng.integers(0, tree + 1)) for k in keep]
    return held, keep, added


@pytest.mark.parametrize("n,longest,tree,page", [(1, 40, 5, 16), (1, 0, 1, 1), (7, 200, 33, 16), (64, 300, 9, 7), (256, 100, 40, 32), (257, 60, 12, 5),
                                                 (1024, 50, 6, 16), (1500, 40, 5, 8), (8192, 20, 3, 4)])
@pytest.mark.parametrize("in_place", [False, True])
def test_step(n, longest, tree, page, in_place):
    """Several steps in turn on one table and pool."""
    rng = np.random.default_rng([n, page])
    held, keep, added = _requests(rng, n, longest, tree)
    s = Steps(held, page, -(-(longest + 4 * tree) // page) + 1, 4 * n * (tree // page + 1) + 3, seed=n)
    for i in range(3):
        want = s.check(added, sum(added) + int(rng.integers(0, 5)), keep=keep, in_place=in_place)
        assert want["status"][0] == 0
        _, _, added = _requests(rng, n, longest, tree)
        keep = [int(rng.integers(max(0, h - tree), h + 1)) if rng.random() < 0.9 else 0 for h in s.held]
    want = s.check([1] * n, n, in_place=in_place)          # keep NULL: plain decoding
    assert want["status"][0] == 0


@pytest.mark.parametrize("n,tree,words", [(1, 1, 1), (1, 64, 2), (5, 33, 2), (40, 70, 3), (3, 1024, 32), (600, 20, 1)])
def test_step_of_trees(n, tree, words):
    rng = np.random.default_rng([n, tree])
    held, keep, added = _requests(rng, n, 100, tree)
    added[0] = tree
    parent = []
    for a in added:
        for i in range(a):
            how = rng.random()
            # chains, roots, any earlier node, and what is no earlier node: a root
            parent.append(i - 1 if how < 0.5 else -1 if how < 0.6 else int(rng.integers(0, max(i, 1))) if how < 0.9 else
                          [i, i + 3, -7, 1 << 30][int(rng.integers(0, 4))])
    tokens = len(parent) + 6
    parent += [0] * 6
    s = Steps(held, 16, -(-(100 + 2 * tree) // 16) + 1, n * (tree // 16 + 2))
    want = s.check(added, tokens, keep=keep, parent=parent, words=words)
    assert want["status"][0] == 0


@pytest.mark.parametrize("bad,code", [
    (dict(added=[30, 40, 20]), MISSING), (dict(held=[20, -1, 0]), LENGTHS), (dict(keep=[20, 41, 0]), LENGTHS), (dict(keep=[-1, 40, 0]), LENGTHS),
    (dict(added=[1, -1, 1]), LENGTHS), (dict(added=[1, 1 << 30, 1]), LENGTHS), (dict(tokens=5), ROWS), (dict(parent=True, added=[1, 33, 1]), ROWS),
    (dict(count=-1), POOL), (dict(count=99), POOL), (dict(held=[20, 40, 1 << 30], keep=[20, 40, 0]), LENGTHS),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_step_refused(bad, code, in_place):
    """All or nothing: the step is empty, table and pool are as they were."""
    s = Steps([20, 40, 0], 16, 8, 4)
    added, tokens = bad.get("added", [1, 2, 3]), bad.get("tokens", 100)
    s.held = bad.get("held", s.held)
    if "count" in bad:
        s.count = bad["count"]
        s.d_count = _i32([s.count])
    keep = bad.get("keep")
    if keep is None and "held" in bad:
        keep = list(s.held)
    want = s.check(added, tokens, keep=keep, parent=[-1] * tokens if "parent" in bad else None, words=1 if "parent" in bad else 0,
                   in_place=in_place)
    assert want["status"][0] & code


def test_step_at_the_end_of_the_pool():
    """The last page is taken; one more is missing; what others give back is there at once."""
    s = Steps([16, 16, 32], 16, 4, 1)
    assert s.check([1, 0, 0], 8)["status"] == [0, 0, 1, 0]
    assert s.check([0, 1, 0], 8)["status"] == [MISSING, 1, 0, 0]
    assert s.check([0, 17, 0], 40, keep=[17, 16, 0])["status"] == [0, 0, 17, 0]
    assert s.table[1][:3] == [s.table[1][0], s.table[2][1], s.table[2][0]]


def test_step_without_sequences_or_rows():
    s = Steps([], 16, 0, 3)
    s.d_table = torch.zeros((0, 2), dtype=torch.int32, device="cuda")
    s.table = []
    assert s.check([], 5)["status"][0] == 0
    s = Steps([7, 0], 16, 2, 3)
    assert s.check([0, 0], 0)["status"][0] == 0
    assert s.check([0, 0], 0, keep=[0, 0])["count"] == 4


def test_step_in_a_graph():
    """Captured once in place, replayed as the sequences grow and shrink; the step's own batch follows."""
    n, page = 5, 4
    s = Steps([0] * n, page, 12, 60)
    held, added, keep = _i32([0] * n), _i32([0] * n), _i32([0] * n)
    pool = nj.PagePool(s.d_stack, s.d_count)
    step = nj.PagedStep(s.d_table, page, 40, kv_len=held)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nj.paged_step(step, pool, held, added, keep)
    rng = np.random.default_rng(4)
    for _ in range(8):
        k = [int(rng.integers(0, h + 1)) for h in s.held]
        a = [int(rng.integers(0, 8)) for _ in range(n)]
        keep.copy_(_i32(k))
        added.copy_(_i32(a))
        want = plain_step(s.held, k, a, s.table, s.stack, s.count, s.capacity, page, 40)
        graph.replay()
        assert (held + 0).tolist() == want["kv_len"]
        assert _host(step.slots).tolist() == want["slots"] and _host(step.status).tolist() == want["status"]
        assert _host(s.d_table).tolist() == s.table and _host(s.d_stack).tolist() == s.stack
        s.held, s.count = want["kv_len"], want["count"]


# --------------------------------------------------------- norms, turns, appends

def _angles(rng, tokens, rot, rows=300):
    table = np.concatenate([np.cos(a := rng.uniform(0, 6.28, (rows, rot // 2))), np.sin(a)], axis=1).astype(np.float32)
    pos = rng.integers(0, rows, tokens).astype(np.int32)
    if tokens > 2:
        pos[0], pos[1] = -4, rows + 9          # clamped to the table
    at = np.clip(pos, 0, rows - 1)
    return table, pos, table[at, :rot // 2].astype(np.float64), table[at, rot // 2:].astype(np.float64)


def _rows(rng, tokens, heads, dim, dtype, gap=0, shift=0, scale=1.0):
    """Head rows that begin `shift` elements into their buffer, `gap` elements between tokens."""
    width = heads * dim + gap
    flat = torch.from_numpy(rng.standard_normal(tokens * width + shift) * scale).to(DT[dtype]).cuda()
    return torch.as_strided(flat, (tokens, heads, dim), (width, dim, 1), shift)


def _np(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _inside(got, want, bound):
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    worst = np.nanmax(np.abs(got - want) - bound, initial=-1.0)
    assert worst <= 0, f"{worst} beyond the bound"


# (dim, rotary dims, layout, elements between tokens, elements before the first)
HEADS = [(128, 128, "half", 0, 0), (64, 64, "interleaved", 0, 0), (96, 48, "half", 8, 0), (128, 64, "interleaved", 0, 1), (256, 256, "half", 0, 0),
         (77, 30, "half", 3, 0), (1, 0, "half", 0, 0), (200, 200, "interleaved", 1, 0), (80, 0, "half", 0, 0), (255, 254, "half", 0, 2),
         (8, 8, "half", 0, 0), (136, 8, "interleaved", 0, 4)]


@pytest.mark.parametrize("dim,rot,layout,gap,shift", HEADS)
@pytest.mark.parametrize("src,dst,wt", [("f32", "f32", "f32"), ("f16", "f16", "f32"), ("f32", "f16", "f16"), ("f16", "f32", "f16")])
@pytest.mark.parametrize("tokens,heads,per_head", [(1, 3, False), (37, 5, True)])
def test_norm_rotary(dim, rot, layout, gap, shift, src, dst, wt, tokens, heads, per_head):
    rng = np.random.default_rng([dim, tokens])
    x = _rows(rng, tokens, heads, dim, src, gap, shift)
    x[tokens // 2, 1] = 0.0
    w = torch.from_numpy(rng.standard_normal((heads, dim) if per_head else dim) * 0.2 + 1).to(DT[wt]).cuda()
    table = None
    want, bound = normed(_np(x), _np(w), 1e-5)
    kw = {}
    if rot:
        t, pos, cos, sin = _angles(rng, tokens, rot)
        table = nj.RotaryTable(torch.from_numpy(t).cuda(), layout)
        kw = dict(positions=torch.from_numpy(pos).cuda(), table=table)
        want, bound = turned_with_bound(want, bound, cos, sin, layout)
    out = _rows(rng, tokens, heads, dim, dst, gap, shift)
    assert nj.norm_rotary(x, w, eps=1e-5, out=out, **kw) is out
    _inside(_np(out), want, rounded(want, bound, dst))
    if src == dst:                        # in place gives the same bits
        again = x.clone()                 # (of one alignment: it picks the kernel)
        other = nj.norm_rotary(again, w, eps=1e-5, **kw)
        nj.norm_rotary(again, w, eps=1e-5, out=again, **kw)
        assert torch.equal(again, other)


@pytest.mark.parametrize("dim,rot,layout,gap,shift", HEADS)
@pytest.mark.parametrize("xt,dt,wt", [("f32", "f32", "f32"), ("f16", "f16", "f16"), ("f32", "f16", "f32"), ("f16", "f32", "f16")])
@pytest.mark.parametrize("tokens,heads,per_head", [(1, 2, False), (70, 6, False), (41, 3, True)])
def test_norm_rotary_grad(dim, rot, layout, gap, shift, xt, dt, wt, tokens, heads, per_head):
    rng = np.random.default_rng([dim, tokens, 1])
    x, dy = _rows(rng, tokens, heads, dim, xt, gap, shift), _rows(rng, tokens, heads, dim, dt, gap, shift)
    w = torch.from_numpy(rng.standard_normal((heads, dim) if per_head else dim) * 0.2 + 1).to(DT[wt]).cuda()
    cos = sin = None
    kw = {}
    if rot:
        t, pos, cos, sin = _angles(rng, tokens, rot)
        kw = dict(positions=torch.from_numpy(pos).cuda(), table=nj.RotaryTable(torch.from_numpy(t).cuda(), layout))
    want, dw, bound, dwb = norm_grad(_np(x), _np(dy), _np(w), 1e-5, cos, sin, layout)
    if not per_head:
        dw, dwb = dw.sum(0), dwb.sum(0) * (1 + heads * 2.0 ** -24) + heads * 2.0 ** -24 * np.abs(dwb.sum(0)) / 2.0 ** -24 / tokens
    dx, dweight = nj.norm_rotary_grad(dy, x, w, eps=1e-5, **kw)
    _inside(_np(dx), want, rounded(want, bound, xt))
    _inside(_np(dweight), dw, rounded(dw, dwb, "f32"))
    again = nj.norm_rotary_grad(dy, x, w, eps=1e-5, **kw)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dweight), "the same bits every time"
    if xt == dt:                          # dx may be dy or x
        a, b = dy.clone(), x.clone()      # (of one alignment: it picks the kernel)
        plain = nj.norm_rotary_grad(a, b, w, eps=1e-5, **kw)[0]
        assert torch.equal(nj.norm_rotary_grad(a.clone(), b, w, eps=1e-5, dx=b.clone(), **kw)[0], plain)
        c = a.clone()
        assert torch.equal(nj.norm_rotary_grad(c, b, w, eps=1e-5, dx=c, **kw)[0], plain)
        assert torch.equal(nj.norm_rotary_grad(a, b, w, eps=1e-5, dx=b, **kw)[0], plain)


def test_norm_rotary_grad_against_differences():
    """The gradients are those of the kernel's own forward pass: central differences of it in fp32 with steps of 2^-6, whose
    third-order term is 2^-12 / 6 times third derivatives of size 10 and whose roundings are 2^-24 of sums of 48 values over the step."""
    rng = np.random.default_rng(3)
    x, w = _rows(rng, 2, 2, 24, "f32"), torch.from_numpy(rng.standard_normal(24) * 0.2 + 1).float().cuda()
    t, pos, _, _ = _angles(rng, 2, 16)
    kw = dict(positions=torch.from_numpy(pos).cuda(), table=nj.RotaryTable(torch.from_numpy(t).cuda()), eps=1e-5)
    dy = _rows(rng, 2, 2, 24, "f32")
    dx, dw = nj.norm_rotary_grad(dy, x, w, **kw)
    loss = lambda a, b: float((nj.norm_rotary(a, b, **kw).double() * dy.double()).sum())  # noqa: E731
    h = 2.0 ** -6
    for at in [(0, 0, 3), (1, 1, 20), (1, 0, 11)]:
        up, down = x.clone(), x.clone()
        up[at] += h
        down[at] -= h
        assert abs((loss(up, w) - loss(down, w)) / (2 * h) - float(dx[at])) < 2e-3
    for i in (0, 9, 23):
        up, down = w.clone(), w.clone()
        up[i] += h
        down[i] -= h
        assert abs((loss(x, up) - loss(x, down)) / (2 * h) - float(dw[i])) < 2e-3


@pytest.mark.parametrize("tokens,heads,per_head", [(4000, 8, False), (1500, 32, True)])
def test_norm_rotary_grad_of_many_rows(tokens, heads, per_head):
    """More rows than workgroups take at once; the weight's gradient against its sum in 64 bits."""
    rng = np.random.default_rng(8)
    x, dy = _rows(rng, tokens, heads, 64, "f32"), _rows(rng, tokens, heads, 64, "f32")
    w = torch.from_numpy(rng.standard_normal((heads, 64) if per_head else 64) * 0.2 + 1).float().cuda()
    want, dw, bound, dwb = norm_grad(_np(x), _np(dy), _np(w), 1e-6, None, None, "half")
    dx, dweight = nj.norm_rotary_grad(dy, x, w)
    _inside(_np(dx), want, rounded(want, bound, "f32"))
    if not per_head:
        dw, dwb = dw.sum(0), heads * dwb.sum(0)
    _inside(_np(dweight), dw, rounded(dw, dwb, "f32"))


def test_norm_grad_of_one_side_only():
    """Through the C entry: dx or dw alone, no tokens."""
    rng = np.random.default_rng(5)
    x, dy, w = _rows(rng, 9, 2, 32, "f32"), _rows(rng, 9, 2, 32, "f32"), torch.ones(32, device="cuda")
    dx, dw = nj.norm_rotary_grad(dy, x, w)
    a, b = torch.full_like(x, 5.0), torch.full_like(w, 5.0)
    call = lambda n, p, q: nj.check(nj.nnjit_norm_rotary_grad(None, n, 2, 32, None, w, 0, 0, 1e-6, x, 64, 32, 0, dy, 64, 32, 0, p, 64, 32, q))  # noqa: E731
    call(9, a, None)
    call(9, None, b)
    torch.cuda.synchronize()
    assert torch.equal(a, dx) and torch.equal(b, dw)
    call(0, None, b)
    torch.cuda.synchronize()
    assert bool((b == 0).all())
    for shape in ((0, 2, 32), (5, 0, 32)):                 # no rows: the sum is 0
        none = torch.zeros(shape, device="cuda")
        b.fill_(5.0)
        dx, dw = nj.norm_rotary_grad(none, none, w, dweight=b)
        assert dx.shape == shape and bool((b == 0).all())
        assert nj.norm_rotary(none, w).shape == shape


@pytest.mark.parametrize("dim,rot,layout,gap,shift", HEADS)
@pytest.mark.parametrize("src,dtype", [("f32", "f32"), ("f32", "f16"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("how", ["both", "keys", "none", "per head"])
def test_kv_append_slots(dim, rot, layout, gap, shift, src, dtype, how):
    rng = np.random.default_rng([dim, 7])
    tokens, hq, hk, page, pages = 29, 6, 2, 5, 9
    qkv = _rows(rng, tokens, hq + 2 * hk, dim, src, gap, shift)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    flat = torch.full((2, pages * page * hk * dim + shift), 3.0, dtype=DT[dtype], device="cuda")
    kc, vc = (f[shift:].view(pages, hk, page, dim).transpose(1, 2) for f in flat)
    cache = nj.PagedCache(kc, vc)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    slots[[3, 17]] = -1
    slots[11], slots[12] = pages * page, 1 << 40                # not in the cache
    weights = [torch.from_numpy(rng.standard_normal((h, dim) if how == "per head" else dim) * 0.2 + 1).to(DT[src]).cuda() for h in (hq, hk)]
    norm = {"both": lambda: nj.HeadNorm(*weights, eps=1e-5), "per head": lambda: nj.HeadNorm(*weights, eps=1e-5),
            "keys": lambda: nj.HeadNorm(None, weights[1], eps=1e-5), "none": lambda: None}[how]()
    kw = {}
    live = (slots >= 0) & (slots < pages * page)
    out = torch.full((tokens, hq, dim), 3.0, dtype=DT[dtype], device="cuda")

    def expected(x, w):
        y, b = normed(_np(x), _np(w), 1e-5) if w is not None else (_np(x), np.zeros(x.shape))
        return turned_with_bound(y, b, cos, sin, layout) if rot else (y, b)

    if rot:
        t, pos, cos, sin = _angles(rng, tokens, rot)
        kw = dict(positions=torch.from_numpy(pos).cuda(), rotary=nj.RotaryTable(torch.from_numpy(t).cuda(), layout))
    assert nj.kv_append_slots(cache, torch.from_numpy(slots).cuda(), k, v, q=q, q_out=out, norm=norm, **kw) is out
    want, bound = expected(q, None if how in ("keys", "none") else weights[0])
    _inside(_np(out)[live], want[live], rounded(want, bound, dtype)[live])
    assert bool((out.cpu()[~torch.from_numpy(live)] == 3.0).all())
    want, bound = expected(k, None if how == "none" else weights[1])
    got_k, got_v = _np(kc).reshape(-1, hk, dim), _np(vc).reshape(-1, hk, dim)
    at = slots[live]
    _inside(got_k[at], want[live], rounded(want, bound, dtype)[live])
    assert np.array_equal(got_v[at], _np(v.to(DT[dtype]))[live])
    rest = np.setdiff1d(np.arange(pages * page), at)
    assert (got_k[rest] == 3.0).all() and (got_v[rest] == 3.0).all(), "other slots are left alone"
    assert nj.kv_append_slots(cache, torch.from_numpy(slots).cuda(), k, v, norm=None if norm is None else nj.HeadNorm(None, weights[1]), **kw) is None


def test_append_slots_is_append():
    """Without norms, with the positions of the batch's rows, it is kv_append: values to the last bit; turned rows within both
    bounds (which product of a turn is fused with the sum is the compiler's choice, so their last bits may differ)."""
    B = Batch([5, 1, 40], [25, 1, 133], 4, 2, 64, 16, "f16", seed=5).device()
    C = Batch([5, 1, 40], [25, 1, 133], 4, 2, 64, 16, "f16", seed=5).device()
    rng = np.random.default_rng(1)
    rows = _rows(rng, 46, 8, 64, "f32")
    table = nj.rotary_table(200, 64)
    past = [m - n for n, m in zip(B.news, B.keys)]
    pos = [p + i for n, p in zip(B.news, past) for i in range(n)]
    slots = [int(B.table[b, (p + i) // 16]) * 16 + (p + i) % 16 for b, (n, p) in enumerate(zip(B.news, past)) for i in range(n)]
    a = nj.kv_append(B.cache, B.batch, rows[:, 4:6], rows[:, 6:], table, rows[:, :4])
    b = nj.kv_append_slots(C.cache, torch.tensor(slots).cuda(), rows[:, 4:6], rows[:, 6:], _i32(pos), table, rows[:, :4])
    cos, sin = _np(table.table)[pos, :32], _np(table.table)[pos, 32:]
    x = _np(rows)
    want, bound = turned_with_bound(x[:, :4], np.zeros((46, 4, 64)), cos, sin, "half")
    _inside(_np(a), _np(b), 2 * rounded(want, bound, "f16"))
    want, bound = turned_with_bound(x[:, 4:6], np.zeros((46, 2, 64)), cos, sin, "half")
    first, second = (_np(k).reshape(-1, 2, 64) for k in (B.dk, C.dk))
    _inside(first[slots], second[slots], 2 * rounded(want, bound, "f16"))
    rest = np.setdiff1d(np.arange(len(first)), slots)
    assert np.array_equal(first[rest], second[rest], equal_nan=True)
    assert np.array_equal(_np(B.dv), _np(C.dv), equal_nan=True)


# ---------------------------------------------------------------- trees

def _tree_case(news, keys, hq, hk, dim, page, dtype, words, kind="tree", window=0, limits=None, scale=None, edit=None, **kw):
    B = Batch(news, keys, hq, hk, dim, page, dtype, **kw)
    rng = np.random.default_rng([len(news), dim, words])
    mask, depth = tree_mask(B, words, rng) if kind == "tree" else (random_mask(B, words, rng, 0.0 if kind == "empty" else 0.4), None)
    positions = np.zeros(B.tokens, dtype=np.int32)
    for b, (n, m) in enumerate(zip(B.news, B.keys)):
        at = slice(B.start[b], B.start[b] + n)
        positions[at] = m - n + (depth[at] if depth is not None else rng.integers(-3, n + 3, n))
    if edit:
        edit(B, mask)
    B.device(**(limits or {}))
    out = torch.full(B.q.shape, 7.0, dtype=DT[dtype], device="cuda")
    how = dict(window=window, positions=torch.from_numpy(positions).cuda()) if window else {}
    nj.tree_attention(B.dq, B.cache, B.batch, torch.from_numpy(mask.view(np.int32)).cuda(), out, scale=scale, **how)
    torch.cuda.synchronize()
    want, bound = attention_of(B, tree_seen(B, mask, window, positions), scale)
    rows = sum(news)
    assert bool((out[rows:] == 7.0).all()), "rows of no sequence are left alone"
    got, want, bound = _np(out)[:rows], want[:rows], bound[:rows]
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf])
    fine = np.isfinite(want)
    _inside(got[fine], want[fine], bound[fine])
    norm = np.linalg.norm(want[fine])
    if norm > 0:
        assert np.linalg.norm(got[fine] - want[fine]) / norm <= (1e-5 if dtype == "f32" else 2 * U16)
    return got


SHAPES = [(4, 4, 64), (8, 2, 128), (6, 2, 96), (16, 1, 64), (5, 1, 256), (3, 3, 40), (2, 2, 200)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", SHAPES)
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("kind", ["tree", "any"])
def test_trees(dtype, hq, hk, dim, page, kind):
    """Trees of one node to sixty at the ends of tiles and pages; masks of any pattern, with bits of tokens that are not there."""
    _tree_case([1, 7, 16, 33, 60, 2], [1, 20, 48, 160, 61, 130], hq, hk, dim, page, dtype, 2, kind)


@pytest.mark.parametrize("case", TREE_COVER, ids=cover_name)
def test_every_kernel_of_trees(case):
    """Every tile height, split and whole, by whole pages and by look-ups a lane, element by element."""
    dtype, news, keys, hq, hk, dim, _, _, _ = case
    _tree_case(news, keys, hq, hk, dim, 16, dtype, 4, "tree", seed=31)
    _tree_case(news, keys, hq, hk, dim, 12, dtype, 4, "any", 150, seed=32)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(4, 4, 64), (16, 2, 128), (3, 1, 96)])
def test_wide_trees_and_short_masks(dtype, hq, hk, dim):
    """More nodes than a mask has bits for: the others are not seen.  Tiles of 64 and 128 rows."""
    _tree_case([130, 64, 97], [330, 64, 500], hq, hk, dim, 16, dtype, 5)
    _tree_case([130, 64, 97], [330, 64, 500], hq, hk, dim, 16, dtype, 1, "any")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(4, 4, 64), (8, 2, 128), (32, 2, 64)])
def test_masks_that_leave_nothing(dtype, hq, hk, dim):
    """No cached key and no bit: zeros; fewer keys than new tokens: the first have no place."""
    got = _tree_case([5, 40, 3], [5, 40, 50], hq, hk, dim, 16, dtype, 2, "empty")
    assert (got[:45] == 0).all() and (got[45:] != 0).any()
    _tree_case([9, 40, 33], [4, 0, 20], hq, hk, dim, 16, dtype, 2, "any")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(4, 4, 64), (8, 2, 128), (32, 2, 64)])
@pytest.mark.parametrize("window", [1, 5, 40, 100000])
def test_trees_with_a_window(dtype, hq, hk, dim, window):
    _tree_case([7, 33, 1, 60], [90, 400, 300, 70], hq, hk, dim, 16, dtype, 2, "tree", window)
    _tree_case([7, 33, 1, 60], [90, 400, 300, 70], hq, hk, dim, 16, dtype, 2, "any", window)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim,new", [(8, 8, 64, 9), (8, 8, 128, 16), (16, 2, 128, 33), (4, 2, 64, 64)])
@pytest.mark.parametrize("window", [0, 1500])
def test_trees_behind_long_contexts(dtype, hq, hk, dim, new, window):
    """Keys split over workgroups, a tree across the last splits."""
    _tree_case([new, 3], [2900 + new, 700], hq, hk, dim, 16, dtype, 2, "tree", window, seed=3)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(4, 4, 64), (8, 2, 128), (32, 2, 64)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_trees_and_values_that_are_not_finite(dtype, hq, hk, dim, bad):
    """In nodes that some rows do not see, in keys and values: those rows are not touched, the others get what the formula gives."""
    def edit(B, mask):
        for b, n in ((1, 20), (2, 41)):
            s = B.key_slots(b)
            B.v[s[B.keys[b] - n + 3]][0, 1] = bad
            B.v[s[B.keys[b] - n + 3]][0, 2] = -bad
            B.v[s[B.keys[b] - n + 7]][0, 2] = bad
            if bad != bad:
                B.k[s[B.keys[b] - n + 5]][0, 3] = bad
        mask[B.start[1]:B.start[1] + 20, 0] &= ~np.uint32(1 << 7)          # no row sees it
    _tree_case([4, 20, 41], [30, 77, 141], hq, hk, dim, 16, dtype, 2, "any", edit=edit)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("dim,shift,row_gap,extra", [(64, 1, 3, 1), (77, 0, 0, 0), (128, 2, 0, 0), (200, 1, 0, 0)])
def test_trees_of_any_alignment(dtype, dim, shift, row_gap, extra):
    _tree_case([9, 50], [60, 130], 4, 2, dim, 7, dtype, 2, shift=shift, row_gap=row_gap, extra_dim=extra, order="hnd", pad=3)


def test_trees_scale_and_limits():
    """Negative and zero scales; a max_q below the new tokens: such rows are the full result or left alone."""
    for scale in (-0.3, 0.0, 1.5):
        _tree_case([9, 20], [60, 90], 4, 2, 64, 16, "f32", 1, scale=scale)
    B = Batch([40, 4], [700, 600], 8, 2, 64, 16, "f16", seed=9)
    rng = np.random.default_rng(2)
    mask, depth = tree_mask(B, 2, rng)
    pos = np.concatenate([660 + depth[:40], 596 + depth[40:]]).astype(np.int32)
    for window in (0, 300):
        B.device(max_q=4, max_kv=700)
        out = torch.full(B.q.shape, 7.0, dtype=torch.float16, device="cuda")
        nj.tree_attention(B.dq, B.cache, B.batch, torch.from_numpy(mask.view(np.int32)).cuda(), out, window=window,
                          positions=torch.from_numpy(pos).cuda())
        want, bound = attention_of(B, tree_seen(B, mask, window, pos))
        got = _np(out)
        alone = (got == 7.0).all(axis=2)
        assert not alone[40:].any() and not alone[:4].any()
        _inside(got[~alone], want[~alone], bound[~alone])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_chain_is_causal_attention(dtype):
    """A tree that is one chain: what paged_attention gives, within both bounds."""
    B = Batch([20, 1, 33], [120, 9, 33], 8, 2, 64, 16, dtype, seed=6).device()
    words = [[(1 << min(i + 1, 32)) - 1, (1 << max(i + 1 - 32, 0)) - 1] for n in B.news for i in range(n)]
    mask = torch.tensor(np.array(words, dtype=np.uint32).view(np.int32)).cuda()
    a, b = nj.paged_attention(B.dq, B.cache, B.batch), nj.tree_attention(B.dq, B.cache, B.batch, mask)
    _, bound = attention_of(B, tree_seen(B, mask.cpu().numpy().view(np.uint32)))
    assert (np.abs(_np(a) - _np(b)) <= 2 * bound).all()


# ---------------------------------------------------------------- moves

def _move_case(news, keys, hk, dim, page, dtype, path, accepted, **kw):
    B = Batch(news, keys, hk, hk, dim, page, dtype, **kw).device()
    before = [[t[s].clone() for s in B.key_slots(b)] for t in (B.k, B.v) for b in range(len(news))]
    nj.kv_move(B.cache, B.batch, _i32(path), _i32(accepted))
    torch.cuda.synchronize()
    for which, t in enumerate((B.dk.cpu(), B.dv.cpu())):
        for b, (n, m) in enumerate(zip(news, keys)):
            rows = list(before[which * len(news) + b])
            want = list(rows)
            for i in range(min(max(accepted[b], 0), len(path[b]))):
                p = path[b][i]
                if i < p < n and m - n + i >= 0:
                    want[m - n + i] = rows[m - n + p]
            for s, w in zip(B.key_slots(b), want):
                assert torch.equal(t[s], w)
    used = {s for b in range(len(news)) for s in B.key_slots(b)}
    for pg in range(B.k.shape[0]):
        for slot in range(page):
            if (pg, slot) not in used:
                assert bool(B.dk[pg, slot].isnan().all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hk,dim,page,kw", [(8, 128, 16, {}), (3, 64, 5, {}), (2, 77, 7, dict(order="hnd")), (1, 33, 1, dict(shift=1)),
                                            (4, 96, 32, dict(order="hnd", extra_dim=4)), (2, 6, 16, dict(shift=2))])
def test_move(dtype, hk, dim, page, kw):
    """Paths whose places are later entries' sources, longer than a thread takes at a time; entries that are skipped."""
    rng = np.random.default_rng(dim)
    news, keys = [1, 40, 17, 30, 5], [9, 90, 17, 31, 60]
    path = np.zeros((5, 33), dtype=np.int64)
    for b, n in enumerate(news):
        steps = np.cumsum(rng.integers(1, 3, 33))
        path[b] = np.minimum(steps - 1 + (b == 2), n + 2)         # past the end: skipped
    path[3, :6] = [2, 1, 1, 9, 9, 4]                              # twice the same, in place, below its own place
    path[4, 1] = -3
    _move_case(news, keys, hk, dim, page, dtype, path.tolist(), [1, 33, 15, 6, 99], **kw)
    _move_case(news, keys, hk, dim, page, dtype, path.tolist(), [0, -5, 2, 33, 3], **kw)


def test_move_of_rows_without_a_place():
    """Fewer keys than new tokens: new token 0 has no place; pages outside the pool are left out."""
    _move_case([9, 4], [4, 30], 2, 64, 16, "f16", [[1, 7, 8, 8, 6, 8], [1, 2, 3, 3, 3, 3]], [6, 3])
    B = Batch([4], [34], 2, 2, 64, 16, "f16").device()
    B.batch.page_table[0, 2] = 1 << 20
    k = B.dk.clone()
    nj.kv_move(B.cache, B.batch, _i32([[3, 3]]), _i32([2]))
    assert np.array_equal(_np(k), _np(B.dk), equal_nan=True)


# ---------------------------------------------------------------- logits

def _logits_case(rows, vocab, history_len, src="f32", dst="f32", rules=("rep", "pres", "freq", "bias", "mask"), gap=0, shift=0, in_place=False,
                 mask_rows=None, length=None, prompt=True, seed=0):
    rng = np.random.default_rng([rows, vocab, seed])
    flat = torch.from_numpy(rng.standard_normal(rows * (vocab + gap) + shift) * 3).to(DT[src]).cuda()
    x = torch.as_strided(flat, (rows, vocab), (vocab + gap, 1), shift)
    kw, plain = {}, {}
    if history_len is not None:
        few = rng.integers(-2, vocab + 2, (rows, max(1, min(40, vocab))))
        h = np.take_along_axis(few, rng.integers(0, few.shape[1], (rows, history_len)), axis=1)
        h[:, ::7] = rng.integers(0, vocab, h[:, ::7].shape)
        kw["history"], plain["history"] = _i32(h), h.tolist()
        n = [history_len] * rows if length is None else length
        kw["length"], plain["length"] = _i32(n), n
        if prompt:
            p = [int(t) for t in rng.integers(-1, history_len + 2, rows)]
            kw["prompt"], plain["prompt"] = _i32(p), p
        for name, key, lo, hi in (("rep", "repetition", 0.7, 1.5), ("pres", "presence", -1, 1), ("freq", "frequency", -0.5, 0.5)):
            if name in rules:
                v = rng.uniform(lo, hi, rows).astype(np.float32)
                kw[key], plain[key] = torch.from_numpy(v).cuda(), v
    if "bias" in rules:
        t = rng.integers(-1, vocab + 1, (rows, 60))
        t[:, 30:] = t[:, :30]                                   # every token twice: the last entry counts
        v = rng.standard_normal((rows, 60)).astype(np.float32)
        kw["bias_token"], kw["bias_value"] = _i32(t), torch.from_numpy(v).cuda()
        plain["bias"] = [list(zip(a, b)) for a, b in zip(t.tolist(), v.tolist())]
    if "mask" in rules:
        allowed = rng.random((mask_rows or rows, vocab)) < 0.5
        allowed[0] = False                                      # nothing is left
        kw["mask"] = words_of(allowed).cuda()
        if mask_rows:
            m = [int(i) for i in rng.integers(-1, mask_rows, rows)]
            kw["mask_row"] = _i32(m)
            plain["allowed"] = np.stack([allowed[i] if i >= 0 else np.ones(vocab, bool) for i in m])
        else:
            plain["allowed"] = allowed
    want, bound = plain_logits(_np(x), **plain)
    r = nj.LogitRules(**kw)
    if in_place:
        out = nj.adjust_logits(x, r, x)
        assert out is x
    else:
        to = torch.full((rows * (vocab + gap) + shift,), 9.0, dtype=DT[dst], device="cuda")
        out = torch.as_strided(to, (rows, vocab), (vocab + gap, 1), shift)
        nj.adjust_logits(x, r, out)
        if gap and rows > 1:
            assert bool((torch.as_strided(to, (rows - 1, gap), (vocab + gap, 1), shift + vocab) == 9.0).all())
    got = _np(out)
    off = np.isneginf(want)
    assert np.array_equal(np.isneginf(got), off)
    _inside(got[~off], want[~off], rounded(want, bound, src if in_place else dst)[~off])


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("f32", "f16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("rows,vocab,history", [(1, 1, 1), (3, 31, 5), (2, 1000, 300), (5, 4097, 64), (1, 32000, 1000), (70, 9000, 400)])
def test_logits(src, dst, rows, vocab, history):
    _logits_case(rows, vocab, history, src, dst)
    _logits_case(rows, vocab, history, src, dst, mask_rows=3, seed=1)


@pytest.mark.parametrize("gap,shift", [(1, 0), (3, 1), (4, 4), (0, 2)])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_logits_of_any_alignment_and_in_place(gap, shift, dtype):
    _logits_case(4, 1030, 50, dtype, dtype, gap=gap, shift=shift)
    _logits_case(4, 1030, 50, dtype, dtype, gap=gap, shift=shift, in_place=True)
    _logits_case(300, 9001, 50, dtype, dtype, gap=gap, shift=shift, in_place=True)


@pytest.mark.parametrize("rules", [("rep",), ("pres",), ("freq",), ("bias",), ("mask",), ("rep", "mask"), ("pres", "freq", "bias")])
def test_logits_one_rule_at_a_time(rules):
    _logits_case(4, 3000, None if rules in (("bias",), ("mask",)) else 200, rules=rules)


def test_logits_lengths():
    """Histories of no token, of more than the columns hold, without a prompt; none at all."""
    _logits_case(5, 500, 30, length=[0, 30, 99, -3, 1])
    _logits_case(5, 500, 30, length=[0, 30, 99, -3, 1], prompt=False)
    _logits_case(2, 500, 0)


def test_logits_of_long_histories_and_many_biases():
    """Counts above 2^15, entries above 2^16: the last of them counts."""
    n, vocab = 70000, 50
    h = np.full((2, n), 7)
    h[1, ::2] = 9
    t = np.full((2, n), -1)
    t[:, [3, 65537, 69999]] = 9
    v = np.arange(n, dtype=np.float32)[None, :].repeat(2, axis=0) / 1024
    x = torch.zeros(2, vocab, device="cuda")
    r = nj.LogitRules(history=_i32(h), prompt=_i32([1, 0]), frequency=torch.tensor([1.0, 0.5], device="cuda"), presence=torch.ones(2, device="cuda"),
                      bias_token=_i32(t), bias_value=torch.from_numpy(v).cuda())
    y = nj.adjust_logits(x, r).cpu()
    assert y[0, 7] == -(n - 1) - 1 and y[1, 7] == -n / 4 - 1
    assert y[0, 9] == np.float32(69999 / 1024) and y[1, 9] == np.float32(-n / 4 - 1) + np.float32(69999 / 1024)
    assert int((y != 0).sum()) == 4
    r = nj.LogitRules(history=_i32(h[:, :32767]), frequency=torch.ones(2, device="cuda"))
    assert nj.adjust_logits(x, r).cpu()[0, 7] == -32767


@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("gap", [0, 3])
def test_logits_of_many_rows(src, dst, gap):
    """Segments of each length, their last ones partly beyond the row; histories that could overflow a narrow count."""
    _logits_case(200, 8193, 90, src, dst, gap=gap)
    _logits_case(400, 16390, 90, src, dst, gap=gap, mask_rows=5)
    _logits_case(130, 9000, 33000, src, dst, gap=gap, length=[33000 if i == 0 else i for i in range(130)], mask_rows=5)
    _logits_case(130, 9000, 33000, src, dst, gap=gap, length=[5000 if i == 0 else i for i in range(130)], mask_rows=5, prompt=False)


def test_logits_that_are_not_finite():
    """Infinities and NaN in places that a mask takes away are gone; elsewhere they stay."""
    x = torch.zeros(1, 64, device="cuda")
    x[0, 3], x[0, 4], x[0, 5], x[0, 6], x[0, 7] = float("nan"), float("inf"), float("nan"), -float("inf"), torch.finfo(torch.float32).min
    allowed = np.ones((1, 64), bool)
    allowed[0, [3, 4]] = False
    r = nj.LogitRules(history=_i32([[5, 6, 7, 8]]), repetition=torch.full((1,), 2.0, device="cuda"), mask=words_of(allowed).cuda())
    y = nj.adjust_logits(x, r).cpu()[0]
    assert y[3] == y[4] == -float("inf") and y[5].isnan() and y[6] == -float("inf") and y[7] == -float("inf") and y[8] == 0


# --------------------------------------------------- streams, graphs, all together

def test_binding_refuses_operands():
    """Tensors on the GPU that the entry points would read or write out of bounds; nothing is launched."""
    r = lambda *shape, dtype=torch.float16: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    cache = nj.PagedCache(r(4, 16, 2, 64), r(4, 16, 2, 64))
    batch = nj.PagedBatch(_i32([0, 3]), _i32([20]), _i32([[0, 1]]), tokens=3)
    table, slots, pos = nj.rotary_table(32, 64), torch.zeros(3, dtype=torch.int64, device="cuda"), _i32([0, 1, 2])
    k, q, w, mask = r(3, 2, 64), r(3, 4, 64), r(64, dtype=torch.float32), _i32([[1]] * 3)
    step, pool = nj.PagedStep(_i32([[0, 1], [2, 3]]), 16, 8, 1), nj.PagePool(_i32([5, 6]), _i32([2]))
    rules = nj.LogitRules(history=_i32([[1], [2]]), mask=_i32([[-1], [-1]]))
    bad = [
        lambda: nj.kv_append_slots(cache, slots.int(), k, k), lambda: nj.kv_append_slots(cache, slots.cpu(), k, k),
        lambda: nj.kv_append_slots(cache, slots[:2], k, k), lambda: nj.kv_append_slots(cache, slots, k[:, :1], k),
        lambda: nj.kv_append_slots(cache, slots, k, k.float()), lambda: nj.kv_append_slots(cache, slots, k, k, rotary=table),
        lambda: nj.kv_append_slots(cache, slots, k, k, pos[:2], table), lambda: nj.kv_append_slots(cache, slots, k, k, q_out=q),
        lambda: nj.kv_append_slots(cache, slots, k, k, q=q[0]), lambda: nj.kv_append_slots(cache, slots, k, k, q=q, q_out=q[:, :3]),
        lambda: nj.kv_append_slots(cache, slots, k, k, q=q, q_out=q[:, :1].expand(3, 4, 64)),
        lambda: nj.kv_append_slots(cache, slots, k, k, norm=nj.HeadNorm(w[:32])),
        lambda: nj.kv_append_slots(cache, slots, k, k, norm=nj.HeadNorm(None, r(3, 64))),
        lambda: nj.kv_append_slots(cache, slots, k, k, q=q, norm=nj.HeadNorm(r(3, 64))),
        lambda: nj.norm_rotary(q, w[:32]), lambda: nj.norm_rotary(q, r(3, 64)), lambda: nj.norm_rotary(q, w, table=table),
        lambda: nj.norm_rotary(q, w, pos.long(), table), lambda: nj.norm_rotary(q, w, out=r(3, 4, 32)), lambda: nj.norm_rotary(q, w.cpu()),
        lambda: nj.norm_rotary(q.transpose(1, 2), r(4)), lambda: nj.norm_rotary(q.double(), w), lambda: nj.norm_rotary(q, w.double()),
        lambda: nj.norm_rotary_grad(q[:2], q, w), lambda: nj.norm_rotary_grad(q, q, w, dweight=w[:32]),
        lambda: nj.norm_rotary_grad(q, q, w, dweight=w.half()), lambda: nj.norm_rotary_grad(q, q, w, dx=q.float()),
        lambda: nj.tree_attention(q, cache, batch, mask[:2]), lambda: nj.tree_attention(q, cache, batch, mask.long()),
        lambda: nj.tree_attention(q, cache, batch, mask[:, :0]), lambda: nj.tree_attention(q, cache, batch, mask.cpu()),
        lambda: nj.tree_attention(q, cache, batch, mask, window=3), lambda: nj.tree_attention(q[:2], cache, batch, mask),
        lambda: nj.tree_attention(q, cache, batch, mask, out=q.float()), lambda: nj.tree_attention(q[:, :3], cache, batch, mask),
        lambda: nj.tree_attention(q, cache, batch, mask, positions=pos[:2], window=3),
        lambda: nj.kv_move(cache, batch, _i32([[0], [0]]), _i32([1])), lambda: nj.kv_move(cache, batch, _i32([[0]]), _i32([1, 1])),
        lambda: nj.kv_move(cache, batch, _i32([[0]]).long(), _i32([1])), lambda: nj.kv_move(cache, batch, _i32([0]), _i32([1])),
        lambda: nj.paged_step(step, pool, pos, pos[:2]), lambda: nj.paged_step(step, pool, pos[:2].cpu(), pos[:2]),
        lambda: nj.paged_step(step, pool, pos[:2].long(), pos[:2]), lambda: nj.paged_step(step, pool, pos[:2], pos[:2], keep=pos),
        lambda: nj.paged_step(step, pool, pos[:2], pos[:2], parent=pos),
        lambda: nj.paged_step(nj.PagedStep(_i32([[0]]), 16, 8), pool, pos[:1], pos[:1], parent=pos),
        lambda: nj.adjust_logits(r(3, 32), rules), lambda: nj.adjust_logits(r(2, 33), rules), lambda: nj.adjust_logits(r(2, 32).cpu(), rules),
        lambda: nj.adjust_logits(r(2, 32), rules, r(2, 31)), lambda: nj.adjust_logits(r(2, 32), rules, r(1, 32).expand(2, 32)),
        lambda: nj.adjust_logits(r(32, 2).t(), rules), lambda: nj.adjust_logits(r(2, 32, dtype=torch.float64), rules),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, nj.NnjitError)):
            call()
            raise AssertionError(f"call {i} was not refused")


def _calls():
    """name -> (inputs, call of them that returns one tensor)"""
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *shape, dtype=torch.float16: torch.randn(shape, device="cuda", generator=g).to(dtype)
    table, w = nj.rotary_table(600, 64), r(64, dtype=torch.float32) + 2
    cache = nj.PagedCache(r(40, 16, 2, 64), r(40, 16, 2, 64))
    pages = torch.randperm(40, generator=g, device="cuda").to(torch.int32)[None]
    batch = nj.PagedBatch(_i32([0, 9]), _i32([600]), pages, tokens=9, max_q=9, max_kv=600)
    pos, slots = _i32(list(range(591, 600))), torch.arange(9, device="cuda") * 3
    mask, path, accepted = _i32([[(2 << i) - 1] for i in range(9)]), _i32([[0, 2, 5, 8]]), _i32([4])
    norm = nj.HeadNorm(w, w)
    rules = nj.LogitRules(history=_i32([[1, 2, 1]] * 6), frequency=torch.ones(6, device="cuda"))
    backup = cache.k.clone(), cache.v.clone()

    def append(k, v, q, **kw):
        out = nj.kv_append_slots(cache, slots, k, v, pos, table, q, norm=norm, **kw)
        return torch.cat([out.flatten(), cache.k.flatten(), cache.v.flatten()])

    def move(k, **kw):
        cache.k.copy_(k)                       # (the same places are moved in every call)
        cache.v.copy_(k)
        nj.kv_move(cache, batch, path, accepted, **kw)
        return torch.cat([cache.k.flatten(), cache.v.flatten()])

    pool = nj.PagePool(torch.arange(100, 160, dtype=torch.int32, device="cuda"), _i32([50]), _i32([0]))
    step = nj.PagedStep(_i32([list(range(20)), list(range(20, 40))]), 4, 30, 1)
    parent = _i32([-1, 0, 0, 1] + [-1, 0, 1, 2] + [0] * 22)

    def arrays(lengths, **kw):
        nj.paged_step(step, pool, lengths[0], lengths[1], lengths[2], parent, **kw)
        return torch.cat([t.flatten().long() for t in (step.q_start, step.kv_len, step.positions, step.slots, step.mask, step.page_table,
                                                       step.status, pool.count_out, pool.free_pages)])

    return {
        "paged_step": ([_i32([[9, 30], [4, 4], [9, 12]])], arrays),
        "kv_append_slots": ([r(9, 2, 64), r(9, 2, 64), r(9, 8, 64)], append),
        "norm_rotary": ([r(9, 8, 64)], lambda x, **kw: nj.norm_rotary(x, w, pos, table, **kw)),
        "norm_rotary_grad": ([r(9, 8, 64), r(9, 8, 64)],
                             lambda dy, x, **kw: torch.cat([t.flatten().float() for t in nj.norm_rotary_grad(dy, x, w, pos, table, **kw)])),
        "tree_attention": ([r(9, 8, 64)], lambda q, **kw: nj.tree_attention(q, cache, batch, mask, **kw)),
        "kv_move": ([backup[0]], move),
        "adjust_logits": ([r(6, 500, dtype=torch.float32)], lambda x, **kw: nj.adjust_logits(x, rules, **kw)),
    }


NAMES = ["paged_step", "kv_append_slots", "norm_rotary", "norm_rotary_grad", "tree_attention", "kv_move", "adjust_logits"]


@pytest.mark.parametrize("name", NAMES)
def test_current_stream(name):
    """The inputs are written behind other work of the current stream, the result is read there."""
    inputs, call = _calls()[name]
    want = call(*inputs).clone()
    torch.cuda.synchronize()
    late = [torch.zeros_like(x) for x in inputs]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                        # about 10 ms
        for x, y in zip(late, inputs):
            x.copy_(y)
        got = call(*late).clone()
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("name", NAMES)
def test_captured_without_a_stream(name):
    """Inside a capture the current stream is the captured one; replays between eager calls of the same inputs give the same."""
    inputs, call = _calls()[name]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = call(*inputs).clone()                         # the stream's scratch
    torch.cuda.synchronize()
    held = [x.clone() for x in inputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = call(*held)
    for rep in range(3):
        got.zero_()
        eager = call(*inputs).clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(eager, want), rep


@pytest.mark.parametrize("name", ["norm_rotary", "norm_rotary_grad", "tree_attention", "adjust_logits"])
def test_outputs_belong_to_the_given_stream(name):
    """Memory that the current stream still writes is not handed to a call on another stream."""
    inputs, call = _calls()[name]
    want = call(*inputs).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for given in (side, side.cuda_stream):
        busy = torch.empty_like(inputs[0])
        torch.cuda._sleep(4_000_000)
        busy.fill_(3.0)                                      # queued behind the sleep, on the current stream
        del busy                                             # its block may be reused there at once
        with torch.cuda.stream(side):
            got = call(*inputs, stream=given)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_capture_that_needs_scratch():
    """A captured call whose stream lacks the scratch is refused; it works once a call of the sizes has run."""
    rng = np.random.default_rng(5)
    x, dy, w = _rows(rng, 3000, 4, 64, "f32"), _rows(rng, 3000, 4, 64, "f32"), torch.ones(64, device="cuda")
    # a stream of its own: torch hands its streams out again and again, with the scratch of earlier calls
    handle = ctypes.c_void_p()
    assert nj.load().hipStreamCreateWithFlags(ctypes.byref(handle), 1) == 0
    s = torch.cuda.ExternalStream(handle.value)
    dx, dw = torch.empty_like(x), torch.empty(64, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(nj.NnjitError, match="run a call of the same sizes once"):
            nj.norm_rotary_grad(dy, x, w, dx=dx, dweight=dw)
    nj.norm_rotary_grad(dy, x, w, dx=dx, dweight=dw, stream=s)
    torch.cuda.synchronize()
    want = dw.clone()
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph(), stream=s):
        nj.norm_rotary_grad(dy, x, w, dx=dx, dweight=dw)
    for _ in range(3):
        dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, want)


@pytest.mark.parametrize("prompts,new,nodes,page", [([40, 7, 1], 24, 12, 16), ([3, 70], 20, 40, 5), ([5], 9, 1, 16)])
def test_decoding_with_drafted_trees(prompts, new, nodes, page):
    """The operators together: every generated token is the best allowed one of the formulas in 64 bits without a cache.

    Logits are sums of 256 products of values rounded to fp16 (the attention's output, x + o and the cache: relative U16 each, against
    logits of size 1 to 4), so a choice may lie a few 2^-11 times 4 below the best."""
    from examples import speculate
    said, steps, worst = speculate.generate(prompts, new, nodes, page_size=page, check=True)
    assert [len(s) for s in said] == [new] * len(prompts)
    assert worst < 4 * 4 * U16
    if nodes > 1:
        plain, more, _ = speculate.generate(prompts, new, 1, page_size=page)
        assert steps < more, "drafts save steps"
        assert plain == said or worst > 0
