"""Host-side tests of the operators of a step of drafted tokens (no GPU):
argument checks come before any HIP call, the binding refuses operands that
the entry points would read or write out of bounds, and the plain forms that
the GPU tests compare with agree with small hand-worked cases."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.drafts_util import (LENGTHS, MISSING, POOL, ROWS, TREE_COVER, attention_of, cover_name, norm_grad, normed, plain_logits, plain_step,
                               tree_plan, tree_seen, words_of)
from tests.serving_util import Batch
from tests.test_serving_cpu import BAD_BATCHES, BAD_CACHES, _batch, _kv, _rot


@pytest.fixture(scope="module", autouse=True)
def lib():
    return nj.load(build_if_missing=True)


def _pool(**kw):
    d = dict(free_pages=16, capacity=8, count=16, count_out=16)
    d.update(kw)
    return nj.PagePoolDesc(**d)


def _arrays(**kw):
    d = dict(sequences=2, tokens=4, held=16, keep=None, added=32, parent=None, page_table=16, ld_table=4, table_pages=4, page_size=16,
             q_start=16, kv_len=48, positions=16, slots=16, mask=None, ld_mask=0, mask_words=0, status=16)
    d.update(kw)
    return nj.StepDesc(**d)


def _norm(**kw):
    d = dict(q_weight=16, k_weight=16, q_head=0, k_head=0, dtype=0, eps=1e-6)
    d.update(kw)
    return nj.HeadNormDesc(**d)


def _rules(**kw):
    return nj.LogitRulesDesc(**kw)


def _step(pool=None, arrays=None):
    return nj.nnjit_paged_step(_pool() if pool is None else pool, _arrays() if arrays is None else arrays)


def _append(kv=None, tokens=1, slots=16, pos=16, rot=None, norm=None, k=16, v=16, kst=(64, 32), heads=4, q=16, out=16, ost=(128, 32), dtype=0):
    return nj.nnjit_kv_append_slots(_kv() if kv is None else kv, tokens, slots, pos, rot, norm, k, *kst, v, 64, 32, heads, q, 128, 32, out,
                                    *ost, dtype)


def _forward(rot=None, tokens=1, heads=2, dim=32, pos=16, w=16, wh=0, wd=0, eps=1e-6, x=16, xst=(64, 32), xd=0, y=16, yst=(64, 32), yd=1):
    return nj.nnjit_norm_rotary(rot, tokens, heads, dim, pos, w, wh, wd, eps, x, *xst, xd, y, *yst, yd)


def _grad(rot=None, tokens=1, heads=2, dim=32, pos=16, w=16, wh=0, wd=0, eps=1e-6, x=16, xd=0, dy=16, dyst=(64, 32), dyd=0, dx=16,
          dxst=(64, 32), dw=16):
    return nj.nnjit_norm_rotary_grad(rot, tokens, heads, dim, pos, w, wh, wd, eps, x, 64, 32, xd, dy, *dyst, dyd, dx, *dxst, dw)


def _tree(kv=None, batch=None, mask=16, ld=1, words=1, pos=None, heads=4, q=16, out=16, ost=(128, 32), scale=0.1, window=0):
    return nj.nnjit_tree_attention(_kv() if kv is None else kv, _batch() if batch is None else batch, mask, ld, words, pos, heads, q, 128, 32,
                                   out, *ost, scale, window)


def _move(kv=None, batch=None, path=16, ld=4, n=4, accepted=16):
    return nj.nnjit_kv_move(_kv() if kv is None else kv, _batch() if batch is None else batch, path, ld, n, accepted)


def _logits(rules=None, rows=2, vocab=100, x=16, ldx=100, xd=0, y=16, ldy=100, yd=0):
    return nj.nnjit_adjust_logits(_rules() if rules is None else rules, rows, vocab, x, ldx, xd, y, ldy, yd)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches(bad):
    want = nj.NNJIT_EDTYPE if "dtype" in bad else nj.NNJIT_EINVAL
    for call in (_append, _tree, _move):
        assert call(kv=_kv(**bad)) == want and nj.nnjit_last_error()


@pytest.mark.parametrize("bad", BAD_BATCHES)
def test_bad_batches(bad):
    for call in (_tree, _move):
        assert call(batch=_batch(**bad)) == nj.NNJIT_EINVAL and nj.nnjit_last_error()


@pytest.mark.parametrize("call", [
    lambda: nj.nnjit_paged_step(None, _arrays()), lambda: nj.nnjit_paged_step(_pool(), None),
    lambda: _step(_pool(capacity=-1)), lambda: _step(_pool(free_pages=None)), lambda: _step(_pool(count=None)), lambda: _step(_pool(count_out=None)),
    lambda: _step(arrays=_arrays(sequences=-1)), lambda: _step(arrays=_arrays(sequences=8193)), lambda: _step(arrays=_arrays(tokens=-1)),
    lambda: _step(arrays=_arrays(tokens=1 << 24)), lambda: _step(arrays=_arrays(page_size=0)), lambda: _step(arrays=_arrays(page_size=(1 << 30) + 1)),
    lambda: _step(arrays=_arrays(table_pages=-1)), lambda: _step(arrays=_arrays(ld_table=3)), lambda: _step(arrays=_arrays(held=None)),
    lambda: _step(arrays=_arrays(added=None)), lambda: _step(arrays=_arrays(page_table=None)), lambda: _step(arrays=_arrays(kv_len=None)),
    lambda: _step(arrays=_arrays(q_start=None)), lambda: _step(arrays=_arrays(status=None)), lambda: _step(arrays=_arrays(kv_len=32)),
    lambda: _step(arrays=_arrays(parent=16)), lambda: _step(arrays=_arrays(parent=16, mask=16, ld_mask=40, mask_words=33)),
    lambda: _step(arrays=_arrays(parent=16, mask=16, ld_mask=1, mask_words=2)), lambda: _step(arrays=_arrays(parent=16, ld_mask=1, mask_words=1)),
    lambda: _append(tokens=-1), lambda: _append(tokens=1 << 24), lambda: _append(slots=None), lambda: _append(rot=_rot(), pos=None),
    lambda: _append(k=None), lambda: _append(v=None), lambda: _append(q=None), lambda: _append(out=None), lambda: _append(heads=-1),
    lambda: _append(kst=(-1, 32)), lambda: _append(ost=(128, 16)), lambda: _append(tokens=2, ost=(127, 32)), lambda: _append(rot=_rot(rotary_dim=34)),
    lambda: _append(kv=_kv(k_token=0)), lambda: _append(norm=_norm(eps=-1.0)), lambda: _append(norm=_norm(eps=math.nan)),
    lambda: _append(norm=_norm(q_head=-1)), lambda: _append(norm=_norm(k_head=31)),
    lambda: _forward(tokens=-1), lambda: _forward(tokens=1 << 24), lambda: _forward(heads=-1), lambda: _forward(heads=(1 << 30) + 1),
    lambda: _forward(dim=0), lambda: _forward(dim=257), lambda: _forward(rot=_rot(), pos=None), lambda: _forward(w=None), lambda: _forward(wh=31),
    lambda: _forward(eps=math.inf), lambda: _forward(x=None), lambda: _forward(xst=(-64, 32)), lambda: _forward(y=None),
    lambda: _forward(tokens=2, yst=(32, 32)), lambda: _forward(rot=_rot(table=None)),
    lambda: _grad(w=None), lambda: _grad(w=None, tokens=0), lambda: _grad(w=None, heads=0), lambda: _grad(x=None), lambda: _grad(dy=None), lambda: _grad(dyst=(64, -1)),
    lambda: _grad(tokens=2, dxst=(63, 32)), lambda: _grad(tokens=1 << 23, heads=256, dxst=(8192, 32)), lambda: _grad(heads=1 << 16, wh=32, dxst=(1 << 21, 32)),
    lambda: nj.nnjit_tree_attention(None, _batch(), 16, 1, 1, None, 4, 16, 128, 32, 16, 128, 32, 0.1),
    lambda: nj.nnjit_tree_attention(_kv(), None, 16, 1, 1, None, 4, 16, 128, 32, 16, 128, 32, 0.1),
    lambda: _tree(mask=None), lambda: _tree(words=0), lambda: _tree(words=(1 << 20) + 1), lambda: _tree(ld=-1), lambda: _tree(window=3),
    lambda: _tree(window=-1, pos=16), lambda: _tree(heads=3), lambda: _tree(q=None), lambda: _tree(out=None), lambda: _tree(ost=(128, 31)),
    lambda: _tree(scale=math.inf), lambda: _tree(batch=_batch(max_q=-1)),
    lambda: _move(path=None), lambda: _move(accepted=None), lambda: _move(n=-1), lambda: _move(ld=3), lambda: _move(kv=_kv(v_token=0)),
    lambda: _move(batch=_batch(sequences=1 << 24)), lambda: _move(kv=_kv(kv_heads=1 << 23, k_token=1 << 30, k_page=1 << 31, v_token=1 << 30, v_page=1 << 31, pages=1, page_size=1)),
    lambda: nj.nnjit_adjust_logits(None, 1, 10, 16, 10, 0, 16, 10, 0),
    lambda: _logits(rows=-1), lambda: _logits(rows=1 << 20), lambda: _logits(vocab=-1), lambda: _logits(vocab=1 << 30), lambda: _logits(x=None),
    lambda: _logits(y=None), lambda: _logits(ldx=-1), lambda: _logits(ldy=99), lambda: _logits(rows=1 << 19, vocab=1 << 20, ldy=1 << 20),
    lambda: _logits(_rules(history=16, history_len=-1)), lambda: _logits(_rules(history=16, history_len=3, ld_history=-1)),
    lambda: _logits(_rules(history_len=3)), lambda: _logits(_rules(bias_token=16)), lambda: _logits(_rules(bias_value=16)),
    lambda: _logits(_rules(bias_token=16, bias_value=16, bias_len=-1)), lambda: _logits(_rules(mask=16)), lambda: _logits(_rules(mask=16, mask_rows=1, ld_mask=-1)),
    lambda: _logits(_rules(mask_row=16)),
])
def test_refused(call):
    assert call() == nj.NNJIT_EINVAL
    assert nj.nnjit_last_error()


def test_dtypes_refused():
    for call in (lambda: _append(dtype=2), lambda: _append(norm=_norm(dtype=5)), lambda: _forward(xd=2), lambda: _forward(yd=-1), lambda: _forward(wd=3),
                 lambda: _grad(xd=2), lambda: _grad(dyd=2), lambda: _logits(xd=2), lambda: _logits(yd=7)):
        assert call() == nj.NNJIT_EDTYPE and nj.nnjit_last_error()


def test_nothing_to_do():
    """Empty calls do not touch the GPU."""
    assert _append(tokens=0, slots=None, k=None, v=None, q=None, out=None) == nj.NNJIT_OK
    assert _forward(tokens=0, x=None, y=None, pos=None) == nj.NNJIT_OK
    assert _forward(heads=0, x=None, y=None, w=None) == nj.NNJIT_OK
    assert _grad(heads=0, x=None, dy=None, dx=None, dw=None, w=None) == nj.NNJIT_OK
    assert _grad(heads=0, x=None, dy=None, dx=None, wh=32) == nj.NNJIT_OK
    assert _grad(tokens=0, x=None, dy=None, dx=None, dw=None) == nj.NNJIT_OK
    assert _tree(batch=_batch(tokens=0), mask=None, q=None, out=None) == nj.NNJIT_OK
    assert _tree(batch=_batch(max_q=0)) == nj.NNJIT_OK
    assert _move(n=0, path=None, accepted=None) == nj.NNJIT_OK
    assert _move(batch=_batch(sequences=0, q_start=None)) == nj.NNJIT_OK
    assert _move(batch=_batch(table_pages=0, page_table=None)) == nj.NNJIT_OK
    assert _logits(rows=0, x=None, y=None) == nj.NNJIT_OK
    assert _logits(vocab=0, x=None, y=None) == nj.NNJIT_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="a GPU is present")
def test_no_gpu_is_an_error():
    for call in (_step, _append, _forward, _grad, _tree, _move, _logits):
        assert call() == nj.NNJIT_EHIP


def test_binding_refuses():
    i32 = dict(dtype=torch.int32)
    with pytest.raises(ValueError, match="free_pages must"):
        nj.PagePool(torch.zeros(3), torch.zeros(1, **i32))
    with pytest.raises(ValueError, match="one GPU"):
        nj.PagePool(torch.zeros(3, **i32), torch.zeros(1, **i32))
    with pytest.raises(ValueError, match="page_table must"):
        nj.PagedStep(torch.zeros(3, **i32), 16, 4)
    with pytest.raises(ValueError, match="mask_words"):
        nj.PagedStep(torch.zeros(3, 2, **i32), 16, 4, mask_words=33)
    with pytest.raises(ValueError, match="kv_len must"):
        nj.PagedStep(torch.zeros(3, 2, **i32), 16, 4, kv_len=torch.zeros(2, **i32))
    with pytest.raises(ValueError, match="one GPU"):
        nj.PagedStep(torch.zeros(3, 2, **i32), 16, 4)
    with pytest.raises(ValueError, match="are needed"):
        nj.HeadNorm()
    with pytest.raises(TypeError, match="float32 or float16"):
        nj.HeadNorm(torch.zeros(8), torch.zeros(8).half())
    with pytest.raises(ValueError, match="one head_dim"):
        nj.HeadNorm(torch.zeros(8), torch.zeros(2, 4))
    with pytest.raises(ValueError, match="eps"):
        nj.HeadNorm(torch.zeros(8), eps=-1.0)
    with pytest.raises(ValueError, match="overlap"):
        nj.HeadNorm(torch.zeros(8).expand(3, 8))
    with pytest.raises(ValueError, match="no rule"):
        nj.LogitRules()
    with pytest.raises(ValueError, match="go together"):
        nj.LogitRules(bias_token=torch.zeros(2, 3, **i32))
    with pytest.raises(ValueError, match="need a history"):
        nj.LogitRules(presence=torch.zeros(2))
    with pytest.raises(ValueError, match="without mask"):
        nj.LogitRules(mask_row=torch.zeros(2, **i32))
    with pytest.raises(ValueError, match="different numbers"):
        nj.LogitRules(history=torch.zeros(2, 3, **i32), presence=torch.zeros(3))
    with pytest.raises(ValueError, match="repetition must"):
        nj.LogitRules(history=torch.zeros(2, 3, **i32), repetition=torch.zeros(2).half())
    with pytest.raises(ValueError, match="same shape"):
        nj.LogitRules(bias_token=torch.zeros(2, 3, **i32), bias_value=torch.zeros(2, 4))
    with pytest.raises(ValueError, match="one GPU"):
        nj.LogitRules(mask=torch.zeros(2, 3, **i32))
    with pytest.raises(ValueError, match="x must"):
        nj.norm_rotary(torch.zeros(2, 8), torch.zeros(8))
    with pytest.raises(ValueError, match="one GPU"):
        nj.norm_rotary(torch.zeros(2, 1, 8), torch.zeros(8))


def test_structs_are_as_in_c():
    """Sizes of the descriptions: eight bytes a field, ints and floats four."""
    assert ctypes.sizeof(nj.PagePoolDesc) == 32 and ctypes.sizeof(nj.HeadNormDesc) == 40
    assert ctypes.sizeof(nj.StepDesc) == 18 * 8 and ctypes.sizeof(nj.LogitRulesDesc) == 16 * 8


# ------------------------------------------------------------- which kernel a tree gets

@pytest.mark.parametrize("case", TREE_COVER, ids=cover_name)
def test_kernel_of_a_tree(case):
    dtype, news, keys, hq, hk, dim, rows, split, waves = case
    p = tree_plan(dtype, news, keys, hq, hk, dim)
    assert (p.tile_rows, p.splits > 1, p.waves) == (rows, split, waves)


def test_tree_cover_is_whole():
    have = {(c[0], c[5], c[6], c[7], c[8]) for c in TREE_COVER}
    for dtype in ("f16", "f32"):
        for dim in (64, 96, 128, 200):
            for rows in (16, 64, 128) if dim <= 128 else (16, 128):
                assert {(dtype, dim, rows, split, 4) for split in (False, True)} <= have
        assert (dtype, 64, 16, False, 8) in have and (dtype, 96, 16, False, 8) in have


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("window", [0, 1, 100, 5000])
def test_tree_plans_reach_every_key(dtype, window):
    """Tiles for all rows, splits over all keys that a row's window and the new tokens behind it span."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        n = int(rng.integers(1, 40))
        new = [int(2 ** rng.uniform(0, 7)) for _ in range(n)]
        keys = [a + int(2 ** rng.uniform(0, 16)) for a in new]
        hk, group, dim = int(rng.choice([1, 4, 8, 32])), int(rng.choice([1, 2, 3, 8])), int(rng.choice([64, 96, 128, 256]))
        p = tree_plan(dtype, new, keys, hk * group, hk, dim, window)
        assert p.row_tiles * p.tile_rows >= max(new) * group and p.split_keys % 32 == 0
        span = min(max(keys), window + max(new) + 31) if window else max(keys)
        assert p.splits * p.split_keys >= span and p.splits <= 256
        assert p.ws_floats == (p.splits * sum(new) * hk * group * ((dim + 3) // 4 * 4 + 2) if p.splits > 1 else 0)


# ------------------------------------------------------------- the plain forms

def test_plain_step_by_hand():
    """Sequence 0 grows into a second page, 1 shrinks from three pages to one, 2 is new and takes two."""
    table = [[4, 0, 0], [7, 8, 9], [0, 0, 0]]
    stack = [1, 2, 0, 0, 0, 0]
    got = plain_step([3, 11, 0], [3, 2, 0], [3, 1, 5], table, stack, 2, 6, 4, 10)
    # given back: 8, 9 on top of 1, 2; taken: 9 (sequence 0), 8 and 2 (sequence 2)
    assert table == [[4, 9, 0], [7, 8, 9], [8, 2, 0]] and got["count"] == 1 and stack[0] == 1
    assert got["q_start"] == [0, 3, 4, 9] and got["kv_len"] == [6, 3, 5] and got["status"] == [0, 0, 9, 1]
    assert got["slots"] == [19, 36, 37, 30, 32, 33, 34, 35, 8, -1]
    assert got["positions"] == [3, 4, 5, 2, 0, 1, 2, 3, 4, 0]


def test_plain_trees_by_hand():
    got = plain_step([5, 0], [5, 0], [4, 2], [[0, 1, 2], [0, 0, 0]], [3, 4, 0], 2, 3, 4, 7, parent=[-1, 0, 0, 1, 5, 0, 9], words=1)
    assert got["mask"] == [[1], [3], [5], [11], [1], [3], [0]]
    assert got["positions"] == [5, 6, 6, 7, 0, 1, 0]


def test_plain_refusals_by_hand():
    one = lambda held, keep, added, count=0, tokens=9, **kw: plain_step([held], [keep], [added], [[0, 1]], [0] * 4, count, 4, 4, tokens, **kw)["status"][0]  # noqa: E731
    assert one(4, 4, 0) == 0 and one(4, 4, 1) == MISSING and one(4, 5, 0) == LENGTHS and one(4, 4, 5) == LENGTHS
    assert one(4, 4, 3, count=1, tokens=2) == ROWS and one(4, 4, 0, count=5) == POOL and one(4, 0, 0, count=4) == POOL
    assert plain_step([0], [0], [33], [[0] * 9], [0] * 9, 9, 9, 4, 40, parent=[-1] * 40, words=1)["status"][0] == ROWS


def test_plain_norms_by_hand_and_by_differences():
    y, _ = normed(np.array([[3.0, 4.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(y, [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]])
    rng = np.random.default_rng(0)
    x, dy, w = rng.standard_normal((3, 2, 6)), rng.standard_normal((3, 2, 6)), rng.standard_normal(6)
    a = rng.uniform(0, 6, (3, 2))
    cos, sin = np.cos(a), np.sin(a)
    from tests.serving_util import turn
    for layout in ("half", "interleaved"):
        loss = lambda p, q: (turn(normed(p, q, 1e-3)[0], cos, sin, layout)[0] * dy).sum()  # noqa: E731
        dx, dw, _, _ = norm_grad(x, dy, w, 1e-3, cos, sin, layout)
        for at in np.ndindex(x.shape):
            d = np.zeros_like(x)
            d[at] = 1e-5
            assert abs((loss(x + d, w) - loss(x - d, w)) / 2e-5 - dx[at]) < 1e-8
        for i in range(6):
            d = np.zeros(6)
            d[i] = 1e-5
            assert abs((loss(x, w + d) - loss(x, w - d)) / 2e-5 - dw.sum(0)[i]) < 1e-8


def test_plain_trees_see_by_hand():
    B = Batch([3, 2], [5, 1], 1, 1, 2, 4, "f32")
    mask = np.array([[1], [3], [5], [3], [3]], dtype=np.uint32)
    seen = tree_seen(B, mask)
    assert seen[0].tolist() == [[True, True, True, False, False], [True, True, True, True, False], [True, True, True, False, True]]
    assert seen[1].tolist() == [[True], [True]]              # new token 0 of two has no place: one key, the second's
    seen = tree_seen(B, mask, window=2, positions=[2, 3, 9, 0, 0])
    assert [r[:2] for r in seen[0].tolist()] == [[False, True], [False, False], [False, False]]
    out, _ = attention_of(B, [np.zeros((3, 5), bool), np.ones((2, 1), bool)])
    assert (out[:3] == 0).all() and np.allclose(out[3:, 0], B.v[B.key_slots(1)[0]][0].double().numpy())


def test_plain_logits_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.5, 3.0]])
    got, _ = plain_logits(x, history=[[0, 1, 3, 3, 9, -1]], prompt=[1], repetition=[2.0], presence=[0.25], frequency=[0.5],
                          bias=[[(2, 1.0), (2, 4.0), (7, 1.0)]], allowed=np.array([[1, 1, 1, 1, 0]], dtype=bool))
    # 0 in the prompt only: 2 / 2; 1: -2 * 2 - 0.5 - 0.25; 2: the last bias; 3 twice: 0.25 - 1 - 0.25; 4: not allowed
    assert got[0].tolist() == [1.0, -4.75, 5.0, -1.0, -math.inf]
    assert words_of(np.array([[1] + [0] * 30 + [1, 1]], dtype=bool)).tolist() == [[1 - (1 << 31), 1]]


@pytest.mark.parametrize("mistake", ["taken", "ancestors", "prompt", "grad"])
def test_planted_mistakes_are_caught(mistake):
    """A plain form with a mistake differs from the right one on the inputs of these tests."""
    if mistake == "taken":            # pages from the bottom of the stack
        a, b = [[0, 0, 0]], [[0, 0, 0]]
        plain_step([0], [0], [5], a, [5, 6, 7], 3, 3, 4, 5)
        assert a != b and a[0][:2] == [7, 6]
    elif mistake == "ancestors":      # only the parent
        got = plain_step([0], [0], [3], [[0, 0]], [1], 1, 1, 4, 3, parent=[-1, 0, 1], words=1)
        assert got["mask"][2] == [7] != [6]
    elif mistake == "prompt":         # counts over the prompt as well
        full, _ = plain_logits(np.ones((1, 2)), history=[[0, 0]], prompt=[0], frequency=[1.0])
        part, _ = plain_logits(np.ones((1, 2)), history=[[0, 0]], prompt=[1], frequency=[1.0])
        assert full[0, 0] == -1 and part[0, 0] == 0
    else:                             # without the mean term
        rng = np.random.default_rng(0)
        x, dy = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
        dx, _, bound, _ = norm_grad(x, dy, np.ones(8), 0.0, None, None, "half")
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True))
        assert (np.abs(r * dy - dx) > bound).any()
