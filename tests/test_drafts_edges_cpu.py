"""Host-side tests of what the entry points of a step of drafted tokens take and
refuse beyond the plain cases (no GPU)."""
import inspect
import textwrap

import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests import drafts_util
from tests.drafts_util import LOGIT_COVER, logit_plan
from tests.test_drafts_cpu import _arrays, _grad, _logits, _step


@pytest.fixture(scope="module", autouse=True)
def lib():
    return nj.load(build_if_missing=True)


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a GPU is present: the pointers are none")


def test_masks_without_trees_are_checked():
    """A mask that a step without parents fills has to hold its words."""
    for bad in (dict(mask_words=33, ld_mask=40), dict(mask_words=-1, ld_mask=4), dict(mask_words=3, ld_mask=2)):
        assert _step(arrays=_arrays(mask=16, **bad)) == nj.NNJIT_EINVAL and nj.nnjit_last_error()


@no_gpu
def test_no_masks_without_words():
    assert _step(arrays=_arrays(mask=16)) == nj.NNJIT_EHIP
    assert _step(arrays=_arrays(mask_words=99)) == nj.NNJIT_EHIP


# ------------------------------------------------------------- memory that is read and written

@pytest.mark.parametrize("arrays", [
    dict(held=1000, kv_len=1004), dict(held=1004, kv_len=1000), dict(keep=1000, kv_len=1012), dict(keep=1012, kv_len=1000), dict(added=1000, kv_len=1000),
    dict(added=1000, kv_len=1012), dict(q_start=1000, kv_len=1016), dict(q_start=1016, kv_len=1004), dict(held=1000, keep=1004, kv_len=1000),
    dict(held=1000, keep=1004, kv_len=1004),
])
def test_lengths_that_overlap_in_part(arrays):
    """kv_len may be held or keep as a whole (a second launch replaces them); it would race with a part of any length."""
    a = dict(held=4000, keep=5000, added=6000, q_start=7000, kv_len=8000, sequences=4)
    a.update(arrays)
    assert _step(arrays=_arrays(**a)) == nj.NNJIT_EINVAL and "kv_len" in nj.nnjit_last_error()


@no_gpu
@pytest.mark.parametrize("arrays", [dict(held=1000, kv_len=1000), dict(keep=1000, kv_len=1000), dict(held=1000, keep=1000, kv_len=1000),
                                    dict(held=1000, kv_len=1016), dict(held=1016, kv_len=1000), dict(q_start=1000, kv_len=1020),
                                    dict(added=1016, kv_len=1000)])
def test_lengths_in_place_or_apart(arrays):
    a = dict(held=4000, keep=5000, added=6000, q_start=7000, kv_len=8000, sequences=4)
    a.update(arrays)
    assert _step(arrays=_arrays(**a)) == nj.NNJIT_EHIP


# rows 4, vocab 100 of fp32 (400 bytes) or fp16 (200), from address 100000 on
OVERLAPPING = [
    dict(y=100000, yd=1),                                   # another type
    dict(y=100000, ldy=104), dict(y=100000, ldx=200),       # another stride
    dict(y=100004), dict(y=99996), dict(y=100400), dict(y=98800 + 4), dict(y=101596),
    dict(x=100000, ldx=0, y=100000), dict(x=100000, ldx=0, y=99000),            # one row for all
    dict(xd=1, yd=1, ldx=150, ldy=150, y=100198), dict(ldx=200, ldy=200, y=100396), dict(ldx=200, ldy=300, y=100400),
]
FINE = [
    dict(y=100000), dict(y=101600), dict(y=98400), dict(y=101600, yd=1), dict(y=99200, yd=1), dict(rows=1, y=100000, ldx=7, ldy=500),
    dict(ldx=200, ldy=200, y=100400), dict(ldx=200, ldy=200, y=99600), dict(ldx=200, ldy=400, y=100400, yd=1), dict(ldx=400, ldy=200, xd=1, y=100200),
    dict(x=100000, ldx=0, y=100400), dict(x=100000, ldx=0, y=98400),
]


@pytest.mark.parametrize("call", OVERLAPPING)
def test_logits_that_overlap(call):
    assert _logits(**{**dict(rows=4, x=100000), **call}) == nj.NNJIT_EINVAL and "overlap" in nj.nnjit_last_error()


@no_gpu
@pytest.mark.parametrize("call", FINE)
def test_logits_in_place_or_apart(call):
    assert _logits(**{**dict(rows=4, x=100000), **call}) == nj.NNJIT_EHIP


# 3 tokens of 2 heads of 32 dims; x (64, 32) floats apart from address 100000 on, dy and dx by default far away
@pytest.mark.parametrize("call", [
    dict(dx=100000, dxst=(96, 32)), dict(dx=100000, dxst=(32, 96)), dict(dx=100004), dict(dx=100128), dict(dx=99900),
    dict(dy=200000, dx=200000, dyd=1), dict(dy=200000, dx=200128), dict(dy=200000, dyst=(0, 0), dx=200000),
    dict(dy=200000, dyst=(64, 0), dx=200000), dict(dy=200124, dyst=(128, 32), dx=200000, dxst=(128, 96)),
    dict(dy=200132, dyst=(128, 32), dx=200000, dxst=(128, 96)), dict(dy=200512, dyst=(256, 32), dyd=1, dx=200000, dxst=(128, 32), x=400000),
])
def test_gradients_that_overlap(call):
    assert _grad(**{**dict(tokens=3, x=100000, dy=200000, dx=300000), **call}) == nj.NNJIT_EINVAL and "overlap" in nj.nnjit_last_error()


@no_gpu
@pytest.mark.parametrize("call", [
    dict(), dict(dx=100000), dict(dx=200000), dict(dy=100000), dict(dx=100768), dict(dx=99232), dict(dy=200000, dyd=1, dx=200384),
    dict(dy=200128, dyst=(128, 64), dx=200000, dxst=(128, 64)),                 # sides of each head
    dict(dy=200256, dyst=(128, 32), dx=200000, dxst=(128, 32)),                 # heads of each token
    dict(dy=200000, dyst=(32, 200), dx=200384, dxst=(32, 200)),                 # tokens of each head
    dict(dy=200128, dyst=(128, 32), dx=200000, dxst=(128, 96)),                 # heads between the heads
    dict(dy=200256, dyst=(256, 32), dyd=1, dx=200000, dxst=(128, 32), x=400000),    # a half row of fp16 behind a row of fp32
])
def test_gradients_in_place_or_apart(call):
    assert _grad(**{**dict(tokens=3, x=100000, dy=200000, dx=300000), **call}) == nj.NNJIT_EHIP


@no_gpu
def test_overlaps_are_those_of_the_bytes():
    """Random strides: what is refused or not, against the sets of bytes; in place only with the same strides and type."""
    rng = np.random.default_rng(0)
    seen = {True: 0, False: 0, "careful": 0}
    for _ in range(4000):
        dim, heads, tokens = int(rng.integers(1, 5)), int(rng.integers(1, 4)), int(rng.integers(1, 4))

        def rows(most):
            if rng.random() < 0.5:
                head = dim + int(rng.integers(0, 4))
                return (heads - 1) * head + dim + int(rng.integers(0, most)), head
            token = dim + int(rng.integers(0, 4))
            return token, (tokens - 1) * token + dim + int(rng.integers(0, most))

        dxst, half = rows(12), int(rng.integers(0, 2))
        dyst = tuple(dxst) if rng.random() < 0.6 else rows(12)
        if half and rng.random() < 0.6:
            dyst = (2 * dxst[0], 2 * dxst[1])
        dx = 1 << 20
        dy = dx + 4 * int(rng.integers(-30, 30)) + 2 * half * int(rng.integers(0, 2))

        def bytes_of(p, st, e):
            return {p + e * (t * st[0] + h * st[1]) + i for t in range(tokens) for h in range(heads) for i in range(dim * e)}

        meet = bool(bytes_of(dx, dxst, 4) & bytes_of(dy, dyst, 2 if half else 4))
        same = dx == dy and not half and (tokens == 1 or dxst[0] == dyst[0]) and (heads == 1 or dxst[1] == dyst[1])
        rc = _grad(tokens=tokens, heads=heads, dim=dim, x=1 << 30, dy=dy, dyst=dyst, dyd=half, dx=dx, dxst=dxst)
        refused = rc == nj.NNJIT_EINVAL and "overlap them otherwise" in nj.nnjit_last_error()
        assert refused or rc == nj.NNJIT_EHIP
        if meet and not same:
            assert refused, (tokens, heads, dim, dxst, dyst, half, dy - dx)
        seen[refused] += 1
        seen["careful"] += refused and not meet
    assert seen[True] > 500 and seen[False] > 500 and seen["careful"] < 0.1 * seen[True], seen


# ------------------------------------------------------------- which kernel a row of logits gets

@pytest.mark.parametrize("case", LOGIT_COVER, ids=str)
def test_kernel_of_logits(case):
    rows, vocab, history, threads, quads, narrow = case
    p = logit_plan(rows, vocab, history)
    assert (p.threads, p.quads, bool(p.narrow)) == (threads, quads, narrow)


def test_logit_cover_is_whole():
    """All that the rule of choice ever gives is among the covered cases."""
    rng = np.random.default_rng(0)
    have = {c[3:] for c in LOGIT_COVER}
    for _ in range(20000):
        p = logit_plan(int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 18)), int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 18)))
        assert (p.threads, p.quads, bool(p.narrow)) in have
    assert len(have) == 6


def test_counts_and_entries_fit_their_words():
    """One word a token: 15 bits of count above 16 of entry, the last bit for the prompt."""
    assert logit_plan(64, 128000, (1 << 15) - 1, (1 << 16) - 1).narrow
    assert not logit_plan(64, 128000, 1 << 15, 60).narrow and not logit_plan(64, 128000, 100, 1 << 16).narrow


# ------------------------------------------------------------- mistakes planted in the plain forms

def _mistaken(module, name, right, wrong):
    """The function with a mistake in its source."""
    source = textwrap.dedent(inspect.getsource(getattr(module, name)))
    assert source.count(right) == 1
    space = dict(vars(module))
    exec(compile(source.replace(right, wrong), name, "exec"), space)
    return space[name]


@pytest.mark.parametrize("right,wrong", [
    ("free.pop()", "free.pop(0)"),                                                   # pages from the bottom of the stack
    ("for b, c in back]", "for b, c in back[::-1]]"),                                # pages given back in another order
    ("(seen[p] if 0 <= p < i else set())", "({p} if 0 <= p < i else set())"),        # the parent only
    ("0 <= p < i", "0 <= p"),                                                        # parents that are no earlier node
    ("keep[b] + len(mine) - 1", "keep[b] + i"),                                      # positions by index, not by depth
    ("place = keep[b] + i", "place = held[b] + i"),                                  # places behind what was held
    ("c in range(need(keep[b] + added[b]), need(held[b]))", "c in range(need(keep[b]), need(held[b]))"),
    ("need = lambda t: -(-t // page)", "need = lambda t: t // page + 1"),
])
def test_mistakes_in_a_step_show(right, wrong):
    """On one of the batches of requests, some array differs (or the step falls over a page that is not there)."""
    bad = _mistaken(drafts_util, "plain_step", right, wrong)
    for seed in range(5):
        rng = np.random.default_rng(seed)
        n, page = 6, 4
        held = [int(x) for x in rng.integers(0, 40, n)]
        keep = [int(rng.integers(0, h + 1)) for h in held]
        added = [int(x) for x in rng.integers(0, 20, n)]
        parent = [int(rng.integers(-1, 12)) for _ in range(sum(added))]
        ids = rng.permutation(200).tolist()
        table = [[ids.pop() for _ in range(-(-h // page))] for h in held]
        table = [row + [0] * (20 - len(row)) for row in table]
        made = []
        for f in (drafts_util.plain_step, bad):
            t, s = [list(r) for r in table], ids[:60] + [0] * 60
            try:
                made.append((f(held, keep, added, t, s, 60, 120, page, sum(added), parent, 1), t, s))
            except IndexError:
                made.append(None)
        if made[0] != made[1]:
            return
    raise AssertionError("no batch shows it")


@pytest.mark.parametrize("right,wrong", [
    ("tokens[max(0, prompt[r]) if prompt is not None else 0:]", "tokens"),           # counts over the prompt as well
    ("z[r, t] > 0 else", "z[r, t] < 0 else"),                                        # penalty the wrong way round
    ("seen = {t for t in tokens", "seen = {t for t in made"),                        # the prompt's tokens not penalised
    ("for t, v in bias[r] if", "for t, v in bias[r][::-1] if"),                      # the first bias, not the last
    ("z[r, t] - f * c - p", "z[r, t] - f * c - p * c"),                              # presence by count
    ("min(max(length[r], 0), len(history[r]))", "len(history[r])"),                  # lengths not looked at
    ("np.where(allowed, z, -math.inf)", "z"),
])
def test_mistakes_in_logits_show(right, wrong):
    rng = np.random.default_rng(0)
    rows, vocab = 3, 12
    kw = dict(history=rng.integers(0, vocab, (rows, 9)).tolist(), length=[9, 5, 7], prompt=[3, 2, 4], repetition=[1.3] * 3, presence=[0.4] * 3,
              frequency=[0.2] * 3, bias=[[(1, 0.5), (1, -0.5), (4, 2.0)]] * 3, allowed=rng.random((rows, vocab)) < 0.7)
    x = rng.standard_normal((rows, vocab))
    want, bound = drafts_util.plain_logits(x, **kw)
    got, _ = _mistaken(drafts_util, "plain_logits", right, wrong)(x, **kw)
    fine = np.isfinite(want) & np.isfinite(got)
    assert (np.isfinite(want) != np.isfinite(got)).any() or (np.abs(got[fine] - want[fine]) > bound[fine]).any()


@pytest.mark.parametrize("right,wrong", [
    ("r * (h - u * m)", "r * h"),                                                    # without the mean term
    ("turn(dy, cos, sin, layout, -1.0)", "turn(dy, cos, sin, layout, 1.0)"),         # turned on, not back
    ("dw = (g * u).sum(0)", "dw = (h * u).sum(0)"),                                  # the weight's gradient times the weight
    ("dw = (g * u).sum(0)", "dw = (g * x).sum(0)"),                                  # ... of rows that are not normed
    ("dw = (g * u).sum(0)", "dw = (g * u)[:-1].sum(0)"),                             # ... without the last token
    ("g * weight\n", "g\n"),
])
def test_mistakes_in_gradients_show(right, wrong):
    rng = np.random.default_rng(0)
    x, dy, w, a = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8)), rng.standard_normal(8), rng.uniform(0, 6, (3, 4))
    dx, dw, bound, dwb = drafts_util.norm_grad(x, dy, w, 1e-5, np.cos(a), np.sin(a), "half")
    bad_dx, bad_dw, _, _ = _mistaken(drafts_util, "norm_grad", right, wrong)(x, dy, w, 1e-5, np.cos(a), np.sin(a), "half")
    assert (np.abs(bad_dx - dx) > bound).any() or (np.abs(bad_dw - dw) > dwb).any()
