"""Host-side tests of what the entry points of a step of drafted tokens take and
refuse beyond the plain cases (no GPU)."""
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.test_drafts_cpu import _arrays, _logits, _step


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
