"""Host-side tests of what the entry points of a step of drafted tokens take and
refuse beyond the plain cases (no GPU)."""
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.test_drafts_cpu import _arrays, _step


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
