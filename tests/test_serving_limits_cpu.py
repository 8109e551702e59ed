"""Sizes that the serving kernels' index arithmetic does not reach are refused
before any HIP call."""
import pytest

import paper_2309_08978_amd as nj


@pytest.fixture(scope="module", autouse=True)
def lib():
    return nj.load(build_if_missing=True)


def _append(q_heads, kv_heads):
    kv = nj.PagedKvDesc(16, 32, 0, 0, 2, 0, 0, 2, 1, 1, kv_heads, 2, nj.NNJIT_F16)
    batch = nj.PagedBatchDesc(1, 1, 16, 16, 16, 1, 1, 1, 1)
    return nj.nnjit_kv_append(kv, batch, None, 16, 0, 2, 16, 0, 2, q_heads, 16, 0, 2, 16, 2 * q_heads, 2, nj.NNJIT_F16)


@pytest.mark.parametrize("heads", [(1 << 30) + 1, (1 << 31) - 1, 1 << 31])
def test_heads_of_a_turn(heads):
    """A thread that steps through 2^31 - 1 heads would pass the last one by an overflow."""
    rot = nj.RotaryDesc(16, 10, 2, nj.NNJIT_ROTARY_HALF)
    assert nj.nnjit_rotary(rot, 1, heads, 2, 16, 16, 0, 2, 1, 16, 2 * heads, 2, 1) == nj.NNJIT_EINVAL
    assert "heads" in nj.nnjit_last_error()


@pytest.mark.parametrize("q_heads,kv_heads", [(1 << 30, 1), ((1 << 31) - 5, 2), (0, (1 << 29) + 1), (-1, 1)])
def test_heads_of_an_append(q_heads, kv_heads):
    assert _append(q_heads, kv_heads) == nj.NNJIT_EINVAL
    assert "heads" in nj.nnjit_last_error()
