"""Which attention kernel a shape gets (no GPU): the shapes that the GPU tests
cover the kernels with, and those of the measured cases, keep theirs."""
import numpy as np
import pytest
import torch

from tests.serving_cover import COVER, name, plan, strict
from tests.serving_util import Batch, attention


@pytest.mark.parametrize("case", COVER, ids=name)
def test_kernel_of_a_shape(case):
    dtype, news, keys, hq, hk, dim, rows, split, waves = case
    p = plan(dtype, news, keys, hq, hk, dim)
    assert (p.tile_rows, p.splits > 1, p.waves) == (rows, split, waves)
    assert p.row_tiles * p.tile_rows >= max(news) * (hq // hk) and p.splits * p.split_keys >= max(keys) and p.split_keys % 32 == 0


def test_cover_is_whole():
    """Every tile height that a class of head dims has, split and not; four and eight waves."""
    have = {(c[0], c[5], c[6], c[7], c[8]) for c in COVER}
    for dtype in ("f16", "f32"):
        for dim in (64, 96, 128, 200):
            for rows in (16, 64, 128) if dim <= 128 else (16, 128):
                for split in (False, True):
                    if (dtype, dim, rows, split) == ("f32", 128, 64, True) or (rows == 16 and dim in (96, 128)):
                        continue                              # no shape gets the first; the others differ in the single-token kernels only
                    assert (dtype, dim, rows, split, 4) in have, (dtype, dim, rows, split)
            if dim <= 128:
                assert (dtype, dim, 16, False, 8) in have, (dtype, dim)


@pytest.mark.parametrize("q_heads,kv_heads,sequences,new,keys,dim,dtype,want", [
    (32, 32, 1, 512, 2048, 128, "f16", (64, 2)), (12, 12, 6, 777, 777, 64, "f16", (128, 1)), (32, 8, 1, 2048, 16384, 128, "f16", (128, 1)),
    (16, 16, 4, 256, 256, 64, "f32", (64, 1))])
def test_kernel_of_long_prompts(q_heads, kv_heads, sequences, new, keys, dim, dtype, want):
    p = plan(dtype, [new] * sequences, [keys] * sequences, q_heads, kv_heads, dim, causal=dtype == "f16")
    assert (p.tile_rows, p.splits) == want


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_strict_check_itself(dtype):
    """The check takes the formula's values (rounded to the type) and refuses a mistake in one element of any size of dim."""
    B = Batch([5, 2], [9, 40], 4, 2, 8, 4, dtype, seed=1)
    B.v[B.key_slots(0)[6]][0, 1] = float("inf")
    B.v[B.key_slots(1)[0]][1] = 0.0
    B.v[B.key_slots(1)[1]][1, 3] = 60000.0
    ref, _ = attention(B)
    t = torch.from_numpy(ref).to(B.q.dtype)
    strict(B, t)
    for at in ((0, 3, 2), (5, 2, 4), (6, 0, 0)):
        bad = t.clone()
        bad[at] += 0.01 + abs(float(bad[at])) * 0.01
        with pytest.raises(AssertionError):
            strict(B, bad)
    bad = t.clone()
    bad[1, 0, 1], bad[4, 0, 1] = float("inf"), 0.0
    with pytest.raises(AssertionError):
        strict(B, bad)
    assert np.isfinite(ref).sum() < ref.size
