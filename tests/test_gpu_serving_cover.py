"""Every attention kernel -- each tile height, split and unsplit, four and
eight waves, pages of any size, any alignment -- element by element against the
formula in 64 bits."""
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.serving_cover import COVER, name, plan, strict
from tests.serving_util import DT, Batch

pytestmark = pytest.mark.gpu


def _attend(B, **kw):
    out = torch.full(B.q.shape, 7.0, dtype=DT[B.dtype], device="cuda")
    nj.paged_attention(B.dq, B.cache, B.batch, out, **kw)
    torch.cuda.synchronize()
    return out


def _batch(case, page, shift, seed):
    dtype, news, keys, hq, hk, dim = case[:6]
    return Batch(news, keys, hq, hk, dim, page, dtype, seed=seed, shift=shift)


@pytest.mark.parametrize("page,shift", [(16, 0), (5, 0), (16, 1)])
@pytest.mark.parametrize("case", COVER, ids=name)
def test_every_kernel(case, page, shift):
    B = _batch(case, page, shift, 51).device()
    got = _attend(B)
    strict(B, got)
    assert torch.equal(got, _attend(B))


@pytest.mark.parametrize("how", [dict(window=37), dict(causal=False), dict(scale=-0.2)], ids=str)
@pytest.mark.parametrize("case", COVER, ids=name)
def test_every_kernel_masked_otherwise(case, how):
    """A window, no mask, a negative scale (a window changes the plan of long contexts)."""
    B = _batch(case, 16, 0, 52).device()
    strict(B, _attend(B, **how), **how)


@pytest.mark.parametrize("window", [700, 1500])
@pytest.mark.parametrize("dtype,news,keys,hq,hk,dim", [("f16", [320, 1], [4020, 54], 16, 16, 64), ("f16", [320, 40], [2620, 900], 16, 4, 128),
                                                       ("f16", [500, 500], [3000, 1600], 8, 4, 96), ("f32", [320, 1], [4020, 54], 16, 16, 64),
                                                       ("f32", [320, 200], [2620, 300], 16, 4, 128)])
def test_windows_on_long_contexts(dtype, news, keys, hq, hk, dim, window):
    """Tall tiles whose window lies anywhere in a long context."""
    assert plan(dtype, news, keys, hq, hk, dim, window=window).tile_rows > 16
    B = Batch(news, keys, hq, hk, dim, 16, dtype, seed=53).device()
    strict(B, _attend(B, window=window), window=window)


@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("case,bad", [pytest.param(c, x, id=f"{name(c)}-{x}") for c in COVER if c[6] > 16 or c[8] == 8
                                      for x in [float("inf"), float("-inf"), float("nan")] + [3.395e38, 3.4e38] * (c[0] == "f32")])
def test_every_kernel_bad_values(case, bad, page):
    """Values that are not finite, or (fp32) close to the largest float or so close that bf16 cannot hold them, at late and early
    keys, in some dims; a query row that is not finite: each reaches the rows and dims that see it, and no other loses a bit."""
    B = _batch(case, page, 0, 54)
    hk, dim = B.hk, B.dim
    s = B.key_slots(0)
    B.v[s[-1]][0, 1] = bad
    B.v[s[len(s) * 2 // 3]][hk - 1, 2] = -bad
    B.v[s[len(s) // 3]][hk - 1, dim - 1] = bad
    B.v[s[0]][0, dim // 2] = bad
    if len(B.keys) > 1 and B.keys[1] > 0:
        B.v[B.key_slots(1)[0]][0, 0] = -bad
    if bad != bad:
        B.q[B.news[0] // 2, 0, 3] = bad
    strict(B.device(), _attend(B))
