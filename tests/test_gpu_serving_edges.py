"""Serving operators on the GPU at the ends of their arguments' ranges: against
the 64-bit forms, with bounds derived where they are used."""
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.serving_util import DT, Batch, check_attention

pytestmark = pytest.mark.gpu


def _attend(B, **kw):
    out = torch.full(B.q.shape, 7.0, dtype=DT[B.dtype], device="cuda")
    nj.paged_attention(B.dq, B.cache, B.batch, out, **kw)
    torch.cuda.synchronize()
    return out


# enough rows for tall tiles as well, some before the first key
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("news,keys,heads", [([12], [9], 2), ([3, 1], [2, 3000], 2), ([320] * 5, [317, 40, 9, 320, 500], 16)])
@pytest.mark.parametrize("window", [(1 << 31) - 1, 1 << 40])
def test_window_past_every_key(dtype, news, keys, heads, window):
    """A window larger than any context is no window, for sequences with fewer keys than new tokens too."""
    B = Batch(news, keys, heads, heads, 64, 16, dtype, seed=31).device()
    got = _attend(B, window=window)
    check_attention(B, got)
    assert torch.equal(got, _attend(B))
