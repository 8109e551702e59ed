"""The operators of a step of drafted tokens where their descriptions allow more
than a plain step does: batches with fewer rows than their starts say, handles
used in turn, the longest lists, calls of many rows."""
import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.serving_util import Batch

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


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
