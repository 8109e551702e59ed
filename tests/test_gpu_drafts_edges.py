"""The operators of a step of drafted tokens where their descriptions allow more
than a plain step does: batches with fewer rows than their starts say, handles
used in turn, the longest lists, calls of many rows."""
import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.drafts_util import attention_of, signed, tree_seen
from tests.serving_util import Batch

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# ------------------------------------------------------------ the step's arrays

def _chain(i, words):
    bits = (2 << min(i, 32 * words - 1)) - 1
    return [signed(bits >> 32 * w & 0xffffffff) for w in range(words)]


@pytest.mark.parametrize("words", [1, 2, 32])
@pytest.mark.parametrize("added", [[1, 1], [70, 3], [0, 33], [64, 31], [1200, 1]])
@pytest.mark.parametrize("in_place", [False, True])
def test_masks_of_a_step_without_trees(added, words, in_place):
    """A step that was a tree's and is filled without parents has the masks of chains, not its last step's; rows behind the last
    sequence, and all rows of a refused step, see nothing."""
    tokens, pages = 1300, 200
    held = _i32([0, 0])
    pool = nj.PagePool(torch.arange(pages, dtype=torch.int32, device="cuda"), _i32([pages]))
    step = nj.PagedStep(torch.zeros((2, 100), dtype=torch.int32, device="cuda"), 16, tokens, words, kv_len=held if in_place else None)
    nj.paged_step(step, pool, held, _i32([20, 32]), parent=_i32([-1] + [0] * (tokens - 1)))
    assert step.status.tolist()[0] == 0 and step.mask[19, 0].tolist() == signed(1 | 1 << 19)
    held = held if in_place else step.kv_len
    nj.paged_step(step, pool, held, _i32(added), keep=_i32([10, 10]))
    want = [_chain(i, words) for n in added for i in range(n)]
    assert step.status.tolist()[0] == 0
    assert step.mask.tolist() == want + [[0] * words] * (tokens - len(want))
    nj.paged_step(step, pool, step.kv_len, _i32([1 << 20, 1]))
    assert step.status.tolist()[0] != 0 and not step.mask.any()


def test_chain_masks_serve_tree_attention():
    """... so that a step of up to 32 mask_words new tokens a sequence may use either attention."""
    B = Batch([20, 1, 33], [120, 9, 33], 4, 2, 64, 16, "f32", seed=6).device()
    pages = int(B.table[B.table < 1 << 29].max()) + 1
    step = nj.PagedStep(B.batch.page_table.clone(), 16, B.tokens, 2)
    pool = nj.PagePool(torch.zeros(pages, dtype=torch.int32, device="cuda"), _i32([0]))
    nj.paged_step(step, pool, _i32(B.keys), _i32(B.news), keep=_i32([m - n for n, m in zip(B.news, B.keys)]))
    assert step.status.tolist()[0] == 0 and step.kv_len.tolist() == B.keys
    got = nj.tree_attention(B.dq, B.cache, step.batch(), step.mask)
    want, bound = attention_of(B, tree_seen(B, step.mask.cpu().numpy().view(np.uint32)))
    causal = [np.tril(np.ones((n, m), dtype=bool), m - n) for n, m in zip(B.news, B.keys)]
    assert all(np.array_equal(a, b) for a, b in zip(causal, tree_seen(B, step.mask.cpu().numpy().view(np.uint32))))
    assert (np.abs(got.double().cpu().numpy() - want) <= bound + 2.0 ** -24 * np.abs(want)).all()


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
