"""Host-side tests of the serving operators (no GPU): argument checks come
before any HIP call, the binding refuses operands that the entry points would
read or write out of bounds, and the plain forms that the GPU tests compare
with agree with small hand-worked cases."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2309_08978_amd as nj
from tests.serving_util import Batch, attention, turn


@pytest.fixture(scope="module", autouse=True)
def lib():
    return nj.load(build_if_missing=True)


def _kv(**kw):
    d = dict(k=16, v=32, k_page=1024, k_token=64, k_head=32, v_page=1024, v_token=64, v_head=32, pages=4, page_size=16, kv_heads=2,
             head_dim=32, dtype=1)
    d.update(kw)
    return nj.PagedKvDesc(**d)


def _batch(**kw):
    d = dict(sequences=1, tokens=1, q_start=16, kv_len=16, page_table=16, ld_table=4, table_pages=4, max_q=1, max_kv=64)
    d.update(kw)
    return nj.PagedBatchDesc(**d)


def _rot(**kw):
    d = dict(table=16, positions=10, rotary_dim=32, layout=0)
    d.update(kw)
    return nj.RotaryDesc(**d)


def _attend(kv=None, batch=None, heads=4, q=16, st=(128, 32), out=16, ost=(128, 32), scale=0.1, causal=1, window=0):
    return nj.nnjit_paged_attention(_kv() if kv is None else kv, _batch() if batch is None else batch, heads, q, *st, out, *ost, scale,
                                    causal, window)


def _append(kv=None, batch=None, rot=None, k=16, v=16, heads=4, q=16, out=16, ost=(128, 32), dtype=0):
    return nj.nnjit_kv_append(_kv() if kv is None else kv, _batch() if batch is None else batch, rot, k, 64, 32, v, 64, 32, heads, q,
                              128, 32, out, *ost, dtype)


def _rotary(rot=None, tokens=1, heads=2, dim=32, pos=16, x=16, xd=0, y=16, yst=(64, 32), yd=1):
    return nj.nnjit_rotary(_rot() if rot is None else rot, tokens, heads, dim, pos, x, 64, 32, xd, y, *yst, yd)


BAD_CACHES = [dict(dtype=2), dict(head_dim=0), dict(head_dim=257), dict(pages=0), dict(page_size=0), dict(kv_heads=0), dict(k=None),
              dict(v=None), dict(k_page=-1), dict(v_head=-1), dict(page_size=(1 << 30) + 1)]
BAD_BATCHES = [dict(sequences=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(table_pages=-1), dict(ld_table=3), dict(q_start=None),
               dict(kv_len=None), dict(page_table=None)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches(bad):
    want = nj.NNJIT_EDTYPE if "dtype" in bad else nj.NNJIT_EINVAL
    assert _attend(kv=_kv(**bad)) == want and nj.nnjit_last_error()
    assert _append(kv=_kv(**bad)) == want


@pytest.mark.parametrize("bad", BAD_BATCHES)
def test_bad_batches(bad):
    assert _attend(batch=_batch(**bad)) == nj.NNJIT_EINVAL and nj.nnjit_last_error()
    assert _append(batch=_batch(**bad)) == nj.NNJIT_EINVAL


@pytest.mark.parametrize("call", [
    lambda: nj.nnjit_paged_attention(None, _batch(), 4, 16, 128, 32, 16, 128, 32, 0.1),
    lambda: nj.nnjit_paged_attention(_kv(), None, 4, 16, 128, 32, 16, 128, 32, 0.1),
    lambda: _attend(heads=3), lambda: _attend(heads=0), lambda: _attend(q=None), lambda: _attend(out=None),
    lambda: _attend(st=(-1, 32)), lambda: _attend(ost=(128, 31)),
    lambda: _attend(batch=_batch(tokens=2), ost=(127, 32)),                        # rows of out overlap
    lambda: _attend(batch=_batch(tokens=2), ost=(32, 63)),                         # head-major: heads overlap
    lambda: _attend(scale=math.nan), lambda: _attend(scale=math.inf), lambda: _attend(window=-1),
    lambda: _attend(window=4, causal=0), lambda: _attend(batch=_batch(max_q=-1)), lambda: _attend(batch=_batch(max_kv=(1 << 30) + 1)),
    lambda: _attend(batch=_batch(tokens=(1 << 31) - 1, max_q=1 << 30), heads=4),   # 2^33 rows
    lambda: _attend(kv=_kv(kv_heads=1), batch=_batch(sequences=(1 << 31) - 1, tokens=100, max_q=100), heads=64),   # workgroups
    lambda: _append(k=None), lambda: _append(v=None), lambda: _append(q=None), lambda: _append(out=None), lambda: _append(heads=-1),
    lambda: _append(ost=(128, 16)), lambda: _append(rot=_rot(rotary_dim=34)), lambda: _append(rot=_rot(rotary_dim=7)),
    lambda: _append(rot=_rot(table=None)), lambda: _append(rot=_rot(layout=2)), lambda: _append(rot=_rot(positions=0)),
    lambda: _rotary(rot=_rot(rotary_dim=0)), lambda: _rotary(tokens=-1), lambda: _rotary(heads=-1), lambda: _rotary(dim=0),
    lambda: _rotary(pos=None), lambda: _rotary(x=None), lambda: _rotary(y=None), lambda: _rotary(tokens=2, yst=(32, 32)),
    lambda: nj.nnjit_rotary(None, 1, 1, 32, 16, 16, 32, 32, 0, 16, 32, 32, 0),
    lambda: nj.nnjit_rotary_fill(16, -1, 32, 1e4), lambda: nj.nnjit_rotary_fill(16, 4, 31, 1e4), lambda: nj.nnjit_rotary_fill(16, 4, 32, 1.0),
    lambda: nj.nnjit_rotary_fill(None, 4, 32, 1e4), lambda: nj.nnjit_rotary_fill(16, 4, 32, math.inf),
    lambda: nj.nnjit_rotary_fill(16, 4, 32, 1e4, nj.RotaryScaling(9, 1, 1, 2, 1, 1)),
    lambda: nj.nnjit_rotary_fill(16, 4, 32, 1e4, nj.RotaryScaling(nj.NNJIT_ROTARY_LINEAR, 0, 1, 2, 1, 1)),
    lambda: nj.nnjit_rotary_fill(16, 4, 32, 1e4, nj.RotaryScaling(nj.NNJIT_ROTARY_TURNS, 4, 2048, 1, 1, 1)),
])
def test_refused(call):
    assert call() == nj.NNJIT_EINVAL
    assert nj.nnjit_last_error()


@pytest.mark.parametrize("call", [
    lambda: _rotary(tokens=1 << 24), lambda: _append(batch=_batch(tokens=1 << 24)),                  # more threads than a launch holds
    lambda: nj.nnjit_rotary_fill(16, 1 << 28, 32, 1e4),
    lambda: _attend(kv=_kv(kv_heads=1), batch=_batch(sequences=1 << 24, tokens=1 << 24, max_q=1), heads=1),
    lambda: _append(kv=_kv(k_token=0)), lambda: _append(kv=_kv(v_token=63)), lambda: _append(kv=_kv(k_head=31)),   # slots overlap
    lambda: _append(kv=_kv(v_page=1023)), lambda: _append(kv=_kv(k_token=32, k_head=511)),
])
def test_refused_by_size_and_overlap(call):
    assert call() == nj.NNJIT_EINVAL
    assert nj.nnjit_last_error()


def test_dtypes_refused():
    assert _append(dtype=2) == nj.NNJIT_EDTYPE
    assert _rotary(xd=3) == nj.NNJIT_EDTYPE and _rotary(yd=-1) == nj.NNJIT_EDTYPE


def test_nothing_to_do():
    """Empty calls do not touch the GPU."""
    assert _attend(batch=_batch(tokens=0), q=None, out=None) == nj.NNJIT_OK
    assert _attend(batch=_batch(sequences=0, q_start=None)) == nj.NNJIT_OK
    assert _attend(batch=_batch(max_q=0)) == nj.NNJIT_OK
    assert _append(batch=_batch(tokens=0), k=None, v=None, q=None, out=None) == nj.NNJIT_OK
    assert _rotary(tokens=0, x=None, y=None, pos=None) == nj.NNJIT_OK
    assert _rotary(heads=0, x=None, y=None) == nj.NNJIT_OK
    assert nj.nnjit_rotary_fill(None, 0, 32, 1e4) == nj.NNJIT_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="a GPU is present")
def test_no_gpu_is_an_error():
    for call in (_attend, _append, _rotary, lambda: nj.nnjit_rotary_fill(16, 4, 32, 1e4)):
        assert call() == nj.NNJIT_EHIP


def test_binding_refuses():
    k = torch.zeros(4, 16, 2, 32)
    with pytest.raises(ValueError, match="one GPU"):
        nj.PagedCache(k, k.clone())
    with pytest.raises(ValueError, match="must be"):
        nj.PagedCache(k[0], k[0])
    with pytest.raises(TypeError, match="unsupported"):
        nj.PagedCache(k.double(), k.double())
    with pytest.raises(ValueError, match="but v is"):
        nj.PagedCache(k, k[:2])
    with pytest.raises(ValueError, match="overlap"):
        nj.PagedCache(k[:1].expand(4, 16, 2, 32), k)
    with pytest.raises(ValueError, match="unit stride"):
        nj.PagedCache(k.transpose(2, 3), k.transpose(2, 3))
    with pytest.raises(ValueError, match="layout"):
        nj.RotaryTable(torch.zeros(4, 8), "other")
    with pytest.raises(ValueError, match="table must"):
        nj.RotaryTable(torch.zeros(4, 7))
    i32 = dict(dtype=torch.int32)
    with pytest.raises(ValueError, match="q_start must"):
        nj.PagedBatch(torch.zeros(2, **i32), torch.zeros(2, **i32), torch.zeros(2, 3, **i32), tokens=2)
    with pytest.raises(ValueError, match="kv_len must"):
        nj.PagedBatch(torch.zeros(3, **i32), torch.zeros(2), torch.zeros(2, 3, **i32), tokens=2)
    with pytest.raises(ValueError, match="page_table must"):
        nj.PagedBatch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(1, 3, **i32), tokens=2)
    with pytest.raises(ValueError, match="one GPU"):
        nj.PagedBatch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 3, **i32), tokens=2)
    # head rows, on stand-ins for the handles
    class Handle:
        pass
    cache, batch = Handle(), Handle()
    cache.head_dim, cache.device_index, cache.dtype, cache.kv_heads = 32, 0, torch.float16, 2
    batch.tokens, batch.device_index = 3, 0
    q = torch.zeros(3, 4, 32, dtype=torch.float16)
    with pytest.raises(ValueError, match="q must be"):
        nj.paged_attention(q[:2], cache, batch)
    with pytest.raises(TypeError, match="q must be"):
        nj.paged_attention(q.float(), cache, batch)
    with pytest.raises(ValueError, match="one GPU"):
        nj.paged_attention(q, cache, batch)
    with pytest.raises(ValueError, match="unit stride"):
        nj.paged_attention(torch.zeros(3, 32, 4, dtype=torch.float16).transpose(1, 2), cache, batch)
    with pytest.raises(ValueError, match="k must be"):
        nj.kv_append(cache, batch, torch.zeros(3, 3, 32), torch.zeros(3, 2, 32))
    with pytest.raises(TypeError, match="unsupported"):
        nj.kv_append(cache, batch, torch.zeros(3, 2, 32).double(), torch.zeros(3, 2, 32))


def test_plain_forms_by_hand():
    """Two keys with logits 0 and ln 3: weights 1/4 and 3/4; a quarter turn swaps a pair."""
    B = Batch([1], [2], 1, 1, 2, 1, "f32")
    s = B.key_slots(0)
    B.q[0, 0] = torch.tensor([1.0, 0.0])
    B.k[s[0]], B.k[s[1]] = torch.tensor([[0.0, 5.0]]), torch.tensor([[math.log(3.0), -2.0]])
    B.v[s[0]], B.v[s[1]] = torch.tensor([[4.0, 0.0]]), torch.tensor([[0.0, 8.0]])
    out, _ = attention(B, scale=1.0)
    assert np.allclose(out[0, 0], [1.0, 6.0], atol=1e-6)
    out, _ = attention(B, scale=1.0, window=1)
    assert np.allclose(out[0, 0], [0.0, 8.0])
    x = np.arange(1.0, 6.0)[None, None]
    for layout, want in (("half", [-3, -4, 1, 2, 5]), ("interleaved", [-2, 1, -4, 3, 5])):
        y, _ = turn(x, np.zeros((1, 2)), np.ones((1, 2)), layout)
        assert np.allclose(y[0, 0], want)
