"""Calls without a stream run on torch's current one, in order with the work
that makes their operands and uses their results; outputs that a call on a
given stream allocates are that stream's."""
import pytest
import torch

import paper_2309_08978_amd as nj

pytestmark = pytest.mark.gpu


NAMES = ["matmul", "batched_matmul", "gemv_q4", "rotary", "kv_append", "paged_attention"]


def _calls():
    """name -> (inputs, call of them)"""
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *shape, dtype=torch.float16: torch.randn(shape, device="cuda", generator=g).to(dtype)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = nj.rotary_table(600, 64)
    cache = nj.PagedCache(r(40, 16, 2, 64), r(40, 16, 2, 64))
    batch = nj.PagedBatch(torch.tensor([0, 4], **i32), torch.tensor([600], **i32), torch.randperm(40, device="cuda").to(torch.int32)[None],
                          tokens=4, max_q=4, max_kv=600)
    pos = torch.arange(4, **i32)
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (96, 16), device="cuda", generator=g).to(torch.int32)
    scales = r(96, 2)
    return {
        "matmul": ([r(64, 96), r(96, 128)], nj.matmul),
        "batched_matmul": ([r(3, 64, 96), r(3, 96, 32)], nj.batched_matmul),
        "gemv_q4": ([r(128)], lambda x, **kw: nj.gemv_q4(x, words, scales, 64, 96, **kw)),
        "rotary": ([r(4, 8, 64)], lambda x, **kw: nj.rotary(x, pos, table, **kw)),
        "kv_append": ([r(4, 2, 64), r(4, 2, 64), r(4, 8, 64)],
                      lambda k, v, q, **kw: torch.cat([nj.kv_append(cache, batch, k, v, table, q, **kw).flatten(), cache.k.flatten(),
                                                       cache.v.flatten()])),
        "paged_attention": ([r(4, 8, 64)], lambda q, **kw: nj.paged_attention(q, cache, batch, **kw)),
    }


@pytest.mark.parametrize("name", NAMES)
def test_current_stream(name):
    """The inputs are written behind other work of the current stream, the result is read there."""
    inputs, call = _calls()[name]
    want = call(*inputs).clone()
    torch.cuda.synchronize()
    late = [torch.zeros_like(x) for x in inputs]
    call(*late)                                              # (a shape's first call may time kernels)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                        # about 10 ms
        for x, y in zip(late, inputs):
            x.copy_(y)
        got = call(*late)
        got = got.clone()
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("name", NAMES)
def test_captured_without_a_stream(name):
    """Inside a capture the current stream is the captured one."""
    inputs, call = _calls()[name]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = call(*inputs).clone()                         # the stream's scratch
    torch.cuda.synchronize()
    held = [x.clone() for x in inputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = call(*held)
    for rep in range(3):
        got.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), rep


@pytest.mark.parametrize("as_handle", [False, True])
def test_outputs_belong_to_the_given_stream(as_handle):
    """Memory that the current stream still writes is not handed to a call on another stream."""
    (q,), call = _calls()["paged_attention"]
    want = call(q).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    given = side.cuda_stream if as_handle else side
    for _ in range(3):
        busy = torch.empty_like(q)
        torch.cuda._sleep(4_000_000)
        busy.fill_(3.0)                                      # queued behind the sleep, on the current stream
        del busy                                             # its block may be reused there at once
        got = call(q, stream=given)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    assert torch.equal(call(q, stream=0), want)
