"""Where the tensor calls launch (no GPU): the operands' GPU, the stream that
was given, or torch's current one there."""
import contextlib

import pytest
import torch

import paper_2309_08978_amd as nj


@pytest.fixture
def gpus(monkeypatch):
    """Two pretended GPUs: current streams 100 and 101; GPU 0 is current."""
    seen = {"current": 0, "calls": []}

    class Cuda:
        @staticmethod
        @contextlib.contextmanager
        def device(index):
            old, seen["current"] = seen["current"], index
            try:
                yield
            finally:
                seen["current"] = old

    class Torch:
        cuda = Cuda

    nj._torch()
    monkeypatch.setattr(nj, "_torch_module", Torch)
    monkeypatch.setattr(nj, "_torch_stream", lambda index: 100 + index)
    monkeypatch.setattr(nj, "_torch_device", lambda: seen["current"])

    def entry(*args):
        seen["calls"].append((seen["current"], args))
        return seen.get("rc", 0)

    seen["entry"] = entry
    return seen


@pytest.mark.parametrize("index", [0, 1])
def test_current_stream_of_the_operands_gpu(gpus, index):
    nj._launch(gpus["entry"], index, None, 7, 8)
    assert gpus["calls"] == [(index, (7, 8, 100 + index))] and gpus["current"] == 0


@pytest.mark.parametrize("index", [0, 1])
def test_given_streams(gpus, index):
    class Stream:
        cuda_stream = 55
    nj._launch(gpus["entry"], index, Stream())
    nj._launch(gpus["entry"], index, 0)
    assert gpus["calls"] == [(index, (55,)), (index, (0,))] and gpus["current"] == 0


def test_errors_pass_and_leave_the_gpu(gpus):
    gpus["rc"] = nj.NNJIT_EINVAL
    with pytest.raises(nj.NnjitError):
        nj._launch(gpus["entry"], 1, None)
    assert gpus["current"] == 0


def test_empty_without_a_gpu():
    t = nj._empty((2, 3), torch.float16, torch.device("cpu"), None)
    assert t.shape == (2, 3) and t.dtype == torch.float16
    assert nj._empty((2,), torch.float32, torch.device("cpu"), 5).shape == (2,)
