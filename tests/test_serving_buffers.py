"""Who owns the serving blocks' buffers: a captured call its own, every CUDA stream its own, for the largest number of rows seen (none among
them).  The rule alone, on host tensors with a stand-in for the current stream."""
import types

import pytest
import torch

from paper_2209_10778_b200 import feed_forward


@pytest.fixture(params=[feed_forward.ServingBlock, feed_forward.GatedServingBlock])
def serve(request, monkeypatch):
    block = object.__new__(request.param)
    block.q1, block.q2, block.dtype, block._kept, block._rows = torch.zeros(96, 32), torch.zeros(32, 96), torch.bfloat16, {}, 0
    block.now = types.SimpleNamespace(cuda_stream=0, capturing=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: block.now.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: block.now)
    monkeypatch.setattr(request.param, "_scratch_bytes", lambda self, rows, n: rows * n)
    return block


def _places(buffers):
    return {t.untyped_storage().data_ptr() for t in buffers}


def test_shapes(serve):
    for rows in (0, 3, 1, 7, 0):
        y1, u, h, scratch = serve._buffers(rows)
        assert y1.shape == (rows, 96) and u.shape == h.shape == (rows, 32) and scratch.numel() >= max(rows * 96, 16)


def test_kept_for_the_largest_number_of_rows(serve):
    first = _places(serve._buffers(5))
    assert _places(serve._buffers(4)) == _places(serve._buffers(5)) == first
    larger = _places(serve._buffers(6))
    assert larger != first and _places(serve._buffers(6)) == larger


def test_streams_do_not_share(serve):
    here = serve._buffers(5)
    serve.now.cuda_stream = 7
    there = serve._buffers(5)
    assert not _places(here) & _places(there)
    serve._buffers(50)
    serve.now.cuda_stream = 0
    assert _places(serve._buffers(5)) == _places(here)


def test_a_captured_call_has_its_own(serve):
    eager = serve._buffers(5)
    serve.now.capturing = True
    one, two = serve._buffers(5), serve._buffers(5)
    assert not _places(one) & _places(two) and not _places(one) & _places(eager) and not _places(two) & _places(eager)
    assert all(t.untyped_storage().data_ptr() not in _places(one) for kept in serve._kept.values() for t in kept[1])
    serve.now.capturing = False
    assert _places(serve._buffers(5)) == _places(eager)
