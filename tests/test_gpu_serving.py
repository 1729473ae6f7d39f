"""The serving blocks called as a program may call them: captured calls beside larger ones, two streams at once, no rows; and the copy
that they are of the block."""
import pytest
import torch

from paper_2209_10778_b200 import feed_forward
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
BLOCKS = [feed_forward.FeedForwardBlock, feed_forward.GatedFeedForwardBlock]


def _block(make, width=128, hidden=384):
    torch.manual_seed(0)
    return make(width, hidden, 1).eval()


def _rows(n, seed, width=128):
    return W.normal(n * width, "bf16", seed, 1.0, DEV).view(n, width)


def _serve(serve, x):
    stream = x.clone()
    h = serve(stream, x)
    return stream, h.clone()


@pytest.mark.parametrize("make", BLOCKS)
def test_captured_calls_outlive_larger_ones(make):
    serve = _block(make).serving()
    xs = [_rows(8, 1), _rows(8, 2)]
    want = [_serve(serve, x) for x in xs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in xs:
        stream = torch.empty_like(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            stream.copy_(x)
            outs.append((stream, serve(stream, x)))
        graphs.append(g)
    large = _serve(serve, _rows(300, 3))                              # keeps larger buffers from now on
    noise = [torch.full((1 << 16,), float("nan"), device=DEV) for _ in range(64)]      # whatever was given back has another owner now
    torch.cuda.synchronize()
    for _ in range(2):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w))
    assert all(torch.isnan(t).all() for t in noise)
    assert all(torch.equal(a, b) for a, b in zip(_serve(serve, _rows(300, 3)), large))


@pytest.mark.parametrize("make", BLOCKS)
def test_two_streams_at_once(make):
    serve = _block(make).serving()
    xs = [_rows(200, 1), _rows(70, 2)]
    want = [_serve(serve, x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    out = _serve(serve, x)
                got.append(out)
        torch.cuda.synchronize()
        for out, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w))


@pytest.mark.parametrize("make", BLOCKS)
def test_no_rows_first(make):
    serve = _block(make).serving()
    for n in (0, 3, 0):
        stream, h = _serve(serve, _rows(n, 1))
        assert stream.shape == h.shape == (n, 128)


@pytest.mark.parametrize("make", BLOCKS)
def test_the_copy_does_not_follow_the_block(make):
    block = _block(make)
    with torch.no_grad():
        for b in (block.b1, block.b2):
            b.normal_()
    serve, x = block.serving(), _rows(9, 1)
    everything = torch.tensor([0, 9], dtype=torch.int32, device=DEV)
    with torch.no_grad():
        want, own = _serve(serve, x), block(x, x, everything)
        for p in block.parameters():
            before = p.clone()
            p.mul_(-0.5).add_(0.25)
            assert not torch.equal(p, before)
            assert all(torch.equal(a, b) for a, b in zip(_serve(serve, x), want))
        assert not any(torch.equal(a, b) for a, b in zip(block(x, x, everything), own))
