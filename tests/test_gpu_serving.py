"""The serving blocks called as a program may call them: with no rows, for one."""
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
def test_no_rows_first(make):
    serve = _block(make).serving()
    for n in (0, 3, 0):
        stream, h = _serve(serve, _rows(n, 1))
        assert stream.shape == h.shape == (n, 128)
