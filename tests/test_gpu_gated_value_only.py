"""The gated wrappers in a pass that nothing will differentiate: the value-only call's bits, without its derivatives' memory."""
import pytest
import torch

import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import autograd
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _case(rows, n_in, hidden, dtype):
    e = 2
    offsets = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device=DEV)
    x, w1, b1 = W.normal(rows * n_in, dtype, 1, 1.0, DEV).view(rows, n_in), W.normal(e * 2 * hidden * n_in, dtype, 2, n_in ** -0.5, DEV).view(e, 2, hidden, n_in), W.normal(e * 2 * hidden, dtype, 3, 0.3, DEV).view(e, 2, hidden)
    w2, b2 = W.normal(e * n_in * hidden, dtype, 4, hidden ** -0.5, DEV).view(e, n_in, hidden), W.normal(e * n_in, dtype, 5, 0.3, DEV).view(e, n_in)
    return x, w1, b1, w2, b2, offsets


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", [None, "gelu_erf", "gelu_tanh", "swish", "mish"])
@pytest.mark.parametrize("rows,n_in,hidden", [(3, 136, 264), (300, 96, 520)])
def test_value(rows, n_in, hidden, kind, dtype):
    x, w1, b1, w2, b2, offsets = _case(rows, n_in, hidden, dtype)
    y = torch.empty(rows, hidden, dtype=x.dtype, device=DEV)
    nfad.nfad_expert_gated_linear(kind, x, w1, b1, offsets, y)
    z = torch.empty_like(x)
    nfad.nfad_expert_linear(None, y, w2, b2, offsets, z)
    leaf = w1.clone().requires_grad_(True)
    with torch.no_grad():
        assert torch.equal(autograd.expert_gated_linear(x, leaf, b1, offsets, kind), y)
        assert torch.equal(autograd.expert_gated_feed_forward(x, leaf, b1, w2, b2, offsets, kind), z)
    trained = autograd.expert_gated_linear(x, leaf, b1, offsets, kind)
    assert trained.requires_grad
    # f by the chain that has f' too, or by the value's own: each within half a spacing of f (a relative eps / 2), then y's two roundings;
    # below the normal numbers spacings are smallest_normal eps, those of f times |u| (below 8: a normal value of deviation about one)
    eps = torch.finfo(x.dtype).eps
    assert bool(((trained - y).float().abs() <= 2 * eps * 1.01 * y.float().abs() + 9 * torch.finfo(x.dtype).smallest_normal * eps).all())


def test_memory():
    x, w1, b1, w2, b2, offsets = _case(4096, 64, 1024, "bf16")
    leaf = w1.clone().requires_grad_(True)
    torch.cuda.synchronize()
    y_bytes = 4096 * 1024 * 2
    with torch.no_grad():
        for call in (lambda: autograd.expert_gated_linear(x, leaf, b1, offsets), lambda: autograd.expert_gated_feed_forward(x, leaf, b1, w2, b2, offsets)):
            torch.cuda.reset_peak_memory_stats()
            before = torch.cuda.memory_allocated()
            y = call()
            # the layer's result, and the second layer's: far from the three of it that a differentiated pass has
            assert torch.cuda.max_memory_allocated() - before < 1.5 * y_bytes
            del y
