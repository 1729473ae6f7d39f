"""The gated wrappers ask for the derivatives only where a gradient can be asked for.  What they ask of the library, on host tensors."""
import pytest
import torch

from paper_2209_10778_b200 import autograd, block


@pytest.fixture
def asked(monkeypatch):
    calls = []
    monkeypatch.setattr(block, "nfad_expert_gated_linear", lambda kind, x, w, bias, offsets, y, partials=None: calls.append(partials is not None))
    monkeypatch.setattr(block, "nfad_expert_linear", lambda *a: None)
    return calls


@pytest.mark.parametrize("layers", [1, 2])
def test_derivatives_only_for_gradients(asked, layers):
    x, w1, b1, w2, b2 = torch.zeros(4, 16), torch.zeros(2, 2, 8, 16), torch.zeros(2, 2, 8), torch.zeros(2, 16, 8), torch.zeros(2, 16)
    offsets = torch.tensor([0, 2, 4], dtype=torch.int32)

    def call(x, w1, b1, w2, b2):
        if layers == 1:
            return autograd.expert_gated_linear(x, w1, b1, offsets)
        return autograd.expert_gated_feed_forward(x, w1, b1, w2, b2, offsets)

    tensors = (x, w1, b1, w2, b2)
    assert not call(*tensors).requires_grad
    assert not call(x, w1, None, w2, None).requires_grad
    every = [t.clone().requires_grad_(True) for t in tensors]
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            assert call(*every).shape == (4, 8 if layers == 1 else 16)
    assert asked == [False] * 4
    del asked[:]
    for i in range(3 if layers == 1 else 5):
        assert call(*(t.clone().requires_grad_(i == j) for j, t in enumerate(tensors))).requires_grad
    assert asked and all(asked)
