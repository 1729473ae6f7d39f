"""The gated feed-forward block: autograd wrappers of the gated layer, of dropout and of the activation with dropout against torch's own autograd in
64 bits, the block trained for some steps with its mask, and served in 8-bit floating point."""
import subprocess
import sys

import pytest
import torch

import dropout_plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import autograd, feed_forward
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _act(z, kind):
    f = torch.nn.functional
    return {"gelu_erf": lambda: f.gelu(z), "gelu_tanh": lambda: f.gelu(z, approximate="tanh"), "swish": lambda: f.silu(z), "mish": lambda: f.mish(z),
            None: lambda: z}[kind]()


def _close(got, want, steps, what):
    """16-bit results that passed through `steps` roundings of 2^-9 of their size: as a whole (2-norm) within steps times that."""
    rel = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
    assert rel <= steps * 2.0 ** -9, (what, rel)


def _leaves(tensors):
    return [t.clone().requires_grad_(True) for t in tensors], [t.double().requires_grad_(True) for t in tensors]


def _gated_case():
    off = [0, 30, 30, 65, 100]
    offsets = torch.tensor(off, dtype=torch.int32, device=DEV)
    x, w1, b1 = W.normal(100 * 64, "bf16", 1, 1.0, DEV).view(100, 64), W.normal(8 * 96 * 64, "bf16", 2, 0.125, DEV).view(4, 2, 96, 64), W.normal(8 * 96, "bf16", 3, 0.3, DEV).view(4, 2, 96)
    w2, b2 = W.normal(4 * 64 * 96, "bf16", 4, 0.1, DEV).view(4, 64, 96), W.normal(4 * 64, "bf16", 5, 0.3, DEV).view(4, 64)
    return off, offsets, (x, w1, b1, w2, b2), W.normal(100 * 64, "bf16", 6, 1.0, DEV).view(100, 64)


def _plain(refs, off, kind):
    x, w1, b1, w2, b2 = refs
    parts = []
    for e in range(4):
        a, u = (x[off[e]:off[e + 1]] @ w1[e, j].t() + b1[e, j] for j in (0, 1))
        parts.append((_act(a, kind) * u) @ w2[e].t() + b2[e])
    return torch.cat(parts)


@pytest.mark.parametrize("kind", ["gelu_erf", "gelu_tanh", "swish", "mish", None])
def test_gated_wrappers_against_torch(kind):
    off, offsets, tensors, g = _gated_case()
    leaves, refs = _leaves(tensors)
    y = autograd.expert_gated_feed_forward(*leaves, offsets, kind)
    y.backward(g)
    y64 = _plain(refs, off, kind)
    y64.backward(g.double())
    # roundings on the longest way: y1, y; back: the derivatives, grad_z, the result, and those of the products' other operand
    _close(y, y64.detach(), 3, "y")
    for name, a, b in zip(("x", "w1", "b1", "w2", "b2"), leaves, refs):
        _close(a.grad, b.grad, 6, name)
    more, _ = _leaves(tensors)
    y2 = autograd.expert_linear(autograd.expert_gated_linear(more[0], more[1], more[2], offsets, kind), more[3], more[4], offsets)
    y2.backward(g)
    assert torch.equal(y, y2)
    for name, a, b in zip(("x", "w1", "b1", "w2", "b2"), more, refs):
        _close(a.grad, b.grad, 7, name)


@pytest.mark.parametrize("frozen", [(0,), (1,), (2,), (3,), (4,), (0, 1, 2), (1, 2, 3, 4), (0, 3)])
def test_frozen_leaves(frozen):
    off, offsets, tensors, g = _gated_case()
    every, _ = _leaves(tensors)
    some = [t.clone().requires_grad_(i not in frozen) for i, t in enumerate(tensors)]
    for leaves in (every, some):
        autograd.expert_gated_feed_forward(*leaves, offsets, "swish").backward(g)
    for i in range(5):
        assert some[i].grad is None if i in frozen else torch.equal(some[i].grad, every[i].grad)
    x, w, b = (t.clone().requires_grad_(i not in frozen) for i, t in enumerate(tensors[:3]))
    if len(set(frozen) & {0, 1, 2}) < 3:
        autograd.expert_gated_linear(x, w, b, offsets).sum().backward()
        assert [t.grad is None for t in (x, w, b)] == [i in frozen for i in range(3)]


def test_without_biases_strided_inputs_and_no_second_derivative():
    _, offsets, (x, w1, b1, w2, b2), g = _gated_case()
    wide = torch.cat([x, x], 1)
    leaf = wide.clone().requires_grad_(True)
    y = autograd.expert_gated_feed_forward(leaf[:, ::2], w1, None, w2, None, offsets, "swish")
    want = autograd.expert_gated_feed_forward(wide[:, ::2].contiguous(), w1, None, w2, None, offsets, "swish")
    assert torch.equal(y, want)
    (gx,) = torch.autograd.grad(y, leaf, g.t().contiguous().t(), create_graph=True)
    assert not gx[:, 1::2].any()
    with pytest.raises(RuntimeError):
        torch.autograd.grad(gx.sum(), leaf)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_dropout_wrapper(dtype):
    n, shape = 3000, (3, 1000)
    x, r, g = (W.normal(n, dtype, i, 1.0, DEV).view(shape) for i in range(3))
    drop = nfad.Dropout(0.3, 77, 5)
    keep, scale = dropout_plain.mask(n, 0.3, 77, 5)
    keep = keep.view(shape).to(DEV)
    x1, r1 = x.clone().requires_grad_(True), r.clone().requires_grad_(True)
    y = autograd.dropout(x1, drop, r1)
    y.backward(g)
    want = torch.where(keep, g.double() * scale, torch.zeros_like(g, dtype=torch.float64))
    # the scale and the product: two fp32 roundings, and the store's
    assert torch.all((x1.grad.double() - want).abs() <= (torch.finfo(x.dtype).eps / 2 + 2.0 ** -23) * want.abs() * 1.01)
    assert torch.equal(x1.grad != 0, keep & (g != 0)) and torch.equal(r1.grad, g)
    assert torch.equal((y - r).abs() > 0, keep & (y != r))
    x2 = x.clone().requires_grad_(True)
    autograd.dropout(x2, drop).backward(g)
    assert torch.equal(x2.grad, x1.grad)
    r2 = r.clone().requires_grad_(True)
    autograd.dropout(x, drop, r2).backward(g)
    assert torch.equal(r2.grad, g)
    # a transposed input: the mask goes by the contiguous order of what the call sees
    assert torch.equal(autograd.dropout(x.t(), drop), autograd.dropout(x.t().contiguous(), drop))
    with pytest.raises(ValueError):
        autograd.dropout(x, drop, r[:1])


def test_dropout_refuses_a_step_counted_up_before_the_backward_pass():
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    x = torch.ones(64, device=DEV, requires_grad=True)
    y = autograd.dropout(x, nfad.Dropout(0.5, 1, 0, step))
    step.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("kind", ["gelu_erf", "gelu_tanh", "swish", "mish"])
def test_activation_with_dropout_wrapper(kind):
    rows, cols = 40, 136
    x, b, g = W.normal(rows * cols, "bf16", 1, 1.0, DEV).view(4, 10, cols), W.normal(cols, "bf16", 2, 0.5, DEV), W.normal(rows * cols, "bf16", 3, 1.0, DEV).view(4, 10, cols)
    keep, scale = dropout_plain.mask(rows * cols, 0.4, 9, 2)
    factor = (keep.double() * scale).view(x.shape).to(DEV)
    for bias in (b, None):
        leaves, refs = _leaves([x] if bias is None else [x, b])
        y = autograd.bias_act_dropout(leaves[0], leaves[1] if bias is not None else None, kind, nfad.Dropout(0.4, 9, 2))
        y.backward(g)
        y64 = _act(refs[0] + refs[1] if bias is not None else refs[0], kind) * factor
        y64.backward(g.double())
        _close(y, y64.detach(), 2, "y")
        assert torch.equal(y != 0, factor.bool() & (y != 0))
        for a, r in zip(leaves, refs):
            _close(a.grad, r.grad, 3, "grad")


def _train(block, x, target, offsets, steps):
    opt = torch.optim.SGD(block.parameters(), lr=0.5)
    for _ in range(steps):
        _, h = block(x, x, offsets)
        loss = (h - target).float().square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        block.advance()
    return [p.detach().clone() for p in block.parameters()]


def test_block_trains_and_serves():
    rows, width, hidden = 256, 128, 384
    x, target = (W.normal(rows * width, "bf16", i, 1.0, DEV).view(rows, width) for i in range(2))
    offsets = torch.tensor([0, 100, 100, rows], dtype=torch.int32, device=DEV)
    results = []
    for seed in (3, 3, 4):
        torch.manual_seed(0)
        block = feed_forward.GatedFeedForwardBlock(width, hidden, 3, p=0.25, seed=seed)
        results.append(_train(block, x, target, offsets, 5))
    # masks are a function of seed, layer and step: the same run again, to the bit, and another one under another seed
    assert all(torch.equal(a, b) for a, b in zip(results[0], results[1])) and not all(torch.equal(a, b) for a, b in zip(results[0], results[2]))
    assert all(torch.isfinite(p).all() for p in results[0]) and block.step.item() == 5
    block.eval()
    s1, h1 = block(x, x, offsets)
    s2, h2 = block(x, x, offsets)
    assert torch.equal(h1, h2) and torch.equal(s1, s2)
    with pytest.raises(ValueError):
        block.serving()
    one = feed_forward.GatedFeedForwardBlock(width, hidden, 1, p=0.25).eval()
    serve = one.serving()
    with torch.no_grad():
        for n in (1, 9, rows, 40):
            stream = x[:n].clone()
            s, h = one(x[:n], x[:n], torch.tensor([0, n], dtype=torch.int32, device=DEV))
            got = serve(stream, x[:n])
            # 8-bit operands: three significand bits and a half step of 2^-4 at each of two products, uniform over it (a factor 1/sqrt 3), two
            # operands each, as random sums; RMS norms keep relative differences
            assert float((got.float() - h.float()).norm() / h.float().norm()) <= 2 * 2.0 ** -4
            assert float((stream.float() - s.float()).norm() / s.float().norm()) <= 2 * 2.0 ** -4
        one.w1.zero_()
        stream = x[:9].clone()
        assert torch.equal(serve(x[:9].clone(), x[:9]), serve(stream, x[:9]))               # the served copy does not follow the block
        assert stream.abs().sum() > 0
    assert nfad.nfad_wait_faults() == 0


def test_training_step_in_a_graph():
    rows, width, hidden = 64, 64, 96
    x = W.normal(rows * width, "bf16", 1, 1.0, DEV).view(rows, width)
    offsets = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    block = feed_forward.GatedFeedForwardBlock(width, hidden, 1, p=0.5, seed=11)
    grads = [torch.zeros_like(p) for p in block.parameters()]

    def step():
        _, h = block(x, x, offsets)
        for g, v in zip(grads, torch.autograd.grad(h.float().square().sum(), list(block.parameters()))):
            g.copy_(v)
        block.advance()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    seen = []
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        seen.append([t.clone() for t in grads])
    assert block.step.item() == 4 and not torch.equal(seen[0][0], seen[1][0])
    # the same masks again, eagerly
    block.step.fill_(1)
    for want in seen:
        step()
        assert all(torch.equal(a, b) for a, b in zip(grads, want))


def test_command():
    r = subprocess.run([sys.executable, "-m", "paper_2209_10778_b200.feed_forward", "--gated", "--rows", "300", "--width", "128", "--hidden", "256", "--experts", "2", "--steps", "3"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "rows in 8 bits" in r.stdout
