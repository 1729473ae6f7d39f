"""The feed-forward block out of the new operators: autograd wrappers against torch's own autograd in 64 bits, the block trained
for a few steps, and served in 8-bit integers."""
import subprocess
import sys

import pytest
import torch

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


def test_block_norm_wrapper_against_torch():
    rows, cols = 24, 256
    t = {k: W.normal(n, "f32", i, 0.5, DEV) for i, (k, n) in enumerate(dict(u=rows * cols, r=rows * cols, post_gain=cols, post_bias=cols, gate=3 * cols,
                                                                               pre_gain=cols, pre_bias=cols).items())}
    t["u"], t["r"], t["gate"] = t["u"].view(2, rows // 2, cols), t["r"].view(2, rows // 2, cols), t["gate"].view(3, cols)
    leaf = {k: v.clone().requires_grad_(True) for k, v in t.items()}
    s, h = autograd.block_norm(leaf["u"], leaf["r"], post="layer", pre="rms", post_gain=leaf["post_gain"], post_bias=leaf["post_bias"], gate=leaf["gate"],
                               pre_gain=leaf["pre_gain"], pre_bias=leaf["pre_bias"], residual_scale=0.7)
    ws, wh = (W.normal(rows * cols, "f32", 20 + i, 1.0, DEV).view(s.shape) for i in range(2))
    ((s * ws).sum() + (h * wh).sum()).backward()
    ref = {k: v.double().requires_grad_(True) for k, v in t.items()}
    a = torch.nn.functional.layer_norm(ref["u"], (cols,), ref["post_gain"], ref["post_bias"], 1e-5)
    s64 = 0.7 * ref["r"] + (a.view(3, -1, cols) * ref["gate"][:, None]).view(a.shape)
    h64 = s64 / (s64.square().mean(-1, keepdim=True) + 1e-5).sqrt() * ref["pre_gain"] + ref["pre_bias"]
    ((s64 * ws.double()).sum() + (h64 * wh.double()).sum()).backward()
    assert torch.allclose(s.double(), s64, rtol=1e-5, atol=1e-5) and torch.allclose(h.double(), h64, rtol=1e-5, atol=1e-5)
    for k in t:
        rel = float((leaf[k].grad.double() - ref[k].grad).norm() / ref[k].grad.norm())
        assert rel < 1e-5, (k, rel)
    # only one of the results used: no gradient comes for the other
    for use_s in (True, False):
        u = t["u"].clone().requires_grad_(True)
        s, h = autograd.block_norm(u, t["r"], post="none", pre="rms", pre_gain=t["pre_gain"])
        (s * ws if use_s else h * wh).sum().backward()
        u64 = t["u"].double().requires_grad_(True)
        s64 = t["r"].double() + u64
        h64 = s64 / (s64.square().mean(-1, keepdim=True) + 1e-5).sqrt() * t["pre_gain"].double()
        (s64 * ws.double() if use_s else h64 * wh.double()).sum().backward()
        assert torch.allclose(u.grad.double(), u64.grad, rtol=1e-5, atol=1e-5)
    s, h = autograd.block_norm(t["u"], t["r"], post="rms", pre="none")
    assert h.numel() == 0 and s.shape == t["u"].shape


@pytest.mark.parametrize("kind", ["gelu_erf", "gelu_tanh", "swish", "mish", None])
def test_expert_wrappers_against_torch(kind):
    off = [0, 30, 30, 65, 100]
    offsets = torch.tensor(off, dtype=torch.int32, device=DEV)
    x, w1, b1 = W.normal(100 * 64, "bf16", 1, 1.0, DEV).view(100, 64), W.normal(4 * 96 * 64, "bf16", 2, 0.125, DEV).view(4, 96, 64), W.normal(4 * 96, "bf16", 3, 0.3, DEV).view(4, 96)
    w2, b2 = W.normal(4 * 64 * 96, "bf16", 4, 0.1, DEV).view(4, 64, 96), W.normal(4 * 64, "bf16", 5, 0.3, DEV).view(4, 64)
    g = W.normal(100 * 64, "bf16", 6, 1.0, DEV).view(100, 64)
    leaves = [t.clone().requires_grad_(True) for t in (x, w1, b1, w2, b2)]
    refs = [t.double().requires_grad_(True) for t in (x, w1, b1, w2, b2)]
    if kind is None:
        y = autograd.expert_linear(autograd.expert_linear(leaves[0], leaves[1], leaves[2], offsets), leaves[3], leaves[4], offsets)
    else:
        y = autograd.expert_feed_forward(*leaves, offsets, kind)
    y.backward(g)
    parts = []
    for e in range(4):
        h = _act(refs[0][off[e]:off[e + 1]] @ refs[1][e].t() + refs[2][e], kind)
        parts.append(h @ refs[3][e].t() + refs[4][e])
    y64 = torch.cat(parts)
    y64.backward(g.double())
    _close(y, y64.detach(), 3, "y")
    for name, a, b in zip(("x", "w1", "b1", "w2", "b2"), leaves, refs):
        _close(a.grad, b.grad, 6, name)
    if kind is not None:
        # the same through the one-layer wrapper
        more = [t.clone().requires_grad_(True) for t in (x, w1, b1, w2, b2)]
        y2 = autograd.expert_linear(autograd.expert_linear(more[0], more[1], more[2], offsets, kind), more[3], more[4], offsets)
        y2.backward(g)
        assert torch.equal(y, y2)
        for name, a, b in zip(("x", "w1", "b1", "w2", "b2"), more, refs):
            _close(a.grad, b.grad, 6, name)


def test_block_trains_and_serves():
    torch.manual_seed(0)
    rows, width, hidden = 256, 128, 512
    x, target = (torch.randn(rows, width, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    offsets = torch.tensor([0, 100, 100, rows], dtype=torch.int32, device=DEV)
    block = feed_forward.FeedForwardBlock(width, hidden, 3, kind="swish")
    opt = torch.optim.SGD(block.parameters(), lr=1.0)
    losses = []
    for _ in range(30):
        _, h = block(x, x, offsets)
        loss = (h - target).float().square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    assert losses[-1] < 0.95 * losses[0], losses
    one = feed_forward.FeedForwardBlock(width, hidden, 1, kind="swish")
    serve = one.serving()
    with torch.no_grad():
        for n in (1, 5, rows):
            s, want = one(x[:n], x[:n], torch.tensor([0, n], dtype=torch.int32, device=DEV))
            stream = x[:n].clone()
            got = serve(stream, x[:n])
            # each quantised operand is off by at most half of 1/127 of its row's largest value, about 1 % of a value's size at four
            # products in a row; the block's part of the sum is about a third of it
            assert float((got - want).float().norm() / want.float().norm()) < 0.03
            assert float((stream - s).float().norm() / s.float().norm()) < 0.03
    assert nfad.nfad_wait_faults() == 0


def test_example_command():
    out = subprocess.run([sys.executable, "-m", "paper_2209_10778_b200.feed_forward", "--rows", "512", "--width", "256", "--hidden", "512", "--steps", "6"],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    assert "rows in 8 bits" in out.stdout


@pytest.mark.parametrize("frozen", [["post_gain"], ["post_bias"], ["gate"], ["pre_gain"], ["pre_bias"], ["post_bias", "pre_bias"], ["post_gain", "post_bias", "pre_bias"]])
@pytest.mark.parametrize("cols", [256, 203])
def test_block_norm_wrapper_with_frozen_parameters(frozen, cols):
    rows = 24
    t = {k: W.normal(n, "f32", 30 + i, 0.5, DEV) for i, (k, n) in enumerate(dict(u=rows * cols, r=rows * cols, post_gain=cols, post_bias=cols, gate=3 * cols,
                                                                               pre_gain=cols, pre_bias=cols).items())}
    t["u"], t["r"], t["gate"] = t["u"].view(rows, cols), t["r"].view(rows, cols), t["gate"].view(3, cols)
    leaf = {k: v.clone().requires_grad_(k not in frozen) for k, v in t.items()}
    s, h = autograd.block_norm(leaf["u"], leaf["r"], post="rms", pre="rms", **{k: leaf[k] for k in list(t)[2:]})
    ws, wh = (W.normal(rows * cols, "f32", 40 + i, 1.0, DEV).view(s.shape) for i in range(2))
    ((s * ws).sum() + (h * wh).sum()).backward()
    ref = {k: v.double().requires_grad_(k not in frozen) for k, v in t.items()}
    rms = lambda x: x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    a = rms(ref["u"]) * ref["post_gain"] + ref["post_bias"]
    s64 = ref["r"] + (a.view(3, -1, cols) * ref["gate"][:, None]).view(a.shape)
    h64 = rms(s64) * ref["pre_gain"] + ref["pre_bias"]
    ((s64 * ws.double()).sum() + (h64 * wh.double()).sum()).backward()
    for k in t:
        if k in frozen:
            assert leaf[k].grad is None
            continue
        rel = float((leaf[k].grad.double() - ref[k].grad).norm() / ref[k].grad.norm())
        assert rel < 1e-5, (k, rel)


@pytest.mark.parametrize("name", ["post_gain", "post_bias", "gate", "pre_gain", "pre_bias"])
def test_block_norm_parameters_changed_before_backward(name):
    rows, cols = 8, 64
    u = W.normal(rows * cols, "bf16", 1, 1.0, DEV).view(rows, cols).requires_grad_(True)
    par = {k: W.normal(cols, "bf16", 2 + i, 0.5, DEV).requires_grad_(True) for i, k in enumerate(("post_gain", "post_bias", "gate", "pre_gain", "pre_bias"))}
    s, h = autograd.block_norm(u, None, post="rms", pre="rms", **par)
    with torch.no_grad():
        par[name].mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (s.float().sum() + h.float().sum()).backward()


def test_block_norm_parameters_pass_saved_tensor_hooks():
    rows, cols = 8, 64
    u = W.normal(rows * cols, "bf16", 1, 1.0, DEV).view(rows, cols).requires_grad_(True)
    gain = W.normal(cols, "bf16", 2, 0.5, DEV).requires_grad_(True)
    seen = []
    # kept on the host between the passes
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.data_ptr()), t.cpu())[1], lambda t: t.to(DEV)):
        s, h = autograd.block_norm(u, None, post="none", pre="rms", pre_gain=gain)
    h.float().sum().backward()
    assert gain.data_ptr() in seen
    want, want_u = gain.grad.clone(), u.grad.clone()
    gain.grad = u.grad = None
    autograd.block_norm(u, None, post="none", pre="rms", pre_gain=gain)[1].float().sum().backward()
    assert torch.equal(gain.grad, want) and torch.equal(u.grad, want_u)


def test_block_norm_stream_in_another_shape():
    u, r = W.normal(12 * 64, "f32", 1, 1.0, DEV).view(2, 6, 64).requires_grad_(True), W.normal(12 * 64, "f32", 2, 1.0, DEV).view(12, 64).requires_grad_(True)
    s, h = autograd.block_norm(u, r, residual_scale=0.5)
    s.sum().backward()
    assert u.grad.shape == u.shape and r.grad.shape == r.shape
    assert torch.equal(u.grad, torch.ones_like(u)) and torch.equal(r.grad, torch.full_like(r, 0.5))


def test_second_derivatives_are_refused():
    # the wrappers' backward passes are kernels without a derivative of their own
    off = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    x = W.normal(8 * 64, "bf16", 1, 1.0, DEV).view(8, 64).requires_grad_(True)
    w1, w2 = (W.normal(64 * 64, "bf16", 2 + i, 0.1, DEV).view(1, 64, 64) for i in range(2))
    for out in (autograd.block_norm(x, None)[1], autograd.expert_linear(x, w1, None, off, "swish"), autograd.expert_feed_forward(x, w1, None, w2, None, off)):
        # a factor that depends on x, so that the first derivative is differentiable as a whole
        g, = torch.autograd.grad((out.float() * x.float()).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.float().sum().backward()


def test_serving_keeps_the_weights_it_was_made_of():
    torch.manual_seed(1)
    block = feed_forward.FeedForwardBlock(64, 128, 1, kind="swish")
    with torch.no_grad():
        for b in (block.b1, block.b2):
            b.normal_()
    x = W.normal(4 * 64, "bf16", 1, 1.0, DEV).view(4, 64)
    serve = block.serving()
    want_s = x.clone()
    want_h = serve(want_s, x).clone()
    with torch.no_grad():
        for p in block.parameters():                                  # training goes on
            p.add_(0.5)
    s = x.clone()
    assert torch.equal(serve(s, x), want_h) and torch.equal(s, want_s)
