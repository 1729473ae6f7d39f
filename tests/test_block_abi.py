"""Argument validation of the operators around the activation, before any device is touched; and their binding's refusals of
host tensors."""
import ctypes

import pytest
import torch

import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import binding, build

BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def p(address):
    return ctypes.c_void_p(address)


def _norm(post=1, pre=1, eps=1e-5, **kw):
    return ctypes.byref(binding.BlockNormDesc(post=post, pre=pre, residual_scale=1.0, eps=eps, **kw))


def test_block_norm(lib):
    f = lib.nfad_block_norm_forward
    u, r, s, h, st = (p(a << 20) for a in range(1, 6))
    assert f(None, BF16, u, r, s, h, st, 4, 64, None) == 3
    assert f(_norm(post=3), BF16, u, r, s, h, st, 4, 64, None) == 1
    assert f(_norm(), 3, u, r, s, h, st, 4, 64, None) == 2
    assert f(_norm(eps=0.0), BF16, u, r, s, h, st, 4, 64, None) == 11
    assert f(_norm(gate=1 << 24, gate_rows=3), BF16, u, r, s, h, st, 4, 64, None) == 11
    assert f(_norm(gate=1 << 24, gate_rows=0), BF16, u, r, s, h, st, 4, 64, None) == 11
    assert f(_norm(), BF16, None, r, s, h, st, 4, 64, None) == 3
    assert f(_norm(), BF16, u, r, s, None, st, 4, 64, None) == 3                       # a norm, and nowhere to put its result
    assert f(_norm(pre=0), BF16, u, r, s, h, st, 4, 64, None) == 3
    assert f(_norm(), BF16, u, r, s, s, st, 4, 64, None) == 4
    assert f(_norm(), BF16, u, r, p((1 << 20) + 16), h, st, 4, 64, None) == 4          # part of u
    assert f(_norm(post_gain=3 << 20), BF16, u, r, s, h, st, 4, 64, None) == 4         # s over a parameter
    assert f(_norm(), BF16, p((1 << 20) + 1), r, s, h, st, 4, 64, None) == 6
    assert f(_norm(), BF16, u, r, s, h, p((5 << 20) + 4), 4, 64, None) == 6
    assert f(_norm(), BF16, u, r, s, h, st, 4, 1 << 31, None) == 9
    assert f(_norm(), BF16, None, None, None, None, None, 0, 64, None) == 0
    b = lib.nfad_block_norm_backward
    g = binding.BlockNormGrads(post_gain=8 << 20)
    assert b(_norm(post=0), BF16, u, None, u, s, st, h, None, ctypes.byref(g), r, 1 << 20, 4, 64, None) == 11
    assert b(_norm(), BF16, None, None, u, s, st, h, None, None, r, 1 << 20, 4, 64, None) == 3
    assert b(_norm(pre=0), BF16, None, None, u, s, st, h, None, None, r, 1 << 20, 4, 64, None) == 3


def test_expert_products(lib):
    x, w, b, off, y, d = (p(a << 20) for a in range(1, 7))
    f = lib.nfad_expert_linear
    assert f(4, BF16, x, w, b, off, y, d, 8, 16, 24, 2, None) == 1
    assert f(-2, BF16, x, w, b, off, y, d, 8, 16, 24, 2, None) == 1
    assert f(0, F32, x, w, b, off, y, d, 8, 16, 24, 2, None) == 2
    assert f(-1, BF16, x, w, b, off, y, d, 8, 16, 24, 2, None) == 11
    assert f(0, BF16, x, w, b, None, y, d, 8, 16, 24, 2, None) == 3
    assert f(0, BF16, None, w, b, off, y, d, 8, 16, 24, 2, None) == 3
    assert f(0, BF16, x, w, b, off, y, y, 8, 16, 24, 2, None) == 4
    assert f(0, BF16, x, w, b, off, x, d, 8, 16, 24, 2, None) == 4
    assert f(0, BF16, x, w, b, p((4 << 20) + 2), y, d, 8, 16, 24, 2, None) == 6
    assert f(0, BF16, x, w, b, off, y, d, 8, 16, 24, 1025, None) == 9
    assert f(0, BF16, x, w, b, off, y, d, 1 << 31, 16, 24, 2, None) == 9
    assert f(0, BF16, x, w, b, off, y, d, 8, 16, 24, 0, None) == 11
    assert f(0, BF16, None, None, None, None, None, None, 0, 16, 24, 2, None) == 0
    assert lib.nfad_expert_act_backward(F32, x, d, off, y, None, None, 0, 8, 24, 2, None) == 2
    assert lib.nfad_expert_act_backward(BF16, x, d, None, y, None, None, 0, 8, 24, 2, None) == 3
    assert lib.nfad_expert_act_backward(BF16, x, d, off, None, None, None, 0, 8, 24, 2, None) == 3
    assert lib.nfad_expert_act_backward(BF16, x, d, off, p((1 << 20) + 32), None, None, 0, 8, 24, 2, None) == 4
    assert lib.nfad_expert_linear_backward_input(BF16, x, w, off, d, x, 8, 16, 24, 2, None) == 4
    assert lib.nfad_expert_linear_backward_input(BF16, x, None, off, d, y, 8, 16, 24, 2, None) == 3
    assert lib.nfad_expert_linear_backward_weight(BF16, x, w, off, x, 8, 16, 24, 2, None) == 4
    assert lib.nfad_expert_linear_backward_weight(BF16, x, w, off, None, 8, 16, 24, 2, None) == 3


def test_bytes(lib):
    x, xs, w, ws, b, y, sc = (p(a << 20) for a in range(1, 8))
    assert lib.nfad_i8_quantize_rows(3, x, w, xs, 4, 16, None) == 2
    assert lib.nfad_i8_quantize_rows(BF16, None, w, xs, 4, 16, None) == 3
    assert lib.nfad_i8_quantize_rows(BF16, x, x, xs, 4, 16, None) == 4
    assert lib.nfad_i8_quantize_rows(BF16, p((1 << 20) + 1), w, xs, 4, 16, None) == 6
    f = lib.nfad_i8_linear
    assert f(9, BF16, x, xs, w, ws, b, y, 4, 16, 8, None) == 1
    assert f(-1, F32, x, xs, w, ws, b, y, 4, 16, 8, None) == 2
    assert f(-1, BF16, x, None, w, ws, b, y, 4, 16, 8, None) == 3
    assert f(-1, BF16, x, xs, w, ws, b, b, 4, 16, 8, None) == 4
    assert f(-1, BF16, x, p((2 << 20) + 2), w, ws, b, y, 4, 16, 8, None) == 6
    assert f(-1, BF16, x, xs, w, ws, b, y, 4, 131072, 8, None) == 9
    g = lib.nfad_i8_linear_dynamic
    need = lib.nfad_i8_linear_dynamic_scratch_bytes(4, 18)
    assert need == 80 + 16
    assert g(-1, BF16, x, w, ws, b, y, sc, need - 1, 4, 18, 8, None) == 7
    assert g(-1, BF16, x, w, ws, b, y, None, need, 4, 18, 8, None) == 3
    assert g(-1, BF16, x, w, ws, b, y, p((7 << 20) + 8), need, 4, 18, 8, None) == 6
    assert g(-1, BF16, x, w, ws, b, y, x, need, 4, 18, 8, None) == 4
    assert lib.nfad_i8_linear_dynamic_scratch_bytes(4, 131072) == 0


def test_status_string():
    assert "range" in binding.nfad_status_string(11)


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    w = torch.zeros(2, 8, 16, dtype=torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int32)
    y = torch.zeros(4, 8, dtype=torch.bfloat16)
    norm = nfad.BlockNorm()
    for call in (lambda: nfad.nfad_expert_linear("swish", x, w, None, off, y), lambda: nfad.nfad_expert_act_backward(y, y, off, y, None, None),
                 lambda: nfad.nfad_block_norm_forward(norm, x, x, x, x), lambda: nfad.nfad_i8_quantize_rows(x, x, x),
                 lambda: nfad.BlockNorm(pre_gain=torch.ones(16))):
        with pytest.raises(TypeError):
            call()


def test_gated(lib):
    x, w, b, off, y, d = (p(a << 20) for a in range(1, 7))
    f = lib.nfad_expert_gated_linear
    assert f(4, BF16, x, w, b, off, y, d, 8, 16, 24, 2, None) == 1
    assert f(0, F32, x, w, b, off, y, d, 8, 16, 24, 2, None) == 2
    assert f(0, BF16, x, w, b, None, y, d, 8, 16, 24, 2, None) == 3
    assert f(0, BF16, x, None, b, off, y, d, 8, 16, 24, 2, None) == 3
    assert f(0, BF16, x, w, b, off, y, y, 8, 16, 24, 2, None) == 4
    assert f(0, BF16, x, w, b, off, y, x, 8, 16, 24, 2, None) == 4
    assert f(0, BF16, x, w, b, off, p((5 << 20) + 1), d, 8, 16, 24, 2, None) == 6
    assert f(0, BF16, x, w, b, off, y, d, 8, 16, 24, 1025, None) == 9
    assert f(0, BF16, x, w, b, off, y, d, 8, 16, 1 << 30, 2, None) == 9             # twice as many outputs
    assert f(0, BF16, x, w, b, off, y, d, 8, 16, (1 << 63) + 8, 2, None) == 9
    assert f(0, BF16, x, w, b, off, y, d, 8, 16, 24, 0, None) == 11
    assert f(0, BF16, None, None, None, None, None, None, 0, 16, 24, 2, None) == 0
    g = lib.nfad_expert_gated_backward
    assert g(F32, x, d, off, y, None, None, 0, 8, 24, 2, None) == 2
    assert g(BF16, x, None, off, y, None, None, 0, 8, 24, 2, None) == 3
    assert g(BF16, x, d, off, None, None, None, 0, 8, 24, 2, None) == 3
    assert g(BF16, x, d, off, x, None, None, 0, 8, 24, 2, None) == 4                   # only the partials' place is as large
    assert g(BF16, x, d, off, p((6 << 20) + 32), None, None, 0, 8, 24, 2, None) == 4
    h = lib.nfad_expert_linear_backward_gated
    assert h(BF16, x, w, off, None, y, 8, 16, 24, 2, None) == 3
    assert h(BF16, x, w, off, d, x, 8, 16, 24, 2, None) == 4
    assert h(BF16, x, w, off, d, y, 8, 1 << 30, 24, 2, None) == 9


def test_dropout(lib):
    x, r, y, d, b = (p(a << 20) for a in range(1, 6))

    def mask(prob=0.5, step=None):
        return ctypes.byref(binding.DropoutMask(prob, 1, 2, step))

    f = lib.nfad_dropout
    assert f(BF16, None, x, r, y, 64, None) == 3
    assert f(3, mask(), x, r, y, 64, None) == 2
    for prob in (-0.1, 1.1, float("nan"), float("inf")):
        assert f(BF16, mask(prob), x, r, y, 64, None) == 11
    assert f(BF16, mask(), None, r, y, 64, None) == 3
    assert f(BF16, mask(), x, r, None, 64, None) == 3
    assert f(BF16, mask(), x, r, p((1 << 20) + 16), 64, None) == 4
    assert f(BF16, mask(step=(3 << 20) + 8), x, r, y, 64, None) == 4                      # the step among the results
    assert f(BF16, mask(step=(6 << 20) + 4), x, r, y, 64, None) == 6
    assert f(BF16, mask(), x, p((2 << 20) + 1), y, 64, None) == 6
    assert f(BF16, mask(), x, r, y, 1 << 62, None) == 9
    assert f(BF16, mask(), None, None, None, 0, None) == 0
    g = lib.nfad_bias_act_dropout_forward
    assert g(-1, BF16, mask(), x, b, y, d, 4, 16, None) == 1
    assert g(0, BF16, mask(2.0), x, b, y, d, 4, 16, None) == 11
    assert g(0, BF16, mask(), x, b, y, None, 4, 16, None) == 3
    assert g(0, BF16, mask(), x, b, y, y, 4, 16, None) == 4
    assert g(0, BF16, mask(), x, b, b, d, 4, 16, None) == 4
    assert g(0, BF16, mask(), x, b, y, d, 4, 1 << 31, None) == 9
    assert g(0, BF16, mask(), None, None, None, None, 0, 16, None) == 0
    with pytest.raises(TypeError):
        nfad.nfad_dropout(nfad.Dropout(0.5, 1), torch.zeros(8), None, torch.zeros(8))


def test_f8(lib):
    x, xs, w, ws, b, y, sc = (p(a << 20) for a in range(1, 8))
    q = lib.nfad_f8_quantize_rows
    assert q(3, x, w, xs, 4, 16, None) == 2
    assert q(BF16, None, w, xs, 4, 16, None) == 3
    assert q(BF16, x, w, None, 4, 16, None) == 3
    assert q(BF16, x, x, xs, 4, 16, None) == 4
    assert q(BF16, p((1 << 20) + 1), w, xs, 4, 16, None) == 6
    assert q(BF16, x, w, p((2 << 20) + 2), 4, 16, None) == 6
    assert q(BF16, x, w, xs, 4, 1 << 31, None) == 9
    assert q(BF16, None, None, None, 0, 16, None) == 0
    m = lib.nfad_f8_quantize_blocks
    assert m(3, x, w, ws, 2, 4, 16, None) == 2
    assert m(BF16, x, None, ws, 2, 4, 16, None) == 3
    assert m(BF16, x, w, p((1 << 20) + 64), 2, 4, 16, None) == 4
    assert m(BF16, x, w, ws, 1 << 62, 4, 16, None) == 9
    assert m(BF16, None, None, None, 0, 4, 16, None) == 0
    for f in (lib.nfad_f8_linear, lib.nfad_f8_gated_linear):
        assert f(9, BF16, x, xs, w, ws, b, y, 4, 16, 8, None) == 1
        assert f(-1, F32, x, xs, w, ws, b, y, 4, 16, 8, None) == 2
        assert f(-1, BF16, x, None, w, ws, b, y, 4, 16, 8, None) == 3
        assert f(-1, BF16, x, xs, w, None, b, y, 4, 16, 8, None) == 3
        assert f(-1, BF16, x, xs, w, ws, b, b, 4, 16, 8, None) == 4
        assert f(-1, BF16, x, xs, w, ws, b, p((3 << 20) + 64), 4, 16, 8, None) == 4
        assert f(-1, BF16, x, p((2 << 20) + 2), w, ws, b, y, 4, 16, 8, None) == 6
        assert f(-1, BF16, x, xs, w, ws, b, p((6 << 20) + 1), 4, 16, 8, None) == 6
        assert f(-1, BF16, x, xs, w, ws, b, y, 1 << 31, 16, 8, None) == 9
        assert f(-1, BF16, None, None, None, None, None, None, 0, 16, 8, None) == 0
    assert lib.nfad_f8_gated_linear(-1, BF16, x, xs, w, ws, b, y, 4, 16, 1 << 30, None) == 9
    need = lib.nfad_f8_linear_dynamic_scratch_bytes(4, 130)
    assert need == 528 + 32                                           # 4 x 130 bytes to the next 16, two blocks of four rows
    for g in (lib.nfad_f8_linear_dynamic, lib.nfad_f8_gated_linear_dynamic):
        assert g(-1, BF16, x, w, ws, b, y, sc, need - 1, 4, 130, 8, None) == 7
        assert g(-1, BF16, x, w, ws, b, y, None, need, 4, 130, 8, None) == 3
        assert g(-1, BF16, x, w, ws, b, y, p((7 << 20) + 8), need, 4, 130, 8, None) == 6
        assert g(-1, BF16, x, w, ws, b, y, x, need, 4, 130, 8, None) == 4
    with pytest.raises(TypeError):
        nfad.nfad_f8_quantize_rows(torch.zeros(4, 16), torch.zeros(4, 16).to(torch.float8_e4m3fn), torch.zeros(1, 4))
