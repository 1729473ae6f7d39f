"""Dropout against the plain mask: every element's fate exactly, its value to one rounding; alone, with a residual, and behind an
activation whose derivative carries the mask."""
import pytest
import torch

import block_plain as block
import dropout_plain as plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
DTYPES = ["f32", "bf16", "f16"]
SEED, OFFSET = 0x123456789abcdef0, (3 << 32) + 17
# around packets, draws, tiles and many CTAs
SIZES = [1, 3, 4, 5, 7, 8, 9, 31, 1000, 8191, 8192, 8200, 24576 + 13, 1 << 20]


def _nan_like(t):
    return torch.full_like(t, float("nan"), device=DEV)


def _check(y, x, r, p, at, what, seed=SEED):
    keep, scale = plain.mask(x.numel(), p, seed, at)
    kept = x.double().flatten() * scale
    want = torch.where(keep, kept, torch.zeros_like(kept)) + (r.double().flatten() if r is not None else 0.0)
    # the scale is an fp32 number and the product and sum one fp32 operation: two roundings of what they form
    mag = torch.where(keep, kept.abs() + (r.double().flatten().abs() if r is not None else 0.0), torch.zeros_like(kept))
    block.check(y.flatten(), want, 2 * block.EPS32 * mag, what)
    if r is None:
        assert torch.equal(y.cpu().flatten() == 0, ~keep | (want.to(y.dtype) == 0)), what + ": dropped places"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", SIZES)
def test_alone_and_with_residual(dtype, n):
    x, r = W.normal(n, dtype, 1, 1.0), W.normal(n, dtype, 2, 2.0)
    for p in (0.0, 0.1, 0.5, 0.999, 1.0):
        drop = nfad.Dropout(p, SEED, OFFSET)
        for res in (None, r):
            y = _nan_like(x)
            nfad.nfad_dropout(drop, x.to(DEV), None if res is None else res.to(DEV), y)
            _check(y, x, res, p, OFFSET, f"p {p}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_step_and_seed(dtype):
    n = 5000
    x = W.normal(n, dtype, 1, 1.0)
    step = torch.tensor([5], dtype=torch.int64, device=DEV)
    for seed, offset, s in ((0, 0, 0), (2 ** 64 - 1, 2 ** 64 - 1, 1), (1 << 40, 1 << 33, 2 ** 62), (7, 3, -2)):
        step.fill_(s)
        y = _nan_like(x)
        nfad.nfad_dropout(nfad.Dropout(0.3, seed, offset, step), x.to(DEV), None, y)
        _check(y, x, None, 0.3, offset + s, f"seed {seed}", seed)          # offset + step modulo 2^64


def _act_check(y, d, z, kind, keep, scale, what):
    """y = m f(z), d = m f'(z).  16-bit storage: the chains' bounds of check_act, scaled; fp32 storage: within 4 spacings of f and f' (or of
    their terms) as the plain pass, one further rounding of the product and the scale's own."""
    want, slope = block.act(z, kind)
    for got, v, terms in ((y, want, 0.0), (d, slope, 1.25)):
        t = got.dtype
        if t == torch.float32:
            err = 8 * block.half_ulp(torch.maximum(v.abs(), torch.full_like(v, terms)), t)
        else:
            err = block.half_ulp(v, t) + (block.half_ulp(torch.full_like(v, terms), t) / 8 if terms else 0.0)
        v, err = v * scale, err * scale + 2 * block.EPS32 * v.abs() * scale
        zero = torch.zeros_like(v)
        block.check(got, torch.where(keep, v, zero), torch.where(keep, err, zero), what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (7, 8), (64, 64), (33, 37), (5, 1000), (129, 264), (300, 1021), (2, 4100)])
def test_behind_an_activation(dtype, rows, cols):
    x, b = W.normal(rows * cols, dtype, 1, 1.5).view(rows, cols), W.normal(cols, dtype, 2, 0.5)
    for kind in ("gelu_erf", "gelu_tanh", "swish", "mish"):
        for bias in (b, None):
            for p in (0.0, 0.2, 1.0):
                y, d = _nan_like(x), _nan_like(x)
                nfad.nfad_bias_act_dropout_forward(kind, nfad.Dropout(p, SEED, OFFSET), x.to(DEV), None if bias is None else bias.to(DEV), y, d)
                z = (x.float() + bias.float() if bias is not None else x.float()).double().flatten()      # the sum is one fp32 addition
                keep, scale = plain.mask(z.numel(), p, SEED, OFFSET)
                _act_check(y.flatten(), d.flatten(), z, kind, keep, scale, f"{kind} p {p}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_without_dropping_it_is_the_plain_pass(dtype):
    x, b = W.normal(64 * 264, dtype, 1, 1.5).view(64, 264).to(DEV), W.normal(264, dtype, 2, 0.5).to(DEV)
    for kind in ("gelu_erf", "gelu_tanh", "swish", "mish"):
        y, d, y2, d2 = (_nan_like(x) for _ in range(4))
        nfad.nfad_bias_act_dropout_forward(kind, nfad.Dropout(0.0, 1), x, b, y, d)
        nfad.nfad_bias_act_forward(kind, x, b, y2, d2)
        assert torch.equal(y, y2) and torch.equal(d, d2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_unaligned_tensors_give_the_same_bits(dtype):
    n, cols = 24 * 1000 + 24, 24
    x, r, b = W.normal(n, dtype, 1, 1.0).to(DEV), W.normal(n, dtype, 2, 1.0).to(DEV), W.normal(cols, dtype, 3, 0.5).to(DEV)

    def shifted(t, by):
        buf = torch.full((t.numel() + by + 9,), 7.0, dtype=t.dtype, device=DEV)
        buf[by:by + t.numel()].copy_(t)
        return buf, buf[by:by + t.numel()]

    drop = nfad.Dropout(0.4, SEED, OFFSET)
    y, ya, da = (_nan_like(x) for _ in range(3))
    nfad.nfad_dropout(drop, x, r, y)
    nfad.nfad_bias_act_dropout_forward("mish", drop, x.view(-1, cols), b, ya.view(-1, cols), da.view(-1, cols))
    for shifts in ((1, 1, 1), (0, 3, 0), (2, 0, 0), (0, 0, 5)):
        (_, x2), (_, r2), (whole, y2) = (shifted(t, s) for t, s in zip((x, r, _nan_like(x)), shifts))
        nfad.nfad_dropout(drop, x2, r2, y2)
        assert torch.equal(y, y2)
        assert (whole[:shifts[2]] == 7).all() and (whole[shifts[2] + n:] == 7).all()          # nothing beside the results is written
        _, b2 = shifted(b, shifts[1])
        ya2, da2 = (shifted(_nan_like(x), shifts[2])[1] for _ in range(2))
        nfad.nfad_bias_act_dropout_forward("mish", drop, x2.view(-1, cols), b2, ya2.view(-1, cols), da2.view(-1, cols))
        assert torch.equal(ya, ya2) and torch.equal(da, da2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_dropped_places_hide_what_they_held(dtype):
    n = 4096
    x, r = W.normal(n, dtype, 1, 1.0), W.normal(n, dtype, 2, 1.0)
    keep, _ = plain.mask(n, 0.5, SEED, OFFSET)
    x[~keep] = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(x.dtype).max], dtype=x.dtype).repeat(n)[:int((~keep).sum())]
    y, z = _nan_like(x), _nan_like(x)
    nfad.nfad_dropout(nfad.Dropout(0.5, SEED, OFFSET), x.to(DEV), None, y)
    nfad.nfad_dropout(nfad.Dropout(0.5, SEED, OFFSET), x.to(DEV), r.to(DEV), z)
    assert torch.isfinite(y).all() and (y.cpu()[~keep] == 0).all() and torch.equal(z.cpu()[~keep], r[~keep])
    x[keep] = float("nan")
    ya, da = _nan_like(x), _nan_like(x)
    nfad.nfad_dropout(nfad.Dropout(0.5, SEED, OFFSET), x.to(DEV), None, y)
    nfad.nfad_bias_act_dropout_forward("gelu_erf", nfad.Dropout(0.5, SEED, OFFSET), x.to(DEV), None, ya, da)
    for t in (y, ya, da):
        assert torch.equal(torch.isnan(t.cpu()), keep)
    nfad.nfad_dropout(nfad.Dropout(1.0, SEED), x.to(DEV), None, y)
    assert (y == 0).all()


def test_in_place():
    x, r = W.normal(1000, "bf16", 1, 1.0).to(DEV), W.normal(1000, "bf16", 2, 1.0).to(DEV)
    drop = nfad.Dropout(0.2, SEED)
    y = torch.empty_like(x)
    nfad.nfad_dropout(drop, x, r, y)
    for place in (0, 1):
        a, b = x.clone(), r.clone()
        nfad.nfad_dropout(drop, a, b, (a, b)[place])
        assert torch.equal((a, b)[place], y)
    d, x2, d2 = torch.empty_like(x), x.clone(), torch.empty_like(x)
    nfad.nfad_bias_act_dropout_forward("swish", drop, x, None, y, d)
    nfad.nfad_bias_act_dropout_forward("swish", drop, x2, None, d2, x2)                    # the derivative in x's place
    assert torch.equal(d2, y) and torch.equal(x2, d)


def test_graph_draws_anew_with_the_step():
    x = W.normal(10000, "bf16", 1, 1.0)
    dx, y, step = x.to(DEV), torch.empty(10000, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    drop = nfad.Dropout(0.25, SEED, 40, step)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        nfad.nfad_dropout(drop, dx, None, y)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nfad.nfad_dropout(drop, dx, None, y)
        step.add_(1)
    for s in range(3):
        g.replay()
        torch.cuda.synchronize()
        _check(y, x, None, 0.25, 40 + s, f"replay {s}")


def test_elements_beyond_32_bits():
    n = (1 << 31) + 8 * 1000 + 3
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_dropout(nfad.Dropout(0.5, SEED, OFFSET), x, None, x)
    for first, count in ((0, 4096), ((1 << 31) - 4096, 12096 + 3)):
        keep, scale = plain.mask(count, 0.5, SEED, OFFSET, first)
        got = x[first:first + count].float().cpu()
        assert torch.equal(got, torch.where(keep, torch.tensor(2.0), torch.tensor(0.0)))


def test_refusals():
    x = torch.zeros(64, dtype=torch.bfloat16, device=DEV)
    drop = nfad.Dropout(0.5, 1)
    for bad in (lambda: nfad.Dropout(1.5, 1), lambda: nfad.Dropout(float("nan"), 1), lambda: nfad.Dropout(0.5, -1), lambda: nfad.Dropout(0.5, 1, 2 ** 64),
                lambda: nfad.Dropout(0.5, 1, 0, torch.zeros(2, dtype=torch.int64, device=DEV)), lambda: nfad.nfad_dropout(drop, x, x[:32], x),
                lambda: nfad.nfad_dropout(drop, x, x.half(), x), lambda: nfad.nfad_bias_act_dropout_forward("swish", drop, x.view(8, 8), x, x.view(8, 8), x.clone()),
                lambda: nfad.nfad_dropout(drop, x.view(8, 8).t(), None, x)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nfad.Dropout(0.5, 1, 0, torch.zeros(1, device=DEV)), lambda: nfad.nfad_dropout(0.5, x, None, x), lambda: nfad.nfad_dropout(drop, x.long(), None, x),
                lambda: nfad.Dropout(0.5, 1, 0, torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(TypeError):
            bad()
    big = torch.zeros(128, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(nfad.NfadError) as e:
        nfad.nfad_dropout(drop, big[:64], None, big[8:72])
    assert e.value.status == 4
