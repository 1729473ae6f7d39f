"""Gated layers grouped by expert against plain 64-bit implementations: value and both partial derivatives, the multiplication of the
backward pass with its bias sums, and the same behind a linear layer.  Bounds: block_plain.dot_error for the two tensor-core sums, the
activation's own accuracy as check_act has it, carried through the product with the other factor, one rounding to the storage type."""
import pytest
import torch

import block_plain as plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
DTYPES = ["bf16", "f16"]
KINDS = [None, "gelu_erf", "gelu_tanh", "swish", "mish"]
# rows of each expert, rows before the first and after the last, in, out
CASES = [
    ([5], 0, 0, 64, 64),
    ([128], 0, 0, 128, 256),
    ([300], 3, 9, 200, 320),
    ([1, 0, 127, 129, 0, 64, 256], 0, 0, 192, 136),
    ([0, 0, 33], 5, 0, 8, 8),
    ([17, 40, 1, 2, 3, 70], 0, 7, 520, 264),
    ([0, 0], 4, 3, 64, 64),
    ([2] * 70, 0, 0, 72, 600),
    ([33, 65], 1, 1, 37, 51),                 # rows off every vector boundary: gathered
    ([3, 0, 200], 0, 2, 1, 1),
    ([130, 20], 0, 0, 100, 44),               # multiples of four only
    ([90, 50], 0, 3, 96, 70),                 # tensor copies in, single elements out
]
# the ways through the products that sizes choose (148 SMs): pairs, single CTAs of both widths, split reductions, few rows
WAYS = [
    ([1100, 700, 800], 0, 0, 1048, 264), ([1101, 701, 900], 1, 3, 520, 1800), ([40, 0, 37], 3, 2, 1288, 136), ([77], 0, 0, 2568, 72),
    ([33], 0, 0, 5128, 72), ([150], 0, 0, 72, 5128), ([260], 0, 0, 264, 2504), ([9, 0, 17, 3], 1, 2, 1032, 200), ([3, 1, 0, 2] * 40, 0, 0, 264, 136),
    ([1], 0, 0, 4096, 1000), ([16], 0, 0, 1032, 520), ([2000, 17, 1500, 0, 500], 0, 5, 328, 776),
]


def _case(case, dtype, seed):
    counts, lead, tail, n_in, n_out = case
    rows = sum(counts) + lead + tail
    off = [lead]
    for c in counts:
        off.append(off[-1] + c)
    e = len(counts)
    x = W.normal(rows * n_in, dtype, seed, 1.0).view(rows, n_in)
    w = W.normal(e * 2 * n_out * n_in, dtype, seed + 1, max(n_in, 1) ** -0.5).view(e, 2, n_out, n_in)
    b = W.normal(e * 2 * n_out, dtype, seed + 2, 0.4).view(e, 2, n_out)
    return x, w, b, torch.tensor(off, dtype=torch.int32), off


def _nan(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def _forward(kind, x, w, b, off, train=True):
    y = _nan(x.shape[0], w.shape[2], dtype=x.dtype)
    both = _nan(x.shape[0], 2, w.shape[2], dtype=x.dtype) if train else None
    nfad.nfad_expert_gated_linear(kind, x.to(DEV), w.to(DEV), None if b is None else b.to(DEV), off.to(DEV), y, both)
    torch.cuda.synchronize()
    return y, both


def _check_forward(kind, x, w, b, off, y, both):
    y, both = y.cpu(), None if both is None else both.cpu()
    covered = torch.zeros(x.shape[0], dtype=torch.bool)
    for e in range(w.shape[0]):
        p = slice(off[e], off[e + 1])
        covered[p] = True
        if off[e + 1] <= off[e]:
            continue
        (a, ea), (u, eu) = (_projection(x[p], w[e, j], None if b is None else b[e, j]) for j in (0, 1))
        f, slope = plain.act(a, kind)
        # the chains' own errors, as check_act counts them (none without an activation), then those of the two products
        own = 0 if kind is None else plain.half_ulp(f, y.dtype)
        own_slope = 0 if kind is None else plain.half_ulp(slope, y.dtype) + plain.half_ulp(torch.full_like(slope, 1.25), y.dtype) / 8
        ef, es = plain.SLOPE * ea + own, plain.CURVATURE * ea + own_slope
        plain.check(y[p], f * u, u.abs() * ef + f.abs() * eu + ef * eu + plain.EPS32 * (f * u).abs(), f"y of expert {e}")
        if both is not None:
            if kind is None:
                es = torch.zeros_like(a)
            plain.check(both[p, 0], slope * u, u.abs() * es + slope.abs() * eu + es * eu + plain.EPS32 * (slope * u).abs(), f"dy/da of expert {e}")
            plain.check(both[p, 1], f, ef if kind is not None else ea, f"dy/du of expert {e}")
    assert not y[~covered].any() and (both is None or not both[~covered].any()), "rows without an expert"


def _projection(x, w, b):
    z, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    return z, plain.dot_error(mag, x.shape[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward(dtype, case):
    x, w, b, off, o = _case(CASES[case], dtype, 10 * case)
    for kind in KINDS:
        for bias in (b, None):
            y, both = _forward(kind, x, w, bias, off)
            _check_forward(kind, x, w, bias, o, y, both)
            _check_forward(kind, x, w, bias, o, *_forward(kind, x, w, bias, off, train=False))
    assert nfad.nfad_wait_faults() == 0


def _backward(g, both, off, experts, bias=True):
    gz = _nan(*both.shape, dtype=g.dtype)
    gb = _nan(experts, 2, g.shape[1], dtype=torch.float32) if bias else None
    scratch = nfad.nfad_expert_act_backward_scratch(gz.flatten(1)).fill_(0xff)
    nfad.nfad_expert_gated_backward(g.to(DEV), both.to(DEV), off.to(DEV), gz, gb, scratch if bias else None)
    torch.cuda.synchronize()
    return gz.cpu(), None if gb is None else gb.cpu()


def _factors(rows, n, dtype, seed):
    return torch.stack([W.normal(rows * n, dtype, seed, 0.7).view(rows, n), W.uniform(rows * n, dtype, seed + 1, -0.2, 1.1).view(rows, n)], 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", list(range(len(CASES))) + ["long"])
def test_backward(dtype, case):
    c = ([900, 0, 1, 4000, 3, 20, 700], 11, 13, 8, 264) if case == "long" else CASES[case]
    _, _, _, off, o = _case(c, dtype, 3)
    rows, n, experts = o[-1] + c[2], c[4], len(c[0])
    g, both = W.normal(rows * n, dtype, 5, 1.0).view(rows, n), _factors(rows, n, dtype, 6)
    gz, gb = _backward(g, both, off, experts)
    for e in range(experts):
        p = slice(o[e], o[e + 1])
        exact = g[p].double()[:, None, :] * both[p].double()
        assert torch.equal(gz[p], exact.to(gz.dtype)), "one rounding of the product"
        plain.check(gb[e], exact.sum(0), plain.EPS32 * (o[e + 1] - o[e] + 40) * exact.abs().sum(0), f"bias of expert {e}")
    assert not gz[:o[0]].any() and not gz[o[-1]:].any()
    again = _backward(g, both, off, experts)
    assert torch.equal(gb, again[1])                                  # the same bits every time
    assert torch.equal(gz, _backward(g, both, off, experts, bias=False)[0])
    if rows:
        place = both.to(DEV)                                          # in place of the partials
        nfad.nfad_expert_gated_backward(g.to(DEV), place, off.to(DEV), place, None, None)
        assert torch.equal(place.cpu(), gz)


def _through_linear(gz, w, off, both):
    out = _nan(*both.shape, dtype=gz.dtype)
    nfad.nfad_expert_linear_backward_gated(gz.to(DEV), w.to(DEV), off.to(DEV), both.to(DEV), out)
    torch.cuda.synchronize()
    return out.cpu()


def _check_through_linear(gz, w, o, both, out):
    covered = torch.zeros(gz.shape[0], dtype=torch.bool)
    for e in range(w.shape[0]):
        p = slice(o[e], o[e + 1])
        covered[p] = True
        g, we = gz[p].double(), w[e].double()
        v, m = g @ we, plain.dot_error(g.abs() @ we.abs(), w.shape[1])
        for j in (0, 1):
            f = both[p, j].double()
            plain.check(out[p, j], v * f, m * f.abs() + plain.EPS32 * (v * f).abs(), f"part {j} of expert {e}")
    assert not out[~covered].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_through_linear(dtype, case):
    counts, lead, tail, n_in, n_out = CASES[case]
    _, _, _, off, o = _case(CASES[case], dtype, 4)
    rows, e = o[-1] + tail, len(counts)
    w = W.normal(e * n_out * n_in, dtype, 8, max(n_out, 1) ** -0.5).view(e, n_out, n_in)
    gz, both = W.normal(rows * n_out, dtype, 9, 1.0).view(rows, n_out), _factors(rows, n_in, dtype, 11)
    out = _through_linear(gz, w, off, both)
    _check_through_linear(gz, w, o, both, out)
    if rows:
        place = both.to(DEV)
        nfad.nfad_expert_linear_backward_gated(gz.to(DEV), w.to(DEV), off.to(DEV), place, place)
        assert torch.equal(place.cpu(), out)
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_ways(dtype, way):
    counts, lead, tail, n_in, n_out = WAYS[way]
    x, w, b, off, o = _case(WAYS[way], dtype, 300 + way)
    _check_forward("gelu_erf", x, w, b, o, *_forward("gelu_erf", x, w, b, off))
    _check_forward("swish", x, w, None, o, *_forward("swish", x, w, None, off, train=False))
    e, rows = len(counts), x.shape[0]
    w2 = W.normal(e * n_in * n_out, dtype, 8, n_in ** -0.5).view(e, n_in, n_out)     # back to the width that came in
    gz, both = W.normal(rows * n_in, dtype, 9, 1.0).view(rows, n_in), _factors(rows, n_out, dtype, 11)
    _check_through_linear(gz, w2, o, both, _through_linear(gz, w2, off, both))
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_neighbours_do_not_mix(dtype):
    # infinities and NaN in one expert's rows and weights, and in rows of nobody, stay there
    counts, n_in, n_out = [70, 61, 90], 136, 72
    x, w, b, off, o = _case((counts, 0, 3, n_in, n_out), dtype, 7)
    gz, both = W.normal(x.shape[0] * n_out, dtype, 9, 1.0).view(x.shape[0], n_out), _factors(x.shape[0], n_in, dtype, 11)
    w2 = W.normal(3 * n_out * n_in, dtype, 8, 0.1).view(3, n_out, n_in)
    first = (*_forward("gelu_erf", x, w, b, off), _through_linear(gz, w2, off, both))
    x, w, gz, w2, both = (t.clone() for t in (x, w, gz, w2, both))
    p = slice(o[1], o[2])
    x[p], w[1], gz[p], w2[1], both[p] = (float("nan"),) * 5
    x[o[3]:], gz[o[3]:], both[o[3]:] = float("nan"), float("inf"), float("nan")
    second = (*_forward("gelu_erf", x, w, b, off), _through_linear(gz, w2, off, both))
    others = [i for i in range(x.shape[0]) if not o[1] <= i < o[2]]
    for a, c in zip(first, second):
        assert torch.equal(a[others], c[others])
        assert torch.isnan(c[p]).all()


def test_gate_and_other_weight_do_not_mix():
    # the last tile along the outputs holds rows behind each weight's last: u's weight must not reach a, nor the next expert's u
    for n_out in (8, 72, 136, 200, 264):
        x, w, b, off, o = _case(([20, 30], 0, 0, 64, n_out), "bf16", 7)
        y, both = _forward("swish", x, w, b, off)
        w2 = w.clone()
        w2[0, 1], w2[1] = float("nan"), float("nan")
        _, both2 = _forward("swish", x, w2, b, off)
        assert torch.equal(both[:20, 1], both2[:20, 1])               # f(a) of the first expert
        assert torch.isnan(both2[:20, 0]).all() and torch.isnan(both2[20:]).all()


def test_unaligned_tensors_give_the_same_bits():
    x, w, b, off, o = _case(([40, 0, 150], 0, 2, 64, 72), "bf16", 7)
    gz, both = W.normal(x.shape[0] * 64, "bf16", 9, 1.0).view(-1, 64), _factors(x.shape[0], 72, "bf16", 11)
    w2 = W.normal(3 * 64 * 72, "bf16", 8, 0.1).view(3, 64, 72)

    def shifted(t):
        buf = torch.zeros(t.numel() + 1, dtype=t.dtype, device=DEV)
        buf[1:].copy_(t.reshape(-1))
        return buf[1:].view(t.shape)

    y, d = _forward("mish", x, w, b, off)
    y2, d2 = shifted(torch.zeros_like(y)), shifted(torch.zeros_like(d))
    nfad.nfad_expert_gated_linear("mish", shifted(x), shifted(w), shifted(b), off.to(DEV), y2, d2)
    assert torch.equal(y, y2) and torch.equal(d, d2)
    out, out2 = _through_linear(gz, w2, off, both), shifted(torch.zeros_like(both))
    nfad.nfad_expert_linear_backward_gated(shifted(gz), shifted(w2), off.to(DEV), shifted(both), out2)
    assert torch.equal(out, out2.cpu())
    gz = gz[:, :1].repeat(1, 72).contiguous()
    back, back2 = _backward(gz, both, off, 3, bias=False)[0], shifted(torch.zeros_like(both))
    nfad.nfad_expert_gated_backward(shifted(gz), shifted(both), off.to(DEV), back2, None, None)
    assert torch.equal(back, back2.cpu())


def test_offsets_out_of_range_are_held_inside():
    x, w, b, _, _ = _case(([50, 30], 0, 0, 64, 64), "bf16", 7)
    off, held = torch.tensor([-7, 1 << 30, 20], dtype=torch.int32), torch.tensor([0, 80, 80], dtype=torch.int32)
    for a, c in zip(_forward("swish", x, w, b, off), _forward("swish", x, w, b, held)):
        assert torch.equal(a, c)
    g, both = W.normal(80 * 64, "bf16", 9, 1.0).view(80, 64), _factors(80, 64, "bf16", 11)
    assert torch.equal(_backward(g, both, off, 2)[0], _backward(g, both, held, 2)[0])
    w2 = w[:, 0].contiguous()
    assert torch.equal(_through_linear(g, w2, off, both), _through_linear(g, w2, held, both))


def test_gradient_against_differences():
    # <wy, f(a) u> along a direction in x, w and b: central differences in 64 bits against the 16-bit gradients
    x, w, b, off, o = _case(([40, 0, 25], 0, 0, 48, 56), "bf16", 7)
    wy = W.normal(x.shape[0] * 56, "bf16", 9, 1.0).view(-1, 56)
    for kind in KINDS:
        _, both = _forward(kind, x, w, b, off)
        gz, gb = _backward(wy, both.cpu(), off, 3)
        gz = gz.flatten(1).to(DEV)
        gx, gw = torch.empty_like(x, device=DEV), torch.empty_like(w, device=DEV)
        nfad.nfad_expert_linear_backward_input(gz, w.to(DEV).flatten(1, 2), off.to(DEV), None, gx)
        nfad.nfad_expert_linear_backward_weight(gz, x.to(DEV), off.to(DEV), gw.flatten(1, 2))
        dx, dw, db = (W.normal(t.numel(), "f32", 20 + i, 0.3).view(t.shape).double() for i, t in enumerate((x, w, b)))

        def value(t):
            total = 0.0
            for e in range(3):
                p = slice(o[e], o[e + 1])
                a, u = ((x[p].double() + t * dx[p]) @ (w[e, j].double() + t * dw[e, j]).t() + b[e, j].double() + t * db[e, j] for j in (0, 1))
                total += float((wy[p].double() * plain.act(a, kind)[0] * u).sum())
            return total

        slope = (value(1e-4) - value(-1e-4)) / 2e-4
        terms = [gx.cpu().double() * dx, gw.cpu().double() * dw, gb.double() * db]
        got = float(sum(t.sum() for t in terms))
        # partials, grad_z and the results are each rounded to 8 bits: three half spacings of 2^-8 of the terms' size, as a random sum
        size = sum(float((t * t).sum()) for t in terms) ** 0.5
        assert abs(got - slope) <= 6 * 3 * 2.0 ** -9 * size + 1e-6 * abs(slope), (kind, got, slope, size)


def test_graph_with_other_offsets():
    x, w, b, off, o = _case(([40, 60, 28], 0, 0, 128, 128), "bf16", 7)
    dx, dw, db, doff = x.to(DEV), w.to(DEV), b.to(DEV), off.to(DEV)
    y, both = torch.zeros(128, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(128, 2, 128, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        nfad.nfad_expert_gated_linear("swish", dx, dw, db, doff, y, both)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nfad.nfad_expert_gated_linear("swish", dx, dw, db, doff, y, both)
    for other in ([0, 0, 128, 128], [0, 100, 101, 120]):
        doff.copy_(torch.tensor(other, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        _check_forward("swish", x, w, b, other, y, both)


def test_elements_beyond_32_bits():
    # partials whose element offsets pass 2^31: the last rows against the plain form
    rows, n_in, n_out = 270000, 64, 4104
    w, b = W.normal(2 * n_out * n_in, "bf16", 2, 0.125).view(1, 2, n_out, n_in), W.normal(2 * n_out, "bf16", 3, 0.4).view(1, 2, n_out)
    x = torch.zeros(rows, n_in, dtype=torch.bfloat16, device=DEV)
    tail = W.normal(5 * n_in, "bf16", 4, 1.0).view(5, n_in)
    x[-5:] = tail.to(DEV)
    off = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    y, both = torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV), torch.empty(rows, 2, n_out, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_expert_gated_linear("swish", x, w.to(DEV), b.to(DEV), off, y, both)
    _check_forward("swish", tail, w, b, [0, 5], y[-5:], both[-5:])
    gz, gb = torch.empty_like(both), torch.empty(1, 2, n_out, device=DEV)
    nfad.nfad_expert_gated_backward(y, both, off, gz, gb, nfad.nfad_expert_act_backward_scratch(gz.flatten(1)))
    assert torch.equal(gz[-5:], (y[-5:, None, :].double() * both[-5:].double()).bfloat16())
    w2 = W.normal(n_in * n_out, "bf16", 8, 0.125).view(1, n_in, n_out)
    nfad.nfad_expert_linear_backward_gated(x, w2.to(DEV), off, both, gz)
    _check_through_linear(tail, w2, [0, 5], both[-5:].cpu(), gz[-5:].cpu())


def test_no_rows_and_no_reduction():
    x, w, b, off, o = _case(([0, 0], 0, 0, 32, 40), "bf16", 7)
    y, _ = _forward("swish", x, w, b, off)
    assert y.shape == (0, 40)
    _, gb = _backward(y.cpu(), torch.empty(0, 2, 40, dtype=torch.bfloat16), off, 2)
    assert not gb.any()
    x, w, b, off, o = _case(([10, 5], 0, 0, 0, 40), "bf16", 7)
    _check_forward("swish", x, w, b, o, *_forward("swish", x, w, b, off))


def test_refusals():
    x, w, b, off, _ = (t.to(DEV) if isinstance(t, torch.Tensor) else t for t in _case(([10, 5], 0, 0, 16, 24), "bf16", 7))
    y, both = torch.empty(15, 24, dtype=torch.bfloat16, device=DEV), torch.empty(15, 2, 24, dtype=torch.bfloat16, device=DEV)

    def status(fn):
        with pytest.raises(nfad.NfadError) as e:
            fn()
        return e.value.status

    assert status(lambda: nfad.nfad_expert_gated_linear(7, x, w, b, off, y)) == 1
    assert status(lambda: nfad.nfad_expert_gated_linear("swish", x.float(), w.float(), b.float(), off, y.float())) == 2
    assert status(lambda: nfad.nfad_expert_gated_linear("swish", x, w, b, off, both.view(-1)[:15 * 24].view(15, 24), both)) == 4
    for bad in (lambda: nfad.nfad_expert_gated_linear("swish", x, w[:, :1], b, off, y), lambda: nfad.nfad_expert_gated_linear("swish", x, w, b[:1], off, y),
                lambda: nfad.nfad_expert_gated_linear("swish", x, w.flatten(1, 2), b, off, y), lambda: nfad.nfad_expert_gated_linear("swish", x, w, b, off[:2], y),
                lambda: nfad.nfad_expert_gated_linear("swish", x, w, b, off, y, both[:, :1]), lambda: nfad.nfad_expert_gated_backward(y, both[:10], off, both, None, None),
                lambda: nfad.nfad_expert_linear_backward_gated(x, w[:, 0], off, both, both)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        nfad.nfad_expert_gated_backward(y, None, off, both, None, None)
    with pytest.raises(TypeError):
        nfad.nfad_expert_gated_linear("swish", x, w, b, off.long(), y)
    gb = torch.empty(2, 2, 24, device=DEV)
    big, big_both = torch.zeros(4000, 24, dtype=torch.bfloat16, device=DEV), torch.zeros(4000, 2, 24, dtype=torch.bfloat16, device=DEV)
    scratch = nfad.nfad_expert_act_backward_scratch(big_both.flatten(1))
    assert status(lambda: nfad.nfad_expert_gated_backward(big, big_both, off, big_both, gb, scratch[:16])) == 7
    assert status(lambda: nfad.nfad_expert_gated_backward(big, big_both, off, big_both, gb, None)) == 3


@pytest.mark.parametrize("way", [0, 3, 5, 7, 9, 11])
def test_the_same_bits_every_time(way):
    counts, lead, tail, n_in, n_out = WAYS[way]
    x, w, b, off, o = _case(WAYS[way], "bf16", 400 + way)
    first = _forward("mish", x, w, b, off)
    streams = [torch.cuda.Stream() for _ in range(3)]
    dx, dw, db, doff = x.to(DEV), w.to(DEV), b.to(DEV), off.to(DEV)
    torch.cuda.synchronize()
    results = []
    for s in streams:                                                 # three calls at once
        with torch.cuda.stream(s):
            y, both = _nan(x.shape[0], n_out, dtype=x.dtype), _nan(x.shape[0], 2, n_out, dtype=x.dtype)
            nfad.nfad_expert_gated_linear("mish", dx, dw, db, doff, y, both)
            results.append((y, both))
    torch.cuda.synchronize()
    for r in results:
        assert torch.equal(r[0], first[0]) and torch.equal(r[1], first[1])
    assert nfad.nfad_wait_faults() == 0


def test_non_finite_values_take_their_way():
    # an infinity in a row of x makes both projections infinite or NaN there, and nothing elsewhere; a value with the same sign on both sides
    # keeps y = f(a) u what the formula gives
    x, w, b, off, o = _case(([40], 0, 0, 64, 72), "bf16", 7)
    x[3, 5], x[7, 9] = float("inf"), float("nan")
    y, both = (t.cpu() for t in _forward("swish", x, w, b, off))
    assert not torch.isfinite(both[3, 1][w[0, 0, :, 5] > 0]).any() and torch.isnan(y[7]).all() and torch.isnan(both[7]).all()
    keep = [r for r in range(40) if r not in (3, 7)]
    assert torch.isfinite(y[keep]).all()
    gate_up = (w[0, 0, :, 5] > 0) & (w[0, 1, :, 5] > 0)
    assert (y[3][gate_up] == float("inf")).all()
