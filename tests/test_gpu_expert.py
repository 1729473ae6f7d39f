"""Products grouped by expert against plain 64-bit implementations: forward with the nested activation, Eq. 4 with its bias
sums, the input's gradient and the weights' gradient.  Bounds: block_plain.dot_error for a tensor-core sum, the activation's own
accuracy, one rounding to the storage type."""
import pytest
import torch

import block_plain as plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
DTYPES = ["bf16", "f16"]
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
]


def _case(case, dtype, seed):
    counts, lead, tail, n_in, n_out = case
    rows = sum(counts) + lead + tail
    off = [lead]
    for c in counts:
        off.append(off[-1] + c)
    e = len(counts)
    x = W.normal(rows * n_in, dtype, seed, 1.0).view(rows, n_in)
    w = W.normal(e * n_out * n_in, dtype, seed + 1, max(n_in, 1) ** -0.5).view(e, n_out, n_in)
    b = W.normal(e * n_out, dtype, seed + 2, 0.4).view(e, n_out)
    return x, w, b, torch.tensor(off, dtype=torch.int32), off


def _nan_like(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def _forward(kind, x, w, b, off, slope=True):
    y = _nan_like(x.shape[0], w.shape[1], dtype=x.dtype)
    d = torch.full_like(y, float("nan")) if slope and kind is not None else None
    nfad.nfad_expert_linear(kind, x.to(DEV), w.to(DEV), None if b is None else b.to(DEV), off.to(DEV), y, d)
    torch.cuda.synchronize()
    return y, d


def _check_forward(kind, x, w, b, off, y, d):
    y, d = y.cpu(), None if d is None else d.cpu()
    covered = torch.zeros(x.shape[0], dtype=torch.bool)
    for e in range(w.shape[0]):
        p = slice(off[e], off[e + 1])
        covered[p] = True
        if off[e + 1] <= off[e]:
            continue
        z, mag = x[p].double() @ w[e].double().t(), x[p].double().abs() @ w[e].double().abs().t()
        if b is not None:
            z, mag = z + b[e].double(), mag + b[e].double().abs()
        plain.check_act(y[p], None if d is None else d[p], z, plain.dot_error(mag, x.shape[1]), kind, f"expert {e}")
    assert not y[~covered].any() and (d is None or not d[~covered].any()), "rows without an expert"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward(dtype, case):
    x, w, b, off, o = _case(CASES[case], dtype, 10 * case)
    for kind in (None, "gelu_erf", "gelu_tanh", "swish", "mish"):
        for bias in (b, None):
            _check_forward(kind, x, w, bias, o, *_forward(kind, x, w, bias, off))
            _check_forward(kind, x, w, bias, o, *_forward(kind, x, w, bias, off, slope=False))
    assert nfad.nfad_wait_faults() == 0


def _act_backward(g, d, off, experts):
    gz = torch.full_like(g, float("nan"), device=DEV)
    gb = _nan_like(experts, g.shape[1], dtype=torch.float32)
    scratch = nfad.nfad_expert_act_backward_scratch(g.to(DEV)).fill_(0xff)
    nfad.nfad_expert_act_backward(g.to(DEV), None if d is None else d.to(DEV), off.to(DEV), gz, gb, scratch)
    torch.cuda.synchronize()
    return gz.cpu(), gb.cpu()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", list(range(len(CASES))) + ["long"])
def test_act_backward(dtype, case):
    c = ([900, 0, 1, 4000, 3, 20, 700], 11, 13, 8, 264) if case == "long" else CASES[case]
    _, _, _, off, o = _case(c, dtype, 3)
    rows, n_out, experts = o[-1] + c[2], c[4], len(c[0])
    g, d = W.normal(rows * n_out, dtype, 5, 1.0).view(rows, n_out), W.uniform(rows * n_out, dtype, 6, -0.2, 1.1).view(rows, n_out)
    for slope in (d, None):
        gz, gb = _act_backward(g, slope, off, experts)
        for e in range(experts):
            p = slice(o[e], o[e + 1])
            exact = g[p].double() * slope[p].double() if slope is not None else g[p].double()
            assert torch.equal(gz[p], exact.to(gz.dtype)), "one rounding of the product"
            plain.check(gb[e], exact.sum(0), plain.EPS32 * (o[e + 1] - o[e] + 40) * exact.abs().sum(0), f"bias of expert {e}")
        assert not gz[:o[0]].any() and not gz[o[-1]:].any()
        assert torch.equal(gb, _act_backward(g, slope, off, experts)[1])          # the same bits every time


def _backward(gz, x, w, off, prev=None):
    gx = torch.full(x.shape, float("nan"), dtype=x.dtype, device=DEV)
    gw = torch.full(w.shape, float("nan"), dtype=x.dtype, device=DEV)
    dgz, doff = gz.to(DEV), off.to(DEV)
    nfad.nfad_expert_linear_backward_input(dgz, w.to(DEV), doff, None if prev is None else prev.to(DEV), gx)
    nfad.nfad_expert_linear_backward_weight(dgz, x.to(DEV), doff, gw)
    torch.cuda.synchronize()
    return gx.cpu(), gw.cpu()


def _check_backward(gz, x, w, o, prev, gx, gw):
    covered = torch.zeros(x.shape[0], dtype=torch.bool)
    for e in range(w.shape[0]):
        p = slice(o[e], o[e + 1])
        covered[p] = True
        g, we, xe = gz[p].double(), w[e].double(), x[p].double()
        v, m = g @ we, plain.dot_error(g.abs() @ we.abs(), w.shape[1])
        if prev is not None:
            f = prev[p].double()
            v, m = v * f, m * f.abs() + plain.EPS32 * (v * f).abs()
        plain.check(gx[p], v, m, f"grad_x of expert {e}")
        plain.check(gw[e], g.t() @ xe, plain.dot_error(g.abs().t() @ xe.abs(), o[e + 1] - o[e]), f"grad_w of expert {e}")
    assert not gx[~covered].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_backward(dtype, case):
    x, w, _, off, o = _case(CASES[case], dtype, 10 * case + 4)
    gz = W.normal(x.shape[0] * w.shape[1], dtype, 9, 1.0).view(x.shape[0], w.shape[1])
    prev = W.uniform(x.numel(), dtype, 11, -0.2, 1.1).view(x.shape)
    for f in (None, prev):
        _check_backward(gz, x, w, o, f, *_backward(gz, x, w, off, f))
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_tiles(dtype):
    # more tiles than SMs, so that every CTA walks over several; tile widths of each size; more than one ring of stages
    for counts, n_in, n_out in (([2000, 17, 3000, 0, 500], 328, 1544), ([700] * 4, 1096, 520), ([3] * 40, 2048, 1024)):
        x, w, b, off, o = _case((counts, 0, 5, n_in, n_out), dtype, 5)
        _check_forward("swish", x, w, b, o, *_forward("swish", x, w, b, off))
        gz = W.normal(x.shape[0] * n_out, dtype, 9, 1.0).view(x.shape[0], n_out)
        _check_backward(gz, x, w, o, None, *_backward(gz, x, w, off))
    assert nfad.nfad_wait_faults() == 0


# shapes that take the ways through the products which depend on size (B200, 148 SMs): pairs of CTAs on 256 x 256 tiles (each
# product), the reduction split over two, four and eight CTAs, tiles of each width, and few rows
WAYS = [
    ([1100, 700, 800], 0, 0, 2048, 264), ([1101, 701, 900], 1, 3, 1040, 1800), ([600, 1, 900], 0, 0, 1048, 2568),
    ([40, 0, 37], 3, 2, 1288, 136), ([77], 0, 0, 2568, 72), ([33], 0, 0, 5128, 72), ([150], 0, 0, 72, 5128), ([40, 0, 60], 0, 5, 136, 2568),
    ([5203], 0, 0, 72, 136), ([2570, 2571], 0, 1, 136, 72), ([260], 0, 0, 264, 5000), ([9, 0, 17, 3], 1, 2, 1032, 200), ([3, 1, 0, 2] * 40, 0, 0, 264, 136),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_ways(dtype, way):
    x, w, b, off, o = _case(WAYS[way], dtype, 300 + way)
    _check_forward("gelu_erf", x, w, b, o, *_forward("gelu_erf", x, w, b, off))
    _check_forward(None, x, w, None, o, *_forward(None, x, w, None, off))
    gz = W.normal(x.shape[0] * w.shape[1], dtype, 9, 1.0).view(x.shape[0], w.shape[1])
    prev = W.uniform(x.numel(), dtype, 11, -0.2, 1.1).view(x.shape)
    _check_backward(gz, x, w, o, prev, *_backward(gz, x, w, off, prev))
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("counts,n_in,n_out", [(list(range(1, 67)), 264, 136), ([513, 527, 528, 529, 545, 575, 576, 577], 1040, 776)])
def test_runs_that_end_anywhere(dtype, counts, n_in, n_out):
    # the weights' gradient multiplies whole groups of rows: what follows an expert's last row must not reach it
    x, w, _, off, o = _case((counts, 3, 2, n_in, n_out), dtype, 17)
    gz = W.normal(x.shape[0] * n_out, dtype, 9, 1.0).view(x.shape[0], n_out)
    gx, gw = _backward(gz, x, w, off)
    _check_backward(gz, x, w, o, None, gx, gw)
    for third in range(3):
        bad_gz, bad_x = gz.clone(), x.clone()
        bad_gz[:o[0]], bad_x[o[-1]:] = float("nan"), float("inf")
        for e in range(third, len(counts), 3):
            bad_gz[o[e]:o[e + 1]], bad_x[o[e]:o[e + 1]] = float("inf"), float("nan")
        _, got = _backward(bad_gz, bad_x, w, off)
        keep = [e for e in range(len(counts)) if e % 3 != third]
        assert torch.equal(got[keep], gw[keep])
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_neighbours_do_not_mix(dtype):
    # infinities and NaN in one expert's rows and weights stay there: tiles and reduction steps reach into the neighbours
    counts, n_in, n_out = [70, 61, 90], 136, 72
    x, w, b, off, o = _case((counts, 0, 3, n_in, n_out), dtype, 7)
    gz = W.normal(x.shape[0] * n_out, dtype, 9, 1.0).view(x.shape[0], n_out)
    y, d = _forward("gelu_erf", x, w, b, off)
    gx, gw = _backward(gz, x, w, off)
    _, gb = _act_backward(gz, None, off, 3)
    x2, w2, gz2 = x.clone(), w.clone(), gz.clone()
    p = slice(o[1], o[2])
    x2[p], gz2[p], w2[1] = float("nan"), float("inf"), float("nan")
    x2[o[3]:], gz2[o[3]:] = float("nan"), float("nan")               # rows without an expert are not read
    y2, d2 = _forward("gelu_erf", x2, w2, b, off)
    gx2, gw2 = _backward(gz2, x2, w2, off)
    gz_out, gb2 = _act_backward(gz2, None, off, 3)
    others = [i for i in range(x.shape[0]) if not o[1] <= i < o[2]]
    for a, c in ((y, y2), (d, d2), (gx, gx2)):
        assert torch.equal(a[others], c[others])
    assert torch.isnan(y2[p]).all() and torch.isnan(gw2[1]).all()
    assert torch.equal(gw[[0, 2]], gw2[[0, 2]]) and torch.equal(gb[[0, 2]], gb2[[0, 2]])
    assert not gz_out[o[3]:].any()


def test_unaligned_tensors_give_the_same_bits():
    x, w, b, off, o = _case(([40, 0, 150], 0, 2, 64, 72), "bf16", 7)
    gz = W.normal(x.shape[0] * 72, "bf16", 9, 1.0).view(-1, 72)

    def shifted(t):
        buf = torch.zeros(t.numel() + 1, dtype=t.dtype, device=DEV)
        buf[1:].copy_(t.reshape(-1))
        return buf[1:].view(t.shape)

    y, d = _forward("mish", x, w, b, off)
    y2, d2 = shifted(torch.zeros_like(y)), shifted(torch.zeros_like(y))
    nfad.nfad_expert_linear("mish", shifted(x), shifted(w), shifted(b), off.to(DEV), y2, d2)
    assert torch.equal(y, y2) and torch.equal(d, d2)
    gx, gw = _backward(gz, x, w, off)
    gx2, gw2 = shifted(torch.zeros_like(x)), shifted(torch.zeros_like(w))
    nfad.nfad_expert_linear_backward_input(shifted(gz), shifted(w), off.to(DEV), None, gx2)
    nfad.nfad_expert_linear_backward_weight(shifted(gz), shifted(x), off.to(DEV), gw2)
    torch.cuda.synchronize()
    assert torch.equal(gx, gx2.cpu()) and torch.equal(gw, gw2.cpu())


def test_offsets_out_of_range_are_held_inside():
    # not a contract to rely on, but nothing outside the tensors may be touched: values below, above and out of order
    x, w, b, _, _ = _case(([50, 30], 0, 0, 64, 64), "bf16", 7)
    off = torch.tensor([-7, 1 << 30, 20], dtype=torch.int32)
    y, _ = _forward(None, x, w, b, off)
    want, _ = _forward(None, x, w, b, torch.tensor([0, 80, 80], dtype=torch.int32))
    assert torch.equal(y, want)
    gz = W.normal(80 * 64, "bf16", 9, 1.0).view(80, 64)
    gx, gw = _backward(gz, x, w, off)
    assert torch.isfinite(gx.float()).all() and torch.isfinite(gw.float()).all()
    gzo, gb = _act_backward(gz, None, off, 2)
    assert torch.isfinite(gzo.float()).all()


def test_gradient_against_differences():
    # <wy, f(x w^T + b)> along a direction in x, w and b: central differences in 64 bits against the 16-bit gradients
    x, w, b, off, o = _case(([40, 0, 25], 0, 0, 48, 56), "bf16", 7)
    wy = W.normal(x.shape[0] * 56, "bf16", 9, 1.0).view(-1, 56)
    for kind in ("gelu_erf", "gelu_tanh", "swish", "mish"):
        _, d = _forward(kind, x, w, b, off)
        gz, gb = _act_backward(wy, d.cpu(), off, 3)
        gx, gw = _backward(gz, x, w, off)
        dx, dw, db = (W.normal(t.numel(), "f32", 20 + i, 0.3).view(t.shape).double() for i, t in enumerate((x, w, b)))

        def value(t):
            total = 0.0
            for e in range(3):
                p = slice(o[e], o[e + 1])
                z = (x[p].double() + t * dx[p]) @ (w[e].double() + t * dw[e]).t() + b[e].double() + t * db[e]
                total += float((wy[p].double() * plain.act(z, kind)[0]).sum())
            return total

        slope = (value(1e-4) - value(-1e-4)) / 2e-4
        terms = [gx.double() * dx, gw.double() * dw, gb.double() * db]
        got = float(sum(t.sum() for t in terms))
        # f', grad_z and the results are each rounded to 8 bits: three half spacings of 2^-8 of the terms' size, as a random sum
        size = sum(float((t * t).sum()) for t in terms) ** 0.5
        assert abs(got - slope) <= 6 * 3 * 2.0 ** -9 * size + 1e-6 * abs(slope), (kind, got, slope, size)


def test_graph_with_other_offsets():
    x, w, b, off, o = _case(([40, 60, 28], 0, 0, 128, 128), "bf16", 7)
    dx, dw, db, doff = x.to(DEV), w.to(DEV), b.to(DEV), off.to(DEV)
    y = torch.zeros(128, 128, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_expert_linear("swish", dx, dw, db, doff, y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nfad.nfad_expert_linear("swish", dx, dw, db, doff, y)
    for other in ([0, 0, 128, 128], [0, 100, 101, 120]):
        doff.copy_(torch.tensor(other, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        _check_forward("swish", x, w, b, other, y, None)


def test_elements_beyond_32_bits():
    # results, and gradients of the input, whose element offsets pass 2^31: the last rows against the plain form
    rows, n_in, n_out = 270000, 64, 8200
    w, b = W.normal(n_out * n_in, "bf16", 2, 0.125).view(1, n_out, n_in), W.normal(n_out, "bf16", 3, 0.4).view(1, n_out)
    x = torch.zeros(rows, n_in, dtype=torch.bfloat16, device=DEV)
    tail = W.normal(5 * n_in, "bf16", 4, 1.0).view(5, n_in)
    x[-5:] = tail.to(DEV)
    off = torch.tensor([0, rows], dtype=torch.int32)
    y, d = torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV), torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_expert_linear("swish", x, w.to(DEV), b.to(DEV), off.to(DEV), y, d)
    _check_forward("swish", tail, w, b, [0, 5], y[-5:], d[-5:])
    _check_forward("swish", torch.zeros(3, n_in, dtype=torch.bfloat16), w, b, [0, 3], y[100:103], d[100:103])
    gx = torch.empty_like(x)
    nfad.nfad_expert_linear_backward_input(y, w.to(DEV), off.to(DEV), None, gx)
    g = y[-5:].cpu().double()
    plain.check(gx[-5:], g @ w[0].double(), plain.dot_error(g.abs() @ w[0].double().abs(), n_out), "grad_x")
    gz = torch.empty_like(y)
    gb = torch.empty(1, n_out, device=DEV)
    nfad.nfad_expert_act_backward(y, d, off.to(DEV), gz, gb, nfad.nfad_expert_act_backward_scratch(y))
    assert torch.equal(gz[-5:], (y[-5:].double() * d[-5:].double()).bfloat16())
    # gradients of many experts' weights: 2.2e9 elements
    experts, n_in, n_out = 1024, 1024, 2056
    gw = torch.full((experts, n_out, n_in), float("nan"), dtype=torch.bfloat16, device=DEV)
    x, gz = W.normal(8 * n_in, "bf16", 5, 1.0).view(8, n_in), W.normal(8 * n_out, "bf16", 6, 1.0).view(8, n_out)
    off = torch.zeros(experts + 1, dtype=torch.int32)
    off[-1] = 8
    nfad.nfad_expert_linear_backward_weight(gz.to(DEV), x.to(DEV), off.to(DEV), gw)
    plain.check(gw[-1], gz.double().t() @ x.double(), plain.dot_error(gz.double().abs().t() @ x.double().abs(), 8), "grad_w")
    assert not gw[:-1].any()


def test_most_experts():
    counts = [1 if i % 3 else 0 for i in range(1024)]
    x, w, b, off, o = _case((counts, 0, 0, 16, 24), "bf16", 7)
    _check_forward("swish", x, w, b, o, *_forward("swish", x, w, b, off))
    gz = W.normal(x.shape[0] * 24, "bf16", 9, 1.0).view(-1, 24)
    _check_backward(gz, x, w, o, None, *_backward(gz, x, w, off))


def test_no_rows_and_no_reduction():
    x, w, b, off, o = _case(([0, 0], 0, 0, 32, 40), "bf16", 7)
    y, d = _forward("swish", x, w, b, off)
    assert y.shape == (0, 40)
    gz = torch.empty(0, 40, dtype=torch.bfloat16)
    gx, gw = _backward(gz, x, w, off)
    assert not gw.any()
    gzo, gb = _act_backward(gz, None, off, 2)
    assert not gb.any()
    x, w, b, off, o = _case(([10, 5], 0, 0, 0, 40), "bf16", 7)
    _check_forward("swish", x, w, b, o, *_forward("swish", x, w, b, off))


def test_refusals():
    x, w, b, off, _ = (t.to(DEV) if isinstance(t, torch.Tensor) else t for t in _case(([10, 5], 0, 0, 16, 24), "bf16", 7))
    y = torch.empty(15, 24, dtype=torch.bfloat16, device=DEV)

    def status(fn):
        with pytest.raises(nfad.NfadError) as e:
            fn()
        return e.value.status

    assert status(lambda: nfad.nfad_expert_linear(7, x, w, b, off, y)) == 1
    assert status(lambda: nfad.nfad_expert_linear("swish", x.float(), w.float(), b.float(), off, y.float())) == 2
    assert status(lambda: nfad.nfad_expert_linear(None, x, w, b, off, y, torch.empty_like(y))) == 11
    assert status(lambda: nfad.nfad_expert_linear("swish", x, w, b, off, y, y)) == 4
    many = torch.zeros(1026, dtype=torch.int32, device=DEV)
    assert status(lambda: nfad.nfad_expert_linear("swish", x, torch.zeros(1025, 24, 16, dtype=torch.bfloat16, device=DEV), None, many, y)) == 9
    for bad in (lambda: nfad.nfad_expert_linear("swish", x, w[:, :, :8], b, off, y), lambda: nfad.nfad_expert_linear("swish", x, w, b[:1], off, y),
                lambda: nfad.nfad_expert_linear("swish", x, w, b, off[:2], y), lambda: nfad.nfad_expert_linear("swish", x, w, b, off, y[:, :8]),
                lambda: nfad.nfad_expert_linear("swish", x, w.transpose(1, 2).contiguous().transpose(1, 2), b, off, y),
                lambda: nfad.nfad_expert_linear_backward_weight(y, x[:4], off, w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        nfad.nfad_expert_linear("swish", x, w, b, off.long(), y)
    with pytest.raises(ValueError):
        nfad.nfad_expert_linear("swish", x, w.half(), b, off, y)
    gb = torch.empty(2, 24, device=DEV)
    big = torch.zeros(4000, 24, dtype=torch.bfloat16, device=DEV)
    scratch = nfad.nfad_expert_act_backward_scratch(big)
    assert status(lambda: nfad.nfad_expert_act_backward(big, None, off, None, gb, scratch[:16])) == 7
    assert status(lambda: nfad.nfad_expert_act_backward(big, None, off, None, gb, None)) == 3


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [24, 25, 1416])
@pytest.mark.parametrize("off", [[0, 60, 20, 80], [0, 10, 5, 20], [5, 3, 10], [70, 0, 80], [-7, 1 << 30, 20], [40, 30, 20, 10], [0, 600, 200, 900, 100, 1500, 2600],
                                 [0] + [100, 40] * 300 + [2500], [3000, 0, 5]])
def test_offsets_out_of_order_mean_the_same_everywhere(dtype, cols, off):
    # an expert begins no earlier than the largest offset before it, in Eq. 4 and its bias sums as in the products
    rows = 80 if len(off) < 5 and max(off) <= 80 else 2600
    held, last = [], 0
    for v in off:
        last = max(last, min(max(v, 0), rows))
        held.append(last)
    experts = len(off) - 1
    g, d = W.normal(rows * cols, dtype, 15, 1.0).view(rows, cols), W.uniform(rows * cols, dtype, 16, -0.2, 1.1).view(rows, cols)
    exact = g.double() * d.double()
    gz, gb = _act_backward(g, d, torch.tensor(off, dtype=torch.int32), experts)
    assert torch.equal(gz[held[0]:held[-1]], exact[held[0]:held[-1]].to(gz.dtype))
    assert not gz[:held[0]].any() and not gz[held[-1]:].any()
    for e in range(experts):
        part = exact[held[e]:held[e + 1]]
        plain.check(gb[e], part.sum(0), plain.EPS32 * (part.shape[0] + 40) * part.abs().sum(0), f"bias of expert {e}")
    gz2, gb2 = _act_backward(g, d, torch.tensor(held, dtype=torch.int32), experts)
    assert torch.equal(gz, gz2) and torch.equal(gb, gb2)
    # the products' rows of the same offsets
    x = W.normal(rows * 16, dtype, 17, 1.0).view(rows, 16)
    w = W.normal(experts * cols * 16, dtype, 18, 0.25).view(experts, cols, 16)
    a, b = (_backward(gz, x, w, torch.tensor(o, dtype=torch.int32)) for o in (off, held))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ya, yb = (_forward("swish", x, w, None, torch.tensor(o, dtype=torch.int32)) for o in (off, held))
    assert torch.equal(ya[0], yb[0]) and torch.equal(ya[1], yb[1])
