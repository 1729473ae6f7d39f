"""The linear layer in 8-bit integers against plain implementations: the quantiser's integers are exact, the products' sums are
exact, and what follows them (two scales, bias, activation) is held to fp32 roundings and one rounding to the storage type."""
import numpy as np
import pytest
import torch

import block_plain as plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
ACTS = [None, "gelu_erf", "gelu_tanh", "swish", "mish"]
# rows, in, out: single tokens, few, a tile and its borders, many tiles; odd sizes (gathered); in a multiple of 4 and of 8 only
SHAPES = [(1, 64, 64), (1, 4096, 1000), (2, 1040, 136), (3, 48, 24), (4, 2064, 520), (5, 128, 40), (8, 512, 256), (9, 512, 264), (16, 1024, 2048),
          (17, 96, 8), (64, 256, 320), (127, 144, 48), (128, 128, 128), (129, 1024, 512), (300, 2048, 1000), (1, 37, 51), (7, 33, 20), (3, 1001, 77),
          (130, 100, 44), (20, 24, 8), (1, 1, 1), (40, 16, 1), (1, 5000, 3), (2, 20000, 40),
          # the reduction over eight, four and two CTAs, one tile for each of two CTAs of an SM, pairs
          (40, 10256, 72), (77, 5136, 136), (60, 2576, 200), (130, 272, 5120), (2600, 272, 2056)]


def quantize(x):
    """The quantiser's definition, every operation rounded to fp32 as stated: q = rint(x (127 / amax)), scale = amax / 127."""
    v = x.float().numpy()
    amax = np.abs(v).max(1) if v.shape[1] else np.zeros(v.shape[0], np.float32)
    zero, bad = amax < np.float32(2.0 ** -120), ~np.isfinite(amax)
    with np.errstate(all="ignore"):
        q = np.rint(v * (np.float32(127) / amax)[:, None])           # numpy: one IEEE division, one product, ties to even
        q[zero | bad] = 0
        scale = np.where(bad, np.float32("nan"), np.where(zero, np.float32(0), amax / np.float32(127)))
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale.astype(np.float32))


def _quantize(x):
    q = torch.full(x.shape, 99, dtype=torch.int8, device=DEV)
    s = torch.full(x.shape[:1], -1.0, device=DEV)
    nfad.nfad_i8_quantize_rows(x.to(DEV), q, s)
    torch.cuda.synchronize()
    return q.cpu(), s.cpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quantizer(dtype):
    for i, (rows, cols) in enumerate([(1, 1), (3, 7), (5, 64), (2, 1000), (4, 4096), (300, 520), (2, 40001), (9, 200), (17, 256), (5, 512), (3, 1024), (4, 2056), (3, 8192), (2, 12000)]):
        x = W.normal(rows * cols, dtype, i, 1.5).view(rows, cols)
        q, s = _quantize(x)
        wq, ws = quantize(x)
        assert torch.equal(q, wq) and torch.equal(s, ws)
        assert q.abs().max() == 127
    # rows of zeros, of subnormals, with one infinity, with a NaN, at the type's largest
    x = W.normal(6 * 256, dtype, 9, 1.0).view(6, 256)
    x[0] = 0
    x[1] = 1e-39 if dtype != "f16" else 0
    x[2, 3], x[3, 200] = float("inf"), float("nan")
    x[4] *= torch.finfo(x.dtype).max / 8
    q, s = _quantize(x)
    wq, ws = quantize(x)
    assert torch.equal(q, wq) and torch.equal(s.nan_to_num(-7), ws.nan_to_num(-7))
    assert torch.isnan(s[2]) and torch.isnan(s[3]) and s[0] == 0


def _check(kind, q, xs, wq, ws, bias, y):
    dot = (q.double() @ wq.double().t())                              # exact: below 2^53
    z = dot * xs.double()[:, None] * ws.double()
    # int to fp32, the two scales' product, that times the sum, and the bias: four roundings
    mag = z.abs()
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    plain.check_act(y.cpu(), None, z, 4 * plain.EPS32 * mag, kind, "y")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_linear(dtype, shape):
    rows, n_in, n_out = SHAPES[shape]
    g = torch.Generator().manual_seed(shape)
    q = torch.randint(-128, 128, (rows, n_in), generator=g, dtype=torch.int8)
    wq = torch.randint(-128, 128, (n_out, n_in), generator=g, dtype=torch.int8)
    xs, ws = torch.rand(rows, generator=g) * 0.02, torch.rand(n_out, generator=g) * 0.01
    bias = W.normal(n_out, dtype, shape + 1, 0.5)
    for kind in ACTS:
        for b in (bias, None):
            y = torch.full((rows, n_out), float("nan"), dtype=W.TORCH_DTYPES[dtype], device=DEV)
            nfad.nfad_i8_linear(kind, q.to(DEV), xs.to(DEV), wq.to(DEV), ws.to(DEV), None if b is None else b.to(DEV), y)
            torch.cuda.synchronize()
            _check(kind, q, xs, wq, ws, b, y)
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_dynamic(dtype, shape):
    rows, n_in, n_out = SHAPES[shape]
    x = W.normal(rows * n_in, dtype, shape, 1.5).view(rows, n_in)
    w = W.normal(n_out * n_in, "f32", shape + 50, n_in ** -0.5).view(n_out, n_in)
    wq, ws = _quantize(w)
    bias = W.normal(n_out, dtype, shape + 1, 0.5)
    q, xs = quantize(x)
    dx = x.to(DEV)
    scratch = nfad.nfad_i8_linear_dynamic_scratch(dx).fill_(0x7f)
    for kind in (None, "swish"):
        y = torch.full((rows, n_out), float("nan"), dtype=dx.dtype, device=DEV)
        nfad.nfad_i8_linear_dynamic(kind, dx, wq.to(DEV), ws.to(DEV), bias.to(DEV), y, scratch)
        torch.cuda.synchronize()
        _check(kind, q, xs, wq, ws, bias, y)


@pytest.mark.parametrize("rows", [3, 140])
def test_bad_rows_stay_by_themselves(rows):
    n_in, n_out = 256, 64
    x = W.normal(rows * n_in, "bf16", 1, 1.0).view(rows, n_in)
    wq, ws = _quantize(W.normal(n_out * n_in, "f32", 2, 0.1).view(n_out, n_in))
    out = []
    for bad in (False, True):
        t = x.clone()
        if bad:
            t[0, 9], t[2, 17] = float("inf"), float("nan")
            t[1] = 0
        dx = t.to(DEV)
        y = torch.zeros(rows, n_out, dtype=torch.bfloat16, device=DEV)
        nfad.nfad_i8_linear_dynamic("gelu_erf", dx, wq.to(DEV), ws.to(DEV), None, y, nfad.nfad_i8_linear_dynamic_scratch(dx))
        torch.cuda.synchronize()
        out.append(y)
    assert torch.isnan(out[1][0]).all() and torch.isnan(out[1][2]).all() and not out[1][1].any()
    assert torch.equal(out[0][3:], out[1][3:])


def test_largest_sums():
    # the longest reduction whose sum of -128 * -128 still fits 32 bits
    n_in = 131071
    q = torch.full((2, n_in), -128, dtype=torch.int8, device=DEV)
    w = torch.full((3, n_in), -128, dtype=torch.int8, device=DEV)
    one = torch.ones(3, device=DEV)
    y = torch.zeros(2, 3, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_i8_linear(None, q, one[:2], w, one, None, y)
    assert (y == torch.tensor(float(n_in * 16384)).bfloat16().to(DEV)).all()
    qa = torch.full((2, 131056), -128, dtype=torch.int8, device=DEV)     # the same through the tensor copies
    wa = torch.full((3, 131056), -128, dtype=torch.int8, device=DEV)
    nfad.nfad_i8_linear(None, qa, one[:2], wa, one, None, y)
    assert (y == torch.tensor(float(131056 * 16384)).bfloat16().to(DEV)).all()


def test_graph_and_other_stream():
    x = W.normal(4 * 512, "bf16", 1, 1.0, DEV).view(4, 512)
    wq, ws = (t.to(DEV) for t in _quantize(W.normal(256 * 512, "f32", 2, 0.1).view(256, 512)))
    scratch = nfad.nfad_i8_linear_dynamic_scratch(x)
    y, y2 = (torch.zeros(4, 256, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        nfad.nfad_i8_linear_dynamic("swish", x, wq, ws, None, y, scratch)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nfad.nfad_i8_linear_dynamic("swish", x, wq, ws, None, y2, scratch)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and y.any()


def test_empty():
    wq, ws = torch.zeros(8, 0, dtype=torch.int8, device=DEV), torch.ones(8, device=DEV)
    x = torch.zeros(3, 0, dtype=torch.bfloat16, device=DEV)
    b = W.normal(8, "bf16", 1, 1.0, DEV)
    y = torch.zeros(3, 8, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_i8_linear_dynamic(None, x, wq, ws, b, y, nfad.nfad_i8_linear_dynamic_scratch(x))
    torch.cuda.synchronize()
    assert torch.equal(y, b.expand(3, 8))
    e = torch.zeros(0, 8, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_i8_linear(None, torch.zeros(0, 16, dtype=torch.int8, device=DEV), torch.zeros(0, device=DEV), torch.zeros(8, 16, dtype=torch.int8, device=DEV), ws, b, e)


def test_refusals():
    x = torch.zeros(4, 32, dtype=torch.bfloat16, device=DEV)
    q, xs = torch.zeros(4, 32, dtype=torch.int8, device=DEV), torch.zeros(4, device=DEV)
    wq, ws = torch.zeros(16, 32, dtype=torch.int8, device=DEV), torch.zeros(16, device=DEV)
    y = torch.zeros(4, 16, dtype=torch.bfloat16, device=DEV)
    scratch = nfad.nfad_i8_linear_dynamic_scratch(x)

    def status(fn):
        with pytest.raises(nfad.NfadError) as e:
            fn()
        return e.value.status

    assert status(lambda: nfad.nfad_i8_linear(4, q, xs, wq, ws, None, y)) == 1
    assert status(lambda: nfad.nfad_i8_linear(None, q, xs, wq, ws, None, y.float())) == 2
    assert status(lambda: nfad.nfad_i8_linear_dynamic(None, x, wq, ws, None, y, scratch[:32])) == 7
    assert status(lambda: nfad.nfad_i8_linear_dynamic(None, x, wq, ws, None, y, scratch[1:])) == 6
    n = 131072
    assert status(lambda: nfad.nfad_i8_linear(None, torch.zeros(4, n, dtype=torch.int8, device=DEV), xs, torch.zeros(16, n, dtype=torch.int8, device=DEV), ws, None, y)) == 9
    with pytest.raises(ValueError):
        nfad.nfad_i8_linear(None, q, xs, wq[:, :16], ws, None, y)
    with pytest.raises(ValueError):
        nfad.nfad_i8_linear(None, q, xs, wq, ws, None, y[:, :8])
    with pytest.raises(TypeError):
        nfad.nfad_i8_linear(None, q, xs, wq.to(torch.uint8), ws, None, y)
    with pytest.raises(TypeError):
        nfad.nfad_i8_linear(None, q.cpu(), xs, wq, ws, None, y)
