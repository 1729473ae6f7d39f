"""The linear layer in 8-bit floating point by blocks of 128 against plain implementations: the quantisers' values are exact, products
of 8-bit values are exact, and their sums, scales, bias and activation are held to fp32 roundings and one rounding to the storage type."""
import pytest
import torch

import block_plain as plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV, F8, SIDE, TOP = "cuda", torch.float8_e4m3fn, 128, 448.0
ACTS = [None, "gelu_erf", "gelu_tanh", "swish", "mish"]
# rows, in, out: single tokens, few, a tile and its borders, many tiles; blocks that end inside; odd sizes (gathered)
SHAPES = [(1, 64, 64), (1, 4096, 1000), (2, 1040, 136), (3, 48, 24), (4, 2064, 520), (5, 128, 40), (8, 512, 256), (9, 528, 264), (16, 1024, 2048),
          (17, 96, 8), (64, 256, 320), (127, 144, 48), (128, 128, 128), (129, 1024, 512), (300, 2048, 1000), (1, 37, 51), (7, 33, 20), (3, 1001, 77),
          (130, 100, 44), (20, 24, 8), (1, 1, 1), (40, 16, 1), (1, 5000, 3), (2, 20000, 40), (70, 1016, 392), (33, 272, 70),
          # the reduction over eight, four and two CTAs, one tile for each of two CTAs of an SM, single CTAs of both widths, pairs
          (40, 10256, 72), (77, 5136, 136), (60, 2576, 200), (130, 272, 5120), (1000, 400, 1500), (2600, 272, 2056)]


def to_f8(v):
    """Nearest value of the type, ties to even, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return ((v / step).round() * step).clamp(-TOP, TOP)


def _blocks(n):
    return -(-n // SIDE)


def _cut(x, side_rows):
    """x [matrices, rows, cols] by blocks: [matrices, row blocks, side_rows, column blocks, 128], padded with zeros."""
    e, n, k = x.shape
    pad = torch.zeros(e, -(-n // side_rows) * side_rows, _blocks(k) * SIDE, dtype=x.dtype)
    pad[:, :n, :k] = x
    return pad.view(e, -1, side_rows, _blocks(k), SIDE)


def quantize(x, side_rows):
    """The definition: (values, scales [matrices, row blocks, column blocks]) of x [matrices, rows, cols]."""
    cut = _cut(x, side_rows)
    amax = cut.abs().amax((2, 4), keepdim=True)
    zero, bad = amax.double() < 2.0 ** -110, ~torch.isfinite(amax)
    if x.dtype == torch.float32:
        ratio = (cut * (torch.tensor(TOP) / amax)).double()           # two fp32 roundings
    else:
        ratio = cut.double() * TOP / amax.double()                    # the exact quotient, or its nearest in 64 bits
    q = to_f8(ratio).masked_fill((zero | bad).expand_as(cut), 0.0)
    scale = (amax.float() / TOP).masked_fill(zero, 0.0).masked_fill(bad, float("nan"))
    n, k = x.shape[1:]
    return q.reshape(q.shape[0], -1, _blocks(k) * SIDE)[:, :n, :k].float(), scale[:, :, 0, :, 0]


def _quantize_rows(x):
    q = torch.full(x.shape, 3.0, device=DEV).to(F8)
    s = torch.full((_blocks(x.shape[1]), x.shape[0]), -1.0, device=DEV)
    nfad.nfad_f8_quantize_rows(x.to(DEV), q, s)
    torch.cuda.synchronize()
    return q.cpu(), s.cpu()


def _quantize_blocks(x):
    q = torch.full(x.shape, 3.0, device=DEV).to(F8)
    s = torch.full((*x.shape[:-2], _blocks(x.shape[-2]), _blocks(x.shape[-1])), -1.0, device=DEV)
    nfad.nfad_f8_quantize_blocks(x.to(DEV), q, s)
    torch.cuda.synchronize()
    return q.cpu(), s.cpu()


def _same(q, s, wq, ws):
    assert torch.equal(q.float(), wq), (q.float() != wq).sum()
    assert torch.equal(s.nan_to_num(-7), ws.nan_to_num(-7))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quantizers(dtype):
    for i, (rows, cols) in enumerate([(1, 1), (3, 7), (5, 64), (2, 1000), (4, 4096), (300, 520), (2, 40001), (129, 200), (17, 256), (5, 132), (260, 1160), (1, 129)]):
        x = W.normal(rows * cols, dtype, i, 1.5).view(rows, cols)
        wq, ws = quantize(x[None], 1)
        _same(*_quantize_rows(x), wq[0], ws[0].t())
        _same(*_quantize_blocks(x), *(v[0] for v in quantize(x[None], SIDE)))
        assert wq.abs().max() == TOP
    for shape in ((3, 40, 136), (2, 130, 264), (4, 1, 5)):
        x = W.normal(shape[0] * shape[1] * shape[2], dtype, 5, 1.5).view(shape)
        _same(*_quantize_blocks(x), *quantize(x, SIDE))
        _same(*_quantize_blocks(x.view(2, -1, *shape[1:]) if shape[0] == 4 else x[None]), *((v.view(2, 2, *v.shape[1:]) if shape[0] == 4 else v[None]) for v in quantize(x, SIDE)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quotients_on_a_border(dtype):
    # every significand against largest magnitudes of every significand: exact quotients halfway between two values go to the even one
    bits = 7 if dtype == "bf16" else 10
    t = torch.bfloat16 if dtype == "bf16" else torch.float16
    mine = torch.arange(2 ** bits, 2 ** (bits + 1), dtype=torch.float32)
    tops = mine if dtype == "bf16" else torch.cat([mine[::7], mine[mine % 7 == 0]])
    n = mine.numel() // 2
    for shift in (0, 1, 3, 9):
        x = torch.zeros(tops.numel(), _blocks(2 * n) * SIDE)
        # below the block's largest; those above it come with the next smaller exponent
        v = torch.where(mine[None] <= tops[:, None], mine[None], mine[None] / 2) * 2.0 ** -shift
        # each block of 128 begins with the row's largest magnitude
        cut = torch.cat([v, torch.zeros(tops.numel(), -v.shape[1] % 127)], 1).view(tops.numel(), -1, 127)
        x = torch.cat([tops[:, None, None].expand(-1, cut.shape[1], 1), cut], 2).reshape(tops.numel(), -1).to(t)
        wq, ws = quantize(x[None], 1)
        _same(*_quantize_rows(x), wq[0], ws[0].t())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quantizers_special_values(dtype):
    # blocks of zeros, of subnormals, with one infinity, with a NaN, at the type's largest: each by itself
    x = W.normal(7 * 384, dtype, 9, 1.0).view(7, 384)
    x[0, 128:256] = 0
    x[1, :128] = 1e-39 if dtype != "f16" else 0
    x[2, 3], x[3, 200] = float("inf"), float("nan")
    x[4, 256:] *= torch.finfo(x.dtype).max / 8
    x[5, :] *= 1e-4
    x[6, 130] = -torch.finfo(x.dtype).max
    wq, ws = quantize(x[None], 1)
    q, s = _quantize_rows(x)
    _same(q, s, wq[0], ws[0].t())
    assert torch.isnan(s[0, 2]) and torch.isnan(s[1, 3]) and s[1, 0] == 0 and torch.isfinite(s[1:, 2]).all()
    for block in (x[:3, :200], x[4:, 130:]):
        _same(*_quantize_blocks(block.contiguous()), *(v[0] for v in quantize(block[None], SIDE)))


def _spread(scale, n, k):
    return scale.repeat_interleave(SIDE, -2)[..., :n, :].repeat_interleave(SIDE, -1)[..., :k]


def _sums(xq, xs, wq, ws):
    """z and its error: products of 8-bit values are exact, 128 of them are summed by the tensor cores, and the blocks' sums, times a
    product of two scales, by fp32 multiply-adds."""
    n, k = wq.shape
    x, w = xq.double() * xs.double().t().repeat_interleave(SIDE, 1)[:, :k], wq.double() * _spread(ws.double(), n, k)
    z, mag = x @ w.t(), x.abs() @ w.abs().t()
    return z, plain.dot_error(mag, SIDE) + plain.EPS32 * (_blocks(k) + 10) * mag, mag


def _check(kind, xq, xs, wq, ws, bias, y):
    if wq.dim() == 2:
        z, err, mag = _sums(xq, xs, wq, ws)
        if bias is not None:
            z, err = z + bias.double(), err + plain.EPS32 * (mag + bias.double().abs())
        plain.check_act(y.cpu(), None, z, err, kind, "y")
        return
    (a, ea), (u, eu) = ((z + (0 if bias is None else bias[j].double()), err + (0 if bias is None else plain.EPS32 * (mag + bias[j].double().abs())))
                        for j, (z, err, mag) in enumerate(_sums(xq, xs, wq[j], ws[j]) for j in (0, 1)))
    f, _ = plain.act(a, kind)
    ef = (plain.SLOPE if kind else 1.0) * ea + (plain.half_ulp(f, y.dtype) if kind else 0.0)
    plain.check(y, f * u, u.abs() * ef + f.abs() * eu + ef * eu + plain.EPS32 * (f * u).abs(), "y")


def _case(rows, n_in, n_out, gated, seed):
    g = torch.Generator().manual_seed(seed)
    lead = (2,) if gated else ()
    xq, wq = (torch.randn(s, generator=g).mul_(60).clamp_(-TOP, TOP).to(F8) for s in ((rows, n_in), (*lead, n_out, n_in)))
    xs = torch.rand(_blocks(n_in), rows, generator=g) * 0.03 + 1e-3
    ws = (torch.rand(*lead, _blocks(n_out), _blocks(n_in), generator=g) * 0.03 + 1e-3) * max(n_in, 1) ** -0.5
    return xq, xs, wq, ws


def _run(kind, xq, xs, wq, ws, bias, dtype):
    call = nfad.nfad_f8_linear if wq.dim() == 2 else nfad.nfad_f8_gated_linear
    y = torch.full((xq.shape[0], wq.shape[-2]), float("nan"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float16, device=DEV)
    call(kind, xq.to(DEV), xs.to(DEV), wq.to(DEV), ws.to(DEV), None if bias is None else bias.to(DEV), y)
    torch.cuda.synchronize()
    return y


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_linear(dtype, shape, gated):
    rows, n_in, n_out = SHAPES[shape]
    xq, xs, wq, ws = _case(rows, n_in, n_out, gated, shape)
    bias = W.normal(2 * n_out, dtype, 1, 0.5).view(2, n_out)
    bias = bias if gated else bias[0].contiguous()
    for kind in ACTS:
        for b in (bias, None):
            _check(kind, xq, xs, wq, ws, b, _run(kind, xq, xs, wq, ws, b, dtype))
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 512, 256), (7, 300, 130), (40, 2064, 200), (300, 512, 520), (2600, 272, 1032)])
def test_sums_are_exact_where_they_can_be(rows, n_in, n_out):
    # small integers and scales that are powers of two: every partial sum is an integer times a power of two that fp32 holds
    g = torch.Generator().manual_seed(3)
    for gated in (False, True):
        lead = (2,) if gated else ()
        xq, wq = (torch.randint(-8, 9, s, generator=g).float().to(F8) for s in ((rows, n_in), (*lead, n_out, n_in)))
        xs = torch.exp2(torch.randint(-2, 3, (_blocks(n_in), rows), generator=g).float())
        ws = torch.exp2(torch.randint(-2, 3, (*lead, _blocks(n_out), _blocks(n_in)), generator=g).float())
        y = _run(None, xq, xs, wq, ws, None, "bf16").cpu()
        parts = [_sums(xq, xs, w, s)[0] for w, s in (zip(wq, ws) if gated else ((wq, ws),))]
        assert max(p.abs().max().item() for p in parts) < 2 ** 19
        want = parts[0].float() * parts[1].float() if gated else parts[0].float()
        assert torch.equal(y, want.bfloat16())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 4096, 520), (3, 1000, 256), (16, 136, 72), (77, 1040, 136), (200, 513, 65), (700, 1024, 392)])
def test_dynamic(dtype, rows, n_in, n_out, gated):
    x = W.normal(rows * n_in, dtype, 2, 1.0).view(rows, n_in)
    lead = (2,) if gated else ()
    w = W.normal(2 * n_out * n_in, "f32", 3, n_in ** -0.5).view(2, n_out, n_in)
    w = w if gated else w[0].contiguous()
    wq, ws = _quantize_blocks(w)
    xq, xs = _quantize_rows(x)
    bias = W.normal(2 * n_out, dtype, 1, 0.5).view(2, n_out)
    bias = bias if gated else bias[0].contiguous()
    call = nfad.nfad_f8_gated_linear_dynamic if gated else nfad.nfad_f8_linear_dynamic
    y = torch.full((rows, n_out), float("nan"), dtype=x.dtype, device=DEV)
    dx = x.to(DEV)
    call("swish", dx, wq.to(DEV), ws.to(DEV), bias.to(DEV), y, nfad.nfad_f8_linear_dynamic_scratch(dx).fill_(0xff))
    torch.cuda.synchronize()
    assert torch.equal(y, _run("swish", xq, xs, wq, ws, bias, dtype))
    _check("swish", xq, xs, wq, ws, bias, y)


@pytest.mark.parametrize("rows", [1, 5, 40, 300])
def test_what_is_not_finite_stays_in_its_row_or_column(rows):
    n_in, n_out = 640, 264
    for gated in (False, True):
        xq, xs, wq, ws = _case(rows, n_in, n_out, gated, 5)
        y = _run(None, xq, xs, wq, ws, None, "bf16")
        bad_s, bad_q = xs.clone(), xq.clone()
        bad_s[2, rows // 2] = float("nan")
        got = _run(None, xq, bad_s, wq, ws, None, "bf16")
        keep = [r for r in range(rows) if r != rows // 2]
        assert torch.isnan(got[rows // 2]).all() and torch.equal(got[keep], y[keep])
        bad_q[rows // 2, 3] = float("nan")
        got = _run(None, bad_q, xs, wq, ws, None, "bf16")
        assert torch.isnan(got[rows // 2]).all() and torch.equal(got[keep], y[keep])
        bad_w = wq.clone()
        bad_w[..., n_out - 1, 7] = float("nan")
        got = _run(None, xq, xs, bad_w, ws, None, "bf16")
        assert torch.isnan(got[:, -1]).all() and torch.equal(got[:, :-1], y[:, :-1])
        bad_ws = ws.clone()
        bad_ws[..., 1, 0] = float("inf")                              # the second block of outputs
        got = _run(None, xq, xs, wq, bad_ws, None, "bf16")
        assert not torch.isfinite(got[:, 128:256]).any() and torch.equal(got[:, :128], y[:, :128]) and torch.equal(got[:, 256:], y[:, 256:])


def test_unaligned_tensors_give_the_same_bits():
    for rows, gated in ((2, False), (50, True), (200, False)):
        xq, xs, wq, ws = _case(rows, 256, 136, gated, 6)
        b = W.normal((2 if gated else 1) * 136, "bf16", 1, 0.5).view((2, 136) if gated else (136,))

        def shifted(t, by=1):
            buf = torch.zeros(t.numel() + by, dtype=t.dtype, device=DEV)
            buf[by:].copy_(t.reshape(-1))
            return buf[by:].view(t.shape)

        y = _run("mish", xq, xs, wq, ws, b, "bf16")
        call = nfad.nfad_f8_gated_linear if gated else nfad.nfad_f8_linear
        for a, c in ((shifted(xq, 1), wq.to(DEV)), (xq.to(DEV), shifted(wq, 3)), (shifted(xq, 8), shifted(wq, 5))):
            y2 = shifted(torch.zeros_like(y))
            call("mish", a, shifted(xs), c, shifted(ws), shifted(b), y2)
            z = (y.float() - y2.float()).abs()
            # the gather's tiles add the blocks in the same order, few rows and split reductions in another
            assert torch.equal(y, y2) or bool((z <= 2.0 ** -7 * y.float().abs() + 1e-5).all())
        x = W.normal(9 * 136, "bf16", 2, 1.0).view(9, 136)
        q, s = torch.empty(9, 136, dtype=F8, device=DEV), torch.empty(2, 9, device=DEV)
        q2, s2 = shifted(torch.zeros(9, 136).to(F8), 1), shifted(torch.zeros(2, 9), 1)
        nfad.nfad_f8_quantize_rows(x.to(DEV), q, s)
        nfad.nfad_f8_quantize_rows(shifted(x), q2, s2)
        assert torch.equal(q.float(), q2.float()) and torch.equal(s, s2)


def test_graph_and_another_stream():
    x = W.normal(33 * 512, "bf16", 2, 1.0).view(33, 512).to(DEV)
    w = W.normal(2 * 264 * 512, "bf16", 3, 0.05).view(2, 264, 512).to(DEV)
    wq, ws = torch.empty(w.shape, dtype=F8, device=DEV), torch.empty(2, 3, 4, device=DEV)
    nfad.nfad_f8_quantize_blocks(w, wq, ws)
    y, scratch = torch.empty(33, 264, dtype=torch.bfloat16, device=DEV), nfad.nfad_f8_linear_dynamic_scratch(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        nfad.nfad_f8_gated_linear_dynamic("swish", x, wq, ws, None, y, scratch)
    side.synchronize()
    want = y.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nfad.nfad_f8_gated_linear_dynamic("swish", x, wq, ws, None, y, scratch)
    other = W.normal(33 * 512, "bf16", 8, 1.0).view(33, 512).to(DEV)
    first = x.clone()
    x.copy_(other)
    g.replay()
    torch.cuda.synchronize()
    assert not torch.equal(y, want)
    x.copy_(first)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_elements_beyond_32_bits():
    # results whose element offsets pass 2^31, and weights of more than 2^31 bytes
    rows, n_in, n_out = 530000, 32, 4104
    xq, xs, wq, ws = _case(5, n_in, n_out, False, 8)
    big, bs = torch.zeros(rows, n_in, device=DEV).to(F8), torch.ones(1, rows, device=DEV)
    big[-5:], bs[:, -5:] = xq.to(DEV), xs.to(DEV)
    y = torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_f8_linear(None, big, bs, wq.to(DEV), ws.to(DEV), None, y)
    _check(None, xq, xs, wq, ws, None, y[-5:])
    assert not y[:100].any()
    del y, big
    n_in, n_out = 16384, 132000
    w = torch.zeros(n_out, n_in, dtype=torch.uint8, device=DEV).view(F8)
    tail, ts = _case(1, n_in, 300, False, 9)[2:]
    w[-300:] = tail.to(DEV)
    s = torch.ones(_blocks(n_out), _blocks(n_in), device=DEV)
    at = (n_out - 300) // SIDE                                        # the first block with values: its scales are one
    for rows in (1, 40):
        xq, xs = _case(rows, n_in, 8, False, 10)[:2]
        y = torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV)
        nfad.nfad_f8_linear(None, xq.to(DEV), xs.to(DEV), w, s, None, y)
        _check(None, xq, xs, tail, torch.ones(_blocks(300), _blocks(n_in)), None, y[:, -300:])
        assert not y[:, :at * SIDE].any()


def test_no_rows_and_no_reduction():
    for gated in (False, True):
        xq, xs, wq, ws = _case(0, 64, 40, gated, 1)
        assert _run("swish", xq, xs, wq, ws, None, "bf16").shape == (0, 40)
        xq, xs, wq, ws = _case(20, 0, 40, gated, 1)
        b = W.normal(80, "bf16", 1, 0.5).view(2, 40)
        b = b if gated else b[0].contiguous()
        _check("swish", xq, xs, wq, ws, b, _run("swish", xq, xs, wq, ws, b, "bf16"))


def test_refusals():
    xq, xs, wq, ws = (t.to(DEV) for t in _case(8, 256, 136, False, 1))
    y, x = torch.empty(8, 136, dtype=torch.bfloat16, device=DEV), torch.zeros(8, 256, dtype=torch.bfloat16, device=DEV)
    scratch = nfad.nfad_f8_linear_dynamic_scratch(x)

    def status(fn):
        with pytest.raises(nfad.NfadError) as e:
            fn()
        return e.value.status

    assert status(lambda: nfad.nfad_f8_linear(9, xq, xs, wq, ws, None, y)) == 1
    assert status(lambda: nfad.nfad_f8_linear(None, xq, xs, wq, ws, None, y.float())) == 2
    assert status(lambda: nfad.nfad_f8_linear_dynamic(None, x, wq, ws, None, y, scratch[:100])) == 7
    for bad in (lambda: nfad.nfad_f8_linear(None, xq, xs, wq[:, :128], ws, None, y), lambda: nfad.nfad_f8_linear(None, xq, xs.t(), wq, ws, None, y),
                lambda: nfad.nfad_f8_linear(None, xq, xs, wq, ws[:1], None, y), lambda: nfad.nfad_f8_linear(None, xq, xs, wq, ws, y[0, :8], y),
                lambda: nfad.nfad_f8_gated_linear(None, xq, xs, wq, ws, None, y), lambda: nfad.nfad_f8_linear(None, xq, xs, wq, ws, None, y[:4]),
                lambda: nfad.nfad_f8_linear_dynamic(None, x.half(), wq, ws, None, y, scratch), lambda: nfad.nfad_f8_quantize_rows(x, xq, xs.t().contiguous())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nfad.nfad_f8_linear(None, xq.view(torch.int8), xs, wq, ws, None, y), lambda: nfad.nfad_f8_linear(None, xq, xs.half(), wq, ws, None, y),
                lambda: nfad.nfad_f8_linear(None, xq.cpu(), xs, wq, ws, None, y)):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.parametrize("rows,n_in,n_out,gated", [(300, 1024, 4100, False), (2600, 384, 1036, True), (1500, 256, 2500, False), (520, 640, 1100, True)])
def test_results_off_the_packets(rows, n_in, n_out, gated):
    # rows of results that no tensor copy can store, in every tile width
    xq, xs, wq, ws = _case(rows, n_in, n_out, gated, 21)
    bias = W.normal(2 * n_out, "bf16", 1, 0.5).view(2, n_out)
    bias = bias if gated else bias[0].contiguous()
    _check("gelu_tanh", xq, xs, wq, ws, bias, _run("gelu_tanh", xq, xs, wq, ws, bias, "bf16"))


def test_several_calls_at_once():
    # streams with their own results and scratch side by side, several times over: each call's bits are those of the call alone
    cases = [(1, 4096, 1000, True), (40, 2064, 520, False), (300, 512, 1032, True), (900, 1024, 1536, False), (50, 300, 130, True)]
    calls = []
    for i, (rows, n_in, n_out, gated) in enumerate(cases):
        x = W.normal(rows * n_in, "bf16", i, 1.0).view(rows, n_in).to(DEV)
        w = W.normal((2 if gated else 1) * n_out * n_in, "bf16", 50 + i, n_in ** -0.5).view((2, n_out, n_in) if gated else (n_out, n_in)).to(DEV)
        wq = torch.empty(w.shape, dtype=F8, device=DEV)
        ws = torch.empty(*w.shape[:-2], _blocks(n_out), _blocks(n_in), device=DEV)
        nfad.nfad_f8_quantize_blocks(w, wq, ws)
        call = nfad.nfad_f8_gated_linear_dynamic if gated else nfad.nfad_f8_linear_dynamic
        y, scratch = torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV), nfad.nfad_f8_linear_dynamic_scratch(x)
        calls.append(lambda y=y, call=call, x=x, wq=wq, ws=ws, scratch=scratch: (call("swish", x, wq, ws, None, y, scratch), y)[1])
    alone = [c().clone() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = []
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    y = c().fill_(0)
                got.append(c())
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for y, want in zip(got, alone))
    assert nfad.nfad_wait_faults() == 0
