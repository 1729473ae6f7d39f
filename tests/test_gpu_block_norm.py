"""The norms before and after a block (nfad_block_norm_forward / _backward) against plain 64-bit implementations.

Bounds (block_plain): a result may be off by 2^-24 times the roundings its terms pass through times the sum of the terms'
magnitudes, and one rounding to the storage type.  Column sums add a term at most rows + 64 times.
"""
import itertools

import pytest
import torch

import block_plain as plain
import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
DTYPES = ["f32", "bf16", "f16"]
# (rows, cols): one warp a row; ragged packets; a CTA a row with one and two packets; odd cols; single elements; long rows
SHAPES = [(13, 64), (37, 1000), (9, 1024), (300, 2048), (21, 4104), (11, 8192), (29, 1021), (1, 1), (5, 3), (3, 20000), (2, 70001)]
NORMS = [("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("rms", "none"), ("layer", "rms"), ("none", "none")]


def _parameters(dtype, cols, rows, post, pre, gates, bias, seed, alpha=0.75, eps=1e-5):
    p = {"post": post, "pre": pre, "alpha": alpha, "eps": eps, "gate": None}
    for side, kind in (("post", post), ("pre", pre)):
        p[side + "_gain"] = (W.normal(cols, "f32", seed, 0.2) + 1).to(W.TORCH_DTYPES[dtype]) if kind != "none" else None
        p[side + "_bias"] = W.normal(cols, dtype, seed + 1, 0.3) if kind != "none" and bias else None
        seed += 2
    if gates:
        p["gate"] = W.normal(gates * cols, dtype, seed, 0.7).view(gates, cols)
    return p


def _module(p, move=lambda t: t.to(DEV)):
    t = {k: (move(p[k]) if p.get(k) is not None else None) for k in nfad.BlockNorm.PARAMETERS}
    return nfad.BlockNorm(post=p["post"], pre=p["pre"], residual_scale=p["alpha"], eps=p["eps"], **t)


def _shifted(t):
    """The same values one element off the 16-byte grid."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
    buf[1:].copy_(t.reshape(-1))
    return buf[1:].view(t.shape)


def _forward(p, u, r, move=lambda t: t.to(DEV), want_s=True):
    norm = _module(p, move)
    du = move(u)
    s = move(torch.zeros_like(u)) if want_s else None
    h = move(torch.zeros_like(u)) if p["pre"] != "none" else None
    stats = torch.full((u.shape[0], 4), 7.0, device=DEV)
    nfad.nfad_block_norm_forward(norm, du, None if r is None else move(r), s, h, stats)
    torch.cuda.synchronize()
    return s, h, stats


def _check_forward(p, u, r, s, h, stats):
    want_s, want_h, want_st, sm, hm = plain.block_norm(p, u, r)
    d = plain.depth(u.shape[1])
    k = plain.EPS32 * d
    if s is not None:
        plain.check(s, want_s, k * sm, "s")
    if h is not None:
        plain.check(h, want_h, 2 * k * hm, "h")
    if stats is not None:
        st = stats.double().cpu()
        for col, mag in ((0, u.double().abs()), (2, sm)):
            mean, rstd = want_st[:, col], want_st[:, col + 1]
            m = mag.mean(1)
            assert ((st[:, col] - mean).abs() <= k * m + 1e-30).all(), "mean"
            x = u.double() if col == 0 else want_s
            rel = k * (1 + (rstd[:, None] ** 2 * (mag + m[:, None]) * (x - mean[:, None]).abs()).mean(1))
            assert ((st[:, col + 1] - rstd).abs() <= rel * rstd).all(), "1/sqrt"


def _tensors(rows, cols, dtype, seed):
    u = (W.normal(rows * cols, "f32", seed, 2.0) + 0.3).to(W.TORCH_DTYPES[dtype]).view(rows, cols)
    return u, W.normal(rows * cols, dtype, seed + 1, 1.5).view(rows, cols)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("post,pre", NORMS)
def test_forward(dtype, post, pre):
    for i, (rows, cols) in enumerate(SHAPES):
        u, r = _tensors(rows, cols, dtype, 10 * i)
        for gates, bias in ((0, False), (1, True), (rows, False)):
            p = _parameters(dtype, cols, rows, post, pre, gates, bias, 1000 + i)
            _check_forward(p, u, r, *_forward(p, u, r))


# rows that do not fill 16-byte packets: by 4 bytes, by single elements; few and many packets a thread; too long to be held
ODD_SHAPES = [(40, 100), (33, 1002), (9, 4098), (6, 14082), (7, 12289), (2, 34007), (400, 202), (333, 997), (200, 6002)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", ODD_SHAPES)
def test_rows_off_the_packets(dtype, rows, cols):
    u, r = _tensors(rows, cols, dtype, cols)
    dh, gs = _tensors(rows, cols, dtype, cols + 2)
    for i, (post, pre) in enumerate(NORMS):
        p = _parameters(dtype, cols, rows, post, pre, 1 if i % 2 else 0, i % 3 == 1, 3000 + i)
        s, h, stats = _forward(p, u, r)
        _check_forward(p, u, r, s, h, stats)
        s = s.cpu()
        _check_backward(p, dh if pre != "none" else None, gs, u, s, stats, *_backward(p, dh if pre != "none" else None, gs, u, s, stats))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(400, 64), (700, 512), (333, 1024), (451, 4096), (310, 6144)])
def test_more_rows_than_multiprocessors(dtype, rows, cols):
    u, r = _tensors(rows, cols, dtype, cols)
    dh, gs = _tensors(rows, cols, dtype, cols + 2)
    for post, pre in (("rms", "rms"), ("layer", "layer"), ("none", "layer")):
        p = _parameters(dtype, cols, rows, post, pre, 1, True, 4000)
        s, h, stats = _forward(p, u, r)
        _check_forward(p, u, r, s, h, stats)
        s = s.cpu()
        _check_backward(p, dh, gs, u, s, stats, *_backward(p, dh, gs, u, s, stats))


@pytest.mark.parametrize("dtype", DTYPES)
def test_forward_without_stream_or_s(dtype):
    rows, cols = 17, 512
    u, r = _tensors(rows, cols, dtype, 3)
    p = _parameters(dtype, cols, rows, "none", "rms", 0, False, 9)
    s, h, st = _forward(p, u, None)
    _check_forward(p, u, None, s, h, st)
    assert torch.equal(s.cpu(), u)
    s, h2, st = _forward(p, u, None, want_s=False)
    assert torch.equal(h2, h)
    # the value-only call and in-place outputs give the same bits
    norm, du, dr = _module(p), u.to(DEV), r.to(DEV)
    s1, h1 = torch.empty_like(du), torch.empty_like(du)
    nfad.nfad_block_norm_forward(norm, du, dr, s1, h1)
    nfad.nfad_block_norm_forward(norm, du, dr, dr, du)
    assert torch.equal(dr, s1) and torch.equal(du, h1)


def _backward(p, dh, gs, u, s, stats, move=lambda t: t.to(DEV), want_r=True):
    norm = _module(p, move)
    gu = move(torch.zeros_like(u))
    gr = move(torch.zeros_like(u)) if want_r else None
    grads = {k: torch.full(norm.tensors[k].shape, 9.0, device=DEV) for k in nfad.BlockNorm.PARAMETERS if norm.tensors[k] is not None}
    scratch = nfad.nfad_block_norm_backward_scratch(norm, gu)
    scratch.fill_(0xff)                                               # NaN everywhere: nothing stale may be added
    nfad.nfad_block_norm_backward(norm, move(dh) if dh is not None else None, move(gs) if gs is not None else None, move(u), move(s),
                                  stats, gu, gr, grads, scratch)
    torch.cuda.synchronize()
    return gu, gr, grads


def _check_backward(p, dh, gs, u, s, stats, gu, gr, grads):
    want = plain.block_norm_backward(p, dh, gs, u, s, stats.cpu())
    rows, cols = u.shape
    k = plain.EPS32 * 2 * plain.depth(cols)
    plain.check(gu, want["u"][0], 2 * k * want["u"][1], "grad_u")
    if gr is not None:
        plain.check(gr, want["r"][0], k * want["r"][1], "grad_r")
    for name, g in grads.items():
        plain.check(g, want[name][0], (2 * k + plain.EPS32 * (rows + 64)) * want[name][1], "grad " + name)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("post,pre", NORMS)
def test_backward(dtype, post, pre):
    for i, (rows, cols) in enumerate(SHAPES):
        u, r = _tensors(rows, cols, dtype, 10 * i + 5)
        dh, gs = (t.clone() for t in _tensors(rows, cols, dtype, 10 * i + 7))
        for gates, bias, stream in ((0, False, True), (1, True, False), (rows, True, True), (0, True, True)):
            p = _parameters(dtype, cols, rows, post, pre, gates, bias, 2000 + i)
            s, _, stats = _forward(p, u, r)
            s = s.cpu()
            a = dh if pre != "none" else None
            b = gs if stream or pre == "none" else None
            _check_backward(p, a, b, u, s, stats, *_backward(p, a, b, u, s, stats))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,gates", [(4000, 4), (3000, 300), (4096, 2048), (2222, 11), (700, 700)])
def test_gate_rows_across_chunks(dtype, rows, gates):
    # gate rows longer than a chunk of rows, shorter than one, and starting in the middle of one
    for cols in (256, 259):
        u, r = _tensors(rows, cols, dtype, rows)
        dh, gs = _tensors(rows, cols, dtype, rows + 1)
        p = _parameters(dtype, cols, rows, "rms", "rms", gates, True, 77)
        s, h, stats = _forward(p, u, r)
        _check_forward(p, u, r, s, h, stats)
        s = s.cpu()
        _check_backward(p, dh, gs, u, s, stats, *_backward(p, dh, gs, u, s, stats))


@pytest.mark.parametrize("dtype", DTYPES)
def test_unaligned_tensors(dtype):
    rows, cols = 12, 512
    u, r = _tensors(rows, cols, dtype, 1)
    dh, gs = _tensors(rows, cols, dtype, 2)
    p = _parameters(dtype, cols, rows, "layer", "layer", 3, True, 5)
    s, h, stats = _forward(p, u, r, move=_shifted)
    _check_forward(p, u, r, s, h, stats)
    s = s.cpu()
    _check_backward(p, dh, gs, u, s, stats, *_backward(p, dh, gs, u, s, stats, move=_shifted))


@pytest.mark.parametrize("cols", [256, 1001])
def test_gradient_against_differences(cols):
    # the derivative of <wh, h> + <ws, s> along a direction in all inputs: central differences of the 64-bit forward
    rows, t = 24, 1e-4
    u, r = _tensors(rows, cols, "f32", 4)
    wh, ws = _tensors(rows, cols, "f32", 6)
    for post, pre in NORMS[:-1]:
        p = _parameters("f32", cols, rows, post, pre, 4, True, 31)
        s, _, stats = _forward(p, u, r)
        gu, gr, grads = _backward(p, wh if pre != "none" else None, ws, u, s.cpu(), stats)
        names = [k for k in grads]
        along = {k: W.normal(p[k].numel(), "f32", 50 + i, 0.3).view(p[k].shape).double() for i, k in enumerate(names)}
        du, dr = (x.double() for x in _tensors(rows, cols, "f32", 8))

        def value(e):
            q = {k: (v.double() + e * along[k] if k in along else v) for k, v in p.items()}
            sv, hv, *_ = plain.block_norm(q, u.double() + e * du, r.double() + e * dr)
            return (ws.double() * sv).sum() + ((wh.double() * hv).sum() if hv is not None else 0.0)

        slope = float((value(t) - value(-t)) / (2 * t))
        got = float((gu.double().cpu() * du).sum() + (gr.double().cpu() * dr).sum() +
                    sum((grads[k].double().cpu() * along[k]).sum() for k in names))
        size = float((gu.double().cpu() * du).abs().sum() + (gr.double().cpu() * dr).abs().sum() +
                     sum((grads[k].double().cpu() * along[k]).abs().sum() for k in names))
        # fp32 gradients (1e-5 of the terms' sum covers the row sums' roundings); the differences' own t^2 term
        assert abs(got - slope) <= 1e-5 * size + 1e-5 * abs(slope), (post, pre, got, slope)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [512, 4096, 515])
def test_bad_rows_stay_by_themselves(dtype, cols):
    rows = 10
    u, r = _tensors(rows, cols, dtype, 21)
    p = _parameters(dtype, cols, rows, "layer", "rms", 1, True, 41)
    clean = _forward(p, u, r)
    u2, r2 = u.clone(), r.clone()
    u2[2, 5] = float("nan")
    r2[4, 7] = float("inf")
    u2[6] = 0.0
    r2[6] = 0.0
    s, h, stats = _forward(p, u2, r2)
    keep = [i for i in range(rows) if i not in (2, 4, 6)]
    assert torch.equal(s[keep], clean[0][keep]) and torch.equal(h[keep], clean[1][keep])
    assert torch.isnan(h[2]).all() and s[4, 7].item() == float("inf") and torch.isnan(h[4, 7])
    _check_forward(p, u2[6:7], r2[6:7], s[6:7], h[6:7], stats[6:7])    # a row of zeros: eps keeps it finite


def test_same_bits_every_time():
    rows, cols = 5000, 1024
    u, r = _tensors(rows, cols, "bf16", 1)
    dh, gs = _tensors(rows, cols, "bf16", 2)
    p = _parameters("bf16", cols, rows, "rms", "rms", 5, False, 3)
    s, _, stats = _forward(p, u, r)
    a = _backward(p, dh, gs, u, s.cpu(), stats)
    b = _backward(p, dh, gs, u, s.cpu(), stats)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all(torch.equal(a[2][k], b[2][k]) for k in a[2])


def test_backward_in_place():
    rows, cols = 40, 512
    u, r = _tensors(rows, cols, "bf16", 1)
    dh, gs = _tensors(rows, cols, "bf16", 2)
    for c in (cols, 509):
        uu, rr, hh, gg = (t[:, :c].contiguous() for t in (u, r, dh, gs))
        p = _parameters("bf16", c, rows, "rms", "layer", 1, False, 3)
        s, _, stats = _forward(p, uu, rr)
        want = _backward(p, hh, gg, uu, s.cpu(), stats)
        norm = _module(p)
        ga, gb = hh.to(DEV), gg.to(DEV)
        scratch = nfad.nfad_block_norm_backward_scratch(norm, ga)
        nfad.nfad_block_norm_backward(norm, ga, gb, uu.to(DEV), s, stats, ga, gb, None, scratch)
        torch.cuda.synchronize()
        assert torch.equal(ga, want[0]) and torch.equal(gb, want[1])


def test_elements_beyond_32_bits():
    rows, cols = (1 << 20) + 3, 4096
    u = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    r = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    tu, tr = _tensors(2, cols, "bf16", 1)
    u[-2:], r[-2:] = tu.to(DEV), tr.to(DEV)
    p = _parameters("bf16", cols, rows, "rms", "rms", 0, False, 3)
    norm = _module(p)
    nfad.nfad_block_norm_forward(norm, u, r, r, u)
    torch.cuda.synchronize()
    _check_forward(p, tu, tr, r[-2:], u[-2:], None)
    assert not r[:-2:4099].any()


def test_other_stream_and_graph():
    rows, cols = 64, 1024
    u, r = _tensors(rows, cols, "bf16", 1)
    p = _parameters("bf16", cols, rows, "rms", "rms", 1, False, 3)
    s, h, _ = _forward(p, u, r)
    norm, du, dr = _module(p), u.to(DEV), r.to(DEV)
    s1, h1 = torch.zeros_like(du), torch.zeros_like(du)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        nfad.nfad_block_norm_forward(norm, du, dr, s1, h1)
    st.synchronize()
    assert torch.equal(s, s1) and torch.equal(h, h1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nfad.nfad_block_norm_forward(norm, du, dr, s1, h1)
    s1.zero_()
    h1.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(s, s1) and torch.equal(h, h1)


def test_no_rows():
    p = _parameters("bf16", 64, 0, "rms", "rms", 0, False, 3)
    norm = _module(p)
    e = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    nfad.nfad_block_norm_forward(norm, e, e, e, e)
    grads = {k: torch.full((64,), 3.0, device=DEV) for k in ("post_gain", "pre_gain")}
    nfad.nfad_block_norm_backward(norm, e, e, e, e, torch.empty(0, 4, device=DEV), e, e, grads, nfad.nfad_block_norm_backward_scratch(norm, e))
    torch.cuda.synchronize()
    assert not grads["post_gain"].any() and not grads["pre_gain"].any()


def test_refusals():
    rows, cols = 8, 64
    u, r = (t.to(DEV) for t in _tensors(rows, cols, "bf16", 1))
    gain = torch.ones(cols, dtype=torch.bfloat16, device=DEV)
    norm = nfad.BlockNorm(post="rms", pre="rms", post_gain=gain, pre_gain=gain)
    s, h = torch.empty_like(u), torch.empty_like(u)
    st = torch.empty(rows, 4, device=DEV)

    def status(fn):
        with pytest.raises(nfad.NfadError) as e:
            fn()
        return e.value.status

    assert status(lambda: nfad.nfad_block_norm_forward(norm, u, r, s, s, st)) == 4
    assert status(lambda: nfad.nfad_block_norm_forward(norm, u, r, s, None, st)) == 3
    for bad in (dict(eps=0.0), dict(eps=float("nan"))):
        q = nfad.BlockNorm(post="rms", pre="rms", pre_gain=gain, **bad)
        assert status(lambda: nfad.nfad_block_norm_forward(q, u, r, s, h, st)) == 11
    q = nfad.BlockNorm(post="none", pre="rms", gate=gain.repeat(3, 1))
    assert status(lambda: nfad.nfad_block_norm_forward(q, u, r, s, h, st)) == 11      # 3 gate rows, 8 rows
    q = nfad.BlockNorm(post=5, pre="rms")
    assert status(lambda: nfad.nfad_block_norm_forward(q, u, r, s, h, st)) == 1
    with pytest.raises(TypeError):
        nfad.nfad_block_norm_forward(norm, u.cpu(), r, s, h, st)
    with pytest.raises(ValueError):
        nfad.nfad_block_norm_forward(norm, u[:, ::2], r, s, h, st)
    with pytest.raises(ValueError):
        nfad.nfad_block_norm_forward(norm, u, r[:4], s, h, st)
    with pytest.raises(TypeError):
        nfad.nfad_block_norm_forward(norm, u, r, s, h, st.double())
    scratch = nfad.nfad_block_norm_backward_scratch(norm, u)
    assert status(lambda: nfad.nfad_block_norm_backward(norm, h, None, u, s, st, s.clone(), None, None, scratch[:64])) == 7
    q = nfad.BlockNorm(post="none", pre="rms", pre_gain=gain)
    assert status(lambda: nfad.nfad_block_norm_backward(q, h, None, u, s, st, s.clone(), None, {"post_gain": torch.empty(cols, device=DEV)}, scratch)) == 11
    assert status(lambda: nfad.nfad_block_norm_backward(norm, None, h, u, s, st, s.clone(), None, None, scratch)) == 3


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [64, 1000, 6144, 1021, 20000])
def test_every_subset_of_the_parameters_gradients(dtype, cols):
    # what is not asked for changes nothing in what is: a frozen bias behind the block still stands in the gate's gradient
    rows = 24
    u, r = _tensors(rows, cols, dtype, 61)
    dh, gs = _tensors(rows, cols, dtype, 63)
    for post, pre, gates in (("rms", "rms", 1), ("rms", "rms", 6), ("rms", "layer", rows), ("layer", "rms", 4), ("rms", "none", 2), ("none", "rms", 3)):
        p = _parameters(dtype, cols, rows, post, pre, gates, True, 6000)
        norm = _module(p)
        s, _, stats = _forward(p, u, r)
        a, du, dgs = dh.to(DEV) if pre != "none" else None, u.to(DEV), gs.to(DEV)
        scratch = nfad.nfad_block_norm_backward_scratch(norm, du)
        want = plain.block_norm_backward(p, dh if pre != "none" else None, gs, u, s.cpu(), stats.cpu())
        k = plain.EPS32 * 2 * plain.depth(cols)
        names = [n for n in nfad.BlockNorm.PARAMETERS if norm.tensors[n] is not None]
        for count in range(len(names) + 1):
            for some in itertools.combinations(names, count):
                scratch.fill_(0xff)
                gu, gr = torch.full_like(du, 9.0), torch.full_like(du, 9.0)
                grads = {n: torch.full(norm.tensors[n].shape, 9.0, device=DEV) for n in some}
                nfad.nfad_block_norm_backward(norm, a, dgs, du, s, stats, gu, gr, grads, scratch)
                plain.check(gu, want["u"][0], 2 * k * want["u"][1], f"grad_u with {some}")
                plain.check(gr, want["r"][0], k * want["r"][1], f"grad_r with {some}")
                for n in some:
                    plain.check(grads[n], want[n][0], (2 * k + plain.EPS32 * (rows + 64)) * want[n][1], f"grad {n} with {some}, {post} {pre}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [64, 1000, 4096, 6144, 515])
def test_gradients_that_begin_on_any_float(dtype, cols):
    # the parameters' gradients as pieces of one flat buffer, as an optimizer keeps them; gate rows that end inside a chunk of rows
    rows = 360
    u, r = _tensors(rows, cols, dtype, 71)
    dh, gs = _tensors(rows, cols, dtype, 73)
    for gates in (rows, rows // 2, 3, 1):
        for post, pre, bias in (("rms", "rms", False), ("layer", "layer", True), ("none", "rms", False)):
            p = _parameters(dtype, cols, rows, post, pre, gates, bias, 7000)
            norm = _module(p)
            s, _, stats = _forward(p, u, r)
            want = _backward(p, dh, gs, u, s.cpu(), stats)
            for shift in (1, 2, 3):
                names = list(want[2])
                flat = torch.full((shift + sum(norm.tensors[n].numel() + 1 for n in names),), 5.0, device=DEV)
                grads, at = {}, shift
                for n in names:
                    t = norm.tensors[n]
                    grads[n] = flat[at:at + t.numel()].view(t.shape)
                    at += t.numel() + 1                               # one float between them, which nothing writes
                du = u.to(DEV)
                gu, gr = torch.empty_like(du), torch.empty_like(du)
                nfad.nfad_block_norm_backward(norm, dh.to(DEV), gs.to(DEV), du, s, stats, gu, gr, grads, nfad.nfad_block_norm_backward_scratch(norm, du))
                assert torch.equal(gu, want[0]) and torch.equal(gr, want[1])
                at = shift
                for n in names:
                    assert torch.equal(grads[n], want[2][n]), n
                    at += norm.tensors[n].numel() + 1
                    assert flat[at - 1] == 5.0
                assert (flat[:shift] == 5.0).all()


def test_threads_with_different_widths():
    # calls from several host threads at once, rows of different lengths through the same kernel: each gets its own answer
    import ctypes
    import threading
    from paper_2209_10778_b200 import binding
    call = binding.load().nfad_block_norm_backward                    # the library's own calls, one behind the other
    jobs = []
    for cols in (256, 4096, 1024, 4088):
        rows = 64
        u, r = _tensors(rows, cols, "bf16", cols)
        dh, gs = _tensors(rows, cols, "bf16", cols + 1)
        p = _parameters("bf16", cols, rows, "rms", "rms", 1, False, 3)
        s, _, stats = _forward(p, u, r)
        want = _backward(p, dh, gs, u, s.cpu(), stats)
        norm, du = _module(p), u.to(DEV)
        given = [dh.to(DEV), gs.to(DEV), du, s, stats, torch.empty_like(du), torch.empty_like(du)]
        grads = {k: torch.empty(norm.tensors[k].shape, device=DEV) for k in want[2]}
        out = binding.BlockNormGrads(**{k: g.data_ptr() for k, g in grads.items()})
        scratch, stream = nfad.nfad_block_norm_backward_scratch(norm, du), torch.cuda.Stream()
        args = (norm.ref, binding.DTYPES["bf16"], *(t.data_ptr() for t in given), ctypes.byref(out), scratch.data_ptr(),
                scratch.numel(), rows, cols, stream.cuda_stream)
        jobs.append((args, given, grads, want, (norm, out, scratch, stream)))
    torch.cuda.synchronize()
    failed = []

    def work(args):
        torch.cuda.set_device(0)
        failed.extend(rc for rc in (call(*args) for _ in range(4000)) if rc)

    threads = [threading.Thread(target=work, args=j[:1]) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, (len(failed), failed[0])
    for _, given, grads, want, _ in jobs:
        assert torch.equal(given[5], want[0]) and torch.equal(given[6], want[1]) and all(torch.equal(grads[k], want[2][k]) for k in grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [64, 1000, 4096, 14336, 1021, 4098, 20000])
def test_rows_whose_squares_overflow(dtype, cols):
    # finite values from about 2^64 on: the sum of their squares is infinite in fp32, its reciprocal root 0, and so is the normalised row
    rows = 9
    u, r = _tensors(rows, cols, dtype, 81)
    sign = torch.ones(cols)
    sign[1::2] = -1
    for post, pre in (("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "none")):
        p = _parameters(dtype, cols, rows, post, pre, 1, True, 8000)
        clean = _forward(p, u, r)
        big_u, big_r = u.clone(), r.clone()
        big_u[2], big_r[6] = (sign * 1e25).to(u.dtype), (sign * 1e25).to(u.dtype)
        s, h, stats = _forward(p, big_u, big_r)
        keep = [i for i in range(rows) if i not in (2, 6)]
        assert torch.equal(s[keep], clean[0][keep]) and torch.equal(stats[keep], clean[2][keep])
        assert torch.isfinite(s).all()
        if post != "none":
            assert stats[2, 1] == 0
            a = p["post_bias"].double() * p["gate"][0].double()       # what is left of a row whose normalised values are 0
            want = p["alpha"] * r[2].double() + a
            plain.check(s[2], want, 4 * plain.EPS32 * (abs(p["alpha"]) * r[2].double().abs() + a.abs()), "s")
        if pre != "none":
            for i in (2, 6) if post == "none" else (6,):
                assert stats[i, 3] == 0
                assert torch.equal(h[i].float().cpu(), p["pre_bias"].float())
            assert torch.isfinite(h).all()
        dh, gs = _tensors(rows, cols, dtype, 83)
        gu, gr, grads = _backward(p, dh if pre != "none" else None, gs, big_u, s.cpu(), stats)
        assert torch.isfinite(gu).all() and torch.isfinite(gr).all() and all(torch.isfinite(g).all() for g in grads.values())


class _Elsewhere(torch.Tensor):
    """A tensor that says it lives on another GPU."""
    device = property(lambda self: torch.device("cuda", 1))


def test_scratch_on_another_device_is_refused():
    rows, cols = 8, 64
    u, r = (t.to(DEV) for t in _tensors(rows, cols, "bf16", 1))
    gain = torch.ones(cols, dtype=torch.bfloat16, device=DEV)
    norm = nfad.BlockNorm(post="rms", pre="rms", pre_gain=gain)
    s, h, st = torch.empty_like(u), torch.empty_like(u), torch.empty(rows, 4, device=DEV)
    nfad.nfad_block_norm_forward(norm, u, r, s, h, st)
    away = nfad.nfad_block_norm_backward_scratch(norm, u).as_subclass(_Elsewhere)
    with pytest.raises(ValueError):
        nfad.nfad_block_norm_backward(norm, h, None, u, s, st, torch.empty_like(u), None, None, away)
    offsets = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        nfad.nfad_expert_act_backward(u, None, offsets, None, torch.empty(1, cols, device=DEV), nfad.nfad_expert_act_backward_scratch(u).as_subclass(_Elsewhere))
    q, qs = torch.zeros(16, cols, dtype=torch.int8, device=DEV), torch.ones(16, device=DEV)
    with pytest.raises(ValueError):
        nfad.nfad_i8_linear_dynamic(None, u, q, qs, None, torch.empty(rows, 16, dtype=u.dtype, device=DEV),
                                    nfad.nfad_i8_linear_dynamic_scratch(u).as_subclass(_Elsewhere))


def test_rows_of_another_length_are_refused():
    # as many elements in rows of another length would be read as other rows
    rows, cols = 8, 64
    u, r = (t.to(DEV) for t in _tensors(rows, cols, "bf16", 1))
    norm = nfad.BlockNorm(post="rms", pre="rms")
    turned = lambda: torch.empty(cols, rows, dtype=u.dtype, device=DEV)
    s, h, st = torch.empty_like(u), torch.empty_like(u), torch.empty(rows, 4, device=DEV)
    for bad in ((u, turned(), s, h), (u, r, turned(), h), (u, r, s, turned())):
        with pytest.raises(ValueError):
            nfad.nfad_block_norm_forward(norm, *bad, st)
    nfad.nfad_block_norm_forward(norm, u.view(2, 4, cols), r, s, h, st)               # the rows are the same
    scratch, gu = nfad.nfad_block_norm_backward_scratch(norm, u), torch.empty_like(u)
    for i in range(5):
        args = [h, r, u, s, torch.empty_like(u)]
        args[i] = turned()
        with pytest.raises(ValueError):
            nfad.nfad_block_norm_backward(norm, *args[:4], st, gu, args[4], None, scratch)
