"""Every kernel that sizes choose among for the gated layer, its gradient through a linear layer, and the products with block scales: its values
against the plain 64-bit forms (bounds as in the operators' own tests), and that it is the one that runs.  The sizes are for 148 SMs."""
import pytest
import torch

import paper_2209_10778_b200 as nfad
import test_gpu_f8 as f8
import test_gpu_gated as gated
from paper_2209_10778_b200 import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda"
UNEVEN = [40 + 37 * i % 171 for i in range(24)]                  # 2964 rows
STORE = {"bf16": "nfad::StoreBF16", "f16": "nfad::StoreF16"}
# kernel, and rows of each expert, rows before and after them, in, out: with results by packets and, where a kernel has them, element by element
GATED = [
    ("product_kernel<4, 256, {s}, false, false>", (UNEVEN, 2, 21, 136, 712)), ("product_kernel<4, 256, {s}, false, false>", (UNEVEN, 0, 5, 136, 708)),
    ("product_kernel<4, 256, {s}, false, false>", ([60], 0, 3, 136, 9500)), ("product_kernel<4, 128, {s}, false, false>", ([260], 0, 0, 264, 2504)),
    ("product_kernel<4, 128, {s}, false, false>", ([260], 1, 0, 264, 2500)), ("product_kernel<4, 256, {s}, false, true>", ([1101, 701, 900], 1, 3, 520, 1800)),
    ("product_kernel<4, 256, {s}, false, true>", ([1101, 701, 900], 0, 0, 264, 1796)), ("product_kernel<4, 128, {s}, true, false>", ([300, 0, 200], 0, 2, 100, 712)),
    ("product_kernel<4, 128, {s}, true, false>", ([33, 65], 1, 1, 37, 51)), ("split_kernel<4, {s}>", ([77], 0, 0, 5128, 72)), ("split_kernel<4, {s}>", ([40, 0, 37], 3, 2, 1288, 136)),
    ("few_rows_kernel<4, {s}, 1>", ([3, 1, 0, 2] * 40, 0, 2, 264, 136)), ("few_rows_kernel<4, {s}, 1>", ([1], 0, 0, 1000, 1001)), ("few_rows_kernel<4, {s}, 2>", ([16], 0, 0, 1032, 520)),
]
THROUGH = [
    ("product_kernel<5, 64, {s}, false, false>", (UNEVEN, 2, 21, 136, 712)), ("product_kernel<5, 128, {s}, false, false>", ([260], 0, 3, 5000, 136)),
    ("product_kernel<5, 256, {s}, false, false>", (UNEVEN, 2, 21, 712, 136)), ("product_kernel<5, 256, {s}, false, true>", ([2000, 17, 1500, 0, 500], 0, 5, 776, 328)),
    ("product_kernel<5, 128, {s}, true, false>", ([33, 65], 1, 1, 37, 51)), ("split_kernel<5, {s}>", ([77], 0, 0, 136, 5128)), ("split_kernel<5, {s}>", ([150], 0, 1, 520, 1288)),
]
# kernel (of the plain layer or the gated one: OP), and rows, in, out
SCALED = [
    ("few_rows_kernel<OP, {s}, 1>", (8, 528, 264)), ("few_rows_kernel<OP, {s}, 1>", (3, 4096, 517)), ("scaled_split_kernel<OP, {s}>", (40, 10256, 72)),
    ("scaled_split_kernel<OP, {s}>", (60, 5136, 200)), ("scaled_split_kernel<OP, {s}>", (300, 2064, 392)), ("scaled_kernel<OP, 128, {s}, false, false>", (300, 400, 1504)),
    ("scaled_kernel<OP, 128, {s}, false, false>", (300, 400, 1500)), ("scaled_kernel<OP, 256, {s}, false, false>", (40, 272, 24000)),
    ("scaled_kernel<OP, 256, {s}, false, false>", (100, 400, 23004)), ("scaled_kernel<OP, 256, {s}, false, true>", (2600, 272, 2056)),
    ("scaled_kernel<OP, 256, {s}, false, true>", (1000, 272, 4100)), ("scaled_kernel<OP, 64, {s}, true, false>", (200, 100, 392)), ("scaled_kernel<OP, 64, {s}, true, false>", (33, 37, 51)),
]
SCALED_GATED = [("scaled_kernel<OP, 256, {s}, false, false>", (40, 272, 14336)), ("scaled_kernel<OP, 256, {s}, false, false>", (300, 272, 6004))]
ALL_SCALED = [(6, *c) for c in SCALED] + [(7, *c) for c in SCALED + SCALED_GATED]


def _ran(call):
    """Names of the library's kernels that the call launched; skips where their activity is not recorded."""
    call()
    torch.cuda.synchronize()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    names = [e.name.replace("(int)", "").replace("(bool)1", "true").replace("(bool)0", "false") for e in p.events()]
    ours = [n.split("(")[0].split("nfad::", 1)[1] for n in names if "nfad::" in n]
    if not ours:
        pytest.skip("the device's activity is not recorded here")
    return ours


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("i", range(len(GATED)))
def test_gated(i, dtype):
    x, w, b, off, o = gated._case(GATED[i][1], dtype, 500 + i)
    for kind, bias, train in (("gelu_erf", b, True), ("swish", None, True), ("mish", b, False), (None, b, True), ("gelu_tanh", None, False)):
        gated._check_forward(kind, x, w, bias, o, *gated._forward(kind, x, w, bias, off, train=train))
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("i", range(len(THROUGH)))
def test_through_linear(i, dtype):
    counts, lead, tail, n_in, n_out = THROUGH[i][1]
    _, _, _, off, o = gated._case((counts, lead, tail, 1, 1), dtype, 4)
    rows, e = o[-1] + tail, len(counts)
    w = W.normal(e * n_out * n_in, dtype, 8, n_out ** -0.5).view(e, n_out, n_in)
    gz, both = W.normal(rows * n_out, dtype, 9, 1.0).view(rows, n_out), gated._factors(rows, n_in, dtype, 11)
    out = gated._through_linear(gz, w, off, both)
    gated._check_through_linear(gz, w, o, both, out)
    place = both.to(DEV)                                              # in place of the derivatives
    nfad.nfad_expert_linear_backward_gated(gz.to(DEV), w.to(DEV), off.to(DEV), place, place)
    assert torch.equal(place.cpu(), out)
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("i", range(len(ALL_SCALED)))
def test_scaled(i, dtype):
    op, _, (rows, n_in, n_out) = ALL_SCALED[i]
    xq, xs, wq, ws = f8._case(rows, n_in, n_out, op == 7, 600 + i)
    bias = W.normal(2 * n_out, dtype, 1, 0.5).view(2, n_out)
    bias = bias if op == 7 else bias[0].contiguous()
    for kind, b in (("gelu_erf", bias), ("swish", None), ("mish", bias), (None, bias), ("gelu_tanh", bias)):
        f8._check(kind, xq, xs, wq, ws, b, f8._run(kind, xq, xs, wq, ws, b, dtype))
    assert nfad.nfad_wait_faults() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_they_are_the_ones_that_run(dtype):
    store = STORE[dtype]
    for i, (name, case) in enumerate(GATED):
        x, w, b, off, _ = (t.to(DEV) if isinstance(t, torch.Tensor) else t for t in gated._case(case, dtype, 500 + i))
        y = torch.empty(x.shape[0], w.shape[2], dtype=x.dtype, device=DEV)
        both = torch.empty(x.shape[0], 2, w.shape[2], dtype=x.dtype, device=DEV)
        assert _ran(lambda: nfad.nfad_expert_gated_linear("swish", x, w, b, off, y, both)) == [name.format(s=store)]
        assert _ran(lambda: nfad.nfad_expert_gated_linear("swish", x, w, b, off, y)) == [name.format(s=store)]
    for name, (counts, lead, tail, n_in, n_out) in THROUGH:
        off, o = (t.to(DEV) if isinstance(t, torch.Tensor) else t for t in gated._case((counts, lead, tail, 1, 1), dtype, 4)[3:])
        rows, e = o[-1] + tail, len(counts)
        gz, w, both = (torch.zeros(s, dtype=torch.bfloat16 if dtype == "bf16" else torch.float16, device=DEV) for s in ((rows, n_out), (e, n_out, n_in), (rows, 2, n_in)))
        assert _ran(lambda: nfad.nfad_expert_linear_backward_gated(gz, w, off, both, torch.empty_like(both))) == [name.format(s=store)]
    for op, name, (rows, n_in, n_out) in ALL_SCALED:
        xq, xs, wq, ws = (t.to(DEV) for t in f8._case(rows, n_in, n_out, op == 7, 1))
        y = torch.empty(rows, n_out, dtype=torch.bfloat16 if dtype == "bf16" else torch.float16, device=DEV)
        call = nfad.nfad_f8_gated_linear if op == 7 else nfad.nfad_f8_linear
        assert _ran(lambda: call(None, xq, xs, wq, ws, None, y)) == [name.replace("OP", str(op)).format(s=store)]


@pytest.mark.parametrize("rows,n_in,n_out", [(40, 272, 14336), (300, 272, 6004), (1000, 272, 4100)])
def test_scaled_gated_from_16_bits(rows, n_in, n_out):
    x = W.normal(rows * n_in, "bf16", 2, 1.0).view(rows, n_in)
    wq, ws = f8._quantize_blocks(W.normal(2 * n_out * n_in, "f32", 3, n_in ** -0.5).view(2, n_out, n_in))
    xq, xs = f8._quantize_rows(x)
    y, dx = torch.full((rows, n_out), float("nan"), dtype=x.dtype, device=DEV), x.to(DEV)
    nfad.nfad_f8_gated_linear_dynamic("swish", dx, wq.to(DEV), ws.to(DEV), None, y, nfad.nfad_f8_linear_dynamic_scratch(dx).fill_(0xff))
    torch.cuda.synchronize()
    assert torch.equal(y, f8._run("swish", xq, xs, wq, ws, None, "bf16"))


def test_every_quotient_of_two_f16_significands():
    # the quantiser's nearest value, ties to even, for largest magnitudes of every significand (a quarter of them at a time)
    mine = torch.arange(1024, 2048, dtype=torch.float32)
    for part in range(4):
        tops = mine[part::4]
        for shift in (0, 1, 9):
            v = torch.where(mine[None] <= tops[:, None], mine[None], mine[None] / 2) * 2.0 ** -shift
            cut = torch.cat([v, torch.zeros(tops.numel(), -v.shape[1] % 127)], 1).view(tops.numel(), -1, 127)
            x = torch.cat([tops[:, None, None].expand(-1, cut.shape[1], 1), cut], 2).reshape(tops.numel(), -1).half()
            wq, ws = f8.quantize(x[None], 1)
            f8._same(*f8._quantize_rows(x), wq[0], ws[0].t())
