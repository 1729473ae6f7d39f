"""A feed-forward block out of the library's operators, trained in 16 bits and served in 8.

    python -m paper_2209_10778_b200.feed_forward [--rows R] [--width C] [--hidden H] [--experts E] [--steps K] [--gated] [--dropout P]

Training: stream, h = norms around the previous block; expert feed-forward with the nested activation in its products; norms
again.  Serving (one expert): the same block with both weight matrices in 8-bit integers and no derivative.  --gated: a gated layer in
the place of the first one, dropout of the block's output before it joins the stream, and serving in 8-bit floating point.
"""
from __future__ import annotations

import argparse
import time

import torch

from . import autograd
from . import block as ops


class FeedForwardBlock(torch.nn.Module):
    """stream, h -> stream + gate N(ffn(h)), N of it: an RMS norm behind the block, its channel gate, and the RMS norm in front of
    the next.  Rows of h are grouped by expert as `offsets` says."""

    projections = ()                                                  # of the first layer, between its experts and its outputs

    def __init__(self, width: int, hidden: int, experts: int = 1, kind: str = "gelu_erf", dtype=torch.bfloat16, device="cuda", residual_scale: float = 1.0):
        super().__init__()
        def weight(*shape):
            return torch.nn.Parameter((torch.randn(*shape, device=device) * shape[-1] ** -0.5).to(dtype))
        def constant(value, *shape):
            return torch.nn.Parameter(torch.full(shape, value, dtype=dtype, device=device))
        self.w1, self.w2 = weight(experts, *self.projections, hidden, width), weight(experts, width, hidden)
        self.b1, self.b2 = constant(0.0, experts, *self.projections, hidden), constant(0.0, experts, width)
        self.post_gain, self.pre_gain, self.gate = constant(1.0, width), constant(1.0, width), constant(0.5, width)
        self.kind, self.residual_scale = kind, residual_scale

    def forward(self, stream: torch.Tensor, h: torch.Tensor, offsets: torch.Tensor):
        return self._join(autograd.expert_feed_forward(h, self.w1, self.b1, self.w2, self.b2, offsets, self.kind), stream)

    def _join(self, u: torch.Tensor, stream: torch.Tensor):
        return autograd.block_norm(u, stream, post="rms", pre="rms", post_gain=self.post_gain, gate=self.gate, pre_gain=self.pre_gain,
                                   residual_scale=self.residual_scale)

    def serving(self) -> "ServingBlock":
        return ServingBlock(self)


class GatedFeedForwardBlock(FeedForwardBlock):
    """The same with a gated layer first, and with dropout (probability p, in training) of what joins the stream.

    The mask is a function of seed, layer and `step`, a buffer on the device: blocks of one model differ in `layer`, and a training program
    counts `step` up after each backward pass (`advance`), in a captured graph too."""

    projections = (2,)

    def __init__(self, width: int, hidden: int, experts: int = 1, kind: str = "swish", dtype=torch.bfloat16, device="cuda", residual_scale: float = 1.0,
                 p: float = 0.0, seed: int = 0, layer: int = 0):
        super().__init__(width, hidden, experts, kind, dtype, device, residual_scale)
        self.register_buffer("step", torch.zeros(1, dtype=torch.int64, device=device))
        self.p, self.seed, self.layer = p, seed, layer

    def advance(self) -> None:
        self.step.add_(1)

    def mask(self) -> ops.Dropout:
        """This step's mask: offsets of different layers are 2^40 steps apart."""
        return ops.Dropout(self.p, self.seed, self.layer << 40, self.step)

    def forward(self, stream: torch.Tensor, h: torch.Tensor, offsets: torch.Tensor):
        u = autograd.expert_gated_feed_forward(h, self.w1, self.b1, self.w2, self.b2, offsets, self.kind)
        if self.training and self.p:
            u = autograd.dropout(u, self.mask())
        return self._join(u, stream)

    def serving(self) -> "GatedServingBlock":
        return GatedServingBlock(self)


class ServingBlock:
    """A one-expert block's value-only pass with its weights in 8-bit integers: a scale for each output channel, formed here once,
    and for each token, formed on the way.  Everything is a copy: training the block on changes nothing here.  Keeps buffers for the
    largest number of rows seen, for each CUDA stream that it is called on."""

    def __init__(self, block: FeedForwardBlock):
        if block.w1.shape[0] != 1:
            raise ValueError("8-bit serving takes a block of one expert")
        (self.q1, self.s1), (self.q2, self.s2) = self._quantized(block.w1), self._quantized(block.w2)
        self.b1, self.b2 = (b.detach()[0].clone() for b in (block.b1, block.b2))
        self.norm = ops.BlockNorm(post="rms", pre="rms", residual_scale=block.residual_scale,
                                  **{k: getattr(block, k).detach().clone() for k in ("post_gain", "gate", "pre_gain")})
        self.kind, self.dtype = block.kind, block.w1.dtype
        self._kept = {}                                               # stream -> (rows, tensors)

    def _quantized(self, w):
        q, s = torch.empty(w.shape[1:], dtype=torch.int8, device=w.device), torch.empty(w.shape[1], device=w.device)
        ops.nfad_i8_quantize_rows(w.detach()[0], q, s)
        return q, s

    def _scratch_bytes(self, rows: int, n: int) -> int:
        return ops.nfad_i8_linear_dynamic_scratch_bytes(rows, n)

    def _products(self, h, y1, u, scratch):
        ops.nfad_i8_linear_dynamic(self.kind, h, self.q1, self.s1, self.b1, y1, scratch)
        ops.nfad_i8_linear_dynamic(None, y1, self.q2, self.s2, self.b2, u, scratch)

    def _make(self, rows: int):
        dev, width, hidden = self.q1.device, *self.q2.shape
        size = max(self._scratch_bytes(rows, n) for n in (width, hidden))
        return (*(torch.empty(rows, n, dtype=self.dtype, device=dev) for n in (hidden, width, width)),
                torch.empty(max(size, 16), dtype=torch.uint8, device=dev))

    def _buffers(self, rows: int):
        """y1, u, h and scratch: what the current stream keeps, which no other stream writes and which is given back in its order.  A captured
        call has its own, in the memory of its graph: a replay may come at any time later."""
        dev = self.q1.device
        if dev.index is not None and dev.index != torch.cuda.current_device():
            with torch.cuda.device(dev):
                return self._buffers(rows)
        if torch.cuda.is_current_stream_capturing():
            return self._make(rows)
        at = torch.cuda.current_stream().cuda_stream
        most, kept = self._kept.get(at, (-1, None))
        if rows > most:
            kept = self._make(rows)
            self._kept[at] = rows, kept
        return (*(t[:rows] for t in kept[:3]), kept[3])

    def __call__(self, stream: torch.Tensor, h: torch.Tensor) -> torch.Tensor:
        """Adds the block to `stream` in place and returns the next block's input (valid until the next call on this CUDA stream)."""
        y1, u, out, scratch = self._buffers(h.shape[0])
        self._products(h, y1, u, scratch)
        ops.nfad_block_norm_forward(self.norm, u, stream, stream, out)
        return out


class GatedServingBlock(ServingBlock):
    """A one-expert gated block's value-only pass with its weights in 8-bit floating point: a scale for each block of 128 x 128, formed here once,
    and for each 128 of a token's values, formed on the way.  Everything is a copy, as in ServingBlock."""

    def _quantized(self, w):
        w = w.detach()[0]
        *lead, n, k = w.shape
        q = torch.empty(w.shape, dtype=ops.F8, device=w.device)
        s = torch.empty(*lead, ops.f8_blocks(n), ops.f8_blocks(k), device=w.device)
        ops.nfad_f8_quantize_blocks(w, q, s)
        return q, s

    def _scratch_bytes(self, rows: int, n: int) -> int:
        return ops.nfad_f8_linear_dynamic_scratch_bytes(rows, n)

    def _products(self, h, y1, u, scratch):
        ops.nfad_f8_gated_linear_dynamic(self.kind, h, self.q1, self.s1, self.b1, y1, scratch)
        ops.nfad_f8_linear_dynamic(None, y1, self.q2, self.s2, self.b2, u, scratch)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("rows", 4096), ("width", 1024), ("hidden", 4096), ("experts", 4), ("steps", 20)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--gated", action="store_true")
    p.add_argument("--dropout", type=float, default=0.1, help="with --gated")
    a = p.parse_args()
    torch.manual_seed(0)
    x = torch.randn(a.rows, a.width, device="cuda", dtype=torch.bfloat16)
    target = torch.randn(a.rows, a.width, device="cuda", dtype=torch.bfloat16)
    # a router's choice, its rows already sorted by expert
    ends = torch.sort(torch.randint(0, a.rows + 1, (a.experts - 1,))).values
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), ends, torch.tensor([a.rows])]).to(torch.int32).cuda()
    make = GatedFeedForwardBlock if a.gated else FeedForwardBlock
    block = make(a.width, a.hidden, a.experts, **({"p": a.dropout} if a.gated else {}))
    opt = torch.optim.SGD(block.parameters(), lr=2.0)
    for step in range(a.steps):
        t0 = time.perf_counter()
        _, h = block(x, x, offsets)
        loss = (h - target).float().square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if a.gated:
            block.advance()
        if step % 5 == 0 or step == a.steps - 1:
            print(f"step {step:3d}: loss {loss.item():.4f}  {1e3 * (time.perf_counter() - t0):.2f} ms")
    one = make(a.width, a.hidden, 1)
    serve = one.serving()
    everything = torch.tensor([0, a.rows], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        for rows in (1, 16, a.rows):
            _, want = one(x[:rows], x[:rows], torch.clamp(everything, max=rows))
            got = serve(x[:rows].clone(), x[:rows])
            print(f"{rows:5d} rows in 8 bits: relative difference from 16 bits {((got - want).float().norm() / want.float().norm()).item():.4f}")


if __name__ == "__main__":
    main()
