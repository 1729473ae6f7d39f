"""Binding of the operators around the activation (the rest of a feed-forward block): the names of the C interface
(``include/nfad.h``), argument marshalling only, as in ``binding``.  Every call works on contiguous CUDA tensors and the
current stream of their device, allocates nothing and raises on anything the library does not take.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional

import torch

from .binding import BlockNormDesc, BlockNormGrads, DropoutMask, _check, _kind, _on_device, _stream, _tensor, _TORCH_TO_CODE, _raw_stream, load

# small calls are a few microseconds on the device: what is looked up for each of them is looked up once
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_functions = {}


def _call(name: str, t: torch.Tensor, *args) -> None:
    """The library's function on t's device and its current stream (the last argument); raises on any status but 0."""
    fn = _functions.get(name)
    if fn is None:
        fn = _functions[name] = getattr(load(), name)
    index = t.get_device()
    if index == _current_device():
        rc = fn(*args, _raw_stream(index) if _raw_stream is not None else _stream(t))
    else:
        with _on_device(t.device):
            rc = fn(*args, _stream(t))
    if rc:
        _check(rc, name)

NORMS = {"none": 0, "rms": 1, "layer": 2}
NO_ACT = -1


def _norm_kind(kind) -> int:
    return NORMS[kind] if isinstance(kind, str) else int(kind)


def _raw(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, shape, device) -> Optional[int]:
    """The address of an optional tensor that must have exactly this type, shape and device."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.is_cuda and t.device == device:
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape or t.device != device:
        raise ValueError(f"{name} must have shape {tuple(shape)} on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _scratch(t: Optional[torch.Tensor], device):
    if t is None:
        return None, 0
    if not t.is_cuda or not t.is_contiguous():
        raise TypeError("scratch must be a contiguous CUDA tensor")
    if t.device != device:
        raise ValueError(f"scratch must be on {device}")
    return t.data_ptr(), t.numel() * t.element_size()


# ---------------------------------------------------------------- the norms before and after a block

class BlockNorm:
    """The parameters of the norms around a block: ``nfad_block_norm`` with the tensors it points to.

    post, pre: "none", "rms" or "layer"; post_gain, post_bias, pre_gain, pre_bias: [cols] or None; gate: [cols],
    [gate_rows, cols] or None.  The tensors are kept and read at every call; changing their values in place is fine.
    """

    PARAMETERS = ("post_gain", "post_bias", "gate", "pre_gain", "pre_bias")

    def __init__(self, post="none", pre="rms", post_gain=None, post_bias=None, gate=None, pre_gain=None, pre_bias=None,
                 residual_scale: float = 1.0, eps: float = 1e-5):
        self.tensors = {"post_gain": post_gain, "post_bias": post_bias, "gate": gate, "pre_gain": pre_gain, "pre_bias": pre_bias}
        given = [t for t in self.tensors.values() if t is not None]
        self.cols = given[0].shape[-1] if given else None
        self.dtype, self.device = (given[0].dtype, given[0].device) if given else (None, None)
        ptr = {}
        for name, t in self.tensors.items():
            rows = t.shape[:1] if name == "gate" and t is not None and t.dim() == 2 else ()
            ptr[name] = _raw(t, name, self.dtype, (*rows, self.cols), self.device)
        self.post, self.pre = _norm_kind(post), _norm_kind(pre)
        self.gate_rows = 0 if gate is None else gate.numel() // max(1, self.cols)
        self.desc = BlockNormDesc(self.post, self.pre, ptr["post_gain"], ptr["post_bias"], ptr["gate"], self.gate_rows,
                                  ptr["pre_gain"], ptr["pre_bias"], residual_scale, eps)
        self.ref = ctypes.byref(self.desc)

    def _fits(self, x: torch.Tensor, name: str) -> int:
        p = _tensor(x, name)
        if x.dim() == 0 or (self.cols is not None and (x.size(-1) != self.cols or x.dtype is not self.dtype or x.device != self.device)):
            raise ValueError(f"{name} must be [..., {self.cols}] of the parameters' dtype and device")
        return p


def _kin(first: torch.Tensor):
    """What tensors like `first` share, for _like: looked up once a call."""
    return first.dtype, first.shape, first.get_device(), first


def _like(t: Optional[torch.Tensor], name: str, kin) -> Optional[int]:
    """The address of an optional contiguous tensor of the first one's type, size, row length and device."""
    if t is None:
        return None
    if type(t) is torch.Tensor and t.dtype is kin[0] and t.shape == kin[1] and t.get_device() == kin[2] and t.is_contiguous():
        return t.data_ptr()
    p = _tensor(t, name, kin[3])                     # a subclass, the same rows in another shape, or it raises
    if t.shape[-1:] != kin[1][-1:]:
        raise ValueError(f"{name} must have rows of {kin[1][-1]}")
    return p


def nfad_block_norm_forward(norm: BlockNorm, u: torch.Tensor, r: Optional[torch.Tensor], s_out: Optional[torch.Tensor],
                            h: Optional[torch.Tensor], stats: Optional[torch.Tensor] = None) -> None:
    """s_out = residual_scale r + gate N_post(u), h = N_pre(s): tensors [..., cols]; stats: fp32 [rows, 4], or None in a
    pass that will not be differentiated."""
    pu = norm._fits(u, "u")
    kin = _kin(u)
    cols = kin[1][-1]
    rows = u.numel() // cols if cols else 0
    ps = None if stats is None else _raw(stats, "stats", torch.float32, (rows, 4), u.device)
    _call("nfad_block_norm_forward", u, norm.ref, _TORCH_TO_CODE[kin[0]], pu, _like(r, "r", kin), _like(s_out, "s_out", kin), _like(h, "h", kin), ps,
          rows, cols)


def nfad_block_norm_backward_scratch_bytes(dtype, rows: int, cols: int, device=None) -> int:
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        return int(load().nfad_block_norm_backward_scratch_bytes(_TORCH_TO_CODE[dtype], rows, cols))


def nfad_block_norm_backward_scratch(norm: BlockNorm, u: torch.Tensor) -> torch.Tensor:
    """A scratch tensor for the backward of tensors like u."""
    cols = u.shape[-1]
    n = nfad_block_norm_backward_scratch_bytes(u.dtype, u.numel() // cols if cols else 0, cols, u.device)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=u.device)


def nfad_block_norm_backward(norm: BlockNorm, grad_h: Optional[torch.Tensor], grad_s: Optional[torch.Tensor], u: Optional[torch.Tensor],
                             s: Optional[torch.Tensor], stats: torch.Tensor, grad_u: torch.Tensor, grad_r: Optional[torch.Tensor],
                             grads: Optional[Dict[str, torch.Tensor]], scratch: torch.Tensor) -> None:
    """grads: fp32 tensors of the wanted parameters' shapes, by the parameters' names."""
    pg = norm._fits(grad_u, "grad_u")
    cols = grad_u.shape[-1]
    rows = grad_u.numel() // cols if cols else 0
    out = BlockNormGrads()
    for name, t in (grads or {}).items():
        if name not in BlockNorm.PARAMETERS:
            raise ValueError(f"no parameter {name}")
        like = norm.tensors[name]
        shape = like.shape if like is not None else (cols,)
        setattr(out, name, _raw(t, "grads[" + name + "]", torch.float32, torch.Size(shape), grad_u.device))
    sp, sb = _scratch(scratch, grad_u.device)
    kin = _kin(grad_u)
    _call("nfad_block_norm_backward", grad_u, norm.ref, _TORCH_TO_CODE[kin[0]], _like(grad_h, "grad_h", kin), _like(grad_s, "grad_s", kin),
          _like(u, "u", kin), _like(s, "s", kin), _raw(stats, "stats", torch.float32, (rows, 4), grad_u.device), pg,
          _like(grad_r, "grad_r", kin), ctypes.byref(out), sp, sb, rows, cols)


# ---------------------------------------------------------------- dropout

class Dropout:
    """A mask: ``nfad_dropout_mask`` with the tensor it points to.

    p in [0, 1] (held to a multiple of 2^-16); seed and offset: 64-bit integers; step: None, or an int64 CUDA tensor of one value that is
    added to offset when a call runs.  The same numbers give the same mask; layers and steps differ in offset (or step).  None of the four
    can be set on a mask that exists: its backward pass draws by the same object, or by its numbers.  Another mask is another object.
    """

    def __init__(self, p: float, seed: int, offset: int = 0, step: Optional[torch.Tensor] = None):
        self._p, self._seed, self._offset, self._step = float(p), int(seed), int(offset), step
        if not 0.0 <= self.p <= 1.0:
            raise ValueError("p must be in [0, 1]")
        if not (0 <= self.seed < 2 ** 64 and 0 <= self.offset < 2 ** 64):
            raise ValueError("seed and offset must be 64-bit numbers")
        if step is not None:
            if not isinstance(step, torch.Tensor) or step.dtype != torch.int64 or not step.is_cuda:
                raise TypeError("step must be an int64 CUDA tensor")
            if step.numel() != 1:
                raise ValueError("step must hold one value")
        self.desc = DropoutMask(self.p, self.seed, self.offset, None)      # the step's address is filled in by the calls
        self.ref, self._at = ctypes.byref(self.desc), None

    p = property(lambda self: self._p)
    seed = property(lambda self: self._seed)
    offset = property(lambda self: self._offset)
    step = property(lambda self: self._step)


def _mask(drop: Dropout, x: torch.Tensor):
    if not isinstance(drop, Dropout):
        raise TypeError("drop must be a Dropout")
    step = drop._step
    if step is not None:
        if step.get_device() != x.get_device():
            raise ValueError("the mask's step must be on the tensors' device")
        at = step.data_ptr()                             # where it is now: a tensor's storage can be exchanged
        if at != drop._at:
            drop._at = drop.desc.step = at
    return drop.ref


def nfad_dropout(drop: Dropout, x: torch.Tensor, residual: Optional[torch.Tensor], y: torch.Tensor) -> None:
    """y = residual + m x (m x without a residual), m the mask times its scale: tensors of one type and shape.  On the gradient, with the same
    mask and no residual, it is its own backward pass."""
    px = _tensor(x, "x")
    _call("nfad_dropout", x, _TORCH_TO_CODE[x.dtype], _mask(drop, x), px, None if residual is None else _tensor(residual, "residual", x),
          _tensor(y, "y", x), x.numel())


def nfad_bias_act_dropout_forward(kind, drop: Dropout, x: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor, dfdx: torch.Tensor) -> None:
    """y = m f(x + bias), dfdx = m f'(x + bias): x, y, dfdx [..., cols], bias [cols] or None.  The backward pass is that of
    nfad_bias_act_forward (without a bias nfad_act_forward): dfdx carries the mask."""
    px, py, pd = _tensor(x, "x"), _tensor(y, "y", x), _tensor(dfdx, "dfdx", x)
    cols = x.shape[-1] if x.dim() else 1
    pb = _raw(bias, "bias", x.dtype, (cols,), x.device)
    _call("nfad_bias_act_dropout_forward", x, _kind(kind), _TORCH_TO_CODE[x.dtype], _mask(drop, x), px, pb, py, pd, x.numel() // cols if cols else 0, cols)


# ---------------------------------------------------------------- products grouped by expert

def _act(kind) -> int:
    return NO_ACT if kind is None else _kind(kind)


def _matrix(t: torch.Tensor, name: str, dims: int = 2) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dim() != dims or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of {dims} dimensions")
    if t.dtype not in _TORCH_TO_CODE:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    return t.data_ptr()


def _offsets(offsets: torch.Tensor, device) -> int:
    if not isinstance(offsets, torch.Tensor) or offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.numel() == 0:
        raise TypeError("offsets must be an int32 tensor of experts + 1 values")
    if offsets.device != device or not offsets.is_contiguous():
        raise ValueError("offsets must be contiguous and on the tensors' device")
    return offsets.data_ptr()


def nfad_expert_linear(kind, x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor], offsets: torch.Tensor, y: torch.Tensor,
                       dfdx: Optional[torch.Tensor] = None) -> None:
    """y = f(x w_e^T + bias_e), dfdx = f' of it: x [rows, in] sorted by expert, w [experts, out, in], bias [experts, out],
    offsets [experts + 1] int32.  kind None: no activation (and no dfdx)."""
    px, pw = _matrix(x, "x"), _matrix(w, "w", 3)
    (rows, n_in), (experts, n_out, w_in) = x.shape, w.shape
    if w_in != n_in or w.dtype != x.dtype or w.device != x.device:
        raise ValueError("w must be [experts, out, in] of x's dtype and device")
    if offsets.numel() != experts + 1:
        raise ValueError("offsets must hold experts + 1 values")
    shape = (rows, n_out)
    pb = _raw(bias, "bias", x.dtype, (experts, n_out), x.device)
    py, pd = _raw(y, "y", x.dtype, shape, x.device), _raw(dfdx, "dfdx", x.dtype, shape, x.device)
    _call("nfad_expert_linear", x, _act(kind), _TORCH_TO_CODE[x.dtype], px, pw, pb, _offsets(offsets, x.device), py, pd, rows, n_in, n_out, experts)


def nfad_expert_act_backward_scratch_bytes(rows: int, out: int, device=None) -> int:
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        return int(load().nfad_expert_act_backward_scratch_bytes(rows, out))


def nfad_expert_act_backward_scratch(grad_out: torch.Tensor, experts: int = 0) -> torch.Tensor:
    """A scratch tensor for nfad_expert_act_backward on tensors like grad_out (the number of experts does not change its size)."""
    n = nfad_expert_act_backward_scratch_bytes(grad_out.shape[0], grad_out.shape[1], grad_out.device)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=grad_out.device)


def nfad_expert_act_backward(grad_out: torch.Tensor, dfdx: Optional[torch.Tensor], offsets: torch.Tensor, grad_z: Optional[torch.Tensor],
                             grad_bias: Optional[torch.Tensor], scratch: Optional[torch.Tensor]) -> None:
    """grad_z = grad_out dfdx; grad_bias (fp32 [experts, out]) = each expert's column sums of the unrounded products."""
    pg = _matrix(grad_out, "grad_out")
    rows, n_out = grad_out.shape
    experts = offsets.numel() - 1
    pd = _raw(dfdx, "dfdx", grad_out.dtype, grad_out.shape, grad_out.device)
    pz = _raw(grad_z, "grad_z", grad_out.dtype, grad_out.shape, grad_out.device)
    pb = _raw(grad_bias, "grad_bias", torch.float32, (experts, n_out), grad_out.device)
    sp, sb = _scratch(scratch, grad_out.device)
    _call("nfad_expert_act_backward", grad_out, _TORCH_TO_CODE[grad_out.dtype], pg, pd, _offsets(offsets, grad_out.device), pz, pb, sp, sb,
          rows, n_out, experts)


def nfad_expert_linear_backward_input(grad_z: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, dfdx_x: Optional[torch.Tensor],
                                      grad_x: torch.Tensor) -> None:
    """grad_x = (grad_z w_e) dfdx_x: the gradient of the layer's input, times the f' of the activation in front when given."""
    pg, pw = _matrix(grad_z, "grad_z"), _matrix(w, "w", 3)
    (rows, n_out), (experts, w_out, n_in) = grad_z.shape, w.shape
    if w_out != n_out or w.dtype != grad_z.dtype or w.device != grad_z.device:
        raise ValueError("w must be [experts, out, in] of grad_z's dtype and device")
    if offsets.numel() != experts + 1:
        raise ValueError("offsets must hold experts + 1 values")
    shape = (rows, n_in)
    pd = _raw(dfdx_x, "dfdx_x", grad_z.dtype, shape, grad_z.device)
    px = _raw(grad_x, "grad_x", grad_z.dtype, shape, grad_z.device)
    _call("nfad_expert_linear_backward_input", grad_z, _TORCH_TO_CODE[grad_z.dtype], pg, pw, _offsets(offsets, grad_z.device), pd, px, rows,
          n_in, n_out, experts)


def nfad_expert_linear_backward_weight(grad_z: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor, grad_w: torch.Tensor) -> None:
    """grad_w[e] = grad_z_e^T x_e, [experts, out, in]."""
    pg, px = _matrix(grad_z, "grad_z"), _matrix(x, "x")
    (rows, n_out), n_in, experts = grad_z.shape, x.shape[1], offsets.numel() - 1
    if x.shape[0] != rows or x.dtype != grad_z.dtype or x.device != grad_z.device:
        raise ValueError("x must have grad_z's rows, dtype and device")
    pw = _raw(grad_w, "grad_w", grad_z.dtype, (experts, n_out, n_in), grad_z.device)
    _call("nfad_expert_linear_backward_weight", grad_z, _TORCH_TO_CODE[grad_z.dtype], pg, px, _offsets(offsets, grad_z.device), pw, rows, n_in,
          n_out, experts)


# ---------------------------------------------------------------- gated layers grouped by expert

def nfad_expert_gated_linear(kind, x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor], offsets: torch.Tensor, y: torch.Tensor,
                             partials: Optional[torch.Tensor] = None) -> None:
    """y = f(a) u, a = x w_e0^T + bias_e0, u = x w_e1^T + bias_e1: x [rows, in] sorted by expert, w [experts, 2, out, in], bias
    [experts, 2, out]; partials [rows, 2, out] = (f'(a) u, f(a)), y's two derivatives.  kind None: y = a u."""
    px, pw = _matrix(x, "x"), _matrix(w, "w", 4)
    (rows, n_in), (experts, two, n_out, w_in) = x.shape, w.shape
    if w_in != n_in or two != 2 or w.dtype != x.dtype or w.device != x.device:
        raise ValueError("w must be [experts, 2, out, in] of x's dtype and device")
    if offsets.numel() != experts + 1:
        raise ValueError("offsets must hold experts + 1 values")
    pb = _raw(bias, "bias", x.dtype, (experts, 2, n_out), x.device)
    py, pp = _raw(y, "y", x.dtype, (rows, n_out), x.device), _raw(partials, "partials", x.dtype, (rows, 2, n_out), x.device)
    _call("nfad_expert_gated_linear", x, _act(kind), _TORCH_TO_CODE[x.dtype], px, pw, pb, _offsets(offsets, x.device), py, pp, rows, n_in, n_out, experts)


def nfad_expert_gated_backward(grad_out: torch.Tensor, partials: torch.Tensor, offsets: torch.Tensor, grad_z: torch.Tensor,
                               grad_bias: Optional[torch.Tensor], scratch: Optional[torch.Tensor]) -> None:
    """grad_z [rows, 2, out] = grad_out times both partials; grad_bias (fp32 [experts, 2, out]) = each expert's column sums of the
    unrounded products.  scratch: nfad_expert_act_backward_scratch of grad_z.flatten(1)."""
    pg = _matrix(grad_out, "grad_out")
    rows, n_out = grad_out.shape
    experts, both = offsets.numel() - 1, (rows, 2, n_out)
    if partials is None or grad_z is None:
        raise TypeError("partials and grad_z must be CUDA tensors")
    pp, pz = _raw(partials, "partials", grad_out.dtype, both, grad_out.device), _raw(grad_z, "grad_z", grad_out.dtype, both, grad_out.device)
    pb = _raw(grad_bias, "grad_bias", torch.float32, (experts, 2, n_out), grad_out.device)
    sp, sb = _scratch(scratch, grad_out.device)
    _call("nfad_expert_gated_backward", grad_out, _TORCH_TO_CODE[grad_out.dtype], pg, pp, _offsets(offsets, grad_out.device), pz, pb, sp, sb,
          rows, n_out, experts)


def nfad_expert_linear_backward_gated(grad_z: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, partials: torch.Tensor, grad: torch.Tensor) -> None:
    """grad [rows, 2, in] = (grad_z w_e) times both partials: the gradient of a linear layer's input, taken on through the gated layer
    that made it."""
    pg, pw = _matrix(grad_z, "grad_z"), _matrix(w, "w", 3)
    (rows, n_out), (experts, w_out, n_in) = grad_z.shape, w.shape
    if w_out != n_out or w.dtype != grad_z.dtype or w.device != grad_z.device:
        raise ValueError("w must be [experts, out, in] of grad_z's dtype and device")
    if offsets.numel() != experts + 1:
        raise ValueError("offsets must hold experts + 1 values")
    if partials is None or grad is None:
        raise TypeError("partials and grad must be CUDA tensors")
    pp, px = (_raw(t, name, grad_z.dtype, (rows, 2, n_in), grad_z.device) for t, name in ((partials, "partials"), (grad, "grad")))
    _call("nfad_expert_linear_backward_gated", grad_z, _TORCH_TO_CODE[grad_z.dtype], pg, pw, _offsets(offsets, grad_z.device), pp, px, rows, n_in,
          n_out, experts)


# ---------------------------------------------------------------- the linear layer in 8-bit integers

def nfad_i8_quantize_rows(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor) -> None:
    """q (int8) and scale (fp32 [rows]) of x [rows, cols]: x = scale q up to half a step of the row's own scale."""
    px = _matrix(x, "x")
    pq, ps = _raw(q, "q", torch.int8, x.shape, x.device), _raw(scale, "scale", torch.float32, x.shape[:1], x.device)
    _call("nfad_i8_quantize_rows", x, _TORCH_TO_CODE[x.dtype], px, pq, ps, x.shape[0], x.shape[1])


def _i8_weight(wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor, n_in: int):
    if not isinstance(wq, torch.Tensor) or wq.dim() != 2 or wq.shape[1] != n_in:
        raise ValueError("wq must be [out, in]")
    n_out = wq.shape[0]
    return (n_out, _raw(wq, "wq", torch.int8, (n_out, n_in), y.device), _raw(w_scale, "w_scale", torch.float32, (n_out,), y.device),
            _raw(bias, "bias", y.dtype, (n_out,), y.device))


def nfad_i8_linear(kind, xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor],
                   y: torch.Tensor) -> None:
    """y = f(x_scale w_scale (xq wq^T) + bias): xq [rows, in] and wq [out, in] int8, scales fp32, bias and y 16-bit."""
    py = _matrix(y, "y")
    rows, n_in = xq.shape
    n_out, pw, pws, pb = _i8_weight(wq, w_scale, bias, y, n_in)
    if y.shape != (rows, n_out):
        raise ValueError("y must be [rows, out]")
    px, pxs = _raw(xq, "xq", torch.int8, (rows, n_in), y.device), _raw(x_scale, "x_scale", torch.float32, (rows,), y.device)
    _call("nfad_i8_linear", y, _act(kind), _TORCH_TO_CODE[y.dtype], px, pxs, pw, pws, pb, py, rows, n_in, n_out)


def nfad_i8_linear_dynamic_scratch_bytes(rows: int, n_in: int) -> int:
    return int(load().nfad_i8_linear_dynamic_scratch_bytes(rows, n_in))


def nfad_i8_linear_dynamic_scratch(x: torch.Tensor) -> torch.Tensor:
    """A scratch tensor for nfad_i8_linear_dynamic on inputs like x."""
    return torch.empty(max(nfad_i8_linear_dynamic_scratch_bytes(*x.shape), 16), dtype=torch.uint8, device=x.device)


def nfad_i8_linear_dynamic(kind, x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor,
                           scratch: torch.Tensor) -> None:
    """nfad_i8_linear from the 16-bit x [rows, in], each row quantised on the way."""
    px, py = _matrix(x, "x"), _matrix(y, "y")
    rows, n_in = x.shape
    n_out, pw, pws, pb = _i8_weight(wq, w_scale, bias, y, n_in)
    if y.shape != (rows, n_out) or y.dtype != x.dtype or y.device != x.device:
        raise ValueError("y must be [rows, out] of x's dtype and device")
    sp, sb = _scratch(scratch, x.device)
    _call("nfad_i8_linear_dynamic", x, _act(kind), _TORCH_TO_CODE[x.dtype], px, pw, pws, pb, py, sp, sb, rows, n_in, n_out)


# ---------------------------------------------------------------- the linear layer in 8-bit floating point

F8 = torch.float8_e4m3fn
F8_BLOCK = 128


def f8_blocks(n: int) -> int:
    """Blocks of 128 along a dimension of n."""
    return -(-n // F8_BLOCK)


def nfad_f8_quantize_rows(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor) -> None:
    """q (float8_e4m3fn [rows, cols]) and scale (fp32 [blocks of cols, rows]) of x [rows, cols]: blocks of 128 along a row."""
    px = _matrix(x, "x")
    rows, cols = x.shape
    pq, ps = _raw(q, "q", F8, (rows, cols), x.device), _raw(scale, "scale", torch.float32, (f8_blocks(cols), rows), x.device)
    _call("nfad_f8_quantize_rows", x, _TORCH_TO_CODE[x.dtype], px, pq, ps, rows, cols)


def nfad_f8_quantize_blocks(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor) -> None:
    """q and scale (fp32 [..., blocks of rows, blocks of cols]) of the matrices x [..., rows, cols]: blocks of 128 x 128."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a CUDA tensor")
    if x.dim() < 2:
        raise ValueError("x must be a matrix or a stack of them")
    px = _matrix(x, "x", x.dim())
    *lead, rows, cols = x.shape
    pq = _raw(q, "q", F8, x.shape, x.device)
    ps = _raw(scale, "scale", torch.float32, (*lead, f8_blocks(rows), f8_blocks(cols)), x.device)
    matrices = 1
    for n in lead:
        matrices *= n
    _call("nfad_f8_quantize_blocks", x, _TORCH_TO_CODE[x.dtype], px, pq, ps, matrices, rows, cols)


def _f8_weight(wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor, n_in: int, lead: tuple):
    if not isinstance(wq, torch.Tensor) or wq.dim() != 2 + len(lead) or wq.shape[:-2] != lead or wq.shape[-1] != n_in:
        raise ValueError(f"wq must be [{'2, ' if lead else ''}out, in]")
    n_out = wq.shape[-2]
    return (n_out, _raw(wq, "wq", F8, wq.shape, y.device), _raw(w_scale, "w_scale", torch.float32, (*lead, f8_blocks(n_out), f8_blocks(n_in)), y.device),
            _raw(bias, "bias", y.dtype, (*lead, n_out), y.device))


def _f8_linear(name, lead, kind, xq, x_scale, wq, w_scale, bias, y) -> None:
    py = _matrix(y, "y")
    if not isinstance(xq, torch.Tensor) or xq.dim() != 2:
        raise ValueError("xq must be [rows, in]")
    rows, n_in = xq.shape
    n_out, pw, pws, pb = _f8_weight(wq, w_scale, bias, y, n_in, lead)
    if y.shape != (rows, n_out):
        raise ValueError("y must be [rows, out]")
    px, pxs = _raw(xq, "xq", F8, (rows, n_in), y.device), _raw(x_scale, "x_scale", torch.float32, (f8_blocks(n_in), rows), y.device)
    _call(name, y, _act(kind), _TORCH_TO_CODE[y.dtype], px, pxs, pw, pws, pb, py, rows, n_in, n_out)


def nfad_f8_linear(kind, xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor],
                   y: torch.Tensor) -> None:
    """y = f(xq wq^T, each block of 128 along the reduction times its scales, + bias): xq [rows, in] and wq [out, in] float8_e4m3fn, scales as
    the quantisers leave them, bias and y 16-bit."""
    _f8_linear("nfad_f8_linear", (), kind, xq, x_scale, wq, w_scale, bias, y)


def nfad_f8_gated_linear(kind, xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor],
                         y: torch.Tensor) -> None:
    """The gated layer y = f(a) u of such products: wq [2, out, in], w_scale [2, ...], bias [2, out]; the gate's first."""
    _f8_linear("nfad_f8_gated_linear", (2,), kind, xq, x_scale, wq, w_scale, bias, y)


def nfad_f8_linear_dynamic_scratch_bytes(rows: int, n_in: int) -> int:
    return int(load().nfad_f8_linear_dynamic_scratch_bytes(rows, n_in))


def nfad_f8_linear_dynamic_scratch(x: torch.Tensor) -> torch.Tensor:
    """A scratch tensor for nfad_f8_linear_dynamic and nfad_f8_gated_linear_dynamic on inputs like x."""
    return torch.empty(max(nfad_f8_linear_dynamic_scratch_bytes(*x.shape), 16), dtype=torch.uint8, device=x.device)


def _f8_dynamic(name, lead, kind, x, wq, w_scale, bias, y, scratch) -> None:
    px, py = _matrix(x, "x"), _matrix(y, "y")
    rows, n_in = x.shape
    n_out, pw, pws, pb = _f8_weight(wq, w_scale, bias, y, n_in, lead)
    if y.shape != (rows, n_out) or y.dtype != x.dtype or y.device != x.device:
        raise ValueError("y must be [rows, out] of x's dtype and device")
    sp, sb = _scratch(scratch, x.device)
    _call(name, x, _act(kind), _TORCH_TO_CODE[x.dtype], px, pw, pws, pb, py, sp, sb, rows, n_in, n_out)


def nfad_f8_linear_dynamic(kind, x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor,
                           scratch: torch.Tensor) -> None:
    """nfad_f8_linear from the 16-bit x [rows, in], quantised on the way."""
    _f8_dynamic("nfad_f8_linear_dynamic", (), kind, x, wq, w_scale, bias, y, scratch)


def nfad_f8_gated_linear_dynamic(kind, x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor], y: torch.Tensor,
                                 scratch: torch.Tensor) -> None:
    """nfad_f8_gated_linear from the 16-bit x [rows, in], quantised on the way."""
    _f8_dynamic("nfad_f8_gated_linear_dynamic", (2,), kind, x, wq, w_scale, bias, y, scratch)


def nfad_wait_faults() -> int:
    """How many CTAs of the products have given up waiting since the library was loaded (0 in a healthy process).  Synchronises."""
    n = int(load().nfad_wait_faults())
    if n < 0:
        _check(-n, "nfad_wait_faults")
    return n
