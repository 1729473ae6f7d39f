"""Binding of the operators around the activation (the rest of a feed-forward block): the names of the C interface
(``include/nfad.h``), argument marshalling only, as in ``binding``.  Every call works on contiguous CUDA tensors and the
current stream of their device, allocates nothing and raises on anything the library does not take.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional

import torch

from .binding import BlockNormDesc, BlockNormGrads, _check, _kind, _on_device, _stream, _tensor, _TORCH_TO_CODE, load

NORMS = {"none": 0, "rms": 1, "layer": 2}
NO_ACT = -1


def _norm_kind(kind) -> int:
    return NORMS[kind] if isinstance(kind, str) else int(kind)


def _raw(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, shape, device) -> Optional[int]:
    """The address of an optional tensor that must have exactly this type, shape and device."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape or t.device != device:
        raise ValueError(f"{name} must have shape {tuple(shape)} on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _scratch(t: Optional[torch.Tensor]):
    if t is None:
        return None, 0
    if not t.is_cuda or not t.is_contiguous():
        raise TypeError("scratch must be a contiguous CUDA tensor")
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
        if x.dim() == 0 or (self.cols is not None and (x.shape[-1] != self.cols or x.dtype != self.dtype or x.device != self.device)):
            raise ValueError(f"{name} must be [..., {self.cols}] of the parameters' dtype and device")
        return p


def _like(t: Optional[torch.Tensor], name: str, first: torch.Tensor) -> Optional[int]:
    return None if t is None else _tensor(t, name, first)


def nfad_block_norm_forward(norm: BlockNorm, u: torch.Tensor, r: Optional[torch.Tensor], s_out: Optional[torch.Tensor],
                            h: Optional[torch.Tensor], stats: Optional[torch.Tensor] = None) -> None:
    """s_out = residual_scale r + gate N_post(u), h = N_pre(s): tensors [..., cols]; stats: fp32 [rows, 4], or None in a
    pass that will not be differentiated."""
    pu = norm._fits(u, "u")
    cols = u.shape[-1]
    rows = u.numel() // cols if cols else 0
    ps = _raw(stats, "stats", torch.float32, (rows, 4), u.device)
    with _on_device(u.device):
        _check(load().nfad_block_norm_forward(norm.ref, _TORCH_TO_CODE[u.dtype], pu, _like(r, "r", u), _like(s_out, "s_out", u),
                                              _like(h, "h", u), ps, rows, cols, _stream(u)), "nfad_block_norm_forward")


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
    sp, sb = _scratch(scratch)
    with _on_device(grad_u.device):
        _check(load().nfad_block_norm_backward(norm.ref, _TORCH_TO_CODE[grad_u.dtype], _like(grad_h, "grad_h", grad_u),
                                               _like(grad_s, "grad_s", grad_u), _like(u, "u", grad_u), _like(s, "s", grad_u),
                                               _raw(stats, "stats", torch.float32, (rows, 4), grad_u.device), pg,
                                               _like(grad_r, "grad_r", grad_u), ctypes.byref(out), sp, sb, rows, cols,
                                               _stream(grad_u)), "nfad_block_norm_backward")
