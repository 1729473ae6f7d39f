"""Plain implementations in 64 bits of the operators around the activation, and the error bounds that go with them.

A bound is 2^-24 times a number of roundings times the sum of the magnitudes that were added: each helper that returns a
value also returns that sum (`mag`), formed like the value with every term replaced by its absolute value.
"""
import numpy as np
import torch

EPS32 = 2.0 ** -24
#: significand bits and smallest normal exponent
FORMATS = {torch.float32: (24, -126), torch.bfloat16: (8, -126), torch.float16: (11, -14)}


def half_ulp(v, dtype):
    """Half the spacing of the type at |v|: what one rounding to nearest may add."""
    p, emin = FORMATS[dtype]
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** emin)))
    # a value at the top of a binade may round into the next
    return torch.exp2(torch.clamp_min(e, emin) - p) * 1.0000001


def check(got, want, err32, what, dtype=None):
    """got (any type) against want (64 bits): fp32 evaluation error err32, then one rounding to got's type."""
    dtype = dtype or got.dtype
    g, want, err32 = got.double().cpu(), want.double().cpu(), torch.as_tensor(err32).double().cpu()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(g[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), f"{what}: infinities differ"
    # the rounding is that of a value up to err32 away from want
    tol = err32 + half_ulp(want.nan_to_num().abs() + err32, dtype)
    bad = finite & ~((g - want).abs() <= tol)
    if bad.any():
        i = int(torch.argmax(((g - want).abs() / tol).masked_fill(~finite, 0)))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, worst at {i}: got {g.flatten()[i]!r} "
                             f"want {want.flatten()[i]!r} tol {tol.flatten()[i]!r}")


# ---------------------------------------------------------------- norms around a block

def _spread(gate, rows):
    return gate.double().reshape(-1, gate.shape[-1]).repeat_interleave(rows // (gate.numel() // gate.shape[-1]), 0)


def _norm_stats(x, kind, eps):
    if kind == "none":
        z = torch.zeros(x.shape[0], 1, dtype=torch.float64)
        return z, z.clone()
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros(x.shape[0], 1, dtype=torch.float64)
    return mean, 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)


def _affine(n, p, side):
    if p.get(side + "_gain") is not None:
        n = n * p[side + "_gain"].double()
    if p.get(side + "_bias") is not None:
        n = n + p[side + "_bias"].double()
    return n


def block_norm(p, u, r):
    """p: dict of post, pre, parameters (CPU tensors or None), alpha, eps.  Returns s, h, stats and the magnitudes of s and h."""
    u = u.double()
    rows, cols = u.shape
    mu, ru = _norm_stats(u, p["post"], p["eps"])
    a, am = u, u.abs()
    if p["post"] != "none":
        a = _affine((u - mu) * ru, p, "post")
        ab = {k: (v.abs() if isinstance(v, torch.Tensor) else v) for k, v in p.items()}
        am = _affine((u.abs() + mu.abs()) * ru, ab, "post")
    if p.get("gate") is not None:
        g = _spread(p["gate"], rows)
        a, am = a * g, am * g.abs()
    s, sm = (a, am) if r is None else (a + p["alpha"] * r.double(), am + abs(p["alpha"]) * r.double().abs())
    if p["pre"] == "none":
        z = torch.zeros(rows, 1, dtype=torch.float64)
        return s, None, torch.cat([mu, ru, z, z], 1), sm, None
    ms, rs = _norm_stats(s, p["pre"], p["eps"])
    h = _affine((s - ms) * rs, p, "pre")
    # the statistics err by the row's own errors, at most the row mean of the magnitudes; 1/sqrt by half their relative size
    ab = {k: (v.abs() if isinstance(v, torch.Tensor) else v) for k, v in p.items()}
    rel = rs * rs * (sm * (s - ms).abs()).mean(1, keepdim=True)
    hm = _affine((sm + sm.mean(1, keepdim=True)) * rs + ((s - ms) * rs).abs() * (1 + rel), ab, "pre")
    return s, h, torch.cat([mu, ru, ms, rs], 1), sm, hm


def depth(cols):
    """Roundings that one term of a row's sum may pass through: its thread's run (at most 32 values, or every 256th column)
    and two trees of five levels; and the element's own handful."""
    return 32 + cols / 256 + 10 + 8


def block_norm_backward(p, dh, gs, u, s, stats):
    """Gradients from the saved stats, and the magnitude of each: dict of (value, magnitude)."""
    st = stats.double()
    mu, ru, ms, rs = (st[:, i:i + 1] for i in range(4))
    rows, cols = u.shape
    one = torch.ones(1, cols, dtype=torch.float64)
    out = {}
    ds = gs.double() if gs is not None else torch.zeros(rows, cols, dtype=torch.float64)
    dsm = ds.abs()

    def through(d, dm, xhat, xm, rstd, kind):
        mean = d.mean(1, keepdim=True) if kind == "layer" else 0.0
        meanm = dm.mean(1, keepdim=True) if kind == "layer" else 0.0
        v = rstd * (d - mean - xhat * (d * xhat).mean(1, keepdim=True))
        return v, rstd * (dm + meanm + xm * (dm * xm).mean(1, keepdim=True))

    if p["pre"] != "none":
        dh = dh.double()
        xhat, xm = (s.double() - ms) * rs, (s.double().abs() + ms.abs()) * rs
        out["pre_gain"] = ((dh * xhat).sum(0), (dh.abs() * xm).sum(0))
        out["pre_bias"] = (dh.sum(0), dh.abs().sum(0))
        g = p["pre_gain"].double() if p.get("pre_gain") is not None else one
        v, m = through(dh * g, (dh * g).abs(), xhat, xm, rs, p["pre"])
        ds, dsm = ds + v, dsm + m
    out["r"] = (p["alpha"] * ds, abs(p["alpha"]) * dsm)
    u = u.double()
    xhat, xm = (u, u.abs()) if p["post"] == "none" else ((u - mu) * ru, (u.abs() + mu.abs()) * ru)
    da, dam = ds, dsm
    if p.get("gate") is not None:
        a, am = xhat, xm
        if p["post"] != "none":
            ab = {k: (v.abs() if isinstance(v, torch.Tensor) else v) for k, v in p.items()}
            a, am = _affine(xhat, p, "post"), _affine(xm, ab, "post")
        n = p["gate"].numel() // cols
        out["gate"] = ((ds * a).view(n, -1, cols).sum(1).view(p["gate"].shape), (dsm * am).view(n, -1, cols).sum(1).view(p["gate"].shape))
        gate = _spread(p["gate"], rows)
        da, dam = ds * gate, dsm * gate.abs()
    if p["post"] != "none":
        out["post_gain"] = ((da * xhat).sum(0), (dam * xm).sum(0))
        out["post_bias"] = (da.sum(0), dam.sum(0))
        g = p["post_gain"].double() if p.get("post_gain") is not None else one
        da, dam = through(da * g, dam * g.abs(), xhat, xm, ru, p["post"])
    out["u"] = (da, dam)
    return out


# ---------------------------------------------------------------- activations

def act(z, kind):
    """f and f' in 64 bits, the derivative from the formulas of the gates."""
    z = z.double()
    if kind is None:
        return z, torch.ones_like(z)
    if kind == "gelu_erf":
        h, dh = 0.5 * torch.special.erfc(-z / np.sqrt(2.0)), torch.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    elif kind == "gelu_tanh":
        v = 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
        h = torch.sigmoid(v)
        dh = h * torch.sigmoid(-v) * 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * z * z)
    elif kind == "swish":
        h = torch.sigmoid(z)
        dh = h * torch.sigmoid(-z)
    else:
        h = torch.tanh(torch.nn.functional.softplus(z))
        dh = (1 - h) * (1 + h) * torch.sigmoid(z)
    return z * h, h + z * dh


#: largest |f'| and |f''| of the four activations are below these
SLOPE, CURVATURE = 1.2, 1.1


def check_act(y, d, z, z_err, kind, what):
    """y = f(z), d = f'(z) for a z that the kernel forms with an error of at most z_err.  The 16-bit chains give y within one
    spacing (not half of one) and f' within one spacing plus a sixteenth of the spacing of its terms, |h| + |z h'| < 1.25."""
    want, slope = act(z, kind)
    if kind is None:
        check(y, want, z_err, what + " y")
        return
    check(y, want, SLOPE * z_err + half_ulp(want, y.dtype), what + " y")
    if d is not None:
        check(d, slope, CURVATURE * z_err + half_ulp(slope, d.dtype) + half_ulp(torch.full_like(slope, 1.25), d.dtype) / 8, what + " f'")


def dot_error(mag, terms):
    """Of a tensor-core sum of `terms` products whose magnitudes add up to mag: each step of 16 terms adds to the fp32
    accumulator with at most 2^-23 (truncation included) of what has been added so far."""
    return 2.0 ** -23 * (terms / 16 + 4) * mag
