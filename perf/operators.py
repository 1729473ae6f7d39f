"""The feed-forward block's operators, as cases with their plain forms and their calls.

Three families: the norms before and after a block with its gate and residual scale (`norm_forward`, `norm_backward`), the
matrix product in 8-bit integers with a scale for each token and channel (`i8_linear`), and matrix products grouped by expert
with the nested activation in their epilogue (`expert_forward`, `expert_backward`).

`own` false: elementary torch operations in 32 bits, rounded once at the end.  `own` true: the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a few requests decoding one token each: both norms of a block's boundary, one row a request, value only
        {"name": "norm_tokens_bf16", "op": "norm_forward", "dtype": "bf16", "rows": 3, "cols": 4096, "post": "rms", "pre": "rms",
         "gates": 1, "alpha": 1.0, "train": False},
        # a training batch of sequences with a gate row for each sequence (12 of 500), LayerNorms with biases, scaled residual
        {"name": "norm_layer_f16", "op": "norm_forward", "dtype": "f16", "rows": 6000, "cols": 2560, "post": "layer", "pre": "layer",
         "gates": 12, "alpha": 0.7071, "train": True},
        # the post-norm block h = LayerNorm(r + u) in 32 bits, its gradient, with odd sizes throughout
        {"name": "norm_grad_odd_f32", "op": "norm_backward", "dtype": "f32", "rows": 1531, "cols": 1021, "post": "none", "pre": "layer",
         "gates": 0, "alpha": 1.0},
        # the gradient of a large training batch's boundary: RMS norms on both sides and a learned gate for each channel
        {"name": "norm_grad_bf16", "op": "norm_backward", "dtype": "bf16", "rows": 32768, "cols": 4096, "post": "rms", "pre": "rms",
         "gates": 1, "alpha": 1.0},
        # one token through the up-projection of an 8-bit feed-forward layer
        {"name": "i8_token", "op": "i8_linear", "dtype": "bf16", "rows": 1, "in": 4096, "out": 12288, "act": "swish", "bias": False},
        # a batch of decoding requests, an odd number of them, through the down-projection
        {"name": "i8_batch", "op": "i8_linear", "dtype": "f16", "rows": 77, "in": 5120, "out": 2048, "act": "none", "bias": True},
        # a long prompt through the up-projection
        {"name": "i8_prompt", "op": "i8_linear", "dtype": "bf16", "rows": 8192, "in": 4096, "out": 16384, "act": "gelu_tanh", "bias": True},
        # a decoding batch of 12 tokens, two experts each of 64: most experts have no row
        {"name": "expert_tokens", "op": "expert_forward", "dtype": "bf16", "rows": 24, "in": 2048, "out": 1408, "experts": 64,
         "act": "swish", "bias": False, "train": False, "spare": 0, "skew": 1.0},
        # fine-grained experts with uneven loads, some empty, and a capacity that is not used up: value and derivative
        {"name": "expert_ragged_f16", "op": "expert_forward", "dtype": "f16", "rows": 4099, "in": 1000, "out": 1416, "experts": 61,
         "act": "mish", "bias": True, "train": True, "spare": 37, "skew": 0.5},
        # a training batch's up-projection on eight experts: value and derivative
        {"name": "expert_train_bf16", "op": "expert_forward", "dtype": "bf16", "rows": 16384, "in": 2048, "out": 8192, "experts": 8,
         "act": "gelu_erf", "bias": True, "train": True, "spare": 0, "skew": 4.0},
        # the gradients of the fine-grained layer
        {"name": "expert_grad_ragged_f16", "op": "expert_backward", "dtype": "f16", "rows": 4099, "in": 1000, "out": 1416, "experts": 61,
         "bias": True, "prev": False, "spare": 37, "skew": 0.5},
        # the gradients of the large layer, the derivative of the activation in front of it multiplied into its input's
        {"name": "expert_grad_bf16", "op": "expert_backward", "dtype": "bf16", "rows": 16384, "in": 2048, "out": 8192, "experts": 8,
         "bias": True, "prev": True, "spare": 0, "skew": 4.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log8(rng, lo, hi):
    return max(8, _log(rng, lo, hi) // 8 * 8)


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "i8_linear", "expert_forward", "expert_backward"])
    if op.startswith("norm"):
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = max(64, cols // 64 * 64)                      # a model's width; otherwise any number
        rows = min(_log(rng, 1, 32768), (32768 * 4096) // cols)
        post, pre = rng.choice([("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("none", "rms"), ("rms", "none"), ("layer", "rms")])
        gates = rng.choice([0, 1, 1, 4])
        if gates == 4:
            rows = -(-rows // 4) * 4
        case = {"op": op, "dtype": rng.choice(["f32", "bf16", "bf16", "f16"]), "rows": rows, "cols": cols, "post": post, "pre": pre,
                "gates": gates, "alpha": rng.choice([1.0, 0.7071, 0.5])}
        if case["dtype"] == "f32":
            case["rows"] = max(4, case["rows"] // 8 * 4)
        if op == "norm_forward":
            case["train"] = rng.random() < 0.7
        return case
    if op == "i8_linear":
        case = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "rows": _log(rng, 1, 8192), "in": _log(rng, 512, 8192), "out": _log(rng, 512, 16384),
                "act": rng.choice(["none", "swish", "gelu_tanh", "gelu_erf", "mish"]), "bias": rng.random() < 0.5}
        if rng.random() < 0.8:
            case["in"], case["out"] = max(64, case["in"] // 64 * 64), max(64, case["out"] // 64 * 64)
        return case
    experts = _log(rng, 1, 128)
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16"]), "rows": _log(rng, 8, 16384), "in": _log8(rng, 256, 4096),
            "out": _log8(rng, 256, 4096), "experts": experts, "bias": rng.random() < 0.5, "spare": rng.choice([0, 0, 5, 64]),
            "skew": rng.choice([0.5, 1.0, 4.0])}
    if rng.random() < 0.15:
        case["in"], case["out"] = case["in"] + 3, case["out"] + 1     # rows that start off every vector boundary
    if op == "expert_forward":
        case["act"] = rng.choice(["none", "swish", "gelu_tanh", "gelu_erf", "mish"])
        case["train"] = case["act"] != "none" and rng.random() < 0.6
    else:
        case["prev"] = rng.random() < 0.5
    return case


def work(case):
    es = SIZE[case["dtype"]]
    if case["op"] == "norm_forward":
        n = case["rows"] * case["cols"]
        return {"bytes": es * n * (3 if case["pre"] == "none" else 4) + (16 * case["rows"] if case["train"] else 0), "flops": 12 * n}
    if case["op"] == "norm_backward":
        n = case["rows"] * case["cols"]
        reads = (2 if case["pre"] == "none" else 3) + (1 if case["post"] != "none" or case["gates"] else 0) - (1 if case["pre"] == "none" else 0)
        return {"bytes": es * n * (reads + 2) + 16 * case["rows"], "flops": 25 * n}
    m, k, n = case["rows"], case["in"], case["out"]
    if case["op"] == "i8_linear":
        return {"bytes": k * n + 4 * n + 2 * m * (k + n), "flops": 2 * m * k * n}
    active = min(case["experts"], m)
    if case["op"] == "expert_forward":
        return {"bytes": 2 * (m * k + active * k * n + m * n * (2 if case["train"] else 1)), "flops": 2 * m * k * n}
    return {"bytes": 2 * (m * (k + 2 * n) + m * k * (2 if case["prev"] else 1) + active * k * n + case["experts"] * k * n), "flops": 4 * m * k * n}


# ---------------------------------------------------------------- inputs

def _offsets(case, seed):
    """Rows of each expert: the tokens' choices under uneven popularity (a smaller `skew` is more uneven)."""
    g = torch.Generator().manual_seed(seed * 7919 + 17)
    e = case["experts"]
    popular = torch.rand(e, generator=g).clamp_min(1e-3).pow(1.0 / case["skew"])
    picks = torch.multinomial(popular, case["rows"], replacement=True, generator=g)
    counts = torch.bincount(picks, minlength=e)
    ends = torch.cumsum(counts, 0)
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends]).to(torch.int32), int(counts.max())


def prepare(case, seed):
    t = TYPES[case["dtype"]]
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)

    s = {"case": dict(case)}
    if case["op"].startswith("norm"):
        rows, cols, g = case["rows"], case["cols"], case["gates"]
        s["u"], s["r"] = normal(rows, cols, std=2.0, mean=0.1), normal(rows, cols, std=3.0, mean=-0.2)
        for side in ("post", "pre"):
            s[side + "_gain"] = normal(cols, std=0.1, mean=1.0) if case[side] != "none" else None
            s[side + "_bias"] = normal(cols, std=0.1) if case[side] == "layer" else None
        s["gate"] = normal(g, cols, std=0.3, mean=0.5) if g else None
        s["r_out"], s["h"] = torch.empty_like(s["u"]), torch.empty_like(s["u"])
        s["stats"] = torch.zeros(rows, 4, device=DEV)
        if case["op"] == "norm_backward":
            stored, _, stats = _norm_plain(s)
            s["r_out"], s["stats"] = stored.to(t), stats
            s["grad_h"] = normal(rows, cols) if case["pre"] != "none" else None
            s["grad_r_out"] = normal(rows, cols)
            s["grad_u"], s["grad_r"] = torch.empty_like(s["u"]), torch.empty_like(s["u"])
            s["grads"] = {k: torch.empty(s[k].shape, device=DEV) for k in ("post_gain", "post_bias", "gate", "pre_gain", "pre_bias")
                          if s[k] is not None}
        else:
            s["stats"] = s["stats"] if case["train"] else None
    elif case["op"] == "i8_linear":
        m, k, n = case["rows"], case["in"], case["out"]
        s["x"] = normal(m, k)
        s["x"][:, 5:: 97] *= 6.0                                   # the few loud channels that activations have
        w = normal(n, k, std=k ** -0.5, dtype=torch.float32)
        s["w_scale"] = w.abs().amax(1) / 127
        s["wq"] = torch.round(w / s["w_scale"][:, None]).clamp_(-127, 127).to(torch.int8)
        s["bias"] = normal(n, std=0.3) if case["bias"] else None
        s["y"] = torch.empty(m, n, dtype=t, device=DEV)
    else:
        m, k, n, e = case["rows"] + case["spare"], case["in"], case["out"], case["experts"]
        off, s["longest"] = _offsets(case, seed)
        s["offsets"] = off.to(DEV)
        s["x"], s["w"] = normal(m, k), normal(e, n, k, std=k ** -0.5)
        if case["op"] == "expert_forward":
            s["bias"] = normal(e, n, std=0.3) if case["bias"] else None
            s["y"] = torch.empty(m, n, dtype=t, device=DEV)
            s["dfdx"] = torch.empty_like(s["y"]) if case["train"] else None
        else:
            s["grad_out"], s["dfdx"] = normal(m, n), (torch.rand(m, n, generator=gen, device=DEV) * 1.2 - 0.1).to(t)
            s["prev"] = (torch.rand(m, k, generator=gen, device=DEV) * 1.2 - 0.1).to(t) if case["prev"] else None
            s["gz"], s["gx"], s["gw"] = torch.empty_like(s["grad_out"]), torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["gb"] = torch.empty(e, n, device=DEV) if case["bias"] else None
    return s


# ---------------------------------------------------------------- the plain forms

def _statistics(x, kind):
    """(mean or 0, reciprocal deviation) of each row."""
    if kind == "none":
        return torch.zeros(x.shape[0], device=x.device), torch.zeros(x.shape[0], device=x.device)
    mean = x.sum(1) / x.shape[1] if kind == "layer" else torch.zeros(x.shape[0], device=x.device)
    c = x - mean[:, None] if kind == "layer" else x
    return mean, 1.0 / torch.sqrt((c * c).sum(1) / x.shape[1] + EPS)


def _affine(x, mean, rstd, gain, bias, kind):
    if kind == "none":
        return x
    y = (x - mean[:, None]) * rstd[:, None] * gain.float()
    return y + bias.float() if bias is not None else y


def _spread(gate, rows):
    """Each gate row over the rows that it governs."""
    return gate.float().repeat_interleave(rows // gate.shape[0], 0)


def _norm_plain(s):
    c = s["case"]
    u = s["u"].float()
    mu, ru = _statistics(u, c["post"])
    a = _affine(u, mu, ru, s["post_gain"], s["post_bias"], c["post"])
    out = c["alpha"] * s["r"].float() + (a * _spread(s["gate"], c["rows"]) if s["gate"] is not None else a)
    ms, rs = _statistics(out, c["pre"])
    h = _affine(out, ms, rs, s["pre_gain"], s["pre_bias"], c["pre"])
    return out, h, torch.stack([mu, ru, ms, rs], 1)


def _norm_gradient(d, xhat, rstd, kind):
    inner = d - xhat * ((d * xhat).sum(1) / d.shape[1])[:, None]
    if kind == "layer":
        inner = inner - (d.sum(1) / d.shape[1])[:, None]
    return inner * rstd[:, None]


def _norm_backward_plain(s):
    c, t = s["case"], TYPES[s["case"]["dtype"]]
    mu, ru, ms, rs = s["stats"].unbind(1)
    grads = {}
    ds = s["grad_r_out"].float()
    if c["pre"] != "none":
        dh = s["grad_h"].float()
        shat = (s["r_out"].float() - ms[:, None]) * rs[:, None]
        grads["pre_gain"] = (dh * shat).sum(0)
        if s["pre_bias"] is not None:
            grads["pre_bias"] = dh.sum(0)
        ds = ds + _norm_gradient(dh * s["pre_gain"].float(), shat, rs, c["pre"])
    u = s["u"].float()
    da = ds
    if s["gate"] is not None:
        a = _affine(u, mu, ru, s["post_gain"], s["post_bias"], c["post"])
        grads["gate"] = (ds * a).view(c["gates"], -1, c["cols"]).sum(1)
        da = ds * _spread(s["gate"], c["rows"])
    du = da
    if c["post"] != "none":
        uhat = (u - mu[:, None]) * ru[:, None]
        grads["post_gain"] = (da * uhat).sum(0)
        if s["post_bias"] is not None:
            grads["post_bias"] = da.sum(0)
        du = _norm_gradient(da * s["post_gain"].float(), uhat, ru, c["post"])
    return [du.to(t), (c["alpha"] * ds).to(t), grads]


def _act_plain(z, kind, slope):
    if kind == "none":
        return z, None
    if kind == "gelu_erf":
        gate = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        dgate = torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)) if slope else None
    elif kind == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        gate = 0.5 * (1 + t)
        dgate = 0.5 * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z) if slope else None
    elif kind == "swish":
        gate = torch.sigmoid(z)
        dgate = gate * (1 - gate) if slope else None
    else:
        gate = torch.tanh(torch.clamp_min(z, 0) + torch.log1p(torch.exp(-torch.abs(z))))
        dgate = (1 - gate * gate) * torch.sigmoid(z) if slope else None
    return z * gate, gate + z * dgate if slope else None


def _i8_plain(s):
    c = s["case"]
    x = s["x"].float()
    amax = x.abs().amax(1, keepdim=True)
    q = torch.round(x * (127.0 / amax))
    z = (q @ s["wq"].float().t()) * (amax / 127.0) * s["w_scale"]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    return _act_plain(z, c["act"], False)[0].to(TYPES[c["dtype"]])


def _places(s):
    """Expert and place within it of each row that has one."""
    off = s["offsets"].long()
    row = torch.arange(s["case"]["rows"], device=DEV)
    e = torch.searchsorted(off, row, right=True) - 1
    return e, row - off[e]


def _pad(x, e, at, s):
    p = torch.zeros(s["case"]["experts"], s["longest"], x.shape[1], device=DEV)
    p[e, at] = x
    return p


def _expert_forward_plain(s):
    c, t = s["case"], TYPES[s["case"]["dtype"]]
    e, at = _places(s)
    rows = c["rows"]
    z = torch.bmm(_pad(s["x"][:rows].float(), e, at, s), s["w"].float().transpose(1, 2))[e, at]
    if s["bias"] is not None:
        z = z + s["bias"].float()[e]
    out = []
    for v in _act_plain(z, c["act"], c["train"]):
        if v is not None:
            full = torch.zeros(s["x"].shape[0], c["out"], dtype=t, device=DEV)
            full[:rows] = v.to(t)
            out.append(full)
    return out


def _expert_backward_plain(s):
    c, t = s["case"], TYPES[s["case"]["dtype"]]
    e, at = _places(s)
    rows = c["rows"]
    gz = _pad(s["grad_out"][:rows].float() * s["dfdx"][:rows].float(), e, at, s)
    gx = torch.zeros(s["x"].shape[0], c["in"], dtype=t, device=DEV)
    g = torch.bmm(gz, s["w"].float())[e, at]
    gx[:rows] = (g * s["prev"][:rows].float() if s["prev"] is not None else g).to(t)
    gw = torch.bmm(gz.transpose(1, 2), _pad(s["x"][:rows].float(), e, at, s)).to(t)
    return [gx, gw, gz.sum(1) if c["bias"] else None]


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "norm_forward":
        t = TYPES[c["dtype"]]
        out, h, stats = _norm_plain(s)
        return [out.to(t), h.to(t) if c["pre"] != "none" else None, stats if c["train"] else None]
    return {"norm_backward": _norm_backward_plain, "i8_linear": _i8_plain, "expert_forward": _expert_forward_plain,
            "expert_backward": _expert_backward_plain}[c["op"]](s)


def _run_own(s):
    import paper_2209_10778_b200 as nfad
    c = s["case"]
    act = None if c.get("act", "none") == "none" else c["act"]
    if c["op"].startswith("norm"):
        if "norm" not in s:
            s["norm"] = nfad.BlockNorm(post=c["post"], pre=c["pre"], post_gain=s["post_gain"], post_bias=s["post_bias"], gate=s["gate"],
                                       pre_gain=s["pre_gain"], pre_bias=s["pre_bias"], residual_scale=c["alpha"], eps=EPS)
        if c["op"] == "norm_forward":
            h = s["h"] if c["pre"] != "none" else None
            nfad.nfad_block_norm_forward(s["norm"], s["u"], s["r"], s["r_out"], h, s["stats"])
            return [s["r_out"], h, s["stats"]]
        if "scratch" not in s:
            s["scratch"] = nfad.nfad_block_norm_backward_scratch(s["norm"], s["u"])
        nfad.nfad_block_norm_backward(s["norm"], s["grad_h"], s["grad_r_out"], s["u"], s["r_out"], s["stats"], s["grad_u"], s["grad_r"],
                                      s["grads"], s["scratch"])
        return [s["grad_u"], s["grad_r"], s["grads"]]
    if c["op"] == "i8_linear":
        if "scratch" not in s:
            s["scratch"] = nfad.nfad_i8_linear_dynamic_scratch(s["x"])
        nfad.nfad_i8_linear_dynamic(act, s["x"], s["wq"], s["w_scale"], s["bias"], s["y"], s["scratch"])
        return s["y"]
    if c["op"] == "expert_forward":
        nfad.nfad_expert_linear(act, s["x"], s["w"], s["bias"], s["offsets"], s["y"], s["dfdx"])
        return [s["y"]] if s["dfdx"] is None else [s["y"], s["dfdx"]]
    if "scratch" not in s:
        s["scratch"] = nfad.nfad_expert_act_backward_scratch(s["grad_out"], c["experts"])
    nfad.nfad_expert_act_backward(s["grad_out"], s["dfdx"], s["offsets"], s["gz"], s["gb"], s["scratch"])
    nfad.nfad_expert_linear_backward_input(s["gz"], s["w"], s["offsets"], s["prev"], s["gx"])
    nfad.nfad_expert_linear_backward_weight(s["gz"], s["x"], s["offsets"], s["gw"])
    return [s["gx"], s["gw"], s["gb"]]


# ---------------------------------------------------------------- 64 bits

def _act_exact(z, kind):
    """f and f' by the definitions, the derivative by automatic differentiation."""
    if kind == "none":
        return z, None
    z = z.detach().requires_grad_(True)
    if kind == "gelu_erf":
        y = z * torch.special.ndtr(z)
    elif kind == "gelu_tanh":
        y = z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    elif kind == "swish":
        y = z / (1 + torch.exp(-z))
    else:
        y = z * torch.tanh(torch.log1p(torch.exp(z)))
    d, = torch.autograd.grad(y.sum(), z)
    return y.detach(), d


def _norm64(x, gain, bias, kind):
    if kind == "none":
        return x
    c = x - x.mean(1, keepdim=True) if kind == "layer" else x
    y = c / (c.square().mean(1, keepdim=True) + EPS).sqrt() * gain
    return y if bias is None else y + bias


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if case["op"] == "norm_forward":
        a = _norm64(d["u"], d["post_gain"], d["post_bias"], case["post"])
        if d["gate"] is not None:
            g = d["gate"]
            a = (a.view(g.shape[0], -1, case["cols"]) * g[:, None, :]).view(a.shape)
        out = case["alpha"] * d["r"] + a
        h = _norm64(out, d["pre_gain"], d["pre_bias"], case["pre"]) if case["pre"] != "none" else None
        stats = None
        if case["train"]:
            cols = []
            for x, kind in ((d["u"], case["post"]), (out, case["pre"])):
                mean = x.mean(1) if kind == "layer" else torch.zeros_like(x[:, 0])
                cols += [mean, ((x - mean[:, None]).square().mean(1) + EPS).rsqrt() if kind != "none" else torch.zeros_like(mean)]
            stats = torch.stack(cols, 1)
        return [out, h, stats]
    if case["op"] == "norm_backward":
        # the gradient with the saved statistics: chain rule over x^ = (x - mean) rstd, with mean and rstd as functions of x
        mu, ru, ms, rs = (v[:, None] for v in d["stats"].unbind(1))
        grads = {}
        ds = d["grad_r_out"].clone()
        if case["pre"] != "none":
            shat = (d["r_out"] - ms) * rs
            g = d["grad_h"] * d["pre_gain"]
            drstd = (g * shat).mean(1, keepdim=True)
            dmean = g.mean(1, keepdim=True) if case["pre"] == "layer" else 0.0
            ds += rs * (g - dmean - shat * drstd)
            grads["pre_gain"] = torch.einsum("rc,rc->c", d["grad_h"], shat)
            if d["pre_bias"] is not None:
                grads["pre_bias"] = d["grad_h"].sum(0)
        uhat = (d["u"] - mu) * ru if case["post"] != "none" else d["u"]
        a = uhat if case["post"] == "none" else uhat * d["post_gain"] + (d["post_bias"] if d["post_bias"] is not None else 0.0)
        da = ds
        if d["gate"] is not None:
            n, group = case["gates"], case["rows"] // case["gates"]
            grads["gate"] = torch.einsum("grc,grc->gc", ds.view(n, group, -1), a.view(n, group, -1))
            da = (ds.view(n, group, -1) * d["gate"][:, None, :]).view(ds.shape)
        du = da
        if case["post"] != "none":
            g = da * d["post_gain"]
            du = ru * (g - (g.mean(1, keepdim=True) if case["post"] == "layer" else 0.0) - uhat * (g * uhat).mean(1, keepdim=True))
            grads["post_gain"] = torch.einsum("rc,rc->c", da, uhat)
            if d["post_bias"] is not None:
                grads["post_bias"] = da.sum(0)
        return [du, case["alpha"] * ds, grads]
    if case["op"] == "i8_linear":
        scale = d["x"].abs().amax(1, keepdim=True) / 127
        z = (d["x"] / scale).round() @ d["wq"].double().t() * scale * d["w_scale"]
        return _act_exact(z + d["bias"] if d["bias"] is not None else z, case["act"])[0]
    off = d["offsets"].tolist()
    parts = [(e, slice(off[e], off[e + 1])) for e in range(case["experts"]) if off[e + 1] > off[e]]
    if case["op"] == "expert_forward":
        z = torch.zeros(d["y"].shape, dtype=torch.float64, device=DEV)
        for e, p in parts:
            z[p] = d["x"][p] @ d["w"][e].t() + (d["bias"][e] if d["bias"] is not None else 0.0)
        y, slope = _act_exact(z, case["act"])
        y[off[-1]:] = 0
        if not case["train"]:
            return [y]
        slope[off[-1]:] = 0
        return [y, slope]
    gz = d["grad_out"] * d["dfdx"]
    gx, gw = torch.zeros_like(d["x"]), torch.zeros_like(d["w"])
    gb = torch.zeros(case["experts"], case["out"], dtype=torch.float64, device=DEV)
    for e, p in parts:
        gx[p], gw[e], gb[e] = gz[p] @ d["w"][e], gz[p].t() @ d["x"][p], gz[p].sum(0)
    return [gx * d["prev"] if d["prev"] is not None else gx, gw, gb if case["bias"] else None]
