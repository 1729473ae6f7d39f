"""The gated feed-forward block's operators, as cases with their plain forms and their calls.

Three families: the gated layer y = f(x Wg^T + bg) (x Wu^T + bu) grouped by expert, both projections, activation and product in
one kernel, and its gradients (`gated_forward`, `gated_backward`); the linear layer, plain or gated, in 8-bit floating point with
a scale for each block of 128 (`f8_linear`); and dropout whose mask is drawn from a counter and never stored, alone, with a
residual, or behind an activation whose derivative then carries the mask (`dropout`).

`own` false: elementary torch operations in 32 bits, rounded once at the end.  `own` true: the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128                                   # side of a block that has one scale
LARGEST = 448.0                               # of the 8-bit type (four exponent bits, three of the significand)


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a few requests decoding one token each through the gated layer, value only
        {"name": "gated_tokens_bf16", "op": "gated_forward", "dtype": "bf16", "rows": 3, "in": 4096, "out": 14336, "experts": 1,
         "act": "swish", "bias": False, "train": False, "spare": 0, "skew": 1.0},
        # small gated experts with uneven loads and a capacity that is not used up: value and both partial derivatives
        {"name": "gated_ragged_f16", "op": "gated_forward", "dtype": "f16", "rows": 3001, "in": 1032, "out": 712, "experts": 24,
         "act": "gelu_tanh", "bias": True, "train": True, "spare": 21, "skew": 0.5},
        # a training batch's gated layer: value and both partial derivatives
        {"name": "gated_train_bf16", "op": "gated_forward", "dtype": "bf16", "rows": 16384, "in": 2048, "out": 5632, "experts": 1,
         "act": "swish", "bias": False, "train": True, "spare": 0, "skew": 4.0},
        # the gradients of the small gated experts
        {"name": "gated_grad_ragged_f16", "op": "gated_backward", "dtype": "f16", "rows": 3001, "in": 1032, "out": 712, "experts": 24,
         "bias": True, "down": False, "spare": 21, "skew": 0.5},
        # the gradients of the training batch's gated layer, from the gradient of the layer behind it
        {"name": "gated_grad_bf16", "op": "gated_backward", "dtype": "bf16", "rows": 16384, "in": 2048, "out": 5632, "experts": 1,
         "bias": False, "down": True, "spare": 0, "skew": 4.0},
        # one token through the gated layer with 8-bit weights
        {"name": "f8_token_gated", "op": "f8_linear", "dtype": "bf16", "rows": 1, "in": 4096, "out": 14336, "gated": True, "act": "swish",
         "bias": False},
        # a batch of decoding requests through the down-projection; the last blocks are ragged both ways
        {"name": "f8_batch_f16", "op": "f8_linear", "dtype": "f16", "rows": 101, "in": 7216, "out": 2056, "gated": False, "act": "none",
         "bias": True},
        # a long prompt through an up-projection with an activation
        {"name": "f8_prompt", "op": "f8_linear", "dtype": "bf16", "rows": 8000, "in": 4096, "out": 16384, "gated": False, "act": "gelu_tanh",
         "bias": True},
        # a long prompt through the gated layer
        {"name": "f8_prompt_gated", "op": "f8_linear", "dtype": "bf16", "rows": 8192, "in": 4096, "out": 8192, "gated": True, "act": "swish",
         "bias": False},
        # the gradient of a small batch's dropout, odd sizes throughout
        {"name": "dropout_grad_f32", "op": "dropout", "dtype": "f32", "rows": 77, "cols": 1021, "p": 0.1, "act": "none", "bias": False,
         "residual": False},
        # a training batch's block output: dropout and the residual stream's addition
        {"name": "dropout_residual_bf16", "op": "dropout", "dtype": "bf16", "rows": 32768, "cols": 4096, "p": 0.1, "act": "none", "bias": False,
         "residual": True},
        # bias, activation and dropout between a block's two layers: value and derivative, both masked
        {"name": "dropout_act_bf16", "op": "dropout", "dtype": "bf16", "rows": 8192, "cols": 12288, "p": 0.2, "act": "gelu_erf", "bias": True,
         "residual": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log8(rng, lo, hi):
    return max(8, _log(rng, lo, hi) // 8 * 8)


def draw(rng):
    op = rng.choice(["gated_forward", "gated_backward", "f8_linear", "f8_linear", "dropout"])
    if op == "dropout":
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = max(64, cols // 64 * 64)                      # a model's width; otherwise any number
        case = {"op": op, "dtype": rng.choice(["f32", "bf16", "bf16", "f16"]), "rows": min(_log(rng, 1, 32768), (32768 * 4096) // cols),
                "cols": cols, "p": rng.choice([0.0, 0.05, 0.1, 0.2, 0.5]), "act": rng.choice(["none", "none", "gelu_erf", "gelu_tanh", "swish", "mish"])}
        if case["dtype"] == "f32":
            case["rows"] = max(1, case["rows"] // 2)
        case["residual"] = case["act"] == "none" and rng.random() < 0.6
        case["bias"] = case["act"] != "none" and rng.random() < 0.6
        if case["act"] != "none":
            case["rows"] = max(1, case["rows"] // 2)
        return case
    if op == "f8_linear":
        case = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "rows": _log(rng, 1, 8192), "in": _log(rng, 512, 8192), "out": _log(rng, 512, 8192),
                "gated": rng.random() < 0.5, "act": rng.choice(["none", "swish", "gelu_tanh", "gelu_erf", "mish"]), "bias": rng.random() < 0.5}
        if rng.random() < 0.8:
            case["in"], case["out"] = max(64, case["in"] // 64 * 64), max(64, case["out"] // 64 * 64)
        case["rows"] = max(1, min(case["rows"], 8192 * 4096 * 8192 // (case["in"] * case["out"])))
        return case
    experts = _log(rng, 1, 64)
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16"]), "rows": _log(rng, 1, 16384), "in": _log8(rng, 256, 4096),
            "out": _log8(rng, 256, 5632), "experts": experts, "bias": rng.random() < 0.5, "spare": rng.choice([0, 0, 5, 64]),
            "skew": rng.choice([0.5, 1.0, 4.0])}
    if rng.random() < 0.15:
        case["in"], case["out"] = case["in"] + 3, case["out"] + 1     # rows that start off every vector boundary
    case["rows"] = max(1, min(case["rows"], 16384 * 2048 * 5632 // (case["in"] * case["out"])))
    if op == "gated_forward":
        case["act"] = rng.choice(["none", "swish", "swish", "gelu_tanh", "gelu_erf", "mish"])
        case["train"] = rng.random() < 0.6
    else:
        case["down"] = not case["bias"] and rng.random() < 0.7
    return case


def work(case):
    es = SIZE[case["dtype"]]
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": es * n * (3 if case["residual"] or case["act"] != "none" else 2), "flops": (20 if case["act"] != "none" else 4) * n}
    m, k, n = case["rows"], case["in"], case["out"]
    if case["op"] == "f8_linear":
        wide = 2 * n if case["gated"] else n
        return {"bytes": k * wide + 2 * m * (k + n), "flops": 2 * m * k * wide}
    active = min(case["experts"], m)
    if case["op"] == "gated_forward":
        return {"bytes": 2 * (m * k + active * k * 2 * n + m * n * (3 if case["train"] else 1)), "flops": 4 * m * k * n}
    down = {"bytes": 2 * active * k * n, "flops": 2 * m * k * n} if case["down"] else {"bytes": 0, "flops": 0}
    first = m * k if case["down"] else m * n                     # the gradient that arrives
    return {"bytes": 2 * (first + 2 * m * n + 2 * m * k + active * k * 2 * n + case["experts"] * k * 2 * n) + down["bytes"],
            "flops": 8 * m * k * n + down["flops"]}


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


def _blocks(w):
    """Largest magnitude of each 128 x 128 block of the last two dimensions, spread over the block again, and once a block."""
    *lead, n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    pad = torch.zeros(*lead, nb * BLOCK, kb * BLOCK, device=w.device, dtype=w.dtype)
    pad[..., :n, :k] = w.abs()
    return pad.view(*lead, nb, BLOCK, kb, BLOCK).amax((-3, -1))


def _spread(scale, n, k):
    """Each block's scale over its elements."""
    return scale.repeat_interleave(BLOCK, -2)[..., :n, :].repeat_interleave(BLOCK, -1)[..., :k]


def prepare(case, seed):
    t = TYPES[case["dtype"]]
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)

    s = {"case": dict(case)}
    if case["op"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["x"] = normal(rows, cols, std=1.5)
        s["residual"] = normal(rows, cols, std=3.0) if case["residual"] else None
        s["bias"] = normal(cols, std=0.3) if case["bias"] else None
        s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 64, seed % 1000003 * 7
        s["step"] = torch.full((1,), seed % 977, dtype=torch.int64, device=DEV)      # a training program's step counter
        s["y"] = torch.empty_like(s["x"])
        s["dfdx"] = torch.empty_like(s["x"]) if case["act"] != "none" else None
    elif case["op"] == "f8_linear":
        m, k, n = case["rows"], case["in"], case["out"]
        lead = (2,) if case["gated"] else ()
        s["x"] = normal(m, k)
        s["x"][:, 5:: 97] *= 6.0                                   # the few loud channels that activations have
        w = normal(*lead, n, k, std=k ** -0.5, dtype=torch.float32)
        s["w_scale"] = _blocks(w) / LARGEST
        s["wq"] = (w / _spread(s["w_scale"], n, k)).clamp_(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
        s["bias"] = normal(*lead, n, std=0.3) if case["bias"] else None
        s["y"] = torch.empty(m, n, dtype=t, device=DEV)
    else:
        m, k, n, e = case["rows"] + case["spare"], case["in"], case["out"], case["experts"]
        off, s["longest"] = _offsets(case, seed)
        s["offsets"] = off.to(DEV)
        s["x"], s["w"] = normal(m, k), normal(e, 2, n, k, std=k ** -0.5)
        if case["op"] == "gated_forward":
            s["bias"] = normal(e, 2, n, std=0.3) if case["bias"] else None
            s["y"] = torch.empty(m, n, dtype=t, device=DEV)
            s["partials"] = torch.empty(m, 2, n, dtype=t, device=DEV) if case["train"] else None
        else:
            # f'(a) u and f(a) as a forward pass leaves them
            s["partials"] = torch.stack([normal(m, n, std=0.7, mean=0.0), normal(m, n, std=0.6, mean=0.3)], 1)
            s["grad_out"] = normal(m, k if case["down"] else n)
            s["w2"] = normal(e, k, n, std=n ** -0.5) if case["down"] else None
            s["gz"], s["gx"], s["gw"] = torch.empty_like(s["partials"]), torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["gb"] = torch.empty(e, 2, n, device=DEV) if case["bias"] else None
    return s


# ---------------------------------------------------------------- the plain forms

def _act_plain(z, kind, slope):
    if kind == "none":
        return z, torch.ones_like(z) if slope else None
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


def _whole(v, rows, like):
    """The rows that have an expert, and zeros behind them."""
    full = torch.zeros_like(like)
    full[:rows] = v.to(like.dtype)
    return full


def _gated_forward_plain(s):
    c, rows, n = s["case"], s["case"]["rows"], s["case"]["out"]
    e, at = _places(s)
    z = torch.bmm(_pad(s["x"][:rows].float(), e, at, s), s["w"].float().flatten(1, 2).transpose(1, 2))[e, at]
    if s["bias"] is not None:
        z = z + s["bias"].float().flatten(1)[e]
    a, u = z[:, :n], z[:, n:]
    f, slope = _act_plain(a, c["act"], c["train"])
    out = [_whole(f * u, rows, s["y"])]
    if c["train"]:
        out.append(_whole(torch.stack([slope * u, f], 1), rows, s["partials"]))
    return out


def _gated_backward_plain(s):
    c, t, rows = s["case"], TYPES[s["case"]["dtype"]], s["case"]["rows"]
    e, at = _places(s)
    g = s["grad_out"][:rows].float()
    if c["down"]:
        g = torch.bmm(_pad(g, e, at, s), s["w2"].float())[e, at]
    gz = _pad((g[:, None, :] * s["partials"][:rows].float()).flatten(1), e, at, s)
    gx = _whole(torch.bmm(gz, s["w"].float().flatten(1, 2))[e, at], rows, s["x"])
    gw = torch.bmm(gz.transpose(1, 2), _pad(s["x"][:rows].float(), e, at, s)).to(t)
    return [gx, gw.view(s["w"].shape), gz.sum(1).view(c["experts"], 2, c["out"]) if c["bias"] else None]


def _f8_plain(s):
    c = s["case"]
    m, k, n = c["rows"], c["in"], c["out"]
    x = s["x"].float()
    pad = torch.zeros(m, -(-k // BLOCK) * BLOCK, device=DEV)
    pad[:, :k] = x
    amax = pad.view(m, -1, BLOCK).abs().amax(2)
    # in 64 bits: many of these quotients lie on a border between two 8-bit values
    q = (x.double() * LARGEST / amax.double().repeat_interleave(BLOCK, 1)[:, :k]).to(torch.float8_e4m3fn).float()
    x = q * (amax / LARGEST).repeat_interleave(BLOCK, 1)[:, :k]
    w = s["wq"].float() * _spread(s["w_scale"], n, k)
    z = x @ w.reshape(-1, k).t()
    if s["bias"] is not None:
        z = z + s["bias"].float().flatten()
    y = _act_plain(z[:, :n], c["act"], False)[0]
    return (y * z[:, n:] if c["gated"] else y).to(s["y"].dtype)


def _random16(s, n):
    """16 random bits for each of n elements: counter-based generator Philox 4x32 with ten rounds (Salmon et al., 2011), eight
    elements a call; the key is the seed, the counter the call's index and offset + step."""
    lo = 0xffffffff
    i = torch.arange(-(-n // 8), device=DEV)
    at = s["offset"] + s["step"]
    c = [i & lo, i >> 32, (at & lo).expand_as(i), (at >> 32 & lo).expand_as(i)]
    k0, k1 = s["seed"] & lo, s["seed"] >> 32
    for _ in range(10):
        # a product of two 32-bit numbers as two sums that stay below 2^63
        words = []
        for v, m in ((c[0], 0xD2511F53), (c[2], 0xCD9E8D57)):
            low, high = v * (m & 0xffff), v * (m >> 16)
            total = low + ((high & 0xffff) << 16)
            words.append(((high >> 16) + (total >> 32) & lo, total & lo))
        (h0, l0), (h1, l1) = words
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & lo, (k1 + 0xBB67AE85) & lo
    return torch.stack([v for w in c for v in (w & 0xffff, w >> 16)], 1).flatten()[:n]


def _dropout_plain(s):
    c, t = s["case"], s["x"].dtype
    dropped = int(c["p"] * 65536 + 0.5)
    keep = (_random16(s, s["x"].numel()) >= dropped).view(s["x"].shape)
    scale = 65536.0 / (65536 - dropped)
    x = s["x"].float()
    if c["act"] == "none":
        y = torch.where(keep, x * scale, torch.zeros_like(x))
        return [(s["residual"].float() + y if s["residual"] is not None else y).to(t)]
    z = x + s["bias"].float() if s["bias"] is not None else x
    return [torch.where(keep, v * scale, torch.zeros_like(x)).to(t) for v in _act_plain(z, c["act"], True)]


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_plain(s):
    return {"gated_forward": _gated_forward_plain, "gated_backward": _gated_backward_plain, "f8_linear": _f8_plain,
            "dropout": _dropout_plain}[s["case"]["op"]](s)


def _run_own(s):
    import paper_2209_10778_b200 as nfad
    c = s["case"]
    act = None if c.get("act", "none") == "none" else c["act"]
    if c["op"] == "dropout":
        if "drop" not in s:
            s["drop"] = nfad.Dropout(c["p"], s["seed"], s["offset"], s["step"])
        if act is None:
            nfad.nfad_dropout(s["drop"], s["x"], s["residual"], s["y"])
            return [s["y"]]
        nfad.nfad_bias_act_dropout_forward(act, s["drop"], s["x"], s["bias"], s["y"], s["dfdx"])
        return [s["y"], s["dfdx"]]
    if c["op"] == "f8_linear":
        call = nfad.nfad_f8_gated_linear_dynamic if c["gated"] else nfad.nfad_f8_linear_dynamic
        if "scratch" not in s:
            s["scratch"] = nfad.nfad_f8_linear_dynamic_scratch(s["x"])
        call(act, s["x"], s["wq"], s["w_scale"], s["bias"], s["y"], s["scratch"])
        return s["y"]
    if c["op"] == "gated_forward":
        nfad.nfad_expert_gated_linear(act, s["x"], s["w"], s["bias"], s["offsets"], s["y"], s["partials"])
        return [s["y"]] if s["partials"] is None else [s["y"], s["partials"]]
    if c["down"]:
        nfad.nfad_expert_linear_backward_gated(s["grad_out"], s["w2"], s["offsets"], s["partials"], s["gz"])
    else:
        if "scratch" not in s:
            s["scratch"] = nfad.nfad_expert_act_backward_scratch(s["gz"].flatten(1))
        nfad.nfad_expert_gated_backward(s["grad_out"], s["partials"], s["offsets"], s["gz"], s["gb"], s["scratch"])
    gz, w = s["gz"].flatten(1), s["w"].flatten(1, 2)
    nfad.nfad_expert_linear_backward_input(gz, w, s["offsets"], None, s["gx"])
    nfad.nfad_expert_linear_backward_weight(gz, s["x"], s["offsets"], s["gw"].flatten(1, 2))
    return [s["gx"], s["gw"], s["gb"]]


# ---------------------------------------------------------------- 64 bits

def _act_exact(z, kind):
    """f and f' by the definitions, the derivative by automatic differentiation."""
    if kind == "none":
        return z, torch.ones_like(z)
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


def _to_eight_bits(v):
    """Nearest value with three fraction bits and exponents from -6 on, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return (v / step).round() * step


def _philox(seed, offset, n):
    """The generator on numpy's unsigned 64-bit integers, which hold a whole 32-bit product."""
    import numpy as np
    u, lo = np.uint64, np.uint64(0xffffffff)
    i = np.arange(-(-n // 8), dtype=u)
    x0, x1, x2, x3 = i & lo, i >> u(32), np.full_like(i, offset & 0xffffffff), np.full_like(i, offset >> 32)
    key = [seed & 0xffffffff, seed >> 32]
    for _ in range(10):
        a, b = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (b >> u(32)) ^ x1 ^ u(key[0]), b & lo, (a >> u(32)) ^ x3 ^ u(key[1]), a & lo
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    out = np.empty((len(i), 8), np.int32)
    for j, w in enumerate((x0, x1, x2, x3)):
        out[:, 2 * j], out[:, 2 * j + 1] = w & u(0xffff), w >> u(16)
    return torch.from_numpy(out.reshape(-1)[:n])


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if case["op"] == "dropout":
        dropped = round(case["p"] * 65536)
        bits = _philox(s["seed"], s["offset"] + int(s["step"]), s["x"].numel())
        factor = (bits >= dropped).view(s["x"].shape).to(DEV).double() / (1 - dropped / 65536)
        if case["act"] == "none":
            return [d["x"] * factor + (d["residual"] if d["residual"] is not None else 0.0)]
        return [v * factor for v in _act_exact(d["x"] + d["bias"] if d["bias"] is not None else d["x"], case["act"])]
    if case["op"] == "f8_linear":
        m, k, n = case["rows"], case["in"], case["out"]
        z = torch.zeros(m, (2 if case["gated"] else 1) * n, dtype=torch.float64, device=DEV)
        w, scales = d["wq"].reshape(-1, n, k), d["w_scale"].reshape(-1, *d["w_scale"].shape[-2:])
        for b, k0 in enumerate(range(0, k, BLOCK)):                # one block of the reduction after another
            x = d["x"][:, k0:k0 + BLOCK]
            amax = x.abs().amax(1, keepdim=True)
            part = _to_eight_bits(x * LARGEST / amax) * (amax / LARGEST)
            for j in range(len(w)):
                ws = scales[j, :, b].repeat_interleave(BLOCK)[:n]
                z[:, j * n:(j + 1) * n].addmm_(part, (w[j, :, k0:k0 + BLOCK] * ws[:, None]).t())
        if d["bias"] is not None:
            z += d["bias"].flatten()
        y = _act_exact(z[:, :n], case["act"])[0]
        return y * z[:, n:] if case["gated"] else y
    off = d["offsets"].tolist()
    parts = [(e, slice(off[e], off[e + 1])) for e in range(case["experts"]) if off[e + 1] > off[e]]
    if case["op"] == "gated_forward":
        y, both = torch.zeros_like(d["y"]), torch.zeros(*d["y"].shape[:1], 2, d["y"].shape[1], dtype=torch.float64, device=DEV)
        for e, p in parts:
            a, u = (d["x"][p] @ d["w"][e, j].t() + (d["bias"][e, j] if d["bias"] is not None else 0.0) for j in (0, 1))
            f, slope = _act_exact(a, case["act"])
            y[p], both[p, 0], both[p, 1] = f * u, slope * u, f
        return [y, both] if case["train"] else [y]
    gx, gw = torch.zeros_like(d["x"]), torch.zeros_like(d["w"])
    gb = torch.zeros(case["experts"], 2, case["out"], dtype=torch.float64, device=DEV)
    for e, p in parts:
        g = d["grad_out"][p] @ d["w2"][e] if case["down"] else d["grad_out"][p]
        for j in (0, 1):
            gz = g * d["partials"][p, j]
            gx[p] += gz @ d["w"][e, j]
            gw[e, j], gb[e, j] = gz.t() @ d["x"][p], gz.sum(0)
    return [gx, gw, gb if case["bias"] else None]
