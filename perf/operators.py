"""What is timed of the operators around a residual block of a language model: its norms, gate and residual scale, and the update.

Two kinds of case, each through the package's public entry points where ``own`` is true and in elementary operations where
it is not:

  adamw   one ``dsp_adamw_step`` over all tensors of a model: decoupled weight decay, optionally a clip by the norm of all
          gradients and a bfloat16 copy of the new parameters; states of 32 bits, or of 8 (e4m3 and e5m2 with one power of
          two for each 256 elements, rounded stochastically from a counter).
  norm    ``dsp_norm_residual_forward`` or ``dsp_norm_residual_backward``: y = alpha x + beta act(gate) N_post(z),
          h = N_pre(y) over rows, and its gradients.

The parameters of a model lie in one buffer, every tensor on a multiple of 256 elements with zeros behind it (``misalign``
shifts the buffer by that many elements), so that a plain form can treat them all at once.
"""
import math
import random

import torch

own = False

_BLOCK = 256  # elements that share a power of two in the 8-bit states
_BETAS = (0.9, 0.999)


def listed():
    return [
        # a network of a few thousand weights: the call is as long as its launches
        {"name": "adamw32_tiny", "kind": "adamw", "bits": 32, "layers": 0, "width": 0, "ff": 0, "vocab": 0, "tensors": 14,
         "largest": 2304, "grad": "fp32", "copy": False, "max_norm": 0.0, "misalign": 0, "lr": 1e-3},
        # a convolutional network's 62 tensors, fp32 gradients, bf16 copies, clipped
        {"name": "adamw32_clip", "kind": "adamw", "bits": 32, "layers": 0, "width": 0, "ff": 0, "vocab": 0, "tensors": 62,
         "largest": 2359296, "grad": "fp32", "copy": True, "max_norm": 1.0, "misalign": 0, "lr": 1e-3},
        # a language model of 270 million parameters, bf16 gradients and copies
        {"name": "adamw32_lm", "kind": "adamw", "bits": 32, "layers": 4, "width": 2048, "ff": 5632, "vocab": 32000, "tensors": 0,
         "largest": 0, "grad": "bf16", "copy": True, "max_norm": 0.0, "misalign": 0, "lr": 1e-4},
        # the same model fine-tuned with 8-bit states, clipped
        {"name": "adamw8_lm", "kind": "adamw", "bits": 8, "layers": 4, "width": 2048, "ff": 5632, "vocab": 32000, "tensors": 0,
         "largest": 0, "grad": "bf16", "copy": True, "max_norm": 1.0, "misalign": 0, "lr": 2e-5},
        # 300 tensors of ragged sizes whose parameters lie on odd addresses, fp32 gradients
        {"name": "adamw8_ragged", "kind": "adamw", "bits": 8, "layers": 0, "width": 0, "ff": 0, "vocab": 0, "tensors": 300,
         "largest": 300001, "grad": "fp32", "copy": False, "max_norm": 0.0, "misalign": 1, "lr": 2e-5},
        # one token at a time through a wide model
        {"name": "norm_fwd_token", "kind": "norm", "back": False, "rows": 1, "width": 4096, "dtype": "bf16", "post": "rms",
         "pre": "rms", "gate": "vector", "gate_rows": 0, "act": "identity", "bias": False, "pad": 0},
        # training rows of the same model, norms on both sides of the block
        {"name": "norm_fwd_rms", "kind": "norm", "back": False, "rows": 32768, "width": 4096, "dtype": "bf16", "post": "rms",
         "pre": "rms", "gate": "vector", "gate_rows": 0, "act": "identity", "bias": False, "pad": 0},
        {"name": "norm_bwd_rms", "kind": "norm", "back": True, "rows": 32768, "width": 4096, "dtype": "bf16", "post": "rms",
         "pre": "rms", "gate": "vector", "gate_rows": 0, "act": "identity", "bias": False, "pad": 0},
        # one gate a picture, as a model conditioned on a time step has it: 32 pictures of 256 positions
        {"name": "norm_bwd_picture_gate", "kind": "norm", "back": True, "rows": 8192, "width": 1152, "dtype": "bf16",
         "post": "none", "pre": "layer", "gate": "rows", "gate_rows": 256, "act": "identity", "bias": False, "pad": 0},
        # a gate for every element, from a branch of its own
        {"name": "norm_fwd_token_gate", "kind": "norm", "back": False, "rows": 6000, "width": 2560, "dtype": "bf16",
         "post": "rms", "pre": "layer", "gate": "rows", "gate_rows": 1, "act": "sigmoid", "bias": True, "pad": 0},
        # odd sizes throughout, fp32, rows that lie apart
        {"name": "norm_fwd_odd", "kind": "norm", "back": False, "rows": 1913, "width": 1431, "dtype": "fp32", "post": "layer",
         "pre": "layer", "gate": "rows", "gate_rows": 137, "act": "tanh", "bias": True, "pad": 6},
        {"name": "norm_bwd_odd", "kind": "norm", "back": True, "rows": 1913, "width": 1431, "dtype": "fp32", "post": "layer",
         "pre": "layer", "gate": "rows", "gate_rows": 137, "act": "tanh", "bias": True, "pad": 6},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        bits = rng.choice([32, 8])
        case = {"kind": "adamw", "bits": bits, "layers": 0, "width": 0, "ff": 0, "vocab": 0, "tensors": 0, "largest": 0,
                "grad": rng.choice(["fp32", "bf16"]), "copy": rng.random() < 0.5, "max_norm": rng.choice([0.0, 1.0]),
                "misalign": rng.choice([0, 0, 0, 1, 3]), "lr": 2e-5 if bits == 8 else 3e-4}
        if rng.random() < 0.5:
            width = 64 * _log(rng, 2, 24)
            return {**case, "layers": rng.randint(1, 8), "width": width, "ff": 32 * _log(rng, width // 16, width // 8) + rng.choice([0, 0, 1]),
                    "vocab": _log(rng, 1000, 50000)}
        return {**case, "tensors": _log(rng, 1, 400), "largest": _log(rng, 100, 4000000)}
    gate = rng.choice(["none", "vector", "rows", "rows"])
    act = rng.choice(["identity", "sigmoid", "tanh"])
    width = _log(rng, 48, 8192)
    if rng.random() < 0.7:
        width = width // 16 * 16
    rows = _log(rng, 1, min(32768, (1 << 26) // width))
    return {"kind": "norm", "back": rng.random() < 0.5, "rows": rows, "width": width, "dtype": rng.choice(["bf16", "bf16", "fp32"]),
            "post": rng.choice(["none", "rms", "rms", "layer"]), "pre": rng.choice(["none", "rms", "rms", "layer"]), "gate": gate,
            "gate_rows": rng.choice([1, _log(rng, 1, 2 * rows)]) if gate == "rows" else 0, "act": act,
            "bias": rng.random() < 0.4, "pad": rng.choice([0, 0, 0, 8, 3])}


def _sizes(case):
    """Elements of every tensor, and whether weight decay applies to it (matrices) or not (gains, biases)."""
    if case["tensors"]:
        r, lo = random.Random(case["tensors"]), math.log(1 if case["largest"] < 1000 else 16)
        sizes = [int(math.exp(r.uniform(lo, math.log(case["largest"])))) for _ in range(case["tensors"] - 1)] + [case["largest"]]
        return [(n, n > 512) for n in sizes]
    w, f = case["width"], case["ff"]
    layer = [(w, False)] + [(w * w, True)] * 4 + [(w, False)] + [(w * f, True)] * 3
    return [(case["vocab"] * w, True)] + layer * case["layers"] + [(w, False)]


# ----------------------------------------------------------------------------- what a program has in hand
_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


class _Object:
    """A library object that is given back when the state goes."""

    def __init__(self, handle, destroy):
        self.handle, self.destroy = handle, destroy

    def __del__(self):
        self.destroy(self.handle)


def _prepare_adamw(case, seed):
    gen = _generator(seed)
    sizes = _sizes(case)
    blocks = [-(-n // _BLOCK) for n, _ in sizes]
    total, shift = sum(blocks) * _BLOCK, case["misalign"]
    starts = [sum(blocks[:j]) * _BLOCK for j in range(len(blocks))]
    per = torch.tensor(blocks, device="cuda")
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), per)
    first = (torch.arange(len(tensor), device="cuda") - (torch.cumsum(per, 0) - per)[tensor]) * _BLOCK
    decay = torch.tensor([float(d) for _, d in sizes], device="cuda")[tensor]
    length = torch.tensor([n for n, _ in sizes], device="cuda")[tensor]

    def flat(values, dtype):
        buffer = torch.zeros(total + shift, dtype=dtype, device="cuda")[shift:]
        return buffer.copy_(values)

    inside = (first[:, None] + torch.arange(_BLOCK, device="cuda") < length[:, None]).reshape(-1)
    # gradients whose size differs from tensor to tensor and, less, from row to row; what their averages look like on the way
    scale = torch.exp(1.5 * _rand(gen, len(sizes)))[tensor] * 1e-4 * torch.exp(0.5 * _rand(gen, len(tensor)))
    scale = scale.repeat_interleave(_BLOCK) * inside
    grad = flat(_rand(gen, total) * scale, _TYPES[case["grad"]])
    x = torch.where(decay.repeat_interleave(_BLOCK) > 0, 0.04 * _rand(gen, total), 1 + 0.05 * _rand(gen, total)) * inside
    m = 0.25 * scale * _rand(gen, total)
    v = scale.square() * torch.exp(0.3 * _rand(gen, total))
    del scale
    s = {"case": case, "seed": seed, "t": 1000, "x": flat(x, torch.float32), "grad": grad, "tensor": tensor, "first": first,
         "decay": decay, "norm": torch.zeros(1, device="cuda"),
         "copy": flat(x, torch.bfloat16) if case["copy"] else None}
    del x
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        for name, a, top, low, dtype in (("m", m, 7, 2.0 ** -9, torch.float8_e4m3fn), ("v", v, 14, 2.0 ** -16, torch.float8_e5m2)):
            a = a.view(-1, _BLOCK)
            e = (torch.floor(torch.log2(a.abs().amax(1).clamp(min=1e-38))) + (127 - top)).clamp(0, 254)
            a = a * torch.exp2(127 - e)[:, None]
            if name == "v":
                a = torch.where(a > 0, a.clamp(min=low), a)
            s[name], s[name + "_exp"] = a.to(dtype).reshape(-1), e.to(torch.uint8).view(torch.float8_e8m0fnu)
    del m, v
    if own:
        import paper_1909_02625_amd as D
        cut = lambda name, j: None if s.get(name) is None else s[name][starts[j]:starts[j] + sizes[j][0]]  # noqa: E731
        exps = lambda name, j: s[name][starts[j] // _BLOCK:starts[j] // _BLOCK + blocks[j]] if name in s else None  # noqa: E731
        tensors = [{"param": cut("x", j), "grad": cut("grad", j), "copy": cut("copy", j), "m": cut("m", j), "v": cut("v", j),
                    "m_exp": exps("m_exp", j), "v_exp": exps("v_exp", j), "decay": sizes[j][1]} for j in range(len(sizes))]
        s["opt"] = _Object(D.dsp_adamw_init(tensors, case["bits"], seed), D.dsp_adamw_destroy)
        D.dsp_adamw_set_steps(s["opt"].handle, s["t"], *_BETAS)
    return s


def _spread(case, a):
    """The rows of ``a`` with ``pad`` elements between them."""
    if not case["pad"]:
        return a
    wide = torch.zeros(a.shape[0], a.shape[1] + case["pad"], dtype=a.dtype, device=a.device)
    wide[:, :a.shape[1]] = a
    return wide[:, :a.shape[1]]


def _prepare_norm(case, seed):
    gen, dtype, rows, width = _generator(seed), _TYPES[case["dtype"]], case["rows"], case["width"]
    n = lambda std: _spread(case, (_rand(gen, rows, width) * std).to(dtype))  # noqa: E731
    s = {"case": case, "alpha": 1.0 if case["post"] != "none" else 0.9, "beta": 0.7, "eps": 1e-5, "gate": None}
    spread = torch.exp(0.4 * _rand(gen, rows, 1))  # the residual stream grows, and not alike for every token
    s["z"] = _spread(case, (_rand(gen, rows, width) * spread + 0.1).to(dtype))
    s["x"] = _spread(case, (_rand(gen, rows, width) * 2 * spread + 0.3).to(dtype))
    for name in ("post", "pre"):
        has = case[name] != "none"
        s[name + "_gain"] = 1 + 0.2 * _rand(gen, width) if has else None
        s[name + "_bias"] = 0.2 * _rand(gen, width) if has and case["bias"] else None
    if case["gate"] == "vector":  # a parameter, small at the start of training
        s["gate"], s["gate_rows"] = 0.5 + 0.1 * _rand(gen, 1, width), max(1, rows)
    elif case["gate"] == "rows":
        s["gate"], s["gate_rows"] = _rand(gen, -(-rows // case["gate_rows"]), width).to(dtype), case["gate_rows"]
    if case["back"]:
        s["x"] = None
        y, _, post, pre = _forward({**s, "x": n(2.0)})
        s["y"], s["post_stats"], s["pre_stats"] = _spread(case, y), post, pre
        s["dy"] = n(0.01)
        s["dh"] = n(0.01) if case["pre"] != "none" else None
    if own:
        import paper_1909_02625_amd as D
        code, stride = {"fp32": D.DSP_FP32, "bf16": D.DSP_BF16}, width + case["pad"]
        kinds = {"none": D.DSP_NORM_NONE, "rms": D.DSP_NORM_RMS, "layer": D.DSP_NORM_LAYER}
        acts = {"identity": D.DSP_GATE_IDENTITY, "sigmoid": D.DSP_GATE_SIGMOID, "tanh": D.DSP_GATE_TANH}
        s["desc"] = D.make_norm_residual_desc(
            rows, width, code[case["dtype"]], post=kinds[case["post"]], pre=kinds[case["pre"]], alpha=s["alpha"], beta=s["beta"],
            eps=s["eps"], gate_rows=0 if s["gate"] is None else s["gate_rows"], gate_act=acts[case["act"]],
            gate_dtype=code["fp32" if case["gate"] == "vector" else case["dtype"]], x_stride=stride, z_stride=stride)
        new = lambda like: torch.empty(like.shape, dtype=like.dtype, device="cuda")  # noqa: E731
        if case["back"]:
            bytes_ = D.dsp_norm_residual_workspace_bytes(s["desc"])
            s["desc"].y_stride = s["desc"].h_stride = stride
            s["ws"] = torch.empty(max(16, bytes_), dtype=torch.uint8, device="cuda"), bytes_
            s["dx"], s["dz"] = _spread(case, new(s["y"])), _spread(case, new(s["z"]))
            s["dgate"] = None if s["gate"] is None else new(s["gate"])
            for name in ("post_gain", "post_bias", "pre_gain", "pre_bias"):
                s["d" + name] = None if s[name] is None else new(s[name])
        else:
            s["y"], s["h"] = new(s["x"]), new(s["x"]) if case["pre"] != "none" else None
            for name in ("post", "pre"):
                s[name + "_stats"] = torch.empty(2, rows, device="cuda") if case[name] != "none" else None
    return s


def prepare(case, seed):
    return _prepare_adamw(case, seed) if case["kind"] == "adamw" else _prepare_norm(case, seed)


# ----------------------------------------------------------------------------- the plain forms
def _mix(x):
    """A bijection of the 32-bit numbers that spreads every bit over all; whole tensors of int64, or a Python int."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_halves(s):
    """The 16 + 16 random bits of every element at step t: a function of seed, step, tensor and element."""
    seed = _mix((s["seed"] & 0xFFFFFFFF) ^ _mix((s["seed"] >> 32) ^ 0xBB67AE85))
    key = _mix(_mix(_mix(seed ^ (s["t"] & 0xFFFFFFFF)) ^ s["tensor"]) ^ (s["first"] >> 32))
    low = (s["first"] & 0xFFFFFFFF)[:, None] + torch.arange(_BLOCK, device="cuda")
    r = _mix(key[:, None] ^ low)
    return r & 0xFFFF, r >> 16


def _stochastic(a, top, lowest, mantissa, r, dtype):
    """Rows of ``a`` over a power of two each, rounded up with the probability of what lies above the value below."""
    e = (torch.frexp(a.abs().amax(1)).exponent + (126 - top)).clamp(0, 254)
    a = torch.ldexp(a.double(), (127 - e)[:, None])
    step = torch.ldexp(torch.ones_like(a), (torch.frexp(a).exponent - 1).clamp(min=lowest) - mantissa)
    rounded = torch.floor(a.abs() / step + r / 65536.0) * step
    if dtype == torch.float8_e5m2:  # what is positive stays positive
        rounded = torch.where((a > 0) & (rounded == 0), step, rounded)
    return torch.copysign(rounded, a).to(dtype), e.to(torch.uint8).view(torch.float8_e8m0fnu)


def _adamw(s):
    case, (b1, b2) = s["case"], _BETAS
    g = s["grad"].float().reshape(-1, _BLOCK)
    s["t"] += 1
    if case["max_norm"]:
        s["norm"] = s["grad"].double().square().sum().sqrt().float().reshape(1)
        g = g * (case["max_norm"] / s["norm"]).clamp(max=1.0)
    if case["bits"] == 32:
        m, v = s["m"].view(-1, _BLOCK), s["v"].view(-1, _BLOCK)
    else:
        m, v = (s[n].float().view(-1, _BLOCK) * s[n + "_exp"].float()[:, None] for n in ("m", "v"))
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    x = s["x"].view(-1, _BLOCK)
    d = m / (1 - b1 ** s["t"]) / ((v / (1 - b2 ** s["t"])).sqrt() + 1e-8)
    x = x - case["lr"] * (d + 0.1 * s["decay"][:, None] * x)
    s["x"].view(-1, _BLOCK).copy_(x)
    if case["copy"]:
        s["copy"].view(-1, _BLOCK).copy_(x)
    if case["bits"] == 32:
        s["m"].view(-1, _BLOCK).copy_(m)
        s["v"].view(-1, _BLOCK).copy_(v)
    else:
        low, high = _random_halves(s)
        for name, a, top, lowest, mantissa, r in (("m", m, 7, -6, 3, low), ("v", v, 14, -14, 2, high)):
            code, e = _stochastic(a, top, lowest, mantissa, r, s[name].dtype)
            s[name].copy_(code.reshape(-1))
            s[name + "_exp"].copy_(e)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    names = ["x", "m", "v"] + (["copy"] if s["case"]["copy"] else []) + (["norm"] if s["case"]["max_norm"] else [])
    return {n: s[n] for n in names + (["m_exp", "v_exp"] if s["case"]["bits"] == 8 else [])}


def _stats(kind, a, eps):
    """Mean (0 for rms) and 1 / deviation of every row."""
    mean = a.mean(1) if kind == "layer" else torch.zeros_like(a[:, 0])
    return torch.stack([mean, torch.rsqrt((a - mean[:, None]).square().mean(1) + eps)])


def _gate(s):
    """act(gate) and its derivative for every row, or 1."""
    if s["gate"] is None:
        return 1.0, None
    g, act = s["gate"].float()[torch.arange(s["case"]["rows"], device="cuda") // s["gate_rows"]], s["case"]["act"]
    if act == "identity":
        return g, torch.ones_like(g)
    a = torch.sigmoid(g) if act == "sigmoid" else torch.tanh(g)
    return a, a * (1 - a) if act == "sigmoid" else 1 - a * a


def _affine(a, stats, gain, bias):
    n = (a - stats[0][:, None]) * stats[1][:, None] * gain
    return n if bias is None else n + bias


def _forward(s):
    case, n, post, pre, h = s["case"], s["z"].float(), None, None, None
    if case["post"] != "none":
        post = _stats(case["post"], n, s["eps"])
        n = _affine(n, post, s["post_gain"], s["post_bias"])
    y = s["alpha"] * s["x"].float() + s["beta"] * _gate(s)[0] * n
    if case["pre"] != "none":
        pre = _stats(case["pre"], y, s["eps"])
        h = _affine(y, pre, s["pre_gain"], s["pre_bias"]).to(s["z"].dtype)
    return y.to(s["z"].dtype), h, post, pre


def _norm_back(kind, d, hat, inv):
    """Gradient of the input of a norm from that of its normalised rows."""
    d = d - hat * (d * hat).mean(1, keepdim=True) - (d.mean(1, keepdim=True) if kind == "layer" else 0.0)
    return d * inv[:, None]


def _backward(s):
    case, out, D = s["case"], {}, s["dy"].float()
    if case["pre"] != "none":
        dh, hat = s["dh"].float(), (s["y"].float() - s["pre_stats"][0][:, None]) * s["pre_stats"][1][:, None]
        out["dpre_gain"], out["dpre_bias"] = (dh * hat).sum(0), dh.sum(0) if case["bias"] else None
        D = D + _norm_back(case["pre"], dh * s["pre_gain"], hat, s["pre_stats"][1])
    z, act, slope = s["z"].float(), *_gate(s)
    if case["post"] != "none":
        z = (z - s["post_stats"][0][:, None]) * s["post_stats"][1][:, None]
    dn = s["beta"] * act * D
    if s["gate"] is not None:
        n = z if case["post"] == "none" else z * s["post_gain"] if s["post_bias"] is None else z * s["post_gain"] + s["post_bias"]
        rows = torch.arange(case["rows"], device="cuda") // s["gate_rows"]
        c = s["beta"] * slope * n * D
        c = c.sum(0, keepdim=True) if len(s["gate"]) == 1 else torch.zeros_like(s["gate"], dtype=torch.float32).index_add_(0, rows, c)
        out["dgate"] = c.to(s["gate"].dtype)
    if case["post"] != "none":
        out["dpost_gain"], out["dpost_bias"] = (dn * z).sum(0), dn.sum(0) if case["bias"] else None
        dn = _norm_back(case["post"], dn * s["post_gain"], z, s["post_stats"][1])
    out["dx"], out["dz"] = (s["alpha"] * D).to(s["y"].dtype), dn.to(s["y"].dtype)
    return out


# ----------------------------------------------------------------------------- one pass
def run(state):
    s, case = state, state["case"]
    if not own:
        if case["kind"] == "adamw":
            return _adamw(s)
        return _backward(s) if case["back"] else dict(zip(("y", "h", "post_stats", "pre_stats"), _forward(s)))
    import paper_1909_02625_amd as D
    if case["kind"] == "adamw":
        D.dsp_adamw_step(s["opt"].handle, case["lr"], *_BETAS, 1e-8, 0.1, case["max_norm"], s["norm"] if case["max_norm"] else None)
        return _adamw_outputs(s)
    if not case["back"]:
        D.dsp_norm_residual_forward(s["desc"], s["x"], s["z"], s["gate"], s["post_gain"], s["post_bias"], s["pre_gain"], s["pre_bias"],
                                    s["y"], s["h"], s["post_stats"], s["pre_stats"])
        return {n: s[n] for n in ("y", "h", "post_stats", "pre_stats")}
    D.dsp_norm_residual_backward(s["desc"], s["dh"], s["dy"], s["y"], s["z"], s["gate"], s["post_gain"], s["post_bias"], s["pre_gain"],
                                 s["post_stats"], s["pre_stats"], s["dx"], s["dz"], s["dgate"], s["dpost_gain"], s["dpost_bias"],
                                 s["dpre_gain"], s["dpre_bias"], *s["ws"])
    return {n: s[n] for n in ("dx", "dz", "dgate", "dpost_gain", "dpost_bias", "dpre_gain", "dpre_bias")}


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "adamw":
        n = sum(n for n, _ in _sizes(case))
        g = 2 if case["grad"] == "bf16" else 4
        # the parameters and both states in and out, the gradients in (once more for their norm), the copy out
        states = 16 if case["bits"] == 32 else 4 + 4 / _BLOCK
        return {"bytes": n * (8 + states + g * (2 if case["max_norm"] else 1) + (2 if case["copy"] else 0)), "flops": 16.0 * n}
    n, e = case["rows"] * case["width"], 2 if case["dtype"] == "bf16" else 4
    pre = case["pre"] != "none"
    gates = 0 if case["gate"] == "none" else 4 * case["width"] if case["gate"] == "vector" else \
        e * case["width"] * -(-case["rows"] // case["gate_rows"])
    stats = 8 * case["rows"] * (pre + (case["post"] != "none"))
    if case["back"]:  # dy, z, dx, dz and, with a norm in front of the next block, dh and y
        vectors = 4 * case["width"] * (2 + case["bias"]) * (pre + (case["post"] != "none"))
        z = n if case["post"] != "none" or case["gate"] != "none" else 0
        return {"bytes": e * ((5 if pre else 3) * n + z) + 2 * gates + stats + vectors, "flops": 30.0 * n}
    vectors = 4 * case["width"] * (1 + case["bias"]) * (pre + (case["post"] != "none"))
    return {"bytes": e * (4 if pre else 3) * n + gates + stats + vectors, "flops": 16.0 * n}


# ----------------------------------------------------------------------------- in 64 bits, from the definitions
def _exact_mixed(seed, t, tensor, first):
    """The random bits once more, by the definition's words: five numbers mixed into one another, 32 bits each."""
    word = 2 ** 32

    def spread(k):
        k = torch.bitwise_xor(k, torch.div(k, 2 ** 16, rounding_mode="floor"))
        k = torch.remainder(k * 2654435769, word)
        k = torch.bitwise_xor(k, torch.div(k, 2 ** 15, rounding_mode="floor"))
        k = torch.remainder(k * 1779033703, word)
        return torch.bitwise_xor(k, torch.div(k, 2 ** 16, rounding_mode="floor"))

    number = lambda k: torch.tensor(k, dtype=torch.int64, device="cuda")  # noqa: E731
    k = spread(number(seed // word) ^ number(3144134277))
    k = spread(number(seed % word) ^ k)
    k = spread(spread(spread(k ^ number(t % word)) ^ tensor) ^ torch.div(first, word, rounding_mode="floor"))
    return spread(torch.remainder(first, word)[:, None] + torch.arange(_BLOCK, device="cuda")[None] ^ k[:, None])


def _exact_adamw(case, seed):
    s = _prepare_adamw({**case, "name": ""}, seed)
    b1, b2, t = _BETAS[0], _BETAS[1], s["t"] + 1
    g = s["grad"].double().reshape(-1, _BLOCK)
    norm = torch.sqrt(torch.sum(g * g)).reshape(1)
    if case["max_norm"] and float(norm) > case["max_norm"]:
        g = g * (case["max_norm"] / float(norm))
    if case["bits"] == 8:
        m, v = (s[n].double().reshape(-1, _BLOCK) * s[n + "_exp"].double()[:, None] for n in ("m", "v"))
    else:
        m, v = s["m"].double().reshape(-1, _BLOCK), s["v"].double().reshape(-1, _BLOCK)
    m = m + (1.0 - b1) * (g - m)
    v = v + (1.0 - b2) * (g * g - v)
    x = s["x"].double().reshape(-1, _BLOCK)
    x = x * (1.0 - case["lr"] * 0.1 * s["decay"].double())[:, None] - case["lr"] * (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + 1e-8)
    out = {"x": x.reshape(-1)}
    if case["copy"]:
        out["copy"] = x.reshape(-1)
    if case["max_norm"]:
        out["norm"] = norm
    if case["bits"] == 32:
        return {**out, "m": m.reshape(-1), "v": v.reshape(-1)}
    r = _exact_mixed(seed, t, s["tensor"], s["first"])
    for name, a, low, high, bits, chance in (("m", m, -6, 7, 3, torch.remainder(r, 65536)), ("v", v, -14, 14, 2, torch.div(r, 65536, rounding_mode="floor"))):
        power = torch.floor(torch.log2(torch.amax(torch.abs(a), 1))) - high
        power = torch.where(torch.isfinite(power), power, torch.full_like(power, -127.0)).clamp(min=-127.0)
        a = a * torch.exp2(-power)[:, None]
        grid = torch.exp2(torch.floor(torch.log2(torch.abs(a).clamp(min=2.0 ** (low - 1)))).clamp(min=low) - bits)
        below = torch.floor(torch.abs(a) / grid)
        value = (below + ((torch.abs(a) / grid - below) * 65536 + chance >= 65536).double()) * grid
        if name == "v":
            value = torch.where((a > 0) & (value == 0), grid, value)
        out[name], out[name + "_exp"] = (value * torch.sign(a)).reshape(-1), torch.exp2(power)
    return out


def _exact_norm(case, seed):
    s = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in _prepare_norm(case, seed).items()}
    rows, width, pre, post = case["rows"], case["width"], case["pre"] != "none", case["post"] != "none"
    of = lambda k, other: s[k] if s.get(k) is not None else other  # noqa: E731
    moments = lambda kind, a: (a.sum(1) / width if kind == "layer" else a.sum(1) * 0)  # noqa: E731
    gate = slope = 1.0
    which = torch.arange(rows, device="cuda") // s.get("gate_rows", 1)
    if s["gate"] is not None:
        raw = torch.index_select(s["gate"], 0, which)
        gate, slope = {"identity": lambda: (raw, 1.0), "tanh": lambda: (torch.tanh(raw), 1 / torch.cosh(raw) ** 2),
                       "sigmoid": lambda: (1 / (1 + torch.exp(-raw)), 1 / ((1 + torch.exp(-raw)) * (1 + torch.exp(raw))))}[case["act"]]()
    if not case["back"]:
        out, n = {}, s["z"]
        if post:
            mean = moments(case["post"], n)
            std = torch.sqrt(((n - mean[:, None]) ** 2).sum(1) / width + s["eps"])
            out["post_stats"] = torch.stack([mean, 1 / std])
            n = (n - mean[:, None]) / std[:, None] * of("post_gain", 1.0) + of("post_bias", 0.0)
        y = s["alpha"] * s["x"] + s["beta"] * gate * n
        if pre:
            mean = moments(case["pre"], y)
            std = torch.sqrt(((y - mean[:, None]) ** 2).sum(1) / width + s["eps"])
            out["pre_stats"] = torch.stack([mean, 1 / std])
            out["h"] = (y - mean[:, None]) / std[:, None] * of("pre_gain", 1.0) + of("pre_bias", 0.0)
        return {**out, "y": y}

    def through(kind, d, hat, inv):  # the Jacobian of the normalised row, applied to d
        centred = d - d.sum(1)[:, None] / width if kind == "layer" else d
        return (centred - hat * (d * hat).sum(1)[:, None] / width) * inv[:, None]

    out, total = {}, s["dy"]
    if pre:
        hat = (s["y"] - s["pre_stats"][0][:, None]) * s["pre_stats"][1][:, None]
        out["dpre_gain"] = torch.sum(s["dh"] * hat, 0)
        if case["bias"]:
            out["dpre_bias"] = torch.sum(s["dh"], 0)
        total = total + through(case["pre"], s["dh"] * s["pre_gain"], hat, s["pre_stats"][1])
    hat = (s["z"] - s["post_stats"][0][:, None]) * s["post_stats"][1][:, None] if post else s["z"]
    if s["gate"] is not None:
        c = s["beta"] * slope * (hat * of("post_gain", 1.0) + of("post_bias", 0.0)) * total
        out["dgate"] = torch.zeros_like(s["gate"]).index_add_(0, which, c)
    branch = s["beta"] * gate * total
    out["dx"] = s["alpha"] * total
    if post:
        out["dpost_gain"] = torch.sum(branch * hat, 0)
        if case["bias"]:
            out["dpost_bias"] = torch.sum(branch, 0)
        branch = through(case["post"], branch * s["post_gain"], hat, s["post_stats"][1])
    return {**out, "dz": branch}


def exact(case, seed):
    return _exact_adamw(case, seed) if case["kind"] == "adamw" else _exact_norm(case, seed)
