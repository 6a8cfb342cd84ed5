"""The operators around a residual block of a language model in plain numpy, 64 bits, from their definitions: test infrastructure."""
import numpy as np

RMS, LAYER = 1, 2


# ---- AdamW
def mix32(x):
    x = np.asarray(x, np.uint64)
    mask = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x9E3779B9)) & mask
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x6A09E667)) & mask
    return x ^ (x >> np.uint64(16))


def random_halves(seed, step, tensor, n, first=0):
    """The 16 + 16 random bits of elements first .. first + n - 1 of tensor ``tensor`` at step ``step``."""
    mask = 0xFFFFFFFF
    i = np.arange(first, first + n, dtype=np.uint64)
    s = mix32(np.uint64(seed & mask) ^ mix32(np.uint64((seed >> 32) ^ 0xBB67AE85)))
    k = mix32(mix32(mix32(s ^ np.uint64(step & mask)) ^ np.uint64(tensor)) ^ (i >> np.uint64(32)))
    r = mix32(k ^ (i & np.uint64(mask)))
    return (r & np.uint64(0xFFFF)).astype(np.float64), (r >> np.uint64(16)).astype(np.float64)


def decode(codes, exps, mantissa, bias):
    """Values of 8-bit floats (sign, exponent, mantissa bits) times their block's power of two; the all-ones code is NaN."""
    c = np.asarray(codes, np.int64)
    mag, sign = c & 127, np.where(c >= 128, -1.0, 1.0)
    e, f = mag >> mantissa, mag & ((1 << mantissa) - 1)
    v = np.where(e == 0, np.ldexp(f.astype(float), 1 - bias - mantissa),
                 np.ldexp((f + (1 << mantissa)).astype(float), (e - bias - mantissa).astype(int)))
    v = np.where(mag == 127, np.nan, v)
    scale = np.ldexp(1.0, np.repeat(np.asarray(exps, np.int64), 256)[:c.size] - 127)
    return sign * v * scale


def encode(a, r, mantissa, bias, top, keep_positive):
    """Blocks of 256: the power of two puts the largest finite magnitude into [2^top, 2^(top+1)); rounded up where the part above
    the value below plus r / 2^16 reaches 1.  Returns codes, exps."""
    a = np.asarray(a, np.float64)
    n = a.size
    codes, exps = np.zeros(n, np.uint8), np.zeros(-(-n // 256), np.uint8)
    for b in range(exps.size):
        s = slice(256 * b, min(n, 256 * b + 256))
        mag, fin = np.abs(a[s]), np.isfinite(a[s])
        big = mag[fin].max() if fin.any() else 0.0
        e = 0 if big < 2.0 ** -126 else max(0, int(np.frexp(big)[1]) - 1 - top + 127)
        exps[b] = e
        x = np.ldexp(np.where(fin, mag, 0.0), 127 - e)
        ex = np.maximum(np.where(x > 0, np.frexp(x)[1] - 1, 1 - bias), 1 - bias)
        step = np.ldexp(1.0, ex - mantissa)
        # (a float's 23 fraction bits below its leading one; subnormal codes take those that 2^-149 leaves, rounded to even)
        q = np.floor((np.rint(x / step * 2.0 ** (23 - mantissa)) + r[s] * 2.0 ** (7 - mantissa)) / 2.0 ** (23 - mantissa))
        if keep_positive:
            q = np.where((x > 0) & (q == 0), 1, q)
        # value q * 2^(ex - mantissa) as a code: counts of steps from 0 on, as floats are ordered
        code = np.where(q == 0, 0, q + (ex - (1 - bias)) * (1 << mantissa))
        code = np.where(fin, code, 127)
        codes[s] = code.astype(np.int64) | np.where(np.signbit(a[s]), 128, 0)
    return codes, exps


def clip_factor(grads, max_norm):
    norm = float(np.sqrt(sum(float(np.sum(np.square(g.astype(np.float64)))) for g in grads)))
    return norm, (1.0 if max_norm == 0 or norm <= max_norm else max_norm / norm)


def adamw(x, g, m, v, t, lr, b1, b2, eps, wd):
    """New x, m, v in 64 bits."""
    x, g, m, v = (np.asarray(a, np.float64) for a in (x, g, m, v))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    d = (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return x - lr * (d + wd * x), m, v


def moments_fp32(g, m, v, b1, b2):
    """The moments with one fp32 rounding per operation, as the kernel forms them."""
    f = np.float32
    g, m, v = (np.asarray(a, f) for a in (g, m, v))
    with np.errstate(all="ignore"):
        return m * f(b1) + g * f(1 - b1), v * f(b2) + g * g * f(1 - b2)


# ---- norms, gate, residual sum
def act(kind, g):
    return [lambda: g, lambda: 1 / (1 + np.exp(-g)), lambda: np.tanh(g)][kind]()


def slope(kind, g):
    return [lambda: np.ones_like(g), lambda: 1 / ((1 + np.exp(-g)) * (1 + np.exp(g))), lambda: 1 / np.cosh(g) ** 2][kind]()


def stats(kind, u, eps):
    mean = u.mean(1, keepdims=True) if kind == LAYER else np.zeros((u.shape[0], 1))
    return mean, 1 / np.sqrt(np.square(u - mean).mean(1, keepdims=True) + eps)


def norm(kind, u, gain, bias, eps):
    if not kind:
        return u
    mean, inv = stats(kind, u, eps)
    return (u - mean) * inv * (1 if gain is None else gain) + (0 if bias is None else bias)


def forward(p):
    """y, h of a dict with x, z, gate, gate_rows, gate_act, post, pre, gains, biases, alpha, beta, eps."""
    a = 1.0
    if p.get("gate") is not None:
        a = act(p["gate_act"], p["gate"])[np.arange(p["x"].shape[0]) // p["gate_rows"]]
    y = p["x"] if p.get("z") is None else \
        p["alpha"] * p["x"] + p["beta"] * a * norm(p["post"], p["z"], p.get("post_gain"), p.get("post_bias"), p["eps"])
    return y, norm(p["pre"], y, p.get("pre_gain"), p.get("pre_bias"), p["eps"]) if p["pre"] else None


def norm_backward(kind, d, hat, inv):
    """Gradient of u from that of (u - mean) * inv; and the sum of the magnitudes it is made of."""
    n = hat.shape[1]
    mean = d.mean(1, keepdims=True) if kind == LAYER else 0.0
    mags = np.abs(d).sum(1, keepdims=True) / n if kind == LAYER else 0.0
    g = inv * (d - mean - hat * (d * hat).mean(1, keepdims=True))
    return g, inv * (np.abs(d) + mags + np.abs(hat) * np.abs(d * hat).mean(1, keepdims=True))


def backward(p, y, dy, dh, pre_stats, post_stats):
    """Gradients, and under the same names with a trailing "~" the sums of magnitudes that bound their rounding."""
    o, M = {}, y.shape[0]
    D = np.zeros_like(y) if dy is None else dy.copy()
    Da = np.abs(D)
    if p["pre"]:
        mean, inv = pre_stats
        hat, hata = (y - mean) * inv, (np.abs(y) + np.abs(mean)) * inv
        o["pre_gain"], o["pre_gain~"] = (dh * hat).sum(0), (np.abs(dh) * hata).sum(0)
        o["pre_bias"], o["pre_bias~"] = dh.sum(0), np.abs(dh).sum(0)
        g, ga = norm_backward(p["pre"], dh * (1 if p.get("pre_gain") is None else p["pre_gain"]), hat, inv)
        D, Da = D + g, Da + ga
    o["x"], o["x~"] = p["alpha"] * D, abs(p["alpha"]) * Da
    if p.get("z") is None:
        return o
    rows = np.arange(M) // p["gate_rows"] if p.get("gate") is not None else None
    w = p["beta"] * (1.0 if rows is None else act(p["gate_act"], p["gate"])[rows]) * np.ones_like(y)
    z, za = p["z"], np.abs(p["z"])
    gain = 1.0 if p.get("post_gain") is None or not p["post"] else p["post_gain"]
    bias = 0.0 if p.get("post_bias") is None or not p["post"] else p["post_bias"]
    if p["post"]:
        mean, inv = post_stats
        z, za = (z - mean) * inv, (za + np.abs(mean)) * inv
        o["post_gain"], o["post_gain~"] = (w * D * z).sum(0), (np.abs(w) * Da * za).sum(0)
        o["post_bias"], o["post_bias~"] = (w * D).sum(0), (np.abs(w) * Da).sum(0)
    if rows is not None:
        c = p["beta"] * slope(p["gate_act"], p["gate"])[rows] * D * (z * gain + bias)
        ca = abs(p["beta"]) * slope(p["gate_act"], p["gate"])[rows] * Da * (za * np.abs(gain) + np.abs(bias))
        o["gate"], o["gate~"] = np.zeros_like(p["gate"]), np.zeros_like(p["gate"])
        np.add.at(o["gate"], rows, c)
        np.add.at(o["gate~"], rows, ca)
    d, da = w * D * gain, np.abs(w) * Da * np.abs(gain)
    if p["post"]:
        n = y.shape[1]
        layer = p["post"] == LAYER
        o["z"] = inv * (d - (d.mean(1, keepdims=True) if layer else 0.0) - z * (d * z).mean(1, keepdims=True))
        o["z~"] = inv * (da + (da.mean(1, keepdims=True) if layer else 0.0) + za * (da * za).sum(1, keepdims=True) / n)
    else:
        o["z"], o["z~"] = d, da
    return o
