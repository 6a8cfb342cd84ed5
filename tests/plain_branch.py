"""The operators inside a residual block's branch and the policy loss in plain numpy, 64 bits, from their definitions: test infrastructure."""
import numpy as np
from scipy.special import expit, ndtr

IDENTITY, RELU, GELU, SILU = 0, 1, 2, 3
SIGMOID, EXP = 0, 1


# ---- products
def act(kind, p):
    with np.errstate(all="ignore"):
        if kind == RELU:
            return np.where(p < 0, 0.0, p)
        if kind == GELU:
            return np.where(np.isneginf(p), 0.0, p * ndtr(p))
        return np.where(np.isneginf(p), 0.0, p * expit(p)) if kind == SILU else p


def slope(kind, p):
    with np.errstate(all="ignore"):
        if kind == RELU:
            return np.where(p > 0, 1.0, 0.0)
        if kind == GELU:
            return np.where(np.isinf(p), p > 0, ndtr(p) + p * np.exp(-0.5 * p * p) / np.sqrt(2 * np.pi))
        return np.where(np.isinf(p), p > 0, expit(p) * (1 + p * expit(-p))) if kind == SILU else np.ones_like(p)


# ---- recurrence
def gates(decay, f):
    """a, 1 - a, da/df"""
    with np.errstate(over="ignore"):
        if decay == SIGMOID:
            return expit(f), expit(-f), expit(f) * expit(-f)
        return np.exp(f), -np.expm1(f), np.exp(f)


def scan(decay, coupled, x, f, state):
    """Rows of one sequence: h, the last state, and what each h may be off by per 2^-24: a step rounds what it keeps once, its gate is off by a few
    units of the smaller of a and 1 - a, and the input by a few of its own."""
    a, b, _ = gates(decay, f)
    h, off, size, rows, offs = state.copy(), np.zeros_like(state), np.abs(state), [], []
    for t in range(len(x)):
        u = b[t] * x[t] if coupled else x[t]
        off = a[t] * off + 3 * a[t] * size + 16 * (np.minimum(a[t], np.abs(b[t])) * size + np.abs(u))
        size = a[t] * size + np.abs(u)
        h = a[t] * h + u
        rows.append(h)
        offs.append(off)
    z = np.zeros((0,) + state.shape)
    return np.array(rows) if rows else z, h, np.array(offs) if offs else z, off


def scan_back(decay, coupled, x, f, h, state, dh, dlast):
    """Gradients of x, f and the state in front, and what each may be off by per 2^-24."""
    a, b, s = gates(decay, f)
    before = np.concatenate([state[None], h[:-1]]) if len(h) else h
    later, off, size = dlast.copy(), np.zeros_like(dlast), np.abs(dlast)
    dx, df, odx, odf = (np.zeros(x.shape) for _ in range(4))
    for t in reversed(range(len(x))):
        g, og, sg = dh[t] + later, off + np.abs(dh[t]) + size, np.abs(dh[t]) + size
        dx[t], odx[t] = (b[t] * g, np.abs(b[t]) * (og + 16 * sg)) if coupled else (g, og)
        diff = before[t] - x[t] if coupled else before[t]
        df[t] = s[t] * g * diff
        odf[t] = s[t] * ((og + 20 * sg) * np.abs(diff) + 2 * sg * (np.abs(before[t]) + (np.abs(x[t]) if coupled else 0)))
        later = a[t] * g
        off = a[t] * og + (3 * a[t] + 16 * np.minimum(a[t], np.abs(b[t]))) * sg
        size = a[t] * sg
    return dx, df, later, odx, odf, off


# ---- policy loss
def policy(z, labels, old, ref, adv, weight, low, high, kl_coef, ent_coef, temperature):
    """loss[5], logp, entropy, terms[4], dz"""
    R, V = z.shape
    z = np.asarray(z, np.float64) / temperature
    with np.errstate(all="ignore"):
        live = (labels >= 0) & ~np.all(np.isneginf(z), 1)
        top = np.where(live, z.max(1), 0.0)
        e = np.exp(z - top[:, None])
        logs = np.log(e.sum(1))
        lo = z - top[:, None] - logs[:, None]
        p = np.exp(lo)
        H = -np.where(np.isneginf(lo), 0.0, p * lo).sum(1)
        inside = (labels >= 0) & (labels < V)
        lp = np.where(inside, lo[np.arange(R), np.where(inside, labels, 0)], np.nan)
        rho = np.exp(lp - old) if old is not None else np.ones(R)
        free, held = -adv * rho, -adv * np.minimum(np.maximum(rho, 1 - low), 1 + high)
        clipped = held > free
        c = np.where(clipped, 0.0, free)
        kl = np.zeros(R)
        if ref is not None:
            d = ref - lp
            kl = np.expm1(d) - d
            c = c - kl_coef * np.expm1(d)
        w = weight if weight is not None else np.full(R, 1.0 / R)
        terms = np.where(live, np.stack([np.where(clipped, held, free), kl, H, clipped.astype(float)]), 0.0)
        parts = (np.where(live, w, 0.0) * terms).sum(1)
        dz = -c[:, None] * p + ent_coef * np.where(np.isneginf(lo), 0.0, p * (lo + H[:, None]))
        hot = np.zeros((R, V))
        hot[np.arange(R)[inside], labels[inside]] = 1.0
        dz = (dz + np.where(hot > 0, c[:, None], 0.0)) * (w / temperature)[:, None]
        dz[~live] = 0.0
    loss = np.concatenate([[parts[0] + kl_coef * parts[1] - ent_coef * parts[2]], parts])
    return loss, np.where(live, lp, 0.0), np.where(live, H, 0.0), terms, dz
