"""Independent CPU model of further operators of a decoding step, in float64 numpy from their definitions: norms of heads with their rotation and
its gradients, and the verification of drafted chains and trees from probabilities.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

OK, BAD_TOKEN, BAD_INDEX = 0, 7, 9


def angles(positions, inv_freq, axes=None):
    """[..., rot / 2] of positions [...], or, with the axis of every frequency, [..., num_axes]."""
    f = np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    pos = np.asarray(positions, dtype=np.float64)
    return pos[..., None] * f if axes is None else pos[..., np.asarray(axes)] * f


def turn(x, angle, layout, amplitude=1.0, inverse=False):
    """x [..., heads, D]; angle [..., rot / 2]."""
    n = angle.shape[-1]
    z = np.exp((-1j if inverse else 1j) * angle)[..., None, :] * amplitude
    y = np.array(x, dtype=np.float64)
    re, im = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = (y[..., re] + 1j * y[..., im]) * z
    y[..., re], y[..., im] = z.real, z.imag
    return y


def normed(x, w, eps):
    """(x w / rms, x / rms, 1 / rms)"""
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r * w, x * r, r


def heads(x, w, eps, angle, layout, amplitude=1.0):
    return turn(normed(x, w, eps)[0], angle, layout, amplitude)


def heads_grad(g, x, w, eps, angle, layout, amplitude=1.0):
    """Gradients of sum(g * heads(x, w)): (by x, by w)."""
    _, n, r = normed(x, w, eps)
    g = turn(g, angle, layout, amplitude, inverse=True)
    gw = g * w
    dx = r * (gw - n * (gw * n).mean(-1, keepdims=True))
    return dx, (g * n).reshape(-1, x.shape[-1]).sum(0)


def draw(w, u):
    """The first entry whose running sum exceeds u times the whole; none has weight: the last entry."""
    run = np.cumsum(w)
    above = np.flatnonzero(run > u * run[-1])
    return int(above[0]) if above.size else len(w) - 1


def verify(p, q, tokens, accept_u, sample_u, parents=None, judged=None, mode="standard", resample="residual", distinct=False):
    """One sequence: p [T, V], q [T - 1, V], tokens, accept_u, judged [T - 1], parents [T]. (path, next token, status)"""
    p, q = np.asarray(p, dtype=np.float64), np.asarray(q, dtype=np.float64)
    T, V = p.shape
    status, children = OK, {i: [] for i in range(T)}
    for i in range(1, T):
        parent = i - 1 if parents is None else int(parents[i])
        if not 0 <= int(tokens[i - 1]) < V:
            status = status or BAD_TOKEN
        if 0 <= parent < i:
            children[parent].append(i)
        else:
            status = status or BAD_INDEX
    at, path = 0, []
    while True:
        w, W, Q, summed = p[at].copy(), 1.0, 1.0, False
        d = q[at].copy() if children[at] else None
        for i in children[at]:
            x = int(tokens[i - 1])
            inside = 0 <= x < V
            standard = inside and float(accept_u[i - 1]) * W * d[x] < w[x] * Q
            judge = inside and judged is not None and bool(judged[i - 1])
            if {"standard": standard, "judge": judge, "judge_or_standard": standard or judge}[mode]:
                path.append(i)
                at = i
                break
            if not (W > 0 and Q > 0):          # nothing to take, or to take from
                continue
            w = np.maximum(0.0, w * Q - W * d)
            e = np.frexp(w.sum())[1]           # kept near 1: the products would leave float64
            w = np.ldexp(w, -e)
            W = w.sum()
            if distinct and inside:
                Q -= d[x]
                d[x] = 0.0
                summed = summed or Q < 0.5     # a row's own rounding is no longer small beside what is left
                Q = d.sum() if summed else Q
        else:
            break
    if resample == "target_p" or w.sum() == 0:
        w = p[at]
    return path, draw(w, float(sample_u)), status
