"""Attention, norms and rotation by their definitions, in 64 bits, a sequence, a head and a query at a time (numpy only,
no code of the HIP path)."""
import numpy as np


def norm_rope(x, weight, eps, inv_freq, position, neighbours):
    """x[T, heads, D] -> (y, size): the result, and |y_i| + |y_j| of the pair an element is turned in (the scale of its
    rounding errors)."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    if weight is not None:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    out, size = y.copy(), np.abs(y)
    half = 0 if inv_freq is None else len(inv_freq)
    for f in range(half):
        i, j = (2 * f, 2 * f + 1) if neighbours else (f, f + half)
        # the angle less its whole turns, from exact whole-number arithmetic on the 32-bit frequency
        a = np.array([_angle(int(p), float(inv_freq[f])) for p in position])[:, None]
        out[..., i] = y[..., i] * np.cos(a) - y[..., j] * np.sin(a)
        out[..., j] = y[..., j] * np.cos(a) + y[..., i] * np.sin(a)
        size[..., i] = size[..., j] = np.abs(y[..., i]) + np.abs(y[..., j])
    return out, size


def _angle(p, f):
    from fractions import Fraction
    exact = Fraction(p) * Fraction(f)
    two_pi = Fraction(884279719003555, 140737488355328) + Fraction(2.4492935982947064e-16)   # 2 pi to 2^-106
    return float(exact - two_pi * round(exact / two_pi))


def visible(p, n, window, sinks):
    """Which of n keys the query at position p sees."""
    j = np.arange(n)
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def attend(q, k, v, p, scale, window=0, sinks=0):
    """One query q[D] at position p over k, v[n, D] -> (out, size, spread): size = sum_j w_j |v_j|; spread: the largest
    scale * sum_d |q_d k_jd|, the scale of a score's rounding errors.  Hidden keys are not looked at."""
    see = visible(p, len(k), window, sinks)
    D = len(q)
    if not see.any():
        return np.zeros(D), np.zeros(D), 0.0
    q, k, v = np.asarray(q, np.float64), np.asarray(k, np.float64)[see], np.asarray(v, np.float64)[see]
    with np.errstate(all="ignore"):
        s = scale * (k @ q)
        w = np.exp(s - s.max())
        w /= w.sum()
        return w @ v, w @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * abs(scale))


def attention(q, k, v, before, scale, window=0, sinks=0):
    """The new tokens q[n, heads, D] of one sequence, the first at position `before`, over k, v[cached, kv_heads, D]."""
    n, heads, D = q.shape
    group = heads // k.shape[1]
    out, size, spread = np.zeros((n, heads, D)), np.zeros((n, heads, D)), np.zeros((n, heads, 1))
    for i in range(n):
        for h in range(heads):
            out[i, h], size[i, h], spread[i, h, 0] = attend(q[i, h], k[:, h // group], v[:, h // group], before + i, scale, window, sinks)
    return out, size, spread
