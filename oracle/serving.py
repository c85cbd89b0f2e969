"""The operators around the blocks' halves by their definitions, in 64 bits (numpy only, no code of the HIP path)."""
import numpy as np

E4M3_MOST = 448.0


def rms_norm(s, weight, eps):
    """Norm of rows s[T, d] as they are kept."""
    s = np.asarray(s, np.float64)
    with np.errstate(all="ignore"):
        y = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    return y if weight is None else y * np.asarray(weight, np.float64)


def adapters(x, adapter, A, B, y, scale=None):
    """out[t] = y[t] + scale B (A x[t]) -> (out, size): size = scale sum |B| sum |A| |x|, the scale of its rounding errors."""
    x, A, B = (np.asarray(t, np.float64) for t in (x, A, B))
    out, size = np.array(y, np.float64), np.zeros(np.shape(y))
    for t, a in enumerate(adapter):
        if 0 <= a < len(A):
            c = 1.0 if scale is None else float(scale[a])
            with np.errstate(all="ignore"):
                out[t] += c * (B[a] @ (A[a] @ x[t]))
                size[t] = abs(c) * (np.abs(B[a]) @ (np.abs(A[a]) @ np.abs(x[t])))
    return out, size


def order(l):
    """The tokens of one row of logits, the largest first, equal ones by the lower index; those that are no numbers left out."""
    at = np.arange(len(l))[~np.isnan(l)]
    return at[np.lexsort((at, -np.asarray(l, np.float64)[at]))]


def logprobs(l):
    """One row -> (log probabilities, entropy, largest logit, mean distance to it)."""
    l = np.asarray(l, np.float64)
    M = l.max()
    if not np.isfinite(M):                       # (NaN is not finite, either)
        return np.full(l.shape, np.nan), np.nan, M, np.nan
    s = np.exp(l - M)
    lp = l - M - np.log(s.sum())
    p = s / s.sum()
    far = np.where(p > 0, M - l, 0.0)
    return lp, float(-(p[p > 0] * lp[p > 0]).sum()), M, float((p * far).sum())
