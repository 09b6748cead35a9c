"""Float64 definitions of the operators around a clipped step (numpy only, no product code).

Layer norm and its backward pass, the preference loss of paired sequences with its gradient, and Newton-Schulz products:
plain, slow, one row / pair / matrix at a time where that is clearer.  Pinned by autograd and differences.
"""
import numpy as np


def layernorm(x, gain=None, shift=None, eps=1e-5):
    """(y, x_hat, mean, rstd) over the last axis."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    rstd = 1.0 / np.sqrt(((x - mean[..., None]) ** 2).mean(-1) + eps)
    hat = (x - mean[..., None]) * rstd[..., None]
    y = hat * (1.0 if gain is None else np.asarray(gain, dtype=np.float64))
    return y + (0.0 if shift is None else np.asarray(shift, dtype=np.float64)), hat, mean, rstd


def layernorm_backward(g, x, gain, mean, rstd):
    """(dx, gain_sums, shift_sums, sq) of g (B, T, p)."""
    g, x = np.asarray(g, dtype=np.float64), np.asarray(x, dtype=np.float64)
    mean, rstd = (np.asarray(v, dtype=np.float64).reshape(x.shape[:2] + (1,)) for v in (mean, rstd))
    hat = (x - mean) * rstd
    u = g * (1.0 if gain is None else np.asarray(gain, dtype=np.float64))
    dx = rstd * (u - u.mean(-1, keepdims=True) - hat * (u * hat).mean(-1, keepdims=True))
    gain_sums, shift_sums = (g * hat).sum(1), g.sum(1)
    return dx, gain_sums, shift_sums, (gain_sums ** 2).sum(-1) + (shift_sums ** 2).sum(-1)


def _softplus(x):
    return max(x, 0.0) + np.log1p(np.exp(-abs(x)))


def _logistic(x):
    return 1.0 / (1.0 + np.exp(-x)) if x >= 0 else np.exp(x) / (1.0 + np.exp(x))


def preference_loss(logits, targets, ref, beta, smoothing=0.0, scale=1.0):
    """(loss, logp, G) of logits (B, 2T, V), targets (B, 2, T); rows whose target is negative or not below V do not count."""
    B, rows, V = logits.shape
    T = rows // 2
    loss, logp, G = np.zeros(B), np.zeros((B, 2)), np.zeros((B, rows, V))
    for i in range(B):
        soft = {}
        for q in range(2):
            for t in range(T):
                k = int(targets[i, q, t])
                if 0 <= k < V:
                    x = np.asarray(logits[i, q * T + t], dtype=np.float64)
                    m = x.max()
                    e = np.exp(x - m)
                    logp[i, q] += (x[k] - m) - np.log(e.sum())
                    soft[q, t] = (k, e / e.sum())
        r = np.zeros(2) if ref is None else np.asarray(ref[i], dtype=np.float64)
        h = beta * ((logp[i, 0] - r[0]) - (logp[i, 1] - r[1]))
        # a term of weight 0 is not there, also where the other one's h is infinite (a target whose logit is -inf)
        loss[i] = sum(w * _softplus(v) for w, v in ((1 - smoothing, -h), (smoothing, h)) if w > 0)
        slope = scale * beta * (smoothing * _logistic(h) - (1 - smoothing) * _logistic(-h))
        for (q, t), (k, p) in soft.items():
            c = slope if q == 0 else -slope
            G[i, q * T + t] = -c * p
            G[i, q * T + t, k] += c
    return loss, logp, G


def orthogonalize(M, coefs, eps=1e-7, scale=1.0):
    """scale * Newton-Schulz iterate of M / (|M|_F + eps), the Gram product on the shorter side."""
    X = np.asarray(M, dtype=np.float64)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    X = X / (np.sqrt((X * X).sum()) + eps)
    for a, b, c in coefs:
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return scale * (X.T if tall else X)
