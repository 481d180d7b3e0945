"""Plain forms of the node-wise operators in 64 bits (host), for their tests."""
import numpy as np
import torch

U = 2.0 ** -24                                     # half a step of fp32, relative
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def half_step(t):
    """Half a step of a value of type t around each number (half the smallest one at zero)."""
    return lambda v: HALF[t] * np.abs(v) + 2.0 ** -134


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def pack(X):
    """q, e of the packed form, number by number from its definition (X float64 [n, K], values of fp32)."""
    n, K = X.shape
    q = np.zeros((n, -(-K // 16) * 16), np.int8)
    e = np.zeros((n, -(-K // 32)), np.uint8)
    for b in range(e.shape[1]):
        x = X[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(x).all(1)
        x = np.where(bad[:, None], 0.0, x)
        k = np.full(n, -126)
        largest = np.abs(x).max(1)
        for _ in range(260):                       # the smallest step that leaves no whole number beyond 127
            k = np.where((np.rint(largest / 2.0 ** k) > 127) & (k < 121), k + 1, k)
        v = np.clip(np.rint(x / (2.0 ** k)[:, None]), -127, 127)         # (beyond 127 only next to the largest number)
        q[:, 32 * b:32 * b + v.shape[1]] = v
        e[:, b] = np.where(bad, 255, k + 127)
    return q, e


def unpack(q, e, K):
    step = np.where(e == 255, np.nan, 2.0 ** (e.astype(np.float64) - 127))
    return q[:, :K].astype(np.float64) * np.repeat(step, 32, axis=1)[:, :K]


def norm_stats(x, eps):
    mean = x.mean(1, keepdims=True)
    return mean, 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)


def norm_fwd(x, gamma, beta, eps):
    mean, r = norm_stats(x, eps)
    return (x - mean) * r * gamma + beta, mean, r


def norm_bwd(dy, x, mean, r, gamma):
    h, d = (x - mean) * r, dy * gamma
    dx = r * (d - d.mean(1, keepdims=True) - h * (d * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def spans(ptr, n):
    ptr = [min(max(int(p), 0), n) for p in ptr]
    return [(t, a, max(a, b)) for t, (a, b) in enumerate(zip(ptr[:-1], ptr[1:]))]
