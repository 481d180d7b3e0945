"""Plain forms of what is taken of rows of class scores, in 64 bits (host), and how far the library's 32 bits may be off, for their tests.

What the library does is counted in units U = 2^-24 of a value: d = x - m is rounded once, d log2(e) / T twice (the factor and the product), so an
exponential is off by 2 units and by 4 |d| / T; a sum of C of them by as many units as it has additions one behind the other."""
import numpy as np

from tests.nodewise import HALF, U, f64, half_step    # noqa: F401

TINY = 2.0 ** -125             # exponentials below 2^-126 may be zero


def additions(C):
    """A lane's values one after the other, the lanes and wavefronts by halves; of rows of more than 2048 a thread's share."""
    return (min(C, 32) if C <= 2048 else C / 256 + 32) + 24


class Softmax:
    """softmax(x / T) of rows x (float64), with what the library's sums of it may be off."""

    def __init__(self, x, T=1.0):
        self.x, self.T = x, T
        C = x.shape[1]
        with np.errstate(all="ignore"):
            m = x.max(1, keepdims=True)
            self.m = np.where(np.isneginf(m), 0.0, m)
            self.d = (x - self.m) / T
            e = np.exp(self.d)
            s = e.sum(1, keepdims=True)
            self.log = np.log(s)
            self.lse = self.m / T + self.log
            self.logp = self.d - self.log
            self.p = e / s
            d = np.where(self.p == 0, 0.0, np.abs(self.d))
            self.d1, self.d2 = (self.p * d).sum(1, keepdims=True), (self.p * d * d).sum(1, keepdims=True)
            self.entropy = -np.where(self.p == 0, 0.0, self.p * self.logp).sum(1, keepdims=True)
            self.off_sum = U * (4 * self.d1 + 4 + additions(C))                      # relative
            self.off_log = self.off_sum + 3 * U * (np.abs(self.log) + 1)
            self.off_lse = self.off_log + 3 * U * (np.abs(self.m) / T + np.abs(self.lse))
            self.off_entropy = (self.off_log + U * (4 * self.d2 + (additions(C) + 6) * self.d1) + self.off_sum * self.d1 +
                                2 * U * (np.abs(self.entropy) + self.d1))

    def off_logp(self, cls_d, logp):
        return self.off_log + 3 * U * (np.abs(cls_d) + np.abs(logp))


def top(x, k):
    """The classes of the k highest scores, of equal ones the lower first; -1 behind the last that is not -inf."""
    order = np.argsort(-x, axis=1, kind="stable")[:, :k]
    out = np.full((x.shape[0], k), -1, np.int64)
    out[:, :order.shape[1]] = np.where(np.isneginf(np.take_along_axis(x, order, 1)), -1, order)
    return out


def logprob_bwd(x, lse, entropy, label, g, h):
    """(gradient, how far 32 bits may be off it); g, h: dlogp, dentropy."""
    n, C = x.shape
    with np.errstate(all="ignore"):
        d = x - lse[:, None]
        p = np.exp(d)
        finite = np.where(p == 0, 0.0, d)
        has = (label >= 0) & (label < C)
        g = np.where(has, g, 0.0)[:, None]
        one = (np.arange(C)[None, :] == label[:, None]) & has[:, None]
        h, H = h[:, None], entropy[:, None]
        want = -p * (g + h * (finite + H)) + one * g
        size = np.abs(g) + np.abs(h) * (np.abs(finite) + np.abs(H))
        off = p * U * (4 * np.abs(finite) + 10) * size + 2 * U * (one * np.abs(g) + np.abs(want)) + TINY * (size + 200 * np.abs(h))
    return want, off


class Teacher:
    """A teacher's softmax over its listed classes."""

    def __init__(self, value, index, T, C):
        self.is_ = (index >= 0) & (index < C)
        v = np.where(self.is_, value, -np.inf)
        with np.errstate(all="ignore"):
            m = v.max(1, keepdims=True) if v.shape[1] else np.full((v.shape[0], 1), -np.inf)
            m = np.where(np.isneginf(m), 0.0, m)
            self.d = (v - m) / T
            e = np.exp(self.d)
            s = e.sum(1, keepdims=True)
            self.none = s[:, 0] == 0
            self.log = np.log(np.where(s == 0, 1.0, s))
            self.q = e / np.where(s == 0, 1.0, s)
            self.abs_d = np.where(self.q == 0, 0.0, np.abs(self.d))
            k = v.shape[1]
            self.off_sum = U * (4 * (self.q * self.abs_d).sum(1, keepdims=True) + 4 + k)
            self.off_q = U * (4 * self.abs_d + 6) + self.off_sum                     # relative


def distill_fwd(x, value, index, T):
    s, t = Softmax(x, T), Teacher(value, index, T, x.shape[1])
    at = np.where(t.is_, index, 0)
    with np.errstate(all="ignore"):
        y = np.take_along_axis(s.d, at, 1)
        part = np.where(t.q == 0, 0.0, t.q * (t.d - y))
        size = np.where(t.q == 0, 0.0, t.q * (t.abs_d + np.abs(y)))
        w = part.sum(1, keepdims=True)
        loss = w - t.log + s.log
        off = ((size * (t.off_q + U * (index.shape[1] + 8))).sum(1, keepdims=True) + t.off_sum + 3 * U * (np.abs(t.log) + 1) + s.off_log +
               3 * U * (np.abs(w) + np.abs(loss)))
    return np.where(t.none, 0.0, loss[:, 0]), np.where(t.none, 0.0, off[:, 0]), s


def distill_bwd(x, value, index, T, lse, g):
    n, C = x.shape
    t = Teacher(value, index, T, C)
    with np.errstate(all="ignore"):
        s = np.exp(x / T - lse[:, None])
        far = np.where(s == 0, 0.0, np.abs(x) / T) + np.abs(lse)[:, None]
        want, off = s.copy(), s * U * (4 * far + 10) + TINY
    q = np.where(t.is_, t.q, 0.0)
    rows = np.arange(n)
    for j in range(index.shape[1]):
        at = np.where(t.is_[:, j], index[:, j], 0)
        want[rows, at] -= q[:, j]
        off[rows, at] += q[:, j] * (t.off_q[:, j] + 8 * U) + 2 * U * (s[rows, at] + 1.0) * t.is_[:, j]
    g = np.where(t.none, 0.0, g / T)[:, None]
    return want * g, (off + 3 * U * np.abs(want)) * np.abs(g) + TINY
