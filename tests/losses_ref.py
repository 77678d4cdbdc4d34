"""The operators of a policy or preference step in 64 bits (NumPy), and bounds on what
fp32 exponentials and sums may differ from them by.

Bounds, with U half a step of fp32 and y_v = (largest logit - z_v) / tau >= 0:
* an exponential's argument takes two roundings (the factor log2 e / tau, which is one
  fp32 number, and the fused operation), the hardware's exp2 is good to a step: a
  term's relative error is U (2 y_v + 2). The bound of a gradient stored in 16 bits
  counts U (4 y_v + 2), more than the steps take (tests/test_gpu_token_losses_bounds.py
  holds such gradients to 2 y_v + 2).
* a sum is a chain over a vector's 8 entries at most, a chain over 16 vectors at most
  and an edge entry in fp32 (26 roundings at most), then in 64 bits; a row in parts
  adds one rounding of a part's sum and one exponential of its offset (2 roundings'
  worth of argument that y_v counts, 2 U). The weighted mean of y_v is below ln n.
"""
from __future__ import annotations

import math

import numpy as np

from tests.row_operators_ref import ROUND, U

TINY = 2.0 ** -126   # exponentials below this are 0 in fp32


class Row:
    """A row z (64 bits) and its token: l, H, what of them and of a gradient fp32 may
    be off by."""

    def __init__(self, z, token, tau):
        self.tau, self.n, self.token = tau, z.size, token
        m = z.max()
        y = np.where(z == -np.inf, np.inf, (m - z) / tau)
        e = np.exp(-y)
        self.e, self.s = e, e.sum()
        self.p = e / self.s
        self.se = np.delete(e, token).sum()
        self.y = np.where(e > 0, y, 0.0)
        # nearly certain tokens: through the sum of the others
        self.l = -math.log1p(self.se / e[token]) if e[token] >= self.se else (
            -y[token] - math.log(self.s))
        self.mean, self.mean2 = (self.p * self.y).sum(), (self.p * self.y ** 2).sum()
        self.entropy = math.log(self.s) + self.mean
        d = U * (2 * (math.log(self.n) + 1) + 2 + 26 + 4) + 3 * U
        self.ds = d
        finite = abs(self.l) if np.isfinite(self.l) else 0.0
        # the token's own exponential is exact to 3 U and no part of the sum's error
        self.l_err = d * min(1.0, finite) + U * finite + self.n * TINY
        t = U * (40 * self.mean + 2 * self.mean2)   # of sum p y
        self.t_err = t
        self.entropy_err = d * (1 + self.mean) + t + 2 * U * abs(self.entropy) + self.n * TINY

    def gradient(self, g, h, g_err, dtype):
        """Of a loss with the slopes g by l and h by H, and its bound."""
        v = self.token
        logp = -self.y - math.log(self.s)
        # entries of no mass have none in the entropy either
        grad = -g * self.p - h * np.where(self.p > 0, self.p * (logp + self.entropy), 0.0)
        grad[v] = g * self.se / self.s - h * (self.p[v] * (self.l + self.entropy) if self.p[v] > 0 else 0)
        arg = 2 if dtype == "f32" else 4
        rel = self.ds + U * (arg * self.y + 4)
        err = self.p * (abs(g) * rel + g_err + abs(h) * ((self.mean + self.y) * (self.ds + rel) + self.t_err))
        err[v] = (abs(g) * 2 * self.ds + g_err) * self.se / self.s + abs(h) * self.p[v] * (
            (self.mean + self.y[v]) * 3 * self.ds + self.t_err)
        # an exponential that is 0 in fp32, times the slopes
        err = err + (abs(g) + abs(h) * (self.mean + 200)) * TINY * self.n
        step, least = ROUND[dtype]
        grad, err = grad / self.tau, err / self.tau + 4 * U * np.abs(grad) / self.tau
        return grad, err * 1.01 + step * np.abs(grad) * 1.01 + least


def policy(row, adv, old=None, ref=None, low=0.2, high=0.2, kl=0.0, bonus=0.0, w=1.0):
    """(loss, its bound, g, h, bound of g)."""
    l, le = row.l, row.l_err
    rho = math.exp(l - old) if old is not None else 1.0
    bound = 1 + high if adv > 0 else 1 - low
    beyond = rho > bound if adv > 0 else rho < bound
    loss = -adv * (bound if beyond else rho) if adv else 0.0
    g = 0.0 if beyond else -adv * rho
    # l's error as the ratio and the gradient feel it (without old there is no ratio)
    dl = 0.0 if beyond or old is None else abs(adv) * rho * le
    err, g_err = dl, dl
    if kl:
        d = ref - l
        loss += kl * (math.expm1(d) - d)
        g -= kl * math.expm1(d)
        err += kl * abs(math.expm1(d)) * le + kl * math.exp(d) * le * le
        g_err += kl * math.exp(d) * le * 1.01
    h = 0.0
    if bonus:
        loss -= bonus * row.entropy
        err += bonus * row.entropy_err
        h = -bonus
    return (w * loss, abs(w) * err * 1.01 + 2 * U * abs(w * loss) + 2.0 ** -149, w * g, w * h, abs(w) * g_err)


def pair_value(u, form, beta, smoothing):
    """(value, slope by u, a bound of the second derivative)."""
    h = beta * u
    if form == "sigmoid":
        soft = lambda x: max(x, 0.0) + math.log1p(math.exp(-abs(x)))
        sig = lambda x: 1 / (1 + math.exp(-x)) if x > -700 else 0.0
        return ((1 - smoothing) * soft(-h) + (smoothing * soft(h) if smoothing else 0.0),
                beta * (-(1 - smoothing) * sig(-h) + smoothing * sig(h)), beta * beta / 4)
    if form == "hinge":
        return max(0.0, 1 - h), (-beta if h < 1 else 0.0), 0.0
    d = u - 0.5 / beta
    return d * d, 2 * d, 2.0


def preference(z, tokens, ends, ref, tau, form, beta, mean=False, smoothing=0.0, margin=0.0, w=1.0,
               dtype="f32"):
    """One pair on rows z[ends[0]:ends[2]]: (loss, bound), [s of both], [bounds], and
    {row: (gradient, bound)}."""
    rows = [{}, {}]
    s, s_err, n = [0.0, 0.0], [0.0, 0.0], [1.0, 1.0]
    for j in range(2):
        for r in range(ends[j], ends[j + 1]):
            if tokens[r] != -1:
                rows[j][r] = q = Row(z[r], tokens[r], tau)
                s[j] += q.l - (ref[r] if ref is not None else 0.0)
                s_err[j] += q.l_err
        n[j] = max(1, len(rows[j])) if mean else 1
        s[j] /= n[j]
        s_err[j] = s_err[j] / n[j]
    u, du = s[0] - s[1] - margin, s_err[0] + s_err[1] + 1e-13 * (abs(s[0]) + abs(s[1]))
    value, slope, second = pair_value(u, form, beta, smoothing)
    err = abs(slope) * du + second * du * du + 2 * U * value + 1e-14
    grads = {}
    for j, sign in enumerate((1.0, -1.0)):
        for r, q in rows[j].items():
            g = w * slope * sign / n[j]
            grads[r] = q.gradient(g, 0.0, abs(w) * second * du / n[j] + 4 * U * abs(g), dtype)
    return ((w * value, abs(w) * err), s, [e + U * abs(x) for e, x in zip(s_err, s)], grads)
