"""The operators on rows of logits in 64 bits (NumPy), and bounds on what fp32
arithmetic may differ from them by."""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24   # half a step of fp32, relative


def top(z, k, tau):
    """values, index, rest of rows z (64 bits)."""
    order = np.argsort(-z, axis=1, kind="stable")
    rows = np.arange(z.shape[0])[:, None]
    index = order[:, :k]
    left = z[rows, order[:, k:]] / tau
    rest = np.full(z.shape[0], -np.inf)
    for r in range(z.shape[0]):
        if left.shape[1] and np.isfinite(left[r].max()):
            m = left[r].max()
            rest[r] = m + np.log(np.exp(left[r] - m).sum())
    return z[rows, index], index, rest


def log_sum_bound(n, typical=40.0):
    """How far fp32 may put the log of a sum of n exponentials whose largest is 1.
    An exponent y <= 0 takes at most 5 roundings (difference, 1/tau, product,
    log2 e, product): a term's relative error is 5 U |y|, and the weighted mean of
    |y| is below ln n + 1. The exponential and the log add 4 U each, and a chain of
    at most n / 64 + 16 additions a rounding each."""
    return U * (5 * (math.log(n) + 1) + 8 + n / 64 + 16)


def distill(z, values, index, rest, w, tau, alpha, beta):
    """One row in 64 bits: loss, gradient, and bounds on the fp32 errors of both.
    index entries of -1 are unused places."""
    V = z.size
    used = index >= 0
    idx, t = index[used], values[used] / tau
    listed = np.zeros(V, bool)
    listed[idx] = True
    y = z / tau
    m = y.max()
    lq_all = y - m - np.log(np.exp(y - m).sum())
    tt = np.append(t, rest) if rest is not None else t
    mt = tt.max()
    lp_all = tt - mt - np.log(np.exp(tt - mt).sum())
    lp, lq = lp_all[:t.size], lq_all[idx]
    with np.errstate(all="ignore"):
        if rest is not None:
            m0 = lq_all[~listed].max() if (~listed).any() else -np.inf
            lq0 = m0 + np.log(np.exp(lq_all[~listed] - m0).sum()) if np.isfinite(m0) else -np.inf
            lp, lq = np.append(lp, lp_all[-1]), np.append(lq, lq0)
        p, q = np.exp(lp), np.exp(lq)
        c = lq - lp
        kl_p = -np.where(p > 0, p * c, 0.0).sum()
        kl_q = np.where(q > 0, q * c, 0.0).sum()
        loss = (alpha * kl_p if alpha else 0.0) + (beta * kl_q if beta else 0.0)
        # fp32: a log probability is a difference of roundings of its parts and of
        # the log of a sum
        s = log_sum_bound(V) + log_sum_bound(max(t.size, 2))
        d_entry = lambda log_p, raw: 6 * U * (np.abs(raw) + np.abs(log_p) + 1) + s
        dq = d_entry(lq, np.append(z[idx] / tau, m + lq0 if rest is not None else 0)[:lq.size])
        dp = d_entry(lp, tt)
        dl = dq + dp
        fin = np.isfinite(c)
        term = lambda x: np.where(fin & (x > 0), x * (dl + np.abs(c) * (dq + dp + 4 * U)), 0).sum()
        chain = U * (t.size / 64 + 16)
        err_p = term(p) + chain * np.where(fin, p * np.abs(c), 0).sum()
        err_q = term(q) + chain * np.where(fin, q * np.abs(c), 0).sum()
        loss_err = alpha * err_p + beta * err_q + 4 * U * abs(loss) if np.isfinite(loss) else 0.0
        qa = np.exp(lq_all)
        # every entry's class
        pv, cv = np.zeros(V), np.zeros(V)
        dv = np.full(V, s)
        if rest is not None:
            pv[~listed] = p[-1] * qa[~listed] / q[-1] if q[-1] > 0 else 0.0
            cv[~listed] = c[-1]
            dv[~listed] = dl[-1] if np.isfinite(dl[-1]) else s
        pv[idx], cv[idx] = p[:t.size], c[:t.size]
        dv[idx] = np.where(np.isfinite(dl[:t.size]), dl[:t.size], s)
        yq = np.where(qa > 0, np.abs(y - m), 0.0)
        dv = dv + 6 * U * (yq + 1)
        reverse = np.where(qa > 0, qa * (cv - kl_q), 0.0) if beta else np.zeros(V)
        g = w / tau * (alpha * (qa - pv) + beta * reverse)
        err = alpha * (qa + pv) * 2 * dv
        if beta:
            err = err + beta * np.where(qa > 0, qa * (np.abs(cv - kl_q) * 2 * dv + dv + err_q), 0.0)
        # the hardware's exp2 gives 0 below 2^-126: an unlisted entry's e_v may be
        # missing, which its factor (alpha (q_0 - P_0) + beta q_0 (c_0 - R)) / s_0, with
        # q_0, P_0 <= 1 <= s_0, makes at most this; a listed one's q likewise
        err = err + 2.0 ** -126 * (alpha + beta * (1 + np.abs(np.where(np.isfinite(cv), cv - kl_q, 0.0))
                                                   if beta else 0.0))
        g_err = abs(w) / tau * err + 4 * U * np.abs(g)
    return w * loss, g, abs(w) * loss_err, g_err


# half a step of the type, relative to the value, and half its smallest step
ROUND = {"f32": (U, 2.0 ** -127), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}


def adjust(x, tokens=None, repetition=None, presence=None, frequency=None, bias=None, allowed=None):
    """One fp32 row, each step rounded to fp32: tokens an int array, bias a list
    of (entry, value), allowed a bool array."""
    x = x.astype(np.float32).copy()
    V = x.size
    f = np.float32
    with np.errstate(all="ignore"):
        if tokens is not None:
            count = np.zeros(V, np.int64)
            np.add.at(count, tokens[(tokens >= 0) & (tokens < V)], 1)
            seen = count > 0
            theta = f(1 if repetition is None else repetition)
            x[seen] = np.where(x[seen] > 0, x[seen] / theta, x[seen] * theta)
            x[seen] = x[seen] - f(0 if frequency is None else frequency) * count[seen].astype(f)
            x[seen] = x[seen] - f(0 if presence is None else presence)
        if bias is not None:
            total = {}
            for v, b in bias:
                if 0 <= v < V:
                    total[int(v)] = f(total[int(v)] + f(b)) if int(v) in total else f(b)
            for v, b in total.items():
                x[v] = x[v] + b
        if allowed is not None:
            x[~allowed] = -np.inf
    return x


def pack_mask(allowed):
    """[masks, V] bools as int32 words, bit v % 32 of word v / 32."""
    n, V = allowed.shape
    pad = np.zeros((n, (V + 31) // 32 * 32), bool)
    pad[:, :V] = allowed
    bits = pad.reshape(n, -1, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)
    return bits.sum(-1).astype(np.uint32).view(np.int32)
