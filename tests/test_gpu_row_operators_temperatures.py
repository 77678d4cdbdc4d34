"""The row operators at temperatures near the ends of their range and on logits
of any size: logits over the temperature of 1e9 and more, where a rounding of the
quotient in fp32 is larger than the exponential's whole range."""
import numpy as np
import pytest

from tests import row_operators_ref as ref
from tests import test_gpu_row_operators as ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = ref.U


def log_softmax(x):
    y = x - x.max()
    return y - np.log(np.exp(y).sum())


def distill(z, t, index, rest, w, tau, alpha, beta):
    """One row: loss, gradient and bounds on their errors. Differences of logits
    are formed before they are divided, as fp32 numbers have them exactly, so a log
    probability has the relative error of a few roundings beside what its
    normaliser's sum is off by. A probability's relative error is e, a log ratio's e
    + 4 U of it."""
    V, k = z.size, t.size
    listed = np.zeros(V, bool)
    listed[index] = True
    lq_all = log_softmax((z - z.max()) / tau)
    top = t.max()
    a = (t - top) / tau
    raw = max(abs(top) / tau, 0 if rest is None else abs(rest))
    if rest is None:
        lp, lq = log_softmax(a), lq_all[index]
    else:
        lp = log_softmax(np.append(a, rest - top / tau))
        m0 = lq_all[~listed].max()
        lq0 = m0 + np.log(np.exp(lq_all[~listed] - m0).sum())
        lq = np.append(lq_all[index], lq0)
    e = ref.log_sum_bound(V) + ref.log_sum_bound(k + 1) + 8 * U
    if raw < 1e10:    # rest less the largest logit over tau, rounded in 64 bits on either side;
        e += 2.0 ** -50 * raw   # beyond that the two differ by 2^-26 of them here at least
    p, q, c = np.exp(lp), np.exp(lq), lq - lp
    kl_p, kl_q = -(p * c).sum(), (q * c).sum()
    loss = alpha * kl_p + beta * kl_q
    err = lambda x: (x * (e + 4 * U) * (np.abs(c) + 1)).sum()
    loss_err = alpha * err(p) + beta * err(q) + 4 * U * abs(loss)
    qv, pv, cv = np.exp(lq_all), np.zeros(V), np.zeros(V)
    if rest is not None:
        pv[~listed] = p[-1] * np.exp(lq_all[~listed] - lq0)
        cv[~listed] = c[-1]
    pv[index], cv[index] = p[:k], c[:k]
    g = alpha * (qv - pv) + beta * qv * (cv - kl_q)
    g_err = 2 * e * alpha * (qv + pv) + beta * qv * (
        np.abs(cv - kl_q) * (2 * e + 4 * U) + e + 4 * U * np.abs(cv) + err(q))
    # the hardware's exp2 gives 0 below 2^-126
    g_err = g_err + 2.0 ** -126 * (alpha + beta * (1 + np.abs(cv - kl_q)))
    return (w * loss, w / tau * g, w * loss_err, w / tau * g_err + 4 * U * np.abs(w / tau * g) + 2.0 ** -126)


@pytest.mark.parametrize("V", [300, 16384, 40000])
@pytest.mark.parametrize("with_rest", [True, False])
@pytest.mark.parametrize("tau,size", [(1e-6, 4e3), (1e-5, 4e4), (0.7, 1.5e9), (3.0, 2e30), (1e6, 4e3),
                                      (1.0, 1e-30)])
def test_distill(tau, size, with_rest, V):
    rng = np.random.default_rng(int(V + size % 97))
    n, k = 12, 8
    tau = float(np.float32(tau))
    z = (size * rng.uniform(0.5, 1.5, (n, V))).astype(np.float32)
    t = (size * rng.uniform(0.75, 1.5, (n, k))).astype(np.float32)
    index = np.argsort(rng.random((n, V)), 1)[:, :k].astype(np.int32)
    t[::3, 4] = t[::3, 1] = t[::3].max(1)                 # two first choices
    t[1::4] = -t[1::4]
    for r in range(0, n, 2):                              # the student's first choice is the teacher's
        z[r, index[r, t[r].argmax()]] = np.float32(1.6 * size)
    w = rng.uniform(0.5, 2, n).astype(np.float32)
    top = t.max(1).astype(np.float64) / tau
    rest = np.where(np.arange(n) % 3 == 0, top - 0.25 * np.abs(top), top + 0.25 * np.abs(top))
    if top.max() < 1e10:
        rest[1::3] = top[1::3]                            # as much as the first choice, rounded
    rest = rest.astype(np.float32) if with_rest else None
    alpha, beta = (0.6, 0.4) if with_rest else (1.0, 0.0)
    loss, grad = ops.P().hbsjd_distill_top_rows(
        ops.dev(z), ops.dev(t), ops.dev(index), ops.dev(rest) if with_rest else None, temperature=tau,
        forward_weight=alpha, reverse_weight=beta, row_weight=ops.dev(w))
    loss, grad = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    alpha, beta = float(np.float32(alpha)), float(np.float32(beta))
    for r in range(n):
        wl, wg, el, eg = distill(z[r].astype(np.float64), t[r].astype(np.float64), index[r],
                                 np.float64(rest[r]) if with_rest else None, float(w[r]), tau, alpha, beta)
        assert abs(loss[r] - wl) <= el, (r, loss[r], wl, el)
        off = np.abs(grad[r] - wg) - eg
        assert off.max() <= 0, (r, int(off.argmax()), grad[r][off.argmax()], wg[off.argmax()])


@pytest.mark.parametrize("V", [300, 16384, 40000])
@pytest.mark.parametrize("tau,size", [(1e-6, 4e3), (1e-5, 4e4), (0.7, 1.5e9), (3.0, 2e30), (1e6, 4e3)])
def test_top_logits(tau, size, V):
    rng = np.random.default_rng(V)
    tau = float(np.float32(tau))
    x = (size * rng.uniform(-1.5, 1.5, (4, V))).astype(np.float32)
    x[1] = np.round(x[1] / size * 8) * np.float32(size / 8)
    x[2] = -np.abs(x[2])
    for k in (1, 8, 200):
        got = ops.P().hbsjd_top_logits_rows(ops.dev(x), k, temperature=tau)
        ops.check_top(x.astype(np.float64), got, k, tau)
