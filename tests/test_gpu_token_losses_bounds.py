"""Token losses against 64 bits within bounds counted from the kernels' steps.

With U half a step of fp32, c = log2 e / tau as one fp32 number and y_v = (largest logit -
z_v) / tau >= 0, an exponent z_v c - k takes two roundings: c's, which puts it off by U y_v
in nats whatever k is (what k is rounded by goes back in 64 bits), and the fused operation's,
U (y_v + 0.03), since k lies within 1/32 of the largest z c. The hardware's exp2 is good to a
step, 2 U. Together U (2 y_v + 2.03) of a term, for every type of the logits. A thread's sum
takes 7 roundings in a vector's chain of 8 entries, 15 in the chain of 16 vectors at most and
one for an edge entry; the rest is in 64 bits, a part's sum and its factor one rounding each.
losses_ref.Row counts 2 y_v + 2 a term, 26 roundings, 4 for parts, and 3 more, which is no
less; its bound of a 16-bit gradient counts 4 y_v, and here it is that of an fp32 gradient and
the one rounding to the type.
"""
import decimal
import math

import numpy as np
import pytest

from tests import losses_ref as ref
from tests.row_operators_ref import ROUND
from tests import test_gpu_row_operators as ops
from tests.test_gpu_token_losses import check_l, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P, dev, rows_of, TYPES = ops.P, ops.dev, ops.rows_of, ops.TYPES


def worst_temperatures():
    """Those of a grid whose factor is rounded the most, up and down."""
    taus = np.linspace(0.3, 3.0, 4001).astype(np.float32)
    c = math.log2(math.e) / taus.astype(np.float64)
    off = (c.astype(np.float32).astype(np.float64) - c) / c
    return [float(taus[off.argmax()]), float(taus[off.argmin()])]


def test_factors_rounding_is_reached():
    for tau in worst_temperatures():
        c = math.log2(math.e) / tau
        assert 0.9 * 2.0 ** -24 < abs(float(np.float32(c)) - c) / c <= 2.0 ** -24


@pytest.mark.parametrize("tau", worst_temperatures())
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,shift", [(70, 0.0), (5003, 0.0), (16384, 0.0), (70001, 0.0), (262144, 0.0),
                                     (5003, 20000.0), (70001, -20000.0)])
def test_sums_and_gradients(V, shift, dtype, tau):
    rng = np.random.default_rng(V)
    n = 3
    t, _ = rows_of(rng, n, V, dtype)
    t = (t.float() * 3 + shift).to(TYPES[dtype])   # entries far below the largest, and far from 0
    x64 = t.double().numpy()
    tok = np.array([x64[0].argmax(), rng.integers(V), x64[2].argmin()], np.int32)
    a, b = (rng.normal(0, 1, n).astype(np.float32) for _ in range(2))
    step, least = ROUND[dtype]
    l, entropy, grad = P().hbsjd_logprob_rows(t.cuda(), dev(tok), temperature=tau, entropy=True,
                                              logprob_weight=dev(a), entropy_weight=dev(b), grad=True)
    alone = P().hbsjd_logprob_rows(t.cuda(), dev(tok), temperature=tau, logprob_weight=dev(a), grad=True)[2]
    for r in range(n):
        q = ref.Row(x64[r], tok[r], tau)
        check_l(l[r], q, r)
        within(np.array(float(entropy[r])), q.entropy, q.entropy_err, r)
        for got, h in ((grad, float(b[r])), (alone, 0.0)):
            want, bound = q.gradient(float(a[r]), h, 0.0, "f32")
            if dtype != "f32":
                bound = bound + step * np.abs(want) * 1.01 + least
            within(got[r], want, bound, (r, h))


def certain(z, tau):
    """-l, H and the gradients of l and H at the first entry, the largest, in 60 digits; and
    the largest distance in nats."""
    with decimal.localcontext() as c:
        c.prec = 60
        D = decimal.Decimal
        y = [(D(float(z[0])) - D(float(v))) / D(tau) for v in z[1:]]
        e = [(-v).exp() for v in y]
        se = sum(e)
        s, ey = 1 + se, sum(a * b for a, b in zip(e, y))
        return [float(v) for v in (s.ln(), s.ln() + ey / s, se / s / D(tau), -ey / (s * s) / D(tau), max(y))]


@pytest.mark.parametrize("gap", [8, 20, 36, 40, 50, 60, 78])
@pytest.mark.parametrize("V", [2, 9, 300, 40000])
def test_nearly_certain_tokens_keep_their_digits(V, gap):
    """Every term of l, H and their gradients at such a token has the same sign, so what they
    are off by is relative: a term's 2 y + 2.03 and 26 roundings of sums as above; y and the
    product in H's terms 2 more, a part's offset 4, the token's own exponential and the
    rounding to fp32 4: U (2 y + 40)."""
    rng = np.random.default_rng(V + gap)
    one = dev(np.ones(1, np.float32))
    for tau in (1.0, 0.25, *worst_temperatures()):
        z = rng.normal(0, tau, (1, V)).astype(np.float32)
        z[0, 0] = z[0, 1:].max() + gap * tau
        x, tok = dev(z), dev(np.zeros(1, np.int32))
        want = certain(z[0], tau)
        l, H, g = P().hbsjd_logprob_rows(x, tok, temperature=tau, entropy=True, logprob_weight=one, grad=True)
        h = P().hbsjd_logprob_rows(x, tok, temperature=tau, entropy_weight=one, grad=True)[2]
        for got, w in zip((-l[0], H[0], g[0, 0], h[0, 0]), want):
            # terms that fp32's exponentials drop: V of them below 2^-126, times 128 nats
            assert abs(float(got) - w) <= 2.0 ** -24 * (2 * want[4] + 40) * abs(w) + V * 128 * 2.0 ** -126 / tau, tau
