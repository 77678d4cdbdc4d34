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
