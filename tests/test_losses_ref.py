"""The 64-bit references of the policy and preference operators against differences
and closed forms (no GPU)."""
import math

import numpy as np
import pytest

from tests import losses_ref as ref

H = 1e-5


def differences(f, z):
    out = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        up, down = z.copy(), z.copy()
        up[i] += H
        down[i] -= H
        out[i] = (f(up) - f(down)) / (2 * H)
    return out


# the differences' own error: H^2 / 6 of a third derivative of a few units, and
# 2^-52 of the loss over H
TOL = 2e-8


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("token", [0, 7])
def test_log_probability_and_entropy(tau, token):
    z = np.random.default_rng(1).normal(0, 2, 19)
    q = ref.Row(z, token, tau)
    p = np.exp(z / tau) / np.exp(z / tau).sum()
    assert math.isclose(q.l, math.log(p[token]), rel_tol=1e-13)
    assert math.isclose(q.entropy, -(p * np.log(p)).sum(), rel_tol=1e-13)
    for g, h in ((1.0, 0.0), (0.0, 1.0), (-1.3, 0.4)):
        def f(x):
            q = ref.Row(x, token, tau)
            return g * q.l + h * q.entropy
        got, _ = q.gradient(g, h, 0.0, "f32")
        assert np.abs(got - differences(f, z)).max() < TOL
        assert abs(got.sum()) < 1e-14


@pytest.mark.parametrize("adv", [1.5, -0.8, 0.0])
@pytest.mark.parametrize("shift", [-0.6, 0.0, 0.6, None])
@pytest.mark.parametrize("kl,bonus", [(0.0, 0.0), (0.3, 0.05)])
def test_policy(adv, shift, kl, bonus):
    """Inside the bounds, and beyond either one."""
    z = np.random.default_rng(2).normal(0, 1, 13)
    l = ref.Row(z, 4, 0.8).l
    old = None if shift is None else l + shift
    kw = dict(old=old, ref=l - 0.7, kl=kl, bonus=bonus, w=1.7)

    def f(x):
        q = ref.Row(x, 4, 0.8)
        # without old the ratio's denominator is the row's own at z, a constant
        return ref.policy(q, adv, **dict(kw, old=l if old is None else old))[0]
    q = ref.Row(z, 4, 0.8)
    loss, _, g, h, _ = ref.policy(q, adv, **kw)
    assert math.isclose(loss, f(z), rel_tol=1e-12, abs_tol=1e-15)
    got, _ = q.gradient(g, h, 0.0, "f32")
    assert np.abs(got - differences(f, z)).max() < TOL


@pytest.mark.parametrize("form,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.2), ("hinge", 0.0), ("square", 0.0)])
@pytest.mark.parametrize("mean", [False, True])
def test_preference(form, smoothing, mean):
    rng = np.random.default_rng(3)
    z = rng.normal(0, 1, (7, 6))
    tokens, ends = np.array([0, 3, -1, 5, 2, 2, -1]), [0, 4, 7]
    base = rng.normal(-2, 0.3, 7)
    kw = dict(form=form, beta=0.7, mean=mean, smoothing=smoothing, margin=0.1, w=1.2)

    def f(x):
        return ref.preference(x, tokens, ends, base, 1.3, **kw)[0][0]
    grads = ref.preference(z, tokens, ends, base, 1.3, **kw)[3]
    want = differences(f, z)
    for r in range(7):
        got = grads[r][0] if r in grads else np.zeros(6)
        assert np.abs(got - want[r]).max() < TOL


def test_preference_of_equal_sequences():
    z = np.random.default_rng(4).normal(0, 1, (2, 9))
    z[1] = z[0]
    (loss, _), s, _, _ = ref.preference(z, np.array([1, 1]), [0, 1, 2], None, 1.0, "sigmoid", 0.1)
    assert math.isclose(loss, math.log(2)) and s[0] == s[1]
