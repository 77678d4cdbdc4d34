"""The 64-bit references of the row operators against differences and closed
forms (no GPU)."""
import numpy as np
import pytest

from tests import row_operators_ref as ref


@pytest.mark.parametrize("alpha,beta,with_rest", [(1, 0, False), (1, 0, True), (0, 1, True),
                                                  (0.5, 0.5, True)])
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_gradient_equals_differences(alpha, beta, with_rest, tau):
    rng = np.random.default_rng(1)
    V, k = 23, 5
    z, t = rng.normal(0, 2, V), rng.normal(0, 2, V)
    values, index, rest = ref.top(t[None], k, tau)
    a = (values[0], index[0], rest[0] if with_rest else None, 1.7, tau, alpha, beta)
    _, g, _, _ = ref.distill(z, *a)
    for v in range(V):
        h = 1e-5
        up, down = z.copy(), z.copy()
        up[v] += h
        down[v] -= h
        d = (ref.distill(up, *a)[0] - ref.distill(down, *a)[0]) / (2 * h)
        # the difference's own error: h^2 / 6 of the third derivative and
        # 2^-52 of the loss over h
        assert abs(d - g[v]) < 1e-8


def test_all_entries_listed_is_the_divergence_of_whole_rows():
    rng = np.random.default_rng(2)
    V = 17
    z, t = rng.normal(0, 2, V), rng.normal(0, 2, V)
    values, index, rest = ref.top(t[None], V, 1.0)
    loss, g, _, _ = ref.distill(z, values[0], index[0], rest[0], 1.0, 1.0, 0.5, 0.5)
    q, p = np.exp(z) / np.exp(z).sum(), np.exp(t) / np.exp(t).sum()
    assert np.isclose(loss, 0.5 * ((p - q) * np.log(p / q)).sum(), rtol=1e-12)
    assert abs(g.sum()) < 1e-14


def test_fewer_entries_give_a_lower_bound():
    rng = np.random.default_rng(3)
    z, t = rng.normal(0, 2, 64), rng.normal(0, 2, 64)
    last = 0.0
    for k in (1, 2, 5, 20, 63, 64):
        values, index, rest = ref.top(t[None], k, 1.0)
        loss = ref.distill(z, values[0], index[0], rest[0], 1.0, 1.0, 0.5, 0.5)[0]
        assert loss >= last - 1e-14
        last = loss


def test_equal_entries_are_listed_by_index():
    values, index, rest = ref.top(np.array([[1.0, 3.0, 3.0, 1.0, 3.0]]), 4, 1.0)
    assert index.tolist() == [[1, 2, 4, 0]] and values.tolist() == [[3, 3, 3, 1]]
    assert np.isclose(rest[0], 1.0)
