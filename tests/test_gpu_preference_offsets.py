"""Preference losses of packed pairs whose offsets are not all in order: which pairs are in
error, and what their rows' gradients hold."""
import numpy as np
import pytest

from tests import test_gpu_row_operators as ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P, dev = ops.P, ops.dev

# A short batch, and one so long that the rows are worked out ahead of the pairs.
SCALES = [1, 400]


def batch(scale, V=50):
    rng = np.random.default_rng(scale)
    rows = 12 * scale
    x = rng.normal(0, 1, (rows, V)).astype(np.float32)
    tok = rng.integers(0, V, rows).astype(np.int32)
    return dev(x), dev(tok)


def call(x, tok, first, scale, **kw):
    return P().hbsjd_preference_rows(x, tok, first=dev(np.array(first, np.int32) * scale), **kw)


@pytest.mark.parametrize("scale", SCALES)
def test_pairs_outside_the_outermost_offsets(scale):
    """A pair that reaches ahead of the first offset or behind the last one is in error,
    though its own offsets ascend; the rows there are nobody's and have no sums."""
    x, tok = batch(scale)
    sound = call(x, tok, [0, 2, 4, 7, 12], scale)
    for first, outside in (([5, 2, 4, 7, 12], 1), ([0, 2, 4, 7, -1], 0), ([0, 6, 12, 8, 10], 0),
                           ([3, 2, 4, 7, 12], 0), ([3, 3, 3, 2, 2], 0)):
        # the workspace that the call gets holds what another one has left there
        call(x, tok, [0, 2, 4, 7, 12], scale)
        loss, grad, s = call(x, tok, first, scale)
        at = [v * scale for v in first[2 * outside:2 * outside + 3]]
        assert bool(torch.isnan(loss[outside])), first
        assert bool(torch.isnan(s[2 * outside:2 * outside + 2]).all()), first
        if at[0] <= at[1] <= at[2]:
            assert bool(torch.isnan(grad[at[0]:at[2]]).all()), first
    again = call(x, tok, [0, 2, 4, 7, 12], scale)
    assert all(torch.equal(a, b) for a, b in zip(again, sound))


@pytest.mark.parametrize("scale", SCALES)
def test_rows_outside_the_outermost_offsets_are_left_out(scale):
    """With offsets in order the same rows as without the others."""
    x, tok = batch(scale)
    loss, grad, s = call(x, tok, [2, 3, 5, 7, 9], scale)
    part = slice(2 * scale, 9 * scale)
    want = call(x[part], tok[part], [0, 1, 3, 5, 7], scale)
    assert torch.equal(loss, want[0]) and torch.equal(s, want[2]) and torch.equal(grad[part], want[1])
    assert bool((grad[:2 * scale] == 0).all()) and bool((grad[9 * scale:] == 0).all())


@pytest.mark.parametrize("scale", SCALES)
def test_rows_that_two_pairs_hold(scale):
    """Pairs 0 and 2 are in order and share the rows 4 and 5: losses as of any pair, NaN in
    the shared rows' gradient, each pair's own in the others, the same at every call."""
    x, tok = batch(scale)
    tok[4 * scale] = -1
    first = [0, 3, 6, 2, 4, 5, 9]
    loss, grad, s = call(x, tok, first, scale, beta=0.7)
    assert bool(torch.isnan(loss[1])) and bool(torch.isnan(s[2:4]).all())
    for pair, own in ((0, slice(0, 2 * scale)), (2, slice(6 * scale, 9 * scale))):
        lone = call(x, tok, first[2 * pair:2 * pair + 3], scale, beta=0.7)
        assert torch.equal(loss[pair], lone[0][0]) and torch.equal(s[2 * pair:2 * pair + 2], lone[2])
        assert torch.equal(grad[own], lone[1][own])
    assert bool((grad[4 * scale] == 0).all())       # no token
    assert bool(torch.isnan(grad[4 * scale + 1:6 * scale]).all())
    assert bool((grad[9 * scale:] == 0).all())
    for _ in range(5):
        again = call(x, tok, first, scale, beta=0.7)
        assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(again, (loss, grad, s)))


@pytest.mark.parametrize("scale", SCALES)
def test_rows_of_pairs_in_error(scale):
    """Their two sequences' rows have NaN, one that descends has no rows; a row that is
    another pair's too is shared; the rest is left out or the other pair's."""
    x, tok = batch(scale)
    tok[7 * scale] = -1
    for first, none in (([0, 2, 4, 3, 12], [(3, 12)]), ([5, 2, 4, 7, 12], [(2, 12)]), ([0, 4, 2, 7, 12], [(0, 4)]),
                        ([0, 2, 9, 4, 12], [(4, 12)]), ([0, 2, 4, 7, 13], [(4, 12)]), ([-5, 2, 4, 7, 12], [(0, 4)]),
                        ([12, 11, 10, 9, 8], []), ([6, 4, 5, 3, 2], [(4, 5)]), ([1, 5, 3, 3, 3], [(1, 5)])):
        want = torch.zeros(12 * scale, dtype=torch.bool, device="cuda")
        for a, b in none:
            want[a * scale:b * scale] = True
        want[7 * scale] = False                      # no token
        _, grad, _ = call(x, tok, first, scale)
        assert torch.equal(torch.isnan(grad).all(1), want), first
        assert torch.equal(torch.isnan(grad).any(1), want), first
