"""Preference losses of batches without pairs: nothing to work out is no error."""
import os

import pytest

torch = pytest.importorskip("torch")
import paper_2608_18183_amd as P
from tests.test_losses_refusals import A, _call


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.library_path()):
        pytest.skip("libhbsjd.so is not built")


NONE = dict(pairs=0, first=A, loss=None, log_ratio=None, grad=None)


def test_no_pairs_and_no_outputs():
    assert _call("preference", **NONE) == "OK"
    assert _call("preference", **dict(NONE, rows=0)) == "OK"
    assert _call("preference", **dict(NONE, loss=A, log_ratio=A)) == "OK"


@pytest.mark.parametrize("bad", [
    dict(pairs=1), dict(first=None), dict(logits=None), dict(tokens=None), dict(first=A + 2), dict(ld=99),
    dict(form=3), dict(workspace=None)])
def test_arguments_are_checked_all_the_same(bad):
    assert _call("preference", **dict(NONE, **bad)) == "EINVAL"


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [0, 5])
@pytest.mark.parametrize("grad", [False, True])
def test_empty_packed_batch(rows, grad):
    x = torch.randn(rows, 64, device="cuda")
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    first = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, g, s = P.hbsjd_preference_rows(x, tok, first=first, grad=grad)
    assert loss.shape == (0,) and s.shape == (0,)
    assert (g is not None and g.shape == x.shape and bool((g == 0).all())) if grad else g is None


@pytest.mark.gpu
def test_no_rows_of_any_strides():
    """A matrix without rows has no entries that could lie apart."""
    x = torch.empty_strided((0, 8), (1, 2), device="cuda")
    f, i = torch.zeros(0, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    assert x.shape == (0, 8) and x.stride(1) != 1
    assert P.hbsjd_logprob_rows(x, i, logprob_weight=f, grad=True)[2].shape == (0, 8)
    assert P.hbsjd_logprob_rows(x, i, logprob_weight=f, grad=x)[2] is x
    assert P.hbsjd_policy_rows(x, i, f)[1].shape == (0, 8)
    loss, grad, s = P.hbsjd_preference_rows(x, i, pairs=2)
    assert loss.shape == (2,) and s.tolist() == [0.0] * 4 and grad.shape == (0, 8)
    assert P.hbsjd_top_logits_rows(x, 3)[0].shape == (0, 3)
