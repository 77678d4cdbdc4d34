"""The row operators refuse bad arguments before any device work: through the C
ABI, without a GPU (no pointer given here is ever read)."""
import ctypes
import os

import pytest

pytest.importorskip("torch")
import paper_2608_18183_amd as P
from paper_2608_18183_amd import binding as B

A = 0x10000   # an address that is never read
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.library_path()):
        pytest.skip("libhbsjd.so is not built")


def _status(st):
    return {0: "OK", 1: "EINVAL"}.get(st, st)


def _top(**kw):
    a = dict(rows=2, V=100, logits=A, elem=0, ld=100, K=5, temperature=1.0, values=A, index=A,
             rest=A, workspace=None, workspace_bytes=0, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return _status(P.load_library().hbsjd_top_logits_rows(*a.values()))


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=1 << 31), dict(V=0), dict(V=262145, ld=300000), dict(K=0), dict(K=101),
    dict(V=5000, ld=5000, K=2049), dict(elem=3), dict(elem=-1), dict(ld=99), dict(ld=1 << 41),
    dict(logits=None), dict(values=None), dict(index=None), dict(rest=None), dict(temperature=0.0),
    dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(logits=A + 2),
    dict(logits=A + 1, elem=1), dict(values=A + 2), dict(index=A + 1), dict(rest=A + 3)])
def test_top_logits_refuses(bad):
    assert _top(**bad) == "EINVAL"
    assert P.load_library().hbsjd_last_error()


def test_no_rows_is_no_work():
    assert _top(rows=0) == "OK"
    assert _top(rows=0, logits=None, values=None, index=None, rest=None) == "OK"
    assert _distill(rows=0) == "OK"
    assert _adjust(rows=0) == "OK"


def _distill(loss=A, grad=A, ld_grad=100, workspace=None, workspace_bytes=0, **kw):
    a = dict(rows=2, V=100, K=5, logits=2 * A, ld=100, elem=0, temperature=1.0, values=A, index=A,
             rest=A, forward_weight=0.5, reverse_weight=0.5, row_weight=None)
    assert set(kw) <= set(a)
    a.update(kw)
    s = B._DistillArgs(*a.values())
    return _status(P.load_library().hbsjd_distill_top_rows(ctypes.byref(s), loss, grad, ld_grad,
                                                           workspace, workspace_bytes, None))


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=1 << 31), dict(V=0), dict(V=262145, ld=300000), dict(K=0), dict(K=2049),
    dict(elem=7), dict(ld=99), dict(logits=None), dict(values=None), dict(index=None),
    dict(rest=None), dict(temperature=0.0), dict(temperature=NAN), dict(forward_weight=-0.1),
    dict(forward_weight=0.0, reverse_weight=0.0), dict(reverse_weight=NAN), dict(forward_weight=INF),
    dict(loss=None, grad=None), dict(ld_grad=99), dict(grad=2 * A, ld=200), dict(grad=A + 2),
    dict(logits=A + 1, elem=2), dict(row_weight=A + 2), dict(loss=A + 1), dict(rest=A + 2)])
def test_distill_refuses(bad):
    assert _distill(**bad) == "EINVAL"


def test_long_rows_need_their_workspace():
    L = P.load_library()
    for f, call in ((L.hbsjd_top_logits_workspace, _top), (L.hbsjd_distill_top_workspace, _distill)):
        for V in (1, 100, 16384):
            assert f(5, V, 0, min(V, 5)) == 0
        need = f(2, 200000, 0, 5)
        assert need > 0
        long = dict(V=200000, ld=200000, **({"ld_grad": 200000} if call is _distill else {}))
        assert call(**long) == "EINVAL"
        assert call(workspace=A, workspace_bytes=need - 1, **long) == "EINVAL"
        assert call(workspace=A + 8, workspace_bytes=need, **long) == "EINVAL"
        for bad in ((0, 200000, 0, 5), (5, 300000, 0, 5), (5, 200000, 4, 5), (5, 200000, 0, 0),
                    (5, 200000, 0, 4000)):
            assert f(*bad) == 0
        # bounded, however many rows
        assert f((1 << 31) - 1, 262144, 0, 2048) <= 256 << 20


def test_distill_refuses_null_args():
    assert _status(P.load_library().hbsjd_distill_top_rows(None, A, A, 100, None, 0, None)) == "EINVAL"
    assert _status(P.load_library().hbsjd_adjust_rows(None, A, 0, 100, None)) == "EINVAL"


def _adjust(out=A, out_elem=0, ld_out=100, **kw):
    a = dict(rows=2, V=100, elem=0, logits=2 * A, ld=100, tokens=A, n_tokens=7, ld_tokens=7,
             token_count=None, repetition=A, presence=None, frequency=None, bias_index=A,
             bias_value=A, n_bias=3, ld_bias=3, mask=A, n_masks=2, mask_row=None)
    assert set(kw) <= set(a)
    a.update(kw)
    s = B._AdjustArgs(*a.values())
    return _status(P.load_library().hbsjd_adjust_rows(ctypes.byref(s), out, out_elem, ld_out, None))


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=1 << 31), dict(V=0), dict(V=262145, ld=300000, ld_out=300000),
    dict(elem=5), dict(out_elem=1), dict(elem=1, out_elem=2), dict(elem=2, out_elem=1),
    dict(ld=99), dict(ld_out=99), dict(logits=None), dict(out=None),
    dict(out=2 * A, ld_out=200), dict(out=2 * A, elem=1, out_elem=0), dict(n_tokens=-1),
    dict(n_bias=-1), dict(n_bias=1025), dict(n_masks=0), dict(n_masks=1), dict(n_masks=-3),
    dict(mask=None, mask_row=A), dict(tokens=None), dict(bias_index=None), dict(bias_value=None),
    dict(ld_tokens=-1), dict(ld_bias=-1), dict(tokens=A + 2), dict(mask=A + 1),
    dict(token_count=A + 2), dict(repetition=A + 3), dict(bias_value=A + 2), dict(out=A + 2),
    dict(logits=A + 1, elem=1, out_elem=1)])
def test_adjust_refuses(bad):
    assert _adjust(**bad) == "EINVAL"


def test_binding_refuses_what_is_not_a_device_matrix():
    import torch
    x = torch.zeros(3, 8)
    for f in (lambda: P.hbsjd_top_logits_rows(x, 2),
              lambda: P.hbsjd_distill_top_rows(x, x[:, :2], x[:, :2].int()),
              lambda: P.hbsjd_adjust_rows(x)):
        with pytest.raises(ValueError):
            f()
