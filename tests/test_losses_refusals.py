"""The operators of a policy or preference step refuse bad arguments before any device
work: through the C ABI, without a GPU (no pointer given here is ever read)."""
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


ROWS = dict(rows=4, V=100, elem=0, logits=2 * A, ld=100, tokens=A, temperature=1.0)
CALLS = {
    "logprob": (B._LogprobArgs, dict(logprob_weight=A, entropy_weight=None), ["logprob", "entropy"]),
    "policy": (B._PolicyArgs, dict(advantage=A, old_logprob=None, ref_logprob=A, clip_low=0.2, clip_high=0.2,
                                   kl_weight=0.1, entropy_weight=0.0, row_weight=None),
               ["loss", "logprob", "entropy"]),
    "preference": (B._PreferenceArgs, dict(pairs=2, first=None, ref_logprob=None, form=0, mean=0, beta=0.1,
                                           smoothing=0.0, margin=0.0, pair_weight=None), ["loss", "log_ratio"]),
}


def _call(name, **kw):
    struct, args, outs = CALLS[name]
    L = P.load_library()
    args = dict(ROWS, **args)
    out = dict({o: A for o in outs}, grad=3 * A, ld_grad=100, workspace=A, workspace_bytes=1 << 40)
    assert set(kw) <= set(args) | set(out)
    args.update((k, v) for k, v in kw.items() if k in args)
    out.update((k, v) for k, v in kw.items() if k in out)
    s = struct(*args.values())
    return _status(getattr(L, f"hbsjd_{name}_rows")(ctypes.byref(s), *out.values(), None))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=1 << 31), dict(V=0), dict(V=262145, ld=300000, ld_grad=300000), dict(elem=3),
    dict(elem=-1), dict(ld=99), dict(ld=1 << 41), dict(logits=None), dict(tokens=None), dict(tokens=A + 2),
    dict(logits=2 * A + 2), dict(logits=2 * A + 1, elem=1), dict(temperature=0.0), dict(temperature=-1.0),
    dict(temperature=NAN), dict(temperature=INF), dict(ld_grad=99), dict(grad=2 * A, ld_grad=200),
    dict(grad=3 * A + 2)])
def test_rows_refuse(name, bad):
    assert _call(name, **bad) == "EINVAL"
    assert P.load_library().hbsjd_last_error()


@pytest.mark.parametrize("name,bad", [
    ("logprob", dict(logprob=None, entropy=None, grad=None)), ("logprob", dict(logprob_weight=None)),
    ("logprob", dict(logprob=A + 1)), ("logprob", dict(entropy=A + 2)), ("logprob", dict(logprob_weight=A + 2)),
    ("logprob", dict(entropy_weight=A + 3)),
    ("policy", dict(loss=None, logprob=None, entropy=None, grad=None)), ("policy", dict(advantage=None)),
    ("policy", dict(ref_logprob=None)), ("policy", dict(clip_low=-0.1)), ("policy", dict(clip_low=1.1)),
    ("policy", dict(clip_low=NAN)), ("policy", dict(clip_high=-0.1)), ("policy", dict(clip_high=INF)),
    ("policy", dict(kl_weight=-1.0)), ("policy", dict(kl_weight=NAN)), ("policy", dict(entropy_weight=-1.0)),
    ("policy", dict(entropy_weight=1e7)), ("policy", dict(advantage=A + 2)), ("policy", dict(old_logprob=A + 1)),
    ("policy", dict(ref_logprob=A + 1)), ("policy", dict(row_weight=A + 1)), ("policy", dict(loss=A + 2)),
    ("preference", dict(loss=None, log_ratio=None, grad=None)), ("preference", dict(pairs=-1)),
    ("preference", dict(pairs=1 << 30)), ("preference", dict(pairs=3)), ("preference", dict(pairs=0)),
    ("preference", dict(rows=5)), ("preference", dict(form=3)), ("preference", dict(form=-1)),
    ("preference", dict(beta=0.0)), ("preference", dict(beta=NAN)), ("preference", dict(beta=1e7)),
    ("preference", dict(smoothing=-0.1)), ("preference", dict(smoothing=1.0)), ("preference", dict(smoothing=NAN)),
    ("preference", dict(form=1, smoothing=0.1)), ("preference", dict(form=2, smoothing=0.1)),
    ("preference", dict(margin=NAN)), ("preference", dict(margin=INF)), ("preference", dict(first=A + 2)),
    ("preference", dict(ref_logprob=A + 2)), ("preference", dict(pair_weight=A + 1)),
    ("preference", dict(log_ratio=A + 1)), ("preference", dict(workspace=None)),
    ("preference", dict(workspace_bytes=16)), ("preference", dict(workspace=A + 8))])
def test_calls_refuse(name, bad):
    assert _call(name, **bad) == "EINVAL"


def test_no_rows_is_no_work():
    assert _call("logprob", rows=0) == "OK"
    assert _call("policy", rows=0, logits=None, tokens=None, advantage=None) == "OK"
    assert _call("preference", rows=0, pairs=0, logits=None, tokens=None) == "OK"
    L = P.load_library()
    for f in (L.hbsjd_logprob_rows, L.hbsjd_policy_rows):
        assert _status(f(None, *[A] * (len(f.argtypes) - 5), 100, None, 0, None)) == "EINVAL"
    assert _status(L.hbsjd_preference_rows(None, A, A, A, 100, None, 0, None)) == "EINVAL"


def test_workspaces():
    L = P.load_library()
    for V in (1, 100, 16384):
        assert L.hbsjd_token_workspace(5, V, 0) == 0
        assert L.hbsjd_preference_workspace(5, V, 0) > 0
    need = L.hbsjd_token_workspace(2, 200000, 0)
    assert need > 0
    long = dict(rows=2, V=200000, ld=200000, ld_grad=200000)
    for name in ("logprob", "policy"):
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=A + 8)):
            assert _call(name, **long, **bad) == "EINVAL"
    for f in (L.hbsjd_token_workspace, L.hbsjd_preference_workspace):
        for bad in ((0, 200000, 0), (-1, 200000, 0), (1 << 31, 200000, 0), (5, 300000, 0), (5, 0, 0),
                    (5, 200000, 4)):
            assert f(*bad) == 0
    # bounded, however many rows
    assert L.hbsjd_token_workspace((1 << 31) - 1, 262144, 0) <= 64 << 20


def _grads(call, count=2, data=(2 * A, 4 * A), sizes=(10, 20), elems=(0, 0), order=2, norm=A, workspace=A,
           workspace_bytes=1 << 30, limit=1.0, out=None):
    L = P.load_library()
    array = lambda t, v: None if v is None else (t * len(v))(*v)
    head = (count, array(ctypes.c_void_p, data), array(ctypes.c_int64, sizes), array(ctypes.c_int32, elems), order)
    if call == "norm":
        return _status(L.hbsjd_grad_norm(*head, norm, workspace, workspace_bytes, None))
    return _status(L.hbsjd_clip_grads(*head, limit, array(ctypes.c_void_p, out), norm, workspace, workspace_bytes,
                                      None))


@pytest.mark.parametrize("call", ["norm", "clip"])
@pytest.mark.parametrize("bad", [
    dict(count=-1), dict(count=65537), dict(data=None), dict(sizes=None), dict(elems=None), dict(norm=None),
    dict(norm=A + 2), dict(order=1), dict(order=3), dict(elems=(0, 3)), dict(sizes=(10, -1)),
    dict(sizes=(10, 1 << 40)), dict(data=(2 * A, None)), dict(data=(2 * A + 2, 4 * A)),
    dict(data=(2 * A, 4 * A + 1), elems=(0, 1)), dict(workspace=None), dict(workspace_bytes=8),
    dict(workspace=A + 8)])
def test_grads_refuse(call, bad):
    assert _grads(call, **bad) == "EINVAL"


@pytest.mark.parametrize("bad", [
    dict(limit=-1.0), dict(limit=NAN), dict(out=(2 * A, None)), dict(out=(2 * A + 1, 4 * A)),
    dict(data=(2 * A, 2 * A)), dict(data=(2 * A, 2 * A + 36)), dict(data=(2 * A + 76, 2 * A)),
    dict(out=(4 * A, 2 * A)), dict(out=(6 * A, 6 * A + 39 // 4 * 4)), dict(out=(2 * A + 4, 4 * A)),
    dict(out=(6 * A, 2 * A))])
def test_clip_refuses(bad):
    assert _grads("clip", **bad) == "EINVAL"


def test_grads_refuse_more_than_a_device_holds():
    n = 200
    big = dict(count=n, data=tuple(A + 16 * i for i in range(n)), sizes=((1 << 40) - 1,) * n, elems=(0,) * n)
    assert _grads("norm", **big) == "EINVAL"
    big["data"] = tuple(A + (i << 43) for i in range(n))
    assert _grads("clip", **big) == "EINVAL"


def test_grads_refuse_what_are_no_device_tensors():
    import torch
    for f in (lambda: P.hbsjd_grad_norm([torch.zeros(3)]), lambda: P.hbsjd_clip_grads([torch.zeros(3)], 1.0),
              lambda: P.hbsjd_logprob_rows(torch.zeros(3, 8), torch.zeros(3).int()),
              lambda: P.hbsjd_policy_rows(torch.zeros(3, 8), torch.zeros(3).int(), torch.zeros(3)),
              lambda: P.hbsjd_preference_rows(torch.zeros(4, 8), torch.zeros(4).int(), pairs=1)):
        with pytest.raises(ValueError):
            f()
