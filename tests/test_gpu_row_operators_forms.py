"""The forms of the row operators that batches take: the largest rows that are
held whole, calls of more rows than a slab of the workspace, parts of many fp32
rows, and the adjustment's workgroups for many rows. Same references and bounds
as tests/test_gpu_row_operators.py; where there are many rows, some of them."""
import numpy as np
import pytest

from tests import row_operators_ref as ref
from tests import test_gpu_row_operators as ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P, dev, placed, untouched, TYPES = ops.P, ops.dev, ops.placed, ops.untouched, ops.TYPES
ELEMS = {"f32": 0, "bf16": 1, "f16": 2}


def device_rows(seed, n, V, dtype):
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((n, V), generator=gen, device="cuda")
    x *= torch.exp(torch.rand((n, 1), generator=gen, device="cuda") * 2 - 1) * 2
    return x.to(TYPES[dtype])


def listed_answers(rng, x, k):
    """Answers that list k spread entries of each row, and a mass for the others."""
    n, V = x.shape
    stride = next(s for s in range(V // k, 0, -1) if np.gcd(s, V) == 1)
    index = (np.arange(k)[None] * stride + rng.integers(0, V, (n, 1))) % V
    near = x.gather(1, dev(index)).float().cpu().numpy()
    values = (near + rng.normal(0, 0.7, (n, k))).astype(np.float32)
    rest = torch.logsumexp(x.float(), 1).cpu().numpy() + rng.normal(0, 0.5, n).astype(np.float32)
    return values, index.astype(np.int32), rest.astype(np.float32)


def check_some(rows, x, values, index, rest, w, alpha, beta, loss, grad, dtype):
    x64 = x[rows].double().cpu().numpy()
    ops.check_distill(x64, values[rows], index[rows], None if rest is None else rest[rows], w[rows],
                      1.0, alpha, beta, loss[rows], grad[rows], dtype)


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("V,dtype", [(32769, "f32"), (50001, "f32"), (65536, "f32"), (65537, "bf16"),
                                     (100003, "bf16"), (131072, "bf16"), (65543, "f16"), (131072, "f16")])
def test_distill_of_many_long_rows_held_whole(V, dtype, layout):
    rng = np.random.default_rng(V)
    n = 112
    # a row that needs no workspace goes whole
    assert P().load_library().hbsjd_distill_top_workspace(n, V, ELEMS[dtype], 64) == 0
    x, _ = placed(device_rows(V, n, V, dtype), layout)
    rows = [0, 1, 2, 55, 110, 111]
    for k, alpha, beta, with_rest in ((64, 0.5, 0.5, True), (2048, 1.0, 0.0, False)):
        values, index, rest = listed_answers(rng, x, k)
        index[1, 2] = -1
        if not with_rest:
            rest = None
        w = rng.uniform(0.5, 2, n).astype(np.float32)
        w[2] = 0.0
        answer = [dev(values), dev(index), None if rest is None else dev(rest)]
        kw = dict(forward_weight=alpha, reverse_weight=beta, row_weight=dev(w))
        grad, gbuf = placed(torch.full((n, V), 3.0, dtype=TYPES[dtype], device="cuda"), layout)
        loss, _ = P().hbsjd_distill_top_rows(x, *answer, grad=grad, **kw)
        check_some(rows, x, values, index, rest, w, alpha, beta, loss, grad, dtype)
        assert float(loss[2]) == 0 and bool((grad[2] == 0).all())
        if gbuf is not None:
            assert untouched(gbuf, grad)
        only, _ = P().hbsjd_distill_top_rows(x, *answer, grad=False, **kw)
        assert torch.equal(only, loss)
        own, obuf = placed(x.clone(), layout)
        again, _ = P().hbsjd_distill_top_rows(own, *answer, grad=own, **kw)
        assert torch.equal(again, loss) and torch.equal(own, grad)
        if obuf is not None:
            assert untouched(obuf, own)


def slab_of(workspace, V, elem, k):
    """Rows of a slab: the workspace grows by a row's bytes up to that many."""
    a = workspace(1024, V, elem, k)
    per_row = a // 1024
    assert per_row * 1024 == a and workspace(1025, V, elem, k) == a + per_row
    most = workspace((1 << 31) - 1, V, elem, k)
    assert most % per_row == 0
    return most // per_row


@pytest.mark.parametrize("V,dtype", [(65537, "f32"), (131073, "bf16")])
def test_distill_of_more_rows_than_a_slab(V, dtype):
    rng = np.random.default_rng(V)
    k = 2048
    slab = slab_of(P().load_library().hbsjd_distill_top_workspace, V, ELEMS[dtype], k)
    n = slab + 5
    assert n < 9000
    x = device_rows(V, n, V, dtype)
    values, index, rest = listed_answers(rng, x, k)
    w = rng.uniform(0.5, 2, n).astype(np.float32)
    rows = [0, 7, slab - 1, slab, slab + 4]
    kept = x[rows]
    answer = [dev(values), dev(index), dev(rest)]
    loss, grad = P().hbsjd_distill_top_rows(x, *answer, row_weight=dev(w), grad=x)
    assert grad is x
    loss, grad = loss[rows], x[rows]
    ops.check_distill(kept.double().cpu().numpy(), values[rows], index[rows], rest[rows], w[rows], 1.0,
                      0.5, 0.5, loss, grad, dtype)


@pytest.mark.parametrize("V,dtype,k", [(16385, "f32", 2048), (40000, "bf16", 2000), (33001, "f16", 2000)])
def test_top_logits_of_more_rows_than_a_slab(V, dtype, k):
    slab = slab_of(P().load_library().hbsjd_top_logits_workspace, V, ELEMS[dtype], k)
    n = slab + 5
    assert n < 9000
    x = device_rows(V, n, V, dtype)
    got = P().hbsjd_top_logits_rows(x, k)
    rows = [0, 7, slab - 1, slab, slab + 4]
    ops.check_top(x[rows].double().cpu().numpy(), [t[rows] for t in got], k, 1.0)


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("V", [16385, 20000, 32768])
def test_top_logits_of_many_fp32_rows_in_parts(V, layout):
    n = 520
    x, _ = placed(device_rows(V, n, V, "f32"), layout)
    x[5] = torch.round(x[5])
    x[6, V // 3:] = -float("inf")
    x[519, 3:] = -float("inf")
    rows = [0, 5, 6, 300, 519]
    x64 = x[rows].double().cpu().numpy()
    for k in (1, 64, 300, 2048):
        got = P().hbsjd_top_logits_rows(x, k)
        ops.check_top(x64, [t[rows] for t in got], k, 1.0)


@pytest.mark.parametrize("dtype,out_type", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"),
                                            ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("n,V", [(512, 16384), (513, 8203), (171, 33001), (64, 128257)])
def test_adjust_of_many_rows(n, V, dtype, out_type):
    """Enough rows, of enough entries, for the adjustment's largest workgroups."""
    rng = np.random.default_rng(V + n)
    for n_tokens, n_bias, masks, layout in ((300, 70, 5, "shifted"), (40, 0, 0, "plain"),
                                            (0, 0, 3, "shifted"), (2000, 300, 4, "plain")):
        ops.adjust_case(rng, n, V, dtype, n_tokens, n_bias, masks, layout, out_type)
    if dtype == out_type:
        ops.adjust_case(rng, n, V, dtype, 300, 70, 5, "shifted", in_place=True)
        ops.adjust_case(rng, n, V, dtype, 576, 0, 0, "plain", in_place=True)
