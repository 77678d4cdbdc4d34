"""Autograd records none of the row operators, and sees what they write."""
import pytest

from tests import row_operators_ref as ref
from tests import test_gpu_row_operators as ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P = ops.P


def answer_of(x, k=4):
    return P().hbsjd_top_logits_rows(x.detach() + 0.5, k)


def write_top(y, out):
    values, index, rest = answer_of(y, y.shape[1])
    P().hbsjd_top_logits_rows(y.detach().clone(), y.shape[1], out=(out, index, rest))


def write_gradient(y, out):
    P().hbsjd_distill_top_rows(y, *answer_of(y), grad=out)


def write_adjusted(y, out):
    P().hbsjd_adjust_rows(y, tokens=torch.zeros(3, dtype=torch.int32, device="cuda"),
                          presence=torch.ones(y.shape[0], device="cuda"), out=out)


@pytest.mark.parametrize("other_stream", [False, True])
@pytest.mark.parametrize("write", [write_top, write_gradient, write_adjusted])
def test_a_saved_tensor_that_is_overwritten_is_noticed(write, other_stream):
    x = torch.randn(3, 40, device="cuda", requires_grad=True)
    y = x.exp()                       # keeps its result for its backward pass
    torch.cuda.synchronize()
    before = y._version
    if other_stream:
        with torch.cuda.stream(torch.cuda.Stream()):
            write(y, y)
        torch.cuda.synchronize()
    else:
        write(y, y)
    assert y._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_every_output_is_marked_and_no_input():
    x = torch.randn(3, 40, device="cuda")
    out = answer_of(x)
    at = [t._version for t in (x, *out)]
    P().hbsjd_top_logits_rows(x, 4, out=out)
    assert x._version == at[0] and all(t._version > v for t, v in zip(out, at[1:]))
    at = [t._version for t in (x, *out)]
    g = torch.empty_like(x)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    P().hbsjd_distill_top_rows(x, *out, grad=g, stream=s)
    P().hbsjd_adjust_rows(x, tokens=out[1], frequency=out[2], stream=s)
    s.synchronize()
    assert [t._version for t in (x, *out)] == at and g._version > 0


def test_results_are_no_part_of_the_graph():
    """Whether or not there is anything to adjust, no gradient reaches the logits."""
    x = torch.randn(3, 40, device="cuda", requires_grad=True)
    pen = dict(tokens=torch.zeros(3, dtype=torch.int32, device="cuda"),
               presence=torch.ones(3, device="cuda"))
    for kw in ({}, pen, dict(out_dtype=torch.float32), dict(out=torch.empty(3, 40, device="cuda"))):
        assert not P().hbsjd_adjust_rows(x, **kw).requires_grad
    y = P().hbsjd_adjust_rows(x)
    assert torch.equal(y, x) and y.data_ptr() == x.data_ptr()
    assert not any(t.requires_grad for t in P().hbsjd_top_logits_rows(x, 3))
    assert not any(t.requires_grad for t in P().hbsjd_distill_top_rows(x, *answer_of(x)))


def test_a_model_takes_its_gradient_in_the_logits_place():
    """The use that in-place gradients are for: the head's product keeps its inputs,
    not the logits."""
    gen = torch.Generator("cuda").manual_seed(2)
    h = torch.randn((5, 16), generator=gen, device="cuda")
    w = torch.randn((16, 70), generator=gen, device="cuda", requires_grad=True)
    answer = answer_of(h @ w)
    logits = h @ w
    _, g = P().hbsjd_distill_top_rows(logits, *answer)
    want = h.t().double() @ g.double()
    logits = h @ w
    P().hbsjd_distill_top_rows(logits, *answer, grad=logits)
    logits.backward(logits.detach())
    # a product of 5 terms in fp32
    bound = 8 * ref.U * (h.t().double().abs() @ g.double().abs())
    assert bool(((w.grad.double() - want).abs() <= bound + 2.0 ** -126).all())
