"""What is no tensor, or no matrix, is refused as such, whichever argument it is."""
import pytest

from tests import test_gpu_row_operators as ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P = ops.P


@pytest.mark.parametrize("other_stream", [False, True])
@pytest.mark.parametrize("what", ["array", "list", "number", "scalar"])
def test_arguments_that_are_no_tensors(what, other_stream):
    x = torch.randn(4, 64, device="cuda")
    v, i, rest = P().hbsjd_top_logits_rows(x, 8)
    words = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    row = torch.zeros(4, dtype=torch.int32, device="cuda")
    not_it = {"array": lambda t: t.cpu().numpy(), "list": lambda t: t.tolist(),
              "number": lambda t: 3, "scalar": lambda t: t.reshape(-1)[0]}[what]
    stream = torch.cuda.Stream() if other_stream else None
    torch.cuda.synchronize()
    distill = dict(logits=x, values=v, index=i, rest=rest, row_weight=rest, grad=x.clone())
    adjust = dict(logits=x, tokens=i, token_count=row, repetition=rest, presence=rest, frequency=rest,
                  bias_index=i, bias_value=v, mask=words, mask_row=row, out=x.clone())
    for f, args in ((P().hbsjd_distill_top_rows, distill), (P().hbsjd_adjust_rows, adjust)):
        f(**args, stream=stream)
        for name in args:
            with pytest.raises(ValueError):
                f(**{**args, name: not_it(args[name])}, stream=stream)
    out = [v, i, rest]
    with pytest.raises(ValueError):
        P().hbsjd_top_logits_rows(not_it(x), 8, stream=stream)
    for j in range(3):
        bad = tuple(not_it(t) if n == j else t for n, t in enumerate(out))
        with pytest.raises(ValueError):
            P().hbsjd_top_logits_rows(x, 8, out=bad, stream=stream)
    torch.cuda.synchronize()


def test_a_refused_call_leaves_the_current_stream():
    """Refused for a tensor in host memory, on a stream that is not the current one."""
    x = torch.randn(4, 64, device="cuda")
    v, i, rest = out = P().hbsjd_top_logits_rows(x, 8)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = torch.cuda.current_stream()
    for f in (lambda: P().hbsjd_top_logits_rows(x, 8, out=(v, i.cpu(), rest), stream=s),
              lambda: P().hbsjd_distill_top_rows(x, v.cpu(), i, rest, stream=s),
              lambda: P().hbsjd_distill_top_rows(x, v, i, rest, grad=x.cpu(), stream=s),
              lambda: P().hbsjd_adjust_rows(x, tokens=i.cpu(), frequency=rest, stream=s)):
        with pytest.raises(ValueError):
            f()
        assert torch.cuda.current_stream() == before
    assert all(a.data_ptr() == b.data_ptr() for a, b in
               zip(P().hbsjd_top_logits_rows(x, 8, out=out, stream=s), out))
    assert torch.cuda.current_stream() == before
    torch.cuda.synchronize()
