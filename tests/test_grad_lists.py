"""How lists of tensors are described for the C calls: what they refuse, without a GPU."""
import pytest

torch = pytest.importorskip("torch")
import paper_2608_18183_amd.binding as B

B._load_torch()
CPU = torch.device("cpu")


@pytest.mark.parametrize("transform", ["vmap", "grad", "jvp"])
def test_tensors_without_an_address_are_refused(transform):
    """Tensors of a function transform have no memory that a kernel could be given."""
    def f(x):
        B._described([x, torch.ones(3)], "grads", CPU)
        return x.sum()
    x = torch.ones(2, 3)
    with pytest.raises(ValueError, match="grads"):
        if transform == "jvp":
            torch.func.jvp(f, (x,), (x,))
        else:
            getattr(torch.func, transform)(f)(x)


def test_lists_on_one_device_are_described():
    a, b = torch.ones(2, 3), torch.ones(4, dtype=torch.bfloat16)
    at, sizes, elems, flat = B._described([a, b, a.t()], "grads", CPU)
    assert list(at) == [a.data_ptr(), b.data_ptr(), a.data_ptr()] and list(sizes) == [6, 4, 6]
    assert list(elems) == [B.ELEM_F32, B.ELEM_BF16, B.ELEM_F32] and not flat
    for bad in (a[:, :2], a.double(), torch.ones(3, device="meta"), 1.0, None):
        with pytest.raises(ValueError, match="grads"):
            B._described([a, bad], "grads", CPU)
