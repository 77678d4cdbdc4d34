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


def test_outputs_laid_out_alike():
    """Strides of dimensions of one entry say nothing about where entries lie, and of two
    contiguous tensors only the number of entries counts, beside others too."""
    turned = torch.ones(4, 3).t()
    odd = torch.ones(5).as_strided((1, 5), (1, 1))
    pairs = [(turned, torch.empty_like(turned)), (odd, torch.empty(1, 5)), (torch.ones(2, 3), torch.ones(6)),
             (torch.ones(5, 1, 2).permute(2, 1, 0), torch.ones(5, 2).t().unsqueeze(1)),
             (torch.ones(0, 3), torch.ones(3, 0).t()), (torch.ones(()), torch.ones(1))]
    assert odd.stride() != pairs[1][1].stride() and pairs[3][0].stride() != pairs[3][1].stride()
    for g, o in pairs:
        assert B._alike(g, o) and B._alike(o, g)
    for g, o in ((turned, turned.contiguous()), (turned, torch.ones(3, 4)), (turned, torch.ones(4, 3)),
                 (turned, torch.ones(2, 6).t()), (torch.ones(3, 4, 2).permute(2, 1, 0), torch.ones(3, 4, 2).permute(2, 0, 1))):
        assert not B._alike(g, o) and not B._alike(o, g)


@pytest.mark.gpu
def test_clips_into_outputs_laid_out_alike():
    import paper_2608_18183_amd as P
    turned = torch.randn(40, 30, device="cuda").t()
    odd = torch.randn(50, device="cuda").as_strided((1, 50), (1, 1))
    grads, out = [turned, odd], [torch.empty_like(turned), torch.empty(1, 50, device="cuda")]
    norm = float(P.hbsjd_clip_grads(grads, 1.0, out=out))
    for g, o in zip(grads, out):   # two roundings of the product, one of the norm
        assert bool(((o.double() - g.double() / norm).abs() <= 4 * 2.0 ** -24 * g.double().abs() / norm).all())
