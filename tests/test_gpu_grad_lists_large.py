"""Norm and clipping of a dense list of more than 256 MB, which the kernels read and write in
part past the caches and describe in several launches, against 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
from tests.test_gpu_grad_norm import P, TYPES, around, check_norm, check_scaled

pytestmark = pytest.mark.gpu

COUNT = 420


def tensors(seed, offset):
    """Tensors of all types, 300 MB together, `offset` entries behind an aligned address."""
    gen = torch.Generator("cuda").manual_seed(seed)
    grads, bufs = [], []
    for i in range(COUNT):
        n = 240_000 + i * 7919 % 60_000
        buf = torch.full((n + offset + 40,), 7.0, dtype=list(TYPES.values())[i % 3], device="cuda")
        buf[offset:offset + n] = torch.randn(n, generator=gen, device="cuda").clamp_(-6, 6)
        bufs.append(buf)
        grads.append(buf[offset:offset + n])
    return grads, bufs


def norm64(grads):
    return math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))


@pytest.mark.parametrize("offset", [0, 3])
def test_norm(offset):
    grads, _ = tensors(1 + offset, offset)
    assert sum(g.numel() * g.element_size() for g in grads) > 256 << 20
    check_norm(P().hbsjd_grad_norm(grads), norm64(grads))
    # one entry that counts, in units from the first to the last
    for i in (0, COUNT // 3, COUNT // 2, COUNT - 1):
        for at in (0, grads[i].numel() // 2, -1):
            keep = float(grads[i][at])
            grads[i][at] = -8.0 - i
            assert float(P().hbsjd_grad_norm(grads, order=math.inf)) == float(grads[i][at].abs())
            grads[i][at] = keep


@pytest.mark.parametrize("offset,to", [(0, 0), (3, 3), (0, 2), (1, 0)])
def test_clip_into_others_and_in_place(offset, to):
    grads, bufs = tensors(5, offset)
    out, obufs = tensors(6, to)
    want = norm64(grads)
    limit = 0.25 * want
    scale = float(torch.tensor(limit, dtype=torch.float32)) / want
    before = [g.clone() for g in grads]
    check_norm(P().hbsjd_clip_grads(grads, 2 * want, out=out), want)
    assert all(torch.equal(o, g) for o, g in zip(out, before))
    check_norm(P().hbsjd_clip_grads(grads, limit, out=out), want)
    for o, buf, g in zip(out, obufs, before):
        check_scaled(o, g, scale)
        assert around(buf, o)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    check_norm(P().hbsjd_clip_grads(grads, limit), want)
    for o, buf, g in zip(grads, bufs, out):
        assert torch.equal(o, g) and around(buf, o)
