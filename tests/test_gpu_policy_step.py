"""Policy and preference steps as they are made: rollouts of the tiny model, the
log-probabilities under the weights that made them, the loss on the rows of a head
that is trained, its gradients, their norm and the clipped update."""
import numpy as np
import pytest

from tests import losses_ref as ref
from tests.row_operators_ref import U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def P():
    import paper_2608_18183_amd
    return paper_2608_18183_amd


@pytest.fixture
def rollout(tiny):
    import synth
    from tests import gpu_util as gu
    w, blob, _ = tiny
    ctx = gu.make_ctx(w.model, "f32", blob)
    batch = synth.make_batch(w, 1)
    out = ctx.hbsjd_rollout(gu.device_batch(batch), batch.prefix_len, batch.labels, batch.temperature,
                            w.window, history=w.history, seed=3)
    tokens, T = out["tokens"], w.model.grid ** 2
    lens = np.full(len(batch.prefix_len), T - 1, np.int32)
    logits = ctx.hbsjd_forward(tokens, lens, batch.labels).view(len(lens) * T, -1)
    target = tokens.clone()
    for b, k in enumerate(batch.prefix_len):
        target[b, :int(k)] = -1
    return logits, target.int().reshape(-1), len(lens), T


def test_policy_step_on_a_rollout(rollout):
    """A bias on the model's logits is trained. On the weights that drew the tokens the
    ratio is 1; the gradient is that of autograd in 64 bits; the update moves the loss's
    parameter by the clipped gradient."""
    logits, tok, images, T = rollout
    V = logits.shape[1]
    gen = torch.Generator("cuda").manual_seed(0)
    old, entropy, _ = P().hbsjd_logprob_rows(logits, tok, entropy=True)
    assert bool((old[tok < 0] == 0).all()) and bool((old[tok >= 0] < 0).all())
    adv = torch.randn(images, generator=gen, device="cuda").repeat_interleave(T)
    weight = torch.full((images * T,), 1.0 / int((tok >= 0).sum()), device="cuda")
    bias = torch.nn.Parameter(0.05 * torch.randn(V, generator=gen, device="cuda"))
    scale = torch.nn.Parameter(torch.ones(1, device="cuda"))
    z = logits * scale + bias
    loss, grad, lp, _ = P().hbsjd_policy_rows(z.detach(), tok, adv, old_logprob=old, ref_logprob=old,
                                              kl_weight=0.1, entropy_weight=0.01, row_weight=weight)
    z.backward(grad)
    z64 = z.detach().double().requires_grad_()
    lsm = torch.log_softmax(z64, 1)
    used = tok >= 0
    l = lsm.gather(1, tok.long().clamp(min=0)[:, None])[:, 0]
    rho = torch.exp(l - old.double())
    d = old.double() - l
    a = adv.double()
    low, high = 1 - float(np.float32(0.2)), 1 + float(np.float32(0.2))
    total = (-torch.minimum(rho * a, rho.clamp(low, high) * a) + float(np.float32(0.1)) * (torch.expm1(d) - d)
             + float(np.float32(0.01)) * (lsm.exp() * lsm).sum(1))
    total = torch.where(used, total * weight.double(), 0.0)
    want, = torch.autograd.grad(total.sum(), z64)
    q = [ref.Row(z.detach()[r].double().cpu().numpy(), int(tok[r]), 1.0) for r in range(0, images * T, 37)
         if tok[r] >= 0]
    # of a row's loss and gradient: the largest errors of the sampled rows' references,
    # with slopes of at most |a| 1.3 + 0.1 and 0.01, three times over for the rows between
    le = 3 * max(x.l_err + x.entropy_err for x in q) * (float(adv.abs().max()) * 1.3 + 0.2)
    wmax = float(weight.max())
    total = total.detach()
    assert float((loss.double() - total).abs().max()) <= wmax * le + 4 * U * float(total.abs().max())
    assert float((grad.double() - want).abs().max()) <= 2 * wmax * le + 8 * U * float(want.abs().max())
    grads = [bias.grad, scale.grad]
    before = [g.clone() for g in grads]
    norm64 = float(torch.cat(before).double().norm())
    limit = norm64 / 3
    norm = P().hbsjd_clip_grads(grads, limit)
    assert abs(float(norm) - norm64) <= 1.001 * U * norm64
    assert torch.equal(norm, P().hbsjd_grad_norm(before))
    for g, b in zip(grads, before):
        assert bool(((g - b / 3).abs() <= 6 * U * b.abs()).all())
    assert abs(float(P().hbsjd_grad_norm(grads)) - limit) <= 4 * U * limit


def test_preference_step_on_a_rollout(rollout):
    """Images as pairs; at the reference's weights the loss is log 2, the implied
    rewards are 0, and the two sequences' gradients are the log-probabilities' own."""
    logits, tok, images, T = rollout
    pairs = images // 2
    base, _, _ = P().hbsjd_logprob_rows(logits, tok)
    loss, grad, s = P().hbsjd_preference_rows(logits, tok, pairs=pairs, ref_logprob=base, beta=0.5)
    # the sums are of the roundings of base to fp32 alone
    n = (tok.view(images, T) >= 0).sum(1)
    assert bool((s.abs() <= n * U * float(base.abs().max()) * 1.01).all())
    slack = 0.25 * float(s.abs().max()) * 2 + 4 * U
    assert bool(((loss - np.log(2)).abs() <= slack).all())
    # -beta sigmoid(0), positive for the chosen
    sign = torch.tensor([-0.25, 0.25], device="cuda").repeat(pairs).repeat_interleave(T)
    _, _, want = P().hbsjd_logprob_rows(logits, tok, logprob_weight=sign, grad=True)
    assert bool(((grad - want).abs() <= (4 * U + slack) * want.abs() + 2.0 ** -126).all())
    # a step along the gradient's other way lowers no chosen sequence's share
    moved = logits - 0.5 * grad
    _, _, after = P().hbsjd_preference_rows(moved, tok, pairs=pairs, ref_logprob=base, beta=0.5, grad=False)
    assert bool((after.view(pairs, 2)[:, 0] > after.view(pairs, 2)[:, 1]).all())
    # packed as a list, without the rows that have no token
    keep = torch.nonzero(tok >= 0)[:, 0]
    first = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int64), n.cumsum(0)]).int()
    got = P().hbsjd_preference_rows(logits[keep].contiguous(), tok[keep].contiguous(), first=first,
                                    ref_logprob=base[keep].contiguous(), beta=0.5)
    # the same numbers added in another order in 64 bits, rounded once more
    assert bool(((got[0] - loss).abs() <= 2 * U).all())
    assert bool(((got[1] - grad[keep]).abs() <= 8 * U * grad[keep].abs() + 2.0 ** -126).all())
