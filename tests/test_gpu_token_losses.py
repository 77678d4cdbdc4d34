"""Tokens' log-probabilities, the policy and the preference loss against their 64-bit
references, within the bounds that tests/losses_ref.py derives."""
import math

import numpy as np
import pytest

from tests import losses_ref as ref
from tests.row_operators_ref import U
from tests import test_gpu_row_operators as ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P, dev, placed, untouched, rows_of, TYPES, SIZES = (
    ops.P, ops.dev, ops.placed, ops.untouched, ops.rows_of, ops.TYPES, ops.SIZES)


def within(got, want, bound, what):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    off = np.abs(got - want) - bound
    assert np.all(off <= 0), (what, int(np.argmax(off)), np.max(off), np.max(bound))


def tokens_of(rng, x64, unused=True):
    """Tokens of every kind: the likeliest, the first, the last, any; the row's own
    finite ones; row 1 left out."""
    n, V = x64.shape
    t = rng.integers(0, V, n)
    t[0] = x64[0].argmax()
    t[n - 1] = V - 1
    for r in range(n):
        if x64[r, t[r]] == -np.inf:
            t[r] = x64[r].argmax()
    if unused and n > 2:
        t[1] = -1
    return t.astype(np.int32)


def check_l(got, q, what):
    if abs(q.l) >= 2.0 ** 128 * (1 - 2.0 ** -25):   # past fp32's numbers the nearest is an infinity
        assert float(got) == -np.inf, what
    else:
        within(np.array(float(got)), q.l, q.l_err, what)


def check_logprob(x64, tokens, tau, a, b, out, dtype):
    l, entropy, grad = out
    grad = None if grad is None else grad.double().cpu().numpy()
    for r in range(len(tokens)):
        if tokens[r] == -1:
            assert float(l[r]) == 0 and (entropy is None or float(entropy[r]) == 0)
            assert grad is None or (grad[r] == 0).all()
            continue
        q = ref.Row(x64[r], tokens[r], tau)
        check_l(l[r], q, ("l", r))
        if entropy is not None:
            within(np.array(float(entropy[r])), q.entropy, q.entropy_err, ("entropy", r))
        if grad is not None:
            g, bound = q.gradient(0.0 if a is None else float(a[r]), 0.0 if b is None else float(b[r]),
                                  0.0, dtype)
            within(grad[r], g, bound, ("grad", r))


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", SIZES)
def test_logprob(V, dtype, layout):
    rng = np.random.default_rng(V)
    n = 4
    for kind in ("noise", "masked", "lowest"):
        t, x64 = rows_of(rng, n, V, dtype, kind)
        x, _ = placed(t.cuda(), layout)
        tok = tokens_of(rng, x64)
        tau = float(rng.choice([0.5, 1.0, 3.0]))
        a, b = (rng.normal(0, 1, n).astype(np.float32) for _ in range(2))
        out = P().hbsjd_logprob_rows(x, dev(tok), temperature=tau, entropy=True)
        check_logprob(x64, tok, tau, a, b, out, dtype)
        assert P().hbsjd_logprob_rows(x, dev(tok), temperature=tau)[1:] == (None, None)
        for wa, wb in ((a, None), (None, b), (a, b)):
            grad, buf = placed(torch.full((n, V), 3.0, dtype=TYPES[dtype], device="cuda"), layout)
            out = P().hbsjd_logprob_rows(
                x, dev(tok), temperature=tau, entropy=wb is not None, grad=grad,
                logprob_weight=None if wa is None else dev(wa),
                entropy_weight=None if wb is None else dev(wb))
            assert out[2] is grad
            check_logprob(x64, tok, tau, wa, wb, out, dtype)
            assert buf is None or untouched(buf, grad)


@pytest.mark.parametrize("V", [1, 64, 16384, 33001])
def test_logprob_of_certain_tokens_keeps_its_digits(V):
    """l next to 0 and the gradient at the token are relative to their own size."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 1, (4, V)).astype(np.float32)
    tok = rng.integers(0, V, 4).astype(np.int32)
    for r, lead in enumerate((5, 20, 40, 300)):
        x[r, tok[r]] += lead + 5
    one = np.ones(4, np.float32)
    out = P().hbsjd_logprob_rows(dev(x), dev(tok), entropy=True, logprob_weight=dev(one), grad=True)
    check_logprob(x.astype(np.float64), tok, 1.0, one, None, out, "f32")


@pytest.mark.parametrize("tau", [1e-6, 1e-3, 1e3, 1e6])
@pytest.mark.parametrize("size", [1e-6, 1.0, 1e30])
def test_logprob_at_any_temperature_and_size(tau, size):
    rng = np.random.default_rng(2)
    for V in (100, 20000):
        x = (rng.normal(0, 1, (4, V)) * size * tau).astype(np.float32)
        tok = x.argmax(1).astype(np.int32)
        tok[2:] = rng.integers(0, V, 2)
        tau32 = float(np.float32(tau))
        a = np.array([1.0, -1.0, 2.0, 0.5], np.float32)
        out = P().hbsjd_logprob_rows(dev(x), dev(tok), temperature=tau, entropy=True,
                                     logprob_weight=dev(a), entropy_weight=dev(a), grad=True)
        l, entropy, grad = (t.double().cpu().numpy() for t in out)
        for r in range(4):
            q = ref.Row(x[r].astype(np.float64), tok[r], tau32)
            check_l(l[r], q, ("l", r))
            within(entropy[r], q.entropy, q.entropy_err, ("entropy", r))
            g, bound = q.gradient(a[r], a[r], 0.0, "f32")
            within(grad[r], g, bound, ("grad", r))


def bad_rows(rng, V):
    """Rows of every kind of error, and which of them are sound."""
    n = 10
    x = rng.normal(0, 2, (n, V)).astype(np.float32)
    tok = rng.integers(0, V, n).astype(np.int32)
    x[1] = np.nan
    tok[1] = -1                       # left out: not read
    x[2] = -np.inf                    # a mask that leaves nothing
    x[3, V // 2] = np.nan
    x[4, V - 1] = np.inf
    tok[5], tok[6] = V, -2            # no such entries
    x[7, tok[7]] = np.nan
    x[8] = -np.inf                    # one entry left, the token
    x[8, tok[8]] = 3.0
    return x, tok, [0, 8, 9]


@pytest.mark.parametrize("V", [2, 96, 4099, 16384, 70000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_in_error_stay_alone(V, dtype):
    rng = np.random.default_rng(V)
    x, tok, sound = bad_rows(rng, V)
    t = torch.from_numpy(x).to(TYPES[dtype])
    x64 = t.double().numpy()
    one = np.ones(len(tok), np.float32)
    l, entropy, grad = P().hbsjd_logprob_rows(t.cuda(), dev(tok), entropy=True, grad=True,
                                              logprob_weight=dev(one), entropy_weight=dev(one))
    loss, pgrad, pl, pe = P().hbsjd_policy_rows(t.cuda(), dev(tok), dev(one), entropy=True)
    for o in (l, entropy, grad, loss, pgrad, pl, pe):
        assert bool((o[1] == 0).all())
        for r in (2, 3, 4, 5, 6, 7):
            assert bool(torch.isnan(o[r]).all()), r
    assert float(l[8]) == 0 and float(entropy[8]) == 0 and bool((grad[8] == 0).all())
    check_logprob(x64[sound], tok[sound], 1.0, one, one,
                  (l[sound], entropy[sound], grad[sound]), dtype)


@pytest.mark.parametrize("V", [50, 40000])
def test_a_token_that_the_mask_bars(V):
    """l is -infinity, its gradient that of the formula; a policy loss is what is
    left of it, or without an end and without a gradient."""
    x = np.random.default_rng(V).normal(0, 1, (3, V)).astype(np.float32)
    x[:, 7] = -np.inf
    tok = np.full(3, 7, np.int32)
    one = np.ones(3, np.float32)
    l, entropy, grad = P().hbsjd_logprob_rows(dev(x), dev(tok), entropy=True, grad=True,
                                              logprob_weight=dev(one))
    assert bool((l == -np.inf).all()) and bool(torch.isfinite(entropy).all())
    for r in range(3):
        q = ref.Row(x[r].astype(np.float64), 7, 1.0)
        g, bound = q.gradient(1.0, 0.0, 0.0, "f32")
        within(grad[r], g, bound, r)
    old = dev(np.full(3, -4.0, np.float32))
    adv = dev(np.array([1.0, -1.0, 0.0], np.float32))
    loss, grad, _, _ = P().hbsjd_policy_rows(dev(x), dev(tok), adv, old_logprob=old)
    # the ratio is 0: nothing for a gain, the lower bound for a loss
    assert loss.tolist() == [0.0, float(np.float32(1 - float(np.float32(0.2)))), 0.0]
    assert bool((grad == 0).all())
    loss, grad, _, _ = P().hbsjd_policy_rows(dev(x), dev(tok), adv, old_logprob=old, ref_logprob=old,
                                             kl_weight=0.1)
    assert bool((loss == np.inf).all()) and bool(torch.isnan(grad).all())


# ------------------------------------------------------------------ policy

def policy_case(rng, n, V, dtype, layout="plain", kl=0.0, bonus=0.0, old=True, low=0.2, high=0.3,
                weights=True, tau=1.0, kind="noise"):
    t, x64 = rows_of(rng, n, V, dtype, kind)
    x, _ = placed(t.cuda(), layout)
    tok = tokens_of(rng, x64)
    for r in range(n):
        if tok[r] >= 0 and x64[r, tok[r]] < -1e4:     # a token that could have been drawn
            tok[r] = x64[r].argmax()
    rows = [ref.Row(x64[r], tok[r], tau) if tok[r] >= 0 else None for r in range(n)]
    l = np.array([q.l if q else 0.0 for q in rows])
    # inside the bounds, beyond either, none within 1e-3 of one
    shift = np.array([0.0, 0.1, -0.1, 0.7, -0.7])[rng.integers(0, 5, n)] + rng.uniform(-0.03, 0.03, n)
    old_l = (l - shift).astype(np.float32)
    ref_l = (l + rng.normal(0, 0.5, n)).astype(np.float32)
    adv = rng.normal(0, 1, n).astype(np.float32)
    adv[-1] = 0.0
    w = rng.uniform(0.5, 2, n).astype(np.float32)
    w[n // 2] = 0.0
    grad, buf = placed(torch.full((n, V), 3.0, dtype=TYPES[dtype], device="cuda"), layout)
    args = (x, dev(tok), dev(adv))
    kw = dict(old_logprob=dev(old_l) if old else None, ref_logprob=dev(ref_l) if kl else None,
              temperature=tau, clip_low=low, clip_high=high, kl_weight=kl, entropy_weight=bonus,
              row_weight=dev(w) if weights else None)
    out = P().hbsjd_policy_rows(*args, **kw, grad=grad)
    low, high, kl, bonus = (float(np.float32(v)) for v in (low, high, kl, bonus))
    loss, g, lp, entropy = (None if o is None else o.double().cpu().numpy() for o in out)
    assert (entropy is None) == (not bonus)
    for r, q in enumerate(rows):
        wr = float(w[r]) if weights else 1.0
        if q is None or wr == 0.0:
            assert loss[r] == 0 and lp[r] == 0 and (g[r] == 0).all()
            continue
        want, err, gl, h, g_err = ref.policy(q, float(adv[r]), float(old_l[r]) if old else None,
                                             float(ref_l[r]), low, high, kl, bonus, wr)
        within(loss[r], want, err, ("loss", r))
        within(lp[r], q.l, q.l_err, ("l", r))
        if entropy is not None:
            within(entropy[r], q.entropy, q.entropy_err, ("entropy", r))
        wg, bound = q.gradient(gl, h, g_err, dtype)
        within(g[r], wg, bound, ("grad", r))
    assert buf is None or untouched(buf, grad)
    return args, kw, out


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", SIZES)
def test_policy(V, dtype, layout):
    rng = np.random.default_rng(V + 1)
    policy_case(rng, 8, V, dtype, layout)
    policy_case(rng, 8, V, dtype, layout, kl=0.2, bonus=0.05, tau=0.7 if V % 2 else 2.0)


@pytest.mark.parametrize("form", [dict(old=False), dict(old=False, kl=0.5), dict(low=1.0, high=0.0),
                                  dict(low=0.0, high=1e6), dict(weights=False, bonus=0.3), dict(kind="masked"),
                                  dict(kind="lowest", kl=0.1, bonus=0.1), dict(kl=100.0)])
def test_policy_forms(form):
    rng = np.random.default_rng(5)
    for V in (300, 16384, 40000):
        policy_case(rng, 12, V, "f32", **form)


@pytest.mark.parametrize("V", [100, 5003, 16384, 70000])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_policy_in_place_and_loss_alone(V, dtype):
    args, kw, (loss, grad, lp, entropy) = policy_case(np.random.default_rng(V), 6, V, dtype, kl=0.1, bonus=0.1)
    out = P().hbsjd_policy_rows(*args, **kw, grad=False)
    assert out[1] is None and all(torch.equal(a, b) for a, b in zip(
        (out[0], out[2], out[3]), (loss, lp, entropy)))
    x = args[0].clone()
    out = P().hbsjd_policy_rows(x, *args[1:], **kw, grad=x)
    assert out[1] is x and torch.equal(x, grad) and torch.equal(out[0], loss)
    # the same through its parts: l's and H's gradients with the loss's slopes as weights
    kw.update(kl_weight=0.0, entropy_weight=0.0, old_logprob=None, ref_logprob=None)
    loss, grad, lp, _ = P().hbsjd_policy_rows(*args, **kw)
    w = kw["row_weight"]
    l, _, g = P().hbsjd_logprob_rows(args[0], args[1], logprob_weight=-args[2] * w, grad=True)
    assert torch.equal(torch.where(w == 0, 0, l), lp)
    # the weight here is a product rounded to fp32, there it is formed in 64 bits: half a
    # step of the slope, as much again of each of the two factors made of it, and the
    # gradient's own roundings, the last one to its type
    step, least = ref.ROUND[dtype]
    assert bool(((g - grad).double().abs() <= (5 * U + 2 * step) * grad.double().abs() + 2 * least).all())


def test_policy_ratio_overflows_and_infinite_inputs():
    """Ratios past every number: bounded for a gain; without an end, and without a
    gradient, for a loss. NaN among a row's numbers stays in the row."""
    x = np.random.default_rng(3).normal(0, 1, (6, 100)).astype(np.float32)
    tok = np.full(6, 3, np.int32)
    adv = np.array([1, -1, 0, 1, np.nan, 1], np.float32)
    old = np.array([-np.inf, -np.inf, -np.inf, -2000, -3, np.nan], np.float32)
    loss, grad, lp, _ = P().hbsjd_policy_rows(dev(x), dev(tok), dev(adv), old_logprob=dev(old))
    up = -float(np.float32(1 + float(np.float32(0.2))))
    lo = loss.cpu().numpy()
    assert lo[0] == lo[3] == up and lo[1] == np.inf and lo[2] == 0
    assert np.isnan(lo[4:]).all()
    g = grad.cpu().numpy()
    assert (g[[0, 2, 3]] == 0).all() and np.isnan(g[[1, 4, 5]]).all()
    assert bool(torch.isfinite(lp).all())


def test_policy_gradient_equals_differences_of_its_loss():
    rng = np.random.default_rng(10)
    V, tok = 260, 31
    x = rng.normal(0, 1.5, (1, V)).astype(np.float32)
    q = ref.Row(x[0].astype(np.float64), tok, 1.0)
    h = 2.0 ** -6
    probes = np.array([tok, int(x.argmax()), 0, 1, 100, 259])
    moved = np.repeat(x, 2 * probes.size, 0)
    for j, v in enumerate(probes):
        moved[2 * j, v] += np.float32(h)
        moved[2 * j + 1, v] -= np.float32(h)
    rep = lambda v, n: dev(np.full(n, v, np.float32))

    def run(rows):
        n = rows.shape[0]
        return P().hbsjd_policy_rows(dev(rows), dev(np.full(n, tok, np.int32)), rep(-0.7, n),
                                     old_logprob=rep(q.l - 0.05, n), ref_logprob=rep(q.l + 0.3, n),
                                     kl_weight=0.2, entropy_weight=0.1)
    loss = run(moved)[0].double().cpu().numpy()
    got = run(x)[1][0].double().cpu().numpy()[probes]
    step = (moved[0::2, probes].diagonal().astype(np.float64)
            - moved[1::2, probes].diagonal().astype(np.float64))
    d = (loss[0::2] - loss[1::2]) / step
    el = ref.policy(q, -0.7, q.l - 0.05, q.l + 0.3, kl=0.2, bonus=0.1)[1]
    # two losses' errors over the step, and h^2 / 6 times a third derivative: l's is at
    # most 1, H's below 8 for these rows, each times slopes of about 1 and 0.1
    assert np.abs(d - got).max() <= 2 * el / (2 * h) * 1.1 + h * h / 6 * 4


# ------------------------------------------------------------------ preference

def preference_case(rng, lengths, V, dtype, layout="plain", packed=True, ahead=0, behind=0, form="sigmoid",
                    mean=False, smoothing=0.0, margin=0.0, beta=0.1, base=True, weights=True, tau=1.0,
                    kind="noise"):
    pairs = len(lengths) // 2
    ends = np.concatenate([[0], np.cumsum(lengths)]) + ahead
    rows = int(ends[-1]) + behind
    t, x64 = rows_of(rng, rows, V, dtype, kind)
    x, _ = placed(t.cuda(), layout)
    tok = rng.integers(0, V, rows).astype(np.int32)
    for r in range(rows):
        if x64[r, tok[r]] < -1e4:
            tok[r] = x64[r].argmax()
    tok[rng.random(rows) < 0.25] = -1
    l = np.array([ref.Row(x64[r], tok[r], tau).l if tok[r] >= 0 else 0 for r in range(rows)])
    r_l = (l + rng.normal(0, 0.5, rows)).astype(np.float32)
    w = rng.uniform(0.5, 2, pairs).astype(np.float32)
    if pairs > 2:
        w[1] = 0.0
    grad, buf = placed(torch.full((rows, V), 3.0, dtype=TYPES[dtype], device="cuda"), layout)
    args = (x, dev(tok))
    kw = dict(ref_logprob=dev(r_l) if base else None, temperature=tau, beta=beta, form=form, mean=mean,
              smoothing=smoothing, margin=margin, pair_weight=dev(w) if weights else None)
    kw.update(first=dev(ends.astype(np.int32))) if packed else kw.update(pairs=pairs)
    out = P().hbsjd_preference_rows(*args, **kw, grad=grad)
    loss, g, s = (o.double().cpu().numpy() for o in out)
    beta, margin, smoothing = (float(np.float32(v)) for v in (beta, margin, smoothing))
    seen = set()
    for i in range(pairs):
        wi = float(w[i]) if weights else 1.0
        (want, err), ws, s_err, grads = ref.preference(
            x64, tok, ends[2 * i:2 * i + 3], r_l.astype(np.float64) if base else None, tau, form, beta, mean,
            smoothing, margin, wi, dtype)
        within(loss[i], want, err, ("loss", i))
        within(s[2 * i:2 * i + 2], np.array(ws), np.array(s_err), ("log_ratio", i))
        for r, (wg, bound) in grads.items():
            within(g[r], wg, bound, ("grad", r))
        seen.update(grads if wi else ())
    for r in set(range(rows)) - seen:     # left out
        assert (g[r] == 0).all(), r
    assert buf is None or untouched(buf, grad)
    return args, kw, out


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", SIZES)
def test_preference(V, dtype, layout):
    rng = np.random.default_rng(V + 2)
    few = V > 40000
    preference_case(rng, [2, 1] if few else [3, 5, 1, 4, 0, 2], V, dtype, layout, ahead=1, behind=2,
                    beta=0.3, tau=0.7 if V % 2 else 2.0)
    preference_case(rng, [2, 2] if few else [3] * 6, V, dtype, layout, packed=False, form="square", mean=True,
                    beta=0.8)


@pytest.mark.parametrize("form", [
    dict(smoothing=0.2), dict(form="hinge"), dict(form="hinge", beta=20.0), dict(form="square", beta=0.5),
    dict(margin=0.7), dict(base=False, mean=True, beta=2.0, margin=0.25), dict(weights=False),
    dict(kind="masked"), dict(kind="lowest"), dict(beta=30.0)])
def test_preference_forms(form):
    rng = np.random.default_rng(6)
    for V in (70, 9000):
        preference_case(rng, [4, 7, 1, 1, 0, 3, 0, 0], V, "f32", **form)


def test_preference_of_long_sequences():
    """Sequences longer than the workgroup that adds them up."""
    preference_case(np.random.default_rng(7), [1500, 1100], 33, "f32", beta=0.01)
    preference_case(np.random.default_rng(8), [2, 2500, 1, 1], 40, "bf16", mean=True, beta=1.0)
    preference_case(np.random.default_rng(9), [1, 2500], 40, "f16", ahead=3, behind=7, mean=True, beta=1.0)
    preference_case(np.random.default_rng(10), [1050, 1010], 17001, "bf16", beta=0.05)


@pytest.mark.parametrize("V", [100, 5003, 16384, 70000])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_preference_in_place_and_loss_alone(V, dtype):
    args, kw, (loss, grad, s) = preference_case(np.random.default_rng(V), [3, 2, 1, 1], V, dtype)
    out = P().hbsjd_preference_rows(*args, **kw, grad=False)
    assert out[1] is None and torch.equal(out[0], loss) and torch.equal(out[2], s)
    x = args[0].clone()
    out = P().hbsjd_preference_rows(x, args[1], **kw, grad=x)
    assert out[1] is x and torch.equal(x, grad) and torch.equal(out[0], loss)


@pytest.mark.parametrize("V", [96, 20000])
def test_preference_errors_stay_in_their_pair(V):
    rng = np.random.default_rng(V)
    pairs, n = 10, 3
    x = rng.normal(0, 2, (2 * pairs * n, V)).astype(np.float32)
    tok = rng.integers(0, V, 2 * pairs * n).astype(np.int32)
    at = lambda pair, seq, r: (2 * pair + seq) * n + r
    w = np.ones(pairs, np.float32)
    x[at(1, 0, 1), 5] = np.nan
    x[at(2, 1, 2)] = -np.inf
    tok[at(3, 0, 0)] = V
    x[at(4, 1, 0), 3] = np.inf
    tok[at(5, 0, 0):at(6, 0, 0)] = -1                # no tokens at all
    x[at(5, 0, 0):at(6, 0, 0)] = np.nan              # and rows that are not read
    x[at(6, 0, 2), tok[at(6, 0, 2)]] = -np.inf       # a chosen token without a probability
    x[at(7, 1, 1), tok[at(7, 1, 1)]] = -np.inf       # a rejected one: nothing left to gain
    w[8] = 0.0
    x[at(8, 0, 0), 2] = np.nan                       # weighted out
    loss, grad, s = P().hbsjd_preference_rows(dev(x), dev(tok), pairs=pairs, pair_weight=dev(w))
    lo, g = loss.cpu().numpy(), grad.view(pairs, -1).cpu().numpy()
    for i in (1, 2, 3, 4):
        assert np.isnan(lo[i]) and np.isnan(g[i]).all(), i
    assert math.isclose(lo[5], math.log(2), rel_tol=1e-6) and (g[5] == 0).all()
    assert lo[6] == np.inf and np.isnan(g[6]).all()
    assert lo[7] == 0 and (g[7] == 0).all()
    assert lo[8] == 0 and (g[8] == 0).all()
    x64 = x.astype(np.float64)
    for i in (0, 9):
        (want, err), _, _, grads = ref.preference(x64, tok, [at(i, 0, 0), at(i, 1, 0), at(i, 1, 0) + n], None, 1.0,
                                                  "sigmoid", float(np.float32(0.1)))
        within(lo[i], want, err, i)
        for r, (wg, bound) in grads.items():
            within(grad[r], wg, bound, r)


def test_preference_offsets_out_of_order_or_range():
    """Their pairs have no loss, and nothing outside the buffers is touched."""
    rng = np.random.default_rng(1)
    x = rng.normal(0, 1, (12, 50)).astype(np.float32)
    tok = rng.integers(0, 50, 12).astype(np.int32)
    big = 2 ** 31 - 1
    sound = P().hbsjd_preference_rows(dev(x), dev(tok), first=dev(np.array([0, 2, 4, 7, 12], np.int32)))
    for first, bad in (([0, 2, 4, 7, 13], [1]), ([0, 2, 4, 7, big], [1]), ([-5, 2, 4, 7, 12], [0]),
                       ([0, 4, 2, 7, 12], [0]), ([0, 2, 4, 3, 12], [1]), ([-big, big, -big, big, -1], [0, 1]),
                       ([12, 11, 10, 9, 8], [0, 1])):
        loss, grad, _ = P().hbsjd_preference_rows(dev(x), dev(tok), first=dev(np.array(first, np.int32)))
        for i in range(2):
            if i in bad:
                assert bool(torch.isnan(loss[i])), first
            elif first[2 * i:2 * i + 3] == [0, 2, 4, 7, 12][2 * i:2 * i + 3]:
                assert torch.equal(loss[i], sound[0][i])
        torch.cuda.synchronize()


def test_no_rows_and_no_pairs():
    x = torch.zeros(0, 64, device="cuda")
    i, f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    l, _, g = P().hbsjd_logprob_rows(x, i, logprob_weight=f, grad=True)
    assert l.shape == (0,) and g.shape == (0, 64)
    assert P().hbsjd_policy_rows(x, i, f)[1].shape == (0, 64)
    assert P().hbsjd_preference_rows(x, i, pairs=0)[0].shape == (0,)
    # two empty sequences are a pair all the same
    loss, _, s = P().hbsjd_preference_rows(x, i, pairs=1)
    assert math.isclose(float(loss[0]), math.log(2), rel_tol=1e-6) and s.tolist() == [0.0, 0.0]
    x = torch.randn(5, 64, device="cuda")
    i = torch.zeros(5, dtype=torch.int32, device="cuda")
    none, g, _ = P().hbsjd_preference_rows(x, i, first=i[:1])
    assert none.shape == (0,) and bool((g == 0).all())


def test_gradients_equal_differences_of_what_they_belong_to():
    """Log-probability, entropy, and the preference loss by a chosen and a rejected row."""
    rng = np.random.default_rng(12)
    V, tok = 260, 31
    x = rng.normal(0, 1.5, (1, V)).astype(np.float32)
    other = rng.normal(0, 1.5, (1, V)).astype(np.float32)
    h = 2.0 ** -6
    probes = np.array([tok, int(x.argmax()), 0, 1, 100, 259])
    moved = np.repeat(x, 2 * probes.size, 0)
    for j, v in enumerate(probes):
        moved[2 * j, v] += np.float32(h)
        moved[2 * j + 1, v] -= np.float32(h)
    step = (moved[0::2, probes].diagonal().astype(np.float64)
            - moved[1::2, probes].diagonal().astype(np.float64))
    q = ref.Row(x[0].astype(np.float64), tok, 1.0)
    one = dev(np.ones(1, np.float32))

    def logprob(rows):
        return P().hbsjd_logprob_rows(dev(rows), dev(np.full(len(rows), tok, np.int32)), entropy=True)

    def preference(rows, which):
        """The loss of pairs of `rows` and the other row, and the gradient by the former."""
        z = np.repeat(other, 2 * len(rows), 0)
        z[which::2] = rows
        loss, grad, _ = P().hbsjd_preference_rows(dev(z), dev(np.full(len(z), tok, np.int32)), pairs=len(rows),
                                                  beta=0.7)
        return loss, grad[which::2]

    at = dev(np.full(1, tok, np.int32))
    cases = [(logprob(moved)[0], P().hbsjd_logprob_rows(dev(x), at, logprob_weight=one, grad=True)[2], q.l_err),
             (logprob(moved)[1], P().hbsjd_logprob_rows(dev(x), at, entropy_weight=one, grad=True)[2],
              q.entropy_err)]
    both = q.l_err + ref.Row(other[0].astype(np.float64), tok, 1.0).l_err
    for which in (0, 1):
        cases.append((preference(moved, which)[0], preference(x, which)[1], both + 2 * U))
    for value, grad, err in cases:
        f = value.double().cpu().numpy()
        d = (f[0::2] - f[1::2]) / step
        got = grad[0].double().cpu().numpy()[probes]
        # two values' errors over the step, and h^2 / 6 times a third derivative: l's is at
        # most 1, H's and the loss's below 8 for these rows
        assert np.abs(d - got).max() <= 2 * err / (2 * h) * 1.1 + h * h / 6 * 8


# ------------------------------------------------------------------ as calls

def all_three(x, tok, f, stream=None):
    """Log-probabilities and their gradient, and both losses on the same rows."""
    l, e, g = P().hbsjd_logprob_rows(x, tok, entropy=True, logprob_weight=f, entropy_weight=f, grad=True,
                                     stream=stream)
    loss, pg, _, _ = P().hbsjd_policy_rows(x, tok, f, old_logprob=l, ref_logprob=l, kl_weight=0.1,
                                           entropy_weight=0.1, stream=stream)
    d, dg, s = P().hbsjd_preference_rows(x, tok, pairs=x.shape[0] // 2, ref_logprob=e, stream=stream)
    return [l, e, g, loss, pg, d, dg, s]


def inputs(gen, n, V):
    return (torch.randn((n, V), generator=gen, device="cuda"),
            torch.randint(-1, V, (n,), generator=gen, device="cuda").int(),
            torch.randn(n, generator=gen, device="cuda"))


@pytest.mark.parametrize("V", [600, 16384, 50001])
def test_captured_and_replayed(V):
    """Two graphs of the calls, replayed in turn with the eager calls on other data
    between the replays, give the eager calls' results each time."""
    gen = torch.Generator("cuda").manual_seed(V)
    data = [inputs(gen, 6, V) for _ in range(2)]
    all_three(*data[0])
    torch.cuda.synchronize()
    graphs = []
    for j in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = all_three(*data[j])
        graphs.append((g, out))
    for rep in range(4):
        for j in range(2):
            for old, new in zip(data[j], inputs(gen, 6, V)):
                old.copy_(new)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for j in range(2):
            want = all_three(*data[j])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(graphs[j][1], want)), (rep, j)


def test_other_streams_and_threads():
    import threading
    gen = torch.Generator("cuda").manual_seed(5)
    data = inputs(gen, 50, 20000)
    want = all_three(*data)
    torch.cuda.synchronize()
    wrong = []

    def work(j):
        s = torch.cuda.Stream()
        for _ in range(5):
            got = all_three(*data, stream=s if j % 2 else s.cuda_stream)
            s.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)):
                wrong.append(j)

    threads = [threading.Thread(target=work, args=(j,)) for j in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@pytest.mark.parametrize("V", [500, 20000])
def test_offsets_past_32_bits(V):
    """Rows 1.2e9 entries apart: the third starts past 2^31 entries and 2^32 bytes."""
    rng = np.random.default_rng(13)
    n, ld = 4, 1_200_000_007
    t, x64 = rows_of(rng, n, V, "bf16")
    buf = torch.empty(3 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (n, V), (ld, 1))
    tok = tokens_of(rng, x64, unused=False)
    a = np.ones(n, np.float32)
    x.copy_(t)
    loss, grad, _ = P().hbsjd_preference_rows(x, dev(tok), pairs=2, grad=x)
    for i in range(2):
        (want, err), _, _, grads = ref.preference(x64, tok, [2 * i, 2 * i + 1, 2 * i + 2], None, 1.0, "sigmoid",
                                                  float(np.float32(0.1)), dtype="bf16")
        within(np.array(float(loss[i])), want, err, i)
        for r, (wg, bound) in grads.items():
            within(grad[r], wg, bound, r)
    x.copy_(t)
    out = P().hbsjd_logprob_rows(x, dev(tok), entropy=True, logprob_weight=dev(a), grad=x)
    check_logprob(x64, tok, 1.0, a, None, (*out[:2], out[2].contiguous()), "bf16")


def test_same_bits_alone_or_among_rows():
    gen = torch.Generator("cuda").manual_seed(11)
    x, tok, f = inputs(gen, 300, 5000)
    x = x.to(torch.bfloat16)
    want = all_three(x, tok, f)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(all_three(x, tok, f), want))
    one = P().hbsjd_logprob_rows(x[7:8], tok[7:8], entropy=True, logprob_weight=f[7:8], entropy_weight=f[7:8],
                                 grad=True)
    assert all(torch.equal(a, b[7:8]) for a, b in zip(one, want))


@pytest.mark.parametrize("rows,V,dtype", [(6144, 16384, "f32"), (4608, 16384, "bf16"), (300, 60000, "f16"),
                                          (300, 80001, "f16"), (420, 50001, "f32"), (4200, 16381, "bf16"),
                                          (130, 128257, "bf16"), (70000, 40, "f32"), (2_200_000, 3, "f16")])
def test_batches(rows, V, dtype):
    """Batches of whole images, long and short rows, more rows than a launch takes:
    samples of them against the references, all of them for being finite."""
    gen = torch.Generator("cuda").manual_seed(rows)
    x = torch.randn((rows, V), generator=gen, device="cuda").mul_(2).to(TYPES[dtype])
    tok = torch.randint(0, V, (rows,), generator=gen, device="cuda").int()
    f = torch.randn(rows, generator=gen, device="cuda")
    out = P().hbsjd_logprob_rows(x, tok, entropy=True, logprob_weight=f, entropy_weight=f, grad=True)
    loss, pg, _, _ = P().hbsjd_policy_rows(x, tok, f, entropy_weight=0.1)
    d, dg, s = P().hbsjd_preference_rows(x, tok, pairs=rows // 2, ref_logprob=f, beta=0.5)
    for o in (*out, loss, pg, d, dg, s):
        assert bool(torch.isfinite(o).all())
    y = x.clone()
    P().hbsjd_policy_rows(y, tok, f, entropy_weight=0.1, grad=y)
    assert torch.equal(y, pg)
    y.copy_(x)
    P().hbsjd_preference_rows(y, tok, pairs=rows // 2, ref_logprob=f, beta=0.5, grad=y)
    assert torch.equal(y, dg)
    del y
    rng = np.random.default_rng(0)
    pick = np.unique(np.concatenate([[0, 1, rows - 2, rows - 1], rng.integers(0, rows, 4)]))
    at = torch.from_numpy(pick).cuda()
    x64, tk, fw = x[at].double().cpu().numpy(), tok[at].cpu().numpy(), f[at].cpu().numpy()
    check_logprob(x64, tk, 1.0, fw, fw, [o[at] for o in out], dtype)
    for j, r in enumerate(pick):
        q = ref.Row(x64[j], tk[j], 1.0)
        want, err, g, h, g_err = ref.policy(q, float(fw[j]), bonus=float(np.float32(0.1)))
        within(np.array(float(loss[r])), want, err, r)
        wg, bound = q.gradient(g, h, g_err, dtype)
        within(pg[r], wg, bound, r)
    for i in (0, rows // 2 - 1):
        two = slice(2 * i, 2 * i + 2)
        z, t2, f2 = x[two].double().cpu().numpy(), tok[two].cpu().numpy(), f[two].double().cpu().numpy()
        (want, err), _, _, grads = ref.preference(z, t2, [0, 1, 2], f2, 1.0, "sigmoid", 0.5, dtype=dtype)
        within(np.array(float(d[i])), want, err, i)
        for r, (wg, bound) in grads.items():
            within(dg[2 * i + r], wg, bound, r)


# ------------------------------------------------------------------ arguments

def test_binding_refuses():
    x = torch.randn(4, 64, device="cuda")
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    f = torch.zeros(4, device="cuda")
    L, Q, R = P().hbsjd_logprob_rows, P().hbsjd_policy_rows, P().hbsjd_preference_rows
    bad = [lambda: L(x.t(), i), lambda: L(x, None), lambda: L(x, i.long()), lambda: L(x, i[:3]),
           lambda: L(x.double(), i), lambda: L(x, i, logprob_weight=f[:2], grad=True),
           lambda: L(x, i, logprob_weight=f, grad=x.half()), lambda: L(x, i.cpu()),
           lambda: Q(x, i, None), lambda: Q(x, i, f.double()), lambda: Q(x, i, f, old_logprob=f[:1]),
           lambda: Q(x, i, f, row_weight=f.cpu()), lambda: Q(x, i, f, grad=x[:, :3]),
           lambda: R(x, i), lambda: R(x, i, pairs=2, form="other"), lambda: R(x, i, first=i),
           lambda: R(x, i, first=f[:3]), lambda: R(x, i, first=i[:3], pairs=2), lambda: R(x, i, pairs=-1),
           lambda: R(x, i, pairs=2, pair_weight=f), lambda: R(x, i, pairs=2, ref_logprob=f[:2])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: L(x, i, grad=True), lambda: L(x, i, temperature=0.0), lambda: Q(x, i, f, clip_low=1.5),
                 lambda: Q(x, i, f, kl_weight=0.1), lambda: Q(x, i, f, entropy_weight=-1.0),
                 lambda: R(x, i, pairs=3), lambda: R(x, i, pairs=2, beta=0.0),
                 lambda: R(x, i, pairs=2, smoothing=1.0),
                 lambda: R(x, i, pairs=2, form="hinge", smoothing=0.1),
                 lambda: R(x, i, pairs=2, margin=float("inf"))):
        with pytest.raises(P().HbsjdError) as e:
            call()
        assert e.value.code == "EINVAL"


@pytest.mark.parametrize("other_stream", [False, True])
def test_arguments_that_are_no_tensors(other_stream):
    x = torch.randn(4, 64, device="cuda")
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    f = torch.zeros(4, device="cuda")
    stream = torch.cuda.Stream() if other_stream else None
    before = torch.cuda.current_stream()
    torch.cuda.synchronize()
    calls = [(P().hbsjd_logprob_rows, dict(logits=x, tokens=i, logprob_weight=f, entropy_weight=f, grad=x.clone())),
             (P().hbsjd_policy_rows, dict(logits=x, tokens=i, advantage=f, old_logprob=f, ref_logprob=f,
                                          row_weight=f, grad=x.clone())),
             (P().hbsjd_preference_rows, dict(logits=x, tokens=i, first=torch.tensor(
                 [0, 1, 4], dtype=torch.int32, device="cuda"), ref_logprob=f, pair_weight=f[:1], grad=x.clone()))]
    for call, args in calls:
        call(**args, stream=stream)
        for name in args:
            for what in (args[name].cpu().numpy(), args[name].tolist(), 3, args[name].reshape(-1)[0]):
                with pytest.raises(ValueError):
                    call(**{**args, name: what}, stream=stream)
                assert torch.cuda.current_stream() == before
    torch.cuda.synchronize()


def test_autograd_sees_what_is_written():
    x = torch.randn(4, 40, device="cuda", requires_grad=True)
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    f = torch.ones(4, device="cuda")
    for write in (lambda y: P().hbsjd_logprob_rows(y, i, logprob_weight=f, grad=y),
                  lambda y: P().hbsjd_policy_rows(y, i, f, grad=y),
                  lambda y: P().hbsjd_preference_rows(y, i, pairs=2, grad=y)):
        assert not any(t.requires_grad for t in write(x * 1) if t is not None and t.shape != x.shape)
        y = x.exp()
        write(y)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
