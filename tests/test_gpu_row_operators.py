"""The operators on rows of logits against their 64-bit references: values and
indices exactly, sums and gradients within bounds on fp32 arithmetic that
tests/row_operators_ref.py derives, adjusted logits bit for bit."""
import numpy as np
import pytest

from tests import row_operators_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# sizes around the vector, wavefront, workgroup and part sizes of the kernels
SIZES = [1, 2, 5, 63, 64, 255, 257, 1000, 2047, 4096, 4099, 8191, 16384, 16385, 32768, 33001, 65537,
         131072, 262144]


def P():
    import paper_2608_18183_amd
    return paper_2608_18183_amd


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def placed(x, layout, fill=7.0):
    """The same rows as a device tensor laid out otherwise: (rows, whole buffer)."""
    rows, V = x.shape
    if layout == "plain":
        return x.contiguous(), None
    pad, first = {"strided": (13, 0), "shifted": (5, 3)}[layout]
    buf = torch.full((rows * (V + pad) + 64,), fill, dtype=x.dtype, device=x.device)
    view = torch.as_strided(buf, (rows, V), (V + pad, 1), first)
    view.copy_(x)
    return view, buf


def untouched(buf, view, fill=7.0):
    """Nothing outside the view was written."""
    keep = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(keep, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((buf[keep] == fill).all())


def rows_of(rng, n, V, dtype, kind="noise"):
    x = rng.normal(0, 2, (n, V)) * np.exp(rng.uniform(-1, 1, (n, 1)))
    if kind == "ties":
        x = np.round(x)
    if kind == "masked":
        x[rng.random((n, V)) < 0.4] = -np.inf
        x[:, V // 2] = 0.5
    if kind == "lowest":
        low = float(torch.finfo(TYPES[dtype]).min)
        x[rng.random((n, V)) < 0.4] = low
        x[:, V // 2] = 0.5
    t = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])
    return t, t.double().numpy()


# ------------------------------------------------------------------ top logits

def check_top(x64, out, k, tau):
    values, index, rest = (t.cpu().numpy() for t in out)
    wv, wi, wr = ref.top(x64, k, tau)
    assert np.array_equal(index, wi)
    assert np.array_equal(values.astype(np.float64), wv)
    n = x64.shape[1]
    for r in range(x64.shape[0]):
        if np.abs(wr[r]) > np.finfo(np.float32).max:
            # rest is fp32: beyond 2^128 (1 - 2^-25) the nearest is an infinity, and
            # the logits here lie well past that or well below it
            assert rest[r] == np.sign(wr[r]) * np.inf
        elif np.isfinite(wr[r]):
            s = wr[r] - np.where(np.isfinite(wv[r, -1]), wv[r, -1], 0) / tau
            left = np.delete(x64[r], wi[r]).max() / tau
            # m / tau (two roundings), the log of the sum, their sum
            tol = ref.log_sum_bound(n) + 3 * ref.U * (abs(left) + abs(wr[r] - left) + abs(wr[r]))
            assert abs(rest[r] - wr[r]) <= tol, (r, rest[r], wr[r], s)
        else:
            assert rest[r] == wr[r]


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", SIZES)
def test_top_logits(V, dtype, layout):
    rng = np.random.default_rng(V)
    n = 3
    for kind in ("noise", "ties", "masked", "lowest"):
        t, x64 = rows_of(rng, n, V, dtype, kind)
        x, buf = placed(t.cuda(), layout)
        for k in sorted({1, min(V, 3), min(V, 64), min(V, 300), min(V, 2048)}):
            tau = float(rng.choice([0.5, 1.0, 3.0]))
            out = (torch.full((n, k), -1.0, device="cuda"),
                   torch.full((n, k), -1, dtype=torch.int32, device="cuda"),
                   torch.full((n,), -1.0, device="cuda"))
            got = P().hbsjd_top_logits_rows(x, k, temperature=tau, out=out)
            check_top(x64, got, k, tau)


@pytest.mark.parametrize("V", [64, 1000, 16384, 70001])
def test_top_logits_of_equal_and_ordered_rows(V):
    """Rows in which a part of the entries, or all, are equal; ascending and
    descending rows (the largest all in one place); one peak."""
    x = np.zeros((8, V), np.float32)
    x[1] = np.arange(V)
    x[2] = -np.arange(V)
    x[3, V // 2] = 50.0
    x[4, ::3] = 1.0
    x[5] = -np.inf
    x[6] = np.where(np.arange(V) % 2 == 0, -0.0, 0.0)
    x[7] = np.float32(3e38) * np.where(np.arange(V) % 3 == 0, 1, -1)
    for k in sorted({1, 5, 64, min(V, 1000)}):
        got = P().hbsjd_top_logits_rows(dev(x), k, temperature=1.0)
        check_top(x.astype(np.float64), got, k, 1.0)


@pytest.mark.parametrize("V", [300, 5000, 40000])
def test_top_logits_far_from_zero(V):
    """Masks left at several values next to fp32's lowest, with and without
    -infinity among them, and rows that are all large."""
    rng = np.random.default_rng(V)
    x = rng.uniform(-3.39e38, -2e38, (5, V)).astype(np.float32)
    x[0, ::V // 5] = rng.normal(0, 1, x[0, ::V // 5].size)
    x[1, ::7] = -np.inf
    x[2] = -x[2]
    x[3] = rng.normal(0, 1, V) * 1e30
    x[4] = rng.normal(0, 1, V) - 90.0
    x[4, :20] += 200.0
    for k in (1, 8, 50, 200):
        for tau in (0.5, 1.0):
            check_top(x.astype(np.float64), P().hbsjd_top_logits_rows(dev(x), k, temperature=tau), k, tau)


@pytest.mark.parametrize("V", [3, 70, 3000, 20000])
def test_top_logits_rest_far_below_the_listed(V):
    """A confident row: the others' mass lies 5 to 80 below the listed logits, and
    its log keeps the digits that its own size asks for."""
    rng = np.random.default_rng(V)
    x = rng.normal(0, 0.3, (8, V)).astype(np.float32)
    x[:, 1] = [2.0, 4.0, 8.0, 14.8, 20.0, 30.0, 40.0, 80.0]
    x[4:, 2] = x[4:, 1] - 1.5
    for k in (1, 2):
        for tau in (0.5, 1.0):
            check_top(x.astype(np.float64), P().hbsjd_top_logits_rows(dev(x), k, temperature=tau), k, tau)


def test_top_logits_of_rows_with_nan_and_infinity():
    rng = np.random.default_rng(0)
    x = rng.normal(0, 1, (4, 500)).astype(np.float32)
    x[0, 100] = np.nan
    x[1, [7, 450]] = np.inf
    x[2, [3, 4, 5]] = [np.nan, -np.nan, np.inf]
    v, i, rest = (t.cpu().numpy() for t in P().hbsjd_top_logits_rows(dev(x), 4))
    assert i[0, 0] == 100 and np.isnan(v[0, 0]) and np.isnan(rest[0])
    assert np.array_equal(i[0, 1:], np.argsort(-np.delete(x[0], 100), kind="stable")[:3]
                          + (np.argsort(-np.delete(x[0], 100), kind="stable")[:3] >= 100))
    assert i[1, :2].tolist() == [7, 450] and np.isfinite(rest[1])
    assert i[2, :3].tolist() == [3, 4, 5] and np.isnan(rest[2])
    v1, i1, rest1 = (t.cpu().numpy() for t in P().hbsjd_top_logits_rows(dev(x[1:2]), 1))
    assert i1[0, 0] == 7 and rest1[0] == np.inf
    check_top(x[3:].astype(np.float64), [t[3:] for t in P().hbsjd_top_logits_rows(dev(x), 4)], 4, 1.0)


def test_top_logits_of_many_rows_and_bounds_of_its_outputs():
    rng = np.random.default_rng(4)
    n, V, k = 5000, 96, 7
    t, x64 = rows_of(rng, n, V, "bf16", "ties")
    out = (torch.full((n + 1, k), -5.0, device="cuda"),
           torch.full((n + 1, k), -5, dtype=torch.int32, device="cuda"),
           torch.full((n + 1,), -5.0, device="cuda"))
    P().hbsjd_top_logits_rows(t.cuda(), k, out=tuple(o[:n] for o in out))
    check_top(x64, [o[:n] for o in out], k, 1.0)
    assert all(bool((o[n:] == -5).all()) for o in out)


# ------------------------------------------------------------------ distillation

def teacher_of(rng, x64, k, tau, noise=0.7):
    z = np.where(np.isfinite(x64), x64, -30.0)
    t = (np.clip(z, -60, 60) + noise * rng.normal(0, 1, x64.shape)).astype(np.float32)
    v, i, rest = ref.top(t.astype(np.float64), k, tau)
    return v.astype(np.float32), i.astype(np.int32), rest.astype(np.float32)


def check_distill(x64, values, index, rest, w, tau, alpha, beta, loss, grad, dtype):
    loss, grad = loss.cpu().numpy().astype(np.float64), grad.double().cpu().numpy()
    rel, small = ref.ROUND[dtype]
    for r in range(x64.shape[0]):
        wl, wg, el, eg = ref.distill(x64[r], values[r].astype(np.float64), index[r],
                                     None if rest is None else np.float64(rest[r]),
                                     np.float64(w[r]), tau, alpha, beta)
        if not np.isfinite(wl):
            assert loss[r] == wl and np.isnan(grad[r]).all()
            continue
        assert abs(loss[r] - wl) <= el, (r, loss[r], wl, el)
        off = np.abs(grad[r] - wg) - (eg + rel * (np.abs(wg) + eg) + small)
        assert off.max() <= 0, (r, int(off.argmax()), grad[r][off.argmax()], wg[off.argmax()])


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", SIZES)
def test_distill(V, dtype, layout):
    rng = np.random.default_rng(V + 1)
    n = 3
    forms = [(0.5, 0.5, True), (1.0, 0.0, False), (1.0, 0.0, True), (0.0, 1.0, True)]
    for j, k in enumerate(sorted({1, min(V, 5), min(V, 64), min(V, 700)})):
        alpha, beta, with_rest = forms[(j + V) % 4]
        tau = float(rng.choice([0.5, 1.0, 2.0]))
        t, x64 = rows_of(rng, n, V, dtype)
        x, _ = placed(t.cuda(), layout)
        values, index, rest = teacher_of(rng, x64, k, tau)
        if V == k:
            rest[:] = -np.inf
        order = rng.permutation(k)
        values, index = values[:, order], index[:, order]
        if k > 2:
            index[1, 2] = -1      # a place not used
        w = rng.uniform(0.5, 2, n).astype(np.float32)
        if not with_rest:
            rest = None
        grad, gbuf = placed(torch.full((n, V), 3.0, dtype=TYPES[dtype], device="cuda"), layout)
        loss, g = P().hbsjd_distill_top_rows(
            x, dev(values), dev(index), None if rest is None else dev(rest), temperature=tau,
            forward_weight=alpha, reverse_weight=beta, row_weight=dev(w), grad=grad)
        assert g is grad
        check_distill(x64, values, index, rest, w, tau, alpha, beta, loss, grad, dtype)
        if gbuf is not None:
            assert untouched(gbuf, grad)


@pytest.mark.parametrize("V", [100, 5003, 16384, 70000])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_distill_in_place_alone_and_without_weights(V, dtype):
    rng = np.random.default_rng(V)
    n, k = 4, 17
    t, x64 = rows_of(rng, n, V, dtype)
    values, index, rest = teacher_of(rng, x64, k, 1.0)
    args = [dev(values), dev(index), dev(rest)]
    x = t.cuda()
    loss, grad = P().hbsjd_distill_top_rows(x, *args)
    check_distill(x64, values, index, rest, np.ones(n), 1.0, 0.5, 0.5, loss, grad, dtype)
    only, none = P().hbsjd_distill_top_rows(x, *args, grad=False)
    assert none is None and torch.equal(only, loss)
    again, same = P().hbsjd_distill_top_rows(x, *args, grad=x)
    assert same is x and torch.equal(again, loss) and torch.equal(x, grad)


@pytest.mark.parametrize("V", [96, 4099, 16384, 40000])
def test_distill_rows_that_have_no_answer(V):
    """Rows of weight zero are not read; the others' data errors stay in them."""
    rng = np.random.default_rng(V)
    n, k = 14, 9
    x = rng.normal(0, 2, (n, V)).astype(np.float32)
    values, index, rest = teacher_of(rng, x.astype(np.float64), k, 1.0)
    w = np.ones(n, np.float32)
    x[1], w[1] = np.nan, 0                   # weighted out
    x[2] = -np.inf                           # a mask that leaves nothing
    x[3, V // 2] = np.nan
    x[4, 5] = np.inf
    index[5, 3] = index[5, 8]                # the same entry twice
    index[6, 0] = V                          # out of range
    index[7, 1] = -2
    index[8, :], rest[8] = -1, -np.inf       # an empty answer
    values[9, 2] = np.nan
    rest[10] = np.nan
    x[11, index[11, 0]] = -np.inf            # the teacher's first choice masked out
    values[12, 0] = np.inf
    index[12, 3] = -1
    keep = [0, 13]
    x[13, np.setdiff1d(np.arange(0, V, 2), index[13])] = -np.inf   # masked entries the teacher does not list
    for alpha, beta in ((0.5, 0.5), (1.0, 0.0)):
        loss, grad = P().hbsjd_distill_top_rows(dev(x), dev(values), dev(index), dev(rest),
                                                forward_weight=alpha, reverse_weight=beta,
                                                row_weight=dev(w))
        lo, g = loss.cpu().numpy(), grad.cpu().numpy()
        assert lo[1] == 0 and (g[1] == 0).all()
        for r in (2, 3, 4, 5, 6, 7, 8, 9, 10, 12):
            assert np.isnan(lo[r]) and np.isnan(g[r]).all(), r
        assert lo[11] == np.inf and np.isnan(g[11]).all()
        check_distill(x[keep].astype(np.float64), values[keep], index[keep], rest[keep], w[keep], 1.0,
                      alpha, beta, loss[keep], grad[keep], "f32")


def test_distill_masks_of_the_lowest_value_and_far_tails():
    """Entries at the type's lowest value have no mass on either side; a student
    whose unlisted mass lies far below fp32's rounding keeps its gradient."""
    rng = np.random.default_rng(8)
    V, k = 3000, 8
    for dtype in ("f32", "bf16", "f16"):
        low = float(torch.finfo(TYPES[dtype]).min)
        x = rng.normal(0, 1, (3, V)).astype(np.float32)
        x[0, 1000:] = low
        x[1, :k] += 40.0                   # the unlisted entries hold e^-40
        x[2, 10:] = -60.0
        t = torch.from_numpy(x).to(TYPES[dtype])
        x64 = t.double().numpy()
        index = np.tile(np.arange(k, dtype=np.int32), (3, 1))
        values = x64[:, :k].astype(np.float32) + rng.normal(0, 0.5, (3, k)).astype(np.float32)
        rest = np.array([0.0, -3.0, -55.0], np.float32)
        w = np.ones(3, np.float32)
        loss, grad = P().hbsjd_distill_top_rows(t.cuda(), dev(values), dev(index), dev(rest),
                                                forward_weight=0.7, reverse_weight=0.3)
        check_distill(x64, values, index, rest, w, 1.0, 0.7, 0.3, loss, grad, dtype)


@pytest.mark.parametrize("V", [300, 20000])
def test_distill_forward_alone_with_entries_of_no_mass(V):
    """Listed entries at -infinity on the teacher's side and a rest of no mass
    leave the forward divergence and its gradient finite."""
    rng = np.random.default_rng(V)
    n, k = 3, 6
    x = rng.normal(0, 2, (n, V)).astype(np.float32)
    values, index, rest = teacher_of(rng, x.astype(np.float64), k, 1.0)
    values[0, 4], values[1, 5], rest[1], rest[2] = -np.inf, -np.inf, -np.inf, -200.0
    for r_ in (rest, None):
        loss, grad = P().hbsjd_distill_top_rows(
            dev(x), dev(values), dev(index), None if r_ is None else dev(r_), forward_weight=1.5,
            reverse_weight=0.0)
        assert bool(torch.isfinite(loss).all())
        check_distill(x.astype(np.float64), values, index, r_, np.ones(n), 1.0, 1.5, 0.0, loss, grad,
                      "f32")


@pytest.mark.parametrize("tau", [0.7, 1.0, 3.0])
def test_distill_of_nearly_equal_rows_keeps_its_digits(tau):
    """A student close to its teacher: the loss is far below the logs it is made
    of. Exponentials good to 2^-22 put q_0 and the entries' q off by that much, to
    which the divergence of near rows is sensitive by |q - P| and |log q - log P|;
    the inputs' own rounding is part of the reference."""
    rng = np.random.default_rng(5)
    n, V, k = 6, 16384, 64
    x = (rng.normal(0, 1, (n, V)) + 20).astype(np.float32)
    values, index, rest = teacher_of(rng, x.astype(np.float64), k, tau, noise=1e-2)
    loss, grad = P().hbsjd_distill_top_rows(dev(x), dev(values), dev(index), dev(rest), temperature=tau)
    for r in range(n):
        wl, wg, _, _ = ref.distill(x[r].astype(np.float64), values[r].astype(np.float64), index[r],
                                   np.float64(rest[r]), 1.0, tau, 0.5, 0.5)
        # |c| is at most about 0.05 / tau here, sum |q - P| and sum (P + q) |c|
        # below 0.05; each rounding above meets one of them, and rest, rounded at
        # about 30 / tau, shifts log P_0 by half an fp32 step of it (in the input)
        assert abs(float(loss[r]) - wl) <= 0.05 * (2.0 ** -22 * 4) + 2.0 ** -22 * wl


def test_distill_over_all_entries_is_the_bidirectional_divergence():
    """With every entry listed the loss is the one hbsjd_bikl_rows computes."""
    rng = np.random.default_rng(9)
    n, V = 40, 2048
    s, t = (rng.normal(0, 2, (n, V)).astype(np.float32) for _ in range(2))
    v, i, rest = P().hbsjd_top_logits_rows(dev(t), V)
    assert bool((rest == -np.inf).all())
    loss, grad = P().hbsjd_distill_top_rows(dev(s), v, i, rest)
    want = P().hbsjd_bikl_rows(dev(s), dev(t)).double().cpu().numpy()
    # both sides' fp32 errors: the bound of this one, and as much for the other
    for r in range(n):
        wl, _, el, _ = ref.distill(s[r].astype(np.float64), v[r].double().cpu().numpy(),
                                   i[r].cpu().numpy(), -np.inf, 1.0, 1.0, 0.5, 0.5)
        assert abs(float(loss[r]) - want[r]) <= 2 * el
        assert abs(wl - want[r]) <= el
    # a distribution's gradient by its logits sums to zero: V roundings of the
    # entries, each within the gradient's own bound
    assert float(grad.double().sum(1).abs().max()) < 1e-5


def test_distill_gradient_equals_differences_of_its_loss():
    rng = np.random.default_rng(10)
    V, k = 260, 12
    x = rng.normal(0, 1.5, (1, V)).astype(np.float32)
    values, index, rest = teacher_of(rng, x.astype(np.float64), k, 1.0)
    h = 2.0 ** -6
    probes = np.concatenate([index[0, :6], [0, 1, 100, 259]])
    moved = np.repeat(x, 2 * probes.size, 0)
    for j, v in enumerate(probes):
        moved[2 * j, v] += np.float32(h)
        moved[2 * j + 1, v] -= np.float32(h)
    m = moved.shape[0]
    rep = lambda a: dev(np.repeat(a, m, 0))
    loss = P().hbsjd_distill_top_rows(dev(moved), rep(values), rep(index), rep(rest),
                                      grad=False)[0].double().cpu().numpy()
    _, grad = P().hbsjd_distill_top_rows(dev(x), dev(values), dev(index), dev(rest))
    _, _, el, _ = ref.distill(x[0].astype(np.float64), values[0].astype(np.float64), index[0],
                              float(rest[0]), 1.0, 1.0, 0.5, 0.5)
    step = (moved[0::2, probes].diagonal().astype(np.float64)
            - moved[1::2, probes].diagonal().astype(np.float64))
    d = (loss[0::2] - loss[1::2]) / step
    got = grad[0].double().cpu().numpy()[probes]
    # two losses' errors over the step, and h^2 / 6 times a third derivative that
    # |c| + 6 bounds for these logits (|c| < 8)
    assert np.abs(d - got).max() <= 2 * el / (2 * h) * 1.1 + h * h / 6 * 14


def test_distill_same_bits_each_time_and_alone_or_among_rows():
    rng = np.random.default_rng(11)
    n, V, k = 300, 5000, 33
    t, x64 = rows_of(rng, n, V, "bf16")
    values, index, rest = teacher_of(rng, x64, k, 1.0)
    x, a = t.cuda(), [dev(values), dev(index), dev(rest)]
    l0, g0 = P().hbsjd_distill_top_rows(x, *a)
    for _ in range(3):
        l1, g1 = P().hbsjd_distill_top_rows(x, *a)
        assert torch.equal(l0, l1) and torch.equal(g0, g1)
    l2, g2 = P().hbsjd_distill_top_rows(x[7:8], *[b[7:8].contiguous() for b in a])
    assert torch.equal(l2, l0[7:8]) and torch.equal(g2, g0[7:8])


# ------------------------------------------------------------------ adjusting

def adjust_case(rng, n, V, dtype, n_tokens, n_bias, masks, layout="plain", out_type=None,
                in_place=False, kind="noise"):
    t, _ = rows_of(rng, n, V, dtype, kind)
    x32 = t.float().numpy()
    out_type = out_type or dtype
    kw, per_row = {}, [dict() for _ in range(n)]
    if n_tokens:
        few = rng.integers(0, max(1, V // 8), (n, n_tokens))
        tok = np.where(rng.random((n, n_tokens)) < 0.5, few, rng.integers(-2, V + 3, (n, n_tokens)))
        tok = tok.astype(np.int32)
        count = rng.integers(0, n_tokens + 1, n).astype(np.int32)
        count[0] = n_tokens
        pen = {"repetition": rng.uniform(0.8, 1.7, n), "presence": rng.normal(0, 1, n),
               "frequency": rng.normal(0, 0.3, n)}
        pen = {k: v.astype(np.float32) for k, v in pen.items()}
        kw.update(tokens=dev(tok), token_count=dev(count), **{k: dev(v) for k, v in pen.items()})
        for r in range(n):
            per_row[r].update(tokens=tok[r, :count[r]], **{k: v[r] for k, v in pen.items()})
    if n_bias:
        bi = rng.integers(-1, V + 1, (n, n_bias)).astype(np.int32)
        bi[:, n_bias // 2] = bi[:, 0]          # the same entry twice
        bv = rng.normal(0, 3, (n, n_bias)).astype(np.float32)
        kw.update(bias_index=dev(bi), bias_value=dev(bv))
        for r in range(n):
            per_row[r]["bias"] = list(zip(bi[r], bv[r]))
    if masks:
        allowed = rng.random((masks, V)) < rng.random((masks, 1))
        allowed[0] = False
        which = rng.integers(-1, masks, n).astype(np.int32)
        kw.update(mask=dev(ref.pack_mask(allowed)), mask_row=dev(which))
        for r in range(n):
            if which[r] >= 0:
                per_row[r]["allowed"] = allowed[which[r]]
    x, xbuf = placed(t.cuda(), layout)
    if in_place:
        out, obuf = x, xbuf
    else:
        out, obuf = placed(torch.zeros((n, V), dtype=TYPES[out_type], device="cuda"), layout)
    got = P().hbsjd_adjust_rows(x, out=out, **kw)
    assert got is out
    want = np.stack([ref.adjust(x32[r], **per_row[r]) for r in range(n)])
    want = torch.from_numpy(want).to(TYPES[out_type])
    g = got.cpu()
    same = (g == want) | (torch.isnan(g) & torch.isnan(want))
    assert bool(same.all()), torch.nonzero(~same)[:5].tolist()
    if obuf is not None:
        assert untouched(obuf, out)


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype,out_type", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"),
                                            ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("V", SIZES)
def test_adjust(V, dtype, out_type, layout):
    rng = np.random.default_rng(V + 2)
    for n_tokens, n_bias, masks in ((0, 0, 0), (40, 0, 0), (0, 9, 0), (0, 0, 3), (300, 70, 5)):
        adjust_case(rng, 3, V, dtype, n_tokens, n_bias, masks, layout, out_type)
        if dtype == out_type:
            adjust_case(rng, 3, V, dtype, n_tokens, n_bias, masks, layout, in_place=True)


@pytest.mark.parametrize("kind", ["ties", "masked", "lowest"])
@pytest.mark.parametrize("n_tokens,n_bias", [(1, 1), (5000, 1024), (70000, 2)])
def test_adjust_long_lists_and_masked_rows(kind, n_tokens, n_bias):
    rng = np.random.default_rng(n_tokens)
    for V in (37, 5001, 40000):
        adjust_case(rng, 2, V, "f32", n_tokens, n_bias, 4, kind=kind)


def test_adjust_shared_lists_nan_and_masks_that_leave_nothing():
    rng = np.random.default_rng(3)
    n, V = 5, 777
    x = rng.normal(0, 1, (n, V)).astype(np.float32)
    x[2, 5] = np.nan
    x[2, 6] = np.inf
    tok = rng.integers(0, V, 50).astype(np.int32)
    bi, bv = np.array([6, 5, 6], np.int32), np.array([1.0, 2.0, -0.5], np.float32)
    freq = np.full(n, 0.25, np.float32)
    allowed = np.ones((3, V), bool)
    allowed[0] = False
    allowed[1, 5] = False
    which = np.array([0, 1, 1, 3, -7], np.int32)      # 3: there is no such mask
    got = P().hbsjd_adjust_rows(dev(x), tokens=dev(tok), frequency=dev(freq), bias_index=dev(bi),
                                bias_value=dev(bv), mask=dev(ref.pack_mask(allowed)),
                                mask_row=dev(which)).cpu().numpy()
    kw = dict(tokens=tok, frequency=freq[0], bias=list(zip(bi, bv)))
    assert (got[0] == -np.inf).all() and np.isnan(got[3]).all()
    for r, ok in ((1, allowed[1]), (2, allowed[1]), (4, None)):
        assert np.array_equal(got[r], ref.adjust(x[r], allowed=ok, **kw), equal_nan=True)
    assert got[2, 5] == -np.inf and got[2, 6] == np.inf
    # without a row list every row has the mask of its number
    own = P().hbsjd_adjust_rows(dev(x[:3]), mask=dev(ref.pack_mask(allowed))).cpu().numpy()
    assert np.array_equal(own, np.where(allowed, x[:3], -np.inf), equal_nan=True)


def test_adjust_ignores_entries_and_counts_out_of_range():
    rng = np.random.default_rng(4)
    big = 2 ** 31 - 1
    x = rng.normal(0, 1, (4, 300)).astype(np.float32)
    tok = rng.integers(0, 300, (4, 9)).astype(np.int32)
    tok[:, ::2] = [-big - 1, -1, 300, 17, big]
    count = np.array([9, -3, big, 0], np.int32)       # clamped to [0, 9]
    bi = np.tile(np.array([-big - 1, 17, -1, 300, big, 17], np.int32), (4, 1))
    bv = rng.normal(0, 1, (4, 6)).astype(np.float32)
    freq = np.full(4, 0.5, np.float32)
    got = P().hbsjd_adjust_rows(dev(x), tokens=dev(tok), token_count=dev(count), frequency=dev(freq),
                                bias_index=dev(bi), bias_value=dev(bv)).cpu().numpy()
    for r, n in enumerate((9, 0, 9, 0)):
        assert np.array_equal(got[r], ref.adjust(x[r], tokens=tok[r, :n], frequency=0.5,
                                                 bias=list(zip(bi[r], bv[r]))))


def test_adjust_of_nothing():
    x = torch.randn(9, 501, device="cuda").to(torch.bfloat16)
    assert P().hbsjd_adjust_rows(x) is x
    out = torch.zeros_like(x)
    assert P().hbsjd_adjust_rows(x, out=out) is out and torch.equal(out, x)
    assert torch.equal(P().hbsjd_adjust_rows(x, out_dtype=torch.float32), x.float())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_in_error_are_nan_in_every_type(dtype):
    rng = np.random.default_rng(12)
    n, V, k = 4, 301, 6
    t, x64 = rows_of(rng, n, V, dtype)
    values, index, rest = teacher_of(rng, x64, k, 1.0)
    index[1, 2] = V + 5
    loss, grad = P().hbsjd_distill_top_rows(t.cuda(), dev(values), dev(index), dev(rest))
    keep = [0, 2, 3]
    assert bool(torch.isnan(loss[1])) and bool(torch.isnan(grad[1]).all())
    check_distill(x64[keep], values[keep], index[keep], rest[keep], np.ones(3), 1.0, 0.5, 0.5,
                  loss[keep], grad[keep], dtype)
    ok = dev(ref.pack_mask(np.ones((1, V), bool)))
    which = dev(np.array([0, 1, -1, 0], np.int32))
    for out_dtype in (TYPES[dtype], torch.float32):
        y = P().hbsjd_adjust_rows(t.cuda(), mask=ok, mask_row=which, out_dtype=out_dtype)
        assert bool(torch.isnan(y[1]).all())
        assert torch.equal(y[keep], t.cuda()[keep].to(out_dtype))


@pytest.mark.parametrize("V", [500, 20000])
def test_offsets_past_32_bits(V):
    """Rows 1.2e9 entries apart: the third starts past 2^31 entries and 2^32 bytes."""
    rng = np.random.default_rng(13)
    n, k, ld = 3, 9, 1_200_000_007
    t, x64 = rows_of(rng, n, V, "bf16")
    buf = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (n, V), (ld, 1))
    x.copy_(t)
    check_top(x64, P().hbsjd_top_logits_rows(x, k), k, 1.0)
    values, index, rest = teacher_of(rng, x64, k, 1.0)
    tok = rng.integers(0, V, (n, 50)).astype(np.int32)
    freq = np.full(n, 0.5, np.float32)
    y = P().hbsjd_adjust_rows(x, tokens=dev(tok), frequency=dev(freq), out_dtype=torch.float32)
    for r in range(n):
        assert np.array_equal(y[r].cpu().numpy(),
                              ref.adjust(t[r].float().numpy(), tokens=tok[r], frequency=0.5))
    loss, grad = P().hbsjd_distill_top_rows(x, dev(values), dev(index), dev(rest), grad=x)
    check_distill(x64, values, index, rest, np.ones(n), 1.0, 0.5, 0.5, loss, grad.contiguous(), "bf16")


def test_list_lengths_and_positions_of_every_kind_of_k():
    """K at the sizes where the selection changes its workgroups, its room and its
    way of placing, on random, tied and ordered rows."""
    rng = np.random.default_rng(14)
    for V in (1024, 1025, 4097, 16384, 50000):
        for dtype in ("f32", "bf16"):
            rows = [rng.normal(0, 2, V), np.round(rng.normal(0, 2, V)), np.sort(rng.normal(0, 2, V)),
                    np.linspace(5, -5, V) + rng.normal(0, 0.5, V)]
            t = torch.from_numpy(np.stack(rows).astype(np.float32)).to(TYPES[dtype])
            for k in (31, 32, 33, 128, 129, 255, 256, 257, 511, 513, 1024):
                check_top(t.double().numpy(), P().hbsjd_top_logits_rows(t.cuda(), k), k, 1.0)


# ------------------------------------------------------------------ as calls

def all_three(x, tok, freq, k, stream=None):
    y = P().hbsjd_adjust_rows(x, tokens=tok, frequency=freq, stream=stream)
    v, i, rest = P().hbsjd_top_logits_rows(y, k, stream=stream)
    loss, grad = P().hbsjd_distill_top_rows(x, v, i, rest, stream=stream)
    return [y, v, i, rest, loss, grad]


@pytest.mark.parametrize("V", [600, 16384, 50001])
def test_captured_and_replayed(V):
    """Two graphs of the three calls, replayed in turn with the eager calls on
    other data between the replays, give the eager calls' results each time."""
    gen = torch.Generator("cuda").manual_seed(V)
    n, k = 6, 20
    x = [torch.randn((n, V), generator=gen, device="cuda") for _ in range(2)]
    tok = torch.randint(0, V, (n, 30), generator=gen, device="cuda").int()
    freq = torch.rand(n, generator=gen, device="cuda")
    all_three(x[0], tok, freq, k)
    torch.cuda.synchronize()
    graphs = []
    for j in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = all_three(x[j], tok, freq, k)
        graphs.append((g, out))
    for rep in range(4):
        for j in range(2):
            x[j].copy_(torch.randn((n, V), generator=gen, device="cuda"))
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for j in range(2):
            want = all_three(x[j], tok, freq, k)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(graphs[j][1], want)), (rep, j)


def test_other_streams_and_threads():
    """Calls at once on several streams from several threads, given as torch's
    streams and as handles, equal the calls made one after another."""
    import threading
    gen = torch.Generator("cuda").manual_seed(5)
    n, V, k = 50, 20000, 40
    x = torch.randn((n, V), generator=gen, device="cuda")
    tok = torch.randint(0, V, (n, 30), generator=gen, device="cuda").int()
    freq = torch.rand(n, generator=gen, device="cuda")
    want = all_three(x, tok, freq, k)
    torch.cuda.synchronize()
    wrong = []

    def work(j):
        s = torch.cuda.Stream()
        for _ in range(5):
            got = all_three(x, tok, freq, k, stream=s if j % 2 else s.cuda_stream)
            s.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)):
                wrong.append(j)

    threads = [threading.Thread(target=work, args=(j,)) for j in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_binding_refuses():
    x = torch.randn(4, 64, device="cuda")
    v, i, rest = P().hbsjd_top_logits_rows(x, 8)
    bad = [lambda: P().hbsjd_top_logits_rows(x.t(), 2), lambda: P().hbsjd_top_logits_rows(x, 0),
           lambda: P().hbsjd_top_logits_rows(x.double(), 2),
           lambda: P().hbsjd_top_logits_rows(x[:1].expand(4, 64), 2),
           lambda: P().hbsjd_distill_top_rows(x, v[:3], i, rest),
           lambda: P().hbsjd_distill_top_rows(x, v, i.long(), rest),
           lambda: P().hbsjd_distill_top_rows(x, v, i, rest[:2]),
           lambda: P().hbsjd_distill_top_rows(x, v, i, rest, grad=x.half()),
           lambda: P().hbsjd_distill_top_rows(x, v.cpu(), i, rest),
           lambda: P().hbsjd_adjust_rows(x, frequency=rest),
           lambda: P().hbsjd_adjust_rows(x, tokens=i, presence=rest[:3]),
           lambda: P().hbsjd_adjust_rows(x, bias_index=i),
           lambda: P().hbsjd_adjust_rows(x, mask=torch.zeros(4, 3, dtype=torch.int32, device="cuda"))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: P().hbsjd_top_logits_rows(x, 65),
              lambda: P().hbsjd_distill_top_rows(x, v, i, None),
              lambda: P().hbsjd_distill_top_rows(x, v, i, rest, temperature=0.0),
              lambda: P().hbsjd_adjust_rows(x, out_dtype=torch.bfloat16)):
        with pytest.raises(P().HbsjdError) as e:
            f()
        assert e.value.code == "EINVAL"


def test_no_rows():
    x = torch.zeros(0, 64, device="cuda")
    v, i, rest = P().hbsjd_top_logits_rows(x, 8)
    loss, grad = P().hbsjd_distill_top_rows(x, v, i, rest)
    assert loss.shape == (0,) and grad.shape == (0, 64)
    assert P().hbsjd_adjust_rows(x).shape == (0, 64)


# ------------------------------------------------------------------ in use

def test_a_distillation_step_on_a_rollout(tiny):
    """A student's rollout; the teacher's answers on the generated positions; the
    student's loss and gradient there. With every entry listed the loss is the
    score the contexts compute themselves; with fewer it is a lower bound."""
    import synth
    from tests import gpu_util as gu
    w, blob, _ = tiny
    student = gu.make_ctx(w.model, "f32", blob)
    teacher = gu.make_ctx(w.model, "f32", synth.make_weights(w.model, 5) * 4)
    batch = synth.make_batch(w, 1)
    out = student.hbsjd_rollout(gu.device_batch(batch), batch.prefix_len, batch.labels,
                                batch.temperature, w.window, history=w.history, seed=3)
    tokens, T, V = out["tokens"], w.model.grid ** 2, w.model.vocab
    per, _ = student.hbsjd_score_bikl(teacher, tokens, batch.prefix_len, batch.labels)
    lens = np.full(len(batch.prefix_len), T - 1, np.int32)
    weight = torch.ones((len(lens), T), device="cuda")
    for b, k in enumerate(batch.prefix_len):
        weight[b, :int(k)] = 0.0
    logits_t = teacher.hbsjd_forward(tokens, lens, batch.labels)
    logits_s = student.hbsjd_forward(tokens, lens, batch.labels)
    z = logits_s.double().cpu().numpy()
    last = None
    for k in (4, 32, V):
        v, i, rest = P().hbsjd_top_logits_rows(logits_t, k)
        loss, grad = P().hbsjd_distill_top_rows(logits_s, v, i, rest, row_weight=weight.view(-1))
        check_distill(z, v.cpu().numpy(), i.cpu().numpy(), rest.cpu().numpy(),
                      weight.view(-1).cpu().numpy(), 1.0, 0.5, 0.5, loss, grad, "f32")
        if last is not None:
            assert bool((loss >= last - 1e-5).all())
        last = loss
    # the score's own fp32 sums of V entries of magnitude |p - q| |ls - lt| < 10
    assert float((last.view(len(lens), T) - per).abs().max()) < 10 * V * 2.0 ** -24


def test_adjusted_rows_are_drawn_from():
    """Penalties, biases and a grammar's masks ahead of the sampler: it draws
    allowed tokens only, and its rows are the softmax of the adjusted logits."""
    gen = torch.Generator("cuda").manual_seed(1)
    n, V = 200, 16384
    x = (torch.randn((n, V), generator=gen, device="cuda") * 2).to(torch.bfloat16)
    tok = torch.randint(0, V, (n, 100), generator=gen, device="cuda").int()
    pen = dict(repetition=torch.full((n,), 1.3, device="cuda"),
               presence=torch.full((n,), 0.5, device="cuda"))
    allowed = np.random.default_rng(0).random((4, V)) < np.array([[0.5], [0.9], [0.01], [0.2]])
    which = torch.randint(0, 4, (n,), generator=gen, device="cuda").int()
    y = P().hbsjd_adjust_rows(x, tokens=tok, **pen, mask=dev(ref.pack_mask(allowed)),
                              mask_row=which, out_dtype=torch.float32)
    tau = torch.ones(n, device="cuda")
    p, amax, draw = P().hbsjd_transform_rows(y, tau, torch.arange(n, device="cuda").int(), seed=9)
    ok = torch.from_numpy(allowed).cuda()[which.long()]
    assert bool(ok[torch.arange(n, device="cuda"), draw.long()].all())
    assert bool((p[~ok] == 0).all())
    want = torch.softmax(y.double(), 1)
    # an exponential's argument of up to 25 and a sum of 16384 terms in fp32
    assert float((p.double() - want).abs().max()) <= 2.0 ** -24 * (16384 / 64 + 6 * 25 + 64)
    assert bool(torch.equal(amax.long(), torch.argmax(y, 1)))
