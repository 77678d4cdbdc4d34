"""Rows whose largest logit stands far above the rest, among masked entries: its place beside
any of them, in every type."""
import numpy as np
import pytest

from tests import losses_ref as ref
from tests.row_operators_ref import U
from tests import test_gpu_row_operators as ops
from tests.test_gpu_token_losses import check_logprob, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

P, dev, placed, TYPES = ops.P, ops.dev, ops.placed, ops.TYPES


def peaked(rng, rows, V, dtype, peak, mask):
    """Noise, a part of the entries at `mask`, one of each row at `peak`: (logits, 64 bits,
    tokens: the peak's and others that are not masked)."""
    x = rng.normal(0, 2, (rows, V)).astype(np.float32)
    x[rng.random((rows, V)) < 0.5] = mask
    at = rng.integers(0, V, rows)
    x[np.arange(rows), at] = peak
    t = torch.from_numpy(x).to(TYPES[dtype])
    x64 = t.double().numpy()
    tok = at.copy()
    for r in range(1, rows, 2):
        open_ = np.flatnonzero(x64[r] > -1e4)
        tok[r] = open_[rng.integers(open_.size)]
    return t, x64, tok.astype(np.int32)


@pytest.mark.parametrize("layout", ["plain", "shifted"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [2, 16, 64, 257, 1024, 4099, 16384, 40001, 100000, 200000])
def test_peaked_and_masked(V, dtype, layout):
    rng = np.random.default_rng(V)
    lowest = float(torch.finfo(TYPES[dtype]).min)
    n = 24 if V < 20000 else 8
    for peak, mask, tau in ((100.0, -np.inf, 1.0), (300.0, -np.inf, 2.0), (20000.0, -np.inf, 1.0),
                            (60.0, -np.inf, 0.25), (300.0, lowest, 1.0), (-20.0, -np.inf, 0.1)):
        tau = float(np.float32(tau))   # as the call takes it: 0.1's rounding is 1.5e-8 of l
        t, x64, tok = peaked(rng, n, V, dtype, peak, mask)
        x, _ = placed(t.cuda(), layout)
        a, b = (rng.normal(0, 1, n).astype(np.float32) for _ in range(2))
        out = P().hbsjd_logprob_rows(x, dev(tok), temperature=tau, entropy=True, logprob_weight=dev(a),
                                     entropy_weight=dev(b), grad=True)
        check_logprob(x64, tok, tau, a, b, out, dtype)
        alone = P().hbsjd_logprob_rows(x, dev(tok), temperature=tau)
        check_logprob(x64, tok, tau, None, None, alone, dtype)
        rows = [ref.Row(x64[r], tok[r], tau) for r in range(n)]
        _, grad, s = P().hbsjd_preference_rows(x, dev(tok), pairs=n // 2, temperature=tau, form="square", beta=0.5)
        for r, q in enumerate(rows):
            within(np.array(float(s[r])), q.l, q.l_err + U * abs(q.l), ("log ratio", peak, r))
        assert not bool(torch.isnan(grad).any())
        loss = P().hbsjd_policy_rows(x, dev(tok), dev(a), temperature=tau)[0]
        for r in range(n):   # without another log-probability the ratio is 1
            assert float(loss[r]) == -a[r], (peak, r)
