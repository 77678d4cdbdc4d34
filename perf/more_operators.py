"""The operators of a policy or preference training step, with inputs, a plain
form of each in elementary torch operations, and their values in 64 bits.

Three calls on rows of logits, with y a row's token, tau the temperature, p =
softmax(z / tau), l = log p_y and H = -sum p log p:

* `logprob`: l and H, or the gradient of a l + b H by the logits.
* `policy`: the clipped policy loss with a KL term and an entropy bonus, and its
  gradient by the logits. With rho = exp(l - old), A the advantage and
  D = exp(ref - l) - (ref - l) - 1,
      L = w (-min(rho A, clip(rho, 1 - low, 1 + high) A) + kl D - ent H).
* `preference`: pairs of sequences, a chosen and a rejected one. With s the sum
  (or the mean) of l - ref over a sequence's tokens, u = s_chosen - s_rejected -
  margin and h = beta u, the loss of a pair is
      sigmoid  -(1 - eps) log sigmoid(h) - eps log sigmoid(-h)
      hinge    max(0, 1 - h)
      square   (u - 1 / (2 beta))^2
  times its weight; its gradient reaches the logits of all rows of both.

Rows whose token is -1 (padding, real prefixes) take no part.

And two on lists of tensors: the norm of all entries of all tensors (`norm`), and
the tensors scaled so that it does not pass a limit (`clip`).

Sizes follow this repository's workloads (vocabulary 16384, 16x16 and 24x24
grids, windows of 16 to 32 drafts; the parameters of its models) and generic
larger vocabularies.
"""
import math
import random

import torch

own = False   # False: the plain forms; True: the framework's operators

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the log-probability of the one token drawn last: launch and latency
        dict(name="logprob_one_row", kind="logprob", rows=1, vocab=16384, type="f32", tau=1.0,
             entropy=True, grad=False, unused=0.0),
        # a finished B batch under the reference weights: every generated position
        dict(name="logprob_b_batch", kind="logprob", rows=6144, vocab=16384, type="f32", tau=1.0,
             entropy=False, grad=False, unused=0.0),
        # the backward pass over whole sequences of the 24x24 grid with their real
        # prefixes left out, 16-bit logits
        dict(name="logprob_l_backward", kind="logprob", rows=18432, vocab=16384, type="bf16",
             tau=1.0, entropy=True, grad=True, unused=0.25),
        # one window of drafts: W + 1 rows, latency
        dict(name="policy_window", kind="policy", rows=17, vocab=16384, type="f32", tau=1.0,
             high=0.2, kl=0.04, entropy=0.01, old=True, unused=0.0),
        # the training step on a finished B batch
        dict(name="policy_b_batch", kind="policy", rows=6144, vocab=16384, type="f32", tau=1.0,
             high=0.28, kl=0.04, entropy=0.01, old=True, unused=0.0),
        # a language model's vocabulary of odd size, a batch of few long rows
        dict(name="policy_wide", kind="policy", rows=64, vocab=128257, type="f16", tau=0.7,
             high=0.2, kl=0.0, entropy=0.0, old=True, unused=0.0),
        # one pair of short continuations, latency
        dict(name="preference_pair", kind="preference", pairs=1, length=16, packed=False,
             vocab=16384, type="f32", tau=1.0, form="sigmoid", mean=False, unused=0.0),
        # sixteen pairs of completed 16x16 images, real prefixes left out, 16-bit logits
        dict(name="preference_b_images", kind="preference", pairs=16, length=256, packed=False,
             vocab=16384, type="bf16", tau=1.0, form="sigmoid", mean=False, unused=0.25),
        # packed texts of odd lengths, a language model's vocabulary, means in place of sums
        dict(name="preference_packed", kind="preference", pairs=4, length=101, packed=True,
             vocab=128257, type="bf16", tau=1.0, form="square", mean=True, unused=0.1),
        # the gradients of the tiny model: launch and latency
        dict(name="norm_tiny_model", kind="norm", sizes="tiny", tensors=18, largest=16384,
             type="f32", order=2.0, flat=False, limit=0.0),
        # the gradients of the B model, matrices in 16 bits, in one flat buffer, clipped
        dict(name="clip_b_model", kind="norm", sizes="b", tensors=88, largest=12582912,
             type="bf16", order=2.0, flat=True, limit=0.5),
        # the gradients of the XL model in 32 bits, clipped
        dict(name="clip_xl_model", kind="norm", sizes="xl", tensors=256, largest=20971520,
             type="f32", order=2.0, flat=False, limit=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprob", "policy", "preference", "norm"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "norm":
        tensors = _log(rng, 1, 600)
        return dict(kind=kind, sizes=rng.randrange(1 << 20), tensors=tensors,
                    largest=_log(rng, 16, min(1 << 25, 600_000_000 // tensors)), type=dtype,
                    order=rng.choice([2.0, 2.0, math.inf]), flat=rng.random() < 0.5,
                    limit=rng.choice([0.0, 0.5, 2.0]))
    vocab = rng.choice([16384, _log(rng, 32, 16384), _log(rng, 16384, 200000)])
    most = max(1, min(6144 * 16384 // vocab, 16384))
    case = dict(kind=kind, vocab=vocab, type=dtype, tau=rng.choice([0.7, 1.0, 2.0]),
                unused=rng.choice([0.0, 0.0, 0.25]))
    if kind == "preference":
        pairs = _log(rng, 1, max(1, min(most // 4, 128)))
        form = rng.choice(["sigmoid", "hinge", "square"])
        # the square of a long sequence's sum would leave fp16's range
        return dict(case, pairs=pairs, length=_log(rng, 1, max(1, most // (2 * pairs))),
                    packed=rng.random() < 0.5, form=form,
                    mean=form == "square" or rng.random() < 0.5)
    case["rows"] = _log(rng, 1, most)
    if kind == "logprob":
        return dict(case, entropy=rng.random() < 0.5, grad=rng.random() < 0.5)
    return dict(case, high=rng.choice([0.2, 0.28]), kl=rng.choice([0.0, 0.04, 0.5]),
                entropy=rng.choice([0.0, 0.01]), old=rng.random() < 0.8)


# ------------------------------------------------------------------ inputs

def _parts(total, size):
    return [(a, min(a + size, total)) for a in range(0, total, size)]


def _rows(rows, vocab, dtype, tau, gen):
    """Logits as a decoder's head gives them (noise over a common profile of the
    tokens, some rows nearly flat and some peaked), each row's token as a slightly
    older model drew it, and the tokens' log-probabilities: the rows' own in 64 bits,
    the older model's and a reference's."""
    x = torch.empty((rows, vocab), dtype=dtype, device="cuda")
    profile = torch.randn(vocab, generator=gen, device="cuda")
    scale = torch.exp(torch.rand((rows, 1), generator=gen, device="cuda") * 1.8 - 0.7)
    token = torch.empty(rows, dtype=torch.int64, device="cuda")
    logs = torch.empty((3, rows), dtype=torch.float64, device="cuda")
    for a, b in _parts(rows, max(1, (1 << 26) // vocab)):
        z = torch.randn((b - a, vocab), generator=gen, device="cuda").add_(profile).mul_(scale[a:b])
        z = z.to(dtype)
        x[a:b] = z
        z = z.float()
        for i, noise in enumerate((0.0, 0.15, 0.4)):
            t = z if not noise else z + noise * scale[a:b] * torch.randn(
                z.shape, generator=gen, device="cuda")
            if i == 1:
                e = torch.rand(z.shape, generator=gen, device="cuda").clamp_(min=1e-30).log_().neg_()
                token[a:b] = (t / tau - e.log_()).argmax(1)
                del e
            if i == 0:
                continue
            logs[i, a:b] = _token_log(t, token[a:b], tau)
        logs[0, a:b] = _token_log(z, token[a:b], tau)
    return x, token.int(), logs


def _token_log(z, token, tau):
    z = z / tau
    m = z.amax(1, keepdim=True)
    total = torch.exp(z - m).sum(1, dtype=torch.float64)
    return z.gather(1, token[:, None])[:, 0].double() - m[:, 0].double() - torch.log(total)


def _loss_scale(dtype):
    return 4096.0 if dtype == torch.float16 else 1.0   # fp16 gradients need the loss scaled up


def _unused(token, share, gen):
    if share:
        token[torch.rand(token.shape, generator=gen, device="cuda") < share] = -1
    return token


def _sizes(case):
    """The tensors' sizes: those of one of this repository's models, or drawn."""
    models = {"tiny": (2, 64, 176, 256, 10), "b": (12, 768, 2048, 16384, 1000),
              "xl": (36, 1280, 3456, 16384, 1000)}
    if case["sizes"] in models:
        n, d, f, vocab, classes = models[case["sizes"]]
        layer = [d, 3 * d * d, d * d, d, f * d, f * d, d * f]
        return [vocab * d, (classes + 1) * d] + layer * n + [d, vocab * d]
    rng = random.Random(case["sizes"])
    return [_log(rng, 1, case["largest"]) for _ in range(case["tensors"] - 1)] + [case["largest"]]


def _buckets(sizes, types):
    """A flat buffer for each type, and the tensors as its parts."""
    flats = {t: torch.empty(sum(n for n, u in zip(sizes, types) if u == t), dtype=t, device="cuda")
             for t in dict.fromkeys(types)}
    at, parts = dict.fromkeys(flats, 0), []
    for n, t in zip(sizes, types):
        parts.append(flats[t][at[t]:at[t] + n])
        at[t] += n
    return list(flats.values()), parts


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    st = dict(case=case)
    dtype = TYPES[case["type"]]
    if case["kind"] == "norm":
        sizes = _sizes(case)
        # gains stay in 32 bits beside 16-bit matrices
        types = [dtype if n > 2048 else torch.float32 for n in sizes]
        spread = torch.exp(torch.randn(len(sizes), generator=gen, device="cuda") - 6).tolist()
        # a flat buffer for each type: where gradients are reduced, or what is clipped into
        flats, grads = _buckets(sizes, types)
        for g, t in zip(grads, spread):
            g.copy_(torch.randn(g.numel(), generator=gen, device="cuda").mul_(t))
        st["grads"] = grads if case["flat"] else [g.clone() for g in grads]
        if case["limit"]:
            if case["order"] == 2.0:
                total = math.sqrt(sum(n * s * s for n, s in zip(sizes, spread)))
            else:
                total = float(max(g.abs().amax().float() for g in st["grads"]))
            st["limit"] = case["limit"] * total
            st["flats"], st["out"] = _buckets(sizes, types)
        return st
    vocab, tau = case["vocab"], case["tau"]
    if case["kind"] == "preference":
        pairs, n = case["pairs"], case["length"]
        if case["packed"]:
            r = random.Random(seed)
            lengths = [r.randint(max(1, n // 2), n) for _ in range(2 * pairs)]
            first = [0]
            for v in lengths:
                first.append(first[-1] + v)
            st["first"] = torch.tensor(first, dtype=torch.int32, device="cuda")
            rows = 2 * pairs * n     # a buffer for the longest: the rows behind are padding
        else:
            st["first"], rows = None, 2 * pairs * n
        st["logits"], st["tokens"], logs = _rows(rows, vocab, dtype, tau, gen)
        st["tokens"] = _unused(st["tokens"], case["unused"], gen)
        st["ref"] = logs[2].float()
        st["weight"] = (torch.rand(pairs, generator=gen, device="cuda") + 0.5) * (
            _loss_scale(dtype) / pairs)
        st["beta"] = 0.1 if not case["mean"] else 2.0
        return st
    rows = case["rows"]
    st["logits"], st["tokens"], logs = _rows(rows, vocab, dtype, tau, gen)
    old = logs[1].float()
    if case["kind"] == "policy" and case["old"]:
        # the gradient jumps where the ratio meets a bound: either side is right there,
        # so no row lies closer to it than rounding reaches
        rho = torch.exp(logs[0] - old.double())
        for bound in (0.8, 1.0 + case["high"]):
            old = torch.where((rho - bound).abs() < 1e-4, old + 1e-3, old)
    st["tokens"] = _unused(st["tokens"], case["unused"], gen)
    st["weight"] = (torch.rand(rows, generator=gen, device="cuda") + 0.5) * (
        _loss_scale(dtype) / rows)
    if case["kind"] == "logprob":
        st["entropy_weight"] = 0.01 * st["weight"]
        return st
    st["old"] = old if case["old"] else None
    st["ref"] = logs[2].float()
    st["advantage"] = torch.randn(rows, generator=gen, device="cuda")
    return st


# ------------------------------------------------------------------ plain forms

def _row_plain(z, tokens, tau):
    """log p of every entry, p, l and H; rows without a token as if it were 0."""
    y = z.float() / tau
    log_p = y - y.amax(1, keepdim=True)
    log_p = log_p - torch.log(torch.exp(log_p).sum(1, keepdim=True))
    p = torch.exp(log_p)
    at = tokens.long().clamp(min=0)[:, None]
    return log_p, p, at, log_p.gather(1, at)[:, 0], -(p * log_p).sum(1)


def _grad_plain(log_p, p, at, entropy, a, b, tau, dtype):
    """The gradient of a l + b H."""
    grad = -(a[:, None] * p)
    grad.scatter_add_(1, at, a[:, None])
    if b is not None:
        grad = grad - b[:, None] * p * (log_p + entropy[:, None])
    return (grad / tau).to(dtype)


def _logprob_plain(st, case):
    z, tokens = st["logits"], st["tokens"]
    log_p, p, at, l, entropy = _row_plain(z, tokens, case["tau"])
    used = tokens >= 0
    zero = torch.zeros_like(l)
    out = [torch.where(used, l, zero)]
    if case["entropy"]:
        out.append(torch.where(used, entropy, zero))
    if case["grad"]:
        a = torch.where(used, st["weight"], zero)
        b = torch.where(used, st["entropy_weight"], zero) if case["entropy"] else None
        out.append(_grad_plain(log_p, p, at, entropy, a, b, case["tau"], z.dtype))
    return tuple(out)


def _policy_plain(st, case):
    z, tokens = st["logits"], st["tokens"]
    log_p, p, at, l, entropy = _row_plain(z, tokens, case["tau"])
    used = tokens >= 0
    zero = torch.zeros_like(l)
    ll = l.double()
    adv = st["advantage"].double()
    rho = torch.exp(ll - st["old"].double()) if st["old"] is not None else torch.ones_like(ll)
    bounded = rho.clamp(0.8, 1.0 + case["high"])
    loss = -torch.minimum(rho * adv, bounded * adv)
    flows = torch.where(adv > 0, rho <= 1.0 + case["high"], rho >= 0.8)
    a = torch.where(flows, -rho * adv, torch.zeros_like(rho))
    if case["kl"]:
        d = st["ref"].double() - ll
        loss = loss + case["kl"] * (torch.exp(d) - d - 1.0)
        a = a + case["kl"] * (1.0 - torch.exp(d))
    b = None
    w = torch.where(used, st["weight"], zero)
    if case["entropy"]:
        loss = loss - case["entropy"] * entropy.double()
        b = -case["entropy"] * w
    out = [loss.float() * w,
           _grad_plain(log_p, p, at, entropy, a.float() * w, b, case["tau"], z.dtype),
           torch.where(used, l, zero)]
    if case["entropy"]:
        out.append(torch.where(used, entropy, zero))
    return tuple(out)


def _sequence_of(st, rows, pairs):
    """Each row's sequence, 2 * pairs for rows behind the last."""
    row = torch.arange(rows, device="cuda")
    if st["first"] is None:
        return row // (rows // (2 * pairs))
    return torch.searchsorted(st["first"][1:].long(), row, right=True)


def _preference_plain(st, case):
    z, tokens, tau = st["logits"], st["tokens"], case["tau"]
    pairs, beta = case["pairs"], st["beta"]
    log_p, p, at, l, entropy = _row_plain(z, tokens, tau)
    seq = _sequence_of(st, z.shape[0], pairs)
    used = (tokens >= 0) & (seq < 2 * pairs)
    ratio = torch.where(used, l.double() - st["ref"].double(), 0.0)
    s = torch.zeros(2 * pairs + 1, dtype=torch.float64, device=z.device).index_add_(0, seq, ratio)
    count = torch.zeros_like(s).index_add_(0, seq, used.double()).clamp(min=1)
    if case["mean"]:
        s = s / count
    u = s[0:2 * pairs:2] - s[1:2 * pairs:2]
    h = beta * u
    if case["form"] == "sigmoid":
        loss = torch.log(1.0 + torch.exp(-h.abs())) + (-h).clamp(min=0)
        du = -beta / (1.0 + torch.exp(h))
    elif case["form"] == "hinge":
        loss = (1.0 - h).clamp(min=0)
        du = torch.where(h < 1.0, -beta, 0.0).double()
    else:
        loss = (u - 0.5 / beta) ** 2
        du = 2.0 * (u - 0.5 / beta)
    w = st["weight"].double()
    c = torch.zeros_like(s)
    c[0:2 * pairs:2], c[1:2 * pairs:2] = du * w, -du * w
    if case["mean"]:
        c = c / count
    a = torch.where(used, c[seq], 0.0).float()
    return (loss * w).float(), _grad_plain(log_p, p, at, None, a, None, tau, z.dtype), \
        s[:-1].float()


def _norm_plain(st, case):
    grads = st["grads"]
    if case["order"] == 2.0:
        parts = [(g.float() * g.float()).sum(dtype=torch.float64) for g in grads]
        norm = torch.sqrt(torch.stack(parts).sum()).float()
    else:
        norm = torch.stack([g.float().abs().amax() for g in grads]).amax()
    if not case["limit"]:
        return norm
    scale = torch.where(norm > st["limit"], st["limit"] / norm, torch.ones_like(norm))
    for g, out in zip(grads, st["out"]):
        out.copy_(g.float() * scale)
    return norm, st["flats"]


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        return _own(st, case, kind)
    if kind == "logprob":
        return _logprob_plain(st, case)
    if kind == "policy":
        return _policy_plain(st, case)
    if kind == "preference":
        return _preference_plain(st, case)
    return _norm_plain(st, case)


def _own(st, case, kind):
    import paper_2608_18183_amd as hb
    if kind == "logprob":
        if case["grad"]:
            out = hb.hbsjd_logprob_rows(
                st["logits"], st["tokens"], temperature=case["tau"], entropy=case["entropy"],
                logprob_weight=st["weight"], grad=True,
                entropy_weight=st["entropy_weight"] if case["entropy"] else None)
        else:
            out = hb.hbsjd_logprob_rows(st["logits"], st["tokens"], temperature=case["tau"],
                                        entropy=case["entropy"])
        return tuple(t for t in out if t is not None)
    if kind == "policy":
        out = hb.hbsjd_policy_rows(
            st["logits"], st["tokens"], st["advantage"], old_logprob=st["old"],
            ref_logprob=st["ref"] if case["kl"] else None, temperature=case["tau"], clip_low=0.2,
            clip_high=case["high"], kl_weight=case["kl"], entropy_weight=case["entropy"],
            row_weight=st["weight"])
        return tuple(t for t in out if t is not None)
    if kind == "preference":
        return hb.hbsjd_preference_rows(
            st["logits"], st["tokens"], first=st["first"],
            pairs=case["pairs"] if st["first"] is None else None, ref_logprob=st["ref"],
            temperature=case["tau"], beta=st["beta"], form=case["form"], mean=case["mean"],
            pair_weight=st["weight"])
    if case["limit"]:
        norm = hb.hbsjd_clip_grads(st["grads"], st["limit"], order=case["order"], out=st["out"])
        return norm, st["flats"]
    return hb.hbsjd_grad_norm(st["grads"], order=case["order"])


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "norm":
        grads = st["grads"]
        if case["order"] == 2.0:
            norm = torch.linalg.vector_norm(
                torch.stack([torch.linalg.vector_norm(g.double()) for g in grads]))
        else:
            norm = max(g.abs().max().double() for g in grads)
        if not case["limit"]:
            return norm
        scale = min(1.0, st["limit"] / float(norm))
        # laid out as the buffers they are clipped into
        return norm, [torch.cat([g.double() * scale for g in grads if g.dtype == f.dtype])
                      for f in st["flats"]]
    if case["kind"] == "preference":
        return _preference_exact(case, st)
    f = _logprob_exact if case["kind"] == "logprob" else _policy_exact
    step = max(1, (1 << 26) // case["vocab"])
    parts = [f(case, st, a, b) for a, b in _parts(case["rows"], step)]
    return tuple(torch.cat([p[i] for p in parts]) for i in range(len(parts[0])))


def _leaf(st, a, b, tau):
    """Rows a to b as a leaf in 64 bits; their tokens' log-probabilities and their
    entropies, 0 where there is no token."""
    z = st["logits"][a:b].double().requires_grad_()
    log_p = torch.log_softmax(z / tau, dim=1)
    tok = st["tokens"][a:b].long()
    used = tok >= 0
    l = log_p[torch.arange(b - a, device=z.device), tok.clamp(min=0)] * used
    return z, l, -(log_p.exp() * log_p).sum(1) * used, used


def _logprob_exact(case, st, a, b):
    z, l, entropy, _ = _leaf(st, a, b, case["tau"])
    out = [l.detach()] + ([entropy.detach()] if case["entropy"] else [])
    if case["grad"]:
        total = (st["weight"][a:b].double() * l).sum()
        if case["entropy"]:
            total = total + (st["entropy_weight"][a:b].double() * entropy).sum()
        out.append(torch.autograd.grad(total, z)[0])
    return out


def _policy_exact(case, st, a, b):
    z, l, entropy, used = _leaf(st, a, b, case["tau"])
    adv = st["advantage"][a:b].double()
    rho = torch.exp(l - (st["old"][a:b].double() if st["old"] is not None else l.detach()))
    bound = torch.where(adv > 0, torch.full_like(adv, 1.0 + case["high"]), torch.full_like(adv, 0.8))
    beyond = torch.where(adv > 0, rho > bound, rho < bound)
    loss = -adv * torch.where(beyond, bound, rho)
    if case["kl"]:
        d = st["ref"][a:b].double() - l
        loss = loss + case["kl"] * (torch.expm1(d) - d)
    loss = (loss - case["entropy"] * entropy) * used * st["weight"][a:b].double()
    grad, = torch.autograd.grad(loss.sum(), z)
    out = [loss.detach(), grad, l.detach()]
    return out + ([entropy.detach()] if case["entropy"] else [])


def _preference_exact(case, st):
    pairs, vocab, beta = case["pairs"], case["vocab"], st["beta"]
    rows = st["logits"].shape[0]
    if st["first"] is None:
        first = [i * (rows // (2 * pairs)) for i in range(2 * pairs + 1)]
    else:
        first = st["first"].tolist()
    grad = torch.zeros((rows, vocab), dtype=torch.float64, device="cuda")
    losses, ratios = [], []
    step = max(1, (1 << 27) // vocab)
    for i in range(pairs):
        ends = first[2 * i:2 * i + 3]
        s, counts = [], []
        for a, b in zip(ends, ends[1:]):
            n = max(1, int((st["tokens"][a:b] >= 0).sum()))
            total = torch.zeros((), dtype=torch.float64, device="cuda")
            for c, d in _parts(b - a, step):
                with torch.no_grad():
                    _, l, _, used = _leaf(st, a + c, a + d, case["tau"])
                total = total + (l - st["ref"][a + c:a + d].double() * used).sum()
            counts.append(n if case["mean"] else 1)
            s.append(total / counts[-1])
        u = (s[0] - s[1]).requires_grad_()
        if case["form"] == "sigmoid":
            loss = torch.nn.functional.softplus(-beta * u)
        elif case["form"] == "hinge":
            loss = torch.relu(1.0 - beta * u)
        else:
            loss = (u - 1.0 / (2.0 * beta)) ** 2
        loss = loss * st["weight"][i].double()
        du, = torch.autograd.grad(loss, u)
        for sign, n, a, b in zip((1.0, -1.0), counts, ends, ends[1:]):
            for c, d in _parts(b - a, step):
                z, l, _, _ = _leaf(st, a + c, a + d, case["tau"])
                grad[a + c:a + d], = torch.autograd.grad(l.sum() * (du * sign / n), z)
        losses.append(loss.detach())
        ratios += s
    return torch.stack(losses), grad, torch.stack(ratios)


# ------------------------------------------------------------------ work

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["type"]]
    if case["kind"] == "norm":
        total = _sizes(case)
        count = sum(total)
        moved = sum(n * (size if n > 2048 else 4) for n in total)
        # the tensors once; where they are clipped, their scaled values too
        return {"bytes": moved * (2 if case["limit"] else 1),
                "flops": count * (3 if case["limit"] else 2)}
    vocab = case["vocab"]
    if case["kind"] == "preference":
        rows, written = 2 * case["pairs"] * case["length"], True
        used = rows * (0.75 if case["packed"] else 1.0)
    else:
        rows, written = case["rows"], case["kind"] == "policy" or case["grad"]
        used = rows
    # rows without a token are not read, their gradient is written
    read = used * (1.0 - case["unused"]) * vocab * size
    per_row = {"logprob": 20, "policy": 28, "preference": 8}[case["kind"]]
    return {"bytes": int(read + (rows * vocab * size if written else 0) + rows * per_row),
            "flops": int((8 if written else 4) * used * vocab)}
