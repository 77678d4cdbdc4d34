"""The row operators around a distillation step, with inputs, a plain form of
each in elementary torch operations, and their values in 64 bits.

Three calls, all on rows of logits:

* `top`: a teacher's answer in short form: each row's K largest logits in
  descending order (the lowest index first among equals), their indices, and the
  log of the mass that the other entries have at the distillation's temperature.
* `distill`: the divergence of a student's full rows from such an answer, and
  its gradient by the student's logits. With tau the temperature, p the teacher
  and q the student, both over the K listed entries and one class for all the
  others (without the rest's mass: p over the K entries alone),
      L = w (alpha KL(p || q) + beta KL(q || p)),
  alpha = beta = 1/2 being the bidirectional divergence that this repository
  scores rollouts with.
* `adjust`: what is done to logits before a draw: penalties for tokens that the
  row's sequence holds already, biases on listed tokens, and a mask of the tokens
  that may follow.

Sizes follow this repository's workloads (vocabulary 16384, 16x16 and 24x24
grids, windows of 16 to 32 drafts, top-k 2000) and generic larger vocabularies.
"""
import math

import torch

own = False   # False: the plain forms; True: the framework's operators

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the teacher's answer for one position: launch and latency
        dict(name="top_one_row", kind="top", rows=1, vocab=16384, k=32, type="f32", tau=1.0),
        # a finished batch of the B workload: every generated position of 32 images
        dict(name="top_b_batch", kind="top", rows=6144, vocab=16384, k=64, type="f32", tau=1.0),
        # as many answers as the samplers' top-k keeps, 16-bit logits (many ties)
        dict(name="top_2000", kind="top", rows=1088, vocab=16384, k=2000, type="bf16", tau=1.0),
        # a language model's vocabulary of odd size, a batch of few long rows
        dict(name="top_wide", kind="top", rows=48, vocab=128257, k=128, type="bf16", tau=2.0),
        # one window of drafts: W + 1 rows, latency
        dict(name="distill_window", kind="distill", rows=17, vocab=16384, k=64, type="f32",
             tau=1.0, alpha=0.5, beta=0.5, rest=True, prefix=0.0),
        # the training step on a finished B batch, the bidirectional divergence
        dict(name="distill_b_batch", kind="distill", rows=6144, vocab=16384, k=64, type="f32",
             tau=1.0, alpha=0.5, beta=0.5, rest=True, prefix=0.0),
        # whole sequences of the 24x24 grid with their real prefixes weighted out,
        # 16-bit logits, the forward divergence from a renormalised answer
        dict(name="distill_l_sequences", kind="distill", rows=18432, vocab=16384, k=256,
             type="bf16", tau=2.0, alpha=1.0, beta=0.0, rest=False, prefix=0.25),
        # a language model's vocabulary of odd size, a batch of few long rows
        dict(name="distill_wide", kind="distill", rows=64, vocab=128257, k=128, type="f16",
             tau=1.0, alpha=0.5, beta=0.5, rest=True, prefix=0.0),
        # one row before its draw, a sequence half done
        dict(name="adjust_one_row", kind="adjust", rows=1, vocab=16384, history=288, biases=16,
             mask=True, penalties=True, type="f32", out="f32"),
        # the rows of a stress round, every one against a 24x24 sequence
        dict(name="adjust_stress", kind="adjust", rows=6400, vocab=16384, history=576, biases=0,
             mask=False, penalties=True, type="f32", out="f32"),
        # 16-bit rows of an XL round widened for the sampler, masked and biased
        dict(name="adjust_xl_masked", kind="adjust", rows=4224, vocab=16384, history=256,
             biases=64, mask=True, penalties=True, type="bf16", out="f32"),
        # a language model's vocabulary of odd size and long histories
        dict(name="adjust_wide", kind="adjust", rows=64, vocab=128257, history=4096, biases=300,
             mask=True, penalties=True, type="bf16", out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["top", "distill", "adjust"])
    vocab = rng.choice([16384, _log(rng, 32, 16384), _log(rng, 16384, 200000)])
    most = {"top": 6144, "distill": 6144, "adjust": 4224}[kind] * 16384
    rows = _log(rng, 1, max(1, min(most // vocab, 16384)))
    case = dict(kind=kind, rows=rows, vocab=vocab, type=rng.choice(["f32", "bf16", "f16"]))
    if kind == "top":
        return dict(case, k=_log(rng, 1, min(vocab, 2048)), tau=rng.choice([0.5, 1.0, 2.0, 4.0]))
    if kind == "distill":
        rest = rng.random() < 0.6
        alpha, beta = rng.choice([(0.5, 0.5), (1.0, 0.0), (0.0, 1.0), (0.9, 0.1)]) if rest else (1.0, 0.0)
        return dict(case, k=_log(rng, 1, min(vocab // 2, 512)), tau=rng.choice([0.7, 1.0, 2.0]),
                    alpha=alpha, beta=beta, rest=rest, prefix=rng.choice([0.0, 0.25]))
    case["history"] = rng.choice([0, _log(rng, 1, 4096)])
    return dict(case, biases=rng.choice([0, _log(rng, 1, min(vocab, 512))]),
                mask=rng.random() < 0.6, penalties=case["history"] > 0,
                out=rng.choice(["f32", case["type"]]))


# ------------------------------------------------------------------ inputs

def _logits(rows, vocab, gen, scale=None):
    """Rows as a decoder's head gives them: noise over a common profile of the
    tokens, some rows nearly flat and some peaked."""
    x = torch.randn((rows, vocab), generator=gen, device="cuda")
    x += torch.randn(vocab, generator=gen, device="cuda")
    if scale is None:
        scale = torch.exp(torch.rand((rows, 1), generator=gen, device="cuda") * 1.8 - 0.7)
    return x.mul_(scale), scale


def _parts(total, size):
    return [(a, min(a + size, total)) for a in range(0, total, size)]


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    dtype = TYPES[case["type"]]
    st = dict(case=case)
    if case["kind"] == "top":
        st["logits"] = _logits(rows, vocab, gen)[0].to(dtype)
        return st
    if case["kind"] == "distill":
        x, scale = _logits(rows, vocab, gen)
        k = case["k"]
        values = torch.empty((rows, k), device="cuda")
        index = torch.empty((rows, k), dtype=torch.int32, device="cuda")
        rest = torch.empty(rows, device="cuda")
        # the teacher agrees with the student up to noise
        for a, b in _parts(rows, max(1, (1 << 26) // vocab)):
            t = x[a:b] + 0.7 * scale[a:b] * torch.randn((b - a, vocab), generator=gen, device="cuda")
            v, i = torch.topk(t, k, dim=1)
            values[a:b], index[a:b] = v, i.int()
            t.scatter_(1, i, -math.inf)
            rest[a:b] = torch.logsumexp(t / case["tau"], dim=1)
        weight = torch.rand(rows, generator=gen, device="cuda") + 0.5
        if case["prefix"]:
            weight[torch.rand(rows, generator=gen, device="cuda") < case["prefix"]] = 0.0
        # the mean over the rows; fp16 gradients need the loss scaled up
        weight *= (4096.0 if dtype == torch.float16 else 1.0) / rows
        st.update(logits=x.to(dtype), values=values, index=index,
                  rest=rest if case["rest"] else None, weight=weight)
        return st
    st["logits"] = _logits(rows, vocab, gen)[0].to(dtype)
    st.update(tokens=None, count=None, repetition=None, presence=None, frequency=None,
              bias_index=None, bias_value=None, mask=None, mask_row=None)
    if case["history"]:
        h = case["history"]
        # sequences repeat themselves: half of the tokens from a small set
        tok = torch.randint(0, vocab, (rows, h), generator=gen, device="cuda")
        few = torch.randint(0, max(1, vocab // 64), (rows, h), generator=gen, device="cuda")
        pick = torch.rand((rows, h), generator=gen, device="cuda") < 0.5
        st["tokens"] = torch.where(pick, few, tok).int()
        st["count"] = torch.randint(h // 2, h + 1, (rows,), generator=gen, device="cuda").int()
        st["repetition"] = 1.0 + torch.rand(rows, generator=gen, device="cuda") * 0.5
        st["presence"] = torch.rand(rows, generator=gen, device="cuda")
        st["frequency"] = torch.rand(rows, generator=gen, device="cuda") * 0.3
    if case["biases"]:
        n = case["biases"]
        pick = torch.rand(vocab, generator=gen, device="cuda").argsort()[:n]
        shift = torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda")
        st["bias_index"] = ((pick[None, :] + shift) % vocab).int()
        st["bias_value"] = torch.randn((rows, n), generator=gen, device="cuda") * 3
    if case["mask"]:
        # a grammar's states: some let a few tokens follow, some nearly all
        states = min(64, rows)
        keep = torch.rand((states, 1), generator=gen, device="cuda") ** 3
        words = (vocab + 31) // 32
        allowed = torch.rand((states, words * 32), generator=gen, device="cuda") < keep
        allowed[:, 0] = True
        bits = allowed.view(states, words, 32).long() << torch.arange(32, device="cuda")
        st["mask"] = _int32(bits.sum(-1))
        st["mask_row"] = torch.randint(-1, states, (rows,), generator=gen, device="cuda").int()
    return st


def _int32(word):
    """The low 32 bits of an int64 as an int32."""
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int()


# ------------------------------------------------------------------ plain forms

def _top_plain(z, k, tau):
    # one ordered integer per entry: its value first, then the lower index, so
    # that no two entries of a row are equal
    x = z.float()
    n = x.shape[1]
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF)
    key = key * n + torch.arange(n - 1, -1, -1, device=x.device)
    index = n - 1 - torch.topk(key, k, dim=1).values % n
    values = x.gather(1, index)
    rest = (x / tau).scatter(1, index, -math.inf)
    m = rest.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    return values, index.int(), torch.log(torch.exp(rest - m).sum(1)) + m[:, 0]


def _distill_plain(z, values, index, rest, weight, tau, alpha, beta):
    y = z.float() / tau
    q_log = y - y.amax(1, keepdim=True)
    q_log = q_log - torch.log(torch.exp(q_log).sum(1, keepdim=True))
    q = torch.exp(q_log)
    idx = index.long()
    t = values / tau
    if rest is not None:
        t = torch.cat([t, rest[:, None]], 1)
    p_log = t - t.amax(1, keepdim=True)
    p_log = p_log - torch.log(torch.exp(p_log).sum(1, keepdim=True))
    k_log = q_log.gather(1, idx)
    if rest is not None:
        others = torch.log(q.scatter(1, idx, 0.0).sum(1, keepdim=True))
        k_log = torch.cat([k_log, others], 1)
    p, k_q = torch.exp(p_log), torch.exp(k_log)
    loss = alpha * (p * (p_log - k_log)).sum(1)
    # by the logits: q_v a_v, less p_v at the listed entries; a_v holds what the
    # class of v has in common
    c = k_log - p_log
    reverse = (k_q * c).sum(1, keepdim=True)
    if beta:
        loss = loss + beta * reverse[:, 0]
    part = alpha * (1.0 - p / k_q) + beta * (c - reverse)
    if rest is not None:
        a = part[:, -1:].expand_as(q).clone()
        part = part[:, :-1]
    else:
        a = torch.full_like(q, alpha)
    # at the listed entries alpha (q - p) without the quotient
    grad = q * a
    kept = q.gather(1, idx)
    n = idx.shape[1]
    grad.scatter_(1, idx, alpha * (kept - p[:, :n]) + beta * kept * (c[:, :n] - reverse))
    w = weight[:, None]
    return loss * weight, (grad * (w / tau)).to(z.dtype)


def _allowed(mask, vocab):
    bit = torch.arange(32, device=mask.device, dtype=torch.int32)
    return ((mask[:, :, None] >> bit) & 1).view(mask.shape[0], -1)[:, :vocab].bool()


def _adjust_plain(st, out):
    z = st["logits"]
    rows, vocab = z.shape
    x = z.float()
    if st["tokens"] is not None:
        h = st["tokens"].shape[1]
        held = torch.arange(h, device=z.device)[None, :] < st["count"][:, None]
        count = torch.zeros((rows, vocab), device=z.device)
        count.scatter_add_(1, st["tokens"].long(), held.float())
        seen = count > 0
        theta = st["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / theta, x * theta), x)
        x = x - st["frequency"][:, None] * count
        x = x - st["presence"][:, None] * seen
    if st["bias_index"] is not None:
        x = x.scatter_add(1, st["bias_index"].long(), st["bias_value"])
    if st["mask"] is not None:
        which = st["mask_row"].long()
        ok = _allowed(st["mask"], vocab)[which.clamp(min=0)] | (which < 0)[:, None]
        x = torch.where(ok, x, torch.full_like(x, -math.inf))
    return x.to(out)


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        import paper_2608_18183_amd as hb
        if kind == "top":
            return hb.hbsjd_top_logits_rows(st["logits"], case["k"], temperature=case["tau"])
        if kind == "distill":
            return hb.hbsjd_distill_top_rows(
                st["logits"], st["values"], st["index"], st["rest"], temperature=case["tau"],
                forward_weight=case["alpha"], reverse_weight=case["beta"], row_weight=st["weight"])
        return hb.hbsjd_adjust_rows(
            st["logits"], tokens=st["tokens"], token_count=st["count"],
            repetition=st["repetition"], presence=st["presence"], frequency=st["frequency"],
            bias_index=st["bias_index"], bias_value=st["bias_value"], mask=st["mask"],
            mask_row=st["mask_row"], out_dtype=TYPES[case["out"]])
    if kind == "top":
        return _top_plain(st["logits"], case["k"], case["tau"])
    if kind == "distill":
        return _distill_plain(st["logits"], st["values"], st["index"], st["rest"], st["weight"],
                              case["tau"], case["alpha"], case["beta"])
    return _adjust_plain(st, TYPES[case["out"]])


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    step = max(1, (1 << 26) // case["vocab"])
    f = {"top": _top_exact, "distill": _distill_exact, "adjust": _adjust_exact}[case["kind"]]
    parts = [f(case, st, a, b) for a, b in _parts(case["rows"], step)]
    if case["kind"] == "adjust":
        return torch.cat(parts)
    return tuple(torch.cat([p[i] for p in parts]) for i in range(len(parts[0])))


def _top_exact(case, st, a, b):
    z = st["logits"][a:b].double()
    v, order = torch.sort(z, dim=1, descending=True, stable=True)
    k = case["k"]
    if k == z.shape[1]:
        rest = torch.full((b - a,), -math.inf, dtype=torch.float64, device=z.device)
    else:
        rest = torch.logsumexp(v[:, k:] / case["tau"], dim=1)
    return v[:, :k], order[:, :k].int(), rest


def _distill_exact(case, st, a, b):
    """Over all entries at once: every entry carries its class's probability."""
    z = st["logits"][a:b].double() / case["tau"]
    log_q = torch.log_softmax(z, dim=1)
    idx = st["index"][a:b].long()
    listed_ = torch.zeros_like(z, dtype=torch.bool).scatter_(1, idx, True)
    t = st["values"][a:b].double() / case["tau"]
    rest = None if st["rest"] is None else st["rest"][a:b, None].double()
    total = torch.logsumexp(t if rest is None else torch.cat([t, rest], 1), 1, keepdim=True)
    log_p = t - total
    at = log_q.gather(1, idx)
    w = st["weight"][a:b, None].double()
    alpha, beta = case["alpha"], case["beta"]
    p = log_p.exp()
    forward = (p * (log_p - at)).sum(1, keepdim=True)
    grad = log_q.exp() * alpha
    grad.scatter_add_(1, idx, -alpha * p)
    if rest is not None:
        log_p0 = rest - total
        log_q0 = torch.logsumexp(log_q.masked_fill(listed_, -math.inf), 1, keepdim=True)
        forward = forward + log_p0.exp() * (log_p0 - log_q0)
        # the class of the others: p0 spread over them as the student spreads it
        grad -= (alpha * (log_p0 + log_q - log_q0).exp()).masked_fill(listed_, 0.0)
        ratio = (log_q0 - log_p0).expand_as(z).scatter(1, idx, at - log_p)
        reverse = (log_q.exp() * ratio).sum(1, keepdim=True)
        grad += beta * log_q.exp() * (ratio - reverse)
        forward = forward * alpha + reverse * beta
    else:
        forward = forward * alpha
    return (w * forward)[:, 0], grad * (w / case["tau"])


def _adjust_exact(case, st, a, b):
    x = st["logits"][a:b].double()
    rows, vocab = x.shape
    row = torch.arange(rows, device=x.device)[:, None]
    if st["tokens"] is not None:
        tok, n = st["tokens"][a:b].long(), st["count"][a:b, None].long()
        kept = torch.arange(tok.shape[1], device=x.device)[None] < n
        flat = (row * vocab + tok)[kept]
        times = torch.bincount(flat, minlength=rows * vocab).view(rows, vocab).double()
        rep = st["repetition"][a:b, None].double()
        x = torch.where(times > 0, torch.where(x > 0, x / rep, x * rep), x)
        x = x - times * st["frequency"][a:b, None].double()
        x = x - (times > 0) * st["presence"][a:b, None].double()
    if st["bias_index"] is not None:
        x.index_put_((row.expand_as(st["bias_index"][a:b]), st["bias_index"][a:b].long()),
                     st["bias_value"][a:b].double(), accumulate=True)
    if st["mask"] is not None:
        v = torch.arange(vocab, device=x.device)
        which = st["mask_row"][a:b].long()
        words = st["mask"].long()[which.clamp(min=0)][:, v // 32]
        barred = ((words >> (v % 32)) & 1 == 0) & (which >= 0)[:, None]
        x = x.masked_fill(barred, -math.inf)
    return x


# ------------------------------------------------------------------ work

def work(case):
    rows, vocab = case["rows"], case["vocab"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    entries = rows * vocab
    row_bytes = entries * size[case["type"]]
    if case["kind"] == "top":
        # the row once; an exponential, a sum and a comparison an entry
        return {"bytes": row_bytes + rows * (case["k"] * 8 + 4), "flops": 4 * entries}
    if case["kind"] == "distill":
        # rows of weight zero are not read
        read = row_bytes * (1.0 - case["prefix"])
        return {"bytes": int(read + row_bytes + rows * (case["k"] * 8 + 12)),
                "flops": 8 * entries}
    out = entries * size[case["out"]]
    lists = rows * (case["history"] * 3 + case["biases"] * 8 + 20)
    mask = min(64, rows) * ((vocab + 31) // 32) * 4 if case["mask"] else 0
    return {"bytes": row_bytes + out + lists + mask, "flops": 2 * entries}
