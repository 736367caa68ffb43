"""Measured operators on rows of logits over a vocabulary: a teacher's top
logits as (idx, val) lists, distillation on such lists (loss, gradient, both in
one pass), and the verification of drafted tokens.

A case is a dict of plain values; `op` names the call:

  top       TopLogitsPlan.execute: each row's k greatest logits, ascending, and
            the log-mass of the others
  forward   DistillPlan.forward: the loss of each row
  backward  DistillPlan.backward: the gradient, from forward's saved sums
  step      DistillPlan.step: loss and gradient
  verify    VerifyPlan.execute: accepted drafts, the token after them, log-probabilities

`own` False computes the operators in their plain form (elementary torch
operations in 32 bits), `own` True calls the package.

`pad` is the distance between two rows beyond the vocabulary (elements);
`banned` words at the end of each row are masked with -inf; `dead` is the share
of rows with weight 0 (their logits hold NaN, as rows of unused positions may);
`ragged` lists have 0 to k entries, ragged drafts 0 to `draft` tokens.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SPREAD = 3.0   # standard deviation of a row's logits at temperature 1
APART = 0.7    # standard deviation between a teacher's logits and its student's
ACCEPT = 0.73  # mean of sum(min(p, q)) at these two: the chance that a drafted token is accepted


def _rows(name, op, rows, vocab, k, dtype, temperature=1.0, val="f32", tail=True, ragged=False,
          dead=0.0, banned=0, pad=0):
    return dict(name=name, op=op, rows=rows, vocab=vocab, k=k, dtype=dtype,
                temperature=temperature, val=val, tail=tail, ragged=ragged, dead=dead,
                banned=banned, pad=pad)


def _verify(name, batch, draft, vocab, dtype, temperature=1.0, ragged=False, banned=0, pad=0):
    return dict(name=name, op="verify", batch=batch, draft=draft, vocab=vocab, dtype=dtype,
                temperature=temperature, ragged=ragged, banned=banned, pad=pad)


def listed():
    return [
        # a teacher behind a server answers for one token: launches and latency
        _rows("top_one_token", "top", 1, 32000, 16, "bf16"),
        # a teacher labels a batch of 8,192 tokens of the 32,000-word configuration
        _rows("top_batch", "top", 8192, 32000, 64, "bf16", temperature=2.0, val="f16"),
        # long lists from a wide vocabulary of an odd size, in 32 bits
        _rows("top_wide_f32", "top", 509, 131071, 256, "f32", banned=63),
        # evaluation: the loss alone over held-out tokens, some of them padding
        _rows("forward_eval", "forward", 4096, 32000, 64, "bf16", temperature=2.0, val="f16",
              dead=0.125),
        # the backward pass of a training step whose loss was taken before
        _rows("backward_train", "backward", 4096, 32000, 64, "bf16", temperature=2.0, val="f16",
              dead=0.125),
        # a training step of a few tokens in 32 bits
        _rows("step_few_tokens", "step", 16, 32000, 8, "f32"),
        # the ordinary training step of the 32,000-word configuration
        _rows("step_train", "step", 8192, 32000, 64, "bf16", temperature=2.0, val="f16"),
        # a wide vocabulary of an odd size, ragged lists without the others' mass,
        # logits that are a view of wider rows
        _rows("step_wide_ragged", "step", 1021, 131071, 128, "f16", tail=False, ragged=True,
              dead=0.0625, banned=63, pad=129),
        # one conversation, four drafted tokens
        _verify("verify_one", 1, 4, 32000, "bf16"),
        # a server's batch
        _verify("verify_batch", 64, 5, 32000, "bf16", temperature=0.8),
        # a wide vocabulary of an odd size in 32 bits, drafts of several lengths
        _verify("verify_wide_ragged", 37, 7, 131071, "f32", ragged=True, banned=63),
        # a large batch with long drafts
        _verify("verify_large", 256, 8, 65536, "f16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["f32", "f16", "bf16"])
    size = 4 if dtype == "f32" else 2
    vocab = rng.choice([32000, 65536, _log_int(rng, 1000, 131072), _log_int(rng, 1000, 131071) | 1])
    temperature = rng.choice([1.0, 1.0, 0.8, 2.0])
    banned = rng.choice([0, 0, 63, 500])
    pad = rng.choice([0, 0, 1, 64, 129])
    most = 8192 * 32000 * 2  # bytes of the largest listed case's logits
    if rng.random() < 0.3:
        draft = rng.randint(1, 8)
        batch = _log_int(rng, 1, min(256, most // (size * (2 * draft + 1) * (vocab + pad))))
        return dict(op="verify", batch=batch, draft=draft, vocab=vocab, dtype=dtype,
                    temperature=temperature, ragged=rng.random() < 0.5, banned=banned, pad=pad)
    op = rng.choice(["top", "top", "forward", "backward", "step", "step"])
    return dict(op=op, rows=_log_int(rng, 1, min(8192, most // (size * (vocab + pad)))),
                vocab=vocab, k=_log_int(rng, 1, 256), dtype=dtype, temperature=temperature,
                val=rng.choice(["f32", "f16"]), tail=rng.random() < 0.7,
                ragged=rng.random() < 0.4, dead=rng.choice([0.0, 0.0, 0.0625, 0.25]),
                banned=banned, pad=pad)


# ----------------------------------------------------------------------------
# inputs

def _view(x, pad):
    """x, laid out as a view of rows that are `pad` elements longer."""
    if not pad:
        return x
    wide = torch.zeros(*x.shape[:-1], x.shape[-1] + pad, dtype=x.dtype, device=x.device)
    wide[..., : x.shape[-1]] = x
    return wide[..., : x.shape[-1]]


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _teacher_lists(teacher, k, temperature):
    """Each row's k greatest (ascending positions), and the log-mass of the rest."""
    idx = teacher.topk(k, dim=1).indices.sort(dim=1).values
    val = teacher.gather(1, idx)
    rest = (teacher / temperature).scatter(1, idx, -math.inf)
    return idx.to(torch.int32), val, torch.logsumexp(rest, dim=1)


def _prepare_rows(c, gen):
    n, vocab, k, t = c["rows"], c["vocab"], c["k"], c["temperature"]
    words = vocab - c["banned"]
    dtype, val_dtype = DTYPES[c["dtype"]], DTYPES[c["val"]]
    teacher = _randn(gen, n, vocab) * (SPREAD * t)
    teacher[:, words:] = -math.inf
    st = {"op": c["op"], "k": k, "temperature": t, "val_dtype": val_dtype}
    if c["op"] == "top":
        st["logits"] = _view(teacher.to(dtype), c["pad"])
    else:
        idx, val, tail = _teacher_lists(teacher, k, t)
        student = teacher.add_(_randn(gen, n, vocab) * (APART * t)).to(dtype)
        st["idx"], st["val"] = idx, val.to(val_dtype)
        st["tail"] = tail if c["tail"] else None
        st["count"] = st["weight"] = None
        if c["ragged"]:
            st["count"] = torch.randint(0, k + 1, (n,), generator=gen, device=DEV,
                                        dtype=torch.int32)
        if c["dead"]:
            # one weight for a row of text; padding has none
            weight = torch.rand(n, generator=gen, device=DEV) + 0.5
            gone = torch.randperm(n, generator=gen, device=DEV)[: int(n * c["dead"])]
            weight[gone] = 0.0
            student[gone] = math.nan
            st["weight"] = weight
        st["logits"] = _view(student, c["pad"])
        if c["op"] == "backward":
            st["dloss"] = torch.rand(n, generator=gen, device=DEV) / n
            st["stats"] = None
    if own:
        import paper_2010_10458_amd as tk
        if c["op"] == "top":
            st["plan"] = tk.TopLogitsPlan(n, vocab, k, dtype=dtype, temperature=t,
                                          val_dtype=val_dtype)
        else:
            st["plan"] = tk.DistillPlan(n, vocab, k, dtype=dtype, temperature=t,
                                        val_dtype=val_dtype)
        if c["op"] == "backward":
            # a training program has run the forward pass before
            st["stats"] = st["plan"].forward(st["logits"], st["idx"], st["val"], tail=st["tail"],
                                             count=st["count"], weight=st["weight"])[1]
    elif c["op"] == "backward":
        st["stats"] = _plain_stats(st)
    return st


def _prepare_verify(c, gen):
    b, draft, vocab, t = c["batch"], c["draft"], c["vocab"], c["temperature"]
    words, dtype = vocab - c["banned"], DTYPES[c["dtype"]]
    target = _randn(gen, b, draft + 1, vocab) * (SPREAD * t)
    drafts = target[:, :draft] + _randn(gen, b, draft, vocab) * (APART * t)
    target[..., words:] = -math.inf
    drafts[..., words:] = -math.inf
    target, drafts = target.to(dtype), drafts.to(dtype)
    # the draft model's own samples from its distribution
    race = torch.rand(b, draft, vocab, generator=gen, device=DEV).clamp_(1e-20)
    tokens = (drafts.float() / t - torch.log(-torch.log(race))).argmax(dim=-1).to(torch.int32)
    st = {"op": "verify", "temperature": t, "target": _view(target, c["pad"]),
          "drafts": _view(drafts, c["pad"]), "tokens": tokens,
          "uniform": torch.rand(b, draft, generator=gen, device=DEV),
          "noise": torch.empty(b, vocab, device=DEV).exponential_(generator=gen).clamp_(1e-30),
          "length": None}
    if c["ragged"]:
        st["length"] = torch.randint(0, draft + 1, (b,), generator=gen, device=DEV,
                                     dtype=torch.int32)
    if own:
        import paper_2010_10458_amd as tk
        st["plan"] = tk.VerifyPlan(b, draft, vocab, dtype=dtype, temperature=t)
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    return _prepare_verify(case, gen) if case["op"] == "verify" else _prepare_rows(case, gen)


# ----------------------------------------------------------------------------
# the plain forms: elementary operations in 32 bits

def _plain_top(st):
    x, k = st["logits"].float(), st["k"]
    kth = x.topk(k, dim=1).values[:, -1:]
    above, at = x > kth, x == kth
    chosen = above | (at & (at.cumsum(1) <= k - above.sum(1, keepdim=True)))
    idx = chosen.nonzero()[:, 1].view(-1, k)
    val = st["logits"].gather(1, idx).to(st["val_dtype"])
    tail = _plain_lse((x / st["temperature"]).masked_fill(chosen, -math.inf))
    return idx.to(torch.int32), val, tail


def _plain_lse(x):
    m = x.amax(1)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    return m + torch.log(torch.exp(x - m[:, None]).sum(1))


def _plain_lists(st):
    """The list's places and mask, the teacher's probabilities, its rest, and their logarithms."""
    idx, k = st["idx"].long(), st["k"]
    used = torch.ones_like(idx, dtype=torch.bool)
    if st["count"] is not None:
        used = torch.arange(k, device=idx.device)[None] < st["count"][:, None]
    n, vocab = st["logits"].shape
    places = torch.where(used, idx, torch.full_like(idx, vocab))
    listed_ = torch.zeros(n, vocab + 1, dtype=torch.bool, device=idx.device)
    listed_ = listed_.scatter_(1, places, True)[:, :vocab]
    t = (st["val"].float() / st["temperature"]).masked_fill(~used, -math.inf)
    tail = st["tail"] if st["tail"] is not None else t.new_full((n,), -math.inf)
    lt = _plain_lse(torch.cat([t, tail[:, None]], 1))
    log_p, log_pr = t - lt[:, None], tail - lt
    return torch.where(used, idx, 0), places, listed_, torch.exp(log_p), torch.exp(log_pr), log_p, log_pr


def _plain_live(st):
    live = torch.ones(st["logits"].shape[0], dtype=torch.bool, device=DEV)
    if st["weight"] is not None:
        live = live & (st["weight"] != 0)
    if st["count"] is not None:
        live = live & (st["count"] > 0)
    return live


def _plain_scale(st):
    t = st["temperature"]
    return st["weight"] * t if st["weight"] is not None else t


def _plain_stats(st):
    """The student's log-sums over the whole row and over what the list leaves out."""
    z = st["logits"].float() / st["temperature"]
    listed_ = _plain_lists(st)[2]
    return _plain_lse(z), _plain_lse(z.masked_fill(listed_, -math.inf))


def _plain_loss(st):
    z = st["logits"].float() / st["temperature"]
    idx, _, listed_, p, pr, log_p, log_pr = _plain_lists(st)
    lz, lr = _plain_lse(z), _plain_lse(z.masked_fill(listed_, -math.inf))
    part = torch.where(p > 0, p * (log_p - (z.gather(1, idx) - lz[:, None])), 0.0).sum(1)
    part = part + torch.where(pr > 0, pr * (log_pr - (lr - lz)), 0.0)
    loss = part * _plain_scale(st) * st["temperature"]
    return torch.where(_plain_live(st), loss, 0.0), (lz, lr)


def _plain_grad(st, stats, dloss=None):
    z = st["logits"].float() / st["temperature"]
    _, places, listed_, p, pr, _, _ = _plain_lists(st)
    lz, lr = stats
    q = torch.exp(z - lz[:, None])
    rest = torch.where(pr > 0, 1.0 - pr * torch.exp(lz - lr), 1.0)
    g = torch.where(listed_, q, q * rest[:, None])
    g = torch.cat([g, torch.zeros_like(g[:, :1])], 1).scatter_add_(1, places, -p)[:, :-1]
    scale = _plain_scale(st) * torch.ones_like(lz) if dloss is None else _plain_scale(st) * dloss
    g = torch.where(_plain_live(st)[:, None], g * scale[:, None], 0.0)
    return g.to(st["logits"].dtype)


def _plain_softmax(x):
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e / total, 0.0)


def _plain_verify(st):
    p = _plain_softmax(st["target"].float() / st["temperature"])
    q = _plain_softmax(st["drafts"].float() / st["temperature"])
    tokens = st["tokens"].long()
    b, draft = tokens.shape
    at = torch.arange(draft, device=DEV)
    length = st["length"].long() if st["length"] is not None else torch.full((b,), draft, device=DEV)
    ps = p[:, :draft].gather(2, tokens[..., None])[..., 0]
    qs = q.gather(2, tokens[..., None])[..., 0]
    ok = (st["uniform"] * qs < ps) & (at < length[:, None])
    accepted = ok.long().cumprod(1).sum(1)
    each = torch.arange(b, device=DEV)
    pn, qn = p[each, accepted], q[each, accepted.clamp(max=draft - 1)]
    qn = torch.where((accepted < length)[:, None], qn, 0.0)
    r = (pn - qn).clamp(min=0.0)
    r = torch.where(r.amax(1, keepdim=True) > 0, r, pn)
    score = r / st["noise"]
    best = score.amax(1, keepdim=True)
    words = torch.arange(score.shape[1], device=DEV)
    last = torch.where(score == best, words, score.shape[1]).amin(1)
    last = torch.where(best[:, 0] > 0, last, -1)
    places = torch.arange(draft + 1, device=DEV)[None]
    out = torch.cat([tokens, tokens[:, :1]], 1)
    out = torch.where(places < accepted[:, None], out, -1)
    out = torch.where(places == accepted[:, None], last[:, None], out)
    logp = torch.log(p.gather(2, out.clamp(min=0)[..., None])[..., 0])
    return accepted.to(torch.int32), out.to(torch.int32), torch.where(out >= 0, logp, 0.0)


def run(state):
    st, op = state, state["op"]
    if not own:
        if op == "top":
            return _plain_top(st)
        if op == "forward":
            return _plain_loss(st)[0]
        if op == "backward":
            return _plain_grad(st, st["stats"], st["dloss"])
        if op == "step":
            loss, stats = _plain_loss(st)
            return loss, _plain_grad(st, stats)
        return _plain_verify(st)
    plan = st["plan"]
    if op == "top":
        return plan.execute(st["logits"])
    if op == "verify":
        return plan.execute(st["target"], st["drafts"], st["tokens"], st["uniform"], st["noise"],
                            length=st["length"])
    lists = dict(tail=st["tail"], count=st["count"], weight=st["weight"])
    if op == "forward":
        return plan.forward(st["logits"], st["idx"], st["val"], **lists)[0]
    if op == "backward":
        return plan.backward(st["logits"], st["idx"], st["val"], st["stats"], dloss=st["dloss"],
                             **lists)
    return plan.step(st["logits"], st["idx"], st["val"], **lists)


# ----------------------------------------------------------------------------

def work(case):
    """Each input read once and each output written once; 4 operations an
    element for a sum of exponentials (difference, exp, sum, and the maximum or
    comparison), 3 more for a gradient."""
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "verify":
        b, draft, vocab = c["batch"], c["draft"], c["vocab"]
        # rows up to the first rejection: a draft's position is reached with
        # probability ACCEPT^i, the row after the last one with ACCEPT^length
        lengths = range(draft + 1) if c["ragged"] else [draft]
        rows = sum(2 * sum(ACCEPT ** i for i in range(n)) + ACCEPT ** n for n in lengths)
        rows *= b / len(lengths)
        return {"bytes": rows * vocab * size + b * vocab * 4 + b * (draft * 8 + 4 + (draft + 1) * 8),
                "flops": rows * vocab * 4 + b * vocab * 6}
    n, vocab, k = c["rows"], c["vocab"], c["k"]
    ev = 4 if c["val"] == "f32" else 2
    lists = n * k * (4 + ev) + n * 4
    if c["op"] == "top":
        return {"bytes": n * vocab * size + lists, "flops": n * vocab * 4}
    live = n - int(n * c["dead"])
    if c["ragged"]:
        live *= k / (k + 1)
        lists /= 2
    data = live * vocab * size
    out = 0 if c["op"] == "forward" else n * vocab * size
    ops = {"forward": 4, "backward": 3, "step": 7}[c["op"]]
    return {"bytes": data + out + lists + n * 8, "flops": live * vocab * ops}


# ----------------------------------------------------------------------------
# the definitions in 64 bits, a block of rows at a time

def _blocks(n, vocab):
    step = max(1, (1 << 26) // vocab)
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


def _exact_top(st):
    val, tail = [], []
    for rows in _blocks(*st["logits"].shape):
        x = st["logits"][rows].double()
        order = x.sort(dim=1, descending=True, stable=True).indices
        first = order[:, : st["k"]].sort(dim=1).values
        val.append(x.gather(1, first))
        left = x.gather(1, order[:, st["k"]:]) / st["temperature"]
        tail.append(torch.logsumexp(left, 1) if left.shape[1] else
                    torch.full((x.shape[0],), -math.inf, device=DEV, dtype=torch.float64))
    val = torch.cat(val)
    return None, val.to(st["val_dtype"]).double(), torch.cat(tail)


def _exact_distill(st):
    """Loss and gradient of each row; the gradient from the loss as the cross
    entropy of k + 1 classes (each listed word, and all others as one)."""
    n, vocab = st["logits"].shape
    t, k = st["temperature"], st["k"]
    losses, grads = [], []
    for rows in _blocks(n, vocab):
        m = rows.stop - rows.start
        z = st["logits"][rows].double() / t
        idx = st["idx"][rows].long()
        count = st["count"][rows] if st["count"] is not None else torch.full((m,), k, device=DEV)
        weight = (st["weight"][rows].double() if st["weight"] is not None
                  else torch.ones(m, device=DEV, dtype=torch.float64))
        alive = (weight != 0) & (count > 0)
        z[~alive] = 0.0
        valid = torch.arange(k, device=DEV)[None] < count[:, None]
        minus = torch.full((m, 1), -math.inf, device=DEV, dtype=torch.float64)
        scores = (st["val"][rows].double() / t).masked_fill(~valid, -math.inf)
        other = st["tail"][rows].double()[:, None] if st["tail"] is not None else minus
        log_t = torch.cat([scores, other], 1)
        log_t[~alive] = 0.0
        log_t = torch.log_softmax(log_t, 1)
        prob = log_t.exp()
        place = idx.masked_fill(~valid, vocab)
        open_ = torch.cat([z, minus], 1).scatter_(1, place, -math.inf)
        log_open = torch.logsumexp(open_, 1, keepdim=True)
        picked = torch.cat([z, minus], 1).gather(1, place)
        classes = torch.cat([picked, log_open], 1)
        log_s = torch.log_softmax(classes, 1)
        loss = torch.where(prob > 0, prob * (log_t - log_s), 0.0).sum(1)
        d = log_s.exp() - prob  # of each class's score
        inside = torch.where(open_ > -math.inf, (open_ - log_open).exp(), 0.0)
        g = (inside * d[:, -1:]).scatter(1, place, torch.where(valid, d[:, :-1], 0.0))[:, :vocab]
        up = st["dloss"][rows].double() if "dloss" in st else torch.ones_like(weight)
        losses.append(torch.where(alive, loss * weight * t * t, 0.0))
        grads.append(torch.where(alive[:, None], g * (weight * up * t)[:, None], 0.0)
                     if st["op"] != "forward" else None)
    if st["op"] == "forward":
        return torch.cat(losses)
    if st["op"] == "backward":
        return torch.cat(grads)
    return torch.cat(losses), torch.cat(grads)


def _exact_verify(st):
    """The chain of decisions of each sequence by itself; the log-probabilities
    of the tokens it ends with."""
    t = st["temperature"]
    b, draft = st["tokens"].shape
    tokens, uniform = st["tokens"].tolist(), st["uniform"].double()
    lengths = st["length"].tolist() if st["length"] is not None else [draft] * b
    logp = np.zeros((b, draft + 1))
    for s in range(b):
        lp = torch.log_softmax(st["target"][s].double() / t, 1)
        lq = torch.log_softmax(st["drafts"][s].double() / t, 1)
        own_tokens = torch.tensor(tokens[s], device=DEV)
        at = torch.arange(draft, device=DEV)
        a, d = lp[at, own_tokens], lq[at, own_tokens]
        passed = (uniform[s] * d.exp() < a.exp()).tolist()
        a, n = a.tolist(), 0
        while n < lengths[s] and passed[n]:
            logp[s, n] = a[n]
            n += 1
        left = lp[n].exp()
        if n < lengths[s]:
            over = left - lq[n].exp()
            left = over if bool((over > 0).any()) else left
        score = torch.where(left > 0, left / st["noise"][s].double(), 0.0)
        if bool((score > 0).any()):
            logp[s, n] = float(lp[n, int(score.argmax())])
    return None, None, logp


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if st["op"] == "top":
        return _exact_top(st)
    return _exact_verify(st) if st["op"] == "verify" else _exact_distill(st)
