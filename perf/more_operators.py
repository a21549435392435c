"""Operators over finished rows of logits, each in its plain form and as the library's call.

  logprobs       log probabilities of given tokens, the entropy and the largest alternatives of every row
  logprobs_grad  the logits' gradient of those log probabilities and that entropy
  distill        the divergence of every row from a teacher of which the largest logits are known
  distill_grad   the logits' gradient of that divergence, from what the forward pass left
  distill_step   both in one call

A case is a dict of plain values:
  op          one of the five
  dtype       type of the logits: "f32" or "bf16"; grad: type of their gradient
  rows, n     rows of n logits
  wide        row strides a few elements larger than rows, so that rows begin at any alignment
  masked      three tenths of the logits are -inf (never a token that is given or that the teacher lists)
  given, top  logprobs: tokens given for a row and alternatives asked for
  lists       logprobs: "none", or the token ids of a row's places: "shared" (one list) or "own" (a list per row)
  tempered    logprobs: every row has its own temperature
  known       distill: tokens that the teacher lists for a row
  kind        distill: "logits" (its largest logits, softmax over the list), "logprobs" (log probabilities, the rest left out), "rest" (log
              probabilities, the rest counted as one more token)
  temp        distill: the temperature
  padded      distill: a fifth of the teacher's entries name no token
  ignored     distill: a fifth of the rows have weight 0
"""
import math

import torch

own = False


def _case(name, op, dtype, rows, n, grad="f32", wide=False, masked=False, given=1, top=0, lists="none", tempered=False,
          known=0, kind="logits", temp=1.0, padded=False, ignored=False):
    c = dict(op=op, dtype=dtype, rows=rows, n=n, grad=grad, wide=wide, masked=masked, given=given, top=top, lists=lists,
             tempered=tempered, known=known, kind=kind, temp=temp, padded=padded, ignored=ignored)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one served token: its log probability and twenty alternatives, nothing but latency
        _case("logprobs_1", "logprobs", "f32", 1, 128256, top=20),
        # a draft tree over a speculative vocabulary: ten children a node and as many alternatives
        _case("logprobs_tree_60", "logprobs", "f32", 60, 8192, given=10, top=10, lists="shared"),
        # a batch that is verified: 16 requests x 32 nodes, every request with its temperature
        _case("logprobs_512", "logprobs", "f32", 512, 151936, top=8, tempered=True),
        # answers that are scored: one token a row, its log probability and the entropy
        _case("logprobs_4096", "logprobs", "bf16", 4096, 128256),
        # a few rows of a vocabulary of odd size, rows at any alignment
        _case("logprobs_grad_60", "logprobs_grad", "f32", 60, 32003),
        # a training step on scored answers, the entropy in its loss
        _case("logprobs_grad_2048", "logprobs_grad", "bf16", 2048, 151936, grad="bf16", tempered=True),
        # validation on a few rows, the teacher's eight largest logits
        _case("distill_16", "distill", "f32", 16, 32003, known=8, temp=2.0),
        # validation of a batch, the rest of the teacher's mass in one token
        _case("distill_1024", "distill", "f32", 1024, 128256, known=64, kind="rest"),
        # the backward pass of float32 logits whose gradient goes into bfloat16 products
        _case("distill_grad_256", "distill_grad", "f32", 256, 151936, grad="bf16", known=32, temp=2.0),
        # the same of a batch in bfloat16 with rows that do not count
        _case("distill_grad_2048", "distill_grad", "bf16", 2048, 128256, grad="bf16", known=128, kind="rest", ignored=True),
        # a micro-batch of a small vocabulary, loss and gradient at once
        _case("distill_step_64", "distill_step", "f32", 64, 32000, known=16),
        # a training batch, loss and gradient at once
        _case("distill_step_4096", "distill_step", "bf16", 4096, 128256, grad="bf16", known=64, kind="rest"),
    ]


MOST = 4096 * 128256 * 4          # bytes of logits and gradient


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("logprobs", "logprobs", "logprobs_grad", "distill", "distill_grad", "distill_step"))
    n = _log(rng, 1, 262144) if rng.random() < 0.3 else _log(rng, 1000, 262144)
    top = rng.choice((0, 0, 1, 5, 20, 64)) if op == "logprobs" else 0
    dtype, grad = rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16"))
    each = (4 if dtype == "f32" else 2) + (0 if op in ("logprobs", "distill") else 4 if grad == "f32" else 2)
    rows = min(_log(rng, 1, 4096), max(1, 512 * 151936 // n if top else MOST // (each * n)))
    c = dict(dtype=dtype, rows=rows, n=n, grad=grad, wide=rng.random() < 0.3, masked=rng.random() < 0.2)
    if op in ("logprobs", "logprobs_grad"):
        lists = rng.choice(("none", "shared", "own")) if op == "logprobs" and n <= 32768 else "none"
        return _case(None, op, given=rng.choice((1, 1, 1, 4, 10, 64)), top=min(top, n), lists=lists, tempered=rng.random() < 0.4, **c)
    return _case(None, op, known=min(n, rng.choice((1, 8, 20, 64, 128, 256, 500))), kind=rng.choice(("logits", "logprobs", "rest")),
                 temp=rng.choice((1.0, 1.0, 0.7, 2.0)), padded=rng.random() < 0.2, ignored=rng.random() < 0.2, **c)


# ---- inputs


_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
KINDS = ("logits", "logprobs", "rest")


def _logits(gen, c):
    """Logits of a language model: most tokens around zero, a few far above them in every row."""
    rows, n = c["rows"], c["n"]
    full = torch.empty((rows, n + (5 if c["wide"] else 0)), dtype=_DTYPES[c["dtype"]], device="cuda").normal_(0.0, 2.5, generator=gen)
    z = full[:, :n]
    some = min(n, 24)
    at = _places(gen, rows, n, some)
    z.scatter_(1, at, (torch.rand((rows, some), device="cuda", generator=gen) * 14).to(z.dtype))
    return z


def _mask(gen, z):
    z.masked_fill_(torch.rand(z.shape, device="cuda", generator=gen, dtype=torch.float16) < 0.3, -math.inf)


def _places(gen, rows, n, k):
    """k places of each row, all different, in no order."""
    j = torch.arange(k, device="cuda")
    lo, hi = j * n // k, (j + 1) * n // k
    at = lo + (torch.rand((rows, k), device="cuda", generator=gen, dtype=torch.float64) * (hi - lo)).long()
    return at[:, torch.randperm(k, device="cuda", generator=gen)]


def _token_inputs(gen, c, s):
    rows, n, m = c["rows"], c["n"], c["given"]
    z = _logits(gen, c)
    at = torch.randint(0, n, (rows, m), device="cuda", generator=gen)
    at[:, 0] = z.argmax(dim=1)                       # the likeliest token is the one most often given
    if c["masked"]:
        keep = z.gather(1, at)
        _mask(gen, z)
        z.scatter_(1, at, keep)
    s["logits"], s["idx"] = z, None
    if c["lists"] != "none":
        own_rows = rows if c["lists"] == "own" else 1
        step = torch.randint(1, 8, (own_rows, n), device="cuda", generator=gen)
        idx = step.cumsum(dim=1)
        at = idx.expand(rows, -1).gather(1, at)
        s["idx"] = idx.to(torch.int32)[0].contiguous() if own_rows == 1 and c["lists"] == "shared" else idx.to(torch.int32)
    s["tokens"] = at.to(torch.int32)
    s["temperature"] = None
    if c["tempered"]:
        choice = torch.tensor([0.0, 0.6, 0.8, 1.0, 1.0, 1.5], device="cuda")
        s["temperature"] = choice[torch.randint(0, 6, (rows,), device="cuda", generator=gen)]
    if c["op"] == "logprobs_grad":
        s["grad_logprob"] = torch.randn((rows, m), device="cuda", generator=gen) / rows
        s["grad_entropy"] = torch.full((rows,), -0.01 / rows, device="cuda")
        s["state"] = _token_state(z, _row_temperature(s, torch.float32))


def _teacher_inputs(gen, c, s):
    rows, n, k = c["rows"], c["n"], c["known"]
    z = _logits(gen, c)
    if c["masked"]:
        _mask(gen, z)
    at = _places(gen, rows, n, k)
    t = torch.randn((rows, k), device="cuda", generator=gen) * 2.5 + 6
    # a student that has learned something: near the teacher where the teacher's mass is
    z.scatter_(1, at, (t + torch.randn((rows, k), device="cuda", generator=gen)).to(z.dtype))
    if c["kind"] != "logits":
        mass = 0.6 + 0.399 * torch.rand((rows, 1), device="cuda", generator=gen)
        t = t / c["temp"]
        t = t - t.exp().sum(dim=1, keepdim=True).log() + mass.log()
    if c["padded"]:
        at = at.masked_fill(torch.rand((rows, k), device="cuda", generator=gen) < 0.2, -1)
    s["logits"], s["tok"], s["teacher"], s["weight"] = z, at.to(torch.int32), t, None
    if c["ignored"]:
        s["weight"] = (torch.rand(rows, device="cuda", generator=gen) >= 0.2).float() / rows
    if c["op"] == "distill_grad":
        s["state"] = _teacher_state(z, s["tok"], c["temp"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": dict(case)}
    (_token_inputs if case["op"].startswith("logprobs") else _teacher_inputs)(gen, case, s)
    return s


# ---- plain forms


def _row_temperature(s, dtype):
    t = s["temperature"]
    if t is None:
        return torch.ones((s["logits"].shape[0], 1), dtype=dtype, device=s["logits"].device)
    return torch.where(t > 0, t.to(dtype).clamp(2.0 ** -20, 2.0 ** 20), 1.0).unsqueeze(1)


def _largest(z):
    """The largest logit of each row, 0 for rows that are masked throughout."""
    most = z.float().amax(dim=1, keepdim=True)
    return torch.where(most > -math.inf, most, 0.0)


def _token_state(z, t):
    """What the gradient needs of the forward pass: largest logit, sum of exp((z - largest) / t), entropy."""
    most = _largest(z)
    x = (z.float() - most) / t
    e = torch.exp(x)
    total = e.sum(dim=1, keepdim=True)
    entropy = torch.log(total) - torch.where(e > 0, e * x, 0.0).sum(dim=1, keepdim=True) / total
    return torch.cat((most, total, torch.where(total > 0, entropy, 0.0), torch.zeros_like(most)), dim=1)


def _at(s, places_of):
    """(places of the given tokens, which of them there are)."""
    tokens, idx = s["tokens"].long(), s["idx"]
    n = s["logits"].shape[1]
    if idx is None:
        return tokens.clamp(0, n - 1), (tokens >= 0) & (tokens < n)
    at = places_of(idx.long().expand(tokens.shape[0], -1), tokens).clamp(0, n - 1)
    return at, idx.long().expand(tokens.shape[0], -1).gather(1, at) == tokens


def _search(idx, tokens):
    return torch.searchsorted(idx.contiguous(), tokens)


def _logprobs(s, c):
    z, t = s["logits"], _row_temperature(s, torch.float32)
    f = z.float()
    most = _largest(z)
    x = (f - most) / t
    e = torch.exp(x)
    total = e.sum(dim=1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * x, 0.0).sum(dim=1, keepdim=True) / total
    at, there = _at(s, _search)
    out = {"logprob": torch.where(there, x.gather(1, at) - log_total, -math.inf), "entropy": torch.where(total > 0, entropy, 0.0)[:, 0]}
    if c["top"]:
        best, order = torch.sort(f, dim=1, descending=True, stable=True)
        best, order = best[:, :c["top"]], order[:, :c["top"]]
        tok = order if s["idx"] is None else s["idx"].long().expand(c["rows"], -1).gather(1, order)
        some = best > -math.inf
        out["top_tok"] = torch.where(some, tok, -1).to(torch.int32)
        out["top_logprob"] = torch.where(some, (best - most) / t - log_total, -math.inf)
    return out


def _logprobs_grad(s, c):
    z, t, state = s["logits"].float(), _row_temperature(s, torch.float32), s["state"]
    most, total, entropy = state[:, :1], state[:, 1:2], state[:, 2:3]
    x = (z - most) / t
    p = torch.exp(x) / total
    g, ge = s["grad_logprob"], s["grad_entropy"].unsqueeze(1)
    grad = -p * (g.sum(dim=1, keepdim=True) + ge * (torch.where(p > 0, x, 0.0) - torch.log(total) + entropy))
    grad.scatter_add_(1, s["tokens"].long(), g)
    return torch.where(z > -math.inf, grad / t, 0.0).to(_DTYPES[c["grad"]])


def _teacher_state(z, tok, temp):
    """What the gradient needs of the forward pass: largest logit and sum of exp((z - largest) / temp), over the row and over
    the places that the teacher does not list."""
    rest = z.float().clone()
    # (an entry that names no token is written where the row ends)
    rest = torch.cat((rest, rest[:, :1]), dim=1).scatter_(1, torch.where(tok >= 0, tok.long(), z.shape[1]), -math.inf)[:, :-1]
    parts = []
    for v in (z, rest):
        most = _largest(v)
        parts += [most, torch.exp((v.float() - most) / temp).sum(dim=1, keepdim=True)]
    return torch.cat(parts, dim=1)


def _teacher_probabilities(s, c):
    """(p, its logarithm, 0 where p is, and the mass left to the rest)."""
    there = s["tok"] >= 0
    t = s["teacher"].float()
    if c["kind"] == "logits":
        t = torch.where(there, t / c["temp"], -math.inf)
        most = t.amax(dim=1, keepdim=True)
        most = torch.where(most > -math.inf, most, 0.0)
        total = torch.exp(t - most).sum(dim=1, keepdim=True)
        t = t - most - torch.log(torch.where(total > 0, total, 1.0))
    p = torch.where(there, torch.exp(t), 0.0)
    left = (1.0 - p.double().sum(dim=1, keepdim=True)).clamp(min=0).float() if c["kind"] == "rest" else torch.zeros_like(p[:, :1])
    return p, torch.where(p > 0, t, 0.0), left


def _distill_loss(s, c, state):
    most, total, rest_most, rest_total = state.unbind(dim=1)
    p, log_p, left = _teacher_probabilities(s, c)
    log_total = torch.log(total).unsqueeze(1)
    log_q = (s["logits"].gather(1, s["tok"].long().clamp(min=0)).float() - most.unsqueeze(1)) / c["temp"] - log_total
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(dim=1)
    left = left[:, 0]
    log_rest = (rest_most - most) / c["temp"] + torch.log(rest_total) - log_total[:, 0]
    loss = loss + torch.where((left > 0) & (rest_total > 0), left * (torch.log(left) - log_rest), 0.0)
    return loss if s["weight"] is None else torch.where(s["weight"] == 0, 0.0, s["weight"] * loss)


def _distill_grad(s, c, state):
    most, total, rest_most, rest_total = (v.unsqueeze(1) for v in state.unbind(dim=1))
    z, tok = s["logits"].float(), s["tok"].long()
    n = z.shape[1]
    p, _, left = _teacher_probabilities(s, c)
    has_rest = (left > 0) & (rest_total > 0)
    mass = p.sum(dim=1, keepdim=True) + torch.where(has_rest, left, 0.0)
    q = torch.exp((z - most) / c["temp"]) / total
    share = torch.where(has_rest, left / rest_total, 0.0)
    grad = mass * q
    listed = torch.zeros((z.shape[0], n + 1), dtype=torch.bool, device=z.device).scatter_(1, torch.where(tok >= 0, tok, n), True)[:, :n]
    grad -= torch.where(listed, 0.0, share * torch.exp((z - rest_most) / c["temp"]))
    grad.scatter_add_(1, tok.clamp(min=0), -p)
    grad /= c["temp"]
    grad = torch.where((z > -math.inf) & (total > 0), grad, 0.0)
    if s["weight"] is not None:
        w = s["weight"].unsqueeze(1)
        grad = torch.where(w == 0, 0.0, w * grad)
    return grad.to(_DTYPES[c["grad"]])


def _own(s):
    import paper_2602_13836_amd as sv
    c = s["case"]
    if c["op"] == "logprobs":
        got = sv.token_logprobs(s["logits"], s["tokens"], top=c["top"], temperature=s["temperature"], idx=s["idx"])
        out = {"logprob": got.logprob, "entropy": got.entropy}
        return dict(out, top_tok=got.top_tok, top_logprob=got.top_logprob) if c["top"] else out
    if c["op"] == "logprobs_grad":
        return sv.token_logprobs_grad(s["logits"], s["tokens"], s["state"], s["grad_logprob"], s["grad_entropy"],
                                      temperature=s["temperature"], grad_dtype=_DTYPES[c["grad"]])
    if c["op"] == "distill_grad":
        return sv.distill_grad(s["logits"], s["tok"], s["teacher"], s["state"], kind=c["kind"], temperature=c["temp"],
                               weight=s["weight"], grad_dtype=_DTYPES[c["grad"]])
    step = c["op"] == "distill_step"
    got = sv.distill(s["logits"], s["tok"], s["teacher"], kind=c["kind"], temperature=c["temp"], weight=s["weight"],
                     grad_dtype=_DTYPES[c["grad"]] if step else None)
    return {"loss": got.loss, "grad": got.grad} if step else {"loss": got.loss}


def run(state):
    if own:
        return _own(state)
    s, c = state, state["case"]
    if c["op"] == "logprobs":
        return _logprobs(s, c)
    if c["op"] == "logprobs_grad":
        return _logprobs_grad(s, c)
    if c["op"] == "distill_grad":
        return _distill_grad(s, c, s["state"])
    stats = _teacher_state(s["logits"], s["tok"], c["temp"])
    out = {"loss": _distill_loss(s, c, stats)}
    return dict(out, grad=_distill_grad(s, c, stats)) if c["op"] == "distill_step" else out


# ---- what a pass cannot do without, and its results in 64 bits


def work(case):
    c = case
    rows, n = c["rows"], c["n"]
    es, eg = (4 if c[t] == "f32" else 2 for t in ("dtype", "grad"))
    read = 0.8 if c["ignored"] else 1.0              # rows of weight 0 need not be read
    of_logits = rows * n * es * read
    if c["op"] == "logprobs":
        lists = {"none": 0, "shared": n, "own": rows * n}[c["lists"]]
        return {"bytes": of_logits + 4 * lists + rows * (8 * c["given"] + 8 * c["top"] + 8), "flops": 6 * rows * n}
    if c["op"] == "logprobs_grad":
        return {"bytes": of_logits + rows * n * eg + rows * (8 * c["given"] + 20), "flops": 7 * rows * n}
    small = rows * (8 * c["known"] + 4)
    if c["op"] == "distill":
        return {"bytes": of_logits + small, "flops": 4 * rows * n * read}
    flops = (4 if c["op"] == "distill_grad" else 8) * rows * n * read
    return {"bytes": of_logits + rows * n * eg + small, "flops": flops}


def _exact_tokens(s, c):
    z = s["logits"].double()
    t = torch.ones(c["rows"], dtype=torch.float64, device=z.device)
    if s["temperature"] is not None:
        t = s["temperature"].double()
        t[t <= 0] = 1.0
    z = z / t[:, None]
    lse = torch.logsumexp(z, dim=1)
    return z, lse, t


def _exact_logprobs(s, c):
    z, lse, _ = _exact_tokens(s, c)
    logp = z - lse[:, None]
    entropy = -(logp.exp() * logp.clamp(min=-1e300)).sum(dim=1)
    if s["idx"] is None:
        at = s["tokens"].long()
    else:
        at = torch.empty_like(s["tokens"], dtype=torch.int64)
        for r in range(c["rows"]):
            ids = s["idx"][r] if s["idx"].dim() == 2 else s["idx"]
            at[r] = (ids[None, :] == s["tokens"][r][:, None]).to(torch.int8).argmax(dim=1)
    out = {"logprob": logp.gather(1, at), "entropy": entropy}
    if c["top"]:
        key = s["logits"].double()
        rows = torch.arange(c["rows"], device=key.device)
        tok, value = [], []
        for _ in range(c["top"]):                    # one after the other: the lowest place among the largest
            best = key.amax(dim=1)
            place = (key == best[:, None]).to(torch.int8).argmax(dim=1)
            some = best > -math.inf
            name = place if s["idx"] is None else (s["idx"][place] if s["idx"].dim() == 1 else s["idx"][rows, place]).long()
            tok.append(torch.where(some, name, -1))
            value.append(torch.where(some, logp[rows, place], -math.inf))
            key[rows, place] = -math.inf
        out["top_tok"], out["top_logprob"] = torch.stack(tok, dim=1).to(torch.int32), torch.stack(value, dim=1)
    return out


def _exact_logprobs_grad(s, c):
    z, lse, t = _exact_tokens(s, c)
    logp = z - lse[:, None]
    p = logp.exp()
    plogp = p * logp.clamp(min=-1e300)
    entropy = -plogp.sum(dim=1, keepdim=True)
    g, ge = s["grad_logprob"].double(), s["grad_entropy"].double()
    grad = torch.zeros_like(z)
    for j in range(c["given"]):
        grad[torch.arange(c["rows"], device=z.device), s["tokens"][:, j].long()] += g[:, j]
    grad -= p * g.sum(dim=1, keepdim=True)
    grad -= ge[:, None] * (plogp + p * entropy)
    return grad / t[:, None]


def _exact_distill(s, c):
    """(loss, its gradient) by rows of a table with one column more: the mass that the list leaves."""
    rows, n, temp = c["rows"], c["n"], c["temp"]
    z = s["logits"].double() / temp
    tok = s["tok"].long()
    there = tok >= 0
    t = s["teacher"].double()
    p = torch.softmax((t / temp).masked_fill(~there, -math.inf), dim=1).nan_to_num(0.0) if c["kind"] == "logits" else t.exp() * there
    left = (1 - p.sum(dim=1)).clamp(min=0) if c["kind"] == "rest" else torch.zeros(rows, dtype=torch.float64, device=z.device)
    w = torch.ones_like(left) if s["weight"] is None else s["weight"].double()
    q = torch.softmax(z, dim=1)
    of_list = torch.zeros((rows, n), dtype=torch.bool, device=z.device)
    r, j = there.nonzero(as_tuple=True)
    of_list[r, tok[r, j]] = True
    lse = torch.logsumexp(z, dim=1)
    rest_lse = torch.logsumexp(z.masked_fill(of_list, -math.inf), dim=1)
    left = torch.where(rest_lse > -math.inf, left, 0.0)
    log_q = z.gather(1, tok.clamp(min=0)) - lse[:, None]
    loss = (torch.special.xlogy(p, p) - torch.where(p > 0, p * log_q, 0.0)).sum(dim=1)
    loss = loss + torch.where(left > 0, torch.special.xlogy(left, left) - left * (rest_lse - lse), 0.0)
    if c["op"] == "distill":
        return w * loss, None
    q_rest = torch.exp(z - rest_lse[:, None]).masked_fill_(of_list, 0.0).nan_to_num_(0.0)
    grad = q * (p.sum(dim=1) + left)[:, None]
    grad -= left[:, None] * q_rest
    grad[r, tok[r, j]] -= p[r, j]
    return w * loss, grad * (w / temp)[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        return _exact_logprobs(s, case)
    if case["op"] == "logprobs_grad":
        return _exact_logprobs_grad(s, case)
    loss, grad = _exact_distill(s, case)
    if case["op"] == "distill":
        return {"loss": loss}
    return grad if case["op"] == "distill_grad" else {"loss": loss, "grad": grad}
