"""Plain forms in 64 bits of the operators over finished rows of logits, from the definitions, and how far float32 arithmetic may be off
them.  torch tensors on any device."""
import math

import torch

STEP = 2.0 ** -24              # half a step of float32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def temperatures(t, rows, device):
    """Of every row: T <= 0 and NaN count as 1, the others are kept within 2^-20 .. 2^20."""
    if t is None:
        return torch.ones(rows, dtype=torch.float64, device=device)
    t = t.double()
    return torch.where(t > 0, t.clamp(2.0 ** -20, 2.0 ** 20), 1.0)


def largest(z):
    """Of every row; 0 where it is masked throughout."""
    most = z.double().amax(dim=1, keepdim=True)
    return torch.where(most == -math.inf, 0.0, most)


def log_softmax(z, t):
    """Rows of log probabilities of z / t; -inf throughout where a row is masked throughout."""
    x = (z.double() - largest(z)) / t[:, None]
    lse = torch.log(torch.exp(x).sum(dim=1, keepdim=True))
    return torch.where(lse > -math.inf, x - lse, torch.where(lse != lse, lse, -math.inf))


def places_of(tokens, idx, n):
    """(the first place of each token, n where it has none), [rows x given]."""
    tokens = tokens.long()
    if idx is None:
        return torch.where((tokens >= 0) & (tokens < n), tokens, n)
    out = torch.full_like(tokens, n)
    for r in range(tokens.shape[0]):
        ids = (idx if idx.dim() == 1 else idx[r]).long()
        for j in range(tokens.shape[1]):
            at = (ids == tokens[r, j]).nonzero()
            if tokens[r, j] >= 0 and len(at):
                out[r, j] = at[0, 0]
    return out


def token_logprobs(z, tokens=None, top=0, temperature=None, idx=None):
    """(logprob [rows x given], entropy, top_tok, top_logprob, log probabilities of all places)."""
    rows, n = z.shape
    logp = log_softmax(z, temperatures(temperature, rows, z.device))
    p = torch.exp(logp)
    entropy = -torch.where(p == 0, 0.0, p * logp).sum(dim=1)
    logprob = tok = value = None
    if tokens is not None:
        at = places_of(tokens, idx, n)
        more = torch.where(entropy != entropy, math.nan, -math.inf)[:, None]
        logprob = torch.cat((logp, more), dim=1).gather(1, at)
    if top:
        order = torch.sort(z.double().nan_to_num(nan=-math.inf) + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        value = logp.gather(1, order)
        some = value > -math.inf
        tok = order if idx is None else idx.long().expand(rows, n).gather(1, order)
        tok = torch.where(some, tok, -1)
    return logprob, entropy, tok, value, logp


def token_grad(z, tokens, g, ge, temperature=None):
    """The logits' gradient, and the sum of the magnitudes that it is made of."""
    rows, n = z.shape
    t = temperatures(temperature, rows, z.device)[:, None]
    _, entropy, _, _, logp = token_logprobs(z, temperature=temperature)
    p = torch.exp(logp)
    g = torch.zeros((rows, 1), dtype=torch.float64, device=z.device) if g is None else g.double()
    at = torch.full((rows, 1), n, device=z.device) if tokens is None else places_of(tokens, None, n)
    there = at < n
    g = torch.where(there, g, 0.0)
    ge = torch.zeros((rows, 1), dtype=torch.float64, device=z.device) if ge is None else ge.double()[:, None]
    onto = torch.zeros((rows, n + 1), dtype=torch.float64, device=z.device).scatter_add_(1, at, g)[:, :n]
    size = torch.zeros((rows, n + 1), dtype=torch.float64, device=z.device).scatter_add_(1, at, g.abs())[:, :n]
    lp = torch.where(p == 0, 0.0, logp)
    grad = onto - p * (g.sum(dim=1, keepdim=True) + ge * (lp + entropy[:, None]))
    size = size + p * (g.abs().sum(dim=1, keepdim=True) + ge.abs() * (lp.abs() + entropy.abs()[:, None]))
    masked = z == -math.inf
    bad = entropy != entropy
    return torch.where(bad[:, None], math.nan, torch.where(masked, 0.0, grad / t)), torch.where(masked, 0.0, size / t)


def teacher_masses(tok, teacher, kind, temp, n):
    """(p of every entry, the mass that the list leaves)."""
    there = (tok >= 0) & (tok < n)
    t = torch.where(there, teacher.double(), -math.inf)
    if kind == "logits":
        e = torch.exp((t - largest(t)) / temp)
        total = e.sum(dim=1, keepdim=True)
        p = torch.where(total == 0, 0.0, e / total)
    else:
        p = torch.exp(t)
    left = (1 - p.sum(dim=1)).clamp(min=0) if kind == "rest" else torch.zeros_like(p[:, 0])
    return p, left


def distill(z, tok, teacher, kind="logits", temp=1.0, weight=None):
    """(loss, gradient, [magnitudes that the loss, the gradient are made of])."""
    rows, n = z.shape
    tok = tok.long()
    p, left = teacher_masses(tok, teacher, kind, temp, n)
    logq = log_softmax(z, torch.full((rows,), float(temp), dtype=torch.float64, device=z.device))
    q = torch.exp(logq)
    at = torch.where((tok >= 0) & (tok < n), tok, n)
    more = torch.cat((logq, torch.zeros_like(logq[:, :1])), dim=1)
    listed = torch.zeros((rows, n + 1), dtype=torch.bool, device=z.device).scatter_(1, at, True)[:, :n]
    of_rest = torch.where(listed, -math.inf, logq)
    lse_rest = torch.logsumexp(of_rest, dim=1) if n else of_rest
    left = torch.where(lse_rest == -math.inf, 0.0, left)
    plogp = torch.where(p == 0, 0.0, p * torch.log(p))
    plogq = torch.where(p == 0, 0.0, p * more.gather(1, at))
    lw = torch.where(left == 0, 0.0, left * (torch.log(left) - lse_rest))
    loss = (plogp - plogq).sum(dim=1) + lw
    size = (plogp.abs() + plogq.abs()).sum(dim=1) + torch.where(left == 0, 0.0, left * (torch.log(left).abs() + lse_rest.abs())) + p.sum(dim=1) + left
    onto = torch.zeros((rows, n + 1), dtype=torch.float64, device=z.device).scatter_add_(1, at, p)[:, :n]
    share = torch.where(listed | (left == 0)[:, None], 0.0, left[:, None] * torch.exp(logq - lse_rest[:, None]))
    mass = (p.sum(dim=1) + left)[:, None]
    empty = (logq == -math.inf).all(dim=1)
    nothing = (z == -math.inf) | empty[:, None]
    grad = torch.where(nothing, 0.0, (mass * q - onto - share) / temp)
    gsize = torch.where(nothing, 0.0, (mass * q + onto + share) / temp)
    bad = (logq != logq).any(dim=1)
    loss = torch.where(bad, math.nan, loss)
    grad = torch.where(bad[:, None], math.nan, grad)
    if weight is not None:
        w = weight.double()
        off = w == 0
        loss, size = torch.where(off, 0.0, w * loss), torch.where(off, 0.0, w.abs() * size)
        grad, gsize = torch.where(off[:, None], 0.0, w[:, None] * grad), torch.where(off[:, None], 0.0, w.abs()[:, None] * gsize)
    return loss, grad, size, gsize


# ---- tolerances
#
# A term 2^y of a sum, y = (z - reference) log2(e) / T: the factor is rounded twice (1.5 half steps with the constant's own), y once, so y
# is off by at most 2.5 half steps of itself, 2^y by that times ln 2, and the exponential itself by a step.  Terms below 2^-40 of the
# sum do not matter, so |y| <= 40 where it counts: 2.5 * 40 * 0.7 + 2 = 72 half steps.  A thread adds its terms one after the other, with
# one rescaling of three roundings for every 16, then 9 + 12 steps join the threads, a wavefront's and the parts, with three roundings each.
# Up to 2^14 places, 256 threads at work, a thread adds at most 64 terms and this is a bound.  In longer rows it may add up to 1024 (2^18 places), of which
# no more than 128 are counted: the roundings of terms of many sizes go either way, and 1024 of them add up like their root, 32 half steps.  Equal terms
# by the thousand, whose roundings may all go one way, could be off by more: 1.2 half steps each.
def sum_error(n):
    terms = n / 256 / max(1, n / 16384) + 64
    return STEP * (72 + 1.2 * terms + 63)


def logprob_error(n, exact, z_range):
    """Of (z - M) / T - log S: the sum's error, and roundings of the two terms and of their difference."""
    return sum_error(n) + STEP * (4 * z_range + 4 * math.log(max(n, 2)) + 2 * exact.abs())
