"""Gradients of rows whose logits over T are far from 0: finite masks (-1e9, -1e10, ...) over whole rows or over all places that a teacher does not list,
single large logits, small temperatures.  Any value but -inf is a logit.  Against the 64-bit plain forms, with the tolerances of ordinary rows: what counts is
the places' distance from the largest."""
import math

import pytest
import torch

import paper_2602_13836_amd as sv
import plain_rows as plain
from test_gpu_distill import errors, inputs
from test_gpu_token_logprobs import grad_check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
TEMPERATURES = [1.0, 0.300000011920929, 3.0, 2.0 ** -20]          # (numbers of float32: the plain forms take them as they are)
TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]
# A reference a m is rounded: up to 2^25 within an octave; from 2^31 on the rounding may leave the range of an exponential; past 2^128 a m itself is infinite.
SIZES = [1e5, 1e7, 12345678.0, 1e8, 1e9, 1e10, 1e12, 1e15, 1e20, 1e29]


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def large_rows(gen, n, dtype):
    """A row for each way in which logits are large, for each size and sign."""
    rows = []
    for v in [s * x for x in SIZES for s in (1.0, -1.0)]:
        for form in range(4):
            z = torch.empty(n, device=DEV).normal_(0, 2, generator=gen)
            if form == 0:
                z[:] = v                                                       # throughout
            elif form == 1:
                z[torch.rand(n, device=DEV, generator=gen) < 0.5] = v           # half of the row
            elif form == 2:
                z[n // 2] = v                                                  # one place
            else:                                                              # neighbours: v and up to three steps of the type below
                step = 2.0 ** (math.floor(math.log2(abs(v))) - (23 if dtype == F32 else 7))
                z = v - step * torch.randint(0, 4, (n,), device=DEV, generator=gen).float()
            rows.append(z.to(dtype))
    return torch.stack(rows)


@pytest.mark.parametrize("dtype, out", TYPES)
@pytest.mark.parametrize("n", [4, 5003, 40001])
def test_token_gradients(n, dtype, out):
    gen = generator(n)
    z = large_rows(gen, n, dtype)
    rows = len(z)
    tokens = torch.randint(0, n, (rows, 3), device=DEV, generator=gen).to(I32)
    tokens[:, 1] = n // 2
    g, ge = torch.randn((rows, 3), device=DEV, generator=gen), torch.randn(rows, device=DEV, generator=gen)
    for temp in TEMPERATURES:
        t = torch.full((rows,), temp, device=DEV)
        grad_check(z, tokens, g, ge, t, out)
        grad_check(z, tokens, g, None, t, out)
        # a row that counts nothing: exactly 0
        got = grad_check(z, tokens, torch.zeros_like(g), torch.zeros_like(ge), t, out)
        assert bool((got == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_gradients_of_rows_cut_into_parts(dtype):
    """Sums of a few long rows come from several workgroups."""
    gen, n = generator(3), 100003
    z = large_rows(gen, n, dtype)
    tokens = torch.full((len(z), 2), n // 2, dtype=I32, device=DEV)
    tokens[:, 1] = n - 1
    g, ge = torch.randn((len(z), 2), device=DEV, generator=gen), torch.randn(len(z), device=DEV, generator=gen)
    for at in range(0, len(z), 40):
        of = slice(at, at + 40)
        assert sv.workspace_bytes(sv.SV_OP_TOKEN_LOGPROBS, 40, k=n, dt=sv.SV_F32 if dtype == F32 else sv.SV_BF16) > 0
        grad_check(z[of], tokens[of], g[of], ge[of], None, F32)


def distillations(gen, n, known, kind, dtype, temp):
    """Rows as above, and rows where only what the teacher does not list is large."""
    z = large_rows(gen, n, dtype)
    rows = len(z)
    _, tok, t = inputs(gen, rows, n, known, kind, dtype, twice=True)
    ordinary, _, _ = inputs(gen, rows, n, 1, kind, dtype)
    beside = torch.cat([z[form::4][:, :1].expand(-1, n) for form in (0,) * 4]).clone()
    # -inf in place of large positive ones: nothing but the list is left there
    beside = torch.where(beside > 0, torch.full_like(beside, -math.inf), beside)
    at = torch.where(tok >= 0, tok, tok[:, :1]).long()
    beside.scatter_(1, at, ordinary.gather(1, at))
    return torch.cat((z, beside)), tok.repeat(2, 1), t.repeat(2, 1)


def distilled(z, tok, teacher, kind, temp):
    """The 64-bit plain form of rows with large logits: (loss, gradient, the magnitudes that each is made of).  The rest's mass is held relative to the rest's own
    largest logit -- added to it, as log q' = -1e20 + log 6, its digits are lost in 64 bits as well."""
    rows, n = z.shape
    tok = tok.long()
    p, left = plain.teacher_masses(tok, teacher, kind, temp, n)
    there = tok >= 0
    at = torch.where(there, tok, n)
    listed = torch.zeros((rows, n + 1), dtype=torch.bool, device=z.device).scatter_(1, at, True)[:, :n]

    def sums(x):
        m = plain.largest(x)
        e = torch.exp((x.double() - m) / temp)
        return m, e, e.sum(dim=1, keepdim=True)

    m, e, s = sums(z)
    rest_m, rest_e, rest_s = sums(torch.where(listed, -math.inf, z))
    other = (left[:, None] > 0) & (rest_s > 0)
    left = torch.where(other, left[:, None], 0.0)
    z_at = torch.cat((z.double(), m), dim=1).gather(1, at)
    of_list = torch.where(p == 0, 0.0, p * (torch.log(p) - (z_at - m) / temp + torch.log(s)))
    size = torch.where(p == 0, 0.0, p * (torch.log(p).abs() + ((z_at - m) / temp).abs() + torch.log(s)))
    loss, size = of_list.sum(dim=1), size.sum(dim=1) + p.sum(dim=1) + left[:, 0]
    log_left, far = torch.where(other, torch.log(left), 0.0), torch.where(other, (rest_m - m) / temp, 0.0)
    log_s = torch.where(other, torch.log(rest_s) - torch.log(s), 0.0)
    loss = loss + (left * (log_left - far - log_s))[:, 0]
    size = size + (left * (log_left.abs() + (far + log_s).abs()))[:, 0]
    mass = p.sum(dim=1, keepdim=True) + left
    share = torch.where(other, left * rest_e / rest_s, 0.0)
    onto = torch.zeros((rows, n + 1), dtype=torch.float64, device=z.device).scatter_add_(1, at, p)[:, :n]
    masked = z == -math.inf
    grad = torch.where(masked, 0.0, (mass * e / s - onto - share) / temp)
    return loss, grad, size, torch.where(masked, 0.0, (mass * e / s + onto + share) / temp)


def distill_check(z, tok, t, kind, temp, out):
    loss, grad, size, gsize = distilled(z, tok, t, kind, temp)
    ltol, gtol = errors(z, size, gsize, loss, grad, out, None)
    step = sv.distill(z, tok, t, kind, temp, grad_dtype=out)
    alone = sv.distill(z, tok, t, kind, temp, want_state=True)
    later = sv.distill_grad(z, tok, t, alone.state, kind, temp, grad_dtype=out)
    n = z.shape[1]
    for got in (step.loss.double(), alone.loss.double()):
        off = (got - loss).abs() - ltol
        assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()))
    for got in (step.grad, later):
        off = (got.double() - grad).abs() - gtol
        assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()) // n, int(off.argmax()) % n)


@pytest.mark.parametrize("dtype, out", TYPES)
@pytest.mark.parametrize("kind", ["logits", "logprobs", "rest"])
@pytest.mark.parametrize("n, known", [(7, 3), (5003, 20), (40001, 20)])
def test_distillation(n, known, kind, dtype, out):
    gen = generator(n + known)
    for temp in TEMPERATURES:
        z, tok, t = distillations(gen, n, known, kind, dtype, temp)
        distill_check(z, tok, t, kind, temp, out=out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["logits", "logprobs", "rest"])
def test_distillation_of_rows_cut_into_parts(kind, dtype):
    gen, n = generator(4), 100003
    z, tok, t = distillations(gen, n, 20, kind, dtype, 1.0)
    for at in range(0, len(z), 40):
        of = slice(at, at + 40)
        assert sv.workspace_bytes(sv.SV_OP_DISTILL, 40, k=n, dt=sv.SV_F32 if dtype == F32 else sv.SV_BF16) > 0
        distill_check(z[of], tok[of], t[of], kind, 1.0, out=F32)


def test_padded_rows_by_hand():
    """Four logits of -1e10: probabilities of a quarter each, whatever the size."""
    for v in (-1e9, -1e10, 1e10, -1e15, 1e20, -1e31):
        z = torch.full((1, 4), v, device=DEV)
        tokens = torch.tensor([[0]], dtype=I32, device=DEV)
        state = sv.token_logprobs(z, tokens, want_state=True).state
        grad = sv.token_logprobs_grad(z, tokens, state, torch.tensor([[0.5]], device=DEV))
        # a sum of four exponentials of 0 and its reciprocal: a few roundings of numbers up to 0.5
        assert torch.allclose(grad, torch.tensor([[0.375, -0.125, -0.125, -0.125]], device=DEV), rtol=0, atol=8 * plain.STEP)
        step = sv.distill(z, tokens, torch.tensor([[math.log(0.5)]], device=DEV), "rest", want_grad=True)
        assert torch.allclose(step.grad, torch.tensor([[-0.25, 0.25 - 0.5 / 3, 0.25 - 0.5 / 3, 0.25 - 0.5 / 3]], device=DEV), rtol=0, atol=8 * plain.STEP)
