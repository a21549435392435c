"""Divergence from a teacher's largest logits and its gradient, against 64-bit plain forms."""
import math

import pytest
import torch

import paper_2602_13836_amd as sv
import plain_rows as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def inputs(gen, rows, n, known, kind, dtype=F32, pad=0, start=0, temp=1.0, mass=0.9, twice=False):
    full = torch.empty(start + rows * (n + pad), dtype=dtype, device=DEV).normal_(0, 2.5, generator=gen)
    z = full[start:].view(rows, n + pad)[:, :n]
    if known <= n:
        tok = torch.rand((rows, n), device=DEV, generator=gen).topk(known, dim=1).indices if rows * n < 1 << 25 else \
            torch.randint(0, n // known, (rows, known), device=DEV, generator=gen) + torch.arange(known, device=DEV) * (n // known)
    else:
        tok = torch.randint(0, n, (rows, known), device=DEV, generator=gen)
    if twice and known > 2:
        tok[:, known // 2] = tok[:, 0]
        tok[:, known - 1] = tok[:, 0]
        tok[:, 1] = -1
    t = torch.randn((rows, known), device=DEV, generator=gen) * 2 + 5
    if kind != "logits":
        t = torch.log_softmax(t.double(), dim=1).float() + math.log(mass)
    return z, tok.to(I32), t


def errors(z, size, gsize, loss, grad, out, weight):
    """Tolerances of loss and gradient: every logarithm of a sum is off by the sum's error, every (z - M) / T by three roundings of itself
    (2^-24 of the magnitudes, which `size` holds), the state holds two float32 sums; a gradient's terms by their exponents' errors."""
    n = z.shape[1]
    e = plain.sum_error(n) + 8 * plain.STEP
    w = torch.ones_like(loss) if weight is None else weight.double().abs()
    per = size * 8 * plain.STEP + w * 2 * e + 1e-37
    return per + loss.abs().nan_to_num(posinf=0.0) * plain.STEP, gsize * 2 * (e + 80 * plain.STEP) + grad.abs() * plain.HALF[out] + 1e-36


def check(z, tok, t, kind="logits", temp=1.0, weight=None, out=F32, **kw):
    loss, grad, size, gsize = plain.distill(z, tok, t, kind, temp, weight)
    ltol, gtol = errors(z, size.nan_to_num(posinf=0.0), gsize, loss, grad, out, weight)
    step = sv.distill(z, tok, t, kind, temp, weight, grad_dtype=out, want_state=True, **kw)
    alone = sv.distill(z, tok, t, kind, temp, weight, want_state=True)
    later = sv.distill_grad(z, tok, t, alone.state, kind, temp, weight, grad_dtype=out)
    assert alone.grad is None and step.grad.dtype == out
    for l in (step.loss.double(), alone.loss.double()):
        assert torch.equal(torch.isnan(l), torch.isnan(loss)) and torch.equal(l == math.inf, loss == math.inf)
        off = ((l - loss).abs() - ltol).nan_to_num(nan=-1.0)
        assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()))
    n = z.shape[1]
    for got in (step.grad, later):
        assert torch.equal(torch.isnan(got), torch.isnan(grad))
        off = ((got.double() - grad).abs() - gtol).nan_to_num(nan=-1.0)
        assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()) // n, int(off.argmax()) % n)
    return step


KINDS = ["logits", "logprobs", "rest"]


@pytest.mark.parametrize("dtype, out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows, n, known", [(1, 1, 1), (3, 2, 1), (2, 7, 7), (3, 9, 4), (4, 33, 8), (2, 255, 20), (3, 4097, 64), (2, 8191, 512),
                                            (3, 16385, 1), (600, 3001, 128), (2, 32768, 30), (2, 40001, 500), (520, 32003, 16)])
def test_distillation_of_every_size(rows, n, known, kind, dtype, out):
    gen = generator(rows + n + known)
    z, tok, t = inputs(gen, rows, n, known, kind, dtype, pad=3, start=1, twice=True)
    check(z, tok, t, kind, 0.7 if n % 2 else 1.0, out=out)
    z, tok, t = inputs(gen, rows, n, known, kind, dtype)
    w = torch.randn(rows, device=DEV, generator=gen)
    w[rows // 2] = 0.0
    check(z, tok, t, kind, 2.0, w, out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows, n, dtype", [(1, 128256, F32), (513, 128256, BF16), (2, 262144, F32), (1, 262145, BF16), (515, 262176, BF16), (3, 500001, F32)])
def test_long_rows(rows, n, dtype, kind):
    gen = generator(n)
    z, tok, t = inputs(gen, rows, n, 64, kind, dtype, pad=1)
    check(z, tok, t, kind, out=dtype)


@pytest.mark.parametrize("rows", [8, 600])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_and_values_at_the_edge(rows, kind, dtype):
    gen = generator(rows)
    n, known = 9001, 6
    z, tok, t = inputs(gen, rows, n, known, kind, dtype, pad=1)
    z[0] = -math.inf                                   # nothing left: the loss is infinite, the gradient 0
    z[1] = torch.finfo(dtype).min                      # all places alike
    z[2, 100] = math.nan
    z[3, tok[3, 2].long()] = math.inf
    z[4, tok[4, 1].long()] = -math.inf                 # the teacher has mass where the student has none
    t[5, 1:4] = -math.inf                              # entries without mass, one of them at a masked place
    z[5, tok[5, 2].long()] = -math.inf
    tok[6] = torch.tensor([-1, n, 2 ** 31 - 1, -2 ** 31, -100, n + 1], dtype=I32)      # no entry that names a place
    keep = z[7, tok[7].long()].clone()
    z[7] = -math.inf                                   # nothing but the list left
    z[7, tok[7].long()] = keep
    check(z, tok, t, kind)
    check(z, tok, t, kind, weight=torch.full((rows,), 0.25, device=DEV))
    w = torch.zeros(rows, device=DEV)                  # rows that do not count are not read
    w[7] = 1.0
    step = check(z, tok, t, kind, weight=w)
    assert bool((step.loss[:7] == 0).all()) and bool((step.grad[:7] == 0).all()) and bool((step.state[:7] == 0).all())
    t[7, 0] = math.nan
    got = sv.distill(z, tok, t, kind, want_grad=True)
    assert math.isnan(float(got.loss[7])) and bool(torch.isnan(got.grad[7, tok[7].long()]).all())


@pytest.mark.parametrize("kind", KINDS)
def test_a_student_that_has_nearly_nothing_beside_the_list(kind):
    """The mass of the rest comes from its own sum: 2^-100 of the row's and less."""
    gen = generator(2)
    z, tok, t = inputs(gen, 3, 5000, 5, kind, mass=0.999)
    z.scatter_add_(1, tok.long(), torch.full((3, 5), 80.0, device=DEV))
    z[1].scatter_add_(0, tok[1].long(), torch.full((5,), 200.0, device=DEV))
    check(z, tok, t, kind)
    z[2] -= 1e6
    check(z, tok, t, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("temp", [2.0 ** -20, 0.01, 100.0, 2.0 ** 20])
def test_temperatures(kind, temp):
    gen = generator(7)
    z, tok, t = inputs(gen, 3, 3001, 9, kind)
    z = (z * min(temp, 4.0)).contiguous()
    check(z, tok, t * (min(temp, 4.0) if kind == "logits" else 1.0), kind, temp)


def test_a_list_of_the_whole_row():
    gen = generator(8)
    for kind in KINDS:
        z, tok, t = inputs(gen, 3, 40, 40, kind, mass=1.0)
        check(z, tok, t, kind)
        z, tok, t = inputs(gen, 3, 4, 512, kind, mass=1.0)             # every token a hundred times
        check(z, tok, t, kind)


def test_a_teacher_that_agrees():
    """Log probabilities that the library itself reports: no divergence, no gradient."""
    gen = generator(4)
    z = torch.empty((5, 30000), device=DEV).normal_(0, 3, generator=gen)
    top = sv.token_logprobs(z, top=64)
    got = sv.distill(z, top.top_tok, top.top_logprob, "rest", want_grad=True)
    # log p, log q and log of the rest off by a log probability's tolerance each, twice
    tol = 4 * plain.sum_error(30000) + 64 * plain.STEP
    assert float(got.loss.abs().max()) <= tol and float(got.grad.abs().max()) <= tol


def test_gradient_against_differences():
    gen = generator(1)
    n, h = 40, 0.03
    for kind in KINDS:
        z, tok, t = inputs(gen, 1, n, 6, kind, mass=0.8)
        z = z * 0.5
        grad = sv.distill(z, tok, t, kind, want_grad=True).grad[0].double()
        at = torch.cat((z + h * torch.eye(n, device=DEV), z - h * torch.eye(n, device=DEV)))
        f = sv.distill(at, tok.expand(2 * n, -1).contiguous(), t.expand(2 * n, -1).contiguous(), kind).loss.double()
        d = (f[:n] - f[n:]) / (2 * h)
        # third derivatives of log q and of log q' are at most 1 each; losses are off by two sums and roundings of terms of at most 16 together
        tol = h * h / 6 * 2 + 2 * (4 * plain.sum_error(n) + 16 * 8 * plain.STEP) / (2 * h)
        assert float((d - grad).abs().max()) <= tol, kind


def test_in_place_and_nothing_beside_it_written():
    gen = generator(5)
    for dtype, rows, n in ((F32, 5, 20003), (BF16, 600, 40007), (BF16, 5, 300007), (BF16, 5, 100)):
        z, tok, t = inputs(gen, rows, n, 7, "rest", dtype, pad=7)
        full = z.as_strided((rows, n + 7), (n + 7, 1))
        before = full[:, n:].clone()
        want = sv.distill(z, tok, t, "rest", want_grad=True, want_state=True)
        copy = full.clone()
        got = sv.distill(copy[:, :n], tok, t, "rest", grad_out=copy[:, :n])
        assert torch.equal(copy[:, :n], want.grad) and torch.equal(copy[:, n:], before) and torch.equal(got.loss, want.loss)
        later = sv.distill_grad(z, tok, t, want.state, "rest")
        sv.distill_grad(z, tok, t, want.state, "rest", grad_out=z)
        assert torch.equal(z, later) and torch.equal(full[:, n:], before)


def test_outputs_given_and_workspace():
    gen = generator(6)
    rows, n = 3, 50000
    z, tok, t = inputs(gen, rows, n, 30, "rest")
    want = sv.distill(z, tok, t, "rest", want_grad=True, want_state=True)
    nbytes = sv.workspace_bytes(sv.SV_OP_DISTILL, rows, k=n, dt=sv.SV_F32)
    ws = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device=DEV)
    loss, state = torch.full((rows + 32,), -77.0, device=DEV), torch.full((rows * 4 + 32,), -77.0, device=DEV)
    grad = torch.full((rows * n + 32,), -77.0, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    sv.distill(z, tok, t, "rest", loss_out=loss[:rows], state_out=state[:rows * 4].view(rows, 4), grad_out=grad[:rows * n].view(rows, n),
               ws=ws[:nbytes], stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(loss[:rows], want.loss) and torch.equal(state[:-32].view(rows, 4), want.state) and torch.equal(grad[:-32].view(rows, n), want.grad)
    assert all(bool((v[-32:] == -77).all()) for v in (loss, state, grad)) and bool((ws[nbytes:] == 0xA5).all())


def test_rows_far_apart():
    """Offsets past 32 bits."""
    gen = generator(9)
    n, ld = 1000, 1_100_000_000
    full = torch.empty(2 * ld + n, dtype=BF16, device=DEV)
    z = full.as_strided((3, n), (ld, 1))
    z.copy_(torch.empty((3, n), device=DEV).normal_(0, 2, generator=gen))
    tok = torch.randint(0, n, (3, 20), device=DEV, generator=gen).to(I32)
    t = torch.randn((3, 20), device=DEV, generator=gen)
    step = check(z, tok, t, "logits", out=BF16)
    state = sv.distill(z, tok, t, want_state=True).state
    sv.distill_grad(z, tok, t, state, grad_out=z)
    assert torch.equal(z, step.grad)


def test_a_row_of_hundreds_of_millions():
    gen = generator(10)
    n = 600_000_000
    z = torch.empty((1, n), device=DEV).normal_(0, 1, generator=gen)
    tok = torch.tensor([[n - 1, 5, n]], dtype=I32, device=DEV)
    t = torch.log(torch.tensor([[0.5, 0.25, 0.9]], device=DEV))
    z[0, n - 1] = 20.0
    got = sv.distill(z, tok, t, "rest", grad_dtype=BF16)
    x = z[0].double()
    lse = torch.logsumexp(x, dim=0)
    rest = x.clone()
    rest[n - 1] = rest[5] = -math.inf
    lse_rest = torch.logsumexp(rest, dim=0)
    want = 0.5 * (math.log(0.5) - x[n - 1] + lse) + 0.25 * (math.log(0.25) - x[5] + lse) + 0.25 * (math.log(0.25) - lse_rest + lse)
    # 2^18 places a part, 2289 of them
    tol = plain.sum_error(1 << 18) * 2 + 16 * plain.STEP
    assert abs(float(got.loss[0] - want)) <= 2 * tol + 64 * plain.STEP
    q = torch.exp(x - lse)
    grad = q - 0.25 * torch.exp(rest - lse_rest)
    grad[n - 1], grad[5] = q[n - 1] - 0.5, q[5] - 0.25
    size = q + 0.25 * torch.exp(rest - lse_rest)
    size[n - 1] += 0.5
    size[5] += 0.25
    assert bool(((grad - grad.float()).abs() <= 1).all())
    assert bool(((got.grad[0].double() - grad).abs() <= grad.abs() * 2.0 ** -8 + size * 4 * (tol + 40 * plain.STEP)).all())


def test_the_step_of_a_draft_model():
    """The teacher's and the student's heads, the teacher's list, the selector's own loss (q_aux), the gradients into both."""
    gen = generator(3)
    rows, d, dp, V, K = 33, 256, 64, 5000, 20
    h_t, h = (torch.empty((rows, d), device=DEV).normal_(0, 1, generator=gen).to(BF16) for _ in range(2))
    U = torch.empty((V, d), device=DEV).normal_(0, 0.15, generator=gen).to(BF16)
    Wd = torch.empty((dp, d), device=DEV).normal_(0, 0.1, generator=gen).to(BF16)
    Wv = torch.empty((V, dp), device=DEV).normal_(0, 0.2, generator=gen).to(BF16)
    teacher = sv.token_logprobs(sv.dense_logits(h_t, U), top=K)
    z, s = sv.dense_logits(h, U), sv.aux_log_softmax(h, Wd, Wv)
    w = torch.full((rows,), 1.0 / rows, device=DEV)
    for logits in (z, s):
        step = check(logits, teacher.top_tok, teacher.top_logprob, "rest", weight=w, out=BF16)
        # a step down the gradient lowers the loss to first order: what is left is the curvature's part
        lr = 1e-2 * rows
        down = logits - lr * step.grad.float()
        after = sv.distill(down, teacher.top_tok, teacher.top_logprob, "rest", weight=w).loss.double().sum()
        g2 = float((step.grad.double() ** 2).sum())
        change = float(after - step.loss.double().sum())
        # second derivatives of w log q are at most w / 2 in size, of the rest's part too; the bfloat16 gradient is within 2^-8
        bound = lr * g2 * 2.0 ** -7 + 0.5 * lr * lr * g2 / rows + 4 * plain.sum_error(V)
        assert abs(change + lr * g2) <= bound
    tok, _ = sv.sample(z, torch.rand(rows, device=DEV, generator=gen))
    scored = sv.token_logprobs(z, tok)
    assert bool((scored.logprob < 0).all()) and scored.logprob.shape == (rows,)


def test_replayed_graphs():
    gen = generator(11)
    sv.init()
    for rows, n in ((4, 60000), (600, 3000)):
        z, tok, t = inputs(gen, rows, n, 12, "rest", twice=True)
        w = torch.rand(rows, device=DEV, generator=gen)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()

        def step():
            a = sv.distill(z, tok, t, "rest", weight=w, want_grad=True, want_state=True)
            return [*a, sv.distill_grad(z, tok, t, a.state, "rest", weight=w, grad_dtype=BF16)]

        with torch.cuda.stream(stream):
            step()
        torch.cuda.synchronize()
        graphs, outs = [], []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                outs.append(step())
            graphs.append(graph)
        for k in range(4):
            z.copy_(torch.empty((rows, n), device=DEV).normal_(0, 1 + k, generator=gen))
            torch.cuda.synchronize()
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            want = step()
            torch.cuda.synchronize()
            for out in outs:
                for a, b in zip(out, want):
                    assert torch.equal(a, b)


def test_the_binding_refuses():
    z, state = torch.zeros((2, 30), device=DEV), torch.zeros((2, 4), device=DEV)
    tok, t = torch.zeros((2, 3), dtype=I32, device=DEV), torch.zeros((2, 3), device=DEV)
    for call in (lambda: sv.distill(z.cpu(), tok, t), lambda: sv.distill(z, tok.long(), t), lambda: sv.distill(z, tok[0], t),
                 lambda: sv.distill(z, tok, t[:, :2]), lambda: sv.distill(z, tok, t.double()), lambda: sv.distill(z, tok, t, "top"),
                 lambda: sv.distill(z, tok, t, weight=torch.ones(3, device=DEV)), lambda: sv.distill(z, tok, t, loss_out=t),
                 lambda: sv.distill(z, tok, t, grad_out=torch.zeros((2, 29), device=DEV)),
                 lambda: sv.distill(z, tok, t, grad_dtype=BF16, grad_out=torch.zeros((2, 30), device=DEV)),
                 lambda: sv.distill(z.t(), tok, t), lambda: sv.distill_grad(z, tok, t, None), lambda: sv.distill_grad(z, tok, t, state[:1])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sv.distill(z.half(), tok, t), lambda: sv.distill(z, [[0]], t), lambda: sv.distill(z, tok, t, grad_dtype=torch.float16)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: sv.distill(z, tok, t, temperature=0.0), lambda: sv.distill(z, tok[:, :0].contiguous(), t[:, :0].contiguous()),
                 lambda: sv.distill(z, tok.repeat(1, 200), t.repeat(1, 200)), lambda: sv.distill_grad(z, tok, t, state, temperature=math.nan)):
        with pytest.raises(sv.SpecVocabError):
            call()
