"""Log probabilities of given tokens, entropy, alternatives and their gradient, against 64-bit plain forms."""
import math

import pytest
import torch

import paper_2602_13836_amd as sv
import plain_rows as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def rows_of(gen, rows, n, dtype, pad=0, start=0):
    """Logits of a language model; rows `pad` elements apart, the first `start` elements into its memory."""
    full = torch.empty(start + rows * (n + pad), dtype=dtype, device=DEV).normal_(0, 2.5, generator=gen)
    z = full[start:].view(rows, n + pad)[:, :n]
    at = torch.randint(0, n, (rows, 1), device=DEV, generator=gen)
    z.scatter_(1, at, 9.0)
    return z


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def check(z, tokens, top=0, temperature=None, idx=None, **kw):
    got = sv.token_logprobs(z, tokens, top=top, temperature=temperature, idx=idx, want_state=True, **kw)
    lp, h, tok, val, logp = plain.token_logprobs(z, tokens, top, temperature, idx)
    n = z.shape[1]
    t = plain.temperatures(temperature, z.shape[0], z.device)
    inf_as = lambda x: x.nan_to_num(neginf=-1e30)  # noqa: E731

    def close(a, b, tol, what):
        assert torch.equal(torch.isnan(a.double()), torch.isnan(b)), what
        a, b = a.double().nan_to_num(nan=0.0, neginf=-1e30), b.nan_to_num(nan=0.0, neginf=-1e30)
        off = (a - b).abs() - tol
        assert bool((off <= 0).all()), (what, float(off.max()), a.flatten()[off.argmax()], b.flatten()[off.argmax()])

    def error(x):
        # (z - M) / T is rounded three times, relative to itself: it is at most |log p| + |log S|
        return plain.sum_error(n) + plain.STEP * (6 * inf_as(x).abs().nan_to_num() + 6 * math.log(max(n, 2)))

    if tokens is not None:
        close(got.logprob, lp, error(lp), "logprob")
    # entropy = log S - sum e y / S: both off by the terms' errors, the second times the y's size, whose mean is at most log S
    mean = 1 + 2 * math.log(max(n, 2))
    close(got.entropy, h, plain.sum_error(n) * mean + plain.STEP * 4 * mean, "entropy")
    if top:
        assert torch.equal(got.top_tok, torch.where(torch.isnan(val), -1, tok).to(I32))
        close(got.top_logprob, val, error(val), "alternatives")
    else:
        assert got.top_tok is None and got.top_logprob is None
    m = z.double().amax(dim=1)
    fine = ~torch.isnan(h)
    some = fine & (m > -math.inf)
    assert bool((got.state[fine & (m == -math.inf), :3] == 0).all())
    # a reference near the row's largest logit, and the sum relative to it
    s = torch.exp((z[some].double() - m[some, None]) / t[some, None]).sum(dim=1)
    above = (got.state[some, 0].double() - m[some]) / t[some]
    assert bool((above <= 0).all())
    close(got.state[some, 1].double().log() + above, s.log(), plain.sum_error(n) + plain.STEP * 6 * above.abs(), "state")
    assert torch.equal(got.state[fine, 2], got.entropy[fine])
    return got


SIZES = [(1, 1), (3, 2), (2, 3), (5, 7), (2, 8), (3, 9), (1, 31), (2, 33), (2, 63), (2, 65), (4, 255), (3, 1000), (2, 2047), (1, 4097), (2, 8191),
         (3, 16385), (300, 32003), (70, 40001), (1, 128256), (1100, 5000), (1030, 131072), (2, 131073), (1, 262145), (2, 300001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n", SIZES)
def test_logprobs_of_every_size(rows, n, dtype):
    gen = generator(rows * 31 + n)
    for pad, start, top, given in ((0, 0, min(20, n), 1), (5, 3, min(64, n), 10), (1, 1, 0, 64)):
        z = rows_of(gen, rows, n, dtype, pad, start)
        tokens = torch.randint(-1, n + 2, (rows, given), device=DEV, generator=gen).to(I32)
        check(z, tokens, top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n", [(4, 100), (40, 5003), (3, 70001), (1500, 20000)])
def test_logprobs_at_temperatures(rows, n, dtype):
    gen = generator(n)
    z = rows_of(gen, rows, n, dtype, 3, 1)
    choice = torch.tensor([0.0, -1.0, math.nan, math.inf, 1e-9, 0.01, 0.7, 1.0, 3.0, 1e9, 2.0 ** -20], device=DEV)
    t = choice[torch.randint(0, len(choice), (rows,), device=DEV, generator=gen)]
    tokens = torch.cat((z.argmax(dim=1, keepdim=True), torch.randint(0, n, (rows, 2), device=DEV, generator=gen)), dim=1).to(I32)
    check(z, tokens, min(n, 7), t)


@pytest.mark.parametrize("rows, n", [(3, 50), (60, 8192), (2, 40000), (1200, 3001)])
@pytest.mark.parametrize("shared", [True, False])
def test_logprobs_over_lists(rows, n, shared):
    gen = generator(n + shared)
    z = rows_of(gen, rows, n, F32)
    z[0, n // 2:] = -math.inf
    step = torch.randint(1, 5, (1 if shared else rows, n), device=DEV, generator=gen)
    idx = step.cumsum(dim=1)[:, torch.randperm(n, device=DEV, generator=gen)].to(I32).contiguous()    # in no order
    idx[:, 0] = idx[:, n - 1]                         # the same token twice: its first place counts
    idx[:, 1] = -1                                    # a padding slot, which names no token
    z[:, 1] = -math.inf
    idx = idx[0].contiguous() if shared else idx
    at = torch.randint(0, n, (rows, 9), device=DEV, generator=gen)
    tokens = idx.long().expand(rows, n).gather(1, at)
    tokens[:, 0] = 2 ** 31 - 1
    tokens[:, 1] = -1
    tokens[:, 2] = idx[n - 1] if shared else idx[:, n - 1]
    check(z, tokens.to(I32), min(n, 10), idx=idx)
    check(z, tokens.to(I32), 0, idx=idx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n", [(9, 20), (9, 5000), (9, 100001), (1200, 9000)])
def test_masked_rows_and_values_at_the_edge(rows, n, dtype):
    gen = generator(n)
    z = rows_of(gen, rows, n, dtype, 1)
    low = torch.finfo(dtype).min
    z[0] = -math.inf
    z[1] = low                                        # a mask of the type's lowest value over the whole row: all places alike
    z[2, :n // 2] = low
    z[3, 1:] = -math.inf                              # one place left
    z[4, n - 1] = math.nan
    z[5, n // 3] = math.inf
    z[6].masked_fill_(torch.rand(n, device=DEV, generator=gen) < 0.5, -math.inf)
    z[7] = z[7] * 1e36                                # beyond what a factor of log2(e) leaves of float32's range
    z[8] = 0.0
    z[8, ::2] = -0.0                                  # equal to 0: by place
    tokens = torch.randint(0, n, (rows, 3), device=DEV, generator=gen).to(I32)
    tokens[:, 0] = 0
    for top in (0, 1, min(n, 64)):
        check(z, tokens, top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n", [(3, 3000), (2, 60001), (1030, 50000)])
def test_alternatives_among_equal_logits(rows, n, dtype):
    """More places reach the bound than a workgroup brings together: selected by digits, equal ones by place."""
    gen = generator(rows)
    z = torch.randint(-2, 3, (rows, n), device=DEV, generator=gen).to(dtype)
    z[0] = 1.5
    z[1, :] = -7.0
    z[1, n - 40:] = 3.0                               # 40 ahead, the rest of 64 among equal ones
    tokens = torch.zeros((rows, 1), dtype=I32, device=DEV)
    for top in (1, 20, 64):
        check(z, tokens, top)
    z = torch.arange(n, device=DEV).expand(rows, n).remainder(2000).to(F32).mul(-0.25).to(dtype).contiguous()      # descending, again and again
    check(z, tokens, 64)
    z = torch.arange(n, device=DEV, dtype=F32).expand(rows, n).mul(1e-3).to(dtype).contiguous()      # ascending: all of them last
    check(z, tokens, 64)
    z[:] = -math.inf
    z[:, n - 5:] = 2.0                                # fewer than asked for, in the last thread's last vector
    check(z, tokens, 64)


def grad_check(z, tokens, g, ge, temperature, out_dtype, **kw):
    state = sv.token_logprobs(z, None, temperature=temperature, want_state=True).state
    want, size = plain.token_grad(z, tokens, g, ge, temperature)
    got = sv.token_logprobs_grad(z, tokens, state, g, ge, temperature=temperature, grad_dtype=out_dtype, **kw)
    assert got.dtype == out_dtype and got.shape == z.shape
    # p is off by its own exponent's and the sum's error, entropy and log p by as much again
    n = z.shape[1]
    tol = size * (2 * plain.sum_error(n) * (1 + math.log(max(n, 2))) + 16 * plain.STEP) + want.abs() * plain.HALF[out_dtype] + 1e-36
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    off = ((got.double() - want).abs() - tol).nan_to_num(nan=-1.0)
    assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()) // n, int(off.argmax()) % n)
    return got


@pytest.mark.parametrize("dtype, out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("rows, n", [(1, 1), (3, 2), (2, 9), (4, 255), (3, 4097), (2, 16384), (60, 32003), (2, 70001)])
def test_gradients_of_every_size(rows, n, dtype, out):
    gen = generator(n + rows)
    z = rows_of(gen, rows, n, dtype, 3, 1)
    tokens = torch.randint(-1, n + 1, (rows, 10), device=DEV, generator=gen).to(I32)
    tokens[:, 1] = tokens[:, 0]                       # given twice: the sum
    tokens[:, 2] = z.argmax(dim=1).to(I32)
    g, ge = torch.randn((rows, 10), device=DEV, generator=gen), torch.randn(rows, device=DEV, generator=gen)
    t = torch.tensor([0.5, 1.0, 0.0, 2.0], device=DEV)[torch.arange(rows, device=DEV) % 4].contiguous()
    grad_check(z, tokens, g, ge, t, out)
    grad_check(z, tokens, g, None, None, out)
    grad_check(z, None, None, ge, t, out)
    grad_check(z, tokens[:, 2].contiguous().unsqueeze(1), g[:, :1].contiguous(), None, t, out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 5000, 50001])
def test_gradients_of_masked_rows(n, dtype):
    gen = generator(n)
    z = rows_of(gen, 7, n, dtype, 1)
    z[0] = -math.inf
    z[1] = torch.finfo(dtype).min
    z[2, 1:] = -math.inf
    z[3, 5] = math.nan
    z[4, 7] = math.inf
    z[5].masked_fill_(torch.rand(n, device=DEV, generator=gen) < 0.5, -math.inf)
    tokens = torch.randint(0, n, (7, 3), device=DEV, generator=gen).to(I32)
    grad_check(z, tokens, torch.randn((7, 3), device=DEV, generator=gen), torch.randn(7, device=DEV, generator=gen), None, F32)


def test_gradient_against_differences():
    """Of the kernels' own log probabilities and entropies."""
    gen = generator(1)
    n, h = 40, 0.03
    z = torch.empty((1, n), device=DEV).normal_(0, 1, generator=gen)
    tokens = torch.tensor([[3, 8]], dtype=I32, device=DEV)
    g, ge = torch.tensor([[0.7, -0.4]], device=DEV), torch.tensor([0.5], device=DEV)
    state = sv.token_logprobs(z, want_state=True).state
    grad = sv.token_logprobs_grad(z, tokens, state, g, ge)[0].double()
    at = torch.cat((z + h * torch.eye(n, device=DEV), z - h * torch.eye(n, device=DEV)))
    f = sv.token_logprobs(at, tokens.expand(2 * n, 2).contiguous())
    value = (f.logprob.double() * g.double()).sum(dim=1) + f.entropy.double() * ge.double()
    d = (value[:n] - value[n:]) / (2 * h)
    # third derivatives of log p are at most 1, those of the entropy at most 10 (log p is at most 8 in size); values are off by a
    # tolerance of `check` each
    tol = h * h / 6 * (1.1 + 5.0) + 2 * plain.sum_error(n) * 10 / (2 * h)
    assert float((d - grad).abs().max()) <= tol


def test_in_place_and_nothing_beside_it_written():
    gen = generator(5)
    for dtype, n in ((F32, 20003), (BF16, 40007), (BF16, 100)):
        rows, pad = 5, 7
        full = torch.empty((rows, n + pad), dtype=dtype, device=DEV).normal_(0, 2, generator=gen)
        z = full[:, :n]
        tokens = torch.randint(0, n, (rows, 2), device=DEV, generator=gen).to(I32)
        g = torch.randn((rows, 2), device=DEV, generator=gen)
        state = sv.token_logprobs(z, want_state=True).state
        want = sv.token_logprobs_grad(z, tokens, state, g)
        before = full[:, n:].clone()
        got = sv.token_logprobs_grad(z, tokens, state, g, grad_out=z)
        assert got is z and torch.equal(full[:, :n], want) and torch.equal(full[:, n:], before)


def test_outputs_given_and_workspace():
    gen = generator(6)
    rows, n, top = 3, 50000, 5
    z = rows_of(gen, rows, n, F32)
    tokens = torch.randint(0, n, (rows,), device=DEV, generator=gen).to(I32)
    want = sv.token_logprobs(z, tokens, top=top, want_state=True)
    nbytes = sv.workspace_bytes(sv.SV_OP_TOKEN_LOGPROBS, rows, k=n, kd=top, dt=sv.SV_F32)
    ws = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device=DEV)
    guard = [torch.full((k + 32,), -77.0, device=DEV) for k in (rows, rows, rows * top, rows * 4)]
    toks = torch.full((rows * top + 32,), -77, dtype=I32, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = sv.token_logprobs(z, tokens, top=top, logprob_out=guard[0][:rows], entropy_out=guard[1][:rows], top_logprob_out=guard[2][:rows * top].view(rows, top),
                            state_out=guard[3][:rows * 4].view(rows, 4), top_tok_out=toks[:rows * top].view(rows, top), ws=ws[:nbytes], stream=stream)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert all(bool((v[-32:] == -77).all()) for v in guard) and bool((toks[-32:] == -77).all()) and bool((ws[nbytes:] == 0xA5).all())
    assert got.logprob.shape == (rows,)


def test_rows_far_apart_and_long_rows():
    """Offsets past 32 bits, in bytes and in elements."""
    gen = generator(9)
    n, ld = 1000, 1_100_000_000
    full = torch.empty(2 * ld + n, dtype=BF16, device=DEV)
    z = full.as_strided((3, n), (ld, 1))
    z.copy_(torch.empty((3, n), device=DEV).normal_(0, 2, generator=gen))
    tokens = torch.randint(0, n, (3, 4), device=DEV, generator=gen).to(I32)
    check(z, tokens, 5)
    g = torch.randn((3, 4), device=DEV, generator=gen)
    state = sv.token_logprobs(z, want_state=True).state
    want = sv.token_logprobs_grad(z, tokens, state, g)
    sv.token_logprobs_grad(z, tokens, state, g, grad_out=z)
    assert torch.equal(z, want)
    del z, full
    n = 600_000_000
    z = torch.empty((1, n), device=DEV).normal_(0, 1, generator=gen)
    z[0, n - 1] = 30.0
    tokens = torch.tensor([[0, n - 1, n]], dtype=I32, device=DEV)
    got = sv.token_logprobs(z, tokens, want_state=True)
    x = z[0].double()
    s = torch.exp(x - 30.0).sum()
    h = torch.log(s) - (torch.exp(x - 30.0) * (x - 30.0)).sum() / s
    # 2^18 places a part, 512 in a thread; 8 parts in a thread of the launch that joins them
    tol = plain.sum_error(1 << 18) * 2
    assert abs(float(got.logprob[0, 1] + torch.log(s))) <= tol + 1e-6 and got.logprob[0, 2] == -math.inf
    assert abs(float(got.logprob[0, 0] - (x[0] - 30.0 - torch.log(s)))) <= tol + 64 * plain.STEP
    assert abs(float(got.entropy[0] - h)) <= tol * 64
    grad = sv.token_logprobs_grad(z, tokens, got.state, torch.ones((1, 3), device=DEV), grad_dtype=BF16)
    want = -2 * torch.exp(x - 30.0) / s
    want[0] += 1
    want[n - 1] += 1
    assert bool(((grad[0].double() - want).abs() <= want.abs() * 2.0 ** -8 + tol * 4 * torch.exp(x - 30.0)).all())


def test_replayed_graphs_that_share_nothing():
    gen = generator(11)
    rows, n, top = 6, 60000, 9
    z = rows_of(gen, rows, n, F32)
    tokens = torch.randint(0, n, (rows, 2), device=DEV, generator=gen).to(I32)
    g, ge = torch.randn((rows, 2), device=DEV, generator=gen), torch.randn(rows, device=DEV, generator=gen)
    sv.init()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def step():
        f = sv.token_logprobs(z, tokens, top=top, want_state=True)
        return [*f, sv.token_logprobs_grad(z, tokens, f.state, g, ge, grad_dtype=BF16)]

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
    z = torch.zeros((2, 30), device=DEV)
    tokens = torch.zeros(2, dtype=I32, device=DEV)
    state = torch.zeros((2, 4), device=DEV)
    bad = [
        lambda: sv.token_logprobs(z.cpu(), tokens), lambda: sv.token_logprobs(z[0], tokens), lambda: sv.token_logprobs(z.t(), tokens),
        lambda: sv.token_logprobs(z, tokens.long()), lambda: sv.token_logprobs(z, tokens[:1]), lambda: sv.token_logprobs(z, tokens.cpu()),
        lambda: sv.token_logprobs(z, tokens, temperature=torch.ones(2, dtype=torch.float64, device=DEV)),
        lambda: sv.token_logprobs(z, tokens, temperature=torch.ones(3, device=DEV)),
        lambda: sv.token_logprobs(z, tokens, idx=torch.zeros(29, dtype=I32, device=DEV)),
        lambda: sv.token_logprobs(z, None, logprob_out=torch.zeros(2, device=DEV)),
        lambda: sv.token_logprobs(z, tokens, top_tok_out=torch.zeros((2, 1), dtype=I32, device=DEV)),
        lambda: sv.token_logprobs(z, tokens, state_out=torch.zeros((2, 3), device=DEV)),
        lambda: sv.token_logprobs_grad(z, tokens, None, torch.zeros(2, device=DEV)),
        lambda: sv.token_logprobs_grad(z, None, state, torch.zeros(2, device=DEV)),
        lambda: sv.token_logprobs_grad(z, tokens, state, torch.zeros((2, 1), device=DEV)),
        lambda: sv.token_logprobs_grad(z, tokens, state, torch.zeros(2, device=DEV), grad_out=torch.zeros((2, 31), device=DEV)),
        lambda: sv.token_logprobs_grad(z, tokens, state, torch.zeros(2, device=DEV), grad_dtype=BF16, grad_out=torch.zeros((2, 30), device=DEV)),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sv.token_logprobs(z.half(), tokens), lambda: sv.token_logprobs(z, [0, 1]), lambda: sv.token_logprobs([z], tokens),
                 lambda: sv.token_logprobs_grad(z, tokens, state, torch.zeros(2, device=DEV), grad_dtype=torch.float16)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: sv.token_logprobs(z, tokens, top=65), lambda: sv.token_logprobs(z, tokens, top=31), lambda: sv.token_logprobs(z[:0], tokens[:0]),
                 lambda: sv.token_logprobs_grad(z, tokens, state)):
        with pytest.raises(sv.SpecVocabError):
            call()
