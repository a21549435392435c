"""Log probabilities and distillation where a call is at its edge: ways to call them that the other tests do not take."""
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_2602_13836_amd as sv
import plain_rows as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n", [(3, 40000), (2, 140000), (1030, 9000)])
def test_rows_whose_first_chunks_say_nothing(rows, n, dtype):
    """The first places are masked, or far below, or far above, the rest: the reference that they give does not serve."""
    gen = generator(n)
    tok = torch.randint(0, n, (rows, 5), device=DEV, generator=gen).to(I32)
    t = torch.randn((rows, 5), device=DEV, generator=gen)
    for first in (-math.inf, -200.0, torch.finfo(dtype).min, 90.0):
        z = torch.empty((rows, n), dtype=dtype, device=DEV).normal_(0, 2, generator=gen)
        z[:, :n - 700] = first
        want, h, top, value, _ = plain.token_logprobs(z, tok, 6)
        got = sv.token_logprobs(z, tok, top=6)
        for a, b in ((got.logprob, want), (got.top_logprob, value), (got.entropy, h)):
            a, b = a.double().nan_to_num(neginf=-1e30), b.nan_to_num(neginf=-1e30)
            # e / s and log s are of the size of the places' distance from the largest where the row is one crowd far below it: |log p| at most
            assert bool(((a - b).abs() <= plain.sum_error(n) * 30 + plain.STEP * 8 * b.abs()).all()), (first, float((a - b).abs().max()))
        assert torch.equal(got.top_tok, top.to(I32))
        for kind in ("logits", "rest"):
            x = torch.log_softmax(t, dim=1) - 0.2 if kind == "rest" else t
            loss, grad, size, gsize = plain.distill(z, tok, x, kind)
            step = sv.distill(z, tok, x, kind, want_grad=True, grad_dtype=F32)
            fine = torch.isfinite(loss)
            off = ((step.loss.double() - loss).abs() - size * 8 * plain.STEP - 2 * plain.sum_error(n) - 16 * plain.STEP)[fine]
            assert bool((off <= 0).all()) and torch.equal(torch.isfinite(step.loss), fine)
            tol = gsize * 2 * (plain.sum_error(n) + 88 * plain.STEP) + grad.abs() * plain.STEP + 1e-36
            assert bool(((step.grad.double() - grad).abs() <= tol).all()), (first, kind)


@pytest.mark.parametrize("n", [3000, 100000, 200000])
def test_the_same_row_gives_the_same_bits(n):
    """Whatever its neighbours hold, and every time; atomics decide nothing."""
    gen = generator(n)
    z = torch.empty((40, n), device=DEV).normal_(0, 3, generator=gen)
    z[:, ::7] = 2.5                                    # crowds of equal logits, listed tokens among them
    z[1:] = z[0]
    tok = torch.randint(0, n, (1, 500), device=DEV, generator=gen).to(I32)
    tok[0, 100:140] = tok[0, 0]
    t = torch.randn((1, 500), device=DEV, generator=gen)
    tok, t = tok.expand(40, -1).contiguous(), t.expand(40, -1).contiguous()
    for _ in range(3):
        f = sv.token_logprobs(z, tok[:, :64].contiguous(), top=64, want_state=True)
        g = sv.token_logprobs_grad(z, tok[:, :64].contiguous(), f.state, t[:, :64].contiguous(), t[:, 0].contiguous())
        d = sv.distill(z, tok, t, want_grad=True, want_state=True)
        e = sv.distill_grad(z, tok, t, d.state, grad_dtype=BF16)
        for out in (*f, g, *d, e):
            assert bool((out[1:] == out[:1]).all())


def test_strides_of_outputs_and_of_a_single_row():
    gen = generator(4)
    n = 5001
    z = torch.empty((3, n), dtype=BF16, device=DEV).normal_(0, 2, generator=gen)
    tok, t = torch.randint(0, n, (3, 4), device=DEV, generator=gen).to(I32), torch.randn((3, 4), device=DEV, generator=gen)
    want = sv.distill(z, tok, t, want_grad=True, want_state=True)
    for dtype in (BF16, F32):
        full = torch.full((3, n + 9), -7.0, dtype=dtype, device=DEV)
        got = sv.distill(z, tok, t, grad_out=full[:, 3:n + 3])
        assert torch.equal(full[:, 3:n + 3].to(BF16), want.grad) and bool((full[:, :3] == -7).all()) and bool((full[:, n + 3:] == -7).all())
        assert torch.equal(got.loss, want.loss)
        full.fill_(-7.0)
        sv.distill_grad(z, tok, t, want.state, grad_out=full[:, 1:n + 1])
        assert bool((full[:, :1] == -7).all()) and bool((full[:, n + 1:] == -7).all())
    every_other = torch.empty((6, n), dtype=BF16, device=DEV)
    every_other[::2] = z
    assert torch.equal(sv.distill(every_other[::2], tok, t).loss, want.loss)
    one = sv.distill(z[1:2], tok[1:2].contiguous(), t[1:2].contiguous())
    assert torch.equal(one.loss, want.loss[1:2])
    with pytest.raises(sv.SpecVocabError):                # rows that lie on one another are refused
        sv.distill(z[:1].expand(3, n), tok, t)


def test_calls_on_two_streams_at_once():
    gen = generator(6)
    n = 120000
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = []
    for k in range(2):
        z = torch.empty((8, n), device=DEV).normal_(0, 2 + k, generator=gen)
        tok, t = torch.randint(0, n, (8, 60), device=DEV, generator=gen).to(I32), torch.randn((8, 60), device=DEV, generator=gen)
        sets.append((z, tok, t))
    torch.cuda.synchronize()
    want = [(sv.token_logprobs(z, tok, top=20), sv.distill(z, tok, t, want_grad=True)) for z, tok, t in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [[], []]
        for _ in range(3):
            for k, (z, tok, t) in enumerate(sets):
                got[k].append((sv.token_logprobs(z, tok, top=20, stream=streams[k]), sv.distill(z, tok, t, want_grad=True, stream=streams[k])))
        torch.cuda.synchronize()
        for k in range(2):
            for f, d in got[k]:
                for a, b in zip((*f, *d), (*want[k][0], *want[k][1])):
                    assert (a is None and b is None) or torch.equal(a, b)


def test_a_workspace_that_is_used_again():
    """What an earlier call left in it changes nothing, nor does what lies in it at first."""
    gen = generator(8)
    ws = torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device=DEV)
    for rows, n in ((3, 150000), (1, 300000), (20, 110000), (2, 100000)):
        z = torch.empty((rows, n), device=DEV).normal_(0, 2, generator=gen)
        tok, t = torch.randint(0, n, (rows, 8), device=DEV, generator=gen).to(I32), torch.randn((rows, 8), device=DEV, generator=gen)
        for a, b in zip(sv.token_logprobs(z, tok, top=33, ws=ws), sv.token_logprobs(z, tok, top=33)):
            assert (a is None and b is None) or torch.equal(a, b)
        assert torch.equal(sv.distill(z, tok, t, "logprobs", ws=ws).loss, sv.distill(z, tok, t, "logprobs").loss)
        assert torch.equal(sv.distill(z, tok, t, want_grad=True, ws=ws).grad, sv.distill(z, tok, t, want_grad=True).grad)


def test_logits_of_the_library_and_a_token_of_its_sampler():
    """A subset's logits, a token drawn from them, its log probability: what the sampler reports as a probability."""
    gen = generator(2)
    rows, d, V, k = 12, 128, 3000, 500
    h = torch.empty((rows, d), device=DEV).normal_(0, 1, generator=gen).to(BF16)
    U = torch.empty((V, d), device=DEV).normal_(0, 0.2, generator=gen).to(BF16)
    idx = torch.rand((rows, V), device=DEV, generator=gen).argsort(dim=1)[:, :k].sort(dim=1).values.to(I32).contiguous()
    z = sv.subset_logits(h, U, idx)
    temperature = torch.tensor([0.7, 1.0, 1.3] * 4, device=DEV)
    tok, prob = sv.sample(z, torch.rand(rows, device=DEV, generator=gen), temperature=temperature, idx=idx)
    got = sv.token_logprobs(z, tok, top=10, temperature=temperature, idx=idx)
    # the probability is rounded once; the log probability as its own tests have it
    assert bool(((got.logprob.double() - prob.double().log()).abs() <= 2 * plain.STEP + plain.sum_error(k) + plain.STEP * 80).all())
    best, p, _ = sv.draft_topk(z, idx, 10)
    assert torch.equal(got.top_tok, best)
    first = sv.token_logprobs(z, best, idx=idx)
    assert bool(((first.logprob.double() - p.double().log()).abs() <= 1e-5).all())


def test_ids_out_of_range_are_named_in_the_debug_mode():
    code = f"""
import sys; sys.path.insert(0, {ROOT!r})
import torch, paper_2602_13836_amd as sv
z = torch.zeros((2, 50), device="cuda")
t = torch.zeros((2, 3), device="cuda")
good = torch.tensor([[0, -1, 49], [1, 2, 3]], dtype=torch.int32, device="cuda")
bad = torch.tensor([[0, -1, 50], [1, 2, 3]], dtype=torch.int32, device="cuda")
state = sv.distill(z, good, t, want_state=True).state
sv.token_logprobs(z, good); sv.token_logprobs_grad(z, good, state, t); sv.distill_grad(z, good, t, state)
for call in (lambda: sv.token_logprobs(z, bad), lambda: sv.token_logprobs_grad(z, bad, state, t), lambda: sv.distill(z, bad, t),
             lambda: sv.distill_grad(z, bad, t, state)):
    try:
        call()
    except sv.SpecVocabError as e:
        assert e.status == 7, e
    else:
        raise AssertionError("no error")
print("named")
"""
    r = subprocess.run([sys.executable, "-c", code], env=dict(os.environ, SPECVOCAB_VALIDATE="1"), capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "named" in r.stdout, r.stderr[-2000:]


def test_a_first_call_may_be_captured_after_init():
    code = f"""
import sys; sys.path.insert(0, {ROOT!r})
import torch, paper_2602_13836_amd as sv
sv.init()
z = torch.randn((4, 120000), device="cuda")
tok = torch.arange(20, dtype=torch.int32, device="cuda").reshape(4, 5)
t = torch.randn((4, 5), device="cuda")
stream = torch.cuda.Stream(); torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=stream):
    a = sv.token_logprobs(z, tok, top=5)
    b = sv.distill(z, tok, t, want_grad=True)
for _ in range(3):
    g.replay()
torch.cuda.synchronize()
c, d = sv.token_logprobs(z, tok, top=5), sv.distill(z, tok, t, want_grad=True)
assert all(torch.equal(x, y) for x, y in zip((a.logprob, a.entropy, a.top_tok, b.loss, b.grad), (c.logprob, c.entropy, c.top_tok, d.loss, d.grad)))
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
