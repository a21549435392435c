"""What the operators over finished rows of logits refuse, without a GPU: every check is made before anything is enqueued.  And the plain
forms that the GPU tests compare with, against values worked out by hand, against autograd and against differences."""
import math
import os

import pytest
import torch

import paper_2602_13836_amd as sv
from paper_2602_13836_amd import build as sv_build
import plain_rows as plain

P = 4096                       # a pointer that is 16-byte aligned and never followed
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sv.LIB_PATH):
        sv_build.build_library()
    return sv.load_library()


def logprobs(lib, **kw):
    a = dict(z=P, ld=100, rows=2, n=100, dt=0, idx=None, mode=0, t=None, tokens=P, given=1, top=4, lp=P, ent=P, tok=P, val=P, state=P, ws=None,
             ws_bytes=0) | kw
    return lib.specvocab_token_logprobs(*a.values(), None)


@pytest.mark.parametrize("kw, status", [
    (dict(z=None), NULL), (dict(tokens=None), NULL), (dict(lp=None), NULL), (dict(tok=None), NULL), (dict(val=None), NULL),
    (dict(given=0, top=0, ent=None, state=None), NULL), (dict(rows=0), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(n=0), SHAPE),
    (dict(n=1 << 31, ld=1 << 31, top=0), SHAPE), (dict(ld=99), SHAPE), (dict(given=-1), SHAPE), (dict(given=65), SHAPE), (dict(top=-1), SHAPE),
    (dict(top=65), SHAPE), (dict(n=3, top=4), SHAPE), (dict(dt=2), DTYPE), (dict(dt=-1), DTYPE), (dict(idx=P, mode=2), DTYPE),
    (dict(n=(1 << 23) + 1, ld=1 << 24), UNSUPPORTED), (dict(z=P + 2), ALIGN), (dict(z=P + 1, dt=1), ALIGN), (dict(state=P + 8), ALIGN),
    (dict(n=100000, ld=100000), WORKSPACE), (dict(n=100000, ld=100000, ws=P, ws_bytes=100), WORKSPACE),
    (dict(n=100000, ld=100000, ws=P + 8, ws_bytes=1 << 30), ALIGN),
])
def test_token_logprobs_refuses(lib, kw, status):
    assert logprobs(lib, **kw) == status


def logprobs_grad(lib, **kw):
    a = dict(z=P, ld=100, rows=2, n=100, dt=0, t=None, tokens=P, given=1, state=P, g=P, ge=P, out=2 * P, ld_grad=100, gdt=0) | kw
    return lib.specvocab_token_logprobs_grad(*a.values(), None)


@pytest.mark.parametrize("kw, status", [
    (dict(z=None), NULL), (dict(state=None), NULL), (dict(out=None), NULL), (dict(g=None, ge=None), NULL), (dict(tokens=None), NULL),
    (dict(rows=0), SHAPE), (dict(n=0), SHAPE), (dict(ld=99), SHAPE), (dict(ld_grad=99), SHAPE), (dict(given=0), SHAPE), (dict(given=65), SHAPE),
    (dict(dt=2), DTYPE), (dict(gdt=2), DTYPE), (dict(z=P + 2), ALIGN), (dict(out=P + 2), ALIGN), (dict(out=P + 1, gdt=1), ALIGN),
    (dict(state=P + 4), ALIGN), (dict(out=P, gdt=1), DTYPE), (dict(out=P, ld_grad=101), SHAPE), (dict(out=P, dt=1), DTYPE),
])
def test_token_logprobs_grad_refuses(lib, kw, status):
    assert logprobs_grad(lib, **kw) == status


def distilled(lib, **kw):
    a = dict(z=P, ld=100, rows=2, n=100, dt=0, tok=P, teacher=P, known=8, kind=0, t=1.0, w=None, loss=P, state=P, out=2 * P, ld_grad=100, gdt=0, ws=None,
             ws_bytes=0) | kw
    return lib.specvocab_distill(*a.values(), None)


def distilled_grad(lib, **kw):
    a = dict(z=P, ld=100, rows=2, n=100, dt=0, tok=P, teacher=P, known=8, kind=0, t=1.0, w=None, state=P, out=2 * P, ld_grad=100, gdt=0) | kw
    return lib.specvocab_distill_grad(*a.values(), None)


@pytest.mark.parametrize("call", [distilled, distilled_grad])
@pytest.mark.parametrize("kw, status", [
    (dict(z=None), NULL), (dict(tok=None), NULL), (dict(teacher=None), NULL), (dict(rows=0), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(n=0), SHAPE),
    (dict(n=1 << 31, ld=1 << 31), SHAPE), (dict(ld=99), SHAPE), (dict(ld_grad=99), SHAPE), (dict(known=0), SHAPE), (dict(known=513), SHAPE),
    (dict(known=1 << 40), SHAPE), (dict(t=0.0), SHAPE), (dict(t=-1.0), SHAPE), (dict(t=math.nan), SHAPE), (dict(t=math.inf), SHAPE),
    (dict(t=1e-7), SHAPE), (dict(t=2e6), SHAPE), (dict(kind=3), DTYPE), (dict(kind=-1), DTYPE), (dict(dt=2), DTYPE), (dict(gdt=2), DTYPE),
    (dict(z=P + 2), ALIGN), (dict(out=P + 2), ALIGN), (dict(out=P + 1, gdt=1), ALIGN), (dict(state=P + 4), ALIGN),
    (dict(out=P, gdt=1), DTYPE), (dict(out=P, ld_grad=101), SHAPE), (dict(out=P, dt=1), DTYPE),
])
def test_distill_refuses(lib, call, kw, status):
    assert call(lib, **kw) == status


def test_distill_refuses_outputs_and_workspaces(lib):
    assert distilled(lib, loss=None) == NULL
    assert distilled_grad(lib, state=None) == NULL and distilled_grad(lib, out=None) == NULL
    long = dict(n=100000, ld=100000, ld_grad=100000)
    assert distilled(lib, **long) == WORKSPACE and distilled(lib, **long, ws=P, ws_bytes=40) == WORKSPACE
    assert distilled(lib, **long, ws=P + 8, ws_bytes=1 << 30) == ALIGN


def test_workspace_sizes(lib):
    for op in (sv.SV_OP_TOKEN_LOGPROBS, sv.SV_OP_DISTILL):
        assert sv.workspace_bytes(op, 4096, k=128256, dt=sv.SV_BF16) == 0
        assert sv.workspace_bytes(op, 1, k=128256, dt=sv.SV_F32) > 0
        assert sv.workspace_bytes(op, 4096, k=1 << 19, dt=sv.SV_BF16) > 0
        for kw, status in ((dict(rows=0), SHAPE), (dict(k=0), SHAPE), (dict(k=1 << 31), SHAPE), (dict(dt=2), DTYPE)):
            with pytest.raises(sv.SpecVocabError) as e:
                sv.workspace_bytes(op, **(dict(rows=2, k=10, dt=sv.SV_F32) | kw))
            assert e.value.status == status
    with pytest.raises(sv.SpecVocabError) as e:
        sv.workspace_bytes(sv.SV_OP_TOKEN_LOGPROBS, 2, k=10, kd=65, dt=sv.SV_F32)
    assert e.value.status == SHAPE
    assert sv.workspace_bytes(sv.SV_OP_TOKEN_LOGPROBS, 1, k=128256, kd=20, dt=0) > sv.workspace_bytes(sv.SV_OP_TOKEN_LOGPROBS, 1, k=128256, dt=0)


# ---- the plain forms themselves
def test_logprobs_by_hand():
    z = torch.log(torch.tensor([[1.0, 4.0, 2.0, 1.0], [0.0, 0.0, 0.0, 0.0]], dtype=torch.float64))
    lp, h, tok, val, _ = plain.token_logprobs(z, torch.tensor([[1, -1, 4], [0, 1, 2]]), top=3)
    assert lp[0].tolist() == [pytest.approx(math.log(0.5)), -math.inf, -math.inf] and lp[1].tolist() == [-math.inf] * 3
    assert float(h[0]) == pytest.approx(0.5 * math.log(2) + 0.25 * math.log(4) + 0.25 * math.log(8)) and float(h[1]) == 0
    assert tok.tolist() == [[1, 2, 0], [-1, -1, -1]] and val[0].exp().tolist() == pytest.approx([0.5, 0.25, 0.125])
    lp, _, tok, _, _ = plain.token_logprobs(z[:1], torch.tensor([[7]]), top=2, temperature=torch.tensor([0.5]), idx=torch.tensor([5, 7, 9, 7]))
    assert float(lp[0, 0]) == pytest.approx(math.log(16 / 22)) and tok.tolist() == [[7, 9]]


def test_distill_by_hand():
    z = torch.log(torch.tensor([[1.0, 4.0, 2.0, 1.0]], dtype=torch.float64))
    tok = torch.tensor([[1, 2, -1]])
    t = torch.log(torch.tensor([[3.0, 1.0, 9.0]]))
    loss, grad, _, _ = plain.distill(z, tok, t)
    assert float(loss[0]) == pytest.approx(0.75 * math.log(0.75 / 0.5) + 0.25 * math.log(1.0))
    # (log 3 = 1.0986 is rounded to float32, by at most 2^-24 of itself: its probability is off by 0.75 * 0.25 * 1.1 * 2^-24 < 2e-8)
    assert grad[0].tolist() == pytest.approx([0.125, -0.25, 0.0, 0.125], abs=2e-8)
    loss, grad, _, _ = plain.distill(z, tok, torch.log(torch.tensor([[0.5, 0.1, 0.9]])), "rest", weight=torch.tensor([2.0]))
    assert float(loss[0]) == pytest.approx(2 * (0.1 * math.log(0.1 / 0.25) + 0.4 * math.log(0.4 / 0.25)))
    assert grad[0].tolist() == pytest.approx([2 * (0.125 - 0.4 / 2), 0.0, 2 * 0.15, 2 * (0.125 - 0.4 / 2)], abs=1.2e-7)     # (log 0.5, log 0.1 in float32: p off by at most 2^-24)
    loss, grad, _, _ = plain.distill(z, torch.tensor([[1, 1, 2]]), torch.log(torch.tensor([[0.25, 0.25, 0.25]])), "logprobs")
    assert grad[0].tolist() == pytest.approx([0.75 / 8, 0.75 / 2 - 0.5, 0.75 / 4 - 0.25, 0.75 / 8])


@pytest.mark.parametrize("kind", ["logits", "logprobs", "rest"])
@pytest.mark.parametrize("temp", [1.0, 0.5])
def test_plain_gradients_against_autograd_and_differences(kind, temp):
    gen = torch.Generator().manual_seed(3)
    z = torch.randn((3, 17), generator=gen, dtype=torch.float64)
    z[0, 3] = -math.inf
    tok = torch.tensor([[1, 5, 5, -1], [0, 16, 2, 3], [7, 8, 9, 10]])
    t = torch.log_softmax(torch.randn((3, 5), generator=gen, dtype=torch.float64), dim=1)[:, :4]
    w = torch.tensor([1.0, 0.3, -2.0], dtype=torch.float64)
    _, grad, _, _ = plain.distill(z, tok, t, kind, temp, w)
    h = 1e-5
    for v in range(17):
        if v == 3:
            continue
        up, down = z.clone(), z.clone()
        up[:, v] += h
        down[:, v] -= h
        d = (plain.distill(up, tok, t, kind, temp, w)[0] - plain.distill(down, tok, t, kind, temp, w)[0]) / (2 * h)
        # third derivatives of a divergence are below 8 |w| / T^3; its roundings 2^-52 of at most 20
        assert torch.allclose(d, grad[:, v], rtol=0, atol=2 * 8 * h * h / temp ** 3 / 6 + 40 * 2.0 ** -52 / h)
    g, ge = torch.randn((3, 4), generator=gen, dtype=torch.float64), torch.randn(3, generator=gen, dtype=torch.float64)
    leaf = z.clone().requires_grad_()
    logp = torch.log_softmax(leaf / temp, dim=1)
    p = logp.exp()
    entropy = -(p * logp.masked_fill(z == -math.inf, 0.0)).sum(dim=1)
    ((logp.gather(1, tok.clamp(min=0)) * g * (tok >= 0)).sum() + (entropy * ge).sum()).backward()
    got, _ = plain.token_grad(z, tok, g, ge, torch.full((3,), temp, dtype=torch.float64))
    assert torch.allclose(got, leaf.grad.masked_fill(z == -math.inf, 0.0), rtol=1e-9, atol=1e-12)
