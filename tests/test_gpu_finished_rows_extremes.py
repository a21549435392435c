"""Log probabilities and distillation at the ends of their ranges: lists of rows that are cut into parts, the longest rows with alternatives, more rows
than one launch takes, rows that just fit a part.  Tolerances are those of the tests of every size."""
import pytest
import torch

import paper_2602_13836_amd as sv
from test_gpu_distill import check as distill_check, inputs
from test_gpu_token_logprobs import check, grad_check, rows_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("rows, n", [(3, 50), (60, 8185), (60, 8192), (2, 100003), (5, 140000), (70, 100001), (3, 300001)])
def test_lists_in_either_type_and_of_rows_in_parts(rows, n, shared, dtype):
    gen = generator(n + shared)
    z = rows_of(gen, rows, n, dtype, 3, 1)
    z[0, n // 2:] = float("-inf")
    step = torch.randint(1, 5, (1 if shared else rows, n), device=DEV, generator=gen)
    idx = step.cumsum(dim=1)[:, torch.randperm(n, device=DEV, generator=gen)].to(I32).contiguous()
    idx[:, 0] = idx[:, n - 1]                         # the same token twice: its first place counts
    idx[:, 1] = -1                                    # a padding slot
    z[:, 1] = float("-inf")
    tokens = idx.long().expand(rows, n).gather(1, torch.randint(0, n, (rows, 9), device=DEV, generator=gen))
    tokens[:, 0], tokens[:, 1] = 2 ** 31 - 1, -1
    tokens[:, 2] = idx[:, n - 1]
    idx = idx[0].contiguous() if shared else idx
    check(z, tokens.to(I32), min(n, 10), idx=idx)
    check(z, tokens.to(I32), 0, idx=idx)


@pytest.mark.parametrize("rows, n, dtype", [(1, 8388608, F32), (3, 8388607, F32), (65, 8388608, BF16), (1, 8388593, BF16)])
def test_alternatives_of_the_longest_rows(rows, n, dtype):
    """As many parts as the launch that joins them takes, 64 alternatives of each."""
    gen = generator(rows)
    z = rows_of(gen, rows, n, dtype)
    tokens = torch.randint(0, n, (rows, 2), device=DEV, generator=gen).to(I32)
    check(z, tokens, 64)
    z[0] = -1.0                                       # equal ones in every part
    z[0, n - 3:] = 2.0
    check(z[:1], tokens[:1], 64)
    with pytest.raises(sv.SpecVocabError):
        sv.token_logprobs(torch.empty((1, 8388609), dtype=dtype, device=DEV), top=1)


def test_more_rows_than_a_launch_takes():
    gen = generator(5)
    for rows, dtype in ((2 ** 24 + 5, F32), (2 ** 24 + 5, BF16)):              # launches of fewer than 2^32 threads, 256 a row
        z = torch.empty((rows, 2), device=DEV).normal_(0, 2, generator=gen).to(dtype)
        z[rows - 1, 0] = float("-inf")
        check(z, torch.randint(-1, 3, (rows, 1), device=DEV, generator=gen).to(I32), 2)
    rows = 2 ** 23 + 3                                                         # 512 a row
    for dtype in (F32, BF16):
        z = torch.empty((rows, 3), device=DEV).normal_(0, 2, generator=gen).to(dtype)
        tokens = torch.randint(0, 3, (rows, 1), device=DEV, generator=gen).to(I32)
        grad_check(z, tokens, torch.randn((rows, 1), device=DEV, generator=gen), torch.randn(rows, device=DEV, generator=gen), None, dtype)
        for kind in ("logits", "rest"):
            teacher = torch.log_softmax(torch.randn((rows, 2), device=DEV, generator=gen), dim=1) - 0.2
            tok = torch.cat((tokens, (tokens + 1) % 3), dim=1).to(I32)
            distill_check(z, tok, teacher, kind, out=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("start", [0, 1, 7])
@pytest.mark.parametrize("n", [262136, 262137, 262138, 262144, 262145])
def test_rows_that_just_fit_a_part(n, start, dtype):
    """A row of up to 2^18 - 7 places is one part wherever it begins, a longer one two."""
    gen = generator(n + start)
    code = sv.SV_F32 if dtype == F32 else sv.SV_BF16
    for op in (sv.SV_OP_TOKEN_LOGPROBS, sv.SV_OP_DISTILL):
        assert (sv.workspace_bytes(op, 260, k=n, dt=code) > 0) == (n > 262137)
    z = rows_of(gen, 260, n, dtype, 1, start)
    check(z, torch.randint(0, n, (260, 2), device=DEV, generator=gen).to(I32), 5)
    z, tok, t = inputs(gen, 260, n, 20, "rest", dtype, pad=1, start=start)
    tok[:, 0], tok[:, 1] = 0, n - 1
    distill_check(z, tok, t, "rest", out=dtype)
