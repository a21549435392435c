"""Distillation of rows whose first 8192 places, from which the sums' reference is taken, lie far below the others: probabilities down to 2^-126 count."""
import math

import pytest
import torch

import paper_2602_13836_amd as sv
from test_gpu_distill import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


@pytest.mark.parametrize("dtype, out", [(F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("kind", ["logits", "logprobs", "rest"])
@pytest.mark.parametrize("rows, n", [(40, 20001), (30, 100003)])
def test_references_far_below(rows, n, kind, dtype, out):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    for below in (0.0, 20.0, 45.0, 60.0, 62.0, 70.0):                     # natural logarithms: 90 octaves are 62.4
        for above in (0.0, 15.0, 28.0, 40.0, 80.0):
            z = torch.empty((rows, n), device=DEV).normal_(0, 1, generator=gen)
            z[:, :n - 5000] -= below
            tok = torch.randint(n - 5000, n, (rows, 3), device=DEV, generator=gen)
            z.scatter_(1, tok, above + torch.randn((rows, 3), device=DEV, generator=gen))
            z = z.to(dtype)
            # the list has all of the teacher's mass, nearly all of it, or half
            for mass in (1.5, 1 - 2.0 ** -20, 0.5):
                t = torch.log_softmax(torch.randn((rows, 3), device=DEV, generator=gen), dim=1) + math.log(mass)
                check(z, tok.to(I32), t, kind, out=out)
            # a small factor, as of a mean over many tokens
            check(z, tok.to(I32), t, kind, weight=torch.full((rows,), 2.0 ** -30, device=DEV), out=out)
