"""Given tokens are looked up in lists of up to 2^31 - 1 ids; the walk over such a list steps past 2^31 before it ends."""
import math

import pytest
import torch

import paper_2602_13836_amd as sv
import plain_rows as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 1024])
def test_a_list_of_2_to_the_31_ids(n):
    # 4.3 GB of logits, 8.6 GB of ids
    z = torch.zeros((1, n), dtype=torch.bfloat16, device=DEV)
    idx = torch.arange(n, dtype=I32, device=DEV)
    z[0, n - 1], z[0, n - 2], z[0, 7], z[0, n - 1023] = 5.0, 3.0, 4.0, -2.0
    idx[n - 4] = 9                                        # a second place of token 9: the first counts
    z[0, n - 4] = 2.0
    tokens = torch.tensor([[n - 1, n - 2, 7, n - 1023, 9, n - 4, -1, n // 2]], dtype=I32, device=DEV)
    log_s = math.log(n - 5 + math.exp(5) + math.exp(3) + math.exp(4) + math.exp(-2) + math.exp(2))
    # (token n - 4 has lost its place to token 9)
    want = [5 - log_s, 3 - log_s, 4 - log_s, -2 - log_s, -log_s, -math.inf, -math.inf, -log_s]
    # 2^18 places a part, 32 of the 8192 parts in a thread of the launch that joins them
    tol = 2 * plain.sum_error(1 << 18) + 64 * plain.STEP
    for ids in (idx, idx.unsqueeze(0)):
        got = sv.token_logprobs(z, tokens, idx=ids).logprob[0].tolist()
        for a, b in zip(got, want):
            assert a == b or abs(a - b) <= tol, (got, want)
