"""Norm, products and sampling where a value, a range or a size is at its edge."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2602_13836_amd as sv
from plain import sample_row

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def drawn(z, u, t=None, k=None, p=None, m=None):
    dev = lambda v, dt=torch.float32: None if v is None else torch.as_tensor(v, dtype=dt).to(DEV)  # noqa: E731
    tok, prob = sv.sample(z.to(DEV), dev(u), dev(t), dev(k, torch.int32), dev(p), dev(m))
    return tok.cpu().numpy(), prob.cpu().numpy()


def check_rows(z, s, which):
    tok, prob = drawn(torch.from_numpy(z), **s)
    for r in which:
        f = {x: float(np.float32(s[x][r])) for x in ("t", "p", "m")}
        at, pr = sample_row(z[r], s["u"][r], f["t"], int(s["k"][r]), f["p"], f["m"])
        # one rounding to float32, and sums that are 64-bit ones up to 2^-40
        assert tok[r] == at and abs(prob[r] - pr) <= pr * (2.0 ** -24 + 2.0 ** -40) + 1e-38, (r, tok[r], at, prob[r], pr)


@pytest.mark.parametrize("rows, n", [(24, 20000), (24, 16385), (24, 49151), (100, 70001), (300, 20000)])
def test_masked_first_places_and_a_rest_far_below_zero(rows, n):
    """The first places, by which a workgroup guesses where its row's logits lie, say nothing; all others have no mass next to zero."""
    rng = np.random.default_rng(n + rows)
    z = np.full((rows, n), -np.inf, np.float32)
    t = rng.choice([0.1, 0.3, 1.0], rows)
    below = np.where(np.arange(rows) % 4 < 2, 80.0, 1000.0) * t        # 61 T below zero the first guess ends
    rest = rng.standard_normal((rows, n - 9000)) * t[:, None] - below[:, None]
    z[:, 9000:] = rest
    z[1::6, :9000] = np.nan
    z[2::6, 9000:] = np.finfo(np.float32).min
    z[3::6, 9000:] = -np.inf
    z[3::6, n - 1] = -500.0
    s = dict(u=rng.random(rows, dtype=np.float32), t=t, k=rng.choice([0, 0, 1, 50, 3000], rows), p=rng.choice([1.0, 0.0, 0.5, 0.95], rows),
             m=rng.choice([0.0, 0.0, 0.05, 1.0], rows))
    check_rows(z, s, range(min(rows, 60)))
    z[:, :9000] = -np.inf
    check_rows(z, dict(s, k=np.zeros(rows), p=np.ones(rows), m=np.zeros(rows)), range(min(rows, 60)))


@pytest.mark.parametrize("rows, n", [(3, 20000), (70, 50000)])
@pytest.mark.parametrize("top, t", [(1e8, 0.243), (-1e8, 0.245), (16777216.0, 0.07), (1000.0, 1.9e-6)])
def test_logits_whose_neighbours_are_dozens_of_octaves_away(rows, n, top, t):
    """Steps of a float between 24 and 48 octaves of weight: what lies one below the largest has little mass, but neither none nor more."""
    rng = np.random.default_rng(rows)
    top = np.float32(top)
    next_down = np.nextafter(top, np.float32(-np.inf))
    z = np.full((rows, n), -np.inf, np.float32)
    for r in range(rows):                                     # a few, whose places are ranked, or a crowd
        z[r, rng.permutation(n)[:n if r % 3 == 2 else 1000]] = next_down
    z[:, 100] = top
    z[1::2, 12000:][z[1::2, 12000:] == next_down] = np.nextafter(next_down, np.float32(-np.inf))
    ones = np.ones(rows)
    s = dict(u=np.where(np.arange(rows) % 2 == 0, np.float32(0.5), np.float32(1 - 2.0 ** -24)), t=ones * t, k=0 * ones, p=ones, m=0 * ones)
    check_rows(z, s, range(min(rows, 6)))


@pytest.mark.parametrize("rows, n", [(1, 1 << 22), (66, 1 << 21)])
@pytest.mark.parametrize("octaves", [39.4, 40.6, 42.0])
@pytest.mark.parametrize("t", [1.0, 0.37, 1.7])
def test_a_crowd_of_far_places_has_its_mass(rows, n, octaves, t):
    """One place of mass 1 and millions of equal ones whose masses only together are something: against exact fractions."""
    t = float(np.float32(t))
    z = torch.full((rows, n), -octaves * math.log(2.0) * t, device=DEV)
    first = 1000
    z[:, first] = 0.0
    w = Fraction(math.exp(float(z[0, 0]) / t))
    most = Fraction(1) - Fraction(1, 1 << 24)
    for p in (None, most):
        u = [most] * rows if p is None else [Fraction(3, 4)] + [most] * (rows - 1)
        tok, prob = drawn(z, [float(x) for x in u], t=[t] * rows, p=None if p is None else [float(p)] * rows)
        kept = 1 + (n - 1) * w
        if p is not None:
            count = max(math.ceil((p * kept - 1) / w), 0)
            kept = 1 + count * w
        for r in range(0, rows, 13):
            j = math.floor((u[r] * kept - 1) / w) if u[r] * kept >= 1 else -1
            place = first if j < 0 else (j if j < first else j + 1)
            # w is right to 2^-46 (an exponent up to 64, rounded twice), the product u * kept to 2^-53: less than one of 2^22 places
            assert abs(int(tok[r]) - place) <= 1, (r, p, int(tok[r]), place)
            want = float((1 if j < 0 else w) / kept)
            assert abs(prob[r] - want) <= want * (2.0 ** -24 + 2.0 ** -40), (r, p, prob[r], want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [16, 256, 4096, 16400, 40000])
@pytest.mark.parametrize("residual", [False, True])
def test_a_norm_of_an_infinity_or_nan_is_nan_throughout(dtype, d, residual):
    x = torch.randn((6, d), generator=torch.Generator().manual_seed(d)).to(dtype)
    x[1, d - 1], x[2, 3], x[3, d // 2], x[4, 0] = math.inf, -math.inf, math.nan, math.inf
    x[4, 1] = -math.inf
    w = torch.ones(d, dtype=dtype, device=DEV)
    res = torch.zeros_like(x).to(DEV) if residual else None
    y, t, q = sv.rms_norm(x.to(DEV), w, 1e-5, residual=res, want_quantized=True)
    assert y[1:5].isnan().all() and not y[0].isnan().any() and not y[5].isnan().any()
    blocks = (d + 127) // 128
    scales = q.scales.view(torch.uint8)
    assert (scales[1:5, :blocks] == 255).all() and (scales[1:5, blocks:] == 127).all()
    assert ((q.q.view(torch.uint8)[1:5] & 127) == 127).all() and (scales[[0, 5], :blocks] != 255).all()
    assert torch.equal(t.cpu().nan_to_num(nan=7.0), x.nan_to_num(nan=7.0))
    alone = sv.rms_norm(x[:1].to(DEV), w, 1e-5)[0]
    assert torch.equal(y[:1], alone)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [16, 272, 4096, 16400, 40000])
@pytest.mark.parametrize("eps", [0.0, 1e-5, 1e-37, 1e38])
def test_a_norm_whose_squares_leave_the_range_of_float32(dtype, d, eps):
    """Values whose squares are too large or too small for float32; the norm itself is an ordinary number."""
    rng = np.random.default_rng(d)
    base = torch.from_numpy(rng.standard_normal(d))
    largest = torch.finfo(dtype).max
    x = torch.stack([(base * s).clamp(-largest, largest).to(dtype) for s in (1e19, 1e30, 1e38, 1e-19, 1e-25, 1e-36, 1.0)] +
                    [torch.full((d,), largest, dtype=dtype), torch.full((d,), -torch.finfo(dtype).tiny, dtype=dtype)])
    x[5, 1::2] = 0.0
    w = torch.from_numpy(rng.standard_normal(d)).to(dtype)
    y, t, q = sv.rms_norm(x.to(DEV), w.to(DEV), eps, residual=torch.zeros_like(x).to(DEV), want_quantized=True)
    assert torch.equal(t.cpu(), x)
    t64 = x.double().numpy()
    ref = t64 / np.sqrt((t64 * t64).mean(axis=1, keepdims=True) + float(np.float32(eps))) * w.double().numpy()
    # the steps counted at test_rms_norm, and two more for eps's factors; results below the smallest normal number are off by half a
    # step of it, whatever they are multiplied with afterwards (|w| < 8)
    chain = 8 * -(-d // 8192) if d > 8192 else 8 * 4
    rel = (0.5 * (2 * chain + 22 + 4) + 6) * 2.0 ** -24
    half = torch.finfo(dtype).eps / 2
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= np.abs(ref) * (rel + half * (1 + rel)) + 8 * torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps).all()
    alone = sv.quantize_rows(y)
    assert torch.equal(q.q.view(torch.uint8), alone.q.view(torch.uint8)) and torch.equal(q.scales.view(torch.uint8), alone.scales.view(torch.uint8))


def small_rows(rows, d, seed):
    """QuantizedRows of small integers, scale 1, and the same in 64 bits: sums are exact in float32."""
    v = torch.randint(-3, 4, (rows, d), generator=torch.Generator().manual_seed(seed)).float()
    s = torch.full((rows, sv.scale_columns(d)), 127, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    return sv.QuantizedRows(v.to(torch.float8_e4m3fn).to(DEV), s.to(DEV)), v.double()


@pytest.mark.parametrize("d", [256, 4096, 8208, 16400])
@pytest.mark.parametrize("rows", [1, 3, 40, 70])
@pytest.mark.parametrize("h8", [True, False], ids=["h8", "hbf16"])
def test_large_hidden_values_by_small_embeddings_and_the_reverse(rows, d, h8):
    """Codes of +-448 at scales of 2^91 and 2^-110, and of 2^-90 and 2^110: every sum is a multiple of 2^12 * 2^(e + f), below 2^24 of them."""
    gen = torch.Generator().manual_seed(d + rows)
    signs = lambda n: torch.randint(0, 2, (n, d), generator=gen).float() * 2 - 1  # noqa: E731
    hv, uv = signs(rows), signs(300)

    def rows8(v, e):
        s = torch.full((v.shape[0], sv.scale_columns(d)), 127 + e, dtype=torch.uint8).view(torch.float8_e8m0fnu)
        return sv.QuantizedRows((v * 448).to(torch.float8_e4m3fn).to(DEV), s.to(DEV))

    for e, f in ((91, -110), (-90, 110)):
        h = rows8(hv, e) if h8 else (hv.double() * 448 * 2.0 ** e).to(torch.bfloat16).to(DEV)
        ref = (hv.double() @ uv.double().t()) * (448.0 ** 2 * 2.0 ** (e + f))
        U = rows8(uv, f)
        assert torch.equal(sv.quantized_dense_logits(h, U).cpu().double(), ref)
        idx = torch.arange(299, -1, -1, dtype=torch.int32)
        assert torch.equal(sv.quantized_subset_logits(h, U, idx.to(DEV)).cpu().double(), ref.flip(1))


def equal_by_parts(got, full, at, part=1 << 24):
    for j in range(0, got.shape[1], part):
        assert torch.equal(got[:, j:j + part], full[:, at[j:j + part].long()]), j


def test_a_vocabulary_of_more_rows_than_a_launch_has_threads_for():
    V, d, kinds = (1 << 28) + 37, 16, 1000
    few, v64 = small_rows(kinds, d, 1)
    h, h64 = small_rows(1, d, 2)
    q = torch.empty((V, d), dtype=torch.uint8, device=DEV)
    at = torch.arange(V, dtype=torch.int32, device=DEV) % kinds
    for j in range(0, V, 1 << 24):
        q[j:j + (1 << 24)] = few.q.view(torch.uint8)[at[j:j + (1 << 24)].long()]
    scales = torch.full((V, 4), 127, dtype=torch.uint8, device=DEV)
    U = sv.QuantizedRows(q.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu))
    equal_by_parts(sv.quantized_dense_logits(h, U), (h64 @ v64.t()).float().to(DEV), at)


@pytest.mark.parametrize("rows, k, d", [(1, (1 << 26) + 5, 4112), (2, (1 << 30) + 5, 8208)])
def test_lists_of_more_tokens_than_a_launch_has_threads_for(rows, k, d):
    V = 100
    U, u64 = small_rows(V, d, 3)
    h, h64 = small_rows(rows, d, 4)
    idx = torch.empty(k, dtype=torch.int32, device=DEV)
    for j in range(0, k, 1 << 24):
        idx[j:j + (1 << 24)] = (torch.arange(j, min(j + (1 << 24), k), device=DEV) * 7 % V).to(torch.int32)
    idx[-1] = 99
    equal_by_parts(sv.quantized_subset_logits(h, U, idx), (h64 @ u64.t()).float().to(DEV), idx)


def test_what_is_no_tensor_is_named():
    z, u = torch.zeros((2, 8), device=DEV), torch.zeros(2, device=DEV)
    x = torch.zeros((2, 256), dtype=torch.bfloat16, device=DEV)
    U = sv.quantize_rows(x)
    for name, call in [("temperature", lambda: sv.sample(z, u, temperature=0.8)), ("top_k", lambda: sv.sample(z, u, top_k=5)),
                       ("top_p", lambda: sv.sample(z, u, top_p=0.9)), ("min_p", lambda: sv.sample(z, u, min_p=0.1)),
                       ("u", lambda: sv.sample(z, 0.5)), ("logits", lambda: sv.sample([[0.0]], u)), ("idx", lambda: sv.sample(z, u, idx=[1])),
                       ("workspace", lambda: sv.sample(z, u, ws=100)), ("tok_out", lambda: sv.sample(z, u, tok_out=[0, 0])),
                       ("x", lambda: sv.quantize_rows(None)), ("weight", lambda: sv.rms_norm(x, 1.0, 1e-5)),
                       ("residual", lambda: sv.rms_norm(x, x[0], 1e-5, residual=0.0)), ("U", lambda: sv.quantized_dense_logits(x, U.q)),
                       ("U", lambda: sv.quantized_dense_logits(x, None)), ("h", lambda: sv.quantized_dense_logits([1.0], U)),
                       ("the quantized output", lambda: sv.quantize_rows(x, U.q)), ("idx", lambda: sv.quantized_subset_logits(x, U, [1, 2]))]:
        with pytest.raises(TypeError, match=name + " must be"):
            call()
