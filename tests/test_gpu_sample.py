"""Tokens drawn from given random numbers against sorting everything in 64 bits, and the steps that end in one."""
import math

import numpy as np
import pytest
import torch

import paper_2602_13836_amd as sv
from plain import sample_row

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NEG = float("-inf")


def check(z, u, t=None, k=None, p=None, m=None, idx=None, name=""):
    """One call over all rows; every row against the plain form."""
    rows, n = z.shape
    dev = lambda v, dt: None if v is None else torch.as_tensor(v, dtype=dt).to(DEV)  # noqa: E731
    f = torch.float32
    tok, prob = sv.sample(z.to(DEV) if not z.is_cuda else z, dev(u, f), dev(t, f), dev(k, torch.int32), dev(p, f), dev(m, f),
                          idx=None if idx is None else idx.to(DEV))
    tok, prob, zc = tok.cpu().numpy(), prob.cpu().numpy(), z.cpu().numpy()
    f32 = lambda v, r, off: off if v is None else float(np.float32(v[r]))  # noqa: E731
    for r in range(rows):
        at, pr = sample_row(zc[r], np.float32(u[r]), f32(t, r, 1.0), 0 if k is None else int(k[r]), f32(p, r, 1.0), f32(m, r, 0.0))
        want = at if at < 0 or idx is None else int(idx[at] if idx.dim() == 1 else idx[r, at])
        assert tok[r] == want, (name, r, tok[r], want, prob[r], pr)
        # one rounding to float32, and sums that are 64-bit ones up to 2^-40
        assert abs(prob[r] - pr) <= pr * (2.0 ** -24 + 2.0 ** -40) + 1e-38, (name, r, prob[r], pr)


def language_like(rng, rows, n):
    z = rng.standard_normal((rows, n)) * 2.5
    for r in range(rows):
        top = rng.integers(0, n, min(24, n))
        z[r, top] += rng.random(top.size) * 12
    return torch.from_numpy(z.astype(np.float32))


def settings(rng, rows):
    return dict(u=rng.random(rows, dtype=np.float32), t=rng.choice([0.0, 0.5, 0.8, 1.0, 1.5, 3.0], rows), k=rng.choice([0, 0, 1, 20, 50, 1000], rows),
                p=rng.choice([1.0, 0.1, 0.8, 0.9, 0.95, 0.999], rows), m=rng.choice([0.0, 0.0, 0.02, 0.1, 0.5], rows))


SIZES = [1, 2, 3, 17, 63, 64, 65, 255, 1000, 1024, 1025, 4095, 4096, 4097, 8192, 16383, 16384, 16385, 20001, 50000, 128256, 151937]


@pytest.mark.parametrize("n", SIZES)
def test_language_like_logits_with_everything(n):
    rng = np.random.default_rng(n)
    rows = 24 if n < 50000 else 9
    s = settings(rng, rows)
    check(language_like(rng, rows, n), **s, name="mixed")
    check(language_like(rng, rows, n), u=s["u"], name="none")


@pytest.mark.parametrize("rows, n", [(300, 20000), (256, 128256), (513, 3000), (255, 17000), (64, 49152), (64, 49151), (65, 60000), (3, 200003)])
def test_many_rows(rows, n):
    rng = np.random.default_rng(rows)
    z = torch.randn((rows, n), generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV) * 3
    s = settings(rng, rows)
    keep = rng.permutation(rows)[:40]                         # (the plain form of a row takes milliseconds)
    got = sv.sample(z, *(torch.as_tensor(s[x], dtype=torch.int32 if x == "k" else torch.float32).to(DEV) for x in ("u", "t", "k", "p", "m")))
    check(z[torch.from_numpy(keep).to(DEV)], **{x: s[x][keep] for x in s}, name="a part")
    part = sv.sample(z[torch.from_numpy(keep).to(DEV)], *(torch.as_tensor(s[x][keep], dtype=torch.int32 if x == "k" else torch.float32).to(DEV)
                                                        for x in ("u", "t", "k", "p", "m")))
    at = torch.from_numpy(keep).to(DEV)
    assert torch.equal(got[0][at], part[0]) and torch.equal(got[1][at], part[1])


@pytest.mark.parametrize("n", [5, 300, 3000, 16384, 40000, 100001])
def test_every_border_by_itself(n):
    rng = np.random.default_rng(n + 1)
    for name, kw in [("k", dict(k=[1, 2, 3, n - 1, n, n + 5, 1400, 3000])), ("p", dict(p=[0.0, -1.0, 1e-7, 0.3, 0.5, 0.9, 0.9999, 1 - 2.0 ** -24])),
                     ("m", dict(m=[1.0, 2.0, 0.99, 0.5, 0.1, 1e-3, 1e-9, 1e-30])), ("t", dict(t=[1e-30, 1e-6, 0.01, 0.1, 2, 30, 1e6, math.inf])),
                     ("odd", dict(t=[math.nan, -1, 1, 1, 1, 1, 1, 1], p=[1, 1, math.nan, 2, 1, 1, 1, 1], m=[0, 0, 0, 0, math.nan, -1, math.inf, 0],
                                  k=[0, 0, 0, 0, 0, 0, 0, -5]))]:
        for u in (rng.random(8, dtype=np.float32), np.zeros(8, np.float32), np.full(8, 1 - 2.0 ** -24, np.float32),
                  np.array([-1, 1, 2, math.inf, -math.inf, 0.5, 0.25, math.nan], np.float32)):
            u = np.where(np.isnan(u), 0, u) if name != "odd" else np.nan_to_num(u, nan=0.0)
            check(language_like(rng, 8, n), u=u, name=name, **kw)


@pytest.mark.parametrize("n", [1, 700, 4096, 16384, 16390, 30000, 60000])
def test_ties_flat_rows_and_clusters(n):
    rng = np.random.default_rng(n + 2)
    few = rng.integers(0, 4, (8, n)).astype(np.float32)                        # four values
    same = np.zeros((8, n), np.float32)
    zeros = np.where(rng.random((8, n)) < 0.5, np.float32(0.0), np.float32(-0.0))
    flat = (1e-6 * rng.standard_normal((8, n)) + 30).astype(np.float32)        # a few neighbouring floats
    far = (rng.standard_normal((8, n)) * 0.01 + 20.0 * (rng.random((8, n)) < 0.3)).astype(np.float32)      # two crowds
    narrow = np.where(np.arange(n) == n // 2, 40.0, 0.001 * rng.standard_normal((8, n))).astype(np.float32)  # one far above a crowd
    s = dict(t=[1, 1, 20, 1, 0.7, 1, 1, 1000], k=[0, 0, 0, n // 2 + 1, 0, 7, 3000, 0], p=[1, 0.5, 0.9, 1, 0.999, 1, 0.7, 0.6],
             m=[0, 0, 0, 0, 0.3, 0, 0, 0.9])
    for name, z in (("few", few), ("same", same), ("zeros", zeros), ("flat", flat), ("far", far), ("narrow", narrow)):
        check(torch.from_numpy(z), u=rng.random(8, dtype=np.float32), name=name, **s)
        check(torch.from_numpy(z), u=rng.random(8, dtype=np.float32), name=name)


@pytest.mark.parametrize("n", [4, 900, 5000, 16400, 70000])
def test_masks(n):
    rng = np.random.default_rng(n + 3)
    z = language_like(rng, 10, n)
    hide = torch.from_numpy(rng.random((10, n)) < 0.9)
    z[hide] = NEG
    z[1] = NEG                                                # nothing left
    z[2] = float("nan")
    z[3, ::2] = float("nan")
    z[4] = torch.finfo(torch.float32).min                     # the lowest value everywhere: all alike
    z[5] = torch.where(hide[5], torch.finfo(torch.float32).min, torch.randn(n))
    z[6] = NEG
    z[6, n - 1] = -3.0                                        # one place left, the last
    z[7, n // 2] = float("inf")
    z[8, :2] = float("inf")
    z[9] = torch.where(hide[9], torch.finfo(torch.float32).min, z[9])
    s = settings(rng, 10)
    check(z, **s)
    check(z, u=s["u"])
    check(z, u=s["u"], p=np.full(10, 0.9), m=np.full(10, 0.01))


@pytest.mark.parametrize("rows, n", [(260, 20000), (257, 100001), (20, 20000), (100, 70001)])
def test_rows_whose_first_places_are_unlike_the_rest(rows, n):
    """Rows that a workgroup each reads, whose first 8192 places say nothing, little or the wrong thing about the rest."""
    rng = np.random.default_rng(n)
    z = language_like(rng, 14, n).numpy()
    z[0, :9000] = -np.inf                                      # nothing there
    z[1, :9000] = np.finfo(np.float32).min                     # a mask's lowest value
    z[2, :9000] = 0.0                                          # all the same
    z[3, :9000] = 0.0
    z[3, 9000:] *= 0.001
    z[4, 12000] = 60.0                                         # one far above
    z[5, 12000:12004] = [200.0, 199.9, 199.8, 150.0]
    z[6, 9000:] -= 100.0                                       # the rest far below
    z[7] = 1e-4 * rng.standard_normal(n)                       # flat, with a rest that spreads more
    z[7, 9000:] *= 50
    z[8] = 7.0                                                 # all equal
    z[9, 15000] = np.inf
    z[10, 100] = np.inf
    z[11] *= 1e37                                              # near the largest float
    z[12, ::3] = np.nan
    z[13] = np.where(rng.random(n) < 0.999, -np.inf, z[13])
    kinds = z.shape[0]
    z = np.concatenate([z] * 19)[:rows]
    s = dict(u=rng.random(rows, dtype=np.float32), t=rng.choice([0.3, 0.7, 1.0, 2.0, 1e30], rows), k=rng.choice([0, 0, 0, 40, 2000], rows),
             p=rng.choice([1.0, 0.9, 0.99], rows), m=rng.choice([0.0, 0.0, 0.05], rows))
    dev = [torch.as_tensor(s[x], dtype=torch.int32 if x == "k" else torch.float32).to(DEV) for x in ("u", "t", "k", "p", "m")]
    tok, prob = (x.cpu().numpy() for x in sv.sample(torch.from_numpy(z).to(DEV), *dev))
    for r in range(min(rows, 5 * kinds)):
        at, pr = sample_row(z[r], s["u"][r], float(np.float32(s["t"][r])), int(s["k"][r]), float(np.float32(s["p"][r])), float(np.float32(s["m"][r])))
        assert tok[r] == at and abs(prob[r] - pr) <= pr * (2.0 ** -24 + 2.0 ** -40) + 1e-38, (r, r % kinds, tok[r], at, prob[r], pr)


@pytest.mark.parametrize("rows, n", [(300, 17000), (100, 20000), (10, 60000), (5, 9000)])
def test_a_mass_of_zero_keeps_the_first_place(rows, n):
    rng = np.random.default_rng(rows)
    z = language_like(rng, rows, n)
    p = rng.choice([0.0, -0.0, -1.0, -math.inf, 1e-45, 1e-30], rows)
    tok, prob = sv.sample(z.to(DEV), torch.rand(rows, device=DEV), top_p=torch.as_tensor(p, dtype=torch.float32).to(DEV))
    assert torch.equal(tok.cpu().long(), z.argmax(dim=1)) and (prob == 1).all()


def test_lists_name_the_tokens():
    rng = np.random.default_rng(8)
    z = language_like(rng, 12, 2048)
    shared = torch.from_numpy(np.sort(rng.permutation(100000)[:2048]).astype(np.int32))
    own = torch.from_numpy(np.stack([rng.permutation(100000)[:2048] for _ in range(12)]).astype(np.int32))
    s = settings(rng, 12)
    check(z, **s, idx=shared)
    check(z, **s, idx=own)
    z[3] = NEG
    check(z, **s, idx=own)


@pytest.mark.parametrize("n, pad, shift", [(2049, 3, 1), (20001, 1, 0), (70003, 5, 3)])
def test_rows_at_any_alignment(n, pad, shift):
    rng = np.random.default_rng(n)
    whole = torch.full((7, n + pad + shift), 50.0, device=DEV)      # what lies around the rows would win
    z = whole[:, shift:shift + n]
    z.copy_(language_like(rng, 7, n))
    check(z, **settings(rng, 7))


def test_the_same_in_every_run_and_in_a_graph():
    rng = np.random.default_rng(77)
    z = torch.randn((40, 100000), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) * 2
    s = settings(rng, 40)
    a = {x: torch.as_tensor(s[x], dtype=torch.int32 if x == "k" else torch.float32).to(DEV) for x in s}
    call = lambda **kw: sv.sample(z, a["u"], a["t"], a["k"], a["p"], a["m"], **kw)  # noqa: E731
    tok, prob = call()
    for _ in range(3):
        again = call()
        assert torch.equal(again[0], tok) and torch.equal(again[1], prob)
    n = sv.workspace_bytes(sv.SV_OP_SAMPLE, 40, k=100000)
    ws, ws2 = (torch.full((n,), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2))
    t1, p1, t2, p2 = torch.empty_like(tok), torch.empty_like(prob), torch.empty_like(tok), torch.empty_like(prob)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(tok_out=t1, prob_out=p1, ws=ws)
    for seed in range(4):
        a["u"].copy_(torch.rand(40, generator=torch.Generator().manual_seed(seed)))
        with torch.cuda.stream(side):                         # at the same time, with a workspace of its own
            side.wait_stream(torch.cuda.default_stream())
            call(tok_out=t2, prob_out=p2, ws=ws2)
        g.replay()
        torch.cuda.synchronize()
        ref = call()
        assert torch.equal(t1, ref[0]) and torch.equal(p1, ref[1]) and torch.equal(t2, ref[0]) and torch.equal(p2, ref[1])
        assert torch.rand(1000, device=DEV).sum() > 0
        torch.cuda.synchronize()


@pytest.mark.parametrize("rows, n", [(1, 49152), (3, 49155), (64, 60001), (7, 151936)])
def test_nothing_beside_the_workspace_and_the_outputs_is_written(rows, n):
    rng = np.random.default_rng(rows)
    full = torch.full((rows, n + 64), 5.0, device=DEV)
    z = full[:, 32:32 + n]
    z.copy_(language_like(rng, rows, n))
    before = full.clone()
    size = sv.workspace_bytes(sv.SV_OP_SAMPLE, rows, k=n)
    ws = torch.full((256 + size + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    tok, prob = torch.full((rows + 8,), -7, dtype=torch.int32, device=DEV), torch.full((rows + 8,), -7.0, device=DEV)
    s = settings(rng, rows)
    dev = [torch.as_tensor(s[x], dtype=torch.int32 if x == "k" else torch.float32).to(DEV) for x in ("u", "t", "k", "p", "m")]
    sv.sample(z, *dev, tok_out=tok[:rows], prob_out=prob[:rows], ws=ws[256:256 + size])
    assert torch.equal(full, before) and (ws[:256] == 0x5A).all() and (ws[256 + size:] == 0x5A).all()
    assert (tok[rows:] == -7).all() and (prob[rows:] == -7).all() and (tok[:rows] >= 0).all()


def test_a_stream_that_is_still_busy_owns_what_a_call_makes():
    """The workspace and the outputs of a call on another stream are not handed out again before that stream is done with them."""
    rng = np.random.default_rng(3)
    n = 60000
    z = language_like(rng, 12, n).to(DEV)
    s = settings(rng, 12)
    dev = [torch.as_tensor(s[x], dtype=torch.int32 if x == "k" else torch.float32).to(DEV) for x in ("u", "t", "k", "p", "m")]
    U = sv.quantize_rows(torch.randn((3000, 1024), device=DEV, dtype=torch.bfloat16))
    h = sv.quantize_rows(torch.randn((80, 1024), device=DEV, dtype=torch.bfloat16))
    want, want_z = sv.sample(z, *dev), sv.quantized_dense_logits(h, U)
    nbytes = [sv.workspace_bytes(sv.SV_OP_SAMPLE, 12, k=n), sv.workspace_bytes(sv.SV_OP_QUANTIZED_DENSE_LOGITS, 80, 1024, 3000, dt=sv.SV_E4M3)]
    big = torch.randn((4096, 4096), device=DEV, dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(40):                                # some milliseconds
                big @ big
        got = sv.sample(z, *dev, stream=side)
        got_z = sv.quantized_dense_logits(h, U, stream=side)
        for b in nbytes + [12 * 4, 80 * 3000 * 4]:              # memory of those sizes, written at once on this stream
            for _ in range(3):
                torch.empty(b, dtype=torch.uint8, device=DEV).fill_(255)
        side.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got_z, want_z)


def test_draws_follow_the_distribution():
    """65000 draws from five tokens: counts of a multinomial, each within six standard deviations (1 in 5e8 for a right sampler)."""
    p = np.array([0.4, 0.3, 0.2, 0.06, 0.04])
    z = torch.from_numpy(np.log(p).astype(np.float32)).to(DEV).expand(65000, 5).contiguous()
    u = torch.rand(65000, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    tok, prob = sv.sample(z, u)
    n = torch.bincount(tok.long(), minlength=5).cpu().numpy()
    assert (np.abs(n - 65000 * p) <= 6 * np.sqrt(65000 * p * (1 - p))).all(), n
    assert np.allclose(prob.cpu().numpy(), p[tok.cpu().numpy()], rtol=1e-6)


def test_from_a_layer_to_a_token():
    """Norm, selection, logits over the selected tokens with the embedding in 8 bits, and a token: as a drafter calls them."""
    gen = torch.Generator().manual_seed(2)
    V, d, dp, k, rows = 6000, 1024, 64, 512, 6
    U = (torch.randn((V, d), generator=gen) * 0.05).to(DEV).to(torch.bfloat16)
    U8 = sv.quantize_rows(U)
    x, res = (torch.randn((rows, d), generator=gen).to(DEV).to(torch.bfloat16) for _ in range(2))
    w = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    Wd, Wv = ((torch.randn(s, generator=gen) * 0.05).to(DEV).to(torch.bfloat16) for s in ((dp, d), (V, dp)))
    u = torch.rand(rows, generator=gen).to(DEV)
    top_p = torch.full((rows,), 0.9, device=DEV)
    y, _, h8 = sv.rms_norm(x, w, 1e-5, residual=res, want_quantized=True)
    idx, _ = sv.select(y, Wd, Wv, k)
    logits, tok, prob = sv.quantized_sample_step(h8, U8, u, idx, top_p=top_p)
    assert torch.equal(logits, sv.quantized_subset_logits(h8, U8, idx))
    assert torch.equal(tok, sv.sample(logits, u, top_p=top_p, idx=idx)[0])
    check(logits.cpu(), u.cpu().numpy(), p=np.full(rows, 0.9), idx=idx.cpu())
    # the embedding in 8 bits is the embedding up to half a step of e4m3 per factor: 2^-4 each of a product, both at random
    exact = sv.subset_logits(y, U, idx)
    assert (logits - exact).abs().max() <= 6 * 2.0 ** -4 * math.sqrt(2) * float((y.float().square().sum(dim=1).max() * U.float().square().max()).sqrt())
    # the whole vocabulary, padded lists, and a workspace of one's own
    logits, tok, _ = sv.quantized_sample_step(h8, U8, u)
    assert torch.equal(logits, sv.quantized_dense_logits(h8, U8)) and torch.equal(tok, sv.sample(logits, u)[0])
    idx[:, 100:] = -1
    n = sv.workspace_bytes(sv.SV_OP_QUANTIZED_SAMPLE_STEP, rows, d, V, k, dt=sv.SV_E4M3, idx_mode=sv.SV_IDX_PADDED)
    _, tok, prob = sv.quantized_sample_step(h8, U8, u, idx, ws=torch.empty(max(n, 1), dtype=torch.uint8, device=DEV), padded=True)
    assert ((tok[:, None] == idx[:, :100]).any(dim=1)).all() and (prob > 0).all()


def test_refusals_of_the_binding():
    z, u = torch.zeros((3, 10), device=DEV), torch.zeros(3, device=DEV)
    for kw in (dict(temperature=u[:2]), dict(top_k=u), dict(top_p=u.double()), dict(min_p=u.cpu()), dict(tok_out=u),
               dict(idx=torch.zeros(9, dtype=torch.int32, device=DEV)), dict(prob_out=torch.zeros(4, device=DEV))):
        with pytest.raises(ValueError):
            sv.sample(z, u, **kw)
    with pytest.raises(TypeError):
        sv.sample(z.double(), u)
    with pytest.raises(ValueError):
        sv.sample(z.t(), u)
    with pytest.raises(ValueError):
        sv.sample(z, None)
