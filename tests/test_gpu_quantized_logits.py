"""Products with an embedding in 8 bits against 64-bit products of the values that codes and scales stand for."""
import numpy as np
import pytest
import torch

import paper_2602_13836_amd as sv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def small_integers(gen, rows, d, most, pad=0):
    return torch.randint(-most, most + 1, (rows, d + pad), generator=gen).float()[:, :d]


def as_rows(codes, exps, pad=0):
    """QuantizedRows of given values (exact in e4m3) and block exponents [rows x blocks]."""
    rows, d = codes.shape
    q = torch.full((rows, d + pad), 0x55, dtype=torch.uint8).view(torch.float8_e4m3fn)
    q[:, :d] = codes.to(torch.float8_e4m3fn)
    s = torch.full((rows, sv.scale_columns(d) + (4 if pad else 0)), 255, dtype=torch.uint8)    # never read past the last block
    s[:, :exps.shape[1]] = (exps + 127).to(torch.uint8)
    return sv.QuantizedRows(q.to(DEV)[:, :d], s.to(DEV).view(torch.float8_e8m0fnu)[:, :sv.scale_columns(d)])


def stands_for(r):
    d = r.q.shape[1]
    e = r.scales.view(torch.uint8).cpu().double() - 127
    return r.q.cpu().float().double() * torch.exp2(e).repeat_interleave(128, dim=1)[:, :d]


def case(seed, rows, d, V, h8, pad=0, most=4):
    """Integers times powers of two small enough that every sum is exact in float32: 16 * 16 * 4096 * 4 < 2^24."""
    gen = torch.Generator().manual_seed(seed)
    nb = (d + 127) // 128
    U = as_rows(small_integers(gen, V, d, most), torch.randint(-1, 2, (V, nb), generator=gen), pad)
    hv = small_integers(gen, rows, d, most)
    if h8:
        h = as_rows(hv, torch.randint(-1, 2, (rows, nb), generator=gen), pad)
        h64 = stands_for(h)
    else:
        h = torch.full((rows, d + pad), 7.0, dtype=torch.bfloat16, device=DEV)[:, :d]
        h.copy_(hv)
        h64 = hv.double()
    return h, U, (h64 @ stands_for(U).t())


def lists(seed, rows, V, k, mode, padded):
    gen = torch.Generator().manual_seed(seed + 1)
    idx = torch.stack([torch.randperm(V, generator=gen)[:k] for _ in range(rows if mode == "own" else 1)]).to(torch.int32)
    if padded:
        idx[torch.rand(idx.shape, generator=gen) < 0.3] = -1
    return idx if mode == "own" else idx[0].contiguous()


def spread(r, stride):
    """The same rows `stride` bytes apart."""
    rows, d = r.q.shape
    q = torch.empty(((rows - 1) * stride + d,), dtype=torch.uint8, device=DEV).as_strided((rows, d), (stride, 1)).view(torch.float8_e4m3fn)
    q.copy_(r.q)
    return sv.QuantizedRows(q, r.scales)


@pytest.mark.parametrize("rows", [1, 5, 40, 70, 140])
def test_rows_gigabytes_apart(rows):
    """An embedding whose rows 32 bits do not reach, by list (5 MB apart) and from a tile's first row (17 MB apart)."""
    h, U, full = case(rows, rows, 256, 900, True)
    far = spread(U, 5_000_000 // 16 * 16)
    idx = lists(rows, rows, 900, 400, "shared", False)
    assert torch.equal(sv.quantized_subset_logits(h, far, idx.to(DEV)).cpu().double(), picked(full, idx))
    own = lists(rows, rows, 900, 500, "own", True)
    assert torch.equal(sv.quantized_subset_logits(h, far, own.to(DEV), padded=True).cpu().double(), picked(full, own))
    del far
    few = sv.QuantizedRows(U.q[:300], U.scales[:300])
    assert torch.equal(sv.quantized_dense_logits(h, spread(few, 17_000_000 // 16 * 16)).cpu().double(), full[:, :300])


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("rows, n, d", [(3, 30000, 144), (20, 30000, 144), (20, 70000, 656), (25, 90000, 144), (40, 40000, 144), (60, 70000, 656),
                                        (33, 82000, 144), (90, 30000, 144), (150, 40000, 144), (300, 40000, 144), (40, 70000, 8192), (20, 40000, 8192)])
def test_long_lists_of_near_and_far_rows(rows, n, d, far):
    """Tokens come several times; rows that 32 bits do not reach."""
    h, U, full = case(rows, rows, d, 900, False)
    idx = torch.randint(0, 900, (n,), generator=torch.Generator().manual_seed(n)).to(torch.int32)
    got = sv.quantized_subset_logits(h, spread(U, 5_000_000 // 16 * 16) if far else U, idx.to(DEV))
    assert torch.equal(got, full.to(DEV).float()[:, idx.to(DEV).long()])


def picked(full, idx):
    at = idx.long().expand(full.shape[0], -1)
    return full.gather(1, at.clamp(min=0)).masked_fill(at < 0, -np.inf)


SHAPES = [
    # rows, d, V, k
    (1, 16, 5, 1), (1, 144, 300, 77), (1, 1024, 1000, 1000), (1, 3840, 700, 301), (1, 4096, 900, 333), (1, 8192, 200, 50), (1, 8208, 150, 33),
    (1, 20000, 64, 7), (2, 256, 300, 100), (3, 4096, 500, 129), (5, 272, 1000, 64), (15, 2048, 1200, 300), (16, 512, 3000, 1100), (17, 528, 2000, 65),
    (32, 1040, 900, 600), (33, 4096, 600, 520), (60, 2560, 3000, 700), (64, 256, 2049, 300), (65, 512, 1500, 400), (100, 4096, 700, 300),
    (128, 1024, 3000, 900), (129, 144, 4000, 200), (200, 3840, 600, 200), (256, 512, 2000, 300), (300, 272, 1111, 1111), (513, 128, 700, 64),
    (20, 16, 300, 50), (70, 48, 300, 20), (33, 128, 500, 1),
    (5000, 64, 40, 3), (700, 16, 20, 1), (70, 48, 3000, 1500), (33, 144, 5000, 1200), (7, 528, 9000, 4000), (300, 272, 40000, 33000),
    (140, 656, 3000, 900), (64, 128, 20000, 1000),
    (90, 272, 30000, 26000), (180, 528, 15000, 13000),
    (20, 8208, 300, 40), (70, 16400, 200, 50),               # scales of a tile's rows do not fit into LDS
    # lists of every length class of the ring (tiles of 32, 64, 128 and 256 items, the last of a width that fills rounds), ragged
    (3, 400, 9000, 8000), (31, 144, 17001, 12345), (8, 272, 33001, 20000), (32, 128, 70001, 66000), (64, 144, 9001, 8500),
    (40, 256, 20000, 16385), (63, 272, 40001, 30000), (50, 144, 80003, 500),
    # tiles of the alternating loop past a round: 128 x 256 and 256 x 256
    (97, 144, 40003, 300), (260, 272, 33333, 300), (129, 400, 35000, 33000),
]


@pytest.mark.parametrize("h8", [True, False], ids=["h8", "hbf16"])
@pytest.mark.parametrize("rows, d, V, k", SHAPES)
def test_logits_are_exact_where_float32_is(rows, d, V, k, h8):
    h, U, full = case(rows * 31 + d, rows, d, V, h8)
    assert torch.equal(sv.quantized_dense_logits(h, U).cpu().double(), full)
    for mode in ("shared", "own"):
        for padded in (False, True):
            idx = lists(rows + d, rows, V, k, mode, padded)
            got = sv.quantized_subset_logits(h, U, idx.to(DEV), padded=padded)
            assert torch.equal(got.cpu().double(), picked(full, idx)), (mode, padded)


@pytest.mark.parametrize("rows, d, V, k", [(1, 528, 500, 100), (4, 528, 500, 100), (40, 272, 2500, 600), (150, 1040, 1300, 200)])
@pytest.mark.parametrize("h8", [True, False], ids=["h8", "hbf16"])
def test_rows_far_apart(rows, d, V, k, h8):
    h, U, full = case(d + rows, rows, d, V, h8, pad=48)
    assert torch.equal(sv.quantized_dense_logits(h, U).cpu().double(), full)
    idx = lists(3, rows, V, k, "own", False)
    assert torch.equal(sv.quantized_subset_logits(h, U, idx.to(DEV)).cpu().double(), picked(full, idx))


@pytest.mark.parametrize("rows, d, V", [(1, 4096, 3000), (2, 4096, 3000), (48, 3840, 2000), (70, 4096, 2000), (256, 4096, 1500)])
@pytest.mark.parametrize("h8", [True, False], ids=["h8", "hbf16"])
def test_logits_of_ordinary_values(rows, d, V, h8):
    gen = torch.Generator().manual_seed(rows)
    U = sv.quantize_rows((torch.randn((V, d), generator=gen) * 0.02).to(DEV))
    h = torch.randn((rows, d), generator=gen).to(DEV).to(torch.bfloat16)
    h64 = h.cpu().double()
    if h8:
        h = sv.quantize_rows(h)
        h64 = stands_for(h)
    u64 = stands_for(U)
    ref = h64 @ u64.t()
    err = (sv.quantized_dense_logits(h, U).cpu().double() - ref).abs()
    # products are exact; any order of d - 1 additions is off by at most (d - 1) 2^-24 of the sum of magnitudes, to first order
    bound = (d * 2.0 ** -24) * (h64.abs() @ u64.abs().t())
    assert (err <= bound).all()
    # and errors of that many independent roundings do not pile up: a tenth of the bound in the mean
    assert err.mean() <= 0.1 * bound.mean()


def test_scales_of_every_size_and_nan():
    d, V = 256, 40
    gen = torch.Generator().manual_seed(1)
    codes = small_integers(gen, V, d, 4)
    exps = torch.zeros((V, 2), dtype=torch.int64)
    exps[1], exps[2], exps[3, 0], exps[4, 1], exps[5] = 100, -100, 128, 128, -127
    U = as_rows(codes, exps)
    U.q.view(torch.uint8)[6, 255] = 0x7F
    U.q.view(torch.uint8)[7, 0] = 0xFF
    for rows in (1, 3, 70):
        hv = small_integers(gen, rows, d, 4)
        hv[:, 0] = hv[:, 255] = 1.0
        h = as_rows(hv, torch.zeros((rows, 2), dtype=torch.int64))
        got = sv.quantized_dense_logits(h, U).cpu().double()
        ref = hv.double() @ stands_for(U).t()
        bad = [3, 4, 6, 7]
        assert got[:, bad].isnan().all()
        ok = [v for v in range(V) if v not in bad + [5]]
        assert torch.equal(got[:, ok], ref[:, ok])
        # 2^-127: a code of 1 widens to a number below the smallest normal one, which the matrix cores may take for nothing:
        # 256 of them times at most 4
        assert ((got[:, 5] - ref[:, 5]).abs() <= 256 * 4 * 2.0 ** -127).all()
        assert (got[:, 5].abs() <= 4096 * 2.0 ** -120).all()
    h.q.view(torch.uint8)[1, 9] = 0x7F
    h.scales.view(torch.uint8)[2, 1] = 255
    got = sv.quantized_dense_logits(h, U)
    assert got[1:3].isnan().all() and not got[0, 0].isnan() and not got[3:, 8:].isnan().any()


def test_hidden_rows_after_a_quantisation_and_many_row_groups_are_the_same_as_alone():
    gen = torch.Generator().manual_seed(11)
    U = sv.quantize_rows(torch.randn((3000, 1024), generator=gen).to(DEV))
    h = torch.randn((90, 1024), generator=gen).to(DEV).to(torch.bfloat16)
    h8 = sv.quantize_rows(h)
    widened = torch.from_numpy(stands_for(h8).float().numpy()).to(DEV).to(torch.bfloat16)
    assert torch.equal(sv.quantized_dense_logits(h8, U), sv.quantized_dense_logits(widened, U))


def test_repeated_tokens_and_lists_of_one():
    h, U, full = case(9, 20, 256, 900, True)
    idx = torch.full((20, 900), 17, dtype=torch.int32)
    idx[:, 400:] = torch.arange(500, dtype=torch.int32)
    assert torch.equal(sv.quantized_subset_logits(h, U, idx.to(DEV)).cpu().double(), picked(full, idx))
    one = torch.tensor([899], dtype=torch.int32)
    assert torch.equal(sv.quantized_subset_logits(h, U, one.to(DEV)).cpu().double(), picked(full, one))


def test_captured_on_another_stream_and_with_workspaces_of_their_own():
    h, U, full = case(21, 40, 512, 2500, True)
    h2, _, _ = case(22, 40, 512, 2500, True)
    ref2 = stands_for(h2) @ stands_for(U).t()
    idx = lists(4, 40, 2500, 700, "own", True)
    dev_idx = idx.to(DEV)
    sv.init()
    side = torch.cuda.Stream()
    n = sv.workspace_bytes(sv.SV_OP_QUANTIZED_SUBSET_LOGITS, 40, 512, 2500, 700, dt=sv.SV_E4M3, idx_mode=sv.SV_IDX_PADDED)
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    out = torch.empty((40, 700), device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sv.quantized_subset_logits(h, U, dev_idx, out=out, ws=ws[:n], padded=True)
    side.synchronize()
    assert torch.equal(out.cpu().double(), picked(full, idx)) and (ws[n:] == 0xA5).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sv.quantized_subset_logits(h, U, dev_idx, out=out, ws=ws[:n], padded=True)
    first = sv.QuantizedRows(h.q.clone(), h.scales.clone())
    for source, ref in ((first, full), (h2, ref2), (first, full), (h2, ref2)):
        h.q.copy_(source.q)
        h.scales.copy_(source.scales)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().double(), picked(ref, idx))
        assert torch.equal(sv.quantized_subset_logits(h, U, dev_idx, padded=True), out)


def test_refusals_of_the_binding():
    h, U, _ = case(1, 3, 256, 100, True)
    with pytest.raises(TypeError):
        sv.quantized_dense_logits(torch.zeros((3, 256), device=DEV), U)
    with pytest.raises(ValueError):
        sv.quantized_dense_logits(sv.QuantizedRows(h.q, h.scales[:2]), U)
    with pytest.raises(ValueError):
        sv.quantized_dense_logits(torch.zeros((3, 128), device=DEV, dtype=torch.bfloat16), U)
    with pytest.raises(ValueError):
        sv.quantized_dense_logits(h, U, out=torch.zeros((3, 99), device=DEV))
    with pytest.raises(ValueError):
        sv.quantized_dense_logits(*case(1, 40, 256, 1000, True)[:2], ws=torch.zeros(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        sv.quantized_dense_logits(sv.QuantizedRows(h.q.cpu(), h.scales.cpu()), U)
    with pytest.raises(ValueError):
        sv.quantized_subset_logits(h, U, torch.zeros((2, 4), dtype=torch.int32, device=DEV))
