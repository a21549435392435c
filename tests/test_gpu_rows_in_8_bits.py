"""Rows in 8 bits and the norm that leaves them, against the plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2602_13836_amd as sv
from plain import quantize

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def wide(rng, rows, d, dtype, std, pad):
    x = torch.from_numpy((rng.standard_normal((rows, d + pad)) * std).astype(np.float32)).to(DEV).to(dtype)
    return x[:, :d]


def out_rows(rows, d, pad):
    q = torch.full((rows, d + pad), 0x55, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    s = torch.full((rows, sv.scale_columns(d) + (4 if pad else 0)), 0x55, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    return q, s, sv.QuantizedRows(q[:, :d], s[:, :sv.scale_columns(d)])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, d, pad", [(1, 16, 0), (3, 144, 0), (2, 512, 16), (5, 528, 32), (7, 1024, 0), (33, 4096, 0), (1, 8208, 16),
                                          (300, 272, 0), (2, 40000, 0)])
def test_quantize_rows_is_exact(dtype, rows, d, pad):
    rng = np.random.default_rng(rows * 100003 + d)
    x = wide(rng, rows, d, dtype, 1.0, pad)
    x *= torch.from_numpy(np.exp2(rng.integers(-30, 30, (rows, 1))).astype(np.float32)).to(DEV).to(dtype)
    q, s, out = out_rows(rows, d, pad)
    assert sv.quantize_rows(x, out) is out
    codes, scales = quantize(x.double().cpu().numpy())
    assert np.array_equal(bits(out.q), codes) and np.array_equal(bits(out.scales), scales)
    if pad:                                                   # what lies between the rows stays
        assert (bits(q[:, d:]) == 0x55).all() and (bits(s[:, sv.scale_columns(d):]) == 0x55).all()
    again = sv.quantize_rows(x)
    assert np.array_equal(bits(again.q), codes) and np.array_equal(bits(again.scales), scales)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_rows_at_the_edges_of_the_format(dtype):
    info = torch.finfo(dtype)
    rows = []
    for first in (0.0, -0.0, 448.0, 450.0, -448.0 * 2.0 ** 60, info.max, info.tiny, info.smallest_normal / 64, float("inf"), float("nan"),
                  -float("inf"), 448.0 * 2.0 ** -126, 450.0 * 2.0 ** -126, 464.0, 2.0 ** -130):
        row = torch.zeros(144, dtype=dtype)
        row[3], row[7], row[8] = first, first / 3, -first / 1000
        row[130] = 1.0625                                     # half way between two codes
        row[131] = 2.0 ** -10                                 # far below the block's largest: half the smallest code after scaling, or not
        rows.append(row)
    x = torch.stack(rows)
    got = sv.quantize_rows(x.to(DEV))
    codes, scales = quantize(x.double().numpy())
    assert np.array_equal(bits(got.scales), scales)
    assert np.array_equal(bits(got.q), codes)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, d, pad, residual, offset", [
    (1, 16, 0, True, 0.0), (1, 4096, 0, True, 0.0), (3, 144, 16, True, 1.0), (5, 3840, 0, True, 0.0), (70, 512, 0, False, 0.0),
    (2, 8208, 32, True, 0.0), (2, 16400, 0, True, 1.0), (3, 32784, 0, True, 0.0), (2, 70000, 0, False, 0.5), (700, 1040, 0, True, 0.0),
])
def test_rms_norm(dtype, rows, d, pad, residual, offset):
    rng = np.random.default_rng(rows * 7919 + d)
    x = wide(rng, rows, d, dtype, 1.0, pad)
    res = wide(rng, rows, d, dtype, 3.0, pad) if residual else None
    w = wide(rng, 1, d, dtype, 0.3, 0)[0].contiguous()
    y, total, q = sv.rms_norm(x, w, 1e-5, residual=res, weight_offset=offset, want_quantized=True)
    # the sum: one float32 addition and one rounding, the same on the CPU
    t = (x.cpu().float() + res.cpu().float()).to(dtype) if residual else x.cpu()
    assert torch.equal(total.cpu(), t)
    t64 = t.double().numpy()
    ref = t64 / np.sqrt((t64 * t64).mean(axis=1, keepdims=True) + np.float32(1e-5)) * (w.double().cpu().numpy() + offset)
    # float32 steps, each half an ulp (2^-24) of what it makes.  The sum of squares: positive terms, a square and an addition each for the
    # at most 8 ceil(d / 8192) values of a thread (a row is spread over 64 threads at least, eight values each at a time, 1024 for
    # long rows), then at most 6 + 16 additions; half of that relative error goes through the root.  Then mean, eps, root, reciprocal,
    # two products and the weight's addition; and the rounding to the storage type.
    chain = 8 * -(-d // 8192) if d > 8192 else 8 * 4
    rel = (0.5 * (2 * chain + 22 + 2) + 6) * 2.0 ** -24
    half = torch.finfo(dtype).eps / 2
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= np.abs(ref) * (rel + half * (1 + rel)) + 1e-30).all(), (err / (np.abs(ref) + 1e-30)).max()
    # the 8 bits are those of y as it is stored
    alone = sv.quantize_rows(y)
    assert torch.equal(q.q.view(torch.uint8), alone.q.view(torch.uint8)) and torch.equal(q.scales.view(torch.uint8), alone.scales.view(torch.uint8))


@pytest.mark.parametrize("d", [4096, 40000])
def test_rms_norm_in_place_and_one_output_at_a_time(d):
    rng = np.random.default_rng(5)
    x, res, w = wide(rng, 4, d, torch.bfloat16, 1.0, 0), wide(rng, 4, d, torch.bfloat16, 2.0, 0), wide(rng, 1, d, torch.bfloat16, 0.5, 0)[0].contiguous()
    y, total, q = sv.rms_norm(x, w, 1e-6, residual=res, want_quantized=True)
    only_y, t, none = sv.rms_norm(x, w, 1e-6, residual=res)
    assert none is None and torch.equal(only_y, y)
    none, t, only_q = sv.rms_norm(x, w, 1e-6, residual=res, want_y=False, want_quantized=True)
    assert none is None and torch.equal(only_q.q.view(torch.uint8), q.q.view(torch.uint8))
    x2, res2 = x.clone(), res.clone()
    y2, t2, _ = sv.rms_norm(x2, w, 1e-6, residual=res2, sum_out=res2, y_out=x2)
    assert y2 is x2 and t2 is res2 and torch.equal(x2, y) and torch.equal(res2, total)
    x3 = x.clone()
    y3, t3, _ = sv.rms_norm(x3, w, 1e-6, y_out=x3)
    assert torch.equal(x3, sv.rms_norm(x, w, 1e-6)[0]) and t3 is x3


def test_more_rows_than_a_launch_takes():
    rows = (1 << 20) + 3
    x = torch.randn((rows, 16), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    w = torch.ones(16, dtype=torch.bfloat16, device=DEV)
    y, total, q = sv.rms_norm(x, w, 1e-5, residual=x, want_quantized=True)
    tail, t2, q2 = sv.rms_norm(x[-10:], w, 1e-5, residual=x[-10:], want_quantized=True)
    assert torch.equal(y[-10:], tail) and torch.equal(total[-10:], t2)
    assert torch.equal(q.q.view(torch.uint8)[-10:], q2.q.view(torch.uint8)) and torch.equal(q.scales.view(torch.uint8)[-10:], q2.scales.view(torch.uint8))


def test_rms_norm_of_zeros_infinities_and_nan():
    x = torch.zeros((4, 256), dtype=torch.bfloat16, device=DEV)
    x[1, 5], x[2, 7] = float("inf"), float("nan")
    x[3, :] = 1.0
    w = torch.ones(256, dtype=torch.bfloat16, device=DEV)
    y, _, q = sv.rms_norm(x, w, 1e-5, want_quantized=True)
    assert (y[0] == 0).all() and (q.scales.view(torch.uint8)[0] == 127).all() and (q.q.view(torch.uint8)[0] == 0).all()
    assert y[1, 5].isnan() and y[2].isnan().all() and (q.scales.view(torch.uint8)[2, :2] == 255).all()
    assert torch.equal(y[3], x[3]) and q.q.double()[3, 0] == 256 and q.scales.double()[3, 0] == 2.0 ** -8
    # eps = 0: a row of zeros has no direction
    assert sv.rms_norm(x[:1], w, 0.0)[0].isnan().all()


def test_refusals_of_the_binding():
    x = torch.zeros((2, 256), dtype=torch.bfloat16, device=DEV)
    w = torch.zeros(256, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        sv.rms_norm(x, w[:128], 1e-5)
    with pytest.raises(ValueError):
        sv.rms_norm(x, w, 1e-5, residual=x[:1])
    with pytest.raises(ValueError):
        sv.rms_norm(x, w, 1e-5, sum_out=x)
    with pytest.raises(ValueError):
        sv.rms_norm(x, w, 1e-5, residual=x.cpu())
    with pytest.raises(TypeError):
        sv.quantize_rows(x.half())
    q = sv.quantize_rows(x)
    with pytest.raises(ValueError):
        sv.quantize_rows(x[:1], q)
    with pytest.raises(TypeError):
        sv.quantize_rows(x, sv.QuantizedRows(q.q.view(torch.uint8), q.scales))
    with pytest.raises(sv.SpecVocabError) as e:
        sv.rms_norm(x, w, -1.0)
    assert e.value.status == 2
