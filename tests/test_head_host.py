"""What the entry points between a layer's output and a token refuse, without a GPU: every check is made before anything is enqueued.
And the plain forms that the GPU tests compare with, against values worked out by hand."""
import math

import numpy as np
import pytest

import paper_2602_13836_amd as sv
from paper_2602_13836_amd import build as sv_build
from plain import E4M3, quantize, sample_row, to_e4m3, values

import os

P = 4096                       # a pointer that is 16-byte aligned and never followed
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sv.LIB_PATH):
        sv_build.build_library()
    return sv.load_library()


def quant(lib, **kw):
    a = dict(x=P, rows=2, d=256, ldx=256, dt=1, q=P, ldq=256, s=P, lds=4) | kw
    return lib.specvocab_quantize_rows(*a.values(), None)


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL), (dict(dt=2), DTYPE), (dict(dt=-1), DTYPE),
    (dict(rows=0), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(d=0), SHAPE), (dict(ldx=255), SHAPE), (dict(ldq=240), SHAPE),
    (dict(lds=0), SHAPE), (dict(d=250, ldx=256), UNSUPPORTED), (dict(d=1 << 25, ldx=1 << 25), UNSUPPORTED),
    (dict(x=P + 8), ALIGN), (dict(q=P + 8), ALIGN), (dict(s=P + 2), ALIGN), (dict(ldx=260), ALIGN), (dict(ldq=264), ALIGN),
    (dict(lds=6), ALIGN), (dict(d=528, ldx=528, ldq=528), SHAPE),
])
def test_quantize_rows_refuses(lib, kw, status):
    assert quant(lib, **kw) == status


def norm(lib, **kw):
    a = dict(x=P, rows=2, d=256, ldx=256, res=P, ldr=256, w=P, off=0.0, eps=1e-5, dt=1, sum=P, ld_sum=256, y=P, ldy=256, q=P, ldq=256,
             s=P, lds=4) | kw
    return lib.specvocab_rms_norm(*a.values(), None)


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(y=None, q=None), NULL), (dict(res=None), NULL), (dict(s=None), NULL),
    (dict(dt=2), DTYPE), (dict(rows=0), SHAPE), (dict(eps=-1e-9), SHAPE), (dict(eps=math.nan), SHAPE), (dict(eps=math.inf), SHAPE),
    (dict(off=math.nan), SHAPE), (dict(ldr=128), SHAPE), (dict(ld_sum=128), SHAPE), (dict(ldy=128), SHAPE), (dict(ldq=128), SHAPE),
    (dict(lds=3), SHAPE), (dict(d=200), UNSUPPORTED), (dict(w=P + 4), ALIGN), (dict(res=P + 4), ALIGN), (dict(y=P + 4), ALIGN),
    (dict(sum=P + 4), ALIGN), (dict(lds=7), ALIGN),
])
def test_rms_norm_refuses(lib, kw, status):
    assert norm(lib, **kw) == status


def logits(lib, name, **kw):
    a = dict(h=P, hs=P, rows=2, d=256, ldh=256, ldhs=4, U=P, Us=P, V=1000, ldu=256, ldus=4)
    if name != "dense":
        a |= dict(idx=P, k=10, mode=0)
    if name == "step":
        a |= dict(t=None, top_k=None, top_p=None, min_p=None, u=P)
    a["out"] = P
    if name == "step":
        a |= dict(tok=P, prob=None)
    a |= dict(ws=P, ws_bytes=1 << 40) | kw
    call = {"dense": lib.specvocab_quantized_dense_logits, "subset": lib.specvocab_quantized_subset_logits,
            "step": lib.specvocab_quantized_sample_step}[name]
    return call(*a.values(), None)


@pytest.mark.parametrize("name", ["dense", "subset", "step"])
@pytest.mark.parametrize("kw, status", [
    (dict(h=None), NULL), (dict(U=None), NULL), (dict(Us=None), NULL), (dict(out=None), NULL), (dict(rows=0), SHAPE),
    (dict(rows=65536), SHAPE), (dict(V=0), SHAPE), (dict(V=1 << 31), SHAPE), (dict(d=0), SHAPE), (dict(ldh=128), SHAPE), (dict(ldu=128), SHAPE),
    (dict(ldhs=2), SHAPE), (dict(ldus=3), SHAPE), (dict(d=250, ldh=256, ldu=256), UNSUPPORTED), (dict(h=P + 4), ALIGN), (dict(U=P + 4), ALIGN),
    (dict(hs=P + 1), ALIGN), (dict(Us=P + 1), ALIGN), (dict(ldh=264), ALIGN), (dict(ldus=6), ALIGN),
    (dict(hs=None, ldh=260), ALIGN), (dict(hs=None, ldh=255), SHAPE),
])
def test_quantized_logits_refuse(lib, name, kw, status):
    assert logits(lib, name, **kw) == status


def test_quantized_logits_refuse_lists_and_workspaces(lib):
    assert logits(lib, "subset", idx=None) == NULL
    for name in ("subset", "step"):
        assert logits(lib, name, k=0) == SHAPE
        assert logits(lib, name, mode=2) == DTYPE
        assert logits(lib, name, rows=64, k=300, ws=None) == WORKSPACE
        assert logits(lib, name, rows=64, k=300, ws_bytes=1000) == WORKSPACE
        assert logits(lib, name, rows=64, k=300, ws=P + 8) == ALIGN
    assert logits(lib, "dense", rows=30, ws=None) == WORKSPACE        # that many rows in 8 bits are widened there
    assert logits(lib, "step", u=None) == NULL
    assert logits(lib, "step", tok=None) == NULL


def sampling(lib, **kw):
    a = dict(z=P, ld=1000, rows=2, n=1000, idx=None, mode=0, t=None, k=None, p=None, m=None, u=P, tok=P, prob=None, ws=None, ws_bytes=0) | kw
    return lib.specvocab_sample(*a.values(), None)


@pytest.mark.parametrize("kw, status", [
    (dict(z=None), NULL), (dict(u=None), NULL), (dict(tok=None), NULL), (dict(idx=P, mode=2), DTYPE), (dict(rows=0), SHAPE),
    (dict(rows=65536), SHAPE), (dict(n=0), SHAPE), (dict(n=1 << 31, ld=1 << 31), SHAPE), (dict(ld=999), SHAPE),
    (dict(n=100000, ld=100000), WORKSPACE), (dict(n=100000, ld=100000, ws=P, ws_bytes=100), WORKSPACE),
    (dict(n=100000, ld=100000, ws=P + 8, ws_bytes=1 << 40), ALIGN),
])
def test_sample_refuses(lib, kw, status):
    assert sampling(lib, **kw) == status


def test_workspace_sizes(lib):
    sub, step = sv.SV_OP_QUANTIZED_SUBSET_LOGITS, sv.SV_OP_QUANTIZED_SAMPLE_STEP
    assert sv.workspace_bytes(sub, 1, 4096, 128256, 8192, dt=sv.SV_E4M3) == 0
    assert sv.workspace_bytes(sv.SV_OP_QUANTIZED_DENSE_LOGITS, 8, 4096, 128256, dt=sv.SV_BF16) == 0
    assert sv.workspace_bytes(sv.SV_OP_QUANTIZED_DENSE_LOGITS, 8, 4096, 128256, dt=sv.SV_E4M3) == 8 * 4096 * 2
    assert sv.workspace_bytes(sv.SV_OP_SAMPLE, 1, k=49151) == 0 and sv.workspace_bytes(sv.SV_OP_SAMPLE, 1, k=49152) > 0
    assert sv.workspace_bytes(sv.SV_OP_SAMPLE, 64, k=128256) > 0 and sv.workspace_bytes(sv.SV_OP_SAMPLE, 65, k=128256) == 0
    assert sv.workspace_bytes(step, 1, 4096, 128256, 0, dt=sv.SV_E4M3) == sv.workspace_bytes(sv.SV_OP_SAMPLE, 1, k=128256)
    plain = sv.workspace_bytes(sub, 60, 4096, 128256, 4096, dt=sv.SV_BF16)
    assert sv.workspace_bytes(sub, 60, 4096, 128256, 4096, dt=sv.SV_E4M3) == plain + 60 * 4096 * 2
    assert sv.workspace_bytes(sub, 60, 4096, 128256, 4096, dt=sv.SV_BF16, idx_mode=sv.SV_IDX_PADDED) == plain + 60 * 4096 * 4
    for op, kw, status in ((sub, dict(dt=sv.SV_F32), DTYPE), (sub, dict(idx_mode=3), DTYPE), (sub, dict(d=250), UNSUPPORTED),
                           (sub, dict(k=0), SHAPE), (step, dict(rows=0), SHAPE), (sv.SV_OP_SAMPLE, dict(k=0), SHAPE)):
        with pytest.raises(sv.SpecVocabError) as e:
            sv.workspace_bytes(op, **(dict(rows=2, d=256, V=1000, k=10, dt=sv.SV_BF16) | kw))
        assert e.value.status == status


# ---- the plain forms themselves
def test_e4m3_by_hand():
    assert E4M3[0x38] == 1.0 and E4M3[0x7E] == 448 and E4M3[1] == 2.0 ** -9 and E4M3[0xC0] == -2.0 and math.isnan(E4M3[0x7F])
    x = np.array([1.0, 1.0625, 1.1875, 448, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17, 19])
    assert [hex(c) for c in to_e4m3(x)] == ["0x38", "0x38", "0x3a", "0x7e", "0x80", "0x0", "0x2", "0x58", "0x5a"]


def test_quantize_by_hand():
    x = np.zeros((1, 272))
    x[0, 0], x[0, 1] = 448.0, 1.0
    x[0, 128] = 449.0
    codes, scales = quantize(x)
    assert list(scales[0]) == [127, 128, 127, 127] and codes[0, 0] == 0x7E and codes[0, 1] == 0x38 and codes[0, 128] == 0x76
    assert values(codes, scales)[0, 128] == 448
    assert quantize(np.full((1, 16), 2.0 ** -140))[1][0, 0] == 1 and quantize(np.full((1, 16), np.inf))[1][0, 0] == 255


def test_sample_by_hand():
    z = np.log(np.array([1.0, 4.0, 2.0, 1.0]))               # masses 4, 2, 1, 1 of 8, in the order 1, 2, 0, 3
    assert [sample_row(z, u)[0] for u in (0, 0.49, 0.51, 0.74, 0.76, 0.87, 0.88)] == [1, 1, 2, 2, 0, 0, 3]
    assert sample_row(z, 0.99, k=2) == (2, pytest.approx(1 / 3)) and sample_row(z, 0.7, p=0.7)[0] == 2
    assert sample_row(z, 0.99, p=0.5) == (1, 1.0) and sample_row(z, 0.99, m=0.3)[0] == 2 and sample_row(z, 0.9, t=0) == (1, 1.0)
    assert sample_row([-np.inf] * 3, 0.5) == (-1, 0.0) and sample_row([5.0, 5.0], 0.5)[0] == 1
