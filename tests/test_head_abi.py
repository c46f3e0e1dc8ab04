"""Refusals of the output head's entry points, on the host: every call here fails an
argument check and returns before any HIP call (dummy pointers, no GPU)."""
import ctypes as C
import os

import pytest

import paper_2005_04680_amd as pk
from paper_2005_04680_amd import head

FAKE = 1 << 20  # a 256-byte aligned non-null address; never dereferenced on these paths
F32, BF16 = pk.EMBBAG_F32, pk.EMBBAG_BF16
BAD, WS, OFF = pk.EMBBAG_ERR_INVALID_ARG, pk.EMBBAG_ERR_WORKSPACE, pk.EMBBAG_ERR_OFFSETS


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pk.LIB_PATH):
        import paper_2005_04680_amd.build as b
        b.build()
    return head._lib()


def call(fn, names, good, **change):
    args = dict(good, **change)
    return fn(*[args[n] for n in names])


Q_NAMES = "src type stride rows dim ids num codes scales status stream".split()
Q = dict(src=FAKE, type=F32, stride=64, rows=10, dim=64, ids=None, num=0, codes=FAKE, scales=FAKE,
         status=None, stream=None)


@pytest.mark.parametrize("change", [
    dict(src=None), dict(src=FAKE + 8), dict(type=2), dict(type=-1), dict(stride=60), dict(stride=66),
    dict(rows=0), dict(rows=2 ** 31), dict(dim=0), dict(dim=6), dict(dim=16388, stride=16388), dict(codes=None),
    dict(codes=FAKE + 8), dict(scales=None), dict(scales=FAKE + 2), dict(num=-1), dict(num=5),
    dict(type=BF16, src=FAKE + 4), dict(ids=FAKE, num=2 ** 31)])
def test_quantize_refusals(L, change):
    assert call(L.embbag_mx4_quantize, Q_NAMES, Q, **change) == BAD


D_NAMES = "codes scales rows dim dst type stride stream".split()
D = dict(codes=FAKE, scales=FAKE, rows=10, dim=64, dst=FAKE, type=F32, stride=64, stream=None)


@pytest.mark.parametrize("change", [
    dict(codes=None), dict(codes=FAKE + 4), dict(scales=FAKE + 1), dict(rows=-1), dict(dim=2),
    dict(dst=None), dict(dst=FAKE + 4), dict(type=7), dict(stride=63), dict(stride=0)])
def test_dequantize_refusals(L, change):
    assert call(L.embbag_mx4_dequantize, D_NAMES, D, **change) == BAD


def mx4_tables(rows=(10, 10), dim=32, codes=None, scales=None):
    n = max(len(rows), 1)
    r = (C.c_int64 * n)(*rows)
    c = (C.c_void_p * n)(*(codes or [FAKE + 4096 * i for i in range(len(rows))]))
    s = (C.c_void_p * n)(*(scales or [FAKE + 4096 * i for i in range(len(rows))]))
    pp = C.POINTER(C.c_void_p)
    return head._Mx4Tables(len(rows), dim, C.cast(r, C.POINTER(C.c_int64)), C.cast(c, pp), C.cast(s, pp)), (r, c, s)


F_NAMES = "tables batch indices offsets num weights pooling out type status stream".split()


@pytest.mark.parametrize("tables,change,code", [
    (dict(rows=()), {}, BAD), (dict(rows=(1,) * 65), {}, BAD), (dict(dim=6), {}, BAD),
    (dict(dim=1028), {}, BAD), (dict(rows=(0, 1)), {}, BAD), (dict(rows=(2 ** 30, 2 ** 30)), {}, BAD),
    (dict(codes=[FAKE, FAKE + 8]), {}, BAD), (dict(scales=[FAKE, 0]), {}, BAD),
    ({}, dict(batch=-1), BAD), ({}, dict(num=-1), BAD), ({}, dict(num=2 ** 31), BAD),
    ({}, dict(batch=2 ** 30), BAD), ({}, dict(indices=None), BAD), ({}, dict(offsets=None), BAD),
    ({}, dict(out=None), BAD), ({}, dict(out=FAKE + 8), BAD), ({}, dict(type=2), BAD),
    ({}, dict(pooling=2), BAD), ({}, dict(weights=FAKE, pooling=pk.EMBBAG_POOL_MEAN), BAD),
    ({}, dict(batch=0), OFF)])
def test_forward_refusals(L, tables, change, code):
    t, keep = mx4_tables(**tables)
    good = dict(tables=C.byref(t), batch=4, indices=FAKE, offsets=FAKE, num=9, weights=None,
                pooling=pk.EMBBAG_POOL_SUM, out=FAKE, type=F32, status=None, stream=None)
    assert call(L.embbag_mx4_forward, F_NAMES, good, **change) == code


def test_forward_needs_tables(L):
    assert L.embbag_mx4_forward(None, 1, FAKE, FAKE, 1, None, 0, FAKE, 0, None, None) == BAD
    t, keep = mx4_tables()
    t.codes = None
    assert L.embbag_mx4_forward(C.byref(t), 1, FAKE, FAKE, 1, None, 0, FAKE, 0, None, None) == BAD


M_NAMES = "x type stride m codes scales n k out otype ostride ws bytes stream".split()


@pytest.mark.parametrize("change,code", [
    (dict(x=None), BAD), (dict(x=FAKE + 4), BAD), (dict(type=3), BAD), (dict(stride=252), BAD),
    (dict(stride=258), BAD), (dict(m=-1), BAD), (dict(m=2 ** 23), BAD), (dict(codes=FAKE + 8), BAD),
    (dict(scales=None), BAD), (dict(n=0), BAD), (dict(n=2 ** 31), BAD), (dict(k=250), BAD),
    (dict(k=16388), BAD), (dict(out=None), BAD), (dict(out=FAKE + 2), BAD), (dict(ostride=999), BAD),
    (dict(m=2 ** 22, n=2 ** 20, ostride=2 ** 20), BAD), (dict(ws=None), WS), (dict(ws=FAKE + 64), WS),
    (dict(bytes=0), WS)])
def test_scores_refusals(L, change, code):
    good = dict(x=FAKE, type=F32, stride=256, m=100, codes=FAKE, scales=FAKE, n=1000, k=256, out=FAKE, otype=F32,
                ostride=1000, ws=FAKE, bytes=1 << 30, stream=None)
    assert call(L.embbag_mx4_matmul, M_NAMES, good, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(x=None), BAD), (dict(x=FAKE + 2), BAD), (dict(type=3), BAD), (dict(stride=999), BAD),
    (dict(m=-1), BAD), (dict(m=2 ** 23), BAD), (dict(codes=None), BAD), (dict(n=0), BAD), (dict(k=0), BAD),
    (dict(out=None), BAD), (dict(out=FAKE + 8), BAD), (dict(ostride=255), BAD), (dict(ostride=258), BAD),
    (dict(otype=9), BAD), (dict(ws=None), WS), (dict(ws=FAKE + 64), WS), (dict(bytes=0), WS)])
def test_gradient_refusals(L, change, code):
    good = dict(x=FAKE, type=F32, stride=1000, m=100, codes=FAKE, scales=FAKE, n=1000, k=256, out=FAKE, otype=F32,
                ostride=256, ws=FAKE, bytes=1 << 30, stream=None)
    assert call(L.embbag_mx4_matmul_grad, M_NAMES, good, **change) == code


def test_workspaces():
    assert pk.embbag_mx4_matmul_workspace_bytes(1, 1000, 256) == 0  # few elements: none
    assert pk.embbag_mx4_matmul_workspace_bytes(4096, 65536, 4096) > 4096 * 2048
    for f in (pk.embbag_mx4_matmul_workspace_bytes, pk.embbag_mx4_matmul_grad_workspace_bytes):
        for m, n, k in [(-1, 10, 64), (2 ** 23, 10, 64), (10, 0, 64), (10, 2 ** 31, 64), (10, 10, 66),
                        (10, 10, 16388), (2 ** 22, 2 ** 20, 64)]:
            assert f(m, n, k) == 0
        for m, n, k in [(0, 10, 64), (1, 1, 4), (300, 2 ** 31 - 1, 4), (2 ** 23 - 1, 7, 16384)]:
            assert f(m, n, k) % 256 == 0
    assert pk.embbag_distill_workspace_bytes(1, 200003, 8) > 0
    for r, v, t in [(-1, 10, 1), (1, 0, 1), (1, 10, 0), (1, 10, 1025), (2 ** 21, 2 ** 20, 1)]:
        assert pk.embbag_distill_workspace_bytes(r, v, t) == 0


def logits_args(**change):
    good = dict(rows=2, vocab=100, type=F32, logits=FAKE, logits_stride=100, out=FAKE + 4096, out_stride=100,
                seen=FAKE, seen_offsets=FAKE, num_seen=5, repetition=FAKE, bias_ids=FAKE, bias_offsets=FAKE,
                biases=FAKE, num_biases=3, masks=FAKE, mask_stride=4, num_masks=2)
    good.update(change)
    a = head._Logits()
    for k, v in good.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), BAD), (dict(vocab=0), BAD), (dict(type=2), BAD), (dict(logits=None), BAD),
    (dict(logits=FAKE + 2), BAD), (dict(logits_stride=99), BAD), (dict(out=None), BAD), (dict(out_stride=50), BAD),
    (dict(out=FAKE, out_stride=101), BAD), (dict(rows=2 ** 30, vocab=2 ** 20, logits_stride=2 ** 20,
                                                 out_stride=2 ** 20), BAD),
    (dict(seen=None), BAD), (dict(num_seen=-1), BAD), (dict(num_seen=2 ** 30), BAD),
    (dict(seen_offsets=None), BAD), (dict(seen_offsets=None, seen=None, num_seen=0), BAD),
    (dict(bias_ids=None), BAD), (dict(biases=None), BAD), (dict(bias_offsets=None), BAD),
    (dict(num_biases=2 ** 30), BAD), (dict(num_masks=0), BAD), (dict(num_masks=1), BAD),
    (dict(mask_stride=3), BAD), (dict(masks=FAKE + 2), BAD), (dict(masks=None, mask_ids=FAKE), BAD),
    (dict(rows=0), OFF)])
def test_logits_refusals(L, change, code):
    assert L.embbag_logits_process(C.byref(logits_args(**change)), None, None) == code


def test_logits_need_arguments(L):
    assert L.embbag_logits_process(None, None, None) == BAD
    assert L.embbag_distill(None, None, 0, None, None) == BAD


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), BAD), (dict(vocab=0), BAD), (dict(type=5), BAD), (dict(teacher_type=5), BAD),
    (dict(top=0), BAD), (dict(top=1025), BAD), (dict(temperature=0.0), BAD), (dict(temperature=-1.0), BAD),
    (dict(temperature=float("nan")), BAD), (dict(temperature=1e7), BAD), (dict(temperature=1e-7), BAD),
    (dict(logits=None), BAD), (dict(logits=FAKE + 1), BAD), (dict(logits_stride=99), BAD), (dict(ids=None), BAD),
    (dict(teacher=None), BAD), (dict(loss=None), BAD), (dict(grad=FAKE + 2), BAD), (dict(grad_stride=10), BAD),
    (dict(grad=FAKE, grad_stride=101), BAD),
    (dict(rows=2 ** 30, vocab=2 ** 20, logits_stride=2 ** 20, grad_stride=2 ** 20), BAD)])
def test_distill_refusals(L, change, code):
    a = head._Distill()
    good = dict(rows=2, vocab=100, type=F32, logits=FAKE, logits_stride=100, top=4, ids=FAKE, teacher_type=F32,
                teacher=FAKE, temperature=1.0, loss=FAKE, grad=FAKE + 4096, grad_stride=100)
    good.update(change)
    for k, v in good.items():
        setattr(a, k, v)
    assert L.embbag_distill(C.byref(a), FAKE, 1 << 30, None, None) == code


def test_distill_workspace_refusals(L):
    a = head._Distill()
    for k, v in dict(rows=1, vocab=200003, type=F32, logits=FAKE, logits_stride=200003, top=4, ids=FAKE, teacher=FAKE,
                     temperature=1.0, loss=FAKE).items():
        setattr(a, k, v)
    need = pk.embbag_distill_workspace_bytes(1, 200003, 4)
    assert L.embbag_distill(C.byref(a), FAKE, need - 1, None, None) == WS
    assert L.embbag_distill(C.byref(a), FAKE + 16, need, None, None) == WS
    assert L.embbag_distill(C.byref(a), None, need, None, None) == WS


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    with pytest.raises(TypeError):
        pk.Mx4Table(torch.zeros(3, 16, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.uint8), 32)
    with pytest.raises(ValueError):
        pk.Mx4Table(torch.zeros(3, 15, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.uint8), 32)
    with pytest.raises(ValueError):
        pk.Mx4Table(torch.zeros(3, 16, dtype=torch.uint8), torch.zeros(3, 3, dtype=torch.uint8), 32)
    x = torch.zeros(2, 5)
    with pytest.raises(TypeError):
        pk.embbag_logits_process(x, x)
    with pytest.raises(TypeError):
        pk.embbag_logits_process(x.double(), x)
    with pytest.raises((TypeError, ValueError)):
        pk.embbag_distill(x, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), 1.0, torch.zeros(2), None)
    assert pk.mx4_code_bytes(33) == 32 and pk.mx4_scale_bytes(129) == 8 and pk.mx4_scale_bytes(4) == 4
