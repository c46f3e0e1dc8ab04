"""Refusals of the norm, of 8-bit rows and of the cross entropy, on the host: every call here fails
an argument check and returns before any HIP call (dummy pointers, no GPU)."""
import os
from types import SimpleNamespace

import pytest
import torch

import paper_2005_04680_amd as pk
from paper_2005_04680_amd import head

FAKE = 1 << 20  # a 256-byte aligned non-null address; never dereferenced on these paths
F32, BF16 = pk.EMBBAG_F32, pk.EMBBAG_BF16
BAD, WS = pk.EMBBAG_ERR_INVALID_ARG, pk.EMBBAG_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pk.LIB_PATH):
        import paper_2005_04680_amd.build as b
        b.build()
    return head._lib()


def packed(cls, good, change):
    a = cls()
    for k, v in dict(good, **change).items():
        setattr(a, k, v)
    import ctypes as C
    return C.byref(a)


NORM = dict(rows=4, dim=64, eps=1e-6, x_type=F32, x=FAKE, x_stride=64, residual_type=F32, residual=FAKE + 4096,
            residual_stride=64, sum_out=FAKE + 8192, sum_stride=64, weight_type=F32, weight=FAKE, out_type=F32,
            out=FAKE + 12288, out_stride=64)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(rows=2 ** 31), dict(dim=0), dict(dim=6), dict(dim=16388), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(x_type=2), dict(residual_type=-1), dict(weight_type=2),
    dict(out_type=2), dict(x=None), dict(x=FAKE + 4), dict(x_stride=63), dict(x_stride=66), dict(residual=FAKE + 8),
    dict(residual_stride=60), dict(sum_out=FAKE + 4), dict(sum_stride=0), dict(out=FAKE + 4), dict(out_stride=62),
    dict(weight=FAKE + 8), dict(codes=FAKE), dict(scales=FAKE), dict(codes=FAKE + 8, scales=FAKE),
    dict(codes=FAKE, scales=FAKE + 2), dict(sum_out=None, out=None), dict(sum_out=FAKE + 4096, sum_stride=68),
    dict(out=FAKE, out_stride=68), dict(out=FAKE, out_type=BF16), dict(out=FAKE + 4096, out_type=BF16),
    dict(sum_out=FAKE, residual_type=BF16), dict(out=FAKE + 8192)])
def test_norm_refusals(L, change):
    assert L.embbag_rmsnorm(packed(head._RmsNorm, NORM, change), None) == BAD


def test_norm_of_no_rows_and_without_arguments(L):
    assert L.embbag_rmsnorm(packed(head._RmsNorm, NORM, dict(rows=0, x=None)), None) == pk.EMBBAG_OK
    assert L.embbag_rmsnorm(None, None) == BAD
    assert L.embbag_rmsnorm_grad(None, FAKE, 1 << 30, None) == BAD


GRAD = dict(rows=4, dim=64, eps=1e-6, dy_type=F32, dy=FAKE, dy_stride=64, h_type=F32, h=FAKE + 4096, h_stride=64,
            weight_type=F32, weight=FAKE, dsum=FAKE + 8192, dsum_stride=64, dh=FAKE + 12288, dh_stride=64,
            dweight=FAKE)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(rows=2 ** 31), dict(dim=2), dict(dim=16388), dict(eps=0.0), dict(eps=float("inf")),
    dict(dy_type=2), dict(h_type=3), dict(weight_type=-1), dict(dy=None), dict(dy=FAKE + 4), dict(dy_stride=65),
    dict(h=None), dict(h_stride=32), dict(dh=None), dict(dh=FAKE + 8), dict(dh_stride=66), dict(dsum=FAKE + 4),
    dict(dsum_stride=0), dict(weight=FAKE + 4), dict(dweight=FAKE + 4), dict(dh=FAKE, dh_stride=68),
    dict(dh=FAKE, dy_type=BF16), dict(dh=FAKE + 4096, dh_stride=68), dict(dh=FAKE + 8192, dh_stride=68)])
def test_norm_gradient_refusals(L, change):
    assert L.embbag_rmsnorm_grad(packed(head._RmsNormGrad, GRAD, change), FAKE, 1 << 30, None) == BAD


def test_norm_gradient_workspace(L):
    need = pk.embbag_rmsnorm_grad_workspace_bytes(4, 64)
    assert need > 0 and need % 256 == 0
    a = packed(head._RmsNormGrad, GRAD, {})
    assert L.embbag_rmsnorm_grad(a, FAKE, need - 1, None) == WS
    assert L.embbag_rmsnorm_grad(a, FAKE + 16, need, None) == WS
    assert L.embbag_rmsnorm_grad(a, None, need, None) == WS
    for rows, dim in [(-1, 64), (2 ** 31, 64), (4, 66), (4, 16388), (4, 0), (4, 2 ** 32 + 64)]:
        assert pk.embbag_rmsnorm_grad_workspace_bytes(rows, dim) == 0


@pytest.mark.parametrize("args", [
    (None, FAKE, 4, 64, FAKE, F32, 64), (FAKE + 8, FAKE, 4, 64, FAKE, F32, 64), (FAKE, None, 4, 64, FAKE, F32, 64),
    (FAKE, FAKE + 2, 4, 64, FAKE, F32, 64), (FAKE, FAKE, -1, 64, FAKE, F32, 64), (FAKE, FAKE, 4, 66, FAKE, F32, 68),
    (FAKE, FAKE, 4, 64, None, F32, 64), (FAKE, FAKE, 4, 64, FAKE, 2, 64), (FAKE, FAKE, 4, 64, FAKE, F32, 60),
    (FAKE, FAKE, 4, 64, FAKE + 4, BF16, 64), (FAKE, FAKE, 2 ** 31, 64, FAKE, F32, 64)])
def test_reading_eight_bit_rows_refusals(L, args):
    assert L.embbag_mx8_dequantize(*args, None) == BAD


def fake(*shape, dtype=torch.float32):
    return SimpleNamespace(is_cuda=True, dtype=dtype, shape=shape, stride=lambda: (shape[-1], 1),
                           data_ptr=lambda: FAKE, is_contiguous=lambda: True,
                           numel=lambda: int(torch.Size(shape).numel()))


def test_binding_refuses_wrong_shapes_and_types():
    x, b = fake(4, 64), fake(4, 64, dtype=torch.bfloat16)
    rows8 = SimpleNamespace(rows=4, dim=64, codes_ptr=FAKE, scales_ptr=FAKE)
    with pytest.raises(TypeError):
        pk.embbag_rmsnorm(torch.zeros(4, 64), None, 1e-6, out=x, stream=0)
    with pytest.raises(TypeError):
        pk.embbag_rmsnorm(x, None, 1e-6, residual=x, sum_out=b, stream=0)
    with pytest.raises(TypeError):
        pk.embbag_rmsnorm(x, fake(64, dtype=torch.float16), 1e-6, out=x, stream=0)
    for bad in (dict(out=fake(3, 64)), dict(out=fake(4, 60)), dict(residual=fake(5, 64), out=x),
                dict(sum_out=fake(4, 68)), dict(mx8=SimpleNamespace(rows=3, dim=64)),
                dict(mx8=SimpleNamespace(rows=4, dim=68))):
        with pytest.raises(ValueError):
            pk.embbag_rmsnorm(x, None, 1e-6, stream=0, **bad)
    with pytest.raises(ValueError):
        pk.embbag_rmsnorm(x, fake(60), 1e-6, out=x, stream=0)
    with pytest.raises(ValueError):
        pk.embbag_mx8_dequantize(rows8, fake(4, 60), stream=0)
    with pytest.raises(TypeError):
        pk.embbag_rmsnorm_grad(x, x, None, 1e-6, b, None, stream=0)
    with pytest.raises(TypeError):
        pk.embbag_rmsnorm_grad(x, x, fake(64), 1e-6, x, None, dweight=fake(64, dtype=torch.bfloat16), stream=0)
    with pytest.raises(ValueError):
        pk.embbag_rmsnorm_grad(fake(3, 64), x, None, 1e-6, x, None, stream=0)
    with pytest.raises(ValueError):
        pk.Mx8Rows(fake(4, 64, dtype=torch.uint8), fake(4, 4, dtype=torch.uint8), 64)
    with pytest.raises(TypeError):
        pk.Mx8Rows(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 64)


M_NAMES = "x xs m codes scales n k out otype ostride ws bytes stream".split()


@pytest.mark.parametrize("change,code", [
    (dict(x=None), BAD), (dict(x=FAKE + 8), BAD), (dict(xs=None), BAD), (dict(xs=FAKE + 2), BAD), (dict(m=-1), BAD),
    (dict(m=2 ** 23), BAD), (dict(codes=FAKE + 8), BAD), (dict(scales=None), BAD), (dict(n=0), BAD),
    (dict(n=2 ** 31), BAD), (dict(k=250), BAD), (dict(k=16388), BAD), (dict(out=None), BAD), (dict(out=FAKE + 2), BAD),
    (dict(ostride=999), BAD), (dict(otype=2), BAD), (dict(m=2 ** 22, n=2 ** 20, ostride=2 ** 20), BAD),
    (dict(ws=None), WS), (dict(ws=FAKE + 64), WS), (dict(bytes=0), WS)])
def test_scores_from_eight_bits_refusals(L, change, code):
    good = dict(x=FAKE, xs=FAKE, m=100, codes=FAKE, scales=FAKE, n=1000, k=256, out=FAKE, otype=F32, ostride=1000,
                ws=FAKE, bytes=1 << 30, stream=None)
    args = dict(good, **change)
    assert L.embbag_mx4_matmul_x8(*[args[n] for n in M_NAMES]) == code


def test_scores_from_eight_bits_sizes():
    f = pk.embbag_mx4_matmul_x8_workspace_bytes
    assert f(16, 1000, 256) == 0 and f(17, 1000, 256) > 0
    for m, n, k in [(-1, 10, 64), (2 ** 23, 10, 64), (10, 0, 64), (10, 2 ** 31, 64), (10, 10, 66), (10, 10, 16388),
                    (2 ** 32 + 17, 10, 64), (17, 10, 2 ** 32 + 64)]:
        assert f(m, n, k) == 0
    x = SimpleNamespace(rows=4, dim=64, codes_ptr=FAKE, scales_ptr=FAKE)
    t = SimpleNamespace(rows=10, dim=68, codes_ptr=FAKE, scales_ptr=FAKE)
    with pytest.raises(ValueError):
        pk.embbag_mx4_matmul_x8(x, t, fake(4, 10), None, stream=0)
    t.dim = 64
    for shape in [(3, 10), (4, 11)]:
        with pytest.raises(ValueError):
            pk.embbag_mx4_matmul_x8(x, t, fake(*shape), None, stream=0)


XENT = dict(rows=4, dim=64, vocab=1000, x_type=F32, x=FAKE, x_stride=64, table_type=F32, table=FAKE, table_stride=64,
            labels=FAKE, scale=1.0, loss=FAKE, grad_x=FAKE + 4096, grad_x_stride=64, grad_table=FAKE + 8192,
            grad_table_stride=64)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(rows=2 ** 20 + 1), dict(vocab=0), dict(vocab=2 ** 31), dict(rows=2 ** 20, vocab=2 ** 20 + 1),
    dict(dim=0), dict(dim=6), dict(dim=16388), dict(x_type=2), dict(table_type=-1), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(scale=-float("inf")), dict(x=None), dict(x=FAKE + 4), dict(x_stride=62),
    dict(x_stride=66), dict(table=None), dict(table=FAKE + 8), dict(table_stride=60), dict(table_stride=2 ** 19 + 4),
    dict(labels=None), dict(loss=None), dict(grad_x=FAKE + 4), dict(grad_x_stride=60), dict(grad_table=FAKE + 8),
    dict(grad_table_stride=65), dict(x_type=BF16, x=FAKE + 4), dict(rows=0, table=None),
    dict(rows=0, grad_table=FAKE + 4), dict(grad_table=FAKE), dict(grad_x=FAKE, grad_x_stride=68)])
def test_xent_refusals(L, change):
    assert L.embbag_xent(packed(head._Xent, XENT, change), FAKE, 1 << 40, None, None) == BAD


def test_xent_workspace(L):
    need = pk.embbag_xent_workspace_bytes(4, 1000, 64, F32, True)
    assert need > pk.embbag_xent_workspace_bytes(4, 1000, 64, F32, False) > 0 and need % 256 == 0
    a = packed(head._Xent, XENT, {})
    assert L.embbag_xent(a, FAKE, need - 1, None, None) == WS
    assert L.embbag_xent(a, FAKE + 16, need, None, None) == WS
    assert L.embbag_xent(a, None, need, None, None) == WS
    assert L.embbag_xent(None, FAKE, need, None, None) == BAD
    for r, v, e, t in [(-1, 10, 64, F32), (2 ** 20 + 1, 10, 64, F32), (4, 0, 64, F32), (4, 2 ** 31, 64, F32),
                       (4, 10, 66, F32), (4, 10, 16388, F32), (4, 10, 64, 2), (2 ** 32 + 4, 10, 64, F32),
                       (4, 10, 2 ** 32 + 64, F32), (2 ** 20, 2 ** 20 + 1, 64, F32)]:
        assert pk.embbag_xent_workspace_bytes(r, v, e, t, True) == 0
    # A piece of the vocabulary at a time: of D 512 MB at most.
    assert pk.embbag_xent_workspace_bytes(4096, 2 ** 27, 256, BF16, True) < 2 ** 36
    for r, v, e in [(0, 1, 4), (1, 1, 4), (2 ** 20, 2 ** 20, 16384), (1, 2 ** 31 - 1, 16384)]:
        for t in (F32, BF16):
            assert pk.embbag_xent_workspace_bytes(r, v, e, t, True) > 0


def test_binding_refuses_wrong_labels_and_gradients():
    x, w = fake(4, 64), fake(10, 64)
    labels, loss = fake(4, dtype=torch.int32), fake(4)
    ok = dict(x=x, table=w, labels=labels, loss=loss, workspace=None, stream=0)
    for bad in (dict(labels=fake(3, dtype=torch.int32)), dict(loss=fake(5)), dict(table=fake(10, 60)),
                dict(grad_x=fake(3, 64)), dict(grad_table=fake(10, 60)), dict(row_weights=fake(3))):
        with pytest.raises(ValueError):
            pk.embbag_xent(**dict(ok, **bad))
    for bad in (dict(labels=fake(4, dtype=torch.int64)), dict(grad_x=fake(4, 64, dtype=torch.bfloat16)),
                dict(grad_table=fake(10, 64, dtype=torch.bfloat16)), dict(x=fake(4, 64, dtype=torch.float16))):
        with pytest.raises(TypeError):
            pk.embbag_xent(**dict(ok, **bad))
    assert pk.embbag_xent(**ok) == WS
