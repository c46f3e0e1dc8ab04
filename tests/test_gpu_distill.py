"""Distillation on the GPU against the 64-bit reference and against differences."""
import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, padded, rounding, status

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def case(rows, vocab, top, type_, seed, repeats=False, spread=3.0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(size=(rows, vocab)) * spread).to(DT[type_])
    ids = np.stack([rng.choice(vocab, size=top, replace=repeats or top > vocab) for _ in range(rows)])
    ids = ids.astype(np.int32)
    ids[rng.random(ids.shape) < 0.1] = -1
    t = (rng.normal(size=(rows, top)) * 2).astype(np.float32)
    w = rng.random(rows).astype(np.float32)
    if rows > 2:
        ids[1] = -1
        w[2] = 0.0
    if rows > 4:
        t[3] = -np.inf
        x[4] = float("-inf")
    return x, ids, t, w


def check(x, ids, t, temperature, w, type_, xs=None, grad=None, loss_only=False):
    rows, vocab = x.shape
    xs = x.to(DEV) if xs is None else xs
    if grad is None and not loss_only:
        grad = torch.full((rows, vocab), float("nan"), dtype=DT[type_], device=DEV)
    loss = torch.full((rows,), float("nan"), device=DEV)
    td = torch.from_numpy(t) if isinstance(t, np.ndarray) else t
    th = td.double().numpy()
    want, wgrad, q, mag = ref.distill(x.double().numpy(), ids, th, temperature, w)
    ws = torch.empty(pk.embbag_distill_workspace_bytes(rows, vocab, ids.shape[1]), dtype=torch.uint8,
                     device=DEV)
    ws.fill_(0xFF)
    st = status()
    pk.check(pk.embbag_distill(xs, torch.from_numpy(ids).to(DEV), td.to(DEV), temperature, loss, ws,
                               grad=grad, d_status=st,
                               row_weights=None if w is None else torch.from_numpy(w).to(DEV)))
    pk.check(pk.embbag_status_read(st))
    # Exponents: the logit's distance to the largest, its product with log2(e)/T (each rounded)
    # and the exponential itself, a few units; the sum of vocab positive terms, in trees over
    # at least 64 lanes.
    with np.errstate(invalid="ignore", divide="ignore"):
        z = np.where(np.isfinite(x.double().numpy()), x.double().numpy(), 0) / temperature
        reach = (z.max(1) - z.min(1))[:, None]
        rel = U * (8 * reach + vocab / 64 + 100)
        pr = U * (8 * np.where(np.isfinite(th), np.abs(th), 0).max(1, keepdims=True) * 2 / temperature +
                  ids.shape[1] + 100)
        wt = np.abs(np.ones(rows) if w is None else w)[:, None] * temperature
        tol = wt * (rel * q + pr * np.abs(q - wgrad / np.where(wt == 0, 1, wt)))
    if grad is not None:
        close(grad, wgrad, tol + np.where(wgrad == 0, 0, rounding(np.abs(wgrad) + tol, type_)), "grad")
    ltol = mag * (pr[:, 0] + U * 100) + wt[:, 0] * temperature * rel[:, 0] * (want != 0)
    close(loss, want, ltol + U * np.where(np.isfinite(want), np.abs(want), 0), "loss")


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,top", [
    (1, 1, 1), (2, 3, 3), (6, 50, 7), (5, 255, 1), (3, 1001, 20), (7, 4096, 64), (2, 8191, 300),
    (2, 8193, 64), (1, 40003, 1024), (6, 20000, 50), (40, 517, 10), (300, 2049, 16)])
@pytest.mark.parametrize("temperature", [1.0, 2.0, 0.3])
def test_distill(rows, vocab, top, temperature, type_):
    x, ids, t, w = case(rows, vocab, top, type_, rows + vocab + top)
    check(x, ids, t, temperature, w, type_)


@pytest.mark.parametrize("rows,vocab", [(3, 777), (2, 30001), (300, 1000)])
def test_loss_alone_is_the_same(rows, vocab):
    x, ids, t, w = case(rows, vocab, 30, "bf16", 5)
    check(x, ids, t, 1.0, w, "bf16", loss_only=True)
    check(x, ids, t, 1.0, None, "bf16")


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,top", [(4, 5, 40), (2, 3000, 500), (1, 20000, 1024), (300, 64, 100)])
def test_repeated_ids_add_up(rows, vocab, top, type_):
    x, ids, t, w = case(rows, vocab, top, type_, 11, repeats=True)
    ids[:, : top // 2] = ids[:, :1]
    check(x, ids, t, 1.0, w, type_)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (8, 2), (0, 3)])
@pytest.mark.parametrize("rows,vocab", [(3, 9001), (300, 1003)])
def test_rows_of_any_alignment_and_in_place(rows, vocab, pad, offset, type_):
    x, ids, t, w = case(rows, vocab, 17, type_, pad + offset)
    out = padded(torch.zeros_like(x), pad + 1, offset + 1)
    check(x, ids, t, 1.5, w, type_, padded(x, pad, offset), out)
    assert torch.isnan(out._base[offset + 1:].view(rows, vocab + pad + 1)[:, vocab:]).all()
    xs = padded(x, pad, offset)
    check(x, ids, t, 1.5, w, type_, xs, xs)


def test_a_bf16_teacher():
    x, ids, t, w = case(4, 600, 12, "f32", 3)
    check(x, ids, torch.from_numpy(t).to(torch.bfloat16), 1.0, w, "f32")


@pytest.mark.parametrize("rows,vocab", [(2, 20000), (300, 500)])
def test_masked_logits_and_far_apart_ones(rows, vocab):
    """-inf has probability 0 (and an infinite loss where the teacher has some left), the type's
    lowest value as well."""
    x, ids, t, w = case(rows, vocab, 9, "f32", 21, spread=30.0)
    x[0, ::2] = float("-inf")
    x[1, 1::2] = torch.finfo(torch.float32).min
    w[:] = 1.0
    want, grad, _, _ = ref.distill(x.double().numpy(), ids, t, 1.0, w)
    loss = torch.empty(rows, device=DEV)
    g = torch.empty(rows, vocab, device=DEV)
    ws = torch.empty(pk.embbag_distill_workspace_bytes(rows, vocab, 9), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_distill(x.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV), 1.0,
                               loss, ws, grad=g))
    got = loss.double().cpu().numpy()
    assert np.isinf(want[0]) and np.array_equal(np.isinf(got), np.isinf(want))
    fin = np.isfinite(want) & (np.abs(want) < 1e30)
    assert np.allclose(got[fin], want[fin], rtol=1e-4, atol=1e-4)
    assert np.allclose(g.double().cpu().numpy(), grad, rtol=1e-3, atol=1e-4)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows,vocab", [(3, 20000), (300, 500)])
def test_nan_and_infinity_stay_in_their_row(rows, vocab, bad):
    x, ids, t, w = case(rows, vocab, 9, "f32", 22)
    w[:] = 1.0
    clean = torch.empty(rows, vocab, device=DEV)
    out = []
    for y in (x, x.clone()):
        if out:
            y[0, vocab - 1] = bad
        loss, g = torch.empty(rows, device=DEV), torch.empty(rows, vocab, device=DEV)
        ws = torch.empty(pk.embbag_distill_workspace_bytes(rows, vocab, 9), dtype=torch.uint8, device=DEV)
        pk.check(pk.embbag_distill(y.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV),
                                   1.0, loss, ws, grad=g))
        out.append((loss.cpu(), g.cpu()))
    assert torch.isnan(out[1][0][0]) and torch.isnan(out[1][1][0]).all()
    assert torch.equal(out[0][0][1:], out[1][0][1:]) and torch.equal(out[0][1][1:], out[1][1][1:])


def test_a_nan_teacher_is_not_left_out():
    x, ids, t, w = case(3, 500, 4, "f32", 23)
    ids[0] = [1, 2, -1, -1]
    t[0] = np.nan
    w[:] = 1.0
    loss, g = torch.empty(3, device=DEV), torch.empty(3, 500, device=DEV)
    ws = torch.empty(pk.embbag_distill_workspace_bytes(3, 500, 4), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_distill(x.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV), 1.0,
                               loss, ws, grad=g))
    assert torch.isnan(loss[0]) and torch.isfinite(loss[1:]).all() and torch.isfinite(g[1:]).all()


def test_gradient_against_differences():
    x, ids, t, w = case(3, 40, 6, "f32", 31, spread=1.0)
    w[:] = [1.0, 0.5, 2.0]
    ids[:] = np.abs(ids)

    def loss_of(v):
        loss = torch.empty(3, device=DEV)
        ws = torch.empty(pk.embbag_distill_workspace_bytes(3, 40, 6), dtype=torch.uint8, device=DEV)
        pk.check(pk.embbag_distill(v.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV),
                                   1.5, loss, ws, row_weights=torch.from_numpy(w).to(DEV)))
        return loss.double().cpu()

    g = torch.empty(3, 40, device=DEV)
    loss = torch.empty(3, device=DEV)
    ws = torch.empty(pk.embbag_distill_workspace_bytes(3, 40, 6), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_distill(x.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV), 1.5, loss,
                               ws, grad=g, row_weights=torch.from_numpy(w).to(DEV)))
    h = 2.0 ** -5
    for v in range(40):
        a, b = x.clone(), x.clone()
        a[:, v] += h
        b[:, v] -= h
        step = (a[:, v] - b[:, v]).double()
        d = (loss_of(a) - loss_of(b)) / step
        # the third derivative of a log-sum-exp is at most 1 (in z): w T^2 (h/T)^3 / 6 / step; the losses'
        # own rounding, 100 units of values up to 20, over the step
        bound = torch.from_numpy(w).double() * (h ** 2 / 1.5 / 6 + 2.25 * 100 * U * 20 / (2 * h))
        assert ((d - g[:, v].double().cpu()).abs() <= bound).all()


def test_bad_ids_are_reported():
    x, ids, t, w = case(2, 100, 4, "f32", 41)
    ids[1, 2] = 100
    loss, g = torch.empty(2, device=DEV), torch.empty(2, 100, device=DEV)
    ws = torch.empty(pk.embbag_distill_workspace_bytes(2, 100, 4), dtype=torch.uint8, device=DEV)
    st = status()
    pk.check(pk.embbag_distill(x.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV), 1.0,
                               loss, ws, grad=g, d_status=st))
    assert pk.embbag_status_read(st) == pk.EMBBAG_ERR_INDEX_RANGE


def test_no_rows():
    x = torch.empty(0, 50, device=DEV)
    ws = torch.empty(max(256, pk.embbag_distill_workspace_bytes(0, 50, 4)), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_distill(x, torch.empty(0, 4, dtype=torch.int32, device=DEV), torch.empty(0, 4, device=DEV),
                               1.0, torch.empty(0, device=DEV), ws, grad=x))
