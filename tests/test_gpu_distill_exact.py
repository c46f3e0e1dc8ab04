"""The digits of distillation's loss and gradient: logits that share an offset, against the 64-bit
reference, and low temperatures, with bounds that follow from the distances to a row's largest
logit, not from the logits' own size."""
import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, rounding, status

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def run(x, ids, t, temperature, w=None, grad=True):
    """loss, gradient (or None) and status of one call."""
    rows, vocab = x.shape
    ws = torch.empty(pk.embbag_distill_workspace_bytes(rows, vocab, ids.shape[1]), dtype=torch.uint8,
                     device=DEV)
    ws.fill_(0xFF)
    loss, st = torch.full((rows,), float("nan"), device=DEV), status()
    g = torch.full((rows, vocab), float("nan"), dtype=x.dtype, device=DEV) if grad else None
    pk.check(pk.embbag_distill(x.to(DEV), torch.from_numpy(ids).to(DEV), t.to(DEV), temperature, loss, ws,
                               grad=g, row_weights=None if w is None else torch.from_numpy(w).to(DEV),
                               d_status=st))
    return loss, g, pk.embbag_status_read(st)


def bounds(x, ids, t, temperature, type_):
    """The reference's loss and gradient, and how far off FP32 may be.

    With U half a unit of FP32: a student's exponential is off by its exponent's relative error (the distance
    to the largest, the constant, their product: 4 roundings, on a number of at most `reach`) and a few units;
    sums of n positive terms in trees over at least 64 lanes by n / 64 + a few; the teacher's likewise with
    `span`.  The loss adds terms p log p, p (z - max) and log of the sum: each off by its probabilities', its own
    few units and, for the last, the sum's relative error."""
    x, t, T = x.double().numpy(), t.double().numpy(), float(temperature)
    loss, grad, q, _ = ref.distill(x, ids, t, T)
    rows, vocab = x.shape
    ltol, gtol = np.zeros(rows), np.zeros((rows, vocab))
    for r in range(rows):
        k = ids[r] >= 0
        z, s = (x[r] - x[r].max()) / T, (t[r, k] - t[r, k].max()) / T
        reach, span = -z.min(), -s.min()
        rel = U * (8 * reach + vocab / 64 + 100)
        pr = U * (8 * span + ids.shape[1] + 100)
        p = np.exp(s) / np.exp(s).sum()
        logp, lse = s - np.log(np.exp(s).sum()), np.log(np.exp(z).sum())
        ltol[r] = T * T * ((pr + 100 * U) * (p @ (np.abs(logp) + np.abs(z[ids[r, k]])) + abs(lse)) + rel)
        gtol[r] = T * (rel * q[r] + pr * np.abs(q[r] - grad[r] / T))
    gtol = gtol + np.where(grad == 0, 0, rounding(np.abs(grad) + gtol, type_))
    return loss, grad, ltol + 1e-38, gtol + 1e-38


@pytest.mark.parametrize("offset", [0.0, 1024.0, -8192.0, 65536.0])
@pytest.mark.parametrize("rows,vocab,top,type_", [
    (3, 1001, 20, "f32"), (300, 517, 16, "f32"), (2, 40003, 20, "f32"), (5, 33001, 300, "f32"),
    (1, 80001, 12, "bf16"), (200, 2049, 20, "bf16")])
@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_an_offset_of_the_logits_changes_no_digit(rows, vocab, top, type_, temperature, offset):
    rng = np.random.default_rng(rows + vocab)
    # (FP32: multiples of 2^-7, which all offsets leave exact; BF16 is taken as it rounds.)
    x = np.round(rng.normal(size=(rows, vocab)) * 3 * 128) / 128 + offset
    x = torch.from_numpy(x).to(DT[type_])
    ids = np.stack([rng.choice(vocab, size=top, replace=False) for _ in range(rows)]).astype(np.int32)
    t = torch.from_numpy((rng.normal(size=(rows, top)) * 2).astype(np.float32))
    want, wgrad, ltol, gtol = bounds(x, ids, t, temperature, type_)
    loss, grad, st = run(x, ids, t, temperature)
    assert st == 0
    close(loss, want, ltol, "loss")
    close(grad, wgrad, gtol, "gradient")
    alone, _, _ = run(x, ids, t, temperature, grad=False)
    assert torch.equal(alone, loss)


@pytest.mark.parametrize("rows,vocab", [(2, 40003), (3, 5000)])
def test_slices_far_apart(rows, vocab):
    """Parts of a row near the type's lowest value, left out by -inf, or a large offset below the rest: the
    loss is the reference's where the teacher has its entries above them, and infinite where it has some left
    at -inf."""
    rng = np.random.default_rng(vocab)
    x = rng.normal(size=(rows, vocab)) + 500
    x[0, : vocab // 3] = float(torch.finfo(torch.float32).min)
    x[0, vocab // 3: vocab // 2] = -np.inf
    x[1, : vocab // 2] -= 1000
    x = torch.from_numpy(x.astype(np.float32))
    ids = np.stack([rng.choice(np.arange(vocab // 2, vocab), size=9, replace=False) for _ in range(rows)])
    ids = ids.astype(np.int32)
    ids[1, 4:] -= vocab // 2
    t = torch.from_numpy(rng.normal(size=(rows, 9)).astype(np.float32))
    want = ref.distill(x.double().numpy(), ids, t.double().numpy(), 1.0)[0]
    loss, grad, _ = run(x, ids, t, 1.0)
    # (p log p, p (z - max) up to 1000, log of the sum: units of 1000 at most, 300 of them.)
    close(loss, want, 300 * U * np.array([20.0] + [1000.0] * (rows - 1)), "loss")
    assert torch.isfinite(grad).all()
    ids[0, 0] = vocab // 2 - 1
    loss, grad, _ = run(x, ids, t, 1.0)
    assert loss[0] == float("inf") and torch.isfinite(loss[1:]).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("rows,vocab", [(4, 900), (200, 333), (2, 33001)])
@pytest.mark.parametrize("temperature", [1e-2, 1e-4, 1e-6, 1e4])
@pytest.mark.parametrize("offset", [20.0, -3.0])
def test_low_temperatures(rows, vocab, temperature, offset):
    """Logits a few temperatures apart around an offset (as FP32 has them)."""
    rng = np.random.default_rng(vocab)
    spread = temperature * 2
    x = torch.from_numpy((rng.normal(size=(rows, vocab)) * spread + offset).astype(np.float32))
    t = torch.from_numpy((rng.normal(size=(rows, 20)) * spread + offset).astype(np.float32))
    ids = np.stack([rng.choice(vocab, size=20, replace=False) for _ in range(rows)]).astype(np.int32)
    ids[1, 3:9] = -1
    want, wgrad, ltol, gtol = bounds(x, ids, t, temperature, "f32")
    loss, grad, _ = run(x, ids, t, temperature)
    close(loss, want, ltol, "loss")
    close(grad, wgrad, gtol, "gradient")


@pytest.mark.parametrize("rows,vocab", [(2, 900), (2, 33001)])
def test_a_teacher_that_the_temperature_would_overflow(rows, vocab):
    rng = np.random.default_rng(1)
    T = 1e-6
    x = torch.from_numpy((rng.normal(size=(rows, vocab)) * T).astype(np.float32))
    t = torch.tensor([[1e33, 1e33, -1e33, -np.inf], [3e38, -3e38, 3e38, 0.0]])
    ids = np.array([[5, 7, 1, 2], [10, 3, vocab - 1, 0]], np.int32)
    loss, grad, _ = run(x, ids, t, T)
    p = np.array([[0.5, 0.5, 0.0, 0.0], [0.5, 0.0, 0.5, 0.0]])
    z = x.double().numpy() / T
    q = np.exp(z - z.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)
    want, wgrad = np.zeros(rows), T * q
    for r in range(rows):
        want[r] = T * T * sum(a * (np.log(a) - np.log(q[r, v])) for a, v in zip(p[r], ids[r]) if a)
        wgrad[r, ids[r]] -= T * p[r]
    # (Exponents up to 10, a sum of vocab terms, and T itself as FP32 has it.)
    rel = U * (8 * 10 + vocab / 64 + 200)
    close(loss, want, rel * T * T * 20, "loss")
    close(grad, wgrad, rel * (T * q + np.abs(wgrad)), "gradient")


@pytest.mark.parametrize("rows,vocab,top", [(2, 50, 3), (2, 5000, 300), (2, 40003, 3), (300, 50, 3), (130, 9000, 1024)])
@pytest.mark.parametrize("left_out", ["weight", "teacher", "logits", "no"])
def test_a_bad_id_is_reported_whatever_its_row(rows, vocab, top, left_out):
    """Also in a row that is left out, and however many rows there are."""
    x = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(1))
    ids = np.tile(np.arange(top, dtype=np.int32) % vocab, (rows, 1))
    t, w = torch.zeros(rows, top), np.ones(rows, np.float32)
    if left_out == "weight":
        w[1] = 0
    elif left_out == "teacher":
        t[1] = float("-inf")
    elif left_out == "logits":
        x[1] = float("-inf")
    for grad in (True, False):
        assert run(x, ids, t, 1.0, w, grad)[2] == 0
        for at in (0, top - 1):
            bad = ids.copy()
            bad[1, at] = vocab
            assert run(x, bad, t, 1.0, w, grad)[2] == pk.EMBBAG_ERR_INDEX_RANGE
