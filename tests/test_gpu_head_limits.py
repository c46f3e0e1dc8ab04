"""The output head at sizes that take more than one launch (2^32 threads and more): outputs over the whole range,
with inputs whose results are exact or known in closed form."""
import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, log, require_gpu
from test_gpu_mx4 import random_table, status

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def pieces(n, step=1 << 26):
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def grid_rows(rows, first, dim=4):
    """Rows `first`.. of values that 4-bit storage holds exactly (products of the grid with one power of two)."""
    at = torch.arange(first * dim, (first + rows) * dim, device=DEV).view(rows, dim)
    v = torch.tensor(GRID, device=DEV, dtype=torch.bfloat16)[(at * 7 + at // 64) % 15]
    return v * torch.exp2(((at[:, :1] // dim) % 9 - 4).to(torch.bfloat16))


def test_a_table_of_more_than_2_30_rows():
    """Quantised (all rows, and a few of them), read back, and scored by 1 and by 17 rows of x."""
    rows = (1 << 30) + 5
    src = torch.empty(rows, 4, dtype=torch.bfloat16, device=DEV)
    for p in pieces(rows):
        src[p] = grid_rows(p.stop - p.start, p.start)
    t = pk.Mx4Table(torch.full((rows, 16), 0xA5, dtype=torch.uint8, device=DEV),
                    torch.full((rows, 4), 0x5A, dtype=torch.uint8, device=DEV), 4)
    log("[limits] quantize")
    pk.check(pk.embbag_mx4_quantize(src, t))
    some = torch.tensor([0, 1, (1 << 29) - 1, 1 << 29, (1 << 29) + 1, (1 << 30) - 1, 1 << 30, rows - 1], device=DEV)
    codes, scales = ref.quantize(src[some].double().cpu().numpy())
    assert np.array_equal(t.codes[some].cpu().numpy(), codes)
    assert np.array_equal(t.scales[some].cpu().numpy(), scales)
    log("[limits] dequantize")
    back = torch.full((rows, 4), float("nan"), dtype=torch.bfloat16, device=DEV)
    pk.check(pk.embbag_mx4_dequantize(t, back))
    assert all(torch.equal(back[p], src[p]) for p in pieces(rows))
    del back

    log("[limits] scores of one row")
    x = torch.tensor([[1.0, 2.0, 0.0, -4.0]], device=DEV)
    out = torch.full((1, rows), float("nan"), device=DEV)
    pk.check(pk.embbag_mx4_matmul(x, t, out, torch.empty(256, dtype=torch.uint8, device=DEV)))

    def want(p, f):
        v = src[p].float() * f  # (exact, as is their sum)
        return v[:, 0] + 2 * v[:, 1] - 4 * v[:, 3]
    assert all(torch.equal(out[0, p], want(p, 1.0)) for p in pieces(rows))
    del out

    log("[limits] scores of 17 rows")
    f = torch.tensor([1.0, -2.0, 0.5] * 5 + [4.0, 1.0], device=DEV)
    out = torch.full((17, rows), float("nan"), dtype=torch.bfloat16, device=DEV)
    ws = torch.full((pk.embbag_mx4_matmul_workspace_bytes(17, rows, 4),), 0xFF, dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul(x * f[:, None], t, out, ws))
    for i in range(17):
        assert all(torch.equal(out[i, p], want(p, float(f[i])).bfloat16()) for p in pieces(rows)), i


def test_x_of_more_than_2_35_elements():
    m, k, n = (1 << 21) + 3, 16384, 40
    t, w = random_table(n, k, 1)
    x = torch.ones(m, k, dtype=torch.bfloat16, device=DEV)
    some = torch.tensor([0, 5, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, 1 << 21, m - 1], device=DEV)
    x[some] = torch.randn(len(some), k, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).bfloat16()
    out = torch.full((m, n), float("nan"), device=DEV)
    ws = torch.full((pk.embbag_mx4_matmul_workspace_bytes(m, n, k),), 0xFF, dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul(x, t, out, ws))
    q = ref.dequantize(*ref.quantize(x[some].double().cpu().numpy()), k)
    tol = 2 * (k + 8) * 2.0 ** -24 * (np.abs(q) @ np.abs(w).T)
    assert (np.abs(out[some].double().cpu().numpy() - q @ w.T) <= tol).all()
    other = torch.ones(m, dtype=torch.bool, device=DEV)
    other[some] = False
    ones = out[1]  # all other rows are the same row of ones (the sums' order is the same as well)
    assert (np.abs(ones.double().cpu().numpy() - w.sum(1)) <= 2 * (k + 8) * 2.0 ** -24 * np.abs(w).sum(1)).all()
    assert bool((out[other] == ones).all())


def test_a_gradient_of_2_34_elements_from_few_rows():
    m, k, n = (1 << 20) + 3, 16384, 3
    t, w = random_table(n, k, 2)
    dy = torch.randn(m, n, device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    dx = torch.full((m, k), float("nan"), dtype=torch.bfloat16, device=DEV)
    pk.check(pk.embbag_mx4_matmul_grad(dy, t, dx, torch.empty(256, dtype=torch.uint8, device=DEV)))
    wd = torch.from_numpy(w).to(DEV)
    for p in pieces(m, 1 << 15):
        d = dy[p].double()
        want = d[:, :1] * wd[0] + d[:, 1:2] * wd[1] + d[:, 2:] * wd[2]
        mag = (d[:, :1] * wd[0]).abs() + (d[:, 1:2] * wd[1]).abs() + (d[:, 2:] * wd[2]).abs()
        # (The nearest BF16 number, of a sum of three FP32 products.)
        assert bool(((dx[p].double() - want).abs() <= want.abs() * 2.0 ** -8 + mag * 2.0 ** -21).all()), p


def test_pooled_forward_of_more_than_2_26_wide_bags():
    dim, rows, batch = 516, 50, (1 << 26) + 7
    t, w = random_table(rows, dim, 3)
    wd = torch.from_numpy(w).to(DEV).bfloat16()
    assert bool((wd.double().cpu() == torch.from_numpy(w)).all())  # codes and scales fit BF16
    idx = (torch.arange(batch, device=DEV, dtype=torch.int32) * 7) % rows
    off = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    st = status()
    for weights in (None, torch.full((batch,), -2.0, device=DEV)):
        y = torch.full((1, batch, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
        pk.check(pk.embbag_mx4_forward(pk.Mx4Tables([t]), batch, idx, off, y, weights, d_status=st))
        for p in pieces(batch, 1 << 22):
            assert torch.equal(y[0, p], wd[idx[p].long()] * (1 if weights is None else -2)), p
        del y
    assert pk.embbag_status_read(st) == 0


@pytest.mark.parametrize("type_", [torch.float32, torch.bfloat16])
def test_logits_of_more_than_2_24_rows(type_):
    rows, vocab = (1 << 24) + 5, 8
    r = torch.arange(rows, device=DEV)
    x = ((r[:, None] + torch.arange(vocab, device=DEV)) % 100).to(type_)
    seen = (r % vocab).to(torch.int32)
    off = torch.arange(rows + 1, dtype=torch.int32, device=DEV)
    out = torch.full_like(x, float("nan"))
    st = status()
    pk.check(pk.embbag_logits_process(x, out, seen=seen, seen_offsets=off, presence=torch.ones(rows, device=DEV),
                                      bias_ids=((r + 1) % vocab).to(torch.int32), bias_offsets=off,
                                      biases=torch.full((rows,), 2.0, device=DEV), d_status=st))
    pk.check(pk.embbag_status_read(st))
    x[r, r % vocab] -= 1
    x[r, (r + 1) % vocab] += 2
    assert torch.equal(out, x)


def test_distillation_of_more_than_2_24_rows():
    rows, vocab = (1 << 24) + 5, 8
    r = torch.arange(rows, device=DEV)
    x = ((r[:, None] * 3 + torch.arange(vocab, device=DEV) * 5) % 11).float() * 0.5
    ids = (r % vocab).to(torch.int32)[:, None].contiguous()
    loss, grad, st = torch.full((rows,), float("nan"), device=DEV), torch.full_like(x, float("nan")), status()
    pk.check(pk.embbag_distill(x, ids, torch.zeros(rows, 1, device=DEV), 1.0, loss, None, grad=grad, d_status=st))
    pk.check(pk.embbag_status_read(st))
    z = x.double()
    lse = torch.logsumexp(z, 1)
    q = torch.exp(z - lse[:, None])
    q[r, r % vocab] -= 1
    assert bool(((grad.double() - q).abs() <= 1e-5).all())
    assert bool(((loss.double() - (lse - z[r, r % vocab])).abs() <= 1e-4).all())


def test_distillation_of_more_than_2_22_longer_rows():
    """Blocks of 1024 threads, in place."""
    rows, vocab = (1 << 22) + 3, 8200
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    some = torch.tensor([0, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, rows - 1], device=DEV)
    x[some] = torch.randn(len(some), vocab, device=DEV, generator=torch.Generator(DEV).manual_seed(4)).bfloat16()
    keep = x[some].double().cpu().numpy()
    ids = (torch.arange(rows, device=DEV) % vocab).to(torch.int32)[:, None].contiguous()
    loss, st = torch.full((rows,), float("nan"), device=DEV), status()
    pk.check(pk.embbag_distill(x, ids, torch.zeros(rows, 1, device=DEV), 1.0, loss, None, grad=x, d_status=st))
    pk.check(pk.embbag_status_read(st))
    want, grad, _, _ = ref.distill(keep, ids[some].cpu().numpy(), np.zeros((len(some), 1)), 1.0)
    assert np.allclose(loss[some].double().cpu().numpy(), want, rtol=1e-4, atol=1e-4)
    assert np.allclose(x[some].double().cpu().numpy(), grad, rtol=2.0 ** -8, atol=1e-7)
    other = torch.ones(rows, dtype=torch.bool, device=DEV)
    other[some] = False
    assert bool(((loss - float(np.log(vocab))).abs()[other] <= 1e-3).all())
    even = torch.tensor(1 / vocab, device=DEV).bfloat16()
    for p in pieces(rows, 1 << 18):
        r = torch.arange(p.start, p.stop, device=DEV)
        g = x[p]
        own = g[r - p.start, r % vocab][other[p]]
        assert bool((own == torch.tensor(1 / vocab - 1, device=DEV).bfloat16()).all())
        # The sum of a row's FP32 terms may put 1 / vocab on the other side of a BF16 midpoint: one unit.
        assert bool((((g.float() - even.float()).abs() > 2.0 ** -20).sum(1)[other[p]] <= 1).all())
