"""Infinities and NaN in dy, in every place of a row: the gradient's infinities and NaN are those of the
64-bit product (an infinity times a zero of the table is NaN, times anything else an infinity)."""
import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, coded_table, random_table

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def gradient(dy, t, k):
    m, n = dy.shape
    ws = torch.empty(pk.embbag_mx4_matmul_grad_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    dx = torch.empty(m, k, device=DEV)
    pk.check(pk.embbag_mx4_matmul_grad(dy.to(DEV), t, dx, ws))
    return dx


@pytest.mark.parametrize("y_type", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 13, 63, 64, 65, 71, 72, 100, 127, 300, 519, 16385, 16390])
def test_an_infinity_in_any_of_the_last_columns(n, y_type):
    """Row i has its infinity in the i-th column from the end, one row none."""
    k = 68
    t, w = random_table(n, k, n)
    m = min(n, 70) + 1
    dy = torch.randn(m, n, generator=torch.Generator().manual_seed(n)).to(DT[y_type])
    for i in range(m - 1):
        dy[i, n - 1 - i] = float("inf") * (-1) ** i
    d = dy.double().numpy()
    with np.errstate(invalid="ignore"):
        want = d @ w
    fin = np.where(np.isfinite(d), np.abs(d), 0)
    close(gradient(dy, t, k), want, 2 * (n + 8) * U * (fin @ np.abs(w)) + 1e-38, f"n={n}")
    assert np.isinf(want[: m - 1]).any() and np.isfinite(want[m - 1]).all()


@pytest.mark.parametrize("m,n,k,y_type", [
    (200, 5003, 256, "bf16"), (700, 16390, 700, "bf16"), (1500, 50001, 100, "bf16"), (900, 8195, 260, "f32"),
    (2100, 15003, 512, "bf16")])
def test_infinities_of_larger_products(m, n, k, y_type):
    t, w = coded_table(n, k, n)
    dy = torch.randn(m, n, generator=torch.Generator().manual_seed(m)).to(DT[y_type])
    rows = [0, 5, m // 2, m - 1]
    for i, r in enumerate(rows):
        dy[r, n - 1 - 2 * i] = float("inf")
    dx = gradient(dy, t, k)
    other = torch.ones(m, dtype=torch.bool)
    other[rows] = False
    assert torch.isfinite(dx[other.to(DEV)]).all()
    with np.errstate(invalid="ignore"):
        want = dy[rows].double().numpy() @ w
    assert np.array_equal(np.isnan(want), torch.isnan(dx[rows]).cpu().numpy())
    assert np.array_equal(want[~np.isnan(want)], dx[rows].double().cpu().numpy()[~np.isnan(want)])


@pytest.mark.parametrize("y_type", ["f32", "bf16"])
@pytest.mark.parametrize("n", [13, 71, 300])
def test_a_nan_makes_its_row_nan(n, y_type):
    t, _ = random_table(n, 64, n)
    dy = torch.randn(n + 1, n, generator=torch.Generator().manual_seed(n)).to(DT[y_type])
    dy[torch.arange(n), torch.arange(n)] = float("nan")
    dx = gradient(dy, t, 64)
    assert torch.isnan(dx[:n]).all() and torch.isfinite(dx[n]).all()
