"""Scores whose blocks take several tiles: what one tile held (a NaN of x or of the table, the
workspace's bytes beside the last rows) must not reach the next."""
import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, coded_table, rounding, some_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


# Tiles of 128 x 128 on 512 blocks with edges of x (300 = 2 * 128 + 44) and of W, of 256 x 256 on 256
# blocks (1100 = 4 * 256 + 76), of 128 x 64; the last group of 128 elements whole and in part.
TILES = [(300, 70000, 128), (1100, 20003, 256), (300, 50001, 256), (1100, 65537, 128),
         (1100, 20003, 1000), (40, 150001, 256)]


def scores(x, t, n, out_type):
    m, k = x.shape
    out = torch.empty(m, n, dtype=DT[out_type], device=DEV)
    ws = torch.empty(pk.embbag_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    pk.check(pk.embbag_mx4_matmul(x.to(DEV), t, out, ws))
    return out


@pytest.mark.parametrize("out_type", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", TILES)
def test_what_the_workspace_held_reaches_no_score(m, n, k, out_type):
    t, w = coded_table(n, k, n + k)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(m)).to(DT["bf16"])
    out = scores(x, t, n, out_type)
    assert torch.isfinite(out).all()
    rows = some_rows(m)
    q = ref.dequantize(*ref.quantize(x[rows].double().numpy()), k)
    want = q @ w.T
    tol = 2 * (k + 8) * U * (np.abs(q) @ np.abs(w).T)
    close(out[rows], want, tol + rounding(np.abs(want) + tol, out_type), f"{m}x{n}x{k}")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("m,n,k", TILES)
def test_a_bad_block_of_x_stays_in_its_row(m, n, k, bad):
    """In every block of the last group, whose scales a tile leaves behind."""
    t, _ = coded_table(n, k, n + k)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(m))
    rows = sorted(r for r in {0, 5, 70, 299, m - 1} if r < m)
    first = (k - 1) // 128 * 128
    for i, r in enumerate(rows):
        x[r, min(first + 32 * (3 - i % 4) + 7, k - 1)] = bad
    out = torch.isnan(scores(x, t, n, "f32"))
    assert out[rows].all()
    assert int(out.sum()) == len(rows) * n


@pytest.mark.parametrize("m,n,k", TILES)
def test_a_bad_block_of_the_table_stays_in_its_column(m, n, k):
    t, _ = coded_table(n, k, n + k)
    cols = [0, 77, 1500, n // 3, n - 1]
    blocks = (k + 31) // 32
    for i, c in enumerate(cols):
        t.scales[c, blocks - 1 - i % min(blocks, 4)] = 255
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(m))
    out = torch.isnan(scores(x, t, n, "f32"))
    assert out[:, cols].all()
    assert int(out.sum()) == len(cols) * m
