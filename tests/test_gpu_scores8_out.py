"""Scores from 8-bit rows into both types of output: bad blocks and codes, rows whose products cancel, and elements at
the ends of the range."""
import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
import train_reference as ref
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import coded_table
from test_gpu_scores8 import check, rows8, scores

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


@pytest.mark.parametrize("out_type", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 150, 128), (3, 150, 260), (16, 150, 1028), (40, 150, 192), (100, 9000, 260),
                                   (300, 70000, 128), (1100, 20003, 1000)])
def test_bad_blocks_and_codes_stay_in_their_row(m, n, k, out_type):
    """The scale 255 and the code that is NaN, in every block of the last group; then bad rows of the table, the first,
    one in a tile's middle and the last.  Blocks take several tiles in the larger sizes."""
    x, _ = rows8(m, k, 3)
    t, _ = coded_table(n, k, n + k)
    first = (k - 1) // 128 * 128
    rows = sorted(r for r in {0, 2, 15, 39, 299, m - 1} if r < m)
    for i, r in enumerate(rows):
        at = min(first + 32 * (3 - i % 4) + 7, k - 1)
        if i % 2:
            x.codes[r, at] = 127 + 128 * (i % 4 == 3)
        else:
            x.scales[r, at // 32] = 255
    out = torch.isnan(scores(x, t, out_type))
    assert out[rows].all()
    out[rows] = False
    assert not out.any()
    x, _ = rows8(m, k, 4)
    columns = [0, n // 2, n - 1]
    for i, c in enumerate(columns):
        t.scales[c, min(i, (k - 1) // 32)] = 255
    out = torch.isnan(scores(x, t, out_type))
    assert out[:, columns].all()
    out[:, columns] = False
    assert not out.any()


@pytest.mark.parametrize("out_type", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 70, 128), (16, 300, 516), (40, 150, 192), (300, 9000, 256), (1100, 20003, 128)])
def test_rows_whose_large_products_cancel(m, n, k, out_type):
    """Neighbours of 448 and -448 against equal elements, beside which the others are 2^-15 of them: into FP32 what is
    left is right to FP32's additions, into BF16 to the bits that the products keep (the bounds of `check`)."""
    x, _ = rows8(m, k, m, spread=0)
    t, _ = coded_table(n, k, n)
    rng = np.random.default_rng(k)
    codes = rng.integers(0, 25, (m, x.codes.shape[1]), np.uint8) + 128 * rng.integers(0, 2, (m, x.codes.shape[1]), np.uint8)
    pair = rng.integers(0, k // 2, (m, 3)) * 2
    for r in range(m):
        codes[r, pair[r]], codes[r, pair[r] + 1] = 126, 126 + 128
    codes[:, k:] = 0
    x.codes.copy_(torch.from_numpy(codes))
    xv = ref.values8(codes, x.scales.cpu().numpy(), k)
    # The table's elements in pairs: both halves of a byte the same.
    t.codes.copy_((t.codes & 15) * 17)
    table = torch.empty(n, k, device=DEV)
    pk.check(pk.embbag_mx4_dequantize(t, table))
    wv = table.double().cpu().numpy()
    some = sorted({0, m // 2, m - 1})
    check(scores(x, t, out_type)[some], xv[some], wv, k, out_type, f"{m}x{n}x{k}")


def test_the_ends_of_the_range():
    """Rows read back: elements of FP32's largest magnitude round to 2^128, which is an infinity, smaller ones do not."""
    g = torch.ones(1, 64, device=DEV)
    w = torch.full((64,), 3.4e38, device=DEV)
    w[32:] = 3.25e38  # 245 * 2^120: rounds to 240
    q, back = pk.Mx8Rows.empty(1, 64), torch.empty(1, 64, device=DEV)
    pk.check(pk.embbag_rmsnorm(g, w, 1e-30, mx8=q))
    codes, scales = ref.quantize8(w[None].double().cpu().numpy())
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)
    pk.check(pk.embbag_mx8_dequantize(q, back))
    assert torch.isinf(back[0, :32]).all() and (back[0, 32:].double() == 240 * 2.0 ** 120).all()
