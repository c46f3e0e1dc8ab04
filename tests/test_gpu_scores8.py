"""Scores of a 4-bit table from 8-bit rows on the GPU against the 64-bit reference: exact products,
so that only the additions and the output's rounding count."""
import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
import train_reference as ref
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, coded_table, random_table, rounding, some_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def rows8(m, k, seed, spread=6):
    """Rows of 8-bit codes: every code but NaN, scales around 1; and their values."""
    rng = np.random.default_rng(seed)
    g = -(-k // 128)
    codes = rng.integers(0, 127, (m, g * 128), np.uint8) + 128 * rng.integers(0, 2, (m, g * 128), np.uint8)
    codes[:, k:] = 0
    scales = np.zeros((m, g * 4), np.uint8)
    nb = -(-k // 32)
    scales[:, :nb] = rng.integers(127 - spread, 128 + spread, (m, nb), np.uint8)
    t = pk.Mx8Rows(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), k)
    return t, ref.values8(codes, scales, k)


def scores(x, t, out_type, pad=0, fill=0xFF):
    buf = torch.full((x.rows, t.rows + pad), -7.0, dtype=DT[out_type], device=DEV)
    out = buf[:, : t.rows]
    ws = torch.empty(pk.embbag_mx4_matmul_x8_workspace_bytes(x.rows, t.rows, x.dim), dtype=torch.uint8, device=DEV)
    ws.fill_(fill)
    pk.check(pk.embbag_mx4_matmul_x8(x, t, out, ws))
    if pad:
        assert (buf[:, t.rows:] == -7.0).all()
    return out


def check(out, xv, wv, k, out_type, what):
    want = xv @ wv.T
    # k products, added in FP32 in any order.  Into BF16 the products come in eights, of which each
    # loses less than 2^-13 of the largest, which is at most their sum.
    tol = (2 * (k + 8) * U + (8 * 2.0 ** -13 if out_type == "bf16" else 0)) * (np.abs(xv) @ np.abs(wv).T)
    close(out, want, tol + rounding(np.abs(want) + tol, out_type), what)


SIZES = [(1, 1, 4), (1, 70, 36), (2, 65, 128), (3, 130, 260), (5, 64, 1024), (16, 77, 516), (16, 300, 4096), (1, 1000, 4100),
         (17, 64, 32), (20, 33, 100), (33, 130, 128), (64, 257, 384), (65, 300, 516), (100, 1000, 1024),
         (129, 2000, 260), (200, 300, 2052), (257, 513, 640)]


@pytest.mark.parametrize("out_type", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_scores8(m, n, k, out_type):
    x, xv = rows8(m, k, m + n)
    t, wv = random_table(n, k, k)
    check(scores(x, t, out_type), xv, wv, k, out_type, f"{m}x{n}x{k}")
    check(scores(x, t, out_type, pad=3), xv, wv, k, out_type, f"{m}x{n}x{k}, padded")


# Tiles of 128 x 128 and 256 x 256 whose blocks take several, of 128 x 64, with edges on both sides.
TILES = [(300, 70000, 128), (1100, 20003, 256), (1100, 65537, 128), (1100, 20003, 1000), (40, 150001, 256),
         (600, 5000, 260), (2100, 66000, 132)]


@pytest.mark.parametrize("out_type", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", TILES)
def test_scores8_of_many_tiles(m, n, k, out_type):
    x, xv = rows8(m, k, m + n)
    t, wv = coded_table(n, k, n)
    rows = some_rows(m)
    check(scores(x, t, out_type)[rows], xv[rows], wv, k, out_type, f"{m}x{n}x{k}")


@pytest.mark.parametrize("m,n,k", [(3, 150, 260), (16, 150, 192), (40, 150, 192), (300, 70000, 128), (1100, 20003, 1000)])
def test_bad_blocks_and_codes_stay_in_their_row(m, n, k):
    """A block with the scale 255, and the code that is NaN, in every block of the last group."""
    x, _ = rows8(m, k, 3)
    t, _ = coded_table(n, k, n + k)
    first = (k - 1) // 128 * 128
    rows = sorted(r for r in {0, 2, 15, 39, 299, m - 1} if r < m)
    for i, r in enumerate(rows):
        at = min(first + 32 * (3 - i % 4) + 7, k - 1)
        if i % 2:
            x.codes[r, at] = 127
        else:
            x.scales[r, at // 32] = 255
    out = torch.isnan(scores(x, t, "f32"))
    assert out[rows].all()
    out[rows] = False
    assert not out.any()
    # A bad row of the table: its column.
    x, _ = rows8(m, k, 4)
    t.scales[n - 1, (k - 1) // 32] = 255
    out = torch.isnan(scores(x, t, "f32"))
    assert out[:, n - 1].all() and not out[:, : n - 1].any()


def test_norm_feeds_the_scores():
    """embbag_rmsnorm's 8-bit rows, scored, against the scores of the values they stand for."""
    for rows, dim, n in [(1, 260, 100), (50, 516, 300)]:
        g = torch.Generator().manual_seed(rows)
        h = torch.randn(rows, dim, generator=g).to(DEV)
        t, wv = random_table(n, dim, 5)
        q = pk.Mx8Rows.empty(rows, dim)
        pk.check(pk.embbag_rmsnorm(h, None, 1e-6, mx8=q))
        xv = ref.values8(q.codes.cpu().numpy(), q.scales.cpu().numpy(), dim)
        check(scores(q, t, "f32"), xv, wv, dim, "f32", "norm and scores")


def test_no_rows():
    t, _ = random_table(10, 32, 12)
    out = scores(pk.Mx8Rows.empty(0, 32), t, "f32")
    assert out.shape == (0, 10)
