"""Cross entropy of few rows over a wide table in FP32, whose products read the table as it stands, and of more
rows, whose scores are kept (300 rows of 260 and the like): at the edges of the tiles (32 and 128 rows, 32 rows of the table, 32 and 128 elements of a row), within the bounds that
count the roundings."""
import pytest
import torch

from gpu_util import DEV, require_gpu
from test_gpu_mx4 import padded
from test_gpu_xent import check, close, expected, inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


@pytest.mark.parametrize("tx,tw", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("N,V,E", [(1, 1, 132), (1, 2000, 132), (2, 31, 136), (31, 33, 160), (32, 255, 164), (33, 1000, 132),
                                   (64, 257, 256), (65, 100, 260), (128, 513, 388), (129, 1003, 516), (257, 64, 516),
                                   (300, 1500, 700), (512, 700, 1028), (513, 700, 1028), (194, 300, 260),
                                   (195, 300, 260), (300, 257, 192), (1000, 1003, 204), (700, 40, 1500)])
def test_sizes(N, V, E, tx, tw):
    check(N, V, E, N + V + E, tx, tw, ignored=0.2 if N > 2 else 0.0)


@pytest.mark.parametrize("N,V,E", [(9, 300, 132), (150, 1030, 260)])
@pytest.mark.parametrize("scale", [0.125, -2.5, 0.0])
def test_weights_and_scale(N, V, E, scale):
    check(N, V, E, N, "f32", "f32", weighted=True, scale=scale)


@pytest.mark.parametrize("N,V,E,t", [(7, 100003, 132, "f32"), (128, 524288, 132, "bf16"), (3, 524289, 132, "f32"),
                                     (200, 20011, 1500, "f32"), (1500, 30001, 260, "f32"), (600, 250001, 196, "f32")])
def test_large(N, V, E, t):
    check(N, V, E, N, "f32", t, sure=4.0)


@pytest.mark.parametrize("N", [5, 70, 150, 300])
def test_rows_left_out_may_hold_anything(N):
    x, w, labels = inputs(N, 700, 260, 3, "f32", "f32", ignored=0.3)
    weights = torch.full((N,), 0.25, device=DEV)
    labels[0], labels[N - 1], weights[N - 1] = -1, 2, 0.0
    clean = run(x, w, labels, weights)
    out = (labels < 0) | (weights == 0)
    x[out] = float("nan")
    got = run(x, w, labels, weights, fill=0x00)
    for a, b in zip(got, clean):
        assert torch.equal(a, b)
    for g, e, what in zip(got, expected(torch.nan_to_num(x, 0), w, labels, weights), ("loss", "dx", "dw")):
        close(g, e, what)


@pytest.mark.parametrize("N", [1, 40, 190, 300])
def test_no_row_counts(N):
    x, w, labels = inputs(N, 700, 260, 3, "f32", "f32")
    labels.fill_(-1)
    for g in run(x, w, labels):
        assert (g == 0).all()


@pytest.mark.parametrize("N,tx,tw", [(5, "f32", "f32"), (70, "f32", "bf16"), (130, "bf16", "f32"), (300, "f32", "f32")])
def test_strides(N, tx, tw):
    x, w, labels = inputs(N, 1000, 260, 8, tx, tw)
    want = run(x, w, labels)
    for extra, offset in [(4, 4), (12, 8)]:
        xs, ws = padded(x, extra, offset), padded(w, extra, offset)
        gx, gw = padded(torch.zeros_like(x), extra, offset), padded(torch.zeros_like(w), extra, offset)
        for a, b in zip(run(xs, ws, labels, grads=(gx, gw)), want):
            assert torch.equal(a, b)
        for t in (xs, ws, gx, gw):
            mask = torch.ones_like(t._base, dtype=torch.bool)
            torch.as_strided(mask, t.shape, t.stride(), t.storage_offset()).fill_(False)
            assert torch.isnan(t._base[mask]).all()
        assert torch.equal(run(xs, ws, labels, grads=(xs, None))[1], want[1])


@pytest.mark.parametrize("N", [1, 70, 190, 300])
def test_each_output_alone_and_again(N):
    x, w, labels = inputs(N, 1000, 260, 9, "f32", "f32")
    loss, dx, dw = run(x, w, labels)
    for a, b in zip(run(x, w, labels, fill=0x7F), (loss, dx, dw)):
        assert torch.equal(a, b)
    assert torch.equal(run(x, w, labels, dx=False, dw=False)[0], loss)
    assert torch.equal(run(x, w, labels, dw=False)[1], dx)
    assert torch.equal(run(x, w, labels, dx=False)[2], dw)


@pytest.mark.parametrize("N,t", [(3, "f32"), (70, "f32"), (300, "f32"), (3, "bf16"), (60, "bf16"), (70, "bf16")])
def test_a_row_with_nan_or_infinity_keeps_it(N, t):
    """The other rows' losses and gradients are the same bits; the row's own, and the table's, are NaN."""
    x, w, labels = inputs(N, 500, 260, 5, t, t, ignored=0.0)
    loss, dx, _ = run(x, w, labels)
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[1, 7] = bad
        got = run(y, w, labels)
        keep = torch.arange(N, device=DEV) != 1
        assert torch.equal(got[0][keep], loss[keep]) and torch.equal(got[1][keep], dx[keep])
        assert not torch.isfinite(got[0][1]) and torch.isnan(got[1][1]).all() and torch.isnan(got[2]).all(1).any()
