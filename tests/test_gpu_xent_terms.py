"""Cross entropy of BF16 sides: where D enters the gradients' products with two BF16 terms (at most 256 rows that
count, however many there are, or a table of fewer than 1024 rows), within the bounds of two."""
import pytest
import torch

from gpu_util import DEV, require_gpu
from test_gpu_xent import close, expected, inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def counting(N, V, E, live, seed):
    """Inputs of which `live` rows count, spread over all of them."""
    x, w, labels = inputs(N, V, E, seed, ignored=0.0, sure=3.0)
    out = torch.randperm(N, generator=torch.Generator().manual_seed(seed))[live:]
    labels[out.to(DEV)] = -1
    return x, w, labels


def check_two_terms(x, w, labels):
    """Against the bounds of 256 rows that count at a time, which are those of two terms: the table's gradient is the
    sum of theirs, and its additions are at most as many times more as there are of them."""
    loss, dx, dw = run(x, w, labels)
    live = torch.nonzero(labels >= 0)[:, 0]
    parts = live.split(256)
    want, tol = torch.zeros(2, *dw.shape, dtype=torch.float64, device=DEV)
    for r in parts:
        l, gx, gw = expected(x[r], w, labels[r])
        close(loss[r], l, "loss")
        close(dx[r], gx, "dx")
        want += gw[0]
        tol += gw[1] * len(parts)
    close(dw, (want, tol), "dw")


# Narrow and wide tables, with D of less and of more elements than the second term is always stored for.
SIZES = [(300, 1200, 64), (2000, 1500, 128), (400, 1100, 36), (300, 1200, 260), (2000, 1100, 132), (70000, 2000, 132),
         (70000, 2048, 516)]


@pytest.mark.parametrize("live", [1, 100, 256])
@pytest.mark.parametrize("N,V,E", SIZES)
def test_few_rows_count(N, V, E, live):
    check_two_terms(*counting(N, V, E, live, N + V + live))


@pytest.mark.parametrize("N,V,E", SIZES)
def test_one_row_more(N, V, E):
    x, w, labels = counting(N, V, E, 257, N + V)
    r = torch.nonzero(labels >= 0)[:, 0]
    loss, dx, dw = run(x, w, labels)
    e = expected(x[r], w, labels[r])
    for g, pair, what in zip((loss[r], dx[r], dw), e, ("loss", "dx", "dw")):
        close(g, pair, what)


@pytest.mark.parametrize("N,V,E", [(600, 500, 64), (513, 1023, 128), (600, 40, 36), (600, 1023, 132)])
def test_small_tables(N, V, E):
    check_two_terms(*counting(N, V, E, N, N + V))


def test_pieces_without_gradients():
    """So many rows that the loss alone takes the vocabulary in pieces: 2^20 rows, 4096 columns at a time."""
    N, V = 1 << 20, 10001
    x, w, labels = counting(N, V, 132, 300, 5)
    r = torch.nonzero(labels >= 0)[:, 0]
    loss = run(x, w, labels, dx=False, dw=False)[0]
    close(loss[r], expected(x[r], w, labels[r])[0], "loss")
    assert int((loss != 0).sum()) <= 300
