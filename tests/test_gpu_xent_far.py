"""Cross entropy where a tile's loads pass 2^28 bytes, at which their base moves, and a side 2^30, which its buffer
covers at a time: D's rows in the table's gradient, and a table read as it stands in rows of the largest stride."""
import pytest
import torch

from gpu_util import DEV, require_gpu
from test_gpu_xent import check, close, expected, inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def test_rows_of_d_past_the_move():
    """4600 rows of D of 66,048 bytes (304 MB), in one piece and one split of the contraction over them."""
    check(4600, 33000, 132, 3, "bf16", "bf16", ignored=0.0, sure=4.0)


@pytest.mark.parametrize("t,N", [("bf16", 300), ("bf16", 20), ("f32", 300), ("f32", 20)])
def test_the_largest_stride(t, N):
    """1100 rows of the table 2^19 elements apart (BF16 1.15 GB, FP32 2.3 GB), and its gradient likewise."""
    V, E, stride = 1100, 264, 1 << 19
    x, w, labels = inputs(N, V, E, N, t, t)
    apart = lambda: torch.empty(V, stride, dtype=w.dtype, device=DEV)[:, 8:8 + E]
    far, gx, gw = apart(), torch.zeros_like(x), apart()
    far._base.fill_(float("nan"))
    far.copy_(w)
    gw._base.fill_(-3.0)
    loss, dx, dw = run(x, far, labels, grads=(gx, gw))
    for g, e, what in zip((loss, dx, dw), expected(x, w, labels), ("loss", "dx", "dw")):
        close(g, e, what)
    for a, b in zip((loss, dx, dw), run(x, w, labels)):
        assert torch.equal(a, b)
    assert (gw._base[:, :8] == -3).all() and (gw._base[:, 8 + E:] == -3).all()
