"""Cross entropy over a table and both gradients on the GPU against a 64-bit evaluation of the
formulas, within bounds that count the roundings on the way."""
import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
import train_reference as ref
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, padded

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def inputs(N, V, E, seed, tx="bf16", tw="bf16", ignored=0.2, sure=6.0):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(V, E, generator=g) * E ** -0.5).to(DT[tw])
    labels = torch.randint(0, V, (N,), generator=g)
    x = torch.randn(N, E, generator=g) + w[labels].float() * (torch.rand(N, 1, generator=g) * sure)
    x = x.to(DT[tx])
    labels[torch.rand(N, generator=g) < ignored] = -1
    return x.to(DEV), w.to(DEV), labels.to(torch.int32).to(DEV)


def run(x, w, labels, weights=None, scale=1.0, dx=True, dw=True, fill=0xFF, want=0, grads=None):
    N, V, E = x.shape[0], w.shape[0], x.shape[1]
    f32 = torch.float32 in (x.dtype, w.dtype)
    loss = torch.full((N,), -7.0, device=DEV)
    if grads is None:
        grads = (torch.full_like(x, -7.0) if dx else None, torch.full_like(w, -7.0) if dw else None)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    n = pk.embbag_xent_workspace_bytes(N, V, E, pk.EMBBAG_F32 if f32 else pk.EMBBAG_BF16,
                                       grads[0] is not None or grads[1] is not None)
    ws = torch.empty(n + 256, dtype=torch.uint8, device=DEV)
    ws.fill_(fill)
    pk.check(pk.embbag_xent(x, w, labels, loss, ws[:n], grad_x=grads[0], grad_table=grads[1], row_weights=weights,
                            scale=scale, d_status=status))
    assert int(status) == want
    assert (ws[n:] == fill).all()
    return (loss,) + tuple(grads)


def expected(x, w, labels, weights=None, scale=1.0):
    """(value, bound) of loss, dx and dw, in 64 bits, some rows at a time."""
    N, V, E = x.shape[0], w.shape[0], x.shape[1]
    f32 = torch.float32 in (x.dtype, w.dtype)
    # D: rounded to BF16 (2^-8), to two terms (2^-16), or whole; products of three terms each lack
    # 2^-22 of each at most.
    qd = U if f32 else 2.0 ** -16 if N <= 256 else 2.0 ** -8
    lack = 2.0 ** -22 if f32 else 0.0
    wd, wa = w.double(), w.double().abs()
    weights = torch.ones(N, device=DEV) if weights is None else weights
    live = torch.nonzero((labels >= 0) & (labels < V) & (weights != 0))[:, 0]
    loss, tloss = torch.zeros(2, N, dtype=torch.float64, device=DEV)
    dx, tdx = torch.zeros(2, N, E, dtype=torch.float64, device=DEV)
    dw, tdw = torch.zeros(2, V, E, dtype=torch.float64, device=DEV)
    for r in live.split(max(1, 40_000_000 // V)):
        xd, k, at = x[r].double(), weights[r].double()[:, None], labels[r].long()
        i = torch.arange(r.numel(), device=DEV)
        z = scale * (xd @ wd.t())
        # A score: E products added in FP32 in some order, the scale's product.
        ez = (2 * (E + 8) * U + lack) * abs(scale) * (xd.abs() @ wa.t()).max(1, keepdim=True).values
        top = z.max(1, keepdim=True).values
        p = torch.exp(z - top)
        total = p.sum(1, keepdim=True)
        p /= total
        loss[r] = k[:, 0] * (torch.log(total) + top - z[i, at][:, None])[:, 0]
        # The sum of exponentials: V terms in chains of at most 64 + V / 2048 and joins.
        esum = 2 * ez + U * (200 + V / 1000)
        size = (torch.log(total) + (top - z[i, at][:, None]).abs() + 2)[:, 0]
        tloss[r] = k.abs()[:, 0] * (2 * ez + esum)[:, 0] + 8 * U * k.abs()[:, 0] * size
        rho = 2 * ez + esum + U * (16 + 4 * (top - z))
        d = p.clone()
        d[i, at] -= 1.0
        derr = p * rho + d.abs() * (qd + 8 * U) + 2 * U * p + 1e-38
        dx[r] = scale * k * (d @ wd)
        tdx[r] = abs(scale) * k.abs() * (derr @ wa + (2 * (V + 8) * U + lack) * (d.abs() @ wa))
        dw += scale * (k * d).t() @ xd
        tdw += abs(scale) * ((k.abs() * derr).t() @ xd.abs() +
                             (2 * (live.numel() + 8) * U + lack) * (k * d).abs().t() @ xd.abs())
    return (loss, tloss), (dx, tdx), (dw, tdw)


def close(got, pair, what):
    if got is None:
        return
    want, tol = pair
    half = {torch.float32: U, torch.bfloat16: 2.0 ** -8}[got.dtype]
    off = (got.double() - want).abs()
    ok = off <= tol + half * (want.abs() + tol) + 1e-37
    if not ok.all():
        i = tuple(torch.nonzero(~ok)[0].tolist())
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} off; first at {i}: got {float(got[i])!r}, "
                             f"want {float(want[i])!r}, allowed {float(tol[i])!r}")


def check(N, V, E, seed, tx="bf16", tw="bf16", weighted=False, scale=1.0, ignored=0.2, sure=6.0):
    x, w, labels = inputs(N, V, E, seed, tx, tw, ignored, sure)
    weights = None
    if weighted:
        g = torch.Generator().manual_seed(seed + 1)
        weights = ((torch.rand(N, generator=g) - 0.3) * 2).to(DEV)
        weights[::7] = 0.0
    got = run(x, w, labels, weights, scale)
    for g, e, what in zip(got, expected(x, w, labels, weights, scale), ("loss", "dx", "dw")):
        close(g, e, f"{what} of {N}x{V}x{E} {tx} {tw}")


SIZES = [(1, 1, 4), (1, 1000, 64), (2, 3, 12), (1, 5003, 260), (3, 100, 36), (17, 129, 64), (32, 257, 100),
         (33, 1000, 128), (40, 2050, 516), (64, 300, 1028), (65, 700, 300), (130, 5000, 32), (200, 40, 260),
         (257, 1000, 256), (300, 513, 1024), (700, 2050, 132)]


@pytest.mark.parametrize("tx,tw", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("N,V,E", SIZES)
def test_xent(N, V, E, tx, tw):
    check(N, V, E, N + V + E, tx, tw)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,E", [(1, 300, 36), (33, 1000, 128), (300, 513, 260), (70, 2050, 64)])
@pytest.mark.parametrize("scale", [1.0, 0.125, -2.5, 0.0])
def test_weights_and_scale(N, V, E, t, scale):
    check(N, V, E, N, t, t, weighted=True, scale=scale)


# Tiles of 256 x 256 in all three products, with edges on every side; several pieces of the vocabulary
# by the size of D, of the table's terms, and by the width of D's rows; a contraction split over rows.
@pytest.mark.parametrize("N,V,E,t", [(300, 25601, 1500, "bf16"), (300, 25001, 1500, "f32"), (600, 20000, 516, "bf16"),
                                     (20000, 14001, 8, "bf16"), (7000, 14000, 36, "f32"), (3, 600001, 8, "bf16"),
                                     (2, 530000, 4, "f32"), (40, 60001, 2052, "f32"), (5000, 300, 260, "bf16"),
                                     (3000, 1, 64, "f32"), (4500, 257, 100, "f32"), (20000, 14001, 132, "bf16"),
                                     (7000, 14000, 132, "f32"), (3, 600001, 136, "bf16"), (2, 530000, 132, "f32"),
                                     (3000, 1, 132, "f32"), (4500, 257, 164, "f32"), (9000, 1000, 128, "bf16"),
                                     (2000, 30001, 128, "f32"), (100, 70001, 64, "bf16"), (1000, 32763, 2052, "bf16"),
                                     (1000, 32763, 512, "f32")])
def test_large(N, V, E, t):
    check(N, V, E, N, t, t, sure=4.0)


def test_gradients_against_differences():
    rng = np.random.default_rng(4)
    N, V, E = 5, 23, 12
    x, w = rng.normal(size=(N, E)), rng.normal(size=(V, E))
    labels, k = np.array([3, -1, 22, 0, 3]), rng.normal(size=N)
    f = lambda x, w: ref.xent(x, w, labels, k, 0.7)[0].sum()
    t = lambda a: torch.from_numpy(a).float().to(DEV)
    loss, dx, dw = run(t(x), t(w), torch.from_numpy(labels).int().to(DEV), t(k), 0.7)
    want = ref.xent(x, w, labels, k, 0.7)
    assert np.abs(loss.cpu().numpy() - want[0]).max() < 1e-5
    step = 1e-5
    for i, e in [(0, 0), (1, 5), (2, 11), (4, 3)]:
        d = np.zeros_like(x)
        d[i, e] = step
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * step) - float(dx[i, e])) < 1e-4
    for v, e in [(3, 0), (22, 7), (11, 11)]:
        d = np.zeros_like(w)
        d[v, e] = step
        assert abs((f(x, w + d) - f(x, w - d)) / (2 * step) - float(dw[v, e])) < 1e-4


@pytest.mark.parametrize("N,V,E,t", [(5, 300, 36, "f32"), (70, 1000, 128, "bf16"), (300, 513, 260, "bf16"),
                                     (300, 25601, 64, "bf16")])
def test_rows_left_out_may_hold_anything(N, V, E, t):
    """NaN and infinities where the label is negative or the weight 0, a row's worth of them at either end."""
    x, w, labels = inputs(N, V, E, 3, t, t, ignored=0.3)
    weights = torch.full((N,), 0.25, device=DEV)
    labels[0], labels[N - 1] = -1, 2
    weights[N - 1] = 0.0
    clean = run(x, w, labels, weights)
    out = (labels < 0) | (weights == 0)
    x[out] = float("nan")
    x[N - 1] = float("inf")
    got = run(x, w, labels, weights, fill=0x00)
    assert (got[0][out] == 0).all() and (got[1][out] == 0).all()
    for a, b in zip(got, clean):
        assert torch.equal(a, b)
    for g, e, what in zip(got, expected(torch.nan_to_num(x, 0, 0, 0), w, labels, weights), ("loss", "dx", "dw")):
        close(g, e, what)


@pytest.mark.parametrize("N", [1, 40, 300])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_no_row_counts(N, t):
    x, w, labels = inputs(N, 700, 36, 3, t, t)
    labels.fill_(-1)
    for g in run(x, w, labels):
        assert (g == 0).all()
    labels.fill_(5)
    for g in run(x, w, labels, torch.zeros(N, device=DEV)):
        assert (g == 0).all()


def test_no_rows():
    x, w, labels = inputs(0, 300, 36, 3)
    loss, dx, dw = run(x, w, labels)
    assert loss.shape == (0,) and (dw == 0).all()
    run(x, w, labels, dw=False)


def test_labels_past_the_vocabulary_are_reported_and_left_out():
    N, V = 40, 500
    x, w, labels = inputs(N, V, 36, 3, ignored=0.0)
    bad = labels.clone()
    bad[3], bad[39] = V, 2 ** 31 - 1
    labels[3], labels[39] = -1, -2 ** 31
    got = run(x, w, bad, want=pk.EMBBAG_ERR_INDEX_RANGE)
    for a, b in zip(got, run(x, w, labels)):
        assert torch.equal(a, b)
    assert got[0][3] == 0 and (got[1][39] == 0).all()


@pytest.mark.parametrize("N,V,E,tx,tw", [(5, 300, 36, "f32", "f32"), (70, 1000, 64, "bf16", "bf16"),
                                         (70, 1000, 68, "bf16", "bf16"), (300, 513, 264, "bf16", "f32")])
def test_strides(N, V, E, tx, tw):
    """Rows apart, at addresses of 4 elements' alignment, in junk that stays as it is; x as its own gradient."""
    x, w, labels = inputs(N, V, E, 8, tx, tw)
    want = run(x, w, labels)
    for extra, offset in [(4, 4), (12, 8), (8, 4)]:
        xs, ws = padded(x, extra, offset), padded(w, extra, offset)
        gx, gw = padded(torch.zeros_like(x), extra, offset), padded(torch.zeros_like(w), extra, offset)
        got = run(xs, ws, labels, grads=(gx, gw))
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for t in (xs, ws, gx, gw):
            mask = torch.ones_like(t._base, dtype=torch.bool)
            torch.as_strided(mask, t.shape, t.stride(), t.storage_offset()).fill_(False)
            assert torch.isnan(t._base[mask]).all()
        got = run(xs, ws, labels, grads=(xs, None))
        assert torch.equal(xs, want[1]) and torch.equal(got[0], want[0])


@pytest.mark.parametrize("N,V,E,t", [(1, 1000, 64, "bf16"), (70, 1000, 260, "f32"), (300, 25601, 64, "bf16"),
                                     (300, 300, 64, "bf16")])
def test_each_output_alone_and_again(N, V, E, t):
    x, w, labels = inputs(N, V, E, 9, t, t)
    loss, dx, dw = run(x, w, labels)
    for a, b in zip(run(x, w, labels, fill=0x7F), (loss, dx, dw)):
        assert torch.equal(a, b)
    assert torch.equal(run(x, w, labels, dx=False, dw=False)[0], loss)
    assert torch.equal(run(x, w, labels, dw=False)[1], dx)
    assert torch.equal(run(x, w, labels, dx=False)[2], dw)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_scores_far_from_zero(t):
    """Scores that share an offset of 1000, and one far above the others: the loss keeps its digits."""
    N, V, E = 9, 300, 64
    x, w, labels = inputs(N, V, E, 11, t, t, ignored=0.0, sure=0.0)
    x[:, 0], w[:, 0] = 1024.0, 1.0
    for g, e, what in zip(run(x, w, labels), expected(x, w, labels), ("loss", "dx", "dw")):
        close(g, e, what)
    x[:, 0], w[:, 0] = 128.0, 0.0
    w[labels.long(), 0] = 1.0  # certain: exp(-128) beside 1
    got = run(x, w, labels)
    assert torch.isfinite(got[0]).all() and (got[0] < 20).all()
    for g, e, what in zip(got, expected(x, w, labels), ("loss", "dx", "dw")):
        close(g, e, what)


@pytest.mark.parametrize("N,V,E,t", [(5, 300, 36, "f32"), (70, 1000, 128, "bf16"), (300, 25601, 64, "bf16")])
def test_nan_of_a_row_stays_in_its_loss_and_gradient(N, V, E, t):
    x, w, labels = inputs(N, V, E, 12, t, t, ignored=0.0)
    clean = run(x, w, labels)
    x[N // 2, E - 1] = float("nan")
    loss, dx, dw = run(x, w, labels)
    assert torch.isnan(loss[N // 2]) and torch.isnan(dx[N // 2]).all() and torch.isnan(dw).all()
    keep = torch.arange(N, device=DEV) != N // 2
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(dx[keep], clean[1][keep])
    # Minus infinity as a score: a token that cannot come.
    x, w, labels = inputs(N, V, E, 12, t, t, ignored=0.0)
    x[:, 0] = x[:, 0].abs() + 1
    w[V - 1, 0] = -float("inf")
    labels[labels == V - 1] = 0
    loss = run(x, w, labels, dx=False, dw=False)[0]
    w[V - 1, 0] = -1e30 if t == "f32" else -1e30
    close(loss, expected(x, w[: V - 1].contiguous(), labels)[0], "loss without the last token")
