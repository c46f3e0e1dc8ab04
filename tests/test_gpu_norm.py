"""RMS norm, 8-bit rows and the norm's gradients on the GPU against the 64-bit reference, within
bounds that count the FP32 roundings on the way."""
import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
import train_reference as ref
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, padded, rounding

pytestmark = pytest.mark.gpu

SHAPES = [(1, 4), (3, 28), (5, 32), (7, 36), (17, 128), (33, 132), (4, 256), (3, 260), (9, 512), (2, 516),
          (5, 1024), (4, 1028), (3, 2048), (2, 2052), (3, 4096), (2, 4100), (2, 8192), (2, 8196), (2, 16384),
          (1, 16380), (5000, 64), (1500, 516)]
# Rounding of h (1), of 1/rms (its mantissa 0.5, square root 1, quotient 1; and h's own in the mean 1),
# of the product with it (1) and with the weight (1).
NORM_U = 6.5


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def rows_of(rows, dim, seed, type_="f32", spread=3):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, dim)) * np.exp(rng.normal(size=(1, dim)) * 0.7)
    x *= np.exp2(rng.integers(-spread, spread + 1, size=(rows, 1)))
    return torch.from_numpy(x).to(DT[type_])


def weight_of(dim, seed, type_):
    if type_ is None:
        return None
    return torch.from_numpy(1.0 + 0.3 * np.random.default_rng(seed).normal(size=dim)).to(DT[type_])


def host(t):
    return t.double().cpu().numpy()


def dev(t):
    return None if t is None else t.to(DEV)


def empty8(rows, dim):
    t = pk.Mx8Rows.empty(rows, dim)
    t.codes.fill_(0x55), t.scales.fill_(0x55)
    return t


@pytest.mark.parametrize("tx,tr,tw,to", [("f32", None, "f32", "f32"), ("bf16", "bf16", "bf16", "bf16"),
                                         ("bf16", "f32", "f32", "bf16"), ("f32", "bf16", None, "f32")])
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_norm(rows, dim, tx, tr, tw, to):
    seed = rows * 31 + dim
    x, w = rows_of(rows, dim, seed, tx), weight_of(dim, seed + 1, tw)
    r = None if tr is None else rows_of(rows, dim, seed + 2, tr)
    h = host(x) if r is None else host(x) + host(r)
    s = torch.empty(rows, dim, dtype=DT[tr or "f32"], device=DEV)
    out = torch.empty(rows, dim, dtype=DT[to], device=DEV)
    pk.check(pk.embbag_rmsnorm(dev(x), dev(w), 1e-6, out=out, residual=dev(r), sum_out=s))
    y, _, _ = ref.rmsnorm(h, 1.0 if w is None else host(w), 1e-6)
    close(s, h, U * np.abs(h) + rounding(h, tr or "f32"), "sum")
    # (h is a sum that may cancel: its rounding error is relative to itself, one FP32 addition.)
    close(out, y, NORM_U * U * np.abs(y) + rounding(y, to), "out")


@pytest.mark.parametrize("tx", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim", SHAPES[:-2] + [(70, 64), (30, 516)])
def test_eight_bit_rows_hold_the_fp32_output(rows, dim, tx):
    seed = rows + dim * 7
    x, w = rows_of(rows, dim, seed, tx, spread=40), weight_of(dim, seed, "f32")
    x[0, : dim // 2] = 0  # blocks of zeros
    w[dim // 3] = 0.0
    x, w = dev(x), dev(w)
    out = torch.empty(rows, dim, device=DEV)
    q = empty8(rows, dim)
    pk.check(pk.embbag_rmsnorm(x, w, 1e-6, out=out, mx8=q))
    codes, scales = ref.quantize8(host(out))
    np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
    np.testing.assert_array_equal(q.codes.cpu().numpy(), codes)
    alone = empty8(rows, dim)
    pk.check(pk.embbag_rmsnorm(x, w, 1e-6, mx8=alone))
    assert torch.equal(alone.codes, q.codes) and torch.equal(alone.scales, q.scales)
    for type_ in ("f32", "bf16"):
        back = torch.empty(rows, dim, dtype=DT[type_], device=DEV)
        pk.check(pk.embbag_mx8_dequantize(q, back))
        np.testing.assert_array_equal(host(back), ref.values8(codes, scales, dim))


def test_every_code_is_rounded_to():
    """Ties and values around every code: weights carry them, rows of equal magnitudes are 1 or -1."""
    v = ref.E4M3[:127]
    mid = (v[1:] + v[:-1]) / 2
    vals = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(1e9)).astype(np.float64),
                           np.nextafter(mid.astype(np.float32), np.float32(0)).astype(np.float64)])
    n = -(-vals.size // 31)
    w = np.zeros((n, 32))
    w[:, 31] = 448.0  # fixes each block's scale
    flat = np.zeros(n * 31)
    flat[: vals.size] = vals
    w[:, :31] = flat.reshape(n, 31)
    dim = n * 32
    sign = np.where(np.arange(dim) % 3 == 0, -1.0, 1.0)
    x = torch.from_numpy(sign[None] * np.array([[2.0 ** 60], [1.0]])).float().to(DEV)
    out, q = torch.empty(2, dim, device=DEV), empty8(2, dim)
    weight = torch.from_numpy(w.reshape(-1)).float().to(DEV)
    # eps vanishes beside a mean square of 1 in FP32, and so does what 1/sqrt(1 + 1e-30) lacks of 1.
    pk.check(pk.embbag_rmsnorm(x, weight, 1e-30, out=out, mx8=q))
    np.testing.assert_array_equal(host(out), sign[None] * w.reshape(1, -1).astype(np.float32).repeat(2, 0))
    codes, scales = ref.quantize8(host(out))
    np.testing.assert_array_equal(q.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)


def test_rows_beyond_the_range_of_fp32_squares():
    base = rows_of(1, 516, 3).double()
    x = torch.cat([base * 1e30, base * 1e-35, base * 1e-20, base * 0]).float()
    y, _, _ = ref.rmsnorm(host(x), 1.0, float(np.float32(1e-38)))
    out = torch.empty(4, 516, device=DEV)
    pk.check(pk.embbag_rmsnorm(x.to(DEV), None, 1e-38, out=out))
    close(out, y, (NORM_U + 1) * U * np.abs(y) + 1e-38)


def test_infinities_and_nan_stay_in_their_row():
    x = rows_of(6, 260, 5)
    x[1, 7], x[3, 259], x[4, 0] = float("inf"), float("nan"), -float("inf")
    y = torch.empty(6, 260, device=DEV)
    q = empty8(6, 260)
    pk.check(pk.embbag_rmsnorm(x.to(DEV), None, 1e-6, out=y, mx8=q))
    want, _, _ = ref.rmsnorm(host(x)[[0, 2, 5]], 1.0, 1e-6)
    close(y[[0, 2, 5]], want, NORM_U * U * np.abs(want))
    bad = torch.isnan(y)
    assert bad[1].sum() == 1 and bad[1, 7] and bad[3].all() and bad[4].sum() == 1 and bad[4, 0]
    assert (y[1][~bad[1]] == 0).all() and (y[4][~bad[4]] == 0).all()
    codes, scales = ref.quantize8(host(y))
    np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
    np.testing.assert_array_equal(q.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("dim", [36, 516, 4100])
def test_strides_and_in_place(dim):
    rows = 5
    x, r, w = rows_of(rows, dim, 1, "bf16"), rows_of(rows, dim, 2, "f32"), weight_of(dim, 3, "f32")
    want, wsum = torch.empty(rows, dim, dtype=DT["bf16"], device=DEV), torch.empty(rows, dim, device=DEV)
    pk.check(pk.embbag_rmsnorm(dev(x), dev(w), 1e-5, out=want, residual=dev(r), sum_out=wsum))
    xp, rp = padded(dev(x), 12, 4), padded(dev(r), 4, 8)
    junk_x, junk_r = xp._base.clone(), rp._base.clone()
    pk.check(pk.embbag_rmsnorm(xp, dev(w), 1e-5, out=xp, residual=rp, sum_out=rp))
    assert torch.equal(xp, want) and torch.equal(rp, wsum)
    for view, was in ((xp, junk_x), (rp, junk_r)):  # what lies between the rows stays
        now = view._base.clone()
        mask = torch.zeros_like(now, dtype=torch.bool)
        torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(True)
        assert torch.equal(now[~mask].view(torch.uint8), was[~mask].view(torch.uint8))


GRAD_U = 14  # see test_norm_gradients


@pytest.mark.parametrize("ty,th,tw,dsum", [("f32", "f32", "f32", False), ("bf16", "bf16", "bf16", True),
                                           ("bf16", "f32", "f32", True), ("f32", "bf16", None, False)])
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_norm_gradients(rows, dim, ty, th, tw, dsum):
    """Roundings: g = w dy 1; n 3.5 (1/rms 2.5, the product 1); mean(n g) 1 for g and 3.5 for the
    factor and its own rounding; n * mean 1 more; the difference 1; times 1/rms 3.5; the sum with dsum
    1: at most 12 of |g| and 14 of |n| mean|n g|."""
    seed = rows * 13 + dim
    h, dy, w = rows_of(rows, dim, seed, th), rows_of(rows, dim, seed + 1, ty), weight_of(dim, seed + 2, tw)
    d = rows_of(rows, dim, seed + 3, th) if dsum else None
    dh = torch.empty(rows, dim, dtype=DT[th], device=DEV)
    dw = torch.empty(dim, dtype=DT[tw or ty], device=DEV)
    ws = torch.empty(pk.embbag_rmsnorm_grad_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    run = lambda **k: pk.check(pk.embbag_rmsnorm_grad(dev(dy), dev(h), dev(w), 1e-6, dh, ws, dsum=dev(d), **k))
    run(dweight=dw)
    want, wdw, size, dwsize = ref.rmsnorm_grad(host(dy), host(h), 1.0 if w is None else host(w), 1e-6,
                                               0.0 if d is None else host(d))
    close(dh, want, GRAD_U * U * size + rounding(want, th), "dh")
    close(dw, wdw, (rows + 8) * U * dwsize + rounding(wdw, tw or ty), "dw")
    first = dh.clone()
    dh.zero_()
    run()
    assert torch.equal(dh, first)


def test_gradients_against_differences():
    rows, dim, eps = 3, 36, 1e-3
    rng = np.random.default_rng(9)
    h, dy, w = rng.normal(size=(rows, dim)), rng.normal(size=(rows, dim)), rng.normal(size=dim)
    f = lambda h, w: (ref.rmsnorm(h, w, eps)[0] * dy).sum()
    dh, dw = torch.empty(rows, dim, device=DEV), torch.empty(dim, device=DEV)
    t = lambda a: torch.from_numpy(a).float().to(DEV)
    ws = torch.empty(pk.embbag_rmsnorm_grad_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_rmsnorm_grad(t(dy), t(h), t(w), eps, dh, ws, dweight=dw))
    step = 1e-5
    for r, c in [(0, 0), (1, 17), (2, 35)]:
        e = np.zeros_like(h)
        e[r, c] = step
        assert abs((f(h + e, w) - f(h - e, w)) / (2 * step) - float(dh[r, c])) < 1e-5
        assert abs((f(h, w + e[r]) - f(h, w - e[r])) / (2 * step) - float(dw[c])) < 1e-5


def test_gradients_in_place_and_of_no_rows():
    rows, dim = 9, 132
    h, dy, d = (rows_of(rows, dim, i) for i in range(3))
    ws = torch.empty(pk.embbag_rmsnorm_grad_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    want = torch.empty(rows, dim, device=DEV)
    pk.check(pk.embbag_rmsnorm_grad(dev(dy), dev(h), None, 1e-6, want, ws, dsum=dev(d)))
    for name in ("dy", "h", "dsum"):
        t = {"dy": padded(dev(dy), 8), "h": padded(dev(h), 4), "dsum": padded(dev(d), 12)}
        pk.check(pk.embbag_rmsnorm_grad(t["dy"], t["h"], None, 1e-6, t[name], ws, dsum=t["dsum"]))
        assert torch.equal(t[name], want), name
    dw = torch.ones(dim, device=DEV)
    none = torch.empty(0, dim, device=DEV)
    pk.check(pk.embbag_rmsnorm_grad(none, none, None, 1e-6, none, ws, dweight=dw))
    assert (dw == 0).all()
    pk.check(pk.embbag_rmsnorm(none, None, 1e-6, out=none))
