"""4-bit microscaled tables on the GPU against the 64-bit reference: codes and
scales byte for byte, values exactly, pooled bags, scores and their gradient within
bounds derived from the number of FP32 additions."""
import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a unit in the last place of FP32, relative
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def rounding(y, type_):
    """Error of storing y: FP32 half a unit, BF16 2^-9 of it (and subnormals)."""
    return np.abs(y) * (2.0 ** -8 if type_ == "bf16" else U) + 1e-38


def close(got, want, tol, what=""):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= tol)
    if not ok.all():
        i = tuple(np.argwhere(~ok)[0])
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.size} off; first at {i}: got "
                             f"{got[i]!r}, want {want[i]!r}, allowed {np.broadcast_to(tol, want.shape)[i]!r}")


def source(rows, dim, seed, type_="f32", special=True):
    """Values of many magnitudes, ties, zeros, infinities and NaN, exact in `type_`."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, dim)) * np.exp2(rng.integers(-20, 20, size=(rows, dim // 4 + 1)).repeat(4, 1)[:, :dim])
    ties = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0], size=x.shape)
    x = np.where(rng.random(x.shape) < 0.3, ties * rng.choice([-1, 1], size=x.shape), x)
    if special:
        flat = x.reshape(-1)
        for i, v in enumerate([np.nan, np.inf, -np.inf, 1e-45, -1e-40, 3.4e38, 2.0 ** -127, 1e-38]):
            flat[(i * 97 + seed) % flat.size] = v
        if rows > 2:
            x[1] = 0.0
            x[2] = -1e-44
    t = torch.from_numpy(x).float().to(DT[type_])
    return t


def padded(t, extra, offset=0):
    """The same rows, `extra` elements apart, in a buffer of junk."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + extra) + offset,), float("nan"), dtype=t.dtype, device=DEV)
    v = buf[offset:].view(rows, cols + extra)[:, :cols]
    v.copy_(t)
    return v


def random_table(rows, dim, seed, spread=4):
    """A table of random codes and scales around 1 (padding as the format has it)."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, dim)) * np.exp2(rng.integers(-spread, spread + 1, size=(rows, 1)))
    codes, scales = ref.quantize(x)
    t = pk.Mx4Table(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), dim)
    return t, ref.dequantize(codes, scales, dim)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim", [(1, 4), (3, 28), (5, 32), (7, 36), (4, 64), (9, 100), (3, 256),
                                      (2, 1024), (33, 132), (1, 4100)])
def test_quantize_is_the_definition(rows, dim, type_):
    x = source(rows, dim, rows * 1000 + dim, type_)
    codes, scales = ref.quantize(x.double().numpy())
    t = pk.Mx4Table(torch.full((rows, pk.mx4_code_bytes(dim)), 0xA5, dtype=torch.uint8, device=DEV),
                    torch.full((rows, pk.mx4_scale_bytes(dim)), 0x5A, dtype=torch.uint8, device=DEV), dim)
    pk.check(pk.embbag_mx4_quantize(padded(x, 8), t))
    assert np.array_equal(t.scales.cpu().numpy(), scales)
    assert np.array_equal(t.codes.cpu().numpy(), codes)
    want = ref.dequantize(codes, scales, dim)
    for back in DT:
        out = padded(torch.zeros(rows, dim, dtype=DT[back]), 4)
        pk.check(pk.embbag_mx4_dequantize(t, out))
        close(out, want, 0.0, back)


def test_every_byte_and_scale_reads_back():
    codes = torch.arange(256, dtype=torch.uint8).repeat_interleave(16).view(256, 16)
    for first in range(0, 256, 64):
        c = codes.repeat(64, 1)
        s = torch.zeros(256 * 64, 4, dtype=torch.uint8)
        s[:, 0] = torch.arange(first, first + 64, dtype=torch.uint8).repeat_interleave(256)
        t = pk.Mx4Table(c.to(DEV), s.to(DEV), 32)
        out = torch.empty(256 * 64, 32, device=DEV)
        pk.check(pk.embbag_mx4_dequantize(t, out))
        with np.errstate(over="ignore"):  # 2^127 * 4 and 6 are infinite in FP32
            want = ref.dequantize(c.numpy(), s.numpy(), 32).astype(np.float32).astype(np.float64)
        close(out, want, 0.0)


def test_quantize_listed_rows_only():
    x = source(50, 100, 5, special=False).to(DEV)
    t = pk.Mx4Table.empty(50, 100)
    t.codes.fill_(0x11)
    t.scales.fill_(0x77)
    ids = torch.tensor([3, 49, 3, 0, 17, 17], dtype=torch.int32, device=DEV)
    st = status()
    pk.check(pk.embbag_mx4_quantize(x, t, row_ids=ids, d_status=st))
    pk.check(pk.embbag_status_read(st))
    codes, scales = ref.quantize(x.double().cpu().numpy())
    named = np.zeros(50, bool)
    named[ids.cpu().numpy()] = True
    assert np.array_equal(t.codes.cpu().numpy(), np.where(named[:, None], codes, 0x11))
    assert np.array_equal(t.scales.cpu().numpy(), np.where(named[:, None], scales, 0x77))
    pk.check(pk.embbag_mx4_quantize(x, t, row_ids=ids[:0], d_status=st))


@pytest.mark.parametrize("bad", [-1, 50, 2 ** 31 - 1])
def test_quantize_reports_a_bad_row(bad):
    x = source(50, 32, 6, special=False).to(DEV)
    t = pk.Mx4Table.empty(50, 32)
    st = status()
    ids = torch.tensor([1, bad, 2], dtype=torch.int32, device=DEV)
    pk.check(pk.embbag_mx4_quantize(x, t, row_ids=ids, d_status=st))
    assert pk.embbag_status_read(st) == pk.EMBBAG_ERR_INDEX_RANGE
    assert int((t.scales != 0).any(1).sum()) == 2


def bags_of(rng, T, rows, batch, longest, empty=0.2):
    n = rng.integers(1, longest + 1, size=T * batch)
    n[rng.random(T * batch) < empty] = 0
    o = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    return o, rng.integers(0, rows, size=o[-1]).astype(np.int32)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pooling", ["sum", "weighted", "mean"])
@pytest.mark.parametrize("T,rows,dim,batch,longest", [
    (1, 1, 4, 1, 1), (3, 40, 16, 7, 5), (2, 100, 32, 33, 3), (4, 50, 64, 20, 40), (2, 30, 100, 9, 17),
    (2, 60, 128, 65, 9), (1, 200, 256, 3, 300), (2, 40, 260, 5, 8), (1, 30, 512, 6, 70),
    (2, 20, 516, 4, 6), (1, 25, 1024, 5, 33)])
def test_pooled_forward(T, rows, dim, batch, longest, pooling, out):
    rng = np.random.default_rng(T * 7 + dim + batch)
    o, idx = bags_of(rng, T, rows, batch, longest)
    made = [random_table(rows, dim, 100 * t + dim) for t in range(T)]
    weights = rng.normal(size=idx.size).astype(np.float32) if pooling == "weighted" else None
    want, mag = ref.pooled([v for _, v in made], batch, idx, o, weights, pooling == "mean")
    y = torch.full((T, batch, dim), float("nan"), dtype=DT[out], device=DEV)
    st = status()
    pk.check(pk.embbag_mx4_forward(
        pk.Mx4Tables([t for t, _ in made]), batch, torch.from_numpy(idx).to(DEV),
        torch.from_numpy(o).to(DEV), y, None if weights is None else torch.from_numpy(weights).to(DEV),
        pk.EMBBAG_POOL_MEAN if pooling == "mean" else pk.EMBBAG_POOL_SUM, st))
    pk.check(pk.embbag_status_read(st))
    tol = (longest + 2) * U * mag * 1.01
    close(y, want, tol + rounding(np.abs(want) + tol, out))
    empty = (np.diff(o) == 0).reshape(T, batch)
    assert not y.cpu().view(torch.int16 if out == "bf16" else torch.int32).numpy()[empty].any()


@pytest.mark.parametrize("pooling", ["sum", "mean", "weighted"])
def test_pooled_forward_of_every_scale_and_code(pooling):
    # Row r: all codes twice, scale byte r.  A bag of one row is the row (a sum of one term).
    t = pk.Mx4Table.empty(256, 32, torch.device(DEV))
    code = np.tile(np.arange(16), 2)
    t.codes[:] = torch.from_numpy((code[::2] | code[1::2] << 4).astype(np.uint8)).to(DEV)
    t.scales.zero_()
    t.scales[:, 0] = torch.arange(256, device=DEV).to(torch.uint8)
    want = torch.empty(256, 32, device=DEV)
    pk.check(pk.embbag_mx4_dequantize(t, want))
    y = torch.empty(1, 256, 32, device=DEV)
    idx = torch.arange(256, dtype=torch.int32, device=DEV)
    o = torch.arange(257, dtype=torch.int32, device=DEV)
    pk.check(pk.embbag_mx4_forward(
        pk.Mx4Tables([t]), 256, idx, o, y,
        torch.ones(256, device=DEV) if pooling == "weighted" else None,
        pk.EMBBAG_POOL_MEAN if pooling == "mean" else pk.EMBBAG_POOL_SUM))
    assert torch.equal(torch.isnan(y[0]), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(y[0]), torch.nan_to_num(want))


@pytest.mark.parametrize("dim", [4, 32, 36, 256, 1024])
def test_pooled_forward_of_lists_of_any_length_in_one_wavefront(dim):
    # Lengths next to each other from none to long: the products of all bags of a wavefront go on
    # until its longest list ends.
    lengths = np.array([0, 1, 2, 3, 700, 0, 5, 8, 9, 16, 17, 33, 0, 64, 1, 129] * 5, np.int64)
    o = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    idx = np.random.default_rng(dim).integers(0, 500, o[-1]).astype(np.int32)
    t, v = random_table(500, dim, dim)
    want, mag = ref.pooled([v], lengths.size, idx, o)
    y = torch.full((1, lengths.size, dim), float("nan"), device=DEV)
    st = status()
    pk.check(pk.embbag_mx4_forward(pk.Mx4Tables([t]), lengths.size, torch.from_numpy(idx).to(DEV),
                                   torch.from_numpy(o).to(DEV), y, d_status=st))
    pk.check(pk.embbag_status_read(st))
    close(y, want, (700 + 2) * U * mag * 1.01)
    assert not y[0].cpu().view(torch.int32).numpy()[lengths == 0].any()


def test_pooled_forward_reports_bad_lists():
    t, _ = random_table(10, 32, 1)
    tb = pk.Mx4Tables([t, t])
    y = torch.zeros(2, 2, 32, device=DEV)
    good = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device=DEV)
    for idx, o, code in [([0, 1, 10, 2], [0, 1, 2, 3, 4], pk.EMBBAG_ERR_INDEX_RANGE),
                         ([0, -1, 1, 2], [0, 1, 2, 3, 4], pk.EMBBAG_ERR_INDEX_RANGE),
                         ([0, 1, 2, 3], [0, 3, 2, 3, 4], pk.EMBBAG_ERR_OFFSETS),
                         ([0, 1, 2, 3], [1, 1, 2, 3, 4], pk.EMBBAG_ERR_OFFSETS),
                         ([0, 1, 2, 3], [0, 1, 2, 3, 3], pk.EMBBAG_ERR_OFFSETS),
                         ([0, 1, 2, 3], [0, 1, 2, 9, 4], pk.EMBBAG_ERR_OFFSETS),
                         ([0, 1, 2, 3], [0, -5, 2, 3, 4], pk.EMBBAG_ERR_OFFSETS)]:
        st = status()
        pk.check(pk.embbag_mx4_forward(tb, 2, torch.tensor(idx, dtype=torch.int32, device=DEV),
                                       torch.tensor(o, dtype=torch.int32, device=DEV), y, d_status=st))
        assert pk.embbag_status_read(st) == code, (idx, o)
    st = status()
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    pk.check(pk.embbag_mx4_forward(tb, 0, none, good[:1], y[:, :0], d_status=st))
    assert pk.embbag_status_read(st) == 0


def test_a_nan_block_stays_in_its_bags_and_columns():
    t, v = random_table(8, 64, 3)
    t.scales[5, 1] = 255
    v[5, 32:] = np.nan
    idx, o = np.array([1, 5, 2, 3, 5, 0], np.int32), np.array([0, 2, 2, 4, 6], np.int32)
    want, _ = ref.pooled([v], 4, idx, o)
    y = torch.empty(1, 4, 64, device=DEV)
    pk.check(pk.embbag_mx4_forward(pk.Mx4Tables([t]), 4, torch.from_numpy(idx).to(DEV),
                                   torch.from_numpy(o).to(DEV), y))
    close(y, want, 1e-4)


# ---- scores -------------------------------------------------------------------
def scores_check(m, n, k, x_type, out_type, seed, pad=0, special=False):
    t, w = random_table(n, k, seed)
    x = source(m, k, seed + 1, x_type, special=special)
    if not special:
        x = (x.double() / x.double().abs().max(1, keepdim=True).values.clamp(min=1e-30)).to(x.dtype)
    q = ref.dequantize(*ref.quantize(x.double().numpy()), k)
    with np.errstate(invalid="ignore"):
        want = q @ w.T
        tol = 2 * (k + 8) * U * (np.abs(q) @ np.abs(w).T)
    xs = padded(x, 4 * pad)
    out = padded(torch.zeros(m, n, dtype=DT[out_type]), pad, offset=pad % 2)
    ws = torch.empty(pk.embbag_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    before = None if pad == 0 else out._base.clone()
    pk.check(pk.embbag_mx4_matmul(xs, t, out, ws))
    close(out, want, tol + rounding(np.abs(want) + tol, out_type), f"{m}x{n}x{k}")
    if pad:  # nothing between the rows is written
        gaps = out._base[pad % 2:].view(m, n + pad)[:, n:]
        assert torch.isnan(gaps).all() and torch.isnan(before[pad % 2:].view(m, n + pad)[:, n:]).all()


SCORES = [(1, 1, 4), (1, 300, 64), (2, 17, 100), (3, 1000, 256), (16, 129, 512), (17, 257, 36),
          (31, 64, 1024), (33, 500, 132), (64, 300, 260), (100, 100, 96), (128, 777, 516),
          (129, 260, 1028), (200, 1030, 320), (257, 513, 64), (5, 90, 4096), (300, 40, 2052)]


@pytest.mark.parametrize("x_type,out_type", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                             ("f32", "bf16")])
@pytest.mark.parametrize("m,n,k", SCORES)
def test_scores(m, n, k, x_type, out_type):
    scores_check(m, n, k, x_type, out_type, m + 3 * n + 5 * k)


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("m,n,k", [(1, 100, 128), (40, 301, 160), (150, 260, 512)])
def test_scores_with_strides(m, n, k, pad):
    scores_check(m, n, k, "bf16", "bf16", 7, pad)
    scores_check(m, n, k, "f32", "f32", 8, pad)


@pytest.mark.parametrize("m", [1, 20, 140])
def test_scores_of_rows_with_infinities_and_nan(m):
    """A bad block of x makes its row NaN and no other."""
    scores_check(m, 150, 192, "f32", "f32", 9, special=True)


@pytest.mark.parametrize("m", [1, 30, 150])
def test_a_nan_block_of_the_table_stays_in_its_column(m):
    t, w = random_table(200, 160, 11)
    t.scales[150, 4] = 255
    x = torch.randn(m, 160, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    out = torch.empty(m, 200, device=DEV)
    ws = torch.empty(pk.embbag_mx4_matmul_workspace_bytes(m, 200, 160), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul(x, t, out, ws))
    bad = torch.isnan(out)
    assert bad[:, 150].all() and int(bad.sum()) == m


def test_scores_of_no_rows():
    t, _ = random_table(10, 32, 12)
    x, out = torch.empty(0, 32, device=DEV), torch.empty(0, 10, device=DEV)
    ws = torch.empty(max(256, pk.embbag_mx4_matmul_workspace_bytes(0, 10, 32)), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul(x, t, out, ws))
    ws = torch.empty(max(256, pk.embbag_mx4_matmul_grad_workspace_bytes(0, 10, 32)), dtype=torch.uint8,
                     device=DEV)
    pk.check(pk.embbag_mx4_matmul_grad(out, t, x, ws))


def coded_table(rows, dim, seed):
    """A large table of random codes and scales around 1, E a multiple of 4."""
    rng = np.random.default_rng(seed)
    nb = (dim + 31) // 32
    pair = rng.integers(0, 256, (rows, nb * 16), np.uint8)
    pair[:, dim // 2:] = 0
    scales = np.zeros((rows, (nb + 3) // 4 * 4), np.uint8)
    scales[:, :nb] = rng.integers(124, 131, (rows, nb), np.uint8)
    value = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    value = np.concatenate([value, -value])
    both = value[np.arange(256)[:, None] >> np.array([0, 4]) & 15]
    w = both[pair].reshape(rows, nb, 32) * np.exp2(scales[:, :nb, None] - 127.0)
    t = pk.Mx4Table(torch.from_numpy(pair).to(DEV), torch.from_numpy(scales).to(DEV), dim)
    return t, w.reshape(rows, nb * 32)[:, :dim]


def some_rows(m):
    """The first and last rows of tiles of 64, 128 and 256 of m rows, and some between."""
    at = {0, 1, 31, 32, 63, 64, 127, 128, 255, 256, 300, m // 2, m - 2, m - 1}
    return sorted(r for r in at if r < m)


@pytest.mark.parametrize("m,n,k,out_type", [(600, 5000, 260, "bf16"), (1100, 20003, 1000, "f32"),
                                            (2048, 20000, 512, "bf16")])
def test_scores_of_many_rows(m, n, k, out_type):
    t, w = coded_table(n, k, n)
    x = source(m, k, m, "bf16", special=False)
    x = (x.double() / x.double().abs().max(1, keepdim=True).values.clamp(min=1e-30)).to(x.dtype)
    out = torch.empty(m, n, dtype=DT[out_type], device=DEV)
    ws = torch.empty(pk.embbag_mx4_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul(x.to(DEV), t, out, ws))
    rows = some_rows(m)
    q = ref.dequantize(*ref.quantize(x[rows].double().numpy()), k)
    want = q @ w.T
    tol = 2 * (k + 8) * U * (np.abs(q) @ np.abs(w).T)
    close(out[rows], want, tol + rounding(np.abs(want) + tol, out_type), f"{m}x{n}x{k}")


# ---- gradient -----------------------------------------------------------------
def grad_check(m, n, k, y_type, x_type, seed, pad=0):
    t, w = random_table(n, k, seed)
    rng = np.random.default_rng(seed)
    dy = torch.from_numpy(rng.normal(size=(m, n)) * np.exp(2 * rng.normal(size=(m, n)))).to(DT[y_type])
    d = dy.double().numpy()
    want = d @ w
    tol = 2 * (n + 8) * U * (np.abs(d) @ np.abs(w))
    dx = padded(torch.zeros(m, k, dtype=DT[x_type]), 4 * pad)
    ws = torch.empty(pk.embbag_mx4_matmul_grad_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    pk.check(pk.embbag_mx4_matmul_grad(padded(dy, pad, offset=pad % 2), t, dx, ws))
    close(dx, want, tol + rounding(np.abs(want) + tol, x_type), f"{m}x{n}x{k}")


@pytest.mark.parametrize("y_type,x_type", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                           ("f32", "bf16")])
@pytest.mark.parametrize("m,n,k", SCORES)
def test_gradient(m, n, k, y_type, x_type):
    grad_check(m, n, k, y_type, x_type, m + 3 * n + 5 * k)


@pytest.mark.parametrize("y_type", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 63, 64, 65, 257, 259, 511, 519, 16385, 16390])
@pytest.mark.parametrize("m", [1, 70])
def test_gradient_ends_of_the_rows(m, n, y_type):
    """Last steps and last splits of a few rows; the buffer ends with dy's last element."""
    grad_check(m, n, 132, y_type, "f32", n)


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("m,n,k", [(1, 100, 128), (40, 301, 160), (150, 260, 512)])
def test_gradient_with_strides(m, n, k, pad):
    grad_check(m, n, k, "bf16", "bf16", 7, pad)
    grad_check(m, n, k, "f32", "f32", 8, pad)


@pytest.mark.parametrize("m,n,k,y_type,x_type", [
    (700, 16390, 700, "bf16", "bf16"), (900, 8195, 1020, "f32", "f32"), (1500, 50001, 100, "bf16", "f32"),
    (4300, 7001, 1004, "bf16", "f32"), (2100, 15003, 1000, "f32", "bf16"),
    (4000, 70000, 128, "bf16", "bf16")])
def test_gradient_of_many_rows(m, n, k, y_type, x_type):
    t, w = coded_table(n, k, n)
    dy = torch.randn(m, n, generator=torch.Generator().manual_seed(m)).to(DT[y_type])
    dx = torch.empty(m, k, dtype=DT[x_type], device=DEV)
    ws = torch.empty(pk.embbag_mx4_matmul_grad_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    pk.check(pk.embbag_mx4_matmul_grad(dy.to(DEV), t, dx, ws))
    rows = some_rows(m)
    d = dy[rows].double().numpy()
    want = d @ w
    tol = 2 * (n + 8) * U * (np.abs(d) @ np.abs(w))
    close(dx[rows], want, tol + rounding(np.abs(want) + tol, x_type), f"{m}x{n}x{k}")


@pytest.mark.parametrize("y_type", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 40, 150])
def test_gradient_rows_with_infinities_and_nan(m, y_type):
    """A row of dy with an infinity or a NaN gives infinities or NaN in its own row alone."""
    t, w = random_table(300, 64, 21)
    dy = torch.randn(m, 300, generator=torch.Generator().manual_seed(2)).to(DT[y_type])
    dy[m - 1, 299] = float("inf")
    if m > 2:
        dy[1, 7] = float("nan")
    dx = torch.empty(m, 64, device=DEV)
    ws = torch.empty(pk.embbag_mx4_matmul_grad_workspace_bytes(m, 300, 64), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul_grad(dy.to(DEV), t, dx, ws))
    bad = ~torch.isfinite(dx)
    rows = {m - 1} | ({1} if m > 2 else set())
    assert bad[m - 1][torch.from_numpy(w[299] != 0).to(DEV)].all()
    assert set(bad.any(1).nonzero().view(-1).tolist()) == rows
    if m > 2:
        assert torch.isnan(dx[1]).all()


def test_gradient_against_differences_of_the_scores():
    """Straight through the rounding of x: on rows of x that are already codes, where a step
    leads to codes again, the difference of the scores is the gradient's step."""
    t, w = random_table(60, 32, 31)
    grid = np.array(ref.GRID)
    rng = np.random.default_rng(0)
    x = rng.choice(grid[:7], size=(6, 32)) * rng.choice([-1.0, 1.0], size=(6, 32))
    x[:, 0] = 6.0  # the blocks' scale is 1 before and after the step
    dy = rng.normal(size=(6, 60)).astype(np.float32)

    def scores(v):
        out = torch.empty(6, 60, device=DEV)
        ws = torch.empty(pk.embbag_mx4_matmul_workspace_bytes(6, 60, 32), dtype=torch.uint8, device=DEV)
        pk.check(pk.embbag_mx4_matmul(torch.from_numpy(v).float().to(DEV), t, out, ws))
        return out.double().cpu().numpy()

    dx = torch.empty(6, 32, device=DEV)
    ws = torch.empty(pk.embbag_mx4_matmul_grad_workspace_bytes(6, 60, 32), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_mx4_matmul_grad(torch.from_numpy(dy).to(DEV), t, dx, ws))
    base = scores(x)
    for e in range(1, 32):
        y = x.copy()
        up = np.array([grid[list(grid).index(abs(v)) + 1] for v in x[:, e]])
        y[:, e] = np.where(x[:, e] < 0, -up, up)
        step = y[:, e] - x[:, e]
        diff = ((scores(y) - base) * dy).sum(1)
        want = dx.double().cpu().numpy()[:, e] * step
        scale = (np.abs(dy) * (np.abs(base) + np.abs(w[:, e]) * 6 + 32 * 6)).sum(1)
        assert (np.abs(diff - want) <= 200 * U * scale + 60 * U * np.abs(want)).all()
