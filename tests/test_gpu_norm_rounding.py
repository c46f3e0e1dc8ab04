"""RMS norm's outputs are the 64-bit values rounded once to FP32, and BF16 and 8-bit rows are rounded from that; the
gradient goes by the row that it is given."""
import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
import train_reference as ref
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, rounding
from test_gpu_norm import GRAD_U, dev, empty8, host, rows_of, weight_of

pytestmark = pytest.mark.gpu

# Half a step of FP32; 1/sqrt is right to 2^-46 before (FP32's 2^-24 squared, a Newton step), FP64 sums and the
# reference to some 2^-43.
ONCE = U * (1 + 2.0 ** -16)


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


SHAPES = [(3, 28), (7, 132), (40, 512), (30, 1028), (64, 4096), (9, 8196), (4, 16384), (5000, 64)]


@pytest.mark.parametrize("tr", [None, "f32"])
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_one_rounding(rows, dim, tr):
    seed = rows * 5 + dim
    x, w = rows_of(rows, dim, seed), weight_of(dim, seed + 1, "f32")
    r = None if tr is None else rows_of(rows, dim, seed + 2, tr)
    h = host(x) if r is None else host(x) + host(r)
    out, wide = torch.empty(rows, dim, device=DEV), torch.empty(rows, dim, device=DEV, dtype=torch.bfloat16)
    pk.check(pk.embbag_rmsnorm(dev(x), dev(w), 1e-6, out=out, residual=dev(r)))
    y, _, _ = ref.rmsnorm(h, host(w), float(np.float32(1e-6)))
    close(out, y, ONCE * np.abs(y), "out")
    pk.check(pk.embbag_rmsnorm(dev(x), dev(w), 1e-6, out=wide, residual=dev(r)))
    assert torch.equal(wide, out.bfloat16())


@pytest.mark.parametrize("rows,dim", SHAPES)
def test_codes_are_those_of_the_exact_norm_but_next_to_a_midpoint(rows, dim):
    seed = rows + dim * 3
    x, w = rows_of(rows, dim, seed), weight_of(dim, seed + 1, "f32")
    q = empty8(rows, dim)
    pk.check(pk.embbag_rmsnorm(dev(x), dev(w), 1e-6, mx8=q))
    y, _, _ = ref.rmsnorm(host(x), host(w), float(np.float32(1e-6)))
    codes, scales = ref.quantize8(y)
    got, got_scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    nb = -(-dim // 32)
    full = np.zeros((rows, nb * 32))
    full[:, :dim] = np.abs(y)
    blocks = full.reshape(rows, nb, 32)
    # A scale may be another's only where its largest element is within the rounding of 448 times a power of two.
    ratio = blocks.max(2) / (448.0 * 2.0 ** (scales[:, :nb].astype(np.float64) - 127))
    edge = (np.abs(ratio - 1) <= 2 * ONCE) | (np.abs(ratio - 0.5) <= 2 * ONCE)
    assert ((scales == got_scales)[:, :nb] | edge).all() and (got_scales[:, nb:] == 0).all()
    a = (blocks * 2.0 ** (127 - scales[:, :nb].astype(np.float64))[:, :, None]).reshape(rows, -1)
    mid = (ref.E4M3[1:127] + ref.E4M3[:126]) / 2
    i = np.searchsorted(mid, a).clip(0, mid.size - 1)
    near = np.minimum(np.abs(a - mid[i]), np.abs(a - mid[np.maximum(i - 1, 0)])) <= ONCE * a
    same = codes[:, :nb * 32] == got[:, :nb * 32]
    assert (same | near | np.repeat(edge, 32, 1)).all()
    assert (got[:, nb * 32:] == 0).all()


@pytest.mark.parametrize("rows,dim", [(3, 36), (17, 516), (4, 4100), (300, 64)])
def test_forward_and_back_over_a_bf16_stream(rows, dim):
    """The gradient is that of the norm of the row it is given: exactly so of a BF16 sum_out, which is the forward's row
    with each element off by half a step of BF16, d = 2^-8 of itself.  Beside the forward's own row: 1/rms is off by d (of
    its size), n by 2 d, so mean(n g) by 2 d of mean|n g|, n * mean by 4 d, and the whole, times 1/rms, by 5 d;
    dweight by 2 d of the sum of |dy n|.  (Squares of d: another d in all.)"""
    seed = rows + dim
    x, r, w = rows_of(rows, dim, seed, "bf16"), rows_of(rows, dim, seed + 1, "bf16"), weight_of(dim, seed + 2, "f32")
    dy = rows_of(rows, dim, seed + 3, "bf16")
    out, s = (torch.empty(rows, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pk.check(pk.embbag_rmsnorm(dev(x), dev(w), 1e-6, out=out, residual=dev(r), sum_out=s))
    assert torch.equal(s, (dev(x).float() + dev(r).float()).bfloat16())
    dh, dw = torch.empty_like(s), torch.empty(dim, device=DEV)
    ws = torch.empty(pk.embbag_rmsnorm_grad_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_rmsnorm_grad(dev(dy), s, dev(w), 1e-6, dh, ws, dweight=dw))
    want, wdw, size, dwsize = ref.rmsnorm_grad(host(dy), host(s), host(w), 1e-6)
    close(dh, want, GRAD_U * U * size + rounding(want, "bf16"), "dh of the rounded row")
    close(dw, wdw, (rows + 8) * U * dwsize + rounding(wdw, "f32"), "dw of the rounded row")
    d = 2.0 ** -8
    want, wdw, size, dwsize = ref.rmsnorm_grad(host(dy), host(x) + host(r), host(w), 1e-6)
    tol = (GRAD_U * U + 6 * d) * size
    close(dh, want, tol + rounding(np.abs(want) + tol, "bf16"), "dh")
    close(dw, wdw, ((rows + 8) * U + 3 * d) * dwsize, "dw")
