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
