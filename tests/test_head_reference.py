"""The 64-bit reference of the output head against independent routines: torch in
float64, hand-worked values, and finite differences."""
import numpy as np
import pytest
import torch

import head_reference as ref


def test_codes_by_hand():
    # Largest magnitude 6: scale 1.  Ties go to the even code.
    x = np.array([[6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.0, -0.25, -0.75, -5.01, 0.26, 4.9,
                   -6.0, 0.5] + [0.0] * 16])
    codes, scales = ref.quantize(x)
    assert scales.tolist() == [[127, 0, 0, 0]]
    flat = [int(c) for b in codes[0] for c in (b & 15, b >> 4)]
    assert flat[:16] == [7, 0, 2, 2, 4, 4, 6, 6, 8, 8, 10, 15, 1, 6, 15, 1]


@pytest.mark.parametrize("top,byte,first", [
    (7.99, 127, 6.0), (8.0, 128, 8.0), (4.0, 127, 4.0), (3.99, 126, 3.0), (2.0 ** -125, 0, 2.0 ** -125),
    (2.0 ** -149, 0, 0.0), (0.0, 0, 0.0), (float(np.finfo(np.float32).max), 252, 6 * 2.0 ** 125)])
def test_scale_of_the_largest(top, byte, first):
    x = np.zeros((1, 32))
    x[0, 0] = top
    codes, scales = ref.quantize(x)
    assert scales[0, 0] == byte
    assert ref.dequantize(codes, scales, 32)[0, 0] == first


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_a_bad_block_reads_back_as_nan(bad):
    x = np.ones((1, 70))
    x[0, 40] = bad
    v = ref.dequantize(*ref.quantize(x), 70)
    assert np.isnan(v[0, 32:64]).all() and (v[0, :32] == 1).all() and (v[0, 64:] == 1).all()


def test_error_of_a_block_is_bounded():
    x = np.random.default_rng(0).normal(size=(20, 96))
    v = ref.dequantize(*ref.quantize(x), 96)
    top = np.abs(x).reshape(20, 3, 32).max(2).repeat(32, 1)
    assert (np.abs(v - x) <= top / 4).all()  # saturation: 8 -> 6 at the worst


def test_bf16_round_is_torchs():
    x = np.random.default_rng(1).normal(size=5000).astype(np.float32)
    want = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    assert np.array_equal(ref.bf16_round(x.astype(np.float64)), want)


@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_distill_is_torchs_kl_and_its_gradient(temperature):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(5, 37, generator=g, dtype=torch.float64, requires_grad=True)
    ids = torch.stack([torch.randperm(37, generator=g)[:6] for _ in range(5)])
    t = torch.randn(5, 6, generator=g, dtype=torch.float64)
    w = torch.tensor([0.5, 1.0, 0.0, 2.0, 1.0], dtype=torch.float64)
    logq = torch.log_softmax(x / temperature, 1).gather(1, ids)
    kl = torch.nn.functional.kl_div(logq, torch.softmax(t / temperature, 1), reduction="none").sum(1)
    loss = w * temperature ** 2 * kl
    loss.sum().backward()
    got, grad, _, _ = ref.distill(x.detach().numpy(), ids.numpy(), t.numpy(), temperature, w.numpy())
    assert np.allclose(got, loss.detach().numpy(), rtol=1e-12, atol=1e-13)
    assert np.allclose(grad, x.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_distill_gradient_by_differences_with_a_repeated_id():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(2, 9))
    ids = np.array([[1, 4, 1, -1], [0, 8, 3, 2]])
    t = rng.normal(size=(2, 4))
    _, grad, _, _ = ref.distill(x, ids, t, 1.7)
    for r in range(2):
        for v in range(9):
            step = np.zeros_like(x)
            step[r, v] = 1e-6
            d = (ref.distill(x + step, ids, t, 1.7)[0][r] - ref.distill(x - step, ids, t, 1.7)[0][r]) / 2e-6
            assert abs(d - grad[r, v]) < 1e-8


def test_distill_rows_left_out():
    x = np.random.default_rng(5).normal(size=(4, 7))
    x[3] = -np.inf
    ids = np.array([[1, 2], [-1, -1], [3, 4], [0, 1]])
    t = np.array([[0.0, 1.0], [0.0, 1.0], [-np.inf, -np.inf], [0.0, 1.0]])
    loss, grad, _, _ = ref.distill(x, ids, t, 1.0, [0.0, 1.0, 1.0, 1.0])
    assert not loss.any() and not grad.any()


def test_logits_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.0, 5.0]])
    y, _ = ref.logits(x, seen=[[0, 1, 2, 2, 3]], prompt_lens=[1], repetition=[2.0], frequency=[0.25],
                      presence=[0.5], bias=[[(4, 1.0), (4, -3.0)]], masks=[[0b10111]])
    assert y.tolist() == [[1.0, -4.75, 0.5 - 1.0, -np.inf, 2.0]]
