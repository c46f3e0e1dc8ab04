"""Penalties, biases and masks on the GPU against the 64-bit reference."""
import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import DT, U, close, padded, rounding, status

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV) if dtype is None else \
        torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def bags(rng, rows, vocab, longest):
    n = rng.integers(0, longest + 1, size=rows)
    n[rng.integers(rows)] = longest
    if rows > 1:
        n[0] = 0
    o = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    hot = rng.integers(0, vocab, size=max(1, longest // 4))
    return o, rng.choice(hot, size=o[-1]).astype(np.int32) if o[-1] else np.zeros(0, np.int32)


def case(rows, vocab, longest, biases, masks, type_, seed, special=True):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(size=(rows, vocab)) * 4).to(DT[type_])
    if special and vocab > 20:
        for i, v in enumerate([np.nan, np.inf, -np.inf, -3e38, 0.0, -0.0]):
            x[rng.integers(rows), rng.integers(vocab)] = v
    kw, want = {}, {}
    if longest:
        o, s = bags(rng, rows, vocab, longest)
        plen = rng.integers(0, longest + 3, size=rows).astype(np.int32)
        rho = (1 + rng.random(rows)).astype(np.float32)
        f, p = rng.random(rows).astype(np.float32), rng.random(rows).astype(np.float32)
        kw.update(seen=dev(s), seen_offsets=dev(o), prompt_lens=dev(plen), repetition=dev(rho),
                  frequency=dev(f), presence=dev(p))
        want.update(seen=[s[o[r]:o[r + 1]].tolist() for r in range(rows)], prompt_lens=plen,
                    repetition=rho, frequency=f, presence=p)
    if biases:
        o, ids = bags(rng, rows, vocab, biases)
        b = rng.normal(size=ids.size).astype(np.float32) * 5
        if b.size:
            b[rng.integers(b.size)] = -np.inf
        kw.update(bias_ids=dev(ids), bias_offsets=dev(o), biases=dev(b))
        want["bias"] = [list(zip(ids[o[r]:o[r + 1]].tolist(), b[o[r]:o[r + 1]].tolist()))
                        for r in range(rows)]
    if masks:
        words = -(-vocab // 32) + (masks % 2)  # rows of words longer than the vocabulary
        m = rng.integers(0, 2 ** 32, size=(masks, words), dtype=np.uint64).astype(np.uint32)
        m[0] = 0
        ids = rng.integers(-1, masks, size=rows).astype(np.int32)
        ids[rows - 1] = 0  # a row that is left nothing
        kw.update(masks=dev(m.view(np.int32)), mask_ids=dev(ids))
        want.update(masks=m, mask_ids=ids)
    return x, kw, want


def check(x, kw, want, type_, out=None, xs=None):
    y, mag = ref.logits(x.double().numpy(), **want)
    xs = x.to(DEV) if xs is None else xs
    out = torch.empty_like(xs) if out is None else out
    st = status()
    pk.check(pk.embbag_logits_process(xs, out, d_status=st, **kw))
    pk.check(pk.embbag_status_read(st))
    with np.errstate(invalid="ignore"):
        tol = 4 * U * np.where(np.isfinite(mag), mag, 0)
        tol = tol + np.where(mag > 0, rounding(np.where(np.isfinite(y), np.abs(y), 0) + tol, type_), 0)
    close(out, y, tol)
    return y


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,longest,biases,masks", [
    (1, 1, 1, 1, 1), (2, 7, 5, 3, 2), (3, 31, 0, 0, 3), (4, 33, 12, 0, 0), (5, 100, 0, 9, 0),
    (3, 1000, 50, 10, 4), (2, 4095, 300, 20, 1), (2, 4097, 300, 20, 2), (1, 8200, 2000, 40, 3),
    (7, 9001, 100, 200, 5), (2, 20000, 0, 0, 0), (1, 40001, 5000, 0, 2)])
def test_logits(rows, vocab, longest, biases, masks, type_):
    check(*case(rows, vocab, longest, biases, masks, type_, rows + vocab), type_)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset,out_pad,out_offset", [
    (1, 0, 1, 0), (3, 1, 3, 1), (0, 2, 5, 2), (8, 0, 0, 0), (1, 0, 2, 1), (7, 3, 7, 4)])
def test_logits_rows_of_any_alignment(pad, offset, out_pad, out_offset, type_):
    x, kw, want = case(4, 5003, 200, 30, 3, type_, pad + 10 * offset)
    out = padded(torch.zeros_like(x), out_pad, out_offset)
    check(x, kw, want, type_, out, padded(x, pad, offset))
    gaps = out._base[out_offset:].view(4, 5003 + out_pad)[:, 5003:]
    assert torch.isnan(gaps).all()


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1])
def test_logits_in_place(offset, type_):
    x, kw, want = case(5, 6001, 200, 30, 3, type_, 77)
    xs = padded(x, 5, offset)
    check(x, kw, want, type_, xs, xs)


def test_parts_left_out():
    """Lists without factors change nothing; a mask per row needs no mask_ids."""
    x, kw, want = case(3, 500, 40, 0, 0, "f32", 5, special=False)
    y = torch.empty(3, 500, device=DEV)
    pk.check(pk.embbag_logits_process(x.to(DEV), y, seen=kw["seen"], seen_offsets=kw["seen_offsets"]))
    assert torch.equal(y.cpu(), x)
    for one in ("repetition", "frequency", "presence"):
        check(x, {k: kw[k] for k in ("seen", "seen_offsets", one)},
              {k: want[k] for k in ("seen", one)}, "f32")
    m = np.random.default_rng(1).integers(0, 2 ** 32, size=(4, 16), dtype=np.uint64).astype(np.uint32)
    check(x, dict(masks=dev(m.view(np.int32))), dict(masks=m), "f32")


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("seen,biases", [(32767, 40), (32768, 40), (40, 65534), (40, 65535), (70000, 70000),
                                         (9, 1023), (9, 1024), (9, 1025)])
def test_long_lists(seen, biases, type_):
    """Lists around the lengths that are treated apart, one token most of the time."""
    x, kw, want = case(2, 9000, 0, 0, 2, type_, 13)
    rng = np.random.default_rng(seen + biases)
    s = np.where(rng.random(seen) < 0.9, 4100, rng.integers(0, 9000, size=seen)).astype(np.int32)
    ids = rng.choice([7, 4100, 8999, 2050], size=biases).astype(np.int32)
    b = rng.normal(size=biases).astype(np.float32)
    s[-1] = ids[-1] = 2049
    f = np.array([1e-4, 1e-3], np.float32)
    kw.update(seen=dev(s), seen_offsets=dev(np.array([0, 0, seen], np.int32)),
              prompt_lens=dev(np.array([0, 5], np.int32)), frequency=dev(f), bias_ids=dev(ids),
              bias_offsets=dev(np.array([0, 0, biases], np.int32)), biases=dev(b))
    want.update(seen=[[], s.tolist()], prompt_lens=[0, 5], frequency=f,
                bias=[[], list(zip(ids.tolist(), b.tolist()))])
    check(x, kw, want, type_)


def test_a_mask_wins_over_everything():
    x = torch.tensor([[float("nan"), float("inf"), 1.0, -1.0]], device=DEV)
    y = torch.empty_like(x)
    pk.check(pk.embbag_logits_process(
        x, y, bias_ids=torch.tensor([2], dtype=torch.int32, device=DEV),
        bias_offsets=torch.tensor([0, 1], dtype=torch.int32, device=DEV),
        biases=torch.tensor([float("inf")], device=DEV),
        masks=torch.zeros(1, 1, dtype=torch.int32, device=DEV)))
    assert (y == float("-inf")).all()


def test_counts_are_the_same_every_time():
    x, kw, _ = case(2, 3000, 4000, 900, 2, "bf16", 9)
    first = None
    for _ in range(5):
        y = torch.empty(2, 3000, dtype=torch.bfloat16, device=DEV)
        pk.check(pk.embbag_logits_process(x.to(DEV), y, **kw))
        bits = y.view(torch.int16).cpu()
        assert first is None or torch.equal(first, bits)
        first = bits


def test_bad_data_is_reported():
    x = torch.randn(2, 50, device=DEV)
    y = torch.empty_like(x)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    masks = torch.full((2, 2), -1, dtype=torch.int32, device=DEV)
    for kw, code in [
            (dict(seen=i32(1, 50), seen_offsets=i32(0, 1, 2)), pk.EMBBAG_ERR_INDEX_RANGE),
            (dict(seen=i32(1, -1), seen_offsets=i32(0, 1, 2)), pk.EMBBAG_ERR_INDEX_RANGE),
            (dict(seen=i32(1, 2), seen_offsets=i32(0, 3, 2)), pk.EMBBAG_ERR_OFFSETS),
            (dict(seen=i32(1, 2), seen_offsets=i32(1, 1, 2)), pk.EMBBAG_ERR_OFFSETS),
            (dict(seen=i32(1, 2), seen_offsets=i32(0, 1, 1)), pk.EMBBAG_ERR_OFFSETS),
            (dict(seen=i32(1, 2), seen_offsets=i32(0, -7, 2)), pk.EMBBAG_ERR_OFFSETS),
            (dict(bias_ids=i32(1, 77), bias_offsets=i32(0, 1, 2), biases=x[0, :2].contiguous()),
             pk.EMBBAG_ERR_INDEX_RANGE),
            (dict(bias_ids=i32(1, 7), bias_offsets=i32(0, 5, 2), biases=x[0, :2].contiguous()),
             pk.EMBBAG_ERR_OFFSETS),
            (dict(masks=masks, mask_ids=i32(0, 2)), pk.EMBBAG_ERR_INDEX_RANGE),
            (dict(masks=masks, mask_ids=i32(-9, 1)), 0)]:
        st = status()
        pk.check(pk.embbag_logits_process(x, y, d_status=st, **kw))
        assert pk.embbag_status_read(st) == code, kw


def test_no_rows():
    x = torch.empty(0, 50, device=DEV)
    pk.check(pk.embbag_logits_process(x, x))
