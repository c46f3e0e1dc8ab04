"""The output head's operators together: the example, graphs, other streams, the same bits
every time, and what the binding refuses."""
import os
import sys

import numpy as np
import pytest
import torch

import head_reference as ref
import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import random_table

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import item_head  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def test_the_example_learns_and_serves():
    losses, choice, fine, model = item_head.main(steps=24, items=3001, dim=64, batch=96, bag=7, top=30)
    assert fine and min(losses[-4:]) < 0.5 * losses[0]
    # the copy that serves is the table's quantisation, also of rows that no step touched
    codes, scales = ref.quantize(model.items[:200].double().cpu().numpy())
    assert np.array_equal(model.copy.codes[:200].cpu().numpy(), codes)
    assert np.array_equal(model.copy.scales[:200].cpu().numpy(), scales)


def test_a_training_step_is_the_references():
    """One step against the 64-bit reference, through the gradient into the updated table."""
    g = torch.Generator(device=DEV).manual_seed(3)
    M, E, B, P, K = 200, 32, 6, 5, 9
    items = torch.randn(M, E, device=DEV, generator=g) * 0.3
    start = items.double().cpu().numpy()
    cat = torch.randn(150, E, device=DEV, generator=g)
    model = item_head.ItemHead(items, cat, B, K, B * P)
    hist = torch.randint(0, M, (B * P,), device=DEV, generator=g, dtype=torch.int32)
    off = torch.arange(0, B * P + 1, P, dtype=torch.int32, device=DEV)
    ids = torch.stack([torch.randperm(150, generator=torch.Generator().manual_seed(r))[:K] for r in range(B)])
    t = torch.randn(B, K, generator=torch.Generator().manual_seed(9))
    loss = model.train_step(hist, off, ids.to(torch.int32).to(DEV), t.to(DEV), 0.5).double().cpu().numpy()

    h = hist.cpu().numpy().reshape(B, P)
    pooled = start[h].sum(1).astype(np.float32).astype(np.float64)
    w = ref.dequantize(*ref.quantize(cat.double().cpu().numpy()), E)
    x = ref.dequantize(*ref.quantize(pooled), E) @ w.T
    want, grad, _, _ = ref.distill(x, ids.numpy(), t.double().numpy(), 1.0)
    assert np.allclose(loss, want, rtol=1e-4, atol=1e-4)
    dx = grad @ w
    table = start.copy()
    for b in range(B):
        for s in range(P):
            table[h[b, s]] -= 0.5 * dx[b]
    assert np.allclose(items.double().cpu().numpy(), table, rtol=1e-4, atol=1e-4)


def head_pass(seed=0, m=70, n=1003, k=160):
    """Inputs and a function that runs every operator once into fixed buffers."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    table, _ = random_table(n, k, 5)
    src = torch.randn(n, k, device=DEV, generator=g)
    again = pk.Mx4Table.empty(n, k)
    back = torch.empty(n, k, device=DEV, dtype=torch.bfloat16)
    idx = torch.randint(0, n, (m * 9,), device=DEV, generator=g, dtype=torch.int32)
    off = torch.arange(0, m * 9 + 1, 9, dtype=torch.int32, device=DEV)
    y = torch.empty(1, m, k, device=DEV)
    out = torch.empty(m, n, device=DEV, dtype=torch.bfloat16)
    done = torch.empty_like(out)
    ids = torch.stack([torch.randperm(n, device=DEV, generator=g)[:12] for _ in range(m)]).to(torch.int32)
    teach = torch.randn(m, 12, device=DEV, generator=g)
    loss, grad = torch.empty(m, device=DEV), torch.empty_like(out)
    dx = torch.empty(m, k, device=DEV)
    few, few_grad, few_loss = torch.empty(3, n, device=DEV), torch.empty(3, n, device=DEV), torch.empty(3, device=DEV)
    tables = pk.Mx4Tables([table])
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    half = torch.full((m,), 0.5, device=DEV)

    def run():
        pk.check(pk.embbag_mx4_quantize(src, again))
        pk.check(pk.embbag_mx4_dequantize(again, back))
        pk.check(pk.embbag_mx4_forward(tables, m, idx, off, y, d_status=status))
        pk.check(pk.embbag_mx4_matmul(y[0], table, out, ws))
        pk.check(pk.embbag_logits_process(out, done, seen=idx, seen_offsets=off, frequency=half,
                                          bias_ids=idx, bias_offsets=off, biases=teach.view(-1)[:1].expand(m * 9).contiguous(),
                                          d_status=status))
        pk.check(pk.embbag_distill(done, ids, teach, 2.0, loss, ws, grad=grad, d_status=status))
        pk.check(pk.embbag_mx4_matmul_grad(grad, table, dx, ws))
        pk.check(pk.embbag_mx4_matmul(y[0, :3], table, few, ws))
        pk.check(pk.embbag_distill(few, ids[:3], teach[:3], 1.0, few_loss, ws, grad=few_grad, d_status=status))
        return [again.codes, again.scales, back, y, out, done, loss, grad, dx, few, few_loss, few_grad]

    return run, src, status


def bits(ts):
    torch.cuda.synchronize()
    return [t.clone().view(torch.uint8).cpu() for t in ts]


def test_the_same_bits_every_time():
    run, _, status = head_pass()
    first = bits(run())
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, bits(run())))
    assert pk.embbag_status_read(status) == 0


def test_in_a_graph():
    run, src, _ = head_pass(1)
    out = run()
    want = [bits(out)]
    values = [src.clone(), src * 1.5 + 0.25, src.flip(0).contiguous()]
    for v in values[1:]:
        src.copy_(v)
        want.append(bits(run()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in (2, 0, 1, 0):
        src.copy_(values[i])
        for t in out:
            t.view(torch.uint8).fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want[i], bits(out))), i
        (src * 2).sum().item()  # the program's own work between replays


def test_on_another_stream():
    run, src, _ = head_pass(2)
    want = bits(run())
    side = torch.cuda.Stream()
    for t in run():
        t.view(torch.uint8).fill_(3)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out = run()
    assert all(torch.equal(a, b) for a, b in zip(want, bits(out)))


def test_the_binding_checks_sizes():
    t, _ = random_table(20, 64, 1)
    f = lambda *s: torch.zeros(*s, device=DEV)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    tb = pk.Mx4Tables([t])
    for err, call in [
            (ValueError, lambda: pk.embbag_mx4_quantize(f(19, 64), t)),
            (ValueError, lambda: pk.embbag_mx4_quantize(f(20, 60), t)),
            (TypeError, lambda: pk.embbag_mx4_quantize(f(20, 64).half(), t)),
            (TypeError, lambda: pk.embbag_mx4_quantize(f(64, 20).t(), t)),
            (TypeError, lambda: pk.embbag_mx4_quantize(f(20, 64), t, row_ids=i(3).long())),
            (ValueError, lambda: pk.embbag_mx4_dequantize(t, f(21, 64))),
            (ValueError, lambda: pk.embbag_mx4_forward(tb, 2, i(4), i(4), f(1, 2, 64))),
            (ValueError, lambda: pk.embbag_mx4_forward(tb, 2, i(4), i(3), f(1, 2, 60))),
            (TypeError, lambda: pk.embbag_mx4_forward(tb, 2, i(4), i(3), f(1, 2, 64).half())),
            (ValueError, lambda: pk.embbag_mx4_forward(tb, 2, i(4), i(3), f(1, 2, 64), f(5))),
            (ValueError, lambda: pk.embbag_mx4_matmul(f(3, 60), t, f(3, 20), ws)),
            (ValueError, lambda: pk.embbag_mx4_matmul(f(3, 64), t, f(3, 21), ws)),
            (ValueError, lambda: pk.embbag_mx4_matmul(f(3, 64), t, f(2, 20), ws)),
            (TypeError, lambda: pk.embbag_mx4_matmul(f(3, 64), t, f(3, 1).expand(3, 20), ws)),
            (ValueError, lambda: pk.embbag_mx4_matmul_grad(f(3, 21), t, f(3, 64), ws)),
            (ValueError, lambda: pk.embbag_mx4_matmul_grad(f(3, 20), t, f(4, 64), ws)),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 10))),
            (TypeError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 9).bfloat16())),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 9), seen=i(4), seen_offsets=i(4))),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 9), seen=i(4))),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 9), seen=i(4), seen_offsets=i(3),
                                                          repetition=f(3))),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 9), bias_ids=i(4), bias_offsets=i(3),
                                                          biases=f(3))),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 33), f(2, 33), masks=i(2, 1))),
            (ValueError, lambda: pk.embbag_logits_process(f(2, 9), f(2, 9), masks=i(1, 1))),
            (ValueError, lambda: pk.embbag_distill(f(2, 9), i(3, 4), f(3, 4), 1.0, f(2), ws)),
            (ValueError, lambda: pk.embbag_distill(f(2, 9), i(2, 4), f(2, 3), 1.0, f(2), ws)),
            (ValueError, lambda: pk.embbag_distill(f(2, 9), i(2, 4), f(2, 4), 1.0, f(3), ws)),
            (ValueError, lambda: pk.embbag_distill(f(2, 9), i(2, 4), f(2, 4), 1.0, f(2), ws, grad=f(3, 9))),
            (TypeError, lambda: pk.embbag_distill(f(2, 9), i(2, 4), f(2, 4), 1.0, f(2), ws,
                                                  grad=f(2, 9).bfloat16()))]:
        with pytest.raises(err):
            call()
