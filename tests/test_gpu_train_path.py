"""The norm, the scores from 8-bit rows and the cross entropy together: the example, graphs,
other streams, the same bits every time."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2005_04680_amd as pk
import train_reference as ref
from gpu_util import DEV, require_gpu
from test_gpu_mx4 import random_table

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import next_item  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def test_the_example_runs_and_serves():
    losses, choice, fine, model = next_item.main(steps=6, items=3001, dim=64, batch=96, bag=7)
    assert fine and np.isfinite(losses).all() and choice.shape == (96,)
    assert torch.isfinite(model.catalogue).all() and torch.isfinite(model.items).all()


@pytest.mark.parametrize("E,V", [(32, 150), (132, 700)])
def test_a_steps_gradients_are_the_references(E, V):
    """Through the whole path, against the 64-bit formulas and against differences."""
    g = torch.Generator(device=DEV).manual_seed(3)
    M, B, P = 200, 6, 5
    model = next_item.NextItem(torch.randn(M, E, device=DEV, generator=g) * 0.3,
                               torch.randn(V, E, device=DEV, generator=g) * E ** -0.5, B, B * P)
    model.weight.add_(torch.randn(E, device=DEV, generator=g) * 0.2)
    hist = torch.randint(0, M, (B * P,), device=DEV, generator=g, dtype=torch.int32)
    off = torch.arange(0, B * P + 1, P, dtype=torch.int32, device=DEV)
    labels = torch.tensor([3, -1, V - 1, 0, 3, 17], dtype=torch.int32, device=DEV)
    k = torch.tensor([1.0, 1.0, 0.5, 0.0, 2.0, -1.0], device=DEV)
    host = lambda t: t.double().cpu().numpy()
    start, cat, w = host(model.items), host(model.catalogue), host(model.weight)
    h = hist.cpu().numpy().reshape(B, P)
    pooled = start[h].sum(1)
    eps = next_item.EPS

    def total(pooled, cat, w):
        return ref.xent(ref.rmsnorm(pooled, w, eps)[0], cat, labels.cpu().numpy(), host(k))[0]

    hidden = ref.rmsnorm(pooled, w, eps)[0]
    loss, dx, dcat, _ = ref.xent(hidden, cat, labels.cpu().numpy(), host(k))
    dpool, dw, _, _ = ref.rmsnorm_grad(dx, pooled, w, eps)
    got = host(model.train_step(hist, off, labels, 0.5, row_weights=k))
    assert np.allclose(got, loss, rtol=1e-5, atol=1e-5)
    assert np.allclose(host(model.grad_catalogue), dcat, rtol=1e-4, atol=1e-5)
    assert np.allclose(host(model.grad_pooled), dpool, rtol=1e-4, atol=1e-5)
    assert np.allclose(host(model.grad_weight), dw, rtol=1e-4, atol=1e-5)
    table = start.copy()
    for b in range(B):
        for s in range(P):
            table[h[b, s]] -= 0.5 * dpool[b]
    assert np.allclose(host(model.items), table, rtol=1e-4, atol=1e-5)
    assert np.allclose(host(model.catalogue), cat - 0.5 * dcat, rtol=1e-4, atol=1e-5)
    step = 1e-5
    for b, e in [(0, 0), (1, 3), (5, E - 1)]:
        d = np.zeros_like(pooled)
        d[b, e] = step
        by = (total(pooled + d, cat, w).sum() - total(pooled - d, cat, w).sum()) / (2 * step)
        assert abs(by - host(model.grad_pooled)[b, e]) < 1e-4


def train_pass(seed=0, n=70, v=1003, e=160, type_="bf16", ws=None):
    """Inputs and a function that runs every operator once into fixed buffers."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[type_]
    x = torch.randn(n, e, device=DEV, generator=g).to(dt)
    r = torch.randn(n, e, device=DEV, generator=g)
    weight = (1 + 0.1 * torch.randn(e, device=DEV, generator=g)).to(dt)
    table4, _ = random_table(v, e, 5)
    table = (torch.randn(v, e, device=DEV, generator=g) * e ** -0.5).to(dt)
    labels = torch.randint(-20, v, (n,), device=DEV, generator=g, dtype=torch.int32)
    k = torch.rand(n, device=DEV, generator=g)
    out, s, q = torch.empty_like(x), torch.empty_like(r), pk.Mx8Rows.empty(n, e)
    logits = torch.empty(n, v, device=DEV)
    loss, dx, dtable = torch.empty(n, device=DEV), torch.empty_like(x), torch.empty_like(table)
    dh, dweight = torch.empty_like(s), torch.empty_like(weight)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    need = max(pk.embbag_xent_workspace_bytes(n, v, e, pk.EMBBAG_F32 if type_ == "f32" else pk.EMBBAG_BF16, True),
               pk.embbag_rmsnorm_grad_workspace_bytes(n, e), pk.embbag_mx4_matmul_x8_workspace_bytes(n, v, e))
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert ws.numel() >= need

    def run(stream=None):
        pk.check(pk.embbag_rmsnorm(x, weight, 1e-6, out=out, mx8=q, residual=r, sum_out=s, stream=stream))
        pk.check(pk.embbag_mx4_matmul_x8(q, table4, logits, ws, stream=stream))
        pk.check(pk.embbag_xent(out, table, labels, loss, ws, grad_x=dx, grad_table=dtable, row_weights=k,
                                d_status=status, stream=stream))
        pk.check(pk.embbag_rmsnorm_grad(dx, s, weight, 1e-6, dh, ws, dweight=dweight, dsum=r, stream=stream))

    outputs = (out, s, q.codes, q.scales, logits, loss, dx, dtable, dh, dweight)
    return run, outputs, (x, r, labels), ws


SIZES = [(70, 1003, 160, "bf16"), (70, 1003, 160, "f32"), (300, 2003, 64, "bf16"), (33, 1003, 100, "f32"),
         (5000, 300, 132, "bf16"), (1, 5003, 260, "bf16")]


@pytest.mark.parametrize("n,v,e,t", SIZES)
def test_graph_replays_are_the_eager_results(n, v, e, t):
    """Replays with other inputs in between, eager work of the same operators and synchronizations."""
    run, outputs, (x, r, labels), ws = train_pass(1, n, v, e, t)
    run()
    torch.cuda.synchronize()
    first = [o.clone() for o in outputs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    other, other_out, _, _ = train_pass(2, n, v, e, t)
    start = (x.clone(), labels.clone())
    for turn in range(4):
        if turn == 2:  # other inputs: fewer rows count
            x.mul_(-0.5), labels[: n // 2 + 1].fill_(-1)
        for o in outputs:
            o.view(torch.uint8).fill_(0xCD)
        ws.fill_(turn * 85)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outputs]
        other()
        run()
        torch.cuda.synchronize()
        for a, b in zip(got, outputs):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        if turn < 2:
            for a, b in zip(got, first):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    x.copy_(start[0]), labels.copy_(start[1])
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outputs, first):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_two_graphs_in_turn_share_a_workspace():
    size = 64 << 20
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    runs = [train_pass(1, 70, 1003, 160, "bf16", ws), train_pass(2, 300, 2003, 64, "f32", ws)]
    want = []
    for run, outputs, _, _ in runs:
        run()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outputs])
    graphs = []
    for run, _, _, _ in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
    for _ in range(3):
        for graph, (_, outputs, _, _), w in zip(graphs, runs, want):
            for o in outputs:
                o.view(torch.uint8).fill_(0xCD)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outputs, w):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_two_streams_at_once():
    """Each with its own workspace, given as an argument and as the current stream."""
    runs = [train_pass(3, 300, 2003, 160, "bf16"), train_pass(4, 300, 2003, 100, "f32")]
    want = []
    for run, outputs, _, _ in runs:
        run()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outputs])
        for o in outputs:
            o.view(torch.uint8).fill_(0xCD)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        runs[0][0](stream=streams[0])
        with torch.cuda.stream(streams[1]):
            runs[1][0]()
    torch.cuda.synchronize()
    for (_, outputs, _, _), w in zip(runs, want):
        for a, b in zip(outputs, w):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_split_tables_high_halves_are_a_table():
    """The high halves of split rows, as BF16: the loss over the truncated weights."""
    g = torch.Generator(device=DEV).manual_seed(1)
    full = torch.randn(500, 64, device=DEV, generator=g) / 8
    hi = torch.empty(500, 64, dtype=torch.int16, device=DEV)
    lo = torch.empty_like(hi)
    pk.check(pk.embbag_split_fp32(full, hi, lo))
    x = torch.randn(20, 64, device=DEV, generator=g).bfloat16()
    labels = torch.arange(20, dtype=torch.int32, device=DEV)
    loss = torch.empty(20, device=DEV)
    table = hi.view(torch.bfloat16)
    ws = torch.empty(pk.embbag_xent_workspace_bytes(20, 500, 64, pk.EMBBAG_BF16, False), dtype=torch.uint8, device=DEV)
    pk.check(pk.embbag_xent(x, table, labels, loss, ws))
    z = x.double() @ table.double().t()
    want = torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0]
    assert (loss.double() - want).abs().max() < 1e-5
