"""Next-item scores from embedding tables: train a look-up table against a teacher's
top logits, keep a 4-bit copy of it up to date, and serve from the copy.

A request's history (a bag of item ids) is pooled from the FP32 table `items`; its
scores are the products with all rows of a catalogue (which is not trained) kept in
4-bit microscaled storage.  A training step is
  embbag_forward -> embbag_mx4_matmul -> embbag_distill -> embbag_mx4_matmul_grad
  -> embbag_backward_sgd -> embbag_mx4_quantize (of the rows the batch touched),
and serving is
  embbag_mx4_forward -> embbag_mx4_matmul -> embbag_logits_process -> the best item.

    python examples/item_head.py [--steps 40] [--items 20000] [--dim 128]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2005_04680_amd as pk  # noqa: E402

DEV = "cuda"


class ItemHead:
    def __init__(self, items, catalogue, batch, top, max_lookups):
        """items: FP32 [M, E], trained; catalogue: FP32 [V, E], kept in 4 bits."""
        self.items, self.batch, self.top = items, batch, top
        self.tables = pk.Tables([items])
        M, E = items.shape
        V = catalogue.shape[0]
        self.catalogue = pk.Mx4Table.empty(V, E, items.device)
        self.copy = pk.Mx4Table.empty(M, E, items.device)
        pk.check(pk.embbag_mx4_quantize(catalogue, self.catalogue), "quantize")
        pk.check(pk.embbag_mx4_quantize(items, self.copy), "quantize")
        self.serving = pk.Mx4Tables([self.copy])
        new = lambda *shape: torch.empty(*shape, device=items.device)
        self.pooled, self.grad_pooled = new(batch, E), new(batch, E)
        self.logits, self.loss = new(batch, V), new(batch)
        self.status = torch.zeros(1, dtype=torch.int32, device=items.device)
        size = max(pk.embbag_mx4_matmul_workspace_bytes(batch, V, E),
                   pk.embbag_mx4_matmul_grad_workspace_bytes(batch, V, E),
                   pk.embbag_distill_workspace_bytes(batch, V, top),
                   pk.embbag_backward_workspace_bytes(1, batch, max_lookups, E))
        self.ws = torch.empty(size, dtype=torch.uint8, device=items.device)

    def scores(self, pooled):
        pk.check(pk.embbag_mx4_matmul(pooled, self.catalogue, self.logits, self.ws), "matmul")
        return self.logits

    def train_step(self, history, offsets, teacher_ids, teacher_logits, lr, temperature=1.0):
        """Returns the rows' losses (each row has the weight 1)."""
        pk.check(pk.embbag_forward(self.tables, self.batch, history, offsets, self.pooled,
                                   self.status), "forward")
        self.scores(self.pooled)
        pk.check(pk.embbag_distill(self.logits, teacher_ids, teacher_logits, temperature, self.loss,
                                   self.ws, grad=self.logits, d_status=self.status), "distill")
        pk.check(pk.embbag_mx4_matmul_grad(self.logits, self.catalogue, self.grad_pooled, self.ws),
                 "matmul_grad")
        pk.check(pk.embbag_backward_sgd(self.grad_pooled, self.batch, history, offsets, lr,
                                        self.tables, self.ws, self.status), "backward")
        pk.check(pk.embbag_mx4_quantize(self.items, self.copy, row_ids=history,
                                        d_status=self.status), "quantize")
        return self.loss

    def serve(self, history, offsets, allowed, penalty):
        """The best item of every row: allowed ones (a row of bits for every request), those of its
        own history penalised."""
        pk.check(pk.embbag_mx4_forward(self.serving, self.batch, history, offsets, self.pooled,
                                       d_status=self.status), "forward")
        self.scores(self.pooled)
        pk.check(pk.embbag_logits_process(self.logits, self.logits, seen=history,
                                          seen_offsets=offsets, presence=penalty, masks=allowed,
                                          d_status=self.status), "logits")
        return self.logits.argmax(1)


def bits_of(allowed):
    """Rows of truth values as rows of 32-bit words."""
    n = -allowed.shape[1] % 32
    b = torch.nn.functional.pad(allowed, (0, n)).view(allowed.shape[0], -1, 32).long()
    w = (b << torch.arange(32, device=allowed.device)).sum(2)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def main(steps=40, items=20000, dim=128, batch=256, bag=20, top=50, lr=0.5, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    catalogue = torch.randn(items, dim, device=DEV, generator=g) * dim ** -0.5
    truth = torch.randn(items, dim, device=DEV, generator=g)  # what the teacher knows
    model = ItemHead(torch.zeros(items, dim, device=DEV), catalogue, batch, top, batch * bag)
    offsets = torch.arange(0, batch * bag + 1, bag, dtype=torch.int32, device=DEV)
    batches = [torch.randint(0, items, (batch * bag,), device=DEV, generator=g, dtype=torch.int32)
               for _ in range(4)]
    losses = []
    for step in range(steps):
        history = batches[step % len(batches)]
        pooled = truth[history.long()].view(batch, bag, dim).sum(1)
        best = (pooled @ catalogue.t()).topk(top, dim=1)
        loss = model.train_step(history, offsets, best.indices.to(torch.int32), best.values.contiguous(), lr)
        losses.append(float(loss.mean()))
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    allowed = torch.rand(batch, items, device=DEV, generator=g) < 0.5
    choice = model.serve(history, offsets, bits_of(allowed), torch.full((batch,), 1e4, device=DEV))
    pk.check(pk.embbag_status_read(model.status), "device status")
    ok = bool(allowed[torch.arange(batch, device=DEV), choice].all())
    new = bool((history.view(batch, bag) != choice[:, None]).all())
    print(f"served {batch} requests: all allowed: {ok}, none from its own history: {new}", flush=True)
    return losses, choice, ok and new, model


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=40)
    p.add_argument("--items", type=int, default=20000)
    p.add_argument("--dim", type=int, default=128)
    a = p.parse_args()
    main(a.steps, a.items, a.dim)
