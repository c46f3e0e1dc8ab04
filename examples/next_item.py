"""The next item from a history, trained on labels: a look-up table, a norm and a catalogue whose
rows are the scores' matrix, all three learned; served from a 4-bit catalogue and 8-bit rows.

A training step is
  embbag_forward -> embbag_rmsnorm -> embbag_xent (the scores of the whole catalogue, kept
  nowhere but in its workspace) -> embbag_rmsnorm_grad -> embbag_backward_sgd, and plain SGD on the catalogue and
  the norm's weights,
and serving is
  embbag_forward -> embbag_rmsnorm (into 8 bits) -> embbag_mx4_matmul_x8 ->
  embbag_logits_process -> the best item.

    python examples/next_item.py [--steps 60] [--items 20000] [--dim 128]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2005_04680_amd as pk  # noqa: E402

DEV = "cuda"
EPS = 1e-6


class NextItem:
    def __init__(self, items, catalogue, batch, max_lookups):
        """items: FP32 [M, E]; catalogue: FP32 [V, E]; both trained."""
        self.items, self.catalogue, self.batch = items, catalogue, batch
        self.tables = pk.Tables([items])
        E, V = items.shape[1], catalogue.shape[0]
        new = lambda *shape: torch.empty(*shape, device=items.device)
        self.weight = torch.ones(E, device=items.device)
        self.pooled, self.hidden, self.grad_hidden, self.grad_pooled = (new(batch, E) for _ in range(4))
        self.grad_weight, self.grad_catalogue = new(E), torch.empty_like(catalogue)
        self.loss, self.logits = new(batch), new(batch, V)
        self.rows8 = pk.Mx8Rows.empty(batch, E, items.device)
        self.catalogue4 = pk.Mx4Table.empty(V, E, items.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=items.device)
        size = max(pk.embbag_xent_workspace_bytes(batch, V, E, pk.EMBBAG_F32, True),
                   pk.embbag_rmsnorm_grad_workspace_bytes(batch, E),
                   pk.embbag_mx4_matmul_x8_workspace_bytes(batch, V, E),
                   pk.embbag_backward_workspace_bytes(1, batch, max_lookups, E))
        self.ws = torch.empty(size, dtype=torch.uint8, device=items.device)

    def gradients(self, history, offsets, labels, row_weights):
        """Losses and all gradients but the look-ups': those of the catalogue, the norm's weights and
        the pooled rows."""
        pk.check(pk.embbag_forward(self.tables, self.batch, history, offsets, self.pooled, self.status), "forward")
        pk.check(pk.embbag_rmsnorm(self.pooled, self.weight, EPS, out=self.hidden), "norm")
        pk.check(pk.embbag_xent(self.hidden, self.catalogue, labels, self.loss, self.ws, grad_x=self.grad_hidden,
                                grad_table=self.grad_catalogue, row_weights=row_weights, d_status=self.status), "xent")
        pk.check(pk.embbag_rmsnorm_grad(self.grad_hidden, self.pooled, self.weight, EPS, self.grad_pooled, self.ws,
                                        dweight=self.grad_weight), "norm_grad")
        return self.loss

    def train_step(self, history, offsets, labels, lr, row_weights=None):
        """Returns the rows' losses (a negative label is no row to learn)."""
        self.gradients(history, offsets, labels, row_weights)
        pk.check(pk.embbag_backward_sgd(self.grad_pooled, self.batch, history, offsets, lr, self.tables, self.ws,
                                        self.status), "backward")
        self.catalogue.add_(self.grad_catalogue, alpha=-lr)
        self.weight.add_(self.grad_weight, alpha=-lr)
        return self.loss

    def freeze(self):
        """The catalogue's 4-bit copy, which serves."""
        pk.check(pk.embbag_mx4_quantize(self.catalogue, self.catalogue4), "quantize")

    def serve(self, history, offsets, penalty):
        """The best item of every row, those of its own history penalised."""
        pk.check(pk.embbag_forward(self.tables, self.batch, history, offsets, self.pooled, self.status), "forward")
        pk.check(pk.embbag_rmsnorm(self.pooled, self.weight, EPS, mx8=self.rows8), "norm")
        pk.check(pk.embbag_mx4_matmul_x8(self.rows8, self.catalogue4, self.logits, self.ws), "matmul_x8")
        pk.check(pk.embbag_logits_process(self.logits, self.logits, seen=history, seen_offsets=offsets,
                                          presence=penalty, d_status=self.status), "logits")
        return self.logits.argmax(1)


def main(steps=60, items=20000, dim=128, batch=256, bag=10, lr=4.0, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new = lambda *shape: torch.randn(*shape, device=DEV, generator=g)
    model = NextItem(new(items, dim) * dim ** -0.5, new(items, dim) * dim ** -0.5, batch, batch * bag)
    offsets = torch.arange(0, batch * bag + 1, bag, dtype=torch.int32, device=DEV)
    # A few batches again and again: the next item follows from the first one of the history.
    batches = [torch.randint(0, items, (batch * bag,), device=DEV, generator=g, dtype=torch.int32) for _ in range(4)]
    mean = torch.full((batch,), 1.0 / (batch - 1), device=DEV)
    losses = []
    for step in range(steps):
        history = batches[step % len(batches)]
        labels = (history[::bag] * 7 + 3) % items
        labels[-1] = -1  # a request without an answer
        losses.append(float(model.train_step(history, offsets, labels, lr, row_weights=mean).sum()))
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    model.freeze()
    choice = model.serve(history, offsets, torch.full((batch,), 1e4, device=DEV))
    pk.check(pk.embbag_status_read(model.status), "device status")
    new_items = bool((history.view(batch, bag) != choice[:, None]).all())
    right = float((choice == labels).float().mean())
    print(f"served {batch} requests: none from its own history: {new_items}, learned answers: {right:.0%}", flush=True)
    return losses, choice, new_items, model


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--items", type=int, default=20000)
    p.add_argument("--dim", type=int, default=128)
    a = p.parse_args()
    main(a.steps, a.items, a.dim)
