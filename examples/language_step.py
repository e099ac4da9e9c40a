"""Workers train a small language model: a layer in 4-bit microscaled floating point between an embedding and a head over the vocabulary.

Every step, each worker on its own batch: the layer's products in MX4, the cross entropy of the next token without keeping the logits, and its
gradients; a padded batch's rows have target -1.  The embedding and the head are tables: their gradients are clipped into the vector that
signum_vote_step takes.  The layer is a matrix: the workers' gradients are added and orthogonal_step takes the update, every singular value of it alike.

    python examples/language_step.py --steps 100
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1802_04434_amd as ss  # noqa: E402


class Model:
    """parameters as views of one vector: embedding (vocab x width), head (vocab x width), layer (width x width)"""

    def __init__(self, vocab, width, rows, gen, device="cuda"):
        self.lengths = [vocab * width, vocab * width]
        self.tables = torch.empty(sum(self.lengths), device=device).normal_(0, width ** -0.5, generator=gen)
        self.embedding, self.head = (t.view(vocab, width) for t in self.tables.split(self.lengths))
        self.layer = torch.empty(width, width, device=device).normal_(0, width ** -0.5, generator=gen)
        self.m = torch.zeros_like(self.layer)
        self.head16 = self.head.bfloat16()
        self.wq, self.wt = ss.new_mx4(width, width), ss.new_mx4(width, width)
        self.orthogonal_scratch = ss.new_orthogonalize_scratch(width, width)
        self.voted = ss.new_bits(self.tables.numel())
        self.refresh()

    def refresh(self):
        """what the products read of the parameters"""
        self.head16.copy_(self.head)
        ss.mx4_quantize(self.layer, self.wq, self.wt)


class Worker:
    def __init__(self, model, rows, device="cuda"):
        vocab, width = model.head.shape
        self.flat, self.m = torch.zeros_like(model.tables), torch.zeros_like(model.tables)
        self.parts = list(self.flat.split(model.lengths))
        self.norm, self.workspace = torch.empty(1, device=device), ss.new_grad_norm_workspace()
        self.xq, self.xt, self.dq, self.dt = (ss.new_mx4(*s) for s in ((rows, width), (width, rows), (rows, width), (width, rows)))
        self.y, self.dx, self.dh = (torch.empty(rows, width, dtype=torch.bfloat16, device=device) for _ in range(3))
        self.loss, self.lse, self.scratch = torch.empty(rows, device=device), torch.empty(rows, device=device), ss.new_cross_entropy_scratch(rows, vocab, width)
        self.dhead, self.dlayer = torch.empty_like(model.head16), torch.empty_like(model.layer)
        self.dembedding = torch.zeros_like(model.embedding)

    def gradients(self, model, tokens, target, max_norm):
        """of the mean loss over the rows that have a target; the tables' clipped into self.flat, the layer's in self.dlayer"""
        x = model.embedding[tokens].bfloat16()
        ss.mx4_quantize(x, self.xq, self.xt)
        active = ss.mx4_matmul(self.xq, model.wq, self.y) > 0
        self.h = x + self.y * active
        ss.cross_entropy(self.h, model.head16, target, self.loss, self.lse, self.scratch)
        there = target >= 0
        self.dloss = there / there.sum().clamp(min=1)
        ss.cross_entropy_grad(self.h, model.head16, target, self.lse, self.dloss, self.dh, self.dhead, self.scratch)
        ss.mx4_quantize(self.dh * active, self.dq, self.dt)
        ss.mx4_matmul(self.dt, self.xt, self.dlayer)
        ss.mx4_matmul(self.dq, model.wt, self.dx)
        self.dembedding.zero_().index_add_(0, tokens, self.dh.float() + self.dx.float())
        g = [self.dembedding, self.dhead]
        ss.grad_norm(g, self.norm, self.workspace)
        ss.grad_clip(g, self.norm, max_norm, self.parts)
        return (self.loss * self.dloss).sum()


def batch(rows, vocab, gen, device="cuda"):
    """tokens and the ones that follow them, by a rule with some noise; the last rows are padding"""
    tokens = torch.randint(0, vocab, (rows,), device=device, generator=gen)
    noise = torch.randint(0, 3, (rows,), device=device, generator=gen)
    target = (tokens * 5 + 7 + noise) % vocab
    target[rows - rows // 8:] = -1
    return tokens, target


def step(model, crew, batches, beta=0.9, delta=2e-3, layer_delta=2e-2, max_norm=1.0):
    """one step of all workers; the loss, averaged over them"""
    loss = sum(w.gradients(model, *b, max_norm) for w, b in zip(crew, batches)) / len(crew)
    ss.signum_vote_step([w.flat for w in crew], [w.m for w in crew], beta, delta, model.tables, model.voted)
    g = crew[0].dlayer
    for w in crew[1:]:
        g.add_(w.dlayer)
    ss.orthogonal_step(g, model.m, beta, layer_delta, model.layer, model.orthogonal_scratch, ahead=True)
    model.refresh()
    return loss


def setup(vocab=509, width=192, rows=256, workers=3, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    model = Model(vocab, width, rows, gen)
    return model, [Worker(model, rows) for _ in range(workers)], lambda: [batch(rows, vocab, gen) for _ in range(workers)]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--workers", type=int, default=3)
    a = ap.parse_args()
    model, crew, batches = setup(workers=a.workers)
    losses = torch.stack([step(model, crew, batches()) for _ in range(a.steps)]).tolist()
    for i in sorted({0, 9, a.steps // 2, a.steps - 1} & set(range(a.steps))):
        print("step %4d  loss %.4f" % (i + 1, losses[i]))


if __name__ == "__main__":
    main()
