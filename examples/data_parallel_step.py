"""A data-parallel training step on k rank buffers of one GPU, collectives and the operators around them together.

Every rank holds the same parameters (an embedding table and a router's matrix) and its own batch.  A step:

  rows of the table -> router's logits -> the k chosen experts, their counts and probability sums
  AllReduce of counts (int32) and sums (fp32) -> the loss over all ranks' tokens, and every rank's part of its gradient
  gradients of the router's matrix and, sorted by token, of the table, both in the rank's gradient buffer
  AllReduce of the gradient buffers along packed trees
  the table moves against its gradient, the router's matrix by an orthogonalised update with momentum

With --balance bias experts are kept evenly used by a bias instead of a loss, and the table moves by AdamW:

  router's logits -> the k experts with the largest sigmoid + bias in the best groups, their counts
  AllReduce of counts -> every rank's bias a step up or down
  AllReduce of the gradient buffers -> the norm of the whole gradient, from which both updates are clipped alike
  the table moves by AdamW with its moments in 8 bits, the router's matrix by the orthogonalised update

All ranks end with the same parameters, bit for bit: the trees fix the order of every sum, no operator adds by atomics, and the random bits that
round moments are those of a seed.

  python examples/data_parallel_step.py [--steps 20] [--ranks 4] [--balance loss|bias]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1910_04940_amd as bl  # noqa: E402


class Trainer:
    def __init__(self, ranks=4, tokens=512, vocab=1000, dim=64, experts=16, k=2, seed=0):
        self.ranks, self.tokens, self.vocab, self.dim, self.experts, self.k = ranks, tokens, vocab, dim, experts, k
        self.balance, self.z = 0.05, 1e-4
        g = torch.Generator("cuda").manual_seed(seed)
        table, router = 0.5 * torch.randn(vocab, dim, generator=g, device="cuda"), 0.1 * torch.randn(dim, experts, generator=g, device="cuda")
        self.label = torch.randint(0, experts, (vocab,), generator=g, device="cuda", dtype=torch.int32)   # the expert that a token should go to
        self.table = [table.clone() for _ in range(ranks)]
        self.router = [router.clone() for _ in range(ranks)]
        self.momentum = [torch.zeros_like(router) for _ in range(ranks)]
        self.batch = [torch.randint(-1, vocab, (tokens,), generator=g, device="cuda") for _ in range(ranks)]   # -1: padding
        # a gradient buffer per rank: the table's, then the router's
        self.n = vocab * dim + dim * experts
        self.grad = [torch.empty(self.n, device="cuda") for _ in range(ranks)]
        self.counts = [torch.empty(experts + 1, dtype=torch.int32, device="cuda") for _ in range(ranks)]
        self.sums = [torch.empty(experts + 1, device="cuda") for _ in range(ranks)]
        self.loss = torch.empty(3, device="cuda")
        size = max(bl.blink_embedding_gradient_workspace(tokens, vocab, dim), bl.blink_route_workspace(tokens, experts),
                   bl.blink_orthogonalize_workspace(1, dim, experts, bl.BLINK_FP32))
        self.work = torch.empty(size, dtype=torch.uint8, device="cuda")     # of one call at a time
        # every rank linked to every other
        arcs = [(a, b) for a in range(ranks) for b in range(ranks) if a != b]
        trees = bl.blink_pack_trees(ranks, [a for a, _ in arcs], [b for _, b in arcs], [1.0] * len(arcs), 0)
        self.sum_of = {n: bl.blink_make_schedule(trees, bl.BLINK_OP_ALLREDUCE, n, 1 << 16) for n in (self.n, experts + 1)}
        self.sum_of_sums = bl.blink_make_schedule(trees, bl.BLINK_OP_ALLREDUCE, experts + 1, 1 << 16)

    def step(self, rate=0.02):
        """One step; the loss over all ranks, as a tensor of (task, balance, z)."""
        stream = torch.cuda.current_stream().cuda_stream
        n, e, k = self.tokens, self.experts, self.k
        held = []
        for r in range(self.ranks):
            rows = torch.empty(n, self.dim, device="cuda")
            bl.blink_embedding(self.table[r], self.batch[r], rows, 1.0, stream)
            logits = rows @ self.router[r]
            keep = self.batch[r] >= 0
            chosen, weights = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
            bl.blink_route(logits, k, chosen, weights, self.counts[r], self.sums[r], self.work, keep, False, stream)
            held.append((rows, logits, keep, chosen, weights))
        bl.blink_allreduce(self.counts, e + 1, bl.BLINK_INT32, self.sum_of[e + 1], stream)
        bl.blink_allreduce(self.sums, e + 1, bl.BLINK_FP32, self.sum_of_sums, stream)
        task = torch.zeros((), device="cuda")
        for r, (rows, logits, keep, chosen, weights) in enumerate(held):
            # the task: weight on the token's own expert, a mean over all ranks' tokens
            own = (chosen == self.label[self.batch[r].clamp(min=0)][:, None]) & keep[:, None]
            grad_weights = -own.float() / self.counts[r][e]
            task -= (own * weights).sum() / self.counts[r][e]
            grad_logits = torch.empty_like(logits)
            bl.blink_route_gradient(logits, k, chosen, self.counts[r], grad_logits, keep, False, grad_weights, None, self.balance, self.z, stream)
            split = self.vocab * self.dim
            torch.mm(rows.t(), grad_logits, out=self.grad[r][split:].view(self.dim, e))
            grad_rows = grad_logits @ self.router[r].t()
            bl.blink_embedding_gradient(self.batch[r], grad_rows, self.grad[r][:split].view(self.vocab, self.dim), self.work, 1.0, False, stream)
        bl.blink_route_loss(self.counts[0], self.sums[0], k, self.loss, self.balance, self.z, stream)
        bl.blink_allreduce(self.grad, self.n, bl.BLINK_FP32, self.sum_of[self.n], stream)
        for r in range(self.ranks):
            split = self.vocab * self.dim
            self.table[r].sub_(self.grad[r][:split].view(self.vocab, self.dim), alpha=50_000 * rate)   # (a row has few of the batch's tokens)
            bl.blink_orthogonal_step(self.router[r], self.momentum[r], self.grad[r][split:].view(self.dim, e), self.router[r], self.momentum[r], self.work,
                                     rate, 0.9, True, stream=stream)
        return torch.stack((task, self.loss[1], self.loss[2]))


class BiasTrainer(Trainer):
    """The same with experts balanced by a bias, gradients clipped by their norm and AdamW for the table."""

    def __init__(self, ranks=4, tokens=512, vocab=1000, dim=64, experts=16, k=2, seed=0, groups=4, kept=2, max_norm=1.0):
        super().__init__(ranks, tokens, vocab, dim, experts, k, seed)
        self.groups, self.kept, self.max_norm = groups, kept, max_norm
        split, blocks = vocab * dim, -(-vocab * dim // 256)
        self.bias = [torch.zeros(experts, device="cuda") for _ in range(ranks)]
        self.moments = [[torch.zeros(split, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)] for _ in range(ranks)]
        self.scales = [[torch.zeros(blocks, device="cuda") for _ in range(2)] for _ in range(ranks)]
        self.norm = [torch.empty(2, device="cuda") for _ in range(ranks)]      # the gradient's norm, and what it is to be multiplied by
        self.count = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(ranks)]
        self.moved = [torch.empty_like(self.router[0]) for _ in range(2)]      # the router's matrix and its momentum after a step
        # the router's matrix has no weights in the list: its gradient counts in the norm, its update is the orthogonalised one
        self.update = [bl.blink_make_update([self.grad[r][:split], self.grad[r][split:]], [self.table[r].view(-1), None], [self.moments[r][0], None],
                                            [self.moments[r][1], None], scales1=[self.scales[r][0], None], scales2=[self.scales[r][1], None])
                       for r in range(ranks)]
        size = max(self.work.numel(), bl.blink_route_biased_workspace(tokens, experts), *(bl.blink_gradient_norm_workspace(u) for u in self.update))
        self.work = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step(self, rate=0.02):
        """One step; the weight that tokens give to their own experts, a mean over all ranks, and how unevenly experts are used (the largest count over the mean)."""
        stream = torch.cuda.current_stream().cuda_stream
        n, e, k = self.tokens, self.experts, self.k
        held = []
        for r in range(self.ranks):
            rows = torch.empty(n, self.dim, device="cuda")
            bl.blink_embedding(self.table[r], self.batch[r], rows, 1.0, stream)
            logits = rows @ self.router[r]
            keep = self.batch[r] >= 0
            chosen, weights = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
            bl.blink_route_biased(logits, k, chosen, weights, self.counts[r], self.work, self.bias[r], keep, self.groups, self.kept, "sigmoid", True, 1.0, stream)
            held.append((rows, logits, keep, chosen, weights))
        bl.blink_allreduce(self.counts, e + 1, bl.BLINK_INT32, self.sum_of[e + 1], stream)
        task = torch.zeros((), device="cuda")
        split = self.vocab * self.dim
        for r, (rows, logits, keep, chosen, weights) in enumerate(held):
            bl.blink_route_bias(self.counts[r], self.bias[r], self.bias[r], 0.01 * rate, stream)
            own = (chosen == self.label[self.batch[r].clamp(min=0)][:, None]) & keep[:, None]
            grad_weights = -own.float() / self.counts[r][e]
            task -= (own * weights).sum() / self.counts[r][e]
            grad_logits = torch.empty_like(logits)
            bl.blink_route_biased_gradient(logits, k, chosen, grad_weights, grad_logits, keep, "sigmoid", True, 1.0, stream)
            torch.mm(rows.t(), grad_logits, out=self.grad[r][split:].view(self.dim, e))
            grad_rows = grad_logits @ self.router[r].t()
            bl.blink_embedding_gradient(self.batch[r], grad_rows, self.grad[r][:split].view(self.vocab, self.dim), self.work, 1.0, False, stream)
        bl.blink_allreduce(self.grad, self.n, bl.BLINK_FP32, self.sum_of[self.n], stream)
        for r in range(self.ranks):
            bl.blink_gradient_norm(self.update[r], self.norm[r], self.work, self.max_norm, 1.0, self.count[r], stream)
            bl.blink_adamw_step(self.update[r], self.count[r], rate, 0.9, 0.99, 1e-8, self.norm[r][1:], None, 1234, stream)
            # AdamW leaves the step out where the factor is NaN (a gradient was no number); the other update is taken or left here, without asking the host
            router = (self.grad[r][split:] * self.norm[r][1]).view(self.dim, e)
            bl.blink_orthogonal_step(self.router[r], self.momentum[r], router, *self.moved, self.work, rate, 0.9, True, stream=stream)
            for old, new in zip((self.router[r], self.momentum[r]), self.moved):
                old.copy_(torch.where(torch.isnan(self.norm[r][1]), old, new))
        return torch.stack((task, self.counts[0][:e].max() * e / self.counts[0][:e].sum()))


def main():
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=20)
    parser.add_argument("--ranks", type=int, default=4)
    parser.add_argument("--balance", choices=("loss", "bias"), default="loss")
    a = parser.parse_args()
    trainer = (BiasTrainer if a.balance == "bias" else Trainer)(ranks=a.ranks)
    for i in range(a.steps):
        if a.balance == "bias":
            task, uneven = trainer.step().tolist()
            print(f"step {i + 1}: weight on a token's own expert {-task:.4f}, busiest expert {uneven:.2f} times the mean", flush=True)
            continue
        task, balance, z = trainer.step().tolist()
        print(f"step {i + 1}: weight on a token's own expert {-task:.4f}, balance loss {balance:.4f}, z loss {z:.5f}", flush=True)
    same = all(torch.equal(t, trainer.table[0]) for t in trainer.table) and all(torch.equal(t, trainer.router[0]) for t in trainer.router)
    print("all ranks hold the same parameters" if same else "THE RANKS DIFFER")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
