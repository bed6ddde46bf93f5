"""The example that runs collectives and the operators around them as one training step."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_ranks_stay_equal_and_learn():
    from data_parallel_step import Trainer
    trainer = Trainer(ranks=4)
    losses = [trainer.step().tolist() for _ in range(30)]
    assert all(torch.equal(t.view(torch.int32), trainer.table[0].view(torch.int32)) for t in trainer.table)
    assert all(torch.equal(t.view(torch.int32), trainer.router[0].view(torch.int32)) for t in trainer.router)
    assert all(torch.equal(t.view(torch.int32), trainer.momentum[0].view(torch.int32)) for t in trainer.momentum)
    assert losses[-1][0] < losses[0][0] - 0.05      # more weight on the tokens' own experts


def test_one_step_against_autograd():
    """The same step from plain products and the loss by automatic differentiation, in 64 bits: gradients of all ranks together."""
    from data_parallel_step import Trainer
    trainer = Trainer(ranks=3, tokens=200, vocab=60, dim=24, experts=8)
    table, router = trainer.table[0].double().requires_grad_(), trainer.router[0].double().requires_grad_()
    batch = torch.cat(trainer.batch)
    keep = batch >= 0
    logits = table[batch[keep]] @ router
    p = torch.softmax(logits, 1)
    chosen = torch.topk(logits.detach(), 2).indices
    n, e = int(keep.sum()), 8
    counts = torch.zeros(e, dtype=torch.float64, device="cuda").index_add_(0, chosen.reshape(-1), torch.ones(chosen.numel(), dtype=torch.float64, device="cuda"))
    weights = p.gather(1, chosen)
    own = chosen == trainer.label[batch[keep]][:, None]
    loss = -(own * weights).sum() / n + trainer.balance * e / 2 / n / n * (counts * p.sum(0)).sum() + trainer.z / n * (torch.logsumexp(logits, 1) ** 2).sum()
    loss.backward()
    got = trainer.step(rate=0.0).double().sum()
    assert abs(float(got - loss.detach())) < 1e-5
    split = 60 * 24
    for r in range(3):
        for part, want in ((trainer.grad[r][:split].view(60, 24), table.grad), (trainer.grad[r][split:].view(24, 8), router.grad)):
            # sums of up to 600 products of 32-bit numbers, each off by a few units
            assert float((part.double() - want).norm()) <= 600 * 2.0 ** -23 * float(want.norm()) + 1e-9
