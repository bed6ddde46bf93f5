"""The example's step with experts balanced by a bias, a clipped gradient and AdamW, all operators together."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_ranks_stay_equal():
    from data_parallel_step import BiasTrainer
    trainer = BiasTrainer(ranks=4)
    before = trainer.table[0].clone()
    for _ in range(20):
        trainer.step()
    same = lambda tensors: all(torch.equal(t.view(torch.uint8), tensors[0].view(torch.uint8)) for t in tensors)   # noqa: E731
    assert all(same(v) for v in (trainer.table, trainer.router, trainer.momentum, trainer.bias, trainer.count, trainer.norm))
    assert all(same([v[i] for v in part]) for part in (trainer.moments, trainer.scales) for i in range(2))
    assert int(trainer.count[0]) == 20 and not torch.equal(before, trainer.table[0]) and bool((trainer.bias[0] != 0).any())
    assert all(torch.isfinite(t).all() for t in (trainer.table[0], trainer.router[0], trainer.norm[0]))


def test_one_step_against_autograd():
    """Gradients of all ranks together by automatic differentiation in 64 bits, and the table after AdamW's first step from them."""
    from data_parallel_step import BiasTrainer
    trainer = BiasTrainer(ranks=3, tokens=200, vocab=60, dim=24, experts=8, max_norm=0.01)
    table, router = trainer.table[0].double().requires_grad_(), trainer.router[0].double().requires_grad_()
    before = trainer.table[0].double()
    batch = torch.cat(trainer.batch)
    keep = batch >= 0
    logits = table[batch[keep]] @ router
    p = torch.sigmoid(logits)
    of_group = p.detach().view(-1, 4, 2).sum(2)
    best = torch.topk(of_group, 2).indices
    stays = torch.zeros_like(of_group).scatter_(1, best, 1).repeat_interleave(2, 1) > 0
    chosen = torch.topk(p.detach().masked_fill(~stays, -1.0), 2).indices
    weights = p.gather(1, chosen)
    weights = weights / weights.sum(1, keepdim=True)
    own = chosen == trainer.label[batch[keep]][:, None]
    loss = -(own * weights).sum() / int(keep.sum())
    loss.backward()
    got = float(trainer.step(rate=0.01)[0])
    assert abs(got - float(loss.detach())) < 1e-5
    split = 60 * 24
    length = float(torch.cat((table.grad.reshape(-1), router.grad.reshape(-1))).norm())
    # sums of up to 600 products of 32-bit numbers, each off by a few units
    tolerance = 600 * 2.0 ** -23
    for r in range(3):
        for part, want in ((trainer.grad[r][:split].view(60, 24), table.grad), (trainer.grad[r][split:].view(24, 8), router.grad)):
            assert float((part.double() - want).norm()) <= tolerance * float(want.norm()) + 1e-9
        assert abs(float(trainer.norm[r][0]) - length) <= tolerance * length + 1e-9 and int(trainer.count[r]) == 1
        # the first step of AdamW on g: m / (1 - b1) = g, v / (1 - b2) = g^2; with the kernel's own gradient and factor, so that only the step's errors count
        g = trainer.grad[r][:split].view(60, 24).double() * float(trainer.norm[r][1])
        want = before - 0.01 * g / (g.abs() + 1e-8)
        assert (trainer.table[r].double() - want).abs().max() <= 0.01 * 16 * 2.0 ** -24 + 2.0 ** -23 * float(before.abs().max())


def test_a_step_that_is_left_out(monkeypatch):
    """One rank's gradient holds an infinity: no parameter, momentum, moment or count of any rank changes; the step after it is an ordinary one."""
    import paper_1910_04940_amd as bl
    from data_parallel_step import BiasTrainer
    trainer = BiasTrainer(ranks=3, tokens=200, vocab=60, dim=24, experts=8)
    trainer.step()
    state = lambda: [t.clone() for part in (trainer.table, trainer.router, trainer.momentum, trainer.count, *trainer.moments, *trainer.scales) for t in part]   # noqa: E731
    before, real = state(), bl.blink_allreduce

    def spoiled(bufs, n, dtype, *rest):
        if dtype == bl.BLINK_FP32:
            bufs[1][5] = float("inf")
        real(bufs, n, dtype, *rest)
    monkeypatch.setattr(bl, "blink_allreduce", spoiled)
    trainer.step()
    assert all(torch.isnan(n[1]) for n in trainer.norm)
    for a, b in zip(before, state()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    monkeypatch.setattr(bl, "blink_allreduce", real)
    trainer.step()
    assert int(trainer.count[0]) == 2 and all(torch.isfinite(t).all() for t in trainer.table + trainer.router + trainer.momentum)
    assert not any(torch.equal(a, b) for a, b in zip(before[:6], state()[:6]))
