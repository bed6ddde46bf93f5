"""A router's choice, its loss and its gradient against the definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_1910_04940_amd as bl  # noqa: E402

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
BALANCE, Z = 0.05, 0.02


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Run:
    def __init__(self, logits, k, keep=None, normalize=False, grad_weights=None, grad_loss=None, counts=None):
        t, e = logits.shape
        self.chosen = torch.full((t, k), 77, dtype=torch.int32, device="cuda")
        self.weights = torch.full((t, k), 7.0, device="cuda")
        self.counts = torch.full((e + 1,), 9, dtype=torch.int32, device="cuda")
        self.sums = torch.full((e + 1,), 9.0, device="cuda")
        self.loss = torch.full((3,), 9.0, device="cuda")
        self.grad = torch.full((t, e), 9.0, device="cuda").to(logits.dtype)
        work = torch.full((max(1, bl.blink_route_workspace(t, e)),), 255, dtype=torch.uint8, device="cuda")
        bl.blink_route(logits, k, self.chosen, self.weights, self.counts, self.sums, work, keep, normalize, _stream())
        bl.blink_route_loss(self.counts, self.sums, k, self.loss, BALANCE, Z, _stream())
        bl.blink_route_gradient(logits, k, self.chosen, self.counts if counts is None else counts, self.grad, keep, normalize, grad_weights, grad_loss, BALANCE, Z,
                                _stream())


def _want(logits, k, keep=None, normalize=False, grad_weights=None, up=1.0):
    """In 64 bits on the host, the choice by counting who comes before."""
    x = logits.cpu().double()
    t, e = x.shape
    counted = (x > -math.inf).any(1)
    if keep is not None:
        counted &= keep.cpu().bool()
    x = torch.where(counted[:, None], x, -math.inf)
    most = torch.where(counted, x.amax(1), 0.0)
    pw = torch.exp(x - most[:, None])
    p = pw / pw.sum(1, keepdim=True).clamp(min=1e-300)
    lse = torch.where(counted, most + torch.log(pw.sum(1).clamp(min=1e-300)), 0.0)
    order = torch.sort(x, dim=1, descending=True, stable=True)
    chosen = torch.where(order.values[:, :k] > -math.inf, order.indices[:, :k], -1)
    hit = torch.zeros(t, e, dtype=torch.float64)
    rows = torch.arange(t)
    up_w = torch.zeros(t, e, dtype=torch.float64)
    weights = torch.zeros(t, k, dtype=torch.float64)
    for j in range(k):
        real = chosen[:, j] >= 0
        hit[rows[real], chosen[real, j]] = 1
        weights[real, j] = p[rows[real], chosen[real, j]]
    if normalize:
        total = weights.sum(1, keepdim=True).clamp(min=1e-300)
        weights = weights / total
    if grad_weights is not None:
        g = grad_weights.cpu().double()
        if normalize:
            g = (g - (g * weights).sum(1, keepdim=True)) / total
        for j in range(k):
            real = chosen[:, j] >= 0
            up_w[rows[real], chosen[real, j]] = g[real, j]
    n = int(counted.sum())
    counts = torch.cat((hit.sum(0), torch.tensor([float(n)], dtype=torch.float64)))
    sums = torch.cat((p.sum(0), (lse ** 2).sum()[None]))
    m = max(n, 1)
    balance, z = BALANCE * e / k * (counts[:e] * sums[:e]).sum() / m / m, Z * sums[e] / m
    d = up * BALANCE * e / k * counts[:e] / m / m + up_w
    dot = (p * d).sum(1, keepdim=True)
    tail = 2 * up * Z / m * lse[:, None]
    grad = p * (d - dot + tail)
    # how far a value may be off: exponents are off by 3 units of the distance from the largest logit, a sum of e numbers by e units
    reach = torch.where(torch.isfinite(x), most[:, None] - x, 0.0).amax(1, keepdim=True)
    rel = (6 * reach + e + 16) * 2.0 ** -24
    if normalize:
        rel = 2 * rel + (k + 4) * 2.0 ** -24
    size = p * (d.abs() + (p * d.abs()).sum(1, keepdim=True) + tail.abs())
    if grad_weights is not None and normalize:   # (g - dot) / total: what cancels counts in full
        size = size + p * ((grad_weights.cpu().double().abs().amax(1, keepdim=True) * 2 / total) * 2)
    return dict(chosen=chosen.int(), weights=weights, counts=counts.int(), sums=sums, loss=torch.stack((balance + z, balance, z)), grad=grad, rel=rel,
                size=size, p=p, n=m, lse=lse)


def _check(run, want, dtype):
    assert torch.equal(run.chosen.cpu(), want["chosen"])
    assert torch.equal(run.counts.cpu(), want["counts"])
    assert ((run.weights.cpu().double() - want["weights"]).abs() <= want["rel"] * want["weights"] + 2.0 ** -120).all()
    e = want["p"].shape[1]
    worst = float(want["rel"].max())
    # sums of n positive numbers in any order, each off by its own error; the logits' sizes to the square
    lse = want["lse"].abs()
    off = (run.sums.cpu().double() - want["sums"]).abs()
    assert (off[:e] <= (worst + want["n"] * 2.0 ** -24) * want["sums"][:e] + 2.0 ** -120).all()
    assert off[e] <= (want["n"] * 2.0 ** -24) * want["sums"][e] + float((2 * lse * (2.0 ** -22 * lse + e * 2.0 ** -23)).sum()) + 2.0 ** -120
    tolerance = worst + (want["n"] + 8) * 2.0 ** -24 + e * 2.0 ** -20
    assert ((run.loss.cpu().double() - want["loss"]).abs() <= tolerance * want["loss"].abs() + 1e-30).all()
    off = (run.grad.cpu().double() - want["grad"]).abs()
    allowed = 4 * want["rel"] * want["size"] + UNIT[dtype] * want["grad"].abs() * 1.01 + TINY[dtype]
    assert (off <= allowed).all(), (off - allowed).max()


def _logits(t, e, dtype, seed, spread=2.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (spread * torch.randn(t, e, generator=g, device="cuda")).to(dtype)


EXPERTS = [(1, 1), (2, 1), (3, 3), (7, 2), (8, 8), (9, 4), (16, 2), (31, 5), (60, 4), (64, 8), (100, 3), (128, 1), (200, 12), (256, 8), (257, 2), (512, 8), (513, 6),
           (1000, 4), (1024, 10)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("e,k", EXPERTS)
def test_experts(e, k, dtype):
    for t, normalize in ((1, False), (333, True)):
        logits = _logits(t, e, dtype, e + k)
        g = torch.randn(t, k, device="cuda", generator=torch.Generator("cuda").manual_seed(4))
        keep = torch.rand(t, device="cuda", generator=torch.Generator("cuda").manual_seed(5)) < 0.8 if t > 1 else None
        up = torch.tensor([0.5], device="cuda")
        run = Run(logits, k, keep, normalize, g, up)
        _check(run, _want(logits, k, keep, normalize, g, 0.5), dtype)


@pytest.mark.parametrize("t", [1, 2, 63, 64, 65, 1000, 4097, 70_001])
def test_tokens(t):
    logits = _logits(t, 48, torch.bfloat16, t)
    run = Run(logits, 3)
    _check(run, _want(logits, 3), torch.bfloat16)
    again = Run(logits, 3)
    for name in ("chosen", "weights", "counts", "sums", "loss", "grad"):
        assert torch.equal(getattr(run, name), getattr(again, name))


def test_no_tokens():
    run = Run(torch.empty(0, 8, device="cuda"), 2)
    assert (run.counts == 0).all() and (run.sums == 0).all() and (run.loss == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_equal_logits_go_to_the_lowest_index(dtype):
    logits = torch.zeros(70, 24, device="cuda").to(dtype)
    logits[1::2, 5] = 1.0
    logits[:, 20] = -0.0     # equal to 0
    run = Run(logits, 4)
    assert run.chosen[0].tolist() == [0, 1, 2, 3] and run.chosen[1].tolist() == [5, 0, 1, 2]
    _check(run, _want(logits, 4), dtype)


def test_masked_experts_and_rows_with_nothing_left():
    logits = _logits(300, 40, torch.float32, 3)
    logits[:, 7] = -math.inf
    logits[10] = -math.inf
    logits[11, 2:] = -math.inf           # two experts for four places
    logits[12] = torch.finfo(torch.float32).min
    logits[13, 1:] = torch.finfo(torch.float32).min
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[20:25] = False
    g = torch.randn(300, 4, device="cuda", generator=torch.Generator("cuda").manual_seed(6))
    for normalize in (False, True):
        run = Run(logits, 4, keep, normalize, g)
        assert run.chosen[10].tolist() == [-1] * 4 and run.chosen[11, 2:].tolist() == [-1, -1] and run.chosen[21].tolist() == [-1] * 4
        assert (run.grad[10] == 0).all() and (run.grad[20:25] == 0).all() and (run.weights[20:25] == 0).all()
        assert (run.counts[7] == 0) and run.counts[40] == 294
        assert all(torch.isfinite(v).all() for v in (run.weights, run.sums[:40], run.grad))
        assert run.sums[40] == math.inf      # 3.4e38 squared
        assert torch.equal(run.chosen.cpu(), _want(logits, 4, keep, normalize, g)["chosen"])
        some = torch.ones(300, dtype=torch.bool, device="cuda")   # (the lowest numbers' squares pass the range of a 32-bit float)
        some[12:14] = False
        logits2 = torch.where(some[:, None], logits, 0.0)
        run = Run(logits2, 4, keep, normalize, g)
        _check(run, _want(logits2, 4, keep, normalize, g), torch.float32)


def test_nothing_kept():
    logits = _logits(50, 8, torch.bfloat16, 3)
    run = Run(logits, 2, torch.zeros(50, dtype=torch.uint8, device="cuda"))
    assert (run.counts == 0).all() and (run.loss == 0).all() and (run.grad == 0).all() and (run.chosen == -1).all()


def test_nan_and_infinity():
    """In rows that are left out they stay out; in a row that counts they show, and are not chosen."""
    logits = _logits(64, 16, torch.float32, 3)
    keep = torch.ones(64, dtype=torch.bool, device="cuda")
    keep[5] = keep[6] = False
    logits[5, 3] = math.nan
    logits[6, 3] = math.inf
    clean = torch.where(keep[:, None], logits, 0.0)
    nan_up = torch.full((1,), 1.0, device="cuda")
    run = Run(logits, 2, keep, False, None, nan_up)
    _check(run, _want(clean, 2, keep), torch.float32)
    bad = logits.clone()
    bad[7, 3] = math.nan
    run = Run(bad, 2, keep)
    assert 3 not in run.chosen[7].tolist() and (run.chosen[7] >= 0).all()
    assert torch.isnan(run.sums[:16]).all() and torch.isnan(run.loss[0]) and torch.isnan(run.grad[7]).all() and (run.grad[5:7] == 0).all()
    up = torch.full((1,), math.nan, device="cuda")
    run = Run(clean, 2, keep, False, None, up)
    assert (run.grad[5:7] == 0).all() and torch.isnan(run.grad[0]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_views(dtype):
    t, e, k = 130, 24, 3
    wide = _logits(t, e + 11, dtype, 8)
    for shift in (0, 1, 8):
        view = wide[:, shift:shift + e]
        run, plain = Run(view, k), Run(view.contiguous(), k)
        for name in ("chosen", "weights", "counts", "sums", "loss", "grad"):
            assert torch.equal(getattr(run, name), getattr(plain, name))


def test_logits_past_32_bits():
    """More than 2^31 logits: the last tokens as they come out of a call of their own, given the same counts."""
    t, e, k, last = 2_200_000, 1000, 2, 700
    g = torch.Generator("cuda").manual_seed(5)
    part = (2 * torch.randn(t // 20, e, generator=g, device="cuda")).bfloat16()
    logits = part.repeat(20, 1)
    run = Run(logits, k)
    tail = Run(logits[-last:].contiguous(), k, counts=run.counts)
    assert torch.equal(run.chosen[-last:], tail.chosen) and torch.equal(run.weights[-last:], tail.weights) and torch.equal(run.grad[-last:], tail.grad)
    once = Run(part, k)
    assert torch.equal(run.counts, once.counts * 20)
    assert ((run.sums - once.sums * 20).abs() <= 2 * t / 1024 * 2.0 ** -24 * run.sums).all()     # a workgroup adds up to t / 1024 of them


def test_ranks_add_up_to_the_whole_batch():
    """Counts and sums of four ranks, summed by the collectives, give the whole batch's loss and every rank's part of its gradient."""
    import synth_inputs as si
    e, k, ranks, each = 60, 4, 4, 501
    logits = _logits(ranks * each, e, torch.float32, 21)
    whole = Run(logits, k)
    parts = [Run(logits[r * each:(r + 1) * each], k) for r in range(ranks)]
    top = si.complete_graph(ranks)
    trees = bl.blink_pack_trees(top.k, top.src, top.dst, top.cap, 0)
    sched = bl.blink_make_schedule(trees, bl.BLINK_OP_ALLREDUCE, e + 1, 1 << 10)
    sums_sched = bl.blink_make_schedule(trees, bl.BLINK_OP_ALLREDUCE, e + 1, 1 << 10)
    counts, sums = ([torch.empty(64, dtype=d, device="cuda")[:e + 1] for _ in range(ranks)] for d in (torch.int32, torch.float32))
    for r, part in enumerate(parts):
        counts[r].copy_(part.counts)
        sums[r].copy_(part.sums)
    bl.blink_allreduce(counts, e + 1, bl.BLINK_INT32, sched, _stream())
    bl.blink_allreduce(sums, e + 1, bl.BLINK_FP32, sums_sched, _stream())
    loss = torch.empty(3, device="cuda")
    for r in range(ranks):
        assert torch.equal(counts[r], whole.counts)
        bl.blink_route_loss(counts[r], sums[r], k, loss, BALANCE, Z, _stream())
        assert torch.allclose(loss, whole.loss, rtol=(ranks * each + e + 16) * 2.0 ** -24, atol=0)
        mine = Run(logits[r * each:(r + 1) * each], k, counts=counts[r])
        assert torch.equal(mine.grad, whole.grad[r * each:(r + 1) * each])


def test_gradient_against_differences():
    """d(loss + sum g w) by central differences of the definition in 64 bits, the choice and the counts held."""
    t, e, k = 12, 10, 3
    for normalize in (False, True):
        logits = _logits(t, e, torch.float32, 31, 1.0)
        g = torch.randn(t, k, device="cuda", generator=torch.Generator("cuda").manual_seed(7))
        run = Run(logits, k, None, normalize, g)
        chosen, counts, n = run.chosen.cpu().long(), run.counts.cpu().double(), t

        def f(x):
            p = torch.softmax(x, 1)
            w = p.gather(1, chosen)
            w = w / w.sum(1, keepdim=True) if normalize else w
            return BALANCE * e / k / n / n * (counts[:e] * p.sum(0)).sum() + Z / n * (torch.logsumexp(x, 1) ** 2).sum() + (g.cpu().double() * w).sum()
        x = logits.cpu().double()
        h = 1e-4      # the third derivative times h^2 is below 1e-7
        for i in range(t):
            for j in range(e):
                up, down = x.clone(), x.clone()
                up[i, j] += h
                down[i, j] -= h
                assert abs(float((f(up) - f(down)) / (2 * h)) - float(run.grad[i, j])) < 1e-6


def test_in_a_graph():
    logits = _logits(5000, 64, torch.bfloat16, 41)
    k = 4
    want = Run(logits, k)
    work = torch.empty(bl.blink_route_workspace(5000, 64), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(v) for v in (want.chosen, want.weights, want.counts, want.sums, want.loss, want.grad)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bl.blink_route(logits, k, out[0], out[1], out[2], out[3], work, stream=_stream())
        bl.blink_route_loss(out[2], out[3], k, out[4], BALANCE, Z, _stream())
        bl.blink_route_gradient(logits, k, out[0], out[2], out[5], balance=BALANCE, z=Z, stream=_stream())
    for _ in range(3):
        for o in out:
            o.fill_(1)
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(out, (want.chosen, want.weights, want.counts, want.sums, want.loss, want.grad)):
            assert torch.equal(o, w)
