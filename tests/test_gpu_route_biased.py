"""The router with scores, a bias and groups, its gradient and the bias's step against the definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_1910_04940_amd as bl  # noqa: E402

F32, B16, H16 = torch.float32, torch.bfloat16, torch.float16
HALF = {F32: 2.0 ** -24, B16: 2.0 ** -8, H16: 2.0 ** -11}      # half a step, relative
TINY = {F32: 2.0 ** -126, B16: 2.0 ** -126, H16: 2.0 ** -24}
SCALE = 2.5


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Run:
    def __init__(self, logits, k, bias=None, keep=None, groups=1, kept=1, scores="sigmoid", normalize=False, grad_weights=None):
        t, e = logits.shape
        self.chosen = torch.full((t, k), 77, dtype=torch.int32, device="cuda")
        self.weights = torch.full((t, k), 7.0, device="cuda")
        self.counts = torch.full((e + 1,), 9, dtype=torch.int32, device="cuda")
        self.grad = torch.full((t, e), 9.0, device="cuda").to(logits.dtype)
        work = torch.full((max(1, bl.blink_route_biased_workspace(t, e)),), 255, dtype=torch.uint8, device="cuda")
        bl.blink_route_biased(logits, k, self.chosen, self.weights, self.counts, work, bias, keep, groups, kept, scores, normalize, SCALE, _stream())
        if grad_weights is not None:
            bl.blink_route_biased_gradient(logits, k, self.chosen, grad_weights, self.grad, keep, scores, normalize, SCALE, _stream())


def _want(logits, k, bias=None, keep=None, groups=1, kept=1, scores="sigmoid", normalize=False, grad_weights=None):
    """In 64 bits on the host, one expert of one group after the other."""
    x = logits.cpu().double()
    t, e = x.shape
    if keep is not None:
        x = torch.where(keep.cpu().bool()[:, None], x, -math.inf)
    b = torch.zeros(e, dtype=torch.float64) if bias is None else bias.cpu().double()
    fits = (x > -math.inf) & (b > -math.inf)
    if scores == "sigmoid":
        p = 1 / (1 + torch.exp(-x))
    else:
        most = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(most > -math.inf, most, 0.0))
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    a = torch.where(fits, p + b, -math.inf)
    size = e // groups
    if groups > 1:
        order = torch.sort(a.view(t, groups, size), dim=2, descending=True).values
        of = order[:, :, 0].clone()
        if size > 1:
            of += torch.where(order[:, :, 1] > -math.inf, order[:, :, 1], 0.0)
        best = torch.sort(of, dim=1, descending=True, stable=True).indices[:, :kept]
        stays = torch.zeros(t, groups, dtype=torch.bool).scatter_(1, best, True)
        a = torch.where(stays.repeat_interleave(size, 1), a, -math.inf)
    order = torch.sort(a, dim=1, descending=True, stable=True)
    found = order.values[:, :k] > -math.inf
    chosen = torch.where(found, order.indices[:, :k], -1)
    counts = torch.zeros(e + 1, dtype=torch.float64)
    counts.index_add_(0, chosen.clamp(min=0).reshape(-1), found.double().reshape(-1))
    counts[e] = found[:, 0].sum()
    # a sigmoid of far below 0 in a sum: all of them by the same factor, which keeps them in range
    at = chosen.clamp(min=0)
    xc = torch.where(found, x.gather(1, at), -math.inf)
    most = xc.amax(1, keepdim=True).clamp(max=0.0 if scores == "sigmoid" else math.inf)
    most = torch.where(most > -math.inf, most, 0.0)
    part = torch.exp(xc - most) / (1 + torch.exp(xc)) if scores == "sigmoid" else torch.exp(xc - most)
    part = torch.where(torch.isnan(part), 1.0, part)      # (far above 0)
    part = torch.where(xc > 700, 1.0, part)
    q = part / part.sum(1, keepdim=True).clamp(min=1e-300)
    s = torch.where(found, p.gather(1, at), 0.0)
    weights = SCALE * (q if normalize else s)
    # how far a weight may be off: an exponential by half a unit of its argument and 2 of its own, a sum of m numbers by m, a quotient by their sum
    whole = scores == "softmax" and not normalize
    far = torch.where(torch.isfinite(x), x.amax(1, keepdim=True) - x, 0.0).amax(1, keepdim=True) if whole else torch.where(found, (xc - most).abs(), 0.0).amax(1, keepdim=True)
    rel = (2 * (2 * far.clamp(max=110) + 8) + (e if whole else k) + 8) * 2.0 ** -24
    out = dict(chosen=chosen.int(), counts=counts.int(), weights=weights, rel=rel)
    if grad_weights is None:
        return out
    g = torch.where(found, grad_weights.cpu().double(), 0.0)
    dx = torch.zeros(t, e, dtype=torch.float64)
    size_of = torch.zeros(t, e, dtype=torch.float64)      # of what cancels
    not_p = torch.where(found, 1 / (1 + torch.exp(xc)), 0.0)
    if normalize:
        # g less its mean by exact differences: the kernel's 64-bit sums are as good
        d = SCALE * q * ((g[:, :, None] - g[:, None, :]) * q[:, None, :]).sum(2)
        # relative errors of the q shift the mean: by rel times the spread of g
        spread = SCALE * q * (g[:, :, None] - g[:, None, :]).abs().mul(q[:, None, :]).sum(2)
        # the kernel takes the mean of g off g, in 64 bits: sums of k products are off by k + 2 half units of 2^-53 of the largest g, which is all there
        # is where one q is within 2^-53 of 1; divided by 3 rel, which `size` is multiplied by
        spread += SCALE * q * (k + 3) * 2.0 ** -53 * g.abs().amax(1, keepdim=True) / (3 * rel)
    else:
        d = SCALE * g * (s if scores == "sigmoid" else torch.ones_like(s))
        spread = d.abs()
    if scores == "sigmoid":
        d, spread = d * not_p, spread * not_p
        if not normalize:      # a p below the normal numbers of 32 bits may be 0, and p times (scale g) is then all off
            spread = spread + torch.where(s < 2.0 ** -126, 2.0 ** -126 * SCALE * g.abs() / (3 * rel), 0.0)
    dx.scatter_add_(1, at, torch.where(found, d, 0.0))
    size_of.scatter_add_(1, at, torch.where(found, spread, 0.0))
    if whole:
        dx, size_of = p * (dx - (p * dx).sum(1, keepdim=True)), p * (size_of + (p * size_of).sum(1, keepdim=True))
        # a p below the normal numbers of 32 bits may be 0, and what it would be times (d less a mean of d) is then all off
        size_of += torch.where(p < 2.0 ** -126, 2.0 ** -126 * 2 * SCALE * g.abs().amax(1, keepdim=True) / (3 * rel), 0.0)
    return out | dict(grad=torch.where(found[:, :1], dx, 0.0), size=size_of)


def _check(run, want, dtype):
    assert torch.equal(run.chosen.cpu(), want["chosen"])
    assert torch.equal(run.counts.cpu(), want["counts"])
    off = (run.weights.cpu().double() - want["weights"]).abs()
    assert (off <= want["rel"] * want["weights"] + 2.0 ** -120).all(), (off / want["weights"]).max()
    if "grad" in want:
        off = (run.grad.cpu().double() - want["grad"]).abs()
        # a gradient has up to three factors that are as far off as a weight
        assert (off <= 3 * want["rel"] * want["size"] + 1.01 * HALF[dtype] * want["grad"].abs() + TINY[dtype]).all(), off.max()


def _logits(t, e, dtype, seed, spread=1.5):
    g = torch.Generator("cuda").manual_seed(seed)
    return (spread * torch.randn(t, e, generator=g, device="cuda") + torch.randn(e, generator=g, device="cuda")).to(dtype)


def _bias(e, seed, size=0.1):
    return size * torch.randn(e, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def _randn(*shape, seed=4):
    return torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


SHAPES = [(1, 1, 1, 1), (2, 1, 2, 1), (3, 3, 1, 1), (8, 4, 4, 2), (9, 4, 3, 2), (16, 2, 16, 3), (31, 5, 1, 1), (30, 10, 3, 1), (60, 4, 6, 3), (60, 6, 60, 8), (64, 6, 1, 1),
          (64, 8, 8, 4), (64, 9, 64, 9), (100, 3, 10, 7), (128, 8, 4, 2), (160, 6, 8, 3), (200, 12, 5, 2), (256, 8, 8, 4), (256, 8, 1, 1), (256, 10, 64, 5),
          (258, 2, 6, 5), (384, 8, 3, 2), (512, 16, 16, 4), (513, 6, 27, 3), (1000, 4, 50, 10), (1024, 10, 32, 8), (1024, 70, 2, 1)]


@pytest.mark.parametrize("dtype", [F32, B16, H16])
@pytest.mark.parametrize("e,k,groups,kept", SHAPES)
def test_shapes(e, k, groups, kept, dtype):
    for t, scores, normalize in ((1, "sigmoid", True), (333, "sigmoid", True), (97, "sigmoid", False), (129, "softmax", True), (65, "softmax", False)):
        logits, bias, g = _logits(t, e, dtype, e + k), _bias(e, k), _randn(t, k)
        keep = torch.rand(t, device="cuda", generator=torch.Generator("cuda").manual_seed(5)) < 0.8 if t % 2 and t > 1 else None
        arguments = (logits, k, bias, keep, groups, kept, scores, normalize, g)
        _check(Run(*arguments), _want(*arguments), dtype)


@pytest.mark.parametrize("t", [0, 1, 2, 15, 16, 17, 1000, 4097, 70_001])
def test_tokens(t):
    arguments = (_logits(t, 64, B16, t), 4, _bias(64, 1), None, 8, 3, "sigmoid", True, _randn(t, 4))
    run = Run(*arguments)
    if t == 0:
        assert (run.counts == 0).all()
        return
    _check(run, _want(*arguments), B16)
    again = Run(*arguments)
    for name in ("chosen", "weights", "counts", "grad"):
        assert torch.equal(getattr(run, name), getattr(again, name))


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_equal_scores_go_to_the_lowest_index(scores, dtype):
    """All logits the same (a router that starts from zeros), a few the same, and the same scores from different logits and biases."""
    t, e = 70, 64
    logits = torch.zeros(t, e, device="cuda").to(dtype)
    logits[1::2, 50] = 1.0
    logits[:, 40] = -0.0
    logits[2::3] = torch.randint(-2, 3, logits[2::3].shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
    for bias in (None, torch.zeros(e, device="cuda"), 0.25 * torch.randint(-1, 2, (e,), device="cuda", generator=torch.Generator("cuda").manual_seed(2))):
        for groups, kept in ((1, 1), (8, 3), (16, 2), (64, 9)):
            arguments = (logits, 5, bias, None, groups, kept, scores, True, _randn(t, 5))
            if kept * e // groups < 5:
                continue
            _check(Run(*arguments), _want(*arguments), dtype)
    run = Run(logits, 5, None, None, 8, 3, scores)
    assert run.chosen[0].tolist() == [0, 1, 2, 3, 4] and run.chosen[1].tolist()[0] == 50


@pytest.mark.parametrize("groups,kept", [(1, 1), (8, 4), (5, 2)])
def test_logits_that_are_often_equal(groups, kept):
    """Multiples of 1/8 without a bias: most tokens have equal experts among their first, in one lane's neighbours, in several lanes, at the end of the choice."""
    for e, dtype in ((80, F32), (80, B16), (240, B16), (1000, H16)):
        logits = (8 * _logits(5000, e, F32, e)).round().div(8).to(dtype)
        e_groups = groups if e % groups == 0 else 1
        for bias in (None, torch.zeros(e, device="cuda"), torch.full((e,), -0.5, device="cuda")):
            arguments = (logits, 8, bias, None, e_groups, min(kept, e_groups), "sigmoid", True)
            _check(Run(*arguments), _want(*arguments), dtype)


@pytest.mark.parametrize("groups,kept", [(1, 1), (8, 4)])
@pytest.mark.parametrize("e", [64, 256])
def test_scores_that_all_but_tie(e, groups, kept):
    """Differences of 2^-33 and more of a score: a 32-bit sum of score and bias shows none of those below 2^-24."""
    t, g = 500, torch.Generator("cuda").manual_seed(3)
    some = torch.rand(8, generator=g, device="cuda", dtype=torch.float64) * 4 - 2
    base = some[torch.randint(0, 8, (e,), generator=g, device="cuda")]
    # a logit and a bias that sum to about the same score for all experts of a kind: the bias makes up for what 32 bits cannot
    x = base.float().expand(t, e) + torch.randint(-64, 65, (t, e), generator=g, device="cuda") * 2.0 ** -20
    p = torch.sigmoid(base.float().double())
    bias = (0.75 - p).float()
    for scores in ("sigmoid", "softmax"):
        arguments = (x, 8, bias, None, groups, kept, scores, True)
        want = _want(*arguments)
        _check(Run(*arguments), want, F32)
    a = torch.sigmoid(x.double()) + bias.double()
    top = torch.sort(a, dim=1, descending=True).values[:, :9]
    assert float((top[:, :-1] - top[:, 1:]).median()) < 2.0 ** -20      # (it is what it says)


def test_far_logits():
    """Scores that are next to 0 and next to 1, and weights from them."""
    t, e = 64, 32
    for low, high in ((-120.0, -80.0), (-1000.0, -300.0), (-20.0, -15.0), (40.0, 400.0), (-30.0, 30.0)):
        x = low + (high - low) * torch.rand(t, e, device="cuda", generator=torch.Generator("cuda").manual_seed(6))
        for scores in ("sigmoid", "softmax"):
            for normalize in (True, False):
                if low == -1000.0 and scores == "sigmoid":
                    x[:, 3] = -700.0 + torch.arange(t, device="cuda") * 0.5      # (below, a 64-bit exponential is 0 and all are equal)
                arguments = (x, 3, None, None, 4, 2, scores, normalize, _randn(t, 3))
                want = _want(*arguments)
                run = Run(*arguments)
                assert torch.isfinite(run.weights).all() and torch.isfinite(run.grad).all()
                if low != -1000.0 or scores == "softmax":
                    _check(run, want, F32)


def test_experts_out_of_service_and_rows_with_nothing_left():
    t, e, k = 300, 40, 4
    logits = _logits(t, e, F32, 3)
    logits[:, 7] = -math.inf
    logits[10] = -math.inf
    logits[11, 2:] = -math.inf               # two experts for four places
    logits[12] = torch.finfo(F32).min        # the lowest number is a number
    logits[13, 5:] = -math.inf               # a group of five is left
    logits[14, 1:] = -math.inf
    bias = _bias(e, 1)
    bias[9] = -math.inf
    bias[10:15] = -math.inf                  # a whole group
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[20:25] = False
    for scores in ("sigmoid", "softmax"):
        for normalize in (False, True):
            arguments = (logits, k, bias, keep, 8, 3, scores, normalize, _randn(t, k))
            run = Run(*arguments)
            _check(run, _want(*arguments), F32)
            assert run.chosen[10].tolist() == [-1] * 4 and run.chosen[11].tolist()[2:] == [-1, -1] and run.chosen[14].tolist() == [0, -1, -1, -1]
            assert (run.grad[10] == 0).all() and (run.grad[20:25] == 0).all() and (run.weights[20:25] == 0).all() and run.counts[7] == 0 and run.counts[9] == 0
            assert run.counts[40] == t - 6


def test_large_and_odd_biases():
    t, e = 100, 64
    logits = _logits(t, e, B16, 8)
    for bias in (1e30 * _randn(e), 1e-30 * _randn(e), torch.full((e,), 1e20, device="cuda"), -5.0 + _randn(e)):
        arguments = (logits, 6, bias, None, 8, 4, "sigmoid", True)
        _check(Run(*arguments), _want(*arguments), B16)
    bias = _bias(e, 2)
    bias[5], bias[6] = math.nan, math.inf
    run = Run(logits, 6, bias)
    assert (run.chosen[:, 0] == 6).all() and run.counts[5] == 0


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_nan_and_infinity(scores):
    """In rows that are left out they stay out; in a row that counts they show, and nothing is chosen."""
    logits = _logits(64, 16, F32, 3)
    keep = torch.ones(64, dtype=torch.bool, device="cuda")
    keep[5] = keep[6] = False
    logits[5, 3] = math.nan
    logits[6, 3] = math.inf
    clean = torch.where(keep[:, None], logits, 0.0)
    for normalize in (False, True):
        g = _randn(64, 2)
        _check(Run(logits, 2, None, keep, 4, 2, scores, normalize, g), _want(clean, 2, None, keep, 4, 2, scores, normalize, g), F32)
        bad = logits.clone()
        bad[7, 3] = math.nan
        run = Run(bad, 2, None, keep, 4, 2, scores, normalize, g)
        assert run.chosen[7].tolist() == [-1, -1] and torch.isnan(run.weights[7]).all() and (run.grad[7] == 0).all() and run.counts[16] == 61
        bad[7, 3] = math.inf
        run = Run(bad, 2, None, keep, 1, 1, scores, normalize, g)
        assert (run.chosen[7, 0] == 3) == (scores == "sigmoid") and torch.isnan(run.weights[7]).all() == (scores == "softmax")
        assert torch.isfinite(run.grad).all()


@pytest.mark.parametrize("dtype", [F32, B16])
def test_views(dtype):
    t, e, k = 130, 24, 3
    wide = _logits(t, e + 11, dtype, 8)
    for shift in (0, 1, 8):
        view = wide[:, shift:shift + e]
        for scores in ("sigmoid", "softmax"):
            run, plain = (Run(x, k, _bias(e, 1), None, 4, 2, scores, False, _randn(t, k)) for x in (view, view.contiguous()))
            for name in ("chosen", "weights", "counts", "grad"):
                assert torch.equal(getattr(run, name), getattr(plain, name))
    out = torch.full((t, e + 5), 7.0, device="cuda").to(dtype)
    run = Run(wide[:, :e], k, grad_weights=_randn(t, k))
    bl.blink_route_biased_gradient(wide[:, :e], k, run.chosen, _randn(t, k), out[:, 2:2 + e], scale=SCALE, stream=_stream())
    assert torch.equal(out[:, 2:2 + e], run.grad) and (out[:, :2] == 7).all() and (out[:, 2 + e:] == 7).all()


def test_logits_past_32_bits():
    """More than 2^31 logits: the last tokens as they come out of a call of their own."""
    t, e, k, last = 2_200_000, 1000, 2, 700
    part = (2 * torch.randn(t // 20, e, generator=torch.Generator("cuda").manual_seed(5), device="cuda")).bfloat16()
    logits, bias, g = part.repeat(20, 1), _bias(e, 1), _randn(t, k)
    run = Run(logits, k, bias, None, 20, 4, "sigmoid", True, g)
    tail = Run(logits[-last:].contiguous(), k, bias, None, 20, 4, "sigmoid", True, g[-last:].contiguous())
    for name in ("chosen", "weights", "grad"):
        assert torch.equal(getattr(run, name)[-last:], getattr(tail, name))
    assert torch.equal(run.counts, Run(part, k, bias, None, 20, 4, "sigmoid", True).counts * 20)


def test_gradient_against_differences():
    """d(sum g w) by central differences of the definition in 64 bits, the choice held."""
    t, e, k = 12, 12, 3
    for scores in ("sigmoid", "softmax"):
        for normalize in (False, True):
            logits, g = _logits(t, e, F32, 31, 1.0), _randn(t, k, seed=7)
            run = Run(logits, k, _bias(e, 3), None, 4, 2, scores, normalize, g)
            chosen = run.chosen.cpu().long()

            def f(x):
                p = (torch.sigmoid(x) if scores == "sigmoid" else torch.softmax(x, 1)).gather(1, chosen)
                return SCALE * (g.cpu().double() * (p / p.sum(1, keepdim=True) if normalize else p)).sum()
            x = logits.cpu().double()
            h = 1e-4      # the third derivative times h^2 is below 1e-7
            for i in range(t):
                for j in range(e):
                    up, down = x.clone(), x.clone()
                    up[i, j] += h
                    down[i, j] -= h
                    assert abs(float((f(up) - f(down)) / (2 * h)) - float(run.grad[i, j])) < 1e-6


@pytest.mark.parametrize("e", [1, 2, 60, 256, 257, 1000, 1024])
def test_bias_step(e):
    g = torch.Generator("cuda").manual_seed(e)
    counts = torch.randint(0, 50, (e + 1,), generator=g, device="cuda", dtype=torch.int32)
    counts[::3] = 25
    bias, out = _randn(e), torch.full((e,), 9.0, device="cuda")
    for c in (counts, torch.full_like(counts, 7), torch.zeros_like(counts), counts * 40_000_000):
        bl.blink_route_bias(c, bias, out, 0.125, _stream())
        n = c[:e].cpu().long()
        assert torch.equal(out.cpu(), bias.cpu() + 0.125 * torch.sign(n.sum() - e * n).float())
    bl.blink_route_bias(counts, bias, bias, -0.125, _stream())      # in place
    n = counts[:e].cpu().long()
    assert torch.equal(bias.cpu(), _randn(e).cpu() - 0.125 * torch.sign(n.sum() - e * n).float())


def test_bias_balances_ranks():
    """Counts of four ranks, summed by the collectives, move every rank's bias alike, until the experts that all preferred have the mean."""
    import synth_inputs as si
    e, k, ranks, each = 32, 4, 4, 1000
    parts = [_logits(each, e, F32, r, 0.5) + 0.5 * _randn(e, seed=9) for r in range(ranks)]
    bias = [torch.zeros(e, device="cuda") for _ in range(ranks)]
    top = si.complete_graph(ranks)
    trees = bl.blink_pack_trees(top.k, top.src, top.dst, top.cap, 0)
    sched = bl.blink_make_schedule(trees, bl.BLINK_OP_ALLREDUCE, e + 1, 1 << 10)
    counts = [torch.empty(64, dtype=torch.int32, device="cuda")[:e + 1] for _ in range(ranks)]
    spread = []
    for step in range(60):
        for r in range(ranks):
            counts[r].copy_(Run(parts[r], k, bias[r], None, 4, 2).counts)
        bl.blink_allreduce(counts, e + 1, bl.BLINK_INT32, sched, _stream())
        whole = Run(torch.cat(parts), k, bias[0], None, 4, 2)
        for r in range(ranks):
            assert torch.equal(counts[r], whole.counts)
            bl.blink_route_bias(counts[r], bias[r], bias[r], 0.005, _stream())
            assert torch.equal(bias[r], bias[0])
        spread.append(float(counts[0][:e].float().std()))
    assert spread[-1] < 0.5 * spread[0]


def test_in_a_graph():
    logits, k, bias, g = _logits(5000, 64, B16, 41), 4, _bias(64, 1), _randn(5000, 4)
    work = torch.empty(bl.blink_route_biased_workspace(5000, 64), dtype=torch.uint8, device="cuda")
    new = lambda: [torch.empty(5000, k, dtype=torch.int32, device="cuda"), torch.empty(5000, k, device="cuda"), torch.empty(65, dtype=torch.int32, device="cuda"),   # noqa: E731
                   torch.empty_like(logits)]
    out, want = new(), new()
    biases = [bias.clone(), bias.clone()]

    def run(o, b):
        bl.blink_route_biased(logits, k, o[0], o[1], o[2], work, b, None, 8, 4, "sigmoid", True, 1.0, _stream())
        bl.blink_route_bias(o[2], b, b, 0.01, _stream())
        bl.blink_route_biased_gradient(logits, k, o[0], g, o[3], None, "sigmoid", True, 1.0, _stream())
    run(want, bias.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, biases[0])
    for _ in range(4):      # the bias moves from replay to replay
        for o in out:
            o.fill_(1)
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        run(want, biases[1])
        for o, w in zip(out + biases[:1], want + biases[1:]):
            assert torch.equal(o, w)


def test_streams():
    """Four at once: as many as there are hardware queues, so that streams of tests after this one fall to the queues that they fell to without it."""
    arguments = [(_logits(20_000, 60, B16, s), 4, _bias(60, s), None, 6, 3, "softmax", False, _randn(20_000, 4, seed=s)) for s in (1, 2, 3, 4)]
    runs, streams = [], [torch.cuda.Stream() for _ in arguments]
    torch.cuda.synchronize()
    for a, s in zip(arguments, streams):
        with torch.cuda.stream(s):
            runs.append(Run(*a))
    torch.cuda.synchronize()
    for a, run in zip(arguments, runs):
        _check(run, _want(*a), B16)


def test_both_ways_from_python(monkeypatch):
    """Through the native call module and through ctypes."""
    from paper_1910_04940_amd import operators
    arguments = (_logits(50, 24, F32, 1), 3, _bias(24, 1), torch.ones(50, dtype=torch.bool, device="cuda"), 4, 2, "softmax", True, _randn(50, 3))

    def all_of():
        run = Run(*arguments)
        bias = _bias(24, 1)
        bl.blink_route_bias(run.counts, bias, bias, 1, _stream())
        w, m, v = (torch.zeros(10, device="cuda") for _ in range(3))
        update = bl.blink_make_update([bias[:10]], [w], [m], [v])
        norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        work = torch.empty(bl.blink_gradient_norm_workspace(update), dtype=torch.uint8, device="cuda")
        bl.blink_gradient_norm(update, norm, work, 1, 0.5, step, _stream())
        bl.blink_adamw_step(update, step, 0.1, 0.9, 0.99, 1e-8, norm[1:], norm[:1], 3, _stream())
        return run.chosen, run.weights, run.counts, run.grad, bias, norm, step, w, m, v
    all_of()
    assert operators._operators, "the native call module is not built"
    longer = operators._rows
    monkeypatch.setattr(operators, "_rows", lambda *a: pytest.fail("the usual call went the longer way"))
    native = all_of()
    monkeypatch.setattr(operators, "_rows", longer)
    monkeypatch.setattr(operators, "_operators", {})
    for a, b in zip(native, all_of()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("e,k", [(5, 2), (8, 8), (64, 2), (64, 6), (256, 8), (1000, 20)])
def test_whole_softmax_with_a_leading_expert(e, k, dtype):
    """dx_i = p_i (d_i - sum_j p_j d_j) where one expert has nearly all: its d_i - mean is about (1 - p_i) d_i."""
    t = 60
    logits = _logits(t, e, F32, e, 0.5)
    lead = torch.arange(t, device="cuda") % e
    # 0 to 29.5 above the others; a chosen expert next to it, but for the last rows
    logits[torch.arange(t, device="cuda"), lead] = logits.amax(1) + 0.5 * torch.arange(t, device="cuda")
    logits = logits.to(dtype)
    g = _randn(t, k, seed=e)
    g[::7] = 1.0                              # nothing to gain by moving between the chosen
    run = Run(logits, k, None, None, 1, 1, "softmax", False, g)
    x = logits.cpu().double()
    p = torch.softmax(x, 1)
    d = torch.zeros(t, e, dtype=torch.float64).scatter_(1, run.chosen.cpu().long(), g.cpu().double())
    moved = p[:, :, None] * p[:, None, :] * (d[:, :, None] - d[:, None, :])
    want = SCALE * moved.sum(2)
    # a power is off by half a step of the difference of logits and 1.25 of its product with log2 e, and two of its own; the sum of the powers by their mean;
    # differences and sums are in 64 bits; five roundings to 32 follow, and the result's own
    far = (x.amax(1, keepdim=True) - x).clamp(max=110)
    off = (2.25 * far + 4) * 2.0 ** -24
    both = off[:, :, None] + off[:, None, :] + 2 * (p * off).sum(1)[:, None, None] + 6 * 2.0 ** -24
    allowed = SCALE * (moved.abs() * both).sum(2) + 1.01 * HALF[dtype] * want.abs() + TINY[dtype]
    # sums of e powers and k products in 64 bits; p below the normal numbers of 32 bits may be 0
    allowed += SCALE * d.abs().amax(1, keepdim=True) * ((e + k + 4) * 2.0 ** -53 * p + torch.where(p < 2.0 ** -126, 2.0 ** -125, 0.0))
    over = (run.grad.cpu().double() - want).abs() / allowed
    assert (over <= 1).all(), (float(over.max()), int(over.amax(1).argmax()))


@pytest.mark.parametrize("kept", [1, 2, 3])
def test_groups_that_lie_in_one_lane(kept):
    """Eight experts to a group and k = 8: one lane, which holds two groups, may have all that are chosen, and what comes after them."""
    for e, dtype in ((64, B16), (64, H16), (128, B16), (128, F32), (256, H16)):
        logits, bias = _logits(3000, e, dtype, e + kept), _bias(e, kept, 0.01)
        logits[1::2] = logits[1::2].mul(8).round().div(8)
        for scores in ("sigmoid", "softmax"):
            arguments = (logits, 8, bias, None, e // 8, kept, scores, True, _randn(3000, 8))
            _check(Run(*arguments), _want(*arguments), dtype)
