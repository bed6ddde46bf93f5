"""The norm of many gradients and the AdamW step against their definitions in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_1910_04940_amd as bl  # noqa: E402

F32, B16, H16, F8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
HALF = {F32: 2.0 ** -24, B16: 2.0 ** -8, H16: 2.0 ** -11}      # half a step, relative
TINY = {F32: 2.0 ** -149, B16: 2.0 ** -133, H16: 2.0 ** -24}   # one below the normal numbers
LR, B1, B2, EPS = 0.01, 0.9, 0.999, 1e-8
SIZES = [1, 3, 256, 255, 257, 0, 2048, 2049, 5000, 70_001]


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _work(update):
    return torch.full((max(1, bl.blink_gradient_norm_workspace(update)),), 255, dtype=torch.uint8, device="cuda")


class Tensors:
    """A list of them, packed at odd places in buffers of each type with a margin that nobody may touch, and their copies in 64 bits."""

    def __init__(self, sizes, weights=F32, grads=F32, master=False, eight=False, seed=0, gap=1, spread=1.0):
        g = torch.Generator("cuda").manual_seed(seed)
        randn = lambda n: torch.randn(n, generator=g, device="cuda")   # noqa: E731
        self.sizes, self.eight, self.flat, self.lists = sizes, eight, {}, {}

        def pack(name, dtype, values, places):
            total = sum(places) + gap * (len(places) + 1)
            flat = torch.full((total,), 7.0, device="cuda").to(dtype) if dtype != F8 else torch.full((total,), 7.0, device="cuda").to(F8)
            views, at = [], gap
            for n, v in zip(places, values):
                views.append(flat[at:at + n])
                views[-1].copy_(v)
                at += n + gap
            self.flat[name], self.lists[name] = flat, views

        blocks = [-(-n // 256) for n in sizes]
        pack("grads", grads, [spread * 1e-2 * randn(n) for n in sizes], sizes)
        w = [randn(n) for n in sizes]
        pack("weights", weights, w, sizes)
        if master:
            pack("masters", F32, w, sizes)
        if eight:
            pack("moments1", F8, [(150 * randn(n)).clamp(-448, 448).to(F8) for n in sizes], sizes)
            pack("moments2", F8, [(150 * randn(n)).abs().clamp(2.0 ** -9, 448).to(F8) for n in sizes], sizes)
            pack("scales1", F32, [1e-5 * torch.exp(randn(n)) for n in blocks], blocks)
            pack("scales2", F32, [1e-4 * torch.exp(randn(n)) for n in blocks], blocks)
        else:
            pack("moments1", F32, [1e-3 * randn(n) for n in sizes], sizes)
            pack("moments2", F32, [(1e-2 * randn(n)).square() for n in sizes], sizes)
        self.rates = [1.0 + 0.5 * (i % 2) for i in range(len(sizes))]
        self.decays = [0.1 * (i % 3) for i in range(len(sizes))]
        self.before = {k: [v.clone() for v in views] for k, views in self.lists.items()}
        self.update = bl.blink_make_update(self.lists["grads"], self.lists["weights"], self.lists["moments1"], self.lists["moments2"],
                                           masters=self.lists.get("masters"), scales1=self.lists.get("scales1"), scales2=self.lists.get("scales2"),
                                           rates=self.rates, decays=self.decays)

    def margins_untouched(self):
        for name, flat in self.flat.items():
            mine = torch.zeros(len(flat), dtype=torch.bool, device="cuda")
            for v in self.lists[name]:
                at = (v.data_ptr() - flat.data_ptr()) // flat.element_size()
                mine[at:at + v.numel()] = True
            assert (flat.float()[~mine] == 7).all(), name


def _mix(h):
    h = np.uint32(h)
    h = (h ^ h >> np.uint32(16)) * np.uint32(0x85ebca6b)
    h = (h ^ h >> np.uint32(13)) * np.uint32(0xc2b2ae35)
    return h ^ h >> np.uint32(16)


def _random(seed, t, tensor, n):
    with np.errstate(over="ignore"):
        at = np.arange(n, dtype=np.uint32)
        key = _mix(_mix(np.uint32((seed + 0x9e3779b9 * t) & 0xffffffff)) ^ np.uint32(tensor))
        h = _mix(_mix(key ^ at // np.uint32(256)) ^ at % np.uint32(256))
    return [torch.from_numpy((h >> np.uint32(s) & np.uint32(0xffff)).astype(np.float64) + 0.5).cuda() / 65536 for s in (0, 16)]


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -len(x) % 256)).view(-1, 256)


def _moments(T, i):
    m, v = T.before["moments1"][i].float().double(), T.before["moments2"][i].float().double()
    if T.eight:
        m = (_blocks(m) * T.before["scales1"][i].double()[:, None]).view(-1)[:len(m)]
        v = (_blocks(v) * T.before["scales2"][i].double()[:, None]).view(-1)[:len(v)].square()
    return m, v


def _check(T, t, scale=1.0, rate=1.0, seed=0):
    for i, n in enumerate(T.sizes):
        if n == 0:
            continue
        g = T.before["grads"][i].double() * scale
        m, v = _moments(T, i)
        # every product and sum below is rounded once: a moment is off by at most 4 half steps of its largest term (6 for v, whose parts are products of
        # products; the 8-bit number's product with its scale is one more, squared), its root by half of that and one
        part = (B1 * m.abs() + (1 - B1) * g.abs())
        m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
        off_m, off_v = 5 * 2.0 ** -24 * part + 2.0 ** -149, 8 * 2.0 ** -24 * v + 2.0 ** -148
        root = v.sqrt()
        by = LR * rate * T.rates[i]
        step = by * (m / (1 - B1 ** t)) / (root / math.sqrt(1 - B2 ** t) + EPS)
        # a divisor is off by 4 + 1 (its root) + 1 (times a factor of half a step's error) + 1, the quotient and the product with the rate by one each
        off_step = step.abs() * (10 + 1) * 2.0 ** -24 + by / (1 - B1 ** t) * off_m / (root / math.sqrt(1 - B2 ** t) + EPS)
        old = (T.before["masters"] if "masters" in T.before else T.before["weights"])[i].double()
        w = old * (1 - by * T.decays[i]) - step
        off_w = off_step + 3 * 2.0 ** -24 * (old.abs() + step.abs())
        if "masters" in T.lists:
            assert ((T.lists["masters"][i].double() - w).abs() <= off_w).all()
            assert torch.equal(T.lists["weights"][i], T.lists["masters"][i].to(T.lists["weights"][i].dtype))
        else:
            dtype = T.lists["weights"][i].dtype
            assert ((T.lists["weights"][i].double() - w).abs() <= off_w + (HALF[dtype] * (w.abs() + off_w) if dtype != F32 else 0) + TINY[dtype]).all()
        if not T.eight:
            assert ((T.lists["moments1"][i].double() - m).abs() <= off_m).all()
            assert ((T.lists["moments2"][i].double() - v).abs() <= off_v).all()
            continue
        up = _random(seed, t, i, n)
        for name, y, u, off in (("1", m, up[0], off_m), ("2", root, up[1], (5 * 2.0 ** -24) * root + 2.0 ** -75)):
            largest, far = _blocks(y.abs()).amax(1), _blocks(off).amax(1)
            scale_got = T.lists["scales" + name][i].double()
            assert ((scale_got - largest / 448).abs() <= far / 448 + 2 * 2.0 ** -24 * largest / 448).all()
            z = (_blocks(y) / scale_got.clamp(min=1e-300)[:, None]).view(-1)[:n]
            code = T.lists["moments" + name][i].float().double()
            unit = torch.exp2(torch.clamp(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))), min=-6) - 3)
            # |z| / unit is below 16, so 8 half steps of z are 2^-17 of a unit; the random numbers are 2^-16 apart
            near = (off / scale_got.clamp(min=1e-300).repeat_interleave(256)[:n] + 4 * 2.0 ** -24 * z.abs()) / unit + 2.0 ** -20
            low, high = (torch.floor(z.abs() / unit + u + d * near) * unit for d in (-1, 1))
            if name == "2":
                low, high = low.clamp(min=2.0 ** -9), high.clamp(min=2.0 ** -9)
            assert ((code.abs() == low) | (code.abs() == high) | (code.abs() == torch.clamp(high, max=448))).all()
            assert ((code == 0) | (torch.sign(code) == torch.sign(y))).all()
            # so that a rule other than this one would show: 5 half steps of terms that are up to four times 448 scales, where they cancel to less than 2^-6, are
            # 5 * 2^-24 * 1792 / 2^-9 = 0.27 of a unit; that much is left to few elements
            assert near.max() < 0.28 and near.mean() < 0.001
    T.margins_untouched()


KINDS = [(F32, F32, False), (F32, B16, False), (F32, H16, False), (B16, F32, False), (B16, B16, True), (B16, F32, True), (H16, F32, True), (H16, H16, False),
         (B16, H16, False), (H16, B16, True)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("weights,grads,master", KINDS)
def test_step(weights, grads, master, eight):
    for t, gap in ((1, 1), (1000, 0)):
        T = Tensors(SIZES, weights, grads, master, eight, seed=t, gap=gap)
        step = torch.tensor([t], dtype=torch.int32, device="cuda")
        scale, rate = torch.tensor([0.25], device="cuda"), torch.tensor([2.0], device="cuda")
        bl.blink_adamw_step(T.update, step, LR, B1, B2, EPS, scale, rate, 77, _stream())
        _check(T, t, 0.25, 2.0, 77)
        assert int(step) == t


@pytest.mark.parametrize("weights,grads,master,eight", [(F32, F32, False, False), (F32, B16, False, True), (B16, F32, True, True), (H16, B16, True, False),
                                                        (B16, F32, False, False)])
def test_lists_larger_than_the_caches(weights, grads, master, eight):
    """More than 256 MiB are read by another variant; here at odd places."""
    T = Tensors([1, 30_000_001, 257, 18_000_003], weights, grads, master, eight, seed=3)
    step, norm = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(2, device="cuda")
    bl.blink_gradient_norm(T.update, norm, _work(T.update), 0.5, 2.0, step, _stream())
    want = 2 * math.sqrt(sum(float(v.double().square().sum()) for v in T.lists["grads"]))
    assert abs(float(norm[0]) - want) <= 1.01 * 2.0 ** -24 * want
    bl.blink_adamw_step(T.update, step, LR, B1, B2, EPS, norm[1:], None, 78, _stream())
    _check(T, 1, float(norm[1]), 1.0, 78)


def test_norm_larger_than_the_caches():
    grads = [torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)) for n in (80_000_001, 5)]
    update = bl.blink_make_update(grads)
    norm = torch.empty(2, device="cuda")
    bl.blink_gradient_norm(update, norm, _work(update), stream=_stream())
    want = math.sqrt(sum(float(v.double().square().sum()) for v in grads))
    assert abs(float(norm[0]) - want) <= 1.01 * 2.0 ** -24 * want


@pytest.mark.parametrize("eight", [False, True])
def test_first_step_from_zeros(eight):
    T = Tensors([1, 300, 4097], eight=eight)
    for name in ("moments1", "moments2", "scales1", "scales2"):
        for v in T.lists.get(name, []) + T.before.get(name, []):
            v.zero_()
    bl.blink_adamw_step(T.update, torch.ones(1, dtype=torch.int32, device="cuda"), LR, B1, B2, EPS, seed=5, stream=_stream())
    _check(T, 1, seed=5)


@pytest.mark.parametrize("grads", [F32, B16, H16])
@pytest.mark.parametrize("sizes", [[1], [0, 5], [2048], [100_003], SIZES, [17] * 3000, [3_000_000, 1, 2_000_001]])
def test_norm(sizes, grads):
    g = torch.Generator("cuda").manual_seed(len(sizes))
    flat = (torch.randn(sum(sizes) + 3, generator=g, device="cuda")).to(grads)
    views, at = [], 3
    for n in sizes:
        views.append(flat[at:at + n])
        at += n
    update = bl.blink_make_update(views)
    want = 0.5 * float(flat[3:].double().norm())
    for most in (math.inf, 10 * want, 0.1 * want):
        norm, step, work = torch.full((2,), 9.0, device="cuda"), torch.full((1,), 41, dtype=torch.int32, device="cuda"), _work(update)
        bl.blink_gradient_norm(update, norm, work, most, 0.5, step, _stream())
        got, scale = norm.double().tolist()
        assert int(step) == 42
        assert abs(got - want) <= 1.01 * 2.0 ** -24 * want      # one rounding; sums in 64 bits
        assert abs(scale - 0.5 * min(1.0, most / want)) <= 1.01 * 2.0 ** -25
        again = torch.empty(2, device="cuda")
        bl.blink_gradient_norm(update, again, work, most, 0.5, None, _stream())
        assert torch.equal(norm, again)


def test_norm_of_all_types_together():
    g = torch.Generator("cuda").manual_seed(1)
    grads = [torch.randn(n, generator=g, device="cuda").to(t) for n, t in ((1000, B16), (3, F32), (5001, H16), (70_000, F32), (9, B16))]
    update = bl.blink_make_update(grads)
    norm = torch.empty(2, device="cuda")
    bl.blink_gradient_norm(update, norm, _work(update), stream=_stream())
    want = math.sqrt(sum(float(v.double().square().sum()) for v in grads))
    assert abs(float(norm[0]) - want) <= 1.01 * 2.0 ** -24 * want and norm[1] == 1


def test_nothing_to_do():
    """Tensors without elements, a list without weights."""
    empty = torch.zeros(0, device="cuda")
    update = bl.blink_make_update([empty, empty], [empty, None], [empty, None], [empty, None])
    norm, step = torch.full((2,), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bl.blink_gradient_norm(update, norm, None, 1.0, 0.5, step, _stream())
    assert norm.tolist() == [0.0, 0.5] and int(step) == 1
    bl.blink_adamw_step(update, step, LR, stream=_stream())
    grad = torch.ones(5, device="cuda")
    bl.blink_adamw_step(bl.blink_make_update([grad]), step, LR, stream=_stream())
    assert (grad == 1).all()


def test_sizes_of_gradients():
    """Squares beyond and below what 32 bits hold; nothing but zeros."""
    for value, most, scale in ((3e38, 1.0, None), (1e-38, 1e-40, None), (0.0, 1.0, 2.0)):
        update = bl.blink_make_update([torch.full((4,), value, device="cuda")])
        norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        bl.blink_gradient_norm(update, norm, _work(update), most, 2.0, step, _stream())
        want = 2 * 2 * float(np.float32(value))
        scale = 2.0 * most / want if scale is None else scale
        assert (norm[0] == math.inf) if want > 3.4e38 else abs(float(norm[0]) - want) <= 2.0 ** -24 * want
        assert abs(float(norm[1]) - scale) <= 2.0 ** -23 * scale + 2.0 ** -149 and int(step) == 1


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("eight", [False, True])
def test_a_step_that_is_left_out(bad, eight):
    """A gradient that is no number: neither weights nor moments nor the step's number change."""
    T = Tensors(SIZES, eight=eight)
    T.lists["grads"][8][4999] = bad
    norm, step = torch.empty(2, device="cuda"), torch.full((1,), 3, dtype=torch.int32, device="cuda")
    bl.blink_gradient_norm(T.update, norm, _work(T.update), 1.0, 1.0, step, _stream())
    assert torch.isnan(norm[1]) and not torch.isfinite(norm[0]) and int(step) == 3
    bl.blink_adamw_step(T.update, step, LR, B1, B2, EPS, norm[1:], stream=_stream())
    bl.blink_adamw_step(T.update, torch.zeros(1, dtype=torch.int32, device="cuda"), LR, stream=_stream())     # no step has number 0
    for name, views in T.lists.items():
        if name != "grads":
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(views, T.before[name]))


def test_a_number_that_is_none_stays_where_it_is():
    """Without a norm in front: one element of 32-bit moments, the 256 of 8-bit ones."""
    for eight in (False, True):
        T = Tensors([1000], eight=eight)
        T.lists["grads"][0][300] = math.nan
        bl.blink_adamw_step(T.update, torch.ones(1, dtype=torch.int32, device="cuda"), LR, stream=_stream())
        w = torch.isnan(T.lists["weights"][0])
        assert w[300] and int(w.sum()) == 1
        if eight:
            assert torch.isnan(T.lists["scales1"][0]).tolist() == [False, True, False, False]
        else:
            assert int(torch.isnan(T.lists["moments1"][0]).sum()) == 1


def test_tensors_that_others_step():
    """Without weights a gradient counts in the norm and nothing is written; a list may hold all kinds."""
    a, b = Tensors([5000], B16, F32, True, True, 1), Tensors([300], F32, B16, False, False, 2)
    other = torch.full((77,), 2.0, device="cuda")
    pick = lambda name: [a.lists.get(name, [None])[0], None, b.lists.get(name, [None])[0]]   # noqa: E731
    update = bl.blink_make_update([a.lists["grads"][0], other, b.lists["grads"][0]], pick("weights"), pick("moments1"), pick("moments2"), pick("masters"),
                                  pick("scales1"), pick("scales2"), [a.rates[0], 1.0, b.rates[0]], [a.decays[0], 0.0, b.decays[0]])
    norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bl.blink_gradient_norm(update, norm, _work(update), step=step, stream=_stream())
    want = math.sqrt(sum(float(v.double().square().sum()) for v in (a.lists["grads"][0], other, b.lists["grads"][0])))
    assert abs(float(norm[0]) - want) <= 1.01 * 2.0 ** -24 * want
    bl.blink_adamw_step(update, step, LR, B1, B2, EPS, norm[1:], seed=9, stream=_stream())
    _check(a, 1, seed=9)
    _check(b, 1)
    assert (other == 2).all()


def test_rounding_is_fair():
    """Moments in 8 bits follow those in 32 on the average where a number nearest by would stand still: v moves by 2^-10 of itself a step, an e4m3 step is 2^-3."""
    n, steps = 1 << 16, 300
    T = Tensors([n], eight=True)
    for name in ("moments1", "moments2", "scales1", "scales2"):
        T.lists[name][0].zero_()
    T.lists["grads"][0].fill_(0.5)
    T.lists["grads"][0][::256] = 1.0      # the largest of every block
    for t in range(1, steps + 1):
        bl.blink_adamw_step(T.update, torch.full((1,), t, dtype=torch.int32, device="cuda"), LR, B1, B2, EPS, seed=3, stream=_stream())
    some = torch.ones(n, dtype=torch.bool, device="cuda")
    some[::256] = False
    m = (_blocks(T.lists["moments1"][0].float()) * T.lists["scales1"][0][:, None]).view(-1)[some].double()
    r = (_blocks(T.lists["moments2"][0].float()) * T.lists["scales2"][0][:, None]).view(-1)[some].double()
    want_r = 0.5 * math.sqrt(1 - B2 ** steps)
    # m: roundings are fair, so its mean over 65280 elements is the sum's own; one element is off by a code (1/8 of it) for each of the 6 steps that halve
    # what a rounding left.  The root r climbs from 0: a climb d adds d (code - d) to the mean of r^2 where a code is r / 8 at most, so r^2 gains r^2 / 16 at most
    # on the way, r half of that; its own spread takes as much from the mean of r at most.
    assert abs(float(m.mean()) - 0.5) < 0.5 * 6 / 8 / math.sqrt(m.numel()) + 1e-4
    assert abs(float(r.mean()) / want_r - 1) < 0.05
    assert float(r.std()) < 0.25 * want_r


def test_in_a_graph():
    """Replays step on: the step's number and the scale are read where the kernel before left them."""
    for eight in (False, True):
        T, U = (Tensors(SIZES, B16, F32, True, eight, 4) for _ in range(2))
        norm, step, work = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), _work(T.update)
        rate = torch.ones(1, device="cuda")

        def run(X, norm, step):
            bl.blink_gradient_norm(X.update, norm, work, 0.3, 0.5, step, _stream())
            bl.blink_adamw_step(X.update, step, LR, B1, B2, EPS, norm[1:], rate, 8, _stream())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(T, norm, step)
        norm2, step2 = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        for k in range(4):
            for X in (T, U):
                for v in X.lists["grads"]:
                    v.mul_(1.0 + 0.5 * k)
            rate.fill_(1.0 / (k + 1))
            work.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            run(U, norm2, step2)
            assert int(step) == k + 1 and torch.equal(norm, norm2)
            for name in T.flat:
                assert torch.equal(T.flat[name].view(torch.uint8), U.flat[name].view(torch.uint8)), name


def test_streams():
    """Four lists on streams of their own: as many as there are hardware queues, so that streams of later tests fall to the queues that they fell to without it."""
    both = [Tensors([200_001, 7], B16, F32, True, True, s) for s in (1, 2, 3, 4)]
    streams = [torch.cuda.Stream() for _ in both]
    state = []
    torch.cuda.synchronize()
    for T, s in zip(both, streams):
        with torch.cuda.stream(s):
            norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
            work = _work(T.update)
            bl.blink_gradient_norm(T.update, norm, work, math.inf, 1.0, step, s.cuda_stream)
            bl.blink_adamw_step(T.update, step, LR, B1, B2, EPS, norm[1:], None, 6, s.cuda_stream)
            state.append((norm, step, work))
    torch.cuda.synchronize()
    for T in both:
        _check(T, 1, seed=6)


def test_a_tensor_past_32_bits():
    """More than 2^32 elements: the last ones as in a tensor of their own that ends alike."""
    n, last = (1 << 32) + 1000, 1000 + 256 * 8
    w, m, v = (torch.zeros(n, dtype=d, device="cuda") for d in (B16, F32, F32))
    g = torch.ones(n, dtype=B16, device="cuda")
    g[-last:] = torch.randn(last, device="cuda").to(B16)
    tail = [x[-last:].clone() for x in (g, w, m, v)]
    update, small = bl.blink_make_update([g], [w], [m], [v]), bl.blink_make_update(*[[x] for x in tail])
    norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bl.blink_gradient_norm(update, norm, _work(update), step=step, stream=_stream())
    want = math.sqrt(n - last + float(tail[0].double().square().sum()))
    assert abs(float(norm[0]) - want) <= 1.01 * 2.0 ** -24 * want
    for u in (update, small):
        bl.blink_adamw_step(u, step, LR, stream=_stream())
    for x, y in zip((w, m, v), tail[1:]):
        assert torch.equal(x[-last:], y)
    assert bool((w[:1 << 20] == w[0]).all()) and float(w[0]) != 0


@pytest.mark.parametrize("weights,grads,master,eight", [(F32, F32, False, False), (F32, F32, False, True), (B16, F32, True, True), (B16, B16, False, False),
                                                        (F32, B16, False, True)])
def test_gradients_whose_squares_32_bits_hold(weights, grads, master, eight):
    """A scaled length below 2^63: moments and weights as in 64 bits, and an ordinary step after it."""
    T = Tensors([5, 1000, 4096], weights, grads, master, eight, seed=6)
    for i, at, value in ((0, 2, 5e18), (1, 300, -3e18), (1, 301, 2e18), (1, 999, 1e15), (2, 4000, 4e18)):
        T.lists["grads"][i][at] = T.before["grads"][i][at] = value
    norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bl.blink_gradient_norm(T.update, norm, _work(T.update), step=step, stream=_stream())
    assert float(norm[1]) == 1 and int(step) == 1
    for t, value in ((1, None), (2, 0.5)):
        if value is not None:
            T.before = {k: [v.clone() for v in views] for k, views in T.lists.items()}
            for v in T.lists["grads"] + T.before["grads"]:
                v.fill_(value)
        bl.blink_adamw_step(T.update, step.fill_(t), LR, B1, B2, EPS, norm[1:], None, 5, _stream())
        _check(T, t, seed=5)
        assert all(torch.isfinite(v.float()).all() for views in T.lists.values() for v in views)


# (gradient, max_norm, factor) and whether a step can be made of it
SCALED = [(1e20, math.inf, 1.0, False), (3e38, math.inf, 1.0, False), (-1e20, math.inf, 1.0, False), (3e38, math.inf, 2.0, False), (3e38, 1e19, 1.0, False),
          (3e38, 1e18, 2.0, True), (3e38, 1.0, -2.0, True), (9e18, math.inf, 1.0, True), (9e18, math.inf, -2.0, False), (1e-3, math.inf, 1e39, False),
          (1e-3, 1.0, 1e39, True), (1e-30, math.inf, 1e39, False), (0.0, 1.0, 1e39, False), (1e-3, math.inf, 1e20, True)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("value,most,factor,fine", SCALED)
def test_a_step_whose_squares_pass_32_bits_is_left_out(value, most, factor, fine, eight):
    """Scaled gradients that 32 bits cannot hold or square are no step, like a gradient that is no number; clipped ones are."""
    T = Tensors([3000], eight=eight)
    T.lists["grads"][0].zero_()
    T.lists["grads"][0][2999] = value
    norm, step = torch.empty(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bl.blink_gradient_norm(T.update, norm, _work(T.update), most, factor, step, _stream())
    value = float(np.float32(value))
    if abs(factor * value) < 3.4e38:
        assert abs(float(norm[0]) - abs(factor * value)) <= 1.01 * 2.0 ** -24 * abs(factor * value)
    assert int(step) == fine and bool(torch.isnan(norm[1])) != fine
    bl.blink_adamw_step(T.update, step, LR, B1, B2, EPS, norm[1:], stream=_stream())
    if fine:
        want = factor * min(1.0, most / abs(factor * value))
        assert abs(float(norm[1]) - want) <= 1.01 * 2.0 ** -24 * abs(want) + 2.0 ** -150      # (half a step of numbers below 2^-126: -2 / 6e38 is one)
        assert all(torch.isfinite(v.float()).all() for views in T.lists.values() for v in views)
        return
    for name, views in T.lists.items():
        if name != "grads":
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(views, T.before[name]))


@pytest.mark.parametrize("sizes", [[1, 300, 4097], [30_000_001, 256]])
def test_first_step_whatever_the_scales_hold(sizes):
    """Moments that are all 0 are 0 with any scales, those of memory that nobody has written among them."""
    both = []
    for fill in (0, 255):
        T = Tensors(sizes, B16, F32, True, True)
        for name in ("moments1", "moments2"):
            for v in T.lists[name]:
                v.zero_()
        for name in ("scales1", "scales2"):
            for v in T.lists[name]:
                v.view(torch.uint8).fill_(fill)
        T.lists["scales1"][0][:1] = math.inf if fill else 0.0
        bl.blink_adamw_step(T.update, torch.ones(1, dtype=torch.int32, device="cuda"), LR, B1, B2, EPS, seed=5, stream=_stream())
        both.append(T)
    for name, views in both[0].lists.items():
        for a, b in zip(views, both[1].lists[name]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name
    assert all(torch.isfinite(v).all() for v in both[1].lists["masters"] + both[1].lists["scales1"] + both[1].lists["scales2"])


@pytest.mark.parametrize("eps", [1e-50, 5e-324])
def test_eps_below_32_bits(eps):
    """It is more than 0: where nothing moves nothing is divided by 0."""
    g = torch.tensor([0.0, 1.0, -1e-3], device="cuda")
    w, m, v = (torch.zeros(3, device="cuda") for _ in range(3))
    w.fill_(2.0)
    update = bl.blink_make_update([g], [w], [m], [v])
    bl.blink_adamw_step(update, torch.ones(1, dtype=torch.int32, device="cuda"), LR, B1, B2, eps, stream=_stream())
    assert (w.cpu() - torch.tensor([2.0, 2.0 - LR, 2.0 + LR])).abs().max() <= 10 * 2.0 ** -24 * LR + 2 * 2.0 ** -23
    assert w[0] == 2


@pytest.mark.parametrize("ratio", [0.5, 1e-2, 1e-4, 1e-6])
def test_roots_next_to_a_larger_one(ratio):
    """Gradients that vary, far below the largest of their block: what rounding adds to v, and the least root."""
    n, steps, b2 = 1 << 16, 600, 0.99
    T = Tensors([n], eight=True)
    for name in ("moments1", "moments2", "scales1", "scales2"):
        T.lists[name][0].zero_()
    g = torch.Generator("cuda").manual_seed(11)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    for t in range(1, steps + 1):
        T.lists["grads"][0].copy_(ratio * torch.randn(n, generator=g, device="cuda"))
        T.lists["grads"][0][::256] = 1.0
        bl.blink_adamw_step(T.update, step.fill_(t), LR, B1, b2, EPS, seed=3, stream=_stream())
    some = torch.ones(n, dtype=torch.bool, device="cuda")
    some[::256] = False
    if ratio == 1e-6:      # a root that would be a fifth of the least code: sqrt(b2) of that code, rounded down to nothing or up, is the least code again
        assert (T.lists["moments2"][0].float()[some] == 2.0 ** -9).all()
        return
    r = (_blocks(T.lists["moments2"][0].float()) * T.lists["scales2"][0][:, None]).view(-1)[some].double()
    # Rounding r + d to one of two codes that are u apart adds at most |d| u to the mean of r^2.  Here d = (1 - b2)(g^2 - v) / 2r and u is r / 8 at most (r is
    # above 2^-6 of a scale's unit): E|z^2 - 1| = 0.968 makes (1 - b2) v 0.968 / 16 a step, against (1 - b2) of the excess that is lost: 0.0605, and 1 / (1 - 0.0605)
    # of it, for the excess itself counts in v.  v of one element varies by sqrt(2 (1 - b2) / (1 + b2)) = 0.1, their mean over 65280 by 0.0004.
    got = float(r.square().mean()) / (ratio * ratio * (1 - b2 ** steps))
    assert -0.003 < got - 1 < 0.0605 / (1 - 0.0605) + 0.003
