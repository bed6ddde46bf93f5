"""The rest of a training step around its collectives, and how fast: the norm of all gradients with the factor that clips them, an
AdamW step over many tensors with its moments in 32 or in 8 bits, and a router that chooses experts by scores and a bias, within groups,
with its gradient and the bias's own step.

`run` makes one pass in one of two ways: where `own` is true through this repository's operators, else in plain form,
elementary torch operations, rounded once at the end.  `exact` gives the results from the definitions in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8
BLOCK = 256          # elements of a tensor that share the scale of a moment in 8 bits
SEED = 0x5eed
BIAS_RATE = 1e-3


def _tensors(op, layers=0, dim=0, hidden=0, vocab=0, odd=0, most=0, weights="fp32", master=False, grads="fp32", moments="fp32"):
    """layers > 0: the tensors of a model; else `odd` tensors of 1 to `most` elements."""
    return {"op": op, "layers": layers, "dim": dim, "hidden": hidden, "vocab": vocab, "odd": odd, "most": most, "weights": weights, "master": master,
            "grads": grads, "moments": moments}


def _route(tokens, experts, k, groups=1, kept=1, scores="sigmoid", dtype="bf16", normalize=True, scale=1.0, masked=0.0):
    return {"op": "route", "tokens": tokens, "experts": experts, "k": k, "groups": groups, "kept": kept, "scores": scores, "dtype": dtype,
            "normalize": normalize, "scale": scale, "masked": masked}


def listed():
    return [{"name": name, **case} for name, case in (
        # gradients of a few small tensors, packed one after the other as the collectives leave them: all latency
        ("a few gradients", _tensors("norm", odd=9, most=5_000)),
        # the summed gradients of a model
        ("a model's gradients", _tensors("norm", layers=8, dim=1_024, hidden=4_096, vocab=16_384)),
        # clipping and a step of a small model: latency of three kernels
        ("a small model's step", _tensors("step", layers=2, dim=128, hidden=512, vocab=1_000)),
        # tensors of all sizes at odd places, 16-bit weights without a copy in 32 bits, 16-bit gradients
        ("odd tensors", _tensors("step", odd=301, most=200_000, weights="bf16", grads="bf16")),
        # clipping and a step of a model with 32-bit weights: seven streams of memory
        ("a model's step", _tensors("step", layers=8, dim=1_024, hidden=4_096, vocab=32_768)),
        # the same with moments in 8 bits: small, odd and large
        ("a small step in 8 bits", _tensors("step", layers=2, dim=128, hidden=512, vocab=1_000, weights="bf16", master=True, moments="8 bits")),
        ("odd tensors in 8 bits", _tensors("step", odd=301, most=200_000, weights="fp32", grads="bf16", moments="8 bits")),
        ("a model's step in 8 bits", _tensors("step", layers=8, dim=1_024, hidden=4_096, vocab=32_768, weights="bf16", master=True, moments="8 bits")),
        # a generated token's experts
        ("one token", _route(1, 64, 6, dtype="fp32")),
        # an odd number of tokens, some of them padding, groups that are no power of two, softmax
        ("sixty experts in groups", _route(20_011, 60, 4, 6, 3, "softmax", normalize=False, masked=0.1)),
        # many experts without groups, logits in 32 bits
        ("128 experts", _route(131_072, 128, 8, dtype="fp32")),
        # a batch's tokens over many experts, in groups that sit together
        ("256 experts in groups", _route(262_144, 256, 8, 8, 4, scale=2.5)),
    )]


def _spread(rng, lo, hi):
    """A whole number, its logarithm evenly spread; every third time as it falls, else near a multiple of eight."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n if rng.random() < 0.4 else (n + 7) // 8 * 8))


def draw(rng):
    op = rng.choice(("norm", "step", "step", "route", "route"))
    if op == "route":
        per, groups = rng.choice((1, 2, 4, 8, 10, 16, 32, 64)), rng.choice((1, 1, 2, 3, 4, 6, 8, 16))
        experts = max(4, per * groups)
        groups = groups if experts == per * groups else 1
        kept = rng.randint(1, groups)
        k = rng.randint(1, min(10, kept * experts // groups))
        return _route(_spread(rng, 1, (1 << 26) // max(16, experts)), experts, k, groups, kept, rng.choice(("sigmoid", "sigmoid", "softmax")),
                      rng.choice(("fp32", "bf16", "fp16")), rng.random() < 0.6, rng.choice((1.0, 2.5)), rng.choice((0.0, 0.2)))
    weights = rng.choice(("fp32", "bf16", "fp16")) if op == "step" else "fp32"
    kinds = {"weights": weights, "master": weights != "fp32" and (weights == "fp16" or rng.random() < 0.6), "grads": rng.choice(("fp32", "fp32", "bf16")),
             "moments": rng.choice(("fp32", "8 bits")) if op == "step" else "fp32"}
    if rng.random() < 0.5:
        odd = _spread(rng, 1, 1_000)
        return _tensors(op, odd=odd, most=_spread(rng, 1, min(1 << 23, (1 << 27) // odd)), **kinds)
    while True:
        layers, dim, hidden, vocab = rng.randint(1, 12), _spread(rng, 32, 2_048), _spread(rng, 64, 8_192), _spread(rng, 100, 65_536)
        if vocab * dim + layers * (4 * dim * dim + 3 * dim * hidden) <= 1 << 27:
            return _tensors(op, layers, dim, hidden, vocab, **kinds)


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _sizes(case):
    if case["layers"]:
        d, h = case["dim"], case["hidden"]
        return [case["vocab"] * d] + case["layers"] * ([d * d] * 4 + [d * h] * 3 + [d] * 2) + [d]
    # spread over the logarithm by the golden ratio's multiples
    return [max(1, min(case["most"], round(case["most"] ** ((i + 1) * 0.6180339887498949 % 1.0)))) for i in range(case["odd"])]


def _views(flat, sizes, each=1):
    """One tensor after the other in a buffer; each: elements to a place in it."""
    out, at = [], 0
    for n in sizes:
        out.append(flat[at:at + -(-n // each)])
        at += -(-n // each)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")   # noqa: E731
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    if case["op"] == "route":
        t, e, k = case["tokens"], case["experts"], case["k"]
        s["logits"] = (1.5 * randn(t, e) + randn(e)).to(TYPES[case["dtype"]])
        s["bias"] = BIAS_RATE * torch.randint(-100, 101, (e,), generator=g, device="cuda").float()   # a hundred steps of it, up or down
        s["keep"] = None
        if case["masked"]:   # padded sequences; and an expert that is out of service
            s["keep"] = torch.rand(t, generator=g, device="cuda") >= case["masked"]
            s["logits"][:, e // 2] = -math.inf
        s["grad_weights"] = 0.01 * randn(t, k)
        if own:
            import paper_1910_04940_amd as bl
            s["chosen"] = torch.empty(t, k, dtype=torch.int32, device="cuda")
            s["weights"] = torch.empty(t, k, device="cuda")
            s["counts"] = torch.empty(e + 1, dtype=torch.int32, device="cuda")
            s["bias_out"] = torch.empty(e, device="cuda")
            s["out"] = torch.empty_like(s["logits"])
            s["workspace"] = torch.empty(bl.blink_route_biased_workspace(t, e), dtype=torch.uint8, device="cuda")
        return s
    sizes = s["sizes"] = _sizes(case)
    n, blocks = sum(sizes), sum(-(-m // BLOCK) for m in sizes)
    # a few directions of a gradient are far larger than the others
    s["grads"] = (1e-3 * randn(n) * torch.exp(0.5 * randn(-(-n // 64)).repeat_interleave(64)[:n])).to(TYPES[case["grads"]])
    s["factor"], s["max_norm"] = 0.125, 0.05 * 0.125 * 1e-3 * math.sqrt(n)      # a mean over eight ranks, a norm that is clipped
    s["step"] = torch.randint(20, 200, (1,), generator=g, device="cuda", dtype=torch.int32)
    s["norm"] = torch.empty(2, device="cuda")
    if case["op"] == "step":
        master = 0.02 * randn(n)
        s["weights"] = master.to(TYPES[case["weights"]])
        s["master"] = master if case["master"] else None
        if case["moments"] == "fp32":
            s["moment1"], s["moment2"] = 1e-5 * randn(n), (1e-5 * randn(n)).square()
            s["scale1"] = s["scale2"] = None
        else:
            s["moment1"] = (100 * randn(n)).clamp_(-448, 448).to(torch.float8_e4m3fn)
            s["moment2"] = (100 * randn(n)).abs_().clamp_(2.0 ** -9, 448).to(torch.float8_e4m3fn)
            s["scale1"], s["scale2"] = 1e-7 * torch.exp(randn(blocks)), 1e-7 * torch.exp(randn(blocks))
        s["rates"] = [1.0 if i % 5 else 0.5 for i in range(len(sizes))]
        s["decays"] = [0.1 if i % 3 else 0.0 for i in range(len(sizes))]
    if own:
        import paper_1910_04940_amd as bl
        grads = _views(s["grads"], sizes)
        if case["op"] == "norm":
            s["update"] = bl.blink_make_update(grads)
        else:
            eight = case["moments"] != "fp32"
            s["update"] = bl.blink_make_update(
                grads, _views(s["weights"], sizes), _views(s["moment1"], sizes), _views(s["moment2"], sizes),
                masters=_views(s["master"], sizes) if case["master"] else None, scales1=_views(s["scale1"], sizes, BLOCK) if eight else None,
                scales2=_views(s["scale2"], sizes, BLOCK) if eight else None, rates=s["rates"], decays=s["decays"])
        s["workspace"] = torch.empty(bl.blink_gradient_norm_workspace(s["update"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _state(s):
    return {key: s[key] for key in ("norm", "step", "weights", "master", "moment1", "moment2", "scale1", "scale2")}


def _own(s):
    import paper_1910_04940_amd as bl
    case, stream = s["case"], s["stream"]
    if case["op"] == "route":
        bl.blink_route_biased(s["logits"], case["k"], s["chosen"], s["weights"], s["counts"], s["workspace"], s["bias"], s["keep"], case["groups"], case["kept"],
                              case["scores"], case["normalize"], case["scale"], stream)
        bl.blink_route_bias(s["counts"], s["bias"], s["bias_out"], BIAS_RATE, stream)
        bl.blink_route_biased_gradient(s["logits"], case["k"], s["chosen"], s["grad_weights"], s["out"], s["keep"], case["scores"], case["normalize"],
                                       case["scale"], stream)
        return {"chosen": s["chosen"], "weights": s["weights"], "counts": s["counts"], "bias": s["bias_out"], "gradient": s["out"]}
    bl.blink_gradient_norm(s["update"], s["norm"], s["workspace"], s["max_norm"], s["factor"], s["step"], stream)
    if case["op"] == "norm":
        return {"norm": s["norm"], "step": s["step"]}
    bl.blink_adamw_step(s["update"], s["step"], LR, BETA1, BETA2, EPS, s["norm"][1:], None, SEED, stream)
    return _state(s)


def _plain(s):
    case = s["case"]
    if case["op"] == "route":
        return _plain_route(s)
    g = s["grads"].float()
    norm = (s["factor"] * s["factor"] * g.double().square().sum()).sqrt()
    fine = torch.isfinite(norm)
    scale = torch.where(fine, s["factor"] * torch.clamp(s["max_norm"] / norm, max=1.0), math.nan).float()
    s["norm"] = torch.stack((norm.float(), scale))
    s["step"] = s["step"] + fine.int()
    return {"norm": s["norm"], "step": s["step"]} if case["op"] == "norm" else _plain_step(s, g * scale)


def _places(sizes):
    """For every element of the packed tensors: its tensor, its place in it, its block among all."""
    n = torch.tensor(sizes, device="cuda")
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), n)
    place = torch.arange(len(tensor), device="cuda") - (torch.cumsum(n, 0) - n)[tensor]
    blocks = (n + BLOCK - 1) // BLOCK
    return tensor, place, (torch.cumsum(blocks, 0) - blocks)[tensor] + place // BLOCK


def _mix(h):
    """The finalizer of MurmurHash3 on whole numbers below 2^32."""
    h = ((h ^ h >> 16) * 0x85ebca6b) & 0xffffffff
    h = ((h ^ h >> 13) * 0xc2b2ae35) & 0xffffffff
    return h ^ h >> 16


def _random(step, tensor, place):
    """The random numbers of a step: two in (0, 1) for every element, of 16 bits."""
    key = _mix((SEED + 0x9e3779b9 * step.long()) & 0xffffffff)
    h = _mix(_mix(_mix(key ^ tensor) ^ place // BLOCK) ^ place % BLOCK)
    return ((h & 0xffff) + 0.5) / 65536, ((h >> 16) + 0.5) / 65536


def _eight(z, u, least):
    """|z| <= 448 rounded to four significant bits (below 2^-6 to multiples of 2^-9), up with the probability of what is left of it."""
    z = z.double()
    unit = torch.exp2(torch.clamp(torch.frexp(z.abs()).exponent - 1, min=-6).double() - 3)
    to = torch.clamp(torch.floor(z.abs() / unit + u) * unit, max=448)
    return torch.where((to == 0) & (z != 0), least, to) * torch.sign(z)


def _plain_step(s, g):
    case = s["case"]
    t = s["step"].double()
    by1, by2 = 1 / (1 - BETA1 ** t), (1 / (1 - BETA2 ** t)).sqrt().float()
    tensor, place, block = _places(s["sizes"])
    rate = LR * torch.tensor(s["rates"], dtype=torch.float64, device="cuda")
    kept = (1 - rate * torch.tensor(s["decays"], dtype=torch.float64, device="cuda")).float()[tensor]
    eight = case["moments"] != "fp32"
    m, v = s["moment1"].float(), s["moment2"].float()
    if eight:
        m, v = m * s["scale1"][block], (v * s["scale2"][block]).square()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g.square()
    w = s["weights"].float() if s["master"] is None else s["master"]
    w = w * kept - (rate * by1).float()[tensor] * (m / (v.sqrt() * by2 + EPS))
    if eight:
        for name, y, u, least in zip("12", (m, v.sqrt()), _random(s["step"], tensor, place), (0.0, 2.0 ** -9)):
            most = torch.zeros_like(s["scale" + name]).scatter_reduce_(0, block, y.abs(), "amax")
            none = most < 2.0 ** -100
            s["scale" + name] = torch.where(none, 0.0, most * (1.0 / 448))
            z = y * torch.where(none, 0.0, 448 / most)[block]
            s["moment" + name] = _eight(z.clamp(-448, 448), u, least).float().to(torch.float8_e4m3fn)
    else:
        s["moment1"], s["moment2"] = m, v
    s["weights"] = w.to(s["weights"].dtype)
    if s["master"] is not None:
        s["master"] = w
    return _state(s)


def _plain_route(s):
    """In 64 bits: scores that all but tie have to come in their order."""
    case = s["case"]
    t, e, k, groups, kept = case["tokens"], case["experts"], case["k"], case["groups"], case["kept"]
    x = s["logits"].double()
    if s["keep"] is not None:
        x = torch.where(s["keep"][:, None], x, -math.inf)
    some = torch.isfinite(x.amax(1, keepdim=True))
    if case["scores"] == "softmax":
        powers = torch.exp(x - torch.where(some, x.amax(1, keepdim=True), 0.0))
        p = powers / powers.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        p = 1 / (1 + torch.exp(-x))
    a = torch.where(x > -math.inf, p + s["bias"].double(), -math.inf)
    if groups > 1:
        two = torch.sort(a.view(t, groups, e // groups), dim=2, descending=True).values[:, :, :2]
        of_group = torch.where(two[:, :, 0] > -math.inf, torch.where(two > -math.inf, two, 0.0).sum(2), -math.inf)
        order = torch.sort(of_group, dim=1, descending=True, stable=True).indices[:, :kept]
        is_kept = torch.zeros(t, groups, dtype=torch.bool, device="cuda").scatter_(1, order, True)
        a = torch.where(is_kept.repeat_interleave(e // groups, 1), a, -math.inf)
    order = torch.sort(a, dim=1, descending=True, stable=True)
    found, at = order.values[:, :k] > -math.inf, order.indices[:, :k]
    picked = torch.where(found, p.gather(1, at), 0.0)
    share = picked.sum(1, keepdim=True) if case["normalize"] else torch.ones_like(picked[:, :1])
    share = torch.where(found[:, :1], share, 1.0)
    shares = picked / share
    weights = case["scale"] * shares
    counts = torch.zeros(e + 1, dtype=torch.int32, device="cuda")
    counts.index_add_(0, torch.where(found, at, e).reshape(-1), found.int().reshape(-1))
    counts[e] = found[:, 0].sum()
    c = counts[:e].long()
    bias = s["bias"] + BIAS_RATE * torch.sign(c.sum() - e * c).float()
    d = torch.where(found, case["scale"] * s["grad_weights"].double(), 0.0)
    if case["normalize"]:
        d = (d - (d * shares).sum(1, keepdim=True)) / share     # (0 where one expert has it all)
    by_p = torch.zeros_like(p).scatter_add_(1, at, torch.where(found, d, 0.0))
    grad = p * (by_p - (p * by_p).sum(1, keepdim=True)) if case["scores"] == "softmax" else by_p * p * (1 - p)
    return {"chosen": torch.where(found, at, -1).int(), "weights": weights.float(), "counts": counts, "bias": bias, "gradient": grad.to(s["logits"].dtype)}


def work(case):
    if case["op"] == "route":   # the gradient reads the logits of the chosen again, or all of them where weights are parts of a whole softmax
        t, e, k = case["tokens"], case["experts"], case["k"]
        b = BYTES[case["dtype"]]
        again = e if case["scores"] == "softmax" and not case["normalize"] else k
        return {"bytes": t * (e * b + again * b + e * b + 16 * k + (2 if case["masked"] else 0)) + 4 * (3 * e + 1), "flops": t * e * (12 + k)}
    n = sum(_sizes(case))
    if case["op"] == "norm":
        return {"bytes": n * BYTES[case["grads"]], "flops": 2 * n}
    state = 2 * (1 + 4 / BLOCK) if case["moments"] != "fp32" else 8
    weights = BYTES[case["weights"]]      # with a master copy they are written only
    each = 2 * BYTES[case["grads"]] + 2 * state + (8 + weights if case["master"] else 2 * weights)
    return {"bytes": n * each, "flops": 2 * n + 20 * n}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        return _exact_route(s)
    g = s["factor"] * s["grads"].double()
    norm = float(torch.linalg.vector_norm(g))
    clip = min(1.0, s["max_norm"] / norm)
    out = {"norm": torch.tensor([norm, s["factor"] * clip], dtype=torch.float64, device="cuda"), "step": None}
    if case["op"] == "norm":
        return out
    g *= clip
    t = int(s["step"]) + 1
    sizes = s["sizes"]
    tensor, place, block = _places(sizes)
    first = s["moment1"].double()
    root = s["moment2"].double()
    if case["moments"] != "fp32":
        first *= s["scale1"].double()[block]
        root *= s["scale2"].double()[block]
    else:
        root.sqrt_()
    first += (1 - BETA1) * (g - first)
    root = torch.hypot(math.sqrt(BETA2) * root, math.sqrt(1 - BETA2) * g)
    rate = torch.repeat_interleave(torch.tensor(s["rates"], dtype=torch.float64), torch.tensor(sizes)).cuda() * LR
    decay = torch.repeat_interleave(torch.tensor(s["decays"], dtype=torch.float64), torch.tensor(sizes)).cuda()
    w = (s["weights"] if s["master"] is None else s["master"]).double()
    w = w - rate * (decay * w + first / (1 - BETA1 ** t) / (root / math.sqrt(1 - BETA2 ** t) + EPS))
    out |= {"weights": w, "master": w if case["master"] else None, "moment1": first, "moment2": root.square(), "scale1": None, "scale2": None}
    if case["moments"] != "fp32":
        up = _random(s["step"] + 1, tensor, place)
        for name, y, u in (("1", first, up[0]), ("2", root, up[1])):
            scale = torch.zeros(len(s["scale1"]), dtype=torch.float64, device="cuda").scatter_reduce_(0, block, y.abs(), "amax") / 448
            z = y.abs() / scale.clamp(min=1e-300)[block]
            # numbers of e4m3 around z: eight to a power of two from 2^-6 on, evenly below it
            unit = torch.where(z < 2.0 ** -6, 2.0 ** -9, 2.0 ** (torch.floor(torch.log2(z.clamp(min=2.0 ** -6))) - 3))
            low = torch.floor(z / unit)
            code = (low + (z / unit - low + u >= 1)) * unit
            if name == "2":
                code = torch.where(z > 0, code.clamp(min=2.0 ** -9), code)
            out["scale" + name], out["moment" + name] = scale, torch.copysign(code, y)
    return out


def _exact_route(s):
    case = s["case"]
    t, e, k, groups = case["tokens"], case["experts"], case["k"], case["groups"]
    x = s["logits"].double()
    out = torch.isinf(x) if s["keep"] is None else torch.isinf(x) | ~s["keep"][:, None]
    p = torch.sigmoid(x) if case["scores"] == "sigmoid" else torch.nan_to_num(torch.softmax(x.masked_fill(out, -math.inf), 1))
    left = (p + s["bias"].double()).masked_fill(out, -math.inf)
    rows = torch.arange(t, device="cuda")
    if groups > 1:   # groups leave one at a time, the first of the best
        most, again = torch.full((t, groups), -math.inf, dtype=torch.float64, device="cuda"), left.view(t, groups, -1).clone()
        for j in range(min(2, e // groups)):
            best, at = again.max(2)
            most = torch.where(best > -math.inf, torch.where(most > -math.inf, most, 0.0) + best, most)
            again.scatter_(2, at[:, :, None], -math.inf)
        stays = torch.zeros(t, groups, dtype=torch.bool, device="cuda")
        for j in range(case["kept"]):
            at = (most == most.amax(1, keepdim=True)).int().argmax(1)
            stays[rows, at] = True
            most[rows, at] = -math.inf
        left = left.view(t, groups, -1).masked_fill(~stays[:, :, None], -math.inf).view(t, e)
    chosen = torch.zeros(t, e, dtype=torch.float64, device="cuda")
    weights = torch.zeros(t, k, dtype=torch.float64, device="cuda")
    upstream = torch.zeros(t, e, dtype=torch.float64, device="cuda")
    for j in range(k):
        most = left.amax(1, keepdim=True)
        at = (left == most).int().argmax(1)
        real = most[:, 0] > -math.inf
        chosen[rows, at] += real
        weights[:, j] = torch.where(real, p[rows, at], 0.0)
        upstream[rows, at] += torch.where(real, s["grad_weights"][:, j].double(), 0.0)
        left[rows, at] = -math.inf
    if case["normalize"]:
        total = (p * chosen).sum(1, keepdim=True).clamp_(min=1e-300)
        weights /= total
        upstream = chosen * (upstream - (upstream * (p / total)).sum(1, keepdim=True)) / total
    upstream *= case["scale"]
    grad = upstream * p * (1 - p) if case["scores"] == "sigmoid" else p * upstream - p * (p * upstream).sum(1, keepdim=True)
    return {"chosen": None, "weights": weights * case["scale"], "counts": None, "bias": None, "gradient": grad}
