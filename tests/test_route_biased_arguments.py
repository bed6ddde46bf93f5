"""What the router with scores, a bias and groups refuses, at the C boundary (addresses that nothing reads) and on tensors."""
import pytest

import paper_1910_04940_amd as bl
from paper_1910_04940_amd import binding

torch = pytest.importorskip("torch")

P = 1 << 20


def route(logits=P, dtype=2, n=1000, experts=8, stride=8, keep=None, bias=P, k=2, groups=2, kept=1, scores=0, normalize=0, scale=1.0, chosen=P, weights=P,
          counts=P, workspace=P, size=1 << 30):
    return binding.lib().blink_route_biased(logits, dtype, n, experts, stride, keep, bias, k, groups, kept, scores, normalize, scale, chosen, weights, counts,
                                            workspace, size, None)


def step(counts=P, bias=P, experts=8, rate=0.1, out=P):
    return binding.lib().blink_route_bias(counts, bias, experts, rate, out, None)


def gradient(logits=P, dtype=2, n=4, experts=8, stride=8, keep=None, k=2, scores=0, normalize=0, scale=1.0, chosen=P, grad_weights=P, out=P, out_stride=8):
    return binding.lib().blink_route_biased_gradient(logits, dtype, n, experts, stride, keep, k, scores, normalize, scale, chosen, grad_weights, out, out_stride,
                                                     None)


NAN, INF = float("nan"), float("inf")
REFUSED = [
    *[(route, a) for a in (dict(dtype=0), dict(dtype=5), dict(experts=0), dict(experts=1025, stride=1025), dict(k=0), dict(k=5), dict(k=9, kept=2), dict(stride=7),
                           dict(groups=0), dict(groups=3), dict(groups=16), dict(kept=0), dict(kept=3), dict(experts=130, stride=130, groups=65), dict(scores=2),
                           dict(scores=-1), dict(normalize=2), dict(scale=NAN), dict(scale=INF), dict(logits=None), dict(logits=P + 1), dict(bias=P + 2),
                           dict(chosen=None), dict(weights=P + 2), dict(counts=None), dict(workspace=None), dict(workspace=P + 64), dict(size=16), dict(n=1 << 31))],
    *[(step, a) for a in (dict(counts=None), dict(bias=None), dict(out=None), dict(out=P + 2), dict(experts=0), dict(experts=1025), dict(rate=NAN))],
    *[(gradient, a) for a in (dict(dtype=4), dict(k=0), dict(k=9), dict(stride=7), dict(out_stride=7), dict(scores=2), dict(normalize=-1), dict(scale=INF),
                              dict(logits=None), dict(out=None), dict(chosen=None), dict(grad_weights=None), dict(grad_weights=P + 1), dict(n=1 << 31))],
]


@pytest.mark.parametrize("call,change", REFUSED, ids=[f"{f.__name__} {c}" for f, c in REFUSED])
def test_refused(call, change):
    assert call(**change) == bl.BLINK_EINVAL


def test_workspace_sizes():
    size = bl.blink_route_biased_workspace
    assert size(1 << 31, 8) == 0 and size(4, 0) == 0 and size(4, 1025) == 0 and size(1, 8) == 0 and size(0, 8) == 0 and size(1 << 20, 8) > 0


def test_no_tokens():
    assert gradient(n=0, logits=None, out=None, chosen=None, grad_weights=None) == bl.BLINK_OK


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_tensors_that_do_not_fit(native, monkeypatch):
    from paper_1910_04940_amd import operators
    if not native:
        monkeypatch.setattr(operators, "_operators", {})
    t = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")   # noqa: E731
    i32 = torch.int32
    good = dict(logits=t(4, 8), k=2, chosen=t(4, 2, dtype=i32), weights=t(4, 2), counts=t(9, dtype=i32), workspace=None, bias=t(8), keep=t(4, dtype=torch.bool),
                groups=2, kept_groups=1)
    back = dict(logits=t(4, 8), k=2, chosen=t(4, 2, dtype=i32), grad_weights=t(4, 2), grad_logits=t(4, 8))
    for _ in range(2):
        for change in (dict(chosen=t(4, 2)), dict(weights=t(4, 1)), dict(counts=t(8, dtype=i32)), dict(bias=t(7)), dict(bias=t(8, dtype=torch.float64)),
                       dict(keep=t(3, dtype=torch.bool)), dict(workspace=torch.zeros(4)), dict(scores="tanh"), dict(logits=t(4, 8, dtype=torch.float64)),
                       dict(logits=t(8, 4).t())):
            with pytest.raises(ValueError):
                bl.blink_route_biased(**{**good, **change})
        for change in (dict(groups=3), dict(kept_groups=3), dict(k=5, chosen=t(4, 5, dtype=i32), weights=t(4, 5))):
            with pytest.raises(bl.BlinkError) as e:
                bl.blink_route_biased(**{**good, **change})
            assert e.value.status == bl.BLINK_EINVAL
        for change in (dict(grad_weights=t(4, 3)), dict(grad_logits=t(4, 8, dtype=torch.bfloat16)), dict(grad_logits=t(3, 8)), dict(chosen=t(4, 2)), dict(scores=1)):
            with pytest.raises(ValueError):
                bl.blink_route_biased_gradient(**{**back, **change})
        for change in (dict(counts=t(8, dtype=i32)), dict(bias_out=t(7)), dict(bias=t(2, 4)), dict(counts=t(9))):
            with pytest.raises(ValueError):
                bl.blink_route_bias(**{**dict(counts=t(9, dtype=i32), bias=t(8), bias_out=t(8), rate=0.1), **change})
        bl.blink_route_biased(**good)
        bl.blink_route_biased_gradient(**back)
