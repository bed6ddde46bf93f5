"""The two ways from Python to an operator, through the native call module and through ctypes, give the same."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_1910_04940_amd as bl  # noqa: E402
from paper_1910_04940_amd import operators  # noqa: E402


def _all(stream):
    g = torch.Generator("cuda").manual_seed(1)
    table = torch.randn(50, 24, generator=g, device="cuda").bfloat16()
    tokens = torch.randint(-1, 50, (3, 40), generator=g, device="cuda")
    rows = torch.empty(120, 24, device="cuda")
    bl.blink_embedding(table, tokens, rows, 2, stream)
    grad = torch.ones(50, 24, device="cuda")
    work = torch.empty(bl.blink_embedding_gradient_workspace(120, 50, 24), dtype=torch.uint8, device="cuda")
    bl.blink_embedding_gradient(tokens, rows, grad, work, 0.5, True, stream)
    logits = torch.randn(120, 12, generator=g, device="cuda")
    keep = torch.rand(120, generator=g, device="cuda") < 0.7
    chosen, weights = torch.empty(120, 3, dtype=torch.int32, device="cuda"), torch.empty(120, 3, device="cuda")
    counts, sums, loss = torch.empty(13, dtype=torch.int32, device="cuda"), torch.empty(13, device="cuda"), torch.empty(3, device="cuda")
    bl.blink_route(logits, 3, chosen, weights, counts, sums, None, keep, True, stream)
    bl.blink_route_loss(counts, sums, 3, loss, 0.1, 0.2, stream)
    out = torch.empty_like(logits)
    bl.blink_route_gradient(logits, 3, chosen, counts, out, keep, True, weights, loss[:1], 0.1, 0.2, stream)
    return rows, grad, chosen, weights, counts, sums, loss, out


def test_both_ways(monkeypatch):
    stream = torch.cuda.current_stream().cuda_stream
    _all(stream)      # the types have been seen
    assert operators._operators, "the native call module is not built"
    longer = operators._code
    monkeypatch.setattr(operators, "_code", lambda *a: pytest.fail("the usual call went the longer way"))
    native = _all(stream)
    monkeypatch.setattr(operators, "_code", longer)
    monkeypatch.setattr(operators, "_operators", {})
    for a, b in zip(native, _all(stream)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_what_does_not_fit(native, monkeypatch):
    if not native:
        monkeypatch.setattr(operators, "_operators", {})
    table, tokens, out = torch.zeros(9, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, 8, device="cuda")
    for _ in range(2):     # types not seen, and seen
        for bad in ((table.cpu(), tokens, out), (table, tokens.cpu(), out), (table, tokens, out[:, :7]), (table, tokens, out[:3]), (table, tokens.float(), out),
                    (table.t(), tokens, out), (table, tokens, out[0]), (table.double(), tokens, out), (table, torch.zeros(8, dtype=torch.int64, device="cuda")[::2], out)):
            with pytest.raises(ValueError):
                bl.blink_embedding(*bad)
        with pytest.raises(ctypes.ArgumentError):      # as a collective's number of another kind
            bl.blink_embedding(table, tokens, out, "scale")
        logits, counts, sums = torch.zeros(4, 8, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(9, device="cuda")
        chosen, weights = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
        for change in (dict(chosen=chosen.long()), dict(weights=weights[:, :1]), dict(counts=counts[:8]), dict(sums=sums.double()),
                       dict(keep=torch.zeros(3, dtype=torch.bool, device="cuda")), dict(workspace=torch.zeros(4))):
            with pytest.raises(ValueError):
                bl.blink_route(**{**dict(logits=logits, k=2, chosen=chosen, weights=weights, counts=counts, sums=sums, workspace=None), **change})
        with pytest.raises(bl.BlinkError) as e:
            bl.blink_route(logits, 0, chosen[:, :0].contiguous(), weights[:, :0].contiguous(), counts, sums, None)
        assert e.value.status == bl.BLINK_EINVAL
