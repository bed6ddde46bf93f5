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


@pytest.mark.parametrize("native", [True, False])
def test_shapes_and_types_do_not_depend_on_earlier_calls(native, monkeypatch):
    """What is refused while a type is new is refused, with the same error, once it has been seen; nothing is written."""
    if not native:
        monkeypatch.setattr(operators, "_operators", {})
    long = torch.zeros(9, 8, dtype=torch.int64, device="cuda")
    tokens, table, out = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(9, 8, device="cuda"), torch.full((4, 8), 7.0, device="cuda")
    logits, chosen, weights = torch.zeros(4, 8, device="cuda"), torch.full((4, 2), 7, dtype=torch.int32, device="cuda"), torch.full((4, 2), 7.0, device="cuda")
    counts, sums, keep = torch.full((9,), 7, dtype=torch.int32, device="cuda"), torch.full((9,), 7.0, device="cuda"), torch.ones(4, dtype=torch.bool, device="cuda")
    loss, grad, up = torch.full((3,), 7.0, device="cuda"), torch.full((4, 8), 7.0, device="cuda"), torch.ones(1, device="cuda")
    work = torch.empty(bl.blink_embedding_gradient_workspace(4, 9, 8), dtype=torch.uint8, device="cuda")
    route = dict(logits=logits, k=2, chosen=chosen, weights=weights, counts=counts, sums=sums, workspace=None, keep=keep)
    of_loss, of_gradient = dict(counts=counts, sums=sums, k=2, loss=loss), dict(logits=logits, k=2, chosen=chosen, counts=counts, grad_logits=grad, keep=keep,
                                                                                  grad_weights=weights, grad_loss=up)
    calls = [(bl.blink_embedding, dict(table=table, tokens=tokens, out=out), [dict(table=long), dict(out=long[:4])]),
             (bl.blink_embedding_gradient, dict(tokens=tokens, grad_out=logits, grad_table=table, workspace=work), [dict(grad_out=long[:4]), dict(grad_table=long)]),
             (bl.blink_route, route, [dict(logits=long[:4]), dict(keep=keep.view(2, 2)), dict(counts=counts.view(1, 9)), dict(sums=sums.view(1, 9)),
                                      dict(chosen=chosen.view(2, 4)), dict(weights=weights.view(8))]),
             (bl.blink_route_loss, of_loss, [dict(counts=counts.view(1, 9)), dict(sums=sums.view(9, 1)), dict(loss=loss.view(1, 3))]),
             (bl.blink_route_gradient, of_gradient, [dict(logits=long[:4]), dict(grad_logits=long[:4]), dict(keep=keep.view(4, 1)), dict(counts=counts.view(3, 3)),
                                                     dict(grad_loss=up.view(1, 1)), dict(grad_loss=up[0]), dict(grad_weights=weights.view(8))])]
    for seen in ({}, dict(operators._seen)):
        monkeypatch.setattr(operators, "_seen", seen)
        for dtype in (torch.float32, torch.int32, torch.int64, torch.bool) if seen else ():
            operators._code(torch.zeros(1, dtype=dtype, device="cuda"), "any", (0, 1, 4, -1))
        for call, arguments, changes in calls:
            for change in changes:
                with pytest.raises(ValueError):
                    call(**{**arguments, **change})
    assert all((t == 7).all() for t in (out, chosen, weights, counts, sums, loss, grad)) and (table == 0).all() and (long == 0).all()
