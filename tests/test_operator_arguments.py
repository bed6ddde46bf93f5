"""What the operators around the collectives refuse, at the C boundary (addresses that nothing reads) and on tensors."""
import ctypes as C

import pytest

import paper_1910_04940_amd as bl
from paper_1910_04940_amd import binding

torch = pytest.importorskip("torch")

P = 1 << 20   # an address on any alignment; every call below is refused, or has nothing to do
STEP = (C.c_float * 3)(1.5, -0.5, 0.0)


def embedding(table=P, table_type=1, vocab=10, dim=8, table_stride=8, tokens=P, token_type=0, n=4, scale=1.0, out=P, out_type=1, out_stride=8):
    return binding.lib().blink_embedding(table, table_type, vocab, dim, table_stride, tokens, token_type, n, scale, out, out_type, out_stride, None)


def gradient(tokens=P, token_type=4, n=4, grad=P, grad_type=2, grad_stride=8, accumulate=0, table=P, table_type=1, vocab=10, dim=8, table_stride=8,
             workspace=P, size=1 << 30):
    return binding.lib().blink_embedding_gradient(tokens, token_type, n, grad, grad_type, grad_stride, 1.0, accumulate, table, table_type, vocab, dim,
                                                  table_stride, workspace, size, None)


def route(logits=P, dtype=2, n=1000, experts=8, stride=8, k=2, normalize=0, chosen=P, weights=P, counts=P, sums=P, workspace=P, size=1 << 30):
    return binding.lib().blink_route(logits, dtype, n, experts, stride, None, k, normalize, chosen, weights, counts, sums, workspace, size, None)


def loss(counts=P, sums=P, experts=8, k=2, out=P):
    return binding.lib().blink_route_loss(counts, sums, experts, k, 0.1, 0.1, out, None)


def route_gradient(logits=P, dtype=2, n=4, experts=8, stride=8, k=2, normalize=0, chosen=P, grad_weights=None, counts=P, grad_loss=None, out=P, out_stride=8):
    return binding.lib().blink_route_gradient(logits, dtype, n, experts, stride, None, k, normalize, chosen, grad_weights, counts, grad_loss, 0.1, 0.1, out,
                                              out_stride, None)


def orthogonalize(matrix=P, dtype=1, batch=1, rows=8, cols=8, row=8, apart=64, co=STEP, steps=1, eps=0.0, out=P, out_row=8, out_apart=64, workspace=P,
                  size=1 << 30):
    return binding.lib().blink_orthogonalize(matrix, dtype, batch, rows, cols, row, apart, co, steps, eps, out, out_row, out_apart, workspace, size, None)


def step(weights=P, weights_out=P, momentum=P, momentum_out=P, grad=P, grad_type=1, batch=1, rows=8, cols=8, nesterov=0, co=STEP, steps=1, eps=0.0,
         workspace=P, size=1 << 30):
    return binding.lib().blink_orthogonal_step(weights, weights_out, momentum, momentum_out, grad, grad_type, batch, rows, cols, 0.9, nesterov, co, steps, eps,
                                               0.1, 0.0, workspace, size, None)


REFUSED = [
    *[(embedding, a) for a in (dict(table_type=0), dict(table_type=4), dict(out_type=-1), dict(token_type=1), dict(n=1 << 31), dict(vocab=1 << 31),
                               dict(table_stride=7), dict(out_stride=7), dict(table=None), dict(tokens=None), dict(out=None), dict(table=P + 2),
                               dict(tokens=P + 2), dict(out=P + 1, out_type=2), dict(dim=(1 << 21) + 1, table_stride=1 << 22, out_stride=1 << 22))],
    *[(gradient, a) for a in (dict(table_type=0), dict(grad_type=4), dict(token_type=2), dict(n=1 << 31), dict(vocab=(1 << 31) - 1), dict(accumulate=2),
                              dict(grad_stride=7), dict(table_stride=7), dict(tokens=P + 4), dict(grad=None), dict(table=None), dict(workspace=None),
                              dict(workspace=P + 128), dict(size=100))],
    *[(route, a) for a in (dict(dtype=0), dict(experts=0), dict(experts=1025, stride=1025), dict(k=0), dict(k=9), dict(stride=7), dict(normalize=2),
                           dict(logits=None), dict(logits=P + 1), dict(chosen=None), dict(weights=P + 2), dict(counts=None), dict(sums=None),
                           dict(workspace=None), dict(size=16), dict(n=1 << 31))],
    *[(loss, a) for a in (dict(counts=None), dict(sums=None), dict(out=None), dict(experts=0), dict(k=9), dict(out=P + 2))],
    *[(route_gradient, a) for a in (dict(dtype=4), dict(k=0), dict(stride=7), dict(out_stride=7), dict(normalize=-1), dict(logits=None), dict(out=None),
                                    dict(counts=None), dict(chosen=None, grad_weights=P), dict(grad_weights=P + 1), dict(grad_loss=P + 2))],
    *[(orthogonalize, a) for a in (dict(dtype=0), dict(batch=0), dict(batch=65536), dict(rows=0), dict(cols=0), dict(rows=(1 << 20) + 1), dict(row=7),
                                   dict(out_row=7), dict(batch=2, out_apart=63), dict(steps=0), dict(steps=65), dict(co=None), dict(eps=-1.0),
                                   dict(eps=float("nan")), dict(eps=float("inf")), dict(matrix=None), dict(out=None), dict(workspace=None), dict(size=64),
                                   dict(workspace=P + 16))],
    *[(step, a) for a in (dict(weights=None), dict(weights_out=None), dict(momentum=None), dict(momentum_out=P + 2), dict(grad=None), dict(grad_type=0),
                          dict(nesterov=2), dict(steps=0), dict(co=None), dict(eps=-1.0), dict(batch=0), dict(size=0), dict(workspace=None))],
]


@pytest.mark.parametrize("call,change", REFUSED, ids=[f"{f.__name__} {c}" for f, c in REFUSED])
def test_refused(call, change):
    assert call(**change) == bl.BLINK_EINVAL


@pytest.mark.parametrize("co", [(2.1, 0.0, 0.0), (7.9, -8.0, 1.0), (float("nan"), 0.0, 0.0), (1.5, float("inf"), 0.0), (1.0, 1.0, 0.0)])
def test_coefficients_that_leave_the_range(co):
    assert orthogonalize(co=(C.c_float * 3)(*co)) == bl.BLINK_EINVAL
    assert step(co=(C.c_float * 3)(*co)) == bl.BLINK_EINVAL


def test_a_later_step_counts():
    """1.9 x from singular values up to 1 is fine once, not twice."""
    assert orthogonalize(co=(C.c_float * 6)(1.9, 0, 0, 1.9, 0, 0), steps=2) == bl.BLINK_EINVAL


def test_calls_with_nothing_to_do():
    assert embedding(n=0, tokens=None, out=None) == bl.BLINK_OK
    assert embedding(dim=0, table=None, out=None) == bl.BLINK_OK
    assert gradient(n=0, tokens=None, grad=None, accumulate=1) == bl.BLINK_OK
    assert gradient(vocab=0, table=None) == bl.BLINK_OK
    assert route_gradient(n=0, logits=None, out=None) == bl.BLINK_OK


def test_workspaces_follow_the_sizes():
    L = binding.lib()
    assert bl.blink_embedding_gradient_workspace(1000, 5000, 64) > 1000 * 16
    assert L.blink_embedding_gradient_workspace(1 << 31, 10, 10) == 0
    assert bl.blink_route_workspace(64, 8) == 0 < bl.blink_route_workspace(100_000, 8)
    assert bl.blink_route_workspace(64, 1025) == 0
    assert bl.blink_orthogonalize_workspace(1, 64, 64, bl.BLINK_BF16) < bl.blink_orthogonalize_workspace(1, 64, 64, bl.BLINK_FP32)
    assert bl.blink_orthogonalize_workspace(1, 300, 200, bl.BLINK_FP32) == bl.blink_orthogonalize_workspace(1, 200, 300, bl.BLINK_FP32)
    assert bl.blink_orthogonalize_workspace(0, 64, 64, bl.BLINK_FP32) == 0 == bl.blink_orthogonalize_workspace(1, 64, 64, bl.BLINK_INT32)


@pytest.mark.parametrize("batch,rows,cols", [(16, 16, 8192), (16, 4096, 22), (8, 32, 8192), (16, 64, 4096), (32, 128, 2048), (200, 16, 16), (128, 64, 64),
                                             (8, 16_000, 16), (48, 180, 1000), (64, 150, 512), (16, 320, 4096), (96, 250, 300), (96, 400, 520)])
def test_narrow_matrices_are_not_blown_up(batch, rows, cols):
    """X, its transposes, A and B with sides rounded up to tiles of 64, or to larger ones that add no more than a third: 16/9 in all at the most,
    and up to 1024 sums of the norm to a matrix."""
    m, n = (max(-(-side // 64) * 64, side * 4 / 3) for side in sorted((rows, cols)))
    assert bl.blink_orthogonalize_workspace(batch, rows, cols, bl.BLINK_FP32) <= batch * (4 * (3 * m * n + 2 * m * m) + 8 * 1024) + 8 * 256


def test_collectives_take_none_of_the_new_types():
    import synth_inputs as si
    t = si.complete_graph(4)
    s = bl.blink_make_schedule(bl.blink_pack_trees(t.k, t.src, t.dst, t.cap, 0), bl.BLINK_OP_ALLREDUCE, 0, 16)
    for dtype in (bl.BLINK_BF16, bl.BLINK_FP16, bl.BLINK_INT64):
        with pytest.raises(bl.BlinkError) as e:
            bl.blink_allreduce([16, 32, 48, 64], 0, dtype, s)
        assert e.value.status == bl.BLINK_EINVAL


def test_tensors_that_do_not_fit():
    f, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: bl.blink_embedding(f, i, f), lambda: bl.blink_embedding_gradient(i, f, f, None),
                 lambda: bl.blink_route(f, 2, i, f, i, f, None), lambda: bl.blink_orthogonalize(f, f, None),
                 lambda: bl.blink_orthogonal_step(f, f, f, f, f, None, 0.1),
                 lambda: bl.blink_route_loss(i.int(), f[0], 2, f[0]), lambda: bl.blink_route_gradient(f, 2, i, i, f)):
        with pytest.raises(ValueError):     # on the host
            call()
    with pytest.raises(ValueError):
        bl.blink_embedding(f.double(), i, f)
