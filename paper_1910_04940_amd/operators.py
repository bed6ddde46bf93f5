"""The operators around the collectives (see include/blink.h): the same names, on tensors.

Sizes, types and strides are taken from the tensors, which must be on the GPU with elements of a row next to one
another; a result goes into the tensor that is given for it.  stream: hipStream_t as int.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

from . import binding
from .binding import BLINK_BF16, BLINK_FP16, BLINK_FP32, BLINK_INT32, BLINK_INT64, _check

# Five steps (a, b, c) that move every singular value above 0.003 to between 0.68 and 1.21.
BLINK_STEPS = ((3.4445, -4.7750, 2.0315),) * 5

_CODES = {"torch.float32": BLINK_FP32, "torch.bfloat16": BLINK_BF16, "torch.float16": BLINK_FP16, "torch.int32": BLINK_INT32,
          "torch.int64": BLINK_INT64, "torch.bool": -1, "torch.uint8": -1}
_seen = {}   # a tensor's dtype -> its code, once asked
_operators = binding._operators


# A small operator takes the GPU 2 to 5 us, less than a wasteful call takes here: what is as usual (tensors of types seen before, plain
# numbers) goes to the library through _blinkcall, which then returns a status; anything else, and what is not allowed, the longer way below.
def _usual(name: str, *arguments):
    native = _operators.get(name)
    return None if native is None else native[0](native[1], _seen, *arguments)


_FLOAT, _TOKEN, _BYTE, _INT32, _FP32 = (BLINK_FP32, BLINK_BF16, BLINK_FP16), (BLINK_INT32, BLINK_INT64), (-1,), (BLINK_INT32,), (BLINK_FP32,)


def _code(t, name: str, types) -> int:
    """The tensor's type, one of `types`; the tensor is on the GPU."""
    dtype = t.dtype
    code = _seen.get(dtype)
    if code is None:
        code = _seen[dtype] = _CODES.get(str(dtype), -2)
    if code not in types:
        raise ValueError(f"{name}: {dtype} is not a type that it may have")
    if not t.is_cuda:
        raise ValueError(f"{name} is not on the GPU")
    return code


def _whole(t, name: str, types, shape: Tuple[int, ...]) -> int:
    """Address of a contiguous tensor of that shape."""
    _code(t, name, types)
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of shape {shape}: got {tuple(t.shape)}")
    return t.data_ptr()


def _rows(t, name: str, types, rows: Optional[int] = None, cols: Optional[int] = None) -> Tuple[int, int, int, int, int]:
    """(address, type, rows, columns, stride of the rows) of a matrix whose rows are contiguous."""
    code = _code(t, name, types)
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name} must be a matrix ({'any' if rows is None else rows} x {'any' if cols is None else cols}): got {tuple(t.shape)}")
    r, c = t.shape
    stride, one = t.stride()
    if c > 1 and one != 1:
        raise ValueError(f"{name}: elements of a row must follow one another")
    return t.data_ptr(), code, r, c, stride if r > 1 else max(stride, c)


def _space(t) -> Tuple[Optional[int], int]:
    if t is None:
        return None, 0
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("workspace must be contiguous, on the GPU")
    return t.data_ptr(), t.numel() * t.element_size()


def blink_embedding(table, tokens, out, scale: float = 1.0, stream: int = 0) -> None:
    """out[i] = scale * table[tokens[i]]; zeros where the token is outside the table."""
    status = _usual("embedding", table, tokens, out, scale, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_embedding")
    at, kind, vocab, dim, stride = _rows(table, "table", _FLOAT)
    token = _code(tokens, "tokens", _TOKEN)
    n = tokens.numel()
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    to, out_kind, _, _, out_stride = _rows(out, "out", _FLOAT, n, dim)
    status = (binding._lib or binding.lib()).blink_embedding(at, kind, vocab, dim, stride, tokens.data_ptr(), token, n, scale, to, out_kind, out_stride, stream)
    if status:
        _check(status, "blink_embedding")


def blink_embedding_gradient_workspace(n_tokens: int, vocab: int, dim: int) -> int:
    return binding.lib().blink_embedding_gradient_workspace(n_tokens, vocab, dim)


def blink_embedding_gradient(tokens, grad_out, grad_table, workspace, scale: float = 1.0, accumulate: bool = False, stream: int = 0) -> None:
    """grad_table[v] = scale * sum of grad_out[i] over the tokens that are v, added to what is there if `accumulate`."""
    status = _usual("embedding_gradient", tokens, grad_out, grad_table, workspace, scale, accumulate, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_embedding_gradient")
    token = _code(tokens, "tokens", _TOKEN)
    n = tokens.numel()
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    to, kind, vocab, dim, stride = _rows(grad_table, "grad_table", _FLOAT)
    at, grad_kind, _, _, grad_stride = _rows(grad_out, "grad_out", _FLOAT, n, dim)
    space, size = _space(workspace)
    status = (binding._lib or binding.lib()).blink_embedding_gradient(tokens.data_ptr(), token, n, at, grad_kind, grad_stride, scale, 1 if accumulate else 0, to,
                                                                      kind, vocab, dim, stride, space, size, stream)
    if status:
        _check(status, "blink_embedding_gradient")


def blink_route_workspace(n_tokens: int, n_experts: int) -> int:
    return binding.lib().blink_route_workspace(n_tokens, n_experts)


def blink_route(logits, k: int, chosen, weights, counts, sums, workspace, keep=None, normalize: bool = False, stream: int = 0) -> None:
    """The k largest logits of every token; per-expert counts and sums of probabilities."""
    status = _usual("route", logits, k, chosen, weights, counts, sums, workspace, keep, normalize, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_route")
    at, kind, n, experts, stride = _rows(logits, "logits", _FLOAT)
    kept = None if keep is None else _whole(keep, "keep", _BYTE, (n,))
    space, size = _space(workspace)
    status = (binding._lib or binding.lib()).blink_route(
        at, kind, n, experts, stride, kept, k, 1 if normalize else 0, _whole(chosen, "chosen", _INT32, (n, k)), _whole(weights, "weights", _FP32, (n, k)),
        _whole(counts, "counts", _INT32, (experts + 1,)), _whole(sums, "sums", _FP32, (experts + 1,)), space, size, stream)
    if status:
        _check(status, "blink_route")


def blink_route_loss(counts, sums, k: int, loss, balance: float = 0.0, z: float = 0.0, stream: int = 0) -> None:
    """loss = (both, the balance loss, the logits' loss) from counts and sums, over all ranks."""
    status = _usual("route_loss", counts, sums, k, loss, balance, z, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_route_loss")
    experts = counts.numel() - 1
    status = (binding._lib or binding.lib()).blink_route_loss(_whole(counts, "counts", _INT32, (experts + 1,)), _whole(sums, "sums", _FP32, (experts + 1,)), experts,
                                                              k, balance, z, _whole(loss, "loss", _FP32, (3,)), stream)
    if status:
        _check(status, "blink_route_loss")


def blink_route_gradient(logits, k: int, chosen, counts, grad_logits, keep=None, normalize: bool = False, grad_weights=None, grad_loss=None,
                         balance: float = 0.0, z: float = 0.0, stream: int = 0) -> None:
    """Gradient of the logits: of the loss (times grad_loss[0]) and through the weights."""
    status = _usual("route_gradient", logits, k, chosen, counts, grad_logits, keep, normalize, grad_weights, grad_loss, balance, z, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_route_gradient")
    at, kind, n, experts, stride = _rows(logits, "logits", _FLOAT)
    to, out_kind, _, _, out_stride = _rows(grad_logits, "grad_logits", _FLOAT, n, experts)
    if out_kind != kind:
        raise ValueError("grad_logits must have the type of logits")
    status = (binding._lib or binding.lib()).blink_route_gradient(
        at, kind, n, experts, stride, None if keep is None else _whole(keep, "keep", _BYTE, (n,)), k, 1 if normalize else 0,
        _whole(chosen, "chosen", _INT32, (n, k)), None if grad_weights is None else _whole(grad_weights, "grad_weights", _FP32, (n, k)),
        _whole(counts, "counts", _INT32, (experts + 1,)), None if grad_loss is None else _whole(grad_loss, "grad_loss", _FP32, (1,)), balance, z, to, out_stride,
        stream)
    if status:
        _check(status, "blink_route_gradient")


def _coefficients(steps: Sequence[Sequence[float]]):
    flat = [float(v) for step in steps for v in step]
    if len(flat) != 3 * len(steps):
        raise ValueError("three coefficients to a step")
    return (C.c_float * len(flat))(*flat), len(steps)


def _matrices(t, name: str, types, shape=None) -> Tuple[int, int, int, int, int, int, int]:
    """(address, type, batch, rows, columns, stride of the rows, of the matrices) of one matrix or a batch."""
    code = _code(t, name, types)
    if t.dim() not in (2, 3) or (shape is not None and tuple(t.shape) != shape):
        raise ValueError(f"{name} must be {'a matrix or a batch of them' if shape is None else f'of shape {shape}'}: got {tuple(t.shape)}")
    batch = t.shape[0] if t.dim() == 3 else 1
    rows, cols = t.shape[-2:]
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: elements of a row must follow one another")
    return t.data_ptr(), code, batch, rows, cols, t.stride(-2) if rows > 1 else max(cols, t.stride(-2)), t.stride(0) if t.dim() == 3 else 0


def blink_orthogonalize_workspace(batch: int, rows: int, cols: int, dtype: int) -> int:
    return binding.lib().blink_orthogonalize_workspace(batch, rows, cols, dtype)


def blink_orthogonalize(matrix, out, workspace, coefficients: Sequence[Sequence[float]] = BLINK_STEPS, eps: float = 1e-7, stream: int = 0) -> None:
    """Every matrix moved towards the nearest one with orthonormal rows (columns, if there are fewer)."""
    at, kind, batch, rows, cols, row, apart = _matrices(matrix, "matrix", _FLOAT)
    to, out_kind, _, _, _, out_row, out_apart = _matrices(out, "out", _FLOAT, tuple(matrix.shape))
    if out_kind != kind:
        raise ValueError("out must have the type of the matrix")
    co, steps = _coefficients(coefficients)
    space, size = _space(workspace)
    status = (binding._lib or binding.lib()).blink_orthogonalize(at, kind, batch, rows, cols, row, apart, co, steps, eps, to, out_row, out_apart, space, size, stream)
    if status:
        _check(status, "blink_orthogonalize")


def blink_orthogonal_step(weights, momentum, grad, weights_out, momentum_out, workspace, rate: float, beta: float = 0.95, nesterov: bool = True,
                          decay: float = 0.0, coefficients: Sequence[Sequence[float]] = BLINK_STEPS, eps: float = 1e-7, stream: int = 0) -> None:
    """momentum_out = beta * momentum + grad; weights_out = (1 - decay) * weights - rate * the update, orthogonalised.  weights_out and momentum_out
    may be weights and momentum."""
    shape = tuple(weights.shape)
    _, _, batch, rows, cols, _, _ = _matrices(weights, "weights", _FP32)
    kind = _code(grad, "grad", _FLOAT)
    co, steps = _coefficients(coefficients)
    space, size = _space(workspace)
    status = (binding._lib or binding.lib()).blink_orthogonal_step(
        _whole(weights, "weights", _FP32, shape), _whole(weights_out, "weights_out", _FP32, shape), _whole(momentum, "momentum", _FP32, shape),
        _whole(momentum_out, "momentum_out", _FP32, shape), _whole(grad, "grad", _FLOAT, shape), kind, batch, rows, cols, beta, 1 if nesterov else 0, co, steps,
        eps, rate, decay, space, size, stream)
    if status:
        _check(status, "blink_orthogonal_step")
