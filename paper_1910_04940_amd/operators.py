"""The operators around the collectives (see include/blink.h): the same names, on tensors.

Sizes, types and strides are taken from the tensors, which must be on the GPU with elements of a row next to one
another; a result goes into the tensor that is given for it.  stream: hipStream_t as int.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Sequence, Tuple

import numpy as np

from . import binding
from .binding import BLINK_BF16, BLINK_FP16, BLINK_FP32, BLINK_FP8, BLINK_INT32, BLINK_INT64, BLINK_SIGMOID, BLINK_SOFTMAX, _check, _handle

# Five steps (a, b, c) that move every singular value above 0.003 to between 0.68 and 1.21.
BLINK_STEPS = ((3.4445, -4.7750, 2.0315),) * 5

_CODES = {"torch.float32": BLINK_FP32, "torch.bfloat16": BLINK_BF16, "torch.float16": BLINK_FP16, "torch.int32": BLINK_INT32,
          "torch.int64": BLINK_INT64, "torch.float8_e4m3fn": BLINK_FP8, "torch.bool": -1, "torch.uint8": -1}
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


_SCORES = {"sigmoid": BLINK_SIGMOID, "softmax": BLINK_SOFTMAX}


def _scores(name: str) -> int:
    code = _SCORES.get(name)
    if code is None:
        raise ValueError(f"scores are {' or '.join(_SCORES)}: got {name!r}")
    return code


def blink_route_biased_workspace(n_tokens: int, n_experts: int) -> int:
    return binding.lib().blink_route_biased_workspace(n_tokens, n_experts)


def blink_route_biased(logits, k: int, chosen, weights, counts, workspace, bias=None, keep=None, groups: int = 1, kept_groups: int = 1, scores: str = "sigmoid",
                       normalize: bool = False, scale: float = 1.0, stream: int = 0) -> None:
    """The k experts with the largest scores + bias of every token, in the kept_groups best of its groups; weights from the scores alone; per-expert counts."""
    code = _scores(scores)
    status = _usual("route_biased", logits, k, chosen, weights, counts, workspace, bias, keep, groups, kept_groups, code, normalize, scale, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_route_biased")
    at, kind, n, experts, stride = _rows(logits, "logits", _FLOAT)
    space, size = _space(workspace)
    status = (binding._lib or binding.lib()).blink_route_biased(
        at, kind, n, experts, stride, None if keep is None else _whole(keep, "keep", _BYTE, (n,)), None if bias is None else _whole(bias, "bias", _FP32, (experts,)),
        k, groups, kept_groups, code, 1 if normalize else 0, scale, _whole(chosen, "chosen", _INT32, (n, k)), _whole(weights, "weights", _FP32, (n, k)),
        _whole(counts, "counts", _INT32, (experts + 1,)), space, size, stream)
    if status:
        _check(status, "blink_route_biased")


def blink_route_bias(counts, bias, bias_out, rate: float, stream: int = 0) -> None:
    """The bias a step up where an expert has fewer than the mean of the counts (over all ranks), down where more.  bias_out may be bias."""
    status = _usual("route_bias", counts, bias, bias_out, rate, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_route_bias")
    experts = bias.numel()
    status = (binding._lib or binding.lib()).blink_route_bias(_whole(counts, "counts", _INT32, (experts + 1,)), _whole(bias, "bias", _FP32, (experts,)), experts,
                                                              rate, _whole(bias_out, "bias_out", _FP32, (experts,)), stream)
    if status:
        _check(status, "blink_route_bias")


def blink_route_biased_gradient(logits, k: int, chosen, grad_weights, grad_logits, keep=None, scores: str = "sigmoid", normalize: bool = False,
                                scale: float = 1.0, stream: int = 0) -> None:
    """Gradient of the logits through the weights of blink_route_biased."""
    code = _scores(scores)
    status = _usual("route_biased_gradient", logits, k, chosen, grad_weights, grad_logits, keep, code, normalize, scale, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_route_biased_gradient")
    at, kind, n, experts, stride = _rows(logits, "logits", _FLOAT)
    to, out_kind, _, _, out_stride = _rows(grad_logits, "grad_logits", _FLOAT, n, experts)
    if out_kind != kind:
        raise ValueError("grad_logits must have the type of logits")
    status = (binding._lib or binding.lib()).blink_route_biased_gradient(
        at, kind, n, experts, stride, None if keep is None else _whole(keep, "keep", _BYTE, (n,)), k, code, 1 if normalize else 0, scale,
        _whole(chosen, "chosen", _INT32, (n, k)), _whole(grad_weights, "grad_weights", _FP32, (n, k)), to, out_stride, stream)
    if status:
        _check(status, "blink_route_biased_gradient")


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


class Update:
    """Owns a blink_update_t handle, and the tensors whose addresses are in it."""

    def __init__(self, handle: int, tensors):
        self._h = C.c_void_p(handle)
        self._update = handle
        self.tensors = tensors

    def __del__(self):
        if getattr(self, "_h", None) and binding is not None and binding._lib is not None:
            binding._lib.blink_update_free(self._h)
            self._h = self._update = None


def blink_make_update(grads: Sequence, weights: Optional[Sequence] = None, moments1: Optional[Sequence] = None, moments2: Optional[Sequence] = None,
                      masters: Optional[Sequence] = None, scales1: Optional[Sequence] = None, scales2: Optional[Sequence] = None,
                      rates: Optional[Sequence[float]] = None, decays: Optional[Sequence[float]] = None) -> Update:
    """The tensors that an optimiser changes, a place in every list for each (None: it has none): contiguous, on one device.  Where weights are
    None the gradient counts in the norm only.  Moments: float32, or float8_e4m3fn with float32 scales, one for every 256 elements; zeros before
    the first step (scales need not be).  Nothing but gradients may overlap: weights that two names stand for are listed once.  Addresses are
    kept: a tensor that moves (a gradient that is freed after each step) needs a new list."""
    lists = {"grad": grads, "weights": weights, "master": masters, "moment1": moments1, "moment2": moments2, "scale1": scales1, "scale2": scales2}
    n = len(grads)
    if n == 0:
        raise ValueError("a list of tensors has at least one")
    for name, values in (*lists.items(), ("rates", rates), ("decays", decays)):
        if values is not None and len(values) != n:
            raise ValueError(f"{name}: {n} tensors, {len(values)} places")
    table = np.zeros(n, binding.UPDATE_TENSOR_DTYPE)
    device = None if grads[0] is None else grads[0].device
    for i, row in enumerate(table):
        got = {name: values[i] for name, values in lists.items() if values is not None and values[i] is not None}
        if "grad" not in got:
            raise ValueError("every tensor has a gradient")
        many = got["grad"].numel()
        eight = "moment1" in got and _code(got["moment1"], "moment1", (BLINK_FP32, BLINK_FP8)) == BLINK_FP8
        for name, t in got.items():
            scale = name.startswith("scale")
            kind = _code(t, name, _FLOAT if name in ("grad", "weights") else (BLINK_FP8 if eight else BLINK_FP32,) if name.startswith("moment") else _FP32)
            if not t.is_contiguous() or t.numel() != (-(-many // 256) if scale else many):
                raise ValueError(f"{name} of tensor {i} must be contiguous, of {-(-many // 256) if scale else many} elements: got {tuple(t.shape)}")
            if t.device != device:
                raise ValueError(f"{name} of tensor {i} is on another device")
            row[name] = t.data_ptr() if t.numel() else 0
            if name == "grad":
                row["grad_type"] = kind
            elif name == "weights":
                row["weight_type"] = kind
        if "weights" in got:
            for name in ("moment1", "moment2", "scale1", "scale2"):
                if (name in got) != (eight or name.startswith("moment")):
                    raise ValueError(f"tensor {i}: weights have moments, moments in 8 bits scales")
            row["moment_type"] = BLINK_FP8 if eight else BLINK_FP32
            if many == 0:   # (nothing to step; an address is what says that there are weights)
                for name in got:
                    row[name] = 0
        elif len(got) > 1:
            raise ValueError(f"tensor {i} has no weights that its other tensors go with")
        row["elements"] = many
        row["rate"], row["decay"] = 1.0 if rates is None else rates[i], 0.0 if decays is None else decays[i]
    out = C.c_void_p()
    import torch
    with torch.cuda.device(device):
        _check(binding.lib().blink_make_update(table.ctypes.data, n, C.byref(out)), "blink_make_update")
    return Update(out.value, [t for values in lists.values() if values is not None for t in values])


def blink_gradient_norm_workspace(update: Update) -> int:
    return binding.lib().blink_gradient_norm_workspace(_handle(update, Update))


def blink_gradient_norm(update: Update, norm, workspace, max_norm: float = math.inf, factor: float = 1.0, step=None, stream: int = 0) -> None:
    """norm = (length of all gradients times factor, what a step is to multiply them by); step, an int32, is counted up where all are finite."""
    status = _usual("gradient_norm", update, norm, workspace, max_norm, factor, step, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_gradient_norm")
    space, size = _space(workspace)
    status = (binding._lib or binding.lib()).blink_gradient_norm(
        _handle(update, Update), max_norm, factor, _whole(norm, "norm", _FP32, (2,)), None if step is None else _whole(step, "step", _INT32, (1,)), space, size, stream)
    if status:
        _check(status, "blink_gradient_norm")


def blink_adamw_step(update: Update, step, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, scale=None, rate=None, seed: int = 0,
                     stream: int = 0) -> None:
    """A step of AdamW on the tensors of `update`, in place; step: which one, from 1 on.  scale, rate: one float32 each that gradients and lr are multiplied by."""
    status = _usual("adamw_step", update, step, lr, beta1, beta2, eps, scale, rate, seed, stream)
    if status == 0:
        return
    if status is not None:
        _check(status, "blink_adamw_step")
    if not 0 <= seed < 1 << 32:
        raise ValueError("seed has 32 bits")
    status = (binding._lib or binding.lib()).blink_adamw_step(
        _handle(update, Update), _whole(step, "step", _INT32, (1,)), lr, beta1, beta2, eps, None if scale is None else _whole(scale, "scale", _FP32, (1,)),
        None if rate is None else _whole(rate, "rate", _FP32, (1,)), seed, stream)
    if status:
        _check(status, "blink_adamw_step")
