"""What the optimiser's list, its norm and its step refuse, at the C boundary (addresses that nothing reads) and on tensors."""
import ctypes as C

import numpy as np
import pytest

import paper_1910_04940_amd as bl
from paper_1910_04940_amd import binding

torch = pytest.importorskip("torch")

P = 1 << 20
GOOD = dict(grad=P, weights=2 * P, master=0, moment1=3 * P, moment2=4 * P, scale1=0, scale2=0, elements=1000, weight_type=1, grad_type=1, moment_type=1, rate=1.0, decay=0.0)
EIGHT = dict(moment_type=5, scale1=5 * P, scale2=6 * P)


def make(n=1, table=True, **change):
    row = np.zeros(2, binding.UPDATE_TENSOR_DTYPE)
    for name, value in {**GOOD, **change}.items():
        row[name] = value
    out = C.c_void_p(1)
    status = binding.lib().blink_make_update(row.ctypes.data if table else None, n, C.byref(out))
    assert status != bl.BLINK_OK and out.value is None
    return status


@pytest.mark.parametrize("change", [
    dict(n=0), dict(n=-1), dict(n=(1 << 20) + 1), dict(table=False), dict(grad=0), dict(grad=P + 2), dict(grad_type=0), dict(grad_type=4), dict(grad_type=5),
    dict(weight_type=0), dict(weight_type=5), dict(weights=2 * P + 2), dict(weights=2 * P + 1, weight_type=2), dict(moment1=0), dict(moment2=0), dict(moment1=3 * P + 2),
    dict(moment_type=2), dict(moment_type=0), dict(master=7 * P), dict(master=7 * P + 2, weight_type=2), dict(scale1=5 * P), dict(scale2=5 * P), dict(moment_type=5),
    {**EIGHT, "scale1": 0}, {**EIGHT, "scale2": 6 * P + 2}, dict(weights=0), dict(weights=0, moment1=0), dict(weights=0, moment1=0, moment2=0, master=7 * P),
    dict(weights=0, moment1=0, moment2=0, scale1=5 * P), dict(elements=(1 << 40) + 1), dict(rate=float("nan")), dict(decay=float("inf")), dict(n=2, elements=1 << 40, rate=float("inf"))],
    ids=str)
def test_lists_that_are_refused(change):
    assert make(**change) == bl.BLINK_EINVAL


def _two(**change):
    """Two tensors of 1000 elements, 8000 bytes from one list to the next, of which `change` moves some: name -> (of which tensor, address)."""
    row = np.zeros(2, binding.UPDATE_TENSOR_DTYPE)
    for i in range(2):
        for name, value in {**GOOD, "grad": P, "weights": P + 8000, "moment1": P + 16000, "moment2": P + 24000}.items():
            row[name][i] = value + 4000 * i if value >= P else value
    for name, (i, value) in change.items():
        row[name][i] = value
    return row


@pytest.mark.parametrize("change", [
    dict(weights=(1, P + 8000)), dict(weights=(1, P + 8004)), dict(weights=(0, P + 12000)), dict(moment1=(1, P + 16000)), dict(moment2=(1, P + 24000 + 3996)),
    dict(moment1=(0, P + 24000)), dict(grad=(1, P + 8000)), dict(grad=(0, P + 8000 - 4)), dict(grad=(1, P + 28000 + 3996)), dict(weights=(0, P))], ids=str)
def test_lists_that_write_a_place_twice(change):
    """The same weights under two names, and what overlaps by an element: two workgroups would step it at once."""
    row, out = _two(**change), C.c_void_p(1)
    assert binding.lib().blink_make_update(row.ctypes.data, 2, C.byref(out)) == bl.BLINK_EINVAL and out.value is None


@pytest.mark.gpu
def test_lists_that_touch():
    """Neighbours in one buffer, and one gradient for two tensors, are no overlap."""
    buffer = torch.zeros(5, 2, 1000, device="cuda")
    grad, weights, moment1, moment2, _ = (list(x) for x in buffer)
    shared = [grad[0], grad[0]]
    for grads in (grad, shared):
        bl.blink_make_update(grads, weights, moment1, moment2)
    for bad in (dict(weights=[weights[0]] * 2), dict(moments1=[moment1[1]] * 2), dict(moments2=[moment1[0], moment2[1]]), dict(grads=[grad[0], weights[0]]),
                dict(weights=[buffer.view(-1)[2001:3001], buffer.view(-1)[3000:4000]])):
        with pytest.raises(bl.BlinkError) as e:
            bl.blink_make_update(**{**dict(grads=grad, weights=weights, moments1=moment1, moments2=moment2), **bad})
        assert e.value.status == bl.BLINK_EINVAL


def test_no_list():
    L = binding.lib()
    assert L.blink_make_update(None, 1, None) == bl.BLINK_EINVAL
    assert L.blink_gradient_norm(None, 1.0, 1.0, P, None, P, 1 << 20, None) == bl.BLINK_EINVAL
    assert L.blink_adamw_step(None, P, 0.1, 0.9, 0.99, 1e-8, None, None, 0, None) == bl.BLINK_EINVAL
    assert L.blink_gradient_norm_workspace(None) == 0
    L.blink_update_free(None)


def test_layout_of_the_c_struct(tmp_path):
    """The binding's mirror of blink_update_tensor_t against the header."""
    import os
    import subprocess
    names = binding.UPDATE_TENSOR_DTYPE.names
    source = tmp_path / "layout.c"
    source.write_text('#include <stdio.h>\n#include "blink.h"\nint main(void) {\n' +
                      "".join(f'    printf("%zu ", offsetof(blink_update_tensor_t, {n}));\n' for n in names) +
                      '    printf("%zu", sizeof(blink_update_tensor_t));\n    return 0;\n}\n')
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", include, str(source), "-o", str(tmp_path / "layout")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [binding.UPDATE_TENSOR_DTYPE.fields[n][1] for n in names] + [binding.UPDATE_TENSOR_DTYPE.itemsize]


def test_tensors_on_the_host():
    for call in (lambda: bl.blink_make_update([torch.zeros(4)]), lambda: bl.blink_make_update([torch.zeros(4)], [None, None]), lambda: bl.blink_make_update([None]),
                 lambda: bl.blink_make_update([])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_tensors_that_do_not_fit():
    t = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda")   # noqa: E731
    eight = torch.float8_e4m3fn
    for bad in (dict(weights=[t(5)]), dict(weights=[t(6)]), dict(weights=[t(6)], moments1=[t(6)]), dict(weights=[t(6)], moments1=[t(6)], moments2=[t(5)]),
                dict(moments1=[t(6)]), dict(weights=[t(12)[::2]], moments1=[t(6)], moments2=[t(6)]),
                dict(weights=[t(6)], moments1=[t(6, eight)], moments2=[t(6, eight)]), dict(weights=[t(6)], moments1=[t(6, eight)], moments2=[t(6)]),
                dict(weights=[t(6)], moments1=[t(6, eight)], moments2=[t(6, eight)], scales1=[t(2)], scales2=[t(1)]),
                dict(weights=[t(6)], moments1=[t(6)], moments2=[t(6)], scales1=[t(1)], scales2=[t(1)]),
                dict(weights=[t(6, torch.float64)], moments1=[t(6)], moments2=[t(6)]), dict(masters=[t(6)])):
        with pytest.raises(ValueError):
            bl.blink_make_update([t(6)], **bad)
    with pytest.raises(bl.BlinkError):      # weights in 32 bits have no copy
        bl.blink_make_update([t(6)], [t(6)], [t(6)], [t(6)], masters=[t(6)])
    update = bl.blink_make_update([t(6)], [t(6)], [t(6)], [t(6)])
    norm, step, work = t(2), t(1, torch.int32), t(bl.blink_gradient_norm_workspace(update), torch.uint8)
    stream = torch.cuda.current_stream().cuda_stream
    for bad in (dict(max_norm=0.0), dict(max_norm=float("nan")), dict(max_norm=-1.0), dict(factor=float("inf")), dict(workspace=None), dict(workspace=work[:-1])):
        with pytest.raises(bl.BlinkError) as e:
            bl.blink_gradient_norm(**{**dict(update=update, norm=norm, workspace=work, stream=stream), **bad})
        assert e.value.status == bl.BLINK_EINVAL
    for bad in (dict(norm=t(3)), dict(norm=t(2, torch.float64)), dict(step=t(1)), dict(step=t(2, torch.int32))):
        with pytest.raises(ValueError):
            bl.blink_gradient_norm(**{**dict(update=update, norm=norm, workspace=work, stream=stream), **bad})
    for bad in (dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=1.0), dict(eps=0.0), dict(eps=float("inf"))):
        with pytest.raises(bl.BlinkError) as e:
            bl.blink_adamw_step(**{**dict(update=update, step=step, lr=0.1, stream=stream), **bad})
        assert e.value.status == bl.BLINK_EINVAL
    for bad in (dict(step=t(1)), dict(scale=t(2)), dict(rate=t(1, torch.int32)), dict(seed=-1), dict(seed=1 << 32)):
        with pytest.raises(ValueError):
            bl.blink_adamw_step(**{**dict(update=update, step=step, lr=0.1, stream=stream), **bad})
