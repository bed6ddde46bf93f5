"""Handles of another kind than a call takes: refused before anything reads what they stand for."""
import math

import pytest

import paper_1910_04940_amd as bl
from paper_1910_04940_amd import binding, operators

AT = 1 << 20     # an address that nothing may read


def _owner(kind):
    """An object of that kind that holds an address, and gives nothing back to the library in the end."""
    class Held(kind):
        __slots__ = ()

        def __del__(self):
            pass
    held = Held.__new__(Held)
    held.__init__(*{"Schedule": (AT, 2, 16, bl.BLINK_OP_ALLREDUCE), "Update": (AT, []), "Trees": (AT,)}[kind.__name__])
    return held


OTHERS = {"Schedule": (operators.Update, binding.Trees), "Update": (binding.Schedule, binding.Trees), "Trees": (binding.Schedule, operators.Update)}
COLLECTIVES = [("blink_allreduce", ()), ("blink_allreduce_noalloc", ()), ("blink_broadcast", ()), ("blink_allgather", ()), ("blink_gather", ()),
               ("blink_allreduce_op", (bl.BLINK_SUM,)), ("blink_reduce", (bl.BLINK_SUM,))]


@pytest.fixture(params=[True, False], ids=["native", "ctypes"])
def way(request, monkeypatch):
    binding.lib()
    if not request.param:
        monkeypatch.setattr(binding, "_call", lambda *a: None)
        monkeypatch.setattr(operators, "_operators", {})


@pytest.mark.parametrize("other", OTHERS["Schedule"], ids=str)
@pytest.mark.parametrize("name,redop", COLLECTIVES, ids=[n for n, _ in COLLECTIVES])
def test_schedules(way, name, redop, other):
    handle = _owner(other)
    with pytest.raises(TypeError):
        getattr(bl, name)([AT, AT], 16, bl.BLINK_FP32, *redop, handle)


@pytest.mark.parametrize("other", OTHERS["Update"], ids=str)
def test_updates(way, other):
    torch = pytest.importorskip("torch")
    handle = _owner(other)
    with pytest.raises(TypeError):
        bl.blink_gradient_norm(handle, torch.empty(2), None, math.inf)
    with pytest.raises(TypeError):
        bl.blink_adamw_step(handle, torch.zeros(1, dtype=torch.int32), 0.1)
    with pytest.raises(TypeError):
        bl.blink_gradient_norm_workspace(handle)


@pytest.mark.parametrize("other", OTHERS["Trees"], ids=str)
def test_trees(other):
    with pytest.raises(TypeError):
        bl.blink_make_schedule(_owner(other), bl.BLINK_OP_ALLREDUCE, 16, 4)
    with pytest.raises(TypeError):
        bl.blink_make_schedule_servers([_owner(other)], [[0, 1]], 16, 4)


def test_handles_that_are_gone(way):
    """An owner that has given its handle back holds none."""
    schedule, update = _owner(binding.Schedule), _owner(operators.Update)
    for owner in (schedule, update):
        for name in [n for n in vars(owner) if n in ("_h", "_address", "_update")]:
            setattr(owner, name, None)
    with pytest.raises(bl.BlinkError) as e:
        bl.blink_allreduce([AT, AT], 16, bl.BLINK_FP32, schedule)
    assert e.value.status == bl.BLINK_EINVAL
    assert bl.blink_gradient_norm_workspace(update) == 0


@pytest.mark.gpu
def test_handles_of_their_kind(way):
    """A GPU call of each with the handle that it takes."""
    torch = pytest.importorskip("torch")
    import synth_inputs as si
    top = si.complete_graph(2)
    schedule = bl.blink_make_schedule(bl.blink_pack_trees(top.k, top.src, top.dst, top.cap, 0), bl.BLINK_OP_ALLREDUCE, 64, 16)
    bufs = [torch.ones(64, device="cuda") for _ in range(2)]
    stream = torch.cuda.current_stream().cuda_stream
    bl.blink_allreduce(bufs, 64, bl.BLINK_FP32, schedule, stream)
    update = bl.blink_make_update([bufs[0]])
    norm, work = torch.empty(2, device="cuda"), torch.empty(bl.blink_gradient_norm_workspace(update), dtype=torch.uint8, device="cuda")
    bl.blink_gradient_norm(update, norm, work, stream=stream)
    assert norm.tolist() == [16.0, 1.0]
