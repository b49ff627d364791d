"""What the lists of addresses and counts may hold, one entry per worker.  No GPU call is made."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from test_layers_host import A, refused
from test_step_calls import BACKWARD, DIST, FORWARD, MORE, NGRAD, NORM, REC

CALLS = {  # with every list of addresses
    "embedding_lookup": dict(table=[A, A], vocab=4, width=16, ids=[2 * A, 3 * A], tokens=[3, 3], out=[4 * A, 5 * A]),
    "embedding_gradient": dict(tensor=0, width=16, ids=[2 * A, 3 * A], tokens=[3, 3], dy=[4 * A, 5 * A], ws=6 * A, ws_bytes=1 << 20),
    "checkpoint_store": dict(tokens=[3, 3], features=16, x=[A, 2 * A], checkpoint=[3 * A, 4 * A]),
    "checkpoint_load": dict(tokens=[3, 3], features=16, checkpoint=[A, 2 * A], x=[3 * A, 4 * A]),
    "weight_gradient": dict(weight=0, bias=1, checkpoint=[A, 2 * A], tokens=[3, 3], features=8, dy=[3 * A, 4 * A], ws=5 * A, ws_bytes=1 << 20),
    "residual_norm": {**NORM, **MORE}, "residual_norm_gradient": {**NGRAD, "dsum": [11 * A, 12 * A]},
    "recurrence": {**REC, **FORWARD}, "recurrence_gradient": {**REC, **BACKWARD}, "distillation": DIST}
COUNTS = ("tokens", "sequences")
LISTS = [(call, name) for call, args in CALLS.items() for name, v in args.items() if isinstance(v, list) and name not in COUNTS]


@pytest.fixture
def plan():
    p = cm.Plan(2, [8 * 16, 16, 24, 1 << 20])
    yield p
    p.close()


@pytest.mark.parametrize("call,name", LISTS)
@pytest.mark.parametrize("wrong", [torch.tensor([A]), torch.tensor(A), np.array([A]), float(A), "0"], ids=["tensor", "scalar", "array", "float", "text"])
def test_what_holds_an_address_is_none(plan, call, name, wrong):
    """A tensor instead of its data_ptr(), even one whose only element could be taken for an address."""
    args = CALLS[call]
    for entry in range(2):
        values = list(args[name])
        values[entry] = wrong
        with pytest.raises(TypeError):
            getattr(plan, call)(**{**args, name: values})


def test_addresses_of_other_kinds(plan):
    """numpy's whole numbers, and ctypes' pointers; tuples and arrays for lists."""
    args = {**NORM, "y": NORM["x"]}                                 # refused for the overlap, and so taken for what they are
    for x in (tuple(NORM["x"]), np.array(NORM["x"]), np.array(NORM["x"], dtype=np.uint64), [C.c_void_p(v) for v in NORM["x"]],
              [np.int64(v) for v in NORM["x"]]):
        with pytest.raises(cm.CaramelError, match="overlap"):
            plan.residual_norm(**{**args, "x": x})
    refused(cm.binding.EINVAL, plan.residual_norm, **{**NORM, "x": [None, A]})
    refused(cm.binding.EINVAL, plan.residual_norm, **{**NORM, "tokens": [-1, 3]})
    with pytest.raises(ValueError):
        plan.residual_norm(**{**NORM, "x": [A]})


LAYER_CALLS = [name for name in cm.binding.EXPORTS
               if any(word in name for word in ("embedding", "checkpoint", "weight_gradient", "residual_norm", "recurrence", "distillation"))]


@pytest.mark.parametrize("name", LAYER_CALLS)
def test_arrays_of_another_type_are_refused(name):
    """By the functions of the library as it is loaded: a list of 32-bit counts would be read past its end."""
    call = getattr(cm.lib(), name)
    numbers, pointers = C.POINTER(C.c_uint64), C.POINTER(C.c_void_p)
    fit = {numbers: (C.c_uint64 * 2)(), pointers: (C.c_void_p * 2)(), C.c_void_p: None, C.c_float: 1.0, C.c_uint64: 1, C.c_uint32: 1, C.c_int: 1}
    lists = [i for i, kind in enumerate(call.argtypes) if kind in (numbers, pointers)]
    assert lists
    for i in lists:
        other = (C.c_void_p * 2)() if call.argtypes[i] == numbers else (C.c_uint64 * 2)()
        for wrong in ((C.c_uint32 * 2)(), (C.c_float * 2)(), other, bytes(16), A):
            with pytest.raises(C.ArgumentError):
                call(*[wrong if k == i else fit[kind] for k, kind in enumerate(call.argtypes)])
