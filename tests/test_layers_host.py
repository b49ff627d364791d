"""The operators that fill gradient tensors: sizes and refusals.  No GPU call is made."""
import ctypes as C

import numpy as np
import pytest

import paper_2004_14020_amd as cm

from layer_util import decode, encode, image

A = 1 << 20          # an address that is aligned to everything
T = (1 << 25) + 1


def refused(status, call, *args, **kw):
    with pytest.raises(cm.CaramelError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value
    return str(e.value)


@pytest.fixture
def plan():
    p = cm.Plan(2, [8 * 16, 16, 24])
    yield p
    p.close()


def test_plain_encoding_reads_back_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((70, 9)) * 10.0 ** rng.integers(-30, 30, 9)).astype(np.float32)
    x[3, 2] = 0.0
    codes, scales = encode(x)
    y = decode(codes, scales, 70)
    step = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, 0)[:70]
    assert (np.abs(y - x) <= step / 2).all()
    # the scale is as small as it can be
    assert (np.abs(codes.astype(int)).max(2) >= 63).all()
    assert image(codes, scales).size == cm.checkpoint_bytes(70, 9)


@pytest.mark.parametrize("tokens,features,want", [(0, 5, 0), (1, 1, 48), (32, 4, 144), (33, 4, 272), (1, 16, 528)])
def test_checkpoint_bytes(tokens, features, want):
    assert cm.checkpoint_bytes(tokens, features) == want


def test_checkpoint_bytes_refusals():
    for t, f in ((1, 0), (1, (1 << 20) + 1), (T, 1)):
        refused(cm.binding.EINVAL, cm.checkpoint_bytes, t, f)
    assert cm.lib().caramel_checkpoint_bytes(1, 1, None) == cm.binding.EINVAL


def test_workspace_refusals(plan):
    E = cm.binding.EINVAL
    for bad in ((3, 16, [1, 1]), (0, 0, [1, 1]), (0, 7, [1, 1]), (0, 16, [T, 1])):
        refused(E, plan.embedding_workspace, *bad)
        refused(E, plan.weight_gradient_workspace, *bad)
    with pytest.raises(ValueError):
        plan.embedding_workspace(0, 16, [1])
    assert plan.embedding_workspace(0, 16, [0, 0]) > 0          # where each row's tokens begin
    assert plan.weight_gradient_workspace(0, 8, [1, 1]) == 0
    n = C.c_uint64()
    one = (C.c_uint64 * 2)(1, 1)
    L = cm.lib()
    assert L.caramel_embedding_workspace(None, 0, 16, one, C.byref(n)) == E
    assert L.caramel_embedding_workspace(plan._h, 0, 16, None, C.byref(n)) == E
    assert L.caramel_embedding_workspace(plan._h, 0, 16, one, None) == E
    assert L.caramel_weight_gradient_workspace(None, 0, 8, one, C.byref(n)) == E
    assert L.caramel_weight_gradient_workspace(plan._h, 0, 8, None, C.byref(n)) == E


def test_workspace_of_split_tokens_grows_with_the_parts(plan):
    big = cm.Plan(1, [1024 * 1024])
    assert big.weight_gradient_workspace(0, 1024, [16]) == 0
    assert big.weight_gradient_workspace(0, 1024, [16384]) >= 2 * 4 * 1024 * 1024
    big.close()


LOOKUP = dict(table=[A, A], vocab=8, width=16, ids=[2 * A, 2 * A], tokens=[3, 3], out=[3 * A, 4 * A])


@pytest.mark.parametrize("change", [
    dict(vocab=0), dict(vocab=(1 << 31) - 1), dict(width=0), dict(width=(1 << 20) + 1), dict(id_bytes=2), dict(tokens=[T, 1]),
    dict(out_pitch=15), dict(out_pitch=(1 << 23) + 1), dict(table=[A, None]), dict(table=[A, A + 2]), dict(ids=[None, A]),
    dict(ids=[2 * A, 2 * A + 4]), dict(out=[3 * A, None]), dict(out=[3 * A, 3 * A + 2]), dict(out=[3 * A, 3 * A]),
    dict(out=[3 * A, 3 * A + 64]), dict(out=[A + 64, 4 * A]), dict(out=[2 * A, 4 * A]),
    dict(tokens=[1 << 25, 1], out_pitch=1 << 23),
], ids=str)
def test_lookup_refusals(plan, change):
    refused(cm.binding.EINVAL, plan.embedding_lookup, **{**LOOKUP, **change})


def test_lookup_null_arguments(plan):
    two = (C.c_void_p * 2)(A, A)
    out = (C.c_void_p * 2)(3 * A, 4 * A)
    n = (C.c_uint64 * 2)(1, 1)
    L, E = cm.lib(), cm.binding.EINVAL
    assert L.caramel_embedding_lookup(None, two, 8, 16, 1.0, two, 8, n, out, 16, None) == E
    assert L.caramel_embedding_lookup(plan._h, None, 8, 16, 1.0, two, 8, n, out, 16, None) == E
    assert L.caramel_embedding_lookup(plan._h, two, 8, 16, 1.0, None, 8, n, out, 16, None) == E
    assert L.caramel_embedding_lookup(plan._h, two, 8, 16, 1.0, two, 8, None, out, 16, None) == E
    assert L.caramel_embedding_lookup(plan._h, two, 8, 16, 1.0, two, 8, n, None, 16, None) == E
    with pytest.raises(ValueError):
        plan.embedding_lookup([A], 8, 16, [A, A], [1, 1], [A, A])


GRAD = dict(tensor=0, width=16, ids=[A, 2 * A], tokens=[3, 3], dy=[3 * A, 4 * A], ws=5 * A, ws_bytes=1 << 16)


@pytest.mark.parametrize("change", [
    dict(tensor=3), dict(width=0), dict(width=7), dict(id_bytes=1), dict(dy_dtype=2), dict(tokens=[1, T]), dict(dy_pitch=15),
    dict(dy_pitch=(1 << 23) + 1), dict(ids=[A, None]), dict(ids=[A, A + 4]), dict(dy=[None, A]), dict(dy=[A, A + 2]),
    dict(ws=None), dict(ws=5 * A + 8), dict(ws_bytes=16), dict(tokens=[1 << 25, 1], dy_pitch=1 << 23),
], ids=str)
def test_embedding_gradient_refusals(plan, change):
    refused(cm.binding.EINVAL, plan.embedding_gradient, **{**GRAD, **change})


STORE = dict(x=[A, 2 * A], tokens=[33, 5], features=7, checkpoint=[3 * A, 4 * A])


@pytest.mark.parametrize("change", [
    dict(features=0), dict(features=(1 << 20) + 1), dict(dtype=2), dict(tokens=[T, 1]), dict(pitch=6), dict(pitch=(1 << 23) + 1),
    dict(x=[None, A]), dict(x=[A, 2 * A + 2]), dict(checkpoint=[3 * A, None]), dict(checkpoint=[3 * A, 4 * A + 8]),
    dict(checkpoint=[3 * A, 3 * A], x=[A, A]), dict(checkpoint=[A, 4 * A]), dict(tokens=[1 << 25, 1], pitch=1 << 23),
], ids=str)
@pytest.mark.parametrize("load", [False, True], ids=["store", "load"])
def test_checkpoint_refusals(plan, change, load):
    call = {**STORE, **change}
    refused(cm.binding.EINVAL, plan.checkpoint_load if load else plan.checkpoint_store, **call)


WGRAD = dict(weight=0, bias=1, checkpoint=[A, 2 * A], tokens=[3, 3], features=8, dy=[3 * A, 4 * A], ws=None, ws_bytes=0)


@pytest.mark.parametrize("change", [
    dict(bias=2), dict(bias=0), dict(features=7), dict(dy_dtype=2), dict(tokens=[1, T]),
    dict(dy_pitch=15), dict(dy_pitch=(1 << 23) + 1), dict(checkpoint=[A, None]), dict(checkpoint=[A, 2 * A + 8]),
    dict(dy=[None, A]), dict(dy=[A, A + 2]), dict(tokens=[1 << 25, 1], dy_pitch=1 << 23), dict(tokens=[4096, 1]),
], ids=str)
def test_weight_gradient_refusals(plan, change):
    refused(cm.binding.EINVAL, plan.weight_gradient, **{**WGRAD, **change})


def test_weight_gradient_refuses_tensors_that_are_not_there(plan):
    for change in (dict(weight=3), dict(weight=-1), dict(bias=3), dict(bias=-1)):
        with pytest.raises(ValueError):
            plan.weight_gradient(**{**WGRAD, **change})
    L, E = cm.lib(), cm.binding.EINVAL
    two, n = (C.c_void_p * 2)(A, A), (C.c_uint64 * 2)(1, 1)
    assert L.caramel_weight_gradient(plan._h, 3, cm.NO_TENSOR, 8, two, n, two, 0, 16, 0, None, 0, None) == E
    assert L.caramel_weight_gradient(plan._h, 0, 3, 8, two, n, two, 0, 16, 0, None, 0, None) == E
    refused(E, plan.embedding_gradient, **{**GRAD, "tensor": -1})


def test_gradients_need_a_bound_plan(plan):
    refused(cm.binding.ESTATE, plan.embedding_gradient, **GRAD)
    refused(cm.binding.ESTATE, plan.weight_gradient, **WGRAD)
    L, E = cm.lib(), cm.binding.EINVAL
    two, n = (C.c_void_p * 2)(A, A), (C.c_uint64 * 2)(1, 1)
    assert L.caramel_embedding_gradient(None, 0, 16, 1.0, two, 8, n, two, 0, 16, 0, A, 1 << 16, None) == E
    assert L.caramel_weight_gradient(None, 0, 1, 8, two, n, two, 0, 16, 0, None, 0, None) == E
    assert L.caramel_checkpoint_store(None, n, 7, two, 0, 7, two, None) == E
    assert L.caramel_checkpoint_load(None, n, 7, two, two, 0, 7, None) == E
