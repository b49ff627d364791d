"""The calls of a training step around the gradients: sizes and refusals.  No GPU call is made."""
import ctypes as C
import math
import os
import random
import shutil
import subprocess

import pytest

import paper_2004_14020_amd as cm

from test_layers_host import A, T, refused

E = cm.binding.EINVAL
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_calls_allocate_nothing(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    exe, libdir = str(tmp_path / "step_alloc_check"), os.path.dirname(cm.binding.LIB_PATH)
    subprocess.run(["gcc", "-std=gnu99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "host", "step_alloc_check.c"), "-L", libdir, "-l:libcaramel.so",
                    "-Wl,-rpath," + libdir, "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "step_alloc_check ok" in res.stdout, (res.returncode, res.stdout + res.stderr)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_overlap_of_rows_of_different_pitch(tmp_path):
    exe = str(tmp_path / "pitch_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2004_14020_amd", "csrc"), os.path.join(ROOT, "tests", "host", "pitch_check.cpp"), "-o", exe],
                   check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "pitch_check ok" in res.stdout, res.stdout[-2000:] + res.stderr[-2000:]


@pytest.fixture
def plan():
    p = cm.Plan(2, [8 * 16, 16, 24, 1 << 20])
    yield p
    p.close()


NORM = dict(gain=[A, A], width=16, tokens=[3, 3], x=[2 * A, 3 * A], y=[4 * A, 5 * A], rstd=[6 * A, 7 * A])
MORE = dict(residual=[8 * A, 9 * A], sum=[10 * A, 11 * A], checkpoint=[12 * A, 13 * A])


@pytest.mark.parametrize("change", [
    dict(width=0), dict(width=32769, pitch=32769), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan), dict(dtype=2),
    dict(tokens=[T, 1]), dict(pitch=15), dict(pitch=(1 << 23) + 1), dict(tokens=[1 << 25, 1], pitch=1 << 23),
    dict(gain=[A, None]), dict(gain=[A, A + 2]), dict(x=[None, A]), dict(x=[2 * A, 3 * A + 1]), dict(y=[4 * A, None]),
    dict(y=[4 * A + 2, 5 * A]), dict(rstd=[None, 7 * A]), dict(rstd=[6 * A + 2, 7 * A]), dict(residual=None), dict(sum=None),
    dict(residual=[8 * A, None]), dict(sum=[None, 11 * A]), dict(checkpoint=[12 * A, None]), dict(checkpoint=[12 * A + 8, 13 * A]),
    # what is written overlaps: the other worker's, an input, the gain
    dict(y=[4 * A, 4 * A]), dict(y=[2 * A, 5 * A]), dict(y=[A + 32, 5 * A]), dict(sum=[8 * A, 11 * A]), dict(sum=[2 * A, 11 * A]),
    dict(sum=[4 * A + 64, 11 * A]), dict(rstd=[2 * A, 7 * A]), dict(rstd=[6 * A, 6 * A + 8]), dict(checkpoint=[12 * A, 12 * A]),
    dict(checkpoint=[4 * A, 13 * A]),
], ids=str)
def test_norm_refusals(plan, change):
    refused(E, plan.residual_norm, **{**NORM, **MORE, **change})


NGRAD = dict(gain_tensor=1, gain=[A, A], tokens=[3, 3], x=[2 * A, 3 * A], rstd=[6 * A, 7 * A], dy=[8 * A, 9 * A], dx=[4 * A, 5 * A],
             ws=10 * A, ws_bytes=1 << 16)


@pytest.mark.parametrize("change", [
    dict(gain_tensor=4, pitch=16), dict(gain_tensor=3), dict(dtype=2), dict(tokens=[1, T]), dict(pitch=15), dict(pitch=(1 << 23) + 1),
    dict(gain=[None, A]), dict(gain=[A, A + 2]), dict(x=[2 * A, None]), dict(rstd=[6 * A, None]), dict(rstd=[6 * A, 7 * A + 2]),
    dict(dy=[None, 9 * A]), dict(dsum=[None, 9 * A]), dict(dsum=[A, A + 2]), dict(dx=[4 * A, None]), dict(ws=None), dict(ws=10 * A + 8),
    dict(ws_bytes=16), dict(tokens=[1 << 25, 1], pitch=1 << 23),
], ids=str)
def test_norm_gradient_refusals(plan, change):
    refused(E, plan.residual_norm_gradient, **{**NGRAD, **change})


def test_norm_gradient_needs_a_bound_plan(plan):
    refused(cm.binding.ESTATE, plan.residual_norm_gradient, **NGRAD)
    with pytest.raises(ValueError):
        plan.residual_norm_gradient(**{**NGRAD, "gain_tensor": -1})
    for bad in ((4, [1, 1]), (3, [1, 1]), (1, [T, 1])):
        refused(E, plan.residual_norm_workspace, *bad)


def test_norm_null_arguments(plan):
    L, two, n, b = cm.lib(), (C.c_void_p * 2)(A, 2 * A), (C.c_uint64 * 2)(0, 0), C.c_uint64()
    forward = [plan._h, two, 16, 1e-5, n, two, None, 0, 16, None, two, two, None, None]
    backward = [plan._h, 1, two, n, two, two, two, None, 0, 16, two, 0, A, 1 << 20, None]
    for call, args, needed in ((L.caramel_residual_norm, forward, (0, 1, 4, 5, 10, 11)),
                               (L.caramel_residual_norm_gradient, backward, (0, 2, 3, 4, 5, 6, 10)),
                               (L.caramel_residual_norm_workspace, [plan._h, 1, n, C.byref(b)], (0, 2, 3))):
        for i in needed:
            assert call(*[None if k == i else v for k, v in enumerate(args)]) == E, (call, i)


def test_norm_workspaces_serve_fewer_tokens():
    rng = random.Random(4)
    for _ in range(200):
        plan = cm.Plan(rng.choice([1, 2, 3, 8, 16, 17, 64]), [rng.randint(1, 4096)])
        tokens = sorted(int(2 ** rng.uniform(0, 25)) for _ in range(30))
        sizes = [plan.residual_norm_workspace(0, [n] * plan.cfg.world) for n in tokens]
        assert sizes == sorted(sizes)
        plan.close()


REC = dict(channels=16, tokens=[3, 3], sequences=[1, 2], starts=[A, A + 64], gate=[2 * A, 3 * A], input=[2 * A + 64, 3 * A + 64],
           pitch=32, ws=None, ws_bytes=0, before=[20 * A, 21 * A])
FORWARD = dict(states=[4 * A, 5 * A], after=[6 * A, 7 * A])
BACKWARD = dict(states=[4 * A, 5 * A], dstates=[6 * A, 7 * A], dgate=[8 * A, 9 * A], dinput=[8 * A + 64, 9 * A + 64],
                dafter=[10 * A, 11 * A], dbefore=[12 * A, 13 * A])
BOTH = [dict(channels=0), dict(channels=(1 << 20) + 1, pitch=1 << 22), dict(id_bytes=2), dict(dtype=2), dict(tokens=[T, 1]),
        dict(sequences=[1, T]), dict(tokens=[3, 0]), dict(pitch=15), dict(pitch=(1 << 23) + 1), dict(states_pitch=15), dict(states_pitch=(1 << 23) + 1),
        dict(tokens=[1 << 25, 1], pitch=1 << 23), dict(starts=[A, None]), dict(starts=[A, A + 4]), dict(gate=[None, A]),
        dict(gate=[2 * A + 2, 3 * A]), dict(input=[None, 3 * A]), dict(before=[20 * A, None]), dict(before=[20 * A + 2, 21 * A]),
        dict(states=[4 * A, None]), dict(states=[4 * A + 2, 5 * A]), dict(tokens=[1000, 3]),
        dict(tokens=[1000, 3], ws=30 * A + 8, ws_bytes=1 << 20), dict(tokens=[1000, 3], ws=30 * A, ws_bytes=16)]


@pytest.mark.parametrize("change", BOTH + [
    dict(after=[None, 7 * A]), dict(after=[6 * A, 6 * A]), dict(after=[20 * A, 7 * A]), dict(states=[2 * A, 5 * A]), dict(states=[A, 5 * A]),
    dict(states=[4 * A, 4 * A + 128]), dict(states=[2 * A + 192, 5 * A]),                       # between rows of another pitch
], ids=str)
def test_recurrence_refusals(plan, change):
    refused(E, plan.recurrence, **{**REC, **FORWARD, **change})


@pytest.mark.parametrize("change", BOTH + [
    dict(dstates=[6 * A, None]), dict(dstates=[6 * A + 2, 7 * A]), dict(dafter=[None, 11 * A]), dict(dgate=[None, 9 * A]),
    dict(dinput=[8 * A + 64, None]), dict(dbefore=[12 * A, None]), dict(dgate=[2 * A, 9 * A]), dict(dinput=[8 * A, 9 * A + 64]),
    dict(dinput=[8 * A + 60, 9 * A + 64]), dict(dgate=[6 * A, 9 * A]), dict(dbefore=[10 * A, 13 * A]), dict(dbefore=[20 * A, 13 * A]),
], ids=str)
def test_recurrence_gradient_refusals(plan, change):
    refused(E, plan.recurrence_gradient, **{**REC, **BACKWARD, **change})


def test_recurrence_null_arguments(plan):
    L, two, n, b = cm.lib(), (C.c_void_p * 2)(A, 2 * A), (C.c_uint64 * 2)(0, 0), C.c_uint64()
    forward = [plan._h, 16, n, n, two, 8, two, two, 0, 16, None, two, 16, None, None, 0, None]
    backward = [plan._h, 16, n, n, two, 8, two, two, 0, 16, None, two, two, 16, None, two, two, None, None, 0, None]
    for call, args, needed in ((L.caramel_recurrence, forward, (0, 2, 3, 4, 6, 7, 11)),
                               (L.caramel_recurrence_gradient, backward, (0, 2, 3, 4, 6, 7, 11, 12, 15, 16)),
                               (L.caramel_recurrence_workspace, [plan._h, 16, n, C.byref(b)], (0, 2, 3))):
        for i in needed:
            assert call(*[None if k == i else v for k, v in enumerate(args)]) == E, (call, i)
    for bad in ((0, [1, 1]), ((1 << 20) + 1, [1, 1]), (16, [1, T])):
        refused(E, plan.recurrence_workspace, *bad)


def test_recurrence_workspaces_serve_fewer_tokens():
    rng = random.Random(4)
    for _ in range(200):
        plan, channels = cm.Plan(rng.choice([1, 2, 3, 8, 16, 17, 64]), [1]), int(2 ** rng.uniform(0, 20))
        tokens = sorted(int(2 ** rng.uniform(0, 25)) for _ in range(30))
        sizes = [plan.recurrence_workspace(channels, [n] * plan.cfg.world) for n in tokens]
        assert sizes == sorted(sizes)
        each = [int(2 ** rng.uniform(0, 16)) for _ in range(plan.cfg.world)]
        for _ in range(20):
            fewer = [rng.randint(0, n) for n in each]
            assert plan.recurrence_workspace(channels, fewer) <= plan.recurrence_workspace(channels, each)
            each = fewer if rng.random() < 0.3 else each
        plan.close()


DIST = dict(vocab=16, tokens=[3, 3], logits=[A, 2 * A], teacher_ids=[3 * A, 4 * A], teacher_logits=[5 * A, 6 * A], top=2,
            loss=[7 * A, 8 * A], ws=None, ws_bytes=0, labels=[9 * A, 10 * A], dlogits=[11 * A, 12 * A], hard=0.5)


@pytest.mark.parametrize("change", [
    dict(vocab=0), dict(vocab=(1 << 20) + 1, pitch=1 << 22, dlogits_pitch=1 << 22), dict(top=0), dict(top=257), dict(id_bytes=1),
    dict(dtype=2), dict(teacher_dtype=2), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=2000.0),
    dict(temperature=math.nan), dict(temperature=math.inf), dict(soft=-1.0), dict(soft=math.nan), dict(hard=-0.5), dict(hard=math.inf),
    dict(soft=0.0, hard=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(labels=None), dict(tokens=[T, 1]), dict(pitch=15),
    dict(pitch=(1 << 23) + 1), dict(dlogits_pitch=15), dict(tokens=[1 << 25, 1], pitch=1 << 23), dict(logits=[None, A]),
    dict(logits=[A + 2, 2 * A]), dict(teacher_ids=[3 * A, None]), dict(teacher_ids=[3 * A + 4, 4 * A]), dict(teacher_logits=[None, A]),
    dict(teacher_logits=[5 * A + 2, 6 * A]), dict(labels=[9 * A, None]), dict(labels=[9 * A + 4, 10 * A]), dict(loss=[None, 8 * A]),
    dict(loss=[7 * A + 2, 8 * A]), dict(dlogits=[11 * A, None]), dict(dlogits=[11 * A + 1, 12 * A]), dict(vocab=61448, pitch=61448),
    dict(vocab=61448, ws=20 * A + 8, ws_bytes=1 << 20), dict(vocab=61448, ws=20 * A, ws_bytes=64),
    # what is written overlaps: the other worker's, inputs; the logits with another pitch or place than theirs
    dict(dlogits=[11 * A, 11 * A]), dict(dlogits=[3 * A, 12 * A]), dict(loss=[7 * A, 7 * A]), dict(loss=[A, 8 * A]),
    dict(dlogits=[2 * A, A]), dict(dlogits=[A, 2 * A], dlogits_pitch=17), dict(dlogits=[A + 64, 2 * A]),
], ids=str)
def test_distillation_refusals(plan, change):
    refused(E, plan.distillation, **{**DIST, **change})


def test_distillation_null_arguments(plan):
    L, two, n, b = cm.lib(), (C.c_void_p * 2)(A, 2 * A), (C.c_uint64 * 2)(0, 0), C.c_uint64()
    args = [plan._h, 16, n, two, 0, 16, two, None, 8, two, 0, 2, 1.0, 1.0, 0.0, 1.0, two, None, 16, None, 0, None]
    for i in (0, 2, 3, 6, 9, 16):
        assert L.caramel_distillation(*[None if k == i else v for k, v in enumerate(args)]) == E, i
    sizes = [plan._h, 16, 2, n, C.byref(b)]
    for i in (0, 3, 4):
        assert L.caramel_distillation_workspace(*[None if k == i else v for k, v in enumerate(sizes)]) == E, i
    for bad in ((0, 1, [1, 1]), ((1 << 20) + 1, 1, [1, 1]), (16, 0, [1, 1]), (16, 257, [1, 1]), (16, 1, [1, T])):
        refused(E, plan.distillation_workspace, *bad)


def test_distillation_workspaces_serve_fewer_tokens():
    rng = random.Random(4)
    for _ in range(200):
        plan = cm.Plan(rng.choice([1, 2, 3, 8, 16, 17, 64]), [1])
        vocab, top = int(2 ** rng.uniform(0, 20)), rng.randint(1, 256)
        tokens = sorted(int(2 ** rng.uniform(0, 25)) for _ in range(30))
        sizes = [plan.distillation_workspace(vocab, top, [n] * plan.cfg.world) for n in tokens]
        assert sizes == sorted(sizes)
        plan.close()
