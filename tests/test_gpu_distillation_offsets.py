"""The loss of distillation does not hang on a number that all of a token's logits have in common, however large it is.

Tolerances: those of the formulas in 64 bits, taken of logits from which the largest of their token has been subtracted (the sums below are exact
in the logits' type): the weights P are fp32 numbers, and what they are off by counts times the distance of a logit to the largest one."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import HALF_STEP, TORCH, f64
from test_gpu_distillation import call, formulas
from test_gpu_layers import DTYPES, close, dtype_id

pytestmark = pytest.mark.gpu

# of every type: the unit of the logits, their size, and what they have in common (at most 24, or 8, bits in all)
UNIT = {cm.F32: 2.0 ** -4, cm.BF16: 1.0}
SIZE = {cm.F32: 3.0, cm.BF16: 2.0}
COMMON = {cm.F32: [0.0, 1000.0, -16384.0, 5.0e5, -5.0e5, 7.0], cm.BF16: [0.0, 100.0, -112.0, 64.0]}


@pytest.mark.parametrize("vocab,n,top", [(9, 12, 5), (50, 12, 8), (777, 300, 32), (9000, 12, 64), (30522, 12, 256), (70000, 12, 16), (70000, 100, 16)])
@pytest.mark.parametrize("T,soft,hard", [(1.0, 1.0, 0.0), (2.0, 0.7, 0.5), (4.0, 1.0, 0.5), (3.0, 1.0, 0.5), (1.0 / 64, 1.0, 0.25), (50.0, 3.0, 0.0)])
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_a_common_number_of_all_logits(dtype, T, soft, hard, vocab, n, top):
    print(f"case: common numbers n={n} vocab={vocab} T={T} {soft} {hard}", flush=True)
    rng = np.random.default_rng(vocab + top)
    unit = UNIT[dtype]
    z = np.round(rng.standard_normal((n, vocab)) * SIZE[dtype] / unit).clip(-15 / unit, 15 / unit) * unit
    common = np.array(COMMON[dtype])[np.arange(n) % len(COMMON[dtype])][:, None]
    shifted = torch.tensor(z + common, dtype=torch.float32).to(TORCH[dtype])
    assert np.array_equal(f64(shifted), z + common)
    ids, labels = rng.integers(-1, vocab, (n, top)), rng.integers(-1, vocab, n)
    ids[::3] = z[::3].argsort(1)[:, ::-1][:, :top] if top <= vocab else ids[::3]     # a teacher who agrees with the student, nearly
    t = rng.standard_normal((n, top)) * 3
    t[::3] = np.take_along_axis(z, np.where(ids >= 0, ids, 0), 1)[::3] + 0.25 * rng.standard_normal(t[::3].shape)
    t = torch.tensor(t, dtype=torch.float32)
    loss, g = call(cm.Plan(1, [1]), shifted, torch.tensor(ids), t, torch.tensor(labels), T, soft, hard, dtype)
    want, dg, off_loss, off = formulas(z - z.max(1, keepdims=True), ids, f64(t), labels, T, soft, hard, 1.0, vocab, T in (2.0, 4.0))
    close(f64(loss), want, off_loss, "loss")
    close(f64(g), dg, off + (HALF_STEP[cm.BF16] * (np.abs(dg) + off) if dtype == cm.BF16 else 0), "dlogits")


@pytest.mark.parametrize("vocab,n", [(50, 12), (9000, 12), (70000, 12), (70000, 100)])
@pytest.mark.parametrize("T", [1.0, 2.0, 3.0, 1.0 / 1024, 1024.0])
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_equal_logits_as_large_as_can_be(dtype, T, vocab, n):
    """All logits the lowest or the largest number, or all that the mask leaves."""
    rng = np.random.default_rng(vocab)
    low, big = torch.finfo(TORCH[dtype]).min, torch.finfo(TORCH[dtype]).max
    z = np.zeros((n, vocab))
    ids, labels = rng.integers(0, vocab, (n, 7)), rng.integers(0, vocab, n)
    t = torch.tensor(rng.standard_normal((n, 7)), dtype=torch.float32)
    x = torch.full((n, vocab), low).to(TORCH[dtype])
    x[1::2] = big
    for r in (2, 3, 6, 7):                                          # masked but for five, of which the teacher asks for some
        kept = rng.permutation(vocab)[:5]
        mask = np.ones(vocab, dtype=bool)
        mask[kept] = False
        z[r, mask] = -np.inf
        x[r, torch.tensor(mask)] = -float("inf")
        ids[r], labels[r] = kept[rng.integers(0, 5, 7)], kept[0]
    loss, g = call(cm.Plan(1, [1]), x, torch.tensor(ids), t, torch.tensor(labels), T, 1.0, 0.5, dtype)
    want, dg, off_loss, off = formulas(z, ids, f64(t), labels, T, 1.0, 0.5, 1.0, vocab, T == 2.0)
    close(f64(loss), want, off_loss, "loss")
    close(f64(g), dg, off + (HALF_STEP[cm.BF16] * (np.abs(dg) + off) if dtype == cm.BF16 else 0), "dlogits")


@pytest.mark.parametrize("vocab,n", [(50, 24), (9000, 24), (70000, 24), (70000, 100)])
@pytest.mark.parametrize("T", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_what_the_teacher_hardly_asks_for(dtype, T, vocab, n):
    """A P as small as the smallest fp32 numbers, and smaller, counts where the student's logit is the type's lowest number, or -infinity."""
    rng = np.random.default_rng(vocab)
    low = float(torch.finfo(TORCH[dtype]).min)
    x = torch.tensor(rng.standard_normal((n, vocab)), dtype=torch.float32).to(TORCH[dtype])
    ids = np.stack([rng.permutation(vocab)[:4] for _ in range(n)])
    labels = ids[:, 0]
    t = np.zeros((n, 4))
    t[:, 1] = -1.0
    t[:, 2] = -T * (70 + np.arange(n) % 24 * 2.0)                  # P from 10^-31 to 10^-51
    t[:, 3] = -T * 90.0
    t = torch.tensor(t, dtype=torch.float32)
    rows = torch.arange(n)
    x[rows, torch.tensor(ids[:, 2])] = low
    nothing = np.arange(n) % 5 == 3
    x[torch.tensor(nothing), torch.tensor(ids[nothing, 3])] = -float("inf")
    loss, g = call(cm.Plan(1, [1]), x, torch.tensor(ids), t, torch.tensor(labels), T, 1.0, 0.5, dtype)
    z = x.double().numpy()
    z -= z.max(1, keepdims=True)
    some = ~nothing
    want, dg, off_loss, off = formulas(z[some], ids[some], f64(t)[some], labels[some], T, 1.0, 0.5, 1.0, vocab, T == 2.0)
    assert want.max() > 1e3 and want.min() < 20
    close(f64(loss)[some], want, off_loss, "loss")
    close(f64(g)[some], dg, off + (HALF_STEP[cm.BF16] * (np.abs(dg) + off) if dtype == cm.BF16 else 0), "dlogits")
    assert bool((loss[torch.tensor(nothing)] == float("inf")).all()) and bool(g.isfinite().all())
