"""Distillation of more rows than are cut into parts, wider than what a workgroup holds (115200 bf16 or 130560 fp32 logits): what is behind that is
summed up as it passes, and read again for the gradient."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import DEV, HALF_STEP, TORCH, addresses, f64, rows, stream, untouched, workspace
from test_gpu_distillation import formulas
from test_gpu_layers import NAMES, close

pytestmark = pytest.mark.gpu

HELD = {cm.F32: 130560, cm.BF16: 115200}
CASES = [  # dtype, tokens of the workers, vocabulary, gap
    (cm.BF16, [97], 115201, 0), (cm.BF16, [97], 115215, 1), (cm.BF16, [60, 41], 151936, 0), (cm.BF16, [99], 256000, 0),
    (cm.F32, [97], 130563, 0), (cm.F32, [60, 41], 150001, 3), (cm.F32, [97], 130561, 0)]


@pytest.mark.parametrize("T,soft,hard", [(1.0, 0.7, 0.5), (2.0, 1.0, 0.5), (4.0, 0.5, 1.0), (3.0, 1.0, 1.5), (2.5, 1.0, 0.0)])
@pytest.mark.parametrize("dtype,ns,vocab,gap", CASES, ids=lambda v: str(v))
def test_rows_that_are_read_twice(dtype, ns, vocab, gap, T, soft, hard):
    print(f"case: wide distillation {ns} vocab={vocab} T={T} {soft} {hard} {NAMES[dtype]}", flush=True)
    rng, top, held = np.random.default_rng(vocab), 12, HELD[dtype]
    plan, pitch, scale = cm.Plan(len(ns), [1]), vocab + gap, 3.0
    gen = torch.Generator(device=DEV)
    gen.manual_seed(vocab)
    logits, ids, teacher, labels = [], [], [], []
    for m in ns:
        z = (torch.randn(m, vocab, device=DEV, generator=gen) * 3).clamp_(-15, 15)
        # the largest logit where it is held, behind that, and in the last column
        at = [int(rng.integers(0, held)) if r % 3 == 0 else int(rng.integers(held, vocab)) if r % 3 == 1 else vocab - 1 for r in range(m)]
        z[torch.arange(m), torch.tensor(at)] = 20.0
        z[4, held:] = -float("inf")                             # nothing behind; nothing held
        z[5, :held] = -float("inf")
        z = z.to(TORCH[dtype])
        if dtype == cm.F32:                                     # so large that the largest one is subtracted first
            z[7] = (z[7] * 16).round() / 16 * 4 + 2.0 ** 21
            z[8] = (z[8] * 16).round() / 16 * 4 - 2.0 ** 21
        i, lab = rng.integers(0, vocab, (m, top)), rng.integers(0, vocab, m)
        i[:, 0] = at
        i[:, 1] = rng.integers(held, vocab, m)
        i[rng.random((m, top)) < 0.1] = -1
        i[4], i[5] = rng.integers(0, held, top), rng.integers(held, vocab, top)
        lab[::2] = rng.integers(held, vocab, len(lab[::2]))
        lab[4], lab[5], lab[6] = 3, vocab - 1, -1
        i[9], lab[9] = -1, -1                                   # nothing to learn
        logits.append(rows(m, vocab, pitch, dtype, z))
        ids.append(i)
        teacher.append(torch.tensor(rng.standard_normal((m, top)) * 3, dtype=torch.float32, device=DEV))
        labels.append(lab)
    on = lambda v: [torch.tensor(x, device=DEV) for x in v]                               # noqa: E731
    di, dl = on(ids), on(labels)
    need = plan.distillation_workspace(vocab, top, ns)
    results = []
    for how in ("apart", "in place", "loss alone"):
        ws, loss = workspace(need), [torch.full((m + 3,), 9.0, device=DEV) for m in ns]
        src = [(mem.clone(), ) for mem, _ in logits] if how == "in place" else [(mem,) for mem, _ in logits]
        out = src if how == "in place" else [(torch.full_like(mem, 7.0),) for mem, _ in logits]
        plan.distillation(vocab, ns, [s[0].data_ptr() for s in src], addresses(di), addresses(teacher), top, addresses(loss), ws.data_ptr(),
                          need, labels=addresses(dl) if hard else None, dlogits=None if how == "loss alone" else [o[0].data_ptr() for o in out],
                          temperature=T, soft=soft, hard=hard, scale=scale, dtype=dtype, teacher_dtype=cm.F32, pitch=pitch,
                          dlogits_pitch=pitch, stream=stream())
        torch.cuda.synchronize()
        assert untouched(ws, need) and all(bool((v[m:] == 9.0).all()) for v, m in zip(loss, ns))
        views = [o[0][:m * pitch].view(m, pitch) for o, m in zip(out, ns)]
        if how == "apart":
            assert all(bool((v[:, vocab:] == 7.0).all()) and bool((o[0][m * pitch:] == 7.0).all()) for v, o, m in zip(views, out, ns))
        results.append((loss, [v[:, :vocab].clone() for v in views]))
    for (loss, out), what in zip(results[1:], ("in place", "loss alone")):
        assert all(torch.equal(a, b) for a, b in zip(loss, results[0][0])), what
        if what == "in place":
            assert all(torch.equal(a, b) for a, b in zip(out, results[0][1])), what
    for w, m in enumerate(ns):
        some = list(range(12)) + [m - 1]
        z = f64(logits[w][1][some])
        z -= z.max(1, keepdims=True)                            # exact: in 64 bits
        want, g, off_loss, off = formulas(z, ids[w][some], f64(teacher[w])[some], labels[w][some], T, soft, hard, scale, vocab, T in (2.0, 4.0))
        close(f64(results[0][0][w][:m])[some], want, off_loss, f"worker {w}: loss")
        close(f64(results[0][1][w][some]), g, off + (HALF_STEP[cm.BF16] * (np.abs(g) + off) if dtype == cm.BF16 else 0), f"worker {w}: dlogits")
        assert float(results[0][0][w][9]) == 0.0 and bool((results[0][1][w][9] == 0.0).all())
    plan.close()
