"""The operators that fill a plan's gradient tensors, against plain statements in 64 bits.

Tolerances.  A sum of n terms in fp32, in whatever order, is off by at most (n - 1) 2^-24 of the sum of the
magnitudes per addition's rounding; the matrix cores may cut instead of round inside an instruction, which
doubles the step.  Multiplying by the scale and adding to what the tensor held are one rounding each, and
the result is rounded once to its type.  Where all numbers are small integers (or the like), every sum is exact in fp32
in any order, and results must be equal."""
import numpy as np
import pytest
import torch

import oracle
import paper_2004_14020_amd as cm

from gpu_util import assert_same_bits
from layer_util import (DEV, HALF_STEP, TORCH, addresses, bound_plan, decode, embedding_gradient, encode, f64, image, lookup, rows,
                        stream, untouched, workspace)

pytestmark = pytest.mark.gpu

DTYPES = [cm.F32, cm.BF16]
NAMES = {cm.F32: "f32", cm.BF16: "bf16"}


def dtype_id(d):
    return NAMES.get(d, str(d))


def close(got, want, bound, what=""):
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: got {got[bad][0]!r}, " \
                          f"want {want[bad][0]!r}, bound {np.broadcast_to(bound, got.shape)[bad][0]!r}"


def counts(world, n):
    """Different numbers of tokens per worker, among them 0 and n."""
    return [n if w == 0 else (0 if w == 1 else max(0, n - 3 * w)) for w in range(world)]


# ---- lookup ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,vocab,width,gap,id_bytes", [
    (1, 1, 1, 1, 0, 8), (2, 1, 5, 3, 0, 4), (3, 7, 9, 8, 5, 4), (8, 65, 100, 17, 1, 8), (2, 300, 512, 1000, 0, 8),
    (3, 129, 2, 1001, 7, 4), (1, 1030, 3000, 64, 64, 8), (2, 33, 40, 2500, 0, 4), (64, 5, 30, 24, 0, 8)])
def test_lookup(world, n, vocab, width, gap, id_bytes, dtype):
    print(f"case: lookup world={world} n={n} vocab={vocab} width={width} gap={gap} dtype={NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n * width)
    plan, ns, scale = cm.Plan(world, [1], dtype=dtype), counts(world, n), 2.7
    table = [torch.randn(vocab, width).to(TORCH[dtype]) for _ in range(world)]
    ids = [rng.integers(-2, vocab + 2, m) for m in ns]
    dt = [t.to(DEV) for t in table]
    di = [torch.tensor(i, dtype=torch.int64 if id_bytes == 8 else torch.int32, device=DEV) for i in ids]
    out = [rows(m, width, width + gap, dtype, fill=7.0) for m in ns]
    plan.embedding_lookup(addresses(dt), vocab, width, addresses(di), ns, addresses([o[0] for o in out]), scale=scale,
                          id_bytes=id_bytes, out_pitch=width + gap, stream=stream())
    torch.cuda.synchronize()
    for w, m in enumerate(ns):
        mem, view = out[w]
        known = torch.tensor((ids[w] >= 0) & (ids[w] < vocab))
        want = table[w].float()[torch.tensor(ids[w]).clamp(0, vocab - 1)] * torch.tensor(scale, dtype=torch.float32)
        want = torch.where(known[:, None], want, torch.zeros(())).to(TORCH[dtype])       # one product, one rounding: exact
        assert torch.equal(view.cpu(), want), f"worker {w}"
        close(f64(view), lookup(f64(table[w]), ids[w], scale), 2 * HALF_STEP[dtype] * np.abs(lookup(f64(table[w]), ids[w], scale)))
        view.fill_(7.0)
        assert bool((mem == 7.0).all()), "the gaps between the rows and what lies behind the last one stay"
    plan.close()


def test_lookup_keeps_infinities_and_nan_and_zeroes_padding():
    plan = cm.Plan(1, [1])
    table = torch.tensor([[float("inf"), float("nan"), -0.0], [1.0, 2.0, float("-inf")]], device=DEV)
    ids = torch.tensor([1, -1, 0, 2, 1 << 40], device=DEV)
    out = torch.full((5, 3), 9.0, device=DEV)
    plan.embedding_lookup([table.data_ptr()], 2, 3, [ids.data_ptr()], [5], [out.data_ptr()], scale=1.0, stream=stream())
    want = torch.tensor([[1.0, 2.0, float("-inf")], [0, 0, 0], [float("inf"), float("nan"), -0.0], [0, 0, 0], [0, 0, 0]])
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=5.0), torch.nan_to_num(want, nan=5.0))
    plan.close()


# ---- embedding gradient ---------------------------------------------------------------------
def make_ids(kind, rng, n, vocab):
    if kind == "uniform":
        return rng.integers(0, vocab, n)
    if kind == "skewed":
        return np.minimum((vocab * rng.random(n) ** 6).astype(np.int64), vocab - 1)
    if kind == "one":
        return np.full(n, vocab - 1)
    if kind == "padded":
        return np.where(rng.random(n) < 0.5, rng.integers(0, vocab, n), rng.choice([-1, vocab, -(1 << 31)], n))
    if kind == "padding":
        return np.full(n, -1)
    return np.arange(n) % vocab


EGRAD = [  # world, tokens, vocab, width, gap, ids
    (1, 1, 1, 1, 0, "one"), (2, 9, 5, 3, 2, "uniform"), (3, 64, 64, 8, 0, "positions"), (8, 65, 100, 17, 1, "skewed"),
    (2, 300, 512, 1000, 0, "padded"), (3, 1025, 2, 1001, 7, "uniform"), (1, 5000, 3000, 64, 0, "skewed"),
    (2, 2000, 7, 260, 4, "one"), (1, 777, 1500, 2500, 0, "uniform"), (64, 40, 30, 24, 0, "uniform"), (2, 100, 50, 16, 0, "padding"),
    (4, 6000, 1025, 36, 0, "positions"), (20, 100, 50, 40, 0, "uniform"), (37, 130, 9, 300, 1, "skewed")]


@pytest.mark.parametrize("accumulate", [False, True], ids=["write", "add"])
@pytest.mark.parametrize("dy_dtype,dtype", [(cm.F32, cm.F32), (cm.BF16, cm.BF16), (cm.BF16, cm.F32), (cm.F32, cm.BF16)],
                         ids=["f32", "bf16", "bf16-f32", "f32-bf16"])
@pytest.mark.parametrize("world,n,vocab,width,gap,kind", EGRAD)
def test_embedding_gradient(world, n, vocab, width, gap, kind, dy_dtype, dtype, accumulate):
    print(f"case: egrad world={world} n={n} vocab={vocab} width={width} {kind} {NAMES[dy_dtype]}->{NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n + width)
    ns, scale, id_bytes = counts(world, n), -1.7, 8 if n % 2 else 4
    plan, grads = bound_plan(world, [5, vocab * width, 3], dtype, fill=0.75)
    ids = [make_ids(kind, rng, m, vocab) for m in ns]
    di = [torch.tensor(i, dtype=torch.int64 if id_bytes == 8 else torch.int32, device=DEV) for i in ids]
    for exact in (True, False):
        dy = []
        for m, i in zip(ns, ids):
            v = torch.tensor(rng.integers(-8, 9, (m, width)).astype(np.float32) if exact
                             else rng.standard_normal((m, width)).astype(np.float32))
            v[torch.tensor((i < 0) | (i >= vocab))] = float("nan")        # padding must not reach any row
            dy.append(rows(m, width, width + gap, dy_dtype, v))
        need = plan.embedding_workspace(1, width, ns)
        ws = workspace(need)
        for w in range(world):
            grads[w][1].fill_(0.75)
        s = 2.0 if exact else scale
        plan.embedding_gradient(1, width, addresses(di), ns, addresses([d[0] for d in dy]), ws.data_ptr(), need, scale=s,
                                id_bytes=id_bytes, dy_dtype=dy_dtype, dy_pitch=width + gap, accumulate=accumulate, stream=stream())
        torch.cuda.synchronize()
        assert untouched(ws, need)
        first = [g[1].clone() for g in grads]
        for w in range(world):
            want, mag, terms = embedding_gradient(vocab, ids[w], f64(dy[w][1]), s)
            old = 0.75 if accumulate else 0.0
            got = f64(grads[w][1]).reshape(vocab, width)
            if exact:
                want32 = torch.tensor(want + old, dtype=torch.float32)    # exact in fp32
                assert torch.equal(grads[w][1].cpu().view(vocab, width), want32.to(TORCH[dtype])), f"worker {w}"
            else:
                bound = (terms + 2) * 2.0 ** -24 * (mag + old) * (1 + 2.0 ** -10)
                close(got, want + old, bound + (HALF_STEP[cm.BF16] * (np.abs(want + old) + bound) if dtype == cm.BF16 else 0),
                      f"worker {w}")
            assert bool((grads[w][0] == 0.75).all()) and bool((grads[w][2] == 0.75).all()), "other tensors stay"
        # the same call again, over a workspace full of something else: the same bits
        ws.fill_(0x5A)
        for w in range(world):
            grads[w][1].fill_(0.75)
        plan.embedding_gradient(1, width, addresses(di), ns, addresses([d[0] for d in dy]), ws.data_ptr(), need, scale=s,
                                id_bytes=id_bytes, dy_dtype=dy_dtype, dy_pitch=width + gap, accumulate=accumulate, stream=stream())
        for w in range(world):
            assert torch.equal(first[w].view(torch.uint8), grads[w][1].view(torch.uint8))
    plan.close()


@pytest.mark.parametrize("world,n,vocab,width,kind", [(2, 4097, 1, 3, "one"), (1, 12289, 40, 8, "skewed"), (2, 20001, 3, 5, "padded"),
                                                      (1, 33000, 2100, 9, "skewed"), (3, 8191, 17, 16, "positions"),
                                                      (1, 70000, 1030, 4, "padded"), (1, 16500, 5000, 70, "skewed")])
def test_embedding_gradient_of_long_lists(world, n, vocab, width, kind):
    """More tokens than the sort keeps in registers: they are counted and dealt out in steps."""
    test_embedding_gradient(world, n, vocab, width, 0, kind, cm.F32, cm.F32, False)


def test_embedding_gradient_agrees_with_differences():
    """<gradient, direction> = <dy, what the lookup gives for the direction>: the lookup is linear in the table."""
    rng = np.random.default_rng(5)
    vocab, width, n, scale = 50, 40, 333, 1.5
    plan, grads = bound_plan(1, [vocab * width], cm.F32)
    ids = torch.tensor(rng.integers(0, vocab, n), device=DEV)
    dy = torch.randn(n, width, device=DEV)
    need = plan.embedding_workspace(0, width, [n])
    ws = workspace(need)
    plan.embedding_gradient(0, width, [ids.data_ptr()], [n], [dy.data_ptr()], ws.data_ptr(), need, scale=scale, stream=stream())
    table, step, out = torch.randn(vocab, width, device=DEV), torch.randn(vocab, width, device=DEV), []
    for t in (table + step, table - step):
        y = torch.empty(n, width, device=DEV)
        plan.embedding_lookup([t.data_ptr()], vocab, width, [ids.data_ptr()], [n], [y.data_ptr()], scale=scale, stream=stream())
        out.append(y)
    torch.cuda.synchronize()
    want = float(((out[0].double() - out[1].double()) / 2 * dy.double()).sum())
    got = float((grads[0][0].double().view(vocab, width) * step.double()).sum())
    # each product carries the roundings of table +- step, of the scaled rows, and of the gradient's sum over ~7 tokens
    mag = float((out[0].abs().double() * dy.abs().double()).sum() + (out[1].abs().double() * dy.abs().double()).sum()) / 2
    assert abs(got - want) <= 30 * 2.0 ** -24 * 2 * mag
    plan.close()


# ---- checkpoints ----------------------------------------------------------------------------
def special(rng, n, k):
    x = (rng.standard_normal((n, k)) * 10.0 ** rng.integers(-6, 6, k)).astype(np.float32)
    kinds = [lambda c: c * 0, lambda c: c * np.float32(1e-38), lambda c: np.full_like(c, np.float32(3.4e38)),
             lambda c: np.full_like(c, 127.0), lambda c: np.full_like(c, 127.25), lambda c: np.full_like(c, 127.5),
             lambda c: np.arange(len(c), dtype=np.float32) - 16.5, lambda c: c * np.float32(1e-45), lambda c: -np.abs(c)]
    for j in range(0, k, 2):
        x[:, j] = kinds[(j // 2) % len(kinds)](x[:, j])
    if n and k > 20:
        x[n // 2, 5], x[n - 1, 7], x[0, 9] = np.inf, np.nan, -np.inf
    return x


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,k,gap", [(1, 1, 1, 0), (2, 31, 3, 1), (3, 32, 4, 0), (8, 33, 5, 3), (2, 100, 255, 0),
                                           (1, 65, 1030, 2), (2, 257, 64, 64), (64, 10, 21, 0), (2, 1000, 2050, 0)])
def test_checkpoint(world, n, k, gap, dtype):
    print(f"case: checkpoint world={world} n={n} k={k} gap={gap} dtype={NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n * k)
    plan, ns = cm.Plan(world, [1]), counts(world, n)
    x = [rows(m, k, k + gap, dtype, torch.tensor(special(rng, m, k))) for m in ns]
    size = [cm.checkpoint_bytes(m, k) for m in ns]
    saved = [torch.full((s + 64,), 0xEE, dtype=torch.uint8, device=DEV) for s in size]
    plan.checkpoint_store(addresses([v[0] for v in x]), ns, k, addresses(saved), dtype=dtype, pitch=k + gap, stream=stream())
    torch.cuda.synchronize()
    want = []
    for w, m in enumerate(ns):
        codes, scales = encode(f64(x[w][1]))
        want.append(decode(codes, scales, m))
        n_bytes = codes.size + scales.size
        assert np.array_equal(saved[w].cpu().numpy()[:n_bytes], image(codes, scales)[:n_bytes]), f"worker {w}"
        assert bool((saved[w][size[w]:] == 0xEE).all())
    for out_dtype in DTYPES:
        out = [rows(m, k, k + gap, out_dtype, fill=7.0) for m in ns]
        plan.checkpoint_load(addresses(saved), ns, k, addresses([o[0] for o in out]), dtype=out_dtype, pitch=k + gap, stream=stream())
        torch.cuda.synchronize()
        for w, m in enumerate(ns):
            assert np.array_equal(f64(out[w][1]), want[w], equal_nan=True)      # exact in either type
            out[w][1].fill_(7.0)
            assert bool((out[w][0] == 7.0).all())
    plan.close()


# ---- weight gradient ------------------------------------------------------------------------
def saved_checkpoints(x):
    return [torch.tensor(image(*encode(v)), device=DEV) if len(v) else torch.empty(16, dtype=torch.uint8, device=DEV) for v in x]


def whole(rng, n, k):
    """Activations that a checkpoint keeps exactly: integers, the largest of every block 64 or less."""
    return rng.integers(-8, 9, (n, k)).astype(np.float64)


WGRAD = [  # world, tokens, features, outputs, gap
    (1, 1, 1, 1, 0), (2, 5, 3, 10, 0), (3, 33, 33, 2, 4), (8, 64, 32, 64, 0), (2, 100, 130, 129, 1), (1, 300, 257, 200, 0),
    (2, 31, 784, 256, 0), (1, 1500, 40, 70, 2), (1, 2100, 300, 131, 3), (64, 20, 17, 12, 0), (8, 260, 1100, 1060, 0),
    (8, 289, 1030, 1301, 0), (12, 2050, 500, 510, 0), (12, 2050, 500, 511, 1), (2, 190, 70, 1, 0), (2, 230, 70, 1, 3),
    (1, 64, 1000, 130, 0), (3, 192, 40, 300, 2),
    (20, 600, 40, 70, 0), (33, 225, 130, 50, 1)]
TYPES = [(cm.F32, cm.F32), (cm.BF16, cm.BF16), (cm.BF16, cm.F32), (cm.F32, cm.BF16)]


@pytest.mark.parametrize("accumulate", [False, True], ids=["write", "add"])
@pytest.mark.parametrize("dy_dtype,dtype", TYPES, ids=["f32", "bf16", "bf16-f32", "f32-bf16"])
@pytest.mark.parametrize("world,n,k,outputs,gap", WGRAD)
def test_weight_gradient(world, n, k, outputs, gap, dy_dtype, dtype, accumulate):
    print(f"case: wgrad world={world} n={n} k={k} outputs={outputs} {NAMES[dy_dtype]}->{NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n + k)
    ns, old = counts(world, n), 0.75 if accumulate else 0.0
    plan, grads = bound_plan(world, [outputs, 3, k * outputs, 5], dtype, fill=0.75)
    need = plan.weight_gradient_workspace(2, k, ns)
    ws = workspace(need)
    for exact in (True, False):
        if exact:
            x = [whole(rng, m, k) for m in ns]
            dv = [rng.integers(-8, 9, (m, outputs)).astype(np.float32) for m in ns]
        else:
            x = [decode(*encode(rng.standard_normal((m, k)).astype(np.float32)), m) for m in ns]
            dv = [rng.standard_normal((m, outputs)).astype(np.float32) for m in ns]
        saved = saved_checkpoints(x)
        dy = [rows(m, outputs, outputs + gap, dy_dtype, torch.tensor(v)) for m, v in zip(ns, dv)]
        results = []
        for again in range(2):
            ws.fill_(0xFF if again else 0x5A)
            ws[max(need, 16):] = 0xFF
            for row in grads:
                for g in row:
                    g.fill_(0.75)
            plan.weight_gradient(2, 0, addresses(saved), ns, k, addresses([d[0] for d in dy]), ws.data_ptr(), need,
                                 dy_dtype=dy_dtype, dy_pitch=outputs + gap, accumulate=accumulate, stream=stream())
            torch.cuda.synchronize()
            results.append([[g.clone() for g in row] for row in grads])
        assert untouched(ws, need)
        for w, m in enumerate(ns):
            for t in (0, 2):
                assert torch.equal(results[0][w][t].view(torch.uint8), results[1][w][t].view(torch.uint8)), "not reproducible"
            assert bool((grads[w][1] == 0.75).all()) and bool((grads[w][3] == 0.75).all()), "other tensors stay"
            d = f64(dy[w][1])
            for got, want, mag in ((grads[w][2].view(k, outputs), x[w].T @ d, np.abs(x[w]).T @ np.abs(d)),
                                   (grads[w][0], d.sum(0), np.abs(d).sum(0))):
                want = want + old
                if exact:
                    assert torch.equal(got.cpu(), torch.tensor(want, dtype=torch.float32).to(TORCH[dtype])), f"worker {w}"
                else:
                    terms = m * (1 if dy_dtype == cm.BF16 else 3) + 2
                    bound = terms * 2.0 ** -23 * (mag * (1 + 2.0 ** -6) + old)
                    close(f64(got), want, bound + (HALF_STEP[cm.BF16] * (np.abs(want) + bound) if dtype == cm.BF16 else 0),
                          f"worker {w}")
    plan.close()


@pytest.mark.parametrize("dy_dtype,dtype", TYPES, ids=["f32", "bf16", "bf16-f32", "f32-bf16"])
@pytest.mark.parametrize("world,n,k,outputs,gap", [(2, 700, 150, 63, 1), (1, 3000, 129, 319, 0), (3, 520, 64, 33, 5), (17, 390, 515, 64, 0),
                                                  (1, 6000, 31, 1, 0), (1, 40000, 20, 9, 1), (2, 1400, 260, 192, 2), (1, 5900, 100, 200, 0)])
def test_weight_gradient_of_few_outputs(world, n, k, outputs, gap, dy_dtype, dtype):
    """Outputs that fill no tile of 128, in one part of the tokens and in many."""
    test_weight_gradient(world, n, k, outputs, gap, dy_dtype, dtype, True)


def test_weight_gradient_loses_no_bit_of_fp32_gradients():
    """dy with 24 significant bits, one token per sum: the product must be right to the last bit."""
    rng = np.random.default_rng(7)
    n, k, outputs = 24, 24, 40
    x = np.zeros((n, k))
    x[np.arange(n), np.arange(k)] = 2.0 ** rng.integers(-3, 4, k)
    dv = (rng.standard_normal((n, outputs)) * 10.0 ** rng.integers(-20, 20, (n, 1))).astype(np.float32)
    plan, grads = bound_plan(1, [k * outputs], cm.F32)
    saved, dy = saved_checkpoints([x]), torch.tensor(dv, device=DEV)
    plan.weight_gradient(0, None, addresses(saved), [n], k, [dy.data_ptr()], None, 0, stream=stream())
    assert np.array_equal(f64(grads[0][0]).reshape(k, outputs), x.T @ dv.astype(np.float64))
    plan.close()


@pytest.mark.parametrize("dy_dtype", DTYPES, ids=dtype_id)
def test_weight_gradient_passes_on_infinities_and_nan(dy_dtype):
    n, k, outputs = 40, 70, 90
    x = np.ones((n, k), np.float32)
    x[3, 5] = np.nan                                        # marks the block of 32 tokens of feature 5
    dv = np.ones((n, outputs), np.float32)
    dv[7, 11], dv[35, 13], dv[39, 17] = np.inf, -np.inf, np.nan
    plan, grads = bound_plan(1, [k * outputs, outputs], cm.F32)
    saved, dy = saved_checkpoints([x.astype(np.float64)]), torch.tensor(dv, device=DEV).to(TORCH[dy_dtype])
    plan.weight_gradient(0, 1, addresses(saved), [n], k, [dy.data_ptr()], None, 0, dy_dtype=dy_dtype, stream=stream())
    want = np.full((k, outputs), float(n))
    want[:, 11], want[:, 13], want[:, 17] = np.inf, -np.inf, np.nan
    want[5] = np.nan
    assert np.array_equal(f64(grads[0][0]).reshape(k, outputs), want, equal_nan=True)
    want = np.full(outputs, float(n))
    want[11], want[13], want[17] = np.inf, -np.inf, np.nan
    assert np.array_equal(f64(grads[0][1]), want, equal_nan=True)
    plan.close()


def test_weight_gradient_agrees_with_differences():
    """The layer is linear in its weights: <dW, direction> = <dy, x direction>."""
    rng = np.random.default_rng(9)
    n, k, outputs = 200, 96, 80
    x = decode(*encode(rng.standard_normal((n, k)).astype(np.float32)), n)
    dv, step = rng.standard_normal((n, outputs)).astype(np.float32), rng.standard_normal((k, outputs))
    plan, grads = bound_plan(1, [k * outputs], cm.F32)
    saved, dy = saved_checkpoints([x]), torch.tensor(dv, device=DEV)
    need = plan.weight_gradient_workspace(0, k, [n])
    ws = workspace(need)
    plan.weight_gradient(0, None, addresses(saved), [n], k, [dy.data_ptr()], ws.data_ptr(), need, stream=stream())
    weights = rng.standard_normal((k, outputs))
    loss = [float(((x @ (weights + s * step)) * dv).sum()) for s in (0.5, -0.5)]
    got = float((f64(grads[0][0]).reshape(k, outputs) * step).sum())
    bound = (3 * n + 2) * 2.0 ** -23 * float(((np.abs(x).T @ np.abs(dv)) * np.abs(step)).sum()) * (1 + 2.0 ** -6)
    assert abs(got - (loss[0] - loss[1])) <= bound + 1e-9 * abs(got)
    plan.close()


# ---- together, as a training step calls them ------------------------------------------------
class Step:
    """One data-parallel step's backward pass of  ids -> embedding -> dense layer, for W workers."""

    def __init__(self, dtype, world=3, n=70, vocab=200, width=72, outputs=50, seed=0):
        self.dtype, self.world, self.vocab, self.width, self.outputs = dtype, world, vocab, width, outputs
        self.ns = [n - 5 * w for w in range(world)]
        self.scale = 4.0
        self.plan = cm.Plan(world, [outputs, width * outputs, vocab * width], dtype=dtype, batch_threshold_bytes=1 << 14)
        T = TORCH[dtype]
        self.grads = [[torch.zeros(n, dtype=T, device=DEV) for n in self.plan.elems] for _ in range(world)]
        self.plan.bind([addresses(r) for r in self.grads], None)
        self.table = torch.zeros(vocab, width, dtype=T, device=DEV)
        self.ids = [torch.zeros(m, dtype=torch.int64, device=DEV) for m in self.ns]
        self.x = [torch.zeros(m, width, dtype=T, device=DEV) for m in self.ns]
        self.dy = [torch.zeros(m, outputs, dtype=T, device=DEV) for m in self.ns]
        self.dx = [torch.zeros(m, width, dtype=T, device=DEV) for m in self.ns]
        self.saved = [torch.zeros(cm.checkpoint_bytes(m, width), dtype=torch.uint8, device=DEV) for m in self.ns]
        self.need = [self.plan.weight_gradient_workspace(1, width, self.ns), self.plan.embedding_workspace(2, width, self.ns)]
        self.ws = [workspace(b) for b in self.need]
        self.fill(seed)

    def fill(self, seed):
        g = torch.Generator().manual_seed(seed)
        T = TORCH[self.dtype]
        self.table.copy_(torch.randint(-8, 9, (self.vocab, self.width), generator=g).to(T))
        for w, m in enumerate(self.ns):
            self.ids[w].copy_(torch.randint(-1, self.vocab, (m,), generator=g))
            self.dy[w].copy_(torch.randint(-4, 5, (m, self.outputs), generator=g).to(T))
            self.dx[w].copy_(torch.randint(-4, 5, (m, self.width), generator=g).to(T))
        torch.cuda.synchronize()

    def forward(self, s):
        self.plan.embedding_lookup([self.table.data_ptr()] * self.world, self.vocab, self.width, addresses(self.ids), self.ns,
                                   addresses(self.x), scale=self.scale, stream=s)
        self.plan.checkpoint_store(addresses(self.x), self.ns, self.width, addresses(self.saved), stream=s)

    def backward(self, s):
        self.plan.weight_gradient(1, 0, addresses(self.saved), self.ns, self.width, addresses(self.dy), self.ws[0].data_ptr(),
                                  self.need[0], stream=s)
        self.plan.embedding_gradient(2, self.width, addresses(self.ids), self.ns, addresses(self.dx), self.ws[1].data_ptr(),
                                     self.need[1], scale=self.scale, stream=s)

    def run(self, s):
        self.forward(s)
        self.backward(s)
        self.plan.allreduce(s)

    def check(self, what):
        torch.cuda.synchronize()
        np_dtype = np.float32 if self.dtype == cm.F32 else np.uint16
        raw = torch.float32 if self.dtype == cm.F32 else torch.int16
        ref = []
        for w in range(self.world):
            x = lookup(f64(self.table), self.ids[w].tolist(), self.scale)
            x = decode(*encode(x), self.ns[w])
            d = f64(self.dy[w])
            e = embedding_gradient(self.vocab, self.ids[w].tolist(), f64(self.dx[w]), self.scale)[0]
            ref.append([torch.tensor(v, dtype=torch.float32).to(TORCH[self.dtype]).view(raw).numpy().view(np_dtype).reshape(-1).copy()
                        for v in (d.sum(0), x.T @ d, e)])                     # integers below 2^24: exact sums
        cfg = oracle.Config(self.world, self.dtype, 1 << 14, oracle.SPLIT_NONE, 8, 0, 16, 2)
        oracle.allreduce(oracle.build_plan(cfg, self.plan.elems), ref)
        got = [[g.view(raw).cpu().numpy().view(np_dtype) for g in row] for row in self.grads]
        assert_same_bits(got, ref, what)


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_a_training_step_end_to_end(dtype):
    step = Step(dtype)
    for seed in (1, 2):
        step.fill(seed)
        step.run(stream())
        step.check(f"step with seed {seed}")
    step.plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_a_training_step_on_another_stream(dtype):
    step = Step(dtype)
    side = torch.cuda.Stream()
    step.fill(3)
    side.wait_stream(torch.cuda.current_stream())
    step.run(side.cuda_stream)
    side.synchronize()
    step.check("side stream")
    step.plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_a_captured_training_step_replays(dtype):
    step, other = Step(dtype), Step(dtype, n=90, outputs=64)
    graphs = []
    for s in (step, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for seed in (4, 5, 6):
        for s, g in zip((step, other), graphs):
            s.fill(seed)
            for row in s.grads:
                for t in row:
                    t.fill_(float("nan"))
            for ws in s.ws:
                ws.fill_(0xFF)
            g.replay()
        for s in (step, other):
            s.check(f"replay with seed {seed}")
    step.fill(7)
    step.run(stream())
    step.check("eager after the replays")
    del graphs
    step.plan.close()
    other.plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_weight_gradient_of_few_tokens_and_large_tensors(dtype):
    """More than the last-level cache holds: streaming stores."""
    rng = np.random.default_rng(12)
    n, k, outputs = 40, 9000, 8192 if dtype == cm.F32 else 16384
    plan, grads = bound_plan(1, [k * outputs], dtype)
    x, d = whole(rng, n, k), torch.tensor(rng.integers(-8, 9, (n, outputs)).astype(np.float32)).to(TORCH[dtype])
    saved, dy = saved_checkpoints([x]), d.to(DEV)
    plan.weight_gradient(0, None, addresses(saved), [n], k, [dy.data_ptr()], None, 0, stream=stream())
    want = (torch.tensor(x.T, dtype=torch.float32, device=DEV) @ d.float().to(DEV)).to(TORCH[dtype])       # integers: exact
    assert torch.equal(grads[0][0].view(k, outputs), want)
    plan.close()


def test_overlap_with_the_bound_tensors_is_refused():
    plan, grads = bound_plan(1, [64 * 32], cm.F32)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    need = plan.embedding_workspace(0, 32, [4])
    ws = workspace(need)
    with pytest.raises(cm.CaramelError) as e:
        plan.embedding_gradient(0, 32, [ids.data_ptr()], [4], [grads[0][0].data_ptr()], ws.data_ptr(), need, stream=stream())
    assert e.value.status == cm.binding.EINVAL
    with pytest.raises(cm.CaramelError) as e:
        plan.weight_gradient(0, None, [ws.data_ptr()], [4], 64, [grads[0][0].data_ptr()], None, 0, stream=stream())
    assert e.value.status == cm.binding.EINVAL
    plan.close()


@pytest.mark.parametrize("accumulate", [False, True], ids=["write", "add"])
def test_no_tokens_at_all(accumulate):
    """Gradients of nothing: zeros, or what was there; no pointer of a worker without tokens is looked at."""
    plan, grads = bound_plan(2, [30 * 20, 20], cm.F32, fill=0.75)
    need = plan.embedding_workspace(0, 20, [0, 0])
    ws = workspace(need)
    none = [None, None]
    plan.embedding_lookup(none, 30, 20, none, [0, 0], none, stream=stream())
    plan.checkpoint_store(none, [0, 0], 30, none, stream=stream())
    plan.checkpoint_load(none, [0, 0], 30, none, stream=stream())
    plan.embedding_gradient(0, 20, none, [0, 0], none, ws.data_ptr(), need, accumulate=accumulate, stream=stream())
    want = 0.75 if accumulate else 0.0
    assert all(bool((row[0] == want).all()) and bool((row[1] == 0.75).all()) for row in grads)
    for row in grads:
        row[0].fill_(0.75)
    plan.weight_gradient(0, 1, none, [0, 0], 30, none, None, 0, accumulate=accumulate, stream=stream())
    assert all(bool((t == want).all()) for row in grads for t in row)
    plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_rows_that_start_on_any_element(dtype):
    """Every buffer of rows one element behind an aligned address, even and odd widths."""
    rng = np.random.default_rng(11)
    n, vocab = 77, 40
    for width in (64, 63, 130):
        plan, grads = bound_plan(1, [vocab * width, 48 * width], cm.F32)
        at = lambda t: [t.data_ptr() + t.element_size()]                               # noqa: E731
        shifted = lambda v: torch.cat([v.new_zeros(1), v.reshape(-1)]).to(DEV)         # noqa: E731
        typed = cm.Plan(1, [1], dtype=dtype)
        table = torch.tensor(rng.integers(-8, 9, (vocab, width)).astype(np.float32)).to(TORCH[dtype])
        rows_ = torch.tensor(rng.integers(-8, 9, (n, width)).astype(np.float32)).to(TORCH[dtype])
        ids = torch.tensor(rng.integers(0, vocab, n), device=DEV)
        src, dy, out = shifted(table), shifted(rows_), torch.full((n * width + 2,), 7.0, dtype=TORCH[dtype], device=DEV)
        typed.embedding_lookup(at(src), vocab, width, [ids.data_ptr()], [n], at(out), stream=stream())
        assert torch.equal(out[1:-1].cpu().view(n, width), table[ids.cpu()]) and float(out[0]) == float(out[-1]) == 7.0
        need = plan.embedding_workspace(0, width, [n])
        ws = workspace(need)
        plan.embedding_gradient(0, width, [ids.data_ptr()], [n], at(dy), ws.data_ptr(), need, dy_dtype=dtype, stream=stream())
        assert np.array_equal(f64(grads[0][0]).reshape(vocab, width), embedding_gradient(vocab, ids.tolist(), f64(rows_), 1.0)[0])
        saved = torch.empty(cm.checkpoint_bytes(n, width), dtype=torch.uint8, device=DEV)
        plan.checkpoint_store(at(dy), [n], width, [saved.data_ptr()], dtype=dtype, stream=stream())
        out.fill_(7.0)
        plan.checkpoint_load([saved.data_ptr()], [n], width, at(out), dtype=dtype, stream=stream())
        assert torch.equal(out[1:-1].cpu().view(n, width), rows_) and float(out[0]) == float(out[-1]) == 7.0
        for tokens in (n, 300):                              # few tokens, and a second kernel
            x = whole(rng, tokens, 48)
            d = torch.tensor(rng.integers(-8, 9, (tokens, width)).astype(np.float32)).to(TORCH[dtype])
            kept, moved = saved_checkpoints([x]), shifted(d)
            need = plan.weight_gradient_workspace(1, 48, [tokens])
            ws = workspace(need)
            plan.weight_gradient(1, None, addresses(kept), [tokens], 48, at(moved), ws.data_ptr(), need, dy_dtype=dtype, stream=stream())
            assert np.array_equal(f64(grads[0][1]).reshape(48, width), x.T @ f64(d))
        plan.close()
        typed.close()


# ---- offsets beyond 32 bits -----------------------------------------------------------------
def test_a_table_of_more_than_four_gib():
    vocab, width = 2_200_000, 1024                           # 4.5 GB in bf16
    plan, grads = bound_plan(1, [vocab * width], cm.BF16)
    table = torch.zeros(vocab, width, dtype=torch.bfloat16, device=DEV)
    picked = torch.tensor([0, vocab - 1, 2_097_151, 2_097_152, 1_048_576, vocab - 1], device=DEV)
    table[picked] = torch.arange(6, dtype=torch.bfloat16, device=DEV)[:, None] + 1
    out = torch.empty(6, width, dtype=torch.bfloat16, device=DEV)
    plan.embedding_lookup([table.data_ptr()], vocab, width, [picked.data_ptr()], [6], [out.data_ptr()], stream=stream())
    assert torch.equal(out, table[picked])
    need = plan.embedding_workspace(0, width, [6])
    ws = workspace(need)
    plan.embedding_gradient(0, width, [picked.data_ptr()], [6], [out.data_ptr()], ws.data_ptr(), need, stream=stream())
    g = grads[0][0].view(vocab, width)
    for v in picked:                                         # a row that is named twice holds either value, column by column
        assert torch.equal(g[v].float(), out[picked == v].float().sum(0))
    named = torch.zeros(vocab, dtype=torch.bool, device=DEV)
    named[picked] = True
    assert bool((g.amax(1)[~named] == 0).all()) and bool((g.amin(1)[~named] == 0).all())
    plan.close()


def test_rows_that_lie_more_than_four_gib_apart():
    n, width, pitch = 300, 64, 1 << 23                       # 300 rows, 5 GB in bf16
    plan, grads = bound_plan(1, [10 * width, 32 * width, width], cm.F32)
    mem = torch.zeros(n * pitch, dtype=torch.bfloat16, device=DEV)
    dy = mem.view(n, pitch)[:, :width]
    dy.copy_(torch.randint(-8, 9, (n, width)).to(torch.bfloat16))
    ids = torch.arange(n, device=DEV) % 10
    need = plan.embedding_workspace(0, width, [n])
    ws = workspace(need)
    plan.embedding_gradient(0, width, [ids.data_ptr()], [n], [mem.data_ptr()], ws.data_ptr(), need, dy_dtype=cm.BF16,
                            dy_pitch=pitch, stream=stream())
    assert np.array_equal(f64(grads[0][0]).reshape(10, width), embedding_gradient(10, ids.tolist(), f64(dy), 1.0)[0])
    saved = torch.empty(cm.checkpoint_bytes(n, width), dtype=torch.uint8, device=DEV)
    plan.checkpoint_store([mem.data_ptr()], [n], width, [saved.data_ptr()], dtype=cm.BF16, pitch=pitch, stream=stream())
    codes, scales = encode(f64(dy))
    b = codes.size + scales.size
    assert np.array_equal(saved.cpu().numpy()[:b], image(codes, scales)[:b])
    x = np.random.default_rng(1).integers(-4, 5, (n, 32)).astype(np.float64)
    kept = saved_checkpoints([x])
    need = plan.weight_gradient_workspace(1, 32, [n])
    ws = workspace(need)
    plan.weight_gradient(1, 2, addresses(kept), [n], 32, [mem.data_ptr()], ws.data_ptr(), need, dy_dtype=cm.BF16, dy_pitch=pitch,
                         stream=stream())
    assert np.array_equal(f64(grads[0][1]).reshape(32, width), x.T @ f64(dy))
    assert np.array_equal(f64(grads[0][2]), f64(dy).sum(0))
    out = mem
    out.zero_()
    plan.checkpoint_load([saved.data_ptr()], [n], width, [out.data_ptr()], dtype=cm.BF16, pitch=pitch, stream=stream())
    assert np.array_equal(f64(dy), decode(codes, scales, n))
    plan.close()
