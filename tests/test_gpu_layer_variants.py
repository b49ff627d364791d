"""The kernel variants that large calls of the gradient-filling operators take: all tilings of the weight gradient."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import DEV, TORCH, addresses, bound_plan, saved_sparse, stream, untouched, workspace
from test_gpu_layers import DTYPES, NAMES, counts, dtype_id

pytestmark = pytest.mark.gpu


# ---- weight gradient: every tiling, in one part of the tokens and in several ------------------
# world, tokens, features, outputs, parts.  With fp32 dy more than 64 tokens leave the kernel for few tokens, with bf16 dy more than
# 192.  An odd number of strips of 64 outputs, five at most: narrow tiles.  At least 192 workgroups of 256 x 256: large ones.
TILES = {"narrow": (1, 200, 150, 64, False), "narrow-parts": (2, 3000, 150, 63, True), "small": (2, 210, 257, 200, False),
         "small-parts": (1, 3000, 300, 120, True), "large": (8, 260, 1100, 1060, False), "large-parts": (1, 1541, 2000, 2042, True)}


def tiles():
    return pytest.mark.parametrize("world,n,k,outputs,parts", TILES.values(), ids=TILES.keys())


def one_token_each(rng, n, k, powers):
    """x with one token per feature, a power of two; all tokens, and all places of a block, where there are features enough."""
    step = next(s for s in range(max(1, n // k) | 1, 2 * n + 3, 2) if np.gcd(s, n) == 1) if n else 1
    at = (int(rng.integers(n)) + step * np.arange(k)) % n if n else np.zeros(0, np.int64)
    return at, 2.0 ** rng.integers(*powers, k)


def sparse_gradient(rng, world, n, k, outputs, dtype, dv, powers):
    """(grads, tokens of the features, their values, tensors to keep) of x with one token per feature and fp32 gradients dv[w]."""
    ns = counts(world, n)
    plan, grads = bound_plan(world, [k * outputs], dtype)
    placed = [one_token_each(rng, m, k, powers) for m in ns]
    saved = [saved_sparse(m, *p) for m, p in zip(ns, placed)]
    dy = [torch.tensor(v, device=DEV) for v in dv]
    need = plan.weight_gradient_workspace(0, k, ns)
    ws = workspace(need)
    plan.weight_gradient(0, None, addresses(saved), ns, k, addresses(dy), ws.data_ptr(), need, dy_dtype=cm.F32, stream=stream())
    torch.cuda.synchronize()
    assert untouched(ws, need)
    plan.close()
    return [row[0] for row in grads], placed, need


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@tiles()
def test_tiles_lose_no_bit_of_fp32_gradients(world, n, k, outputs, parts, dtype):
    """One product per sum, dy with 24 significant bits: right to the last bit, in all places of a tile."""
    print(f"case: bits of dy, world={world} n={n} k={k} outputs={outputs} ->{NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n + outputs)
    dv = [(rng.standard_normal((m, outputs)) * 10.0 ** rng.integers(-20, 20, (m, 1))).astype(np.float32) for m in counts(world, n)]
    grads, placed, need = sparse_gradient(rng, world, n, k, outputs, dtype, dv, (-3, 4))
    assert (need > 0) == parts
    for w, v in enumerate(dv):
        at, x = placed[w]
        want = torch.zeros(k, outputs) if len(v) == 0 else torch.tensor(v)[at] * torch.tensor(x, dtype=torch.float32)[:, None]
        assert torch.equal(grads[w].view(k, outputs).cpu(), want.to(TORCH[dtype])), f"worker {w}"


@pytest.mark.parametrize("dy_dtype", DTYPES, ids=dtype_id)
@tiles()
def test_tiles_pass_on_infinities_and_nan(world, n, k, outputs, parts, dy_dtype):
    print(f"case: special values, world={world} n={n} k={k} outputs={outputs} dy={NAMES[dy_dtype]}", flush=True)
    ns = counts(world, n)
    plan, grads = bound_plan(world, [k * outputs, outputs], cm.F32)
    need = plan.weight_gradient_workspace(0, k, ns)
    ws = workspace(need)
    saved, dy = [], []
    for m in ns:
        codes, scales = np.zeros(((m + 31) // 32, k, 32), np.int8), np.full(((m + 31) // 32, k), 121, np.uint8)      # 64 * 2^-6
        codes[:] = 64
        if m % 32:
            codes[-1, :, m % 32:] = 0
        d = torch.ones(m, outputs)
        if m:
            codes[m // 2 // 32, 5], scales[m // 2 // 32, 5] = 0, 255
            codes[-1, k - 1], scales[-1, k - 1] = 0, 255
            d[0, 11], d[m // 2, outputs - 1], d[m - 1, 17], d[m - 1, 0] = float("inf"), float("-inf"), float("nan"), float("-inf")
        saved.append(torch.tensor(np.frombuffer(codes.tobytes() + scales.tobytes() + bytes(16), np.uint8).copy(), device=DEV))
        dy.append(d.to(TORCH[dy_dtype]).to(DEV))
    plan.weight_gradient(0, 1, addresses(saved), ns, k, addresses(dy), ws.data_ptr(), need, dy_dtype=dy_dtype, stream=stream())
    torch.cuda.synchronize()
    for w, m in enumerate(ns):
        bias = torch.full((outputs,), float(m))
        if m:
            bias[11], bias[outputs - 1], bias[17], bias[0] = float("inf"), float("-inf"), float("nan"), float("-inf")
        want = bias.expand(k, outputs).clone()
        if m:
            want[5], want[k - 1] = float("nan"), float("nan")
        for got, ref in ((grads[w][0].view(k, outputs), want), (grads[w][1], bias)):
            assert torch.equal(torch.nan_to_num(got.cpu(), nan=-5.0), torch.nan_to_num(ref, nan=-5.0)), f"worker {w}"
    plan.close()
