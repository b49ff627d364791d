"""The kernel variants that large calls of the gradient-filling operators take: all tilings of the weight gradient, the embedding
gradient of wide rows and long lists, the lookup with streaming stores."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import (DEV, HALF_STEP, TORCH, addresses, bound_plan, embedding_gradient, f64, rows, saved_sparse, stream, untouched,
                        workspace)
from test_gpu_layers import DTYPES, NAMES, TYPES, close, counts, dtype_id, make_ids, saved_checkpoints

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


@pytest.mark.parametrize("world,n,k,outputs", [(1, 50, 150, 64)] + [t[:4] for t in TILES.values()], ids=["few-tokens", *TILES])
def test_tiny_fp32_gradients_lose_only_what_lies_below_bf16(world, n, k, outputs):
    """From 2^-110 on a product is exact; below, dy's bits under 2^-133 are cut off.  x >= 1, so that no product is subnormal for x's
    sake alone."""
    print(f"case: tiny dy, world={world} n={n} k={k} outputs={outputs}", flush=True)
    rng = np.random.default_rng(n + k)
    dv = [(rng.choice([-1, 1], (m, outputs)) * 2.0 ** rng.uniform(-149, -100, (m, outputs))).astype(np.float32) for m in counts(world, n)]
    grads, placed, _ = sparse_gradient(rng, world, n, k, outputs, cm.F32, dv, (0, 100))
    for w, v in enumerate(dv):
        if len(v) == 0:
            assert not bool(grads[w].any())
            continue
        at, x = placed[w]
        v, x, got = v[at].astype(np.float64), x[:, None], f64(grads[w]).reshape(k, outputs)
        assert np.array_equal(got[np.abs(v) >= 2.0 ** -110], (v * x)[np.abs(v) >= 2.0 ** -110])
        assert (np.abs(got - v * x) < 2.0 ** -133 * x).all()


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


# ---- embedding gradient: wide rows, chunks of 16 and 32 ----------------------------------------
@pytest.mark.parametrize("accumulate", [False, True], ids=["write", "add"])
@pytest.mark.parametrize("dy_dtype,dtype", TYPES, ids=["f32", "bf16", "bf16-f32", "f32-bf16"])
@pytest.mark.parametrize("world,n,vocab,width,gap,kind", [
    (4, 4100, 3000, 300, 0, "skewed"), (4, 4111, 2, 300, 3, "uniform"), (4, 4100, 3000, 1001, 0, "padded"), (5, 4099, 2, 1001, 1, "padded"),
    (1, 17001, 700, 520, 0, "skewed"), (1, 17001, 500, 264, 4, "skewed"), (17, 1000, 29, 1024, 0, "skewed"), (2, 9000, 40, 96, 0, "skewed")])
def test_embedding_gradient_of_wide_rows_and_many_tokens(world, n, vocab, width, gap, kind, dy_dtype, dtype, accumulate):
    """From 16384 tokens over all workers on, chunks of 16 tokens (more than tokens / 32 rows) and of 32; rows that many chunks cut."""
    print(f"case: egrad world={world} n={n} vocab={vocab} width={width} {kind} {NAMES[dy_dtype]}->{NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n + width)
    ns, id_bytes, scale = counts(world, n), 8 if width % 2 else 4, -1.7
    plan, grads = bound_plan(world, [5, vocab * width, 3], dtype, fill=0.75)
    ids = [make_ids(kind, rng, m, vocab) for m in ns]
    di = [torch.tensor(i, dtype=torch.int64 if id_bytes == 8 else torch.int32, device=DEV) for i in ids]
    need = plan.embedding_workspace(1, width, ns)
    ws = workspace(need)
    gen = torch.Generator(device=DEV).manual_seed(n)
    for exact in (True, False):
        dy, old = [], 0.75 if accumulate else 0.0
        for m, i in zip(ns, di):
            v = (torch.randint(-8, 9, (m, width), device=DEV, generator=gen).float() if exact
                 else torch.randn(m, width, device=DEV, generator=gen))
            v[(i < 0) | (i >= vocab)] = float("nan")                                  # padding must not reach any row
            dy.append(rows(m, width, width + gap, dy_dtype, v))
        s, first = 2.0 if exact else scale, None
        for again in range(2):                               # the second time over other leftovers: the same bits
            ws[:max(need, 16)] = 0x5A if again else 0xFF
            for row in grads:
                row[1].fill_(0.75)
            plan.embedding_gradient(1, width, addresses(di), ns, addresses([d[0] for d in dy]), ws.data_ptr(), need, scale=s,
                                    id_bytes=id_bytes, dy_dtype=dy_dtype, dy_pitch=width + gap, accumulate=accumulate, stream=stream())
            torch.cuda.synchronize()
            assert untouched(ws, need)
            now = [row[1].clone() for row in grads]
            assert first is None or all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, now))
            first = now
        for w in range(world):
            known = ((di[w] >= 0) & (di[w] < vocab)).nonzero().flatten()
            at, d = di[w][known].long(), dy[w][1][known].double()
            zero = torch.zeros(vocab, width, dtype=torch.float64, device=DEV)
            want = float(np.float32(s)) * zero.index_add(0, at, d) + old
            got = grads[w][1].view(vocab, width)
            if exact:                                        # integers below 2^24: exact in fp32 in any order
                assert torch.equal(got, want.float().to(TORCH[dtype])), f"worker {w}"
            else:
                mag = abs(float(np.float32(s))) * zero.index_add(0, at, d.abs())
                terms = torch.bincount(at, minlength=vocab).double()[:, None]
                bound = (terms + 2) * 2.0 ** -24 * (mag + old) * (1 + 2.0 ** -10)
                if dtype == cm.BF16:
                    bound = bound + HALF_STEP[cm.BF16] * (want.abs() + bound)
                close(f64(got), f64(want), f64(bound), f"worker {w}")
            assert bool((grads[w][0] == 0.75).all()) and bool((grads[w][2] == 0.75).all()), "other tensors stay"
    plan.close()


@pytest.mark.parametrize("n,vocab,width", [(50, 30, 20), (50, 30, 3), (300, 200, 300), (300, 200, 33), (3000, 3, 301), (3000, 3, 2)])
@pytest.mark.parametrize("dy_dtype,dtype", TYPES, ids=["f32", "bf16", "bf16-f32", "f32-bf16"])
def test_accumulating_rounds_once(n, vocab, width, dy_dtype, dtype):
    """old + scale * sum in one rounding to fp32, for rows of few tokens, of a sorted list, and cut by chunks.  Sums of integers, a
    scale and old values of 24 bits in [1, 2): in 64 bits all of it is exact."""
    print(f"case: accumulate once, n={n} vocab={vocab} width={width} {NAMES[dy_dtype]}->{NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n + width)
    plan, grads = bound_plan(1, [vocab * width], dtype)
    ids = torch.tensor(rng.integers(0, vocab, n), device=DEV)
    dy = torch.tensor(rng.integers(-8, 9, (n, width)).astype(np.float32), device=DEV).to(TORCH[dy_dtype])
    old = torch.tensor((1 + rng.random(vocab * width)).astype(np.float32), device=DEV).to(TORCH[dtype])
    grads[0][0].copy_(old)
    scale = float(np.float32(1.7))
    need = plan.embedding_workspace(0, width, [n])
    ws = workspace(need)
    plan.embedding_gradient(0, width, [ids.data_ptr()], [n], [dy.data_ptr()], ws.data_ptr(), need, scale=scale, dy_dtype=dy_dtype,
                            accumulate=True, stream=stream())
    total = torch.zeros(vocab, width, dtype=torch.float64, device=DEV).index_add(0, ids, dy.double())
    want = (old.double().view(vocab, width) + scale * total).float().to(TORCH[dtype])
    assert torch.equal(grads[0][0].view(vocab, width), want)
    plan.close()


# ---- lookup: more than 32 MiB of output --------------------------------------------------------
@pytest.mark.parametrize("id_bytes", [4, 8])
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,vocab,width,gap", [(3, 9000, 500, 1001, 0), (2, 12001, 70, 1024, 8), (2, 400_000, 1000, 35, 1)])
def test_lookup_with_streaming_stores(world, n, vocab, width, gap, dtype, id_bytes):
    print(f"case: lookup world={world} n={n} vocab={vocab} width={width} gap={gap} dtype={NAMES[dtype]}", flush=True)
    ns, scale = [n] * (world - 1) + [n // 2 + 9], 2.7
    assert sum(ns) * width * 2 > 32 << 20
    gen = torch.Generator(device=DEV).manual_seed(n)
    plan = cm.Plan(world, [1], dtype=dtype)
    table = [torch.randn(vocab, width, device=DEV, generator=gen).to(TORCH[dtype]) for _ in range(world)]
    ids = [torch.randint(-2, vocab + 2, (m,), device=DEV, generator=gen).to(torch.int64 if id_bytes == 8 else torch.int32) for m in ns]
    out = [rows(m, width, width + gap, dtype, fill=7.0) for m in ns]
    plan.embedding_lookup(addresses(table), vocab, width, addresses(ids), ns, addresses([o[0] for o in out]), scale=scale,
                          id_bytes=id_bytes, out_pitch=width + gap, stream=stream())
    torch.cuda.synchronize()
    for w in range(world):
        mem, view = out[w]
        known = (ids[w] >= 0) & (ids[w] < vocab)
        want = table[w].float()[ids[w].long().clamp(0, vocab - 1)] * torch.tensor(scale, dtype=torch.float32, device=DEV)
        want = torch.where(known[:, None], want, torch.zeros((), device=DEV)).to(TORCH[dtype])       # one product, one rounding: exact
        assert torch.equal(view, want), f"worker {w}"
        view.fill_(7.0)
        assert bool((mem == 7.0).all()), "the gaps between the rows and what lies behind the last one stay"
    plan.close()


# ---- the workers' rows side by side in one array -------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,width", [(2, 70, 33), (3, 5, 1), (8, 40, 260), (64, 33, 7)])
def test_rows_of_all_workers_interleave(world, n, width, dtype):
    """[token][worker][column]: lookup, store and load, and both gradients, one column free behind the last worker's."""
    print(f"case: interleaved rows world={world} n={n} width={width} dtype={NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n + width)
    vocab, k, pitch, es = 40, 24, world * width + 1, 2 if dtype == cm.BF16 else 4
    plan, grads = bound_plan(world, [vocab * width, k * width], dtype)
    side_by_side = lambda fill: torch.full((n, pitch), fill, dtype=TORCH[dtype], device=DEV)                # noqa: E731
    at = lambda t: [t.data_ptr() + w * width * es for w in range(world)]                                 # noqa: E731
    of = lambda t, w: t[:, w * width:(w + 1) * width]                                                    # noqa: E731
    table = torch.tensor(rng.integers(-8, 9, (vocab, width)).astype(np.float32)).to(TORCH[dtype])
    ids = [torch.tensor(rng.integers(-1, vocab, n)) for _ in range(world)]
    dt, di, ns = table.to(DEV), [i.to(DEV) for i in ids], [n] * world
    x, back = side_by_side(7.0), side_by_side(7.0)
    plan.embedding_lookup([dt.data_ptr()] * world, vocab, width, addresses(di), ns, at(x), out_pitch=pitch, stream=stream())
    saved = [torch.empty(cm.checkpoint_bytes(n, width), dtype=torch.uint8, device=DEV) for _ in range(world)]
    plan.checkpoint_store(at(x), ns, width, addresses(saved), dtype=dtype, pitch=pitch, stream=stream())
    plan.checkpoint_load(addresses(saved), ns, width, at(back), dtype=dtype, pitch=pitch, stream=stream())
    torch.cuda.synchronize()
    for w in range(world):
        want = torch.where((ids[w] >= 0)[:, None], table[ids[w].clamp(min=0)], torch.zeros((), dtype=TORCH[dtype]))
        assert torch.equal(of(x, w).cpu(), want) and torch.equal(of(back, w).cpu(), want)                 # integers: kept as they are
    assert bool((x[:, -1] == 7.0).all()) and bool((back[:, -1] == 7.0).all())
    dy = side_by_side(float("nan"))
    for w in range(world):
        of(dy, w).copy_(torch.tensor(rng.integers(-8, 9, (n, width)).astype(np.float32)))
    need = [plan.embedding_workspace(0, width, ns), plan.weight_gradient_workspace(1, k, ns)]
    ws = [workspace(b) for b in need]
    kept = [rng.integers(-8, 9, (n, k)).astype(np.float64) for _ in range(world)]
    codes = saved_checkpoints(kept)
    plan.embedding_gradient(0, width, addresses(di), ns, at(dy), ws[0].data_ptr(), need[0], dy_pitch=pitch, stream=stream())
    plan.weight_gradient(1, None, addresses(codes), ns, k, at(dy), ws[1].data_ptr(), need[1], dy_pitch=pitch, stream=stream())
    torch.cuda.synchronize()
    for w in range(world):
        d = f64(of(dy, w))
        for got, want in ((grads[w][0].view(vocab, width), embedding_gradient(vocab, ids[w].tolist(), d, 1.0)[0]),
                          (grads[w][1].view(k, width), kept[w].T @ d)):
            assert torch.equal(got.cpu(), torch.tensor(want, dtype=torch.float32).to(TORCH[dtype])), f"worker {w}"
    plan.close()
