"""The residual norm and its gradient, against plain statements in 64 bits.

Tolerances.  Everything the forward pass does with a row but its mean square is one fp32 operation after the other, so given
rstd its results must be equal; rstd itself is a sum of `width` squares in 64 bits, rounded once.  In the gradient a product
or sum of fp32 numbers is off by at most 2^-24 of its magnitude, and a sum of n terms by n times that of the magnitudes'."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import DEV, HALF_STEP, TORCH, addresses, bound_plan, encode, f64, image, rows, stream, untouched, workspace
from test_gpu_layers import DTYPES, NAMES, close, counts, dtype_id

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
TYPES = [(cm.F32, cm.F32), (cm.BF16, cm.BF16), (cm.BF16, cm.F32), (cm.F32, cm.BF16)]
TYPE_IDS = ["f32", "bf16", "bf16-f32", "f32-bf16"]          # rows, gains


def same(a, b):
    """Equal bits, but for which NaN it is."""
    a, b = a.cpu(), b.cpu()
    return a.shape == b.shape and bool(((a == b) | (a.isnan() & b.isnan())).all())


def norm64(x, gain, eps):
    r = 1.0 / np.sqrt((x * x).mean(1) + eps)
    return x * r[:, None] * gain, r


def gradient64(x, gain, r, dy, dsum):
    """dx, dgain, and how far fp32 may be off each."""
    width, n = x.shape[1], x * r[:, None]
    u = dy * gain
    c, mag = (u * n).mean(1, keepdims=True), np.abs(u * n).mean(1, keepdims=True)
    dx = r[:, None] * (u - n * c) + dsum
    off = 4 * STEP * (r[:, None] * (np.abs(u) + np.abs(n * c)) + np.abs(dsum)) + r[:, None] * np.abs(n) * (width + 4) * STEP * mag
    return dx, (dy * n).sum(0), off, (len(x) + 3) * STEP * np.abs(dy * n).sum(0)


def inputs(rng, n, width, dtype, size=1.0):
    x = rng.standard_normal((n, width)) * size * 10.0 ** rng.uniform(-1, 1, width)
    return torch.tensor(x, dtype=torch.float32).to(TORCH[dtype])


FORWARD = [  # world, tokens, width, gap
    (1, 1, 1, 0), (2, 3, 2, 1), (3, 7, 7, 0), (8, 33, 9, 3), (2, 65, 255, 0), (64, 5, 40, 0), (1, 70, 512, 8), (20, 9, 513, 1),
    (2, 129, 1024, 0), (3, 40, 1025, 2), (2, 31, 2047, 1), (1, 64, 2048, 0), (2, 33, 4096, 0), (1, 20, 4097, 3), (2, 5, 8191, 0),
    (1, 9, 16385, 1), (1, 4, 32768, 0), (1, 700, 64, 0)]


def check_forward(world, n, width, gap, dtype, gain_dtype, residual, saved, ns=None, eps=1e-5):
    print(f"case: norm world={world} n={n} width={width} gap={gap} {NAMES[dtype]} gain {NAMES[gain_dtype]}", flush=True)
    rng = np.random.default_rng(n * width)
    ns = counts(world, n) if ns is None else ns
    plan, pitch = cm.Plan(world, [1], dtype=gain_dtype), width + gap
    gain = [inputs(rng, 1, width, gain_dtype)[0].to(DEV) for _ in ns]
    x = [rows(m, width, pitch, dtype, inputs(rng, m, width, dtype)) for m in ns]
    res = [rows(m, width, pitch, dtype, inputs(rng, m, width, dtype, 3.0)) for m in ns]
    total, y = ([rows(m, width, pitch, dtype, fill=7.0) for m in ns] for _ in range(2))
    rstd = [torch.full((m + 3,), 9.0, device=DEV) for m in ns]
    size = [cm.checkpoint_bytes(m, width) for m in ns]
    kept = [torch.full((s + 64,), 0xEE, dtype=torch.uint8, device=DEV) for s in size]
    plan.residual_norm(addresses(gain), width, ns, addresses([v[0] for v in x]), addresses([v[0] for v in y]), addresses(rstd), eps=eps,
                       residual=addresses([v[0] for v in res]) if residual else None,
                       sum=addresses([v[0] for v in total]) if residual else None,
                       checkpoint=addresses(kept) if saved else None, dtype=dtype, pitch=pitch, stream=stream())
    torch.cuda.synchronize()
    for w, m in enumerate(ns):
        h = x[w][1]
        if residual:
            h = (x[w][1].float() + res[w][1].float()).to(TORCH[dtype])
            assert same(total[w][1], h), f"worker {w}"
        _, want = norm64(f64(h), f64(gain[w]), float(np.float32(eps)))
        close(f64(rstd[w][:m]), want, (STEP + (width + 8) * 2.0 ** -52) * want, f"worker {w}: rstd")
        assert bool((rstd[w][m:] == 9.0).all())
        # (on the CPU, one operation at a time)
        r, g = rstd[w][:m, None].cpu(), gain[w].float().cpu()
        assert same(y[w][1], ((h.float().cpu() * r) * g).to(TORCH[dtype])), f"worker {w}"
        if saved:
            codes, scales = encode(f64(y[w][1]))
            whole = codes.size + scales.size
            assert np.array_equal(kept[w].cpu().numpy()[:whole], image(codes, scales)[:whole]), f"worker {w}"
            assert bool((kept[w][size[w]:] == 0xEE).all())
        else:
            assert bool((kept[w] == 0xEE).all())
        for mem, view in (y[w], total[w]):
            view.fill_(7.0)
            assert bool((mem == 7.0).all()), "the gaps between the rows and what lies behind the last one stay"
    plan.close()


@pytest.mark.parametrize("residual,saved", [(False, False), (True, False), (True, True), (False, True)],
                         ids=["plain", "residual", "residual-saved", "saved"])
@pytest.mark.parametrize("dtype,gain_dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("world,n,width,gap", FORWARD)
def test_norm(world, n, width, gap, dtype, gain_dtype, residual, saved):
    check_forward(world, n, width, gap, dtype, gain_dtype, residual, saved)


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("n,width,gap", [(4096, 1024, 0), (4099, 1000, 0), (2050, 4096, 0), (1100, 2048, 2), (9000, 130, 0), (300, 8192, 0),
                                         (4200, 2049, 1), (8200, 1111, 0)])
def test_norm_of_many_tokens(n, width, gap, dtype):
    """As many blocks of 32 tokens as fill the GPU, whole and not; matrices of more than 28 MiB."""
    check_forward(2, n, width, gap, dtype, dtype, True, True, ns=[n, n - 37])


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("n", [5, 9000])
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_norm_of_extreme_rows(dtype, n, saved):
    """Infinities, NaN, zeros, the largest and smallest numbers: by the formulas, and in their own row (block) only."""
    width, plan = 40, cm.Plan(1, [1])
    big, small = torch.finfo(TORCH[dtype]).max, 2.0 ** -126
    x = torch.randn(n, width).to(TORCH[dtype])
    x[0], x[1, 3], x[2, 5], x[3], x[4] = 0.0, float("inf"), float("nan"), big, small
    gain = torch.randn(width)
    y, rstd = rows(n, width, width, dtype, fill=7.0), torch.empty(n, device=DEV)
    kept = torch.empty(cm.checkpoint_bytes(n, width), dtype=torch.uint8, device=DEV)
    dx, dg = x.to(DEV), gain.to(DEV)
    plan.residual_norm([dg.data_ptr()], width, [n], [dx.data_ptr()], [y[0].data_ptr()], [rstd.data_ptr()], eps=1e-6,
                       checkpoint=[kept.data_ptr()] if saved else None, dtype=dtype, stream=stream())
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        _, r = norm64(x.double().numpy(), gain.double().numpy(), float(np.float32(1e-6)))
    got = rstd.cpu().double().numpy()
    assert got[1] == 0.0 and np.isnan(got[2]) and np.isfinite(np.delete(got, 2)).all()
    close(np.delete(got, 2), np.delete(r, 2), np.delete(r, 2) * (STEP + 2.0 ** -40))
    assert same(y[1], ((x.float() * rstd.cpu()[:, None]) * gain).to(TORCH[dtype]))
    if saved:
        codes, scales = encode(f64(y[1]))
        assert np.array_equal(kept.cpu().numpy()[:codes.size + scales.size], image(codes, scales)[:codes.size + scales.size])
    plan.close()


GRADIENT = [  # world, tokens, width, gap
    (1, 1, 1, 0), (2, 3, 2, 1), (3, 9, 7, 0), (8, 33, 9, 3), (64, 6, 40, 0), (1, 700, 64, 0), (2, 300, 255, 0), (20, 17, 513, 1),
    (2, 129, 1024, 0), (3, 40, 1025, 2), (2, 31, 2047, 1), (2, 33, 4096, 0), (1, 20, 4097, 3), (2, 9, 8191, 0), (1, 9, 16385, 1),
    (1, 4, 32768, 0), (2, 4100, 100, 0)]

LARGE = [(2, 3700, 2049, 1), (3, 4900, 1024, 0)]   # more than 28 MiB of bf16


@pytest.mark.parametrize("accumulate", [False, True], ids=["write", "add"])
@pytest.mark.parametrize("with_dsum", [False, True], ids=["alone", "dsum"])
@pytest.mark.parametrize("dtype,gain_dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("world,n,width,gap", GRADIENT)
def test_norm_gradient(world, n, width, gap, dtype, gain_dtype, with_dsum, accumulate):
    print(f"case: norm gradient world={world} n={n} width={width} {NAMES[dtype]} gain {NAMES[gain_dtype]}", flush=True)
    rng = np.random.default_rng(n + width)
    ns, pitch, old = counts(world, n), width + gap, 0.75 if accumulate else 0.0
    plan, grads = bound_plan(world, [3, width, 5], gain_dtype, fill=0.75)
    gain = [inputs(rng, 1, width, gain_dtype)[0].to(DEV) for _ in ns]
    x, dy, dsum = ([rows(m, width, pitch, dtype, inputs(rng, m, width, dtype, s)) for m in ns] for s in (1.0, 0.1, 0.1))
    rstd = [torch.tensor(norm64(f64(v[1]), 1.0, 1e-5)[1], dtype=torch.float32, device=DEV) for v in x]
    need = plan.residual_norm_workspace(1, ns)
    results = []
    for again in range(2):
        ws = workspace(need)
        ws[:need] = 0x5A if again else 0xFF
        dx = [rows(m, width, pitch, dtype, fill=7.0) for m in ns]
        for row in grads:
            row[1].fill_(0.75)
        plan.residual_norm_gradient(1, addresses(gain), ns, addresses([v[0] for v in x]), addresses(rstd), addresses([v[0] for v in dy]),
                                    addresses([v[0] for v in dx]), ws.data_ptr(), need,
                                    dsum=addresses([v[0] for v in dsum]) if with_dsum else None, dtype=dtype, pitch=pitch,
                                    accumulate=accumulate, stream=stream())
        torch.cuda.synchronize()
        assert untouched(ws, need)
        results.append([t.clone() for v in dx for t in v[:1]] + [row[1].clone() for row in grads])
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*results)), "not reproducible"
    for w, m in enumerate(ns):
        want, dg, off, off_g = gradient64(f64(x[w][1]), f64(gain[w]), f64(rstd[w]), f64(dy[w][1]), f64(dsum[w][1]) if with_dsum else
                                          np.zeros((m, width)))
        half = HALF_STEP[cm.BF16]
        close(f64(dx[w][1]), want, off + (half * (np.abs(want) + off) if dtype == cm.BF16 else 0), f"worker {w}: dx")
        off_g = off_g + STEP * (np.abs(dg) + old)
        close(f64(grads[w][1]), dg + old, off_g + (half * (np.abs(dg + old) + off_g) if gain_dtype == cm.BF16 else 0), f"worker {w}: dgain")
        assert bool((grads[w][0] == 0.75).all()) and bool((grads[w][2] == 0.75).all()), "other tensors stay"
        dx[w][1].fill_(7.0)
        assert bool((dx[w][0] == 7.0).all())
    plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,width,gap", LARGE)
def test_norm_gradient_of_many_tokens(world, n, width, gap, dtype):
    test_norm_gradient(world, n, width, gap, dtype, dtype, True, False)


def test_norm_gradient_agrees_with_differences():
    """Of <dy, y> + <dsum, x>, in 64 bits, along directions of x and of the gain."""
    rng = np.random.default_rng(3)
    n, width, eps, h = 23, 37, 1e-5, 1e-6
    plan, grads = bound_plan(1, [width], cm.F32)
    x, dy, dsum = (inputs(rng, n, width, cm.F32) for _ in range(3))
    gain = inputs(rng, 1, width, cm.F32)[0]
    d = [t.to(DEV) for t in (gain, x, dy, dsum)]
    y, dx, rstd = (torch.empty(s, device=DEV) for s in ((n, width), (n, width), (n,)))
    need = plan.residual_norm_workspace(0, [n])
    ws = workspace(need)
    plan.residual_norm([d[0].data_ptr()], width, [n], [d[1].data_ptr()], [y.data_ptr()], [rstd.data_ptr()], eps=eps, stream=stream())
    plan.residual_norm_gradient(0, [d[0].data_ptr()], [n], [d[1].data_ptr()], [rstd.data_ptr()], [d[2].data_ptr()], [dx.data_ptr()],
                                ws.data_ptr(), need, dsum=[d[3].data_ptr()], stream=stream())
    torch.cuda.synchronize()
    x, dy, dsum, gain = (f64(t) for t in (x, dy, dsum, gain))

    def value(x, gain):
        return (dy * norm64(x, gain, float(np.float32(eps)))[0]).sum() + (dsum * x).sum()

    _, _, off, off_g = gradient64(x, gain, f64(rstd), dy, dsum)
    off += STEP * (np.abs(gradient64(x, gain, f64(rstd), dy, 0 * dsum)[0]) * 4 + np.abs(x * dy * gain).sum(1, keepdims=True))  # rstd's rounding
    for _ in range(3):
        a, b = rng.standard_normal((n, width)), rng.standard_normal(width)
        want = (value(x + h * a, gain) - value(x - h * a, gain)) / (2 * h)
        # the differences: curvature of relative size h^2, and the roundings of value over h
        slack = 1e-8 * (np.abs(dy * gain).sum() + np.abs(dsum).sum()) * 10
        assert abs((f64(dx) * a).sum() - want) <= (off * np.abs(a)).sum() + slack
        want = value(x, gain + b) - value(x, gain)                               # linear in the gain
        assert abs((f64(grads[0][0]) * b).sum() - want) <= ((off_g + STEP * np.abs(dy * x).sum(0)) * np.abs(b)).sum() + slack
    plan.close()


def test_norm_without_any_tokens():
    for accumulate in (False, True):
        plan, grads = bound_plan(2, [6], cm.F32, fill=0.75)
        plan.residual_norm([None] * 2, 6, [0, 0], [None] * 2, [None] * 2, [None] * 2, residual=[None] * 2, sum=[None] * 2,
                           checkpoint=[None] * 2, stream=stream())
        need = plan.residual_norm_workspace(0, [0, 0])
        ws = workspace(need)
        plan.residual_norm_gradient(0, [None] * 2, [0, 0], [None] * 2, [None] * 2, [None] * 2, [None] * 2, ws.data_ptr(), need,
                                    accumulate=accumulate, stream=stream())
        torch.cuda.synchronize()
        assert all(bool((row[0] == (0.75 if accumulate else 0.0)).all()) for row in grads)
        plan.close()


def test_rows_of_a_norm_more_than_four_gib_apart():
    """The last of 300 rows, 2^23 elements apart, is behind 2^32 bytes, and behind 2^31 elements."""
    n, width, pitch = 300, 16, 1 << 23
    plan, grads = bound_plan(1, [width], cm.F32)
    free, _ = torch.cuda.mem_get_info()
    need = 4 * n * pitch * 2
    if free < need + (4 << 30):
        pytest.skip("not enough memory")
    x, y, dx, dy = (torch.empty(n * pitch, dtype=torch.bfloat16, device=DEV) for _ in range(4))
    view = lambda t: t.view(n, pitch)[:, :width]                                  # noqa: E731
    values = torch.randn(n, width).to(torch.bfloat16)
    view(x).copy_(values)
    view(dy).copy_(values.flip(0))
    gain, rstd = torch.ones(width, device=DEV), torch.empty(n, device=DEV)
    plan.residual_norm([gain.data_ptr()], width, [n], [x.data_ptr()], [y.data_ptr()], [rstd.data_ptr()], dtype=cm.BF16, pitch=pitch,
                       stream=stream())
    size = plan.residual_norm_workspace(0, [n])
    ws = workspace(size)
    plan.residual_norm_gradient(0, [gain.data_ptr()], [n], [x.data_ptr()], [rstd.data_ptr()], [dy.data_ptr()], [dx.data_ptr()],
                                ws.data_ptr(), size, dtype=cm.BF16, pitch=pitch, stream=stream())
    torch.cuda.synchronize()
    assert same(view(y), (values.float() * rstd.cpu()[:, None]).to(torch.bfloat16))
    want, dg, off, off_g = gradient64(f64(values), np.ones(width), f64(rstd), f64(values.flip(0)), 0.0)
    close(f64(view(dx)), want, off + HALF_STEP[cm.BF16] * (np.abs(want) + off))
    close(f64(grads[0][0]), dg, off_g + STEP * np.abs(dg))
    plan.close()


def test_norm_calls_captured_into_a_graph():
    """Replayed three times, with new inputs and eager calls of the same buffers in between."""
    n, width = 1200, 200
    plan, grads = bound_plan(2, [width], cm.BF16)
    make = lambda: [torch.empty(n, width, dtype=torch.bfloat16, device=DEV) for _ in range(2)]      # noqa: E731
    x, res, total, y, dy, dx = (make() for _ in range(6))
    gain, rstd = [torch.randn(width, device=DEV).bfloat16() for _ in range(2)], [torch.empty(n, device=DEV) for _ in range(2)]
    kept = [torch.empty(cm.checkpoint_bytes(n, width), dtype=torch.uint8, device=DEV) for _ in range(2)]
    need = plan.residual_norm_workspace(0, [n, n])
    ws = workspace(need)

    def step():
        plan.residual_norm(addresses(gain), width, [n, n], addresses(x), addresses(y), addresses(rstd), residual=addresses(res),
                           sum=addresses(total), checkpoint=addresses(kept), stream=stream())
        plan.residual_norm_gradient(0, addresses(gain), [n, n], addresses(total), addresses(rstd), addresses(dy), addresses(dx),
                                    ws.data_ptr(), need, dsum=addresses(y), stream=stream())

    def outputs():
        torch.cuda.synchronize()
        return [t.clone() for t in total + y + rstd + kept + dx + [row[0] for row in grads]]

    def fill(seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        for t in x + res + dy:
            t.copy_(torch.randn(t.shape, device=DEV, generator=g))
        for t in total + y + rstd + kept + dx + [row[0] for row in grads] + [ws]:
            t.fill_(1)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fill(0)
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        fill(seed)
        step()
        want = outputs()
        fill(seed)
        graph.replay()
        assert all(same(a, b) for a, b in zip(outputs(), want))
    plan.close()
