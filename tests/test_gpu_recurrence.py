"""The gated recurrence and its gradient, against plain loops in 64 bits.

Tolerances.  With M_t = a M_(t-1) + b |u|, the sum of the magnitudes of everything that state t is made of, each part of it
has been through a multiplication by a (off by `off` at most, relatively, in fp32) and up to five roundings per step: two of
the step itself, one in the product of the steps that a map holds, two where maps are joined.  So an error E_t grows as
a (E + k M) + k b |u| with k = off + 5 * 2^-24.  a and b: the exponent's product is off by |gate| 2^-24 in bf16 gates and by
2^-24 in fp32 ones; the exponential, 1 + e and the reciprocal by another 2^-23 each."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import DEV, HALF_STEP, TORCH, addresses, f64, rows, stream, untouched, workspace
from test_gpu_layers import DTYPES, NAMES, close, dtype_id

pytestmark = pytest.mark.gpu

STEP, TINY = 2.0 ** -24, 2.0 ** -120          # TINY: what is lost of numbers next to the smallest


def factor(dtype, gate):
    largest = np.abs(gate).max() if gate.size else 0.0
    return (min(largest, 150.0) if dtype == cm.BF16 else 1.0) * STEP + 8 * STEP + 5 * STEP


def gates64(gate):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-gate)), 1.0 / (1.0 + np.exp(gate))


def scan64(gate, u, starts, before, k, states, after, off, off_after):
    """Fills states, after and how far fp32 may be off, for one worker; rows that belong to no sequence stay."""
    a, b = gates64(gate)
    for s in range(len(starts) - 1):
        h = before[s].copy()
        M, E = np.abs(h), np.zeros_like(h)
        for t in range(starts[s], starts[s + 1]):
            E = a[t] * (E + k * M) + k * b[t] * np.abs(u[t]) + TINY * (M + np.abs(u[t]))
            M = a[t] * M + b[t] * np.abs(u[t])
            h = a[t] * h + b[t] * u[t]
            states[t], off[t] = h, E
        after[s], off_after[s] = h, E


def back64(gate, u, starts, before, prior, ds, dafter, k):
    """dgate, dinput, dbefore and how far each may be off; NaN where a row belongs to no sequence."""
    a, b = gates64(gate)
    n, ch = gate.shape
    dg, du, off_g, off_u = (np.full((n, ch), np.nan) for _ in range(4))
    db, off_b = dafter.copy(), np.zeros_like(dafter)
    for s in range(len(starts) - 1):
        e, M, E = dafter[s].copy(), np.abs(dafter[s]), np.zeros(ch)
        for t in range(starts[s + 1] - 1, starts[s] - 1, -1):
            p = before[s] if t == starts[s] else prior[t - 1]
            e, M, E = e + ds[t], M + np.abs(ds[t]), E + STEP * (M + np.abs(ds[t]))
            du[t], off_u[t] = b[t] * e, b[t] * (E + k * M) + TINY * M
            dg[t] = a[t] * b[t] * e * (p - u[t])
            off_g[t] = a[t] * b[t] * (E + 2 * k * M) * (np.abs(p) + np.abs(u[t])) + TINY * M * (np.abs(p) + np.abs(u[t]))
            e, M, E = a[t] * e, a[t] * M, a[t] * (E + k * M) + TINY * M
        db[s], off_b[s] = e, E
    return dg, du, db, off_g, off_u, off_b


def cut(rng, n, s, kind):
    """Where s sequences of n tokens start."""
    if kind == "even":
        return [n * k // s for k in range(s + 1)]
    if kind == "steps":                                       # one token each
        return list(range(n + 1))
    if kind == "gaps":                                        # tokens in front and behind that belong to no sequence
        lo, hi = n // 5, n - n // 7
        return sorted(int(v) for v in rng.integers(lo, hi + 1, s + 1))
    if kind == "empty":                                       # many without tokens, more than 64 of them in one place
        return sorted([0] * 3 + [n // 3] * 70 + [n // 3 + 1] * 2 + [n] * 5 + [int(v) for v in rng.integers(0, n + 1, s)])
    return sorted([0, n] + [int(v) for v in rng.integers(0, n + 1, s - 1)])


CASES = [  # world, tokens, channels, sequences, kind, gap
    (1, 1, 1, 1, "even", 0), (2, 3, 2, 1, "even", 1), (1, 9, 3, 2, "even", 0), (3, 64, 5, 3, "random", 2), (2, 65, 127, 4, "gaps", 0),
    (1, 200, 128, 7, "random", 0), (2, 300, 129, 9, "empty", 1), (1, 77, 130, 77, "steps", 0), (20, 30, 33, 5, "random", 0),
    (64, 6, 7, 2, "random", 0), (1, 513, 300, 1, "even", 0), (1, 1500, 64, 1, "even", 0), (2, 1100, 40, 3, "random", 3),
    (1, 1300, 70, 90, "random", 0), (1, 700, 20, 300, "random", 0), (1, 1000, 17, 5, "gaps", 0), (1, 900, 1, 4, "random", 0),
    (1, 2000, 9, 20, "empty", 0), (2, 640, 24, 5, "even", 0), (1, 500, 12, 500, "steps", 0), (1, 70, 6, 63, "random", 0),
    (1, 130, 6, 64, "random", 0), (1, 600, 260, 5, "random", 0),
    # two tokens or less to a sequence
    (2, 65, 127, 60, "random", 1), (1, 100, 5, 90, "gaps", 2), (3, 64, 130, 9, "empty", 1), (1, 1024, 66, 600, "random", 0),
    (20, 40, 40, 40, "steps", 0), (1, 30, 1, 30, "random", 0), (64, 3, 256, 3, "steps", 0), (1, 2, 300, 1, "even", 0)]


def tokens_of(world, n):
    return [n if w == 0 else (0 if w == 1 else max(0, n - 3 * w)) for w in range(world)]


def make(rng, world, n, ch, sequences, kind):
    ns = tokens_of(world, n)
    starts = [cut(rng, m, min(sequences, max(m, 1)), kind) if m else [0] for m in ns]
    gate = [rng.standard_normal((m, ch)) * 2 + 1.5 for m in ns]
    for g in gate:
        if g.size:
            g[rng.random(g.shape) < 0.01] = 60.0               # channels that keep their state, and that let go of it
            g[rng.random(g.shape) < 0.01] = -60.0
    return ns, starts, gate


@pytest.mark.parametrize("carry", [False, True], ids=["from-zero", "carried"])
@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,ch,sequences,kind,gap", CASES)
def test_recurrence_and_its_gradient(world, n, ch, sequences, kind, gap, dtype, carry):
    print(f"case: recurrence world={world} n={n} channels={ch} {sequences} {kind} {NAMES[dtype]}", flush=True)
    rng = np.random.default_rng(n * ch)
    ns, starts, gate = make(rng, world, n, ch, sequences, kind)
    counts = [len(s) - 1 for s in starts]
    id_bytes, ids = (8, torch.int64) if n % 2 else (4, torch.int32)
    plan, pitch, spitch = cm.Plan(world, [1]), 2 * ch + gap, ch + 2 * gap
    t32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.float32)                # noqa: E731
    product = [rows(m, 2 * ch, pitch, dtype, torch.cat([t32(g), t32(rng.standard_normal((m, ch)))], 1)) for m, g in zip(ns, gate)]
    halves = lambda p: [v[0].data_ptr() for v in p], lambda p: [v[0].data_ptr() + ch * v[0].element_size() for v in p]   # noqa: E731
    st = [torch.tensor(s, dtype=ids, device=DEV) for s in starts]
    per = lambda scale: [t32(rng.standard_normal((c, ch)) * scale).to(DEV) for c in counts]     # noqa: E731
    before, dafter = per(0.5), per(0.1)
    after, dbefore = ([torch.full((c * ch + 3,), 9.0, device=DEV) for c in counts] for _ in range(2))
    states = [rows(m, ch, spitch, dtype, fill=7.0) for m in ns]
    dstates = [rows(m, ch, spitch, dtype, t32(rng.standard_normal((m, ch)) * 0.1)) for m in ns]
    dproduct = [rows(m, 2 * ch, pitch, dtype, fill=7.0) for m in ns]
    need = plan.recurrence_workspace(ch, ns)
    kept = []
    for again in range(2):
        ws = workspace(need)
        ws[:need] = 0x5A if again else 0xFF
        plan.recurrence(ch, ns, counts, addresses(st), halves[0](product), halves[1](product), addresses([v[0] for v in states]),
                        ws.data_ptr(), need, before=addresses(before) if carry else None, after=addresses(after) if carry else None,
                        id_bytes=id_bytes, dtype=dtype, pitch=pitch, states_pitch=spitch, stream=stream())
        ws2 = workspace(need)
        plan.recurrence_gradient(ch, ns, counts, addresses(st), halves[0](product), halves[1](product), addresses([v[0] for v in states]),
                                 addresses([v[0] for v in dstates]), halves[0](dproduct), halves[1](dproduct), ws2.data_ptr(), need,
                                 before=addresses(before) if carry else None, dafter=addresses(dafter) if carry else None,
                                 dbefore=addresses(dbefore) if carry else None, id_bytes=id_bytes, dtype=dtype, pitch=pitch,
                                 states_pitch=spitch, stream=stream())
        torch.cuda.synchronize()
        assert untouched(ws, need) and untouched(ws2, need)
        kept.append([t.clone() for t in [v[0] for v in states + dproduct] + after + dbefore])
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*kept)), "not reproducible"
    half = HALF_STEP[dtype]
    for w, m in enumerate(ns):
        if not m:
            assert bool((after[w] == 9.0).all()) and bool((dbefore[w] == 9.0).all())
            continue
        p = f64(product[w][1])
        g, u, k = p[:, :ch], p[:, ch:], factor(dtype, p[:, :ch])
        zero = np.zeros((counts[w], ch))
        b0, da = (f64(before[w]), f64(dafter[w])) if carry else (zero, zero)
        want, off = np.full((m, ch), 7.0), np.zeros((m, ch))
        end, off_end = zero.copy(), zero.copy()
        scan64(g, u, starts[w], b0, k, want, end, off, off_end)
        close(f64(states[w][1]), want, off + half * (np.abs(want) + off) * (off > 0) + 1e-30, f"worker {w}: states")
        dg, du, db, off_g, off_u, off_b = back64(g, u, starts[w], b0, f64(states[w][1]), f64(dstates[w][1]), da, k)
        got = f64(dproduct[w][1])
        for part, ref, bound in ((got[:, :ch], dg, off_g), (got[:, ch:], du, off_u)):
            nowhere = np.isnan(ref)
            assert (part[nowhere] == 7.0).all(), "tokens of no sequence"
            close(part[~nowhere], ref[~nowhere], (bound + half * (np.abs(ref) + bound) + 1e-30)[~nowhere], f"worker {w}: gradient")
        if carry:
            # STEP: stored in fp32, equal where nothing was added
            close(f64(after[w][:counts[w] * ch]).reshape(-1, ch), end, off_end + STEP * (np.abs(end) + off_end) + 1e-30, "after")
            close(f64(dbefore[w][:counts[w] * ch]).reshape(-1, ch), db, off_b + STEP * (np.abs(db) + off_b) + 1e-30, "dbefore")
        c = counts[w] * ch if carry else 0
        assert bool((after[w][c:] == 9.0).all()) and bool((dbefore[w][c:] == 9.0).all())
        for mem, view in (states[w], dproduct[w]):
            view.fill_(7.0)
            assert bool((mem == 7.0).all()), "the gaps between the rows and what lies behind the last one stay"
    plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("n,ch", [(300, 70), (3000, 70)])
def test_nothing_leaves_its_sequence(n, ch, dtype):
    """Infinities and NaN in one sequence, in tokens of none, and in the states: the other sequences' results stay the same to the bit."""
    rng = np.random.default_rng(n)
    starts = [5, 40, n // 3, n // 3, n // 2 + 1, n - 9]
    plan, S = cm.Plan(1, [1]), 5
    st = torch.tensor(starts, device=DEV)
    clean = torch.tensor(rng.standard_normal((n, 2 * ch))).to(TORCH[dtype])
    ds, before, dafter = torch.tensor(rng.standard_normal((n, ch))).to(TORCH[dtype]), torch.randn(S, ch), torch.randn(S, ch)
    bad_rows = torch.zeros(n, dtype=torch.bool)
    bad_rows[:5] = bad_rows[40:n // 3] = bad_rows[n - 9:] = True
    results = []
    for spoiled in (False, True):
        x, d, b, a = clean.clone(), ds.clone(), before.clone(), dafter.clone()
        if spoiled:
            x[:5], x[n - 9:], d[:5], d[n - 9:] = float("nan"), float("inf"), float("nan"), float("nan")
            x[40, ch:], x[n // 3 - 1, ch:] = float("inf"), float("nan")
            x[44, :ch], d[n // 3 - 2], d[41] = float("nan"), float("inf"), float("-inf")
            b[1], a[1] = float("nan"), float("inf")
        x, d, b, a = (t.to(DEV) for t in (x, d, b, a))
        out, dx = torch.full((n, ch), 7.0, dtype=TORCH[dtype], device=DEV), torch.full((n, 2 * ch), 7.0, dtype=TORCH[dtype], device=DEV)
        end, db = torch.empty(S, ch, device=DEV), torch.empty(S, ch, device=DEV)
        need = plan.recurrence_workspace(ch, [n])
        ws = workspace(need)
        lo, hi = [x.data_ptr()], [x.data_ptr() + ch * x.element_size()]
        plan.recurrence(ch, [n], [S], [st.data_ptr()], lo, hi, [out.data_ptr()], ws.data_ptr(), need, before=[b.data_ptr()],
                        after=[end.data_ptr()], dtype=dtype, pitch=2 * ch, stream=stream())
        plan.recurrence_gradient(ch, [n], [S], [st.data_ptr()], lo, hi, [out.data_ptr()], [d.data_ptr()], [dx.data_ptr()],
                                 [dx.data_ptr() + ch * dx.element_size()], ws.data_ptr(), need, before=[b.data_ptr()],
                                 dafter=[a.data_ptr()], dbefore=[db.data_ptr()], dtype=dtype, pitch=2 * ch, stream=stream())
        torch.cuda.synchronize()
        results.append([t.cpu() for t in (out, dx, end, db)])
    (o0, x0, e0, b0), (o1, x1, e1, b1) = results
    assert torch.equal(o0[~bad_rows], o1[~bad_rows]) and torch.equal(x0[~bad_rows], x1[~bad_rows])
    others = [0, 2, 3, 4]
    assert torch.equal(e0[others], e1[others]) and torch.equal(b0[others], b1[others])
    assert bool(torch.isfinite(o0.float()).all()) and bool(o1[40:n // 3].isnan().all())
    plan.close()


@pytest.mark.parametrize("n,ch", [(100, 30), (2500, 30)])
def test_starts_that_are_none(n, ch):
    """Out of range and out of order: the outputs are unspecified, but nothing outside them is written."""
    plan = cm.Plan(1, [1])
    for k, (ids, starts) in enumerate([(torch.int64, [-(1 << 62), 5, 1 << 62, 7, -1]), (torch.int32, [n, 40, 3, 0, n // 2]),
                                       (torch.int32, [-5] * 40 + [n + 9] * 40 + [3, 2, 1] * 20), (torch.int64, [n // 2] * 200)]):
        print("case: starts", k, flush=True)
        S = len(starts) - 1
        st = torch.tensor(starts, dtype=ids, device=DEV)
        x, ds = torch.randn(n, 2 * ch, device=DEV), torch.randn(n, ch, device=DEV)
        before = torch.randn(S, ch, device=DEV)
        out, dx = torch.full((n + 2, ch), 7.0, device=DEV), torch.full((n + 2, 2 * ch), 7.0, device=DEV)
        end, db = torch.full((S + 2, ch), 7.0, device=DEV), torch.full((S + 2, ch), 7.0, device=DEV)
        need = plan.recurrence_workspace(ch, [n])
        ws = workspace(need)
        at = lambda t, rows=1: [t.data_ptr() + rows * t.shape[1] * 4]                # noqa: E731
        ib = 8 if ids == torch.int64 else 4
        lo, hi = [x.data_ptr()], [x.data_ptr() + ch * 4]
        plan.recurrence(ch, [n], [S], [st.data_ptr()], lo, hi, at(out), ws.data_ptr(), need, before=[before.data_ptr()], after=at(end),
                        id_bytes=ib, pitch=2 * ch, stream=stream())
        plan.recurrence_gradient(ch, [n], [S], [st.data_ptr()], lo, hi, at(out), [ds.data_ptr()], at(dx),
                                 [at(dx)[0] + ch * 4], ws.data_ptr(), need, before=[before.data_ptr()], dafter=[before.data_ptr()],
                                 dbefore=at(db), id_bytes=ib, pitch=2 * ch, stream=stream())
        torch.cuda.synchronize()
        assert untouched(ws, need)
        assert all(bool((t[i] == 7.0).all()) for t in (out, dx, end, db) for i in (0, -1))
    plan.close()


def test_recurrence_gradient_agrees_with_differences():
    """Of <ds, states> + <dafter, after>, in 64 bits, along directions of gates, inputs and states before."""
    rng = np.random.default_rng(8)
    n, ch, starts, h = 90, 11, [0, 30, 30, 61, 90], 1e-6
    S = len(starts) - 1
    x, ds, b, da = (torch.tensor(rng.standard_normal(s), dtype=torch.float32) for s in ((n, 2 * ch), (n, ch), (S, ch), (S, ch)))
    d = [t.to(DEV) for t in (x, ds, b, da)]
    st = torch.tensor(starts, device=DEV)
    out, dx, end, db = (torch.empty(s, device=DEV) for s in ((n, ch), (n, 2 * ch), (S, ch), (S, ch)))
    plan = cm.Plan(1, [1])
    need = plan.recurrence_workspace(ch, [n])
    ws = workspace(need)
    lo, hi = [d[0].data_ptr()], [d[0].data_ptr() + ch * 4]
    plan.recurrence(ch, [n], [S], [st.data_ptr()], lo, hi, [out.data_ptr()], ws.data_ptr(), need, before=[d[2].data_ptr()],
                    after=[end.data_ptr()], pitch=2 * ch, stream=stream())
    plan.recurrence_gradient(ch, [n], [S], [st.data_ptr()], lo, hi, [out.data_ptr()], [d[1].data_ptr()], [dx.data_ptr()],
                             [dx.data_ptr() + ch * 4], ws.data_ptr(), need, before=[d[2].data_ptr()], dafter=[d[3].data_ptr()],
                             dbefore=[db.data_ptr()], pitch=2 * ch, stream=stream())
    torch.cuda.synchronize()
    x, ds, b, da = (f64(t) for t in (x, ds, b, da))

    def value(x, b):
        s, e, o = np.zeros((n, ch)), np.zeros((S, ch)), np.zeros((n, ch))
        scan64(x[:, :ch], x[:, ch:], starts, b, 0.0, s, e, o, np.zeros((S, ch)))
        return (ds * s).sum() + (da * e).sum()

    k = factor(cm.F32, x[:, :ch])
    *_, off_g, off_u, off_b = back64(x[:, :ch], x[:, ch:], starts, b, f64(out), ds, da, k)
    # the stored states that the gradient reads are themselves off
    off_s = np.zeros((n + 1, ch))
    scan64(x[:, :ch], x[:, ch:], starts, b, k, np.zeros((n, ch)), np.zeros((S, ch)), off_s[1:], np.zeros((S, ch)))
    off_s[1:] += STEP * (np.abs(f64(out)) + off_s[1:])
    off = np.concatenate([off_g + off_s[:-1] * np.abs(f64(dx)[:, ch:]), off_u], 1)
    for _ in range(3):
        p, q = rng.standard_normal((n, 2 * ch)), rng.standard_normal((S, ch))
        want = (value(x + h * p, b + h * q) - value(x - h * p, b - h * q)) / (2 * h)
        got = (f64(dx) * p).sum() + (f64(db) * q).sum()
        assert abs(got - want) <= (off * np.abs(p)).sum() + (off_b * np.abs(q)).sum() + 1e-8 * (np.abs(ds).sum() + np.abs(da).sum())
    plan.close()


@pytest.mark.parametrize("n", [9, 40, 3000])
def test_recurrence_calls_captured_into_a_graph(n):
    """Replayed three times, with new inputs and starts and eager calls of the same buffers in between."""
    ch, S, W = 33, 6, 2
    plan = cm.Plan(W, [1], dtype=cm.BF16)
    new = lambda *s: [torch.empty(*s, dtype=torch.bfloat16, device=DEV) for _ in range(W)]                   # noqa: E731
    new32 = lambda: [torch.empty(S, ch, device=DEV) for _ in range(W)]                                        # noqa: E731
    x, dx, out, ds, before, after, dafter, dbefore = new(n, 2 * ch), new(n, 2 * ch), new(n, ch), new(n, ch), new32(), new32(), new32(), new32()
    st = [torch.zeros(S + 1, dtype=torch.int32, device=DEV) for _ in range(W)]
    need = plan.recurrence_workspace(ch, [n] * W)
    ws = workspace(need)
    second = lambda p: [t.data_ptr() + 2 * ch for t in p]                                                     # noqa: E731

    def step():
        plan.recurrence(ch, [n] * W, [S] * W, addresses(st), addresses(x), second(x), addresses(out), ws.data_ptr(), need,
                        before=addresses(before), after=addresses(after), id_bytes=4, pitch=2 * ch, stream=stream())
        plan.recurrence_gradient(ch, [n] * W, [S] * W, addresses(st), addresses(x), second(x), addresses(out), addresses(ds),
                                 addresses(dx), second(dx), ws.data_ptr(), need, before=addresses(before), dafter=addresses(dafter),
                                 dbefore=addresses(dbefore), id_bytes=4, pitch=2 * ch, stream=stream())

    def outputs():
        torch.cuda.synchronize()
        return [t.clone() for t in out + dx + after + dbefore]

    def fill(seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        for t in x + ds + before + dafter:
            t.copy_(torch.randn(t.shape, device=DEV, generator=g))
        for t in st:
            t.copy_(torch.randint(0, n + 1, (S + 1,), device=DEV, generator=g).sort().values)
        for t in out + dx + after + dbefore + [ws]:
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
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    plan.close()


def test_recurrence_rows_more_than_four_gib_apart():
    """The last of 300 rows, 2^23 elements apart, is behind 2^32 bytes, and behind 2^31 elements; some channels of a long cache of states."""
    n, ch, pitch = 300, 16, 1 << 23
    free, _ = torch.cuda.mem_get_info()
    if free < 2 * 2 * n * pitch + (4 << 30):
        pytest.skip("not enough memory")
    x, out = (torch.empty(n * pitch, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    view = lambda t, c: t.view(n, pitch)[:, :c]                                       # noqa: E731
    values = torch.randn(n, 2 * ch).to(torch.bfloat16)
    view(x, 2 * ch).copy_(values)
    plan, S = cm.Plan(1, [1]), 300000
    starts = torch.zeros(S + 1, dtype=torch.int64, device=DEV)                        # the last sequence alone has tokens
    starts[S] = n
    before = torch.randn(S, 1, device=DEV).expand(S, ch).contiguous()
    after = torch.empty(S, ch, device=DEV)
    need = plan.recurrence_workspace(ch, [n])
    ws = workspace(need)
    plan.recurrence(ch, [n], [S], [starts.data_ptr()], [x.data_ptr()], [x.data_ptr() + 2 * ch], [out.data_ptr()], ws.data_ptr(), need,
                    before=[before.data_ptr()], after=[after.data_ptr()], dtype=cm.BF16, pitch=pitch, states_pitch=pitch,
                    stream=stream())
    torch.cuda.synchronize()
    v = f64(values)
    k = factor(cm.BF16, v[:, :ch])
    want, off, end, off_end = np.zeros((n, ch)), np.zeros((n, ch)), np.zeros((1, ch)), np.zeros((1, ch))
    scan64(v[:, :ch], v[:, ch:], [0, n], f64(before[-1:]), k, want, end, off, off_end)
    close(f64(view(out, ch)), want, off + HALF_STEP[cm.BF16] * (np.abs(want) + off))
    close(f64(after[-1:]), end, off_end + STEP * np.abs(end))
    assert torch.equal(after[:-1], before[:-1])
    plan.close()
