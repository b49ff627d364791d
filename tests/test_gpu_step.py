"""A training step from token ids to aggregated gradients: lookup, norm with an 8-bit copy, dense layer, recurrence, norm, logits,
distillation, and all of it backwards, for several workers.

Every operator's outputs are checked against its formulas in 64 bits on the inputs that it had in the step, with the tolerances of its
own test, so that what passes between them (types, pitches, halves of a product, checkpoints, places in the plan) is checked and
nothing has to be said of how errors grow from one to the next.  The products between them are torch's.  The last test goes the
other way: derivatives through all of them, against differences of losses."""
import numpy as np
import pytest
import torch

import oracle
import paper_2004_14020_amd as cm

from gpu_util import assert_same_bits
from layer_util import DEV, HALF_STEP, TORCH, addresses, decode, embedding_gradient, encode, f64, image, stream, untouched, workspace
from test_gpu_distillation import formulas
from test_gpu_layers import DTYPES, close, dtype_id
from test_gpu_norm import STEP, gradient64, norm64, same
from test_gpu_recurrence import back64, factor, scan64

pytestmark = pytest.mark.gpu

EPS, SCALE, T, SOFT, HARD = 1e-5, 4.0, 2.0, 1.0, 0.5
GAIN1, WEIGHT1, BIAS1, GAIN2, WEIGHT2, TABLE = range(6)


class Step:
    def __init__(self, dtype, world=3, n=70, sequences=4, vocab=333, width=72, channels=40, top=5):
        self.dtype, self.world, self.vocab, self.width, self.ch, self.top = dtype, world, vocab, width, channels, top
        self.ns = [max(0, n - 9 * w) for w in range(world)]
        self.sequences = [min(sequences, m) for m in self.ns]
        self.mean = 1.0 / max(1, sum(self.ns))
        elems = [width, width * 2 * channels, 2 * channels, channels, channels * vocab, vocab * width]
        self.plan = cm.Plan(world, elems, dtype=dtype, batch_threshold_bytes=1 << 14)
        t = TORCH[dtype]
        make = lambda *cols: [torch.zeros(m, *cols, dtype=t, device=DEV) for m in self.ns]                  # noqa: E731
        fp32 = lambda: [torch.zeros(m, device=DEV) for m in self.ns]                                     # noqa: E731
        ints = lambda *cols: [torch.zeros(m, *cols, dtype=torch.int64, device=DEV) for m in self.ns]     # noqa: E731
        saved = lambda k: [torch.zeros(cm.checkpoint_bytes(m, k), dtype=torch.uint8, device=DEV) for m in self.ns]   # noqa: E731
        self.params = [torch.zeros(e, dtype=t, device=DEV) for e in elems]
        self.w1t, self.w2t = torch.zeros(2 * channels, width, dtype=t, device=DEV), torch.zeros(vocab, channels, dtype=t, device=DEV)
        self.grads = [[torch.zeros(e, dtype=t, device=DEV) for e in elems] for _ in range(world)]
        self.plan.bind([addresses(r) for r in self.grads], None)
        self.ids, self.labels, self.teacher_ids, self.teacher = ints(), ints(), ints(top), make(top)
        self.starts = [torch.zeros(s + 1, dtype=torch.int64, device=DEV) for s in self.sequences]
        self.x, self.res, self.sum, self.y1, self.rstd1, self.saved1 = make(width), make(width), make(width), make(width), fp32(), saved(width)
        self.product, self.states, self.y2, self.rstd2, self.saved2 = make(2 * channels), make(channels), make(channels), fp32(), saved(channels)
        self.logits, self.loss, self.dlogits = make(vocab), fp32(), make(vocab)
        self.dy2, self.dstates, self.dproduct, self.dy1, self.dsum = make(channels), make(channels), make(2 * channels), make(width), make(width)
        self.local = [[torch.zeros_like(g) for g in row] for row in self.grads]                           # before they are added up
        p, ns = self.plan, self.ns
        self.need = dict(norm1=p.residual_norm_workspace(GAIN1, ns), norm2=p.residual_norm_workspace(GAIN2, ns),
                         rec=p.recurrence_workspace(channels, ns), loss=p.distillation_workspace(vocab, top, ns),
                         weight1=p.weight_gradient_workspace(WEIGHT1, width, ns), weight2=p.weight_gradient_workspace(WEIGHT2, channels, ns),
                         table=p.embedding_workspace(TABLE, width, ns))
        self.ws = {k: workspace(b) for k, b in self.need.items()}

    def matrix(self, t, rows):
        return self.params[t].view(rows, -1)

    def transposed(self):
        """Of the weights, for the products of the backward pass (in place: a graph has their addresses)."""
        self.w1t.copy_(self.matrix(WEIGHT1, self.width).t())
        self.w2t.copy_(self.matrix(WEIGHT2, self.ch).t())

    def fill(self, seed):
        g, t = torch.Generator().manual_seed(seed), TORCH[self.dtype]
        size = {GAIN1: 0.0, GAIN2: 0.0, WEIGHT1: self.width ** -0.5, WEIGHT2: self.ch ** -0.5, BIAS1: 0.5, TABLE: 0.25}
        for i, v in enumerate(self.params):
            r = torch.randn(v.shape, generator=g)
            v.copy_((r * size[i] if size[i] else 1 + 0.1 * r).to(t))
        for w, m in enumerate(self.ns):
            self.ids[w].copy_(torch.randint(-1, self.vocab, (m,), generator=g))
            self.labels[w].copy_(torch.randint(-1, self.vocab, (m,), generator=g))
            self.teacher_ids[w].copy_(torch.randint(-1, self.vocab, (m, self.top), generator=g))
            self.teacher[w].copy_(torch.randn(m, self.top, generator=g) * 2)
            self.res[w].copy_(torch.randn(m, self.width, generator=g) * 0.5)
            cuts = torch.sort(torch.randint(0, m + 1, (max(0, self.sequences[w] - 1),), generator=g)).values.tolist()
            self.starts[w].copy_(torch.tensor([0, *cuts, m] if self.sequences[w] else [0]))
        self.transposed()
        for row in self.grads:
            for v in row:
                v.fill_(float("nan"))
        for ws in self.ws.values():
            ws.fill_(0xFF)
        torch.cuda.synchronize()

    def halves(self, p):
        return addresses(p), [v.data_ptr() + self.ch * v.element_size() for v in p]

    def work(self, name):
        return self.ws[name].data_ptr(), self.need[name]

    def forward(self, s):
        p, ns, one = self.plan, self.ns, lambda t: [self.params[t].data_ptr()] * self.world
        p.embedding_lookup(one(TABLE), self.vocab, self.width, addresses(self.ids), ns, addresses(self.x), scale=SCALE, stream=s)
        p.residual_norm(one(GAIN1), self.width, ns, addresses(self.x), addresses(self.y1), addresses(self.rstd1), eps=EPS,
                        residual=addresses(self.res), sum=addresses(self.sum), checkpoint=addresses(self.saved1), stream=s)
        for y, out in zip(self.y1, self.product):
            torch.addmm(self.params[BIAS1], y, self.matrix(WEIGHT1, self.width), out=out)
        p.recurrence(self.ch, ns, self.sequences, addresses(self.starts), *self.halves(self.product), addresses(self.states),
                     *self.work("rec"), pitch=2 * self.ch, stream=s)
        p.residual_norm(one(GAIN2), self.ch, ns, addresses(self.states), addresses(self.y2), addresses(self.rstd2), eps=EPS,
                        checkpoint=addresses(self.saved2), stream=s)
        for y, out in zip(self.y2, self.logits):
            torch.mm(y, self.matrix(WEIGHT2, self.ch), out=out)
        p.distillation(self.vocab, ns, addresses(self.logits), addresses(self.teacher_ids), addresses(self.teacher), self.top,
                       addresses(self.loss), *self.work("loss"), labels=addresses(self.labels), dlogits=addresses(self.dlogits),
                       temperature=T, soft=SOFT, hard=HARD, scale=self.mean, stream=s)

    def backward(self, s):
        p, ns, one = self.plan, self.ns, lambda t: [self.params[t].data_ptr()] * self.world
        p.weight_gradient(WEIGHT2, None, addresses(self.saved2), ns, self.ch, addresses(self.dlogits), *self.work("weight2"), stream=s)
        for d, out in zip(self.dlogits, self.dy2):
            torch.mm(d, self.w2t, out=out)
        p.residual_norm_gradient(GAIN2, one(GAIN2), ns, addresses(self.states), addresses(self.rstd2), addresses(self.dy2),
                                 addresses(self.dstates), *self.work("norm2"), stream=s)
        p.recurrence_gradient(self.ch, ns, self.sequences, addresses(self.starts), *self.halves(self.product), addresses(self.states),
                              addresses(self.dstates), *self.halves(self.dproduct), *self.work("rec"), pitch=2 * self.ch, stream=s)
        p.weight_gradient(WEIGHT1, BIAS1, addresses(self.saved1), ns, self.width, addresses(self.dproduct), *self.work("weight1"), stream=s)
        for d, out in zip(self.dproduct, self.dy1):
            torch.mm(d, self.w1t, out=out)
        p.residual_norm_gradient(GAIN1, one(GAIN1), ns, addresses(self.sum), addresses(self.rstd1), addresses(self.dy1),
                                 addresses(self.dsum), *self.work("norm1"), stream=s)
        p.embedding_gradient(TABLE, self.width, addresses(self.ids), ns, addresses(self.dsum), *self.work("table"), scale=SCALE, stream=s)

    def run(self, s):
        self.forward(s)
        self.backward(s)
        for kept, row in zip(self.local, self.grads):
            for k, g in zip(kept, row):
                k.copy_(g)
        self.plan.allreduce(s)

    def outputs(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.loss + self.dlogits + self.dsum + [g for row in self.local + self.grads for g in row]]

    def check(self, what):
        torch.cuda.synchronize()
        assert all(untouched(self.ws[k], self.need[k]) for k in self.ws), what
        half = HALF_STEP[self.dtype]
        typed = lambda want, off: off + half * (np.abs(want) + off) + 1e-30                              # noqa: E731
        gain1, gain2 = f64(self.params[GAIN1]), f64(self.params[GAIN2])
        for w, m in enumerate(self.ns):
            if not m:
                continue
            at = f"{what}, worker {w}: "
            h = f64((self.x[w].float() + self.res[w].float()).to(TORCH[self.dtype]))
            assert np.array_equal(f64(self.sum[w]), h), at + "sum"
            for x, gain, rstd, y, saved, name in ((h, gain1, self.rstd1[w], self.y1[w], self.saved1[w], "norm 1"),
                                                  (f64(self.states[w]), gain2, self.rstd2[w], self.y2[w], self.saved2[w], "norm 2")):
                want, r = norm64(x, gain, float(np.float32(EPS)))
                close(f64(rstd), r, (STEP + (x.shape[1] + 8) * 2.0 ** -52) * r, at + name)
                close(f64(y), want, typed(want, 4 * STEP * np.abs(want)), at + name)                     # r, and two products
                codes, scales = encode(f64(y))
                whole = codes.size + scales.size
                assert np.array_equal(saved.cpu().numpy()[:whole], image(codes, scales)[:whole]), at + name + ": checkpoint"
            p, ch = f64(self.product[w]), self.ch
            gate, u, k = p[:, :ch], p[:, ch:], factor(self.dtype, p[:, :ch])
            starts, zero = self.starts[w].tolist(), np.zeros((self.sequences[w], ch))
            want, off = np.zeros((m, ch)), np.zeros((m, ch))
            scan64(gate, u, starts, zero, k, want, zero.copy(), off, zero.copy())
            close(f64(self.states[w]), want, typed(want, off), at + "states")
            dg, du, _, off_g, off_u, _ = back64(gate, u, starts, zero, f64(self.states[w]), f64(self.dstates[w]), zero, k)
            close(f64(self.dproduct[w]), np.hstack([dg, du]), typed(np.hstack([dg, du]), np.hstack([off_g, off_u])), at + "dproduct")
            loss, dz, off_loss, off = formulas(f64(self.logits[w]), self.teacher_ids[w].cpu().numpy(), f64(self.teacher[w]),
                                               self.labels[w].cpu().numpy(), T, SOFT, HARD, float(np.float32(self.mean)), self.vocab, True)
            close(f64(self.loss[w]), loss, off_loss, at + "loss")
            close(f64(self.dlogits[w]), dz, typed(dz, off), at + "dlogits")
            local = [f64(g) for g in self.local[w]]
            for x, gain, rstd, dy, dx, t, name in ((f64(self.states[w]), gain2, self.rstd2[w], self.dy2[w], self.dstates[w], GAIN2, "norm 2"),
                                                   (h, gain1, self.rstd1[w], self.dy1[w], self.dsum[w], GAIN1, "norm 1")):
                want, dgain, off, off_g = gradient64(x, gain, f64(rstd), f64(dy), np.zeros_like(x))
                close(f64(dx), want, typed(want, off), at + name + ": dx")
                close(local[t], dgain, typed(dgain, off_g + STEP * np.abs(dgain)), at + name + ": dgain")
            for y, dy, t, b in ((self.y2[w], self.dlogits[w], WEIGHT2, None), (self.y1[w], self.dproduct[w], WEIGHT1, BIAS1)):
                x, d = decode(*encode(f64(y)), m), f64(dy)
                terms = (m * (1 if self.dtype == cm.BF16 else 3) + 2) * 2.0 ** -23 * (1 + 2.0 ** -6)
                want = x.T @ d
                close(local[t].reshape(want.shape), want, typed(want, terms * (np.abs(x).T @ np.abs(d))), at + "weight")
                if b is not None:
                    close(local[b], d.sum(0), typed(d.sum(0), terms * np.abs(d).sum(0)), at + "bias")
            want, mag, n = embedding_gradient(self.vocab, self.ids[w].tolist(), f64(self.dsum[w]), SCALE)
            close(local[TABLE].reshape(want.shape), want, typed(want, (n + 2) * STEP * (1 + 2.0 ** -10) * mag), at + "table")
        raw, kind = (torch.float32, np.float32) if self.dtype == cm.F32 else (torch.int16, np.uint16)
        host = lambda rows: [[g.view(raw).cpu().numpy().view(kind).copy() for g in row] for row in rows]  # noqa: E731
        ref = host(self.local)
        cfg = oracle.Config(self.world, self.dtype, 1 << 14, oracle.SPLIT_NONE, 8, 0, 16, 2)
        oracle.allreduce(oracle.build_plan(cfg, self.plan.elems), ref)
        assert_same_bits(host(self.grads), ref, what)


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
@pytest.mark.parametrize("world,n,sequences", [(3, 70, 4), (1, 1, 1), (2, 9, 9), (8, 600, 3)])
def test_a_step(world, n, sequences, dtype):
    """Also with a worker that has no token, with one token in all, and with sequences of one token."""
    print(f"case: step world={world} n={n} sequences={sequences} dtype={dtype}", flush=True)
    step = Step(dtype, world, n, sequences)
    for seed in (1, 2):
        step.fill(seed)
        step.run(stream())
        step.check(f"seed {seed}")
    step.plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_a_step_on_another_stream(dtype):
    step, side = Step(dtype), torch.cuda.Stream()
    step.fill(3)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run(side.cuda_stream)
    side.synchronize()
    step.check("side stream")
    step.plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_two_steps_on_two_streams_at_once(dtype):
    """Each with its own workspaces, so neither sees the other."""
    steps, sides = [Step(dtype, n=2000), Step(dtype, n=1900, channels=56)], [torch.cuda.Stream() for _ in range(2)]
    for k, (s, side) in enumerate(zip(steps, sides)):
        s.fill(k)
        s.run(stream())
    want = [s.outputs() for s in steps]
    for k, (s, side) in enumerate(zip(steps, sides)):
        s.fill(k)
        side.wait_stream(torch.cuda.current_stream())
    for s, side in zip(steps, sides):
        with torch.cuda.stream(side):
            s.run(side.cuda_stream)
    for s, w in zip(steps, want):
        assert all(same(a, b) for a, b in zip(s.outputs(), w))
        s.plan.close()


@pytest.mark.parametrize("dtype", DTYPES, ids=dtype_id)
def test_captured_steps_replay(dtype):
    """Two graphs, replayed in turn with new inputs, with eager steps between them."""
    steps = [Step(dtype), Step(dtype, n=90, sequences=2, channels=24)]
    graphs = []
    for s in steps:
        s.fill(0)
        s.run(stream())                                       # the library products' own first calls, outside the graph
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for seed in (4, 5, 6):
        for s, g in zip(steps, graphs):
            s.fill(seed)
            s.run(stream())
            want = s.outputs()
            s.fill(seed)
            g.replay()
            assert all(same(a, b) for a, b in zip(s.outputs(), want)), f"replay with seed {seed}"
            s.check(f"replay with seed {seed}")
    del graphs
    for s in steps:
        s.plan.close()


def test_the_gradient_agrees_with_differences():
    """Along two directions in the table, fp32, whose gradient no 8-bit copy has a part in: the chain of the operators' gradients against
    the central difference of the loss in 64 bits.  A term or factor that is missing anywhere shows in the first digit.  The chain is 14
    operators and products, whose sums have at most 333 terms in fp32: 14 * 340 * 2^-24 = 2^-11.8, relative to the magnitudes that are
    added, and 16 times that where they cancel.  The step of 2^-13 is off by 2^-26 of the third derivative, itself of the size
    of the first: 2^-20 allows for the factors in between."""
    step = Step(cm.F32, world=1, n=40, sequences=3)
    step.fill(9)
    rng = np.random.default_rng(1)
    direction = rng.standard_normal((step.vocab, step.width)) * 0.25
    p = [f64(v) for v in step.params]

    def loss(table):
        ids = step.ids[0].tolist()
        x = np.array([SCALE * table[i] if i >= 0 else np.zeros(step.width) for i in ids]) + f64(step.res[0])
        z = norm64(x, p[GAIN1], float(np.float32(EPS)))[0] @ p[WEIGHT1].reshape(step.width, -1) + p[BIAS1]
        ch, starts = step.ch, step.starts[0].tolist()
        states, zero = np.zeros((len(ids), ch)), np.zeros((len(starts) - 1, ch))
        scan64(z[:, :ch], z[:, ch:], starts, zero, 0.0, states, zero.copy(), np.zeros_like(states), zero.copy())
        logits = norm64(states, p[GAIN2], float(np.float32(EPS)))[0] @ p[WEIGHT2].reshape(ch, -1)
        return formulas(logits, step.teacher_ids[0].cpu().numpy(), f64(step.teacher[0]), step.labels[0].cpu().numpy(), T, SOFT, HARD, 1.0,
                        step.vocab, True)[0].sum() * step.mean

    step.run(stream())
    torch.cuda.synchronize()
    gradient, table, h = f64(step.local[0][TABLE]).reshape(step.vocab, -1), p[TABLE].reshape(step.vocab, -1), 2.0 ** -13
    # a direction at random, which most of the gradient is at right angles to, and the gradient's own
    for d in (direction, gradient * np.sqrt((direction ** 2).sum() / (gradient ** 2).sum())):
        got, want = (gradient * d).sum(), (loss(table + h * d) - loss(table - h * d)) / (2 * h)
        norm = np.sqrt((gradient ** 2).sum() * (d ** 2).sum())    # what the sum over the table may be off, by Cauchy and Schwarz
        assert abs(got - want) <= (2.0 ** -11.8 * 16 + 2.0 ** -20) * norm, (got, want, norm)
    step.plan.close()
