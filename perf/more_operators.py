"""The calls of a training step between the embedding and the gradients, as they are timed: the residual
norm and its gradient, the gated recurrence and its gradient, distillation from a teacher's top logits.

`run` computes each in elementary torch operations while `own` is False, and through the library
while it is True.  All W workers of a data-parallel program go through one call.  Their rows lie one
worker after the other in one array, so that the elementary operations run over all of them at once.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ES = {"f32": 4, "bf16": 2}
DEV = "cuda:0"
BLOCK = 32                     # tokens that share a scale in a checkpoint
EPS = 2.0 ** -17               # of the norm


def _case(op, world, tokens, cols, dtype="f32", ragged=False, params=None, residual=False, saved=False, sequences=1,
          carry=False, top=1, temperature=1.0, hard=0.0, gradient=True, pad=0.0, id_bytes=8, **name):
    """op        norm, ngrad, rec, rgrad or distill
    tokens    of the largest worker; ragged: the others have fewer, and sequences have different lengths
    cols      the norm's width, the recurrence's channels, the vocabulary
    dtype     of the rows; params: of the norm's gain and its gradient
    residual  norm: x is added to the residual stream; ngrad: the stream's gradient is added to dx
    saved     norm: also an 8-bit checkpoint of the result, which is read back as the backward pass does
    sequences of every worker; carry: states go in and come out, and so do their gradients
    top       teacher's entries per token; hard: weight of the labels; gradient: not only the loss; pad: share of
              the tokens at the end that are padding"""
    return dict(name, op=op, world=world, tokens=tokens, cols=cols, dtype=dtype, ragged=ragged, params=params or dtype,
                residual=residual, saved=saved, sequences=sequences, carry=carry, top=top, temperature=temperature, hard=hard,
                gradient=gradient, pad=pad, id_bytes=id_bytes)


def listed():
    return [
        # the norm before a dense layer of the Transformer encoder, whose input is kept in 8 bits; eight workers
        _case("norm", 8, 4096, 1024, "bf16", residual=True, saved=True, name="norm-encoder-bf16-w8"),
        # one token at each of two workers, as when a model is tried out: latency alone
        _case("norm", 2, 1, 1024, "f32", residual=True, name="norm-one-token-f32-w2"),
        # rows of the feed-forward product's width and one more, ragged, fp32
        _case("norm", 3, 1500, 4097, "f32", ragged=True, saved=True, name="norm-wide-odd-f32-w3"),
        # the encoder's norm backward, with the gradient that comes along the residual stream
        _case("ngrad", 8, 4096, 1024, "bf16", residual=True, name="ngrad-encoder-bf16-w8"),
        # an odd width, gains kept in fp32, ragged batches that fit the caches
        _case("ngrad", 4, 1000, 777, "bf16", ragged=True, params="f32", name="ngrad-odd-mixed-w4"),
        # the encoder's tokens mixed by the recurrence: eight sequences of 512 tokens at each of eight workers
        _case("rec", 8, 4096, 1024, "bf16", sequences=8, name="rec-encoder-bf16-w8"),
        # one more token of each of 48 running sequences, their states in and out: single tokens
        _case("rec", 2, 48, 1024, "f32", sequences=48, carry=True, id_bytes=4, name="rec-step-f32-w2"),
        # one worker, one long sequence: there is little beside the tokens to work on at once
        _case("rgrad", 1, 16384, 1000, "f32", carry=True, name="rgrad-long-f32-w1"),
        # the encoder's recurrence backward, sequences of different lengths
        _case("rgrad", 8, 4096, 1024, "bf16", ragged=True, sequences=24, id_bytes=4, name="rgrad-encoder-bf16-w8"),
        # a student of the Transformer's vocabulary learns from a teacher's 32 best logits and from labels
        _case("distill", 8, 512, 30522, "bf16", top=32, temperature=2.0, hard=0.5, pad=0.05, name="distill-encoder-bf16-w8"),
        # a handful of tokens: few rows, long ones
        _case("distill", 1, 3, 30522, "f32", top=8, hard=1.0, name="distill-few-f32-w1"),
        # a large odd vocabulary in fp32, ragged, from the teacher alone
        _case("distill", 2, 200, 129_999, "f32", ragged=True, top=64, temperature=3.0, id_bytes=4, name="distill-wide-f32-w2"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["norm", "norm", "ngrad", "ngrad", "rec", "rgrad", "distill", "distill"])
        world, dtype = rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice(["f32", "bf16"])
        c = dict(ragged=rng.random() < 0.5)
        if op in ("norm", "ngrad"):
            cols = rng.choice([_log(rng, 16, 8192), 8 * _log(rng, 2, 1024)])
            case = _case(op, world, _log(rng, 1, 16384), cols, dtype, params=rng.choice([None, None, "f32"]),
                         residual=rng.random() < 0.6, saved=op == "norm" and rng.random() < 0.6, **c)
        elif op in ("rec", "rgrad"):
            tokens = _log(rng, 1, 32768)
            sequences = tokens if tokens <= 1024 and rng.random() < 0.25 else _log(rng, 1, min(tokens, 64))
            cols = rng.choice([_log(rng, 16, 4096), 8 * _log(rng, 2, 512)])
            case = _case(op, world, tokens, cols, dtype, sequences=sequences, carry=rng.random() < 0.5,
                         id_bytes=rng.choice([4, 8]), **c)
        else:
            vocab = _log(rng, 200, 130_000)
            case = _case(op, world, _log(rng, 1, 4096), vocab, dtype, top=_log(rng, 1, 128),
                         temperature=rng.choice([1.0, 1.0, 2.0, 4.0, 0.7]), hard=rng.choice([0.0, 0.5, 1.0]),
                         gradient=rng.random() < 0.85, pad=rng.choice([0.0, 0.0, 0.2]), id_bytes=rng.choice([4, 8]), **c)
        if work(case)["bytes"] <= most:
            return case


def _tokens(case):
    """Tokens of every worker."""
    n = case["tokens"]
    return [max(1, n - (n * w) // (3 * case["world"])) if case["ragged"] else n for w in range(case["world"])]


def _sequences(case):
    """Sequences of every worker: no more than its tokens where each has one."""
    return [min(case["sequences"], n) for n in _tokens(case)]


def _starts(case):
    """Where the sequences of every worker start, and the end of the last one."""
    rng = random.Random(case["tokens"] * 64 + case["cols"])
    out = []
    for n, s in zip(_tokens(case), _sequences(case)):
        even = [n * k // s for k in range(s + 1)]
        out.append(sorted([0, n] + [rng.randint(0, n) for _ in range(s - 1)]) if case["ragged"] and s < n else even)
    return out


def _generator(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + what)
    return g


def _randn(shape, seed, what, size=1.0, dtype="f32"):
    return torch.randn(shape, device=DEV, generator=_generator(seed, what)).mul_(size).to(DT[dtype])


def _stream(case, seed):
    """The residual stream: features of different sizes, a few of them far larger than the rest."""
    n, k = sum(_tokens(case)), case["cols"]
    size = torch.exp(0.5 * _randn((k,), seed, 0))
    size = torch.where(_randn((k,), seed, 1) < -2.3, 20 * size, size)
    return _randn((n, k), seed, 2).mul_(size).to(DT[case["dtype"]])


def _gain(case, seed):
    return (1.0 + 0.1 * _randn((case["cols"],), seed, 3)).to(DT[case["params"]])


def _inputs(case, seed):
    """What the user's program has, all workers in one array."""
    n, k, dt = sum(_tokens(case)), case["cols"], case["dtype"]
    if case["op"] == "norm":
        d = {"x": _stream(case, seed), "gain": _gain(case, seed)}
        if case["residual"]:
            d["residual"], d["x"] = d["x"], _randn((n, k), seed, 4, 0.5, dt)
        return d
    if case["op"] == "ngrad":
        x = _stream(case, seed)
        d = {"x": x, "gain": _gain(case, seed), "rstd": _rstd(x), "dy": _randn((n, k), seed, 4, 1e-2, dt)}
        if case["residual"]:
            d["dsum"] = _randn((n, k), seed, 5, 1e-2, dt)
        return d
    if case["op"] in ("rec", "rgrad"):
        # a dense layer has made gates and inputs side by side; channels remember for a few to a few hundred tokens
        product = torch.randn(n, 2 * k, device=DEV, generator=_generator(seed, 2))
        product[:, :k] += 1.0 + 3.0 * torch.rand(k, device=DEV, generator=_generator(seed, 0))
        d = {"product": product.to(DT[dt]), "starts": _start_tensors(case)}
        if case["carry"]:
            d["before"] = _randn((sum(_sequences(case)), k), seed, 3, 0.3)
        if case["op"] == "rgrad":
            d["states"] = _scan(case, d)[0].to(DT[dt])
            d["dstates"] = _randn((n, k), seed, 4, 1e-2, dt)
            if case["carry"]:
                d["dafter"] = _randn((sum(_sequences(case)), k), seed, 5, 1e-2)
        return d
    top, ids = min(case["top"], k), torch.int64 if case["id_bytes"] == 8 else torch.int32
    common = -0.7 * torch.log(torch.arange(k, device=DEV) + 3.0)            # words are not equally frequent
    logits = _randn((n, k), seed, 0, 2.0).add_(common).to(DT[dt])
    teacher = _randn((n, k), seed, 1).add_(logits)
    best, named = teacher.topk(top, dim=1)
    rank = (torch.rand(n, device=DEV, generator=_generator(seed, 2)) ** 3 * top).long().clamp_(max=top - 1)
    label = named.gather(1, rank[:, None])[:, 0]
    other = torch.randint(0, k, (n,), device=DEV, generator=_generator(seed, 3))
    label = torch.where(torch.rand(n, device=DEV, generator=_generator(seed, 4)) < 0.2, other, label)
    padding = torch.cat([torch.arange(t, device=DEV) >= t - int(t * case["pad"]) for t in _tokens(case)])
    return {"logits": logits, "teacher_ids": torch.where(padding[:, None], -1, named).to(ids), "teacher": best.to(DT[dt]),
            "labels": torch.where(padding, -1, label).to(ids)}


def _start_tensors(case):
    dt = torch.int64 if case["id_bytes"] == 8 else torch.int32
    return [torch.tensor(s, dtype=dt, device=DEV) for s in _starts(case)]


def _rows(tensor, counts):
    """Every worker's rows of an array of all."""
    return list(torch.split(tensor, counts))


def prepare(case, seed):
    st = _inputs(case, seed)
    counts, W, n, k, dt = _tokens(case), case["world"], sum(_tokens(case)), case["cols"], DT[case["dtype"]]
    st["case"], st["tokens"], st["sequences"] = case, counts, _sequences(case)
    st["stream"] = torch.cuda.current_stream().cuda_stream
    blocks = [(t + BLOCK - 1) // BLOCK for t in counts]
    st["place"] = torch.cat([torch.arange(t, device=DEV) + BLOCK * sum(blocks[:w]) for w, t in enumerate(counts)])
    st["blocks"] = sum(blocks)
    if own:
        import paper_2004_14020_amd as cm
        code, new = {"f32": cm.F32, "bf16": cm.BF16}, lambda *s, dtype=dt: torch.empty(s, dtype=dtype, device=DEV)
        at = lambda t, c=counts: [r.data_ptr() for r in _rows(t, c)]        # noqa: E731
        plan = st["plan"] = cm.Plan(W, [k], dtype=code[case["params"]])
        st["dtype"] = code[case["dtype"]]
        a = st["at"] = {}
        ws = 0
        if case["op"] in ("norm", "ngrad"):
            st["gains"] = [st["gain"].clone() for _ in range(W)]            # every worker has its copy
            a["gain"] = [g.data_ptr() for g in st["gains"]]
            a |= {key: at(st[key]) for key in ("x", "residual", "dy", "dsum") if key in st}
            st["rstd"] = st.get("rstd", new(n, dtype=torch.float32))
            a["rstd"] = at(st["rstd"])
        if case["op"] == "norm":
            st["out"] = {key: new(n, k) for key in (["sum"] if case["residual"] else []) + ["y"]}
            if case["saved"]:
                st["bytes"] = [new(cm.checkpoint_bytes(t, k), dtype=torch.uint8) for t in counts]
                a["checkpoint"] = [b.data_ptr() for b in st["bytes"]]
                st["out"]["saved"] = new(n, k, dtype=torch.bfloat16)        # what is kept in 8 bits is exact in bf16
        elif case["op"] == "ngrad":
            st["grad"] = [new(k, dtype=DT[case["params"]]) for _ in range(W)]
            plan.bind([[g.data_ptr()] for g in st["grad"]], None)
            st["out"] = {"dx": new(n, k)}
            ws = plan.residual_norm_workspace(0, counts)
        elif case["op"] in ("rec", "rgrad"):
            a["starts"] = [s.data_ptr() for s in st["starts"]]
            a["gate"], a["input"] = at(st["product"]), at(st["product"][:, k:])
            a |= {key: at(st[key], st["sequences"]) for key in ("before", "dafter") if key in st}
            per_sequence = lambda: new(sum(st["sequences"]), k, dtype=torch.float32)    # noqa: E731
            if case["op"] == "rec":
                st["out"] = {"states": new(n, k)} | ({"after": per_sequence()} if case["carry"] else {})
            else:
                a |= {"states": at(st["states"]), "dstates": at(st["dstates"])}
                st["out"] = {"dproduct": new(n, 2 * k)} | ({"dbefore": per_sequence()} if case["carry"] else {})
                a["dgate"], a["dinput"] = at(st["out"]["dproduct"]), at(st["out"]["dproduct"][:, k:])
            a |= {key: at(st["out"][key], st["sequences"]) for key in ("after", "dbefore") if key in st["out"]}
            ws = plan.recurrence_workspace(k, counts)
        else:
            st["top"] = st["teacher"].shape[1]
            a |= {key: at(st[key]) for key in ("logits", "teacher_ids", "teacher", "labels")}
            st["out"] = {"loss": new(n, dtype=torch.float32)} | ({"dlogits": new(n, k)} if case["gradient"] else {})
            ws = plan.distillation_workspace(k, st["top"], counts)
        a |= {key: at(st["out"][key]) for key in ("sum", "y", "saved", "dx", "states", "loss", "dlogits") if key in st["out"]}
        st["ws"] = torch.empty(max(ws, 16), dtype=torch.uint8, device=DEV)
    return st


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    case, plan, a, out, k, tokens = st["case"], st["plan"], st["at"], st["out"], st["case"]["cols"], st["tokens"]
    stream, ws = st["stream"], (st["ws"].data_ptr(), st["ws"].numel())
    if case["op"] == "norm":
        plan.residual_norm(a["gain"], k, tokens, a["x"], a["y"], a["rstd"], eps=EPS, residual=a.get("residual"), sum=a.get("sum"),
                           checkpoint=a.get("checkpoint"), dtype=st["dtype"], stream=stream)
        if case["saved"]:
            plan.checkpoint_load(a["checkpoint"], tokens, k, a["saved"], dtype=1, stream=stream)
        return {"rstd": st["rstd"], **out}
    if case["op"] == "ngrad":
        plan.residual_norm_gradient(0, a["gain"], tokens, a["x"], a["rstd"], a["dy"], a["dx"], *ws, dsum=a.get("dsum"),
                                    dtype=st["dtype"], stream=stream)
        return {"dgain": st["grad"], **out}
    if case["op"] == "rec":
        plan.recurrence(k, tokens, st["sequences"], a["starts"], a["gate"], a["input"], a["states"], *ws, before=a.get("before"),
                        after=a.get("after"), id_bytes=case["id_bytes"], dtype=st["dtype"], pitch=2 * k, stream=stream)
        return out
    if case["op"] == "rgrad":
        plan.recurrence_gradient(k, tokens, st["sequences"], a["starts"], a["gate"], a["input"], a["states"], a["dstates"],
                                 a["dgate"], a["dinput"], *ws, before=a.get("before"), dafter=a.get("dafter"),
                                 dbefore=a.get("dbefore"), id_bytes=case["id_bytes"], dtype=st["dtype"], pitch=2 * k, stream=stream)
        return out
    plan.distillation(k, tokens, a["logits"], a["teacher_ids"], a["teacher"], st["top"], a["loss"], *ws,
                      labels=a["labels"] if case["hard"] else None, dlogits=a.get("dlogits"), temperature=case["temperature"],
                      soft=1.0, hard=case["hard"], scale=_scale(case), id_bytes=case["id_bytes"], dtype=st["dtype"], stream=stream)
    return out


def _scale(case):
    """Of the loss's gradient: the mean over a worker's tokens, and a loss scale."""
    return 64.0 / case["tokens"]


# ---- plain forms
def _rstd(x):
    """The mean square in 64 bits: results that lie next to a border of the 8-bit codes do not hang on a sum's order."""
    return torch.rsqrt(x.double().square().mean(1) + EPS).float()


def _encode(y, st):
    """A block is 32 tokens of one feature; it has one power of two as its scale: (codes [blocks][features][32], exponents)."""
    full = torch.zeros(st["blocks"] * BLOCK, y.shape[1], dtype=torch.float32, device=DEV)
    full[st["place"]] = y.float()
    full = full.view(st["blocks"], BLOCK, y.shape[1]).transpose(1, 2)
    m, e = torch.frexp(full.abs().amax(2))                           # m in [1/2, 1)
    e = torch.where(m > 127.0 / 128.0, e - 6, e - 7).clamp(min=-126)
    return torch.ldexp(full, -e[..., None]).round().to(torch.int8), e


def _decode(q, e, st):
    x = torch.ldexp(q.float(), e[..., None])
    return x.transpose(1, 2).reshape(-1, q.shape[1])[st["place"]]


def _doubled(factor, value, longest):
    """x_i = value_i + factor_i x_(i-1), over spans that double; a factor of 0 starts anew."""
    step = 1
    while step < longest:
        value = torch.cat([value[:step], torch.addcmul(value[step:], factor[step:], value[:-step])])
        factor = torch.cat([factor[:step], factor[step:] * factor[:-step]])
        step *= 2
    return value


def _ends(case, starts):
    """(first and last row of every sequence in the array of all workers, which of them have a token, the longest's length)."""
    offsets = [sum(_tokens(case)[:w]) for w in range(case["world"])]
    first = torch.cat([s[:-1].long() + o for s, o in zip(starts, offsets)])
    last = torch.cat([s[1:].long() + o for s, o in zip(starts, offsets)]) - 1
    longest = max(b - a for s in _starts(case) for a, b in zip(s, s[1:]))
    return first, last, last >= first, longest


def _gates(d, k):
    g = d["product"][:, :k].double()
    return torch.sigmoid(g), torch.sigmoid(-g), d["product"][:, k:].double()


def _scan(case, d):
    """(states, states after the sequences) in 64 bits: a sum over a channel's long memory."""
    first, last, some, longest = _ends(case, d["starts"])
    a, b, u = _gates(d, case["cols"])
    value, at = b * u, first[some]
    if case["carry"]:
        value[at] += a[at] * d["before"].double()[some]
    a[at] = 0.0
    s = _doubled(a, value, longest)
    return s, torch.where(some[:, None], s[last.clamp(min=0)], d["before"].double()) if case["carry"] else None


def _run_plain(st):
    case, k, dt = st["case"], st["case"]["cols"], DT[st["case"]["dtype"]]
    if case["op"] == "norm":
        out, x = {}, st["x"]
        if case["residual"]:
            out["sum"] = x = (x.float() + st["residual"].float()).to(dt)
        out["rstd"] = _rstd(x)
        out["y"] = (x.float() * out["rstd"][:, None] * st["gain"].float()).to(dt)
        if case["saved"]:
            out["saved"] = _decode(*_encode(out["y"], st), st).to(torch.bfloat16)
        return out
    if case["op"] == "ngrad":
        normed, dy = st["x"].float() * st["rstd"][:, None], st["dy"].float()
        u = dy * st["gain"].float()
        dx = (u - normed * (u * normed).mean(1, keepdim=True)) * st["rstd"][:, None]
        if case["residual"]:
            dx += st["dsum"].float()
        return {"dgain": [p.sum(0).to(DT[case["params"]]) for p in _rows(dy * normed, st["tokens"])], "dx": dx.to(dt)}
    if case["op"] == "rec":
        s, after = _scan(case, st)
        return {"states": s.to(dt)} | ({"after": after.float()} if case["carry"] else {})
    if case["op"] == "rgrad":
        first, last, some, longest = _ends(case, st["starts"])
        a, b, u = _gates(st, k)
        value, at, end = st["dstates"].double(), first[some], last[some]
        previous = torch.cat([st["states"][:1], st["states"][:-1]]).double()
        previous[at] = 0.0
        if case["carry"]:
            value[end] += st["dafter"].double()[some]
            previous[at] = st["before"].double()[some]
        factor = torch.cat([a[1:], a[:1]])
        factor[end] = 0.0
        e = _doubled(factor.flip(0), value.flip(0), longest).flip(0)
        out = {"dproduct": torch.cat([a * b * e * (previous - u), b * e], 1).to(dt)}
        if case["carry"]:
            out["dbefore"] = torch.where(some[:, None], (a * e)[first.clamp(max=len(e) - 1)], st["dafter"].double()).float()
        return out
    z, hard, T = st["logits"].float(), case["hard"], case["temperature"]
    ids = st["teacher_ids"].long()
    there, label = ids >= 0, st["labels"].long()
    soft = there.any(1).float()
    lab = (label >= 0).float() * hard
    d = z - z.amax(1, keepdim=True)
    warm = torch.exp(d / T)
    sum_warm = warm.sum(1, dtype=torch.float64)
    t = torch.where(there, st["teacher"].double() / T, float("-inf"))
    p = torch.exp(t - t.amax(1, keepdim=True))
    p = torch.where(there, p / p.sum(1, keepdim=True), 0.0)
    ids = ids.clamp(min=0)
    part = p * (torch.log(p) - d.gather(1, ids).double() / T + torch.log(sum_warm)[:, None])
    loss = torch.where(p > 0, part, 0.0).sum(1)
    if hard:
        cold = torch.exp(d)
        sum_cold = cold.sum(1, dtype=torch.float64)
        label = label.clamp(min=0)[:, None]
        loss = loss + lab * (torch.log(sum_cold) - d.gather(1, label)[:, 0].double())
    out = {"loss": loss.float()}
    if case["gradient"]:
        g = warm * (soft / T / sum_warm.float())[:, None]
        g.scatter_add_(1, ids, -p.float() / T)
        if hard:
            g += cold * (lab / sum_cold.float())[:, None]
            g.scatter_add_(1, label, -lab[:, None])
        out["dlogits"] = (g * _scale(case)).to(dt)
    return out


def work(case):
    n, W, k, es, S = sum(_tokens(case)), case["world"], case["cols"], ES[case["dtype"]], sum(_sequences(case))
    values = n * k
    if case["op"] == "norm":
        kept = sum((t + BLOCK - 1) // BLOCK for t in _tokens(case)) * k * (BLOCK + 1) if case["saved"] else 0
        rows = 4 if case["residual"] else 2
        return {"bytes": values * es * rows + 4 * n + k * ES[case["params"]] + 2 * kept + (2 * values if kept else 0),
                "flops": values * (12 if kept else 6)}
    if case["op"] == "ngrad":
        return {"bytes": values * es * (4 if case["residual"] else 3) + 4 * n + (W + 1) * k * ES[case["params"]],
                "flops": values * 10}
    carried = 4 * S * k if case["carry"] else 0
    if case["op"] == "rec":
        return {"bytes": 3 * values * es + 2 * carried, "flops": values * 8}
    if case["op"] == "rgrad":
        return {"bytes": 6 * values * es + 3 * carried, "flops": values * 14}
    top = min(case["top"], k)
    told = n * (top * (es + case["id_bytes"]) + (case["id_bytes"] if case["hard"] else 0) + 4)
    return {"bytes": values * es * (2 if case["gradient"] else 1) + told,
            "flops": values * (5 + (4 if case["gradient"] else 0)) * (2 if case["hard"] else 1)}


def exact(case, seed):
    """The definitions in 64 bits."""
    d, k = _inputs(case, seed), case["cols"]
    if case["op"] == "norm":
        out, x = {}, d["x"].double()
        if case["residual"]:
            out["sum"] = x + d["residual"].double()
            x = out["sum"].to(DT[case["dtype"]]).double()               # the norm is that of the stream as it is kept
        out["rstd"] = 1.0 / torch.sqrt((x * x).sum(1) / k + EPS)
        out["y"] = x * out["rstd"][:, None] * d["gain"].double()
        if case["saved"]:
            kept, at = out["y"].to(DT[case["dtype"]]).double(), 0
            out["saved"] = torch.empty_like(kept)
            for t in _tokens(case):
                for b in range(at, at + t, BLOCK):
                    part = kept[b:min(b + BLOCK, at + t)]
                    step = torch.exp2(torch.ceil(torch.log2(part.abs().amax(0).clamp(min=1e-300) / 127.0)).clamp(min=-126.0))
                    out["saved"][b:b + len(part)] = torch.round(part / step) * step
                at += t
        return out
    if case["op"] == "ngrad":
        r, g, out, at = d["rstd"].double()[:, None], d["gain"].double(), {"dgain": [], "dx": []}, 0
        for t in _tokens(case):
            x, dy = d["x"][at:at + t].double(), d["dy"][at:at + t].double()
            out["dgain"].append((x * dy * r[at:at + t]).sum(0))
            inner = (x * dy * g).sum(1, keepdim=True) / k
            dx = r[at:at + t] * (dy * g) - r[at:at + t] ** 3 * x * inner
            out["dx"].append(dx + d["dsum"][at:at + t].double() if case["residual"] else dx)
            at += t
        return {"dgain": out["dgain"], "dx": torch.cat(out["dx"])}
    if case["op"] in ("rec", "rgrad"):
        # token by token, the longest sequences first, so that those that still run are the first so many
        spans, at = [], 0
        for s, t in zip(_starts(case), _tokens(case)):
            spans += [(at + a, b - a) for a, b in zip(s, s[1:])]
            at += t
        order = sorted(range(len(spans)), key=lambda i: -spans[i][1])
        first = torch.tensor([spans[i][0] for i in order], device=DEV)
        length = [spans[i][1] for i in order]
        running, m = [], len(order)
        for t in range(length[0]):
            while m and length[m - 1] <= t:
                m -= 1
            running.append(m)
        x = d["product"].double()
        a, u = 1.0 / (1.0 + torch.exp(-x[:, :k])), x[:, k:]
        back = torch.empty(len(order), dtype=torch.long, device=DEV)
        back[torch.tensor(order, device=DEV)] = torch.arange(len(order), device=DEV)
        zeros = torch.zeros(len(order), k, dtype=torch.float64, device=DEV)
        begin = d["before"].double()[torch.tensor(order, device=DEV)] if case["carry"] else zeros
        if case["op"] == "rec":
            s, out = begin.clone(), torch.empty_like(a)
            for t, m in enumerate(running):
                at = first[:m] + t
                s[:m] = u[at] + a[at] * (s[:m] - u[at])
                out[at] = s[:m]
            return {"states": out} | ({"after": s[back]} if case["carry"] else {})
        e, out = zeros.clone(), torch.empty_like(x)
        if case["carry"]:
            e = d["dafter"].double()[torch.tensor(order, device=DEV)]
        states, ds = d["states"].double(), d["dstates"].double()
        for t in range(length[0] - 1, -1, -1):
            m = running[t]
            at = first[:m] + t
            total = e[:m] + ds[at]
            prior = states[at - 1] if t else begin[:m]
            out[at] = torch.cat([total * (prior - u[at]) * a[at] * (1.0 - a[at]), total * (1.0 - a[at])], 1)
            e[:m] = a[at] * total
        return {"dproduct": out} | ({"dbefore": e[back]} if case["carry"] else {})
    T, losses, grads = case["temperature"], [], []
    step = max(1, (1 << 26) // k)
    for r in range(0, d["logits"].shape[0], step):
        z, ids, label = d["logits"][r:r + step].double(), d["teacher_ids"][r:r + step].long(), d["labels"][r:r + step].long()
        taught = ids >= 0                                               # either all of a row's entries or none
        rows, some = torch.arange(len(z), device=DEV)[:, None], taught.any(1)
        P = torch.zeros_like(z)
        P[rows, ids.clamp(min=0)] = torch.softmax(d["teacher"][r:r + step].double() / T, 1) * taught
        logQ = torch.log_softmax(z / T, 1)
        loss = torch.where(P > 0, P * (torch.log(P) - logQ), 0.0).sum(1)
        g = (torch.exp(logQ) - P) / T * some[:, None]
        if case["hard"]:
            logq, known = torch.log_softmax(z, 1), (label >= 0).double() * case["hard"]
            loss -= known * logq.gather(1, label.clamp(min=0)[:, None])[:, 0]
            one = torch.zeros_like(z)
            one[rows[:, 0], label.clamp(min=0)] = 1.0
            g += known[:, None] * (torch.exp(logq) - one)
        losses.append(loss)
        if case["gradient"]:
            grads.append(g * _scale(case))
    return {"loss": torch.cat(losses)} | ({"dlogits": torch.cat(grads)} if case["gradient"] else {})
