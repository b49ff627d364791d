"""The calls that fill a plan's gradient tensors, as they are timed: the embedding lookup and its
gradient, activation checkpoints in 8 bits, and the weight and bias gradients that read them.

`run` computes each in elementary torch operations while `own` is False, and through the library
while it is True.  All W workers of a data-parallel program go through one call, as they do in the
library's other calls; a worker has its own tokens, tables, activations and gradients.
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
LARGEST = {"bytes": 1.0e9, "flops": 2.8e11}


def _case(op, world, tokens, rows, cols, dtype="f32", grads=None, ids="zipf", id_bytes=8, ragged=False, pad=0.0,
          bias=False, **name):
    """op      lookup, egrad, checkpoint or wgrad
    tokens  of the largest worker; ragged: the others have fewer
    rows    lookup, egrad: the table's rows; checkpoint, wgrad: the layer's input features
    cols    lookup, egrad: the table's width; wgrad: the layer's outputs
    dtype   of the table, the activations, the plan's tensors; grads: of the incoming gradients
    ids     zipf (words), positions (0, 1, 2, ... in every sequence) or types (a few segments);
            pad: share of the tokens at the end that are padding (id -1)"""
    return dict(name, op=op, world=world, tokens=tokens, rows=rows, cols=cols, dtype=dtype, grads=grads or dtype,
                ids=ids, id_bytes=id_bytes, ragged=ragged, pad=pad, bias=bias)


def listed():
    return [
        # word embeddings of the Transformer encoder: eight sequences of 512 tokens at each of eight workers
        _case("lookup", 8, 4096, 30522, 1024, "bf16", name="lookup-word-bf16-w8"),
        # one token at each of two workers, as when a model is tried out: latency alone
        _case("lookup", 2, 1, 30522, 1024, "f32", id_bytes=4, name="lookup-one-token-f32-w2"),
        # the gradient of the word embeddings: mostly rows that no token names
        _case("egrad", 8, 4096, 30522, 1024, "bf16", name="egrad-word-bf16-w8"),
        # of the segment embeddings: two rows, on which all tokens fall
        _case("egrad", 8, 4096, 2, 1024, "f32", ids="types", id_bytes=4, name="egrad-type-f32-w8"),
        # of the position embeddings, mixed precision, odd width, sequences that end in padding
        _case("egrad", 4, 2050, 512, 1001, "f32", "bf16", ids="positions", ragged=True, pad=0.1,
              name="egrad-position-mixed-w4"),
        # the input of the encoder's second feed-forward product, saved in the forward pass and read back
        _case("checkpoint", 4, 4096, 4096, 1, "bf16", name="checkpoint-ffn-bf16-w4"),
        # an image classifier's features, fp32, a batch that is no whole number of blocks
        _case("checkpoint", 8, 200, 2048, 1, "f32", ragged=True, name="checkpoint-fc-f32-w8"),
        # the small network's input: the smallest call
        _case("checkpoint", 4, 50, 784, 1, "f32", name="checkpoint-mlp-f32-w4"),
        # the encoder's first feed-forward product: the largest matrix product of its backward pass
        _case("wgrad", 8, 4096, 1024, 4096, "bf16", bias=True, name="wgrad-ffn-bf16-w8"),
        # one worker's attention projection over a long batch, gradients kept in fp32: few tiles, a long sum
        _case("wgrad", 1, 16384, 1024, 1024, "f32", name="wgrad-attn-f32-w1"),
        # VGG-16's first dense layer, a batch of 64 images: little to add, 400 MB to write at each worker
        _case("wgrad", 2, 64, 25088, 4096, "f32", bias=True, name="wgrad-vgg-fc1-f32-w2"),
        # the small network's first layer: latency
        _case("wgrad", 4, 128, 784, 256, "f32", bias=True, name="wgrad-mlp-f32-w4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges."""
    while True:
        op = rng.choice(["lookup", "egrad", "egrad", "checkpoint", "wgrad", "wgrad"])
        world = rng.choice([1, 2, 3, 4, 8, 8, 16])
        dtype = rng.choice(["f32", "bf16"])
        c = dict(id_bytes=rng.choice([4, 8]), ragged=rng.random() < 0.5)
        if op in ("lookup", "egrad"):
            ids = rng.choice(["zipf", "zipf", "positions", "types"])
            rows = {"zipf": _log(rng, 1000, 130_000), "positions": _log(rng, 64, 4096), "types": rng.choice([1, 2, 3])}[ids]
            case = _case(op, world, _log(rng, 1, 16384), rows, rng.choice([_log(rng, 16, 4096), 8 * _log(rng, 4, 512)]),
                         dtype, "bf16" if op == "egrad" and rng.random() < 0.3 else None, ids=ids,
                         pad=rng.choice([0.0, 0.0, 0.2]), **c)
        elif op == "checkpoint":
            case = _case(op, world, _log(rng, 1, 8192), _log(rng, 32, 16384), 1, dtype, **c)
        else:
            case = _case(op, world, _log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 10, 8192), dtype,
                         rng.choice([None, None, "bf16"]), bias=rng.random() < 0.5, **c)
        w = work(case)
        if all(w[k] <= LARGEST[k] for k in w):
            return case


def _tokens(case):
    """Tokens of every worker."""
    n = case["tokens"]
    return [max(1, n - (n * w) // (3 * case["world"])) if case["ragged"] else n for w in range(case["world"])]


def _generator(seed, worker, what):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 64 + worker) * 8 + what)
    return g


def _zipf(case):
    p = 1.0 / (torch.arange(case["rows"], dtype=torch.float64, device="cpu") + 3.0)
    return p / p.sum()


def _ids(case, seed, worker, n):
    g = _generator(seed, worker, 0)
    if case["ids"] == "zipf":
        u = torch.rand(n, dtype=torch.float64, device=DEV, generator=g)
        v = torch.searchsorted(_zipf(case).cumsum(0).to(DEV), u).clamp_(max=case["rows"] - 1)
    elif case["ids"] == "positions":
        v = torch.arange(n, device=DEV) % case["rows"]
    else:
        v = torch.randint(0, case["rows"], (n,), device=DEV, generator=g)
    if case["pad"]:
        v[n - int(n * case["pad"]):] = -1
    return v.to(torch.int64 if case["id_bytes"] == 8 else torch.int32)


def _activations(case, seed, worker, n):
    """What a layer is fed with: features of different sizes, a few of them far larger than the rest."""
    g = _generator(seed, worker, 1)
    x = torch.randn(n, case["rows"], device=DEV, generator=g)
    size = torch.exp(0.5 * torch.randn(case["rows"], device=DEV, generator=g))
    size = torch.where(torch.rand(case["rows"], device=DEV, generator=g) < 0.01, 20 * size, size)
    return (x * size).to(DT[case["dtype"]])


def _incoming(case, seed, worker, n):
    g = _generator(seed, worker, 2)
    return (torch.randn(n, case["cols"], device=DEV, generator=g) * 1e-2).to(DT[case["grads"]])


def _scale(case):
    return math.sqrt(case["cols"])


# ---- activations in 8 bits: a block is 32 tokens of one feature; it has one power of two as its scale.
# In memory: codes [blocks][features][32], then the exponents plus 127, [blocks][features].
def _encode(x):
    n, k = x.shape
    blocks = (n + BLOCK - 1) // BLOCK
    full = torch.zeros(blocks * BLOCK, k, dtype=torch.float32, device=x.device)
    full[:n] = x
    full = full.view(blocks, BLOCK, k).transpose(1, 2)               # [blocks][k][32]
    largest = full.abs().amax(2)
    m, e = torch.frexp(largest)                                      # m in [1/2, 1)
    e = torch.where(m > 127.0 / 128.0, e - 6, e - 7).clamp(min=-126)
    e = torch.where(largest == 0, torch.full_like(e, -126), e)
    bad = ~torch.isfinite(largest)
    e = torch.where(bad, torch.zeros_like(e), e)
    q = torch.ldexp(full.to(torch.float64), -e[..., None])           # exact in 64 bits at both ends of the range
    q = torch.where(bad[..., None], torch.zeros_like(q), q).round().to(torch.int8)
    s = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return q, s


def _decode(q, s, n):
    e = s.to(torch.int32) - 127
    size = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
    size = torch.where(s == 255, torch.full_like(size, float("nan")), size)
    x = q.to(torch.float32) * size[..., None]
    return x.transpose(1, 2).reshape(-1, q.shape[1])[:n]


def prepare(case, seed):
    counts, W, dt = _tokens(case), case["world"], DT[case["dtype"]]
    st = {"case": case, "tokens": counts, "stream": torch.cuda.current_stream().cuda_stream}
    op = case["op"]
    if op in ("lookup", "egrad"):
        st["ids"] = [_ids(case, seed, w, n) for w, n in enumerate(counts)]
    if op == "lookup":
        g = _generator(seed, 0, 3)
        table = torch.randn(case["rows"], case["cols"], device=DEV, generator=g).mul_(0.02).to(dt)
        st["table"] = [table if w == 0 else table.clone() for w in range(W)]   # every worker has its copy
        st["out"] = [torch.empty(n, case["cols"], dtype=dt, device=DEV) for n in counts]
        tensors = [case["rows"] * case["cols"]]
    elif op == "egrad":
        st["dy"] = [_incoming(case, seed, w, n) for w, n in enumerate(counts)]
        tensors = [case["rows"] * case["cols"]]
        st["grad"] = [[torch.empty(case["rows"], case["cols"], dtype=dt, device=DEV)] for _ in range(W)]
    elif op == "checkpoint":
        st["x"] = [_activations(case, seed, w, n) for w, n in enumerate(counts)]
        st["out"] = [torch.empty_like(x) for x in st["x"]]
        tensors = [case["rows"]]
    else:
        saved = [_encode(_activations(case, seed, w, n)) for w, n in enumerate(counts)]
        st["saved"] = [torch.cat([q.view(torch.uint8).reshape(-1), s.reshape(-1)]) for q, s in saved]
        st["dy"] = [_incoming(case, seed, w, n) for w, n in enumerate(counts)]
        tensors = [case["rows"] * case["cols"]] + ([case["cols"]] if case["bias"] else [])
        st["grad"] = [[torch.empty(case["rows"], case["cols"], dtype=dt, device=DEV)]
                      + ([torch.empty(case["cols"], dtype=dt, device=DEV)] if case["bias"] else []) for _ in range(W)]
    if own:
        import paper_2004_14020_amd as cm
        plan = st["plan"] = cm.Plan(W, tensors, dtype=cm.F32 if case["dtype"] == "f32" else cm.BF16)
        st["code"] = {"f32": cm.F32, "bf16": cm.BF16}
        st["at"] = {k: [t.data_ptr() for t in st[k]] for k in ("ids", "table", "out", "dy", "x", "saved") if k in st}
        st["ws"] = None
        if "grad" in st:
            plan.bind([[t.data_ptr() for t in row] for row in st["grad"]], None)
            if op == "egrad":
                size = plan.embedding_workspace(0, case["cols"], counts)
            else:
                size = plan.weight_gradient_workspace(0, case["rows"], counts)
            st["ws"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
        if op == "checkpoint":
            st["saved"] = [torch.empty(cm.checkpoint_bytes(n, case["rows"]), dtype=torch.uint8, device=DEV) for n in counts]
            st["at"]["saved"] = [t.data_ptr() for t in st["saved"]]
    return st


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    case, plan, at, code = st["case"], st["plan"], st["at"], st["code"]
    op, tokens, stream = case["op"], st["tokens"], st["stream"]
    if op == "lookup":
        plan.embedding_lookup(at["table"], case["rows"], case["cols"], at["ids"], tokens, at["out"], scale=_scale(case),
                              id_bytes=case["id_bytes"], stream=stream)
        return st["out"]
    if op == "egrad":
        plan.embedding_gradient(0, case["cols"], at["ids"], tokens, at["dy"], st["ws"].data_ptr(), st["ws"].numel(),
                                scale=_scale(case), id_bytes=case["id_bytes"], dy_dtype=code[case["grads"]], stream=stream)
        return [row[0] for row in st["grad"]]
    if op == "checkpoint":
        plan.checkpoint_store(at["x"], tokens, case["rows"], at["saved"], dtype=code[case["dtype"]], stream=stream)
        plan.checkpoint_load(at["saved"], tokens, case["rows"], at["out"], dtype=code[case["dtype"]], stream=stream)
        return st["out"]
    plan.weight_gradient(0, 1 if case["bias"] else None, at["saved"], tokens, case["rows"], at["dy"], st["ws"].data_ptr(),
                         st["ws"].numel(), dy_dtype=code[case["grads"]], stream=stream)
    return st["grad"]


def _run_plain(st):
    case, dt = st["case"], DT[st["case"]["dtype"]]
    op, out = case["op"], []
    for w, n in enumerate(st["tokens"]):
        if op in ("lookup", "egrad"):
            ids = st["ids"][w].long()
            known = (ids >= 0) & (ids < case["rows"])
            ids = torch.where(known, ids, torch.zeros_like(ids))
        if op == "lookup":
            rows = st["table"][w][ids].float() * _scale(case)
            out.append(torch.where(known[:, None], rows, torch.zeros_like(rows)).to(dt))
        elif op == "egrad":
            dy = st["dy"][w].float()
            dy = torch.where(known[:, None], dy, torch.zeros_like(dy))
            g = torch.zeros(case["rows"], case["cols"], device=DEV).index_add_(0, ids, dy)
            out.append((g * _scale(case)).to(dt))
        elif op == "checkpoint":
            out.append(_decode(*_encode(st["x"][w]), n).to(dt))
        else:
            k, blocks = case["rows"], (n + BLOCK - 1) // BLOCK
            q = st["saved"][w][:blocks * BLOCK * k].view(torch.int8).view(blocks, k, BLOCK)
            x = _decode(q, st["saved"][w][blocks * BLOCK * k:].view(blocks, k), n)
            dy = st["dy"][w].float()
            out.append([(x.t() @ dy).to(dt)] + ([dy.sum(0).to(dt)] if case["bias"] else []))
    return out


def work(case):
    counts, es, gs = _tokens(case), ES[case["dtype"]], ES[case["grads"]]
    n, W, rows, cols = sum(counts), case["world"], case["rows"], case["cols"]
    if case["op"] == "lookup":
        if case["ids"] == "zipf":
            p = _zipf(case)
            named = sum(float((1.0 - torch.exp(t * torch.log1p(-p))).sum()) for t in counts)
        else:
            named = sum(min(t, rows) for t in counts)
        return {"bytes": int(n * case["id_bytes"] + (named + n) * cols * es), "flops": n * cols}
    if case["op"] == "egrad":
        return {"bytes": n * case["id_bytes"] + n * cols * gs + W * rows * cols * es, "flops": n * cols + W * rows * cols}
    blocks = sum((t + BLOCK - 1) // BLOCK for t in counts)
    saved = blocks * rows * (BLOCK + 1)
    if case["op"] == "checkpoint":
        return {"bytes": 2 * (n * rows * es + saved), "flops": 4 * n * rows}
    tensors = W * cols * (rows + (1 if case["bias"] else 0))
    return {"bytes": saved + n * cols * gs + tensors * es, "flops": 2 * n * rows * cols + (n * cols if case["bias"] else 0)}


def exact(case, seed):
    """The definitions in 64 bits."""
    out = []
    for w, n in enumerate(_tokens(case)):
        if case["op"] == "lookup":
            g = _generator(seed, 0, 3)
            table = torch.randn(case["rows"], case["cols"], device=DEV, generator=g).mul_(0.02).to(DT[case["dtype"]])
            ids = _ids(case, seed, w, n).long()
            y = torch.zeros(n, case["cols"], dtype=torch.float64, device=DEV)
            there = torch.nonzero((ids >= 0) & (ids < case["rows"])).flatten()
            y[there] = torch.tensor(_scale(case), dtype=torch.float32).double().item() * table.index_select(0, ids[there]).double()
            out.append(y)
        elif case["op"] == "egrad":
            ids = _ids(case, seed, w, n).long()
            order = torch.argsort(ids, stable=True)
            order = order[int((ids < 0).sum()):]
            y = torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device=DEV)
            dy = _incoming(case, seed, w, n).double()[order]
            y.index_put_((ids[order],), dy, accumulate=True)
            out.append(y * torch.tensor(_scale(case), dtype=torch.float32).double().item())
        else:
            x = _activations(case, seed, w, n).double()
            y = torch.empty_like(x)
            for b in range(0, n, BLOCK):
                part = x[b:b + BLOCK]
                step = torch.exp2(torch.ceil(torch.log2(part.abs().amax(0).clamp(min=1e-300) / 127.0)).clamp(min=-126.0))
                y[b:b + BLOCK] = torch.round(part / step) * step
            if case["op"] == "checkpoint":
                out.append(y)
            else:
                dy = _incoming(case, seed, w, n).double()
                out.append([y.t().contiguous() @ dy] + ([dy.sum(0)] if case["bias"] else []))
    return out
