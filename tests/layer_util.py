"""Plain CPU statements, in 64 bits, of the operators that fill gradient tensors, and device plumbing for
their tests (not collected by pytest)."""
from __future__ import annotations

import numpy as np
import torch

import paper_2004_14020_amd as cm

DEV = "cuda:0"
TORCH = {cm.F32: torch.float32, cm.BF16: torch.bfloat16}
HALF_STEP = {cm.F32: 2.0 ** -24, cm.BF16: 2.0 ** -8}      # largest relative error of one rounding


def lookup(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            out[i] = float(np.float32(scale)) * table[v].astype(np.float64)
    return out


def embedding_gradient(vocab, ids, dy, scale):
    """(gradient, sum of the magnitudes, number of terms) in 64 bits."""
    g, mag, n = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros((vocab, 1))
    for i, v in enumerate(ids):
        if 0 <= v < vocab:
            g[v] += dy[i]
            mag[v] += np.abs(dy[i])
            n[v] += 1
    s = float(np.float32(scale))
    return s * g, abs(s) * mag, n


def encode(x):
    """(codes [block][feature][32] int8, scale bytes [block][feature]) of activations [token][feature]."""
    n, k = x.shape
    blocks = (n + 31) // 32
    full = np.zeros((blocks * 32, k))
    full[:n] = x
    full = full.reshape(blocks, 32, k).transpose(0, 2, 1)
    with np.errstate(invalid="ignore"):
        largest = np.abs(full).max(2)                       # a NaN stays one
    bad = ~np.isfinite(largest)
    largest = np.where(bad, 0.0, largest)
    e = np.maximum(np.frexp(largest)[1] - 7, -126)
    e = np.where(largest > 127 * 2.0 ** e, e + 1, e)        # m in [1/2, 1): never more than one step
    e = np.minimum(np.where(largest == 0, -126, e), 121)
    codes = np.rint(np.where(bad[:, :, None], 0.0, full) / 2.0 ** e[:, :, None]).clip(-127, 127).astype(np.int8)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, scales, n):
    size = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (codes * size[:, :, None]).transpose(0, 2, 1).reshape(-1, codes.shape[1])[:n]


def image(codes, scales):
    """The bytes of a checkpoint."""
    b = codes.tobytes() + scales.tobytes()
    return np.frombuffer(b + bytes(-len(b) % 16), np.uint8)


def f64(t):
    return t.detach().cpu().double().numpy()


def addresses(tensors):
    return [t.data_ptr() for t in tensors]


def bound_plan(world, elems, dtype, fill=None):
    """A plan over freshly allocated gradient tensors; grads[w][t]."""
    plan = cm.Plan(world, elems, dtype=dtype)
    grads = [[torch.full((n,), float("nan") if fill is None else fill, dtype=TORCH[dtype], device=DEV) for n in elems]
             for _ in range(world)]
    plan.bind([addresses(row) for row in grads], None)
    return plan, grads


def workspace(nbytes):
    """Workspace of exactly that size, full of what would be wrong to read, and bytes behind it that must stay."""
    return torch.full((max(nbytes, 16) + 256,), 0xFF, dtype=torch.uint8, device=DEV)


def untouched(ws, nbytes):
    return bool((ws[max(nbytes, 16):] == 0xFF).all())


def rows(n, cols, pitch, dtype, values=None, fill=float("nan")):
    """(memory, view of n rows of `cols` columns `pitch` apart): all of the memory that is no row is `fill`."""
    mem = torch.full((max(n, 1) * pitch + 8,), fill, dtype=TORCH[dtype], device=DEV)
    view = mem[:n * pitch].view(n, pitch)[:, :cols]
    if values is not None:
        view.copy_(values)
    return mem, view


def stream():
    return torch.cuda.current_stream().cuda_stream


def saved_sparse(n, at, values):
    """The checkpoint of n tokens in which feature k is values[k], a power of two from 2^-114 on, at token at[k], and 0 elsewhere."""
    k, blocks = len(values), (n + 31) // 32
    codes, scales = np.zeros((blocks, k, 32), np.int8), np.ones((blocks, k), np.uint8)
    f, at = np.arange(len(at)), np.asarray(at)
    codes[at // 32, f, at % 32] = 64
    if n:
        scales[at // 32, f] = np.log2(values).astype(int) - 6 + 127
    return torch.tensor(np.frombuffer(image(codes, scales).tobytes() + bytes(16), np.uint8).copy(), device=DEV)
