"""Where the norm's results are known to the last bit: 1 / sqrt of a mean square that is exact in 64 bits or nearly, and sums of small whole numbers."""
import numpy as np
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import DEV, bound_plan, stream, workspace

pytestmark = pytest.mark.gpu


def rstd_of(x, eps):
    n, width = x.shape
    plan, at = cm.Plan(1, [1]), torch.tensor(x, device=DEV)
    y, rstd, gain = torch.empty_like(at), torch.empty(n, device=DEV), torch.ones(width, device=DEV)
    plan.residual_norm([gain.data_ptr()], width, [n], [at.data_ptr()], [y.data_ptr()], [rstd.data_ptr()], eps=eps, stream=stream())
    torch.cuda.synchronize()
    plan.close()
    return rstd.cpu().numpy()


def check(got, m):
    """1 / sqrt(m), right to 2^-50 and then rounded: nothing else between two fp32 numbers than either, within 2^-50 of where they meet."""
    r = 1 / np.sqrt(m)                                              # 2^-63 and as much again
    low, high = ((r * (1 + s * np.longdouble(2) ** -50)).astype(np.float32) for s in (-1, 1))
    wrong = (got < low) | (got > high)
    assert not wrong.any(), f"{wrong.sum()} of {len(m)} rows, first {np.argmax(wrong)}: {got[wrong][0]!r}, want {low[wrong][0]!r}"


@pytest.mark.parametrize("eps", [2.0 ** -17, 1e-5, 1e-12])
def test_rstd_of_rows_of_all_sizes(eps):
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((1 << 20, 1)) * np.exp(6 * rng.standard_normal((1 << 20, 1))).clip(1e-8, 1e8)).astype(np.float32)
    x64 = x[:, 0].astype(np.float64)                                # whose squares are exact
    check(rstd_of(x, eps), (x64 * x64 + float(np.float32(eps))).astype(np.longdouble))


@pytest.mark.parametrize("side", [-1, 1])
def test_rstd_next_to_where_two_numbers_meet(side):
    """Two columns whose mean square puts 1 / sqrt as near to the middle of two fp32 numbers as columns in fp32 can, mostly within 2^-45."""
    n, eps = 1 << 18, np.longdouble(np.float32(2.0 ** -20))
    rng = np.random.default_rng(6 + side)
    low = (0.5 + rng.integers(0, 1 << 23, n) * 2.0 ** -24).astype(np.float32)
    middle = low.astype(np.longdouble) + np.longdouble(2) ** -25
    r = middle * (1 + side * np.longdouble(2) ** -rng.uniform(47, 49, n).astype(np.longdouble))
    squares = 2 * (1 / (r * r) - eps)
    x = np.empty((n, 2), np.float32)
    x[:, 0] = np.sqrt(squares * (1 - np.longdouble(2) ** -22))      # the second one makes up for what the first leaves
    x[:, 1] = np.sqrt(squares - x[:, 0].astype(np.longdouble) ** 2)
    x64 = x.astype(np.float64)
    m = (x64[:, 0] * x64[:, 0] + x64[:, 1] * x64[:, 1]) * 0.5 + float(eps)      # as near as 2^-52: 1 / sqrt to 2^-53
    near = np.abs(1 / np.sqrt(m.astype(np.longdouble)) / middle - 1)
    assert np.median(near) < np.longdouble(2) ** -45
    check(rstd_of(x, float(eps)), m.astype(np.longdouble))


@pytest.mark.parametrize("dtype", [cm.F32, cm.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,width", [(4 * (1 << 20) + 4 * 777 + 3, 4), (600_001, 9), (50_001, 1030), (20_000, 4100)])
def test_every_row_counts_once_in_the_gains_gradient(n, width, dtype):
    """rstd = 1 and whole numbers, none of which is 0 or below, with a sum below 2^24: exact in fp32 in any order, so that no row is lost and none
    counted twice."""
    plan, grads = bound_plan(1, [width], cm.F32)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    t = torch.float32 if dtype == cm.F32 else torch.bfloat16
    x = torch.randint(1, 3, (n, width), device=DEV, generator=g).to(t)
    dy = torch.ones_like(x)
    some = torch.randint(0, n, (1000,), device=DEV, generator=g)
    dy[some] = torch.randint(1, 9, (1000, width), device=DEV, generator=g).to(t)
    gain, rstd, dx = torch.ones(width, device=DEV), torch.ones(n, device=DEV), torch.empty_like(x)
    want = sum((x[i:i + (1 << 20)].double() * dy[i:i + (1 << 20)].double()).sum(0) for i in range(0, n, 1 << 20))
    assert float(want.max()) < 2 ** 24
    for accumulate in (False, True):
        need = plan.residual_norm_workspace(0, [n])
        ws = workspace(need)
        plan.residual_norm_gradient(0, [gain.data_ptr()], [n], [x.data_ptr()], [rstd.data_ptr()], [dy.data_ptr()], [dx.data_ptr()],
                                    ws.data_ptr(), need, dtype=dtype, accumulate=accumulate, stream=stream())
        torch.cuda.synchronize()
        assert torch.equal(grads[0][0].double(), want * (2 if accumulate else 1))
    plan.close()
