"""More rows than one direction of a grid has places for, or nearly as many as a call may have: the same rows over and over, whose
results have to be those of a small call to the bit."""
import pytest
import torch

import paper_2004_14020_amd as cm

from layer_util import DEV, addresses, bound_plan, stream, workspace

pytestmark = pytest.mark.gpu

PERIOD = 4099


def repeated(t, n):
    return t.repeat((n + PERIOD - 1) // PERIOD, *[1] * (t.dim() - 1))[:n].contiguous()


def equal(got, want, n):
    """Row i of got is row i % PERIOD of want."""
    whole = n // PERIOD * PERIOD
    assert torch.equal(got[:whole].view(-1, *want.shape), want.expand(n // PERIOD, *want.shape))
    assert torch.equal(got[whole:], want[:n - whole])


def test_norm_of_more_rows():
    n, width = 4 * (1 << 20) + 4 * 777 + 3, 4                    # four rows to a workgroup
    plan, grads = bound_plan(1, [width], cm.F32)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x, res, dy = (torch.randn(PERIOD, width, device=DEV, generator=g) for _ in range(3))
    gain = torch.randn(width, device=DEV, generator=g)
    results = []
    for m in (PERIOD, n):
        at = [repeated(t, m) for t in (x, res, dy)]
        total, y, dx = (torch.full((m, width), 7.0, device=DEV) for _ in range(3))
        rstd = torch.full((m,), 7.0, device=DEV)
        plan.residual_norm([gain.data_ptr()], width, [m], [at[0].data_ptr()], [y.data_ptr()], [rstd.data_ptr()], residual=[at[1].data_ptr()],
                           sum=[total.data_ptr()], stream=stream())
        need = plan.residual_norm_workspace(0, [m])
        ws = workspace(need)
        plan.residual_norm_gradient(0, [gain.data_ptr()], [m], [total.data_ptr()], [rstd.data_ptr()], [at[2].data_ptr()], [dx.data_ptr()],
                                    ws.data_ptr(), need, stream=stream())
        torch.cuda.synchronize()
        results.append((total, y, rstd, dx))
        n64 = total.double() * rstd.double()[:, None]
        want, mag = (at[2].double() * n64).sum(0), (at[2].double() * n64).abs().sum(0)
        # a part's rows one after the other, of which there are at most 2^13 by a wavefront, then 1024 parts and the joins: fp32 sums
        assert bool(((grads[0][0].double() - want).abs() <= (2.0 ** 13 + 1024 + 40) * 2.0 ** -24 * mag).all())
    for got, want in zip(results[1], results[0]):
        equal(got, want, n)
    plan.close()


def test_distillation_of_more_rows():
    n, vocab, top = (1 << 20) + 777, 8, 2
    plan = cm.Plan(1, [1])
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    z, t = torch.randn(PERIOD, vocab, device=DEV, generator=g), torch.randn(PERIOD, top, device=DEV, generator=g)
    ids, labels = (torch.randint(-1, vocab, s, device=DEV, generator=g) for s in ((PERIOD, top), (PERIOD,)))
    results = []
    for m in (PERIOD, n):
        at = [repeated(v, m) for v in (z, ids, t, labels)]
        loss, dz = torch.full((m,), 7.0, device=DEV), torch.full((m, vocab), 7.0, device=DEV)
        assert plan.distillation_workspace(vocab, top, [m]) == 0
        plan.distillation(vocab, [m], [at[0].data_ptr()], [at[1].data_ptr()], [at[2].data_ptr()], top, [loss.data_ptr()], None, 0,
                          labels=[at[3].data_ptr()], dlogits=[dz.data_ptr()], temperature=2.0, hard=0.5, stream=stream())
        torch.cuda.synchronize()
        results.append((loss, dz))
    for got, want in zip(results[1], results[0]):
        equal(got, want, n)
    plan.close()


@pytest.mark.parametrize("channels", [1, 3])
def test_recurrence_of_more_tokens_and_sequences(channels):
    """Sequences of one token, so that rows repeat; the small call has a kernel of its own, and no other arithmetic."""
    few, n = 1000, (1 << 21) + 777
    plan = cm.Plan(1, [1])
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x, ds, before, dafter = (torch.randn(few, c * channels, device=DEV, generator=g) for c in (2, 1, 1, 1))
    results = []
    for m in (few, n):
        at = [t.repeat((m + few - 1) // few, 1)[:m].contiguous() for t in (x, ds, before, dafter)]
        starts = torch.arange(m + 1, device=DEV)
        states, after, dbefore = (torch.full((m, channels), 7.0, device=DEV) for _ in range(3))
        dx = torch.full((m, 2 * channels), 7.0, device=DEV)
        need = plan.recurrence_workspace(channels, [m])
        ws = workspace(need)
        halves = lambda t: ([t.data_ptr()], [t.data_ptr() + 4 * channels])                               # noqa: E731
        plan.recurrence(channels, [m], [m], [starts.data_ptr()], *halves(at[0]), [states.data_ptr()], ws.data_ptr(), need,
                        before=[at[2].data_ptr()], after=[after.data_ptr()], pitch=2 * channels, stream=stream())
        plan.recurrence_gradient(channels, [m], [m], [starts.data_ptr()], *halves(at[0]), [states.data_ptr()], [at[1].data_ptr()],
                                 *halves(dx), ws.data_ptr(), need, before=addresses([at[2]]), dafter=[at[3].data_ptr()],
                                 dbefore=[dbefore.data_ptr()], pitch=2 * channels, stream=stream())
        torch.cuda.synchronize()
        results.append((states, after, dbefore, dx))
    for got, want in zip(results[1], results[0]):
        whole = n // few * few
        assert torch.equal(got[:whole].view(-1, *want.shape), want.expand(n // few, *want.shape))
        assert torch.equal(got[whole:], want[:n - whole])
    plan.close()
