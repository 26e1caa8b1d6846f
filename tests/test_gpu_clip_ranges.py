"""Clipping where the factor alone is below binary32's normal numbers and its products are not: gradients that have grown beyond 1e38 times their bound."""
import math

import pytest
import torch

from tests import operator_ref as ref
from tests.test_gpu_clip import TYPES, U, check, clipped64, norm64, work
from tests.test_gpu_parity import dq  # noqa: F401  (dq is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("max_norm", [100.0, 1.0, 1e-3, 1e-6, 1e-20, 1e-38])
@pytest.mark.parametrize("lens", [[5000], [100, 70000, 3, 200001]])
def test_factors_below_binary32(dq, dtype, max_norm, lens):
    """One launch and two; into others, in place and into the row.  Beside the large values there are ordinary ones, which become 0 or nearly."""
    gen = torch.Generator().manual_seed(len(lens))
    grads = []
    for n in lens:
        g = (torch.rand(n, generator=gen) + 0.5) * 2e38 * torch.where(torch.rand(n, generator=gen) < 0.5, -1.0, 1.0)
        g[::7] = torch.randn(len(g[::7]), generator=gen)
        grads.append(g.to(dtype).cuda())
    n = norm64(grads)
    want = clipped64(grads, max_norm)
    assert max_norm / n < 2.0 ** -126
    norm, ws = work(dq)
    plan = dq.Plan(lens)
    row, out = torch.full((plan.padded_elems,), math.nan, device="cuda"), [torch.full_like(g, math.nan) for g in grads]
    dq.clip_grads(grads, max_norm, norm, ws, out=out)
    dq.clip_gather(plan, grads, max_norm, norm, row, ws)
    dq.clip_grads(grads, max_norm, norm, ws)
    torch.cuda.synchronize()
    for l, w in enumerate(want):
        check(out[l], w, dtype)
        assert torch.equal(grads[l], out[l])
        check(row[plan.segment_start(l):plan.segment_start(l) + lens[l]], w, torch.float32)
    plan.close()


@pytest.mark.parametrize("M,n_seg", [(3, 62), (2, 50001)])
@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e-20])
def test_norms_whose_factor_is_below_binary32(dq, M, n_seg, max_norm):
    gen = torch.Generator().manual_seed(n_seg)
    norms = (torch.rand((M, n_seg), generator=gen) + 0.5) * 2e38
    total = norms.double().square().sum(1).sqrt()
    ws = torch.empty(dq.clip_norms_workspace_bytes(M, n_seg), dtype=torch.uint8, device="cuda")
    dev, out, tot = norms.cuda(), torch.full((M, n_seg), math.nan, device="cuda"), torch.full((M,), math.nan, device="cuda")
    dq.clip_norms(dev, max_norm, tot, out, ws)
    assert tot.isinf().all()  # beyond binary32; the factor is of the norm in binary64
    want = norms.double() * (max_norm / total)[:, None]
    ref.close(out, want, want * 4 * U + 2.0 ** -149)
    dq.clip_norms(dev, max_norm, tot, dev, ws)
    assert torch.equal(dev, out)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_ordinary_factors(dq, dtype):
    """A factor that binary32 holds is one product, rounded as it always was."""
    gen = torch.Generator().manual_seed(9)
    g = (torch.randn(70003, generator=gen) * 3).to(dtype).cuda()
    norm, ws = work(dq)
    for max_norm in (1.0, 1e-3, 1e-30):
        out = [torch.full_like(g, math.nan)]
        dq.clip_grads([g], max_norm, norm, ws, out=out)
        f = torch.tensor(max_norm / norm64([g]), dtype=torch.float64).float().cuda()
        wide = (g.float() * f).to(dtype)
        # the norm's binary64 sum may differ in its last bits, and with it the factor by one unit
        assert float((out[0].float() - wide.float()).abs().max()) <= 4 * ref.TYPE_U[dtype][0] * float(wide.float().abs().max()) + 2 * ref.TYPE_U[dtype][1]
