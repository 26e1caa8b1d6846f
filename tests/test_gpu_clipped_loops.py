"""Algorithm 1 with clipped gradients, in every loop: what the server subtracts is the clipped gradients' average."""
import numpy as np
import pytest
import torch

from tests.test_gpu_parity import SEED, dq  # noqa: F401  (dq is a fixture)

pytestmark = pytest.mark.gpu

MODES = [dict(), dict(lagged=False), dict(one_pass=False), dict(norm_margin=0.1), dict(device_rule=True), dict(device_rule=True, lagged=False), dict(device_rule=True, norm_margin=0.1),
         dict(device_rule=True, per_tensor=True), dict(per_tensor=True), dict(per_tensor=True, lagged=False), dict(per_worker=True), dict(per_worker=True, lagged=False),
         dict(per_worker=True, per_tensor=True)]


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("chunk_local", [False, True])
def test_steps_are_those_of_clipped_gradients(dq, mode, chunk_local):
    """Workers' gradients of the norms 1.5^t, clipped to 0.25: along the mean gradient the steps add up to eta * 0.25 * T of it, where unclipped ones are 14 times as long.  Stochastic
    rounding moves an element by a variance of |g| * level at most, and independently; six standard deviations along one direction are a few per cent."""
    lens, M, T, eta, most = ([500] * 28 if chunk_local else [5000, 300, 9000]), 3, 6, 0.125, 0.25
    plan = dq.Plan(lens)
    assert plan.chunk_local == chunk_local
    gen = torch.Generator().manual_seed(3)
    fixed = torch.zeros((M, plan.padded_elems))
    for l, n in enumerate(lens):
        fixed[:, plan.segment_start(l):plan.segment_start(l) + n] = torch.randn((M, n), generator=gen)
    fixed = (fixed / fixed.norm(dim=1, keepdim=True)).cuda()
    x0 = torch.randn(plan.padded_elems, generator=gen).cuda()

    def grad_fn(t, x, grads):
        grads.copy_(fixed * 1.5 ** t)

    from paper_2107_14575_amd import dqsgd
    result = dqsgd.run(plan, x0, grad_fn, M, T, eta, 1.0, 1.0, b0=5, b_min=4, seed=SEED, max_norm=most, **mode)
    mean = fixed.double().mean(0)
    along = float((x0 - result.x).double() @ mean / (mean @ mean))
    b = int(np.min(np.asarray(result.bits)))
    variance = 0.0
    for l, n in enumerate(lens):
        g = fixed[:, plan.segment_start(l):plan.segment_start(l) + n].double() * most
        level = g.norm(dim=1, keepdim=True) / (2 ** b - 1)
        m = mean[plan.segment_start(l):plan.segment_start(l) + n] / (mean @ mean)
        variance += float((m ** 2 * g.abs() * level).sum()) / M ** 2 * T
    sigma = eta * variance ** 0.5
    assert 6 * sigma < 0.3 * eta * most * T, (b, sigma)
    assert abs(along - eta * most * T) <= 6 * sigma + 1e-4, (along, sigma, b)
    plan.close()
