"""The operators at the ends of what their calls take: the most pairs, and values whose differences, exponentials or products pass binary32 where the
result does not."""
import math

import pytest
import torch

from tests import operator_ref as ref
from tests.test_gpu_token_logprob import TYPES, dq, forward, make_logits  # noqa: F401  (dq is a fixture)

pytestmark = pytest.mark.gpu

U = ref.U


@pytest.mark.parametrize("pairs", [(1 << 20) - 1, 1 << 20, (1 << 20) + 1, 1 << 24])
def test_the_most_pairs(dq, pairs):
    """More workgroups than one dimension of a grid takes.  The first and the last pair have a sequence with rows each; all others are empty."""
    z, y, gen = make_logits(7, 50, torch.float32, 3)
    start = torch.full((2 * pairs + 1,), 3, device="cuda")
    start[0], start[-1] = 0, 7
    loss, seq = torch.full((4,), math.nan, device="cuda"), torch.full((2 * pairs,), math.nan, device="cuda")
    out = torch.full((7, 50), math.nan, device="cuda")
    ws = torch.empty(dq.preference_loss_workspace_bytes(7, 50, pairs), dtype=torch.uint8, device="cuda")
    # a loss scale keeps the gradient, which is 1 / pairs, in the range where the bounds are relative
    dq.preference_loss(z.cuda(), y.cuda(), start, loss, seq, out, ws, beta=0.5, grad_scale=float(1 << 20))
    torch.cuda.synchronize()
    sm = ref.softmax(z, y)
    first, last = sm["logp"][:3].sum(), sm["logp"][3:].sum()
    bound = sm["logp_err"].sum() + 4 * U * (first.abs() + last.abs())
    assert abs(float(seq[0]) - float(first)) <= bound and abs(float(seq[-1]) - float(last)) <= bound and int((seq != 0).sum()) == 2
    h = 0.5 * torch.stack([first, -last])
    want = torch.stack([(torch.nn.functional.softplus(-h).sum() + (pairs - 2) * math.log(2)) / pairs, (h > 0).sum() / pairs, 0.5 * first / pairs, 0.5 * last / pairs])
    ref.close(loss, want, 2 * U * want.abs() + bound / pairs)
    g = 0.5 * torch.sigmoid(-h) / pairs
    d = torch.cat([-g[0].expand(3), g[1].expand(4)])
    want, err = ref.dlogits(sm, d, scale=float(1 << 20), d_err=(0.25 * bound / pairs + 4 * U * d.abs()))
    ref.close(out, want, err)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("temperature", [1.0, 100.0, 1e20, 3.2e36])
@pytest.mark.parametrize("vocab", [9, 700, 3000, 9000, 70000])
def test_logits_at_both_ends_of_the_type(dq, dtype, temperature, vocab):
    """z_y - m passes binary32 and (z_y - m) / T need not: -6.8e36 at T = 100, -6.8e18 at 1e20, and -213 at the largest temperature."""
    ends = torch.finfo(dtype)
    z, y, gen = make_logits(4, vocab, dtype, vocab)
    for r in range(4):
        z[r, (y[r] + 1) % vocab] = ends.max
    z[0, y[0]] = ends.min
    z[1, y[1]] = ends.min / 2
    z[2] = ends.min
    z[2, (y[2] + 1) % vocab] = ends.max
    sm = ref.softmax(z, y, temperature)
    want = sm["logp"].clone()
    want[want < -ends.max] = -math.inf  # of binary32: its largest number is bfloat16's but for half a unit
    if temperature > 1.0:
        assert want.isfinite().all() and float(want[0]) < -200.0
    logp, softmax = forward(dq, z.cuda(), y.cuda(), temperature)
    ref.close(logp, want, torch.nan_to_num(sm["logp_err"], posinf=0.0))
    ws = torch.empty(dq.policy_loss_workspace_bytes(4, vocab), dtype=torch.uint8, device="cuda")
    loss, lp, out = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(z).cuda()
    ones = torch.full((4,), 0.25, device="cuda")
    dq.policy_loss(z.cuda(), y.cuda(), torch.zeros(4, device="cuda"), ones, ones, loss, lp, out, ws, temperature=temperature)
    torch.cuda.synchronize()
    ref.close(lp, want, torch.nan_to_num(sm["logp_err"], posinf=0.0))
