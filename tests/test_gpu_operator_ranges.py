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
