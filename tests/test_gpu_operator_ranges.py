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


@pytest.mark.parametrize("lens,vocab", [([3, 2, 4, 3], 60), ([70, 40, 50, 30], 9000)])
@pytest.mark.parametrize("own_stream", [False, True])
def test_sequences_of_probability_zero(dq, lens, vocab, own_stream):
    """A token of probability 0 in one sequence of a pair: h is infinite, and a term of the loss whose factor is 0 adds nothing (-1 ln sigma(inf) - 0 ln sigma(-inf)
    is 0).  The gradient is that of a sigmoid of 0 or 1."""
    rows, pairs = sum(lens), 2
    stream = torch.cuda.Stream() if own_stream else None
    start = torch.tensor([0] + lens).cumsum(0)
    for which, side in ((0, -math.inf), (2, math.inf)):  # the first pair's preferred sequence, or its other one
        z, y, gen = make_logits(rows, vocab, torch.float32, 5)
        row = int(start[which])
        z[row, y[row]] = -math.inf
        sm = ref.softmax(z, y)
        S = torch.stack([sm["logp"][a:b].sum() for a, b in zip(start[:-1], start[1:])])
        h1 = 0.5 * (S[1] - S[3])
        sp = torch.nn.functional.softplus
        for eps in (0.0, 0.25, 1.0):
            # the first pair's loss: -ln sigma(h) has the factor 1 - eps, -ln sigma(-h) eps
            infinite = (1 - eps if side < 0 else eps) > 0
            l0 = math.inf if infinite else 0.0
            want = torch.tensor([(l0 + float((1 - eps) * sp(-h1) + eps * sp(h1))) / 2])
            g0 = (1 - eps) if side < 0 else -eps          # (1 - eps) sigma(-h) - eps sigma(h)
            g1 = (1 - eps) * torch.sigmoid(-h1) - eps * torch.sigmoid(h1)
            loss, seq = torch.full((4,), math.nan, device="cuda"), torch.full((4,), math.nan, device="cuda")
            out = torch.full((rows, vocab), math.nan, device="cuda")
            ws = torch.empty(dq.preference_loss_workspace_bytes(rows, vocab, pairs), dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            dq.preference_loss(z.cuda(), y.cuda(), start.cuda(), loss, seq, out, ws, beta=0.5, label_smoothing=eps, stream=stream)
            torch.cuda.synchronize()
            err = torch.nan_to_num(sm["logp_err"], posinf=0.0).sum() + 8 * U * S[S.isfinite()].abs().sum()
            ref.close(loss[:1], want, (err + 4 * U) * (1 + want.abs().nan_to_num(posinf=0.0)))
            assert float(loss[1]) == ((side > 0) + (float(h1) > 0)) / 2
            assert float(seq[which]) == -math.inf and seq[[k for k in range(4) if k != which]].isfinite().all()
            d = torch.zeros(rows, dtype=torch.float64)
            for k, g in ((0, -g0), (1, -float(g1)), (2, g0), (3, float(g1))):
                d[start[k]:start[k + 1]] = 0.5 * g / pairs
            grad, bound = ref.dlogits(sm, d, d_err=err.expand(rows) * 0.25 + 4 * U)
            ref.close(out, grad, torch.nan_to_num(bound))


def policy_rows(dq, logp_minus_old, adv, ref_minus_logp=None, beta=0.0, at_zero=(), vocab=90, dtype=torch.float32, rows=None):
    """One policy loss whose rows have the given differences; rows in at_zero take a token of probability 0.  -> sums, logp, dlogits, and what they are of"""
    n = len(adv)
    z, y, gen = make_logits(n, vocab, dtype, 17)
    for r in at_zero:
        z[r, y[r]] = -math.inf
    sm = ref.softmax(z, y)
    logp32 = torch.nan_to_num(sm["logp"], neginf=0.0)
    old = (logp32 - torch.tensor(logp_minus_old, dtype=torch.float64)).float()
    reference = None if ref_minus_logp is None else (logp32 + torch.tensor(ref_minus_logp, dtype=torch.float64)).float()
    a, w = torch.tensor(adv, dtype=torch.float32), torch.full((n,), 1.0 / n)
    loss, logp, out = torch.empty(4, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(z).cuda()
    ws = torch.empty(dq.policy_loss_workspace_bytes(n, vocab), dtype=torch.uint8, device="cuda")
    alone, ignored = torch.empty(4, device="cuda"), torch.empty(n, device="cuda")
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    for gradient, l, lp in ((out, loss, logp), (None, alone, ignored)):
        dq.policy_loss(z.cuda(), y.cuda(), old.cuda(), a.cuda(), w.cuda(), l, lp, gradient, ws, ref_logp=up(reference), clip_low=0.2, clip_high=0.3, beta=beta)
    torch.cuda.synchronize()
    return loss, alone, logp, out, (sm, old, reference, a, w, z, y)


@pytest.mark.parametrize("vocab", [5, 90, 3000, 9000, 70000])
def test_ratios_beyond_binary32(dq, vocab):
    """exp(logp - old_logp) beyond binary32 where its product with the advantage is not: 0 for an advantage of 0, 1e33 for one of -1e-10; a positive advantage is clipped."""
    loss, alone, logp, out, (sm, old, _, a, w, z, y) = policy_rows(dq, [100.0, 100.0, 100.0, 0.1, 120.0, -200.0], [0.0, -1e-10, 2.0, 1.0, -1e-30, 1.0], vocab=vocab)
    sums, d, sum_err, d_err, lp = ref.policy(sm, old, None, a, w, 0.2, 0.3, 0.0)
    assert sums.isfinite().all() and float(sums[1]) > 1e32
    # where the exponential overflows it is the square of one of half the exponent, whose error is twice one's
    for l in (loss, alone):
        ref.close(l, sums, 2 * sum_err)
    ref.close(logp, lp, sm["logp_err"])
    want, bound = ref.dlogits(sm, d, d_err=2 * d_err)
    ref.close(out, want, bound)
    assert not out[0].any() and not out[2].any()
    # an advantage of 0 beside ordinary rows
    loss, alone, logp, out, (sm, old, _, a, w, z, y) = policy_rows(dq, [95.0, 0.1, -0.1], [0.0, 1.0, -0.5], vocab=vocab)
    sums, d, sum_err, d_err, lp = ref.policy(sm, old, None, a, w, 0.2, 0.3, 0.0)
    for l in (loss, alone):
        ref.close(l, sums, sum_err)
    want, bound = ref.dlogits(sm, d, d_err=d_err)
    ref.close(out, want, bound)


@pytest.mark.parametrize("vocab", [5, 90, 3000, 9000, 70000])
def test_divergence_of_a_token_of_probability_zero(dq, vocab):
    """exp(u) - 1 - u is infinite for an infinite u of either sign, not NaN: with beta = 0 in its own sum alone, otherwise in the loss as well."""
    for ref_minus in (0.5, -math.inf):
        zero = (1,) if ref_minus == 0.5 else ()
        for beta in (0.0, 0.1):
            loss, alone, logp, out, (sm, old, reference, a, w, z, y) = policy_rows(dq, [0.1, 0.0, -0.1], [1.0, 0.5, -1.0], [0.2, ref_minus, -0.3], beta=beta, at_zero=zero, vocab=vocab)
            assert float(loss[2]) == math.inf and float(alone[2]) == math.inf
            assert (float(logp[1]) == -math.inf) == bool(zero) and logp[[0, 2]].isfinite().all()
            assert out[[0, 2]].isfinite().all()
            if beta:
                assert float(loss[0]) == math.inf and float(alone[0]) == math.inf
            else:
                plain = ref.policy(sm, old, None, a, w, 0.2, 0.3, 0.0)
                bound = torch.nan_to_num(plain[2], nan=4e-6, posinf=4e-6)
                for l in (loss, alone):
                    ref.close(l[:2], plain[0][:2], bound[:2])
                assert out.isfinite().all()
