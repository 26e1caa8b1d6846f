"""Every element of a row counts once, in every form of the kernels over logits: at heads, tails, the seams between registers, LDS, what is read again, and slices.

Row r has the logit 0 at the elements v = r (mod rows) and at its token, and -inf elsewhere.  Its sum is then a number n of ones, exact in binary32 in any order, so that
logp = -ln n to the accuracy of one logarithm and a probability is 1/n to that of one division: an element that is left out or counted twice, anywhere, moves
logp by 1/n, hundreds of times the bound.  The rows together have each element of the vocabulary once.

Random rows go through the same forms with a bound that has the additions which these make: 4 roundings a vector of a thread, not one for each 64 elements."""
import math

import pytest
import torch

from tests import operator_ref as ref
from tests.test_gpu_token_logprob import TYPES, dq, make_logits  # noqa: F401  (dq is a fixture)

pytestmark = pytest.mark.gpu

U = ref.U
PER = {torch.float32: 4, torch.float16: 8, torch.bfloat16: 8}
SLICED_ROWS, SLICED_VECS = 64, 8192  # up to so many rows of at least so many vectors are sliced
# vectors of a row: the ends of what each fused form holds in registers, 16384 with 9216 more in LDS, and rows of which some vectors are read again
VECS = [0, 1, 16, 17, 32, 33, 64, 65, 128, 129, 256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 25600, 25601, 30001]


def room(rows, vocab, dtype, how):
    """Memory for rows of logits: contiguous, or at every alignment with room between."""
    if how == "contiguous":
        return torch.empty((rows, vocab), dtype=dtype, device="cuda")
    return torch.empty(rows * (vocab + 3) + 1, dtype=dtype, device="cuda")[1:].view(rows, vocab + 3)[:, :vocab]


def classes(rows, vocab, dtype, how):
    """-> logits, tokens, the count of ones of each row"""
    z = room(rows, vocab, dtype, how)
    z.fill_(-math.inf)
    v = torch.arange(vocab, device="cuda")
    z[v % rows, v] = 0.0
    r = torch.arange(rows, device="cuda")
    y = (r * 7919 + 13) % vocab
    z[r, y] = 0.0
    n = torch.bincount(v % rows, minlength=rows) + (y % rows != r)
    return z, y, n


def same(got, want, relative, tiny=0.0):
    """Within so much of the value wanted, on the GPU, and `tiny`, the rounding of a type's subnormals; what is to be 0 exactly."""
    got = got.double()
    off = (got - want).abs()
    assert not got.isnan().any() and bool((off <= relative * want.abs() + tiny * (want != 0)).all()), float((off / want.abs().clamp(min=1e-30)).max())


def gradient(z, y, n, d):
    p = torch.where(z.double() == 0.0, 1.0 / n.double()[:, None], 0.0)
    g = -p * d[:, None]
    g[torch.arange(len(y), device="cuda"), y] += d
    return g


def check(dq, rows, vocab, dtype, how, stream=None):
    z, y, n = classes(rows, vocab, dtype, how)
    new = lambda *s: torch.full(s, math.nan, device="cuda")  # noqa: E731
    u, tiny = ref.TYPE_U[dtype]
    logp_want = -n.double().log()

    # forward with and without what the backward pass takes
    logp, only, softmax = new(rows), new(rows), new(rows, 2)
    ws = torch.empty(dq.token_logprob_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    dq.token_logprob(z, y, logp, ws, softmax_out=softmax, stream=stream)
    dq.token_logprob(z, y, only, ws, stream=stream)
    torch.cuda.synchronize()
    same(logp, logp_want, 4 * U)
    assert torch.equal(only, logp)
    assert not softmax[:, 0].any()
    same(softmax[:, 1], 1.0 / n.double(), 2 * U)

    # backward: d = 1, so that the token's own element is 1 - 1/n, a subtraction of numbers at least 1/2 apart where n > 1 and exactly 0 where n = 1
    out = room(rows, vocab, dtype, how)
    out.fill_(math.nan)
    ones = torch.ones(rows, device="cuda")
    torch.cuda.synchronize()
    dq.token_logprob_backward(z, y, softmax, ones, out, stream=stream)
    torch.cuda.synchronize()
    want = gradient(z, y, n, ones.double())
    same(out, want, 8 * U + u, tiny)

    # the policy loss: ratio 1, advantage -1, so that dL/dlogp = weight
    loss, logp, grad, alone = new(4), new(rows), room(rows, vocab, dtype, how), new(4)
    grad.fill_(math.nan)
    weights = torch.ones(rows, device="cuda")
    ws = torch.empty(dq.policy_loss_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
    old = only.clone()  # so that the ratio is 1 exactly: the same logits, and s exact in any order
    torch.cuda.synchronize()
    dq.policy_loss(z, y, old, -ones, weights, loss, logp, grad, ws, stream=stream)
    dq.policy_loss(z, y, old, -ones, weights, alone, only, None, ws, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(logp, old) and torch.equal(only, old)
    sums = torch.tensor([rows, rows, 0, 0], dtype=torch.float64, device="cuda")
    same(loss, sums, 4 * U)
    same(alone, sums, 4 * U)
    same(grad, want, 8 * U + u, tiny)
    dq.policy_loss(z, y, old, -ones, weights, loss, logp, z, ws, stream=stream)  # in place
    torch.cuda.synchronize()
    assert torch.equal(z, grad) and torch.equal(logp, old)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vecs", VECS)
def test_every_element_counts_once(dq, dtype, vecs):
    """More rows than are sliced: the fused forms, in one launch each."""
    rows = SLICED_ROWS + 3
    side = torch.cuda.Stream()
    for extra in (0, PER[dtype] - 1) if vecs else (1, PER[dtype] - 1):
        for how in ("contiguous", "odd"):
            check(dq, rows, vecs * PER[dtype] + extra, dtype, how)
        check(dq, rows, vecs * PER[dtype] + extra, dtype, "odd", side)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vecs", [8192, 8193, 9215, 9216, 16384, 30001, 65536, 65537])
def test_every_element_counts_once_in_slices(dq, dtype, vecs):
    """Slices of 1024 vectors, or of 2048 beyond 65536; few rows by the last slice to arrive, and more by a kernel a row."""
    side = torch.cuda.Stream()
    for rows in (1, 2, 11, SLICED_ROWS):
        if rows * vecs > 11 * 65537:
            continue
        for stream in (None, side):
            check(dq, rows, vecs * PER[dtype] + 3, dtype, "odd", stream)
    assert vecs >= SLICED_VECS


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,vecs", [(600, 2000), (600, 3000), (1100, 700), (1100, 2049), (1100, 5000)])
def test_every_element_counts_once_in_many_rows(dq, dtype, rows, vecs):
    """The forms of calls of many rows: more than 512 for the fused kernel, 1024 for the forward pass."""
    check(dq, rows, vecs * PER[dtype] + 1, dtype, "odd")


def tight(z, y, rows, temperature=1.0):
    """ref.softmax, whose bounds have a sum's additions as these kernels make them: 256 threads a row in forward passes of 1024 rows, otherwise 1024 from 2049 vectors on, and
    the same in the fused forms of up to 512 rows; a slice's threads have fewer vectors.  In units of 2^-24: a vector is an addition to its thread's sum and a rescaling of that (a product,
    and 2 for its factor's exponential; the error of that one's argument is in the elements' own) beside a tree of 3 and 2 for an element's exponential; two joins over
    lanes and one over slices are 6 additions and a rescaling each."""
    sm = ref.softmax(z, y, temperature)
    vecs = z.shape[1] // PER[z.dtype]
    chain = math.ceil(vecs / (16 if vecs <= 128 else 64 if vecs <= 512 else 256 if vecs <= 2048 or rows >= 1024 else 1024)) + 1
    loose = U * (z.shape[1] / 64 + 18)
    own = U * (4 * chain + 3 + 2 + 3 * (6 + 3))
    better = min(own - loose, 0.0)  # short rows' bound was as tight as this one
    for key in ("sum", "logp_err", "p_err"):
        sm[key] = sm[key] + better
    return sm


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vecs", [2047, 4095, 8191, 8193, 16383, 16385, 25599, 25601, 30001])
def test_random_rows_in_the_longest_forms(dq, dtype, vecs):
    """Against binary64, in a call of more rows than are sliced, most of which do not count."""
    rows, vocab, counted = SLICED_ROWS + 5, vecs * PER[dtype] + 5, [0, 1, 33, 64, 67]
    z, y, gen = make_logits(len(counted), vocab, dtype, vecs)
    side = torch.cuda.Stream()
    for temperature in (1.0, 0.7):
        sm = tight(z, y, rows, temperature)
        old = sm["logp"].float() - torch.randn(len(counted), generator=gen) * 0.1
        adv, w, reference = torch.randn(len(counted), generator=gen), torch.rand(len(counted), generator=gen) / 5, sm["logp"].float() + 0.3
        sums, d, sum_err, d_err, lp = ref.policy(sm, old, reference, adv, w, 0.2, 0.2, 0.1)
        want, bound = ref.dlogits(sm, d, temperature, d_err=d_err, dtype=dtype)
        plain, plain_bound = ref.dlogits(sm, adv.double(), temperature, dtype=dtype)
        for how, stream in (("contiguous", None), ("odd", None), ("odd", side)):
            at = room(rows, vocab, dtype, how)
            at.fill_(math.nan)
            at[counted] = z.cuda()

            def spread(values, fill):
                all_rows = torch.full((rows,), fill, dtype=values.dtype, device="cuda")
                all_rows[counted] = values.cuda()
                return all_rows
            tokens, weights = spread(y, 3), spread(w, 0.0)
            out = room(rows, vocab, dtype, how)
            out.fill_(math.nan)
            loss, logp = torch.full((4,), math.nan, device="cuda"), torch.full((rows,), math.nan, device="cuda")
            ws = torch.empty(dq.policy_loss_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
            args = [spread(t, math.nan) for t in (old, adv)]
            ref_logp = spread(reference, math.nan)
            rest = [r for r in range(rows) if r not in counted]
            torch.cuda.synchronize()
            for destination in (out, at):  # then in place
                dq.policy_loss(at, tokens, *args, weights, loss, logp, destination, ws, ref_logp=ref_logp, clip_low=0.2, clip_high=0.2, beta=0.1, temperature=temperature, stream=stream)
                torch.cuda.synchronize()
                ref.close(loss, sums, sum_err)
                ref.close(logp[counted], lp, sm["logp_err"])
                ref.close(destination[counted], want, bound)
                assert not destination[rest].any() and not logp[rest].any()
            # the same rows forward, with and without what the gradient takes, and backward
            at.fill_(math.nan)
            at[counted] = z.cuda()
            tokens = spread(y, -100)
            softmax, only = torch.full((rows, 2), math.nan, device="cuda"), torch.full((rows,), math.nan, device="cuda")
            logp.fill_(math.nan), out.fill_(math.nan)
            ws = torch.empty(dq.token_logprob_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
            dlogp = spread(adv, math.nan)
            torch.cuda.synchronize()
            dq.token_logprob(at, tokens, logp, ws, softmax_out=softmax, temperature=temperature, stream=stream)
            dq.token_logprob(at, tokens, only, ws, temperature=temperature, stream=stream)
            dq.token_logprob_backward(at, tokens, softmax, dlogp, out, temperature=temperature, stream=stream)
            torch.cuda.synchronize()
            for values in (logp, only):
                ref.close(values[counted], sm["logp"], sm["logp_err"])
                assert not values[rest].any()
            ref.close(out[counted], plain, plain_bound)
            assert not out[rest].any()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,vocab", [(1, 131072), (3, 262147), (20, 65536), (5, 50001), (70, 12000), (30, 5000), (1030, 9001)])
def test_random_rows_forward(dq, dtype, rows, vocab):
    """The forward pass with and without softmax_out against binary64, rows that do not count and a NaN among them."""
    z, y, gen = make_logits(rows, vocab, dtype, rows)
    sm = tight(z, y, rows)
    if rows > 2:
        y[1], z[2, 5] = -100, math.nan
        sm["logp"][1], sm["logp"][2] = 0.0, math.nan
    ws = torch.empty(dq.token_logprob_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
    zd, yd = z.cuda(), y.cuda()
    for stream in (None, torch.cuda.Stream()):
        for softmax in (None, torch.full((rows, 2), math.nan, device="cuda")):
            logp = torch.full((rows,), 7.0, device="cuda")
            torch.cuda.synchronize()
            dq.token_logprob(zd, yd, logp, ws, softmax_out=softmax, stream=stream)
            torch.cuda.synchronize()
            ref.close(logp, sm["logp"], sm["logp_err"])
