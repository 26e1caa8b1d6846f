"""Numbers that the operators' calls take and refuse, at the ends of what their kernels can serve; no GPU is needed: calls without rows launch nothing."""
import ctypes as C
import math

import pytest

OK, INVALID = 0, -1
FAKE = 0x1000  # aligned, never read: no call here launches


@pytest.fixture(scope="module")
def lib():
    import paper_2107_14575_amd as dq
    return dq.load_library()


def no_rows():
    from paper_2107_14575_amd.binding import Logits
    return Logits(data_dev=FAKE, dtype=0, batch=1, rows=0, vocab=100, batch_stride=0, row_stride=100)


# log2(e) / T has to be a number of binary32, and where a difference of two logits passes binary32 the exponential has to be 0: beyond T = 3.27e36
# log2(e) / T times the largest binary32 number is below 150, beyond 1e38 the factor is subnormal, beyond 2e45 it is 0 and 0 times infinity NaN.
TEMPERATURES = [(5e-39, OK), (1e-30, OK), (1.0, OK), (1e30, OK), (3.2e36, OK), (3.4e36, INVALID), (1e37, INVALID), (2e38, INVALID), (1e45, INVALID), (3e45, INVALID),
                (1e300, INVALID), (4e-39, INVALID)]


@pytest.mark.parametrize("temperature,want", TEMPERATURES, ids=str)
def test_temperatures(lib, temperature, want):
    m = no_rows()
    assert lib.dq_token_logprob(m, FAKE, temperature, FAKE, None, FAKE, None) == want
    assert lib.dq_token_logprob_backward(m, FAKE, temperature, FAKE, FAKE, 1.0, m, None) == want
    if want != OK:  # these two write their sums without rows as well
        assert lib.dq_policy_loss(m, FAKE, temperature, FAKE, None, FAKE, FAKE, 0.2, 0.2, 0.0, 1.0, FAKE, FAKE, None, FAKE, None) == want
        assert lib.dq_preference_loss(m, FAKE, temperature, FAKE, 2, None, 0.1, 0.0, 0, 1.0, FAKE, FAKE, None, FAKE, None) == want


def test_no_product_passes_the_range():
    """What the temperatures rest on: the factor at the largest one makes the overflown difference worth 2^-150 or less, which binary32 does not hold."""
    largest = float(2 ** 128 - 2 ** 104)
    assert 1 / math.log(2) / 3.2e36 * largest >= 150 > 1 / math.log(2) / 3.4e36 * largest
    assert C.c_float(1 / math.log(2) / 3e45).value == 0.0 and math.isinf(C.c_float(1 / math.log(2) / 4e-39).value)
