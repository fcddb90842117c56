"""What the checks of long attention results accept and reject, on results spoilt on purpose in the model.  No kernel runs."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import workloads as wl
from tests.cache_utils import NORM_LIMIT, bf16, norm_error


@pytest.fixture(scope="module")
def case():
    """One row of two heads over 24901 tokens, as the longest of the GPU tests has them."""
    rng = np.random.default_rng(0)
    n, d = 24901, 128
    k, v = (np.moveaxis(co.dequantize(*co.quantize(bf16(rng, (n, 1, d)))), 0, 1) for _ in range(2))
    q = bf16(rng, (1, 2, d))
    want, w = co.attend(q, k, v, n, d ** -0.5)
    return v, want, w


def spoilt(case, weight):
    """The result with the keys' weights times `weight` (and their sum, as a kernel's would be)."""
    v, _, w = case
    out = np.stack([(w[0, h] * weight) @ v[0] / max((w[0, h] * weight).sum(), 1e-30) for h in range(2)])[None]
    return wl.round_to_bf16(out.astype(np.float32))


def test_the_rounded_result_is_within_the_norm(case):
    assert norm_error(spoilt(case, np.ones(24901)), case[1]).max() <= 2.0 ** -8


@pytest.mark.parametrize("first,last,factor", [(0, 64, 0), (6400, 6464, 0), (6400, 6464, 2), (24896, 24901, 0), (0, 448, 0), (448, 896, 2), (12000, 24901, 0), (0, 24901, 0)])
def test_a_lost_or_doubled_page_or_part_is_not(case, first, last, factor):
    weight = np.ones(24901)
    weight[first:last] = factor
    assert norm_error(spoilt(case, weight), case[1]).max() > NORM_LIMIT


def test_a_row_that_sees_nothing_has_to_be_zero():
    want = np.zeros((1, 1, 64))
    assert norm_error(np.zeros((1, 1, 64)), want).max() == 0
    assert norm_error(np.full((1, 1, 64), 1e-6), want).max() == np.inf
