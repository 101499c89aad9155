"""Limits of rows to 8 bits, as the header states them (runs without a GPU)."""
import pytest

import paper_2605_29843_b200 as harp
from paper_2605_29843_b200 import build as harp_build

OK, DIM, LARGE = 0, 2, 11
P = 1 << 20         # an address that is never followed


@pytest.fixture(scope="module", autouse=True)
def _built():
    harp_build.build()


@pytest.mark.parametrize("ld_x,ld_q,n,d,code", [
    ((1 << 37) + 1, 64, 4, 64, LARGE), (64, (1 << 37) + 1, 4, 64, LARGE), (1 << 62, 1 << 62, 4, 64, LARGE), (1 << 62, 64, 1, 64, LARGE),
    (63, 1 << 62, 4, 64, DIM), (1 << 37, 1 << 37, 0, 64, OK), (64, 64, 1 << 31, 64, DIM), (1 << 21, 1 << 21, 4, (1 << 20) + 1, DIM)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_quantiser_limits(ld_x, ld_q, n, d, code, dtype):
    assert harp.lib().harp_quantize_rows(P, ld_x, n, d, dtype, P, ld_q, P, None) == code
