"""bf16 results of long sums: the tensor core cuts its fp32 sums off, so that one run of products over a million rows would come out
more than a bf16 step too small.

Bound, for products of one sign.  An addition that is cut off loses at most a step (2^-23) of the sum: m 2^-23 for a run of m
products, runs of 512 where more than 32768 are summed; n / 512 additions of runs, rounded to nearest (2^-24 each), and the result's
half step (2^-8)."""
import pytest
import torch

import paper_2605_29843_b200 as harp
from test_linear_gpu import bf16_want, check, gen, group_rows, normal, offsets_of

pytestmark = pytest.mark.gpu

LONE, RUN = 32768, 512


def uniform(seed, *shape):
    return torch.rand(shape, generator=gen(seed), device="cuda").to(torch.bfloat16)


def one_sign(y, want, n):
    summed = (RUN if n > LONE else n) * 2.0 ** -23 + (n / RUN + 2) * 2.0 ** -24
    far = ((y.double() - want).abs() / want).max().item()
    assert far <= summed * (1 + 2.0 ** -8) + 2.0 ** -8, far
    assert harp.harp_linear_error_word() == 0


@pytest.mark.parametrize("rows", [1, 8, 100, 300])
@pytest.mark.parametrize("d", [LONE, 1 << 17, 1 << 20])
def test_long_contracted_dimension(rows, d):
    x, w = uniform(1, rows, d), uniform(2, 1, 256, d)
    one_sign(harp.grouped_linear(x, w, offsets_of([rows])), x.double() @ w[0].double().T, d)
    w = w.view(1, d, 256)
    one_sign(harp.grouped_grad_rows(x, w, offsets_of([rows])), x.double() @ w[0].double(), d)


@pytest.mark.parametrize("rows", [1 << 17, 1 << 20, (1 << 20) + 3])
def test_long_groups(rows):
    gy, x = uniform(3, rows, 64), uniform(4, rows, 200)
    want = sum(gy[r:r + (1 << 17)].double().T @ x[r:r + (1 << 17)].double() for r in range(0, rows, 1 << 17))
    one_sign(harp.grouped_grad_weights(gy, x, offsets_of([rows]), out_dtype=torch.bfloat16)[0], want, rows)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("d_in,d_out", [(72, 264), (35, 33)])
def test_long_and_short_groups_of_one_call(d_in, d_out, accumulate):
    """Lengths on both sides of the limit, empty groups among them, rows around the groups that are not finite."""
    sizes = [100, LONE + 1, 0, LONE, 3 * LONE + 17, 1, 0]
    n = sum(sizes) + 5
    gy, x = normal(1, n, d_out).to(torch.bfloat16), normal(2, n, d_in).to(torch.bfloat16)
    gy[:2], x[n - 3:] = float("nan"), float("inf")
    before = normal(5, len(sizes), d_out, d_in).to(torch.bfloat16)
    gw = before.clone()
    harp.grouped_grad_weights(gy, x, offsets_of(sizes, 2), out=gw, accumulate=accumulate)
    for e, r in group_rows(sizes, 2):
        want, bound = bf16_want(gy[r].T, x[r].T, torch.bfloat16)
        if accumulate:
            want = want + before[e].double()
            bound = bound + want.abs() * 2.0 ** -8 + before[e].double().abs() * 2.0 ** -23
        check(gw[e], want, bound)
