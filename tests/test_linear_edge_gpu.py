"""Layer products at the edges of what they accept.  Bounds as in test_linear_gpu."""
import pytest
import torch

import paper_2605_29843_b200 as harp
from test_linear_gpu import bf16_want, check, group_rows, normal, offsets_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_weights_of_one_row(rows):
    """d_out = 1: the row's own stride says nothing, the groups' is the leading dimension."""
    sizes, d_in = [rows, 0, 7], 100
    n, off = sum(sizes), offsets_of(sizes)
    x, gy = normal(1, n, d_in).to(torch.bfloat16), normal(2, n, 1).to(torch.bfloat16)
    base = normal(3, len(sizes), 2, 112).to(torch.bfloat16)
    for w in (base[:, :1, :d_in], base[:, 0, :d_in].unsqueeze(1), base.as_strided((3, 1, d_in), (112, 1, 1)), base.as_strided((3, 1, d_in), (d_in, 7, 1))):
        y = harp.grouped_linear(x, w, off, out_dtype=torch.float32)
        gx = harp.grouped_grad_rows(gy, w, off, out_dtype=torch.float32)
        full = torch.full((len(sizes), 120), -3.0, device="cuda")
        gw = harp.grouped_grad_weights(gy, x, off, out=full[:, :d_in].unsqueeze(1))
        for e, r in group_rows(sizes):
            check(y[r], *bf16_want(x[r], w[e], torch.float32))
            check(gx[r], *bf16_want(gy[r], w[e].T, torch.float32))
            check(gw[e], *bf16_want(gy[r].T, x[r].T, torch.float32))
        assert (full[:, d_in:] == -3).all()
    with pytest.raises(ValueError):
        harp.grouped_linear(x, base.as_strided((3, 1, d_in), (d_in - 1, d_in, 1)), off)


def test_no_offsets():
    x, gy, off = normal(1, 4, 8).to(torch.bfloat16), normal(2, 4, 8).to(torch.bfloat16), torch.empty(0, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        harp.grouped_grad_weights(gy, x, off)
    with pytest.raises(harp.HarpError):
        harp.grouped_grad_weights(gy, x, offsets_of([]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_out", [1, 2])
def test_no_rows_and_results_far_apart(d_out, dtype):
    """Rows of a cleared result 2^31 bytes apart and more; a padded copy afterwards."""
    d_in, ld = 5, 2 ** 31 // dtype.itemsize + 8
    flat = torch.full((ld + 16,), 2.0, dtype=dtype, device="cuda")
    gw = flat.as_strided((1, d_out, d_in), (d_out * ld, ld, 1))
    harp.grouped_grad_weights(torch.empty((0, d_out), dtype=torch.bfloat16, device="cuda"), torch.empty((0, d_in), dtype=torch.bfloat16, device="cuda"),
                              offsets_of([0]), out=gw)
    assert (gw == 0).all() and (flat[d_in:ld] == 2).all() and (flat[ld + d_in:] == 2).all()
    x, w = normal(1, 9, 33).to(torch.bfloat16), normal(2, 1, 7, 33).to(torch.bfloat16)
    check(harp.grouped_linear(x, w, offsets_of([9]), out_dtype=torch.float32), *bf16_want(x, w[0], torch.float32))
