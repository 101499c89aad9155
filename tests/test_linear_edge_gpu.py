"""Layer products at the edges of what they accept.  Bounds as in test_linear_gpu."""
import pytest
import torch

import paper_2605_29843_b200 as harp
from test_linear_gpu import bf16_want, check, normal, offsets_of

pytestmark = pytest.mark.gpu


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
