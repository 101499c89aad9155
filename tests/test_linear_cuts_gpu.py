"""Layer products through every cut of their tiles (columns of a tile, CTAs that divide the contracted dimension, length of the ring), at sizes that
are no multiple of anything, against the definitions in 64 bits.  Bounds as in test_linear_gpu and, for sums of more than 32768 products, as there."""
import pytest
import torch

import paper_2605_29843_b200 as harp
from test_linear_gpu import bf16_want, check, eight_bits, group_rows, i8_want, normal, offsets_of, padded, scales

pytestmark = pytest.mark.gpu

CUTS = [(256, 1, False), (32, 1, False), (32, 1, True), (32, 2, False), (32, 4, False), (64, 1, False), (64, 1, True), (64, 2, False),
        (64, 2, True), (64, 4, False), (64, 4, True)]
OUT = [torch.bfloat16, torch.float32]
# rows of the groups; d_in and d_out; leading dimensions of x and w (d_in), of gy (d_out) and of results, beyond those
SHAPES = [
    ([1], 64, 8, 0, 0, 0),                             # fewer blocks than CTAs of a split
    ([17, 0, 40, 255, 257, 1], 264, 136, 0, 0, 0),     # pieces of 16 bytes, but of no chunk of 64
    ([17, 0, 40, 255, 257, 1], 257, 131, 0, 0, 0),     # off the 16-byte grid: padded copies, element stores
    ([300, 33], 1002, 514, 22, 30, 2),                 # padded rows; results two lanes at a time
    ([31, 64, 65], 1600, 320, 0, 0, 8),                # whole chunks of 64, results beside others
    ([40], 1001, 4100, 7, 12, 1),
    ([513], 4104, 264, 8, 0, 0),
]


@pytest.fixture(params=CUTS, ids=lambda c: "%d-%d-%s" % (c[0], c[1], "long" if c[2] else "short"))
def cut(request):
    harp.harp_linear_set_cut(*request.param)
    yield request.param
    harp.harp_linear_set_cut(0)


def result(n, d, more, dtype):
    full = torch.full((n + 1, d + more), -3.0, dtype=dtype, device="cuda")
    return full, full[:n, :d]


def untouched(full, n, d):
    assert (full[n:] == -3).all() and (full[:, d:] == -3).all()


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("sizes,d_in,d_out,more_in,more_out,more_y", SHAPES)
def test_eight_bits(cut, sizes, d_in, d_out, more_in, more_out, more_y, out):
    n = sum(sizes)
    x, w = padded(eight_bits(1, n, d_in), d_in + more_in), padded(eight_bits(2, len(sizes), d_out, d_in), d_in + more_in)
    sx, sw = scales(3, n), scales(4, len(sizes), d_out)
    full, y = result(n, d_out, more_y, out)
    harp.grouped_linear_i8(x, sx, w, sw, offsets_of(sizes), out=y)
    assert harp.harp_linear_last_cut() == cut
    for e, r in group_rows(sizes):
        check(y[r], *i8_want(x[r], sx[r], w[e], sw[e], out))
    untouched(full, n, d_out)


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("sizes,d_in,d_out,more_in,more_out,more_y", SHAPES)
def test_bf16(cut, sizes, d_in, d_out, more_in, more_out, more_y, out):
    n = sum(sizes)
    x, w = padded(normal(1, n, d_in).to(torch.bfloat16), d_in + more_in), padded(normal(2, len(sizes), d_out, d_in).to(torch.bfloat16), d_in + more_in)
    full, y = result(n, d_out, more_y, out)
    harp.grouped_linear(x, w, offsets_of(sizes), out=y)
    assert harp.harp_linear_last_cut() == cut
    for e, r in group_rows(sizes):
        check(y[r], *bf16_want(x[r], w[e], out))
    untouched(full, n, d_out)


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("sizes,d_in,d_out,more_in,more_out,more_y", SHAPES)
def test_gradient_of_rows(cut, sizes, d_in, d_out, more_in, more_out, more_y, out):
    n = sum(sizes)
    gy, w = padded(normal(1, n, d_out).to(torch.bfloat16), d_out + more_out), padded(normal(2, len(sizes), d_out, d_in).to(torch.bfloat16), d_in + more_in)
    full, gx = result(n, d_in, more_y, out)
    harp.grouped_grad_rows(gy, w, offsets_of(sizes), out=gx)
    assert harp.harp_linear_last_cut() == cut
    for e, r in group_rows(sizes):
        check(gx[r], *bf16_want(gy[r], w[e].T, out))
    untouched(full, n, d_in)


@pytest.mark.parametrize("d", [32769, 40000])
def test_long_sums(cut, d):
    """bf16 results of more than 32768 products: kernels of their own."""
    sizes = [3, 60, 0, 270]
    n = sum(sizes)
    x, w = normal(1, n, d).to(torch.bfloat16), normal(2, len(sizes), 40, d).to(torch.bfloat16)
    y = harp.grouped_linear(x, w, offsets_of(sizes))
    assert harp.harp_linear_last_cut() == cut
    w = w.view(len(sizes), d, 40)
    gx = harp.grouped_grad_rows(x, w, offsets_of(sizes))
    assert harp.harp_linear_last_cut() == cut
    for e, r in group_rows(sizes):
        check(y[r], *bf16_want(x[r], w.view(len(sizes), 40, d)[e], torch.bfloat16))
        check(gx[r], *bf16_want(x[r], w[e].T, torch.bfloat16))


@pytest.mark.parametrize("d_in,d_out", [(1001, 515), (264, 136)])
def test_same_result_in_every_cut(d_in, d_out):
    """8-bit sums are exact, so the cuts give the same bits."""
    sizes = [17, 0, 40, 300]
    n = sum(sizes)
    x, w, sx, sw = eight_bits(1, n, d_in), eight_bits(2, len(sizes), d_out, d_in), scales(3, n), scales(4, len(sizes), d_out)
    want = harp.grouped_linear_i8(x, sx, w, sw, offsets_of(sizes))
    try:
        for c in CUTS:
            harp.harp_linear_set_cut(*c)
            assert torch.equal(harp.grouped_linear_i8(x, sx, w, sw, offsets_of(sizes)), want), c
    finally:
        harp.harp_linear_set_cut(0)


@pytest.mark.parametrize("tiles", ["many", "few"])
def test_captured_beside_another_stream(cut, tiles):
    """More tiles than CTAs of a launch, and one; replayed while the same cut runs on another stream."""
    sizes = [700, 5, 64] * 3 if tiles == "many" else [9]
    n, d_in, d_out = sum(sizes), 520, 1024
    off, w = offsets_of(sizes), normal(2, len(sizes), d_out, d_in).to(torch.bfloat16)
    xs = [normal(s, n, d_in).to(torch.bfloat16) for s in (3, 4)]
    want = [harp.grouped_linear(x, w, off) for x in xs]
    ys = [torch.zeros_like(v) for v in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        harp.grouped_linear(xs[0], w, off, out=ys[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        g.replay()
        with torch.cuda.stream(side):
            harp.grouped_linear(xs[1], w, off, out=ys[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ys, want)) and harp.harp_linear_error_word() == 0
