"""Layer products against their definitions in 64 bits: rows to 8 bits, the 8-bit product, products grouped by expert and their
gradients.

Bounds.  8 bits: the sum is exact in 32-bit integers, so the result carries its rounding to fp32 and those of two scales (three half
steps, 3 * 2^-24 of the value, 2^-22 with room for their product terms), and that of the output type.  bf16: d products summed in fp32 by a tensor core that may cut
off instead of rounding, a step (2^-23) of the sum of magnitudes an addition at most: d * 2^-23 * sum |x||w|, two more for the last
additions, and the output type's half step of the value."""
import math
import random

import pytest
import torch

import paper_2605_29843_b200 as harp

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 2.0 ** -126


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(seed, *shape):
    return torch.randn(shape, generator=gen(seed), device="cuda")


def eight_bits(seed, *shape):
    return torch.randint(-128, 128, shape, generator=gen(seed), device="cuda", dtype=torch.int32).to(torch.int8)


def scales(seed, *shape):
    return torch.rand(shape, generator=gen(seed), device="cuda") * 0.1 + 1e-3


def offsets_of(sizes, start=0):
    o = [start]
    for n in sizes:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device="cuda")


def padded(t, ld):
    """The same matrix (or matrices) with a longer leading dimension, its padding poisoned."""
    full = torch.full((*t.shape[:-1], ld), float("nan") if t.is_floating_point() else 77, dtype=t.dtype, device="cuda")
    full[..., :t.shape[-1]] = t
    return full[..., :t.shape[-1]]


def check(y, want, bound):
    far = (y.double() - want).abs() - bound
    assert not torch.isnan(far).any()
    assert far.max().item() <= 0 if far.numel() else True, far.max().item()
    assert harp.harp_linear_error_word() == 0


def i8_want(x, sx, w, sw, dtype):
    y = (x.double() @ w.double().T) * sx.double()[:, None] * sw.double()
    return y, y.abs() * (2.0 ** -22 + HALF[dtype]) + TINY


def bf16_want(a, b, dtype):
    """a b^T and its bound"""
    a, b = a.double(), b.double()
    y = a @ b.T
    return y, (a.shape[1] + 2) * 2.0 ** -23 * (a.abs() @ b.abs().T) + y.abs() * HALF[dtype] + TINY


# ---- rows to 8 bits

def quantised(x):
    most = x.double().abs().amax(1)
    t = 127 * x.double() / torch.where(most > 0, most, 1.0)[:, None]
    return t.round().to(torch.int8), (most / 127).float()      # (torch divides fp32 by a number through its reciprocal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 8), (3, 7), (5, 16), (1, 14336), (300, 2048), (7, 4096), (3, 5120), (2, 11008),
                                    (1, 28672), (4, 28672), (297, 4104), (2, 65536), (1, 1 << 20), (33, 1000), (9, 1001)])
def test_quantize_rows(rows, d, dtype):
    x = (normal(rows * d, rows, d) * torch.exp(4 * normal(d, 1, d))).to(dtype)
    q, s = harp.quantize_rows(x)
    want, scale = quantised(x)
    assert torch.equal(q, want) and torch.equal(s, scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_ties_and_ranges(dtype):
    """Halves of the largest value and other exact ties; rows of the smallest and largest magnitudes."""
    rows = []
    for most in (1.0, 1.984375, 127.0, 254.0, 2.0 ** -120, 2.0 ** -133, 2.0 ** -126, 2.0 ** 127, 3.0e38, 1e-30, 130.0):
        k = torch.arange(-127, 128, device="cuda").double()
        v = torch.cat([(k + 0.5) * most / 127, k * most / 254, torch.tensor([most, -most, most / 2, -most / 2], device="cuda").double()])
        rows.append(v.clamp(-most, most).float().to(dtype))
    x = torch.stack(rows)
    for cols in (x.shape[1], 520):                     # element by element, and in pieces
        x = torch.cat([x, torch.zeros((x.shape[0], cols - x.shape[1]), dtype=dtype, device="cuda")], 1)
        q, s = harp.quantize_rows(x)
        want, scale = quantised(x)
        assert torch.equal(q, want) and torch.equal(s, scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [40, 41, 4096])
def test_quantize_zero_and_unfinite_rows(dtype, d):
    x = normal(d, 6, d).to(dtype)
    x[1] = 0
    x[2] = -0.0
    x[3, d - 1] = float("inf")
    x[4, 0] = float("-inf")
    x[5, d // 2] = float("nan")
    q, s = harp.quantize_rows(x)
    assert (q[1:] == 0).all() and (s[1:3] == 0).all() and torch.isnan(s[3:]).all()
    assert torch.equal(q[:1], quantised(x[:1])[0])
    y = harp.linear_i8(q, s, eight_bits(1, 5, d), scales(2, 5))
    assert (y[1:3] == 0).all() and torch.isnan(y[3:]).all() and torch.isfinite(y[0]).all()


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_quantize_strides(shift):
    base = normal(9, 10, 300).to(torch.bfloat16)
    x = base[:, shift:shift + 160]
    out = torch.full((10, 200), 99, dtype=torch.int8, device="cuda")
    q, s = harp.quantize_rows(x, out=out[:, 16:176])
    want, scale = quantised(x)
    assert torch.equal(q, want) and torch.equal(s, scale)
    assert (out[:, :16] == 99).all() and (out[:, 176:] == 99).all()


# ---- the 8-bit product

@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d_in,d_out", [
    (1, 1, 1), (1, 16, 8), (1, 4096, 4096), (2, 128, 130), (5, 2048, 1001), (8, 14336, 512), (9, 512, 14336), (15, 17, 33), (16, 4096, 2048),
    (17, 2048, 300), (31, 100, 100), (33, 8192, 640), (64, 4096, 4096), (65, 1000, 129), (100, 11008, 256), (128, 2048, 5120), (129, 256, 257),
    (255, 5120, 384), (256, 4096, 4096), (257, 272, 513), (300, 4097, 1023), (513, 128, 2048), (1000, 2048, 2048), (2051, 1024, 4096), (4100, 384, 600)])
def test_linear_i8(rows, d_in, d_out, out):
    x, w = eight_bits(rows, rows, d_in), eight_bits(d_out + 7, d_out, d_in)
    sx, sw = scales(1, rows), scales(2, d_out)
    check(harp.linear_i8(x, sx, w, sw, out_dtype=out), *i8_want(x, sx, w, sw, out))


def test_linear_i8_extremes():
    """Sums at the ends of 32 bits."""
    d = 131071
    for rows in (1, 20, 40):
        x = torch.full((rows, d), -128, dtype=torch.int8, device="cuda")
        w = torch.full((24, d), -128, dtype=torch.int8, device="cuda")
        w[1::2] = 127
        one = torch.ones(24, device="cuda")
        y = harp.linear_i8(x, torch.ones(rows, device="cuda"), w, one, out_dtype=torch.float32)
        assert (y[:, 0::2] == 128 * 128 * d).all() and (y[:, 1::2].double() - (-128.0 * 127 * d)).abs().max() <= 128 * 127 * d * 2.0 ** -24
        assert harp.harp_linear_error_word() == 0


@pytest.mark.parametrize("rows", [1, 7, 16, 40, 300])
@pytest.mark.parametrize("ldx,ldw,ldy,sx,sw", [(512, 512, 700, 0, 0), (501, 512, 601, 0, 0), (512, 503, 640, 0, 0), (520, 528, 608, 3, 5)])
def test_linear_i8_strides(rows, ldx, ldw, ldy, sx, sw):
    """Padded and odd leading dimensions and bases; what lies beside the result stays."""
    d_in, d_out = 500, 600
    x, w = eight_bits(rows, rows, ldx)[:, sx:sx + d_in], eight_bits(3, d_out, ldw)[:, sw:sw + d_in]
    x_scale, w_scale = scales(1, rows), scales(2, d_out)
    full = torch.full((rows + 2, ldy), -5.0, dtype=torch.bfloat16, device="cuda")
    y = harp.linear_i8(x, x_scale, w, w_scale, out=full[1:-1, :d_out])
    check(y, *i8_want(x, x_scale, w, w_scale, torch.bfloat16))
    assert (full[0] == -5).all() and (full[-1] == -5).all() and (full[:, d_out:] == -5).all()


# ---- products grouped by expert

GROUPS = [
    ([1], 64, 64), ([5, 0, 3], 128, 96), ([0, 0, 7, 0], 256, 200), ([0], 64, 64), ([16, 16, 16, 16], 512, 512), ([1] * 40, 256, 320),
    ([17, 1, 33, 0, 63, 64, 65], 264, 136), ([300, 0, 5], 2048, 512), ([130, 129, 128, 127], 1001, 515), ([257, 255, 600], 512, 1000),
    ([0, 1000, 0, 24], 4096, 264), ([3] * 129, 72, 72), ([2, 700, 31, 1], 40, 24), ([515], 1, 1), ([127, 1, 70, 15], 4096, 4096),
    ([751, 383, 10], 4096, 2048), ([40, 60], 1, 300), ([40, 60], 300, 1)]


def group_rows(sizes, start=0):
    at = start
    for e, n in enumerate(sizes):
        yield e, slice(at, at + n)
        at += n


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sizes,d_in,d_out", GROUPS)
def test_grouped_linear(sizes, d_in, d_out, out):
    """Rows before the first group and behind the last one are left as they were."""
    n = sum(sizes) + 5
    x, w = normal(1, n, d_in).to(torch.bfloat16), normal(2, len(sizes), d_out, d_in).to(torch.bfloat16)
    x[:2] = float("nan")
    x[n - 3:] = float("inf")
    y = torch.full((n, d_out), -3.0, dtype=out, device="cuda")
    harp.grouped_linear(x, w, offsets_of(sizes, 2), out=y)
    for e, r in group_rows(sizes, 2):
        check(y[r], *bf16_want(x[r], w[e], out))
    assert (y[:2] == -3).all() and (y[n - 3:] == -3).all()


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sizes,d_in,d_out", GROUPS)
def test_grouped_linear_i8(sizes, d_in, d_out, out):
    n = sum(sizes) + 5
    x, w = eight_bits(1, n, d_in), eight_bits(2, len(sizes), d_out, d_in)
    sx, sw = scales(3, n), scales(4, len(sizes), d_out)
    y = torch.full((n, d_out), -3.0, dtype=out, device="cuda")
    harp.grouped_linear_i8(x, sx, w, sw, offsets_of(sizes, 2), out=y)
    for e, r in group_rows(sizes, 2):
        check(y[r], *i8_want(x[r], sx[r], w[e], sw[e], out))
    assert (y[:2] == -3).all() and (y[n - 3:] == -3).all()


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sizes,d_in,d_out", GROUPS)
def test_grouped_grad_rows(sizes, d_in, d_out, out):
    n = sum(sizes) + 5
    gy, w = normal(1, n, d_out).to(torch.bfloat16), normal(2, len(sizes), d_out, d_in).to(torch.bfloat16)
    gy[:2] = float("nan")
    gy[n - 3:] = float("inf")
    gx = torch.full((n, d_in), -3.0, dtype=out, device="cuda")
    harp.grouped_grad_rows(gy, w, offsets_of(sizes, 2), out=gx)
    for e, r in group_rows(sizes, 2):
        check(gx[r], *bf16_want(gy[r], w[e].T, out))
    assert (gx[:2] == -3).all() and (gx[n - 3:] == -3).all()


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("sizes,d_in,d_out", GROUPS)
def test_grouped_grad_weights(sizes, d_in, d_out, accumulate, out):
    """The rows around a group, whose values are not finite, leave no trace in it."""
    n = sum(sizes) + 5
    gy, x = normal(1, n, d_out).to(torch.bfloat16), normal(2, n, d_in).to(torch.bfloat16)
    gy[:2], x[n - 3:] = float("nan"), float("inf")
    if len(sizes) > 2 and sizes[2]:                   # ... nor does a group whose rows are not finite in others
        x[2 + sizes[0] + sizes[1]] = float("inf")
    before = normal(5, len(sizes), d_out, d_in).to(out)
    gw = before.clone()
    harp.grouped_grad_weights(gy, x, offsets_of(sizes, 2), out=gw, accumulate=accumulate)
    for e, r in group_rows(sizes, 2):
        if e == 2 and sizes[2]:
            assert not torch.isfinite(gw[e]).all()
            continue
        want, bound = bf16_want(gy[r].T, x[r].T, out)
        if accumulate:
            want = want + before[e].double()
            bound = bound + want.abs() * HALF[out] + before[e].double().abs() * 2.0 ** -23
        check(gw[e], want, bound)


@pytest.mark.parametrize("d_in,d_out,ld_in,ld_out", [(200, 136, 256, 200), (201, 137, 208, 144), (64, 64, 72, 72), (203, 139, 203, 140), (77, 33, 81, 35)])
@pytest.mark.parametrize("sizes", [[5, 0, 27], [300, 40]])
def test_padding_leaves_no_trace(sizes, d_in, d_out, ld_in, ld_out):
    """Rows longer than they say, NaN behind their ends, on the 16-byte grid and off it; what lies beside a result stays."""
    n, off = sum(sizes), offsets_of(sizes)
    x, gy = padded(normal(1, n, d_in).to(torch.bfloat16), ld_in), padded(normal(2, n, d_out).to(torch.bfloat16), ld_out)
    w = padded(normal(3, len(sizes), d_out, d_in).to(torch.bfloat16), ld_in)
    full = [torch.full((n, d_out + 3), -3.0, device="cuda"), torch.full((n, d_in + 5), -3.0, device="cuda"),
            torch.full((len(sizes), d_out, d_in + 7), -3.0, device="cuda")]
    y, gx, gw = full[0][:, :d_out], full[1][:, :d_in], full[2][..., :d_in]
    harp.grouped_linear(x, w, off, out=y)
    harp.grouped_grad_rows(gy, w, off, out=gx)
    harp.grouped_grad_weights(gy, x, off, out=gw)
    for e, r in group_rows(sizes):
        check(y[r], *bf16_want(x[r], w[e], torch.float32))
        check(gx[r], *bf16_want(gy[r], w[e].T, torch.float32))
        check(gw[e], *bf16_want(gy[r].T, x[r].T, torch.float32))
    assert (full[0][:, d_out:] == -3).all() and (full[1][:, d_in:] == -3).all() and (full[2][..., d_in:] == -3).all()


@pytest.mark.parametrize("d", [9000, 20000])
def test_long_fp32_sums(d):
    """Sums of d products of one sign, which a tensor core's truncation would shrink by 1e-9 of the sum each: runs of 512 keep the error
    below that of 512 additions cut off (2^-23 each) and d / 512 rounded ones."""
    x, w = normal(1, 300, d).abs().to(torch.bfloat16), normal(2, 1, 256, d).abs().to(torch.bfloat16)
    bound = 512 * 2.0 ** -23 / 16 + (d / 512 + 2) * 2.0 ** -24        # sixteen products an addition
    for rows in (8, 300):
        y = harp.grouped_linear(x[:rows], w, offsets_of([rows]), out_dtype=torch.float32).double()
        want = x[:rows].double() @ w[0].double().T
        assert ((y - want).abs() / want).max() <= bound
    gw = harp.grouped_grad_weights(w[0].T.contiguous(), x.T.contiguous()[:, :296], offsets_of([d])).double()[0]
    want = w[0].double() @ x[:296].double().T
    assert ((gw - want).abs() / want).max() <= bound
