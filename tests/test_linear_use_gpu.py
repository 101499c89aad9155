"""Layer products as a program uses them: in a chain, captured, on several streams, beside each other, at sizes past 32 bits, and
what the torch conveniences refuse.  Bounds as in test_linear_gpu."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2605_29843_b200 as harp
from oracle import harp_oracle as orc
from paper_2605_29843_b200 import workloads as wl
from test_linear_gpu import bf16_want, check, eight_bits, group_rows, i8_want, normal, offsets_of, scales

pytestmark = pytest.mark.gpu


# ---- offsets

@pytest.mark.parametrize("raw", [[-5, 3, 2, 40, 1000, 7], [50, 50, 50, 50, 50, 50], [0, 64, 64, 10, 12, 64], [2 ** 31 - 1, -2 ** 31, 0, 5, 9, 64],
                                 [-1, -1, -1, -1, -1, -1], [10, 20, 30, 25, 40, 41]])
def test_offsets_are_clamped(raw):
    """Rising and within the batch, whatever they say; the rows that are then in no group stay."""
    n, d_in, d_out, groups = 64, 128, 160, len(raw) - 1
    clamped, most = [], 0
    for o in raw:
        most = max(most, min(max(o, 0), n))
        clamped.append(most)
    off = torch.tensor(raw, dtype=torch.int32, device="cuda")
    x, gy = normal(1, n, d_in).to(torch.bfloat16), normal(2, n, d_out).to(torch.bfloat16)
    w = normal(3, groups, d_out, d_in).to(torch.bfloat16)
    xq, sx, wq, sw = eight_bits(4, n, d_in), scales(5, n), eight_bits(6, groups, d_out, d_in), scales(7, groups, d_out)
    y, yq = (torch.full((n, d_out), -3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gx = torch.full((n, d_in), -3.0, dtype=torch.bfloat16, device="cuda")
    harp.grouped_linear(x, w, off, out=y)
    harp.grouped_linear_i8(xq, sx, wq, sw, off, out=yq)
    harp.grouped_grad_rows(gy, w, off, out=gx)
    gw = harp.grouped_grad_weights(gy, x, off)
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    for e in range(groups):
        r = slice(clamped[e], clamped[e + 1])
        outside[r] = False
        check(y[r], *bf16_want(x[r], w[e], torch.bfloat16))
        check(yq[r], *i8_want(xq[r], sx[r], wq[e], sw[e], torch.bfloat16))
        check(gx[r], *bf16_want(gy[r], w[e].T, torch.bfloat16))
        check(gw[e], *bf16_want(gy[r].T, x[r].T, torch.float32))
    assert (y[outside] == -3).all() and (yq[outside] == -3).all() and (gx[outside] == -3).all()


@pytest.mark.parametrize("groups", [1, 31, 32, 33, 64, 1000, 1024])
def test_many_groups(groups):
    rng = np.random.default_rng(groups)
    sizes = [int(v) for v in rng.integers(0, 4, groups)]
    n = sum(sizes)
    x, w = normal(1, n, 64).to(torch.bfloat16), normal(2, groups, 40, 64).to(torch.bfloat16)
    y = harp.grouped_linear(x, w, offsets_of(sizes), out_dtype=torch.float32)
    gw = harp.grouped_grad_weights(y.to(torch.bfloat16), x, offsets_of(sizes))
    for e, r in group_rows(sizes):
        check(y[r], *bf16_want(x[r], w[e], torch.float32))
        check(gw[e], *bf16_want(y[r].to(torch.bfloat16).T, x[r].T, torch.float32))


def test_no_rows():
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    x, w = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), normal(1, 3, 32, 64).to(torch.bfloat16)
    assert harp.grouped_linear(x, w, off).shape == (0, 32)
    gw = torch.full((3, 32, 64), 2.0, device="cuda")
    harp.grouped_grad_weights(torch.empty((0, 32), dtype=torch.bfloat16, device="cuda"), x, off, out=gw, accumulate=True)
    assert (gw == 2).all()
    harp.grouped_grad_weights(torch.empty((0, 32), dtype=torch.bfloat16, device="cuda"), x, off, out=gw)
    assert (gw == 0).all()
    q, s = harp.quantize_rows(torch.empty((0, 64), device="cuda"))
    assert q.shape == (0, 64) and s.shape == (0,)
    assert harp.linear_i8(q, s, eight_bits(1, 8, 64), scales(1, 8)).shape == (0, 8)


# ---- gradients against differences

@pytest.mark.parametrize("sizes", [[3, 0, 17], [130, 70], [1]])
def test_gradients_against_differences(sizes):
    """Small whole numbers: every product and sum is exact, and so is the difference of a linear function."""
    n, d_in, d_out, groups = sum(sizes), 96, 72, len(sizes)
    rng = np.random.default_rng(5)

    def whole(*shape):
        return torch.from_numpy(rng.integers(-8, 9, shape).astype(np.float32)).cuda().to(torch.bfloat16)
    x, v, w, u, gy, off = whole(n, d_in), whole(n, d_in), whole(groups, d_out, d_in), whole(groups, d_out, d_in), whole(n, d_out), offsets_of(sizes)

    def loss(x, w):
        return (harp.grouped_linear(x, w, off, out_dtype=torch.float32).double() * gy.double()).sum()
    gx = harp.grouped_grad_rows(gy, w, off, out_dtype=torch.float32)
    gw = harp.grouped_grad_weights(gy, x, off)
    assert (loss(x + v, w) - loss(x - v, w)) / 2 == (gx.double() * v.double()).sum()
    assert (loss(x, w + u) - loss(x, w - u)) / 2 == (gw.double() * u.double()).sum()


# ---- a run of them together

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 5, 33, 300])
def test_processed_layer(n, dtype):
    """y = x W^T through the 8-bit W~.  The steps one by one give the same bits; against the layer itself the error of a row is that
    of the two quantisations, half a step a value, which Q_out^T leaves as long as it is, and the applies' own."""
    spec_in, spec_out = wl.tiny_plan(3, (8, 8, 4), kind="qr", perm="identity", signs=True), wl.tiny_plan(4, (8, 4, 4), kind="qr", perm="identity", signs=True)
    plan_in, plan_out = harp.plan_from_spec(spec_in), harp.plan_from_spec(spec_out)
    o_in, o_out = orc.OraclePlan.from_spec(spec_in), orc.OraclePlan.from_spec(spec_out)
    rng = np.random.default_rng(n)
    W = rng.standard_normal((spec_out.d, spec_in.d)) * 0.05
    x = torch.from_numpy(rng.standard_normal((n, spec_in.d)).astype(np.float32)).cuda().to(dtype)
    wt = torch.from_numpy(np.ascontiguousarray(orc.two_sided(o_out, o_in, W), dtype=np.float32)).cuda()
    wq, sw = harp.quantize_rows(wt)
    y = harp.processed_linear_i8(x.clone(), plan_in, plan_out, wq, sw)
    scratch = torch.empty(harp.harp_processed_linear_scratch_bytes(plan_in, n), dtype=torch.uint8, device="cuda")
    assert torch.equal(harp.processed_linear_i8(x.clone(), plan_in, plan_out, wq, sw, scratch=scratch), y)
    xt = harp.apply_(plan_in, x.clone())
    q, sx = harp.quantize_rows(xt)
    z = harp.linear_i8(q, sx, wq, sw, out_dtype=dtype)
    assert torch.equal(harp.apply_(plan_out, z, transpose=True), y)
    exact = x.double().cpu().numpy() @ W.T
    xt64, wt64 = torch.from_numpy(orc.forward(o_in, x.double().cpu().numpy())), torch.from_numpy(orc.two_sided(o_out, o_in, W))
    sx64, sw64 = sx.double().cpu()[:, None], sw.double().cpu()[None, :]
    bound = xt64.abs().sum(1, keepdim=True) * sw64 / 2 + wt64.abs().sum(1)[None, :] * sx64 / 2 + spec_in.d * sx64 * sw64 / 4
    far = np.linalg.norm(y.double().cpu().numpy() - exact, axis=1)
    tol = 8e-3 if dtype == torch.bfloat16 else 1e-5               # of a row, an apply: per coordinate, hence the root
    own = 2 * tol * np.sqrt(max(spec_in.d, spec_out.d)) * np.linalg.norm(exact, axis=1) + 2.0 ** -8 * np.linalg.norm(exact, axis=1)
    assert (far <= np.linalg.norm(bound.numpy(), axis=1) + own).all()


def test_expert_layers_forward_and_backward():
    """Two grouped products and their gradients, as a step takes them, twice: the same bits."""
    sizes, d, f = [70, 0, 33, 129], 256, 384
    n, off = sum(sizes), offsets_of(sizes)
    x, w1, w2 = normal(1, n, d).to(torch.bfloat16), (normal(2, 4, f, d) * 0.1).to(torch.bfloat16), (normal(3, 4, d, f) * 0.1).to(torch.bfloat16)
    gy = normal(4, n, d).to(torch.bfloat16)

    def step():
        h = harp.grouped_linear(x, w1, off)
        y = harp.grouped_linear(h, w2, off, out_dtype=torch.float32)
        gh = harp.grouped_grad_rows(gy, w2, off)
        return y, harp.grouped_grad_rows(gh, w1, off), harp.grouped_grad_weights(gy, h, off), harp.grouped_grad_weights(gh, x, off)
    a, b = step(), step()
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    for e, r in group_rows(sizes):
        h = harp.grouped_linear(x, w1, off)[r]
        check(a[0][r], *bf16_want(h, w2[e], torch.float32))


# ---- captures, streams, order

def _calls(seed, misaligned=False):
    """Inputs and one call of every operator on them; the outputs are kept."""
    sizes, d_in, d_out = [40, 0, 3, 200, 21], 501 if misaligned else 512, 384
    n, off = sum(sizes), offsets_of(sizes)
    s = dict(x=normal(seed, n, d_in).to(torch.bfloat16), w=normal(seed + 1, 5, d_out, d_in).to(torch.bfloat16), gy=normal(seed + 2, n, d_out).to(torch.bfloat16),
             q=torch.empty((n, d_in), dtype=torch.int8, device="cuda"), scale=torch.empty(n, device="cuda"), wq=eight_bits(seed + 3, 5, d_out, d_in),
             sw=scales(seed + 4, 5, d_out), off=off, y=torch.zeros((n, d_out), dtype=torch.bfloat16, device="cuda"),
             y1=torch.zeros((7, d_out), dtype=torch.float32, device="cuda"), y8=torch.zeros((n, d_out), dtype=torch.bfloat16, device="cuda"),
             gx=torch.zeros((n, d_in), dtype=torch.bfloat16, device="cuda"), gw=torch.zeros((5, d_out, d_in), device="cuda"))

    def run():
        harp.quantize_rows(s["x"], out=s["q"], scale=s["scale"])
        harp.linear_i8(s["q"][:7], s["scale"][:7], s["wq"][0], s["sw"][0], out=s["y1"])
        harp.grouped_linear_i8(s["q"], s["scale"], s["wq"], s["sw"], s["off"], out=s["y8"])
        harp.grouped_linear(s["x"], s["w"], s["off"], out=s["y"])
        harp.grouped_grad_rows(s["gy"], s["w"], s["off"], out=s["gx"])
        harp.grouped_grad_weights(s["gy"], s["x"], s["off"], out=s["gw"])
    return s, run


OUTPUTS = ("q", "scale", "y1", "y8", "y", "gx", "gw")


@pytest.mark.parametrize("misaligned", [False, True])
def test_captured_and_replayed(misaligned):
    """A replay reads what the inputs and offsets hold by then."""
    s, run = _calls(1, misaligned)
    t, run_t = _calls(50, misaligned)
    run()
    run_t()
    torch.cuda.synchronize()
    want = {k: t[k].clone() for k in OUTPUTS}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for k in ("x", "w", "gy", "wq", "sw"):
        s[k].copy_(t[k])
    for k in OUTPUTS:
        s[k].zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for k in OUTPUTS:
        assert torch.equal(s[k], want[k]), k
    s["off"].copy_(offsets_of([0, 100, 100, 0, 64]))
    t["off"].copy_(s["off"])
    g.replay()
    run_t()
    torch.cuda.synchronize()
    for k in OUTPUTS:
        assert torch.equal(s[k], t[k]), k
    assert harp.harp_linear_error_word() == 0


@pytest.mark.parametrize("d_in", [512, 500])
def test_the_first_call_of_a_process_may_be_captured(d_in):
    code = f"""
import torch
import paper_2605_29843_b200 as harp
x, w = torch.randn(37, {d_in}, device='cuda').bfloat16(), torch.randn(1, 64, {d_in}, device='cuda').bfloat16()
off, y = torch.tensor([0, 37], dtype=torch.int32, device='cuda'), torch.zeros(37, 64, dtype=torch.bfloat16, device='cuda')
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    harp.grouped_linear(x, w, off, out=y)
g.replay()
torch.cuda.synchronize()
z = harp.grouped_linear(x, w, off)
assert torch.equal(y, z) and z.abs().sum() > 0
"""
    subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), check=True, timeout=100)


def test_a_captured_layer():
    """The whole layer without scratch of the caller's, its first call captured, replayed on other rows."""
    code = """
import torch
import paper_2605_29843_b200 as harp
from paper_2605_29843_b200 import workloads as wl
plan_in, plan_out = (harp.plan_from_spec(wl.tiny_plan(s, r, kind='qr', perm='identity', signs=True)) for s, r in ((3, (8, 8, 4)), (4, (8, 4, 4))))
wq = torch.randint(-127, 128, (plan_out.d, plan_in.d), dtype=torch.int8, device='cuda')
sw = torch.rand(plan_out.d, device='cuda')
rows, y = torch.randn(2, 9, plan_in.d, device='cuda').bfloat16(), torch.empty(9, plan_out.d, dtype=torch.bfloat16, device='cuda')
x = rows[0].clone()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    harp.processed_linear_i8(x, plan_in, plan_out, wq, sw, out=y)
for r in rows:
    x.copy_(r)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, harp.processed_linear_i8(r.clone(), plan_in, plan_out, wq, sw)) and y.abs().sum() > 0
"""
    subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), check=True, timeout=100)


@pytest.mark.parametrize("misaligned", [False, True])
def test_two_graphs_and_two_streams_at_once(misaligned):
    sets = [_calls(1 + 10 * i, misaligned) for i in range(4)]
    for s, run in sets:
        run()
    torch.cuda.synchronize()
    want = [{k: s[k].clone() for k in OUTPUTS} for s, _ in sets]
    graphs = []
    for s, run in sets[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(4):
                run()
        graphs.append(g)
    for s, _ in sets:
        for k in OUTPUTS:
            s[k].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                if i < 2:
                    graphs[i].replay()
                else:
                    for _ in range(4):
                        sets[i][1]()
    torch.cuda.synchronize()
    for (s, _), w in zip(sets, want):
        for k in OUTPUTS:
            assert torch.equal(s[k], w[k]), k
    assert harp.harp_linear_error_word() == 0


def test_chained_calls_see_each_other():
    """Each call's input is the output of the one before it: a hundred products by a permutation and its inverse."""
    d = 512
    p = torch.randperm(d, generator=torch.Generator().manual_seed(1)).cuda()
    w = torch.zeros((1, d, d), dtype=torch.bfloat16, device="cuda")
    w[0, torch.arange(d, device="cuda"), p] = 1
    off = offsets_of([37])
    x = normal(1, 37, d).to(torch.bfloat16)
    y = x.clone()
    for _ in range(50):
        y = harp.grouped_linear(y, w, off)
        y = harp.grouped_grad_rows(y, w, off)
    assert torch.equal(x, y)


@pytest.mark.parametrize("rows", [1, 16, 31, 64, 100, 300])
def test_same_bits_every_time(rows):
    x, w, off = normal(1, rows, 4096).to(torch.bfloat16), normal(2, 1, 2048, 4096).to(torch.bfloat16), offsets_of([rows])
    y = harp.grouped_linear(x, w, off, out_dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(harp.grouped_linear(x, w, off, out_dtype=torch.float32), y)


# ---- sizes past 32 bits

def test_results_past_32_bits():
    n, d_in, d_out = 66000, 64, 33000
    x, w, off = normal(1, n, d_in).to(torch.bfloat16), normal(2, 1, d_out, d_in).to(torch.bfloat16), offsets_of([n])
    y = harp.grouped_linear(x, w, off)
    for r in (slice(0, 40), slice(n // 2, n // 2 + 40), slice(n - 40, n)):
        check(y[r], *bf16_want(x[r], w[0], torch.bfloat16))


def test_weights_past_32_bits():
    sizes, d = [3, 0, 1] + [0] * 30 + [2, 30], 8192
    n, off = sum(sizes), offsets_of(sizes)
    x = normal(1, n, d).to(torch.bfloat16)
    w = torch.zeros((len(sizes), d, d), dtype=torch.bfloat16, device="cuda")
    for e in (0, 2, len(sizes) - 2, len(sizes) - 1):
        w[e] = normal(e + 2, d, d).to(torch.bfloat16)
    y = harp.grouped_linear(x, w, off, out_dtype=torch.float32)
    gx = harp.grouped_grad_rows(x, w, off, out_dtype=torch.float32)
    for e, r in group_rows(sizes):
        check(y[r], *bf16_want(x[r], w[e], torch.float32))
        check(gx[r], *bf16_want(x[r], w[e].T, torch.float32))
    gw = harp.grouped_grad_weights(x, x, off, out=w)
    for e, r in group_rows(sizes):
        if e in (0, 1, len(sizes) - 1):
            check(gw[e], *bf16_want(x[r].T, x[r].T, torch.bfloat16))


# ---- refusals of the torch conveniences

def test_refusals():
    x, w, off = normal(1, 8, 64).to(torch.bfloat16), normal(2, 2, 32, 64).to(torch.bfloat16), offsets_of([3, 5])
    q, s, wq, sw = eight_bits(1, 8, 64), scales(1, 8), eight_bits(2, 32, 64), scales(2, 32)
    gy = normal(3, 8, 32).to(torch.bfloat16)
    before = harp.harp_launch_count()
    for error, call in [
            (TypeError, lambda: harp.quantize_rows(x.half())), (ValueError, lambda: harp.quantize_rows(x[0])),
            (ValueError, lambda: harp.quantize_rows(x.cpu())), (ValueError, lambda: harp.quantize_rows(x.T)),
            (ValueError, lambda: harp.quantize_rows(x, out=q[:4])), (TypeError, lambda: harp.quantize_rows(x, out=x)),
            (ValueError, lambda: harp.quantize_rows(x, scale=s[:4])), (TypeError, lambda: harp.quantize_rows(x, scale=s.double())),
            (TypeError, lambda: harp.linear_i8(x, s, wq, sw)), (ValueError, lambda: harp.linear_i8(q, s, wq[:, :32], sw)),
            (ValueError, lambda: harp.linear_i8(q, s[:7], wq, sw)), (ValueError, lambda: harp.linear_i8(q, s, wq, sw[:31])),
            (ValueError, lambda: harp.linear_i8(q, s, wq.cpu(), sw)), (ValueError, lambda: harp.linear_i8(q, s.cpu(), wq, sw)),
            (TypeError, lambda: harp.linear_i8(q, s, wq, sw, out=q[:, :32])), (ValueError, lambda: harp.linear_i8(q, s, wq, sw, out=gy[:4])),
            (TypeError, lambda: harp.linear_i8(q, s, wq, sw, out=gy, out_dtype=torch.float32)),
            (ValueError, lambda: harp.linear_i8(q[:1].expand(8, 64), s, wq, sw)),
            (TypeError, lambda: harp.grouped_linear(x.float(), w, off)), (TypeError, lambda: harp.grouped_linear(x, w, off.long())),
            (ValueError, lambda: harp.grouped_linear(x, w, off[:2])), (ValueError, lambda: harp.grouped_linear(x, w, off.cpu())),
            (ValueError, lambda: harp.grouped_linear(x, w[0], off)), (ValueError, lambda: harp.grouped_linear(x[:, :32], w, off)),
            (ValueError, lambda: harp.grouped_linear(x, w.transpose(1, 2), off)), (ValueError, lambda: harp.grouped_linear(x, w[:, :16], off)),
            (ValueError, lambda: harp.grouped_grad_rows(gy[:, :16], w, off)), (ValueError, lambda: harp.grouped_grad_weights(gy[:4], x, off)),
            (ValueError, lambda: harp.grouped_grad_weights(gy, x, off, accumulate=True)),
            (ValueError, lambda: harp.grouped_grad_weights(gy, x, off, out=torch.zeros((3, 32, 64), device="cuda"))),
            (harp.HarpError, lambda: harp.grouped_linear(x, w[:0], off[:1]))]:
        with pytest.raises(error):
            call()
    assert harp.harp_launch_count() == before
