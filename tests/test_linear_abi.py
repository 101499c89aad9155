"""Layer products: what their entry points refuse, before the first CUDA call (runs without a GPU)."""
import ctypes

import pytest

import paper_2605_29843_b200 as harp
from paper_2605_29843_b200 import build as harp_build

OK, NULL, DIM, DTYPE, LARGE = 0, 1, 2, 6, 11
P = 1 << 20         # an address that is never followed: the calls below end before any launch


@pytest.fixture(scope="module", autouse=True)
def _built():
    harp_build.build()


def quantize(x=P, ld_x=64, n=4, d=64, dtype=1, q=P, ld_q=64, scale=P):
    return harp.lib().harp_quantize_rows(x, ld_x, n, d, dtype, q, ld_q, scale, None)


def linear(x=P, ld_x=64, xs=P, w=P, ld_w=64, ws=P, n=4, d_in=64, d_out=32, y=P, ld_y=32, dtype=1):
    return harp.lib().harp_linear_i8(x, ld_x, xs, w, ld_w, ws, n, d_in, d_out, y, ld_y, dtype, None)


def grouped_i8(x=P, ld_x=64, xs=P, w=P, ld_w=64, ws=P, off=P, groups=2, n=4, d_in=64, d_out=32, y=P, ld_y=32, dtype=1):
    return harp.lib().harp_grouped_linear_i8(x, ld_x, xs, w, ld_w, ws, off, groups, n, d_in, d_out, y, ld_y, dtype, None)


def grouped(x=P, ld_x=64, w=P, ld_w=64, off=P, groups=2, n=4, d_in=64, d_out=32, y=P, ld_y=32, dtype=1):
    return harp.lib().harp_grouped_linear(x, ld_x, w, ld_w, off, groups, n, d_in, d_out, y, ld_y, dtype, None)


def grad_rows(gy=P, ld_gy=32, w=P, ld_w=64, off=P, groups=2, n=4, d_in=64, d_out=32, gx=P, ld_gx=64, dtype=1):
    return harp.lib().harp_grouped_grad_rows(gy, ld_gy, w, ld_w, off, groups, n, d_in, d_out, gx, ld_gx, dtype, None)


def grad_weights(gy=P, ld_gy=32, x=P, ld_x=64, off=P, groups=2, n=4, d_in=64, d_out=32, gw=P, ld_gw=64, dtype=0, acc=0):
    return harp.lib().harp_grouped_grad_weights(gy, ld_gy, x, ld_x, off, groups, n, d_in, d_out, gw, ld_gw, dtype, acc, None)


@pytest.mark.parametrize("call,kwargs,code", [
    (quantize, dict(x=None), NULL), (quantize, dict(q=None), NULL), (quantize, dict(scale=None), NULL),
    (quantize, dict(dtype=2), DTYPE), (quantize, dict(d=0), DIM), (quantize, dict(n=-1), DIM), (quantize, dict(ld_x=63), DIM),
    (quantize, dict(ld_q=63), DIM), (quantize, dict(x=P + 1), DIM), (quantize, dict(scale=P + 2), DIM), (quantize, dict(x=P + 2, dtype=0), DIM),
    (quantize, dict(d=(1 << 20) + 1, ld_x=1 << 21, ld_q=1 << 21), DIM), (quantize, dict(n=1 << 31), DIM),
    (quantize, dict(n=0, x=None, q=None, scale=None), OK),
    *[(linear, {k: None}, NULL) for k in ("x", "xs", "w", "ws", "y")],
    (linear, dict(dtype=3), DTYPE), (linear, dict(d_in=0), DIM), (linear, dict(d_out=0), DIM), (linear, dict(n=-1), DIM),
    (linear, dict(ld_x=63), DIM), (linear, dict(ld_w=63), DIM), (linear, dict(ld_y=31), DIM), (linear, dict(y=P + 1), DIM),
    (linear, dict(y=P + 2, dtype=0), DIM), (linear, dict(xs=P + 1), DIM), (linear, dict(ws=P + 2), DIM),
    (linear, dict(d_in=131072, ld_x=131072, ld_w=131072), LARGE), (linear, dict(n=(1 << 30) + 1), LARGE),
    (linear, dict(d_out=(1 << 20) + 1, ld_y=1 << 21), LARGE), (linear, dict(ld_w=1 << 62), LARGE), (linear, dict(ld_y=1 << 38), LARGE),
    (grad_rows, dict(ld_gy=1 << 38), LARGE), (grad_weights, dict(ld_gw=1 << 38), LARGE), (grouped, dict(ld_x=1 << 38), LARGE), (linear, dict(n=0, x=None, y=None), OK),
    *[(grouped_i8, {k: None}, NULL) for k in ("x", "xs", "w", "ws", "off", "y")],
    (grouped_i8, dict(groups=0), DIM), (grouped_i8, dict(groups=1025), LARGE), (grouped_i8, dict(off=P + 2), DIM),
    *[(grouped, {k: None}, NULL) for k in ("x", "w", "off", "y")],
    (grouped, dict(x=P + 1), DIM), (grouped, dict(w=P + 1), DIM), (grouped, dict(dtype=-1), DTYPE), (grouped, dict(groups=-1), DIM),
    (grouped, dict(d_in=(1 << 20) + 1, ld_x=1 << 21, ld_w=1 << 21), LARGE), (grouped, dict(n=0), OK),
    *[(grad_rows, {k: None}, NULL) for k in ("gy", "w", "off", "gx")],
    (grad_rows, dict(ld_gy=31), DIM), (grad_rows, dict(ld_gx=63), DIM), (grad_rows, dict(gx=P + 1), DIM), (grad_rows, dict(n=0), OK),
    *[(grad_weights, {k: None}, NULL) for k in ("gy", "x", "off", "gw")],
    (grad_weights, dict(ld_gw=63), DIM), (grad_weights, dict(gw=P + 2), DIM), (grad_weights, dict(dtype=5), DTYPE),
    (grad_weights, dict(n=0, gw=None), NULL), (grad_weights, dict(n=0, gy=None, x=None, off=None, acc=1), OK),
])
def test_refusals(call, kwargs, code):
    assert call(**kwargs) == code


def test_processed_layer_refusals():
    L = harp.lib()
    assert L.harp_processed_linear_i8(None, P, P, 1, 1, P, 64, P, P, None, None) == NULL
    assert L.harp_processed_linear_i8(P, None, P, 1, 1, P, 64, P, P, None, None) == NULL
    assert L.harp_processed_linear_scratch_bytes(None, 4) == 0


@pytest.mark.parametrize("kind,n_args", [("quantize", 9), ("linear_i8", 13), ("grouped_linear_i8", 15), ("grouped", 13), ("grad_weights", 14)])
def test_calls_without_ctypes(kind, n_args):
    """The extension's calls refuse what ctypes refuses, and hand every argument on in its place."""
    name = {"quantize": "harp_quantize_rows", "grouped": "harp_grouped_linear", "grad_weights": "harp_grouped_grad_weights"}.get(kind, "harp_" + kind)
    plain = getattr(harp.lib(), name)
    quick = harp._without_ctypes(plain, kind)
    assert quick is not plain
    pointers = [k for k, t in enumerate(plain.argtypes) if t is ctypes.c_void_p]
    good = {"quantize": (P, 64, 4, 64, 1, P, 64, P, 0), "linear_i8": (P, 64, P, P, 64, P, 4, 64, 32, P, 32, 1, 0),
            "grouped_linear_i8": (P, 64, P, P, 64, P, P, 2, 4, 64, 32, P, 32, 1, 0), "grouped": (P, 64, P, 64, P, 2, 4, 64, 32, P, 32, 1, 0),
            "grad_weights": (P, 32, P, 64, P, 2, 4, 64, 32, P, 64, 0, 0, 0)}[kind]
    assert len(good) == n_args == len(plain.argtypes)
    for k in range(n_args - 1):
        bad = list(good)
        if k in pointers:
            bad[k] = None
            assert quick(*bad) == plain(*bad) == NULL
        else:
            for value in (None, 1.0, "1"):
                bad[k] = value
                with pytest.raises(TypeError):
                    quick(*bad)
            if kind == "grad_weights" and k == 12:
                continue                      # accumulate takes any value
            bad[k] = -1
            assert quick(*bad) == plain(*bad) != OK
    with pytest.raises(TypeError):
        quick(*good[:-1])
